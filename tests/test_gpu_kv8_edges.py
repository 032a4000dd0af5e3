"""The 8-bit key/value cache and token scores where calls are unusual: paths that only sizes reach, padding, two streams, captured graphs; against the fp64 oracle, with the bounds of
test_gpu_kv8.py and test_gpu_token_scores.py."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import kv8_oracle as K
from tests import test_gpu_kv8 as T
from tests import test_gpu_token_scores as S

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dm():
    from paper_2511_15927_b200 import build
    build.build()
    from paper_2511_15927_b200 import binding
    return binding


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


# ---- attention and weights --------------------------------------------------------------------------------------------------------------

def test_weights_of_a_sequence_without_queries_are_copied(dm):
    """counts = 0: what was accumulated stays what it was, beside NaN codes too."""
    c = T.random_cache(2, 2, 1, 64, 64, [40, 40], rubbish=False)
    c["k"][0, 0, 3, 5] = 0x7f
    q = np.ones((2, 2, 1, 64)) * 0.125
    acc = np.random.default_rng(0).random((2, 1, 64)).astype(np.float32)
    _, got = T.run_attention(dm, c, q, [40, 38], [0, 2], 40, acc)
    assert np.array_equal(got[0, 0, :40], acc[0, 0, :40].astype(np.float64)) and np.all(got[0, 0, 40:] == -5)
    assert not np.isnan(got[1]).any()


@pytest.mark.parametrize("D,Hq,H,G,lens,counts", [
    (64, 2, 2, 3, [(37 * i * i) % 1900 for i in range(40)], [i % 4 for i in range(40)]),      # more sequences than lanes, shares that begin and end anywhere
    (80, 2, 1, 17, [(911 * i) % 2500 for i in range(70)], None),
    (128, 1, 1, 2, [0] * 33 + [5000], [0] * 20 + [2] * 14),                                   # most of the batch empty
    (64, 1, 1, 2, [9000, 0], [2, 1]),                                                         # two sequences, cut by pair
    (128, 4, 2, 1, [7000, 1], [1, 0])])
def test_many_and_few_sequences(dm, D, Hq, H, G, lens, counts):
    rng = np.random.default_rng(len(lens))
    B = len(lens)
    n = [a + b for a, b in zip(lens, counts or [G] * B)]
    cap = (max(n) + 31) // 32 * 32
    c = T.random_cache(7, B, H, cap, D, n)
    q = bf16(rng.normal(size=(B, G, Hq, D)))
    acc = rng.random((B, H, cap)).astype(np.float32)
    got, acc_got = T.run_attention(dm, c, q, lens, counts, max(lens), acc)
    T.check_attention(got, c, q, lens, counts, acc.astype(np.float64), acc_got)


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("D,Hq,H,G", [(64, 4, 1, 40), (80, 5, 1, 64), (128, 2, 2, 129)])
def test_weights_of_more_rows_than_one_launch_takes(dm, D, Hq, H, G, alias):
    rng = np.random.default_rng(G)
    lens, counts, cap = [200, 0], [G, G - 3], 352
    c = T.random_cache(9, 2, H, cap, D, [a + b for a, b in zip(lens, counts)])
    q = bf16(rng.normal(size=(2, G, Hq, D)))
    acc = rng.random((2, H, cap)).astype(np.float32)
    got, acc_got = T.run_attention(dm, c, q, lens, counts, 200, acc, alias=alias)
    T.check_attention(got, c, q, lens, counts, acc.astype(np.float64), acc_got, fill=None)


@pytest.mark.parametrize("D,Hq,H,G,lens,counts", [
    (64, 16, 2, 40, [4000, 3511, 17, 4090], [40, 1, 40, 39]), (80, 10, 2, 32, [4096, 0, 1, 33, 4000, 2999, 127, 129], [32, 32, 0, 5, 32, 32, 32, 31]),
    (64, 32, 32, 32, [14400, 9000], None), (80, 24, 24, 32, [11000, 200, 9601, 4096], [32, 32, 17, 32])])
def test_much_work_for_many_queries(dm, D, Hq, H, G, lens, counts):
    """Enough of it for 32 rows of queries with each tile."""
    rng = np.random.default_rng(D + H)
    B = len(lens)
    cap = (max(a + b for a, b in zip(lens, counts or [G] * B)) + 31) // 32 * 32
    c = T.random_cache(7, B, H, 64, D, [64] * B, rubbish=False)
    c = {k: np.tile(v, (1, 1, -(-cap // 64)) + (1,) * (v.ndim - 3))[:, :, :cap if k == "k" else cap // 32].copy() for k, v in c.items()}
    for b in range(B):                               # no row like another: signs and scales change along the cache
        c["k"][b] ^= (rng.integers(0, 2, (H, cap, 1), dtype=np.uint8) << 7).astype(np.uint8)
    for k in ("ks", "vs"):
        c[k] = c[k] * 2.0 ** rng.integers(-2, 3, c[k].shape)
    q = bf16(rng.normal(size=(B, G, Hq, D)))
    acc = rng.random((B, H, cap)).astype(np.float32)
    got, acc_got = T.run_attention(dm, c, q, lens, counts, max(lens), acc)
    T.check_attention(got, c, q, lens, counts, acc.astype(np.float64), acc_got)


def test_padding_may_hold_anything(dm):
    """NaN and infinities in the padding tokens' queries, keys and values change nothing."""
    B, G, Hq, H, D, cap = 3, 9, 4, 2, 64, 128
    rng = np.random.default_rng(31)
    lens, counts = [5, 60, 31], [4, 0, 9]
    cfg = dm.dm_kv8_cfg(B, G, Hq, H, D, dm.DM_BF16)
    width = (Hq + 2 * H) * D
    x = torch.from_numpy(rng.normal(size=(B, G, width))).to(torch.bfloat16)
    y = x.clone()
    for b, m in enumerate(counts):
        y[b, m:] = math.nan
        y[b, m:, ::3] = math.inf
    start = T.random_cache(4, B, H, cap, D, lens, rubbish=True)
    res = []
    for z in (x.cuda(), y.cuda()):
        d = T.to_gpu(start)
        n, m = T.i32(lens), T.i32(counts)
        nb = dm.dm_kv8_attention_workspace_bytes(cfg, 64)
        ws, out, acc = T.workspace(nb), torch.full((B * G, Hq * D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.ones(B, H, cap, device="cuda")
        p = z.data_ptr()
        dm.dm_kv8_append(cfg, T.handle(dm, d), p + 2 * Hq * D, p + 2 * (Hq + H) * D, width, n.data_ptr(), m.data_ptr(), T.stream())
        dm.dm_kv8_attention(cfg, T.handle(dm, d), p, width, n.data_ptr(), m.data_ptr(), 64, acc.data_ptr(), acc.data_ptr(), out.data_ptr(), Hq * D, ws.data_ptr(), nb, T.stream())
        dm.dm_check(T.stream())
        res.append((d, out, acc))
    assert torch.equal(res[0][1], res[1][1]) and torch.equal(res[0][2], res[1][2]) and all(torch.equal(res[0][0][k], res[1][0][k]) for k in ("k", "v"))
    assert torch.all(res[0][1].view(B, G, -1)[1] == 7)


def test_a_prompt_into_an_empty_cache(dm):
    """max_len = 0: everything that is attended to is the block's own, more rows of queries than shares."""
    rng = np.random.default_rng(2)
    G, Hq, H, D, cap = 300, 4, 2, 80, 320
    c = T.random_cache(12, 2, H, cap, D, [G, 77])
    q = bf16(rng.normal(size=(2, G, Hq, D)))
    got, _ = T.run_attention(dm, c, q, [0, 0], [G, 77], 0)
    T.check_attention(got, c, q, [0, 0], [G, 77])


def tiled(seed, B, H, cap, D):
    """A full cache whose 64 rows repeat with other signs."""
    rng = np.random.default_rng(seed)
    c = T.random_cache(7, B, H, 64, D, [64] * B, rubbish=False)
    c = {k: np.tile(v, (1, 1, -(-cap // 64)) + (1,) * (v.ndim - 3))[:, :, :cap if k == "k" else cap // 32].copy() for k, v in c.items()}
    c["k"] ^= (rng.integers(0, 2, (B, H, cap, 1), dtype=np.uint8) << 7).astype(np.uint8)
    return c


def check_wide(got, acc_got, c, q, lens, acc):
    """As check_attention, where V's scales differ: a probability is held to half a step of 2^-24 where the row's largest product of probability and scale is at 2^8 or above, so 2^-33 of
    that for every code beside the relative bound."""
    B, G, Hq, D = q.shape
    H = c["k"].shape[1]
    want, acc_want, spread, reach = K.attend(c, q, lens, [G] * B, acc)
    ds = reach[..., None] / math.sqrt(D) * (D + 8) * 2.0 ** -23 * 2
    for b in range(B):
        n = lens[b] + G
        for h in range(Hq):
            k = K.decode(c["k"][b, h * H // Hq], c["ks"][b, h * H // Hq])[:n]
            s = np.repeat(c["vs"][b, h * H // Hq], 32)[:n]
            codes = np.abs(K.VALUES[K.v_rows(c["v"][b, h * H // Hq])[:n]])
            for t in range(G):
                p = k @ q[b, t, h] / math.sqrt(D)
                p = np.exp(p - p.max())
                p /= p.sum()
                tol = 2.0 ** -8 * np.abs(want[b, t, h]) + (2.0 ** -11 + 2 * ds[b, t, h] + 2.0 ** -18) * spread[b, t, h] + 2.0 ** -33 * (p * s).max() * codes.sum(0) + 1e-38
                err = np.abs(got[b, t, h] - want[b, t, h])
                assert np.all(err <= tol), (b, h, t, float((err / tol).max()))
    if acc is not None:
        there = ~np.isnan(acc_want)
        bound = (2 * ds.max() + (Hq // H * G + 16) * 2.0 ** -23) * np.abs(np.where(there, acc_want, 0)) + 1e-30
        err = np.abs(np.where(there, acc_got - acc_want, 0))
        assert np.all(err <= bound), float((err / bound).max())


WIDE = [(64, 2, 1, 3, [700, 31]), (80, 2, 2, 17, [3000]), (128, 4, 2, 2, [1500, 96, 0]), (64, 1, 1, 1, [40000]), (64, 32, 32, 32, [14400, 9000])]      # the last: 32 rows of queries with each tile


@pytest.mark.parametrize("top", [100, 118])
@pytest.mark.parametrize("D,Hq,H,G,lens", WIDE)
def test_values_near_the_end_of_the_range(dm, D, Hq, H, G, lens, top):
    """Magnitudes of 1e32 and of 1e38, shared by all rows: what fits bf16 is not infinite."""
    rng = np.random.default_rng(top)
    B, cap = len(lens), (max(lens) + G + 31) // 32 * 32
    c = tiled(top, B, H, cap, D)
    c["v"] = np.where(c["v"] & 0x7f, c["v"] & 0x7f, 0x38).astype(np.uint8)       # all of one sign: an average is as large as they are
    c["vs"] = np.full_like(c["vs"], 2.0 ** top)
    q = bf16(rng.normal(size=(B, G, Hq, D)))
    acc = rng.random((B, H, cap)).astype(np.float32)
    got, acc_got = T.run_attention(dm, c, q, lens, None, max(lens), acc)
    assert np.isfinite(got).all()
    T.check_attention(got, c, q, lens, None, acc.astype(np.float64), acc_got)


@pytest.mark.parametrize("top", [0, 30, 60, 110])
@pytest.mark.parametrize("D,Hq,H,G,lens", WIDE[:4])
def test_blocks_of_zeros_beside_large_values(dm, D, Hq, H, G, lens, top):
    """Rows whose values are zeros, in blocks whose scale is the smallest there is: they take their part of the weight, however large the other blocks' values are."""
    rng = np.random.default_rng(top + D)
    B, cap = len(lens), (max(lens) + G + 31) // 32 * 32
    c = tiled(top, B, H, cap, D)
    c["vs"] = np.full_like(c["vs"], 2.0 ** top)
    for b in range(B):
        for h in range(H):
            zero = rng.random(cap // 32) < 0.4
            zero[0] = h % 2 == 0
            c["v"][b, h, zero], c["vs"][b, h, zero] = 0, K.FLOOR
    q = bf16(rng.normal(size=(B, G, Hq, D)) * 0.5)
    acc = rng.random((B, H, cap)).astype(np.float32)
    got, acc_got = T.run_attention(dm, c, q, lens, None, max(lens), acc)
    T.check_attention(got, c, q, lens, None, acc.astype(np.float64), acc_got)


@pytest.mark.parametrize("order", ["any", "rising", "falling", "one"])
@pytest.mark.parametrize("D,Hq,H,G,lens", WIDE[:4])
def test_scales_of_every_magnitude_in_one_head(dm, D, Hq, H, G, lens, order):
    """V's scales from 2^-100 to 2^100 in one head, and rows of queries that see the smaller ones alone, or nearly."""
    rng = np.random.default_rng(D + G)
    B, cap = len(lens), (max(lens) + G + 31) // 32 * 32
    c = tiled(D, B, H, cap, D)
    e = rng.integers(-100, 101, c["vs"].shape)
    if order == "rising" or order == "falling":
        e.sort(-1)
        e = e if order == "rising" else e[..., ::-1].copy()
    elif order == "one":
        e = np.zeros_like(e)
        e[..., 0] = 100
    c["vs"] = 2.0 ** e
    # the larger the scale, the less the row is attended to: channel 0 of K says how much
    k = K.decode(c["k"], np.ones_like(c["ks"]))
    c["k"][..., 0] = K.encode(np.repeat(-np.clip(e, -100, 100) * 2.0 + rng.normal(size=e.shape), 32, -1))
    c["ks"] = np.ones_like(c["ks"])
    c["k"][..., 1:] = K.encode(k[..., 1:] / 256)
    q = rng.normal(size=(B, G, Hq, D))
    # up to twice as steep as would balance the scales
    q[..., 0] = rng.uniform(0, 1, (B, G, Hq)) * math.log(2) / 2 * 2 * math.sqrt(D)
    q[:, 0, :, 0] = 0
    q = bf16(q)
    acc = rng.random((B, H, cap)).astype(np.float32)
    got, acc_got = T.run_attention(dm, c, q, lens, None, max(lens), acc)
    check_wide(got, acc_got, c, q, lens, acc.astype(np.float64))


@pytest.mark.parametrize("D,Hq,H,G", [(80, 4, 2, 4), (64, 2, 2, 32), (128, 4, 1, 1)])
def test_a_sequence_beside_other_sequences(dm, D, Hq, H, G):
    """The same sequence alone, at either end of a batch, and beside long, empty and padded sequences of other contents: where it is cut and joined depends on them, so the results agree within the
    bound of each; the same batch again gives the same bits."""
    rng = np.random.default_rng(D)
    n, cap = 3000, 9600
    own = T.random_cache(11, 1, H, cap, D, [n + G])
    q0, acc0 = rng.normal(size=(1, G, Hq, D)), rng.random((1, H, cap)).astype(np.float32)
    for at, others, counts in ((0, [], [G]), (0, [9500], [G, G]), (1, [9500], [1, G]), (2, [0, 77, 5000, 9000], [G, 0, G, G, G]), (0, [3000] * 20, None)):
        lens = others[:at] + [n] + others[at:]
        B = len(lens)
        cn = counts or [G] * B
        rest = T.random_cache(B, B, H, 64, D, [64] * B, rubbish=False)
        c = {k: np.tile(v, (1, 1, cap // 64) + (1,) * (v.ndim - 3)) for k, v in rest.items()}
        for k in c:
            c[k][at] = own[k][0]
        q = np.concatenate([rng.normal(size=(at, G, Hq, D)), q0, rng.normal(size=(B - at - 1, G, Hq, D))])
        q = bf16(q)
        acc = rng.random((B, H, cap)).astype(np.float32)
        acc[at] = acc0[0]
        got, acc_got = T.run_attention(dm, c, q, lens, counts, max(lens), acc)
        again, acc_again = T.run_attention(dm, c, q, lens, counts, max(lens), acc)
        assert np.array_equal(got, again) and np.array_equal(acc_got, acc_again, equal_nan=True)
        mine = slice(at, at + 1)
        assert cn[at] == G
        T.check_attention(got[mine], own, q[mine], [n], None, acc0.astype(np.float64), acc_got[mine])


# ---- evict --------------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [8193, 20000, 32768, 40000])
@pytest.mark.parametrize("scores", ["random", "equal", "few", "nan"])
def test_evict_from_long_sequences(dm, n, scores):
    """Each way of holding the weights: 32 per thread, none; thousands of equal ones, whose bin no list holds; more NaN than rows that leave."""
    rng = np.random.default_rng(n)
    lens, cap, D = [n, n // 3], (n + 31) // 32 * 32, 64
    c = T.random_cache(3, 2, 1, 64, D, [64, 64], rubbish=False)
    c = {k: np.tile(v, (1, 1, -(-cap // 64)) + (1,) * (v.ndim - 3))[:, :, :cap if k == "k" else cap // 32] for k, v in c.items()}      # 64 rows over and over
    for k in ("ks", "vs"):
        c[k] = c[k] * 2.0 ** rng.integers(-6, 7, c[k].shape)
    acc = rng.random((2, 1, cap)).astype(np.float32)
    if scores == "equal":
        acc[:] = 0.5
    elif scores == "few":
        acc = rng.integers(0, 3, acc.shape).astype(np.float32)
    elif scores == "nan":
        acc[rng.random(acc.shape) < 0.7] = math.nan
    keep, recent = n // 2 + 3, 77
    dst = T.random_cache(22, 2, 1, (keep + 31) // 32 * 32, D, [0, 0], rubbish=False)
    acc_dst = rng.random((2, 1, dst["k"].shape[2])).astype(np.float32)
    want, a, m, r = K.evict(c, acc, np.array(lens), keep, recent, dst, acc_dst)
    got, ga, gm, gr = T.run_evict(dm, c, acc, lens, keep, recent, dst, acc_dst)
    assert np.array_equal(gm, m) and np.array_equal(gr, r) and np.array_equal(ga, a, equal_nan=True)
    T.same(got, want)


@pytest.mark.parametrize("n", [1020, 2047, 1024])
def test_evict_where_nan_weights_are_all_that_is_left(dm, n):
    """The threshold falls among a few NaN weights, in a sequence that leaves a few of the threads without a row; sequences before it have many ordinary ones."""
    rng = np.random.default_rng(n)
    B, H, D, cap, keep = 40, 4, 64, 2048, n - 4
    lens = [2048 - b for b in range(B - 1)] + [n]
    c = T.random_cache(3, B, H, 64, D, [64] * B, rubbish=False)
    c = {k: np.tile(v, (1, 1, 32) + (1,) * (v.ndim - 3)) for k, v in c.items()}
    acc = rng.random((B, H, cap)).astype(np.float32)
    acc[-1][:, rng.permutation(n)[:9]] = math.nan
    acc[-1][:, rng.permutation(n)[:3]] = -1.0
    dst = T.random_cache(22, B, H, (keep + 31) // 32 * 32, D, [0] * B, rubbish=False)
    acc_dst = rng.random((B, H, dst["k"].shape[2])).astype(np.float32)
    for first, recent in ((0, 0), (B - 1, 2)):
        l = np.array(lens[first:])
        part = {k: np.ascontiguousarray(v[first:]) for k, v in c.items()}
        to = {k: np.ascontiguousarray(v[first:]) for k, v in dst.items()}
        want, a, m, r = K.evict(part, acc[first:], l, keep, recent, to, acc_dst[first:])
        got, ga, gm, gr = T.run_evict(dm, part, acc[first:], l.tolist(), keep, recent, to, acc_dst[first:])
        assert np.array_equal(gm, m) and np.array_equal(gr, r) and np.array_equal(ga, a, equal_nan=True)
        T.same(got, want)


@pytest.mark.parametrize("keep,recent,cap_to", [(40, 40, 64), (1, 1, 32), (500, 500, 512), (64, 64, 256)])
def test_evict_that_keeps_the_last_rows_or_all(dm, keep, recent, cap_to):
    rng = np.random.default_rng(keep)
    c = T.random_cache(5, 3, 2, 128, 128, [128, 41, 40])
    acc = rng.random((3, 2, 128)).astype(np.float32)
    dst = T.random_cache(6, 3, 2, cap_to, 128, [0] * 3)
    acc_dst = rng.random((3, 2, cap_to)).astype(np.float32)
    want, a, m, r = K.evict(c, acc, np.array([128, 41, 40]), keep, recent, dst, acc_dst)
    got, ga, gm, gr = T.run_evict(dm, c, acc, [128, 41, 40], keep, recent, dst, acc_dst, max_len=40000 if keep == 64 else None)
    assert np.array_equal(gm, m) and np.array_equal(gr, r) and np.array_equal(ga, a)
    T.same(got, want)


@pytest.mark.parametrize("n,B,H", [(32768, 6, 40), (20000, 4, 40), (40000, 2, 30)])
@pytest.mark.parametrize("scores", ["uniform", "far", "levels"])
def test_evict_that_counts_in_several_passes(dm, n, B, H, scores):
    """More than 32 weights in the first pass's step, for every head and in many more CTAs than run at a time: uniform weights (two passes), a few weights 2^200 from the others, which leaves
    those in one step (three), a handful of values (a pass for each digit of the key).  The kept rows against a stable sort, call after call, the words behind them untouched."""
    D, keep, recent = 64, n // 3 + 1, 37
    cap, to = (n + 31) // 32 * 32, (keep + 31) // 32 * 32
    g = torch.Generator(device="cuda").manual_seed(n + H)
    src = {"k": torch.zeros(B, H, cap, D, dtype=torch.uint8, device="cuda"), "v": torch.zeros(B, H, cap // 32, D, 32, dtype=torch.uint8, device="cuda"),
           "ks": torch.ones(B, H, cap // 32, device="cuda"), "vs": torch.ones(B, H, cap // 32, device="cuda")}
    dst = {"k": torch.empty(B, H, to, D, dtype=torch.uint8, device="cuda"), "v": torch.empty(B, H, to // 32, D, 32, dtype=torch.uint8, device="cuda"),
           "ks": torch.empty(B, H, to // 32, device="cuda"), "vs": torch.empty(B, H, to // 32, device="cuda")}
    cfg = dm.dm_kv8_cfg(B, 1, H, H, D, dm.DM_BF16)
    lens = [n - 500 * b for b in range(B)]
    li, lo = T.i32(lens), T.i32([0] * B)
    acc2 = torch.empty(B, H, to, device="cuda")
    rows = torch.empty(B * H * keep + 4096, dtype=torch.int32, device="cuda")
    nb = dm.dm_kv8_evict_workspace_bytes(cfg, n, keep)
    ws = T.workspace(nb)
    at = torch.arange(cap, device="cuda")
    there = at < li.long()[:, None, None]
    for _ in range(6):
        acc = torch.rand(B, H, cap, generator=g, device="cuda")
        if scores == "far":
            acc = torch.where(torch.rand(B, H, cap, generator=g, device="cuda") < 1e-3, acc * 2.0 ** 100, acc * 2.0 ** -100)
            acc[:, :, ::977] *= -1
        elif scores == "levels":
            acc = torch.floor(acc * 5) * 0.1 + 1
        rows.fill_(-7)
        dm.dm_kv8_evict(cfg, T.handle(dm, src), T.handle(dm, dst), acc.data_ptr(), acc2.data_ptr(), li.data_ptr(), lo.data_ptr(), n, keep, recent, rows.data_ptr(),
                        ws.data_ptr(), nb, T.stream())
        dm.dm_check(T.stream())
        key = torch.where(at >= (li.long() - recent)[:, None, None], math.inf, acc)
        order = torch.sort(torch.where(there, key, -math.inf), dim=-1, descending=True, stable=True).indices[..., :keep]
        want = torch.sort(order, dim=-1).values
        assert lo.tolist() == [keep] * B
        assert torch.equal(rows[:B * H * keep].view(B, H, keep).long(), want)
        assert torch.all(rows[B * H * keep:] == -7)
        assert torch.equal(acc2[:, :, :keep], acc.gather(2, want))


# ---- token scores -------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 32), (3, 31, 32), (2, 262147, 32), (601, 20011, 32), (1, 8192, 1), (1, 8191, 1)])
def test_scores_of_equal_logits_and_extreme_sizes(dm, dtype, rows, vocab, k):
    """Every logit the same: the lowest ids, more candidates than there is room for; then two that are larger, at the ends."""
    x = torch.full((rows, vocab), -2.5, dtype=dtype, device="cuda")
    S.check(dm, x[:3], list(range(min(rows, 3))), -1, k)
    x[:, -1] = 1.5
    x[:, vocab // 3] = 1.5
    tokens = [r % vocab for r in range(rows)]
    if rows < 10:
        S.check(dm, x, tokens, 0, k)
    else:
        lp, en, ids, tops = S.run(dm, x, tokens, 0, k)
        assert np.all(ids[:, 0] == vocab // 3) and np.all(ids[:, 1] == vocab - 1) and np.all(ids[:, 2:] == np.arange(1, k - 1))
        assert np.all(lp[1:] == lp[1]) and lp[0] == -math.inf and np.all(en == en[0])


@pytest.mark.parametrize("vocab,shift", [(12 * 1024, 0), (13 * 1024 + 5, 3), (15 * 1024, 1), (18 * 1024 - 7, 0), (35 * 1024 + 1, 5), (50257, 0), (1023, 7)])
def test_scores_of_many_rows_with_each_length_of_round(dm, vocab, shift):
    """Rows enough for one CTA each; the rounds of loads are chosen by the vocabulary."""
    rows, g = 300, torch.Generator(device="cuda").manual_seed(vocab)
    x = (torch.randn(rows, vocab + 16, generator=g, device="cuda") * 4).to(torch.bfloat16)[:, shift:shift + vocab]
    tokens = [(r * 7919) % vocab for r in range(rows)]
    lp, en, ids, tops = S.run(dm, x, tokens, 11, 8)
    few = [0, 1, 150, 299]
    S.check(dm, x[few], [tokens[r] for r in few], 11, 8)      # (by clusters)
    wl, we, wi, wt = K.token_scores(x[few].double().cpu().numpy(), [tokens[r] for r in few], 11, 8)
    rel = (vocab / 1024 + 16) * 2.0 ** -24 + 2.0 ** -21       # 128 threads instead of the 256 of a cluster's CTAs: half as many rows' ends, at most vocab / 1024 pieces of 8 each
    assert np.array_equal(ids[few], wi)
    S.close(lp[few], wl, 2.0 ** -22 * np.abs(np.where(np.isfinite(wl), wl, 0)) + 2 * rel)
    S.close(en[few], we, 2.0 ** -22 * np.abs(we) + rel * (4 + 2 * np.abs(we)))
    S.close(tops[few], wt, 2.0 ** -22 * np.abs(wt) + 2 * rel)


def crowded(rows, vocab, dtype, threads, parts, seed):
    """Rows whose alternatives are narrowed down in several rounds.  A row is taken in pieces of 16 bytes, piece i of a part by thread i % threads; the last warp's threads, and one of each
    other warp's, hold nothing above 1, so that 1 is the bound of the first look, while a few threads hold hundreds of 2 (more than `threads` in all) and 40 values above that: those are
    too few, or lie too close together, to be the next bound every time."""
    rng = np.random.default_rng(seed)
    N = 8 if dtype == torch.bfloat16 else 4
    pieces = vocab // N
    per = -(-pieces // parts)
    x = -5 - rng.random((rows, pieces, N))
    i = np.arange(per)
    high = (i % threads < threads - 32) & (i % 32 != 31)
    x[:, i[~high], 0] = 1
    for r in range(rows):
        few = rng.permutation(np.unique(i[high] % threads))
        mine = i[np.isin(i % threads, few[:1 + (threads + 40) // (N * max(1, per // threads))])]
        x[r, mine] = 2
        at = rng.choice(len(mine) * N, 40, replace=False)
        x[r, mine[at // N], at % N] = 3 + rng.integers(0, 30, 40) * 0.125
        assert threads < (x[r] >= 2).sum() and (x[r, :per] >= 1).sum() <= 2048
    x = x.reshape(rows, -1)
    return torch.from_numpy(np.concatenate([x, np.full((rows, vocab - x.shape[1]), -9.0)], 1)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,threads,parts", [(320, 20008, 128, 1), (4, 50304, 256, 8), (60, 32000, 256, 4)])
def test_alternatives_narrowed_down_in_several_rounds(dm, dtype, rows, vocab, threads, parts):
    for seed in range(3):
        S.check(dm, crowded(rows, vocab, dtype, threads, parts, seed), [(r * 7919) % vocab for r in range(rows)], -1, 32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [0, 1, 2, 3, 4, 5, 6, 7])
def test_masked_rows_at_any_alignment(dm, dtype, shift):
    """Far from zero and beginning anywhere between two 16-byte pieces: the first piece is an end of the row, and what follows it belongs to other threads."""
    V = 9001
    low = torch.finfo(dtype).min
    x = torch.randn(8, V, generator=torch.Generator().manual_seed(3)).to(dtype)
    x[0] = low
    x[1] = torch.finfo(dtype).max
    x[2] = 1e30
    x[3] = -1e30; x[3, 9] = -0.5e30
    x[4] = low; x[4, :3] = 1.0
    x[5] = -1e9; x[5, 4000:4003] = 1.5
    x[6] = 3e6; x[6, 5] = 3.5e6
    x[7] = -math.inf; x[7, 1::2] = -2.5e7
    for ld in (V, V + 7):
        store = torch.full((8 * ld + 16,), 1e30, dtype=dtype, device="cuda")
        y = store[shift:shift + 8 * ld].view(8, ld)
        y[:, :V] = x
        S.check(dm, y, [5, 9000, 0, 9, 2, 4001, 5, 1], -1, 8, V)
        S.check(dm, y, [5, 9000, 0, 9, 2, 4001, 5, 1], 1, 8, V)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [16, 320])
def test_one_id_left_by_a_finite_mask(dm, dtype, rows):
    """All ids but one masked with the type's lowest value, the one in each piece of the first rounds in turn, rows at every alignment: it is certain."""
    V, N = 50257 if rows == 16 else 20011, 8 if dtype == torch.bfloat16 else 4
    x = torch.full((rows, V), torch.finfo(dtype).min, dtype=dtype, device="cuda")
    at = [(r * (V // 16) + 3) % V if r % 3 == 0 else ((128 if rows > 296 else 256) * (1 + r % 7) * N + r % (2 * N)) % V for r in range(rows)]
    at[1] = 5
    x[torch.arange(rows), at] = 2.25
    lp, en, ids, tops = S.run(dm, x, at, -1, 3)
    rel = (V / 1024 + 16) * 2.0 ** -24 + 2.0 ** -21           # the bounds of test_gpu_token_scores.py, where log p = H = 0
    assert np.array_equal(ids[:, 0], at) and np.all(np.abs(lp) <= 2 * rel) and np.all(np.abs(en) <= 4 * rel) and np.array_equal(tops[:, 0], lp)
    assert np.all(tops[:, 1:] <= torch.finfo(dtype).min) and np.array_equal(ids[:, 1], [0 if a else 1 for a in at])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [3, 400])
def test_log_probabilities_of_masked_ids_are_finite(dm, dtype, rows):
    """A finite mask, the type's lowest value included, gives a finite log probability, x minus the logarithm of the sum, wherever that is not below fp32's range."""
    V, low = 8200, torch.finfo(dtype).min
    x = torch.randn(rows, V, generator=torch.Generator().manual_seed(6)).to(dtype).cuda()
    x[0, 5:] = low
    x[1, 5:] = -2e6
    x[2] = low; x[2, 7] = -3e38
    t = [77 + r for r in range(rows)]
    few = [0, 1, 2, rows - 1]
    lp, en, ids, tops = S.run(dm, x, t, -1, 12)
    wl, we, wi, wt = K.token_scores(x[few].double().cpu().numpy(), [t[r] for r in few], -1, 12)
    assert np.isfinite(lp).all() and np.isfinite(tops).all() and lp[0] <= float(low) and np.array_equal(ids[few], wi)
    rel = (V / 1024 + 16) * 2.0 ** -24 + 2.0 ** -21
    for got, want in ((lp[few], wl), (tops[few], wt)):
        S.close(got, want, 2.0 ** -22 * np.abs(want) + 2 * rel)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [40, 700])
def test_no_probability_is_above_one(dm, dtype, rows):
    """Certain ids of every magnitude: the exponential of a log probability is never above 1, nor an entropy below 0."""
    V = 5000
    x = torch.full((rows, V), -1e4, dtype=dtype)
    at = torch.arange(rows) * 7 % V
    x[torch.arange(rows), at] = torch.exp(torch.linspace(-3, 9, rows)).to(dtype)
    lp, en, ids, tops = S.run(dm, x.cuda(), at.tolist(), -1, 2)
    rel = (V / 1024 + 16) * 2.0 ** -24 + 2.0 ** -21
    assert np.array_equal(ids[:, 0], at.numpy()) and np.all(lp <= 0) and np.all(lp >= -2 * rel) and np.all(tops <= 0) and np.all(en >= 0) and np.all(en <= 4 * rel)


# ---- streams and graphs -----------------------------------------------------------------------------------------------------------------

def test_two_streams_and_two_graphs_at_once(dm):
    """Append, attention with weights, eviction and scores: eager on one stream, and two captured graphs on two others with buffers of their own, all at the same time and
    replayed, give the same bits."""
    rng = np.random.default_rng(41)
    B, G, H, D, cap, keep, V = 3, 4, 2, 64, 4096, 600, 5003
    cfg = dm.dm_kv8_cfg(B, G, H, H, D, dm.DM_BF16)
    start = T.random_cache(3, B, H, cap, D, [cap] * B, rubbish=False)
    width = 3 * H * D
    x = torch.from_numpy(rng.normal(size=(B * G, width))).to(torch.bfloat16).cuda()
    logits = torch.from_numpy(rng.normal(size=(B * G, V)) * 3).to(torch.bfloat16).cuda()
    tokens = T.i32(rng.integers(0, V, B * G).tolist())
    nb, ne = dm.dm_kv8_attention_workspace_bytes(cfg, cap), dm.dm_kv8_evict_workspace_bytes(cfg, cap, keep)

    class Side:
        def __init__(self):
            self.a, self.b = T.to_gpu(start), T.to_gpu(T.random_cache(4, B, H, 608, D, [0] * B, rubbish=False))
            self.n, self.m = T.i32([4000, 17, 1500]), T.i32([0] * B)
            self.acc, self.acc2 = torch.zeros(B, H, cap, device="cuda"), torch.zeros(B, H, 608, device="cuda")
            self.out = torch.zeros(B * G, H * D, dtype=torch.bfloat16, device="cuda")
            self.lp, self.en = torch.zeros(B * G, device="cuda"), torch.zeros(B * G, device="cuda")
            self.ids, self.tops = torch.zeros(B * G, 5, dtype=torch.int32, device="cuda"), torch.zeros(B * G, 5, device="cuda")
            self.ws, self.we = T.workspace(nb), T.workspace(ne)

        def step(self, s):
            p = x.data_ptr()
            dm.dm_kv8_append(cfg, T.handle(dm, self.a), p + 2 * H * D, p + 4 * H * D, width, self.n.data_ptr(), 0, s)
            dm.dm_kv8_attention(cfg, T.handle(dm, self.a), p, width, self.n.data_ptr(), 0, cap, self.acc.data_ptr(), self.acc.data_ptr(), self.out.data_ptr(), H * D,
                                self.ws.data_ptr(), nb, s)
            dm.dm_kv8_evict(cfg, T.handle(dm, self.a), T.handle(dm, self.b), self.acc.data_ptr(), self.acc2.data_ptr(), self.n.data_ptr(), self.m.data_ptr(), cap, keep, 100, 0,
                            self.we.data_ptr(), ne, s)
            dm.dm_token_scores(B * G, V, V, dm.DM_BF16, logits.data_ptr(), tokens.data_ptr(), 7, 5, self.lp.data_ptr(), self.en.data_ptr(), self.ids.data_ptr(),
                               self.tops.data_ptr(), s)

        def results(self):
            return [self.b["k"], self.b["v"], self.b["ks"], self.b["vs"], self.m, self.acc, self.acc2, self.out, self.lp, self.en, self.ids, self.tops]

    sides, streams = [Side() for _ in range(3)], [torch.cuda.Stream() for _ in range(3)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for i in range(2):
        with torch.cuda.stream(streams[i]), torch.cuda.graph(graphs[i], stream=streams[i]):
            sides[i].step(streams[i].cuda_stream)
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        sides[2].step(streams[2].cuda_stream)
    torch.cuda.synchronize()
    dm.dm_check(T.stream())
    for r0, r1, r2 in zip(*(s.results() for s in sides)):
        assert torch.equal(r0, r2) and torch.equal(r1, r2)
    assert sides[2].m.tolist() == [600, 17, 600] and sides[2].ids.min() >= 0
