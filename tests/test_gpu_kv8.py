"""The 8-bit key/value cache on the GPU against the fp64 oracle: append and evict bit by bit, attention and accumulated weights within derived bounds.

Bounds.  Attention: the output's rounding to bf16 is half a step, 2^-8 of the value; P's rounding to f16 is 2^-11 of each term, so 2^-11 sum_j p_j |v_j|; a score's error
is that of D + 8 fp32 additions of terms that sum to `reach` in magnitude, twice that in log2 units, and shifts p and the normalisation by as much each.
Weights: fp32 throughout, the scores' error and one rounding per addition.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import kv8_oracle as K


@pytest.fixture(scope="module")
def dm():
    from paper_2511_15927_b200 import build
    build.build()
    from paper_2511_15927_b200 import binding
    return binding


torch = pytest.importorskip("torch")


def random_cache(seed, B, H, cap, D, lens, rubbish=True):
    """Codes and scales as appending leaves them; behind each sequence's rows anything, NaN codes and wild scales included."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(2, B, H, cap, D)) * np.exp(rng.normal(size=(2, B, H, 1, D)) * 0.5)
    c = {}
    for i, n in enumerate("kv"):
        s = np.array([[[K.scale_of(x[i, b, h, j * 32:(j + 1) * 32]) for j in range(cap // 32)] for h in range(H)] for b in range(B)])
        codes = K.encode(x[i] / np.repeat(s, 32, -1)[..., None])
        if rubbish:
            for b in range(B):
                codes[b, :, lens[b]:] = rng.integers(0, 256, codes[b, :, lens[b]:].shape)
                codes[b, :, lens[b]:, ::3] = 0x7f
                s[b, :, -(-lens[b] // 32):] = math.nan
        c[n], c[n + "s"] = codes, s
    c["v"] = K.v_blocks(c["v"])
    return c


def to_gpu(c):
    return {n: torch.from_numpy(np.ascontiguousarray(c[n] if n in "kv" else c[n].astype(np.float32))).cuda() for n in ("k", "v", "ks", "vs")}


def to_cpu(d):
    return {n: d[n].cpu().numpy().astype(np.float64 if n.endswith("s") else np.uint8) for n in ("k", "v", "ks", "vs")}


def same(a, b):
    for n in ("k", "v", "ks", "vs"):
        assert np.array_equal(a[n], b[n], equal_nan=n.endswith("s")), (n, np.argwhere(~((a[n] == b[n]) | (a[n] != a[n])))[:5])


def handle(dm, d):
    return dm.dm_kv8_cache(d["k"].data_ptr(), d["v"].data_ptr(), d["ks"].data_ptr(), d["vs"].data_ptr(), d["k"].shape[2])


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def stream():
    return torch.cuda.current_stream().cuda_stream


def workspace(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda").fill_(0xff)


# ---- append ---------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,G,lens,counts", [
    (64, 2, 1, [0, 31, 32, 63], None), (80, 3, 32, [0, 5, 32, 95], None), (128, 1, 33, [0, 1], [33, 0]), (64, 2, 100, [3, 64, 17], [100, 1, 50]),
    (80, 1, 7, [123, 126, 128, 200], [7, 7, 7, 7])])     # the last: rows past the capacity of 128 are dropped
def test_append(dm, dtype, D, H, G, lens, counts):
    rng = np.random.default_rng(D + G)
    B, cap = len(lens), 128 if G <= 33 else 192
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    ld = 2 * H * D + 24 if dtype == "bf16" else 2 * H * D + 12           # [K | V | something else]
    x = torch.from_numpy(rng.normal(size=(B * G, ld)).astype(np.float32) * np.exp(rng.normal(size=(B * G, 1)) * 4)).to(t).cuda()
    c = random_cache(1, B, H, cap, D, [min(n, cap) for n in lens])
    d = to_gpu(c)
    cfg = dm.dm_kv8_cfg(B, G, H, H, D, dm.DM_BF16 if dtype == "bf16" else dm.DM_F32)
    n, m = i32(lens), i32(counts or [G] * B)
    dm.dm_kv8_append(cfg, handle(dm, d), x.data_ptr(), x.data_ptr() + H * D * x.element_size(), ld, n.data_ptr(), m.data_ptr() if counts else 0, stream())
    dm.dm_check(stream())
    host = x.double().cpu().numpy().reshape(B, G, ld)
    want = K.append(c, host[:, :, :H * D].reshape(B, G, H, D), host[:, :, H * D:2 * H * D].reshape(B, G, H, D), [min(v, cap) for v in lens], counts or [G] * B)
    same(to_cpu(d), want)
    assert n.tolist() == lens


def test_append_of_special_values(dm):
    """Zeros of both signs, infinities, NaN, the smallest and the largest values of bf16, a block of nothing but them."""
    B, G, H, D = 1, 64, 1, 64
    x = torch.zeros(G, 2 * D, dtype=torch.bfloat16)
    x[0, :6] = torch.tensor([-0.0, math.inf, -math.inf, math.nan, 1e-40, -1.5])
    x[1, 64:70] = torch.tensor([3.38e38, -3.38e38, math.inf, 1.0, 1e-30, -math.nan])
    x[32, :3] = torch.tensor([math.nan, math.inf, 1e-38])
    d = to_gpu(random_cache(0, 1, 1, 64, D, [0]))
    xg = x.cuda()
    n = i32([0])
    dm.dm_kv8_append(dm.dm_kv8_cfg(B, G, H, H, D, dm.DM_BF16), handle(dm, d), xg.data_ptr(), xg.data_ptr() + 2 * D, 2 * D, n.data_ptr(), 0, stream())
    dm.dm_check(stream())
    host = x.double().numpy().reshape(B, G, 2, D)
    want = K.append(random_cache(0, 1, 1, 64, D, [0]), host[:, :, :1], host[:, :, 1:], [0], [G])
    got = to_cpu(d)
    same(got, want)
    assert got["k"][0, 0, 0, 1] == got["k"][0, 0, 0, 3] == 0x7f and got["ks"][0, 0, 1] == K.FLOOR


# ---- attention ------------------------------------------------------------------------------------------------------------------------

def run_attention(dm, c, q, lens, counts, max_len, acc=None, out=None, alias=False, ws=None):
    B, G, Hq, D = q.shape
    d = c if isinstance(c["k"], torch.Tensor) else to_gpu(c)
    cfg = dm.dm_kv8_cfg(B, G, Hq, d["k"].shape[1], D, dm.DM_BF16)
    ldq, ldo = Hq * D + 16, Hq * D + 8
    qg = torch.full((B * G, ldq), math.nan, dtype=torch.bfloat16, device="cuda")
    qg[:, :Hq * D] = torch.from_numpy(q.reshape(B * G, -1)).to(torch.bfloat16)
    out = torch.full((B * G, ldo), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    n, m = i32(lens), i32(counts or [G] * B)
    nb = dm.dm_kv8_attention_workspace_bytes(cfg, max_len)
    ws = workspace(nb) if ws is None else ws
    ai = torch.from_numpy(acc.astype(np.float32)).cuda() if acc is not None else None
    ao = ai if alias else torch.full_like(ai, -5.0) if acc is not None else None
    dm.dm_kv8_attention(cfg, handle(dm, d), qg.data_ptr(), ldq, n.data_ptr(), m.data_ptr() if counts else 0, max_len, ai.data_ptr() if acc is not None else 0,
                        ao.data_ptr() if acc is not None else 0, out.data_ptr(), ldo, ws.data_ptr(), ws.numel(), stream())
    dm.dm_check(stream())
    o = out.double().cpu().numpy()
    assert np.all(o[:, Hq * D:] == 7)
    return o[:, :Hq * D].reshape(B, G, Hq, D), None if acc is None else ao.double().cpu().numpy()


def check_attention(got, c, q, lens, counts, acc=None, acc_got=None, fill=-5.0):
    B, G, Hq, D = q.shape
    counts = counts or [G] * B
    want, acc_want, spread, reach = K.attend(c, q, lens, counts, acc)
    ds = reach[..., None] / math.sqrt(D) * (D + 8) * 2.0 ** -23 * 2
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * ds + 2.0 ** -18) * spread + 1e-30
    for b in range(B):
        assert np.all(got[b, counts[b]:] == 7), "rows of padding tokens were written"
        live = slice(0, counts[b])
        err = np.abs(got[b, live] - want[b, live])
        assert np.array_equal(np.isnan(got[b, live]), np.isnan(want[b, live]))
        ok = (err <= tol[b, live]) | np.isnan(want[b, live])
        assert ok.all(), (b, float(np.nanmax(err / tol[b, live])))
    if acc is not None:
        there = ~np.isnan(acc_want)
        assert np.all(acc_got[~there] == fill if fill is not None else True)
        group = Hq // c["k"].shape[1]
        bound = (2 * ds.max() + (group * G + 16) * 2.0 ** -23) * np.abs(np.where(there, acc_want, 0)) + 1e-30
        err = np.abs(np.where(there, acc_got - acc_want, 0))
        assert np.all(err <= bound), float((err / bound).max())


CASES = [  # D, query heads, kv heads, block, lens, counts, cap
    (64, 2, 2, 1, [0, 1, 31, 32], None, 96),
    (64, 4, 1, 3, [0, 5, 100], [3, 0, 2], 128),
    (80, 3, 3, 32, [7, 60, 200], None, 288),
    (80, 4, 2, 5, [33, 255], [5, 1], 288),
    (128, 8, 2, 1, [300, 1], None, 320),
    (128, 2, 2, 17, [64, 65, 0], [17, 16, 0], 96),
    (64, 2, 2, 64, [500, 129], None, 608),
    (64, 16, 1, 9, [250, 11], None, 288),
    (80, 1, 1, 33, [1500], None, 1536),
    (64, 1, 1, 1, [2000], None, 2048),
]


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("D,Hq,H,G,lens,counts,cap", CASES)
def test_attention(dm, D, Hq, H, G, lens, counts, cap, weights):
    rng = np.random.default_rng(G * D)
    B = len(lens)
    n = [a + b for a, b in zip(lens, counts or [G] * B)]
    c = random_cache(5, B, H, cap, D, n)
    q = torch.from_numpy(rng.normal(size=(B, G, Hq, D)) * np.exp(rng.normal(size=(B, G, Hq, 1)))).to(torch.bfloat16).double().numpy()
    acc = rng.random((B, H, cap)) if weights else None
    got, acc_got = run_attention(dm, c, q, lens, counts, max(lens), acc)
    check_attention(got, c, q, lens, counts, np.float32(acc).astype(np.float64) if weights else None, acc_got)


def test_attention_of_extreme_queries_and_scales(dm):
    """Rows of Q from 2^-100 to 2^100 and with channels 2^30 apart, scales of neighbouring blocks far apart, one key far ahead of all the others."""
    rng = np.random.default_rng(9)
    D, n, cap = 64, 400, 416
    c = random_cache(3, 1, 1, cap, D, [n], rubbish=False)
    c["vs"] *= 2.0 ** rng.integers(-40, 40, c["vs"].shape)
    c["ks"][0, 0, 4] *= 16
    q = rng.normal(size=(1, 6, 1, D))
    q[0, 1] *= 2.0 ** -100
    q[0, 2] *= 30
    q[0, 3, :, ::2] *= 2.0 ** -30
    q[0, 4] = 0
    c["ks"][0, 0, 7] = 2.0 ** -100
    q = torch.from_numpy(q).to(torch.bfloat16).double().numpy()
    got, _ = run_attention(dm, c, q, [n - 6], None, n - 6)
    check_attention(got, c, q, [n - 6], None)
    # huge queries against a cache of tiny scale: every product is ordinary again
    c["ks"] = np.full_like(c["ks"], 2.0 ** -90)
    got, _ = run_attention(dm, c, q * 2.0 ** 84, [n - 6], None, n - 6)
    check_attention(got, c, q * 2.0 ** 84, [n - 6], None)


def test_flat_attention_over_many_rows(dm):
    """Equal scores and one peak e^20 above 30000 others: small probabilities must not be lost."""
    D, n = 64, 30000
    cap = (n + 31) // 32 * 32
    rng = np.random.default_rng(4)
    c = random_cache(8, 1, 1, cap, D, [n], rubbish=False)
    c["k"][:] = 0
    c["v"] &= 0x7f                                   # positive values: nothing cancels
    c["k"][0, 0, 777, 0] = K.encode(np.array([1.0]))[0]
    c["ks"][:] = 1
    q = np.zeros((1, 2, 1, D))
    q[0, 1, 0, 0] = 8 * 18.0                         # s = 18 at the peak, 0 elsewhere
    got, _ = run_attention(dm, c, q, [n - 2], None, n)
    check_attention(got, c, q, [n - 2], None)


def test_nan_codes_show_where_they_are_read(dm):
    c = random_cache(2, 2, 1, 64, 64, [40, 40], rubbish=False)
    c["k"][0, 0, 3, 5] = 0x7f
    c["v"][1, 0, 1, 9, 2] = 0xff                     # sequence 1, channel 9, row 34
    q = np.ones((2, 2, 1, 64)) * 0.125
    got, _ = run_attention(dm, c, q, [38, 38], None, 38)
    assert np.isnan(got[0]).all()
    assert np.isnan(got[1, :, 0, 9]).all() and not np.isnan(np.delete(got[1], 9, -1)).any()


def test_lengths_beyond_the_cache_or_max_len_are_cut(dm):
    c = random_cache(6, 3, 2, 96, 64, [96, 96, 96], rubbish=False)
    q = np.random.default_rng(0).normal(size=(3, 1, 2, 64)).astype(np.float32)
    q = torch.from_numpy(q).to(torch.bfloat16).double().numpy()
    got, _ = run_attention(dm, c, q, [500, -3, 95], None, 2000)
    check_attention(got, c, q, [96, 0, 95], None)
    got, _ = run_attention(dm, c, q, [60, 90, 10], None, 31)
    check_attention(got, c, q, [31, 31, 10], None)


def test_results_do_not_depend_on_the_rows_beside_or_the_run(dm):
    D, cap = 80, 3200
    lens = [3000, 17, 900]
    c = random_cache(11, 3, 2, cap, D, [n + 4 for n in lens])
    q = torch.from_numpy(np.random.default_rng(1).normal(size=(3, 4, 2, D))).to(torch.bfloat16).double().numpy()
    acc = np.zeros((3, 2, cap))
    a, wa = run_attention(dm, c, q, lens, None, 3000, acc)
    b, wb = run_attention(dm, c, q, lens, None, 3000, acc, alias=True)
    assert np.array_equal(a, b)
    for i, n in enumerate(lens):
        assert np.array_equal(wa[i, :, :n + 4], wb[i, :, :n + 4])
    assert np.allclose(wa[:, :, :10].sum() + wa[:, :, 10:].clip(0).sum(), 3 * 2 * 4, rtol=1e-5)


def test_long_cache_offsets_past_32_bits(dm):
    """20 heads' codes past 4 GiB: the last sequence reads the right rows."""
    D, H, cap, B = 128, 8, 1 << 20, 5
    k = torch.zeros(B, H, cap, D, dtype=torch.uint8, device="cuda")
    v = torch.zeros(B, H, cap // 32, D, 32, dtype=torch.uint8, device="cuda")
    ks, vs = (torch.ones(B, H, cap // 32, device="cuda") for _ in range(2))
    assert k.numel() > 1 << 32
    n = 200
    small = random_cache(13, 1, H, 224, D, [n])
    k[-1, :, :224] = torch.from_numpy(small["k"][0]).cuda()
    v[-1, :, :7] = torch.from_numpy(small["v"][0]).cuda()
    ks[-1, :, :7] = torch.from_numpy(small["ks"][0]).cuda()
    vs[-1, :, :7] = torch.from_numpy(small["vs"][0]).cuda()
    q = torch.from_numpy(np.random.default_rng(3).normal(size=(B, 1, H, D))).to(torch.bfloat16).double().numpy()
    got, _ = run_attention(dm, {"k": k, "v": v, "ks": ks, "vs": vs}, q, [1, 1, 1, 1, n - 1], None, cap - 1)
    check_attention(got[-1:], small, q[-1:], [n - 1], None)
    assert np.all(got[:-1] == 0)


# ---- evict ----------------------------------------------------------------------------------------------------------------------------

def run_evict(dm, c, acc, lens, keep, recent, dst, acc_dst, max_len=None, rows=True):
    B, H, cap, D = c["k"].shape
    s, d = to_gpu(c), to_gpu(dst)
    cfg = dm.dm_kv8_cfg(B, 1, H, H, D, dm.DM_BF16)
    ai, ao = torch.from_numpy(acc.astype(np.float32)).cuda(), torch.from_numpy(acc_dst.astype(np.float32)).cuda()
    li, lo, r = i32(lens), i32([-9] * B), torch.full((B, H, keep), -7, dtype=torch.int32, device="cuda")
    max_len = max(lens) if max_len is None else max_len
    nb = dm.dm_kv8_evict_workspace_bytes(cfg, max_len, keep)
    ws = workspace(nb)
    dm.dm_kv8_evict(cfg, handle(dm, s), handle(dm, d), ai.data_ptr(), ao.data_ptr(), li.data_ptr(), lo.data_ptr(), max_len, keep, recent, r.data_ptr() if rows else 0,
                    ws.data_ptr(), nb, stream())
    dm.dm_check(stream())
    same(to_cpu(s), {n: np.float32(c[n]).astype(np.float64) if n.endswith("s") else c[n] for n in c})
    return to_cpu(d), ao.cpu().numpy(), lo.cpu().numpy(), r.cpu().numpy()


@pytest.mark.parametrize("D,H,cap,lens,keep,recent,scores", [
    (64, 2, 96, [0, 1, 33, 96], 33, 5, "random"), (80, 1, 320, [300, 320, 31], 64, 64, "random"), (128, 2, 160, [150, 129], 70, 0, "random"),
    (64, 1, 512, [500, 77], 100, 30, "ties"), (80, 2, 256, [256], 1, 0, "random"), (64, 1, 256, [255], 200, 1, "special"), (80, 1, 64, [64, 50], 64, 3, "random"),
    (64, 1, 9600, [9600, 5000], 4000, 100, "random"), (128, 1, 96, [90], 40, 7, "equal")])
def test_evict(dm, D, H, cap, lens, keep, recent, scores):
    rng = np.random.default_rng(keep)
    B = len(lens)
    c = random_cache(21, B, H, cap, D, lens)
    for n in ("ks", "vs"):                           # scales of neighbouring blocks apart, so that rows change theirs
        c[n] = c[n] * 2.0 ** rng.integers(-6, 7, c[n].shape)
    acc = np.float32(np.exp(rng.normal(size=(B, H, cap)) * 2))
    if scores == "ties":
        acc = np.float32(rng.integers(0, 4, acc.shape))
    elif scores == "equal":
        acc[:] = 0.25
    elif scores == "special":
        acc[..., ::5] = math.nan
        acc[..., 1::7] = math.inf
        acc[..., 2::7] = -0.0
        acc[..., 3::7] = 0.0
        acc[..., 4::11] = -1.0
        acc[..., 5::11] = 1e-42
    dst = random_cache(22, B, H, (keep + 31) // 32 * 32 + 32, D, [0] * B)
    acc_dst = rng.random((B, H, dst["k"].shape[2])).astype(np.float32)
    want, a, n, r = K.evict(c, acc, np.array(lens), keep, recent, dst, acc_dst)
    got, ga, gn, gr = run_evict(dm, c, acc, lens, keep, recent, dst, acc_dst)
    assert np.array_equal(gn, n) and np.array_equal(gr, r) and np.array_equal(ga, a, equal_nan=True)
    same(got, want)


def test_evict_cuts_lengths_to_max_len(dm):
    c = random_cache(1, 2, 1, 96, 64, [96, 96], rubbish=False)
    acc = np.random.default_rng(0).random((2, 1, 96)).astype(np.float32)
    dst = random_cache(2, 2, 1, 96, 64, [0, 0])
    got = run_evict(dm, c, acc, [900, 20], 50, 10, dst, np.zeros((2, 1, 96), np.float32), max_len=60, rows=False)
    want = K.evict(c, acc, np.array([60, 20]), 50, 10, dst, np.zeros((2, 1, 96), np.float32))
    same(got[0], want[0])
    assert got[2].tolist() == [50, 20]
    got = run_evict(dm, c, acc, [900, 20], 50, 10, dst, np.zeros((2, 1, 96), np.float32), max_len=0, rows=True)
    assert got[2].tolist() == [0, 0] and np.all(got[3] == -1)
    same(got[0], dst)


# ---- together -------------------------------------------------------------------------------------------------------------------------

def test_decoding_with_a_bounded_cache(dm):
    """Blocks are appended and attended to, weights accumulate, the cache is cut when it is full, and decoding goes on in the other one: every step against the oracle
    carried along in the same way."""
    rng = np.random.default_rng(17)
    B, G, Hq, H, D, cap, keep, recent = 2, 32, 4, 2, 64, 160, 64, 40
    cfg = dm.dm_kv8_cfg(B, G, Hq, H, D, dm.DM_BF16)
    ref, other = random_cache(0, B, H, cap, D, [0] * B), random_cache(1, B, H, cap, D, [0] * B)
    gpu = [to_gpu(ref), to_gpu(other)]
    acc = np.zeros((B, H, cap))
    accs = [torch.zeros(B, H, cap, device="cuda"), torch.zeros(B, H, cap, device="cuda")]
    lens, glens = [0] * B, [i32([0] * B), i32([0] * B)]
    width = (Hq + 2 * H) * D
    nb = max(dm.dm_kv8_attention_workspace_bytes(cfg, cap), dm.dm_kv8_evict_workspace_bytes(cfg, cap, keep))
    ws, out = workspace(nb), torch.zeros(B * G, Hq * D, dtype=torch.bfloat16, device="cuda")
    cur = 0
    for step in range(8):
        counts = [G, int(rng.integers(1, G + 1))]
        if max(lens) + G > cap:
            dm.dm_kv8_evict(cfg, handle(dm, gpu[cur]), handle(dm, gpu[1 - cur]), accs[cur].data_ptr(), accs[1 - cur].data_ptr(), glens[cur].data_ptr(), glens[1 - cur].data_ptr(),
                            cap, keep, recent, 0, ws.data_ptr(), nb, stream())
            a32 = accs[cur].cpu().numpy().astype(np.float64)      # the same weights for both: they agree to a few units in the last place, a choice may not
            assert np.allclose(np.where(np.arange(cap) < np.array(lens)[:, None, None], a32 - acc, 0), 0, atol=1e-4)
            other = to_cpu(gpu[1 - cur])
            ref, acc, n, _ = K.evict(ref, a32, np.array(lens), keep, recent, {**other}, np.zeros((B, H, cap)))
            lens, cur = n.tolist(), 1 - cur
            dm.dm_check(stream())
            got = to_cpu(gpu[cur])
            for b in range(B):
                assert np.array_equal(got["k"][b, :, :lens[b]], ref["k"][b, :, :lens[b]])
            assert glens[cur].tolist() == lens
        x = torch.from_numpy(rng.normal(size=(B * G, width)) * 1.5).to(torch.bfloat16).cuda()
        q, kp, vp = x.data_ptr(), x.data_ptr() + Hq * D * 2, x.data_ptr() + (Hq + H) * D * 2
        m = i32(counts)
        dm.dm_kv8_append(cfg, handle(dm, gpu[cur]), kp, vp, width, glens[cur].data_ptr(), m.data_ptr(), stream())
        dm.dm_kv8_attention(cfg, handle(dm, gpu[cur]), q, width, glens[cur].data_ptr(), m.data_ptr(), cap, accs[cur].data_ptr(), accs[cur].data_ptr(), out.data_ptr(), Hq * D,
                            ws.data_ptr(), nb, stream())
        dm.dm_check(stream())
        host = x.double().cpu().numpy().reshape(B, G, Hq + 2 * H, D)
        ref = K.append(ref, host[:, :, Hq:Hq + H], host[:, :, Hq + H:], lens, counts)
        for b in range(B):
            assert np.array_equal(to_cpu(gpu[cur])["k"][b, :, :lens[b] + counts[b]], ref["k"][b, :, :lens[b] + counts[b]])
        got = out.double().cpu().numpy().reshape(B, G, Hq, D).copy()
        for b in range(B):
            got[b, counts[b]:] = 7
        before = acc.copy()
        check_attention(got, ref, host[:, :, :Hq], lens, counts)
        _, acc, _, _ = K.attend(ref, host[:, :, :Hq], lens, counts, before)
        acc = np.nan_to_num(acc)
        lens = [a + b for a, b in zip(lens, counts)]
        glens[cur] += m
    assert max(lens) <= cap


def test_captured_graph_follows_the_lengths(dm):
    """One graph of append and attention, replayed with other lengths, inputs and on a stream of its own: the same bits as eager calls."""
    rng = np.random.default_rng(23)
    B, G, H, D, cap = 2, 8, 2, 80, 1024
    cfg = dm.dm_kv8_cfg(B, G, H, H, D, dm.DM_BF16)
    start = random_cache(3, B, H, cap, D, [cap, cap], rubbish=False)
    g, e = to_gpu(start), to_gpu(start)
    width = 3 * H * D
    x = torch.zeros(B * G, width, dtype=torch.bfloat16, device="cuda")
    nb = dm.dm_kv8_attention_workspace_bytes(cfg, cap)
    n, ws, out = i32([5, 900]), workspace(nb), torch.zeros(B * G, H * D, dtype=torch.bfloat16, device="cuda")
    acc = torch.zeros(B, H, cap, device="cuda")

    def step(d, w, o, a, s):
        q = x.data_ptr()
        dm.dm_kv8_append(cfg, handle(dm, d), q + 2 * H * D, q + 4 * H * D, width, n.data_ptr(), 0, s)
        dm.dm_kv8_attention(cfg, handle(dm, d), q, width, n.data_ptr(), 0, cap, a.data_ptr(), a.data_ptr(), o.data_ptr(), H * D, w.data_ptr(), nb, s)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(g, ws, out, acc, side.cuda_stream)
    out2, acc2, ws2 = torch.zeros_like(out), torch.zeros_like(acc), workspace(nb)
    for lens in ([5, 900], [0, 1000], [700, 33]):
        torch.cuda.synchronize()
        n.copy_(i32(lens))
        x.copy_(torch.from_numpy(rng.normal(size=(B * G, width))).to(torch.bfloat16))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        step(e, ws2, out2, acc2, stream())
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(acc, acc2)
        assert all(torch.equal(g[k], e[k]) for k in ("k", "v"))
    dm.dm_check(stream())
