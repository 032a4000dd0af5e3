"""The 8-bit cache and the token scores without a GPU: pins of the fp64 oracle, and what the library refuses (nothing is launched)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as K


def test_code_values_are_e4m3():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(K.VALUES, want, equal_nan=True)


def test_encode_rounds_to_nearest_even():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * np.exp(rng.normal(size=4000) * 3), K.VALUES[~np.isnan(K.VALUES)], [0.0, -0.0, 2.0 ** -10, -2.0 ** -10, 3 * 2.0 ** -10, 447.9]])
    mids = (K.VALUES[:0x7e] + K.VALUES[1:0x7f]) / 2                      # every tie
    x = np.concatenate([x, mids, -mids])
    x = np.float32(x[np.abs(x) <= 448]).astype(np.float64)
    want = torch.from_numpy(np.float32(x)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(K.encode(x), want)
    assert np.array_equal(K.encode(np.array([math.nan, math.inf, -math.inf])), [0x7f] * 3)


def test_scale_is_the_smallest_power_of_two():
    for top, s in ((448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1.75, 2.0 ** -8), (1.7501, 2.0 ** -7), (0.0, K.FLOOR), (1e-40, K.FLOOR), (3e38, 2.0 ** 120)):
        assert K.scale_of(np.array([top, -top / 2, math.nan, math.inf])) == s


def test_moving_a_row_to_another_scale_loses_nothing_above_the_smallest_normal_code():
    codes = np.arange(0x08, 0x7f)                                        # normal values
    for up in range(0, 5):
        x = K.VALUES[codes] * 2.0 ** -up
        keep = np.abs(x) >= 2.0 ** -6
        assert np.array_equal(K.VALUES[K.encode(x)][keep], x[keep])


def _cache(rng, B, H, cap, D):
    c = {"k": rng.integers(0, 256, (B, H, cap, D)).astype(np.uint8), "v": rng.integers(0, 256, (B, H, cap // 32, D, 32)).astype(np.uint8),
         "ks": 2.0 ** rng.integers(-8, 1, (B, H, cap // 32)), "vs": 2.0 ** rng.integers(-8, 1, (B, H, cap // 32))}
    for n in ("k", "v"):
        c[n][(c[n] & 0x7f) == 0x7f] = 0x11
    return c


def test_append_keeps_what_it_does_not_write():
    rng = np.random.default_rng(1)
    c = _cache(rng, 2, 2, 96, 16)
    new = rng.normal(size=(2, 2, 5, 2, 16))
    got = K.append(c, new[0], new[1], [30, 7], [5, 0])
    assert np.array_equal(got["k"][1], c["k"][1]) and np.array_equal(got["v"][1], c["v"][1])
    assert np.array_equal(got["k"][0, :, 35:], c["k"][0, :, 35:])
    # the new rows come back within half a step of their block's scale, the committed ones exactly where the scale did not grow
    x = K.decode(got["k"], got["ks"])[0, :, 30:35]
    want = new[0][0].transpose(1, 0, 2)
    assert np.all(np.abs(x - want) <= np.maximum(np.abs(want) * 2.0 ** -4, np.repeat(got["ks"][0], 32, -1)[:, 30:35, None] * 2.0 ** -10))
    # one call or two: committed rows are only ever rounded to coarser scales, so a block filled at once has the finest
    one = K.append(c, new[0], new[1], [64, 64], [5, 5])
    two = K.append(K.append(c, new[0][:, :2], new[1][:, :2], [64, 64], [2, 2]), new[0][:, 2:], new[1][:, 2:], [66, 66], [3, 3])
    assert np.array_equal(one["ks"][:, :, 2], two["ks"][:, :, 2])


def test_what_discarded_drafts_leave_behind_is_bounded():
    """Drafts of every magnitude into a block with committed rows, up and down again: a committed value ends less than 2^-9 of the largest scale away, and moves only when the scale is a new largest."""
    rng = np.random.default_rng(5)
    start = K.append(_cache(rng, 1, 1, 64, 16), *(rng.normal(size=(2, 1, 40, 1, 16)) * np.exp(rng.normal(size=(2, 1, 40, 1, 16)) * 2)), [0], [40])
    first = {n: K.decode(start["k"] if n == "k" else K.v_rows(start["v"]), start[n + "s"])[0, 0, :40] for n in "kv"}
    for up in (0.1, 3.0, 40.0):
        c, top, seen = start, {n: start[n + "s"][0, 0, 1] for n in "kv"}, None
        for e in list(rng.normal(size=12) * up) + [12 * up] + list(rng.normal(size=12) * up):
            c = K.append(c, *(rng.normal(size=(2, 1, 24, 1, 16)) * 2.0 ** e), [40], [24])
            now = {n: K.decode(c["k"] if n == "k" else K.v_rows(c["v"]), c[n + "s"])[0, 0, :40] for n in "kv"}
            for n in "kv":
                grown = c[n + "s"][0, 0, 1] > top[n]
                top[n] = max(top[n], c[n + "s"][0, 0, 1])
                assert np.array_equal(now[n][:32], first[n][:32])
                assert np.all(np.abs(now[n][32:] - first[n][32:]) < 2.0 ** -9 * top[n])
                assert grown or seen is None or np.array_equal(now[n], seen[n])
            seen = now


def test_attend_is_attention():
    rng = np.random.default_rng(2)
    c = _cache(rng, 1, 2, 64, 16)
    q = rng.normal(size=(1, 3, 4, 16)) * 0.01
    out, acc, _, _ = K.attend(c, q, [37], [3], np.zeros((1, 2, 64)))
    k, v = torch.from_numpy(K.decode(c["k"], c["ks"]))[0, :, :40], torch.from_numpy(K.decode(K.v_rows(c["v"]), c["vs"]))[0, :, :40]
    for h in range(4):
        p = torch.softmax(torch.from_numpy(q[0, :, h]) @ k[h // 2].T / 4, -1)
        assert np.allclose(out[0, :, h], p @ v[h // 2], rtol=1e-12, atol=1e-14)
    assert np.allclose(acc[0, :, :40].sum(-1), 6.0) and np.isnan(acc[0, :, 40:]).all()
    # no queries: the mean value vector
    out, _, _, _ = K.attend(c, q * 0, [37], [3])
    assert np.allclose(out[0, 0, 0], v[0].mean(0))


def test_evict_by_hand():
    rng = np.random.default_rng(3)
    c, d = _cache(rng, 1, 1, 64, 16), _cache(rng, 1, 1, 32, 16)
    acc = np.zeros((1, 1, 64))
    acc[0, 0, :10] = [5, 1, 1, 9, math.nan, 1, 0, 7, 100, 100]
    got, a2, lens, rows = K.evict(c, acc, np.array([10]), 6, 2, d, np.zeros((1, 1, 32)))
    assert rows[0, 0].tolist() == [0, 1, 3, 7, 8, 9] and lens[0] == 6 and a2[0, 0, :6].tolist() == [5, 1, 9, 7, 100, 100]
    assert np.array_equal(K.decode(got["k"], got["ks"])[0, 0, :6] * (got["ks"][0, 0, 0] <= c["ks"][0, 0, 0]),
                          K.decode(c["k"], c["ks"])[0, 0, [0, 1, 3, 7, 8, 9]] * (got["ks"][0, 0, 0] <= c["ks"][0, 0, 0]))
    assert np.array_equal(got["k"][0, 0, 6:], d["k"][0, 0, 6:])


def test_token_scores_by_hand():
    x = np.array([[0.0, math.log(3), -math.inf, 0.0], [-math.inf] * 4, [1.0, math.nan, 2.0, 0.0]])
    lp, en, ids, tops = K.token_scores(x, [1, 0, 0], -1, 3)
    assert np.isclose(lp[0], math.log(3 / 5)) and np.isclose(en[0], -(0.6 * math.log(0.6) + 0.4 * math.log(0.2)))
    assert ids[0].tolist() == [1, 0, 3] and ids[1].tolist() == [-1] * 3 and lp[1] == -math.inf and en[1] == 0
    assert math.isnan(lp[2]) and math.isnan(en[2]) and ids[2].tolist() == [2, 0, 3]
    lp, _, ids, _ = K.token_scores(x, [1, 0, 0], 1, 2)
    assert lp[0] == -math.inf and ids[0].tolist() == [0, 3]


# ---- refusals ------------------------------------------------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def dm():
    from paper_2511_15927_b200 import build
    build.build()
    from paper_2511_15927_b200 import binding
    return binding


P, Q = 4096, 8192                    # addresses that are never followed


def _cfg(dm, **kw):
    base = dict(batch=2, block_len=4, n_heads=8, n_kv_heads=4, head_dim=64, dtype=dm.DM_BF16)
    base.update(kw)
    return dm.dm_kv8_cfg(*base.values())


def _refused(dm, status, f, *args):
    before = dm.dm_kernel_launch_count()
    with pytest.raises(dm.DmError) as e:
        f(*args)
    assert e.value.status == status, str(e.value)
    assert dm.dm_last_error_message() and dm.dm_kernel_launch_count() == before


def test_kv8_configurations_that_are_refused(dm):
    c = dm.dm_kv8_cache(P, P, P, P, 64)
    for bad, status in ((dict(batch=0), dm.DM_ERR_INVALID_ARG), (dict(block_len=0), dm.DM_ERR_INVALID_ARG), (dict(n_heads=6), dm.DM_ERR_INVALID_ARG),
                        (dict(n_kv_heads=0), dm.DM_ERR_INVALID_ARG), (dict(dtype=7), dm.DM_ERR_INVALID_ARG), (dict(head_dim=32), dm.DM_ERR_UNSUPPORTED),
                        (dict(head_dim=96), dm.DM_ERR_UNSUPPORTED), (dict(batch=65536), dm.DM_ERR_UNSUPPORTED), (dict(batch=60000, block_len=60000), dm.DM_ERR_UNSUPPORTED)):
        cfg = _cfg(dm, **bad)
        _refused(dm, status, dm.dm_kv8_append, cfg, c, P, P, 512, P, 0)
        _refused(dm, status, dm.dm_kv8_attention_workspace_bytes, cfg, 100)
        _refused(dm, status, dm.dm_kv8_evict_workspace_bytes, cfg, 100, 10)
    _refused(dm, dm.DM_ERR_UNSUPPORTED, dm.dm_kv8_attention_workspace_bytes, _cfg(dm, dtype=dm.DM_F32), 100)
    _refused(dm, dm.DM_ERR_INVALID_ARG, dm.dm_kv8_attention_workspace_bytes, _cfg(dm), -1)
    _refused(dm, dm.DM_ERR_INVALID_ARG, dm.dm_kv8_evict_workspace_bytes, _cfg(dm), 100, 0)
    assert dm.dm_kv8_attention_workspace_bytes(_cfg(dm), 100000) >= dm.dm_kv8_attention_workspace_bytes(_cfg(dm), 100) > 0


def test_kv8_calls_that_are_refused(dm):
    cfg, good = _cfg(dm), dm.dm_kv8_cache(P, P, P, P, 64)
    bad = dm.DM_ERR_INVALID_ARG
    for c in (dm.dm_kv8_cache(0, P, P, P, 64), dm.dm_kv8_cache(P, P, P, 0, 64), dm.dm_kv8_cache(P + 8, P, P, P, 64), dm.dm_kv8_cache(P, P, P, P, 0), dm.dm_kv8_cache(P, P, P, P, 40)):
        _refused(dm, bad, dm.dm_kv8_append, cfg, c, P, P, 512, P, 0)
        _refused(dm, bad, dm.dm_kv8_attention, cfg, c, P, 512, P, 0, 64, 0, 0, Q, 512, P, 1 << 30)
        _refused(dm, bad, dm.dm_kv8_evict, cfg, c, dm.dm_kv8_cache(Q, Q, Q, Q, 64), P, Q, P, Q, 64, 32, 0, 0, P, 1 << 30)
    for k, v, ld, lens, counts in ((0, P, 512, P, 0), (P, P, 255, P, 0), (P, P, 260, P, 0), (P, P, 512, 0, 0), (P + 8, P, 512, P, 0), (P, P, 512, P + 2, 0), (P, P, 512, P, P + 1)):
        _refused(dm, bad, dm.dm_kv8_append, cfg, good, k, v, ld, lens, counts)
    ok = [cfg, good, P, 512, P, 0, 64, 0, 0, Q, 512, P, 1 << 30]
    for i, x in ((2, 0), (2, Q), (2, P + 8), (3, 504), (3, 516), (4, 0), (4, P + 2), (6, -1), (7, P), (8, P), (9, 0), (10, 511)):
        _refused(dm, bad, dm.dm_kv8_attention, *(ok[:i] + [x] + ok[i + 1:]))
    for ws, n in ((P, 16), (0, 1 << 30), (P + 16, 1 << 30)):
        _refused(dm, dm.DM_ERR_WORKSPACE, dm.dm_kv8_attention, *ok[:11], ws, n)
    ok = [cfg, good, dm.dm_kv8_cache(Q, Q, Q, Q, 64), P, Q, P, Q, 64, 32, 8, 0, P, 1 << 30]
    for i, x in ((2, good), (3, 0), (3, Q), (4, P), (5, Q), (6, 0), (7, -1), (8, 0), (8, 65), (9, -1), (9, 33), (10, P + 2)):
        _refused(dm, bad, dm.dm_kv8_evict, *(ok[:i] + [x] + ok[i + 1:]))
    _refused(dm, dm.DM_ERR_WORKSPACE, dm.dm_kv8_evict, *ok[:11], P, 16)


def test_token_scores_that_are_refused(dm):
    ok = [4, 100, 100, dm.DM_BF16, P, P, -1, 4, P, P, P, P]
    for i, x in ((0, 0), (1, 0), (2, 99), (3, 9), (4, 0), (4, P + 1), (5, 0), (5, P + 2), (6, -2), (7, -1), (7, 33), (8, 0), (9, P + 1), (11, P + 2)):
        _refused(dm, dm.DM_ERR_INVALID_ARG, dm.dm_token_scores, *(ok[:i] + [x] + ok[i + 1:]))
    _refused(dm, dm.DM_ERR_INVALID_ARG, dm.dm_token_scores, 4, 100, 100, dm.DM_BF16, P, 0, -1, 0, 0, 0, P, P)       # nothing to compute
    _refused(dm, dm.DM_ERR_UNSUPPORTED, dm.dm_token_scores, (1 << 28) + 1, *ok[1:])


def test_paths_on_the_cache_that_are_refused(dm):
    cfg, good, bad = _cfg(dm), dm.dm_kv8_cache(P, P, P, P, 64), dm.DM_ERR_INVALID_ARG
    ok = [cfg, 256, P, P, P, good, P, 64, 0, 0, Q, P, 1 << 30]
    for i, x in ((1, 0), (2, 0), (3, P + 8), (4, Q), (5, dm.dm_kv8_cache(P, P, P, P, 33)), (6, 0), (6, P + 1), (7, -1), (8, P), (9, P), (10, 0)):
        _refused(dm, bad, dm.dm_attention_block_step_kv8, *(ok[:i] + [x] + ok[i + 1:]))
    _refused(dm, dm.DM_ERR_UNSUPPORTED, dm.dm_attention_block_step_kv8, *([cfg, 252] + ok[2:]))
    _refused(dm, dm.DM_ERR_UNSUPPORTED, dm.dm_attention_block_step_kv8, *([_cfg(dm, dtype=dm.DM_F32)] + ok[1:]))
    _refused(dm, dm.DM_ERR_WORKSPACE, dm.dm_attention_block_step_kv8, *ok[:11], P, 256)
    mix = dm.make_mixer_cfg(1, 32, 128, 2, 128, 4, 4, dm.DM_BF16)
    scfg, hyb = dm.dm_stack_cfg(mix, 2, 504, 1e-5), dm.dm_hybrid_cfg(2, 2)
    n = dm.dm_denoise_hybrid_kv8_workspace_bytes(scfg, None, hyb, 1000)
    assert n > dm.dm_denoise_hybrid_workspace_bytes(scfg) and dm.dm_denoise_hybrid_kv8_workspace_bytes(scfg, None, dm.dm_hybrid_cfg(0, 0), 1000) == dm.dm_denoise_hybrid_workspace_bytes(scfg)
    _refused(dm, bad, dm.dm_denoise_hybrid_kv8_workspace_bytes, scfg, None, hyb, -1)
    _refused(dm, dm.DM_ERR_UNSUPPORTED, dm.dm_denoise_hybrid_kv8_workspace_bytes, scfg, None, dm.dm_hybrid_cfg(2, 3), 10)
    layers = (dm.dm_layer_weights * 2)()
    for l in layers:
        l.norm_w = P
        l.dir[0] = l.dir[1] = dm.dm_dir_weights(*([P] * 8))
    sw = dm.dm_stack_weights(P, C.cast(layers, C.POINTER(dm.dm_layer_weights)), P, P)
    aw = (dm.dm_attn_weights * 2)(dm.dm_attn_weights(P, P))

    def call(states, n=1 << 40):
        return dm.dm_denoise_step_hybrid_block_kv8, scfg, None, hyb, sw, None, aw, P, 0, P, 0, None, states, P, n

    good = (dm.dm_kv8_cache(P, P, P, P, 64), P, 32, None, None)
    for i, x in ((0, dm.dm_kv8_cache(P, P, P, 0, 64)), (1, None), (1, P + 2), (2, -1), (3, P), (4, P)):
        one = list(good)
        one[i] = x
        _refused(dm, bad, *call((dm.dm_kv8_state * 2)(dm.dm_kv8_state(*one))))
    _refused(dm, bad, *call(None))
    _refused(dm, dm.DM_ERR_WORKSPACE, *call((dm.dm_kv8_state * 2)(dm.dm_kv8_state(*good)), 1024))


def test_token_scores_refuse_ids_over_the_tokens(dm):
    """Other rows' tokens may still be read when a row's ids are written."""
    _refused(dm, dm.DM_ERR_INVALID_ARG, dm.dm_token_scores, 4, 100, 100, dm.DM_BF16, P, Q, -1, 4, P, 0, Q, 0)


def test_a_workspace_serves_every_shorter_cache(dm):
    """The stack sizes one workspace by the longest of its layers' caches."""
    for D, H, kv, G, B in ((64, 16, 16, 32, 2), (64, 16, 16, 1, 4), (80, 24, 24, 32, 1), (128, 32, 8, 4, 8), (64, 1, 1, 1, 1), (80, 24, 24, 32, 16)):
        cfg = _cfg(dm, batch=B, block_len=G, n_heads=H, n_kv_heads=kv, head_dim=D)
        sizes = [dm.dm_kv8_attention_workspace_bytes(cfg, n) for n in list(range(0, 70000, 250)) + [1 << 20, 1 << 30]]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), (D, H, kv, G, B)


def test_waits_of_whole_warps_are_agreed_upon():
    """A wait that runs out is noticed lane by lane: where a whole warp waits and goes on together, the answer is the warp's (the self-test of the waits has lanes that disagree)."""
    import os
    import re
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_15927_b200", "csrc")
    for name, waits in (("kv8_attention.cu", 2), ("kv8_evict.cu", 1)):
        text = open(os.path.join(csrc, name)).read()
        assert not re.search(r"\bmbar_wait\(", text) and len(re.findall(r"\bmbar_wait_warp\(", text)) == waits
