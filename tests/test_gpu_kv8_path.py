"""The 8-bit key/value cache on the library's own paths: the attention mixer's block step and the hybrid stack in block mode, against the fp64 oracle.

The oracle takes keys and values from the cache as the call left it (append is tested bit by bit elsewhere; a projection rounded to bf16 next to a code's boundary may fall on either side,
so codes made from the oracle's own projection are no reference), and everything else from its own arithmetic, at the tolerances of the bf16 paths.
The cache itself: a code is at most half a step from the value, 2^-4 of it, plus the projection's rounding to bf16.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import bimamba_oracle as O
from oracle import kv8_oracle as K
from paper_2511_15927_b200 import inputs as I

torch = pytest.importorskip("torch")
F64 = np.float64


@pytest.fixture(scope="module")
def G():
    from paper_2511_15927_b200 import build
    build.build()
    import tests.gpu_util as g
    return g


@pytest.fixture(scope="module")
def dm():
    from paper_2511_15927_b200 import binding
    return binding


class Cache:
    def __init__(self, dm, B, H, cap, D):
        self.k = torch.full((B, H, cap, D), 0x7f, dtype=torch.uint8, device="cuda")
        self.v = torch.full((B, H, cap // 32, D, 32), 0x7f, dtype=torch.uint8, device="cuda")
        self.ks, self.vs = (torch.full((B, H, cap // 32), float("nan"), device="cuda") for _ in range(2))
        self.handle = dm.dm_kv8_cache(self.k.data_ptr(), self.v.data_ptr(), self.ks.data_ptr(), self.vs.data_ptr(), cap)

    def rows(self, b, n):
        """Keys and values [H, n, D] of sequence b."""
        k = K.decode(self.k[b].cpu().numpy(), self.ks[b].cpu().numpy().astype(F64))
        v = K.decode(K.v_rows(self.v[b].cpu().numpy()), self.vs[b].cpu().numpy().astype(F64))
        return k[:, :n], v[:, :n]


def attend(q, cache, b, n):
    """q [G, Hq, D] over the cache's rows: [G, Hq * D] and the weights [H, n]."""
    k, v = cache.rows(b, n)
    group = q.shape[1] // k.shape[0]
    out, w = np.empty(q.shape), np.zeros((k.shape[0], n))
    for h in range(q.shape[1]):
        s = q[:, h] @ k[h // group].T / np.sqrt(q.shape[2])
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        out[:, h] = p @ v[h // group]
        w[h // group] += p.sum(0)
    return out.reshape(q.shape[0], -1), w


@pytest.mark.parametrize("D,Hq,H,d", [(64, 4, 4, 256), (80, 3, 3, 240), (64, 6, 2, 200), (128, 4, 1, 256)])
def test_block_step_chain(G, dm, D, Hq, H, d):
    """Three steps: a prefix committed, a block twice without a commit (the second time with other tokens), weights accumulated on the last."""
    rng = np.random.default_rng(D + Hq)
    B, cap, max_len = 2, 160, 100
    wide = (Hq + 2 * H) * D
    wq = I.round_to_bf16((1.5 / np.sqrt(d)) * rng.standard_normal((wide, d), dtype=np.float32))
    wo = I.round_to_bf16((1.0 / np.sqrt(Hq * D)) * rng.standard_normal((d, Hq * D), dtype=np.float32))
    dwq, dwo = G.dev(wq, I.BF16), G.dev(wo, I.BF16)
    cache = Cache(dm, B, H, cap, D)
    lens_h = [0, 0]
    lens = torch.tensor(lens_h, dtype=torch.int32, device="cuda")
    acc = torch.zeros(B, H, cap, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    for step, (n, weights) in enumerate(((70, False), (17, False), (17, True))):
        x = I.round_to_bf16(rng.standard_normal((B, n, d), dtype=np.float32))
        xd = G.dev(x, I.BF16)
        yd = torch.empty(B, n, d, dtype=torch.bfloat16, device="cuda")
        cfg = dm.dm_kv8_cfg(B, n, Hq, H, D, dm.DM_BF16)
        nb = dm.dm_attention_block_step_kv8_workspace_bytes(cfg, d, max_len)
        ws = G.workspace(nb)
        a = acc.data_ptr() if weights else 0
        dm.dm_attention_block_step_kv8(cfg, d, dwq.data_ptr(), dwo.data_ptr(), xd.data_ptr(), cache.handle, lens.data_ptr(), max_len, a, a, yd.data_ptr(), ws.data_ptr(), nb, st)
        dm.dm_check(st)
        qkv = (x.astype(F64) @ wq.astype(F64).T).reshape(B, n, Hq + 2 * H, D)
        for b in range(B):
            k, v = cache.rows(b, lens_h[b] + n)
            for got, want in ((k, qkv[b, :, Hq:Hq + H]), (v, qkv[b, :, Hq + H:])):
                new, want = got[:, lens_h[b]:], want.transpose(1, 0, 2)
                assert np.all(np.isfinite(new)) and G.rel_l2(new, want) <= 2.0 ** -4 + 2.0 ** -8
            out, w = attend(qkv[b, :, :Hq], cache, b, lens_h[b] + n)
            want = out @ wo.astype(F64).T
            got = yd[b].double().cpu().numpy()
            assert G.rel_l2(got, want) <= 1e-2 and G.max_abs(got, want) <= 5e-2, (step, G.rel_l2(got, want))
            if weights:
                # q reaches the scores through its rounding to bf16: 2^-8 of the channels' products, below 2 % of a weight here
                gw = acc[b].double().cpu().numpy()[:, :lens_h[b] + n]
                assert G.rel_l2(gw, w) <= 2e-2 and np.isclose(gw.sum(), Hq * n, rtol=1e-4)
        if step == 0:
            lens_h = [70, 33]                        # sequence 1 keeps less of its prefix
            lens.copy_(torch.tensor(lens_h, dtype=torch.int32))


def test_a_draft_that_is_given_up(G, dm):
    """A draft with an outlier into a block that the commit boundary cuts, then the real one: committed rows of whole blocks keep every bit, those of the cut one stay within 2^-9 of the
    largest scale that it has had, and the block's own rows are those of a cache that has never seen the draft, but for half a step of the smallest codes at each one's scale."""
    rng = np.random.default_rng(19)
    B, Hq, H, D, d, n0, n = 1, 4, 2, 64, 256, 41, 20
    wide, cap = (Hq + 2 * H) * D, 96
    dwq = G.dev(I.round_to_bf16(rng.standard_normal((wide, d), dtype=np.float32) / 16), I.BF16)
    dwo = G.dev(I.round_to_bf16(rng.standard_normal((d, Hq * D), dtype=np.float32) / 16), I.BF16)
    prefix, draft, real = (I.round_to_bf16(rng.standard_normal((B, m, d), dtype=np.float32)) for m in (n0, n, n))
    draft[0, 3] *= 2.0 ** 9
    st = torch.cuda.current_stream().cuda_stream

    def step(cache, x, before):
        cfg = dm.dm_kv8_cfg(B, x.shape[1], Hq, H, D, dm.DM_BF16)
        lens = torch.tensor([before], dtype=torch.int32, device="cuda")
        xd, y = G.dev(x, I.BF16), torch.empty(B, x.shape[1], d, dtype=torch.bfloat16, device="cuda")
        nb = dm.dm_attention_block_step_kv8_workspace_bytes(cfg, d, cap)
        ws = G.workspace(nb)
        dm.dm_attention_block_step_kv8(cfg, d, dwq.data_ptr(), dwo.data_ptr(), xd.data_ptr(), cache.handle, lens.data_ptr(), cap, 0, 0, y.data_ptr(), ws.data_ptr(), nb, st)
        dm.dm_check(st)
        return y

    a, b = Cache(dm, B, H, cap, D), Cache(dm, B, H, cap, D)
    for c in (a, b):
        step(c, prefix, 0)
    first = a.rows(0, n0)
    step(a, draft, n0)
    top = [s[0, :, 1].cpu().numpy().astype(F64) for s in (a.ks, a.vs)]
    ya, yb = step(a, real, n0), step(b, real, n0)
    for i, (x, ra, rb) in enumerate(zip(first, a.rows(0, n0 + n), b.rows(0, n0 + n))):
        sa, sb = ((c.ks, c.vs)[i][0].cpu().numpy().astype(F64) for c in (a, b))
        assert np.all(top[i] > 2.0 ** 4 * sb[:, 1])                                # the outlier did make the scale grow
        assert np.array_equal(ra[:, :32], x[:, :32])
        moved = np.abs(ra[:, 32:n0] - x[:, 32:])
        assert moved.max() > 0 and np.all(moved < 2.0 ** -9 * top[i][:, None, None])
        assert np.all(np.abs(ra[:, n0:] - rb[:, n0:]) <= 2.0 ** -9 * np.maximum(sa, sb).repeat(32, -1)[:, n0:n0 + n, None])
    assert torch.isfinite(ya.float()).all() and torch.isfinite(yb.float()).all()


def test_hybrid_stack_block_mode_on_the_8_bit_cache(G, dm, monkeypatch):
    """The prefix is committed (Mamba states, 8-bit caches), then a block runs from it, twice with the same result."""
    import tests.test_gpu_attention as A
    import tests.gpu_util as U
    B, G1, G2, V, layers, period, heads = 2, 96, 32, 504, 4, 2, 2
    full = I.MixerShape(B, G1 + G2, 128, 2, 128, 4, 4)
    sw, _, _ = A._hybrid_stack(full, layers, V, 41, False)
    tok = I.make_tokens(B, G1 + G2, V - 1, V - 1, seed=41)
    kw = G.oracle_kwargs(full)
    dsw = U.dev_stack_weights(sw, I.BF16)
    csw, keep = dm.make_stack_weights(dsw)
    daw = [{"w_qkv": G.dev(l["w_qkv"], I.BF16), "w_o": G.dev(l["w_o"], I.BF16)} for l in sw["layers"]]
    caw = dm.make_attn_weights(daw)
    caches = [Cache(dm, B, heads, 160, 64) if i % period == 0 else None for i in range(layers)]
    accs = [torch.zeros(B, heads, 160, device="cuda") for _ in range(layers)]
    ssm = [torch.zeros((B, full.n_heads, full.headdim, full.d_state), device="cuda") for _ in range(layers)]
    conv = [torch.zeros((B, full.d_conv - 1, full.conv_ch), device="cuda", dtype=torch.bfloat16) for _ in range(layers)]
    st = torch.cuda.current_stream().cuda_stream
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    hyb = dm.dm_hybrid_cfg(period, heads)

    def step(tokens, L, first):
        shape = I.MixerShape(B, L, full.d_model, 2, full.d_state, 4, full.n_heads)
        scfg = dm.dm_stack_cfg(U.cfg_of(shape, I.BF16), layers, V, 1e-5)
        states, k8 = (dm.dm_layer_state * layers)(), (dm.dm_kv8_state * layers)()
        for i in range(layers):
            states[i] = dm.dm_layer_state(None, None, ssm[i].data_ptr(), conv[i].data_ptr()) if first else dm.dm_layer_state(ssm[i].data_ptr(), conv[i].data_ptr(), None, None)
            if caches[i]:
                k8[i] = dm.dm_kv8_state(caches[i].handle, lens.data_ptr(), 128, None if first else accs[i].data_ptr(), None if first else accs[i].data_ptr())
        td = G.dev(np.asarray(tokens, np.int32))
        logits = torch.empty((B, L, V), device="cuda", dtype=torch.bfloat16)
        nb = dm.dm_denoise_hybrid_kv8_workspace_bytes(scfg, None, hyb, 128)
        ws = G.workspace(nb)
        dm.dm_denoise_step_hybrid_block_kv8(scfg, None, hyb, csw, None, caw, td.data_ptr(), 0, logits.data_ptr(), 0, states, k8, ws.data_ptr(), nb, st)
        dm.dm_check(st)
        return logits.float().cpu().numpy().astype(F64)

    def want(tokens, n_before, L, states_in):
        """The oracle's stack, its attention layers reading the library's caches in turn."""
        order = iter([c for c in caches if c])

        def mixer(u, w_qkv, w_o, n_heads, kc=None, vc=None):
            c, d = next(order), u.shape[-1]
            q = (u @ np.asarray(w_qkv, F64)[:d].T).reshape(B, L, n_heads, -1)
            y = np.stack([attend(q[b], c, b, n_before + L)[0] for b in range(B)])
            return y @ np.asarray(w_o, F64).T, None, None

        monkeypatch.setattr(O, "attention_block_step", mixer)
        out, _ = O.denoise_step_hybrid(tokens, sw, attn_period=period, attn_heads=heads, states_in=states_in, return_states=True, **kw)
        return out

    got1 = step(tok[:, :G1], G1, True)
    want1 = want(tok[:, :G1], 0, G1, None)
    assert G.rel_l2(got1, want1) <= 1e-2, G.rel_l2(got1, want1)
    lens.fill_(G1)
    st_in = [None if caches[i] else (ssm[i].cpu().numpy().astype(F64), conv[i].float().cpu().numpy().astype(F64)) for i in range(layers)]
    got2 = step(tok[:, G1:], G2, False)
    want2 = want(tok[:, G1:], G1, G2, st_in)
    assert G.rel_l2(got2, want2) <= 1e-2, G.rel_l2(got2, want2)
    for i in range(0, layers, period):
        assert np.isclose(accs[i].sum().item(), B * heads * G2, rtol=1e-4)
    assert np.array_equal(step(tok[:, G1:], G2, False), got2)
    # 8 bits against 16: the same stack with a bf16 cache differs by what the codes cost, some per cent of the attention layers' part
    monkeypatch.undo()
    plain, _ = O.denoise_step_hybrid(tok[:, :G1], sw, attn_period=period, attn_heads=heads, return_states=True, **kw)
    assert G.rel_l2(got1, plain) <= 2.0 ** -4
