"""Log probabilities, entropy and the most likely tokens of rows of logits against the fp64 oracle.

Bound.  Sums run over at most V / 2048 + 16 fp32 additions per thread and joint, each off by 2^-24 of the sum, each term by 2^-21 (the exponential's 2 units in the last place and
its argument's rounding); log S takes that over as it is, T / S takes it times the mean distance from the reference.  Ids are exact: equal logits go by the lower id.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import kv8_oracle as K

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dm():
    from paper_2511_15927_b200 import build
    build.build()
    from paper_2511_15927_b200 import binding
    return binding


def run(dm, x, tokens, exclude, k, vocab=None, only=None):
    """x [rows, ld] on the GPU (a view of a larger tensor may start at any element)."""
    rows, vocab = x.shape[0], vocab or x.shape[1]
    t = torch.tensor(tokens, dtype=torch.int32, device="cuda")
    lp, en = torch.full((rows,), 5.0, device="cuda"), torch.full((rows,), 5.0, device="cuda")
    ids, tops = torch.full((rows, max(k, 1)), -5, dtype=torch.int32, device="cuda"), torch.full((rows, max(k, 1)), 5.0, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    want = only or ("lp", "en", "ids", "tops")
    p = lambda n, v: v.data_ptr() if n in want else 0
    dm.dm_token_scores(rows, vocab, x.stride(0), dm.DM_BF16 if x.dtype == torch.bfloat16 else dm.DM_F32, x.data_ptr(), p("lp", t), exclude, k, p("lp", lp), p("en", en),
                       p("ids", ids) if k else 0, p("tops", tops) if k else 0, s)
    dm.dm_check(s)
    return lp.double().cpu().numpy(), en.double().cpu().numpy(), ids.cpu().numpy()[:, :k], tops.double().cpu().numpy()[:, :k]


def close(got, want, tol):
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    err = np.abs(got - want)[fin]
    assert np.all(err <= np.broadcast_to(tol, got.shape)[fin]), float((err / np.broadcast_to(tol, got.shape)[fin]).max())


def check(dm, x, tokens, exclude=-1, k=8, vocab=None):
    vocab = vocab or x.shape[1]
    lp, en, ids, tops = run(dm, x, tokens, exclude, k, vocab)
    h = x[:, :vocab].double().cpu().numpy()
    wl, we, wi, wt = K.token_scores(h, tokens, exclude, k)
    assert np.array_equal(ids, wi), np.argwhere(ids != wi)[:4]
    rel = (vocab / 2048 + 16) * 2.0 ** -24 + 2.0 ** -21
    mag = 2.0 ** -22 * np.abs(np.where(np.isfinite(wl), wl, 0))
    close(lp, wl, mag + 2 * rel)
    close(en, we, 2.0 ** -22 * np.abs(np.nan_to_num(we)) + rel * (4 + 2 * np.abs(np.nan_to_num(we))))
    close(tops, wt, 2.0 ** -22 * np.abs(np.where(np.isfinite(wt), wt, 0)) + 2 * rel)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,ld,k,exclude", [
    (1, 50304, 50304, 8, -1), (3, 50257, 50304, 32, 50256), (1, 1, 1, 1, -1), (2, 7, 9, 5, 3), (5, 1000, 1047, 16, 999), (700, 257, 257, 3, 0), (2, 2049, 2049, 32, 7),
    (40, 20000, 20001, 1, -1), (2, 150001, 150001, 4, 5), (4, 33, 40, 0, -1), (3, 31, 31, 32, 30), (300, 4100, 4100, 20, -1)])
def test_shapes(dm, dtype, rows, vocab, ld, k, exclude):
    g = torch.Generator().manual_seed(vocab + k)
    x = (torch.randn(rows, ld, generator=g) * 3).to(dtype).cuda()
    x[:, vocab:] = 1e30                                              # what lies between the rows is not read
    t = torch.randint(vocab, (rows,), generator=g).tolist()
    check(dm, x, t, exclude, k, vocab)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [1, 3, 5, 7])
def test_rows_at_any_alignment(dm, dtype, shift):
    g = torch.Generator().manual_seed(shift)
    store = (torch.randn(5 * 3001 + 16, generator=g) * 2).to(dtype).cuda()
    check(dm, store[shift:shift + 5 * 3001].view(5, 3001), [0, 1, 3000, 1500, 7], 1500, 9)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 9])
def test_ties_go_to_the_lower_id(dm, dtype, rows):
    V = 30011
    x = torch.zeros(rows, V, dtype=dtype, device="cuda")             # all alike
    check(dm, x, [5] * rows, -1, 32)
    x[:, 20000:] = 1.0                                               # ten thousand alike at the top
    check(dm, x, [20000] * rows, 20001, 17)
    x[:] = torch.randint(0, 5, (rows, V), generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    check(dm, x, [20000] * rows, -1, 32)
    x[:] = -2.0
    x[:, ::4096] = 3.0                                               # fewer at the top than asked for
    check(dm, x, [4096] * rows, -1, 20)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_and_special_rows(dm, dtype):
    V = 9000
    low = torch.finfo(dtype).min
    x = torch.randn(12, V, generator=torch.Generator().manual_seed(2)).to(dtype)
    x[0] = -math.inf                                                 # nothing left
    x[1] = -math.inf; x[1, 8999] = 2.0                               # one left
    x[2, 5:] = -math.inf                                             # fewer left than asked for
    x[3] = low                                                       # a mask of the lowest value everywhere: uniform
    x[4, 100:] = low
    x[5, 77] = math.nan
    x[6, 4000] = math.inf
    x[7, ::2] = -math.inf
    x[8] = x[8] * 0 + torch.finfo(dtype).max                         # as large as they come: uniform
    x[9] = 1e4; x[9, 3] = 1.01e4                                     # far from zero
    x[10] = -1e30; x[10, 9] = -0.5e30
    x[11, 1] = 200.0                                                 # certain
    check(dm, x.cuda(), [0, 8999, 3, 10, 99, 1, 1, 2, 0, 3, 9, 1], -1, 8)
    check(dm, x.cuda(), [0, 8999, 3, 10, 99, 1, 1, 3, 0, 3, 9, 2], 8999, 8)      # of row 1 nothing is left


def test_tokens_that_cannot_be(dm):
    x = torch.randn(5, 100, device="cuda")
    lp, en, _, _ = run(dm, x, [-1, 100, 2 ** 31 - 1, 42, 41], 42, 0)
    assert np.all(lp[:4] == -math.inf) and np.isfinite(lp[4]) and np.isfinite(en).all()


def test_what_is_not_asked_for_is_not_written(dm):
    x = torch.randn(3, 500, device="cuda")
    full = run(dm, x, [1, 2, 3], -1, 4)
    for name, i in (("lp", 0), ("en", 1), ("ids", 2), ("tops", 3)):
        part = run(dm, x, [1, 2, 3], -1, 4, only=(name,))
        assert np.array_equal(part[i], full[i])
        assert all(np.all(np.abs(part[j]) == 5) for j in range(4) if j != i)


def test_many_rows_are_each_like_one(dm):
    """Rows taken by one CTA and rows shared by a cluster agree to the sums' order."""
    x = (torch.randn(600, 12345, generator=torch.Generator().manual_seed(5)) * 2).to(torch.bfloat16).cuda()
    t = list(range(600))
    many = run(dm, x, t, -1, 6)
    for r in (0, 299, 599):
        one = run(dm, x[r:r + 1], [t[r]], -1, 6)
        assert np.array_equal(one[2][0], many[2][r])
        for i in (0, 1, 3):
            assert np.allclose(one[i][0], many[i][r], rtol=1e-6, atol=2e-6)
    again = run(dm, x, t, -1, 6)
    assert all(np.array_equal(a, b) for a, b in zip(many, again))


def test_scores_of_a_stack_steps_logits(dm):
    """dm_denoise_step's logits, scored where they lie: the arg-max is the first alternative and its probability the largest."""
    import tests.gpu_util as G
    from paper_2511_15927_b200 import inputs as I
    shape = I.MixerShape(2, 24, 64, 2, 16, 4, 4)
    for dtype in (I.F32, I.BF16):
        sw = I.make_stack_weights(shape, 2, 96, seed=0, dtype=dtype, perturb=True)
        tok = I.make_tokens(2, 24, 95, 95, seed=0)
        logits, amax, _ = G.run_denoise(shape, dtype, sw, tok, 96)
        x = torch.from_numpy(logits.reshape(48, 96)).to(torch.bfloat16 if dtype == I.BF16 else torch.float32).cuda()
        lp, en, ids, tops = run(dm, x, amax.reshape(-1).tolist(), -1, 2)
        assert np.array_equal(ids[:, 0], amax.reshape(-1)) and np.array_equal(lp, tops[:, 0]) and np.all(tops[:, 0] >= tops[:, 1])
        check(dm, x, tok.reshape(-1).tolist(), 95, 4)
