"""Operators of block-autoregressive decoding with a bounded 8-bit key/value cache, and of what a decoding step reads off its logits.

    append   the block's keys and values into the cache: e4m3 codes with one power-of-two scale per 32 rows and head
    attend   the block's queries over the cache, one length per sequence; with `weights` also what each row has received
    evict    the rows with the least accumulated weight leave the cache, the others move up into another one
    scores   log probability of given tokens, entropy and the most likely alternatives of each row of logits

Every case takes queries, keys and values as a program has them: as columns of the projection [Q | K | V] of the block's tokens.
Sizes are those of the configurations in `inputs.CONFIGS` and `bench.py` (16 heads of 64, the paper's 24 heads of 80, blocks of 32,
16 sequences, vocabulary 50304 with 50257 real ids) and ragged ones between them; grouped heads of 128 are a generic size.

    own            False: `run` computes the plain form; True: it calls the library
    listed()       the named cases
    draw(rng)      one more case of the same kinds and ranges
    prepare(c, s)  inputs on the GPU, from the seed
    run(state)     one call
    work(case)     bytes and operations of one call that no implementation can avoid
    exact(c, s)    what `run` returns, in 64 bits
"""
import math

import torch

own = False

BLOCK = 32             # rows of the cache that share a scale
TOP = 448.0            # largest e4m3 value
FLOOR = 2.0 ** -100    # smallest scale
VOCAB, VOCAB_REAL = 50304, 50257


def _decode(name, kind, batch, block, heads, kv_heads, dim, length, **more):
    c = {"kind": kind, "batch": batch, "block": block, "heads": heads, "kv_heads": kv_heads, "dim": dim, "len": length,
         "dtype": "bf16", "padded": False, "weights": False, "keep": 0, "recent": 0, **more}
    return dict(c, name=name) if name else c


def _scores(name, rows, vocab, pitch, dtype, top, exclude=-1):
    c = {"kind": "scores", "rows": rows, "vocab": vocab, "pitch": pitch, "dtype": dtype, "top": top, "exclude": exclude}
    return dict(c, name=name) if name else c


def listed():
    return [
        # single-token decoding of a batch: one row per sequence joins a block that is already half full
        _decode("append_token", "append", 16, 1, 16, 16, 64, 4096),
        # a committed block of 32 tokens of the paper's hybrid, 16 sequences whose prefixes end inside a block of the cache
        _decode("append_block", "append", 16, 32, 24, 24, 80, 2048),
        # a prompt goes into the empty cache in one call, its length no multiple of anything
        _decode("append_prompt", "append", 4, 8191, 24, 24, 80, 0),
        # the latency of a single token of a single sequence
        _decode("attend_token", "attend", 1, 1, 16, 16, 64, 8192),
        # a denoising pass of the paper's hybrid over one sequence's active block
        _decode("attend_block", "attend", 1, 32, 24, 24, 80, 8192),
        # long contexts of unequal length: the cache is what has to be read
        _decode("attend_long", "attend", 4, 32, 16, 16, 64, 65536),
        # grouped heads, single tokens, a batch of unequal lengths
        _decode("attend_grouped", "attend", 16, 1, 32, 8, 128, 16384),
        # the pass that commits a block and keeps count of what each row receives, blocks of a padded batch partly empty
        _decode("attend_weights", "attend", 16, 32, 24, 24, 80, 8192, padded=True, weights=True),
        # one sequence's cache cut to a quarter: the latency of the choice
        _decode("evict_one", "evict", 1, 32, 16, 16, 64, 8192, keep=2048, recent=256),
        # long caches of unequal length, some of them short enough to stay whole
        _decode("evict_batch", "evict", 8, 32, 24, 24, 80, 32768, keep=8000, recent=1000),
        # the positions of one active block, fp32 logits: which of them are certain enough to be committed
        _scores("scores_block", 32, VOCAB, VOCAB, "f32", 4),
        # scoring whole sequences: real ids only, rows padded to the projection's pitch
        _scores("scores_batch", 8192, VOCAB_REAL, VOCAB, "bf16", 8),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "evict", "scores"])
    if kind == "scores":
        vocab = _log(rng, 1000, VOCAB)
        rows = min(_log(rng, 1, 8192), 8192 * VOCAB // (2 * vocab))
        return _scores(None, rows, vocab, vocab + rng.choice([0, 1, 47, 64]), rng.choice(["bf16", "f32"]), rng.randint(1, 16),
                       rng.choice([-1, vocab - 1, vocab // 3]))
    heads, kv_heads, dim = rng.choice([(16, 16, 64), (24, 24, 80), (8, 8, 64), (12, 12, 80), (32, 8, 128), (16, 4, 64), (20, 5, 80), (14, 2, 64)])
    batch = rng.randint(1, 16)
    if kind == "append":
        block = min(_log(rng, 1, 8192), 4 * 8191 // batch)
        return _decode(None, kind, batch, block, heads, kv_heads, dim, rng.choice([0, _log(rng, 1, 8192)]), padded=rng.random() < 0.3,
                       dtype=rng.choice(["bf16", "f32"]))
    room = 4 * 65536 * 16 * 64 // (batch * kv_heads * dim)          # rows per sequence at the largest case's bytes
    length = min(_log(rng, 1, 65536), room * 2 // 3)
    if kind == "evict":
        length = max(length, 64)
        keep = rng.randint(16, length)
        return _decode(None, kind, batch, 32, heads, kv_heads, dim, length, keep=keep, recent=rng.randint(0, keep // 2))
    block = rng.choice([1, 1, 8, 16, 32, 32, 64, rng.randint(2, 64)])
    length = min(length, max(1, 4 * 65536 * 16 * 32 // (batch * heads * block)))   # and at its products
    return _decode(None, kind, batch, block, heads, kv_heads, dim, length, padded=rng.random() < 0.3, weights=rng.random() < 0.4)


def _lens(c):
    """Committed rows of each sequence: from `len` down to a half of it."""
    return [c["len"] - (b * c["len"]) // (2 * c["batch"]) - (5 * b if c["len"] > 64 * c["batch"] else 0) for b in range(c["batch"])]


def _counts(c):
    """Rows of the block that each sequence really has."""
    return [c["block"] if not c["padded"] else c["block"] - (b * 7) % (c["block"] + 1) for b in range(c["batch"])]


def _capacity(c):
    return (c["len"] + c["block"] + 2 * BLOCK + BLOCK - 1) // BLOCK * BLOCK


def _scale(top):
    """The smallest power of two s with 448 s >= top, and not below FLOOR."""
    m, e = torch.frexp(top / TOP)                                   # top / 448 = m 2^e, m in [0.5, 1): the quotient rounds up past a power of
    s = torch.ldexp(torch.ones_like(top), torch.where(m > 0.5, e, e - 1))   # two only where it is one
    s = torch.where(s * TOP < top, 2 * s, s)
    return torch.where(top > 0, s, 0.0).clamp_min(FLOOR)


def _unblock(v):
    """V as it lies in the cache, [.., blocks, dim, 32], to [.., rows, dim]."""
    return v.transpose(-1, -2).flatten(-3, -2)


def _rows(codes, scale, dt=torch.float32):
    """Values of codes [.., rows, dim] with a scale per BLOCK rows."""
    return codes.view(torch.float8_e4m3fn).to(dt) * scale.to(dt).repeat_interleave(BLOCK, -1).unsqueeze(-1)


def _quantised(x, there):
    """Codes and scales of rows x [.., rows, dim] where `there` [.., rows]; rows a multiple of BLOCK."""
    x = torch.where(there.unsqueeze(-1), x, torch.zeros_like(x)).unflatten(-2, (-1, BLOCK))
    s = _scale(torch.where(x.isfinite(), x.abs(), 0.0).amax((-1, -2)))
    q = (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(x.isfinite(), q, torch.full_like(q, 0x7f)).flatten(-3, -2), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    c = dict(case)
    if c["kind"] == "scores":
        # a language model's logits: a broad floor, a few ids far above it, some positions certain and others not
        x = normal(c["rows"], c["pitch"]) * 2
        x[torch.arange(c["rows"], device="cuda"), torch.randint(c["vocab"], (c["rows"],), generator=g, device="cuda")] += 12 * torch.rand(c["rows"], generator=g, device="cuda")
        t = torch.randint(c["vocab"], (c["rows"],), generator=g, device="cuda", dtype=torch.int32)
        t = torch.where(t == c["exclude"], (t + 1) % c["vocab"], t)
        x = x.to(torch.bfloat16) if c["dtype"] == "bf16" else x
        k = max(1, c["top"])
        return {"case": c, "logits": x, "tokens": t, "logprob": torch.empty(c["rows"], device="cuda"), "entropy": torch.empty(c["rows"], device="cuda"),
                "top_ids": torch.empty(c["rows"], k, device="cuda", dtype=torch.int32), "top_logprobs": torch.empty(c["rows"], k, device="cuda")}
    B, G, H, K, D = c["batch"], c["block"], c["heads"], c["kv_heads"], c["dim"]
    cap = _capacity(c)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    # channels of unequal size, as trained projections have them
    width = torch.exp(0.5 * normal(K, D))
    st = {"case": c, "cap": cap, "lens": torch.tensor(_lens(c), dtype=torch.int32, device="cuda"),
          "counts": torch.tensor(_counts(c), dtype=torch.int32, device="cuda")}
    qkv = normal(B, G, H + 2 * K, D)
    qkv[:, :, :H] *= 2.0
    qkv[:, :, H:H + K] *= width
    qkv[:, :, H + K:] *= width.flip(0)
    st["qkv"] = qkv.to(dt).view(B * G, (H + 2 * K) * D)
    del qkv
    kc = torch.empty(B, K, cap, D, dtype=torch.uint8, device="cuda")
    vc = torch.empty(B, K, cap // BLOCK, D, BLOCK, dtype=torch.uint8, device="cuda")
    ks, vs = (torch.empty(B, K, cap // BLOCK, device="cuda") for _ in range(2))
    on = torch.ones((), dtype=torch.bool, device="cuda").expand(K, cap)
    for b in range(B):
        q, ks[b] = _quantised(normal(K, cap, D) * width[:, None], on)
        kc[b] = q
        q, vs[b] = _quantised(normal(K, cap, D) * width.flip(0)[:, None], on)
        vc[b] = q.unflatten(1, (-1, BLOCK)).transpose(-1, -2)
    st.update(k=kc, v=vc, ks=ks, vs=vs)
    if c["kind"] == "attend":
        st["out"] = torch.zeros(B * G, H * D, dtype=torch.bfloat16, device="cuda")
        if c["weights"]:
            st["acc"] = torch.rand(B, K, cap, generator=g, device="cuda")
            st["acc_out"] = torch.zeros(B, K, cap, device="cuda")
    if c["kind"] == "evict":
        cap2 = (c["keep"] + BLOCK - 1) // BLOCK * BLOCK
        # accumulated attention is heavy-tailed: a few rows have most of it
        st["acc"] = torch.exp(2 * normal(B, K, cap))
        st.update(k2=torch.zeros(B, K, cap2, D, dtype=torch.uint8, device="cuda"), v2=torch.zeros(B, K, cap2 // BLOCK, D, BLOCK, dtype=torch.uint8, device="cuda"),
                  ks2=torch.zeros(B, K, cap2 // BLOCK, device="cuda"), vs2=torch.zeros(B, K, cap2 // BLOCK, device="cuda"),
                  acc2=torch.zeros(B, K, cap2, device="cuda"), lens2=torch.zeros(B, dtype=torch.int32, device="cuda"),
                  rows2=torch.zeros(B, K, c["keep"], dtype=torch.int32, device="cuda"))
    return st


def _heads(st, what):
    """[B, heads, block, dim] of the projection's Q, K or V columns."""
    c = st["case"]
    x = st["qkv"].view(c["batch"], c["block"], c["heads"] + 2 * c["kv_heads"], c["dim"])
    at = {"q": 0, "k": c["heads"], "v": c["heads"] + c["kv_heads"]}[what]
    return x[:, :, at:at + c["heads" if what == "q" else "kv_heads"]].transpose(1, 2)


def _f8(codes):
    return codes.view(torch.float8_e4m3fn)


# ---- plain forms -----------------------------------------------------------------------------------------------------------------

def _append_side(codes, scale, at, new, lens, counts):
    """The block's rows into one side of the cache; at(b, h, row): the index of a row's channels in `codes`."""
    B, H, G, D = new.shape
    dev = new.device
    j = lens.long()[:, None] // BLOCK + torch.arange((2 * (BLOCK - 1) + G) // BLOCK, device=dev)                # blocks that may be touched
    pos = (j[:, :, None] * BLOCK + torch.arange(BLOCK, device=dev)).flatten(1)                                   # [B, rows]
    old, g = pos < lens[:, None], pos - lens.long()[:, None]
    there = old | (g < counts[:, None])
    b, h = torch.arange(B, device=dev)[:, None, None], torch.arange(H, device=dev)[None, :, None]
    place = at(b, h, pos[:, None])
    was, was_s = codes[place], scale[b, h, j[:, None]]
    rows = new.gather(2, g.clamp(0, G - 1)[:, None, :, None].expand(B, H, -1, D)).float()
    q, s = _quantised(torch.where(old[:, None, :, None], _rows(was, was_s), rows), there[:, None])
    touched = (j * BLOCK < lens[:, None] + counts[:, None]) & (counts[:, None] > 0)
    changed = touched.repeat_interleave(BLOCK, 1) & there
    codes[place] = torch.where(changed[:, None, :, None], q, was)
    scale[b, h, j[:, None]] = torch.where(touched[:, None], s, was_s)


def _append(st):
    _append_side(st["k"], st["ks"], lambda b, h, r: (b, h, r), _heads(st, "k"), st["lens"], st["counts"])
    _append_side(st["v"], st["vs"], lambda b, h, r: (b, h, r // BLOCK, slice(None), r % BLOCK), _heads(st, "v"), st["lens"], st["counts"])


def _attend(st):
    c = st["case"]
    n = st["lens"].long() + st["counts"]
    rows = torch.arange(st["cap"], device="cuda")
    there = (rows < n[:, None])[:, None, :, None]
    k = torch.where(there, _rows(st["k"], st["ks"]), 0.0)
    v = torch.where(there, _rows(_unblock(st["v"]), st["vs"]), 0.0)
    q = _heads(st, "q").float().unflatten(1, (c["kv_heads"], -1)).flatten(2, 3)                # [B, kv_heads, group * block, dim]
    s = (q @ k.transpose(-1, -2)) / math.sqrt(c["dim"])
    s = s.masked_fill(~there.transpose(-1, -2), -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = (p @ v).unflatten(2, (-1, c["block"])).flatten(1, 2).transpose(1, 2).flatten(2)          # [B, block, heads * dim]
    live = torch.arange(c["block"], device="cuda") < st["counts"][:, None]
    out = st["out"].view(o.shape)
    out.copy_(torch.where(live[..., None], o.to(out.dtype), out))
    if c["weights"]:
        w = (p.unflatten(2, (-1, c["block"])) * live[:, None, None, :, None]).sum((2, 3))
        w = w + torch.where(rows < st["lens"][:, None, None], st["acc"], 0.0)
        st["acc_out"].copy_(torch.where(there[..., 0], w, st["acc_out"]))


def _evict(st):
    c = st["case"]
    n, rows = st["lens"].long()[:, None, None], torch.arange(st["cap"], device="cuda")
    key = torch.where(rows >= n - c["recent"], math.inf, st["acc"].nan_to_num(nan=-math.inf))
    order = torch.sort(torch.where(rows < n, key, -math.inf), dim=-1, descending=True, stable=True).indices[..., :c["keep"]]
    kept = torch.sort(torch.where(order < n, order, st["cap"]), dim=-1).values                    # ascending, what is not there last
    there = kept < st["cap"]
    pad = -c["keep"] % BLOCK
    at = torch.nn.functional.pad(kept.clamp_max(st["cap"] - 1), (0, pad))
    there = torch.nn.functional.pad(there, (0, pad))
    at4 = at[..., None].expand(*at.shape, c["dim"])
    blocks = there.unflatten(-1, (-1, BLOCK)).any(-1)
    k, ks = _quantised(_rows(st["k"], st["ks"]).gather(2, at4), there)
    v, vs = _quantised(_rows(_unblock(st["v"]), st["vs"]).gather(2, at4), there)
    st["k2"].copy_(torch.where(there[..., None], k, st["k2"]))
    st["v2"].copy_(torch.where(there[..., None], v, _unblock(st["v2"])).unflatten(-2, (-1, BLOCK)).transpose(-1, -2))
    st["ks2"].copy_(torch.where(blocks, ks, st["ks2"]))
    st["vs2"].copy_(torch.where(blocks, vs, st["vs2"]))
    st["acc2"].copy_(torch.where(there, st["acc"].gather(2, at), st["acc2"]))
    st["lens2"].copy_(st["lens"].clamp_max(c["keep"]))
    st["rows2"].copy_(torch.where(kept < st["cap"], kept, -1))


def _token_scores(st):
    c = st["case"]
    x = st["logits"][:, :c["vocab"]].float()
    if c["exclude"] >= 0:
        x = x.masked_fill(torch.arange(c["vocab"], device="cuda") == c["exclude"], -math.inf)
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    st["logprob"].copy_((x.gather(1, st["tokens"].long()[:, None]) - lse)[:, 0])
    st["entropy"].copy_((torch.log(total) - (e * torch.where(e > 0, x - m, 0.0)).sum(1, keepdim=True) / total)[:, 0])
    if c["top"]:
        v, i = torch.sort(x, dim=1, descending=True, stable=True)
        st["top_ids"].copy_(i[:, :c["top"]])
        st["top_logprobs"].copy_(v[:, :c["top"]] - lse)


# ---- the library's calls ---------------------------------------------------------------------------------------------------------

def _library(st):
    from paper_2511_15927_b200 import binding as dm
    c = st["case"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["kind"] == "scores":
        dm.dm_token_scores(c["rows"], c["vocab"], c["pitch"], dm.DM_BF16 if c["dtype"] == "bf16" else dm.DM_F32, st["logits"].data_ptr(), st["tokens"].data_ptr(),
                           c["exclude"], c["top"], st["logprob"].data_ptr(), st["entropy"].data_ptr(), st["top_ids"].data_ptr(), st["top_logprobs"].data_ptr(),
                           stream)
        return
    if "cfg" not in st:                                             # what a program keeps with its cache: the descriptions and the workspace
        st["cfg"] = dm.dm_kv8_cfg(c["batch"], c["block"], c["heads"], c["kv_heads"], c["dim"], dm.DM_BF16 if c["dtype"] == "bf16" else dm.DM_F32)
        st["cache"] = dm.dm_kv8_cache(st["k"].data_ptr(), st["v"].data_ptr(), st["ks"].data_ptr(), st["vs"].data_ptr(), st["cap"])
        need = 0
        if c["kind"] == "attend":
            need = dm.dm_kv8_attention_workspace_bytes(st["cfg"], c["len"])
        if c["kind"] == "evict":
            need = dm.dm_kv8_evict_workspace_bytes(st["cfg"], c["len"], c["keep"])
            st["cache2"] = dm.dm_kv8_cache(st["k2"].data_ptr(), st["v2"].data_ptr(), st["ks2"].data_ptr(), st["vs2"].data_ptr(), st["k2"].shape[2])
        st["ws"] = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    cfg, es = st["cfg"], st["qkv"].element_size()
    pitch, q = st["qkv"].shape[1], st["qkv"].data_ptr()
    counts = st["counts"].data_ptr() if c["padded"] else 0
    if c["kind"] == "append":
        k = q + c["heads"] * c["dim"] * es
        dm.dm_kv8_append(cfg, st["cache"], k, k + c["kv_heads"] * c["dim"] * es, pitch, st["lens"].data_ptr(), counts, stream)
    elif c["kind"] == "attend":
        w = c["weights"]
        dm.dm_kv8_attention(cfg, st["cache"], q, pitch, st["lens"].data_ptr(), counts, c["len"], st["acc"].data_ptr() if w else 0,
                            st["acc_out"].data_ptr() if w else 0, st["out"].data_ptr(), c["heads"] * c["dim"], st["ws"].data_ptr(), st["ws"].numel(), stream)
    else:
        dm.dm_kv8_evict(cfg, st["cache"], st["cache2"], st["acc"].data_ptr(), st["acc2"].data_ptr(), st["lens"].data_ptr(), st["lens2"].data_ptr(), c["len"],
                        c["keep"], c["recent"], st["rows2"].data_ptr(), st["ws"].data_ptr(), st["ws"].numel(), stream)


def run(state):
    kind = state["case"]["kind"]
    if own:
        _library(state)
    else:
        {"append": _append, "attend": _attend, "evict": _evict, "scores": _token_scores}[kind](state)
    if kind == "append":
        return {"k": _f8(state["k"]), "v": _f8(state["v"]), "k_scale": state["ks"], "v_scale": state["vs"]}
    if kind == "attend":
        return {"out": state["out"], **({"acc": state["acc_out"]} if state["case"]["weights"] else {})}
    if kind == "evict":
        return {"k": _f8(state["k2"]), "v": _f8(state["v2"]), "k_scale": state["ks2"], "v_scale": state["vs2"], "acc": state["acc2"], "lens": state["lens2"],
                "rows": state["rows2"]}
    return {n: state[n] for n in ("logprob", "entropy") + (("top_ids", "top_logprobs") if state["case"]["top"] else ())}


def work(case):
    c = case
    if c["kind"] == "scores":
        es = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": c["rows"] * (c["vocab"] * es + 12 + 8 * c["top"]), "flops": c["rows"] * c["vocab"] * 5}
    lens, counts, K, D = _lens(c), _counts(c), c["kv_heads"], c["dim"]
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "append":
        rows = sum(counts)
        return {"bytes": 2 * rows * K * D * (es + 1) + rows * K * 8 // BLOCK, "flops": 4 * rows * K * D}
    if c["kind"] == "attend":
        seen = sum(a + b for a, b in zip(lens, counts) if b)
        pairs = sum((a + b) * b for a, b in zip(lens, counts))
        w = c["weights"]
        return {"bytes": seen * K * (2 * D + 8 / BLOCK + (8 if w else 0)) + 4 * sum(counts) * c["heads"] * D, "flops": pairs * c["heads"] * (4 * D + (1 if w else 0))}
    kept = sum(min(n, c["keep"]) for n in lens)
    return {"bytes": K * (sum(lens) * 4 + kept * (4 * D + 4 + 4 + 16 / BLOCK)), "flops": kept * K * 4 * D}


# ---- 64 bits ---------------------------------------------------------------------------------------------------------------------

def _e4m3(x):
    """The e4m3 value next to x (|x| <= 448), ties to the even one."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6)))
    e = torch.where(torch.exp2(e) > x.abs().clamp_min(2.0 ** -6), e - 1, torch.where(torch.exp2(e + 1) <= x.abs(), e + 1, e))
    return torch.round(x * torch.exp2(3 - e)) * torch.exp2(e - 3)


def exact(case, seed):
    def _codes64(x):
        """Values of the codes and the scale of one block of rows x [rows, dim] in 64 bits."""
        top = float(x.abs().max())
        s = FLOOR
        while s * TOP < top:
            s *= 2
        while s > FLOOR and s / 2 * TOP >= top:
            s /= 2
        return _e4m3(x / s), s

    def _exact_side(codes, scale, new, lens, counts):
        """One side of an append, block by block: codes' values [B, H, cap, dim] and scales, changed in place."""
        for b in range(new.shape[0]):
            lo, hi = lens[b], lens[b] + counts[b]
            for j in range(lo // BLOCK, (hi + BLOCK - 1) // BLOCK if hi > lo else 0):
                r0, r1 = j * BLOCK, min(hi, (j + 1) * BLOCK)
                at = max(lo, r0)
                for h in range(new.shape[1]):
                    x = torch.cat([codes[b, h, r0:at] * scale[b, h, j], new[b, h, at - lo:r1 - lo]])
                    codes[b, h, r0:r1], scale[b, h, j] = _codes64(x)

    c = case
    st = prepare(c, seed)
    if c["kind"] == "scores":
        lp, en, tops = [], [], []
        for r in range(0, c["rows"], 1024):
            x = st["logits"][r:r + 1024, :c["vocab"]].double()
            if c["exclude"] >= 0:
                x[:, c["exclude"]] = -math.inf
            q = torch.log_softmax(x, 1)
            lp.append(q.gather(1, st["tokens"][r:r + 1024].long()[:, None])[:, 0])
            en.append(-torch.nan_to_num(q.exp() * q, nan=0.0).sum(1))
            tops.append(q.topk(c["top"], 1).values)
        return {"logprob": torch.cat(lp), "entropy": torch.cat(en), "top_ids": None, "top_logprobs": torch.cat(tops)}
    lens, counts, B, K, D = _lens(c), _counts(c), c["batch"], c["kv_heads"], c["dim"]
    k, v = st["k"].view(torch.float8_e4m3fn).float(), st["v"].view(torch.float8_e4m3fn).float().permute(0, 1, 2, 4, 3).reshape(st["k"].shape)
    ks, vs = st["ks"].double(), st["vs"].double()
    if c["kind"] == "append":
        if 2 * K * sum(counts) // BLOCK > 20000:                    # block by block: too many of them for a few seconds
            return None
        host = [t.cpu().double() for t in (k, ks, v, vs, _heads(st, "k"), _heads(st, "v"))]
        _exact_side(host[0], host[1], host[4], lens, counts)
        _exact_side(host[2], host[3], host[5], lens, counts)
        v = host[2].unflatten(2, (-1, BLOCK)).transpose(-1, -2).contiguous()
        return {"k": host[0], "v": v, "k_scale": host[1], "v_scale": host[3]}
    if c["kind"] == "attend":
        G, group = c["block"], c["heads"] // K
        out = torch.zeros(B, G, c["heads"], D, dtype=torch.float64, device="cuda")
        acc = torch.zeros(B, K, st["cap"], dtype=torch.float64, device="cuda")
        q = _heads(st, "q").double()
        for b in range(B):
            n, live = lens[b] + counts[b], counts[b]
            if not n or not live:
                if n:
                    acc[b, :, :n] = st["acc"][b, :, :n].double() if c["weights"] else 0
                continue
            for h in range(K):
                kk = k[b, h, :n].double() * ks[b, h].repeat_interleave(BLOCK)[:n, None]
                vv = v[b, h, :n].double() * vs[b, h].repeat_interleave(BLOCK)[:n, None]
                qq = q[b, h * group:(h + 1) * group, :live].reshape(-1, D)
                p = torch.softmax(qq @ kk.T / math.sqrt(D), -1)
                out[b, :live, h * group:(h + 1) * group] = (p @ vv).view(group, live, D).transpose(0, 1)
                if c["weights"]:
                    acc[b, h, :n] = p.sum(0)
                    acc[b, h, :lens[b]] += st["acc"][b, h, :lens[b]].double()
        return {"out": out.view(B * G, -1), **({"acc": acc} if c["weights"] else {})}
    if B * K * c["keep"] // BLOCK > 10000:
        return None
    keep, cap2 = c["keep"], st["k2"].shape[2]
    score = st["acc"].cpu().double()
    k, v, ks, vs = (t.cpu().double() for t in (k, v, ks, vs))
    k2, v2 = torch.zeros(B, K, cap2, D, dtype=torch.float64), torch.zeros(B, K, cap2 // BLOCK, D, BLOCK, dtype=torch.float64)
    ks2, vs2 = torch.zeros(B, K, cap2 // BLOCK, dtype=torch.float64), torch.zeros(B, K, cap2 // BLOCK, dtype=torch.float64)
    acc2 = torch.zeros(B, K, cap2, dtype=torch.float64)
    for b in range(B):
        n = lens[b]
        for h in range(K):
            old = max(0, n - c["recent"])
            best = score[b, h, :old].tolist()
            first = sorted(range(old), key=lambda i: (-best[i], i))[:keep - (n - old)] if n > keep else range(old)
            rows = torch.tensor(sorted(first) + list(range(old, n)))
            acc2[b, h, :len(rows)] = score[b, h, rows]
            for j in range((len(rows) + BLOCK - 1) // BLOCK):
                r = rows[j * BLOCK:(j + 1) * BLOCK]
                k2[b, h, j * BLOCK:j * BLOCK + len(r)], ks2[b, h, j] = _codes64(k[b, h, r] * ks[b, h, r // BLOCK, None])
                x, vs2[b, h, j] = _codes64(v[b, h, r] * vs[b, h, r // BLOCK, None])
                v2[b, h, j, :, :len(r)] = x.T
    return {"k": k2, "v": v2, "k_scale": ks2, "v_scale": vs2, "acc": acc2, "lens": None, "rows": None}
