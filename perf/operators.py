"""Performance cases of the paged serving operators: appending rotated keys and
values to a paged cache (bf16, or 8 bits with a scale per block of tokens and
head), attention over that cache, and the draw of tokens from given uniforms.

Each case runs in one of two forms.  With ``own`` false it is the plain form:
elementary torch operations in 32 bits (64 for the draw, whose cumulative sums
decide between neighbouring tokens).  With ``own`` true it is the library's
calls, as a serving loop makes them.  Both read and write the same tensors:

    k cache  [n_pages][hkv][page][hd]            v cache [n_pages][hkv][page/16][hd][16]
    scales   [n_pages][hkv][page/block] float32  (powers of two; 8-bit caches)
    table    [B][pages of a sequence] int32      row_start [B + 1], pos0 [B] int32

Head shapes and context lengths are those of the Llama-3-8B- and Qwen3-8B-shaped
decoders and of the tiny float32 one.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

MIN_EXP = -100  # smallest scale: 2^-100


# ---------------------------------------------------------------- the cases
def listed():
    llama = dict(hq=32, hkv=8, hd=128)
    return [
        # one decode step of one sequence: latency of the smallest call
        dict(name="append_one", op="append", B=1, lo=1, hi=1, ctx=8191, **llama, page=64, block=16,
             kind="e4m3", dtype="bf16"),
        # one verify step of a served batch: 1 to 9 rows a sequence, float32 rows, 32-token scales
        dict(name="append_verify_48", op="append", B=48, lo=1, hi=9, ctx=1500, **llama, page=32,
             block=32, kind="e4m3", dtype="f32"),
        # prompts entering together, one scale per page
        dict(name="append_prompts", op="append", B=5, lo=900, hi=4096, ctx=300, **llama, page=64,
             block=64, kind="e4m3", dtype="bf16"),
        # a decode step at 8K context, one sequence
        dict(name="attend_one_8k", op="attend", B=1, lo=1, hi=1, ctx_lo=8191, ctx=8191, **llama,
             page=64, block=16, kind="e4m3", dtype="bf16"),
        # the verify rows of one round at 32K context (gamma 6)
        dict(name="attend_verify_32k", op="attend", B=1, lo=7, hi=7, ctx_lo=32761, ctx=32761,
             **llama, page=256, block=32, kind="e4m3", dtype="bf16"),
        # a decode step of a served batch with ragged contexts: cache bandwidth
        dict(name="attend_batch_64", op="attend", B=64, lo=1, hi=1, ctx_lo=500, ctx=15000, **llama,
             page=64, block=16, kind="e4m3", dtype="bf16"),
        # the tiny decoder's heads, float32 rows, bf16 cache in the smallest pages
        dict(name="attend_tiny_17", op="attend", B=17, lo=1, hi=5, ctx_lo=1, ctx=900, hq=4, hkv=2,
             hd=64, page=16, block=16, kind="bf16", dtype="f32"),
        # a prompt chunk against its history: matrix-product rate
        dict(name="attend_chunk_2048", op="attend", B=1, lo=2048, hi=2048, ctx_lo=6000, ctx=6000,
             **llama, page=64, block=16, kind="e4m3", dtype="bf16"),
        # ragged chunks of several prompts over a bf16 cache
        dict(name="attend_chunks_6", op="attend", B=6, lo=100, hi=700, ctx_lo=0, ctx=3000, **llama,
             page=128, block=16, kind="bf16", dtype="bf16"),
        # one token of one sequence
        dict(name="draw_one", op="draw", rows=1, vocab=128256, dtype="f32", mix="paper"),
        # the rows of a verify round, each request with its own settings
        dict(name="draw_7", op="draw", rows=7, vocab=151936, dtype="f32", mix="mixed"),
        # a served batch
        dict(name="draw_256", op="draw", rows=256, vocab=128256, dtype="f32", mix="mixed"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "draw"])
    if op == "draw":
        return dict(op=op, rows=_log(rng, 1, 200), vocab=_log(rng, 1000, 152000),
                    dtype=rng.choice(["f32", "f32", "bf16"]),
                    mix=rng.choice(["paper", "mixed", "open"]))
    heads = rng.choice([dict(hq=32, hkv=8, hd=128), dict(hq=32, hkv=8, hd=128),
                        dict(hq=8, hkv=2, hd=128), dict(hq=4, hkv=2, hd=64),
                        dict(hq=12, hkv=4, hd=64), dict(hq=9, hkv=1, hd=128)])
    page = rng.choice([16, 32, 64, 128, 256])
    c = dict(op=op, **heads, page=page,
             block=rng.choice([b for b in (16, 32, 64) if b <= page]),
             kind=rng.choice(["e4m3", "e4m3", "bf16"]), dtype=rng.choice(["bf16", "bf16", "f32"]),
             spread=rng.randint(1, 10 ** 6))
    if op == "append":
        hi = _log(rng, 1, 3000)
        return dict(c, B=_log(rng, 1, max(1, min(64, 12000 // hi))), lo=rng.randint(1, hi), hi=hi,
                    ctx=_log(rng, 1, 4000))
    if rng.random() < 0.7:  # decode and verify steps
        hi = rng.choice([1, 1, rng.randint(2, 16)])
        ctx = _log(rng, 16, 32000)
        return dict(c, B=_log(rng, 1, max(1, min(64, 400000 // ctx))), lo=rng.randint(1, hi),
                    hi=hi, ctx_lo=rng.randint(0, ctx), ctx=ctx)
    hi = _log(rng, 17, 1500)
    ctx = _log(rng, 1, 5000)
    return dict(c, B=_log(rng, 1, max(1, min(8, 2000 // hi))), lo=rng.randint(1, hi), hi=hi,
                ctx_lo=rng.randint(0, ctx), ctx=ctx)


# ------------------------------------------------------------------- inputs
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _sizes(case):
    """(new rows, position of the first of them) of every sequence: by the case alone."""
    r = random.Random(case.get("spread", 7))
    n = [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    lo = case.get("ctx_lo", 0 if case["B"] > 1 else case["ctx"])
    return n, [r.randint(lo, case["ctx"]) for _ in range(case["B"])]


def _gen(seed, part):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1009 + part)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def prepare(case, seed):
    if case["op"] == "draw":
        return _prepare_draw(case, seed)
    n, p0 = _sizes(case)
    B, page, hkv, hd = case["B"], case["page"], case["hkv"], case["hd"]
    rows = sum(n)
    need = [-(-(p + m) // page) for p, m in zip(p0, n)]
    n_pages = sum(need) + 1
    order = np.random.RandomState(seed % (1 << 31)).permutation(n_pages)
    table = np.zeros((B, max(need)), np.int32)  # page 0 where a sequence needs none
    at = 0
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    g = _gen(seed, 1)
    heads = case["hq"] + 2 * hkv
    # rows of a fused projection: some channels of the keys an order larger than the rest
    qkv = _randn(g, rows, heads, hd)
    qkv[:, case["hq"]:case["hq"] + hkv] *= 1 + 7 * (torch.rand(hkv, hd, generator=g, device="cuda") > 0.97)
    qkv = qkv.to(DT[case["dtype"]])
    st = dict(case=case, rows=rows, max_rows=max(n), max_len=max(p + m for p, m in zip(p0, n)),
              table=torch.from_numpy(table).cuda(),
              row_start=torch.from_numpy(np.cumsum([0] + n).astype(np.int32)).cuda(),
              pos0=torch.from_numpy(np.array(p0, np.int32)).cuda(),
              q=qkv[:, :case["hq"]], k=qkv[:, case["hq"]:case["hq"] + hkv],
              v=qkv[:, case["hq"] + hkv:])
    for name, shape in (("kc", (n_pages, hkv, page, hd)), ("vc", (n_pages, hkv, page // 16, hd, 16))):
        if case["kind"] == "bf16":
            st[name] = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        else:  # codes with a spread of about 100 and scales of 2^-6 or 2^-7
            x = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0, 90, generator=g)
            st[name] = x.clamp_(-448, 448).to(torch.float8_e4m3fn)
            s = torch.randint(0, 2, (n_pages, hkv, page // case["block"]), generator=g, device="cuda")
            st[name + "_scale"] = torch.exp2(-6.0 - s)
    st.setdefault("kc_scale", None)
    st.setdefault("vc_scale", None)
    if case["op"] == "append":
        f = torch.arange(hd // 2, device="cuda", dtype=torch.float64)
        ang = torch.arange(table.shape[1] * page, device="cuda", dtype=torch.float64)[:, None] * \
            5e5 ** (-2 * f / hd)
        st["rope"] = torch.stack([ang.cos(), ang.sin()], -1).float()
        st["q_out"] = torch.empty(rows, case["hq"], hd, dtype=qkv.dtype, device="cuda")
    else:
        st["out"] = torch.empty(rows, case["hq"], hd, dtype=qkv.dtype, device="cuda")
        st["lse"] = torch.empty(rows, case["hq"], dtype=torch.float32, device="cuda")
    return st


def _prepare_draw(case, seed):
    rows, vocab = case["rows"], case["vocab"]
    g = _gen(seed, 2)
    lg = _randn(g, rows, vocab) * 2.5
    # a few likely tokens a row, as a language model gives
    top = torch.randint(0, vocab, (rows, 8), generator=g, device="cuda")
    lg.scatter_add_(1, top, 8 + 3 * _randn(g, rows, 8))
    # some tokens barred by a mask
    lg.masked_fill_(torch.rand(rows, vocab, generator=g, device="cuda") < 0.01, -math.inf)
    r = np.random.RandomState(seed % (1 << 31))
    if case["mix"] == "paper":  # the paper's setting
        t, k, p, m = np.full(rows, 0.7), np.full(rows, 50), np.full(rows, 0.95), np.zeros(rows)
    elif case["mix"] == "open":  # temperature alone
        t, k, p, m = r.uniform(0.5, 1.5, rows), np.zeros(rows), np.ones(rows), np.zeros(rows)
    else:
        t = r.choice([0.0, 0.6, 0.8, 1.0, 1.3], rows)
        k = r.choice([0, 20, 50, 1000], rows)
        p = r.choice([1.0, 0.95, 0.9, 0.5], rows)
        m = r.choice([0.0, 0.02, 0.1], rows)
    dev = lambda a, d: torch.from_numpy(a.astype(d)).cuda()  # noqa: E731
    return dict(case=case, logits=lg.to(DT[case["dtype"]]), temperature=dev(t, np.float32),
                top_k=dev(k, np.int32), top_p=dev(p, np.float32), min_p=dev(m, np.float32),
                u=dev(r.uniform(0, 1, rows), np.float32).clamp_(max=1 - 2 ** -24),
                tokens=torch.empty(rows, dtype=torch.int32, device="cuda"),
                logprob=torch.empty(rows, dtype=torch.float32, device="cuda"),
                kept=torch.empty(rows, dtype=torch.int32, device="cuda"))


# ------------------------------------------------------------------ one pass
def run(st):
    op = st["case"]["op"]
    if op == "append":
        (_own_append if own else _plain_append)(st)
        out = dict(q=st["q_out"], k=st["kc"], v=st["vc"])
        if st["kc_scale"] is not None:
            out.update(k_scale=st["kc_scale"], v_scale=st["vc_scale"])
        return out
    if op == "attend":
        (_own_attend if own else _plain_attend)(st)
        return dict(out=st["out"], lse=st["lse"])
    (_own_draw if own else _plain_draw)(st)
    return dict(tokens=st["tokens"], logprob=st["logprob"], kept=st["kept"])


def _cache(st):
    """The cache handle and the workspace that a serving loop keeps."""
    from paper_2602_20217_amd import engine as E
    if "handle" not in st:
        st["handle"] = E.PagedCache.over(st["kc"], st["vc"], st["kc_scale"], st["vc_scale"])
        if st["case"]["op"] == "attend":
            st["ws"] = E.paged_attention_workspace(st["handle"], st["case"]["B"], st["rows"],
                                                   st["case"]["hq"], st["max_rows"], st["max_len"])
    return E, st["handle"]


def _own_append(st):
    E, cache = _cache(st)
    E.paged_append(cache, st["table"], st["row_start"], st["pos0"], st["k"], st["v"], q=st["q"],
                   rope=st["rope"], q_out=st["q_out"], max_rows=st["max_rows"])


def _own_attend(st):
    E, cache = _cache(st)
    E.paged_attention(cache, st["table"], st["row_start"], st["pos0"], st["q"], out=st["out"],
                      lse=st["lse"], max_rows=st["max_rows"], max_len=st["max_len"],
                      workspace=st["ws"])


def _own_draw(st):
    from paper_2602_20217_amd import engine as E
    if "ws" not in st:
        st["ws"] = E.sample_draw_workspace(*st["logits"].shape, device=st["logits"].device)
    E.sample_draw(st["logits"], st["u"], st["temperature"], st["top_k"], st["top_p"], st["min_p"],
                  tokens=st["tokens"], logprob=st["logprob"], kept=st["kept"], workspace=st["ws"])


# --------------------------------------------------------------- plain forms
def _rows_of(st):
    """Sequence and position of every row."""
    n = st["row_start"][1:] - st["row_start"][:-1]
    seq = torch.repeat_interleave(torch.arange(st["case"]["B"], device="cuda"), n,
                                  output_size=st["rows"])
    pos = st["pos0"][seq] + torch.arange(st["rows"], device="cuda") - st["row_start"][seq]
    return seq, pos.long()


def _rotate(x, cs):
    h = x.shape[-1] // 2
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _needed(amax):
    """Smallest power of two s with amax <= 448 s (448 = 0.875 2^9), at least 2^-100."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.exp2(torch.where(amax > 0, e, MIN_EXP).clamp(min=MIN_EXP).float())


def _plain_append(st):
    c = st["case"]
    page, block = c["page"], c["block"]
    seq, pos = _rows_of(st)
    cs = st["rope"][pos]
    st["q_out"].copy_(_rotate(st["q"].float(), cs))
    pg, slot = st["table"][seq, pos // page].long(), pos % page
    new = dict(kc=_rotate(st["k"].float(), cs), vc=st["v"].float())
    if c["kind"] == "bf16":
        st["kc"][pg, :, slot] = new["kc"].to(torch.bfloat16)
        st["vc"][pg, :, slot // 16, :, slot % 16] = new["vc"].to(torch.bfloat16)
        return
    nb = page // block
    blk = pg * nb + slot // block  # the row's scale block, over all pages
    old = (pos - pos % block) < st["pos0"][seq]  # it holds earlier tokens
    # the one block of every sequence that its first new row shares with earlier tokens
    p0 = st["pos0"].long()
    shared = p0 % block != 0
    pg0 = st["table"][torch.arange(c["B"], device="cuda"), p0 // page].long()
    in0 = (p0 % page) // block * block  # its first token in the page
    t = torch.arange(block, device="cuda")
    earlier = (t[None] < (p0 % block)[:, None]) & shared[:, None]  # [B][block]
    tok = in0[:, None] + t
    for name in ("kc", "vc"):
        x = new[name]
        sc = st[name + "_scale"]
        flat = sc.transpose(1, 2).reshape(-1, c["hkv"])  # [pages * nb][hkv]
        amax = torch.zeros_like(flat).scatter_reduce(
            0, blk[:, None].expand(-1, c["hkv"]), x.abs().amax(-1), "amax")[blk]
        s = torch.maximum(_needed(amax), torch.where(old[:, None], flat[blk], 0))
        # earlier tokens of a shared block take its new scale
        code = st[name].view(torch.uint8)
        s_old = sc[pg0, :, in0 // block]
        s_new = torch.zeros_like(flat)
        s_new[blk] = s
        s_new = torch.where(shared[:, None], s_new[pg0 * nb + in0 // block], s_old)
        sel = (pg0[:, None], slice(None), tok) if name == "kc" else \
            (pg0[:, None], slice(None), tok // 16, slice(None), tok % 16)
        was = code[sel]  # [B][block][hkv][hd]
        val = was.view(torch.float8_e4m3fn).float() * (s_old / s_new)[:, None, :, None]
        code[sel] = torch.where(earlier[:, :, None, None],
                                val.to(torch.float8_e4m3fn).view(torch.uint8), was)
        sel = (pg, slice(None), slot) if name == "kc" else \
            (pg, slice(None), slot // 16, slice(None), slot % 16)
        code[sel] = (x / s[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        sc[pg, :, slot // block] = s


def _plain_attend(st):
    c = st["case"]
    B, page, hq, hkv, hd, R, N = (c["B"], c["page"], c["hq"], c["hkv"], c["hd"], st["max_rows"],
                                  st["max_len"])
    t = torch.arange(N, device="cuda")
    pg, slot = st["table"][:, t // page].long(), (t % page).expand(B, -1)
    k = st["kc"].view(torch.uint8 if c["kind"] == "e4m3" else torch.bfloat16)[pg, :, slot]
    v = st["vc"].view(torch.uint8 if c["kind"] == "e4m3" else torch.bfloat16)[
        pg, :, slot // 16, :, slot % 16]  # [B][N][hkv][hd]
    if c["kind"] == "e4m3":
        k = k.view(torch.float8_e4m3fn).float() * st["kc_scale"][pg, :, slot // c["block"]][..., None]
        v = v.view(torch.float8_e4m3fn).float() * st["vc_scale"][pg, :, slot // c["block"]][..., None]
    seq, pos = _rows_of(st)
    i = pos - st["pos0"][seq]
    q = torch.zeros(B, R, hq, hd, device="cuda")
    q[seq, i] = st["q"].float()
    # [B][hkv][R G][hd] x [B][hkv][hd][N]
    q = q.view(B, R, hkv, hq // hkv, hd).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, hd)
    s = q @ k.float().permute(0, 2, 3, 1).contiguous() * hd ** -0.5
    far = t[None, None] > (st["pos0"][:, None] + torch.arange(R, device="cuda"))[..., None]
    s = s.view(B, hkv, R, -1, N).masked_fill_(far[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    s = s.sub_(m).exp_()
    l = s.sum(-1, keepdim=True)
    o = (s.view(B, hkv, -1, N) @ v.float().permute(0, 2, 1, 3).contiguous()).view(B, hkv, R, -1, hd) / l
    st["out"].copy_(o.permute(0, 2, 1, 3, 4).reshape(B, R, hq, hd)[seq, i])
    st["lse"].copy_((m + l.log())[..., 0].permute(0, 2, 1, 3).reshape(B, R, hq)[seq, i])


def _plain_draw(st):
    lg, ids = st["logits"].float().sort(dim=1, descending=True, stable=True)
    t = st["temperature"].double()[:, None]
    greedy = t <= 0
    x = (lg.double() - lg[:, :1].double()) / torch.where(greedy, 1, t)
    w = x.exp()
    V = lg.shape[1]
    rank = torch.arange(V, device="cuda")
    k = torch.where(st["top_k"] > 0, st["top_k"], V)[:, None]
    k = torch.where(greedy, 1, k)
    keep = (rank < k) & (w >= st["min_p"].double()[:, None]) & (lg > -math.inf)
    w = w * keep
    cum = w.cumsum(1)
    p = st["top_p"].double()[:, None]
    keep &= (cum - w < p * cum[:, -1:]) | (p >= 1) | (rank == 0)
    w = w * keep
    cum = w.cumsum(1)
    z = cum[:, -1]
    kept = keep.sum(1)
    j = (cum <= st["u"].double()[:, None] * z[:, None]).sum(1)
    j = torch.minimum(j, kept - 1)[:, None]
    st["tokens"].copy_(ids.gather(1, j)[:, 0])
    st["logprob"].copy_(x.gather(1, j)[:, 0] - z.log())
    st["kept"].copy_(kept)


# -------------------------------------------------------------- what it takes
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "draw":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * e + 28 * case["rows"], "flops": 12 * n}
    n, p0 = _sizes(case)
    rows, hq, hkv, hd = sum(n), case["hq"], case["hkv"], case["hd"]
    per = 2 * hkv * (hd * (1 + 4 / (hd * case["block"])) if case["kind"] == "e4m3" else 2 * hd)
    if case["op"] == "append":
        return {"bytes": rows * ((2 * hq + 2 * hkv) * hd * e + per + 4 * hd),
                "flops": rows * ((hq + hkv) * 3 * hd + 4 * hkv * hd)}
    keys = sum(m * p + m * (m + 1) // 2 for m, p in zip(n, p0))  # (row, key) pairs
    return {"bytes": sum(p + m for m, p in zip(n, p0)) * per + rows * hq * (2 * hd * e + 4),
            "flops": 4 * hq * hd * keys}


# ------------------------------------------------------ 64 bits, written apart
def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "draw": _exact_draw}[case["op"]](st)


def _e4m3(x):
    """float64 values to the nearest e4m3 value (ties to even), |x| <= 448."""
    _, e = np.frexp(np.abs(x))
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.round(x / step) * step


def _exact_append(st):
    c = st["case"]
    page, block, hd = c["page"], c["block"], c["hd"]
    h = hd // 2
    host = lambda x: x.double().cpu().numpy()  # noqa: E731
    q, k, v, rope = host(st["q"]), host(st["k"]), host(st["v"]), host(st["rope"])
    kc, vc = host(st["kc"]), host(st["vc"])
    e4 = c["kind"] == "e4m3"
    if e4:
        ks, vs = host(st["kc_scale"]), host(st["vc_scale"])
    table, start, pos0 = (st[x].cpu().numpy() for x in ("table", "row_start", "pos0"))
    qo = np.empty_like(q)
    for b in range(c["B"]):
        r = slice(start[b], start[b + 1])
        pos = pos0[b] + np.arange(start[b + 1] - start[b])
        cos, sin = rope[pos, :, 0][:, None], rope[pos, :, 1][:, None]
        turn = lambda x: np.concatenate([x[..., :h] * cos - x[..., h:] * sin,  # noqa: E731,B023
                                         x[..., h:] * cos + x[..., :h] * sin], -1)
        qo[r] = turn(q[r])
        kb, vb = turn(k[r]), v[r]
        at = 0
        while at < len(pos):  # one scale block after the other
            p = int(pos[at])
            end = min(len(pos), at + block - p % block)
            pg, s0 = table[b, p // page], p % page
            for x, cache, sc in ((kb, kc, ks if e4 else None), (vb, vc, vs if e4 else None)):
                y = x[at:end]
                slots = s0 + np.arange(end - at)
                first = s0 - s0 % block

                def place(slot, val):
                    if cache is kc:
                        cache[pg][:, slot] = val.transpose(1, 0, 2)
                    else:
                        cache[pg][:, slot // 16, :, slot % 16] = val

                if not e4:
                    place(slots, y)
                    continue
                amax = np.abs(y).max(axis=(0, 2))
                s = np.exp2(np.ceil(np.log2(np.maximum(amax, 1e-300) / 448.0)))
                n_old = s0 - first if p - p % block < pos0[b] else 0
                was = sc[pg, :, first // block].copy()
                if n_old:
                    s = np.maximum(s, was)
                    old = first + np.arange(n_old)
                    val = cache[pg][:, old].transpose(1, 0, 2) if cache is kc else \
                        cache[pg][:, old // 16, :, old % 16]
                    place(old, _e4m3(val * (was / s)[None, :, None]))
                place(slots, _e4m3(y / s[None, :, None]))
                sc[pg, :, first // block] = s
            at = end
    out = dict(q=torch.from_numpy(qo), k=torch.from_numpy(kc), v=torch.from_numpy(vc))
    if e4:
        out.update(k_scale=torch.from_numpy(ks), v_scale=torch.from_numpy(vs))
    return out


def _exact_attend(st):
    c = st["case"]
    page, hq, hkv, hd = c["page"], c["hq"], c["hkv"], c["hd"]
    table, start, pos0 = (st[x].cpu().numpy() for x in ("table", "row_start", "pos0"))
    out = torch.empty(st["rows"], hq, hd, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["rows"], hq, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        n = int(start[b + 1] - start[b])
        N = int(pos0[b]) + n
        pages = torch.from_numpy(table[b, :-(-N // page)]).cuda().long()
        k = st["kc"].view(torch.uint8)[pages] if c["kind"] == "e4m3" else st["kc"][pages]
        v = st["vc"].view(torch.uint8)[pages] if c["kind"] == "e4m3" else st["vc"][pages]
        if c["kind"] == "e4m3":
            k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
        v = v.to(torch.float32).transpose(3, 4).reshape(len(pages), hkv, page, hd).double()
        k = k.double()
        if c["kind"] == "e4m3":
            k *= st["kc_scale"][pages].double().repeat_interleave(c["block"], 2)[..., None]
            v *= st["vc_scale"][pages].double().repeat_interleave(c["block"], 2)[..., None]
        k = k.transpose(0, 1).reshape(hkv, -1, hd)[:, :N]
        v = v.transpose(0, 1).reshape(hkv, -1, hd)[:, :N]
        last = int(pos0[b]) + torch.arange(n, device="cuda")
        off = torch.arange(N, device="cuda")[None] > last[:, None]
        for h in range(hq):
            q = st["q"][start[b]:start[b + 1], h].double()
            s = (q @ k[h // (hq // hkv)].T.contiguous()) / math.sqrt(hd)
            s = s.masked_fill(off, -math.inf)
            z = torch.logsumexp(s, 1)
            lse[start[b]:start[b + 1], h] = z
            out[start[b]:start[b + 1], h] = torch.exp(s - z[:, None]) @ v[h // (hq // hkv)]
    return dict(out=out, lse=lse)


def _exact_draw(st):
    lg = st["logits"].double().cpu().numpy()
    T, K, P, M, U = (st[x].double().cpu().numpy() for x in
                     ("temperature", "top_k", "top_p", "min_p", "u"))
    tok, lp, kept = [], [], []
    for r, row in enumerate(lg):
        order = np.argsort(-row, kind="stable")
        order = order[:int(np.sum(row > -np.inf))]
        if T[r] <= 0:
            tok.append(order[0]), lp.append(0.0), kept.append(1)
            continue
        x = (row[order] - row[order[0]]) / T[r]
        if 0 < K[r] < len(x):
            x = x[:int(K[r])]
        if M[r] > 0:
            x = x[x >= np.log(M[r])]
        w = np.exp(x)
        c = np.cumsum(w)
        if P[r] < 1:
            x = x[:int(np.searchsorted(c, P[r] * c[-1])) + 1]
        z = c[len(x) - 1]
        j = min(int(np.searchsorted(c[:len(x)], U[r] * z, side="right")), len(x) - 1)
        tok.append(order[j]), lp.append(x[j] - np.log(z)), kept.append(len(x))
    return dict(tokens=torch.tensor(tok, dtype=torch.int32),
                logprob=torch.tensor(lp, dtype=torch.float64),
                kept=torch.tensor(kept, dtype=torch.int32))
