"""The paged cache through the C ABI: append with rotation and attention, against a
plain float64 implementation on the host.

Tolerances.  A rounding is off by at most half a step, relative to the value: 2^-24
in float32, 2^-8 in bf16, 2^-4 in e4m3.  Attention averages values of the cache, so
its error is held against the largest |value|:
  scores        about eight float32 roundings (the sum of products, the scale, the
                distance to the maximum): 2^-21 |score|, which moves a probability by
                as much, relative
  float32 rows  a probability to 2^-16 (two bf16 planes): 2^-15 with what else rounds
  bf16 rows     a probability to 2^-8 and the output to 2^-8: 2^-7
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2602_20217_amd import engine
    return engine


# ------------------------------------------------------------ plain form
def e4m3(x):
    """Nearest e4m3 value (ties to even) of float64 x, |x| <= 448; NaN stays."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(np.abs(np.nan_to_num(x)))
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.round(x / step) * step


def needed(amax):
    """Smallest power of two s >= 2^-100 with amax <= 448 s."""
    s = 2.0 ** -100
    while amax > 448 * s:
        s *= 2
    return s


class Plain:
    """The cache as float64 values by (page, head, slot), and its scales."""

    def __init__(self, n_pages, page, hkv, hd, kind, block):
        self.page, self.block, self.kind = page, block, kind
        self.k = np.zeros((n_pages, hkv, page, hd))
        self.v = np.zeros((n_pages, hkv, page, hd))
        self.known = np.zeros((n_pages, page), bool)  # slots that hold a token
        self.ks = np.zeros((n_pages, hkv, page // block))
        self.vs = np.zeros((n_pages, hkv, page // block))

    def append(self, table, start, pos0, k, v, rope, rows_of=None):
        """k, v float64 (already the values of their type)."""
        h = k.shape[2] // 2
        for b in range(len(pos0)):
            new = {}
            for i in range(start[b], start[b + 1]):
                p = pos0[b] + i - start[b]
                if p < 0:
                    continue
                kk = k[i]
                if rope is not None:
                    c, s = rope[p, :, 0], rope[p, :, 1]
                    kk = np.concatenate([kk[:, :h] * c - kk[:, h:] * s,
                                         kk[:, h:] * c + kk[:, :h] * s], 1)
                new[p] = (kk, v[i])
            for p in sorted(new):
                pg, sl = table[b, p // self.page], p % self.page
                first = p - p % self.block
                if p == first or p == min(new):  # a block's first new token: its scale
                    mem = [t for t in new if first <= t < first + self.block]
                    bl = (p % self.page) // self.block
                    for x, cache, sc in ((0, self.k, self.ks), (1, self.v, self.vs)):
                        if self.kind == "bf16":
                            continue
                        for hh in range(k.shape[1]):
                            a = np.abs(np.concatenate([new[t][x][hh] for t in mem]))
                            a = a[np.isfinite(a)]
                            s = needed(a.max() if a.size else 0.0)
                            old = [t for t in range(first, max(pos0[b], 0)) if t < p]
                            if old:
                                was = sc[pg, hh, bl]
                                s = max(s, was)
                                for t in old:
                                    y = cache[pg, hh, t % self.page]
                                    cache[pg, hh, t % self.page] = e4m3(y / s) * s
                            sc[pg, hh, bl] = s
                for x, cache, sc in ((0, self.k, self.ks), (1, self.v, self.vs)):
                    y = new[p][x]
                    if self.kind == "bf16":
                        y = torch.from_numpy(y).float().bfloat16().double().numpy()
                    else:
                        s = sc[pg, :, (p % self.page) // self.block][:, None]
                        with np.errstate(invalid="ignore"):
                            y = np.where(np.isfinite(y), e4m3(np.nan_to_num(y) / s) * s, np.nan)
                    cache[pg, :, sl] = y
                self.known[pg, sl] = True

    def attend(self, table, start, pos0, q, scale):
        rows, hq, hd = q.shape
        hkv = self.k.shape[1]
        out, lse = np.zeros((rows, hq, hd)), np.full((rows, hq), -np.inf)
        for b in range(len(pos0)):
            for i in range(start[b], start[b + 1]):
                n = pos0[b] + i - start[b] + 1
                t = [p for p in range(max(n, 0)) if 0 <= table[b, p // self.page] < len(self.k)]
                if not t:
                    continue
                pg, sl = table[b][np.array(t) // self.page], np.array(t) % self.page
                for h in range(hq):
                    g = h // (hq // hkv)
                    s = self.k[pg, g, sl] @ q[i, h] * scale
                    m = s.max()
                    w = np.exp(s - m)
                    out[i, h] = w @ self.v[pg, g, sl] / w.sum()
                    lse[i, h] = m + math.log(w.sum())
        return out, lse


def values(cache):
    """The cache's tensors as float64 (keys, values) [n_pages][hkv][page][hd]."""
    k = cache.k.float().cpu().double().numpy()
    v = cache.v.float().cpu().double().numpy()
    n, hkv, ng, hd, _ = v.shape
    v = v.transpose(0, 1, 2, 4, 3).reshape(n, hkv, ng * 16, hd)
    if cache.k_scale is not None:
        k = k * np.repeat(cache.k_scale.cpu().double().numpy(), cache.block, 2)[..., None]
        v = v * np.repeat(cache.v_scale.cpu().double().numpy(), cache.block, 2)[..., None]
    return k, v


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def rope_table(n, hd, theta=1e4):
    ang = np.arange(n)[:, None] * theta ** (-2.0 * np.arange(hd // 2) / hd)
    return np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)


class Case:
    """A cache, its plain twin, and sequences with tables of shuffled pages."""

    def __init__(self, E, B, hq, hkv, hd, page, block, kind, dtype, width, seed=0):
        self.E, self.B, self.hq, self.hkv, self.hd = E, B, hq, hkv, hd
        self.rng = np.random.RandomState(seed)
        self.dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        n_pages = B * width + 2
        self.cache = E.PagedCache(n_pages, page, hkv, hd, kind, block)
        if kind == "e4m3":  # what no token was stored in holds anything, NaN included
            self.cache.k.view(torch.uint8).fill_(0x7F)
            self.cache.v.view(torch.uint8).fill_(0xFF)
            self.cache.k_scale.fill_(math.nan)
            self.cache.v_scale.fill_(math.inf)
        else:
            self.cache.k.fill_(math.nan)
            self.cache.v.fill_(-math.inf)
        self.plain = Plain(n_pages, page, hkv, hd, kind, block)
        self.table = self.rng.permutation(n_pages)[:B * width].reshape(B, width).astype(np.int32)
        self.rope = rope_table(width * page, hd)
        self.len = np.zeros(B, int)

    def rows(self, n, std=1.0):
        """Fused rows of this type, as device slices and float64 values."""
        x = self.rng.randn(n, self.hq + 2 * self.hkv, self.hd) * std
        x = torch.from_numpy(x).to(self.dt)
        f = x.double().numpy()
        d = x.cuda()
        a, b = self.hq, self.hq + self.hkv
        return (d[:, :a], d[:, a:b], d[:, b:]), (f[:, :a], f[:, a:b], f[:, b:])

    def step(self, n, std=1.0, rope=True, pos0=None, check=True, tail=0):
        """Appends n[b] rows to every sequence and attends them; tail more rows lie
        behind the last sequence."""
        start = np.cumsum([0] + list(n))
        pos0 = self.len.copy() if pos0 is None else np.asarray(pos0)
        (q, k, v), (fq, fk, fv) = self.rows(int(start[-1]) + tail, std)
        tab, rs, p0 = i32(self.table), i32(start), i32(pos0)
        rp = torch.from_numpy(self.rope).cuda() if rope else None
        err = torch.zeros(self.B, dtype=torch.int32, device="cuda")
        qo = self.E.paged_append(self.cache, tab, rs, p0, k, v, q=q, rope=rp, err=err,
                                 q_out=torch.full_like(q.contiguous(), 7.0))
        self.plain.append(self.table, start, pos0, fk, fv, self.rope if rope else None)
        self.len = np.maximum(self.len, pos0 + np.asarray(n))
        out = torch.full_like(qo, 7.0)
        lse = torch.full(qo.shape[:2], 7.0, device="cuda")
        self.E.paged_attention(self.cache, tab, rs, p0, qo, out=out, lse=lse, err=err)
        torch.cuda.synchronize()
        assert err.abs().sum().item() == 0
        N = int(start[-1])
        assert bool((out[N:] == 7).all()) and bool((qo[N:] == 7).all()) and bool((lse[N:] == 7).all())
        if check:
            self.check_queries(fq[:N], qo[:N], start, pos0, rope)
            self.check_cache()
            self.check_attention(qo[:N], out[:N], lse[:N], start, pos0)
        return qo, out, lse

    def check_queries(self, fq, qo, start, pos0, rope):
        h = self.hd // 2
        ref = fq.copy()
        for b in range(self.B):
            for i in range(start[b], start[b + 1]):
                p = pos0[b] + i - start[b]
                if p < 0:
                    ref[i] = 0
                elif rope:
                    c, s = self.rope[p, :, 0], self.rope[p, :, 1]
                    x = fq[i]
                    ref[i] = np.concatenate([x[:, :h] * c - x[:, h:] * s,
                                             x[:, h:] * c + x[:, :h] * s], 1)
        # two products and a sum in float32, then the type's rounding
        tol = 2.0 ** -22 if self.dt == torch.float32 else 2.0 ** -8
        assert np.abs(qo.double().cpu().numpy() - ref).max(initial=0) <= tol * max(1.0, np.abs(ref).max(initial=0)) * 1.5

    def check_cache(self):
        k, v = values(self.cache)
        for got, ref in ((k, self.plain.k), (v, self.plain.v)):
            for pg, sl in zip(*np.nonzero(self.plain.known)):
                a, b = got[pg, :, sl], ref[pg, :, sl]
                assert np.array_equal(np.isnan(a), np.isnan(b))
                d = np.abs(np.nan_to_num(a) - np.nan_to_num(b))
                # the float32 rotation may put a value on the other side of a tie: one
                # step (2^-3 e4m3, 2^-7 bf16 of the value) in a few places
                step = 2.0 ** (-3 if self.plain.kind == "e4m3" else -7)
                assert (d <= step * np.abs(np.nan_to_num(b)) + 1e-30).all()
                assert (d > 0).mean() < 0.02

    def check_attention(self, qo, out, lse, start, pos0, scale=None):
        q = qo.double().cpu().numpy()
        p = Plain.__new__(Plain)
        p.__dict__.update(self.plain.__dict__)
        p.k, p.v = values(self.cache)  # the cache as it is: its own check is above
        ro, rl = p.attend(self.table, start, pos0, q, scale or self.hd ** -0.5)
        o = out.double().cpu().numpy()
        assert np.array_equal(np.isnan(o), np.isnan(ro))
        big = np.abs(np.nan_to_num(p.v[self.plain.known.nonzero()[0], :, self.plain.known.nonzero()[1]])).max()
        top = np.abs(rl[np.isfinite(rl)]).max(initial=0)  # as large as the largest score
        tol = ((2.0 ** -15 if self.dt == torch.float32 else 2.0 ** -7) + 2.0 ** -21 * top) * big
        assert np.abs(np.nan_to_num(o) - np.nan_to_num(ro)).max(initial=0) <= tol
        l = lse.double().cpu().numpy()
        fin = np.isfinite(rl)
        assert np.array_equal(fin, np.isfinite(l)) and (l[np.isneginf(rl)] == -np.inf).all()
        assert np.abs(l[fin] - rl[fin]).max(initial=0) <= 2.0 ** -20 + 2.0 ** -21 * top


CASES = [
    # B, hq, hkv, hd, page, block, kind, dtype, width
    (1, 4, 1, 128, 16, 16, "e4m3", "bf16", 6),
    (3, 8, 2, 128, 64, 16, "e4m3", "bf16", 3),
    (3, 8, 2, 128, 32, 32, "e4m3", "f32", 5),
    (2, 9, 1, 128, 128, 64, "e4m3", "bf16", 2),
    (2, 4, 4, 64, 16, 16, "e4m3", "f32", 9),
    (5, 6, 2, 64, 64, 32, "e4m3", "bf16", 2),
    (3, 8, 2, 128, 64, 16, "bf16", "bf16", 3),
    (2, 4, 2, 64, 16, 16, "bf16", "f32", 8),
    (2, 8, 2, 128, 32, 16, "bf16", "f32", 4),
    (1, 40, 1, 64, 64, 16, "e4m3", "f32", 2),
    (2, 33, 1, 128, 256, 256, "e4m3", "bf16", 1),
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(map(str, c)))
def test_steps(E, c):
    """Prompts of ragged lengths (one empty), single tokens, verify rows, a chunk; each
    step's queries, cache, scales and attention against the plain form."""
    print("steps", c, flush=True)
    B = c[0]
    x = Case(E, *c, seed=B)
    cap = c[8] * c[4]
    x.step([min(cap // 3, 17 + 13 * b) if b != 1 else 0 for b in range(B)])
    x.step([1] * B, std=0.3)          # smaller: the block keeps its scale
    x.step([1] * B, std=9.0, tail=3)  # larger: its scale grows
    x.step([(b * 3) % 5 for b in range(B)], std=2.0)
    x.step([min(11, cap - int(n)) for n in x.len], rope=False)


SMALL = (3, 8, 2, 128, 32, 16, "e4m3", "bf16", 4)


def forget(x, n):
    """The tokens of the sequences from n[b] on are no longer theirs."""
    for b in range(x.B):
        for p in range(int(n[b]), x.table.shape[1] * x.cache.page):
            x.plain.known[x.table[b, p // x.cache.page], p % x.cache.page] = False
        x.len[b] = min(x.len[b], n[b])


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_rollback_and_padding(E, kind):
    """Rejected rows are overwritten; rows at negative positions are padding."""
    x = Case(E, *SMALL[:6], kind, *SMALL[7:], seed=5)
    qo, out, lse = x.step([5, 40, 7], pos0=[-2, 0, -7])
    assert bool((qo[:2] == 0).all()) and bool((out[:2] == 0).all())
    assert bool((out[45:] == 0).all()) and bool(torch.isneginf(lse[45:]).all())
    for n, std in (([5, 5, 5], 1.0), ([5, 5, 5], 4.0), ([3, 1, 2], 1.0), ([1, 1, 1], 0.5)):
        x.step(n, std)
        keep = np.maximum(x.len - [2, 4, 0], 0)
        forget(x, keep)
    x.step([2, 3, 4])


@pytest.mark.parametrize("c", [
    (3, 8, 2, 128, 64, 16, "e4m3", "bf16", 7), (2, 4, 2, 128, 16, 16, "bf16", "bf16", 25),
    (2, 6, 2, 64, 32, 32, "e4m3", "f32", 14), (1, 3, 1, 128, 128, 64, "e4m3", "f32", 3),
    (2, 5, 1, 64, 16, 16, "bf16", "bf16", 25), (2, 2, 2, 128, 256, 32, "bf16", "f32", 2)],
    ids=lambda c: "-".join(map(str, c)))
def test_chunks(E, c):
    """Prompt chunks next to single tokens and an empty sequence, then a chunk that
    continues its own prompt."""
    print("chunks", c, flush=True)
    B = c[0]
    x = Case(E, *c, seed=20 + B)
    cap = c[8] * c[4]
    x.step([(151, 1, 0)[b] for b in range(B)])
    x.step([(cap - 155, 70, 3)[b] for b in range(B)], std=0.7)
    x.step([(1, 90, 129)[b] for b in range(B)], tail=2)


def test_same_rows_again_and_no_queries(E):
    x = Case(E, *SMALL, seed=6)
    x.step([9, 21, 40])
    (q, k, v), _ = x.rows(6)
    args = (x.cache, i32(x.table), i32([0, 1, 4, 6]), i32(x.len), k, v)
    assert E.paged_append(*args) is None
    was = [t.view(torch.uint8).clone() for t in (x.cache.k, x.cache.v)] + \
        [x.cache.k_scale.clone(), x.cache.v_scale.clone()]
    qc = q.contiguous()
    ref = E.paged_append(*args, q=qc, rope=None)
    assert torch.equal(ref, qc)
    now = [t.view(torch.uint8) for t in (x.cache.k, x.cache.v)] + [x.cache.k_scale, x.cache.v_scale]
    assert all(torch.equal(a.nan_to_num(-1) if a.is_floating_point() else a,
                           b.nan_to_num(-1) if b.is_floating_point() else b)
               for a, b in zip(was, now))
    rope = torch.from_numpy(x.rope).cuda()
    ref = E.paged_append(*args, q=qc, rope=rope)
    got = E.paged_append(*args, q=qc, rope=rope, q_out=qc)  # in place
    assert got is qc and torch.equal(ref, qc)


@pytest.mark.parametrize("kind,dtype,hd,block", [("e4m3", "bf16", 128, 256), ("e4m3", "f32", 64, 128),
                                                 ("bf16", "f32", 128, 16), ("e4m3", "bf16", 64, 64)])
def test_append_long_blocks_and_unaligned_rows(E, kind, dtype, hd, block):
    """Blocks of several passes, begun and ended anywhere; rows at addresses that are
    no multiple of 16 bytes."""
    x = Case(E, 2, 3, 1, hd, 256, block, kind, dtype, 2, seed=14)
    for n, off in (([37, 300], 0), ([150, 9], 1), ([1, 1], 3), ([200, 130], 5), ([3, 0], 0)):
        start, pos0 = np.cumsum([0] + n), x.len.copy()
        r = int(start[-1])
        (q, k, v), (fq, fk, fv) = x.rows(r, 1.0 + off)
        pad = lambda t, h: torch.zeros(r * (h * hd + off) + 16, dtype=t.dtype, device="cuda")[
            off:off + r * (h * hd + off)].view(r, h * hd + off)[:, :h * hd].view(r, h, hd)
        k2, v2, q2 = pad(k, 1).copy_(k), pad(v, 1).copy_(v), pad(q, 3).copy_(q)
        qo = E.paged_append(x.cache, i32(x.table), i32(start), i32(pos0), k2, v2, q=q2,
                            rope=torch.from_numpy(x.rope).cuda(), q_out=pad(q, 3))
        x.plain.append(x.table, start, pos0, fk, fv, x.rope)
        x.len += n
        x.check_queries(fq, qo, start, pos0, True)
        x.check_cache()


@pytest.mark.parametrize("std", [1e-40, 1e-33, 1e30])
def test_magnitudes(E, std):
    """Scales down to 2^-100 and values near the float32 limits."""
    x = Case(E, 2, 2, 1, 64, 16, 16, "e4m3", "f32", 3, seed=7)
    start, pos0 = [0, 20, 25], [0, 3]
    (q, k, v), (_, fk, fv) = x.rows(25, std)
    E.paged_append(x.cache, i32(x.table), i32(start), i32(pos0), k, v)
    x.plain.append(x.table, start, pos0, fk, fv, None)
    gk, gv = values(x.cache)
    for got, ref in ((gk, x.plain.k), (gv, x.plain.v)):
        for pg, sl in zip(*np.nonzero(x.plain.known)):
            assert np.array_equal(got[pg, :, sl], ref[pg, :, sl])


def test_bad_pages_are_left_out(E):
    x = Case(E, *SMALL, seed=8)
    x.step([60, 33, 50])
    was = [t.view(torch.uint8).clone() for t in (x.cache.k, x.cache.v)]
    tab = x.table.copy()
    tab[0, 1] = -1          # holds positions 32..59 of sequence 0
    tab[2, 0] = 14          # n_pages is 14
    tab[2, 1] = 2 ** 31 - 1
    start, pos0 = [0, 2, 4, 5], [60, 33, 50]
    (q, k, v), (fq, fk, fv) = x.rows(5)
    err = torch.zeros(3, dtype=torch.int32, device="cuda")
    E.paged_append(x.cache, i32(tab), i32(start), i32(pos0), k, v, err=err)
    assert err.tolist() == [1, 0, 1]
    err.zero_()
    qo, lse = q.contiguous(), torch.zeros(5, 8, device="cuda")
    out = E.paged_attention(x.cache, i32(tab), i32(start), i32(pos0), qo, lse=lse, err=err)
    assert err.tolist() == [1, 0, 1]
    for a, t in zip(was, (x.cache.k, x.cache.v)):  # only sequence 1's page was written
        t = t.view(torch.uint8)
        other = [p for p in range(14) if p != tab[1, 1]]
        assert torch.equal(a[other], t[other])
    p = Plain.__new__(Plain)
    p.__dict__.update(x.plain.__dict__)
    p.k, p.v = values(x.cache)
    t2 = tab.copy()
    t2[2, 1] = -1
    x.plain.append(x.table, [0, 0, 2, 2], pos0, fk[2:4], fv[2:4], None)
    ro, rl = p.attend(t2, start, pos0, fq, 128 ** -0.5)
    assert np.abs(out.double().cpu().numpy() - ro).max() <= 2.0 ** -6 * 4
    assert bool((out[4] == 0).all()) and bool(torch.isneginf(lse[4]).all())


def test_bounds_that_do_not_hold(E):
    """More rows than max_rows, positions past max_len, past the table, past the
    rotation table: left out and reported, nothing else touched."""
    x = Case(E, *SMALL, seed=9)
    x.step([60, 33, 50])
    (q, k, v), (fq, _, _) = x.rows(12)
    tab, start, pos0 = i32(x.table), [0, 2, 8, 12], [60, 33, 50]
    q = q.contiguous()

    def attend(**kw):
        err = torch.zeros(3, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 7.0)
        E.paged_attention(x.cache, tab, i32(start), i32(kw.pop("pos0", pos0)), q, out=out, err=err, **kw)
        return out, err.tolist()

    full, err = attend(pos0=[58, 20, 40])
    assert err == [0, 0, 0]
    out, err = attend(pos0=[58, 20, 40], max_rows=4)
    assert err == [0, 1, 0] and bool((out[6:8] == 7).all())
    ok = [0, 1, 2, 3, 4, 5, 8, 9, 10, 11]
    assert (out[ok] - full[ok]).abs().max() <= 2.0 ** -6
    out, err = attend(pos0=[58, 20, 40], max_len=43)
    assert err == [1, 0, 1]
    assert (out[2:8] - full[2:8]).abs().max() <= 2.0 ** -6
    assert (out[8:11] - full[8:11]).abs().max() <= 2.0 ** -6  # positions 40..42
    out, err = attend(pos0=[2 ** 31 - 1, 20, -2 ** 31])
    assert err == [1, 0, 0] and bool((out[8:] == 0).all())
    err = torch.zeros(3, dtype=torch.int32, device="cuda")
    was = [t.view(torch.uint8).clone() for t in (x.cache.k, x.cache.v)]
    rope = torch.from_numpy(x.rope).cuda()
    qo = E.paged_append(x.cache, tab, i32(start), i32([2 ** 31 - 1, -2 ** 31, 128]), k, v, q=q,
                        rope=rope, err=err)
    assert err.tolist() == [1, 0, 1] and bool((qo == 0).all())
    assert all(torch.equal(a, t.view(torch.uint8)) for a, t in zip(was, (x.cache.k, x.cache.v)))
    # garbage row boundaries stay inside the tensors
    E.paged_attention(x.cache, tab, i32([-5, 400, 3, 2 ** 31 - 1]), i32(pos0), q)
    E.paged_append(x.cache, tab, i32([2 ** 31 - 1, -2 ** 31, 1000, 5]), i32(pos0), k, v, q=q)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind,dtype,hd", [("e4m3", "bf16", 128), ("bf16", "bf16", 128),
                                           ("bf16", "f32", 64), ("e4m3", "f32", 64)])
@pytest.mark.parametrize("many", [False, True])
def test_infinities_and_nan(E, kind, dtype, hd, many):
    """What is not finite reaches the rows that attend it and no others."""
    x = Case(E, 2, 4, 2, hd, 32, 16, kind, dtype, 8, seed=10)
    x.step([70, 20])
    n = [90, 6] if many else [5, 6]
    start, pos0 = np.cumsum([0] + n), x.len.copy()
    (q, k, v), (fq, fk, fv) = x.rows(sum(n))
    a, b = (k.clone(), v.clone())
    a[3, 1, 5] = math.inf
    b[2, 0, 7] = math.nan
    b[4, 1, 9] = math.inf
    b[n[0] + 1, 0, 0] = -math.inf
    b[n[0] + 3, 0, 0] = math.inf
    a[n[0] + 5, 1, 0] = math.nan
    E.paged_append(x.cache, i32(x.table), i32(start), i32(pos0), a, b)
    for i in range(2):
        for p in range(pos0[i], pos0[i] + n[i]):
            x.plain.known[x.table[i, p // 32], p % 32] = True
    lse = torch.zeros(sum(n), 4, device="cuda")
    out = E.paged_attention(x.cache, i32(x.table), i32(start), i32(pos0), q, lse=lse,
                            **(dict() if many else dict(max_rows=6)))
    assert bool(torch.isfinite(out[:2]).all()) and not bool(torch.isfinite(out[2]).all())
    p = Plain.__new__(Plain)
    p.__dict__.update(x.plain.__dict__)
    p.k, p.v = values(x.cache)
    with np.errstate(invalid="ignore"):
        ro, rl = p.attend(x.table, start, pos0, fq, hd ** -0.5)
    o = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(o), np.isnan(ro))
    inf = np.isinf(ro)
    assert np.array_equal(o[inf], ro[inf])
    fin = np.isfinite(ro)
    assert np.abs(o[fin] - ro[fin]).max() <= 2.0 ** -6 * 4
    l = lse.double().cpu().numpy()
    assert np.array_equal(np.isfinite(l), np.isfinite(rl))


def test_replays_of_a_captured_step(E):
    """Append and attention captured once and replayed with other rows, positions and
    tables, the eager twin's work in between: the same bits each time."""
    x, y = Case(E, *SMALL, seed=11), Case(E, *SMALL, seed=11)
    x.step([60, 33, 50]), y.step([60, 33, 50])
    (q, k, v), _ = x.rows(9)
    rope = torch.from_numpy(x.rope).cuda()
    tab, rs, p0 = i32(x.table), i32([0, 2, 5, 9]), i32(x.len)
    qo, out = torch.empty_like(q.contiguous()), torch.empty_like(q.contiguous())
    ws = E.paged_attention_workspace(x.cache, 3, 9, 8, 5, 128)

    def step(c, tab, rs, p0, q, k, v, qo, out, ws):
        E.paged_append(c.cache, tab, rs, p0, k, v, q=q, rope=rope, q_out=qo, max_rows=5)
        E.paged_attention(c.cache, tab, rs, p0, qo, out=out, workspace=ws, max_rows=5, max_len=128)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):  # also: another stream than the tensors' own
        step(x, tab, rs, p0, q, k, v, qo, out, ws)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(x, tab, rs, p0, q, k, v, qo, out, ws)
    step(y, tab, rs, p0, q, k, v, torch.empty_like(qo), torch.empty_like(qo),
         torch.empty_like(ws))
    at, n = x.len.copy(), [[0, 2, 5, 9], [0, 5, 6, 9], [0, 0, 4, 8], [0, 3, 6, 9]]
    for i in range(4):
        (q2, k2, v2), _ = x.rows(9, 1.0 + i)
        q.copy_(q2), k.copy_(k2), v.copy_(v2)
        rs.copy_(i32(n[i])), p0.copy_(i32(at))
        out.fill_(7.0)
        g.replay()
        q3, o3 = torch.empty_like(qo), torch.full_like(out, 7.0)
        step(y, tab, rs, p0, q2, k2, v2, q3, o3, torch.empty_like(ws))
        torch.cuda.synchronize()
        m = n[i][-1]
        assert torch.equal(qo[:m], q3[:m]) and torch.equal(out, o3)
        for b in range(3):
            for p in range(int(at[b]), int(at[b]) + n[i][b + 1] - n[i][b]):
                x.plain.known[x.table[b, p // 32], p % 32] = True
        kx, vx = values(x.cache)
        ky, vy = values(y.cache)
        for pg, sl in zip(*np.nonzero(x.plain.known)):
            assert np.array_equal(kx[pg, :, sl], ky[pg, :, sl])
            assert np.array_equal(vx[pg, :, sl], vy[pg, :, sl])
        at = at + np.diff(n[i])


def test_cache_past_32_bit_offsets(E):
    """Pages beyond 4 GiB of codes: 8 heads of 128, pages of 1024."""
    n = 4200  # pages of 1 MiB of keys
    c = E.PagedCache(n, 1024, 8, 128, "e4m3", 64)
    rng = np.random.RandomState(12)
    table = np.array([[4199, 3], [2100, 4150]], np.int32)
    x = Case.__new__(Case)
    x.rng, x.hq, x.hkv, x.hd, x.dt = rng, 8, 8, 128, torch.bfloat16
    (q, k, v), (fq, fk, fv) = x.rows(1100 + 30)
    start, pos0 = [0, 1100, 1130], [0, 1010]
    E.paged_append(c, i32(table), i32(start), i32(pos0), k, v)
    out = E.paged_attention(c, i32(table), i32([0, 1, 2]), i32([1099, 1039]), q[[1099, 1129]].contiguous())
    for b in range(2):
        lo, m = (0, 1100) if b == 0 else (1010, 1040)
        kk, vv = np.zeros((m, 8, 128)), np.zeros((m, 8, 128))
        kk[lo:], vv[lo:] = fk[start[b]:start[b + 1]], fv[start[b]:start[b + 1]]
        for h in range(8):
            s = kk[:, h] @ fq[[1099, 1129][b], h] * 128 ** -0.5
            w = np.exp(s - s.max())
            ref = w @ vv[:, h] / w.sum()
            # half a step of the codes moves scores (of std 1) and values by 2^-4
            assert np.linalg.norm(out[b, h].double().cpu().numpy() - ref) <= 0.1 * np.linalg.norm(ref) + 0.02


def test_table_rows_of_a_wider_table_and_strided_rows(E):
    x = Case(E, *SMALL, seed=13)
    x.step([60, 33, 50])
    wide = torch.full((3, 9), -1, dtype=torch.int32, device="cuda")
    wide[:, 2:6] = i32(x.table)
    (q, k, v), _ = x.rows(4)
    pad = torch.zeros(4, 8 * 128 + 64, dtype=torch.bfloat16, device="cuda")
    out = pad[:, 32:32 + 1024].view(4, 8, 128)
    rs, p0 = i32([0, 1, 2, 4]), i32(x.len)
    E.paged_append(x.cache, wide[:, 2:6], rs, p0, k, v)
    E.paged_attention(x.cache, wide[:, 2:6], rs, p0, q, out=out)
    ref = E.paged_attention(x.cache, i32(x.table), rs, p0, q.contiguous())
    assert torch.equal(out, ref) and bool((pad[:, :32] == 0).all()) and bool((pad[:, 1056:] == 0).all())
    for bad in (lambda: E.paged_attention(x.cache, wide[:, 2:6].t(), rs, p0, q),
                lambda: E.paged_attention(x.cache, i32(x.table), rs.long(), p0, q),
                lambda: E.paged_attention(x.cache, i32(x.table), rs, p0, q.transpose(1, 2)),
                lambda: E.paged_append(x.cache, i32(x.table), rs, p0, k, v.float()),
                lambda: E.paged_append(x.cache, i32(x.table), rs, p0.cpu(), k, v)):
        with pytest.raises(ValueError):
            bad()


def test_one_workspace_for_smaller_calls(E):
    """A workspace for many sequences takes one long one, split more finely, and rows
    behind the last sequence, which have places in it; the same results as with its own."""
    x = Case(E, 3, 32, 2, 128, 64, 16, "e4m3", "bf16", 40, seed=14)
    x.step([2400, 70, 30], check=False)
    (q, _, _), _ = x.rows(64)
    ws = E.paged_attention_workspace(x.cache, 64, 64, 32, 64, 2560)
    for rows, rs, at in ((64, [0, 40], [2360]), (64, [0, 1], [2399]), (3, [0, 3], [2397]),
                         (64, [0, 1, 33], [2399, 38]), (1, [0, 1], [2399])):
        n = len(at)
        for m in (None, max(np.diff(rs))):
            a = [i32(x.table[:n]), i32(rs), i32(at), q[:rows].contiguous()]
            out = torch.full_like(a[3], 7.0)
            lse = torch.zeros(rows, 32, device="cuda")
            E.paged_attention(x.cache, *a, out=out, lse=lse, max_rows=m, workspace=ws)
            own = E.paged_attention(x.cache, *a, max_rows=m, out=torch.full_like(out, 7.0))
            assert torch.equal(out, own) and bool((out[rs[-1]:] == 7).all())
            x.check_attention(a[3][:rs[-1]], out[:rs[-1]], lse[:rs[-1]], rs, at)
