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
