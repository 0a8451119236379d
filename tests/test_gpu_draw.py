"""ks_sample_draw against a plain float64 implementation on the host: tokens and the
number of entries kept are equal, the log-probability to its float32 rounding.

The places searched for are decided in units of 2^-44 of the largest entry's mass, so
a uniform nearer than that to a border could fall either way; with random uniforms of
24 bits and at most 2^18 entries that has a chance below 2^18 2^-44 a row."""
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


def plain(row, T, k, p, m, u):
    """(token, log-probability, entries kept) of one row (float64 values)."""
    ids = np.argsort(-row, kind="stable")
    ids = ids[~np.isnan(row[ids])]
    ids = ids[row[ids] > -np.inf]
    if not len(ids):
        return -1, -math.inf, 0
    if not T > 0:
        return int(ids[0]), 0.0, 1
    l = row[ids]
    with np.errstate(invalid="ignore"):
        x = np.where(l == l[0], 0.0, (l - l[0]) / T)
    n = len(x) if k <= 0 else min(k, len(x))
    w = np.exp(x[:n])
    if m > 0:
        w = w[w >= min(m, 1.0)]
    if p < 1:
        c = np.cumsum(w)
        w = w[:int(np.argmax(c >= max(p, 0.0) * c[-1])) + 1]
    c = np.cumsum(w)
    u = u if u > 0 else 0.0
    j = int(np.sum(c <= u * c[-1]))
    if j >= len(w):
        j = int(np.max(np.nonzero(w)[0]))
    return int(ids[j]), float(x[j] - math.log(c[-1])), len(w)


def run(E, logits, T, k, p, m, u, **kw):
    R = logits.shape[0]
    f = lambda a: None if a is None else torch.tensor(np.broadcast_to(np.float32(a), R).copy(), device="cuda")
    i = lambda a: None if a is None else torch.tensor(np.broadcast_to(np.int32(a), R).copy(), device="cuda")
    lp = torch.full((R,), 9.0, device="cuda")
    kept = torch.full((R,), -9, dtype=torch.int32, device="cuda")
    tok = E.sample_draw(logits, f(u), f(T), i(k), f(p), f(m), logprob=lp, kept=kept, **kw)
    torch.cuda.synchronize()
    return tok.cpu().numpy(), lp.cpu().numpy(), kept.cpu().numpy()


def check(E, logits, T, k, p, m, u):
    R = logits.shape[0]
    tok, lp, kept = run(E, logits, T, k, p, m, u)
    host = logits.double().cpu().numpy()
    b = lambda a, d, dt: np.broadcast_to(dt(d if a is None else a), R)
    T, p, m, u = (b(a, d, np.float32) for a, d in ((T, 1), (p, 1), (m, 0), (u, 0)))
    k = b(k, 0, np.int64)
    for r in range(R):
        want = plain(host[r], float(T[r]), int(k[r]), float(p[r]), float(m[r]), float(u[r]))
        assert (tok[r], kept[r]) == (want[0], want[2]), (r, T[r], k[r], p[r], m[r], u[r], want)
        # the sum's units and the float32 rounding
        assert lp[r] == want[1] or abs(lp[r] - want[1]) <= 2.0 ** -23 * abs(want[1]) + 2.0 ** -26


@pytest.mark.parametrize("V", [1, 2, 63, 64, 1000, 1025, 4097, 50257, 128256, 262144])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_settings(E, V, dt):
    print("settings", V, dt, flush=True)
    g = torch.Generator(device="cuda").manual_seed(V)
    R = 24
    lg = (torch.randn(R, V, generator=g, device="cuda") * 3).to(dt)
    lg[torch.rand(R, V, generator=g, device="cuda") < 0.05] = -math.inf
    r = np.random.RandomState(V)
    check(E, lg, r.choice([0, 0.3, 0.7, 1.0, 2.0], R), r.choice([0, 1, 5, 50, 700, 10 ** 9], R),
          r.choice([0.0, 0.1, 0.5, 0.95, 1.0, 1.0], R), r.choice([0, 0, 0.01, 0.3, 1.0], R),
          r.uniform(0, 1, R).astype(np.float32))


def test_defaults_and_uniform_edges(E):
    lg = torch.randn(6, 5000, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    top = 1 - 2.0 ** -24
    check(E, lg, None, None, None, None, [0.0, -1.0, top, 0.5, 2.0 ** -30, math.nan])
    check(E, lg, 0.8, 40, 0.9, 0.02, [0.0, top, 0.25, 0.75, 1.0, 3.0])


@pytest.mark.parametrize("V", [1, 700, 20000, 151936])
def test_dense_bins(E, V):
    """Equal logits and high temperatures: more entries in a bin than are gathered."""
    print("dense", V, flush=True)
    g = torch.Generator(device="cuda").manual_seed(V)
    R = 9
    r = np.random.RandomState(V)
    u = r.uniform(0, 1, R).astype(np.float32)
    k, p = r.choice([0, 7, 300, 10000], R), r.choice([1.0, 0.9, 0.3], R)
    check(E, torch.zeros(R, V, device="cuda"), 1.0, k, p, 0, u)
    check(E, torch.full((R, V), torch.finfo(torch.float32).min, device="cuda"), 0.7, k, p, 0.5, u)
    check(E, torch.randn(R, V, generator=g, device="cuda"), 500.0, k, p, None, u)
    few = torch.randint(0, 3, (R, V), generator=g, device="cuda").float()  # three values
    check(E, few, [0.5, 1, 3] * 3, k, p, [0, 0.2, 0.9] * 3, u)


def test_barred_rows_and_infinities(E):
    V = 3001
    lg = torch.randn(8, V, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    lg[0] = -math.inf
    lg[1] = math.nan
    lg[2, :] = -math.inf
    lg[2, 1234] = -7.0
    lg[3, 5] = math.inf
    lg[4, 5] = lg[4, 77] = math.inf
    lg[5, ::2] = math.nan
    lg[6, 10:] = torch.finfo(torch.float32).min
    for T in (0.0, 0.9, 1e-30):
        check(E, lg, T, None, None, None, [0.1, 0.2, 0.3, 0.4, 0.7, 0.6, 0.9, 0.99])
    check(E, lg, 1.0, 3, 0.8, 0.1, [0.1, 0.2, 0.3, 0.4, 0.7, 0.6, 0.9, 0.99])


def test_row_strides_and_alignment(E):
    g = torch.Generator(device="cuda").manual_seed(3)
    for dt, off, ld in ((torch.float32, 1, 1031), (torch.bfloat16, 3, 1027), (torch.bfloat16, 8, 1032)):
        buf = torch.randn(5 * ld + 16, generator=g, device="cuda").to(dt)
        lg = buf[off:off + 5 * ld].view(5, ld)[:, :1013]
        check(E, lg, 0.9, 100, 0.9, None, [0.05, 0.3, 0.5, 0.7, 0.95])


def test_many_rows(E):
    g = torch.Generator(device="cuda").manual_seed(4)
    R = 1500
    lg = torch.randn(R, 300, generator=g, device="cuda") * 2
    r = np.random.RandomState(4)
    check(E, lg, r.uniform(0.2, 2, R), r.randint(0, 200, R), r.uniform(0.2, 1, R),
          r.uniform(0, 0.2, R), r.uniform(0, 1, R).astype(np.float32))


def test_same_as_the_tabulated_filter(E):
    """With the settings that ks_sample_filter takes and its uniforms, the same tokens
    (float32 there: rows whose uniform is not next to a border)."""
    g = torch.Generator(device="cuda").manual_seed(5)
    R, V = 16, 32000
    lg = torch.randn(R, V, generator=g, device="cuda") * 3
    ids, probs, cnt, _, tok = E.sample_filter(lg, 0.7, 50, 0.95, seed=9, pos0=100)
    u = E.sample_uniforms(9, torch.arange(100, 100 + R, dtype=torch.int32, device="cuda"), 2)
    t2, _, kept = run(E, lg, 0.7, 50, 0.95, None, u.cpu().numpy())
    tok, c = tok.cpu().numpy(), cnt.cpu().numpy()
    cum = np.cumsum(probs.double().cpu().numpy(), 1)
    for r in range(R):
        near = np.abs(cum[r, :c[r]] - float(u[r])).min()
        assert near < 1e-5 or tok[r] == t2[r]
