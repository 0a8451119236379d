"""Contexts on paged caches against the oracle: each attention sublayer on the cache
as it is held (bf16, or 8 bits with block scales), the cache against the oracle's
keys and values, and generation."""
import numpy as np
import pytest

import workloads as W
from oracle import model as M
from tests.gpu_helpers import check_rows, rel_err

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TOL = {"tiny": 1e-4, "small_bf16": 2e-2, "small_qwen_bf16": 2e-2}
LAT = {"tiny": (W.TINY_LATENCY, "bins", 64), "small_bf16": ((1.0, 0.004, 0.3), "bins", 32),
       "small_qwen_bf16": ((1.0, 0.004, 0.3), "bins", 32)}


class Held(np.ndarray):
    """Keys or values that a write leaves as they are: the device's."""

    def __setitem__(self, at, x):
        pass


def held_cache(cfg, dm, n_max=320):
    c = M.KVCache(cfg, n_max)
    for l, pg in enumerate(dm.pages):
        k, v = pg.k.float().cpu().double().numpy(), pg.v.float().cpu().double().numpy()
        v = v.transpose(0, 1, 2, 4, 3).reshape(k.shape)
        if pg.k_scale is not None:
            k = k * np.repeat(pg.k_scale.cpu().double().numpy(), pg.block, 2)[..., None]
            v = v * np.repeat(pg.v_scale.cpu().double().numpy(), pg.block, 2)[..., None]
        tab = dm.page_table.cpu().numpy()
        for x, dst in ((k, c.K), (v, c.V)):
            x = x[tab].transpose(1, 0, 2, 3).reshape(cfg.hkv, -1, cfg.hd)[:, :n_max]
            dst[l] = np.ascontiguousarray(x).view(Held)
    return c


@pytest.fixture(scope="module", params=[(n, k) for n in TOL for k in ("bf16", "e4m3")],
                ids=lambda p: "-".join(p))
def setup(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2602_20217_amd.engine import DeviceModel
    name, kind = request.param
    print(f"\n[setup] building {name} on {kind} pages", flush=True)
    cfg = W.config(name)
    weights = W.generate_weights(cfg, seed=0)
    dm = DeviceModel(cfg, n_max=320, gamma_max=4, m_rounds=5, cap_max=128, prefill_chunk=64,
                     cache=kind).upload_all(weights)
    yield name, kind, cfg, dm, M.Model(cfg, weights)
    dm.close()


def test_prefill_cache(setup):
    """The first layer's keys and values (deeper ones follow the held cache's rounding):
    the model's tolerance, and half a step of the held type."""
    name, kind, cfg, dm, model = setup
    n = 100
    prompt = W.prompt_ids(cfg.vocab, n, 1)
    dm.prefill(prompt)
    st = M.prefill(model, prompt, 320, 25)
    c = held_cache(cfg, dm)
    for h in range(cfg.hkv):
        for got, ref in ((c.K[0][h, :n], st.cache.K[0][h, :n]), (c.V[0][h, :n], st.cache.V[0][h, :n])):
            assert rel_err(got, ref) < TOL[name] + 2.0 ** (-4 if kind == "e4m3" else -8)


@pytest.mark.parametrize("R,mode", [(1, 0), (5, 0), (16, 0), (40, 0), (3, 1), (50, 1)])
def test_sublayers(setup, R, mode):
    name, kind, cfg, dm, model = setup
    n = 90
    dm.prefill(W.prompt_ids(cfg.vocab, n, 5))
    x = W.synthetic_rows(R, cfg.d, seed=4, std=0.5, index=R)
    pos = (np.arange(R) + n) if mode == 0 else np.sort(
        np.random.default_rng(R).integers(0, n, size=R))
    xd = torch.from_numpy(x).cuda()
    for l in range(cfg.L):
        out = torch.empty_like(xd)
        dm.sublayer_apply(2 * l + 1, xd, pos, mode=mode, out=out)
        ref = M.sublayer(model, 2 * l + 1, x.astype(np.float64), pos, held_cache(cfg, dm),
                         mode="write" if mode == 0 else "own")
        check_rows(out.cpu().numpy(), x, ref, TOL[name], (name, kind, R, mode, l))


def test_generate(setup):
    """Speculative generation through prefill, selection, drafts and verify.  On bf16
    pages it gives the autoregressive run's tokens; on 8-bit ones it may part from them
    where a rejected draft raised a scale, so only its first token has to agree."""
    name, kind, cfg, dm, model = setup
    from paper_2602_20217_amd.engine import select_params
    c, mode, bins = LAT[name]
    prompt = W.prompt_ids(cfg.vocab, 128, 1)
    ar, _, _ = dm.generate(prompt, 32, gamma=0)
    ssd, st, sels = dm.generate(prompt, 32, gamma=4, reselect_every=8,
                                params=select_params(c, mode, bins))
    assert st.n_selections == len(sels) >= 2 and st.n_rounds >= 1
    if kind == "bf16":
        np.testing.assert_array_equal(ssd, ar)
    assert ssd[0] == ar[0] and ((0 <= ssd) & (ssd < cfg.vocab)).all()
    prof = dm.profile_decode(steps=1)
    assert prof["launches"]["qkv_post"] == cfg.L


def test_shuffled_pages_and_back(setup):
    """The pages' order and size do not change a prefill's token or the cache; the flat
    cache is refused where the context was made without one."""
    name, kind, cfg, dm, model = setup
    from paper_2602_20217_amd import _lib as K
    from paper_2602_20217_amd.engine import PagedCache
    old, tab = dm.pages, dm.page_table
    prompt = W.prompt_ids(cfg.vocab, 128, 1)
    first = dm.prefill(prompt)
    ref = held_cache(cfg, dm)
    perm = torch.from_numpy(np.random.RandomState(0).permutation(23)[:21].astype(np.int32)).cuda()
    dm.use_paged([PagedCache(23, 16, cfg.hkv, cfg.hd, kind, 16, device=dm.dev)
                  for _ in range(cfg.L)], perm)
    with pytest.raises(K.KsError) as e:  # the decode state is cleared
        dm.draft_step(np.ones(2 * cfg.L, bool))
    assert e.value.status == K.KS_ESTATE
    assert dm.prefill(prompt) == first
    got = held_cache(cfg, dm)
    for l in range(cfg.L):
        assert np.array_equal(got.K[l][:, :128], ref.K[l][:, :128])
        assert np.array_equal(got.V[l][:, :128], ref.V[l][:, :128])
    dm.use_paged(None, None)
    for call in (lambda: dm.prefill(prompt), lambda: dm.set_context(3, 0)):
        with pytest.raises(K.KsError) as e:
            call()
        assert e.value.status == K.KS_ESTATE
    for bad in (perm[:10], perm + 30, perm - 3):
        with pytest.raises(K.KsError):
            dm.use_paged([PagedCache(23, 16, cfg.hkv, cfg.hd, kind, 16, device=dm.dev)
                          for _ in range(cfg.L)], bad.contiguous())
    dm.use_paged(old, tab)
    assert dm.prefill(prompt) == first
    with pytest.raises(K.KsError) as e:
        x = torch.zeros(2, cfg.d, device=dm.dev)
        dm.sublayer_apply(1, x, [5, 9], mode=0)
    assert e.value.status == K.KS_EINVAL
