"""The refinement step with the 8-bit latent cache, step by step: what each block's slice holds after a step, the rows
and blocks that a step leaves alone, and latents that show the cache's rounding."""
import numpy as np
import pytest

import oracle as O
import workloads as W

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding

from test_gpu_kv8 import MODELS  # noqa: E402

pytestmark = pytest.mark.gpu


def workload(model):
    shapes = [W.Request(4, 16, 16)] if model == "bf16_72" else [W.Request(3, 24, 20), W.Request(2, 10, 14),
                                                                 W.Request(1, 4, 4)]
    n = len(shapes)
    return W.custom("kv8_steps_" + model, MODELS[model], shapes, [0.4, 0.7, 0.5][:n],
                    [("uniform", 0.3, 0.7), 0.5, 0.2][:n], [5, 4, 3][:n])


def slices(R, bounds):
    cfg = R.cfg
    return R.kv_cache.view(cfg.L, B.sphinx_kv8_bytes(cfg.heads, cfg.head_dim, bounds))


def held(R, bounds):
    """Keys and values of every block [L][2][N][heads][head_dim], as numbers."""
    cfg, n = R.cfg, int(bounds[-1])
    out = torch.empty(cfg.L, 2, n, cfg.heads, cfg.head_dim, device="cuda")
    for l, s in enumerate(slices(R, bounds)):
        B.sphinx_kv8_load(B.F32, cfg.heads, cfg.head_dim, s, bounds, None, n, out[l, 0], out[l, 1], cfg.D)
    return out.double().cpu().numpy()


def load(R, bounds, state_nchw, cache):
    """The oracle's state and cache into the Refiner; the cache's numbers are exact in 8 bits."""
    cfg, n = R.cfg, int(bounds[-1])
    P = O.patchify(state_nchw, R.shapes).astype(np.float32)
    R.z.copy_(torch.from_numpy(np.ascontiguousarray(P.ravel())).cuda())
    R.kv_cache.zero_()
    for s, kv in zip(slices(R, bounds), cache):
        k, v = (torch.from_numpy(x.astype(np.float32)).cuda() for x in kv)
        B.sphinx_kv8_store(B.F32, cfg.heads, cfg.head_dim, k, v, cfg.D, None, n, bounds, s)


@pytest.mark.parametrize("model", list(MODELS))
def test_slices_after_each_step(model):
    """Before each step the GPU gets the oracle's state and cache.  A key or value may then differ from the oracle's by
    what the model's type allows (1e-4 and 3e-2, as for the unrounded cache) and by one 8-bit step, which is at most 2^-3
    of it; nearly all are the same (a bf16 number that is off by two of its steps, 2^-6, crosses the middle of two 8-bit
    numbers one time in eight at most).  Blocks that no forwarded row falls into keep every byte."""
    wl = workload(model)
    cfg = wl.model
    M = O.model_from_workload(wl)
    bounds = np.asarray(wl.tok_offset, np.int32)
    plans = O.plan_steps([r.frames for r in wl.requests], wl.s_start, wl.nsteps, 2)
    info = O.token_info(wl.requests)
    R = S.from_workload(wl, cache_period=2, cache_dtype="fp8")
    R.reset()
    state, cache = np.asarray(wl.z0, np.float64), O.sphinx_oracle.Kv8Cache(O.new_cache(M, wl.N), wl.tok_offset)
    off, same, tol = (1e-4, 0.999, 1e-4) if cfg.dtype == "f32" else (3e-2, 0.875, 2e-2)
    left = 0
    for i, p in enumerate(plans):
        load(R, bounds, state, cache)
        before = held(R, bounds)
        n = R.step(i, force_select=True)
        res = O.step_cached(wl, M, state, p, cache, "model", info)
        assert n == res.n_sel and R.n_fwd == res.qidx.size
        got = held(R, bounds)
        want = np.stack([np.stack(kv) for kv in cache]).reshape(got.shape)
        touched = np.zeros(wl.N, bool)
        for a, b in O.kv8.blocks(bounds):
            touched[a:b] = np.isin(np.arange(a, b), res.qidx).any()
        assert np.array_equal(got[:, :, ~touched], before[:, :, ~touched])
        left += int((~touched).sum())
        d = np.abs(got - want) - off - 2.0 ** -3 * np.maximum(np.abs(got), np.abs(want))
        rows = res.qidx
        eq = float((got[:, :, rows] == want[:, :, rows]).mean()) if rows.size else 1.0
        err = np.abs(R.state.cpu().numpy().astype(np.float64) - res.state).max()
        print(f"[kv8 step {model} {i}] forwarded {rows.size} of {wl.N}, over bound {d.max():.3e}, equal {eq:.5f}, "
              f"latents {err:.3e}", flush=True)
        assert d.max() <= 0.0 and eq >= same and err <= tol
        state = res.state
    assert left > 0  # some steps did leave blocks alone


@pytest.mark.parametrize("model", list(MODELS))
def test_latents_show_the_rounding_of_the_cache(model):
    """The loop's latents are nearer to the oracle with an 8-bit cache than to the one without: for an fp32 model,
    whose own roundings are far below the cache's, at most a tenth as far."""
    wl = workload(model)
    got = S.from_workload(wl, cache_period=3, cache_dtype="fp8").run().cpu().numpy().astype(np.float64)
    ref = O.refine(wl, precision="model", period=3, cache8=True)
    plain = O.refine(wl, precision="model", period=3)
    a, b = (float(np.sqrt(((got - x) ** 2).mean())) for x in (ref, plain))
    print(f"[kv8 loop {model}] rms to the 8-bit oracle {a:.3e}, to the unrounded one {b:.3e}", flush=True)
    assert a < b * (0.1 if wl.model.dtype == "f32" else 1.0)
