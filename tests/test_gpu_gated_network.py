"""Networks with gated blocks in the sampler: the model call against the oracle, and whole samples.

The device and the oracle round at the same places; they differ where fp32 accuracy moves a number across a border of its
rounding: by 2^-8 of a bf16 number, by a step, 1/127 of the row's largest, of an 8-bit one.  With one number in a hundred moved
-- fp32 errors of 1e-6 against borders 2^-8 or 2^-7 apart make it one in some thousands -- a block's result moves by
sqrt(0.01) / 127 of its size, 8e-4, and three blocks and the output layer, which add up, by 2.4e-3."""
import numpy as np
import pytest
import torch

import asd_workloads as W
import gpu_helpers as H
from oracle import denoisers, schedule
from oracle_helpers import chain_randoms
from oracle import asd as oasd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def setup(cfg):
    from paper_2505_03983_amd import runtime
    T = schedule.ddpm_tables(cfg["K"], W.BETA_MIN, W.BETA_MAX)
    p = W.make_params(cfg)
    net = denoisers.GatedOracle(p, abar=T["abar"])

    def model(idx, rows):
        return net(rows, T["tau"][np.asarray(idx)])
    return T, p, model, runtime


CASES = [dict(d=16, E=8, width=64, hidden=96, n_blocks=2), dict(d=112, E=128, width=256, hidden=688, n_blocks=3),
         dict(d=48, E=16, width=1040, hidden=400, n_blocks=1), dict(d=64, E=64, width=512, hidden=1024, n_blocks=0)]


@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("shape", CASES)
def test_model_call(shape, eight_bit):
    for rows, act, terms in ((1, 0, 2), (50, 1, 2), (700, 0, 1)):
        cfg = dict(shape, kind="gated", K=100, chains=50, L=16, eight_bit=eight_bit, act=act, act_terms=terms)
        T, p, model, runtime = setup(cfg)
        p["out_clip"] = 0.0
        net = denoisers.GatedOracle(p)
        ctx = runtime.open_ctx(cfg, p)
        rng = np.random.default_rng(rows)
        x = rng.standard_normal((rows, cfg["d"])).astype(np.float32)
        tau = rng.integers(1, 101, rows).astype(np.int32)
        out = torch.zeros(rows, cfg["d"], device=DEV)
        ctx.denoise(torch.from_numpy(x).to(DEV), torch.from_numpy(tau).to(DEV), out)
        torch.cuda.synchronize()
        want = net(x.astype(np.float64), tau)
        got = out.cpu().numpy()
        # (one term: the roundings of the first and last layer's activations, 2^-9 each, besides)
        assert np.linalg.norm(got - want) <= (2.4e-3 if terms == 2 else 6e-3) * np.linalg.norm(want), (rows, act, terms)
        ctx.close()


@pytest.mark.parametrize("eight_bit", [False, True])
def test_samples_follow_the_oracle(eight_bit):
    cfg = dict(kind="gated", d=16, E=8, width=64, hidden=160, n_blocks=2, K=30, chains=6, L=12, eight_bit=eight_bit)
    T, p, model, runtime = setup(cfg)
    ctx = runtime.open_ctx(cfg, p, seed=3)
    a, b = runtime.alloc_traj(ctx), runtime.alloc_traj(ctx)
    ctx.sample(a)
    for c in range(cfg["chains"]):
        f = H.follow_chain(cfg, T, model, 3, c, a[c].cpu().numpy(), 2e-2)
        assert H.rel_err(a[c].cpu().numpy(), f["y"]) <= 2e-2, c
    # plain launches, and the entry that allocates nothing
    ctx.use_graphs(False)
    ctx.sample(b)
    assert torch.equal(a, b)
    ctx.sample_noalloc(b)
    assert H.rel_err(b.cpu().numpy(), a.cpu().numpy()) <= 2e-2
    ctx.close()


@pytest.mark.parametrize("eight_bit", [False, True])
def test_sequential_and_windows_of_one(eight_bit):
    cfg = dict(kind="gated", d=32, E=16, width=96, hidden=224, n_blocks=2, K=20, chains=5, L=1, eight_bit=eight_bit)
    T, p, model, runtime = setup(cfg)
    ctx = runtime.open_ctx(cfg, p, seed=2)
    a, s = runtime.alloc_traj(ctx), runtime.alloc_traj(ctx)
    ctx.sample(a)
    ctx.sample_sequential(s)
    assert torch.equal(a, s)
    for c in (0, 4):
        xi, _ = chain_randoms(2, c, cfg["K"], cfg["d"])
        ys = oasd.sequential_chain(xi[0], T["c_x"], T["c_0"], T["sigma"], model, xi)
        assert H.rel_err(s[c].cpu().numpy(), ys) <= 2e-2
    ctx.close()


@pytest.mark.parametrize("control", [False, True])
def test_windows_in_pieces_and_by_the_controller(control):
    """Sizes at which windows are taken in pieces or rounds differ in rows.  A random-weight network is no contraction: over 60 steps
    the 2e-3 that two correct model calls differ by grows to a tenth of the state.  So every round is compared from the device's own
    state, where a round's rows hold one model call's difference, scaled by c_0 < 1."""
    cfg = dict(kind="gated", d=112, E=128, width=512, hidden=1376, n_blocks=3, K=60, chains=64, L=16, eight_bit=True)
    T, p, model, runtime = setup(cfg)
    ctx = runtime.open_ctx(cfg, p, seed=7)
    ctx.use_adaptive_window(control)
    a = runtime.alloc_traj(ctx)
    rounds = torch.zeros(64, dtype=torch.int32, device=DEV)
    for _ in range(2):
        ctx.sample(a, rounds)
        assert bool(torch.isfinite(a).all())
        assert 60 / 16 <= float(rounds.min()) and float(rounds.max()) <= 60
        for c in (5, 60):
            f = H.follow_chain(cfg, T, model, 7, c, a[c].cpu().numpy(), 2e-2, adaptive=control, resync=True)
            assert f["a"] == 60 and f["R"] == int(rounds[c]) and f["round_err"] <= 2e-2, f["round_err"]
    ctx.close()
