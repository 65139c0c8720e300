"""Networks with gated blocks: how a window is launched -- whole, in pieces, for the rows the controller expects -- changes no bit."""
import pytest
import torch

import asd_workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def setup(cfg):
    from paper_2505_03983_amd import runtime
    return W.make_params(cfg), runtime


@pytest.mark.parametrize("width, hidden, chains, L, K, eight_bit", [
    (4096, 8192, 64, 32, 40, False),     # whole windows on 256 x 256 tiles, pieces on smaller ones
    (4096, 1024, 8, 128, 150, False),    # pieces of as many rows as the kernel for few rows may take, windows of a thousand
    (512, 1376, 200, 16, 60, False),
    (1040, 528, 100, 24, 60, True),
])
def test_windows_in_pieces_change_no_bit(width, hidden, chains, L, K, eight_bit):
    cfg = dict(kind="gated", d=112, E=16, width=width, hidden=hidden, n_blocks=3 if L == 128 else 1, K=K, L=L, chains=chains,
               eight_bit=eight_bit)
    p, runtime = setup(cfg)
    ctx = runtime.open_ctx(cfg, p, seed=0)
    runs = []
    for pieces, graphs, profile in ((False, True, False), (True, True, False), (True, False, False), (False, True, True), (True, True, True)):
        ctx.use_window_pieces(pieces)
        ctx.use_graphs(graphs)
        ctx.profile_enable(profile)
        ctx.set_seed(6)
        traj = torch.full((chains, K + 1, 112), float("nan"), device=DEV)
        rounds = torch.zeros(chains, dtype=torch.int32, device=DEV)
        n = ctx.sample(traj, rounds)
        torch.cuda.synchronize()
        runs.append((traj, rounds, n, ctx.profile_rows()))
    ctx.close()
    traj, rounds, n, _ = runs[0]
    assert bool(torch.isfinite(traj).all()) and n == int(rounds.max())
    for t, r, m, _ in runs[1:]:
        assert m == n and torch.equal(r, rounds) and torch.equal(t, traj)
    (starts, whole), (starts_p, pieces) = runs[3][3], runs[4][3]
    # (small networks take windows whole: fewer rows are no faster there)
    assert starts == starts_p and (pieces < 0.8 * whole if width == 4096 else pieces <= whole)


@pytest.mark.parametrize("chains, eight_bit", [(90, False), (90, True), (8, False)])
def test_controlled_windows_change_no_bit_with_the_rows_that_are_expected(chains, eight_bit):
    """A batch whose chains all start alike and one in which half of them start elsewhere go through the launches' forms in their own
    time; what the chains they share do is the same."""
    cfg = dict(kind="gated", d=112, E=16, width=1024, hidden=2048, n_blocks=1, K=100, L=48, chains=chains, eight_bit=eight_bit)
    p, runtime = setup(cfg)
    ctx = runtime.open_ctx(cfg, p, seed=3)
    ctx.use_adaptive_window(True)
    runs = []
    g = torch.Generator(device=DEV).manual_seed(2)
    y0 = torch.randn(chains, 112, generator=g, device=DEV)
    for scale in (1.0, 0.0, 30.0):
        start = y0.clone()
        start[chains // 2:] *= scale
        for graphs in (True, False):
            ctx.use_graphs(graphs)
            ctx.set_seed(3)
            traj, rounds = torch.full((chains, 101, 112), float("nan"), device=DEV), torch.zeros(chains, dtype=torch.int32, device=DEV)
            ctx.sample(traj, rounds, start)
            runs.append((traj[: chains // 2].clone(), rounds[: chains // 2].clone()))
    ctx.close()
    assert bool(torch.isfinite(runs[0][0]).all())
    for t, r in runs[1:]:
        assert torch.equal(t, runs[0][0]) and torch.equal(r, runs[0][1])


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16, torch.int8])
@pytest.mark.parametrize("cols", [2080, 333])
def test_a_rows_bits_do_not_depend_on_the_tile(cols, t):
    """Calls of 65 rows and more, on tiles of 64, 128 and 256 rows; numbers of very different sizes, so that every order of addition
    rounds differently."""
    from paper_2505_03983_amd import operators as O
    g = torch.Generator(device=DEV).manual_seed(cols)
    rows, channels = 5000, 2100

    def matrix(n):
        if t == torch.int8:
            return torch.randint(-128, 128, (n, cols), generator=g, device=DEV, dtype=torch.int32).to(t)
        return (torch.randn(n, cols, generator=g, device=DEV) * torch.exp2(-4 * torch.rand(n, cols, generator=g, device=DEV)) / 16).to(t)
    x, wg, wu = matrix(rows), matrix(channels), matrix(channels)
    one, more = torch.full((rows,), 1e-3, device=DEV), torch.full((channels,), 1e-3, device=DEV)

    def call(n):
        if t == torch.int8:
            return O.gated_ff(x[:n], wg, wu, x_scale=one[:n], gate_scale=more, up_scale=more)
        return O.gated_ff(x[:n], wg, wu)
    whole = call(rows)
    for n in (65, 130, 300, 700, 1500, 2600, 4000):
        assert torch.equal(call(n), whole[:n]), n
