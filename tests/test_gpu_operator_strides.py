"""Outputs and inputs of the gradients at pitches of their own, and as columns of one wider matrix: the same bits as side by side, and
nothing written besides."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def O():
    from paper_2505_03983_amd import operators
    return operators


def randn(g, *shape, t=F32, scale=1.0):
    return (scale * torch.randn(*shape, generator=g, device=DEV)).to(t)


class Wide:
    """Matrices as columns of one wider one that holds 7 elsewhere."""

    def __init__(self, t, rows, *cols, gap):
        self.held = torch.full((rows, sum(c + gap for c in cols)), 7.0, device=DEV).to(t)
        self.views, at = [], 0
        self.free = torch.ones(self.held.shape[1], dtype=torch.bool, device=DEV)
        for c in cols:
            self.views.append(self.held[:, at:at + c])
            self.free[at:at + c] = False
            at += c + gap

    def untouched(self):
        return bool((self.held[:, self.free] == 7).all())


@pytest.mark.parametrize("gap", [1, 8, 40])
@pytest.mark.parametrize("rows, cols", [(5, 777), (33, 1032), (70, 4104), (9, 9000)])
@pytest.mark.parametrize("t", [F32, BF16])
def test_norm_gradient(rows, cols, gap, t):
    g = torch.Generator(device=DEV).manual_seed(cols + gap)
    values = [randn(g, rows, cols, t=t) for _ in range(3)]
    gain = randn(g, cols, t=t)
    want, want_gain = O().rms_norm_backward(values[0], values[1], gain, dsum=values[2])
    w = Wide(t, rows, cols, cols, cols, cols, gap=gap)
    for v, a in zip(w.views, values):
        v.copy_(a)
    dy, r, dsum, out = w.views
    dx, dgain = O().rms_norm_backward(dy, r, gain, dsum=dsum, dx=out)
    assert dx is out and torch.equal(dx, want) and torch.equal(dgain, want_gain)
    for v, a in zip(w.views, values):
        assert torch.equal(v, a)
    assert w.untouched()
    for into in (dsum, dy):       # in place
        keep = into.clone()
        O().rms_norm_backward(dy, r, gain, dsum=dsum, dx=into)
        assert torch.equal(into, want) and w.untouched()
        into.copy_(keep)


# few rows, sums that are split (and finish into rows apart), one tile and many
@pytest.mark.parametrize("gap", [1, 8])
@pytest.mark.parametrize("rows, cols, channels", [(3, 72, 40), (40, 520, 6000), (130, 520, 1030), (9000, 264, 72), (700, 1100, 1500)])
@pytest.mark.parametrize("t", [BF16, F16])
def test_gated_gradient(rows, cols, channels, gap, t):
    g = torch.Generator(device=DEV).manual_seed(rows + gap)
    x, dh = randn(g, rows, cols, t=t), randn(g, rows, channels, t=t)
    wg, wu = (randn(g, channels, cols, t=t, scale=cols ** -0.5) for _ in range(2))
    want = O().gated_ff_backward(dh, x, wg, wu)
    dx = Wide(t, rows, cols, gap=gap)
    dw = Wide(t, channels, cols, cols, gap=gap)
    got = O().gated_ff_backward(dh, x, wg, wu, dx=dx.views[0], dw_gate=dw.views[0], dw_up=dw.views[1])
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert dx.untouched() and dw.untouched()
    # dx between dh's rows, the weights' gradients below one another
    side = Wide(t, rows, channels, cols, gap=gap)
    side.views[0].copy_(dh)
    both = torch.zeros(2 * channels, cols, dtype=t, device=DEV)
    got = O().gated_ff_backward(side.views[0], x, wg, wu, dx=side.views[1], dw_gate=both[:channels], dw_up=both[channels:])
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert side.untouched() and torch.equal(side.views[0], dh)


def test_forward_calls_between_columns():
    g = torch.Generator(device=DEV).manual_seed(4)
    rows, cols, channels = 150, 264, 320
    w = Wide(BF16, rows, cols, channels, cols, gap=8)
    x, out, total = w.views
    x.copy_(randn(g, rows, cols, t=BF16))
    keep, res = x.clone(), randn(g, rows, cols, t=BF16)
    wg, wu = randn(g, channels, cols, t=BF16), randn(g, channels, cols, t=BF16)
    h = O().gated_ff(x, wg, wu, out=out)
    assert torch.equal(h, O().gated_ff(keep, wg, wu)) and torch.equal(x, keep) and w.untouched()
    y, _, r = O().rms_norm(x, residual=res, sum_out=total)
    z, _, s = O().rms_norm(keep, residual=res)
    assert torch.equal(y, z) and torch.equal(r, s) and torch.equal(x, keep) and w.untouched()
