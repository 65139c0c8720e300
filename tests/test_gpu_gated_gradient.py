"""How exact the gradient of the gated unit is: as exact as its results' own rounding, at every size.

Let D be the gradient in 64 bits, R that rounded once to the results' type, and x a kernel's number before it is rounded, off from D
by at most s.  Then what the kernel returns, the number of the type nearest to x, is off from D by at most |R - D| + 2 s: no number of
the type is nearer to x than R is up to s on either side.  dg and du are the sum of two numbers of 8 bits (bf16), which leave
2^-16 of them at most; fp16 operands are such a sum, too, an exact one, and the product of both second numbers, 2^-16 of the whole at
most, is left out; u = 2^-24 is half a step of fp32, in which g, u and all sums are formed."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def O():
    from paper_2505_03983_amd import operators
    return operators


def randn(g, *shape, t=F32, scale=1.0):
    return (scale * torch.randn(*shape, generator=g, device=DEV)).to(t)


def act_def(z, kind):
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    c = (2 / torch.pi) ** 0.5
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def definition(dh, x, wg, wu, act):
    """[(D, s)] of dx, dw_gate, dw_up: the gradient in 64 bits, and what a kernel's may be off by before its last rounding.

    g and u: sums of K products in fp32, (K + 1) u times the products' magnitudes.  |act'| <= 1.13, |act''| <= 1.2; the slope is
    formed to 2^-20 (1 + |z|)^3 of its size (exp2 and reciprocal to 1 ulp each on an argument rounded to fp32, its polynomial
    included), the value to 2^-20 (1 + |z|).  The products' sums: their length in roundings, and 130 for the parts they are added in."""
    half = x.dtype == F16
    dh, x, wg, wu = dh.double(), x.double(), wg.double(), wu.double()
    zg, zu = x @ wg.T, x @ wu.T
    k = (x.shape[1] + 1) * U
    eg, eu = k * (x.abs() @ wg.abs().T), k * (x.abs() @ wu.abs().T)
    a, da = act_def(zg, act)
    dg, du = dh * zu * da, dh * a
    bent = 2.0 ** -20 * (1 + zg.abs()) ** 3
    sdg = dh.abs() * (1.2 * eg * (zu.abs() + eu) + da.abs() * eu + bent * zu.abs())
    sdu = dh.abs() * (1.13 * eg + bent * a.abs())
    left = 2.0 ** (-15 if half else -16)
    sdg, sdu = sdg + left * (dg.abs() + sdg), sdu + left * (du.abs() + sdu)
    out = []
    s = sdg @ wg.abs() + sdu @ wu.abs()
    out.append((dg @ wg + du @ wu, s + (4 * wg.shape[0] + 260) * U * ((dg.abs() + sdg) @ wg.abs() + (du.abs() + sdu) @ wu.abs())))
    for d, sd in ((dg, sdg), (du, sdu)):
        out.append((d.T @ x, sd.T @ x.abs() + (2 * x.shape[0] + 260) * U * ((d.abs() + sd).T @ x.abs())))
    return out


def rms(v):
    return float(v.square().mean().sqrt())


# few rows and one more; few numbers in dg and du, few weights, and one row or channel more; many of everything; odd sizes; tall and
# wide ones
SIZES = [(4, 1024, 520), (64, 320, 136), (65, 320, 136), (512, 96, 256), (513, 96, 256), (700, 512, 256), (700, 512, 257),
         (300, 300, 450), (31, 768, 2048), (129, 400, 999), (2100, 300, 500), (9001, 640, 72), (20, 72, 6000), (1100, 2049, 1031)]


def check(dh, x, wg, wu, act):
    t = x.dtype
    got = O().gated_ff_backward(dh, x, wg, wu, act)
    for name, y, (D, s) in zip(("dx", "dw_gate", "dw_up"), got, definition(dh, x, wg, wu, act)):
        R = D.to(t).double()
        e = (y.double() - D).abs()
        over = e - (R - D).abs() - 2 * s
        assert float(over.max()) <= 0.0, (name, float(over.max()))
        # what is left out of dg and du, 2^-16 or 2^-15 at most, is 2^-7 (bf16) or 2^-4 (fp16) of the results' rounding at most; in root
        # mean square it is less, and errors that do not depend on each other add as squares
        more = rms(e) / rms(R - D)
        assert more <= 1.05, (name, more)


@pytest.mark.parametrize("rows, cols, channels", SIZES)
@pytest.mark.parametrize("t, act", [(BF16, "silu"), (F16, "gelu")])
def test_errors_are_those_of_the_results_rounding(rows, cols, channels, t, act):
    g = torch.Generator(device=DEV).manual_seed(rows + channels)
    x, dh = randn(g, rows, cols, t=t), randn(g, rows, channels, t=t)
    wg, wu = (randn(g, channels, cols, t=t, scale=cols ** -0.5) for _ in range(2))
    check(dh, x, wg, wu, act)


@pytest.mark.parametrize("rows, cols, channels", [(40, 320, 136), (4096, 128, 1100), (700, 512, 257)])
@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("scale", [1e-5, 2e-6, 2.0 ** -24])
def test_small_gradients(rows, cols, channels, t, scale):
    """dh next to fp16's smallest numbers: dg and du are below them, their sums over rows are not."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    x, dh = randn(g, rows, cols, t=t), randn(g, rows, channels, t=t, scale=scale)
    wg, wu = (randn(g, channels, cols, t=t, scale=cols ** -0.5) for _ in range(2))
    check(dh, x, wg, wu, "silu")


@pytest.mark.parametrize("rows", [50, 130])
@pytest.mark.parametrize("t", [BF16, F16])
def test_large_gradients(rows, t):
    """dh u act'(g) above fp16's largest number, dx and the weights' gradients below it."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    cols, channels = 256, 520
    x, dh = randn(g, rows, cols, t=t, scale=0.02), randn(g, rows, channels, t=t, scale=2000.0)
    wg, wu = randn(g, channels, cols, t=t, scale=0.01), randn(g, channels, cols, t=t, scale=125.0)
    D = definition(dh, x, wg, wu, "silu")
    assert all(float(d.abs().max()) < 65000 for d, _ in D)
    zg, zu = x.double() @ wg.double().T, x.double() @ wu.double().T
    assert float((dh.double() * zu * act_def(zg, "silu")[1]).abs().max()) > 2 * 65504
    check(dh, x, wg, wu, "silu")


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("rows", [5, 90])
def test_what_is_not_finite_stays_in_its_row_and_channel(t, rows):
    """An infinity in dh reaches its row of dx and its channel of the weights' gradients, and nothing else."""
    g = torch.Generator(device=DEV).manual_seed(1)
    cols, channels = 72, 136
    x, dh = randn(g, rows, cols, t=t), randn(g, rows, channels, t=t)
    wg, wu = (randn(g, channels, cols, t=t, scale=0.1) for _ in range(2))
    clean = O().gated_ff_backward(dh, x, wg, wu)
    dh[3, 7] = float("inf")
    dx, dwg, dwu = O().gated_ff_backward(dh, x, wg, wu)
    others = [i for i in range(rows) if i != 3]
    assert torch.equal(dx[others], clean[0][others]) and not bool(torch.isfinite(dx[3]).any())
    others = [i for i in range(channels) if i != 7]
    for a, b in ((dwg, clean[1]), (dwu, clean[2])):
        assert torch.equal(a[others], b[others]) and not bool(torch.isfinite(a[7]).any())
