"""The operators of a gated residual network against their definitions in 64 bits.

Tolerances are sums of what each rounding may do.  u = 2^-24 is half a step of fp32, h that of the output's type.  A sum of K
products in fp32, in any order, is off by at most (K + 1) u times the sum of the products' magnitudes; sums of 8-bit products are
exact.  The activation's exp2 and reciprocal are the hardware's (1 ulp each) on an argument rounded to fp32: 2^-20 (1 + |z|) of
the value covers them."""
import pytest
import torch

from paper_2505_03983_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-6


def O():
    from paper_2505_03983_amd import operators
    return operators


def half(t):
    return torch.finfo(t).eps / 2


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, t=F32, scale=1.0, gap=0):
    x = (scale * torch.randn(*shape, generator=g, device=DEV)).to(t)
    if gap:
        held = torch.full((shape[0], shape[1] + gap), float("nan"), device=DEV).to(t)
        held[:, : shape[1]] = x
        return held[:, : shape[1]]
    return x


def rand_i8(g, rows, cols, gap=0):
    x = torch.randint(-128, 128, (rows, cols + gap), generator=g, device=DEV, dtype=torch.int32).to(torch.int8)
    return x[:, :cols]


def close(got, want, tol, what=""):
    """|got - want| <= tol everywhere, and the smallest number a type holds besides."""
    assert got.shape == want.shape
    tiny = float(torch.finfo(got.dtype).smallest_normal) * 2 if got.dtype == F16 else 0.0
    d = (got.double() - want).abs() - tol - tiny
    assert bool(torch.isfinite(got.double()).all()), what
    assert float(d.max()) <= 0.0, (what, float(d.max()), float(want.abs().max()))


# ---- norm ------------------------------------------------------------------------------------------------------------------
def norm_def(x, gain, residual, eps=EPS):
    """(r in fp32, rstd, v) of the definition."""
    r = x.float() if residual is None else x.float() + residual.float()
    d = r.double()
    rstd = 1.0 / torch.sqrt(d.square().mean(1, keepdim=True) + eps)
    return r, rstd, d if gain is None else d * gain.double()


def integers(v):
    top = v.abs().amax(1, keepdim=True)
    q = torch.round(127.0 * v / top)
    return torch.where(top > 0, q, torch.zeros_like(q)).to(torch.int8), top


WIDTHS = [(1, 1), (3, 2), (1, 64), (5, 7), (4, 512), (7, 513), (6, 1000), (2, 2048), (3, 2056), (5, 4104), (3, 8192), (2, 8193),
          (3, 16384), (2, 30001), (2, 32768)]


@pytest.mark.parametrize("rows, cols", WIDTHS)
@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_norm_of_every_width(rows, cols, t):
    g = gen(cols)
    x, gain = randn(g, rows, cols, t=t, scale=3.0), randn(g, cols, t=t)
    res = randn(g, rows, cols, t=t)
    for residual in (None, res):
        r, rstd, v = norm_def(x, gain, residual)
        q, scale, total = O().rms_norm(x, gain, EPS, residual=residual, out_type=torch.int8)
        want, top = integers(v)
        assert torch.equal(q, want)
        close(scale[:, None], top * rstd / 127.0, 2 * U * top * rstd / 127.0, "scale")
        assert total is None if residual is None else torch.equal(total, r.to(t))
        for ot in (F32, BF16, F16):
            y, none, _ = O().rms_norm(x, gain, EPS, residual=residual, out_type=ot)
            assert none is None and y.dtype == ot
            close(y, v * rstd, (v * rstd).abs() * (half(ot) + 4 * U), "y")
    q, scale = O().quantize_rows(x)
    want, top = integers(x.double())
    assert torch.equal(q, want)
    close(scale[:, None], top / 127.0, U * top / 127.0, "scale")


@pytest.mark.parametrize("gap", [1, 3, 8])
@pytest.mark.parametrize("t", [F32, BF16])
def test_norm_of_rows_apart(gap, t):
    g = gen(gap)
    rows, cols = 9, 777
    x, res, gain = randn(g, rows, cols, t=t, gap=gap), randn(g, rows, cols, t=t, gap=gap + 2), randn(g, cols + 1, t=t)[1:]
    held = torch.full((rows, cols + gap), 7, dtype=torch.int8, device=DEV)
    sums = torch.zeros(rows, cols + gap, dtype=t, device=DEV)
    q, scale, total = O().rms_norm(x, gain, EPS, residual=res, out_type=torch.int8, out=held[:, :cols], sum_out=sums[:, :cols])
    r, rstd, v = norm_def(x, gain, res)
    assert torch.equal(q, integers(v)[0]) and torch.equal(total, r.to(t))
    assert bool((held[:, cols:] == 7).all()) and bool((sums[:, cols:] == 0).all())


def test_norm_in_place_and_without_gain():
    g = gen(1)
    for alias in ("x", "res"):
        x, res = randn(g, 12, 4104, t=BF16), randn(g, 12, 4104, t=BF16)
        r, rstd, v = norm_def(x, None, res)
        y, _, total = O().rms_norm(x, None, EPS, residual=res, sum_out=x if alias == "x" else res)
        assert torch.equal(total, r.to(BF16)) and total is (x if alias == "x" else res)
        close(y, v * rstd, (v * rstd).abs() * (half(BF16) + 4 * U))


def test_integers_at_ties_zeros_infinities():
    """v = max / 2 is 63.5 steps: to even, 64; odd multiples of max / 254 are ties with any power of two as max."""
    k = torch.arange(-127, 128, device=DEV)
    x = torch.zeros(8, 600, dtype=F32, device=DEV)
    x[0, :255] = (k * 2 - 1).clamp(-254, 254).float() / 254.0
    x[1, :4] = torch.tensor([1.0, 0.5, -0.5, 0.25], device=DEV)
    x[3, 5], x[3, 9] = 1.0, float("inf")
    x[4, 2] = float("nan")
    x[5] = 1e-38
    x[6, :3] = torch.tensor([3e38, -3e38, 1.5e38], device=DEV)
    x[7, 0] = -2.0 ** -140
    q, scale = O().quantize_rows(x)
    good = [0, 1, 2, 5, 6, 7]
    want, top = integers(x[good].double())
    assert torch.equal(q[good], want)
    assert q[1, :4].tolist() == [127, 64, -64, 32] and scale[2] == 0 and int(q[2].abs().max()) == 0
    assert bool(torch.isnan(scale[3:5]).all()) and int(q[3:5].abs().max()) == 0
    n, ns, _ = O().rms_norm(x, None, EPS, out_type=torch.int8)
    assert torch.equal(n[good], want) and bool(torch.isnan(ns[3:5]).all()) and ns[2] == 0
    # rows whose squares leave fp32
    y, _, _ = O().rms_norm(x[5:8], None, 0.0)
    d = x[5:8].double()
    want = d / d.square().mean(1, keepdim=True).sqrt()
    close(y, want, 4 * U * want.abs())


@pytest.mark.parametrize("rows, cols", [(1, 1), (3, 5), (40, 64), (33, 1000), (300, 1024), (70, 1032), (17, 4104), (5, 8200),
                                        (3, 20000), (2, 32768), (9000, 72)])
@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_norm_gradient(rows, cols, t):
    g = gen(rows + cols)
    gap = 3 if rows == 33 else 0
    r, dy, dsum = randn(g, rows, cols, t=t, gap=gap), randn(g, rows, cols, t=t, gap=gap), randn(g, rows, cols, t=t)
    gain = randn(g, cols, t=t)
    d, gd, dyd = r.double(), gain.double(), dy.double()
    rstd = 1.0 / torch.sqrt(d.square().mean(1, keepdim=True) + EPS)
    n = d * rstd
    along = (gd * dyd * n).mean(1, keepdim=True)
    want = rstd * (gd * dyd - n * along)
    # each term to a few roundings of fp32 (g dy, rstd, n, mean, n mean, their difference, the last product and sum); along is
    # summed in fp32 over up to 32 products of a thread, in 64 bits from there
    slack = 40 * U * rstd * ((gd * dyd).abs() + (n * along).abs() + n.abs() * (gd * dyd * n).abs().mean(1, keepdim=True))
    for ds in (None, dsum):
        dx, dgain = O().rms_norm_backward(dy, r, gain, EPS, dsum=ds)
        w = want if ds is None else want + ds.double()
        close(dx, w, slack + (0 if ds is None else 2 * U * ds.double().abs()) + half(t) * (w.abs() + slack), "dx")
        terms = (dyd * n).abs().sum(0)
        wg = (dyd * n).sum(0)
        close(dgain, wg, (rows + 4) * U * terms + half(t) * (wg.abs() + (rows + 4) * U * terms), "dgain")
    none, dgain2 = O().rms_norm_backward(dy, r, gain, EPS, dx=dy if gap == 0 else None)
    assert torch.equal(dgain2, dgain)
    if gap == 0:
        assert none is dy


def test_norm_gradient_by_differences():
    g = gen(3)
    rows, cols = 4, 40
    x, gain, dy = randn(g, rows, cols), 1 + 0.2 * randn(g, cols), randn(g, rows, cols)
    dx, dgain = O().rms_norm_backward(dy, x, gain, EPS)

    def loss(xd, gd):
        return (dy.double() * xd * gd / torch.sqrt(xd.square().mean(1, keepdim=True) + EPS)).sum()
    h = 1e-5
    for i, j in ((0, 0), (1, 17), (3, 39)):
        e = torch.zeros(rows, cols, dtype=torch.float64, device=DEV)
        e[i, j] = h
        num = (loss(x.double() + e, gain.double()) - loss(x.double() - e, gain.double())) / (2 * h)
        assert abs(float(num - dx[i, j])) <= 1e-5 * (1 + abs(float(num)))
        num = (loss(x.double(), gain.double() + e[i]) - loss(x.double(), gain.double() - e[i])) / (2 * h)
        assert abs(float(num - dgain[j])) <= 1e-5 * (1 + abs(float(num)))


# ---- products ----------------------------------------------------------------------------------------------------------------
# rows, cols, channels: a few rows and many, whole tiles and what is left over, k below and above a stage, one of each
SIZES = [(1, 1, 1), (1, 16, 3), (2, 4096, 48), (1, 1000, 777), (16, 272, 16), (17, 640, 100), (33, 2048, 33), (64, 1040, 130),
         (65, 16, 5), (65, 128, 64), (100, 144, 257), (200, 1003, 129), (129, 400, 999), (257, 96, 1100), (500, 2064, 2000),
         (1025, 333, 2051), (2048, 512, 4096)]


@pytest.mark.parametrize("rows, cols, channels", SIZES + [(3, 131071, 20), (70, 131071, 70), (300, 16400, 200), (64, 14848, 768)])
def test_linear_i8(rows, cols, channels):
    g = gen(rows + channels)
    x, w = rand_i8(g, rows, cols), rand_i8(g, channels, cols)
    if cols == 131071:
        x[:2], w[:2] = -128, -128     # the largest sums there are
    xs, ws = torch.rand(rows, generator=g, device=DEV), torch.rand(channels, generator=g, device=DEV)
    bias = randn(g, channels)
    total = x.double() @ w.double().T
    for b in (None, bias):
        scaled = total * xs.double()[:, None] * ws.double()
        want = scaled if b is None else scaled + b.double()
        slack = 4 * U * (scaled.abs() + want.abs())     # the sum as fp32, two scalings, the bias
        for t in (F32, BF16, F16):
            s = 1.0 if t != F16 else 2.0 ** -14 / max(1.0, cols / 256.0)    # (inside fp16's range)
            if t == F16:
                y = O().linear_i8(x, xs * s, w, ws, None if b is None else b * s, t)
            else:
                y = O().linear_i8(x, xs, w, ws, b, t)
            close(y, want * s, (slack + half(t) * (want.abs() + slack)) * s, str(t))


@pytest.mark.parametrize("rows", [3, 50, 130, 700])
def test_linear_i8_of_rows_apart(rows):
    g = gen(rows)
    cols, channels = 323, 210
    for gx, gw, go in ((1, 0, 3), (13, 13, 0), (0, 5, 8)):
        x, w = rand_i8(g, rows, cols, gx), rand_i8(g, channels, cols, gw)
        held = torch.full((rows, channels + go), 3.0, dtype=BF16, device=DEV)
        ones = torch.ones(max(rows, channels), device=DEV)
        O().linear_i8(x, ones[:rows], w, ones[:channels], out=held[:, :channels])
        want = x.double() @ w.double().T
        close(held[:, :channels], want, half(BF16) * want.abs() + 2 * U * want.abs())
        assert bool((held[:, channels:] == 3.0).all())


def act_def(z, kind):
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    c = (2 / torch.pi) ** 0.5
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def gated_def(x, wg, wu, act):
    """(g, u, act(g), act'(g), bounds of the errors of g and u) in 64 bits."""
    x, wg, wu = x.double(), wg.double(), wu.double()
    zg, zu = x @ wg.T, x @ wu.T
    k = (x.shape[1] + 1) * U
    a, da = act_def(zg, act)
    return zg, zu, a, da, k * (x.abs() @ wg.abs().T), k * (x.abs() @ wu.abs().T)


@pytest.mark.parametrize("rows, cols, channels", SIZES)
@pytest.mark.parametrize("t, act", [(BF16, "silu"), (F16, "gelu")])
def test_gated(rows, cols, channels, t, act):
    g = gen(rows + cols)
    x = randn(g, rows, cols, t=t, gap=5 if rows == 200 else 0)
    wg, wu = (randn(g, channels, cols, t=t, scale=2.0 / cols ** 0.5) for _ in range(2))
    zg, zu, a, da, eg, eu = gated_def(x, wg, wu, act)
    want = a * zu
    # |act'| <= 1.13
    slack = 1.13 * eg * (zu.abs() + eu) + (a.abs() + 1.13 * eg) * eu + 2.0 ** -20 * (1 + zg.abs()) * want.abs()
    close(O().gated_ff(x, wg, wu, act), want, slack + half(t) * (want.abs() + slack))


@pytest.mark.parametrize("rows, cols, channels", SIZES)
@pytest.mark.parametrize("t, act", [(BF16, "gelu"), (F16, "silu")])
def test_gated_of_integers(rows, cols, channels, t, act):
    g = gen(rows + cols)
    x, wg, wu = rand_i8(g, rows, cols), rand_i8(g, channels, cols), rand_i8(g, channels, cols)
    s = (2.0 / (74.0 * cols ** 0.5)) / 74.0
    xs, gs, us = (0.5 + torch.rand(n, generator=g, device=DEV) for n in (rows, channels, channels))
    gs, us = gs * s, us * s
    zg = (x.double() @ wg.double().T) * xs.double()[:, None] * gs.double()
    zu = (x.double() @ wu.double().T) * xs.double()[:, None] * us.double()
    a, da = act_def(zg, act)
    want = a * zu
    slack = 1.13 * 3 * U * zg.abs() * zu.abs() + 4 * U * want.abs() + 2.0 ** -20 * (1 + zg.abs()) * want.abs()
    y = O().gated_ff(x, wg, wu, act, x_scale=xs, gate_scale=gs, up_scale=us, out_type=t)
    close(y, want, slack + half(t) * (want.abs() + slack))


@pytest.mark.parametrize("rows, cols, channels", [(1, 1, 1), (2, 16, 64), (5, 7, 9), (64, 64, 64), (65, 130, 67), (100, 1000, 300),
                                                  (200, 72, 129), (130, 520, 1030), (1000, 256, 512), (700, 1100, 1500),
                                                  (5000, 100, 140), (20, 72, 6000), (9001, 640, 72), (16, 33, 47), (300, 1001, 700),
                                                  (2100, 300, 500)])
@pytest.mark.parametrize("t, act", [(BF16, "silu"), (F16, "gelu")])
def test_gated_gradient(rows, cols, channels, t, act):
    g = gen(rows + cols)
    gap = 3 if rows in (5, 100) else 0
    x, dh = randn(g, rows, cols, t=t, gap=gap), randn(g, rows, channels, t=t, gap=gap)
    wg, wu = (randn(g, channels, cols, t=t, scale=2.0 / cols ** 0.5, gap=gap) for _ in range(2))
    zg, zu, a, da, eg, eu = gated_def(x, wg, wu, act)
    dhd, h = dh.double(), half(t)
    dg, du = dhd * zu * da, dhd * a
    # errors of dg and du: of g and u (|act''| <= 1.2, |act'| <= 1.13), the slope's two terms to 2^-20 (1 + |z|)^3 (its polynomial
    # included), and the rounding to the operands' type
    eps_act = 2.0 ** -20 * (1 + zg.abs()) ** 3
    sdg = dhd.abs() * (1.2 * eg * (zu.abs() + eu) + da.abs() * eu + eps_act * zu.abs())
    sdu = dhd.abs() * (1.13 * eg + eps_act * a.abs())
    tiny = float(torch.finfo(t).smallest_normal) if t == F16 else 0.0
    sdg, sdu = sdg + h * (dg.abs() + sdg) + tiny, sdu + h * (du.abs() + sdu) + tiny
    dx, dwg, dwu = O().gated_ff_backward(dh, x, wg, wu, act)
    xd, wgd, wud = x.double(), wg.double(), wu.double()
    want = dg @ wgd + du @ wud
    size = (dg.abs() + sdg) @ wgd.abs() + (du.abs() + sdu) @ wud.abs()
    s = sdg @ wgd.abs() + sdu @ wud.abs() + (2 * channels + 130) * U * size
    close(dx, want, s + h * (want.abs() + s), "dx")
    for got, d, sd in ((dwg, dg, sdg), (dwu, du, sdu)):
        want = d.T @ xd
        s = sd.T @ xd.abs() + (rows + 65) * U * ((d.abs() + sd).T @ xd.abs())
        close(got, want, s + h * (want.abs() + s), "dw")
    only, n1, n2 = O().gated_ff_backward(dh, x, wg, wu, act, need_dw=False)
    assert torch.equal(only, dx) and n1 is None and n2 is None
    n0, g2, u2 = O().gated_ff_backward(dh, x, wg, wu, act, need_dx=False)
    assert n0 is None and torch.equal(g2, dwg) and torch.equal(u2, dwu)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_gradient_by_differences(act):
    """One row through one channel, the pre-activation from far below zero to far above: what the formulas' derivative has to
    be, from differences of the definition in 64 bits."""
    z = torch.tensor([-100.0, -20.0, -5.0, -1.0, -0.25, 0.0, 0.25, 1.0, 5.0, 20.0, 100.0], device=DEV)
    rows = z.numel()
    x = torch.zeros(rows, 16, dtype=BF16, device=DEV)
    x[:, 0], x[:, 1] = z.to(BF16), 1.5
    wg, wu = torch.zeros(1, 16, dtype=BF16, device=DEV), torch.zeros(1, 16, dtype=BF16, device=DEV)
    wg[0, 0], wu[0, 1] = 1.0, 1.0
    dx, _, _ = O().gated_ff_backward(torch.ones(rows, 1, dtype=BF16, device=DEV), x, wg, wu, act)
    h = 1e-6
    zd = z.to(BF16).double()
    slope = (act_def(zd + h, act)[0] - act_def(zd - h, act)[0]) / (2 * h)
    # dg rounded to bf16, and the same number (times a weight of 1) once more: no second error; differences to 1e-8 of z
    close(dx[:, 0], 1.5 * slope, half(BF16) * 1.5 * slope.abs() + 1e-5)
    close(dx[:, 1], act_def(zd, act)[0], (half(BF16) + 2.0 ** -18) * act_def(zd, act)[0].abs() + 1e-12)


def test_extreme_preactivations():
    """Where the sigmoid's exponential overflows or vanishes, the unit has its limits, and a NaN or an infinity stays in its row."""
    for act in ("silu", "gelu"):
        for rows in (4, 80):
            x = torch.zeros(rows, 32, dtype=BF16, device=DEV)
            x[0, 0], x[1, 0], x[2, 0] = 3e38, -3e38, float("nan")
            w = torch.ones(40, 32, dtype=BF16, device=DEV)
            up = torch.full((40, 32), 2.0 ** -10, dtype=BF16, device=DEV)
            y = O().gated_ff(x, w, up, act)
            assert bool(torch.isinf(y[0]).all()) and bool((y[1] == 0).all()) and bool(torch.isnan(y[2]).all()) and bool((y[3:] == 0).all())


# ---- calls --------------------------------------------------------------------------------------------------------------------
def block(x, res, p, used=None):
    """A gated block on 8-bit integers: the operators together, as a network's block has them."""
    o = O()
    n, ns, r = o.rms_norm(x, p["gain"], EPS, residual=res, out_type=torch.int8, rows_used=used)
    h = o.gated_ff(n, p["wg"], p["wu"], "silu", x_scale=ns, gate_scale=p["gs"], up_scale=p["us"], rows_used=used)
    q, qs = o.quantize_rows(h, rows_used=used)
    return o.linear_i8(q, qs, p["wd"], p["ds"], rows_used=used), r


def block_params(g, width, hidden):
    o = O()
    p = dict(gain=(1 + 0.1 * randn(g, width)).to(BF16))
    for w, s, n, k in (("wg", "gs", hidden, width), ("wu", "us", hidden, width), ("wd", "ds", width, hidden)):
        p[w], p[s] = o.quantize_rows(randn(g, n, k) / k ** 0.5)
    return p


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_block_of_integers(rows):
    """The whole block, against itself in 64 bits with its roundings where they are."""
    g = gen(rows)
    width, hidden = 328, 520
    p = block_params(g, width, hidden)
    x, res = randn(g, rows, width, t=BF16), randn(g, rows, width, t=BF16)
    y, r = block(x, res, p)
    r32, rstd, v = norm_def(x, p["gain"], res)
    q, top = integers(v)
    n = q.double() * (top * rstd / 127).float().double()
    wide = lambda w, s: p[w].double() * p[s].double()[:, None]   # noqa: E731
    a, _ = act_def(n @ wide("wg", "gs").T, "silu")
    h = (a * (n @ wide("wu", "us").T)).to(BF16)
    hq, htop = integers(h.double())
    want = (hq.double() * htop / 127) @ wide("wd", "ds").T
    # h may round to its neighbour in bf16, 2^-8 of it, and an integer to the next, top / 127, where the two sides' h (equal to
    # fp32 accuracy) straddle a border: at most one element in 2^9 does; as a bound, 16 of a row's 520
    slack = 16 * htop / 127 * 2 * wide("wd", "ds").abs().amax()
    close(y, want, slack + half(BF16) * (want.abs() + slack))
    assert torch.equal(r, r32.to(BF16))


def test_rows_used_and_what_is_left_alone():
    g = gen(5)
    o = O()
    for rows, used in ((10, 0), (10, 3), (300, 129), (300, 300), (300, 500), (900, 257), (6, -4)):
        n = torch.tensor([used], dtype=torch.int32, device=DEV)
        keep = min(max(used, 0), rows)
        x, wg, wu = randn(g, rows, 80, t=BF16), randn(g, 144, 80, t=BF16), randn(g, 144, 80, t=BF16)
        out = torch.full((rows, 144), 9.0, dtype=BF16, device=DEV)
        o.gated_ff(x, wg, wu, out=out, rows_used=n)
        assert torch.equal(out[:keep], o.gated_ff(x, wg, wu)[:keep]) and bool((out[keep:] == 9.0).all())
        xq, wq = rand_i8(g, rows, 80), rand_i8(g, 144, 80)
        xs, ws = torch.ones(rows, device=DEV), torch.ones(144, device=DEV)
        out = torch.full((rows, 144), 9.0, dtype=F32, device=DEV)
        o.linear_i8(xq, xs, wq, ws, out=out, out_type=F32, rows_used=n)
        assert torch.equal(out[:keep], o.linear_i8(xq, xs, wq, ws, out_type=F32)[:keep]) and bool((out[keep:] == 9.0).all())
        q, s = torch.full((rows, 80), 9, dtype=torch.int8, device=DEV), torch.full((rows,), 9.0, device=DEV)
        tot = torch.full((rows, 80), 9.0, dtype=BF16, device=DEV)
        o.rms_norm(x, None, EPS, residual=x, out_type=torch.int8, out=q, scale=s, sum_out=tot, rows_used=n)
        assert bool((q[keep:] == 9).all()) and bool((s[keep:] == 9).all()) and bool((tot[keep:] == 9).all())
        assert torch.equal(tot[:keep], (x + x)[:keep])


def test_no_rows():
    o = O()
    x = torch.zeros(0, 64, dtype=BF16, device=DEV)
    w = torch.zeros(32, 64, dtype=BF16, device=DEV)
    assert o.gated_ff(x, w, w).shape == (0, 32)
    assert o.quantize_rows(x)[0].shape == (0, 64)
    q = torch.zeros(0, 64, dtype=torch.int8, device=DEV)
    s = torch.zeros(0, device=DEV)
    assert o.linear_i8(q, s, w.to(torch.int8), torch.ones(32, device=DEV)).shape == (0, 32)
    dx, dw, du = o.gated_ff_backward(torch.zeros(0, 32, dtype=BF16, device=DEV), x, w, w)
    assert dx.shape == (0, 64) and bool((dw == 0).all()) and bool((du == 0).all())
    dx, dgain = o.rms_norm_backward(x, x)
    assert dx.shape == (0, 64) and bool((dgain == 0).all())


def test_graphs_and_streams():
    """A block and a training step captured once and replayed on new inputs, with eager work between; and on another stream."""
    g = gen(8)
    o = O()
    p = block_params(g, 264, 333)
    x, res = randn(g, 70, 264, t=BF16), randn(g, 70, 264, t=BF16)
    wg, wu = randn(g, 333, 264, t=BF16, scale=0.1), randn(g, 333, 264, t=BF16, scale=0.1)
    dh, gain = randn(g, 70, 333, t=BF16), p["gain"]

    def step():
        y, r = block(x, res, p)
        n, _, tot = o.rms_norm(x, gain, EPS, residual=res)
        h = o.gated_ff(n, wg, wu)
        dn, dwg, dwu = o.gated_ff_backward(dh, n, wg, wu)
        dx, dgain = o.rms_norm_backward(dn, tot, gain, EPS, dsum=res)
        return [y, r, h, dwg, dwu, dx, dgain]

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(4):
        x.copy_(randn(gen(seed), 70, 264, t=BF16))
        dh.copy_(randn(gen(seed + 9), 70, 333, t=BF16))
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)
        with torch.cuda.stream(side):
            again = step()
        side.synchronize()
        for a, b in zip(again, want):
            assert torch.equal(a, b)


def test_calls_on_a_stream_of_their_own():
    g = gen(6)
    o = O()
    x, w, dy = randn(g, 77, 333, t=BF16), randn(g, 130, 333, t=BF16, scale=0.1), randn(g, 77, 130, t=BF16)
    q, qs = o.quantize_rows(x)
    wq, ws = o.quantize_rows(w)
    gain = randn(g, 333, t=BF16)
    calls = [lambda s: o.rms_norm(x, gain, EPS, residual=x, stream=s), lambda s: o.quantize_rows(x, stream=s),
             lambda s: o.rms_norm_backward(x, x, gain, EPS, stream=s), lambda s: o.linear_i8(q, qs, wq, ws, stream=s),
             lambda s: o.gated_ff(x, w, w, stream=s), lambda s: o.gated_ff_backward(dy, x, w, w, stream=s)]
    want = [c(None) for c in calls]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [c(side) for c in calls]
    side.synchronize()
    for a, b in zip(got, want):
        for u, v in zip(a if isinstance(a, tuple) else (a,), b if isinstance(b, tuple) else (b,)):
            assert (u is None and v is None) or torch.equal(u, v)
    with pytest.raises(binding.AsdError):
        o.quantize_rows(x, stream=side.cuda_stream)


def test_results_do_not_depend_on_the_other_rows():
    """In a call of the same size, a row's bits are its own."""
    g = gen(4)
    o = O()
    for rows in (20, 300, 600):
        x = randn(g, rows, 200, t=BF16)
        wg, wu = randn(g, 2100, 200, t=BF16), randn(g, 2100, 200, t=BF16)
        y = o.gated_ff(x, wg, wu)
        x2 = randn(g, rows, 200, t=BF16)
        x2[rows - 7] = x[3]
        assert torch.equal(o.gated_ff(x2, wg, wu)[rows - 7], y[3])


def test_offsets_past_32_bits():
    o = O()
    rows, cols = 70000, 32768
    x = torch.zeros(rows, cols, dtype=BF16, device=DEV)        # 4.6 GB
    x[-1, -3:] = torch.tensor([1.0, -2.0, 4.0], dtype=BF16, device=DEV)
    q, s = o.quantize_rows(x)
    assert q[-1, -3:].tolist() == [32, -64, 127] and float(s[-1]) == pytest.approx(4 / 127) and int(q[:100].abs().max()) == 0
    w = torch.zeros(cols, 16, dtype=torch.int8, device=DEV)
    w[-1] = 1
    a = torch.zeros(rows, 16, dtype=torch.int8, device=DEV)
    a[-1] = 2
    ones = torch.ones(rows, device=DEV)
    o.linear_i8(a, ones, w, ones[:cols], out=x)
    assert float(x[-1, -1]) == 32.0 and float(x[-1, :-1].abs().max()) == 0 and float(x[: rows - 1].abs().max()) == 0


def test_more_rows_than_threads_in_a_dimension():
    """70 million rows of 8, four to a workgroup: 2^32 threads and more."""
    o = O()
    rows = 70_000_000
    x = torch.ones(rows, 8, dtype=F16, device=DEV)
    x[-1] = 2.0
    q, s = o.quantize_rows(x)
    assert bool((q == 127).all()) and float(s[0]) == float(s[rows // 2]) and float(s[-1]) == 2 * float(s[0])
    y, _, _ = o.rms_norm(x, eps=0.0)
    assert bool((y == 1.0).all())
    dx, dgain = o.rms_norm_backward(y, x, eps=0.0)
    assert float(dx.float().abs().max()) == 0.0 and dgain.shape == (8,)


def test_first_call_in_a_graph():
    """Kernels that no call has used before, captured at once (in a process of its own: nothing is warm there)."""
    import subprocess
    import sys
    code = """
import torch
from paper_2505_03983_amd import operators as O
x = torch.randn(600, 512, device="cuda:0").half()
w = torch.randn(8192, 512, device="cuda:0").half() / 20
g = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(g):
    h = O.gated_ff(x, w, w, "gelu")
    dx, dg, du = O.gated_ff_backward(h, x, w, w, "gelu")
g.replay()
torch.cuda.synchronize()
want = O.gated_ff(x, w, w, "gelu")
assert torch.equal(h, want)
a = O.gated_ff_backward(want, x, w, w, "gelu")
assert torch.equal(dx, a[0]) and torch.equal(dg, a[1]) and torch.equal(du, a[2])
print("done")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=100)
    assert r.stdout.strip().endswith("done"), r.stderr[-2000:]


def test_refused_tensors():
    o = O()
    x, w = torch.zeros(4, 32, dtype=BF16, device=DEV), torch.zeros(8, 32, dtype=BF16, device=DEV)
    q, s = torch.zeros(4, 32, dtype=torch.int8, device=DEV), torch.ones(4, device=DEV)
    for call in (lambda: o.gated_ff(x, w, w[:, :16]), lambda: o.gated_ff(x, w, w.half()), lambda: o.gated_ff(x, w, w, "relu"),
                 lambda: o.gated_ff(x.float(), w.float(), w.float()), lambda: o.gated_ff(x.t(), w, w),
                 lambda: o.gated_ff(x, w, w, out=x[:, :8]), lambda: o.gated_ff(x, w.cpu(), w),
                 lambda: o.gated_ff(q, w.to(torch.int8), w.to(torch.int8)), lambda: o.linear_i8(q, s[:3], q, s),
                 lambda: o.linear_i8(q, s, q, s, out_type=torch.int8), lambda: o.linear_i8(x, s, q, s),
                 lambda: o.rms_norm(x, s), lambda: o.rms_norm(x, eps=-1.0), lambda: o.rms_norm(x, out=x), lambda: o.quantize_rows(q),
                 lambda: o.rms_norm(x.expand(4, 32)[:1].expand(4, 32)), lambda: o.quantize_rows(x.cpu()),
                 lambda: o.gated_ff_backward(x, x, w, w), lambda: o.rms_norm_backward(x, x.half()),
                 lambda: o.gated_ff(x, w, w, rows_used=s[:1])):
        with pytest.raises(binding.AsdError) as e:
            call()
        assert e.value.status == binding.ASD_EINVAL
