"""What the operators' C entries refuse, on the host: no call here reaches a device."""
import ctypes as C

import pytest

from paper_2505_03983_amd import binding as b

L = b.lib()
EINVAL, EUNSUPPORTED = b.ASD_EINVAL, b.ASD_EUNSUPPORTED
A = 1 << 40     # addresses that are never read: a gigabyte apart


def at(k):
    return A + (k << 30)


def norm(**kw):
    p = b.asd_norm(rows=4, cols=64, type=b.ASD_BF16, out_type=b.ASD_I8, x=at(1), residual=at(2), gain=at(3), sum=at(4), out=at(5),
                   scale=at(6), ld_x=64, ld_residual=64, ld_sum=64, ld_out=64, eps=1e-6)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw, status", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(cols=32769, ld_x=32769), EUNSUPPORTED), (dict(type=b.ASD_I8), EINVAL),
    (dict(type=9), EINVAL), (dict(out_type=4), EINVAL), (dict(eps=-1e-9), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(eps=float("inf")), EINVAL), (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(scale=None), EINVAL),
    (dict(ld_x=63), EINVAL), (dict(ld_sum=0), EINVAL), (dict(ld_out=1 << 60), EINVAL), (dict(x=at(1) + 1), EINVAL),
    (dict(scale=at(6) + 2), EINVAL), (dict(out=at(1) + 8), EINVAL), (dict(sum=at(1) + 2), EINVAL), (dict(sum=at(1), ld_sum=65), EINVAL),
    (dict(sum=at(3)), EINVAL), (dict(out=at(4)), EINVAL), (dict(scale=at(5)), EINVAL),
])
def test_norm_refusals(kw, status):
    assert L.asd_rms_norm(C.byref(norm(**kw)), None) == status, b.last_error()


def test_quantize_refusals():
    assert L.asd_rms_norm(None, None) == EINVAL and L.asd_quantize_rows(None, None) == EINVAL
    # eps, sum and the like are not its own; rows = 0 is nothing to do
    assert L.asd_quantize_rows(C.byref(norm(rows=0, eps=-1.0, sum=at(1) + 1)), None) == b.ASD_OK
    assert L.asd_quantize_rows(C.byref(norm(scale=None)), None) == EINVAL
    assert L.asd_quantize_rows(C.byref(norm(out=at(1))), None) == EINVAL


def grad(**kw):
    p = b.asd_norm_grad(rows=4, cols=64, type=b.ASD_F32, dy=at(1), sum=at(2), gain=at(3), dsum=at(4), dx=at(5), dgain=at(6), ld_dy=64,
                        ld_sum=64, ld_dsum=64, ld_dx=64, eps=1e-6, workspace=at(7), workspace_bytes=1 << 20)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw, status", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(type=3), EINVAL), (dict(dy=None), EINVAL), (dict(sum=None), EINVAL),
    (dict(workspace=None), EINVAL), (dict(workspace_bytes=100), EINVAL), (dict(workspace=at(7) + 8), EINVAL),
    (dict(dx=at(2)), EINVAL), (dict(dgain=at(3)), EINVAL), (dict(dx=at(7)), EINVAL), (dict(dx=at(1), ld_dx=65), EINVAL),
    (dict(cols=32769, ld_dy=32769, ld_sum=32769, ld_dsum=32769, ld_dx=32769), EUNSUPPORTED),
])
def test_norm_gradient_refusals(kw, status):
    assert L.asd_rms_norm_backward(C.byref(grad(**kw)), None) == status, b.last_error()


def test_norm_gradient_workspace():
    assert L.asd_rms_norm_backward_workspace(None) == 0
    assert L.asd_rms_norm_backward_workspace(C.byref(grad(dgain=None))) == 0
    assert L.asd_rms_norm_backward_workspace(C.byref(grad(rows=0))) == 0
    assert L.asd_rms_norm_backward_workspace(C.byref(grad())) >= 4 * 64
    assert L.asd_rms_norm_backward_workspace(C.byref(grad(rows=1 << 30, cols=65536))) <= 4 * 4096 * 65536


def linear(**kw):
    p = b.asd_linear8(rows=4, cols=64, channels=32, out_type=b.ASD_BF16, x=at(1), x_scale=at(2), w=at(3), w_scale=at(4), bias=at(5),
                      out=at(6), ld_x=64, ld_w=64, ld_out=32)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw, status", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(channels=0), EINVAL), (dict(cols=131072, ld_x=131072, ld_w=131072), EUNSUPPORTED),
    (dict(out_type=b.ASD_I8), EINVAL), (dict(x=None), EINVAL), (dict(x_scale=None), EINVAL), (dict(w=None), EINVAL),
    (dict(w_scale=None), EINVAL), (dict(out=None), EINVAL), (dict(ld_x=10), EINVAL), (dict(ld_out=31), EINVAL), (dict(out=at(6) + 1), EINVAL),
    (dict(w_scale=at(4) + 1), EINVAL), (dict(out=at(1)), EINVAL), (dict(out=at(5)), EINVAL), (dict(x=at(1) + 1), EINVAL),
    (dict(ld_w=65), EINVAL), (dict(ld_w=65, workspace=at(8), workspace_bytes=64), EINVAL),
    (dict(ld_w=65, workspace=at(8) + 4, workspace_bytes=1 << 20), EINVAL), (dict(ld_w=65, workspace=at(6), workspace_bytes=1 << 20), EINVAL),
])
def test_linear_refusals(kw, status):
    assert L.asd_linear_i8(C.byref(linear(**kw)), None) == status, b.last_error()


def test_workspaces_are_for_rows_off_sixteen_bytes():
    w = lambda **kw: L.asd_linear_i8_workspace(C.byref(linear(**kw)))   # noqa: E731
    assert L.asd_linear_i8_workspace(None) == 0 and w() == 0 and w(rows=0, ld_x=65) == 0
    assert w(ld_w=65) >= 32 * 64 and w(x=at(1) + 1) >= 4 * 64 and w(cols=63) >= 36 * 64
    assert w(rows=1, ld_x=65) == 0      # one row is at no pitch
    assert L.asd_linear_i8(C.byref(linear(rows=0, x=None)), None) == b.ASD_OK


def gated(**kw):
    p = b.asd_gated(rows=4, cols=64, channels=32, type=b.ASD_BF16, out_type=b.ASD_BF16, act=0, x=at(1), w_gate=at(2), w_up=at(3), out=at(4),
                    ld_x=64, ld_w_gate=64, ld_w_up=64, ld_out=32, x_scale=at(5), gate_scale=at(6), up_scale=at(7), dh=at(8), dx=at(9),
                    dw_gate=at(10), dw_up=at(11), ld_dh=32, ld_dx=64, ld_dw_gate=64, ld_dw_up=64, workspace=at(12), workspace_bytes=1 << 24)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw, status", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(channels=-3), EINVAL), (dict(type=b.ASD_F32, out_type=b.ASD_F32), EINVAL),
    (dict(out_type=b.ASD_F16), EINVAL), (dict(type=b.ASD_I8, out_type=b.ASD_F32), EINVAL), (dict(act=2), EINVAL), (dict(x=None), EINVAL),
    (dict(w_up=None), EINVAL), (dict(out=None), EINVAL), (dict(type=b.ASD_I8, gate_scale=None), EINVAL),
    (dict(type=b.ASD_I8, cols=131072, ld_x=131072, ld_w_gate=131072, ld_w_up=131072), EUNSUPPORTED), (dict(out=at(2)), EINVAL),
    (dict(ld_w_gate=63), EINVAL), (dict(x=at(1) + 2, workspace_bytes=0), EINVAL), (dict(rows=(1 << 28) + 1), EUNSUPPORTED),
    (dict(cols=(1 << 20) + 8, ld_x=1 << 21, ld_w_gate=1 << 21, ld_w_up=1 << 21), EUNSUPPORTED), (dict(out=at(12)), EINVAL),
])
def test_gated_refusals(kw, status):
    assert L.asd_gated_ff(C.byref(gated(**kw)), None) == status, b.last_error()


@pytest.mark.parametrize("kw, status", [
    (dict(type=b.ASD_I8), EINVAL), (dict(dh=None), EINVAL), (dict(dw_up=None), EINVAL), (dict(rows_used=at(20)), EINVAL),
    (dict(dx=at(1)), EINVAL), (dict(dw_gate=at(2)), EINVAL), (dict(dw_gate=at(11)), EINVAL), (dict(workspace=None), EINVAL),
    (dict(workspace_bytes=1000), EINVAL), (dict(workspace=at(9)), EINVAL), (dict(ld_dh=31), EINVAL), (dict(act=-1), EINVAL),
    (dict(rows=(1 << 20) + 1), EUNSUPPORTED),
])
def test_gated_gradient_refusals(kw, status):
    assert L.asd_gated_ff_backward(C.byref(gated(**kw)), None) == status, b.last_error()


def test_gated_gradient_workspace():
    w = lambda **kw: L.asd_gated_ff_backward_workspace(C.byref(gated(**kw)))   # noqa: E731
    assert L.asd_gated_ff_backward_workspace(None) == 0 and L.asd_gated_ff_workspace(None) == 0
    assert w() > w(dx=None) > 0 and w() > w(dw_gate=None, dw_up=None) > 0 and w(rows=0) == 0
    assert L.asd_gated_ff(C.byref(gated(rows=0, x=None)), None) == b.ASD_OK


@pytest.mark.parametrize("kw, status", [
    (dict(hidden=0), EINVAL), (dict(block_type=b.ASD_F32), EINVAL), (dict(act=5), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(w_up=None), EINVAL), (dict(w_down=24), EINVAL), (dict(hidden=20), EUNSUPPORTED), (dict(hidden=65536), EUNSUPPORTED),
    (dict(block_type=b.ASD_I8), EINVAL), (dict(block_type=b.ASD_I8, gate_scale=16, up_scale=16, down_scale=16, width=24), EUNSUPPORTED),
    (dict(w_out=None), EINVAL), (dict(d=12), EUNSUPPORTED),
])
def test_gated_network_refusals(kw, status):
    s = b.asd_schedule_ddpm_linear(10)
    den = dict(kind="gated", d=16, n_tau=11, width=32, hidden=48, n_blocks=2, temb_dim=8, w_in=16, w_out=16, temb=16, w_gate=16, w_up=16,
               w_down=16)
    den.update(kw)
    with pytest.raises(b.AsdError) as e:
        b.Ctx(s, den, 4, 2)
    assert e.value.status == status, b.last_error()


def test_gated_gradient_workspace_of_a_tall_call():
    """A million rows of 2048 through 64 channels: dg and du twice (as they lie and transposed, two numbers each) and x transposed;
    nothing of rows times columns besides."""
    n = L.asd_gated_ff_backward_workspace(C.byref(gated(rows=1 << 20, cols=2048, channels=64, ld_x=2048, ld_w_gate=2048, ld_w_up=2048,
                                                        ld_dh=64, ld_dx=2048, ld_dw_gate=2048, ld_dw_up=2048)))
    assert n <= (1 << 20) * 2 * (2048 + 2 * 4 * 64) + (64 << 20)


@pytest.mark.parametrize("shape", [(2 ** 31, 8), (2 ** 32 + 3, 8), (8, 2 ** 32 + 16)])
def test_sizes_that_32_bits_do_not_hold(shape):
    """Not what is left of them: a call on the first three rows of four billion."""
    import torch
    from paper_2505_03983_amd import operators as O
    x = torch.empty(shape, dtype=torch.bfloat16, device="meta")
    for call in (lambda: O.quantize_rows(x), lambda: O.rms_norm(x), lambda: O.rms_norm_backward(x, x), lambda: O.gated_ff(x, x, x),
                 lambda: O.gated_ff_backward(x, x, x, x), lambda: O.linear_i8(x, x[:, 0], x, x[:, 0])):
        with pytest.raises(b.AsdError) as e:
            call()
        assert e.value.status == EUNSUPPORTED


def test_columns_of_one_matrix_are_no_overlap():
    """Outputs and inputs that are columns of one wider matrix, their rows between each other's, share no byte."""
    status = lambda call, p: call(C.byref(p), None)   # noqa: E731
    ld = 256
    # the shape of a refusal shows where the overlap check ended: with them apart, the next check (no workspace) speaks
    wide = dict(ld_dw_gate=ld, ld_dw_up=ld, workspace=None, workspace_bytes=0)
    for off, apart in ((64, True), (192, True), (63, False), (193, False), (1, False), (256 * 5 + 64, True), (0, False)):
        p = gated(dw_gate=at(10), dw_up=at(10) + 2 * off, **wide)
        assert status(L.asd_gated_ff_backward, p) == EINVAL
        assert ("overlaps" not in b.last_error()) == apart, (off, b.last_error())
    # other pitches, and a row alone
    p = gated(dw_gate=at(10), dw_up=at(10) + 128, ld_dw_gate=256, ld_dw_up=255, workspace=None, workspace_bytes=0)
    assert status(L.asd_gated_ff_backward, p) == EINVAL and "overlaps" in b.last_error()
    p = gated(dx=at(1) + 2 * 128, ld_x=ld, ld_dx=ld, workspace=None, workspace_bytes=0)
    assert status(L.asd_gated_ff_backward, p) == EINVAL and "overlaps" not in b.last_error()
    p = gated(dx=at(1) + 2 * 32, ld_x=ld, ld_dx=ld, workspace=None, workspace_bytes=0)
    assert status(L.asd_gated_ff_backward, p) == EINVAL and "overlaps" in b.last_error()
    # int8 rows between bf16 ones: pitches in bytes
    p = norm(x=at(1), ld_x=96, cols=64, out=at(1) + 128, ld_out=192, scale=None)
    assert status(L.asd_quantize_rows, p) == EINVAL and "scale" in b.last_error()
    p = norm(x=at(1), ld_x=96, out=at(1) + 127, ld_out=192)
    assert status(L.asd_quantize_rows, p) == EINVAL and "overlaps" in b.last_error()


def test_sizes_that_are_refused_need_no_workspace():
    """The refusal is the call's, not that of an allocation for it."""
    wide = dict(ld_x=1 << 21, ld_w_gate=1 << 21, ld_w_up=1 << 21, ld_dh=1 << 21, ld_dx=1 << 21, ld_dw_gate=1 << 21, ld_dw_up=1 << 21)
    for kw in (dict(rows=(1 << 20) + 1), dict(channels=(1 << 20) + 1), dict(cols=(1 << 20) + 8), dict(type=b.ASD_F32), dict(rows=-5),
               dict(channels=2 ** 31 - 1)):
        p = gated(**{**wide, **kw})
        assert L.asd_gated_ff_backward_workspace(C.byref(p)) == 0, kw
        p.workspace, p.workspace_bytes = None, 0
        assert L.asd_gated_ff_backward(C.byref(p), None) in (EINVAL, EUNSUPPORTED) and "workspace" not in b.last_error()
    assert L.asd_gated_ff_workspace(C.byref(gated(cols=(1 << 20) + 8, x=at(1) + 2))) == 0
    assert L.asd_gated_ff_workspace(C.byref(gated(rows=(1 << 28) + 1, x=at(1) + 2))) == 0
    assert L.asd_linear_i8_workspace(C.byref(linear(cols=131073, ld_x=131073, ld_w=131073))) == 0
    assert L.asd_linear_i8_workspace(C.byref(linear(rows=-1, ld_x=65))) == 0
    assert L.asd_rms_norm_backward_workspace(C.byref(grad(cols=32769))) == 0
    # ... and the largest that are taken say what they need
    assert L.asd_gated_ff_backward_workspace(C.byref(gated(rows=1 << 20))) > 0 and L.asd_linear_i8_workspace(C.byref(linear(cols=131071))) > 0
