"""The operators and torch's autograd: nothing is detached in silence, and the pairs of calls make an autograd function."""
import pytest
import torch

from paper_2505_03983_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def O():
    from paper_2505_03983_amd import operators
    return operators


def tensors(seed=1, rows=9, cols=72, channels=40):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV).to(BF16)   # noqa: E731
    return r(rows, cols), r(channels, cols), r(channels, cols), r(cols), r(rows, channels)


def test_arguments_that_require_a_gradient_are_refused_where_it_is_recorded():
    o = O()
    x, wg, wu, gain, dh = tensors()
    ones = torch.ones(40, device=DEV)
    q, qs = o.quantize_rows(x)
    w, ws = o.quantize_rows(wg)

    def calls(x, wg, gain, ws):
        return [lambda: o.rms_norm(x, gain), lambda: o.rms_norm(x, gain, residual=x), lambda: o.quantize_rows(x), lambda: o.gated_ff(x, wg, wu),
                lambda: o.gated_ff_backward(dh, x, wg, wu), lambda: o.rms_norm_backward(x, x, gain), lambda: o.linear_i8(q, qs, w, ws, ones)]
    plain = [c() for c in calls(x, wg, gain, ws)]
    leaves = [t.clone().requires_grad_() for t in (x, wg, gain, ws)]
    for c in calls(*leaves):
        with pytest.raises(binding.AsdError) as e:
            c()
        assert e.value.status == binding.ASD_EINVAL
    with pytest.raises(binding.AsdError):
        o.gated_ff(x, wg, wu, out=dh.clone().requires_grad_())
    with torch.no_grad():
        for c, want in zip(calls(*leaves), plain):
            got = c()
            for a, b in zip(got if isinstance(got, tuple) else (got,), want if isinstance(want, tuple) else (want,)):
                assert (a is None and b is None) or torch.equal(a, b)


def test_an_autograd_function_of_the_pairs():
    o = O()

    class Block(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, gain, wg, wu):
            n, _, total = o.rms_norm(x, gain, sum_out=torch.empty_like(x))
            ctx.save_for_backward(n, total, gain, wg, wu)
            return o.gated_ff(n, wg, wu)

        @staticmethod
        def backward(ctx, dh):
            n, total, gain, wg, wu = ctx.saved_tensors
            dn, dwg, dwu = o.gated_ff_backward(dh, n, wg, wu)
            dx, dgain = o.rms_norm_backward(dn, total, gain)
            return dx, dgain, dwg, dwu

    x, wg, wu, gain, dh = tensors(2)
    leaves = [t.clone().requires_grad_() for t in (x, gain, wg, wu)]
    Block.apply(*leaves).backward(dh)
    n, _, _ = o.rms_norm(x, gain)
    dn, dwg, dwu = o.gated_ff_backward(dh, n, wg, wu)
    dx, dgain = o.rms_norm_backward(dn, x, gain)
    for leaf, want in zip(leaves, (dx, dgain, dwg, dwu)):
        assert torch.equal(leaf.grad, want)
