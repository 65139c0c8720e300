"""Parameters on their way to the device (here: the CPU)."""
import pytest

import asd_workloads as W
from paper_2505_03983_amd import runtime

SHAPE = dict(d=16, E=8, width=32, n_blocks=2, K=10)


@pytest.mark.parametrize("kind, missing", [("mlp", k) for k in ("w_in", "w_blk", "w_out", "b_in", "b_blk", "b_out", "temb")] +
                         [("gated", k) for k in ("w_in", "w_out", "b_in", "b_out", "temb")])
def test_a_missing_parameter_is_an_error(kind, missing):
    """Not a network without that bias."""
    cfg = dict(SHAPE, kind=kind, hidden=48)
    p = W.make_params(cfg)
    out = runtime.device_params(cfg, p, device="cpu")
    assert out["kind"] == kind and missing in out
    del p[missing]
    with pytest.raises(KeyError):
        runtime.device_params(cfg, p, device="cpu")


def test_gated_blocks_have_arrays_of_their_own():
    out = runtime.device_params(dict(SHAPE, kind="gated", hidden=48), W.make_params(dict(SHAPE, kind="gated", hidden=48)), device="cpu")
    assert "w_blk" not in out and "b_blk" not in out and out["w_gate"].shape == (2, 48, 32)
