"""Mask-token training calls that the binding turns away before any device work."""
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2504_18583_amd", "libpard.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libpard.so not built")


@pytest.fixture(scope="module")
def b():
    from paper_2504_18583_amd import binding
    return binding


def test_tensors_that_require_gradients_are_refused(b):
    """Their gradients would be lost without a word; where torch records none
    (no_grad, an autograd.Function's forward) the call goes on to the next check."""
    t, table, pos = torch.zeros(4, 2, 64), torch.zeros(16, 32, 2), torch.zeros(4, dtype=torch.int32)
    gain = torch.ones(64)

    def calls(x, g):
        return [lambda: b.qk_rope(x, None, pos, table), lambda: b.qk_rope(t, x, pos, table), lambda: b.qk_rope(t, None, pos, table, q_gain=g),
                lambda: b.qk_rope(t, t, pos, table, q_gain=gain, k_gain=g), lambda: b.cod_attn(x, t, t, None), lambda: b.cod_attn(t, x, t, None),
                lambda: b.cod_attn(t, t, x, None)]
    for f in calls(t.clone().requires_grad_(), gain.clone().requires_grad_()):
        with pytest.raises(b.PardError, match="autograd.Function") as e:
            f()
        assert e.value.status == b.PARD_ERR_ARG
        with torch.no_grad(), pytest.raises((b.PardError, AttributeError)) as e:
            f()
        assert "autograd" not in str(e.value)


def test_rope_table_of_a_host_device_is_refused(b):
    """The kernel would write to host memory."""
    for device in ("cpu", torch.device("cpu"), "cpu:0", "meta"):
        with pytest.raises(b.PardError, match="GPU") as e:
            b.rope_table(8, 64, 1e4, device=device)
        assert e.value.status == b.PARD_ERR_ARG


def test_cod_plan_of_host_tensors_is_refused(b):
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(b.PardError, match="device tensors") as e:
        b.cod_plan(z, z, [0, 4], z[:1])
    assert e.value.status == b.PARD_ERR_ARG
