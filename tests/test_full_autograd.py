"""What full attention and rotary positions tell autograd, without a GPU: the front end as it is, its launches left out."""
import importlib

import numpy as np
import pytest

torch = pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")

# (the package's names of both modules' functions hide the modules)
full, rotary_module = (importlib.import_module("paper_2604_03815_amd." + n) for n in ("full", "rotary"))

BF, SF = torch.bfloat16, torch.float32
F = np.ones(8)


@pytest.fixture
def no_launch(monkeypatch):
    for module, launch in ((full, "_launch"), (rotary_module, "_launch_on")):
        monkeypatch.setattr(module, "_check_devices", lambda *named: named[0][0].device)
        monkeypatch.setattr(module, launch, lambda device, call, *args: None)


def z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


def attend_args():
    return z(40, 4, 32), z(50, 2, 32), z(50, 2, 16), 0.25


def test_given_outputs_count_as_written(no_launch):
    out, lse = z(40, 4, 16), z(40, 4, dtype=SF)
    kmip.full_fwd(*attend_args(), out=out, lse=lse)
    assert out._version == 1 and lse._version == 1
    grads = z(40, 4, 32), z(50, 2, 32), z(50, 2, 16)
    q, k, v, scale = attend_args()
    kmip.full_bwd(q, k, v, z(40, 4, 16), out, lse, scale, dq=grads[0], dk=grads[1], dv=grads[2])
    assert [t._version for t in (out, lse, *grads)] == [1] * 5 and [t._version for t in (q, k, v)] == [0] * 3
    q, k = z(9, 2, 16), z(9, 1, 16)
    q_out = z(9, 2, 16)
    kmip.rotary(q, k, freqs=F, q_out=q_out, k_out=k)
    assert (q._version, q_out._version, k._version) == (0, 1, 1)
    with torch.inference_mode():   # (such tensors have no counter)
        kmip.rotary(z(9, 2, 16), freqs=F, q_out=z(9, 2, 16))


def test_saved_tensor_turned_in_place(no_launch):
    """w * q saves q; turning q in place afterwards makes w's gradient an error, as torch's own operations in place do."""
    w, q = torch.ones(2, 1, dtype=BF, requires_grad=True), torch.ones(9, 2, 16, dtype=BF)
    y = w * q
    kmip.rotary(q, freqs=F, q_out=q)
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()


def test_outputs_of_a_graph_are_refused(no_launch):
    """A given output that requires a gradient would keep the gradient of the values it had."""
    def of_graph(*shape, dtype=BF):
        return torch.ones(*shape, dtype=dtype, requires_grad=True) * 2

    calls = [lambda: kmip.full_fwd(*attend_args(), out=of_graph(40, 4, 16)), lambda: kmip.full_fwd(*attend_args(), lse=of_graph(40, 4, dtype=SF)),
             lambda: kmip.full_bwd(*attend_args()[:3], z(40, 4, 16), z(40, 4, 16), z(40, 4, dtype=SF), 0.25, dk=of_graph(50, 2, 32)),
             lambda: kmip.rotary(z(9, 2, 16), freqs=F, q_out=of_graph(9, 2, 16)),
             lambda: kmip.rotary(z(9, 2, 16), z(9, 2, 16), freqs=F, k_out=of_graph(9, 4, 16)[:, ::2])]
    for one in calls:
        with pytest.raises(ValueError, match="requires a gradient"):
            one()
        with torch.no_grad():
            one()


def test_dual_tensors_are_refused(no_launch):
    """No forward-mode derivative: an error, not a result without its tangent."""
    forward_ad = torch.autograd.forward_ad
    with forward_ad.dual_level():
        x = forward_ad.make_dual(z(9, 2, 16), z(9, 2, 16))
        for q, k in ((x, None), (z(9, 2, 16), x)):
            with pytest.raises(NotImplementedError):
                kmip.rotary(q, k, freqs=F)
            with pytest.raises(ValueError, match="differentiable"):
                kmip.rotary(q, k, freqs=F, q_out=z(9, 2, 16))
        with pytest.raises(NotImplementedError):
            kmip.full_attention(z(9, 2, 16), x, z(9, 2, 16), 0.25)
        y = kmip.rotary(z(9, 2, 16), freqs=F)   # tensors without a tangent are as ever
        assert forward_ad.unpack_dual(y).tangent is None
