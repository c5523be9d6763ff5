"""The k-MIP layer's calls of before it had a rotary, without a GPU (the attention itself is replaced)."""
import importlib

import pytest

torch = pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")

layer_module = importlib.import_module("paper_2604_03815_amd.layer")


@pytest.fixture
def plain_attention(monkeypatch):
    monkeypatch.setattr(layer_module, "attention", lambda q, k, v, kk, scale, **kw: v.float())


class Doubled(kmip.KMIPAttention):
    """A subclass with a projection of its own, that takes the features alone."""

    def project(self, x):
        return super().project(2.0 * x)


def test_subclass_with_its_own_projection(plain_attention):
    layer = Doubled(16, 2, 16, generator=torch.Generator().manual_seed(1))
    x = torch.randn(10, 16, generator=torch.Generator().manual_seed(2))
    want = (2.0 * x @ layer.w_v).to(torch.bfloat16).float() @ layer.w_o
    assert torch.equal(layer(x), want) and torch.equal(layer(x, [0, 4, 10]), want)


def test_layer_without_the_attribute(plain_attention):
    """As a layer unpickles that was saved by a version without rotary positions."""
    layer = kmip.KMIPAttention(16, 2, 16, generator=torch.Generator().manual_seed(1))
    x = torch.randn(10, 16, generator=torch.Generator().manual_seed(2))
    want = layer(x)
    del layer.__dict__["rotary"]
    assert torch.equal(layer(x), want)
    with pytest.raises(ValueError, match="rotary"):
        layer(x, positions=torch.zeros(10, dtype=torch.int32))
