"""Layer norm's gradients of rows that do not fit registers, with several workgroups to a device,
whose sums of the columns are joined."""
import pytest

from test_gpu_layer_norm import run, sc  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,weights,pad,bias", [("f32", "f32", 0, True), ("bf16", "f32", 3, True), ("bf16", "bf16", 0, False), ("f32", "bf16", 1, False)])
@pytest.mark.parametrize("T,dim,K", [(700, 8193, 3), (100, 9001, 1), (33, 8200, 1), (260, 16_385, 20)])
def test_long_rows(sc, T, dim, K, kind, weights, pad, bias):  # noqa: F811
    run(sc, T, dim, K, kind, weights, pad, bias)
