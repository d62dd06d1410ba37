"""Arguments that the binding refuses behind good tensors."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2509_06362_amd import instance as I  # noqa: E402
from tests.test_gpu_kv_attention import inst  # noqa: E402, F401


class Neither:
    def __bool__(self):
        raise ValueError("neither")


def test_an_interleaving_that_is_neither_true_nor_false(inst):  # noqa: F811
    """Its own error comes out, and nothing is written."""
    k, v = torch.zeros(1, 2, 1, 16, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 2, 1, 64, 16, dtype=torch.bfloat16, device="cuda")
    x, out = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    cache, slot = I.KvCache(k, v), torch.zeros(1, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError, match="neither"):
        I.maaso_kv_append(inst, cache, layer=0, q=x, k=x, v=x, q_out=out, slot=slot, interleaved=Neither())
    assert not out.any() and not k.any()
    I.maaso_kv_append(inst, cache, layer=0, q=x, k=x, v=x, q_out=out, slot=slot, interleaved=[1])
    assert (out == 1).all() and (k[0, 0, 0, 0] == 1).all()
