"""Edges of the serving operators: sizes, lengths, page numbers and values at the ends of what the calls take, beside
the ordinary ones of test_gpu_serve.py."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_serve import Paged, dev  # noqa: E402,F401


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,Hkv,hd", [(28, 4, 128), (4, 4, 64)])
def test_attention_first_blocks_far_from_zero(dev, H, Hkv, hd, dtype):
    """The first block of a run's every unit makes its probabilities twice, with no reference and with the block's
    maximum: with scores beyond 100 the first ones are infinities and zeros, and must not be what is used."""
    x = Paged([900, 3, 0, 64, 130] * 4, [1, 32, 100, 7, 2] * 4, 700, 32, H, Hkv, hd, dtype=dtype, seed=21, spread=30.0)
    first = x.check()
    for _ in range(20):
        assert torch.equal(x.call(), first)
