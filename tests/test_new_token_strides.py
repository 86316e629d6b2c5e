"""rgd_cache_write takes views: a dimension of one element may have any stride."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_20791_gb300 import binding  # noqa: E402
from paper_2607_20791_gb300.build import build  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    return binding.load_library(build())


def _write(k, v, heads):
    """Host tensors: a call whose arguments are all right is refused for that alone, at the end."""
    shape = binding.CacheShape(num_layers=1, num_pages=4, num_kv_heads=heads, page_size=16, head_dim=64)
    pool = torch.empty(4 * heads * 16 * 64, dtype=torch.bfloat16)
    rows = k.shape[0]
    table, per_row = torch.empty(rows, 4, dtype=torch.int32), torch.empty(rows, dtype=torch.int32)
    binding.rgd_cache_write(shape, 0, k, v, per_row, table, per_row, None, pool, pool)


def _strided(size, stride):
    need = 1 + sum((n - 1) * s for n, s in zip(size, stride))
    return torch.empty(need, dtype=torch.bfloat16).as_strided(size, stride)


@pytest.mark.parametrize("size, stride", [
    ((2, 3, 1, 64), (192, 64, 7, 1)),     # one head, as a transposed [rows, heads, tokens, D] has it
    ((1, 3, 2, 64), (5, 128, 64, 1)),     # one row
    ((2, 1, 2, 64), (128, 3, 64, 1)),     # one token
])
def test_the_stride_of_one_element_does_not_matter(lib, size, stride):
    dense = torch.empty(size, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        _write(_strided(size, stride), dense, size[2])
    with pytest.raises(ValueError, match="CUDA"):
        _write(dense, _strided(size, stride), size[2])


def test_other_strides_are_refused_as_before(lib):
    with pytest.raises(ValueError, match="dense"):
        _write(_strided((2, 3, 2, 64), (384, 128, 72, 1)), torch.empty(2, 3, 2, 64, dtype=torch.bfloat16), 2)
    with pytest.raises(ValueError, match="dense"):
        _write(_strided((2, 3, 2, 64), (768, 256, 128, 2)), torch.empty(2, 3, 2, 64, dtype=torch.bfloat16), 2)
    with pytest.raises(ValueError, match="strides"):
        _write(_strided((2, 3, 2, 64), (512, 128, 64, 1)), torch.empty(2, 3, 2, 64, dtype=torch.bfloat16), 2)
