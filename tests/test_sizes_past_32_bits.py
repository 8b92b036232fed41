"""Sizes of the norm and of the update that do not fit the 32 bits their structures have are refused, not wrapped (no GPU needed)."""
import pytest
import torch

from paper_2411_10003_amd import binding


@pytest.mark.parametrize("rows", [2 ** 30, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 33])
def test_rows_of_a_norm(rows):
    """Wrapped, 2^32 + 5 rows are five: the call would leave the others as they are and report success."""
    n = binding.Norm(d=1, dtype="bf16", alloc_workspace=False)
    X = torch.empty(rows, 1, dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match=f"{rows} rows"):
        n._for_rows(X)
    assert n._calls == {}
    n._for_rows(X[:2 ** 30 - 1])                           # the most there may be


@pytest.mark.parametrize("d", [2 ** 32 + 64, -2 ** 32 + 64, 2 ** 31])
def test_width_of_a_norm(d):
    with pytest.raises((ValueError, binding.MoeError)):
        binding.Norm(d=d, dtype="bf16", alloc_workspace=False)


@pytest.mark.parametrize("name", ["count", "rows", "cols", "steps"])
@pytest.mark.parametrize("off", [2 ** 32, -2 ** 32, 2 ** 31])
def test_sizes_of_an_update(name, off):
    sizes = dict(count=2, rows=4, cols=4, steps=5)
    sizes[name] += off
    with pytest.raises((ValueError, binding.MoeError)):
        binding.Muon(**sizes, dtype="bf16", alloc_workspace=False)
