"""What a call object of the binding holds an address of lives as long as the call does, also where the object that made it has let go of it (no GPU
needed: calls of no rows)."""
import gc
import weakref

import pytest
import torch

from paper_2411_10003_amd import binding


@pytest.mark.parametrize("kind", ["native", "python"])
def test_sizes_of_a_norm_outlive_its_memory_of_row_counts(monkeypatch, kind):
    """A thread may hold a call, or be inside one, while another brings more row counts than the object keeps."""
    if kind == "python":
        monkeypatch.setattr(binding, "_call_class", binding.PythonCall)
    made = []

    class Norm(binding._Norm):
        def __init__(self, *a):
            super().__init__(*a)
            made.append(weakref.ref(self))
    n = binding.Norm(d=64, dtype="f32", alloc_workspace=False)
    monkeypatch.setattr(binding, "_Norm", Norm)
    rows = lambda r: torch.empty(r, 64, device="meta")  # noqa: E731
    call = n._for_rows(rows(0))[0]
    sizes, = made
    assert call(*[None] * 8, 0) == 0
    for r in range(1, 2 * n.MAX_CALLS):
        n._for_rows(rows(r))
    gc.collect()
    assert sizes() is not None and sizes().rows == 0
    assert call(*[None] * 8, 0) == 0
    # and no longer than that
    del call
    gc.collect()
    assert sizes() is None
