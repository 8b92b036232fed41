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


def test_a_step_of_the_update_has_its_own_rates(monkeypatch):
    """The library reads a step's constants without the interpreter's lock: a step that begins meanwhile with other rates leaves them alone."""
    mu = binding.Muon(count=1, rows=8, cols=8, dtype="f32", alloc_workspace=False)
    mu.ws = torch.empty(1)
    monkeypatch.setattr(binding, "_ptr", lambda *a: 0x1000)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    seen, one = [], [torch.empty(1, 8, 8, device="meta")]

    class Library:
        def moe_muon_step(self, cfg, *rest):
            c = cfg._obj
            before = (c.lr, c.weight_decay, c.scale)
            if not seen:
                seen.append(None)
                mu.step(one, one, one, lr=0.5, weight_decay=0.25, scale=4.0)           # another thread's
            seen.append((before, (c.lr, c.weight_decay, c.scale), (c.rows, c.cols, c.steps, c.momentum)))
            return 0
    monkeypatch.setattr(mu, "lib", Library())
    mu.step(one, one, one, lr=0.125)
    constants = (8, 8, 5, seen[1][2][3])
    assert seen[1:] == [((0.5, 0.25, 4.0), (0.5, 0.25, 4.0), constants), ((0.125, 0.0, 1.0), (0.125, 0.0, 1.0), constants)]
