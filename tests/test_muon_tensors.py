"""Which tensors a step of the update takes for matrices of its sides (no GPU needed: their shapes are looked at first)."""
import pytest
import torch

from paper_2411_10003_amd import binding


def _step(monkeypatch, rows, cols, transposed, shapes, count=2, which="weights"):
    """Addresses and the call itself left out: what reaches the library is counted."""
    mu = binding.Muon(count=count, rows=rows, cols=cols, dtype="f32", transposed=transposed, alloc_workspace=False)
    mu.ws = torch.empty(1)
    made = []
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype, numel, name: 0x1000)
    monkeypatch.setattr(binding, "_stream", lambda: 0)

    class Library:
        def moe_muon_step(self, *a):
            made.append(a)
            return 0
    monkeypatch.setattr(mu, "lib", Library())
    right = [torch.empty(count, cols, rows, device="meta") if t else torch.empty(count, rows, cols, device="meta") for t in transposed]
    kinds = {n: right for n in ("grads", "momenta", "weights", "copies")}
    kinds[which] = [torch.empty(s, device="meta") for s in shapes]
    mu.step(kinds["grads"], kinds["momenta"], kinds["weights"], lr=0.1, copies=kinds["copies"])
    return len(made)


@pytest.mark.parametrize("which", ["grads", "momenta", "weights", "copies"])
@pytest.mark.parametrize("transposed,shapes", [
    ((False,), [(2, 96, 64)]),                             # W2 where W1 belongs
    ((True,), [(2, 64, 96)]),
    ((False, True, False), [(2, 64, 96), (2, 64, 96), (2, 96, 64)]),       # W1, W3, W2
    ((False,), [(192, 64)]),                               # the same, matrices end to end
    ((False,), [(2, 64, 100)]),                            # wider rows
])
def test_sides_the_other_way_round(monkeypatch, which, transposed, shapes):
    with pytest.raises(ValueError, match=rf"{which}\[\d\]: shape"):
        _step(monkeypatch, 64, 96, transposed, shapes, which=which)


@pytest.mark.parametrize("rows,cols,count,transposed,shape", [
    (64, 96, 2, False, (2, 64, 96)), (64, 96, 2, True, (2, 96, 64)),
    (64, 96, 2, False, (3, 64, 96)),                       # more matrices than the call takes
    (64, 96, 1, False, (64, 96)), (64, 96, 2, False, (128, 96)),           # one matrix; matrices end to end
    (64, 96, 2, False, (2, 64 * 96)), (64, 96, 2, False, (2 * 64 * 96,)), (64, 96, 2, False, (2 * 64 * 96 + 5,)),     # flat
    (64, 96, 2, False, (2, 64, 8, 12)), (64, 96, 2, False, (2, 1, 64, 96)),                # rows in pieces, sides of one
    (64, 96, 2, False, (2, 64, 96, 1)),
    (64, 64, 2, True, (2, 64, 64)), (1, 96, 2, False, (2, 96, 1)), (96, 1, 2, False, (2, 1, 96)),       # either way the same bytes
    (1, 1, 1, False, ()),
])
def test_shapes_that_are_the_matrices(monkeypatch, rows, cols, count, transposed, shape):
    assert _step(monkeypatch, rows, cols, (transposed,), [shape], count=count) == 1
