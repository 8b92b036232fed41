"""The workspace of an update is as large as its sizes need (no GPU needed), and nothing is written past it."""
import pytest
import torch

import muon_util as U
from paper_2411_10003_amd import binding


def _bytes(rows, cols, dtype, count=1, tensors=1):
    return binding.Muon(count=count, rows=rows, cols=cols, dtype=dtype, transposed=(False,) * tensors, alloc_workspace=False).workspace_bytes


@pytest.mark.parametrize("rows,cols,dtype,count,tensors", [(8, 8, "f32", 1, 1), (8, 8, "bf16", 1, 1), (64, 256, "f32", 2, 2), (128, 192, "bf16", 4, 3), (65, 129, "f32", 1, 1),
                                                            (192, 320, "bf16", 1, 1), (200, 300, "f32", 2, 1)])
def test_small_matrices_need_little(rows, cols, dtype, count, tensors):
    """The iterates (two X, four A, padded to multiples of 64), and for the parts of cut tiles no more than eight of each tile: 1 MB and less beside the
    iterates for a handful of 64 x 64 tiles, 2 MB for a 256 x 256 one that a long contraction may cut."""
    m, n = (-(-v // 64) * 64 for v in sorted((rows, cols)))
    iterates = count * tensors * (2 * m * n + 4 * m * m) * 2 * (2 if dtype == "f32" else 1)
    got = _bytes(rows, cols, dtype, count, tensors)
    tiles = count * tensors * -(-m // 256) * -(-n // 256)
    assert iterates <= got <= iterates + 2 ** 16 + tiles * 8 * 256 * 256 * 4
    if m <= 64:
        assert got <= iterates + 2 ** 16                   # a block takes a matrix: no tiles at all


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,count,transposed,dtype", [
    (1024, 1088, 20, (False,), "bf16"), (1100, 1500, 10, (True,), "f32"), (576, 4032, 3, (False, True), "bf16"), (320, 3840, 2, (True,), "f32"), (640, 704, 40, (False,), "bf16"),
    (512, 16384, 1, (False,), "bf16"), (200, 300, 2, (False,), "f32"), (65, 4000, 1, (True,), "f32"), (100, 9000, 1, (False,), "bf16"), (64, 4096, 1, (False,), "f32"),
    (64, 256, 2, (False, True), "f32"), (100, 70, 2, (False,), "bf16")])
def test_nothing_is_written_past_it(rows, cols, count, transposed, dtype):
    dev = "cuda:0"
    g = torch.Generator(device=dev).manual_seed(rows + cols)
    shapes = [(count, cols, rows) if t else (count, rows, cols) for t in transposed]
    grads = [U.gradient(g, *s, dev) for s in shapes]
    momenta, weights = [torch.zeros_like(x) for x in grads], [torch.zeros_like(x, dtype=U.TYPES[dtype]) for x in grads]
    mu = binding.Muon(count=count, rows=rows, cols=cols, dtype=dtype, transposed=transposed, device=dev, alloc_workspace=False)
    guard = 4 << 20
    held = torch.full((mu.workspace_bytes + 2 * guard,), 0xa5, dtype=torch.uint8, device=dev)
    mu.ws = held[guard:guard + mu.workspace_bytes]
    assert mu.ws.data_ptr() % 256 == 0
    mu.step(grads, momenta, weights, lr=0.5, scale=2.0)
    assert (held[:guard] == 0xa5).all() and (held[guard + mu.workspace_bytes:] == 0xa5).all()
    for x, w in zip(grads, weights):
        U.check(dtype, U.orthogonalised(U.direction(x, torch.zeros_like(x))[1]), torch.zeros_like(w), w, lr=0.5, wd=0.0, scale=2.0)
