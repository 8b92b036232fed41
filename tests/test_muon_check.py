"""That the check of the update's weights notices what a wrong epilogue would do: it passes the definition rounded once, and none of the mistakes (no
GPU: they are planted in the oracle)."""
import pytest
import torch

import muon_util as U

RATES = dict(lr=0.5, wd=0.5, scale=2.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(192, 320), (320, 576), (333, 517), (517, 333), (640, 385), (8, 8), (63, 200)])
def test_mistakes_are_noticed(rows, cols, dtype):
    g = torch.Generator().manual_seed(rows + cols)
    x = U.orthogonalised(U.gradient(g, 2, rows, cols, "cpu"))
    W0 = U.weights_like(x, g, dtype, lr=RATES["lr"], scale=RATES["scale"])

    def new(x=x, wd=RATES["wd"], rate=1.0):
        return ((1.0 - RATES["lr"] * wd) * W0.double() - rate * RATES["lr"] * RATES["scale"] * x).to(U.TYPES[dtype])
    right = new()
    U.check(dtype, x, W0, right, **RATES)

    def old(where):
        w = right.clone()
        w[where] = W0[where]
        return w
    last = slice(-1, None)
    wrong = {
        "last column left": old((0, slice(None), last)), "last row left": old((1, last, slice(None))), "first column left": old((1, slice(None), slice(0, 1))),
        "a corner left": old((0, last, last)), "one element left": old((1, rows // 2, cols // 2)),
        "no decay": new(wd=0.0), "update 5 % too large": new(rate=1.05), "update 5 % too small": new(rate=0.95), "no update": new(rate=0.0),
        "matrices exchanged": new(x=x.flip(0)), "columns moved by one": new(x=x.roll(1, 2)), "rows moved by one": new(x=x.roll(1, 1)),
    }
    for name, w in wrong.items():
        # an element may be within the tolerance by chance: then nothing is wrong with it
        if name in ("a corner left", "one element left"):
            i = (0, -1, -1) if name == "a corner left" else (1, rows // 2, cols // 2)
            if abs(float(W0[i]) - float(right[i])) < 0.2 * RATES["lr"] * RATES["scale"] * float(x.square().mean().sqrt()):
                continue
        with pytest.raises(AssertionError):
            U.check(dtype, x, W0, w, **RATES)
            print(name)
