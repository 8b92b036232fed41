"""The norm's gradient written over dY or dS, in rows of several waves whose last piece is short: that piece is requested together with columns that
another wave stores.  A width just past a number of threads has the short piece with the first thread and the columns with the last.  Rows enough
that blocks walk several."""
import pytest
import torch

import gpu_util as G
from paper_2411_10003_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", d) for d in (131, 517, 1021, 2049, 2055, 4099, 6147, 8201, 12290, 16383)] +
                         [("f32", d) for d in (65, 259, 510, 1025, 1027, 2049, 4097, 6145, 8195, 16383)])
def test_gradient_over_its_inputs(dtype, d):
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    for rows in (1, 3, 1500):
        g = torch.Generator(device=G.DEV).manual_seed(rows + d)
        randn = lambda *s: torch.randn(*s, generator=g, device=G.DEV)  # noqa: E731
        S, dY, dS, gamma = randn(rows, d).to(t), randn(rows, d).to(t), randn(rows, d).to(t), 1.0 + 0.3 * randn(d)
        n = binding.Norm(d=d, dtype=dtype, device=G.DEV)
        mean, rstd = torch.empty(rows, device=G.DEV), torch.empty(rows, device=G.DEV)
        n.fwd(S, gamma, None, torch.empty_like(S), mean=mean, rstd=rstd)
        for residual in (True, False):
            dX, dg, db = torch.empty_like(S), torch.empty(d, device=G.DEV), torch.empty(d, device=G.DEV)
            n.bwd(dY, S, gamma, mean, rstd, dX, dg, db, residual_grad=dS if residual else None)
            for over in ("dY", "dS")[:1 + residual]:
                a = dict(dY=dY.clone(), dS=dS.clone() if residual else None)
                dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
                n.bwd(a["dY"], S, gamma, mean, rstd, a[over], dg2, db2, residual_grad=a["dS"])
                assert torch.equal(a[over], dX) and torch.equal(dg2, dg) and torch.equal(db2, db), (rows, over)
