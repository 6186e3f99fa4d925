"""Fp8Weight and the products of a pass on tensors as programs hold them: views with gaps between their rows, and what is refused."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2505_10951_amd import sgc
from paper_2505_10951_amd.harness import DraftPass, Fp8Weight

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _project(x, w, y):
    holder = types.SimpleNamespace(workspace=torch.empty(sgc.sgc_project_fp8_workspace(x.shape[0], w.n_features, w.d_model), dtype=torch.uint8, device=DEV))
    DraftPass.project(holder, x, w, y)
    torch.cuda.synchronize()


@pytest.mark.parametrize("rows,features,d", [(5, 77, 144), (130, 300, 512)])
def test_views_give_what_copies_give(rows, features, d):
    g = torch.Generator().manual_seed(rows)
    w = Fp8Weight((torch.randn((features, d), generator=g) * 0.1).bfloat16().to(DEV))
    wide = torch.randn((rows, d + 32), generator=g).bfloat16().to(DEV)
    x = wide[:, 16: 16 + d]
    out = torch.full((rows, features + 9), 7.0, device=DEV)
    _project(x, w, out[:, 4: 4 + features])
    plain = torch.empty((rows, features), device=DEV)
    _project(x.contiguous(), w, plain)
    assert torch.equal(out[:, 4: 4 + features], plain)
    assert (out[:, :4] == 7.0).all() and (out[:, 4 + features:] == 7.0).all()


def test_what_is_refused():
    with pytest.raises(ValueError):
        Fp8Weight(torch.zeros((64, 64), device=DEV).bfloat16().t()[:, ::2])
    w = Fp8Weight(torch.zeros((48, 64), device=DEV).bfloat16())
    x, y = torch.zeros((8, 64), device=DEV).bfloat16(), torch.zeros((8, 48), device=DEV)
    for a, b in ((x[:, :48], y), (x, y[:4]), (x, y[:, :40]), (torch.zeros((64, 8), device=DEV).t(), y), (x, torch.zeros((48, 8), device=DEV).t())):
        with pytest.raises(ValueError):
            _project(a, w, b)
