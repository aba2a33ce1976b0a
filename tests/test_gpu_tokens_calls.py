"""What a call of the token operators answers and refuses whatever its sizes."""
import numpy as np
import pytest

from test_gpu_tokens import native_mod, torch_type

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,v", [(3, 40), (3, 20011), (1500, 300), (300, 20001), (300, 140003)])
def test_ids_of_a_row_of_weight_0(gpu, n, v, dtype):
    """They may hold anything, however the rows are split: one out of range is no
    error there, and one elsewhere is."""
    import torch

    native = native_mod()
    z = torch.randn(n, v, device=gpu).to(torch_type(dtype))
    ids = torch.randint(0, v, (n, 5), device=gpu, dtype=torch.int32)
    t = torch.randn(n, 5, device=gpu)
    w = torch.ones(n, device=gpu)
    off = torch.arange(n, device=gpu) % 3 == 1
    w[off] = 0.0
    ids[off, 2] = v
    status = torch.zeros(1, dtype=torch.int32, device=gpu)
    for grad in (True, False):
        loss, d = native.pdb_distill(z, ids, t, weight=w, grad=grad, status=status)
        assert int(status) == native.PDB_OK
        assert not loss[off].any() and bool((loss[~off] != 0).all())
        assert not grad or (not d[off].any() and bool(d[~off].any(dim=1).all()))
    ids[n - 1 if (n - 1) % 3 != 1 else 0, 4] = v
    for grad in (True, False):
        status.zero_()
        native.pdb_distill(z, ids, t, weight=w, grad=grad, status=status)
        assert int(status) == native.PDB_ERR_INVALID_ARG
