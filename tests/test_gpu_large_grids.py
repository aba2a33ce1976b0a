"""Calls of more blocks than one launch takes (2^32 threads): the same results as the
calls on pieces of them, which fit."""
import pytest

from test_gpu_tokens import native_mod

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,k,v", [((1 << 24) + 1234, 0, 5), ((1 << 22) + 17, 3, 4)])
def test_verification_of_many_sequences(gpu, b, k, v):
    import torch

    native = native_mod()
    gen = torch.Generator(device=gpu).manual_seed(b)
    t = torch.randn(b * (k + 1), v, generator=gen, device=gpu).to(torch.bfloat16)
    u = torch.rand(b, k + 1, generator=gen, device=gpu)
    q = torch.randn(b * k, v, generator=gen, device=gpu).to(torch.bfloat16) if k else None
    x = torch.randint(-1, v, (b, k), generator=gen, device=gpu, dtype=torch.int32) if k else None
    x_out = torch.tensor([b - 3], device=gpu)
    if k:
        x[x_out, 0] = v      # behind the first launch: noted there, too
    status = torch.zeros(1, dtype=torch.int32, device=gpu)
    got = native.pdb_draft_verify(t, u, tokens=x, draft=q, status=status)
    assert int(status) == (native.PDB_ERR_INVALID_ARG if k else native.PDB_OK)
    step = 1 << 21
    for i in range(0, b, step):
        j = min(i + step, b)
        part = native.pdb_draft_verify(t[i * (k + 1):j * (k + 1)], u[i:j], tokens=x[i:j] if k else None,
                                       draft=q[i * k:j * k] if k else None)
        assert torch.equal(got.tokens[i:j], part.tokens) and torch.equal(got.accepted[i:j], part.accepted), i
