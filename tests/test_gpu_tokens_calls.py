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


@pytest.mark.parametrize("n,v", [(3, 20011), (1000, 1500)])
def test_memory_freed_by_a_busy_stream(gpu, n, v):
    """The current stream has freed blocks of just the sizes that the call wants and has
    yet to read them: a call on another stream leaves them alone."""
    import torch

    native = native_mod()
    z = torch.randn(n, v, device=gpu)
    tok = torch.randint(0, v, (n,), device=gpu)
    ids = torch.randint(0, v, (n, 8), device=gpu, dtype=torch.int32)
    t, g = torch.randn(n, 8, device=gpu), torch.randn(n, device=gpu)
    w, dy = torch.randn(v, 24, device=gpu), torch.randn(n, 24, device=gpu)
    grad = torch.empty(v, 24, device=gpu)
    a = torch.randn(4096, 4096, device=gpu)
    sizes = [native.pdb_token_logprobs_workspace_bytes(n, v, 20), native.pdb_distill_workspace_bytes(n, v),
             native.pdb_embed_grad_workspace_bytes(n, v, 24), 4 * n, 8 * n, 80 * n, 96 * n, 4 * n * v]

    def calls(stream):
        f = native.pdb_token_logprobs(z, tok, top=20, stream=stream)
        d = native.pdb_token_logprobs_grad(z, tok, f.stats, g, f.entropy, g, stream=stream)
        loss, e = native.pdb_distill(z, ids, t, stream=stream)
        out = native.pdb_embed_lookup(w, tok, stream=stream)
        return [f.logp, f.entropy, f.top_id, f.top_logp, d, loss, e, out,
                native.pdb_embed_grad(dy, tok, grad, stream=stream)]

    want = [x.clone() for x in calls(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        blocks = [torch.full((s,), 7, dtype=torch.uint8, device=gpu) for s in sizes for _ in range(3)]
        torch.cuda.synchronize()
        for _ in range(8):  # some milliseconds of work ahead of the reading
            b = a @ a
        seen = [x.clone() for x in blocks]
        del blocks
        got = calls(side)
        side.synchronize()
        torch.cuda.synchronize()
        assert all(bool((x == 7).all()) for x in seen)
        for x, y in zip(got, want):
            assert torch.equal(x, y)
        del b, seen, got


def test_arguments_by_name(gpu):
    import torch

    native = native_mod()
    w, tok = torch.randn(30, 8, device=gpu), torch.randint(0, 30, (5,), device=gpu)
    z, g = torch.randn(5, 30, device=gpu), torch.randn(5, device=gpu)
    ids = tok[:, None].int().contiguous()
    x = native.pdb_embed_lookup(table=w, tokens=tok)
    assert torch.equal(x, w[tok])
    assert torch.equal(native.pdb_embed_grad(dy=x, tokens=tok, grad=torch.empty_like(w)),
                       native.pdb_embed_grad(x, tok, torch.empty_like(w)))
    f = native.pdb_token_logprobs(logits=z, tokens=tok)
    assert torch.equal(f.logp, native.pdb_token_logprobs(z, tok).logp)
    assert torch.equal(native.pdb_token_logprobs_grad(logits=z, tokens=tok, stats=f.stats, d_logp=g),
                       native.pdb_token_logprobs_grad(z, tok, f.stats, g))
    for a, b in zip(native.pdb_distill(logits=z, ids=ids, teacher=g[:, None]),
                    native.pdb_distill(z, ids, g[:, None])):
        assert torch.equal(a, b)
