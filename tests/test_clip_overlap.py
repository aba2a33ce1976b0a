"""Outputs of the clipping that share memory: with their own gradient they may, all of it,
and with nothing else that the call reads or writes."""
import ctypes

import pytest

from test_layers_host import native  # noqa: F401  (the fixture)
from test_tokens_host import P

F32, F16, BF16 = 0, 1, 2
AT = 0x100000   # never dereferenced: these calls are refused


def tensors(*ts):
    """pdb_tensor of (address, rows, columns, stride, type)."""
    flat = [v for t in ts for v in t]
    return ctypes.cast((ctypes.c_int64 * len(flat))(*flat), ctypes.c_void_p)


def clip(native, grads, outs, accumulate=0):  # noqa: F811
    need = native.pdb_grad_workspace_bytes()
    return native.load().pdb_grad_clip(tensors(*grads), len(grads), 1.0, 1.0, 1.0, accumulate, tensors(*outs), P, P,
                                       need, None)


def vec(at, n, dtype=F32):
    return (at, 1, n, n, dtype)


REFUSED = {
    "another's gradient": ([vec(AT, 8), vec(AT + 64, 8)], [vec(AT + 64, 8), vec(AT, 8)]),
    "another's gradient, in place": ([vec(AT, 8), vec(AT, 8)], [vec(AT, 8), vec(AT + 64, 8)]),
    "another output": ([vec(AT, 8), vec(AT + 64, 8)], [vec(AT + 256, 8), vec(AT + 256, 8)]),
    "another output, in part": ([vec(AT, 8), vec(AT + 64, 8)], [vec(AT + 256, 8), vec(AT + 284, 8)]),
    "another output, inside it": ([vec(AT, 80), vec(AT + 400, 2)], [vec(AT + 4096, 80), vec(AT + 4200, 2)]),
    "its own gradient in part": ([vec(AT, 8)], [vec(AT + 4, 8)]),
    "its own gradient from behind": ([vec(AT + 4, 8)], [vec(AT, 8)]),
    "another's gradient in part": ([vec(AT, 8), vec(AT + 64, 8)], [vec(AT + 256, 8), vec(AT + 20, 8)]),
    "in place twice": ([vec(AT, 8), vec(AT, 8)], [vec(AT, 8), vec(AT, 8)]),
    "wider elements": ([vec(AT, 8, BF16), vec(AT + 16, 8, BF16)], [vec(AT + 256, 8), vec(AT + 256 + 28, 8)]),
    "rows further apart": ([(AT, 4, 5, 9, F32), vec(AT + 4096, 3)], [(AT + 512, 4, 5, 9, F32), vec(AT + 516, 3)]),
    "rows without gaps": ([(AT, 4, 5, 5, F32), vec(AT + 4096, 3)], [(AT + 512, 4, 5, 5, F32), vec(AT + 580, 3)]),
    "the last of many": ([vec(AT + 64 * i, 8) for i in range(700)],
                         [vec(AT + 64 * (i if i < 699 else 0), 8) for i in range(700)]),
}


@pytest.mark.parametrize("what", list(REFUSED))
@pytest.mark.parametrize("accumulate", [0, 1])
def test_refused(native, what, accumulate):  # noqa: F811
    grads, outs = REFUSED[what]
    assert clip(native, grads, outs, accumulate) == native.PDB_ERR_INVALID_ARG


@pytest.mark.gpu
def test_refused_by_the_binding(gpu):
    import torch

    from paper_1508_00703_amd import native as nat

    a, b = torch.randn(2, 100, device=gpu)
    before = a.clone(), b.clone()
    with pytest.raises((ValueError, nat.PdbError)):
        nat.pdb_grad_clip([a, b], 1.0, out=[b, a])
    with pytest.raises((ValueError, nat.PdbError)):
        nat.pdb_grad_clip([a[:50]], 1.0, out=[a[25:75]], accumulate=True)
    assert torch.equal(a, before[0]) and torch.equal(b, before[1])


@pytest.mark.gpu
def test_taken(gpu):
    """Neighbours, columns of one buffer, a gradient read twice, tensors of no elements."""
    import torch

    from paper_1508_00703_amd import native as nat

    def check(grads, out, **kw):
        want = [0.25 * g.double() + (o.double() if kw.get("accumulate") else 0) for g, o in zip(grads, out)]
        nat.pdb_grad_clip(grads, float("inf"), scale=0.25, out=out, **kw)
        for w, o in zip(want, out):
            torch.testing.assert_close(o.double(), w, rtol=2 ** -23, atol=2.0 ** -24 * float(w.abs().max() if w.numel() else 0))

    buf, other = torch.randn(2, 4000, device=gpu)
    parts = [buf[i:i + 100] for i in range(0, 4000, 100)]
    check(parts, [other[i:i + 100] for i in range(0, 4000, 100)], accumulate=True)
    check(parts, parts)                                             # in place, one behind another
    check(parts, parts, accumulate=True)
    wide = torch.randn(50, 60, device=gpu)
    columns = [wide[:, i:i + 12] for i in range(0, 60, 12)]
    check(columns, columns)                                         # in place, side by side
    check([w.contiguous() for w in columns], columns, accumulate=True)
    check([buf[:100], buf[:100]], [other[:100], other[100:200]])    # read twice
    check([buf[:100], buf[:0], buf[50:50]], [buf[:100], buf[:0], buf[:0]])
    half = buf[:200].to(torch.bfloat16)
    check([half[:100], half[100:]], [other[:100], other[100:200]])
