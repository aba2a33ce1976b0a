"""Calls that share a workspace at the same time, which the header forbids: their results
are unspecified, but nothing outside their outputs is written, and they end."""
import pytest

from test_gpu_tokens import native_mod

pytestmark = pytest.mark.gpu
GUARD = 4096  # rows before and behind each matrix


def test_two_chains_in_one_workspace(gpu):
    import torch

    native = native_mod()
    lib = native.load()
    n, d, b = 60_000, 520, 3

    def rows(fill=None):
        m = torch.randn(n + 2 * GUARD, d, device=gpu) if fill is None else \
            torch.full((n + 2 * GUARD, d), fill, device=gpu)
        return m.to(torch.bfloat16)

    def at(m):
        return m[GUARD:].data_ptr()

    x, g, dy = rows(), rows(), rows()
    starts = torch.tensor([0, 20_000, 20_001, n], dtype=torch.int32, device=gpu)
    marks = torch.zeros(-(-n // 64), d, device=gpu)
    ws = torch.empty(native.pdb_gated_scan_workspace_bytes(n, d), dtype=torch.uint8, device=gpu)
    outs = [rows(7.0) for _ in range(8)]
    states = [torch.full((b + 2, d), 7.0, device=gpu) for _ in range(4)]
    status = torch.zeros(1, dtype=torch.int32, device=gpu)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(4):
        stream = streams[k % 2].cuda_stream
        y, dg = outs[2 * k], outs[2 * k + 1]
        last = states[k][1:].data_ptr()
        if k < 2:
            rc = lib.pdb_gated_scan(at(x), d, at(g), d, native.PDB_BF16, n, d, starts.data_ptr(), b, None, at(y), d,
                                    last, None, status.data_ptr(), ws.data_ptr(), ws.numel(), stream)
        else:
            rc = lib.pdb_gated_scan_grad(at(dy), d, at(x), d, at(g), d, native.PDB_BF16, n, d, starts.data_ptr(), b,
                                         None, marks.data_ptr(), None, at(y), d, at(dg), d, last, status.data_ptr(),
                                         ws.data_ptr(), ws.numel(), stream)
        assert rc == native.PDB_OK
    torch.cuda.synchronize()
    assert int(status) in (native.PDB_OK, native.PDB_ERR_DEVICE)
    for m in outs:
        assert bool((m[:GUARD] == 7).all()) and bool((m[GUARD + n:] == 7).all())
    for m in states:
        assert bool((m[0] == 7).all()) and bool((m[-1] == 7).all())
    # and by itself, in the same workspace, the call gives what it gives in its own
    want = native.pdb_gated_scan(x[GUARD:GUARD + n], g[GUARD:GUARD + n], starts=starts)
    f = native.pdb_gated_scan(x[GUARD:GUARD + n], g[GUARD:GUARD + n], starts=starts, ws=ws)
    assert torch.equal(f.y, want.y) and torch.equal(f.state, want.state)
