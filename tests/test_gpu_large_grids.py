"""Calls of more blocks than one launch takes (2^32 threads): the same results as the
calls on pieces of them, which fit."""
import pytest

from test_gpu_tokens import native_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory(gpu):
    """What a test took goes back to the device, not to the tests behind it."""
    import torch

    yield
    torch.cuda.empty_cache()


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


def test_scan_gradient_of_the_most_rows(gpu):
    """2^31 - 1 rows of a channel, in sequences that are also run by themselves."""
    import torch

    native = native_mod()
    n, length = 2 ** 31 - 1, 1 << 25
    gen = torch.Generator(device=gpu).manual_seed(1)
    x = torch.empty(n, 1, dtype=torch.bfloat16, device=gpu).normal_(generator=gen)
    starts = torch.cat([torch.arange(0, n, length), torch.tensor([n])]).to(torch.int32).to(gpu)
    status = torch.zeros(1, dtype=torch.int32, device=gpu)
    f = native.pdb_gated_scan(x, x, starts=starts, marks=True, status=status)
    r = native.pdb_gated_scan_grad(x, x, x, f.marks, starts=starts, status=status)
    assert int(status) == 0
    for i in (0, 1, 17, 62, 63):
        rows = slice(i * length, min((i + 1) * length, n))
        f1 = native.pdb_gated_scan(x[rows], x[rows], marks=True)
        r1 = native.pdb_gated_scan_grad(x[rows], x[rows], x[rows], f1.marks)
        assert torch.equal(f.y[rows], f1.y) and torch.equal(f.state[i], f1.state[0]), i
        assert torch.equal(r.dx[rows], r1.dx) and torch.equal(r.dgate[rows], r1.dgate), i


@pytest.mark.parametrize("n,d,spare", [(100_000_003, 17, 20), (1_431_700_001, 17, 130)])
def test_decoding_steps_of_many_vectors(gpu, n, d, spare):
    """More vectors of rows than threads of a launch; states of no interest."""
    import torch

    native = native_mod()
    if torch.cuda.mem_get_info(gpu)[0] < spare << 30:
        pytest.skip("needs %d GiB of device memory" % spare)
    x = torch.empty(n, d, dtype=torch.bfloat16, device=gpu).normal_()
    y = torch.full_like(x, 7.0)

    def step(a, b, out):
        rc = native.load().pdb_gated_scan(x[a:b].data_ptr(), d, x[a:b].data_ptr(), d, native.PDB_BF16, b - a, d,
                                          None, b - a, None, out.data_ptr(), d, None, None, None, None, 0,
                                          torch.cuda.current_stream().cuda_stream)
        assert rc == native.PDB_OK

    step(0, n, y)
    part = 1 << 22
    for a in (0, n // 3, n // 4 * 3, n - part):
        want = torch.empty(part, d, dtype=x.dtype, device=gpu)
        step(a, a + part, want)
        assert torch.equal(y[a:a + part], want), a


def test_rows_of_many_channels(gpu):
    """One tile of more strips than a launch has blocks."""
    import torch

    native = native_mod()
    n, d = 3, (1 << 25) + 1001
    x, g, dy = torch.randn(3, n, d, device=gpu)
    h0 = torch.randn(1, d, device=gpu)
    f = native.pdb_gated_scan(x, g, h0=h0, marks=True)
    r = native.pdb_gated_scan_grad(dy, x, g, f.marks, h0=h0)
    for at in (slice(0, 999), slice(12_345_600, 12_350_000), slice(d - 2000, d)):
        f1 = native.pdb_gated_scan(x[:, at], g[:, at], h0=h0[:, at].contiguous(), marks=True)
        r1 = native.pdb_gated_scan_grad(dy[:, at], x[:, at], g[:, at], f1.marks, h0=h0[:, at].contiguous())
        for a, b in ((f.y, f1.y), (f.state, f1.state), (f.marks, f1.marks), (r.dx, r1.dx), (r.dgate, r1.dgate),
                     (r.dh0, r1.dh0)):
            assert torch.equal(a[:, at], b), at
