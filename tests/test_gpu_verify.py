"""The verification of drafted tokens on the GPU against the 64-bit form of layerref:
the same tokens, at every size, type and mask."""
import numpy as np
import pytest

import layerref as ref
from test_gpu_tokens import DTYPES, f64, native_mod, on_gpu

pytestmark = pytest.mark.gpu
NINF = -np.inf


def draw_case(gpu, rng, b, k, v, dtype, pad=0, shift=0, apart=0.5, spread=3.0):
    import torch

    t, t64 = on_gpu(rng.normal(size=(b * (k + 1), v)) * spread, dtype, gpu, pad, shift)
    t64 = t64.reshape(b, k + 1, v)
    q, q64 = on_gpu((t64[:, :k] + apart * rng.normal(size=(b, k, v))).reshape(b * k, v), dtype, gpu, pad, shift)
    q64 = q64.reshape(b, k, v)
    x = np.zeros((b, k), np.int64)
    for i in range(b):
        for j in range(k):
            x[i, j] = ref.draw(ref.softmax(q64[i, j], 1.0), rng.random())
    u = torch.from_numpy(rng.random((b, k + 1)).astype(np.float32)).to(gpu)
    return t, t64, q, q64, x, u


def same(gpu, t, t64, q, q64, x, u, temp=1.0, index=None):
    import torch

    native = native_mod()
    b, k = x.shape
    tok = torch.from_numpy(x).to(gpu, index or torch.int32) if k else None
    status = torch.zeros(1, dtype=torch.int32, device=gpu)
    r = native.pdb_draft_verify(t, u, tokens=tok, draft=q if k else None, temp=temp, status=status)
    out, acc = ref.verify(t64, q64 if q is not None else None, x, f64(u), temp)
    assert np.array_equal(r.tokens.cpu().numpy(), out)
    assert np.array_equal(r.accepted.cpu().numpy(), acc)
    return r, int(status)


SIZES = [(1, 0, 1), (1, 1, 1), (3, 2, 2), (1, 0, 131_072), (4, 3, 100), (70, 1, 333), (5, 8, 4096), (2, 4, 4097),
         (33, 0, 8191), (9, 5, 20_011), (300, 2, 50), (2, 64, 30), (1, 3, 200_003)]


@pytest.mark.parametrize("b,k,v", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("model", [True, False])
def test_verify(gpu, b, k, v, dtype, model):
    import torch

    rng = np.random.default_rng(b + k + v)
    pad, shift = (0, 0) if v % 2 == 0 else (3, 1)
    t, t64, q, q64, x, u = draw_case(gpu, rng, b, k, v, dtype, pad, shift)
    for temp in (1.0, 0.7, 2.0):
        r, status = same(gpu, t, t64, q if model else None, q64, x, u, temp,
                         torch.int64 if k % 2 else torch.int32)
        assert status == 0
    if model and k and b * k > 20 and v > 40:
        assert 0 < int(r.accepted.sum()) < b * k     # both answers occur


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("b,k,v", [(40, 3, 500), (12, 5, 9001)])
def test_masks_and_ragged_drafts(gpu, b, k, v, dtype):
    import torch

    rng = np.random.default_rng(v)
    t, _, q, _, x, u = draw_case(gpu, rng, b, k, v, dtype)
    t[:, ::3] = NINF
    q[::2, 1::5] = NINF
    t[5] = NINF
    q[3] = NINF
    lowest = torch.finfo(t.dtype).min
    t[7, : v // 2] = lowest
    q[7, v // 3:] = lowest
    t[9] = lowest
    x[rng.random((b, k)) < 0.2] = -3
    x[4] = -1
    same(gpu, t, f64(t).reshape(b, k + 1, v), q, f64(q).reshape(b, k, v), x, u)
    same(gpu, t, f64(t).reshape(b, k + 1, v), None, None, x, u)


def test_the_same_distribution_accepts_all(gpu):
    rng = np.random.default_rng(0)
    b, k, v = 30, 4, 5000
    t, t64, q, q64, x, u = draw_case(gpu, rng, b, k, v, "bf16", apart=0.0)
    r, _ = same(gpu, t, t64, q, q64, x, u)
    assert bool((r.accepted == k).all())


def test_numbers_at_their_ends(gpu):
    """u = 0: the first entry of weight > 0, and accepted wherever p > 0; u = 1 (never
    given, but no fault): the last one."""
    import torch

    rng = np.random.default_rng(3)
    for v in (7, 4096, 9000):
        b, k = 6, 2
        t, t64, q, q64, x, u = draw_case(gpu, rng, b, k, v, "f32")
        t[:, 0] = t[:, -1] = NINF
        t64 = f64(t).reshape(b, k + 1, v)
        r, _ = same(gpu, t, t64, q, q64, x, torch.zeros_like(u))
        r0 = r.tokens[torch.arange(b), r.accepted.long()]
        assert bool((r0 >= 1).all())
        native = native_mod()
        one = native.pdb_draft_verify(t, torch.ones(b * (k + 1), 1, device=gpu))
        assert bool((one.tokens == v - 2).all())


def test_ids_out_of_range(gpu):
    import torch

    rng = np.random.default_rng(4)
    t, t64, q, q64, x, u = draw_case(gpu, rng, 8, 4, 300, "f16")
    x[2, 0] = 300
    x[5, 1] = -1
    x[5, 2] = 2 ** 40          # behind the end: not looked at
    _, status = same(gpu, t, t64, q, q64, x, u, index=torch.int64)
    assert status == native_mod().PDB_ERR_INVALID_ARG
    x[2, 0] = -1
    _, status = same(gpu, t, t64, q, q64, x, u, index=torch.int64)
    assert status == 0


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_rows_without_a_distribution(gpu, bad):
    rng = np.random.default_rng(5)
    b, k, v = 6, 2, 700
    t, t64, q, q64, x, u = draw_case(gpu, rng, b, k, v, "f32")
    u.mul_(0.01)               # whatever can be accepted is
    t[0 * 3 + 0, 99] = bad     # sequence 0: its first row
    t[1 * 3 + 2, 5] = bad      # sequence 1: the row behind its draft
    q[2 * 2 + 1, 7] = bad      # sequence 2: the draft's second row
    r = native_mod().pdb_draft_verify(t, u, tokens=__import__("torch").from_numpy(x).to(gpu), draft=q)
    out, acc = r.tokens.cpu().numpy(), r.accepted.cpu().numpy()
    assert acc.tolist() == [0, 2, 1, 2, 2, 2]
    assert out[0].tolist() == [-1, -1, -1] and out[1, 2] == -1
    assert out[2, 1] == ref.draw(ref.softmax(t64[2, 1], 1.0), float(u[2, 2])) and out[2, 2] == -1


def test_drawn_tokens_follow_the_distribution(gpu):
    import torch

    native = native_mod()
    v, n = 50, 200_000
    z = torch.randn(1, v, device=gpu)
    g = torch.Generator(device=gpu).manual_seed(1)
    r = native.pdb_draft_verify(z.expand(n, v).contiguous(), torch.rand(n, 1, generator=g, device=gpu))
    got = torch.bincount(r.tokens[:, 0], minlength=v).double() / n
    assert float((got - torch.softmax(z[0].double(), 0)).abs().max()) < 5 * (0.25 / n) ** 0.5


@pytest.mark.parametrize("temp", [1.0, 0.7])
def test_near_borders(gpu, temp):
    """Random numbers a part in 1e7 to either side of a border of the running sum, and a
    vocabulary in which many borders lie as near to a number as a temperature of 32 bits
    would move them."""
    import torch

    rng = np.random.default_rng(6)
    n, v = 4000, 131_072
    row, row64 = on_gpu(rng.normal(size=(1, v)), "f16", gpu)
    run = np.cumsum(ref.softmax(row64[0], temp))
    u = rng.random(n).astype(np.float32)
    got = native_mod().pdb_draft_verify(row.expand(n, v).contiguous(), torch.from_numpy(u[:, None]).to(gpu), temp=temp)
    assert np.array_equal(got.tokens[:, 0].cpu().numpy(),
                          np.searchsorted(run, u.astype(np.float64) * run[-1], side="right"))
    v, n = 4500, 400
    z = np.repeat(rng.normal(size=(1, v)).astype(np.float32), n, 0)
    t, t64 = on_gpu(z, "f32", gpu)
    run = np.cumsum(ref.softmax(t64[0], temp))
    at = np.sort(rng.choice(v, n // 2, replace=False))
    edge = run[at].astype(np.float32)
    u = np.concatenate([np.nextafter(edge, np.float32(0)), np.nextafter(edge, np.float32(1))])
    u = np.minimum(u, np.float32(1 - 2 ** -24))
    same(gpu, t, t64.reshape(n, 1, v), None, None, np.zeros((n, 0), np.int64),
         torch.from_numpy(u[:, None]).to(gpu), temp)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("model", [True, False])
def test_near_the_bar(gpu, dtype, model):
    """Random numbers next to p / q, where 32-bit sums cannot tell: at every position of
    a draft, those before it accepted."""
    import torch

    rng = np.random.default_rng(7)
    b, k, v = 60, 4, 3001
    t, t64, q, q64, x, u = draw_case(gpu, rng, b, k, v, dtype)
    un = np.full((b, k + 1), 0.0, np.float32)
    un[:, k] = rng.random(b)
    for i in range(b):
        j = i % k
        p = ref.softmax(t64[i, j], 1.0)
        w = ref.softmax(q64[i, j], 1.0) if model else np.ones(v)
        x[i, j] = np.nonzero((p < w) & (p > 0))[0][i % 5]
        bar = np.float32(p[x[i, j]] / w[x[i, j]])
        un[i, j] = (bar, np.nextafter(bar, np.float32(0)), np.nextafter(bar, np.float32(1)))[i % 3]
    r, _ = same(gpu, t, t64, q if model else None, q64, x, torch.from_numpy(un).to(gpu))
    at = np.arange(b) % k
    stopped = r.accepted.cpu().numpy() == at
    assert stopped.any() and not stopped.all()   # both sides of the bar


def test_residual_of_nearly_equal_rows(gpu):
    """The draft has the target's logits but for the token that it proposes: what is left
    of every other entry is a part in 1e5 of it, and its sign hangs on the exact sums."""
    import torch

    rng = np.random.default_rng(8)
    b, k, v = 24, 1, 20_011
    t, t64 = on_gpu(rng.normal(size=(b * 2, v)), "f32", gpu)
    t64 = t64.reshape(b, 2, v)
    q = t.view(b, 2, v)[:, 0].clone()
    x = rng.integers(0, v, (b, 1))
    for i in range(b):
        p = ref.softmax(t64[i, 0], 1.0)
        x[i, 0] = np.argmin(np.abs(p - 1e-5))
        q[i, x[i, 0]] += 0.7
    u = torch.from_numpy(rng.random((b, 2)).astype(np.float32)).to(gpu)
    u[:, 0] = 0.9
    r, _ = same(gpu, t, t64, q, f64(q).reshape(b, 1, v), x, u)
    assert not r.accepted.any()


def test_captured_and_replayed(gpu):
    """Recorded into a graph, replayed on other inputs, with eager work between."""
    import torch

    native = native_mod()
    rng = np.random.default_rng(9)
    cases = [draw_case(gpu, rng, 6, 3, 9001, "bf16") for _ in range(3)]
    t, _, q, _, x, u = (c.clone() if hasattr(c, "clone") else c for c in cases[0])
    tok = torch.from_numpy(x).to(gpu)
    native.pdb_draft_verify(t, u, tokens=tok, draft=q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = native.pdb_draft_verify(t, u, tokens=tok, draft=q)
        one = native.pdb_draft_verify(t, u.view(-1, 1))
    for c in cases + cases:
        t.copy_(c[0])
        q.copy_(c[2])
        tok.copy_(torch.from_numpy(c[4]))
        u.copy_(c[5])
        graph.replay()
        torch.cuda.synchronize()
        out, acc = ref.verify(c[1], c[3], c[4], f64(c[5]), 1.0)
        assert np.array_equal(r.tokens.cpu().numpy(), out) and np.array_equal(r.accepted.cpu().numpy(), acc)
        eager = native.pdb_draft_verify(t, u.view(-1, 1))
        assert torch.equal(one.tokens, eager.tokens)


@pytest.mark.parametrize("dtype,v", [("f32", 300_000), ("bf16", 700_001)])
def test_rising_rows(gpu, dtype, v):
    """Logits that rise along the row, so that the maximum is raised all the way: sums
    next to the bar."""
    import torch

    rng = np.random.default_rng(10)
    b, k = 3, 2
    z = np.sort(rng.normal(size=(b * (k + 1), v)) * 2, axis=1)
    t, t64 = on_gpu(z, dtype, gpu)
    q, q64 = on_gpu(z[: b * k] * 0.9, dtype, gpu)
    t64, q64 = t64.reshape(b, k + 1, v), q64.reshape(b, k, v)
    x = np.zeros((b, k), np.int64)
    u = rng.random((b, k + 1)).astype(np.float32)
    for i in range(b):
        p, w = ref.softmax(t64[i, 0], 1.0), ref.softmax(q64[i, 0], 1.0)
        x[i, 0] = np.nonzero(p < w)[0][-1 - i]
        x[i, 1] = v - 1 - i
        u[i, 0] = np.nextafter(np.float32(p[x[i, 0]] / w[x[i, 0]]), np.float32(i % 2))
    same(gpu, t, t64, q, q64, x, torch.from_numpy(u).to(gpu))
    same(gpu, t, t64, None, None, x, torch.from_numpy(u).to(gpu))
    u[:, 0] = 0.99
    same(gpu, t, t64, None, None, x, torch.from_numpy(u).to(gpu))
