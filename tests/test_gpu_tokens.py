"""The token operators on the GPU against the 64-bit forms of tokenref, whose
bounds hold for every case here: sizes from one up, odd ones, ragged strides,
every type, masks that leave a row little or nothing, special values, ties."""
import numpy as np
import pytest

import tokenref as ref

pytestmark = pytest.mark.gpu

DTYPES = ["f32", "f16", "bf16"]
NINF = -np.inf


def native_mod():
    from paper_1508_00703_amd import native
    return native


def torch_type(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def on_gpu(x, dtype, dev, pad=0, shift=0):
    """x (2-D) on the GPU in dtype, its rows pad elements further apart and its
    first element shift elements behind an allocation's start; and the values it
    then holds, in 64 bits."""
    import torch

    t = torch_type(dtype)
    n, v = x.shape
    buf = torch.full((n * (v + pad) + shift + 8,), 7.0, dtype=t, device=dev)
    m = buf[shift:shift + n * (v + pad)].view(n, v + pad)[:, :v]
    m.copy_(torch.from_numpy(np.ascontiguousarray(x)).to(t))
    return m, m.double().cpu().numpy()


def f64(t):
    return t.double().cpu().numpy()


def check(got, want, bound, what):
    """Equal where the expected value is infinite or NaN, within bound elsewhere."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    fin = np.isfinite(want)
    over = (np.abs(got - want) - bound)[fin]
    assert over.size == 0 or over.max() <= 0, (what, over.max(), np.argmax(over))


# ---------------------------------------------------------------------------
# embedding

def draw_tokens(rng, n, v, how):
    if how == "one":
        t = np.full(n, v // 2)
    elif how == "zipf":
        p = np.arange(1, v + 1) ** -1.1
        t = rng.choice(v, n, p=p / p.sum())
    elif how == "holes":
        t = np.where(rng.random(n) < 0.3, -1 - rng.integers(0, 3, n), rng.integers(0, v, n))
    elif how == "none":
        t = np.full(n, -1)
    else:
        t = rng.integers(0, v, n)
    return t.astype(np.int64)


@pytest.mark.parametrize("table_type", DTYPES)
@pytest.mark.parametrize("out_type", DTYPES)
@pytest.mark.parametrize("n,v,d,pad,shift", [(1, 1, 1, 0, 0), (7, 5, 3, 1, 1), (300, 1000, 32, 0, 0),
                                             (65, 40, 777, 5, 3), (129, 300, 4104, 0, 0)])
def test_lookup(gpu, table_type, out_type, n, v, d, pad, shift):
    import torch

    native = native_mod()
    rng = np.random.default_rng(n + d)
    w, _ = on_gpu(rng.normal(size=(v, d)), table_type, gpu, pad, shift)
    tok = draw_tokens(rng, n, v, "holes" if n > 1 else "uniform")
    for index in (torch.int32, torch.int64):
        t = torch.from_numpy(tok).to(gpu, index)
        got = native.pdb_embed_lookup(w, t, scale=0.3, out_dtype=torch_type(out_type))
        # one product and one rounding: the same bits
        want = (w.float()[t.long().clamp(min=0)] * np.float32(0.3)).to(torch_type(out_type))
        want[t < 0] = 0
        assert torch.equal(got, want)


def test_lookup_shapes_and_out(gpu):
    import torch

    native = native_mod()
    w = torch.randn(50, 24, device=gpu)
    t = torch.randint(0, 50, (4, 6), device=gpu)
    assert torch.equal(native.pdb_embed_lookup(w, t), w[t])
    buf = torch.full((24, 40), 5.0, device=gpu)
    native.pdb_embed_lookup(w, t, out=buf[:, 3:27])
    assert torch.equal(buf[:, 3:27], w[t].view(24, 24))
    assert bool((buf[:, :3] == 5).all()) and bool((buf[:, 27:] == 5).all())
    assert native.pdb_embed_lookup(w, t[:0]).shape == (0, 6, 24)


EMBED = [  # n, v, d, tokens, pad
    (1, 1, 1, "uniform", 0), (1, 300, 32, "uniform", 0), (100, 1000, 32, "zipf", 0),
    (100, 7, 33, "uniform", 2), (700, 50, 20, "one", 0), (257, 300, 777, "holes", 23),
    (64, 40, 4104, "zipf", 0), (5000, 300, 64, "zipf", 0), (5000, 5000, 16, "holes", 1),
    (3000, 100, 1, "zipf", 0), (4097, 2, 40, "uniform", 0), (9000, 20000, 24, "one", 0),
    (20, 30, 8, "none", 0), (30011, 1003, 17, "zipf", 0), (2100, 30, 1030, "one", 3)]


@pytest.mark.parametrize("n,v,d,how,pad", EMBED)
@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"),
                                   ("f32", "f16")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad(gpu, n, v, d, how, pad, types, accumulate):
    import torch

    native = native_mod()
    rng = np.random.default_rng(n + v + d)
    dy, dy64 = on_gpu(rng.normal(size=(n, d)), types[0], gpu, pad, pad % 3)
    tok = draw_tokens(rng, n, v, how)
    old, old64 = on_gpu(rng.normal(size=(v, d)), types[1], gpu, pad)
    want, bound = ref.embed_grad(dy64, tok, old64, -0.25, accumulate)
    index = torch.int32 if n % 2 else torch.int64
    got = native.pdb_embed_grad(dy, torch.from_numpy(tok).to(gpu, index), old, scale=-0.25,
                                accumulate=accumulate)
    if types[1] != "f32":
        touched = np.isin(np.arange(v), tok)[:, None]
        bound = bound + np.where(touched | (not accumulate), ref.rounded(np.abs(want) + bound, types[1]), 0)
    check(f64(got), want, bound, "grad")


def test_embed_grad_repeats_and_workspace(gpu):
    """The same bits on a repeated call, whatever the workspace held; and on a
    workspace larger than asked for."""
    import torch

    native = native_mod()
    rng = np.random.default_rng(3)
    for n, v, d in [(200, 100, 48), (20000, 700, 40)]:
        dy = torch.from_numpy(rng.normal(size=(n, d)).astype(np.float32)).to(gpu)
        tok = torch.from_numpy(draw_tokens(rng, n, v, "zipf")).to(gpu)
        need = native.pdb_embed_grad_workspace_bytes(n, v, d)
        got = []
        for fill, more in ((0, 0), (255, 0), (90, 4096)):
            ws = torch.full((need + more,), fill, dtype=torch.uint8, device=gpu)
            got.append(native.pdb_embed_grad(dy, tok, torch.empty(v, d, device=gpu), ws=ws))
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_embed_grad_is_the_lookups(gpu):
    """The lookup is linear in its table: along any direction its difference
    equals the gradient's product with that direction."""
    import torch

    native = native_mod()
    g = torch.Generator(device=gpu)
    g.manual_seed(5)
    n, v, d = 900, 200, 36
    tok = torch.randint(-20, v, (n,), device=gpu, generator=g)
    w, dw = (torch.randn(v, d, device=gpu, generator=g) for _ in range(2))
    dy = torch.randn(n, d, device=gpu, generator=g)
    grad = native.pdb_embed_grad(dy, tok, torch.empty_like(w), scale=0.5)
    f = lambda x: float((native.pdb_embed_lookup(x, tok, scale=0.5).double() * dy.double()).sum())
    got = float((grad.double() * dw.double()).sum())
    # 1/16 steps: the products stay exact up to the roundings of w +- h dw
    h = 2.0 ** -4
    diff = (f(w + h * dw) - f(w - h * dw)) / (2 * h)
    # n d terms of order 1, each rounded by 2 u / h
    assert abs(got - diff) <= n * d * 4 * ref.U / h


def test_sgd_step_on_the_table(gpu):
    """Accumulating into the table with scale -lr is the step, and rows that no
    token picked keep their bits."""
    import torch

    native = native_mod()
    w = torch.randn(5000, 32, device=gpu)
    before = w.clone()
    tok = torch.randint(0, 200, (1000,), device=gpu, dtype=torch.int32)
    dy = torch.randn(1000, 32, device=gpu)
    native.pdb_embed_grad(dy, tok, w, scale=-0.1, accumulate=True)
    assert torch.equal(w[200:], before[200:])
    want, bound = ref.embed_grad(f64(dy), tok.cpu().numpy(), f64(before), float(np.float32(-0.1)), True)
    check(f64(w), want, bound, "step")


def test_embed_out_of_range_tokens(gpu):
    import torch

    native = native_mod()
    w = torch.randn(10, 8, device=gpu)
    status = torch.zeros(1, dtype=torch.int32, device=gpu)
    for bad in (10, 2 ** 31 - 1, 2 ** 40 + 3):
        tok = torch.tensor([3, bad, -5, 9], device=gpu)
        status.zero_()
        out = native.pdb_embed_lookup(w, tok, status=status)
        assert int(status) == native.PDB_ERR_INVALID_ARG
        assert torch.equal(out[[0, 3]], w[[3, 9]]) and not out[1:3].any()
        status.zero_()
        g = native.pdb_embed_grad(torch.ones(4, 8, device=gpu), tok, torch.empty(10, 8, device=gpu),
                                  status=status)
        assert int(status) == native.PDB_ERR_INVALID_ARG
        assert float(g.sum()) == 16.0 and float(g[3].sum()) == 8.0
    status.zero_()
    native.pdb_embed_lookup(w, torch.tensor([0, -1, 9], device=gpu), status=status)
    assert int(status) == 0


def test_embed_no_tokens(gpu):
    import torch

    native = native_mod()
    g = torch.full((40, 12), 3.0, device=gpu)
    none, dy = torch.empty(0, dtype=torch.int64, device=gpu), torch.empty(0, 12, device=gpu)
    native.pdb_embed_grad(dy, none, g, accumulate=True)
    assert bool((g == 3).all())
    native.pdb_embed_grad(dy, none, g)
    assert not g.any()


def test_embed_offsets_past_32_bits(gpu):
    """A table of more than 2^32 bytes and 2^31 elements: its last rows."""
    import torch

    native = native_mod()
    v, d = 70_000_000, 32
    w = torch.empty(v, d, dtype=torch.bfloat16, device=gpu)
    w[-100:] = torch.randn(100, d, device=gpu)
    tok = torch.arange(v - 100, v, device=gpu)
    assert torch.equal(native.pdb_embed_lookup(w, tok), w[-100:])
    dy = torch.ones(200, d, device=gpu)
    want = (w[-100:].float() + 2.0).bfloat16()
    native.pdb_embed_grad(dy, torch.cat([tok, tok]), w, accumulate=True)
    assert torch.equal(w[-100:], want)
    native.pdb_embed_grad(dy, torch.cat([tok, tok]), w, scale=0.5)
    assert bool((w[-100:] == 1).all()) and not w[:-100].any()


# ---------------------------------------------------------------------------
# rows of logits

def draw_logits(rng, n, v, how):
    z = 3.0 * rng.normal(size=(n, v))
    if how == "equal":
        z[:] = 1.5
    elif how == "coarse":  # many ties
        z = np.round(z)
    elif how == "falling":
        z = np.broadcast_to(np.linspace(20, -20, v), (n, v)).copy()
    elif how == "rising":
        z = np.broadcast_to(np.linspace(-20, 20, v), (n, v)).copy()
    elif how == "waves":  # the largest logits 2048 elements apart, then next to them
        z = np.broadcast_to(30 - (np.arange(v) % 2048) * 0.01 - np.arange(v) / (8.0 * v), (n, v)).copy()
    elif how == "large":
        z = z * 3000.0
    elif how == "masked":
        z[rng.random((n, v)) < 0.7] = NINF
        z[::3, v // 2:] = NINF
        z[1::4] = NINF                                   # nothing left
        z[2::5, :(v + 1) // 2] = -65504.0                # a lowest value
    elif how == "lowest":
        z[:] = -65504.0
        z[::2, v // 2] = 0.0
    elif how == "special":
        z[0, v // 2] = np.nan
        z[-1, v - 1] = np.inf
        z[n // 2, v // 3:] = np.nan
    return z


HOWS = ["normal", "equal", "coarse", "falling", "rising", "waves", "large", "masked", "lowest",
        "special"]
SIZES = [  # n, v, top, pad, shift
    (1, 1, 1, 0, 0), (3, 2, 2, 1, 1), (5, 63, 20, 0, 0), (4, 257, 128, 3, 2), (7, 1000, 5, 0, 0),
    (6, 8193, 64, 7, 1), (2, 20011, 20, 0, 0), (1, 140001, 128, 0, 0), (1500, 300, 3, 5, 0),
    (1030, 2501, 64, 0, 0)]


@pytest.mark.parametrize("n,v,top,pad,shift", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("how", HOWS)
def test_logprobs(gpu, n, v, top, pad, shift, dtype, how):
    import torch

    native = native_mod()
    rng = np.random.default_rng(v + n)
    z, z64 = on_gpu(draw_logits(rng, n, v, how), dtype, gpu, pad, shift)
    tok = rng.integers(0, v, n)
    tok[rng.random(n) < 0.1] = -1
    temp = (1.0, 0.7, 2.0)[v % 3]
    t = torch.from_numpy(tok).to(gpu, torch.int32 if n % 2 else torch.int64)
    want = ref.logprobs(z64, tok, float(np.float32(temp)), top)
    for k in (top, 0):
        r = native.pdb_token_logprobs(z, t, top=k, temp=temp)
        check(f64(r.logp), want["logp"], want["b_logp"], "logp")
        check(f64(r.entropy), want["entropy"], want["b_entropy"], "entropy")
        if k:
            assert np.array_equal(r.top_id.cpu().numpy(), want["top_id"])
            check(f64(r.top_logp), want["top_logp"], want["b_top"], "top_logp")
    # without tokens no row is skipped
    r = native.pdb_token_logprobs(z, top=top, temp=temp)
    want = ref.logprobs(z64, None, float(np.float32(temp)), top)
    assert r.logp is None
    check(f64(r.entropy), want["entropy"], want["b_entropy"], "entropy")
    assert np.array_equal(r.top_id.cpu().numpy(), want["top_id"])


@pytest.mark.parametrize("n,v,top,pad,shift", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("how", ["normal", "equal", "large", "masked", "lowest"])
def test_logprobs_grad(gpu, n, v, top, pad, shift, dtype, how):
    import torch

    native = native_mod()
    rng = np.random.default_rng(v + n)
    z, z64 = on_gpu(draw_logits(rng, n, v, how), dtype, gpu, pad, shift)
    tok = rng.integers(0, v, n)
    tok[rng.random(n) < 0.1] = -1
    temp = (1.0, 0.7, 2.0)[v % 3]
    t = torch.from_numpy(tok).to(gpu, torch.int32 if n % 2 else torch.int64)
    f = native.pdb_token_logprobs(z, t, temp=temp)
    g, gh = (torch.from_numpy(rng.normal(size=n).astype(np.float32)).to(gpu) for _ in range(2))
    for a, b in ((g, gh), (g, None), (None, gh)):
        want, bound = ref.logprobs_grad(z64, tok, float(np.float32(temp)), a if a is None else f64(a),
                                        b if b is None else f64(b))
        bound = bound + ref.rounded(np.abs(want) + bound, dtype)
        got = native.pdb_token_logprobs_grad(z, t, f.stats, a, f.entropy, b, temp=temp)
        check(f64(got), want, bound, "dlogits")
    # entropies alone need no tokens; in place gives the same bits
    if not (tok < 0).any():
        none = native.pdb_token_logprobs_grad(z, None, f.stats, None, f.entropy, gh, temp=temp)
        assert torch.equal(none, got)
    got = native.pdb_token_logprobs_grad(z, t, f.stats, g, f.entropy, gh, temp=temp)
    native.pdb_token_logprobs_grad(z, t, f.stats, g, f.entropy, gh, temp=temp, out=z)
    assert torch.equal(z, got)


def central_difference(f, z, h):
    d = np.zeros_like(z)
    for i in np.ndindex(z.shape):
        a, b = z.copy(), z.copy()
        a[i] += h
        b[i] -= h
        d[i] = (f(a) - f(b)) / (2 * h)
    return d


def test_logprobs_grad_against_differences(gpu):
    import torch

    native = native_mod()
    rng = np.random.default_rng(8)
    z, z64 = on_gpu(rng.normal(size=(3, 37)), "f32", gpu)
    tok = np.array([5, 36, 0])
    g, gh = rng.normal(size=3), rng.normal(size=3)

    def value(x):
        r = ref.logprobs(x, tok, 0.5, 0)
        return float((g * r["logp"] + gh * r["entropy"]).sum())

    t = torch.from_numpy(tok).to(gpu)
    f = native.pdb_token_logprobs(z, t, temp=0.5)
    got = native.pdb_token_logprobs_grad(z, t, f.stats, torch.from_numpy(g).float().to(gpu),
                                         f.entropy, torch.from_numpy(gh).float().to(gpu), temp=0.5)
    # h^2 / 6 times a third derivative of at most 8 |g| / T^3 each, and the 32-bit bound
    _, bound = ref.logprobs_grad(z64, tok, 0.5, g, gh)
    h = 1e-4
    check(f64(got), central_difference(value, z64, h),
          bound + h * h / 6 * 8 * 8 * (np.abs(g) + 4 * np.abs(gh))[:, None] + 1e-10, "differences")


def draw_teacher(rng, n, v, k, how):
    ids = rng.integers(0, v, (n, k))
    t = 2.0 * rng.normal(size=(n, k))
    if how == "holes":
        ids[rng.random((n, k)) < 0.4] = -1
        ids[1::3] = -1
        t[rng.random((n, k)) < 0.2] = NINF
        t[2::7] = NINF
    elif how == "same":  # one id many times
        ids[:] = ids[:, :1]
    return ids.astype(np.int32), t


DISTILL = [  # n, v, k, pad, shift
    (1, 1, 1, 0, 0), (3, 2, 5, 1, 1), (5, 63, 20, 0, 0), (4, 257, 128, 3, 2), (7, 1000, 1, 0, 0),
    (6, 8193, 64, 7, 1), (2, 30011, 300, 0, 0), (1, 140001, 1024, 0, 0), (1500, 300, 3, 5, 0),
    (1030, 2501, 64, 0, 0)]


@pytest.mark.parametrize("n,v,k,pad,shift", DISTILL)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("how,teacher", [("normal", "plain"), ("normal", "holes"), ("coarse", "same"),
                                         ("large", "plain"), ("masked", "holes"),
                                         ("lowest", "plain")])
def test_distill(gpu, n, v, k, pad, shift, dtype, how, teacher):
    import torch

    native = native_mod()
    rng = np.random.default_rng(v + n + k)
    z, z64 = on_gpu(draw_logits(rng, n, v, how), dtype, gpu, pad, shift)
    ids, t = draw_teacher(rng, n, v, k, teacher)
    tt, t64 = on_gpu(t, ("f32", "bf16", "f16")[n % 3], gpu)
    tt = tt.contiguous()
    w = rng.normal(size=n).astype(np.float32)
    w[rng.random(n) < 0.1] = 0.0
    temp = (1.0, 0.7, 2.0)[v % 3]
    ig, wg = torch.from_numpy(ids).to(gpu), torch.from_numpy(w).to(gpu)
    loss, d, bl, bd = ref.distill(z64, ids, t64, float(np.float32(temp)), w.astype(np.float64))
    bd = bd + ref.rounded(np.abs(d) + bd, dtype)
    got_loss, got = native.pdb_distill(z, ig, tt, temp=temp, weight=wg)
    check(f64(got_loss), loss, bl, "loss")
    check(f64(got), d, bd, "dlogits")
    only, none = native.pdb_distill(z, ig, tt, temp=temp, weight=wg, grad=False)
    assert none is None
    check(f64(only), loss, bl, "loss alone")
    # in place
    again, _ = native.pdb_distill(z, ig, tt, temp=temp, weight=wg, out=z)
    check(f64(again), loss, bl, "loss in place")
    assert torch.equal(z, got)


def test_distill_special_values(gpu):
    import torch

    native = native_mod()
    z = torch.randn(4, 3000, device=gpu)
    z[0, 7] = float("nan")
    z[1, 9] = float("inf")
    ids = torch.tensor([[1, 2]] * 4, dtype=torch.int32, device=gpu)
    t = torch.zeros(4, 2, device=gpu)
    t[2, 0] = float("nan")
    loss, d = native.pdb_distill(z, ids, t)
    assert bool(loss[:3].isnan().all()) and bool(d[0].isnan().all())
    assert bool(torch.isfinite(loss[3])) and bool(torch.isfinite(d[3]).all())
    # a row of weight 0 is not looked at
    loss, d = native.pdb_distill(z, ids, t, weight=torch.tensor([0.0, 0.0, 0.0, 1.0], device=gpu))
    assert not loss[:3].any() and not d[:3].any()


def test_distill_against_differences(gpu):
    import torch

    native = native_mod()
    rng = np.random.default_rng(9)
    z, z64 = on_gpu(rng.normal(size=(3, 41)), "f32", gpu)
    ids, t = draw_teacher(rng, 3, 41, 6, "plain")
    ids[0, 2] = -1
    ids[1, 3] = ids[1, 0]
    w = np.array([1.0, -0.5, 2.0])
    tt, t64 = on_gpu(t, "f32", gpu)
    _, got = native.pdb_distill(z, torch.from_numpy(ids).to(gpu), tt.contiguous(), temp=2.0,
                                weight=torch.from_numpy(w).float().to(gpu))
    _, _, _, bound = ref.distill(z64, ids, t64, 2.0, w)
    h = 1e-4
    want = central_difference(lambda x: float(ref.distill(x, ids, t64, 2.0, w)[0].sum()), z64, h)
    check(f64(got), want, bound + h * h / 6 * 8 + 1e-10, "differences")


def test_teacher_to_student(gpu):
    """What pdb_token_logprobs gives of a teacher is what pdb_distill takes; a
    student with the teacher's logits, and all of the vocabulary handed over,
    has loss 0 and gradient 0."""
    import torch

    native = native_mod()
    z = 2.0 * torch.randn(40, 100, device=gpu)
    f = native.pdb_token_logprobs(z, top=100, temp=1.0)
    loss, d = native.pdb_distill(z, f.top_id, f.top_logp)
    # 200 u for the two log sums, times the magnitudes of up to 12 of log p
    assert float(loss.abs().max()) <= 200 * ref.U * 12 and float(d.abs().max()) <= 200 * ref.U * 12


def test_out_of_range_ids_and_tokens(gpu):
    import torch

    native = native_mod()
    z = torch.randn(3, 50, device=gpu)
    status = torch.zeros(1, dtype=torch.int32, device=gpu)
    r = native.pdb_token_logprobs(z, torch.tensor([4, 50, 2 ** 35], device=gpu), top=2, status=status)
    assert int(status) == native.PDB_ERR_INVALID_ARG
    assert not r.logp[1:].any() and bool((r.top_id[1:] == -1).all())
    status.zero_()
    g = torch.ones(3, device=gpu)
    d = native.pdb_token_logprobs_grad(z, torch.tensor([4, 50, 51], device=gpu), r.stats, g,
                                       status=status)
    assert int(status) == native.PDB_ERR_INVALID_ARG and not d[1:].any()
    status.zero_()
    ids = torch.tensor([[1, 50], [2 ** 31 - 1, 50], [3, 4]], dtype=torch.int32, device=gpu)
    loss, d = native.pdb_distill(z, ids, torch.zeros(3, 2, device=gpu), status=status)
    assert int(status) == native.PDB_ERR_INVALID_ARG
    assert float(loss[1]) == 0.0 and not d[1].any()
    want, _ = native.pdb_distill(z[:1], ids[:1, :1].contiguous(), torch.zeros(1, 1, device=gpu))
    assert abs(float(loss[0]) - float(want[0])) <= 100 * ref.U * 8


def test_logits_past_32_bits(gpu):
    """More than 2^32 bytes and 2^31 elements of logits: the last rows."""
    import torch

    native = native_mod()
    n, v = 20_000, 131_072
    z = torch.zeros(n, v, dtype=torch.bfloat16, device=gpu)
    z[-2:] = 3 * torch.randn(2, v, device=gpu)
    tok = torch.full((n,), -1, device=gpu)
    tok[-2:] = torch.tensor([v - 1, 17], device=gpu)
    want = ref.logprobs(f64(z[-2:]), tok[-2:].cpu().numpy(), 1.0, 20)
    r = native.pdb_token_logprobs(z, tok, top=20)
    check(f64(r.logp[-2:]), want["logp"], want["b_logp"], "logp")
    assert np.array_equal(r.top_id[-2:].cpu().numpy(), want["top_id"])
    g = torch.ones(n, device=gpu)
    d64, bound = ref.logprobs_grad(f64(z[-2:]), tok[-2:].cpu().numpy(), 1.0, np.ones(2), None)
    ids = torch.full((n, 4), -1, dtype=torch.int32, device=gpu)
    ids[-2:] = torch.tensor([5, 9, v - 1, 77], device=gpu, dtype=torch.int32)
    t = torch.randn(n, 4, device=gpu)
    loss, d = native.pdb_distill(z, ids, t)
    l2, d2, b1, b2 = ref.distill(f64(z[-2:]), ids[-2:].cpu().numpy(), f64(t[-2:]), 1.0, np.ones(2))
    check(f64(loss[-2:]), l2, b1, "loss")
    check(f64(d[-2:]), d2, b2 + ref.rounded(np.abs(d2) + b2, "bf16"), "dlogits")
    del d
    native.pdb_token_logprobs_grad(z, tok, r.stats, g, out=z)
    check(f64(z[-2:]), d64, bound + ref.rounded(np.abs(d64) + bound, "bf16"), "dlogits")
    assert not z[:-2].any()


# ---------------------------------------------------------------------------
# streams and graphs

def every_operator(native, s):
    """One call of each on the inputs s; their outputs."""
    f = native.pdb_token_logprobs(s["z"], s["tok"], top=20, temp=0.7, stream=s.get("stream"))
    g = native.pdb_token_logprobs_grad(s["z"], s["tok"], f.stats, s["g"], f.entropy, s["g"],
                                       temp=0.7, stream=s.get("stream"))
    loss, d = native.pdb_distill(s["z"], s["ids"], s["t"], stream=s.get("stream"))
    e = native.pdb_embed_lookup(s["w"], s["tok"], scale=2.0, stream=s.get("stream"))
    w = native.pdb_embed_grad(s["dy"], s["tok"], s["grad"], stream=s.get("stream"))
    return [f.logp, f.entropy, f.stats, f.top_id, f.top_logp, g, loss, d, e, w]


def operator_inputs(gpu, n, v):
    import torch

    return dict(z=torch.randn(n, v, device=gpu).bfloat16(), tok=torch.randint(0, v, (n,), device=gpu),
                g=torch.randn(n, device=gpu), t=torch.randn(n, 8, device=gpu),
                ids=torch.randint(0, v, (n, 8), device=gpu, dtype=torch.int32),
                w=torch.randn(v, 40, device=gpu), dy=torch.randn(n, 40, device=gpu),
                grad=torch.empty(v, 40, device=gpu))


@pytest.mark.parametrize("n,v", [(3, 20011), (2000, 600)])
def test_on_another_stream(gpu, n, v):
    import torch

    native = native_mod()
    s = operator_inputs(gpu, n, v)
    want = [x.clone() for x in every_operator(native, s)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = [x.clone() for x in every_operator(native, s)]
    b = every_operator(native, dict(s, stream=side))
    # tensors made on the current stream meanwhile must not land in the calls' workspaces
    junk = [torch.full((1 << 20,), 9.0, device=gpu) for _ in range(8)]
    side.synchronize()
    torch.cuda.synchronize()
    for x, y, z in zip(want, a, b):
        assert torch.equal(x, y) and torch.equal(x, z)
    del junk


@pytest.mark.parametrize("n,v", [(3, 20011), (5000, 600)])
def test_in_a_graph(gpu, n, v):
    import torch

    native = native_mod()
    s = operator_inputs(gpu, n, v)
    every_operator(native, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = every_operator(native, s)
    for k in range(4):
        fresh = operator_inputs(gpu, n, v)
        for name in ("z", "tok", "g", "t", "ids", "w", "dy"):
            s[name].copy_(fresh[name])
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        want = every_operator(native, dict(fresh, grad=torch.empty_like(s["grad"])))
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), k
