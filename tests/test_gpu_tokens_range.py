"""The softmax statistics over the range that their types hold: rows whose largest
logit, or whose masked stretch, lies anywhere between ordinary logits and the type's
lowest value, and temperatures from far below to far above the logits' spread."""
import numpy as np
import pytest

import tokenref as ref
from test_gpu_tokens import check, f64, native_mod, on_gpu, torch_type

pytestmark = pytest.mark.gpu

# few rows, cut into parts; a block to a row; a wave to a row
SIZES = [(6, 20011), (300, 9001), (2100, 700)]
VALUES = [s * x for x in (1e6, 1e9, 1e10, 1e12, 1e20, 1e30, 1e37) for s in (-1, 1)]


def rows_of(rng, n, v, value):
    """Row i mod 6: value alone; before ordinary logits (more than a first tile of
    them); behind them (the whole last part); once among ordinary ones; ordinary ones
    alone; value and its negative in turn."""
    z = 3.0 * rng.normal(size=(n, v))
    z[0::6] = value
    z[1::6, :v - v // 3] = value
    z[2::6, min(16384, v // 2):] = value
    z[3::6, v // 2] = value
    z[5::6, 0::2] = value
    z[5::6, 1::2] = -value
    return z


def draw_tokens(rng, z):
    """A given token is a row's best or its last or any other."""
    n, v = z.shape
    tok = rng.integers(0, v, n)
    tok[::2] = z[::2].argmax(axis=1)
    tok[1::4] = v - 1
    return tok


def in_binary32(x):
    """A result past the range of binary32 is infinite."""
    return np.where(np.abs(x) > np.finfo(np.float32).max, np.sign(x) * np.inf, x)


def check_scores(gpu, rng, z, z64, temp, dtype, top=3):
    import torch

    native = native_mod()
    n, v = z64.shape
    t64 = float(np.float32(temp))
    tok = draw_tokens(rng, z64)
    tg = torch.from_numpy(tok).to(gpu)
    want = ref.logprobs(z64, tok, t64, top)
    want["logp"], want["top_logp"] = in_binary32(want["logp"]), in_binary32(want["top_logp"])
    # gradients of the size of temp, so that their quotient stays in every type's range
    g, gh = (torch.from_numpy((t64 * rng.normal(size=n)).astype(np.float32)).to(gpu) for _ in range(2))
    for k in (top, 0):
        f = native.pdb_token_logprobs(z, tg, top=k, temp=temp)
        check(f64(f.logp), want["logp"], want["b_logp"], "logp")
        check(f64(f.entropy), want["entropy"], want["b_entropy"], "entropy")
        if k:
            assert np.array_equal(f.top_id.cpu().numpy(), want["top_id"])
            check(f64(f.top_logp), want["top_logp"], want["b_top"], "top_logp")
    d, bound = ref.logprobs_grad(z64, tok, t64, f64(g), f64(gh))
    got = native.pdb_token_logprobs_grad(z, tg, f.stats, g, f.entropy, gh, temp=temp)
    check(f64(got), d, bound + ref.rounded(np.abs(d) + bound, dtype), "dlogits")


def check_distill(gpu, rng, z, z64, ids, teacher, temp, dtype):
    import torch

    native = native_mod()
    n, v = z64.shape
    t64 = float(np.float32(temp))
    tg, teacher64 = on_gpu(teacher, "f32", gpu)
    tg = tg.contiguous()
    w = (t64 * rng.normal(size=n)).astype(np.float32)
    ig, wg = torch.from_numpy(ids).to(gpu), torch.from_numpy(w).to(gpu)
    loss, d, bl, bd = ref.distill(z64, ids, teacher64, t64, w.astype(np.float64))
    got_loss, got = native.pdb_distill(z, ig, tg, temp=temp, weight=wg)
    check(f64(got_loss), loss, bl, "loss")
    check(f64(got), d, bd + ref.rounded(np.abs(d) + bd, dtype), "distill dlogits")
    only, _ = native.pdb_distill(z, ig, tg, temp=temp, weight=wg, grad=False)
    check(f64(only), loss, bl, "loss alone")


@pytest.mark.parametrize("n,v", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", VALUES)
def test_logits_of_any_size(gpu, n, v, dtype, value):
    rng = np.random.default_rng(n + v)
    z, z64 = on_gpu(rows_of(rng, n, v, value), dtype, gpu)
    temp = (1.0, 0.7, 5.0)[n % 3]
    check_scores(gpu, rng, z, z64, temp, dtype)
    ids = rng.integers(0, v, (n, 8)).astype(np.int32)
    ids[:, 0] = z64.argmax(axis=1)
    check_distill(gpu, rng, z, z64, ids, 2.0 * rng.normal(size=(n, 8)), temp, dtype)


@pytest.mark.parametrize("n,v", SIZES)
@pytest.mark.parametrize("value", VALUES)
def test_teachers_of_any_size(gpu, n, v, value):
    rng = np.random.default_rng(n + v + 1)
    z, z64 = on_gpu(3.0 * rng.normal(size=(n, v)), "bf16", gpu)
    k = 70  # more than a wave
    ids = rng.integers(0, v, (n, k)).astype(np.int32)
    check_distill(gpu, rng, z, z64, ids, rows_of(rng, n, k, value), 0.7, "bf16")


@pytest.mark.parametrize("n,v", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("temp", [1e-20, 1e-10, 1e-8, 1e-6, 1e-3, 1e3, 1e30])
def test_temperatures_of_any_size(gpu, n, v, dtype, temp):
    rng = np.random.default_rng(n + v + 2)
    z, z64 = on_gpu(rows_of(rng, n, v, 30.0), dtype, gpu)
    check_scores(gpu, rng, z, z64, temp, dtype)
    ids = rng.integers(0, v, (n, 8)).astype(np.int32)
    check_distill(gpu, rng, z, z64, ids, 2.0 * rng.normal(size=(n, 8)), temp, dtype)


@pytest.mark.parametrize("n,v", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("temp", [0.7, 5.0, 10.0, 1e4])
def test_the_lowest_value_at_any_temperature(gpu, n, v, dtype, temp):
    """A mask by the type's lowest value: whole rows, stretches, all but one entry."""
    import torch

    rng = np.random.default_rng(n + v + 3)
    z = rows_of(rng, n, v, np.inf)
    z[np.isinf(z)] = torch.finfo(torch_type(dtype)).min
    z, z64 = on_gpu(z, dtype, gpu)
    check_scores(gpu, rng, z, z64, temp, dtype)
    # a teacher under the same mask proposes none of its entries
    ids = np.repeat(z64.argmax(axis=1).astype(np.int32)[:, None], 2, axis=1)
    check_distill(gpu, rng, z, z64, ids, rng.normal(size=(n, 2)), temp, dtype)


@pytest.mark.parametrize("n,v", SIZES)
@pytest.mark.parametrize("temp", [1.0, 0.7, 3.0])
@pytest.mark.parametrize("side", [-1, 1])
def test_rows_across_the_two_forms(gpu, n, v, temp, side):
    """The running maximum passes |log2(e) m / T| = 2^20, where the sums go from one form
    of their powers to the other, while both sides count: rising, falling, in any order."""
    rng = np.random.default_rng(n + v + 4)
    edge = side * 2.0 ** 20 * np.log(2.0) * temp
    z = np.broadcast_to(np.linspace(-6.0, 6.0, v) * temp, (n, v)).copy()
    z[1::3] = z[1::3, ::-1]
    z[2::3] = rng.permuted(z[2::3], axis=1)
    z += rng.uniform(-5.0, 5.0, (n, 1)) * temp + edge
    z, z64 = on_gpu(z, "f32", gpu)
    check_scores(gpu, rng, z, z64, temp, "f32")
    ids = rng.integers(0, v, (n, 8)).astype(np.int32)
    check_distill(gpu, rng, z, z64, ids, edge + rng.normal(size=(n, 8)), temp, "f32")
