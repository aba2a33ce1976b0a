"""The token operators where a kernel is chosen by size: several rows to a team, rows
held in registers of every size and rows too long for that, a wave to a row, the
sorts of many tokens.  Rows are independent, so some of each call's are held against
the 64-bit forms of tokenref, and all of them against the call on them in another order."""
import numpy as np
import pytest

import tokenref as ref
from test_gpu_tokens import DTYPES, NINF, check, f64, native_mod, on_gpu, torch_type

pytestmark = pytest.mark.gpu


def some_rows(rng, n, most=48):
    return np.unique(np.concatenate([[0, n - 1], rng.integers(0, n, most)]))


def many_logits(gpu, rng, n, v, dtype, pad):
    """(n, v) on the GPU, rows pad elements further apart, some of them special: every
    eleventh holds one value only, every thirteenth is masked but for its last logit."""
    import torch

    gen = torch.Generator(device=gpu).manual_seed(int(rng.integers(1 << 30)))
    z = torch.empty(n, v + pad, dtype=torch_type(dtype), device=gpu)
    z.copy_(3.0 * torch.randn(n, v + pad, generator=gen, device=gpu))
    z = z[:, :v]
    z[5::11] = 1.5
    z[7::13, :v - 1] = NINF
    return z


DISTILL = [  # n, v, k, pad: lengths on either side of each share of a team's registers
    (20011, 3, 2, 0), (9001, 300, 5, 1), (6007, 2048, 20, 0), (3001, 2049, 128, 0),
    (1501, 7001, 129, 3), (901, 16384, 20, 0), (701, 30011, 257, 0), (401, 60001, 64, 7),
    (301, 131073, 1, 0), (270, 140009, 513, 1)]


@pytest.mark.parametrize("n,v,k,pad", DISTILL)
@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_rows(gpu, n, v, k, pad, dtype):
    import torch

    native = native_mod()
    rng = np.random.default_rng(n + v + k)
    z = many_logits(gpu, rng, n, v, dtype, pad)
    ids = rng.integers(0, v, (n, k)).astype(np.int32)
    t = (2.0 * rng.normal(size=(n, k))).astype(np.float32)
    ids[3::8] = -1                      # no teacher
    ids[4::9, k // 2:] = -1
    w = rng.normal(size=n).astype(np.float32)
    w[2::5] = 0.0
    ig, tg, wg = (torch.from_numpy(x).to(gpu) for x in (ids, t, w))
    loss, d = native.pdb_distill(z, ig, tg, temp=0.7, weight=wg)
    rows = some_rows(rng, n)
    at = torch.from_numpy(rows).to(gpu)
    want, want_d, bl, bd = ref.distill(f64(z[at]), ids[rows], t[rows].astype(np.float64),
                                       float(np.float32(0.7)), w[rows].astype(np.float64))
    check(f64(loss[at]), want, bl, "loss")
    check(f64(d[at]), want_d, bd + ref.rounded(np.abs(want_d) + bd, dtype), "dlogits")
    off = torch.from_numpy((w == 0) | (ids < 0).all(axis=1)).to(gpu)
    assert not loss[off].any() and not d[off].any()
    # rows are independent of the rows beside them: another order, the same bits
    turn = torch.from_numpy(rng.permutation(n)).to(gpu)
    l2, d2 = native.pdb_distill(z[turn], ig[turn], tg[turn], temp=0.7, weight=wg[turn])
    assert torch.equal(l2, loss[turn]) and torch.equal(d2, d[turn])
    native.pdb_distill(z, ig, tg, temp=0.7, weight=wg, out=z)
    assert torch.equal(z, d)


LOGPROBS = [  # n, v, top, pad
    (20011, 3, 3, 0), (4096, 33, 20, 0), (4100, 1000, 0, 1), (5003, 1001, 64, 0),
    (4099, 2500, 65, 0), (4097, 9001, 128, 5), (4111, 5000, 1, 0), (2049, 4099, 128, 0),
    (300, 65537, 100, 0), (40, 200003, 128, 1)]


@pytest.mark.parametrize("n,v,top,pad", LOGPROBS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_logprobs_rows(gpu, n, v, top, pad, dtype):
    import torch

    native = native_mod()
    rng = np.random.default_rng(n + v + top)
    z = many_logits(gpu, rng, n, v, dtype, pad)
    tok = rng.integers(0, v, n)
    tok[3::8] = -1
    tg = torch.from_numpy(tok).to(gpu)
    f = native.pdb_token_logprobs(z, tg, top=top, temp=2.0)
    g, gh = (torch.from_numpy(rng.normal(size=n).astype(np.float32)).to(gpu) for _ in range(2))
    d = native.pdb_token_logprobs_grad(z, tg, f.stats, g, f.entropy, gh, temp=2.0)
    rows = some_rows(rng, n)
    at = torch.from_numpy(rows).to(gpu)
    z64 = f64(z[at])
    want = ref.logprobs(z64, tok[rows], 2.0, top)
    check(f64(f.logp[at]), want["logp"], want["b_logp"], "logp")
    check(f64(f.entropy[at]), want["entropy"], want["b_entropy"], "entropy")
    if top:
        assert np.array_equal(f.top_id[at].cpu().numpy(), want["top_id"])
        check(f64(f.top_logp[at]), want["top_logp"], want["b_top"], "top_logp")
    want_d, bound = ref.logprobs_grad(z64, tok[rows], 2.0, f64(g[at]), f64(gh[at]))
    check(f64(d[at]), want_d, bound + ref.rounded(np.abs(want_d) + bound, dtype), "dlogits")
    off = tg < 0
    assert not f.logp[off].any() and not d[off].any()
    turn = torch.from_numpy(rng.permutation(n)).to(gpu)
    f2 = native.pdb_token_logprobs(z[turn], tg[turn], top=top, temp=2.0)
    for a, b in ((f2.logp, f.logp), (f2.entropy, f.entropy), (f2.stats, f.stats)):
        assert torch.equal(a, b[turn])
    if top:
        assert torch.equal(f2.top_id, f.top_id[turn]) and torch.equal(f2.top_logp, f.top_logp[turn])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,v", [(3, 40), (2, 30011), (600, 1001), (4100, 300), (300, 20001)])
def test_rows_of_the_lowest_value(gpu, dtype, n, v):
    """Rows that hold nothing but their type's lowest value, as a mask by that value
    leaves them, are uniform; one other logit takes everything."""
    import torch

    native = native_mod()
    z = torch.full((n, v), torch.finfo(torch_type(dtype)).min, dtype=torch_type(dtype), device=gpu)
    z[1::2, v // 3] = 1.0
    z64 = f64(z)
    rng = np.random.default_rng(v)
    tok = np.full(n, v // 3)
    tg = torch.from_numpy(tok).to(gpu)
    top = 3
    f = native.pdb_token_logprobs(z, tg, top=top, temp=0.7)
    temp = float(np.float32(0.7))
    want = ref.logprobs(z64, tok, temp, 1)
    check(f64(f.logp), want["logp"], want["b_logp"], "logp")
    check(f64(f.entropy), want["entropy"], want["b_entropy"], "entropy")
    assert np.array_equal(f.top_id[:, :1].cpu().numpy(), want["top_id"])
    check(f64(f.top_logp[:, :1]), want["top_logp"], want["b_top"], "top_logp")
    g, gh = (torch.from_numpy(rng.normal(size=n).astype(np.float32)).to(gpu) for _ in range(2))
    want_d, bound = ref.logprobs_grad(z64, tok, temp, f64(g), f64(gh))
    got = native.pdb_token_logprobs_grad(z, tg, f.stats, g, f.entropy, gh, temp=0.7)
    check(f64(got), want_d, bound + ref.rounded(np.abs(want_d) + bound, dtype), "dlogits")
    # the teacher's entries where the student has something left
    ids = tok[:, None].astype(np.int32)
    t = np.zeros((n, 1), np.float32)
    w = np.ones(n)
    loss, want_d, bl, bd = ref.distill(z64, ids, t.astype(np.float64), temp, w)
    got_loss, got = native.pdb_distill(z, torch.from_numpy(ids).to(gpu), torch.from_numpy(t).to(gpu),
                                       temp=0.7)
    check(f64(got_loss), loss, bl, "loss")
    check(f64(got), want_d, bd + ref.rounded(np.abs(want_d) + bd, dtype), "distill dlogits")


@pytest.mark.parametrize("n,v,d,pad", [
    (12288, 40000, 5, 0), (12289, 40000, 5, 1), (300007, 256, 3, 0), (300007, 65536, 12, 0),
    (1000003, 20, 8, 0), (131072, 131072, 33, 0), (8388609, 1000003, 2, 0)])
@pytest.mark.parametrize("how", ["uniform", "hot"])
def test_embed_grad_many_tokens(gpu, n, v, d, pad, how):
    import torch

    native = native_mod()
    rng = np.random.default_rng(n + v)
    tok = rng.integers(0, v, n)
    if how == "hot":  # a tenth of the positions share a token, some hold padding
        tok[rng.random(n) < 0.1] = v // 2
        tok[rng.random(n) < 0.05] = -1
    dy, dy64 = on_gpu(rng.normal(size=(n, d)), "f32", gpu, pad)
    old, old64 = on_gpu(rng.normal(size=(v, d)), "f32", gpu)
    tg = torch.from_numpy(tok).to(gpu, torch.int32)
    for accumulate in (True, False):
        want, bound = ref.embed_grad(dy64, tok, old64, 0.5, accumulate)
        got = native.pdb_embed_grad(dy, tg, old.clone(), scale=0.5, accumulate=accumulate)
        check(f64(got), want, bound, "grad")
        assert torch.equal(got, native.pdb_embed_grad(dy, tg, old.clone(), scale=0.5,
                                                      accumulate=accumulate))


@pytest.mark.parametrize("grad_type", DTYPES)
@pytest.mark.parametrize("v,d", [(1, 255), (70, 256), (130, 257), (4097, 300), (63, 2048)])
def test_rows_without_tokens_are_zero(gpu, grad_type, v, d):
    """All of a gradient is written, and nothing around it."""
    import torch

    native = native_mod()
    rng = np.random.default_rng(v * d)
    for n in (1, 300):
        tok = rng.integers(0, v, n)
        tok[n // 3:] = v - 1
        for pad in (0, 3):
            grad, _ = on_gpu(np.full((v, d), 5.0), grad_type, gpu, pad, 1)
            dy = torch.ones(n, d, device=gpu)
            base = grad._base
            native.pdb_embed_grad(dy, torch.from_numpy(tok).to(gpu), grad)
            want = torch.bincount(torch.from_numpy(tok), minlength=v).double()[:, None].expand(v, d)
            assert torch.equal(grad.double().cpu(), want)
            assert float(base[0]) == 7.0 and bool((base[1 + v * (d + pad):] == 7.0).all())
            if pad:
                assert bool((base[1:1 + v * (d + pad)].view(v, d + pad)[:, d:] == 7.0).all())
