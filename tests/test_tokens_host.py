"""Host-side checks of the token operators' C ABI: no kernel is launched, and
what cannot be computed is refused before any device work.  Also checks of the
64-bit forms that the GPU tests compare with."""
import ctypes
import os

import numpy as np
import pytest

import tokenref as ref


@pytest.fixture(scope="module")
def native():
    from paper_1508_00703_amd import native

    if not os.path.exists(native.LIB_PATH):
        pytest.fail("libpdb.so is not built (run __graft_entry__.build())")
    native.load()
    return native


P = ctypes.c_void_p(0x10000)   # never dereferenced: every call here is refused
ODD = ctypes.c_void_p(0x10001)


def call(native, name, base, **changes):
    args = dict(base)
    args.update(changes)
    assert set(args) == set(base)
    return getattr(native.load(), name)(*args.values())


def sweep(native, name, base, refusals):
    for changes, code in refusals:
        assert call(native, name, base, **changes) == code, (name, changes)


def test_lookup_refusals(native):
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    base = dict(table=P, dtype=0, ld=8, v=10, d=8, tokens=P, index=0, n=4, scale=1.0, out=P,
                out_dtype=0, ldo=8, status=None, stream=None)
    sweep(native, "pdb_embed_lookup", base, [
        (dict(table=None), bad), (dict(tokens=None), bad), (dict(out=None), bad),
        (dict(table=ODD), bad), (dict(out=ODD), bad), (dict(tokens=ODD), bad),
        (dict(dtype=3), bad), (dict(out_dtype=-1), bad), (dict(index=2), bad), (dict(ld=7), bad),
        (dict(ldo=7), bad), (dict(v=-1), bad), (dict(n=-1), bad), (dict(d=-1), bad),
        (dict(n=2 ** 31), big), (dict(v=2 ** 31), big), (dict(d=2 ** 31, ld=2 ** 31, ldo=2 ** 31), big)])
    assert call(native, "pdb_embed_lookup", base, n=0, tokens=None, out=None) == native.PDB_OK


def test_embed_grad_refusals(native):
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    need = native.pdb_embed_grad_workspace_bytes(4, 10, 8)
    base = dict(dy=P, dtype=0, ldy=8, tokens=P, index=0, n=4, grad=P, grad_dtype=0, ldg=8, v=10, d=8,
                scale=1.0, accumulate=0, status=None, ws=P, ws_bytes=need, stream=None)
    sweep(native, "pdb_embed_grad", base, [
        (dict(dy=None), bad), (dict(tokens=None), bad), (dict(grad=None), bad), (dict(dy=ODD), bad),
        (dict(dtype=9), bad), (dict(grad_dtype=9), bad), (dict(index=-1), bad), (dict(ldy=7), bad),
        (dict(ldg=7), bad), (dict(accumulate=2), bad), (dict(n=-1), bad), (dict(v=-1), bad),
        (dict(n=2 ** 31), big), (dict(v=2 ** 31), big),
        (dict(ws=None), native.PDB_ERR_WORKSPACE),
        (dict(ws_bytes=need - 1), native.PDB_ERR_WORKSPACE)])
    assert call(native, "pdb_embed_grad", base, n=0, dy=None, tokens=None, accumulate=1) == native.PDB_OK
    assert call(native, "pdb_embed_grad", base, v=0, grad=None) == native.PDB_OK


def test_logprobs_refusals(native):
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    need = native.pdb_token_logprobs_workspace_bytes(4, 100, 5)
    base = dict(logits=P, dtype=2, ldz=100, n=4, v=100, tokens=P, index=0, temp=1.0, logp=P,
                entropy=P, stats=P, top=5, top_id=P, top_logp=P, status=None, ws=P, ws_bytes=need,
                stream=None)
    sweep(native, "pdb_token_logprobs", base, [
        (dict(logits=None), bad), (dict(logits=ODD), bad), (dict(tokens=None), bad),
        (dict(dtype=5), bad), (dict(index=7), bad), (dict(ldz=99), bad), (dict(n=-2), bad),
        (dict(v=0, ldz=0), bad), (dict(temp=0.0), bad), (dict(temp=-1.0), bad),
        (dict(temp=float("nan")), bad), (dict(temp=float("inf")), bad), (dict(temp=1e-45), bad),
        (dict(top=-1), bad), (dict(v=4, top=5), bad), (dict(v=1000, ldz=1000, top=129), big),
        (dict(n=2 ** 31), big), (dict(ws=None), native.PDB_ERR_WORKSPACE),
        (dict(ws_bytes=need - 1), native.PDB_ERR_WORKSPACE)])
    assert call(native, "pdb_token_logprobs", base, n=0, logits=None, tokens=None) == native.PDB_OK


def test_logprobs_grad_refusals(native):
    bad = native.PDB_ERR_INVALID_ARG
    base = dict(logits=P, dtype=2, ldz=100, n=4, v=100, tokens=P, index=0, temp=1.0, stats=P,
                entropy=P, d_logp=P, d_entropy=P, dlogits=P, ldd=100, status=None, stream=None)
    sweep(native, "pdb_token_logprobs_grad", base, [
        (dict(logits=None), bad), (dict(dlogits=None), bad), (dict(tokens=None), bad),
        (dict(stats=None), bad), (dict(entropy=None), bad), (dict(ldd=99), bad),
        (dict(ldd=101), bad),           # in place with another stride
        (dict(temp=0.0), bad), (dict(dtype=-1), bad), (dict(index=3), bad)])
    assert call(native, "pdb_token_logprobs_grad", base, n=0, logits=None, dlogits=None) == native.PDB_OK


def test_distill_refusals(native):
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    need = native.pdb_distill_workspace_bytes(4, 100)
    base = dict(logits=P, dtype=0, ldz=100, n=4, v=100, ids=P, teacher=P, teacher_dtype=2, k=8,
                temp=1.0, weight=None, loss=P, dlogits=P, ldd=100, status=None, ws=P, ws_bytes=need,
                stream=None)
    sweep(native, "pdb_distill", base, [
        (dict(logits=None), bad), (dict(ids=None), bad), (dict(teacher=None), bad),
        (dict(loss=None), bad), (dict(k=0), bad), (dict(k=-1), bad), (dict(k=1025), big),
        (dict(teacher_dtype=4), bad), (dict(temp=0.0), bad), (dict(ldz=99), bad),
        (dict(ldd=101), bad), (dict(ids=ODD), bad), (dict(v=0, ldz=0, ldd=0), bad),
        (dict(ws=None), native.PDB_ERR_WORKSPACE), (dict(ws_bytes=need - 1), native.PDB_ERR_WORKSPACE)])
    assert call(native, "pdb_distill", base, n=0, logits=None, ids=None, teacher=None, loss=None,
                dlogits=None) == native.PDB_OK


def test_workspace_queries(native):
    lib, sz = native.load(), ctypes.c_size_t(0)
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    assert lib.pdb_embed_grad_workspace_bytes(-1, 1, 1, ctypes.byref(sz)) == bad
    assert lib.pdb_embed_grad_workspace_bytes(1, 1, 1, None) == bad
    assert lib.pdb_embed_grad_workspace_bytes(2 ** 31, 1, 1, ctypes.byref(sz)) == big
    assert lib.pdb_token_logprobs_workspace_bytes(1, 1, -1, ctypes.byref(sz)) == bad
    assert lib.pdb_token_logprobs_workspace_bytes(1, 1000, 129, ctypes.byref(sz)) == big
    assert lib.pdb_distill_workspace_bytes(1, -1, ctypes.byref(sz)) == bad
    # bounded: rows are cut into parts only where they are few
    assert native.pdb_token_logprobs_workspace_bytes(10 ** 6, 10 ** 5, 128) < 64 << 20
    assert native.pdb_distill_workspace_bytes(10 ** 6, 10 ** 5) < 64 << 20


def test_binding_refuses_what_it_cannot_pass(native):
    import torch

    z = torch.zeros(3, 10)
    with pytest.raises(ValueError):           # not on a device
        native.pdb_token_logprobs(z)
    with pytest.raises(TypeError):
        native.pdb_token_logprobs(z.double())
    with pytest.raises(ValueError):
        native.pdb_token_logprobs(z[0])
    with pytest.raises(ValueError):
        native.pdb_embed_lookup(z.t(), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError):
        native._status(torch.zeros(1))
    with pytest.raises(TypeError):
        native._tokens(torch.zeros(4, dtype=torch.int16), 4)
    with pytest.raises(ValueError):
        native._tokens(torch.zeros(4, dtype=torch.int32), 5)


# ---------------------------------------------------------------------------
# the 64-bit forms themselves

def test_reference_by_hand():
    # two logits ln 3 and 0: probabilities 3/4 and 1/4
    z = np.array([[np.log(3.0), 0.0, -np.inf]])
    r = ref.logprobs(z, np.array([1]), 1.0, 3)
    assert np.isclose(r["logp"][0], np.log(0.25))
    assert np.isclose(r["entropy"][0], -(0.75 * np.log(0.75) + 0.25 * np.log(0.25)))
    assert r["top_id"][0].tolist() == [0, 1, 2] and r["top_logp"][0, 2] == -np.inf
    d, _ = ref.logprobs_grad(z, np.array([1]), 1.0, np.array([1.0]), None)
    assert np.allclose(d, [[-0.75, 0.75, 0.0]])
    loss, d, _, _ = ref.distill(z, np.array([[0, 1]]), np.array([[0.0, 0.0]]), 1.0, np.array([2.0]))
    assert np.isclose(loss[0], 2 * (0.5 * np.log(0.5 / 0.75) + 0.5 * np.log(0.5 / 0.25)))
    assert np.allclose(d, [[2 * 0.25, -2 * 0.25, 0.0]])
    g, _ = ref.embed_grad(np.array([[1.0], [2.0], [4.0]]), np.array([1, -1, 1]), np.zeros((2, 1)), 0.5,
                          False)
    assert g.tolist() == [[0.0], [2.5]]


def test_reference_gradients_against_differences():
    rng = np.random.default_rng(0)
    z = rng.normal(size=(2, 9))
    tok, g, gh = np.array([3, 8]), rng.normal(size=2), rng.normal(size=2)
    ids = np.array([[1, 4, 4], [0, -1, 8]])
    t, w = rng.normal(size=(2, 3)), np.array([1.5, -1.0])

    def scores(x):
        r = ref.logprobs(x, tok, 0.5, 0)
        return (g * r["logp"] + gh * r["entropy"]).sum()

    for f, d in ((scores, ref.logprobs_grad(z, tok, 0.5, g, gh)[0]),
                 (lambda x: ref.distill(x, ids, t, 2.0, w)[0].sum(),
                  ref.distill(z, ids, t, 2.0, w)[1])):
        for i in np.ndindex(z.shape):
            a, b = z.copy(), z.copy()
            a[i] += 1e-5
            b[i] -= 1e-5
            assert abs((f(a) - f(b)) / 2e-5 - d[i]) < 1e-8


@pytest.mark.parametrize("plant", ["sign", "temperature", "entropy", "duplicate"])
def test_planted_mistakes_are_seen(plant):
    """A mistake in a form is far outside its bound."""
    rng = np.random.default_rng(1)
    z, tok = rng.normal(size=(4, 50)), np.array([1, 2, 3, 4])
    g, gh = rng.normal(size=4), rng.normal(size=4)
    d, bound = ref.logprobs_grad(z, tok, 0.5, g, gh)
    ids = np.array([[1, 1, 2]] * 4)
    e, be = ref.distill(z, ids, np.zeros((4, 3)), 1.0, np.ones(4))[1::2]
    if plant == "sign":
        bad = ref.logprobs_grad(z, tok, 0.5, -g, gh)[0]
    elif plant == "temperature":
        bad = 0.5 * d
    elif plant == "entropy":
        bad = ref.logprobs_grad(z, tok, 0.5, g, 1.001 * gh)[0]
    else:
        bad, d, bound = ref.distill(z, np.array([[1, -1, 2]] * 4), np.zeros((4, 3)), 1.0, np.ones(4))[1], e, be
    assert (np.abs(bad - d) > 4 * bound).any()
