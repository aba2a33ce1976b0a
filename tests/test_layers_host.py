"""Host-side checks of the layer operators and of the verification of drafts: what
cannot be computed is refused before any device work; and checks of the 64-bit forms
that the GPU tests compare with."""
import ctypes
import os

import numpy as np
import pytest

import layerref as ref
from test_tokens_host import ODD, P, call, sweep


@pytest.fixture(scope="module")
def native():
    from paper_1508_00703_amd import native

    if not os.path.exists(native.LIB_PATH):
        pytest.fail("libpdb.so is not built (run __graft_entry__.build())")
    native.load()
    return native


def test_scan_refusals(native):
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    need = native.pdb_gated_scan_workspace_bytes(12, 8)
    base = dict(x=P, ldx=8, gate=P, ldg=8, dtype=2, n=12, d=8, starts=None, b=3, h0=P, y=P, ldy=8,
                state=P, marks=P, status=None, ws=P, ws_bytes=need, stream=None)
    refusals = [
        (dict(x=None), bad), (dict(gate=None), bad), (dict(y=None), bad), (dict(x=ODD), bad),
        (dict(gate=ODD), bad), (dict(y=ODD), bad), (dict(dtype=3), bad), (dict(ldx=7), bad),
        (dict(ldg=7), bad), (dict(ldy=7), bad), (dict(n=-1), bad), (dict(d=-1), bad), (dict(b=-1), bad),
        (dict(b=5), bad),               # 12 rows are not five equal sequences
        (dict(b=0), bad), (dict(starts=ODD), bad), (dict(h0=ODD), bad), (dict(state=ODD), bad),
        (dict(marks=ODD), bad), (dict(n=2 ** 31), big), (dict(starts=P, b=2 ** 31 - 1), big),
        (dict(ldx=2 ** 41), big), (dict(ws=None), native.PDB_ERR_WORKSPACE),
        (dict(ws_bytes=need - 1), native.PDB_ERR_WORKSPACE)]
    sweep(native, "pdb_gated_scan", base, refusals)
    assert call(native, "pdb_gated_scan", base, starts=P, b=0) == native.PDB_OK
    assert call(native, "pdb_gated_scan", base, n=0, b=0, x=None, gate=None, y=None) == native.PDB_OK
    assert call(native, "pdb_gated_scan", base, d=0) == native.PDB_OK


def test_scan_grad_refusals(native):
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    need = native.pdb_gated_scan_workspace_bytes(12, 8)
    base = dict(dy=P, lddy=8, x=P, ldx=8, gate=P, ldg=8, dtype=0, n=12, d=8, starts=None, b=3, h0=P,
                marks=P, d_state=P, dx=P, lddx=8, dgate=P, lddg=8, dh0=P, status=None, ws=P,
                ws_bytes=need, stream=None)
    sweep(native, "pdb_gated_scan_grad", base, [
        (dict(dy=None), bad), (dict(x=None), bad), (dict(gate=None), bad), (dict(dx=None), bad),
        (dict(dgate=None), bad), (dict(marks=None), bad), (dict(dy=ODD), bad), (dict(dtype=-1), bad),
        (dict(lddy=7), bad), (dict(lddx=7), bad), (dict(lddg=7), bad), (dict(b=5), bad),
        (dict(d_state=ODD), bad), (dict(dh0=ODD), bad), (dict(n=2 ** 31), big),
        (dict(ws=None), native.PDB_ERR_WORKSPACE), (dict(ws_bytes=need - 1), native.PDB_ERR_WORKSPACE)])
    assert call(native, "pdb_gated_scan_grad", base, starts=P, b=0) == native.PDB_OK


def one(native, **changes):
    t = dict(data=0x10000, rows=3, cols=5, ld=5, dtype=0)
    t.update(changes)
    a = (ctypes.c_int64 * 5)(t["data"], t["rows"], t["cols"], t["ld"], t["dtype"])
    return ctypes.cast(a, ctypes.c_void_p)


def test_clip_refusals(native):
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    nan, inf = float("nan"), float("inf")
    need = native.pdb_grad_workspace_bytes()
    good = one(native)
    norm = dict(grads=good, count=1, scale=1.0, norm=P, ws=P, ws_bytes=need, stream=None)
    of_tensor = [(dict(data=0), bad), (dict(data=0x10002), bad), (dict(rows=-1), bad),
                 (dict(cols=-1), bad), (dict(ld=4), bad), (dict(dtype=3), bad), (dict(rows=2 ** 31), big),
                 (dict(rows=1, cols=2 ** 40), big), (dict(rows=2 ** 20, cols=2 ** 20, ld=2 ** 20), big),
                 (dict(ld=2 ** 41), big)]
    common = [(dict(grads=None), bad), (dict(count=-1), bad), (dict(count=2 ** 20), big),
              (dict(scale=nan), bad), (dict(scale=inf), bad), (dict(norm=None), bad), (dict(norm=ODD), bad),
              (dict(ws=None), native.PDB_ERR_WORKSPACE), (dict(ws_bytes=need - 1), native.PDB_ERR_WORKSPACE)]
    sweep(native, "pdb_grad_norm", norm,
          common + [(dict(grads=one(native, **c)), e) for c, e in of_tensor])
    base = dict(grads=good, count=1, scale=1.0, max_norm=1.0, step=1.0, accumulate=0, outs=good, norm=P,
                ws=P, ws_bytes=need, stream=None)
    sweep(native, "pdb_grad_clip", base, common + [(dict(outs=one(native, **c)), e) for c, e in of_tensor] + [
        (dict(outs=None), bad), (dict(outs=one(native, rows=5, cols=3)), bad), (dict(max_norm=-1.0), bad),
        (dict(max_norm=nan), bad), (dict(step=inf), bad), (dict(accumulate=2), bad),
        (dict(outs=one(native, dtype=2)), bad),      # in place in another type
        (dict(outs=one(native, ld=6)), bad)])        # in place with another stride


def test_verify_refusals(native):
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    need = native.pdb_draft_verify_workspace_bytes(2, 3, 100)
    base = dict(target=P, ldt=100, draft=P, ldq=100, dtype=2, b=2, k=3, v=100, tokens=P, index=0, u=P,
                temp=1.0, out=P, accepted=P, status=None, ws=P, ws_bytes=need, stream=None)
    sweep(native, "pdb_draft_verify", base, [
        (dict(target=None), bad), (dict(target=ODD), bad), (dict(draft=ODD), bad), (dict(ldt=99), bad),
        (dict(ldq=99), bad), (dict(dtype=4), bad), (dict(b=-1), bad), (dict(k=-1), bad),
        (dict(k=65), big), (dict(v=0), bad), (dict(v=-1), bad), (dict(v=2 ** 31, ldt=2 ** 31), big),
        (dict(b=2 ** 30), big), (dict(tokens=None), bad), (dict(tokens=ODD), bad), (dict(index=2), bad),
        (dict(u=None), bad), (dict(u=ODD), bad), (dict(out=None), bad), (dict(accepted=None), bad),
        (dict(temp=0.0), bad), (dict(temp=float("nan")), bad), (dict(temp=float("inf")), bad),
        (dict(ws=None), native.PDB_ERR_WORKSPACE), (dict(ws_bytes=need - 1), native.PDB_ERR_WORKSPACE)])
    assert call(native, "pdb_draft_verify", base, b=0, target=None, draft=None, tokens=None, u=None,
                out=None, accepted=None) == native.PDB_OK


def test_workspace_queries(native):
    lib, sz = native.load(), ctypes.c_size_t(0)
    bad, big = native.PDB_ERR_INVALID_ARG, native.PDB_ERR_UNSUPPORTED
    assert lib.pdb_gated_scan_workspace_bytes(-1, 1, ctypes.byref(sz)) == bad
    assert lib.pdb_gated_scan_workspace_bytes(1, 1, None) == bad
    assert lib.pdb_gated_scan_workspace_bytes(2 ** 31, 1, ctypes.byref(sz)) == big
    assert lib.pdb_grad_workspace_bytes(None) == bad
    assert lib.pdb_draft_verify_workspace_bytes(1, -1, 1, ctypes.byref(sz)) == bad
    assert lib.pdb_draft_verify_workspace_bytes(1, 65, 1, ctypes.byref(sz)) == big
    assert native.pdb_gated_scan_workspace_bytes(2 ** 20, 4096) < 512 << 20
    assert native.pdb_draft_verify_workspace_bytes(1024, 8, 2 ** 17) < 64 << 20


def test_binding_refuses_what_it_cannot_pass(native):
    import torch

    x, h = torch.zeros(6, 8), torch.zeros(2, 8)
    marks = torch.zeros(1, 8)
    with pytest.raises(ValueError, match="device"):
        native.pdb_gated_scan(x, x)
    with pytest.raises(TypeError):
        native.pdb_gated_scan(x.double(), x)
    with pytest.raises(ValueError, match="device"):
        native.pdb_gated_scan_grad(x, x, x, marks)
    with pytest.raises(ValueError):
        native._sequences(x, torch.zeros(3, dtype=torch.int32), 5, -1)
    with pytest.raises(TypeError):
        native._sequences(x, torch.zeros(3, dtype=torch.int64), None, -1)
    with pytest.raises(ValueError):
        native._sequences(x.view(2, 3, 8), None, 3, -1)
    with pytest.raises(ValueError):
        native._rows(x[:, :4], "gate", x, -1)
    with pytest.raises(ValueError):
        native._rows(x.half(), "gate", x, -1)
    with pytest.raises(ValueError):
        native._state(h[:, :4], "h0", 2, 8, -1)
    with pytest.raises(ValueError, match="at least one"):
        native.pdb_grad_norm([])
    with pytest.raises(ValueError, match="device"):
        native.pdb_grad_norm([x])
    with pytest.raises(TypeError):
        native.pdb_grad_norm([x.double()])
    with pytest.raises(ValueError, match="same shape"):
        native.pdb_grad_clip([x], 1.0, out=[x.t()])
    with pytest.raises(ValueError, match="device"):
        native.pdb_draft_verify(x, torch.zeros(6, 1))
    for name, given in (("pdb_gated_scan", ("x", "gate")), ("pdb_draft_verify", ("target", "u")),
                        ("pdb_gated_scan_grad", ("dy", "x", "gate", "marks"))):
        with pytest.raises(ValueError, match="device"):
            getattr(native, name)(**{g: x for g in given})


# ---------------------------------------------------------------------------
# the 64-bit forms themselves

def test_scan_by_hand():
    # gates 0: the state moves half of the way to the input
    x = np.array([[4.0], [8.0], [1.0]])
    r = ref.scan(x, np.zeros((3, 1)), [(0, 2), (2, 2), (2, 3)], np.array([[2.0], [5.0], [3.0]]))
    assert r["y"][:, 0].tolist() == [3.0, 5.5, 2.0]
    assert r["before"][:, 0].tolist() == [2.0, 3.0, 3.0]
    assert r["state"][:, 0].tolist() == [5.5, 5.0, 2.0]


def test_scan_gradients_against_differences():
    rng = np.random.default_rng(0)
    n, d, seqs = 9, 2, [(0, 4), (4, 4), (4, 9)]
    x, g, dy = rng.normal(size=(3, n, d))
    h0, ds = rng.normal(size=(2, 3, d))
    want = ref.scan_grad(dy, x, g, seqs, h0, ds)

    def value(x, g, h0):
        r = ref.scan(x, g, seqs, h0)
        return (r["y"] * dy).sum() + (r["state"] * ds).sum()

    for k, name in enumerate(("dx", "dgate", "dh0")):
        args = [x, g, h0]
        for i in np.ndindex(args[k].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[k][i] += 1e-5
            down[k][i] -= 1e-5
            assert abs((value(*up) - value(*down)) / 2e-5 - want[name][i]) < 1e-8


@pytest.mark.parametrize("plant", ["gate", "reset", "last", "order"])
def test_planted_mistakes_are_seen(plant):
    """A mistake in a form is far outside its bound."""
    rng = np.random.default_rng(1)
    x, g, dy = rng.normal(size=(3, 30, 4))
    seqs, ds = [(0, 13), (13, 30)], rng.normal(size=(2, 4))
    r = ref.scan_grad(dy, x, g, seqs, None, ds)
    if plant == "gate":
        bad = ref.scan_grad(dy, x, 1.0001 * g, seqs, None, ds)
    elif plant == "reset":
        bad = ref.scan_grad(dy, x, g, [(0, 30), (30, 30)], None, ds)
    elif plant == "last":
        bad = ref.scan_grad(dy, x, g, seqs, None, None)
    else:
        bad = ref.scan_grad(dy[::-1], x, g, seqs, None, ds)
    assert (np.abs(bad["dgate"] - r["dgate"]) > 4 * r["bdgate"]).any()


def test_verify_by_hand():
    ln = np.log
    p, q = ln(np.array([0.5, 0.25, 0.25])), ln(np.array([0.25, 0.25, 0.5]))
    target, draft = np.stack([p, p])[None], q[None, None]

    def run(x, u0, u1, draft=draft):
        out, acc = ref.verify(target, draft, np.array([[x]]), np.array([[u0, u1]]), 1.0)
        return out[0].tolist(), int(acc[0])

    assert run(0, 0.99, 0.1) == ([0, 0], 1)       # p > q: always accepted, then from p
    assert run(0, 0.99, 0.6) == ([0, 1], 1)
    assert run(2, 0.49, 0.9) == ([2, 2], 1)       # p / q = 1 / 2
    assert run(2, 0.51, 0.9) == ([0, -1], 0)      # the draft has too little of 0 only
    assert run(1, 0.26, 0.5, None) == ([0, -1], 0)
    assert run(1, 0.26, 0.7, None) == ([2, -1], 0)  # without a distribution: p but for 1
    assert run(-1, 0.0, 0.6) == ([1, -1], 0)      # nothing drafted


def test_verified_tokens_follow_the_target():
    """The first token out is distributed as the target's, whatever the draft."""
    rng = np.random.default_rng(2)
    v, many = 5, 4000
    zt, zq = rng.normal(size=(2, v))
    q, p = ref.softmax(zq, 1.0), ref.softmax(zt, 1.0)
    x = rng.choice(v, many, p=q)[:, None]
    target = np.broadcast_to(zt, (many, 2, v))
    out, _ = ref.verify(target, np.broadcast_to(zq, (many, 1, v)), x, rng.random((many, 2)), 1.0)
    got = np.bincount(out[:, 0], minlength=v) / many
    assert np.abs(got - p).max() < 5 * np.sqrt(0.25 / many)   # five deviations


def test_clip_by_hand():
    g = [np.array([3.0]), np.array([4.0])]
    norm, _, out, _ = ref.clip(g, [np.array([1.0])] * 2, 2.0, 5.0, -1.0, True)
    assert norm == 10.0 and out[0][0] == -2.0 and out[1][0] == -3.0
