"""The layer operators on the GPU against the 64-bit forms of layerref, whose bounds
hold for every case here: one row and many, odd channels, ragged strides, every type,
empty sequences, sequences that end inside tiles, rows of no sequence, special values."""
import numpy as np
import pytest

import layerref as ref
from test_gpu_tokens import DTYPES, check, f64, native_mod, on_gpu, torch_type
from tokenref import rounded

pytestmark = pytest.mark.gpu


def store(dtype, want, bound):
    return bound if dtype == "f32" else bound + rounded(np.abs(want) + bound, dtype)


def cut(rng, n, b, how):
    """(starts or None, sequences) of n rows."""
    if how == "equal":
        return None, ref.spans(n, None, b)
    at = np.sort(rng.integers(0, n + 1, b + 1))
    if how == "all":
        at[0], at[-1] = 0, n
    elif how == "empty":
        at[: b // 2] = at[b // 2]
        at[-1] = n
    return at.astype(np.int32), ref.spans(n, at, b)


SCANS = [  # n, d, b, sequences, pad, shift
    (1, 1, 1, "equal", 0, 0), (1, 8, 1, "equal", 0, 0), (5, 3, 2, "all", 1, 1), (64, 64, 1, "equal", 0, 0),
    (63, 7, 3, "inside", 2, 0), (256, 64, 1, "equal", 0, 0), (257, 65, 3, "empty", 0, 0),
    (1000, 40, 7, "inside", 3, 5), (3000, 16, 1, "equal", 0, 0), (2048, 72, 2048, "equal", 0, 0),
    (700, 130, 300, "all", 0, 0), (512, 200, 2, "equal", 8, 0), (1300, 33, 5, "empty", 0, 0),
    (300, 5, 299, "all", 0, 0), (2600, 9, 1, "inside", 0, 1), (96, 2, 96, "equal", 5, 1),
    (77, 777, 11, "equal", 23, 0)]


def draw_scan(gpu, rng, n, d, b, how, pad, shift, dtype, wide=2.0):
    import torch

    x, x64 = on_gpu(rng.normal(size=(n, d)), dtype, gpu, pad, shift)
    g, g64 = on_gpu(rng.normal(size=(n, d)) * wide + 1.0, dtype, gpu, pad, shift)
    starts, seqs = cut(rng, n, b, how)
    on = None if starts is None else torch.from_numpy(starts).to(gpu)
    h0 = rng.normal(size=(b, d)).astype(np.float32)
    return x, x64, g, g64, on, seqs, h0


@pytest.mark.parametrize("n,d,b,how,pad,shift", SCANS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("first", [True, False])
def test_scan(gpu, n, d, b, how, pad, shift, dtype, first):
    import torch

    native = native_mod()
    rng = np.random.default_rng(n + d + b)
    x, x64, g, g64, starts, seqs, h0 = draw_scan(gpu, rng, n, d, b, how, pad, shift, dtype)
    h = torch.from_numpy(h0).to(gpu) if first else None
    want = ref.scan(x64, g64, seqs, h0 if first else None)
    out = torch.full((n, d + pad), 7.0, dtype=x.dtype, device=gpu)[:, :d]
    status = torch.zeros(1, dtype=torch.int32, device=gpu)
    f = native.pdb_gated_scan(x, g, starts=starts, batch=b, h0=h, marks=True, out=out, status=status)
    assert int(status) == 0
    y = f64(f.y)
    none = np.isnan(want["y"])
    assert (y[none] == 7).all()            # rows of no sequence
    check(np.where(none, 0, y), np.where(none, 0, want["y"]),
          store(dtype, np.where(none, 0, want["y"]), want["by"]), "y")
    check(f64(f.state), want["state"], want["bstate"], "state")
    at = np.arange(0, n, 64)
    some = ~np.isnan(want["before"][at])
    check(np.where(some, f64(f.marks), 0), np.where(some, want["before"][at], 0), want["bbefore"][at],
          "marks")
    # repeated, with a used workspace, and without marks: the same bits
    ws = torch.full((native.pdb_gated_scan_workspace_bytes(n, d) + 512,), 255, dtype=torch.uint8, device=gpu)
    again = native.pdb_gated_scan(x, g, starts=starts, batch=b, h0=h, out=torch.full_like(out, 7.0), ws=ws)
    assert torch.equal(again.y, f.y) and torch.equal(again.state, f.state) and again.marks is None


@pytest.mark.parametrize("n,d,b,how,pad,shift", SCANS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ends", [True, False])
def test_scan_grad(gpu, n, d, b, how, pad, shift, dtype, ends):
    import torch

    native = native_mod()
    rng = np.random.default_rng(n + 2 * d + b)
    x, x64, g, g64, starts, seqs, h0 = draw_scan(gpu, rng, n, d, b, how, pad, shift, dtype)
    dy, dy64 = on_gpu(rng.normal(size=(n, d)), dtype, gpu, pad, shift)
    ds = rng.normal(size=(b, d)).astype(np.float32) if ends else None
    h = torch.from_numpy(h0).to(gpu) if ends else None
    want = ref.scan_grad(dy64, x64, g64, seqs, h0 if ends else None, ds)
    f = native.pdb_gated_scan(x, g, starts=starts, batch=b, h0=h, marks=True)
    r = native.pdb_gated_scan_grad(dy, x, g, f.marks, starts=starts, batch=b, h0=h,
                                   d_state=None if ds is None else torch.from_numpy(ds).to(gpu))
    for name in ("dx", "dgate"):
        none = np.isnan(want[name])
        w = np.where(none, 0, want[name])
        check(np.where(none, 0, f64(getattr(r, name))), w, store(dtype, w, want["b" + name]), name)
    if ends:
        check(f64(r.dh0), want["dh0"], want["bdh0"], "dh0")
    else:
        assert r.dh0 is None
    again = native.pdb_gated_scan_grad(dy, x, g, f.marks, starts=starts, batch=b, h0=h,
                                       d_state=None if ds is None else torch.from_numpy(ds).to(gpu))
    inside = torch.from_numpy(~np.isnan(want["dx"])).to(gpu)
    assert torch.equal(again.dx[inside], r.dx[inside]) and torch.equal(again.dgate[inside], r.dgate[inside])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,b", [(40_000, 8, 1), (20_001, 130, 3), (9_000, 72, 500)])
def test_long_sequences(gpu, dtype, n, d, b):
    """Many tiles, gates that keep for thousands of rows: the chain over tiles."""
    import torch

    native = native_mod()
    rng = np.random.default_rng(n)
    x, x64, g, g64, starts, seqs, h0 = draw_scan(gpu, rng, n, d, b, "all", 0, 0, dtype, 4.0)
    g += 4.0
    g64 = f64(g)
    want = ref.scan(x64, g64, seqs, h0)
    h = torch.from_numpy(h0).to(gpu)
    f = native.pdb_gated_scan(x, g, starts=starts, h0=h, marks=True)
    check(f64(f.y), want["y"], store(dtype, want["y"], want["by"]), "y")
    check(f64(f.state), want["state"], want["bstate"], "state")
    dy, dy64 = on_gpu(rng.normal(size=(n, d)), dtype, gpu)
    back = ref.scan_grad(dy64, x64, g64, seqs, h0, None)
    r = native.pdb_gated_scan_grad(dy, x, g, f.marks, starts=starts, h0=h)
    for name in ("dx", "dgate"):
        check(f64(getattr(r, name)), back[name], store(dtype, back[name], back["b" + name]), name)
    check(f64(r.dh0), back["dh0"], back["bdh0"], "dh0")
    for _ in range(3):
        again = native.pdb_gated_scan(x, g, starts=starts, h0=h)
        assert torch.equal(again.y, f.y) and torch.equal(again.state, f.state)
        more = native.pdb_gated_scan_grad(dy, x, g, f.marks, starts=starts, h0=h)
        assert torch.equal(more.dx, r.dx) and torch.equal(more.dgate, r.dgate)


def test_scan_shapes_and_states(gpu):
    """[b, t, d]; decoding row by row with the states in place gives what one call gives."""
    import torch

    native = native_mod()
    b, t, d = 5, 37, 43
    x, g = torch.randn(2, b, t, d, device=gpu)
    h0 = torch.randn(b, d, device=gpu)
    whole = native.pdb_gated_scan(x, g, h0=h0)
    assert whole.y.shape == x.shape
    flat = native.pdb_gated_scan(x.view(b * t, d), g.view(b * t, d), batch=b, h0=h0)
    assert torch.equal(flat.y.view_as(x), whole.y)
    h = h0.clone()
    for i in range(t):
        f = native.pdb_gated_scan(x[:, i], g[:, i], batch=b, h0=h, state=h)
        assert f.state is h
        torch.testing.assert_close(f.y, whole.y[:, i], rtol=1e-5, atol=1e-5)
        assert torch.equal(f.y, h)
    torch.testing.assert_close(h, whole.state, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,b", [(5000, 65, 7), (3000, 130, 2), (700, 9, 40), (2000, 5, 3)])
def test_states_in_place(gpu, n, d, b, dtype):
    """Text read in pieces: the last states written over the first ones."""
    import torch

    native = native_mod()
    rng = np.random.default_rng(n)
    x, _, g, _, starts, _, h0 = draw_scan(gpu, rng, n, d, b, "all", 0, 0, dtype)
    h = torch.from_numpy(h0).to(gpu)
    want = native.pdb_gated_scan(x, g, starts=starts, h0=h, marks=True)
    for _ in range(5):
        now = h.clone()
        f = native.pdb_gated_scan(x, g, starts=starts, h0=now, state=now, marks=True)
        assert torch.equal(f.y, want.y) and torch.equal(now, want.state) and torch.equal(f.marks, want.marks)


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_values_that_are_not_finite_stay_in_their_sequence(gpu, bad):
    import torch

    native = native_mod()
    n, d = 900, 24
    starts = torch.tensor([0, 300, 301, 620, 900], dtype=torch.int32, device=gpu)
    x, g, dy = torch.randn(3, n, d, device=gpu)
    x[350, 3] = bad
    h0 = torch.randn(4, d, device=gpu)
    h0[1, 5] = bad
    f = native.pdb_gated_scan(x, g, starts=starts, h0=h0, marks=True)
    y = f64(f.y)
    fin = np.isfinite(y)
    assert not fin[350:620, 3].any() and not fin[300, 5]
    fin[350:620, 3] = fin[300, 5] = True
    assert fin.all()
    r = native.pdb_gated_scan_grad(dy, x, g, f.marks, starts=starts, h0=h0)
    ok = np.isfinite(f64(r.dgate))
    ok[350:620, 3] = ok[300, 5] = True
    assert ok.all() and np.isfinite(f64(r.dx)).all()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("d", [24, 600])
def test_gates_that_are_not_finite(gpu, bad, d):
    """A gate that is no number behind a sequence's first row, many tiles before the end:
    its channel only, to the end of its sequence, forth and back."""
    import torch

    native = native_mod()
    n = 12_000
    starts = torch.tensor([0, 900, 1000, 5000, 5001, n], dtype=torch.int32, device=gpu)
    x, g, dy = torch.randn(3, n, d, device=gpu)
    want = native.pdb_gated_scan(x, g, starts=starts, marks=True)
    back = native.pdb_gated_scan_grad(dy, x, g, want.marks, starts=starts)
    g[1010, 3] = g[5003, 7] = bad
    status = torch.zeros(1, dtype=torch.int32, device=gpu)
    f = native.pdb_gated_scan(x, g, starts=starts, marks=True, status=status)
    r = native.pdb_gated_scan_grad(dy, x, g, f.marks, starts=starts, status=status)
    assert int(status) == 0
    for got, ref_, name in ((f.y, want.y, "y"), (r.dx, back.dx, "dx"), (r.dgate, back.dgate, "dgate")):
        same = got == ref_
        for c, a, b in ((3, 1010, 5000), (7, 5003, n)):
            lo, hi = (a, b) if name == "y" else (1000 if c == 3 else 5001, b)
            if np.isnan(bad) and name == "y":
                assert not torch.isfinite(got[lo:hi, c]).any()
            same[lo:hi, c] = True
        assert bool(same.all()), name


def test_gates_at_their_ends(gpu):
    """Gates of +-inf and far out: the state is kept, or taken from the input, exactly."""
    import torch

    native = native_mod()
    n, d = 70, 8
    x = torch.randn(n, d, device=gpu)
    h0 = torch.randn(1, d, device=gpu)
    for v in (np.inf, 200.0):
        keep = torch.full((n, d), v, device=gpu)
        f = native.pdb_gated_scan(x, keep, h0=h0, marks=True)
        assert torch.equal(f.y, h0.expand(n, d)) and torch.equal(f.marks, h0.expand(2, d))
        f = native.pdb_gated_scan(x, -keep, h0=h0, marks=True)
        assert torch.equal(f.y, x) and torch.equal(f.state[0], x[-1])
        r = native.pdb_gated_scan_grad(x, x, -keep, f.marks, h0=h0)
        assert torch.equal(r.dx, x) and not r.dgate.any() and not r.dh0.any()


@pytest.mark.parametrize("starts", [[0, 50, 40, 300], [-5, 10, 20, 300], [0, 10, 20, 301], [300, 200, 100, 0],
                                    [2 ** 31 - 1, 5, -2 ** 31, 7], [301, 400, 500, 600]])
def test_offsets_out_of_order(gpu, starts):
    """Noted in status; nothing outside the outputs is written."""
    import torch

    native = native_mod()
    n, d, b = 300, 20, 3
    x, g, dy = torch.randn(3, n, d, device=gpu)
    h0 = torch.randn(b, d, device=gpu)
    at = torch.tensor(starts, dtype=torch.int32, device=gpu)
    for grad in (False, True):
        status = torch.zeros(1, dtype=torch.int32, device=gpu)
        buf = torch.full((b + 2, d), 7.0, device=gpu)
        if grad:
            native.pdb_gated_scan_grad(dy, x, g, torch.zeros(5, d, device=gpu), starts=at, h0=h0, status=status)
        else:
            native.pdb_gated_scan(x, g, starts=at, h0=h0, state=buf[1:-1], marks=True, status=status)
            assert bool((buf[0] == 7).all()) and bool((buf[-1] == 7).all())
        assert int(status) == native.PDB_ERR_INVALID_ARG


def test_no_rows(gpu):
    import torch

    native = native_mod()
    x, h0 = torch.zeros(0, 6, device=gpu), torch.randn(3, 6, device=gpu)
    for starts in (None, torch.zeros(4, dtype=torch.int32, device=gpu)):
        f = native.pdb_gated_scan(x, x, starts=starts, batch=3, h0=h0, marks=True)
        assert torch.equal(f.state, h0) and f.marks.shape == (0, 6)
        assert not native.pdb_gated_scan(x, x, starts=starts, batch=3).state.any()
        r = native.pdb_gated_scan_grad(x, x, x, f.marks, starts=starts, batch=3, h0=h0, d_state=2 * h0)
        assert torch.equal(r.dh0, 2 * h0)
    y = torch.full((5, 6), 7.0, device=gpu)   # rows, but no sequence
    f = native.pdb_gated_scan(y, y, starts=torch.zeros(1, dtype=torch.int32, device=gpu), out=y.clone())
    assert bool((f.y == 7).all()) and f.state.shape == (0, 6)


def test_offsets_beyond_32_bits(gpu):
    import torch

    native = native_mod()
    n, d, ld = 2100, 16, 1 << 20
    buf = torch.empty(n * ld, dtype=torch.bfloat16, device=gpu)
    x, g, y = (buf.as_strided((n, d), (ld, 1), o) for o in (0, 64, 128))
    x.copy_(torch.randn(n, d, device=gpu))
    g.copy_(torch.randn(n, d, device=gpu))
    f = native.pdb_gated_scan(x, g, out=y, marks=True)
    want = native.pdb_gated_scan(x.contiguous(), g.contiguous(), marks=True)
    assert torch.equal(f.y, want.y) and torch.equal(f.state, want.state) and torch.equal(f.marks, want.marks)
    a = native.pdb_gated_scan_grad(x, x, g, f.marks)
    c = native.pdb_gated_scan_grad(x.contiguous(), x.contiguous(), g.contiguous(), f.marks)
    assert torch.equal(a.dx, c.dx) and torch.equal(a.dgate, c.dgate)


# ---------------------------------------------------------------------------
# norm and clipping

SHAPES = [[(1,)], [(5,), (0,), (3, 4), ()], [(8192,), (8193,), (16384,), (7,)], [(100, 33), (3, 9000), (1, 1)],
          [(k % 13 + 1, k % 7 + 1) for k in range(150)], [(100_003,), (2, 50_001)], [(0,)]]


def draw_grads(gpu, rng, shapes, types, pad, size=1.0):
    import torch

    out = []
    for i, s in enumerate(shapes):
        t = torch_type(types[i % len(types)])
        z = torch.from_numpy(np.asarray(rng.normal(size=s) * size)).to(gpu).to(t)
        if pad and len(s) == 2:
            wide = torch.full((s[0], s[1] + pad), 7.0, dtype=t, device=gpu)
            wide[:, :s[1]] = z
            z = wide[:, :s[1]]
        out.append(z)
    return out


@pytest.mark.parametrize("shapes", SHAPES)
@pytest.mark.parametrize("types", [["f32"], ["bf16"], ["f16", "f32", "bf16"]])
@pytest.mark.parametrize("pad", [0, 3])
def test_norm_and_clip(gpu, shapes, types, pad):
    import torch

    native = native_mod()
    rng = np.random.default_rng(len(shapes) + pad)
    grads = draw_grads(gpu, rng, shapes, types, pad)
    g64 = [f64(g) for g in grads]
    for out_types, acc, most, step, scale in ((["f32"], False, 1.0, 1.0, 1.0), (["f32"], True, 1.0, -0.1, 0.25),
                                              (types[::-1], True, 1e9, 0.5, 2.0), (types, False, np.inf, 1.0, 1.0)):
        outs = draw_grads(gpu, rng, shapes, out_types, 2 * pad)
        want, bound, res, bounds = ref.clip(g64, [f64(o) for o in outs], scale, most, step, acc)
        got = native.pdb_grad_norm(grads, scale=scale)
        assert abs(float(got) - want) <= bound
        norm = native.pdb_grad_clip(grads, most, scale=scale, out=outs, step=step, accumulate=acc)
        assert torch.equal(norm, got)
        for i, o in enumerate(outs):
            t = out_types[i % len(out_types)]
            check(f64(o), res[i], store(t, res[i], bounds[i]), (i, t))
            if pad and o.dim() == 2 and o.numel():
                wide = o.as_strided((o.shape[0], o.shape[1] + 2 * pad), o.stride())
                assert bool((wide[:, o.shape[1]:] == 7).all())
    # in place
    want, bound, res, bounds = ref.clip(g64, g64, 1.0, 0.5, 1.0, False)
    native.pdb_grad_clip(grads, 0.5)
    for i, g in enumerate(grads):
        t = types[i % len(types)]
        check(f64(g), res[i], store(t, res[i], bounds[i]), (i, t))
    before = [g.clone() for g in grads]
    native.pdb_grad_clip(grads, 1e9)          # below: nothing changes
    assert all(torch.equal(a, b) for a, b in zip(grads, before))


def test_norm_of_large_and_small_values(gpu):
    import torch

    native = native_mod()
    for v in (3e38, 1e30, 1e-30, 1e-44):
        g = torch.full((4,), v, device=gpu)
        want = 2 * float(g[0])
        got = float(native.pdb_grad_norm([g]))
        assert got == (np.inf if want > 3.41e38 else np.float32(want))
    many = torch.full((1 << 24,), 1e-3, device=gpu)
    assert abs(float(native.pdb_grad_norm([many])) / (4096 * float(many[0])) - 1) < 2 ** -24
    g = [torch.zeros(100, device=gpu)]
    assert float(native.pdb_grad_clip(g, 1.0)) == 0 and not g[0].any()
    g = [torch.randn(100, device=gpu)]
    native.pdb_grad_clip(g, 0.0)
    assert not g[0].any()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_norm_that_is_not_finite(gpu, bad):
    """Nothing is written: the step is skipped."""
    import torch

    native = native_mod()
    g = [torch.randn(300, device=gpu), torch.randn(20_000, device=gpu)]
    g[1][777] = bad
    w = [torch.randn_like(t) for t in g]
    before, old = [t.clone() for t in w], [t.clone() for t in g]
    for acc in (True, False):
        norm = float(native.pdb_grad_clip(g, 1.0, out=w, step=-0.1, accumulate=acc))
        assert np.isnan(norm) if np.isnan(bad) else norm == np.inf
        assert all(torch.equal(a, b) for a, b in zip(w, before))
    native.pdb_grad_clip(g, 1.0)
    assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(g, old))


def test_large_tensor(gpu):
    """More than 2^31 elements."""
    import torch

    native = native_mod()
    n = (1 << 31) + 12345
    g = torch.ones(n, dtype=torch.bfloat16, device=gpu)
    g[-3:] = 256.0
    want = np.sqrt(n - 3 + 3 * 65536.0)
    assert abs(float(native.pdb_grad_norm([g])) / want - 1) < 2 ** -23
    native.pdb_grad_clip([g], float(want) / 2)
    assert bool((g[:-3] == 0.5).all()) and bool((g[-3:] == 128).all())


def test_layouts_that_differ(gpu):
    """Gradients in rows further apart, outputs without gaps, and the other way round;
    tensors of other dimensions among them."""
    import torch

    native = native_mod()
    rng = np.random.default_rng(5)
    shapes = [(40, 9), (7,), (2, 3, 4), (1, 300), (300, 1), (), (90, 130)]
    for pads in ((4, 0), (0, 4), (4, 2), (0, 0)):
        g = draw_grads(gpu, rng, shapes, ["bf16", "f32"], pads[0])
        o = draw_grads(gpu, rng, shapes, ["f32"], pads[1])
        want, bound, res, bounds = ref.clip([f64(t) for t in g], [f64(t) for t in o], 1.0, 2.0, -0.1, True)
        norm = native.pdb_grad_clip(g, 2.0, out=o, step=-0.1, accumulate=True)
        assert abs(float(norm) - want) <= bound
        for i, t in enumerate(o):
            check(f64(t), res[i], bounds[i], (pads, i))
    with pytest.raises(ValueError):
        native.pdb_grad_norm([torch.zeros(4, 6, device=gpu).t()])
    with pytest.raises(ValueError):
        native.pdb_grad_norm([torch.zeros(8, device=gpu)[::2]])
    with pytest.raises(ValueError):
        native.pdb_grad_norm([torch.zeros(8, device=gpu), torch.zeros(8)])
    with pytest.raises(TypeError):
        native.pdb_grad_norm([torch.zeros(8, device=gpu), torch.zeros(8, device=gpu).double()])
    with pytest.raises(ValueError):
        native.pdb_grad_clip([torch.zeros(4, 6, device=gpu)], 1.0, out=[torch.zeros(6, 4, device=gpu)])
    w = torch.ones(4, 6, device=gpu)
    with pytest.raises(ValueError, match="twice"):
        native.pdb_grad_clip([w, w], 1.0)
    assert abs(float(native.pdb_grad_norm([w, w])) / 48 ** 0.5 - 1) < 1e-6   # to read twice is no harm
    native.pdb_grad_clip([w, w[:0], w[:0]], 1.0)   # nothing is written at the same address
    assert abs(float(native.pdb_grad_norm([w])) - 1) < 1e-6


def test_captured_layers(gpu):
    """The layer operators recorded into one graph and replayed on other values, with eager
    work between the replays: the bits of the eager calls."""
    import torch

    native = native_mod()
    n, d = 3000, 72
    starts = torch.tensor([0, 700, 700, 1999, 3000], dtype=torch.int32, device=gpu)
    x, g, dy = (t.to(torch.bfloat16) for t in torch.randn(3, n, d, device=gpu))
    h0 = torch.randn(4, d, device=gpu)
    w = [torch.randn(500, 33, device=gpu), torch.randn(d, device=gpu)]

    def calls(w):
        f = native.pdb_gated_scan(x, g, starts=starts, h0=h0, marks=True)
        r = native.pdb_gated_scan_grad(dy, x, g, f.marks, starts=starts, h0=h0)
        norm = native.pdb_grad_clip([r.dx, r.dgate, r.dh0], 0.5)
        second = native.pdb_grad_clip([t * 2 for t in w], 1.0, out=w, step=-0.1, accumulate=True)
        return [f.y, f.state, f.marks, r.dx, r.dgate, r.dh0, norm, second]

    calls([t.clone() for t in w])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls(w)
    for k in range(5):
        with torch.no_grad():
            for t in (x, g, dy):
                t.copy_(torch.randn(n, d, device=gpu))
            h0.copy_(torch.randn(4, d, device=gpu))
        eager = [t.clone() for t in w]
        want = calls(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert all(torch.equal(a, b) for a, b in zip(w, eager))


def test_memory_and_streams_of_layers(gpu):
    """On a stream of its own, while the current one still reads blocks that it has freed."""
    import torch

    native = native_mod()
    n, d = 4000, 136
    x, g, dy = torch.randn(3, n, d, device=gpu)
    big = torch.randn(4096, 4096, device=gpu)

    def calls(stream):
        f = native.pdb_gated_scan(x, g, batch=5, marks=True, stream=stream)
        r = native.pdb_gated_scan_grad(dy, x, g, f.marks, batch=5, stream=stream)
        return [f.y, f.state, f.marks, r.dx, r.dgate, native.pdb_grad_norm([x, g], stream=stream),
                native.pdb_draft_verify(x, dy[:, :1].contiguous().sigmoid(), stream=stream).tokens]

    want = [t.clone() for t in calls(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    sizes = [4 * n * d, 4 * 5 * d, 4 * d * 63, 4, 4 * n, native.pdb_gated_scan_workspace_bytes(n, d),
             native.pdb_grad_workspace_bytes(), native.pdb_draft_verify_workspace_bytes(n, 0, d)]
    for _ in range(3):
        blocks = [torch.full((s,), 7, dtype=torch.uint8, device=gpu) for s in sizes for _ in range(3)]
        torch.cuda.synchronize()
        for _ in range(8):
            big @ big
        seen = [t.clone() for t in blocks]
        del blocks
        side.wait_stream(torch.cuda.current_stream())
        got = calls(side)
        side.synchronize()
        torch.cuda.synchronize()
        assert all(bool((t == 7).all()) for t in seen)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_scans_at_once(gpu):
    """Two chains of tiles on two streams, each in a workspace of its own."""
    import torch

    native = native_mod()
    n, d = 60_000, 520
    x, g = (t.to(torch.bfloat16) for t in torch.randn(2, n, d, device=gpu))
    want = native.pdb_gated_scan(x, g, marks=True)
    back = native.pdb_gated_scan_grad(x, x, g, want.marks)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        a = native.pdb_gated_scan(x, g, marks=True, stream=streams[0])
        b = native.pdb_gated_scan_grad(x, x, g, want.marks, stream=streams[1])
        c = native.pdb_gated_scan(x, g, stream=streams[2])
        torch.cuda.synchronize()
        assert torch.equal(a.y, want.y) and torch.equal(c.y, want.y) and torch.equal(a.marks, want.marks)
        assert torch.equal(b.dx, back.dx) and torch.equal(b.dgate, back.dgate)
