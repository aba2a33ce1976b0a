"""The gates of the recurrence over their whole range, forth, back and in the decoding
step: every finite value of the 16-bit types, and binary32 values densely around +-87 to
+-89, where exp(-gate) passes from 2^126 to beyond binary32's range.

The bounds are tighter than layerref's where a gate is far out.  With u = 2^-24, s the
smaller one of f and k = 1 - f, and eg = (2 |g| + 8) u as there (the error of
s = t / (1 + t), relatively):

* the larger one is 1 / (1 + t): off by s eg through t, and by the roundings of the sum
  (u), the reciprocal (2 u) and a product (u).  So f is within s eg + 4 u f of the true
  one, k within s eg + 4 u k;
* h' = f h + k x: two roundings more of either product and their sum, and three where
  rows are joined through maps;
* results, and parts of them, below binary32's normal numbers are lost."""
import numpy as np
import pytest

import layerref as ref
from test_gpu_layers import store
from test_gpu_tokens import DTYPES, check, f64, native_mod, on_gpu, torch_type

U, LEAST = ref.U, ref.LEAST


def all_gates(dtype):
    """Finite gates of the type, as 256 columns."""
    import torch

    if dtype != "f32":
        bits = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16)
        g = bits.view(torch_type(dtype)).double().numpy()
        g = g[np.isfinite(g)]
    else:
        ends = [p * np.log(2.0) for p in (100, 125, 126, 127, 128, 149)]
        near = np.concatenate([np.float32(e) + np.arange(-512, 512) * np.spacing(np.float32(e)) for e in ends])
        g = np.concatenate([np.linspace(-150, 150, 40_001), np.linspace(86, 90, 20_001),
                            -np.linspace(86, 90, 20_001), near, -near, [0.0, 1e-30, -1e-30, 1e30, -1e30, 3e38, -3e38]])
        g = np.float32(g).astype(np.float64)
    return np.resize(g, -(-len(g) // 256) * 256).reshape(-1, 256)


def spread(g):
    """(f, k, and what they may be off by)."""
    f, k, eg = ref.gates(g)
    far = np.where(np.abs(g) > 150, 0.0, eg) * np.minimum(f, k)
    return f, k, far + 4 * U * f, far + 4 * U * k


def forth(x, g, h0):
    """States [b, t, d] of sequences of equal length, those before, and their bounds."""
    f, k, ef, ek = spread(g)
    h, err = h0, np.zeros_like(h0)
    y, before, by, bb = (np.zeros_like(x) for _ in range(4))
    for t in range(x.shape[1]):
        before[:, t], bb[:, t] = h, err
        mag = f[:, t] * np.abs(h) + k[:, t] * np.abs(x[:, t])
        err = f[:, t] * err + ef[:, t] * (np.abs(h) + err) + ek[:, t] * np.abs(x[:, t]) + 5 * U * mag + LEAST
        h = f[:, t] * h + k[:, t] * x[:, t]
        y[:, t], by[:, t] = h, err
    return y, before, by, bb


def back(dy, x, g, h0, ds):
    """dict of dx, dgate, dh0 and their bounds."""
    f, k, ef, ek = spread(g)
    _, before, _, bb = forth(x, g, h0)
    r = {n: np.zeros_like(x) for n in ("dx", "dgate", "bdx", "bdgate")}
    e, err = ds, np.zeros_like(ds)
    for t in range(x.shape[1] - 1, -1, -1):
        err = err + 2 * U * (np.abs(dy[:, t]) + np.abs(e))
        e = dy[:, t] + e
        ft, kt, gap = f[:, t], k[:, t], before[:, t] - x[:, t]
        r["dx"][:, t] = kt * e
        r["bdx"][:, t] = kt * err + ek[:, t] * (np.abs(e) + err) + U * kt * np.abs(e) + LEAST
        # the product of both gates: the smaller one's error and the larger one's
        both = ft * ek[:, t] + kt * ef[:, t] + 4 * U * ft * kt
        wide = bb[:, t] + U * np.abs(gap)
        r["dgate"][:, t] = e * gap * ft * kt
        r["bdgate"][:, t] = (both * (np.abs(e) + err) * (np.abs(gap) + wide)
                             + ft * kt * (err * (np.abs(gap) + wide) + np.abs(e) * wide) + LEAST)
        err = ft * err + ef[:, t] * (np.abs(e) + err) + 3 * U * ft * np.abs(e) + LEAST
        e = ft * e
    r["dh0"], r["bdh0"] = e, err
    return r


def test_bounds_against_a_computation_in_32_bits():
    """The formulas in numpy's 32 bits, by |g|, stay inside the bounds."""
    rng = np.random.default_rng(0)
    g = all_gates("f32")[:, None].repeat(3, 1)
    x, dy = rng.normal(size=(2, *g.shape)).astype(np.float32).astype(np.float64)
    h0, ds = rng.normal(size=(2, len(g), 256)).astype(np.float32).astype(np.float64)
    y, _, by, _ = forth(x, g, h0)
    want = back(dy, x, g, h0, ds)
    with np.errstate(all="ignore"):
        s = np.exp2(np.abs(g).astype(np.float32) * np.float32(-np.log2(np.e)))
        r = 1 / (1 + s)
        f, k = np.where(g >= 0, r, s * r), np.where(g >= 0, s * r, r)
        x32, h, e = x.astype(np.float32), h0.astype(np.float32), ds.astype(np.float32)
        gap = []
        for t in range(3):
            gap.append(h - x32[:, t])
            h = f[:, t] * h + k[:, t] * x32[:, t]
            check(h, y[:, t], by[:, t], ("y", t))
        for t in (2, 1, 0):
            e = dy[:, t].astype(np.float32) + e
            check(k[:, t] * e, want["dx"][:, t], want["bdx"][:, t], ("dx", t))
            check(gap[t] * (k[:, t] * (f[:, t] * e)), want["dgate"][:, t], want["bdgate"][:, t], ("dgate", t))
            e = f[:, t] * e
        check(e, want["dh0"], want["bdh0"], "dh0")


def draw(gpu, dtype, rows):
    """Gates of every value at each of `rows` places of a sequence, the others drawn."""
    rng = np.random.default_rng(rows)
    g = all_gates(dtype)
    b = len(g)
    gates = rng.normal(size=(rows * b, rows, 256)) * 2
    for t in range(rows):
        gates[t * b:(t + 1) * b, t] = g
        if t:
            gates[t * b:(t + 1) * b, t - 1] = g[::-1, ::-1]
    n = rows * b * rows
    out = [on_gpu(z.reshape(n, 256), dtype, gpu) for z in (gates, *rng.normal(size=(2, *gates.shape)))]
    h0, ds = rng.normal(size=(2, rows * b, 256)).astype(np.float32)
    return out, h0, ds, gates.shape


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_decoding_step(gpu, dtype):
    import torch

    ((g, g64), (x, x64), _), h0, _, shape = draw(gpu, dtype, 1)
    h = torch.from_numpy(h0).to(gpu)
    f = native_mod().pdb_gated_scan(x, g, batch=len(h), h0=h)
    y, _, by, _ = forth(x64.reshape(shape), g64.reshape(shape), h0.astype(np.float64))
    check(f64(f.state), y[:, 0], by[:, 0], "state")
    check(f64(f.y), y[:, 0], store(dtype, y[:, 0], by[:, 0]), "y")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_sequences(gpu, dtype):
    import torch

    native = native_mod()
    ((g, g64), (x, x64), (dy, dy64)), h0, ds, shape = draw(gpu, dtype, 3)
    h, d = torch.from_numpy(h0).to(gpu), torch.from_numpy(ds).to(gpu)
    x64, g64, dy64 = (z.reshape(shape) for z in (x64, g64, dy64))
    y, _, by, _ = forth(x64, g64, h0.astype(np.float64))
    f = native.pdb_gated_scan(x, g, batch=len(h), h0=h, marks=True)
    check(f64(f.y).reshape(shape), y, store(dtype, y, by), "y")
    check(f64(f.state), y[:, -1], by[:, -1], "state")
    want = back(dy64, x64, g64, h0.astype(np.float64), ds.astype(np.float64))
    r = native.pdb_gated_scan_grad(dy, x, g, f.marks, batch=len(h), h0=h, d_state=d)
    for name in ("dx", "dgate"):
        check(f64(getattr(r, name)).reshape(shape), want[name], store(dtype, want[name], want["b" + name]), name)
    check(f64(r.dh0), want["dh0"], want["bdh0"], "dh0")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [5, 24, 600])
def test_a_gate_that_is_no_number(gpu, dtype, d):
    """What hangs on it is no number either, the gradient by its own row's input among it;
    the rest keeps its bits."""
    import torch

    native = native_mod()
    n, at, col = 3000, 1010, 3
    starts = torch.tensor([0, 900, 1000, 2500, n], dtype=torch.int32, device=gpu)
    x, g, dy = (t.to(torch_type(dtype)) for t in torch.randn(3, n, d, device=gpu))
    h0 = torch.randn(4, d, device=gpu)

    def calls():
        f = native.pdb_gated_scan(x, g, starts=starts, h0=h0, marks=True)
        r = native.pdb_gated_scan_grad(dy, x, g, f.marks, starts=starts, h0=h0)
        step = native.pdb_gated_scan(x, g, batch=n)
        return dict(y=f.y, state=f.state, dx=r.dx, dgate=r.dgate, dh0=r.dh0, step=step.y)

    want = calls()
    g[at, col] = np.nan
    got = calls()
    lost = {name: torch.zeros_like(t, dtype=torch.bool) for name, t in want.items()}
    lost["y"][at:2500, col] = lost["state"][2, col] = True     # from its row to the sequence's end
    lost["dx"][1000:at + 1, col] = lost["dh0"][2, col] = True  # from its row to the beginning
    lost["dgate"][1000:2500, col] = True                       # before it by e, behind it by h
    lost["step"][at, col] = True
    for name, t in got.items():
        assert torch.equal(t.isnan(), lost[name]), name
        assert torch.equal(t[~lost[name]], want[name][~lost[name]]), name
