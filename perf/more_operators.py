"""The measured cases of a recurrent layer and its gradient, of the norm of many
gradients with the clipped step, and of the verification of drafted tokens.

A case's ``op`` is the call that one pass makes:

  scan       pdb_gated_scan: h_t = f_t h_{t-1} + (1 - f_t) x_t, f = sigmoid(gate), in
             every channel of every sequence; the states that the sequences end with
             and, ``marks`` true, the state before every 64th row
  scan_grad  pdb_gated_scan_grad: the gradients by inputs, gates and first states
  norm       pdb_grad_norm: the norm of many tensors together
  clip       pdb_grad_clip: the tensors scaled to a norm of at most ``most``, into
             others (``acc`` false), or a step along them added to others (``acc``
             true: clipped stochastic gradient descent)
  verify     pdb_draft_verify: how many of ``k`` drafted tokens stand, and the token
             after them, from given random numbers; ``k`` 0 draws a token

Recurrence: ``n`` rows, ``d`` channels, ``b`` sequences: ``equal`` of the same length,
else of lengths that an array of offsets gives; ``empty``: some hold no row;
``first``: with first states; ``last``: with the gradient by the last ones; ``step``:
one row each, the states updated in place.  Norm and clip: ``tensors`` of ``total``
elements together, ``out`` the type of what is written.  Verification: ``b`` sequences,
``v`` logits a row, ``model`` false: the draft has no distribution (text copied from
before); ``apart``: how far its logits are from the target's; ``holes``: masked logits,
target rows without a distribution, sequences with fewer drafted tokens.  ``pad``: the
rows of a matrix are that many elements further apart than its columns need.
"""
import math
import random

import torch

own = False  # False: the plain forms below; True: the framework's operators

DEV = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
NINF = -math.inf
MARK = 64  # rows between two marks


# ---------------------------------------------------------------------------
# the cases

def _scan(op, n, d, b, dtype, equal=False, empty=False, first=False, last=False, marks=False,
          step=False, pad=0):
    return dict(op=op, n=n, d=d, b=b, dtype=dtype, equal=equal, empty=empty, first=first, last=last,
                marks=marks, step=step, pad=pad)


def _grads(op, tensors, total, dtype, out="f32", most=1.0, scale=1.0, acc=False, pad=0):
    return dict(op=op, tensors=tensors, total=total, dtype=dtype, out=out, most=most, scale=scale,
                acc=acc, pad=pad)


def _verify(b, k, v, dtype, temp=1.0, model=True, apart=0.5, idx="i32", pad=0, holes=False):
    return dict(op="verify", b=b, k=k, v=v, dtype=dtype, temp=temp, model=model, apart=apart, idx=idx,
                pad=pad, holes=holes)


def listed():
    return [
        # one decoding step of 256 sequences, their states updated in place: latency
        dict(_scan("scan", 256, 2_048, 256, "bf16", equal=True, first=True, step=True),
             name="scan-step"),
        # a training batch: texts of unequal lengths one behind another
        dict(_scan("scan", 32_768, 2_048, 24, "bf16", marks=True), name="scan-batch"),
        # a long text read at once: all the parallelism is in cutting it
        dict(_scan("scan", 131_072, 1_024, 1, "bf16", equal=True, first=True), name="scan-long"),
        # the backward pass of the training batch
        dict(_scan("scan_grad", 32_768, 2_048, 24, "bf16"), name="scan-grad-batch"),
        # odd sizes, rows further apart than their channels, empty sequences, states at
        # both ends (text cut into pieces that are trained one after another)
        dict(_scan("scan_grad", 10_007, 777, 37, "f32", empty=True, first=True, last=True, pad=23),
             name="scan-grad-odd"),
        # the two tables of a factor model of 5,003 tokens: the smallest model
        dict(_grads("norm", 2, 240_144, "f32"), name="norm-factors"),
        # the gradients of a whole model in 16 bits: matrices and many small vectors
        dict(_grads("norm", 200, 200_000_000, "bf16", scale=1 / 1024), name="norm-model"),
        # clipping into the 32-bit buffers that the optimizer reads
        dict(_grads("clip", 48, 60_000_000, "bf16"), name="clip-model"),
        # the clipped step on parameters in 32 bits: odd sizes, strided matrices
        dict(_grads("clip", 61, 30_000_001, "f32", acc=True, pad=5), name="clip-step"),
        # one token drawn for one sequence
        dict(_verify(1, 0, 131_072, "bf16", temp=0.7), name="verify-token"),
        # speculative decoding of 64 sequences, five drafted tokens each
        dict(_verify(64, 5, 131_072, "bf16"), name="verify-batch"),
        # odd vocabulary in 32 bits, masks, drafts that end early
        dict(_verify(23, 3, 50_001, "f32", temp=0.7, idx="i64", pad=31, holes=True), name="verify-odd"),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["scan", "scan", "scan_grad", "scan_grad", "norm", "clip", "verify", "verify"])
    dtype, pad = rng.choice(["f32", "bf16", "bf16", "f16"]), rng.choice([0, 0, rng.randint(1, 96)])
    if op in ("scan", "scan_grad"):
        d = rng.choice([_log(rng, 16, 4_096), 8 * _log(rng, 4, 512)])
        most = (134_000_000 if op == "scan" else 67_000_000) // (2 if dtype == "f32" else 1)
        if op == "scan" and rng.random() < 0.25:
            n = min(_log(rng, 1, 4_096), most // d)
            return _scan(op, n, d, n, dtype, True, first=True, step=True, pad=pad)
        n = min(_log(rng, 1, 131_072), most // d)
        b = _log(rng, 1, min(n, 256))
        equal = rng.random() < 0.3
        if equal:
            n -= n % b
        return _scan(op, n, d, b, dtype, equal, not equal and rng.random() < 0.5, rng.random() < 0.5,
                     op == "scan_grad" and rng.random() < 0.5, op == "scan" and rng.random() < 0.5,
                     pad=pad)
    if op in ("norm", "clip"):
        tensors = _log(rng, 1, 400 if op == "norm" else 62)
        total = max(_log(rng, 1_000, 200_000_000 if op == "norm" else 60_000_000), 2 * tensors)
        if op == "norm":
            return _grads(op, tensors, total, dtype, scale=rng.choice([1.0, 1 / 1024]), pad=pad)
        acc = rng.random() < 0.5
        return _grads(op, tensors, total, dtype, rng.choice(["f32", dtype]), rng.choice([1.0, 1e3]),
                      rng.choice([1.0, 1 / 8]), acc, pad)
    v = rng.choice([32_768, 131_072, _log(rng, 1_000, 200_000), _log(rng, 1_000, 200_000)])
    k = rng.choice([0, 1, 3, 5, 8])
    b = min(_log(rng, 1, 256), 92_000_000 // (v * (2 * k + 1)))
    return _verify(max(b, 1), k, v, dtype, rng.choice([1.0, 0.7, 2.0]), rng.random() < 0.75,
                   rng.choice([0.2, 0.5, 1.0]), rng.choice(["i32", "i64"]), pad, rng.random() < 0.4)


# ---------------------------------------------------------------------------
# inputs

def _rows(g, n, d, pad, dtype, spread=1.0, mean=0.0):
    """n x d normal values whose rows are d + pad apart."""
    x = torch.randn(n, d + pad, generator=g, device=DEV).mul_(spread).add_(mean)
    return x.to(DTYPES[dtype])[:, :d]


def _shapes(c):
    """Sizes of the tensors: spread over their logarithm, ``total`` together; rows and
    columns where rows are further apart than columns."""
    rng = random.Random(c["tensors"] * 7919 + c["total"])
    share = [math.exp(rng.gauss(0.0, 1.5)) for _ in range(c["tensors"])]
    room = c["total"] - c["tensors"]
    sizes = [1 + int(room * s / sum(share)) for s in share]
    sizes[0] += c["total"] - sum(sizes)
    if not c["pad"]:
        return [(s,) for s in sizes]
    cols = [max(1, int(s ** 0.5)) for s in sizes]
    return [(max(1, s // k), k) for s, k in zip(sizes, cols)]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = dict(case=c)
    if c["op"] in ("scan", "scan_grad"):
        n, d, b = c["n"], c["d"], c["b"]
        s["x"] = _rows(g, n, d, c["pad"], c["dtype"])
        # gates of trained layers: most keep for tens of rows, some for one, some for ever
        s["gate"] = _rows(g, n, d, c["pad"], c["dtype"], 2.0, 2.0)
        s["starts"] = None
        if not c["equal"]:
            cuts = torch.randint(0, n + 1, (b - 1,), generator=g, device=DEV)
            if c["empty"] and b > 3:
                cuts[::3] = cuts[-1]
            ends = torch.tensor([0, n], device=DEV)
            s["starts"] = torch.cat([cuts, ends]).sort().values.to(torch.int32)
        s["h0"] = torch.randn(b, d, generator=g, device=DEV) if c["first"] else None
        if c["op"] == "scan_grad":
            s["dy"] = _rows(g, n, d, c["pad"], c["dtype"])
            s["d_state"] = torch.randn(b, d, generator=g, device=DEV) if c["last"] else None
            s["marks"] = _marks(s, c, _states(s, c)[0])
    elif c["op"] in ("norm", "clip"):
        spread = 0.01 / c["scale"]
        s["grads"] = [(torch.randn(*z[:-1], z[-1] + c["pad"], generator=g, device=DEV) * spread)
                      .to(DTYPES[c["dtype"]])[..., :z[-1]] for z in _shapes(c)]
        if c["op"] == "clip":
            s["out"] = [torch.randn(z, generator=g, device=DEV).to(DTYPES[c["out"]])
                        for z in _shapes(c)]
    else:
        _prepare_verify(s, c, g)
    return s


def _prepare_verify(s, c, g):
    b, k, v = c["b"], c["k"], c["v"]
    z = s["target"] = _rows(g, b * (k + 1), v, c["pad"], c["dtype"], 3.0)
    s["u"] = torch.rand(b, k + 1, generator=g, device=DEV)
    s["draft"] = s["tokens"] = None
    if k:
        near = z.view(b, k + 1, v)[:, :k] if not c["pad"] else \
            z.as_strided((b, k, v), ((k + 1) * z.stride(0), z.stride(0), 1))
        near = near.reshape(b * k, v).float()
        q = torch.randn(b * k, v + c["pad"], generator=g, device=DEV).mul_(c["apart"])
        q[:, :v] += near
        q = q.to(DTYPES[c["dtype"]])[:, :v]
        # the drafted tokens: drawn from the draft's distribution
        e = torch.empty(b * k, v, device=DEV).exponential_(generator=g)
        t = (q.float() / c["temp"] - e.log_()).argmax(dim=1).view(b, k)
        s["tokens"] = t.to(torch.int32 if c["idx"] == "i32" else torch.int64)
        if c["model"]:
            s["draft"] = q
    if c["holes"]:
        # a mask that the draft does not know, target rows that it leaves empty, and
        # drafts that end early
        z[:, torch.rand(v, generator=g, device=DEV) < 0.125] = NINF
        z.masked_fill_((torch.rand(len(z), 1, generator=g, device=DEV) < 0.03), NINF)
        if k:
            have = torch.randint(0, 2 * k, (b, 1), generator=g, device=DEV)
            s["tokens"].masked_fill_(torch.arange(k, device=DEV) >= have, -1)


# ---------------------------------------------------------------------------
# the plain forms: 32 bits whatever the inputs' type, rounded once at the end

def _bounds(s, c):
    """First row of each sequence and the row behind its last."""
    if s["starts"] is not None:
        at = s["starts"].long()
        return at[:-1], at[1:]
    at = torch.arange(c["b"] + 1, device=DEV) * (c["n"] // c["b"])
    return at[:-1], at[1:]


def _compose(a, h):
    """h_t <- a_t h_{t-1} + h_t for all t, in place: doubling steps."""
    reach = 1
    while reach < len(h):
        h[reach:] += a[reach:] * h[:-reach]
        a[reach:] *= a[:-reach].clone()
        reach *= 2
    return h


def _states(s, c):
    """The states h after every row, and the states before."""
    first, end = _bounds(s, c)
    f = torch.sigmoid(s["gate"].float())
    h = torch.sigmoid(-s["gate"].float()) * s["x"].float()
    some = first < end
    enter = torch.zeros(c["b"], c["d"], device=DEV) if s["h0"] is None else s["h0"]
    h[first[some]] += f[first[some]] * enter[some]
    f[first[some]] = 0.0
    h = _compose(f, h)
    before = torch.zeros_like(h)
    before[1:] = h[:-1]
    before[first[some]] = enter[some]
    return h, before


def _marks(s, c, h):
    first, end = _bounds(s, c)
    some = first < end
    before = torch.zeros_like(h)
    before[1:] = h[:-1]
    before[first[some]] = 0.0 if s["h0"] is None else s["h0"][some]
    return before[::MARK].contiguous()


def _plain_scan(s, c):
    first, end = _bounds(s, c)
    if c["step"]:  # one row a sequence: the recurrence itself
        f = torch.sigmoid(s["gate"].float())
        h = f * s["h0"] + torch.sigmoid(-s["gate"].float()) * s["x"].float()
        s["h0"].copy_(h)
        return dict(y=h.to(s["x"].dtype), state=s["h0"])
    h, before = _states(s, c)
    state = h[(end - 1).clamp(min=0)]
    none = torch.zeros_like(state) if s["h0"] is None else s["h0"]
    r = dict(y=h.to(s["x"].dtype), state=torch.where((first < end).unsqueeze(1), state, none))
    if c["marks"]:
        r["marks"] = before[::MARK].contiguous()
    return r


def _plain_scan_grad(s, c):
    first, end = _bounds(s, c)
    some = first < end
    _, before = _states(s, c)
    x, dy = s["x"].float(), s["dy"].float()
    f, keep = torch.sigmoid(s["gate"].float()), torch.sigmoid(-s["gate"].float())
    # from the last row to the first: e_t = dy_t + f_{t+1} e_{t+1}
    a = torch.zeros_like(f)
    a[:-1] = f[1:]
    a[end[some] - 1] = 0.0
    e = dy.clone() if dy.data_ptr() == s["dy"].data_ptr() else dy
    if s["d_state"] is not None:
        e[end[some] - 1] += s["d_state"][some]
    e = _compose(a.flip(0), e.flip(0)).flip(0)
    r = dict(dx=(keep * e).to(s["x"].dtype), dgate=(e * (before - x) * (f * keep)).to(s["x"].dtype))
    if s["h0"] is not None:
        d0 = torch.zeros_like(s["h0"]) if s["d_state"] is None else s["d_state"].clone()
        d0[some] = f[first[some]] * e[first[some]]
        r["dh0"] = d0
    return r


def _plain_norm(s, c):
    # a sum of up to 2e8 squares: in 64 bits
    return abs(c["scale"]) * torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()


def _plain_clip(s, c):
    norm = _plain_norm(s, c)
    factor = (c["scale"] * (c["most"] / norm).clamp(max=1.0)).float()
    for g, o in zip(s["grads"], s["out"]):
        if c["acc"]:
            o.copy_(o.float() - 0.01 * factor * g.float())
        else:
            o.copy_(factor * g.float())
    return dict(norm=norm.float(), out=s["out"])


def _weights64(z, temp):
    """exp((z - max) / temp) in 64 bits and its sum: the choices below stand next to
    borders.  Logits 700 temperatures below the largest count as -inf."""
    z = z.double()
    m = z.max(dim=-1, keepdim=True).values
    y = (z - torch.where(m == NINF, torch.zeros_like(m), m)) / temp
    e = torch.where(y < -700.0, torch.zeros_like(y), y.exp())
    return e, e.sum(dim=-1, keepdim=True)


def _plain_verify(s, c):
    b, k, v, u = c["b"], c["k"], c["v"], s["u"].double()
    e, total = _weights64(s["target"], c["temp"])
    p = (e / torch.where(total == 0, torch.ones_like(total), total)).view(b, k + 1, v)
    rows = torch.arange(b, device=DEV)
    at, drawn_from = torch.zeros(b, dtype=torch.int64, device=DEV), p[:, 0]
    if k:
        t = s["tokens"].long()
        x = t.clamp(min=0).unsqueeze(2)
        px, q = p[:, :k].gather(2, x).squeeze(2), None
        if s["draft"] is not None:
            eq, tq = _weights64(s["draft"], c["temp"])
            q = (eq / torch.where(tq == 0, torch.ones_like(tq), tq)).view(b, k, v)
        qx = torch.ones_like(px) if q is None else q.gather(2, x).squeeze(2)
        good = (t >= 0) & (u[:, :k] * qx < px)
        at = good.long().cumprod(dim=1).sum(dim=1)
        # what a refused token leaves: the part of p that the draft has too little of
        j = at.clamp(max=k - 1)
        here = p[rows, at]
        left = here.clone().scatter_(1, x[rows, j], 0.0) if q is None else \
            (here - q[rows, j]).clamp(min=0.0)
        refused = (at < k) & (t[rows, j] >= 0) & (left.sum(dim=1) > 0)
        drawn_from = torch.where(refused.unsqueeze(1), left, here)
    run = drawn_from.cumsum(dim=1)
    some = drawn_from > 0
    last = torch.where(some, torch.arange(v, device=DEV), -1).max(dim=1).values
    next_ = (run <= (u[:, k] * run[:, -1]).unsqueeze(1)).sum(dim=1).minimum(last)
    out = torch.full((b, k + 1), -1, dtype=torch.int32, device=DEV)
    if k:
        out[:, :k] = s["tokens"].masked_fill(torch.arange(k, device=DEV) >= at.unsqueeze(1), -1)
    out[rows, at] = next_.to(torch.int32)
    return dict(tokens=out, accepted=at.to(torch.int32))


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        return {"scan": _plain_scan, "scan_grad": _plain_scan_grad, "norm": _one(_plain_norm),
                "clip": _plain_clip, "verify": _plain_verify}[op](s, c)
    from paper_1508_00703_amd import native

    if op == "scan":
        f = native.pdb_gated_scan(s["x"], s["gate"], starts=s["starts"], batch=c["b"], h0=s["h0"],
                                  state=s["h0"] if c["step"] else None, marks=c["marks"])
        r = dict(y=f.y, state=f.state)
        return dict(r, marks=f.marks) if c["marks"] else r
    if op == "scan_grad":
        g = native.pdb_gated_scan_grad(s["dy"], s["x"], s["gate"], s["marks"], starts=s["starts"],
                                       batch=c["b"], h0=s["h0"], d_state=s["d_state"])
        r = dict(dx=g.dx, dgate=g.dgate)
        return r if s["h0"] is None else dict(r, dh0=g.dh0)
    if op == "norm":
        return native.pdb_grad_norm(s["grads"], scale=c["scale"])
    if op == "clip":
        norm = native.pdb_grad_clip(s["grads"], c["most"], scale=c["scale"], out=s["out"],
                                    step=-0.01 if c["acc"] else 1.0, accumulate=c["acc"])
        return dict(norm=norm, out=s["out"])
    f = native.pdb_draft_verify(s["target"], s["u"], tokens=s["tokens"], draft=s["draft"],
                                temp=c["temp"])
    return dict(tokens=f.tokens, accepted=f.accepted)


def _one(f):
    return lambda s, c: f(s, c).float()


# ---------------------------------------------------------------------------
# what one pass cannot do without

def work(case):
    c = case
    if c["op"] in ("scan", "scan_grad"):
        cells, ends = c["n"] * c["d"], c["b"] * c["d"] * 4
        if c["op"] == "scan":
            size = 3 * cells * SIZE[c["dtype"]] + ends * (2 if c["first"] else 1)
            if c["marks"]:
                size += 4 * c["d"] * -(-c["n"] // MARK)
            return dict(bytes=size, flops=8 * cells)
        size = 5 * cells * SIZE[c["dtype"]] + ends * (2 * c["first"] + c["last"])
        return dict(bytes=size, flops=16 * cells)
    if c["op"] in ("norm", "clip"):
        n = sum(math.prod(z) for z in _shapes(c))
        if c["op"] == "norm":
            return dict(bytes=n * SIZE[c["dtype"]], flops=2 * n)
        return dict(bytes=n * (SIZE[c["dtype"]] + SIZE[c["out"]] * (2 if c["acc"] else 1)),
                    flops=4 * n)
    rows = c["b"] * (c["k"] + 1 + (c["k"] if c["model"] else 0))
    return dict(bytes=rows * c["v"] * SIZE[c["dtype"]], flops=4 * rows * c["v"])


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def _walk(a, h):
    """h_t <- a_t h_{t-1} + h_t row by row: inside stretches side by side, then over them."""
    n, d = h.shape
    long = max(1, math.isqrt(n))
    rows = -(-n // long) * long
    a = torch.nn.functional.pad(a, (0, 0, 0, rows - n)).view(-1, long, d)
    h = torch.nn.functional.pad(h, (0, 0, 0, rows - n)).view(-1, long, d)
    for t in range(1, long):
        h[:, t] += a[:, t] * h[:, t - 1]
        a[:, t] *= a[:, t - 1]
    for i in range(1, len(h)):
        h[i] += a[i] * h[i - 1, -1]
    return h.reshape(rows, d)[:n]


def _exact_scan(s, c):
    first, end = (t.tolist() for t in _bounds(s, c))
    x, f = s["x"].double(), 1.0 / (1.0 + (-s["gate"].double()).exp())
    keep = 1.0 / (1.0 + s["gate"].double().exp())
    start = [torch.zeros(c["d"], dtype=torch.float64, device=DEV) if s["h0"] is None else
             s["h0"][i].double() for i in range(c["b"])]
    used = [i for i in range(c["b"]) if first[i] < end[i]]
    at = torch.tensor([first[i] for i in used], device=DEV)
    enter = torch.stack([start[i] for i in used])
    a, h = f.clone(), keep * x
    h[at] += f[at] * enter
    a[at] = 0.0
    h = _walk(a, h)
    before = torch.roll(h, 1, 0)
    before[at] = enter
    if c["op"] == "scan":
        r = dict(y=h, state=torch.stack([h[end[i] - 1] if first[i] < end[i] else start[i]
                                         for i in range(c["b"])]))
        return dict(r, marks=before[::MARK]) if c["marks"] else r
    e, a = s["dy"].double(), torch.roll(f, -1, 0)
    tail = torch.tensor([end[i] - 1 for i in used], device=DEV)
    if s["d_state"] is not None:
        e[tail] += s["d_state"][torch.tensor(used, device=DEV)].double()
    a[tail] = 0.0
    e = _walk(a.flip(0), e.flip(0)).flip(0)
    r = dict(dx=keep * e, dgate=e * (before - x) * f * keep)
    if s["h0"] is not None:
        d0 = [torch.zeros_like(start[0]) if s["d_state"] is None else s["d_state"][i].double()
              for i in range(c["b"])]
        for i in used:
            d0[i] = f[first[i]] * e[first[i]]
        r["dh0"] = torch.stack(d0)
    return r


def exact(case, seed):
    c = case
    if c["op"] == "verify":
        return None  # whole numbers: equal or not
    s = prepare(case, seed)
    if c["op"] in ("scan", "scan_grad"):
        return _exact_scan(s, c)
    squares = [torch.linalg.vector_norm(g.double()).item() for g in s["grads"]]
    norm = abs(c["scale"]) * math.hypot(*squares)
    if c["op"] == "norm":
        return torch.tensor(norm, dtype=torch.float64, device=DEV)
    by = c["scale"] * min(1.0, c["most"] / norm) * (-0.01 if c["acc"] else 1.0)
    return dict(norm=torch.tensor(norm, dtype=torch.float64, device=DEV),
                out=[by * g.double() + (o.double() if c["acc"] else 0.0)
                     for g, o in zip(s["grads"], s["out"])])
