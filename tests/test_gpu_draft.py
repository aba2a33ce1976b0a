"""The example runs the layer and token operators together: its gradients are those of the
same model in 64 bits, and what it serves is what its models say."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def draft():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import draft
    finally:
        sys.path.pop(0)
    return draft


def model64(tables, text):
    """Mean log probability of a text, by the plain recurrence, differentiable."""
    import torch

    inp, gate, out = tables
    b, t = text.shape
    h, total = torch.zeros(b, inp.shape[1], dtype=torch.float64), 0.0
    for i in range(t - 1):
        f = torch.sigmoid(gate[text[:, i]])
        h = f * h + (1 - f) * inp[text[:, i]]
        total = total + torch.log_softmax(h @ out.t(), 1).gather(1, text[:, i + 1:i + 2]).sum()
    return total / (b * (t - 1))


def test_gradients_and_clipped_step(gpu, draft):
    import torch

    gen = torch.Generator(device=gpu).manual_seed(3)
    m = draft.Recurrent(61, 24, gen, gpu)
    text = draft.draw_text(61, 7, 150, gen, gpu)
    tables = [w.double().cpu().requires_grad_() for w in m.tables]
    logp = model64(tables, text.cpu())
    want = torch.autograd.grad(-logp, tables)
    tokens, after = text[:, :-1].contiguous(), text[:, 1:].reshape(-1)
    native = draft.native
    x, g, scan = m.read(tokens, marks=True)
    z = m.logits(scan.y)
    f = native.pdb_token_logprobs(z, after)
    assert abs(float(f.logp.double().mean()) - float(logp.detach())) < 1e-5
    dz = native.pdb_token_logprobs_grad(z, after, f.stats, torch.full_like(f.logp, -1.0 / len(f.logp)))
    got = m.gradients(tokens, x, g, scan, dz)
    # sums of some thousand terms in 32 bits, through products over 24 and 61 entries
    for a, b in zip(got, want):
        assert float((a.double().cpu() - b).abs().max()) < 1e-4 * float(b.abs().max())
    # and along a direction, against differences
    way = [torch.randn(w.shape, dtype=torch.float64, generator=torch.Generator().manual_seed(k))
           for k, w in enumerate(tables)]
    slope = sum((a.double().cpu() * v).sum() for a, v in zip(got, way))
    with torch.no_grad():
        up, down = (model64([w + s * v for w, v in zip(tables, way)], text.cpu()) for s in (1e-6, -1e-6))
    assert abs(float(-(up - down) / 2e-6 - slope)) < 1e-3 * abs(float(slope)) + 1e-5
    norm = torch.stack([w.square().sum() for w in want]).sum().sqrt()
    before = [w.clone() for w in m.tables]
    got_norm = m.step(got, 0.5, float(norm) / 3)
    assert abs(float(got_norm) / float(norm) - 1) < 1e-4
    for w, old, d in zip(m.tables, before, want):
        step = -0.5 / 3 * d
        assert float(((w - old).double().cpu() - step).abs().max()) < 1e-3 * float(step.abs().max()) + 1e-6


def test_a_model_drafting_for_itself(gpu, draft):
    """Its drafted tokens are accepted but for rounding, and the states it leaves are
    those of reading what was said."""
    import torch

    gen = torch.Generator(device=gpu).manual_seed(4)
    m = draft.Recurrent(97, 40, gen, gpu)
    b, k = 16, 5
    token = torch.randint(0, 97, (b, 1), generator=gen, device=gpu, dtype=torch.int32)
    first, state = token.clone(), torch.zeros(b, 40, device=gpu)
    small = state.clone()
    heard = [[int(t)] for t in first]
    accepted = 0
    for _ in range(6):
        said, n = draft.draft_and_verify(m, m, k, token, state, small, gen)
        accepted += int(n.sum())
        for i in range(b):
            heard[i] += said[i, :int(n[i]) + 1].tolist()
            assert (said[i, int(n[i]) + 1:] == -1).all() and heard[i][-1] == int(token[i])
    assert accepted >= 6 * b * k - 2
    for i in range(b):
        text = torch.tensor([heard[i][:-1]], device=gpu)
        h = m.read(text)[2].state
        torch.testing.assert_close(h[0], state[i], rtol=1e-4, atol=1e-5)
        torch.testing.assert_close(h[0], small[i], rtol=1e-4, atol=1e-5)


def test_run(gpu, draft):
    lines = []
    r = draft.run(vocabulary=101, batch=8, length=20, steps=3, channels=24, small_channels=16, top=5, k=3, passes=4,
                  report=lines.append)
    t = r["tokens"]
    assert t.shape == (8, 16) and int(t.max()) < 101 and int(t.min()) >= -1
    assert 0 <= r["accepted"] <= 3 and len(lines) == 2
    again = draft.run(vocabulary=101, batch=8, length=20, steps=3, channels=24, small_channels=16, top=5, k=3, passes=4,
                      report=None)
    assert again["start"] == r["start"]


def test_command(gpu):
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "draft.py"), "--vocabulary", "101", "--batch",
                          "8", "--length", "24", "--steps", "100"], check=True, capture_output=True, text=True,
                         timeout=100).stdout
    assert "small step  100" in out and "tokens a pass" in out and "nan" not in out
