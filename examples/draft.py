"""Recurrent next-token models, one drafting for the other, with the layer and token
operators.

A model reads a token by two rows of tables, an input and its gate; a gated recurrence
carries them along the text, and the state times the output factors are the logits of
what follows.  A large model learns from a synthetic text in which a token depends on
the two before it; a small one learns from the large one's best alternatives; every
step is clipped by the norm of all its gradients.  Then text is drawn from the large
model, one token at a time, and with the small one drafting several that the large one
verifies in one pass: the same distribution, in fewer passes.

    python examples/draft.py                       # 503 tokens, 128 -> 32 channels
    python examples/draft.py --vocabulary 5003 --batch 64
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1508_00703_amd import native  # noqa: E402


class Recurrent:
    """Tables in float32; activations in float32, so that an output is a state."""

    def __init__(self, vocabulary, d, gen, device):
        self.inp, self.gate, self.out = (torch.randn(vocabulary, d, generator=gen, device=device) / d ** 0.5
                                         for _ in range(3))

    @property
    def tables(self):
        return [self.inp, self.gate, self.out]

    def read(self, tokens, state=None, marks=False):
        """Tokens [b, t] behind the state [b, d]: their inputs, gates and the scan."""
        x, g = native.pdb_embed_lookup(self.inp, tokens), native.pdb_embed_lookup(self.gate, tokens)
        return x, g, native.pdb_gated_scan(x, g, h0=state, marks=marks)

    def logits(self, y):
        return y.reshape(-1, y.shape[-1]) @ self.out.t()

    def gradients(self, tokens, x, g, scan, dz):
        """Those of the tables, from the logits' (rows as the tokens)."""
        dy = (dz @ self.out).view_as(x)
        s = native.pdb_gated_scan_grad(dy, x, g, scan.marks)
        return [native.pdb_embed_grad(s.dx, tokens, torch.empty_like(self.inp)),
                native.pdb_embed_grad(s.dgate, tokens, torch.empty_like(self.gate)),
                dz.t() @ scan.y.reshape(-1, x.shape[-1])]

    def step(self, grads, lr, max_norm):
        """The clipped step, in place; the norm."""
        return native.pdb_grad_clip(grads, max_norm, out=self.tables, step=-lr, accumulate=True)


def draw_text(vocabulary, b, t, gen, device):
    """b texts of t + 1 tokens: each follows from the two before it, by one of four rules."""
    x = torch.randint(0, vocabulary, (b, t + 1), generator=gen, device=device)
    turn = torch.rand(b, t + 1, generator=gen, device=device).clamp_min_(1 / 16).log2_().neg_().long()
    for i in range(2, t + 1):
        x[:, i] = (x[:, i - 1] * 5 + x[:, i - 2] % 7 + 1 + turn[:, i].clamp(max=3) * (vocabulary // 5)) % vocabulary
    return x


def learn_from_text(model, text, lr, max_norm):
    """One step of likelihood; (mean log probability, norm of the gradients)."""
    tokens, after = text[:, :-1].contiguous(), text[:, 1:].reshape(-1)
    x, g, scan = model.read(tokens, marks=True)
    z = model.logits(scan.y)
    f = native.pdb_token_logprobs(z, after)
    weight = torch.full_like(f.logp, -1.0 / len(f.logp))
    dz = native.pdb_token_logprobs_grad(z, after, f.stats, weight, out=z)
    return f.logp.mean(), model.step(model.gradients(tokens, x, g, scan, dz), lr, max_norm)


def learn_from_teacher(model, teacher, text, top, lr, max_norm):
    """One step on the teacher's best alternatives; (mean divergence, norm)."""
    tokens = text[:, :-1].contiguous()
    told = native.pdb_token_logprobs(teacher.logits(teacher.read(tokens)[2].y), top=top)
    x, g, scan = model.read(tokens, marks=True)
    z = model.logits(scan.y)
    weight = torch.full((len(z),), 1.0 / len(z), device=z.device)
    loss, dz = native.pdb_distill(z, told.top_id, told.top_logp, weight=weight, out=z)
    return loss.sum(), model.step(model.gradients(tokens, x, g, scan, dz), lr, max_norm)


def draw(model, token, state, u):
    """The next token [b, 1] of each sequence; the states go on in place."""
    x, g = (native.pdb_embed_lookup(w, token.view(-1)) for w in (model.inp, model.gate))
    h = native.pdb_gated_scan(x, g, batch=len(x), h0=state, state=state)
    z = model.logits(h.y)
    return native.pdb_draft_verify(z, u).tokens, z


def draft_and_verify(model, small, k, token, state, small_state, gen):
    """Up to k + 1 tokens of each sequence, in one pass of the model: (tokens [b, k + 1],
    -1 behind, how many were accepted); token [b, 1] and the states go on in place."""
    b = len(token)
    u = torch.rand(b, k + 1, generator=gen, device=token.device)
    at, said, ahead, z = small_state.clone(), [], token, []
    for _ in range(k):
        ahead, logits = draw(small, ahead, at, torch.rand(b, 1, generator=gen, device=token.device))
        said.append(ahead)
        z.append(logits)
    drafted = torch.cat(said, 1)
    read = torch.cat([token, drafted], 1)
    y = model.read(read, state)[2].y
    f = native.pdb_draft_verify(model.logits(y), u, tokens=drafted, draft=torch.stack(z, 1).view(b * k, -1))
    # the states behind the last token that stands
    rows, n = torch.arange(b, device=token.device), f.accepted.long()
    state.copy_(y[rows, n])
    small_state.copy_(small.read(read, small_state)[2].y[rows, n])
    token.copy_(f.tokens.gather(1, n.unsqueeze(1)))
    return f.tokens, f.accepted


def run(vocabulary=503, batch=32, length=48, steps=600, channels=128, small_channels=32, top=20, k=4, lr=100.0,
        max_norm=0.05, passes=32, seed=1, report=print):
    device = torch.device("cuda", 0)
    gen = torch.Generator(device=device).manual_seed(seed)
    model, small = (Recurrent(vocabulary, d, gen, device) for d in (channels, small_channels))
    result = {}

    def score(m, text):
        z = m.logits(m.read(text[:, :-1].contiguous())[2].y)
        return float(native.pdb_token_logprobs(z, text[:, 1:].reshape(-1)).logp.mean())

    test = draw_text(vocabulary, batch, length, gen, device)
    result["start"] = score(model, test), score(small, test)
    for i in range(steps):
        logp, norm = learn_from_text(model, draw_text(vocabulary, batch, length, gen, device), lr, max_norm)
        if report and i % 100 == 99:
            report("model step %4d  log probability %.3f, norm %.3f" % (i + 1, float(logp), float(norm)))
    for i in range(steps):
        loss, norm = learn_from_teacher(small, model, draw_text(vocabulary, batch, length, gen, device), top, lr,
                                        max_norm)
        if report and i % 100 == 99:
            report("small step %4d  divergence %.3f, norm %.3f" % (i + 1, float(loss), float(norm)))
    result["end"] = score(model, test), score(small, test)

    token = test[:, :1].to(torch.int32).contiguous()
    state, small_state = (torch.zeros(batch, d, device=device) for d in (channels, small_channels))
    counts, tokens = [], []
    for _ in range(passes):
        said, accepted = draft_and_verify(model, small, k, token, state, small_state, gen)
        tokens.append(said)
        counts.append(accepted)
    result["accepted"] = float(torch.stack(counts).float().mean())
    result["tokens"] = torch.cat(tokens, 1)
    if report:
        report("unseen text, log probability: model %.3f -> %.3f, small %.3f -> %.3f"
               % (result["start"][0], result["end"][0], result["start"][1], result["end"][1]))
        report("%d passes with %d drafted: %.2f tokens a pass" % (passes, k, 1 + result["accepted"]))
    return result


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocabulary", type=int, default=503)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--length", type=int, default=48)
    ap.add_argument("--steps", type=int, default=600)
    ap.add_argument("--channels", type=int, default=128)
    ap.add_argument("--small-channels", type=int, default=32)
    ap.add_argument("--top", type=int, default=20)
    ap.add_argument("--drafted", type=int, default=4)
    ap.add_argument("--lr", type=float, default=100.0)
    ap.add_argument("--max-norm", type=float, default=0.05)
    ap.add_argument("--seed", type=int, default=1)
    a = ap.parse_args()
    run(a.vocabulary, a.batch, a.length, a.steps, a.channels, a.small_channels, a.top, a.drafted, a.lr,
        a.max_norm, seed=a.seed)


if __name__ == "__main__":
    main()
