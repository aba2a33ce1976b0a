"""Next-token factor models that learn from one another, with the token operators.

A model is two tables: the factors that a token is read by and those that it is
predicted by; the logits of what follows token x are its input factors times every
output factor.  A teacher learns from a synthetic text by likelihood (with an
entropy reward, which keeps it from being too sure).  A student of fewer factors
then learns from the teacher's best alternatives alone, and both are scored on text
that neither has seen and go on from one token, greedily.

    python examples/distill.py                      # 5,003 tokens, 64 -> 24 factors
    python examples/distill.py --vocabulary 50001 --batch 8192
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1508_00703_amd import native  # noqa: E402


class Factors:
    """Tables in float32; logits and their gradients in bf16."""

    def __init__(self, vocabulary, d, gen, device):
        self.inp = torch.randn(vocabulary, d, generator=gen, device=device) / d ** 0.5
        self.out = torch.randn(vocabulary, d, generator=gen, device=device) / d ** 0.5

    def logits(self, x):
        h = native.pdb_embed_lookup(self.inp, x, out_dtype=torch.bfloat16)
        return h, h @ self.out.to(torch.bfloat16).t()

    def step(self, x, h, dz, lr):
        """SGD on both tables: of the input factors only the rows in use."""
        dh = dz @ self.out.to(torch.bfloat16)
        self.out.sub_((dz.t() @ h).float(), alpha=lr)
        native.pdb_embed_grad(dh, x, self.inp, scale=-lr, accumulate=True)


def draw_text(vocabulary, n, gen, device):
    """(x, y): token y follows x.  Each token has four successors, half of the time the
    first of them, a quarter of the time the second, and so on."""
    x = (vocabulary * torch.rand(n, generator=gen, device=device) ** 2).long()
    turn = torch.rand(n, generator=gen, device=device).clamp_min_(1 / 16).log2_().neg_().long()
    return x, (x * 7 + 1 + turn.clamp_max_(3) * (vocabulary // 5)) % vocabulary


def learn_from_text(model, x, y, lr, entropy_reward=0.01):
    """One step of likelihood on the observed tokens; the mean log probability."""
    n = x.numel()
    h, z = model.logits(x)
    f = native.pdb_token_logprobs(z, y)
    d_logp = torch.full((n,), -1.0, device=z.device)
    d_entropy = torch.full((n,), -entropy_reward, device=z.device)
    dz = native.pdb_token_logprobs_grad(z, y, f.stats, d_logp, f.entropy, d_entropy, out=z)
    model.step(x, h, dz, lr)
    return f.logp.mean()


def learn_from_teacher(model, teacher, x, top, temp, lr):
    """One step on the teacher's `top` best alternatives; the mean divergence."""
    told = native.pdb_token_logprobs(teacher.logits(x)[1], top=top)
    h, z = model.logits(x)
    loss, dz = native.pdb_distill(z, told.top_id, told.top_logp, temp=temp, out=z)
    model.step(x, h, dz, lr)
    return loss.mean()


def go_on(model, token, steps):
    """Greedy continuation of one token, a call for each."""
    x = torch.tensor([token], dtype=torch.int32, device=model.inp.device)
    said = []
    for _ in range(steps):
        best = native.pdb_token_logprobs(model.logits(x)[1], top=1)
        x = best.top_id.view(1)
        said.append(int(x))
    return said


def run(vocabulary=5003, batch=2048, steps=300, teacher_factors=64, factors=24, top=20, lr=0.03, seed=1,
        report=print):
    device = torch.device("cuda", 0)
    gen = torch.Generator(device=device).manual_seed(seed)
    teacher = Factors(vocabulary, teacher_factors, gen, device)
    student = Factors(vocabulary, factors, gen, device)
    test = draw_text(vocabulary, batch, gen, device)

    def score(model):
        f = native.pdb_token_logprobs(model.logits(test[0])[1], test[1])
        return float(f.logp.mean()), float(f.entropy.mean())

    result = {"start": score(student)}
    for i in range(steps):
        logp = learn_from_text(teacher, *draw_text(vocabulary, batch, gen, device), lr)
        if report and i % 50 == 49:
            report("teacher step %4d  log probability %.3f" % (i + 1, float(logp)))
    for i in range(steps):
        x, _ = draw_text(vocabulary, batch, gen, device)
        loss = learn_from_teacher(student, teacher, x, top, 1.0, lr)
        if i == 0:
            result["first_loss"] = float(loss)
        if report and i % 50 == 49:
            report("student step %4d  divergence %.3f" % (i + 1, float(loss)))
    result.update(loss=float(loss), teacher=score(teacher), student=score(student),
                  said=(go_on(teacher, 1, 8), go_on(student, 1, 8)))
    if report:
        report("unseen text, log probability and entropy: student before %.3f %.3f, teacher %.3f %.3f, "
               "student %.3f %.3f" % (result["start"] + result["teacher"] + result["student"]))
        report("after token 1: teacher %s, student %s" % result["said"])
    return result


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocabulary", type=int, default=5003)
    ap.add_argument("--batch", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--teacher-factors", type=int, default=64)
    ap.add_argument("--factors", type=int, default=24)
    ap.add_argument("--top", type=int, default=20)
    ap.add_argument("--lr", type=float, default=0.03)
    ap.add_argument("--seed", type=int, default=1)
    a = ap.parse_args()
    run(a.vocabulary, a.batch, a.steps, a.teacher_factors, a.factors, a.top, a.lr, a.seed)


if __name__ == "__main__":
    main()
