"""On-policy distillation of a bigram model, on one GPU: the token operators as they run together.

The student is a table of logits [V, V], one row per preceding token; the teacher is a fixed one. A
step
  1. rolls out: draws each next token from the student (SampleCall) and records its log-probability,
  2. has the teacher leave its K largest logits and their tail at the visited positions
     (TopLogitsCall),
  3. takes the distillation loss of the student's logits there and its gradient (DistillCall),
  4. adds the CIS loss of the drawn tokens (LossCall), whose log-probabilities are the recorded ones,
     with the teacher's preference for a token as its advantage,
and descends on both gradients. The calls keep their outputs and workspaces from step to step.

    python examples/on_policy_distillation.py [--steps N] [--vocab V] [--batch B] [--length L] [--k K]
"""

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2609_32444_amd as cis  # noqa: E402


def train(steps=40, vocab=1000, batch=64, length=32, k=32, lr=6.0, seed=0):
    """Mean KL to the teacher over the visited positions, step by step, and the largest difference
    between a recorded log-probability and the loss's own."""
    if vocab % 4:
        raise ValueError("vocab must be a multiple of 4: rows are whole 16-byte vectors")
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    teacher = torch.randn(vocab, vocab, generator=g, device=dev) * 2
    student = torch.randn(vocab, vocab, generator=g, device=dev) * 0.5
    T = batch * length
    # what the calls read: the rollout's current rows, and the logits of the visited positions
    now, u = torch.empty(batch, vocab, device=dev), torch.empty(batch, device=dev)
    zs, zt = torch.empty(T, vocab, device=dev), torch.empty(T, vocab, device=dev)
    ids, logp = torch.empty(T, dtype=torch.int64, device=dev), torch.empty(T, device=dev)
    advantage = torch.empty(T, device=dev)
    draw = cis.SampleCall(now, u)
    top = cis.TopLogitsCall(zt, k)
    distill = cis.DistillCall(zs, top.out["ids"], top.out["values"], top.out["tail"],
                              kind=cis.KL_REVERSE, scale=1.0 / T)
    loss = cis.LossCall(zs, ids, logp, advantage, lam=2.3, scale=-0.05 / T, bwd=True)
    kl, off = [], 0.0
    for _ in range(steps):
        at = torch.randint(0, vocab, (batch,), generator=g, device=dev)
        visited = []
        for t in range(length):
            visited.append(at)
            torch.index_select(student, 0, at, out=now)
            u.uniform_(generator=g)
            out = draw.run()
            at = out["ids"].clone()
            ids[t * batch:(t + 1) * batch] = at
            logp[t * batch:(t + 1) * batch] = out["logp"]
        rows = torch.cat(visited)
        torch.index_select(student, 0, rows, out=zs)
        torch.index_select(teacher, 0, rows, out=zt)
        top.run()
        gain = zt.gather(1, ids[:, None])[:, 0] - torch.logsumexp(zt, 1) - logp
        advantage.copy_((gain - gain.mean()).clamp_(-3, 3))
        d, p = distill.run(), loss.run()
        grad = d["dlogits"] + p["dlogits"]
        # rows that are visited often take the mean of their gradients
        count = torch.bincount(rows, minlength=vocab).clamp_(min=1).float()
        student.index_add_(0, rows, grad * (-lr * T / count[rows])[:, None])
        kl.append(d["loss"].clone())
        off = max(off, float((p["logp_train"] - logp).abs().max()))
    return [float(x) for x in kl], off


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("steps", 40), ("vocab", 1000), ("batch", 64), ("length", 32), ("k", 32)):
        ap.add_argument("--" + name, type=int, default=value)
    kl, off = train(**vars(ap.parse_args()))
    for i in range(0, len(kl), max(1, len(kl) // 10)):
        print(f"step {i:4d}  KL to the teacher {kl[i]:.4f}")
    print(f"step {len(kl) - 1:4d}  KL to the teacher {kl[-1]:.4f}; recorded and training "
          f"log-probabilities differ by {off:.2g} at most")


if __name__ == "__main__":
    main()
