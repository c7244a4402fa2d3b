"""A student learns from the short lists of a teacher that answers with 8-bit weights: the operators on packed weights and on
logits next to the quantized step, on one GPU.

Per batch:
  1. the teacher's hidden states meet its output matrix as the codec packed it (qsdp_quantize_weight, a bucket per channel):
     qsdp_linear_codes rounds the states to 8 bits and multiplies; no weight is decoded;
  2. qsdp_token_logprobs leaves the 16 most likely tokens of every position with their log probabilities: what a training run
     stores of a teacher;
  3. the student's logits, the lists and the labels go into qsdp_distill_loss, which returns the loss and, from the same pass,
     the gradient of the logits;
  4. the gradient of the student's matrix (a plain product) updates it by qsdp_fused_step: W8 G8, the iterate lives on its grid.

    python examples/distill_student.py            # prints the loss and how often student and teacher agree
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2302_02390_amd import binding as qb  # noqa: E402

VOCAB, HIDDEN, WIDTH, TOP = 4001, 512, 256, 16  # tokens, the teacher's and the student's hidden size, length of a list


def train(steps=120, batch=512, lr=10.0, temperature=2.0, alpha=0.9, device="cuda:0", trace=None):
    """[(mean loss, share of positions where student and teacher put the same token first)] per step."""
    device = torch.device(device)
    gen = torch.Generator(device=device).manual_seed(0)

    def normal(*shape):
        return torch.randn(shape, device=device, generator=gen)

    teacher = normal(VOCAB, HIDDEN) * (4.0 / HIDDEN ** 0.5)
    codes, meta = qb.alloc_packed(teacher.numel(), 8, HIDDEN, device)
    qb.qsdp_quantize_weight(teacher.view(-1), 8, HIDDEN, 0.0, 0, codes, meta.view(-1))
    del teacher                                                     # from here on there are only its codes
    student = normal(VOCAB, WIDTH) * 0.01
    into = normal(HIDDEN, WIDTH) / HIDDEN ** 0.5                    # the student sees the states through a narrow map

    logits_t = torch.empty((batch, VOCAB), dtype=torch.bfloat16, device=device)
    logprob, entropy, loss = (torch.empty(batch, device=device) for _ in range(3))
    top_logprob = torch.empty((batch, TOP), device=device)
    top_index = torch.empty((batch, TOP), dtype=torch.int32, device=device)
    workspace = torch.empty(qb.tokens_bytes(batch, HIDDEN, HIDDEN), dtype=torch.uint8, device=device)
    d_logits = torch.empty((batch, VOCAB), device=device)
    scale = torch.full((batch,), 1.0 / batch, device=device)
    seen = normal(4 * batch, HIDDEN)                                # a small data set, passed over again and again
    history = []
    for step in range(steps):
        states = seen[step % 4 * batch:(step % 4 + 1) * batch]
        qb.qsdp_linear_codes(states, codes, meta.view(-1), VOCAB, HIDDEN, None, logits_t, workspace)                 # 1
        labels = logits_t.argmax(1)
        qb.qsdp_token_logprobs(logits_t, labels, 1.0, logprob, entropy, None, top_logprob, top_index)                # 2
        features = states @ into
        logits = features @ student.t()
        qb.qsdp_distill_loss(logits, top_index, top_logprob, labels, temperature, alpha, scale, loss, None, d_logits)  # 3
        gradient = d_logits.t() @ features
        qb.qsdp_fused_step(student.view(-1), gradient.view(-1), lr, 8, 8, WIDTH, 0.0, step)                          # 4
        history.append((float(loss.mean()), float((logits.argmax(1) == labels).float().mean())))
        if trace is not None and step % trace == 0:
            print(f"step {step:4d}  loss {history[-1][0]:.4f}  agreement {history[-1][1]:.3f}  "
                  f"teacher's entropy {float(entropy.mean()):.3f}")
    return history


if __name__ == "__main__":
    if not torch.cuda.is_available():
        print("distill_student.py needs a GPU", file=sys.stderr)
        sys.exit(2)
    result = train(trace=20)
    print(f"loss {result[0][0]:.4f} -> {result[-1][0]:.4f}, agreement {result[0][1]:.3f} -> {result[-1][1]:.3f}")
