"""Data-parallel distillation of a small student on one GPU, with the whole library: the layers' products on microscaled 4-bit
matrices, the loss against a teacher's top logits, the workers' gradients compressed, averaged and applied.

    python examples/distill_student.py [steps]

Each of the simulated workers has its own tokens.  A step of a worker:
    h = relu(x W1^T), z = h W2^T          tq_mx_quantize, tq_mx_matmul
    loss, dz                              tq_distill
    dW2 = dz^T h, dh = dz W2, dW1 = ...   tq_mx_quantize (gradients rounded stochastically, both ways at once), tq_mx_matmul
and of the server: statistics, parameters, codes, average and momentum SGD in the calls of tq.h.  At the end the student
answers for one token at a time (tq_mx_linear).
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2402_01798_amd import binding as tq                                        # noqa: E402

WORKERS, TOKENS, WIDTH, HIDDEN, VOCAB, TOP, BITS = 4, 512, 256, 512, 1000, 16, 4
TAU, RATE, MOMENTUM, SEED = 2.0, 0.1, 0.9, 7


class Matrix:
    """A matrix of one shape, in both 4-bit forms.  What is rounded stochastically has a seed of its own: casts and payloads of one
    (seed, worker, step) would draw the same numbers."""

    def __init__(self, rows, cols, seed=0):
        self.form, self.form_t = tq.alloc_mx(rows, cols), tq.alloc_mx(cols, rows)
        self.seed = seed

    def take(self, x, rounding=tq.MX_NEAREST, worker=0, step=0):
        tq.tq_mx_quantize(x, self.form, self.form_t, rounding, self.seed, worker, step)
        return self


class Student:
    """W1 and W2 are views of one flat fp32 parameter vector, the gradients of one flat gradient for each worker."""

    def __init__(self):
        d = HIDDEN * WIDTH + VOCAB * HIDDEN
        g = torch.Generator(device="cuda").manual_seed(SEED)
        self.theta = torch.empty(d, device="cuda")
        self.velocity = torch.zeros(d, device="cuda")
        self.w1, self.w2 = self.split(self.theta)
        self.w1.normal_(0, (2 / WIDTH) ** 0.5, generator=g)
        self.w2.normal_(0, HIDDEN ** -0.5, generator=g)
        self.m1, self.m2 = Matrix(HIDDEN, WIDTH), Matrix(VOCAB, HIDDEN)
        self.mx, self.mh = Matrix(TOKENS, WIDTH), Matrix(TOKENS, HIDDEN)
        self.mdz, self.mdh = Matrix(TOKENS, VOCAB, SEED + 1), Matrix(TOKENS, HIDDEN, SEED + 2)
        shapes = ((TOKENS, HIDDEN, WIDTH), (TOKENS, VOCAB, HIDDEN), (TOKENS, HIDDEN, VOCAB), (VOCAB, HIDDEN, TOKENS), (HIDDEN, WIDTH, TOKENS))
        self.ws = torch.empty(max(tq.mx_matmul_workspace_bytes(*s) for s in shapes) or 1, dtype=torch.uint8, device="cuda")
        self.h = torch.empty(TOKENS, HIDDEN, dtype=torch.bfloat16, device="cuda")
        self.z = torch.empty(TOKENS, VOCAB, dtype=torch.bfloat16, device="cuda")
        self.dh = torch.empty_like(self.h)
        self.loss = torch.empty(TOKENS, device="cuda")
        self.grad = torch.full((TOKENS,), 1 / TOKENS, device="cuda")
        self.gradients = [torch.empty(d, device="cuda") for _ in range(WORKERS)]
        self.stats = [tq.alloc_stats(d) for _ in range(WORKERS)]
        self.params = [tq.alloc_params(d) for _ in range(WORKERS)]
        self.payloads = [tq.alloc_payload(d, BITS) for _ in range(WORKERS)]
        self.stats_ws = torch.empty(WORKERS * tq.stats_workspace_bytes(d), dtype=torch.uint8, device="cuda")

    @staticmethod
    def split(flat):
        return flat[:HIDDEN * WIDTH].view(HIDDEN, WIDTH), flat[HIDDEN * WIDTH:].view(VOCAB, HIDDEN)

    def worker(self, i, step, x, ids, t):
        """Loss of worker i's tokens; its gradient into self.gradients[i]."""
        dw1, dw2 = self.split(self.gradients[i])
        x = self.mx.take(x)
        tq.tq_mx_matmul(x.form, self.m1.form, self.h, self.ws)
        self.h.relu_()
        h = self.mh.take(self.h)
        tq.tq_mx_matmul(h.form, self.m2.form, self.z, self.ws)
        tq.tq_distill(self.z, ids, t, self.grad, self.loss, self.z, TAU)                # dz in place of z
        dz = self.mdz.take(self.z, tq.MX_STOCHASTIC, i, step)
        tq.tq_mx_matmul(dz.form_t, h.form_t, dw2, self.ws)
        tq.tq_mx_matmul(dz.form, self.m2.form_t, self.dh, self.ws)
        self.dh.masked_fill_(self.h <= 0, 0)
        dh = self.mdh.take(self.dh, tq.MX_STOCHASTIC, i, step)
        tq.tq_mx_matmul(dh.form_t, x.form_t, dw1, self.ws)
        return self.loss.mean()

    def step(self, step, batches):
        self.m1.take(self.w1)
        self.m2.take(self.w2)
        loss = sum(self.worker(i, step, *batch) for i, batch in enumerate(batches)) / len(batches)
        tq.tq_stats_multi(self.gradients, self.stats, self.stats_ws)
        tq.tq_params_multi(self.stats, self.params, BITS, tq.GRID_NONUNIFORM)
        tq.tq_compress_multi(self.gradients, self.params, self.payloads, BITS, SEED, 0, step, grid=tq.GRID_NONUNIFORM)
        tq.tq_decompress_aggregate_update(self.payloads, self.params, self.theta, BITS, RATE, MOMENTUM, 0.0, self.velocity)
        return loss

    def answer(self, x):
        """The logits of a few tokens [m, WIDTH], cast inside the products."""
        h = torch.empty(x.shape[0], HIDDEN, dtype=torch.bfloat16, device="cuda")
        z = torch.empty(x.shape[0], VOCAB, dtype=torch.bfloat16, device="cuda")
        tq.tq_mx_linear(x, self.m1.form, h, self.scratch(x.shape[0], HIDDEN, WIDTH))
        return tq.tq_mx_linear(h.relu_(), self.m2.form, z, self.scratch(x.shape[0], VOCAB, HIDDEN))

    @staticmethod
    def scratch(m, n, k):
        nbytes = tq.mx_linear_workspace_bytes(m, n, k)
        return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def teacher_of(seed):
    """A network of the same kind, wider and in fp32, that hands out the largest of its logits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    a = torch.randn(WIDTH, 4 * WIDTH, generator=g, device="cuda") * WIDTH ** -0.5
    b = torch.randn(4 * WIDTH, VOCAB, generator=g, device="cuda") * 0.2
    return lambda x: torch.topk(torch.relu(x @ a) @ b, TOP, dim=1)


def train(steps):
    student, teacher = Student(), teacher_of(SEED + 1)
    g = torch.Generator(device="cuda").manual_seed(SEED + 2)
    data = []
    for _ in range(WORKERS):
        x = torch.randn(TOKENS, WIDTH, generator=g, device="cuda")
        t, ids = teacher(x)
        data.append((x.bfloat16(), ids, t))                                            # ids as torch.topk gives them: int64
    losses = [student.step(step, data) for step in range(steps)]
    return student, data, [float(v) for v in losses]


def main():
    steps = int(sys.argv[1]) if len(sys.argv) > 1 else 200
    student, data, losses = train(steps)
    for i in range(0, steps, max(1, steps // 10)):
        print("step %4d  loss %.4f" % (i, losses[i]))
    print("step %4d  loss %.4f" % (steps - 1, losses[-1]))
    x, ids, _ = data[0]
    student.m1.take(student.w1)
    student.m2.take(student.w2)
    right = sum(int(student.answer(x[i:i + 1]).argmax()) in ids[i].tolist() for i in range(64))
    print("one token at a time: %d of 64 answers among the teacher's %d" % (right, TOP))


if __name__ == "__main__":
    main()
