"""A training loop around the pipeline, small enough to read: users compute gradients, encode them with error feedback; the server
decodes and averages, clips by the global norm, and takes an AdamW step with 32-bit or 8-bit moments.

    python -m paper_2203_09044_b200.train_step [--iterations 60] [--users 4] [--d 200000] [--state-bits 8]
    python -m paper_2203_09044_b200.train_step --model tokens [--vocab 2000] [--dim 128] [--tokens 256] [--teacher 4]

The first model is a separable quadratic over the tensors of the ResNet-18 layer mix (scaled to d parameters): the loss of weights w is
mean(h (w - w*)^2) / 2 with curvatures h over two decades, and a user's gradient is the true one plus noise of its own.  It needs
nothing but the library, and one can tell from the loss whether the step works.

The second predicts the next token from the last one: embedding, layer norm, head.  Every user has sequences of its own, of different
lengths; its gradient goes layer by layer into its row, which is what is encoded.  The forward pass reads the 16-bit copies that the optimizer
leaves.  With --teacher k users learn from the k most likely next tokens of a teacher instead of from the ones drawn.
"""
import argparse

from . import binding, inputs


def run(iterations=60, n_users=4, d=200_000, state_bits=8, lr=0.05, max_norm=1.0, weight_decay=0.0, seed=0, report=None):
    """The losses before each iteration and after the last (a list of floats).  report(t, loss, norm, bits per element) is called after
    every iteration."""
    import torch
    wl = inputs.workload(1, d=d, n_users=n_users)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    plan = binding.Plan(wl.d, wl.n_users, wl.exp_bits, wl.mant_bits, wl.seg_offsets, gamma=wl.gamma, bias_mode=binding.BIAS_CURRENT)
    out = plan.alloc_outputs()
    residual = torch.zeros((n_users, plan.ld), device="cuda")
    gradient = torch.zeros((n_users, plan.ld), device="cuda")

    target = torch.randn(wl.d, generator=gen, device="cuda")
    curvature = 10.0 ** (torch.rand(wl.d, generator=gen, device="cuda") * 2 - 2)
    weights = torch.zeros(wl.d, device="cuda")
    layers = list(zip(wl.seg_offsets[:-1], wl.seg_offsets[1:]))
    optimizer = binding.AdamW([weights[a:b] for a, b in layers], lr=lr, weight_decay=weight_decay, state_bits=state_bits, seed=seed)
    averaged = optimizer.bind_grads([out["avg"][a:b] for a, b in layers])       # the decoder's output row, layer by layer
    info = torch.zeros(4, device="cuda")

    losses = []
    for t in range(iterations):
        error = weights - target
        losses.append(float((curvature * error * error).mean()) / 2)
        noise = torch.randn((n_users, wl.d), generator=gen, device="cuda")
        gradient[:, :wl.d] = (curvature * error + 0.05 * noise) / wl.d
        plan.encode(gradient, residual, out)
        plan.decode_aggregate(out)
        optimizer.grad_norm(averaged, info, max_norm=max_norm, grad_scale=float(wl.d))
        optimizer.step(averaged, info)
        if report:
            report(t, losses[-1], float(info[1]), float(out["user_bits"].sum()) / (n_users * wl.d))
    error = weights - target
    losses.append(float((curvature * error * error).mean()) / 2)
    flags, _ = plan.status()
    if flags or optimizer.status()[0]:
        raise RuntimeError(f"pipeline flags {flags}, optimizer flags {optimizer.status()[0]}")
    return losses


class TokenModel:
    """Embedding, layer norm and head over the tokens of several users, with a gradient row for each.  Weights in float32; the forward
    pass reads copies in bfloat16, which whoever changes the weights keeps up to date (AdamW does)."""

    def __init__(self, vocab, dim, n_users, tokens, top=1, seed=0):
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.vocab, self.dim, self.n_users = vocab, dim, n_users
        self.embedding = binding.Embedding(vocab, dim, n_users=n_users, tokens=tokens)
        self.norm = binding.LayerNorm(dim, n_users=n_users)
        self.head = binding.TokenLoss(vocab, dim, n_users=n_users, tokens=tokens, dtype=torch.bfloat16, grad_dtype=torch.float32, top=top)
        self.shapes = [(vocab, dim), (dim,), (dim,), (vocab, dim)]              # table, scale and shift of the norm, head
        self.seg_offsets = [0]
        for shape in self.shapes:
            self.seg_offsets.append(self.seg_offsets[-1] + (shape[0] * shape[1] if len(shape) == 2 else shape[0]))
        self.d = self.seg_offsets[-1]
        self.weights = [torch.randn(self.shapes[0], generator=gen, device="cuda"), torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda"),
                        torch.randn(self.shapes[3], generator=gen, device="cuda") * dim ** -0.5]
        self.copies = [w.bfloat16() for w in self.weights]

    def segments(self, rows):
        """The layers' parts of gradient rows [users][ld], or of one row."""
        return [rows[..., a:b] for a, b in zip(self.seg_offsets[:-1], self.seg_offsets[1:])]

    def gradients(self, inputs, targets, rows, teacher=None, temperature=1.0):
        """Loss of each token ([users][tokens], 0 where there is none); the gradient of each user's mean goes into its row.  teacher: (index,
        logits) of its entries for each token, in place of targets."""
        table, scale, shift, head = self.copies
        d_table, d_scale, d_shift, d_head = self.segments(rows)
        x = self.embedding.forward(inputs, table)
        h, mean, rstd = self.norm.forward(x, scale, shift)
        if teacher is None:
            loss, lse = self.head.loss(h, head, targets)
            dh = self.head.loss_grad(h, head, targets, lse, dweight=d_head)
        else:
            loss, lse = self.head.distill(h, head, *teacher, temperature)
            dh = self.head.distill_grad(h, head, *teacher, lse, temperature=temperature, dweight=d_head)
        dx = self.norm.backward(dh, x, scale, mean, rstd, dweight=d_scale, dbias=d_shift)
        self.embedding.backward(dx, inputs, d_table)
        return loss


def token_batch(successors, n_users, tokens, gen):
    """Sequences in which a token's successor is one of its `successors` [vocab][k], the first half of the time, the second a quarter, ...;
    inputs, targets and how many there are of each user's (-1 behind them)."""
    import torch
    vocab, k = successors.shape
    pick = torch.rand((n_users, tokens), generator=gen, device="cuda").clamp(min=1e-6).log2().neg().long().clamp(max=k - 1)
    at = [torch.randint(0, vocab, (n_users,), generator=gen, device="cuda")]
    for t in range(tokens):
        at.append(successors[at[-1], pick[:, t]])
    sequence = torch.stack(at, 1)
    length = torch.randint(max(1, tokens // 2), tokens + 1, (n_users, 1), generator=gen, device="cuda")
    behind = torch.arange(tokens, device="cuda")[None] >= length
    return sequence[:, :-1].masked_fill(behind, -1), sequence[:, 1:].masked_fill(behind, -1)


def run_tokens(iterations=60, n_users=4, vocab=2000, dim=128, tokens=256, teacher=0, state_bits=8, lr=0.01, max_norm=1.0, seed=0, report=None):
    """The mean losses before each iteration (a list of floats).  teacher: entries of the teacher's logits, or 0.  report: as in run()."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    model = TokenModel(vocab, dim, n_users, tokens, top=max(1, teacher), seed=seed)
    successors = torch.randint(0, vocab, (vocab, max(4, teacher)), generator=gen, device="cuda")
    halves = -0.6931471805599453 * torch.arange(teacher, device="cuda").float()              # logits of 1/2, 1/4, ...
    plan = binding.Plan(model.d, n_users, 4, 3, model.seg_offsets, gamma=0.9, bias_mode=binding.BIAS_CURRENT)
    out = plan.alloc_outputs()
    residual, gradient = torch.zeros((n_users, plan.ld), device="cuda"), torch.zeros((n_users, plan.ld), device="cuda")
    optimizer = binding.AdamW(model.weights, grad_dtype=torch.float32, copies=model.copies, lr=lr, weight_decay=[0.01, 0.0, 0.0, 0.01], state_bits=state_bits, seed=seed)
    averaged = optimizer.bind_grads([g.view(shape) for g, shape in zip(model.segments(out["avg"]), model.shapes)])
    info = torch.zeros(4, device="cuda")
    losses = []
    for t in range(iterations):
        inputs, targets = token_batch(successors, n_users, tokens, gen)
        entries = None
        if teacher:
            index = successors[inputs.clamp(min=0), :teacher].masked_fill((inputs < 0)[..., None], -1)
            entries = index, halves.expand(index.shape).contiguous()
        loss = model.gradients(inputs, targets, gradient, entries)
        plan.encode(gradient, residual, out)
        plan.decode_aggregate(out)
        optimizer.grad_norm(averaged, info, max_norm=max_norm)
        optimizer.step(averaged, info)
        losses.append(float(loss.sum() / (targets >= 0).sum()))
        if report:
            report(t, losses[-1], float(info[1]), float(out["user_bits"].sum()) / (n_users * model.d))
    flags = [plan.status()[0], optimizer.status()[0], model.embedding.status()[0], model.head.status()[0]]
    if any(flags):
        raise RuntimeError(f"flags of pipeline, optimizer, embedding and head: {flags}")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--iterations", type=int, default=60)
    ap.add_argument("--users", type=int, default=4)
    ap.add_argument("--d", type=int, default=200_000)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    ap.add_argument("--model", choices=("quadratic", "tokens"), default="quadratic")
    ap.add_argument("--vocab", type=int, default=2000)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--teacher", type=int, default=0)
    a = ap.parse_args()

    def show(t, loss, norm, bits):
        if t % 10 == 0:
            print(f"iteration {t:4d}  loss {loss:.5f}  gradient norm {norm:.3f}  {bits:.2f} bits/element")

    if a.model == "tokens":
        final = run_tokens(a.iterations, a.users, a.vocab, a.dim, a.tokens, a.teacher, a.state_bits, report=show)
    else:
        final = run(a.iterations, a.users, a.d, a.state_bits, report=show)
    print(f"loss {final[0]:.5f} -> {final[-1]:.5f}")
