"""A training loop around the pipeline, small enough to read: users compute gradients, encode them with error feedback; the server
decodes and averages, clips by the global norm, and takes an AdamW step with 32-bit or 8-bit moments.

    python -m paper_2203_09044_b200.train_step [--iterations 60] [--users 4] [--d 200000] [--state-bits 8]

The model is a separable quadratic over the tensors of the ResNet-18 layer mix (scaled to d parameters): the loss of weights w is
mean(h (w - w*)^2) / 2 with curvatures h over two decades, and a user's gradient is the true one plus noise of its own.  It needs
nothing but the library, and one can tell from the loss whether the step works.
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


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--iterations", type=int, default=60)
    ap.add_argument("--users", type=int, default=4)
    ap.add_argument("--d", type=int, default=200_000)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    a = ap.parse_args()
    final = run(a.iterations, a.users, a.d, a.state_bits,
                report=lambda t, loss, norm, bits: t % 10 or print(f"iteration {t:4d}  loss {loss:.5f}  gradient norm {norm:.3f}  {bits:.2f} bits/element"))
    print(f"loss {final[0]:.5f} -> {final[-1]:.5f}")
