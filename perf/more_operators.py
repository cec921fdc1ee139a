"""Cases of the operators at a language model's two ends, which make the gradients that the pipeline encodes: embedding lookup and its
gradient, layer norm forward and backward, and the losses over a large vocabulary (cross entropy against tokens, distillation from a
teacher's top logits) with their gradients, without the logits being kept.

A batch is [users][tokens]; every user has a weight gradient of its own, which goes into a segment of that user's row of a gradient
array, as the encoder takes it (`at`: the element of the row at which the segment begins, which may be any), or into an array of its own
(`at` = 0).  A token below zero is none: the places behind the last token of a shorter sequence.
"""
import math
import random

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases --------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # lookup: one short sequence of a small model, where the call is what counts; the prompt batch of a wide one
        dict(name="embed_512", op="embed", users=1, tokens=512, vocab=32000, dim=768, table="f32", act="bf16"),
        dict(name="embed_64k", op="embed", users=4, tokens=16384, vocab=131072, dim=4096, table="bf16", act="bf16"),
        # its gradient: eight users' rows of 32 bits, at an odd element; one long batch into an array in 16 bits
        dict(name="embed_grad_8users", op="embed_grad", users=8, tokens=2000, vocab=32000, dim=768, act="bf16", grad="f32", at=1001),
        dict(name="embed_grad_64k", op="embed_grad", users=1, tokens=65536, vocab=131072, dim=2048, act="bf16", grad="bf16", at=0),
        # layer norm: a long batch in 16 bits; backward for users with rows of an odd width in 32 bits, and for the long batch
        dict(name="norm_64k", op="norm", users=1, tokens=65536, dim=4096, act="bf16"),
        dict(name="norm_grad_8users_odd", op="norm_grad", users=8, tokens=1023, dim=1001, act="f32", grad="f32", at=77),
        dict(name="norm_grad_64k", op="norm_grad", users=1, tokens=65536, dim=4096, act="bf16", grad="f32", at=0),
        # the losses: evaluation of a few tokens; a training pass of four users with an odd vocabulary into their rows; the largest
        dict(name="loss_200", op="loss", users=1, tokens=200, vocab=32000, dim=768, act="bf16", top=1),
        dict(name="loss_grad_4users", op="loss_grad", users=4, tokens=1000, vocab=50257, dim=768, act="bf16", grad="f32", at=5, top=1),
        dict(name="loss_grad_8k", op="loss_grad", users=1, tokens=8192, vocab=131072, dim=4096, act="bf16", grad="bf16", at=0, top=1),
        # distillation: a training pass on a teacher's 64 logits a token
        dict(name="distill_512", op="loss", users=2, tokens=256, vocab=32000, dim=1024, act="f16", top=20, temperature=2.0),
        dict(name="distill_grad_4users", op="loss_grad", users=4, tokens=1024, vocab=50257, dim=2048, act="bf16", grad="bf16", at=0, top=64, temperature=1.5),
    ]


def spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_grad", "norm_grad", "loss", "loss_grad", "loss_grad"])
    users = rng.choice([1, 1, 2, 3, 8])
    case = dict(op=op, users=users, act=rng.choice(["bf16", "bf16", "f16"] if op.startswith("loss") else ["bf16", "bf16", "f16", "f32"]))
    if not op.startswith("norm"):
        case["vocab"] = spread(rng, 1000, 96000 // users)
    if op.startswith("loss"):
        case.update(tokens=spread(rng, 1, 4096 // users), dim=8 * spread(rng, 16, 400), top=rng.choice([1, 1, spread(rng, 2, 64)]))
        if case["top"] > 1:
            case["temperature"] = rng.choice([1.0, 2.0, round(rng.uniform(0.7, 4.0), 2)])
    else:
        case["tokens"], case["dim"] = spread(rng, 1, 32768 // users), spread(rng, 64, 4096)
        if rng.random() < 0.5:
            case["dim"] = case["dim"] // 8 * 8
    if op == "embed":
        case["table"] = rng.choice(["f32", case["act"]])
    if op.endswith("grad"):
        case.update(grad=rng.choice(["f32", "f32", "bf16" if case["act"] == "f32" else case["act"]]), at=rng.choice([0, 0, rng.randrange(1, 5000)]))
    return case


def rows_written(case):
    """Elements of the weight gradient of one user."""
    return case["dim"] * (2 if case["op"] == "norm_grad" else case["vocab"])


def work(case):
    width = {"f32": 4, "bf16": 2, "f16": 2}
    n, d, op = case["users"] * case["tokens"], case["dim"], case["op"]
    act = width[case["act"]]
    grad = case["users"] * rows_written(case) * width[case["grad"]] if "grad" in case else 0
    if op == "embed":
        return {"bytes": n * (8 + d * (width[case["table"]] + act)), "flops": n * d}
    if op == "embed_grad":
        return {"bytes": n * (8 + d * act) + grad, "flops": n * d}
    if op == "norm":
        return {"bytes": n * (8 + 2 * d * act), "flops": 7 * n * d}
    if op == "norm_grad":
        return {"bytes": n * (8 + 3 * d * act) + grad, "flops": 12 * n * d}
    tokens = int(sum(lengths(case)))                      # the others cost nothing
    entries = n * (8 if case["top"] == 1 else 12 * case["top"])
    product = 2 * tokens * case["vocab"] * d
    if op == "loss":
        return {"bytes": act * d * (tokens + case["vocab"]) + entries + 8 * n, "flops": product}
    # one product for the logits, one for each gradient
    return {"bytes": act * d * (tokens + n + case["vocab"]) + entries + 8 * n + grad, "flops": 3 * product}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def lengths(case):
    """Tokens of each user's sequence: the first has them all, the others from half on."""
    rng = random.Random(case["tokens"] * 64 + case["users"])
    return [case["tokens"]] + [rng.randint((case["tokens"] + 1) // 2, case["tokens"]) for _ in range(case["users"] - 1)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    u, t, d, op = case["users"], case["tokens"], case["dim"], case["op"]
    act = TYPES[case["act"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    s = dict(case=case)
    there = torch.arange(t, device="cuda")[None, :] < torch.tensor(lengths(case), device="cuda")[:, None]
    if not op.startswith("norm"):
        # tokens as a language has them: the lower the more frequent
        often = (torch.rand((u, t), generator=gen, device="cuda").pow_(3) * case["vocab"]).long().clamp_(max=case["vocab"] - 1)
        s["tokens"] = torch.where(there, often, -1)
    if op == "embed":
        s["table"] = (normal(case["vocab"], d) * 0.02).to(TYPES[case["table"]])
        s["scale"] = float(d) ** 0.5
    elif op == "embed_grad":
        s["dout"] = (normal(u, t, d) * 0.01).to(act)
        s["scale"] = float(d) ** 0.5
    elif op.startswith("norm"):
        x = normal(u, t, d) * (0.5 + 2 * torch.rand((u, t, 1), generator=gen, device="cuda")) + normal(u, t, 1)
        s["x"] = x.to(act)
        s["weight"], s["bias"] = 1 + 0.1 * normal(d), 0.1 * normal(d)
        if op == "norm_grad":
            s["dy"] = (normal(u, t, d) * 0.01).to(act)
            x = s["x"].double()
            mean = x.mean(2)
            s["mean"] = mean.float()
            s["rstd"] = (x.sub_(mean[:, :, None]).square_().mean(2) + EPS).rsqrt().float()
        del x
    else:
        s["weight"] = (normal(case["vocab"], d) * 0.05).to(act)
        s["hidden"] = normal(u, t, d).to(act)             # behind a sequence's end lies what the model computes of padding
        if case["top"] > 1:
            k = case["top"]
            # a teacher's k entries of each token, largest first, all different
            step = torch.randint(1, max(2, case["vocab"] // k), (u, t, k), generator=gen, device="cuda")
            s["index"] = torch.where(there[:, :, None], (s["tokens"].clamp(min=0)[:, :, None] + step.cumsum(2) - step[:, :, :1]) % case["vocab"], -1)
            s["logits"] = (normal(u, t, k) * 3).sort(2, descending=True)[0].to(act)
        s["share"] = torch.where(there, 1.0 / there.sum(1, keepdim=True), 0.0).float()       # of each token in its user's mean
    if "grad" in case:
        n = rows_written(case)
        ld = (case["at"] + n + 4 + 3) // 4 * 4
        s["rows"] = torch.zeros((u, ld), dtype=TYPES[case["grad"]], device="cuda")
        s["part"] = s["rows"][:, case["at"]:case["at"] + n]
    if own:
        from paper_2203_09044_b200 import binding
        if op.startswith("embed"):
            s["own"] = binding.Embedding(case["vocab"], d, n_users=u, tokens=t)
        elif op.startswith("norm"):
            s["own"] = binding.LayerNorm(d, n_users=u, eps=EPS)
        else:
            s["own"] = binding.TokenLoss(case["vocab"], d, n_users=u, tokens=t, dtype=act, grad_dtype=TYPES[case.get("grad", "f32")], top=case["top"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------
def run(s):
    return kernels(s) if own else plain(s)


def kernels(s):
    case, op, mine = s["case"], s["case"]["op"], s["own"]
    if op == "embed":
        return {"out": mine.forward(s["tokens"], s["table"], scale=s["scale"], out_dtype=TYPES[case["act"]])}
    if op == "embed_grad":
        mine.backward(s["dout"], s["tokens"], s["part"], scale=s["scale"])
        return {"dtable": s["part"]}
    if op == "norm":
        y, mean, rstd = mine.forward(s["x"], s["weight"], s["bias"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        d = case["dim"]
        dx = mine.backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], dweight=s["part"][:, :d], dbias=s["part"][:, d:])
        return {"dx": dx, "dparams": s["part"]}
    if case["top"] == 1:
        loss, lse = mine.loss(s["hidden"], s["weight"], s["tokens"])
        if op == "loss":
            return {"loss": loss, "lse": lse}
        dhidden = mine.loss_grad(s["hidden"], s["weight"], s["tokens"], lse, s["share"], dweight=s["part"])
    else:
        loss, lse = mine.distill(s["hidden"], s["weight"], s["index"], s["logits"], case["temperature"])
        if op == "loss":
            return {"loss": loss, "lse": lse}
        dhidden = mine.distill_grad(s["hidden"], s["weight"], s["index"], s["logits"], lse, s["share"], case["temperature"], dweight=s["part"])
    return {"loss": loss, "lse": lse, "dhidden": dhidden, "dweight": s["part"]}


def plain(s):
    case, op = s["case"], s["case"]["op"]
    act = TYPES[case["act"]]
    u, t, d = case["users"], case["tokens"], case["dim"]
    if op == "embed":
        rows = s["table"][s["tokens"].clamp(min=0)].float() * s["scale"]
        return {"out": torch.where((s["tokens"] < 0)[:, :, None], 0.0, rows).to(act)}
    if op == "embed_grad":
        # tokens that are none go to a row behind the last one
        v = case["vocab"]
        row = torch.where(s["tokens"] < 0, v, s["tokens"]) + torch.arange(u, device="cuda")[:, None] * (v + 1)
        sums = torch.zeros((u * (v + 1), d), device="cuda").index_add_(0, row.view(-1), s["dout"].view(-1, d).float())
        s["part"].copy_((sums.view(u, v + 1, d)[:, :v] * s["scale"]).view(u, v * d))
        return {"dtable": s["part"]}
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(2, keepdim=True)
        x = x - mean
        rstd = ((x * x).mean(2, keepdim=True) + EPS).rsqrt()
        return {"y": (x * rstd * s["weight"] + s["bias"]).to(act), "mean": mean.view(u, t), "rstd": rstd.view(u, t)}
    if op == "norm_grad":
        dy, rstd = s["dy"].float(), s["rstd"][:, :, None]
        xhat = (s["x"].float() - s["mean"][:, :, None]) * rstd
        g = dy * s["weight"]
        dx = (g - g.mean(2, keepdim=True) - xhat * (g * xhat).mean(2, keepdim=True)) * rstd
        s["part"].copy_(torch.cat([(dy * xhat).sum(1), dy.sum(1)], 1))
        return {"dx": dx.to(act), "dparams": s["part"]}
    return plain_loss(s)


def plain_loss(s):
    case = s["case"]
    act, tau = TYPES[case["act"]], case.get("temperature", 1.0)
    u, t, d, v = case["users"], case["tokens"], case["dim"], case["vocab"]
    there = s["tokens"] >= 0
    weight = s["weight"].float()
    hidden = torch.where(there[:, :, None], s["hidden"].float(), 0.0)
    z = hidden.view(u * t, d) @ weight.T
    if tau != 1.0:
        z = z / tau
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    lse = (total.log() + top).view(u, t)
    if case["top"] == 1:
        at = s["tokens"].clamp(min=0).view(u * t, 1)
        q = torch.ones_like(top)
        loss = lse - z.gather(1, at).view(u, t)
    else:
        at = s["index"].clamp(min=0).view(u * t, -1)
        teacher = s["logits"].float().view(u * t, -1) / tau
        q = (teacher - teacher.amax(1, keepdim=True)).exp()
        q = q / q.sum(1, keepdim=True)
        loss = (q * (q.clamp(min=1e-38).log() + lse.view(u * t, 1) - z.gather(1, at))).sum(1).view(u, t)
    out = {"loss": torch.where(there, loss, 0.0), "lse": torch.where(there, lse, 0.0)}
    del z
    if case["op"] == "loss":
        return out
    dz = e.div_(total).scatter_add_(1, at, -q).mul_(s["share"].view(u * t, 1) / tau)
    out["dhidden"] = (dz @ weight).view(u, t, d).to(act)
    s["part"].copy_(torch.bmm(dz.view(u, t, v).transpose(1, 2), hidden).view(u, v * d))
    out["dweight"] = s["part"]
    return out


# ---- the same in 64 bits ----------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    op, u, d = case["op"], case["users"], case["dim"]
    if op == "embed":
        hot = s["tokens"] >= 0
        out = torch.zeros((u, case["tokens"], d), dtype=f64, device="cuda")
        out[hot] = s["table"].to(f64)[s["tokens"][hot]] * s["scale"]
        return {"out": out}
    if op == "embed_grad":
        out = torch.zeros((u, case["vocab"], d), dtype=f64, device="cuda")
        for i in range(u):
            mine = s["tokens"][i]
            out[i].index_put_((mine[mine >= 0],), s["dout"][i].to(f64)[mine >= 0] * s["scale"], accumulate=True)
        return {"dtable": out.reshape(u, -1)}
    if op.startswith("norm"):
        x = s["x"].to(f64)
        if op == "norm":
            var, mean = torch.var_mean(x, 2, correction=0)
            rstd = 1 / torch.sqrt(var + EPS)
            y = (x - mean.unsqueeze(2)) / torch.sqrt(var + EPS).unsqueeze(2) * s["weight"].to(f64) + s["bias"].to(f64)
            return {"y": y, "mean": mean, "rstd": rstd}
        dy, r, w = s["dy"].to(f64), s["rstd"].to(f64).unsqueeze(2), s["weight"].to(f64)
        xhat = (x - s["mean"].to(f64).unsqueeze(2)) * r
        along = torch.einsum("utd,utd,d->ut", dy, xhat, w).unsqueeze(2)
        dx = r * (dy * w) - r / d * (torch.einsum("utd,d->ut", dy, w).unsqueeze(2) + xhat * along)
        return {"dx": dx, "dparams": torch.cat([torch.einsum("utd,utd->ud", dy, xhat), dy.sum(1)], 1)}
    tau, w = case.get("temperature", 1.0), s["weight"].to(f64)
    loss = torch.zeros((u, case["tokens"]), dtype=f64, device="cuda")
    lse, dhidden = torch.zeros_like(loss), torch.zeros(s["hidden"].shape, dtype=f64, device="cuda")
    dweight = torch.zeros((u, case["vocab"], d), dtype=f64 if case["vocab"] * d * u < 1 << 30 else torch.float32, device="cuda") if "grad" in case else None
    for i, n in enumerate(lengths(case)):
        h = s["hidden"][i, :n].to(f64)
        logp = torch.log_softmax(h @ w.T / tau, 1)
        first = h @ w[0] / tau
        lse[i, :n] = first - logp[:, 0]
        if case["top"] == 1:
            loss[i, :n] = torch.nn.functional.nll_loss(logp, s["tokens"][i, :n], reduction="none")
            at, q = s["tokens"][i, :n, None], torch.ones((n, 1), dtype=f64, device="cuda")
        else:
            at = s["index"][i, :n]
            logq = torch.log_softmax(s["logits"][i, :n].to(f64) / tau, 1)
            q = logq.exp()
            loss[i, :n] = (q * (logq - logp.gather(1, at))).sum(1)
        if dweight is not None:
            dz = logp.exp_().scatter_add_(1, at, -q) * (s["share"][i, :n, None].to(f64) / tau)
            dhidden[i, :n] = dz @ w
            dweight[i] = (dz.T @ h).to(dweight.dtype)
    out = {"loss": loss, "lse": lse}
    if dweight is not None:
        out.update(dhidden=dhidden, dweight=dweight.reshape(u, -1))
    return out
