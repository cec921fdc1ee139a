"""Cases of the optimizer operators: the gradient norm with its clipping factor, and the AdamW step over many tensors
with its two moments held in 32 bits or in 8.

Each case is one set of tensors, as a parameter server (or a user that trains locally) holds it.  `layout` says how they lie in
memory: "row" back to back, the segments of one row as the gradient pipeline has them, so that a tensor may start at an odd
element; "apart" each at a multiple of 256 elements, as an allocator gives them.  The two moments always start at a multiple of
256 elements for each tensor (the blocks of the 8-bit states).
"""
import math
import random

import torch

own = False

BETA1, BETA2, EPS, LR = 0.9, 0.999, 1e-8, 1e-3
DECAY = 0.1            # of tensors with 1024 elements or more; biases and scales of norms have none
MAX_NORM = 1.0
BLOCK = 256            # elements that share an exponent in the 8-bit states
SEED = 20220917        # of the rounding of 8-bit states
T0 = 1000              # steps taken before the measured one
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases --------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the norm alone: a monitor of a small flat model, of the ResNet-18 layer mix, and of a large half-precision gradient
        dict(name="norm_2p20", op="norm", d=1 << 20, split="one", layout="row", grad="f32"),
        dict(name="norm_resnet18", op="norm", d=11_173_962, split="resnet18", layout="row", grad="f32"),
        dict(name="norm_2p28_bf16", op="norm", d=1 << 28, split="mixed", n=290, layout="apart", grad="bf16"),
        # 32-bit states: the smallest step (a layer of a head), where the call itself is what counts
        dict(name="step32_2p16", op="step", bits=32, d=1 << 16, split="one", layout="row", weight="f32", grad="f32", copy="", clip=False),
        # ... norm, factor and step of the ResNet-18 layers on the averaged gradient row
        dict(name="step32_resnet18_clip", op="step", bits=32, d=11_173_962, split="resnet18", layout="row", weight="f32", grad="f32", copy="", clip=True),
        # ... sixteen segments that start at odd elements
        dict(name="step32_16seg_odd", op="step", bits=32, d=14_728_266, split="equal", n=16, layout="row", weight="f32", grad="f32", copy="", clip=False),
        # ... mixed precision: 32-bit weights, gradients in 16 bits, a 16-bit copy of the weights for the next forward pass
        dict(name="step32_124m_bf16", op="step", bits=32, d=124_439_808, split="mixed", n=148, layout="apart", weight="f32", grad="bf16", copy="bf16", clip=False),
        dict(name="step32_2p28", op="step", bits=32, d=1 << 28, split="mixed", n=290, layout="apart", weight="f32", grad="f32", copy="", clip=False),
        # 8-bit states: the smallest step, the ResNet-18 layers, and the largest ones with all else in 32 bits and in 16
        dict(name="step8_2p16", op="step", bits=8, d=1 << 16, split="one", layout="row", weight="f32", grad="f32", copy="", clip=False),
        dict(name="step8_resnet18", op="step", bits=8, d=11_173_962, split="resnet18", layout="row", weight="f32", grad="f32", copy="", clip=False),
        dict(name="step8_124m_bf16w", op="step", bits=8, d=124_439_808, split="mixed", n=148, layout="apart", weight="bf16", grad="bf16", copy="", clip=False),
        dict(name="step8_2p28", op="step", bits=8, d=1 << 28, split="mixed", n=290, layout="apart", weight="f32", grad="bf16", copy="bf16", clip=False),
    ]


def draw(rng):
    op, bits = rng.choice([("norm", 0), ("step", 32), ("step", 32), ("step", 8), ("step", 8)])
    d = int(2.0 ** rng.uniform(13.0, 27.0)) | rng.choice([0, 1])
    n = min(max(1, int(2.0 ** rng.uniform(0.0, 8.6))), d // 64)
    case = dict(op=op, d=d, split=rng.choice(["mixed", "equal"]), n=n, layout=rng.choice(["row", "apart"]), grad=rng.choice(["f32", "f32", "bf16", "f16"]))
    if op == "step":
        weight = rng.choice(["f32", "f32", "bf16"])
        copy = rng.choice(["", "", "bf16", "f16"]) if weight == "f32" else ""
        case.update(bits=bits, weight=weight, copy=copy, clip=bits == 32 and rng.random() < 0.4)
    return case


def sizes_of(case):
    """Element counts of the case's tensors."""
    d, split = case["d"], case["split"]
    if split == "one":
        return [d]
    if split == "equal":
        base, extra = divmod(d, case["n"])
        return [base + (1 if i < extra else 0) for i in range(case["n"])]
    if split == "resnet18":
        sizes = [64 * 3 * 9, 64, 64] + 4 * [64 * 64 * 9, 64, 64]
        for c in (128, 256, 512):
            h = c // 2
            sizes += [c * h * 9, c, c, c * c * 9, c, c, c * h, c, c] + 2 * [c * c * 9, c, c]
        sizes += [5120, 10]
        assert sum(sizes) == d
        return sizes
    rng = random.Random(d * 1000 + case["n"])            # "mixed": a few large ones, many small ones
    part = [2.0 ** rng.uniform(0.0, 12.0) for _ in range(case["n"])]
    sizes = [max(1, int(d * p / sum(part))) for p in part]
    sizes[sizes.index(max(sizes))] += d - sum(sizes)
    return sizes


def work(case):
    d = case["d"]
    width = {"f32": 4, "bf16": 2, "f16": 2, "": 0}
    if case["op"] == "norm":
        return {"bytes": d * width[case["grad"]] + 4 * len(sizes_of(case)), "flops": 2 * d}
    each = 2 * width[case["weight"]] + width[case["grad"]] + width[case["copy"]]
    # both moments read and written; with 8 bits also an exponent each per block, and their values written in 16 bits
    each += 16 if case["bits"] == 32 else 4 * (1 + 1 / BLOCK) + 4
    return {"bytes": d * each, "flops": (16 if case["clip"] else 14) * d}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    """Tensors of a training run under way: weights, a heavy-tailed gradient with a scale of its own for every tensor, and moments
    such as a run of T0 steps with such gradients leaves."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    sizes = sizes_of(case)
    n = len(sizes)
    count = torch.tensor(sizes, device="cuda")
    blocks = (count + BLOCK - 1) // BLOCK
    block0 = blocks.cumsum(0) - blocks                    # first block of each tensor
    owner = torch.repeat_interleave(torch.arange(n, device="cuda"), blocks)          # tensor of each block
    n_blocks = owner.numel()
    start = count.cumsum(0) - count if case["layout"] == "row" else block0 * BLOCK    # first element of each tensor
    index = valid = None
    if case["layout"] == "row":                          # where the element of each place of the blocks lies
        inside = (torch.arange(n_blocks, device="cuda") - block0[owner])[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
        valid = inside < count[owner][:, None]
        index = torch.where(valid, start[owner][:, None] + inside, torch.zeros_like(inside))
        if bool(valid.all()):
            index = valid = None                          # one tensor of whole blocks
    in_use = valid
    if case["layout"] == "apart":
        in_use = ((torch.arange(n_blocks, device="cuda") - block0[owner])[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")) < count[owner][:, None]
    scale = 10.0 ** (torch.rand(n, generator=gen, device="cuda") * 2 - 4)

    def heavy(shape_of):                                  # values with heavy tails, per block and zero outside the tensors
        x = torch.rand(shape_of, generator=gen, device="cuda").clamp_(min=1e-7).log_().neg_().pow_(1.25)
        x = torch.where(torch.rand(shape_of, generator=gen, device="cuda") < 0.5, -x, x) * scale[owner][:, None]
        return x if in_use is None else torch.where(in_use, x, torch.zeros_like(x))

    def laid_out(x, kind):                                # as the layout has it
        x = x.to(TYPES[kind])
        return x[valid] if valid is not None else x.reshape(-1)

    s = dict(case=case, index=index, valid=valid, owner=owner, n=n, t=T0)
    s["grad"] = laid_out(heavy((n_blocks, BLOCK)), case["grad"])
    if case["op"] == "step":
        w = torch.randn((n_blocks, BLOCK), generator=gen, device="cuda") * 0.05
        s["weight"] = laid_out(w if in_use is None else torch.where(in_use, w, torch.zeros_like(w)), case["weight"])
        s["copy"] = torch.zeros_like(s["weight"], dtype=TYPES[case["copy"]]) if case["copy"] else None
        del w
        m = heavy((n_blocks, BLOCK)) * 0.25
        v = heavy((n_blocks, BLOCK)).square_() * 0.3 + m.square()
        decay = torch.where(count >= 1024, DECAY, 0.0)
        s["decay"] = decay[owner][:, None].float()
        # what an earlier norm of this gradient would have left: factor, norm, and the count of non-finite elements in 64 bits
        s["info"] = torch.tensor([0.25 + 0.5 * random.Random(seed).random(), 1.0, 0.0, 0.0], device="cuda")
        if case["bits"] == 8:
            zero = torch.zeros((), dtype=torch.int64, device="cuda")
            s["m"], s["m_exp"] = encode(m, M_OCTAVES, zero, True)
            s["v"], s["v_exp"] = encode(v, V_OCTAVES, zero, False)
            s["m_values"] = torch.empty((n_blocks, BLOCK), dtype=torch.bfloat16, device="cuda")
            s["v_values"] = torch.empty((n_blocks, BLOCK), dtype=torch.bfloat16, device="cuda")
        else:
            s["m"], s["v"] = m, v
    s["norms"], s["info_out"] = torch.empty(n, device="cuda"), torch.zeros(4, device="cuda")
    s["factor_norm"], s["nonfinite"] = s["info_out"][:2], s["info_out"][2:].view(torch.int64)
    if own:
        from paper_2203_09044_b200.binding import AdamW, GradNorm
        begin = start.tolist()

        def tensors(flat):
            return [flat[b:b + k] for b, k in zip(begin, sizes)]

        if case["op"] == "norm":
            s["opt"] = GradNorm(sizes, grad_dtype=TYPES[case["grad"]])
        else:
            s["opt"] = AdamW(tensors(s["weight"]), grad_dtype=TYPES[case["grad"]], copies=tensors(s["copy"]) if case["copy"] else None, lr=LR,
                             betas=(BETA1, BETA2), eps=EPS, weight_decay=[DECAY if k >= 1024 else 0.0 for k in sizes], state_bits=case["bits"], seed=SEED,
                             state={k: s[k] for k in ("m", "v", "m_exp", "v_exp") if k in s})
            s["opt"].set_steps(T0)
        s["grads"] = s["opt"].bind_grads(tensors(s["grad"]))
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------
def run(s):
    return kernels(s) if own else plain(s)


def kernels(s):
    case, opt = s["case"], s["opt"]
    if case["op"] == "norm":
        opt.grad_norm(s["grads"], s["info_out"], max_norm=MAX_NORM, tensor_norms=s["norms"])
        return {"norms": s["norms"], "info": s["factor_norm"], "nonfinite": s["nonfinite"]}
    info = opt.grad_norm(s["grads"], s["info_out"], max_norm=MAX_NORM) if case["clip"] else s["info"]
    opt.step(s["grads"], info)
    out = {"weight": s["weight"]}
    if case["copy"]:
        out["copy"] = s["copy"]
    if case["bits"] == 8:
        opt.state_values(s["m_values"], s["v_values"])
        out.update(m=s["m_values"], v=s["v_values"])
    else:
        out.update(m=s["m"], v=s["v"])
    return out


def in_blocks(x, s):
    """[blocks][256] in 32 bits, zero outside the tensors."""
    if s["index"] is None:
        return x.view(-1, BLOCK).float()
    return torch.where(s["valid"], x[s["index"]].float(), torch.zeros((), device="cuda"))


def plain_norm(s):
    g = in_blocks(s["grad"], s)
    fine = g.abs() < math.inf
    square = torch.where(fine, g * g, torch.zeros_like(g)).sum(1)
    # the sums of a tensor's blocks are joined in 64 bits: a chain of a million additions in 32 would lose what is compared
    of_tensor = torch.zeros(s["n"], dtype=torch.float64, device="cuda").index_add_(0, s["owner"], square.double())
    norm = of_tensor.sum().sqrt().float()
    factor = (MAX_NORM / norm).clamp(max=1.0)
    nonfinite = (~fine).sum()
    return of_tensor.sqrt().float(), torch.stack([factor, norm]), nonfinite.reshape(1)


def plain(s):
    case = s["case"]
    if case["op"] == "norm":
        norms, info, nonfinite = plain_norm(s)
        return {"norms": norms, "info": info, "nonfinite": nonfinite}
    factor = plain_norm(s)[1][0] if case["clip"] else s["info"][0]
    s["t"] += 1
    g = in_blocks(s["grad"], s) * factor
    w = in_blocks(s["weight"], s)
    if case["bits"] == 8:
        m, v = decode(s["m"], s["m_exp"], M_OCTAVES, True), decode(s["v"], s["v_exp"], V_OCTAVES, False)
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    c1, c2 = 1 - BETA1 ** s["t"], 1 - BETA2 ** s["t"]
    w = w - (w * (s["decay"] * LR) + (m * (LR / c1)) / (v.sqrt() * c2 ** -0.5 + EPS))
    rand = counters(w, s["t"]) if case["bits"] == 8 or case["weight"] == "bf16" else None
    new = w
    if case["weight"] == "bf16":                          # sixteen of the counter's bits decide which neighbour a weight goes to
        new = ((w.view(torch.int32) + ((rand >> 10) & 0xFFFF).int()) & -65536).view(torch.float32)
    for name, x in (("weight", new), ("copy", w)):
        if s[name] is not None:
            x = x.to(s[name].dtype)
            s[name].copy_(x.view(-1) if s["valid"] is None else x[s["valid"]])
    out = {"weight": s["weight"]}
    if case["copy"]:
        out["copy"] = s["copy"]
    if case["bits"] == 8:
        code, top = encode(m, M_OCTAVES, rand & 0xFFFFF, True)
        s["m"].copy_(code)
        s["m_exp"].copy_(top)
        code, top = encode(v, V_OCTAVES, rand >> 12, False)
        s["v"].copy_(code)
        s["v_exp"].copy_(top)
        out["m"] = decode(s["m"], s["m_exp"], M_OCTAVES, True).bfloat16()
        out["v"] = decode(s["v"], s["v_exp"], V_OCTAVES, False).bfloat16()
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        out.update(m=s["m"], v=s["v"])
    return out


# ---- the 8-bit states, in plain form --------------------------------------------------------------------------------------
# A code of 8 bits is a float with three bits of mantissa, below the exponent `top` that its block of 256 has: that of the largest
# magnitude, kept as 32-bit floats keep theirs.  OCTAVES is how many octaves below the top one still have all mantissa bits; below
# them the grid is even.  First moments: a sign and four exponent bits.  Second moments: five exponent bits, no sign, and no
# positive value goes to zero.  A value goes to the grid point above it with a probability equal to its distance from the one below.
# The top is never so low that the grid would leave the normal 32-bit floats.
M_OCTAVES, V_OCTAVES = 13, 29


def power2(e):
    """2^e for whole e of -126 .. 127."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def encode(x, octaves, rand, signed):
    mag = x.abs()
    top = (mag.amax(1, keepdim=True).view(torch.int32) >> 23).clamp(min=octaves + 4)
    least = top - 127 - octaves
    octave = torch.maximum((mag.view(torch.int32) >> 23) - 127, least)
    steps = (mag * power2(3 - octave) * 1048576.0).round().to(torch.int64)           # in 2^-20 of a grid step
    steps = ((steps + rand) >> 20).to(torch.int32)
    code = (octave - least) * 8 + steps
    code = torch.where(x < 0, code + 128, code) if signed else torch.maximum(code, (x > 0).int())
    return code.to(torch.uint8), top.view(-1).to(torch.uint8)


def decode(code, top, octaves, signed):
    least = (top.int() - 127 - octaves)[:, None]
    code = code.int()
    mag = code & 127 if signed else code
    octave = ((mag >> 3) - 1).clamp(min=0)
    x = (mag - octave * 8).float() * power2(octave + least - 3)
    return torch.where(code > 127, -x, x) if signed else x


def mixed(x):
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x046CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def counters(like, t):
    """32 bits for each place of the blocks at step t."""
    s = (torch.arange(like.numel(), device="cuda").view(-1, BLOCK) * 0x9E3779B9 + mixed((mixed(SEED) + t) & 0xFFFFFFFF)) & 0xFFFFFFFF
    return ((s ^ (s >> 15)) * 0x2C1B3C6D) & 0xFFFFFFFF


# ---- the same in 64 bits ----------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    rows = s["owner"].numel()

    def blocks(flat):
        if s["valid"] is None:
            return flat.to(f64).reshape(rows, BLOCK)
        full = torch.zeros((rows, BLOCK), dtype=f64, device="cuda")
        full[s["valid"]] = flat.to(f64)
        return full

    g = blocks(s["grad"])
    fine = torch.isfinite(g)
    sums = torch.zeros(s["n"], dtype=f64, device="cuda").index_add_(0, s["owner"], torch.where(fine, g, 0.0).pow(2).sum(1))
    norm = sums.sum().sqrt()
    factor = torch.clamp(MAX_NORM / norm, max=1.0)
    if case["op"] == "norm":
        return {"norms": sums.sqrt(), "info": torch.stack([factor, norm]), "nonfinite": (~fine).sum().reshape(1)}
    if not case["clip"]:
        factor = s["info"][0].to(f64)
    t = T0 + 1
    if case["bits"] == 8:
        m, v = value64(s["m"], s["m_exp"], 4), value64(s["v"], s["v_exp"], 5)
    else:
        m, v = s["m"].to(f64), s["v"].to(f64)
    m = BETA1 * m + (1 - BETA1) * factor * g
    v = BETA2 * v + (1 - BETA2) * (factor * g) ** 2
    w = blocks(s["weight"])
    w = w - LR * (s["decay"].to(f64) * w + (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS))
    flat = w.reshape(-1) if s["valid"] is None else w[s["valid"]]
    out = {"weight": flat}
    if case["copy"]:
        out["copy"] = flat
    if case["bits"] == 8:
        place = torch.arange(rows * BLOCK, device="cuda").reshape(rows, BLOCK)
        r = (mixed((mixed(SEED) + t) % 2 ** 32) + place * 0x9E3779B9) % 2 ** 32
        r = (r.bitwise_xor(r // 2 ** 15) * 0x2C1B3C6D) % 2 ** 32
        m, v = grid64(m, (r % 2 ** 20).to(f64) / 2 ** 20, 4, 0), grid64(v, (r // 2 ** 12).to(f64) / 2 ** 20, 5, 1)
    out.update(m=m, v=v)
    return out


def value64(code, top, exponent_bits):
    """What codes stand for: sign, exponent field and three mantissa bits, the block's top exponent in the field 2^bits - 2."""
    c = code.to(torch.int64)
    sign = torch.where((c >= 128) & torch.tensor(exponent_bits == 4, device="cuda"), -1.0, 1.0).double()
    c = c % 2 ** (exponent_bits + 3)
    field, low = c // 8, c % 8
    n = torch.where(field > 0, 8 + low, low).double()
    unit = torch.clamp(field, min=1) - (2 ** exponent_bits - 2) - 3 + (top.to(torch.int64) - 127)[:, None]
    return sign * n * torch.exp2(unit.double())


def grid64(x, u, exponent_bits, least):
    """Nearest grid values at or below |x| + u steps."""
    a = x.abs()
    e = torch.frexp(a)[1].double() - 1
    top = torch.clamp(torch.frexp(a.amax(1, keepdim=True))[1].double() - 1, min=2 ** exponent_bits + 1 - 127)
    step = torch.exp2(torch.maximum(e, top - (2 ** exponent_bits - 3)) - 3)
    n = torch.floor(a / step + u)
    n = torch.where(a > 0, torch.clamp(n, min=least), torch.zeros_like(n))
    return torch.sign(x) * n * step
