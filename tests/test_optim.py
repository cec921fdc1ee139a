"""The optimizer operators: gradient norm with its clipping factor, AdamW with moments in 32 bits and in 8.

The reference is numpy.  The moments are compared bit for bit with the same products and sums rounded one by one to
32 bits (and those with the formula in 64 bits), the codes of the 8-bit moments as whole numbers with the rounding rule
carried out in 64 bits, where every scaled value is exact.  Weights: each of the roughly twelve roundings of an update
costs at most 2^-24 of it, square root and quotient taken to two units in the last place; 2^-20 of the update and one
rounding of the weight bound their sum."""
import ctypes as C
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
f32 = np.float32

M_FIELD, V_FIELD = 14, 30          # exponent field of a block's top octave


# ---- reference --------------------------------------------------------------------------------------------------------------
def mix32(x):
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x046CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def counter_bits(seed, t, places):
    """The 32 random bits of each place of the moment arrays at step t."""
    p = np.asarray(places, np.uint64)
    key = np.uint64(mix32((mix32(seed) + t) & 0xFFFFFFFF)) + (p >> np.uint64(32)) * np.uint64(0x632BE5AB)
    s = (key + (p & np.uint64(0xFFFFFFFF)) * np.uint64(0x9E3779B9)) & np.uint64(0xFFFFFFFF)
    return (((s ^ (s >> np.uint64(15))) * np.uint64(0x2C1B3C6D)) & np.uint64(0xFFFFFFFF)).astype(np.int64)


def decode_ref(code, top, field, signed):
    """[blocks][256] codes -> float64 values."""
    c = code.astype(np.int64)
    mag = c & 127 if signed else c
    e, k = mag >> 3, mag & 7
    n = np.where(e > 0, 8 + k, k)
    x = np.ldexp(n.astype(np.float64), (np.maximum(e, 1) - 1 + top.astype(np.int64)[:, None] - 127 - field - 2).astype(np.int32))
    return np.where(c > 127, -x, x) if signed else x


def encode_ref(x, rand, field, signed):
    """[blocks][256] float64 that hold float32 values -> codes, top exponents."""
    a = np.abs(x)
    big = a.max(1).astype(f32)
    top = np.maximum(big.view(np.uint32) >> 23, field + 3).astype(np.int64)
    least = (top - 127 - field + 1)[:, None]                            # octave of field 1
    octave = np.maximum(np.frexp(np.where(a > 0, a, 1e-300))[1] - 1, least)
    steps = np.rint(np.ldexp(a, (23 - octave).astype(np.int32))).astype(np.int64)    # in 2^-20 of a grid step
    code = (octave - least) * 8 + ((steps + rand) >> 20)
    if signed:
        code = np.where(x < 0, code + 128, code)
    else:
        code = np.maximum(code, (x > 0).astype(np.int64))
    return code.astype(np.uint8), top.astype(np.uint8)


def bf16_to_f32(bits):
    return (bits.astype(np.uint32) << 16).view(f32)


class Reference:
    """AdamW over tensors of the given sizes; the moments in blocks, weights as one float32 array per tensor."""

    def __init__(self, weights, decay, bits, lr, betas, eps, seed, w16):
        self.w = [np.array(w, f32) for w in weights]
        self.sizes = [w.size for w in self.w]
        self.decay, self.bits, self.lr, self.betas, self.eps, self.seed, self.w16 = decay, bits, lr, betas, eps, seed, w16
        self.nb = [(n + 255) // 256 for n in self.sizes]
        self.b0 = np.concatenate([[0], np.cumsum(self.nb)])[:-1]
        total = int(sum(self.nb))
        self.m, self.v = np.zeros((total, 256), f32), np.zeros((total, 256), f32)
        self.mc = self.vc = np.zeros((total, 256), np.uint8)
        self.mt = self.vt = np.zeros(total, np.uint8)
        self.t = 0
        self.kept = 0
        self.w_tol = None

    def blocks(self, tensors):
        out = np.zeros(self.m.size, f32)
        for b, x in zip(self.b0, tensors):
            out[b * 256:b * 256 + x.size] = x
        return out.reshape(-1, 256)

    def step(self, grads, factor=1.0, lr=None):
        self.t += 1
        lr = self.lr if lr is None else lr
        b1, b2 = self.betas
        with np.errstate(all="ignore"):
            g = self.blocks(grads) * f32(factor)
            m0, v0 = self.m, self.v
            if self.bits == 8:
                m0, v0 = decode_ref(self.mc, self.mt, M_FIELD, True).astype(f32), decode_ref(self.vc, self.vt, V_FIELD, False).astype(f32)
            m = m0 * f32(b1) + g * f32(1.0 - b1)
            v = v0 * f32(b2) + (g * g) * f32(1.0 - b2)
            fine = v < f32(2.0 ** 126)
        # the same in 64 bits: three roundings of 32 bits each, and those of the two constants
        g64 = self.blocks(grads).astype(np.float64) * factor
        m64, v64 = m0.astype(np.float64) * b1 + g64 * (1 - b1), v0.astype(np.float64) * b2 + g64 * g64 * (1 - b2)
        tiny = 1e-44
        with np.errstate(invalid="ignore"):
            assert (np.abs(m - m64) <= 6 * 2.0 ** -24 * (np.abs(m0 * b1) + np.abs(g64 * (1 - b1))) + tiny)[fine].all()
            assert (np.abs(v - v64) <= 8 * 2.0 ** -24 * (np.abs(v0 * b2) + g64 * g64 * (1 - b2)) + tiny)[fine].all()
        self.kept += int((~fine).sum())
        m, v = np.where(fine, m, m0), np.where(fine, v, v0)
        w = self.blocks(self.w).astype(np.float64)
        decay = np.concatenate([np.full((n, 1), d) for n, d in zip(self.nb, self.decay)]) if sum(self.nb) else np.zeros((0, 1))
        with np.errstate(all="ignore"):
            upd = lr * (m.astype(np.float64) / (1 - b1 ** self.t)) / (np.sqrt(v.astype(np.float64) / (1 - b2 ** self.t)) + self.eps)
            new = np.where(fine, w - (lr * decay * w + upd), w)
        tol = np.where(fine, 2.0 ** -23 * np.abs(new) + 2.0 ** -20 * (np.abs(upd) + np.abs(lr * decay * w)), 0.0) + tiny
        self.rand = counter_bits(self.seed, self.t, np.arange(m.size)).reshape(m.shape)
        if self.bits == 8:
            m, v = np.where(np.isfinite(m), m, 0), np.where(np.isfinite(v), v, 0)
            self.mc, self.mt = encode_ref(m.astype(np.float64), self.rand & 0xFFFFF, M_FIELD, True)
            self.vc, self.vt = encode_ref(v.astype(np.float64), self.rand >> 12, V_FIELD, False)
        else:
            self.m, self.v = m, v
        self.new, self.fine = new, fine

        def back(x):
            flat = x.reshape(-1)
            return [flat[b * 256:b * 256 + n] for b, n in zip(self.b0, self.sizes)]
        return back(new), back(tol), back(fine), back(self.rand)


DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def make(sizes, dtype, gen, off=0, scale=1.0, device="cuda"):
    """Tensors back to back in one buffer, each `off` elements further on than it has to be."""
    out = []
    buf = torch.empty(sum(sizes) + off * (len(sizes) + 1) + 64, dtype=dtype, device=device)
    at = off
    for n in sizes:
        x = torch.randn(n, generator=gen) * scale * 10.0 ** (torch.rand(1, generator=gen).item() * 2 - 1)
        buf[at:at + n] = x.to(dtype).to(device)
        out.append(buf[at:at + n])
        at += n + off
    return out


def as_f32(ts):
    return [t.detach().float().cpu().numpy() for t in ts]


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2203_09044_b200 import binding as b
    b.lib()
    return b


SETS = {
    "one": [1], "block": [256], "over": [257], "empty": [0, 5, 0, 300, 0], "many": [1, 7, 64, 255, 256, 513] * 50,
    "long": [70_001, 8, 131_072], "table": [3] * 1400,
}


# ---- gradient norm -------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("name", list(SETS))
@pytest.mark.parametrize("off", [0, 1])
def test_norm(binding, name, dtype, off):
    sizes = SETS[name]
    gen = torch.Generator().manual_seed(len(name) + off)
    grads = make(sizes, DT[dtype], gen, off)
    ref = [x.astype(np.float64) for x in as_f32(grads)]
    sq = np.array([(x * x).sum() for x in ref])
    opt = binding.GradNorm(sizes, DT[dtype])
    norms = torch.full((len(sizes),), -1.0, device="cuda")
    for scale, most in ((1.0, 0.0), (0.5, 1e9), (2.0, 0.25)):
        info = opt.grad_norm(grads, max_norm=most, grad_scale=scale, tensor_norms=norms)
        f, n = info[:2].tolist()
        want = scale * math.sqrt(sq.sum())
        # 64-bit sums, rounded once to 32 bits
        assert abs(n - want) <= 2.0 ** -23 * want
        factor = scale * (min(1.0, most / want) if most > 0 else 1.0)
        assert abs(f - factor) <= 2.0 ** -23 * factor
        assert info[2:].view(torch.int64).item() == 0
        np.testing.assert_allclose(norms.cpu().numpy(), scale * np.sqrt(sq), rtol=2.0 ** -23, atol=0)
    again = opt.grad_norm(opt.bind_grads(grads), max_norm=0.25, grad_scale=2.0)
    assert torch.equal(again.view(torch.int32), info.view(torch.int32))


@pytest.mark.gpu
def test_norm_of_extreme_values(binding):
    """Squares that leave the range of 32 bits at either end, zeros, and non-finite elements, which are counted and left out."""
    sizes = [1000, 1000, 300, 1000]
    gen = torch.Generator().manual_seed(5)
    grads = make(sizes, torch.float32, gen, 1)
    grads[0].mul_(1e37)
    grads[1].mul_(1e-42)
    grads[2].zero_()
    opt = binding.GradNorm(sizes)
    norms = torch.empty(4, device="cuda")

    def check(bad):
        info = opt.grad_norm(grads, tensor_norms=norms)
        ref = [x.astype(np.float64) for x in as_f32(grads)]
        sq = [float((x[np.isfinite(x)] ** 2).sum()) for x in ref]
        np.testing.assert_allclose(norms.cpu().numpy(), np.sqrt(sq).astype(f32), rtol=2.0 ** -22, atol=2e-45)
        assert abs(info[1].item() - math.sqrt(sum(sq))) <= 2.0 ** -23 * math.sqrt(sum(sq))
        assert info[2:].view(torch.int64).item() == bad
    check(0)
    grads[3][[0, 255, 256, 999]] = torch.tensor([float("inf"), float("nan"), -float("inf"), float("nan")], device="cuda")
    check(4)
    for g in grads:
        g.fill_(float("nan"))
    info = opt.grad_norm(grads, max_norm=1.0)
    assert info[:2].tolist() == [1.0, 0.0] and info[2:].view(torch.int64).item() == sum(sizes)


# ---- the step ---------------------------------------------------------------------------------------------------------------------
def run_steps(binding, sizes, bits, weight="f32", grad="f32", copy=None, off=0, steps=3, factor=None, betas=(0.9, 0.999), eps=1e-8, lr=1e-2,
              seed=7, decay=None, grads_of=None, stream=None, scale=1.0):
    gen = torch.Generator().manual_seed(sum(sizes) + bits)
    params = make(sizes, DT[weight], gen, off)
    copies = None if copy is None else make(sizes, DT[copy], gen, off)
    decay = [0.1 * (i % 3) for i in range(len(sizes))] if decay is None else decay
    opt = binding.AdamW(params, grad_dtype=DT[grad], copies=copies, lr=lr, betas=betas, eps=eps, weight_decay=decay, state_bits=bits, seed=seed)
    ref = Reference(as_f32(params), np.array(decay, f32).astype(np.float64), bits, lr, betas, eps, seed, weight == "bf16")
    info = None if factor is None else torch.tensor([factor, 0, 0, 0], device="cuda", dtype=torch.float32)
    for t in range(steps):
        grads = make(sizes, DT[grad], gen, off, scale) if grads_of is None else grads_of(t, gen)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        opt.step(grads, info, stream=stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        f = 1.0 if info is None else float(info[0].item())
        new, tol, fine, rand = ref.step(as_f32(grads), f)
        if bits == 8:
            for got, want, what in ((opt.m_exp, ref.mt, "m_exp"), (opt.v_exp, ref.vt, "v_exp"), (opt.m, ref.mc, "m"), (opt.v, ref.vc, "v")):
                assert np.array_equal(got.cpu().numpy(), want), f"t={t} {what}"
            for dt in (torch.bfloat16, torch.float32):
                mv = opt.state_values(*(torch.empty((opt.n_blocks, 256), dtype=dt, device="cuda") for _ in range(2)))
                assert np.array_equal(mv[0].double().cpu().numpy(), decode_ref(ref.mc, ref.mt, M_FIELD, True))
                assert np.array_equal(mv[1].double().cpu().numpy(), decode_ref(ref.vc, ref.vt, V_FIELD, False))
        else:
            assert np.array_equal(opt.m.cpu().numpy().view(np.uint32), ref.m.view(np.uint32)), f"t={t} m"
            assert np.array_equal(opt.v.cpu().numpy().view(np.uint32), ref.v.view(np.uint32)), f"t={t} v"
        for i, p in enumerate(params):
            got = as_f32([p])[0]
            if weight == "bf16":
                # the neighbour that the counter's bits choose; where 32 bits of the update differ from 64, either of the two choices
                lo, hi = (new[i] - tol[i]).astype(f32), (new[i] + tol[i]).astype(f32)
                r = ((rand[i] >> 10) & 0xFFFF).astype(np.uint32)
                a, b = (bf16_to_f32(((x.view(np.uint32) + r) >> 16)) for x in (lo, hi))
                ok = (got >= np.minimum(a, b)) & (got <= np.maximum(a, b)) | (~fine[i] & (got == ref.w[i]))
                assert ok.all(), f"t={t} weights {i}"
            else:
                assert (np.abs(got - new[i]) <= tol[i]).all(), f"t={t} weights {i}"
                if copies is not None:
                    assert torch.equal(copies[i], p.to(DT[copy])), f"t={t} copy {i}"
            ref.w[i] = got
    assert opt.steps() == steps
    return opt, ref, params


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("name", list(SETS))
def test_step_over_sets_of_tensors(binding, name, off, bits):
    opt, _, _ = run_steps(binding, SETS[name], bits, off=off, factor=0.3)
    assert opt.status() == (0, 0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("weight,grad,copy", [("f32", "bf16", "bf16"), ("f32", "f16", "f16"), ("f32", "f32", "bf16"), ("bf16", "bf16", None),
                                              ("bf16", "f32", None), ("bf16", "f16", None), ("f32", "bf16", None)])
@pytest.mark.parametrize("off", [0, 1, 4, 8])
def test_step_over_types_and_alignments(binding, weight, grad, copy, bits, off):
    run_steps(binding, [4097, 512, 3, 2048, 40], bits, weight, grad, copy, off)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("betas", [(0.0, 0.0), (0.9, 0.95), (0.0, 0.999), (0.5, 0.0), (1e-3, 0.9), (2.0 ** -9, 1e-6)])
@pytest.mark.parametrize("eps", [0.0, 1e-8, 1.0])
def test_step_over_constants(binding, bits, betas, eps):
    run_steps(binding, [1000, 5], bits, betas=betas, eps=eps)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_step_over_magnitudes(binding, bits):
    """Gradients from 1e-30 to 1e17 in one block each, one block across all of them, and zeros: block exponents at both ends of
    their range, subnormal codes, positive second moments below the grid."""
    def grads_of(t, gen):
        x = torch.randn(256 * 8, generator=gen)
        for b, s in enumerate((1e-30, 1e-18, 1e-12, 1e-3, 1e6, 1e17)):
            x[256 * b:256 * b + 256] *= s
        x[256 * 6:256 * 7] *= 10.0 ** torch.linspace(-20, 10, 256)
        x[256 * 7:] = 0
        return [x.cuda()]
    opt, ref, _ = run_steps(binding, [2048], bits, grads_of=grads_of, eps=1e-8, steps=4)
    assert opt.status() == (0, 0, 0)
    if bits == 8:
        assert (ref.vc[6] >= 1).all() and (ref.vc[6] == 1).any() and (ref.vc[7] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("weight", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_elements_without_a_finite_second_moment_stay(binding, bits, weight):
    def grads_of(t, gen):
        x = torch.randn(700, generator=gen)
        x[[0, 31, 32, 255, 256, 699]] = torch.tensor([float("inf"), float("nan"), -float("inf"), 1e30, -float("nan"), 3e38])
        return [x.cuda(), torch.full((40,), float("nan")).cuda()]
    opt, ref, params = run_steps(binding, [700, 40], bits, weight, grads_of=grads_of)
    flags, elements, steps = opt.status(clear=True)
    assert flags == binding.FLAG_NONFINITE and elements == ref.kept == 3 * 46 and steps == 0
    assert opt.status() == (0, 0, 0)
    assert all(torch.isfinite(p).all() for p in params)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_is_left_out_when_the_norm_found_a_bad_element(binding, bits):
    gen = torch.Generator().manual_seed(1)
    sizes = [300, 1, 0, 5000]
    params, grads = make(sizes, torch.float32, gen), make(sizes, torch.float32, gen)
    opt = binding.AdamW(params, state_bits=bits)
    opt.step(grads, opt.grad_norm(grads, max_norm=1.0))
    before = [t.clone() for t in params + [opt.m, opt.v]]
    grads[3][77] = float("nan")
    info = opt.grad_norm(grads, max_norm=1.0)
    opt.step(grads, info)
    assert all(torch.equal(a, b) for a, b in zip(before, params + [opt.m, opt.v]))
    assert opt.steps() == 1 and opt.status() == (binding.FLAG_NONFINITE, 0, 1)
    grads[3][77] = 0.5
    opt.step(grads, opt.grad_norm(grads, info, max_norm=1.0))
    assert opt.steps() == 2 and not torch.equal(before[3], params[3])


@pytest.mark.gpu
def test_clipped_steps_follow_the_formula_in_64_bits(binding):
    """Norm, factor and step as a training loop calls them, against the whole formula in 64 bits."""
    gen = torch.Generator().manual_seed(3)
    sizes = [5000, 10, 777]
    params = make(sizes, torch.float32, gen)
    w = [x.astype(np.float64) for x in as_f32(params)]
    m, v = [np.zeros_like(x) for x in w], [np.zeros_like(x) for x in w]
    opt = binding.AdamW(params, lr=1e-2, weight_decay=0.1)
    for t in range(1, 6):
        grads = make(sizes, torch.float32, gen)
        opt.step(grads, opt.grad_norm(grads, max_norm=1.0))
        g = [x.astype(np.float64) for x in as_f32(grads)]
        f = min(1.0, 1.0 / math.sqrt(sum((x * x).sum() for x in g)))
        for i in range(3):
            m[i] = 0.9 * m[i] + 0.1 * f * g[i]
            v[i] = 0.999 * v[i] + 0.001 * (f * g[i]) ** 2
            w[i] = w[i] - 1e-2 * (0.1 * w[i] + m[i] / (1 - 0.9 ** t) / (np.sqrt(v[i] / (1 - 0.999 ** t)) + 1e-8))
            # at most t times the bound of one step, whose updates are below 10 lr here
            assert np.abs(as_f32([params[i]])[0] - w[i]).max() <= t * (2.0 ** -23 * np.abs(w[i]).max() + 2.0 ** -19 * 0.1)


@pytest.mark.gpu
def test_channels_last_weights(binding):
    gen = torch.Generator().manual_seed(4)
    w = torch.randn(16, 8, 3, 3, generator=gen).cuda()
    g = torch.randn(16, 8, 3, 3, generator=gen).cuda()
    a, b = w.clone(), w.clone(memory_format=torch.channels_last)
    oa, ob = binding.AdamW([a]), binding.AdamW([b])
    oa.step([g])
    ob.step([g.contiguous(memory_format=torch.channels_last)])
    assert torch.equal(a, b) and not b.is_contiguous()
    with pytest.raises(ValueError, match="another order"):
        ob.step([g])
    with pytest.raises(ValueError, match="another order"):
        oa.step([g.contiguous(memory_format=torch.channels_last)])


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_on_another_stream(binding, bits):
    run_steps(binding, [3000, 77], bits, stream=torch.cuda.Stream(), factor=0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 200])
@pytest.mark.parametrize("bits", [32, 8])
def test_replayed_from_a_graph(binding, bits, n):
    """A captured norm + step, replayed with other gradients and learning rates, gives the bits of the calls one by one."""
    gen = torch.Generator().manual_seed(6)
    sizes = [(37 * i) % 600 for i in range(1, n + 1)]
    w0 = make(sizes, torch.float32, gen)
    data = [make(sizes, torch.float32, gen) for _ in range(4)]
    one = [w.clone() for w in w0]
    oa = binding.AdamW(one, state_bits=bits, seed=9)
    for t, g in enumerate(data):
        oa.step(g, oa.grad_norm(g, max_norm=1.0), lr=1e-3 * (t + 1))
    two, grads = [w.clone() for w in w0], [torch.zeros_like(w) for w in w0]
    ob = binding.AdamW(two, state_bits=bits, seed=9)
    info, lr = torch.zeros(4, device="cuda"), torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    bound = ob.bind_grads(grads)
    with torch.cuda.graph(graph):
        ob.grad_norm(bound, info, max_norm=1.0)
        ob.step(bound, info, lr=lr)
    for t, g in enumerate(data):
        for x, y in zip(grads, g):
            x.copy_(y)
        lr.fill_(1e-3 * (t + 1))
        graph.replay()
    assert ob.steps() == 4
    assert all(torch.equal(a, b) for a, b in zip(one, two)) and torch.equal(oa.m, ob.m) and torch.equal(oa.v, ob.v)


@pytest.mark.gpu
def test_resumed_run_gives_the_same_bits(binding):
    gen = torch.Generator().manual_seed(8)
    sizes = [1000, 30]
    w0, data = make(sizes, torch.bfloat16, gen), [make(sizes, torch.bfloat16, gen) for _ in range(6)]
    a, b = [w.clone() for w in w0], [w.clone() for w in w0]
    oa = binding.AdamW(a, state_bits=8, seed=2)
    for g in data:
        oa.step(g)
    ob = binding.AdamW(b, state_bits=8, seed=2)
    for g in data[:3]:
        ob.step(g)
    saved = {k: getattr(ob, k).clone() for k in ("m", "v", "m_exp", "v_exp")}
    oc = binding.AdamW(b, state_bits=8, seed=2, state=saved)
    oc.set_steps(ob.steps())
    for g in data[3:]:
        oc.step(g)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(oa.m, oc.m) and torch.equal(oa.v_exp, oc.v_exp)
    # far into a run: one optimizer that took the steps, one that is told so
    w = [torch.ones(64, device="cuda") for _ in range(2)]
    z, g = [torch.zeros(64, device="cuda")], [torch.full((64,), 0.5, device="cuda")]
    od, oe = binding.AdamW([w[0]], weight_decay=0.0), binding.AdamW([w[1]], weight_decay=0.0)
    bound = od.bind_grads(z)
    for _ in range(3000):
        od.step(bound)
    oe.set_steps(3000)
    od.step(g)
    oe.step(g)
    assert od.steps() == oe.steps() == 3001 and torch.equal(w[0], w[1]) and not torch.equal(w[0], torch.ones_like(w[0]))
    m, v = oc.moments_of(1)
    assert m.numel() == v.numel() == 30 and m.data_ptr() == oc.m.data_ptr() + 1024


@pytest.mark.gpu
def test_rounding_is_unbiased(binding):
    """65,536 second moments that each step moves by less than a tenth of a grid step: under rounding to nearest they would stay
    where they are; their mean has to follow the 32-bit average.  One value's standard deviation is at most a quarter of it
    (about 8 grid steps of 1/16 .. 1/8, squared and weighted), so 1% is over ten standard deviations of the mean."""
    n = 1 << 16
    g = torch.full((n,), 1e-3, device="cuda")
    p8, p32 = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    o8, o32 = binding.AdamW([p8], state_bits=8, lr=0.0), binding.AdamW([p32], state_bits=32, lr=0.0)
    for t in range(1, 1001):
        o8.step([g])
        o32.step([g])
        if t in (10, 100, 1000):
            m, v = (x.double().mean().item() for x in o8.state_values())
            assert abs(v / o32.v.double().mean().item() - 1) < 0.01
            assert abs(m / o32.m.double().mean().item() - 1) < 0.01


@pytest.mark.gpu
def test_more_than_2_to_the_32_elements(binding):
    """Offsets beyond 32 bits: the ends of a tensor of 2^32 + 300 elements and one after it, with the smallest types."""
    n = (1 << 32) + 300
    p, g = torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    q, h = torch.ones(5, dtype=torch.bfloat16, device="cuda"), torch.full((5,), 0.25, dtype=torch.bfloat16, device="cuda")
    g[-300:] = torch.linspace(-1, 1, 300, device="cuda").bfloat16()
    g[:256] = 0.5
    opt = binding.AdamW([p, q], state_bits=8, lr=1e-2, weight_decay=0.0, seed=3)
    info = opt.grad_norm([g, h], max_norm=0.0)
    want = math.sqrt(float((g[-300:].double() ** 2).sum() + 256 * 0.25 + 5 * 0.0625))
    assert abs(info[1].item() - want) <= 2.0 ** -23 * want
    opt.step([g, h], info)
    places = np.arange(n - 300, n)
    r = counter_bits(3, 1, places)
    x = g[-300:].float().cpu().numpy()
    m = (x * f32(1 - 0.9)).astype(np.float64)
    for lo, hi in ((0, 0), (0, 256), (256, 300)):
        if hi == lo:
            continue
        a, b = slice(lo, hi), (n - 300 + lo) // 256
        pad = np.zeros((1, 256))
        rr = np.zeros((1, 256), np.int64)
        start = (n - 300 + lo) % 256
        pad[0, start:start + hi - lo], rr[0, start:start + hi - lo] = m[a], r[a] & 0xFFFFF
        code, top = encode_ref(pad, rr, M_FIELD, True)
        got = opt.m[b].cpu().numpy()
        assert np.array_equal(got[start:start + hi - lo], code[0, start:start + hi - lo]) and opt.m_exp[b].item() == top[0]
    assert (p[:256] != 1).all() and (p[256:1 << 20] == 1).all() and (p[-300:-150] > 0.98).all() and (q != 1).all()


# ---- refusals ----------------------------------------------------------------------------------------------------------------------
def test_bad_configurations_are_refused_on_the_host():
    from paper_2203_09044_b200 import binding as b, build
    build.build()
    L = b.lib()

    def create(sizes=(10, 20), **kw):
        n = np.array(sizes, np.int64)
        d = dict(n_tensors=len(sizes), decay=None, weight=b.F32, grad=b.F32, copy=b.NONE, bits=32, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, reserved=0)
        d.update(kw)
        dec = None if d["decay"] is None else np.array(d["decay"], np.float32)
        cfg = b.AdamwConfig(d["n_tensors"], n.ctypes.data_as(C.POINTER(C.c_int64)), None if dec is None else dec.ctypes.data_as(C.POINTER(C.c_float)),
                            d["weight"], d["grad"], d["copy"], d["bits"], d["b1"], d["b2"], d["eps"], d["wd"], 0, d["reserved"])
        h = C.c_void_p()
        rc = L.co3_adamw_create(C.byref(h), C.byref(cfg))
        if rc == 0:
            L.co3_adamw_destroy(h)
        else:
            assert not h.value
        return rc

    nan, inf = float("nan"), float("inf")
    for bad in (dict(n_tensors=0), dict(sizes=(-1,)), dict(sizes=((1 << 40) + 1,)), dict(sizes=(1 << 40,)), dict(weight=b.F16), dict(weight=3), dict(grad=b.NONE),
                dict(copy=b.F32), dict(copy=b.BF16, weight=b.BF16), dict(bits=16), dict(b1=1.0), dict(b1=-0.1), dict(b2=nan), dict(b2=1.0),
                dict(eps=-1e-8), dict(eps=inf), dict(wd=nan), dict(wd=-1.0), dict(decay=(0.0, nan)), dict(decay=(0.0, -1.0)), dict(reserved=1)):
        assert create(**bad) == b.EINVAL, bad
    assert L.co3_adamw_create(None, None) == b.EINVAL
    for call in (lambda: L.co3_adamw_sizes(None, None, None), lambda: L.co3_grad_norm(None, None, 1.0, 0.0, None, None, None),
                 lambda: L.co3_adamw_step(None, None, None, None, None, 0.0, None, None, None), lambda: L.co3_adamw_values(None, None, None, None, 0, None),
                 lambda: L.co3_adamw_status(None, None, None, None, 0), lambda: L.co3_adamw_steps_export(None, None), lambda: L.co3_adamw_steps_import(None, 0)):
        assert call() == b.EINVAL
    L.co3_adamw_destroy(None)
    if not torch.cuda.is_available():
        assert create() in (b.ENOMEM, b.ECUDA)


@pytest.mark.gpu
def test_bad_calls_are_refused(binding):
    b = binding
    dev = dict(device="cuda")
    p, g = torch.ones(300, **dev), torch.ones(300, **dev)
    opt = b.AdamW([p, torch.ones(4, **dev)], state_bits=8)
    good = [g, torch.ones(4, **dev)]
    for bad, word in ((good[:1], "2 gradients"), ([g[:299], good[1]], "300 elements"), ([g.half(), good[1]], "float32"), ([g.cpu(), good[1]], "cuda"),
                      ([torch.ones(600, **dev)[::2], good[1]], "one piece")):
        with pytest.raises(ValueError, match=word):
            opt.step(bad)
        with pytest.raises(ValueError, match=word):
            opt.grad_norm(bad)
    with pytest.raises(ValueError, match="info"):
        opt.step(good, torch.ones(3, **dev))
    with pytest.raises(ValueError, match="lr"):
        opt.step(good, lr=torch.ones(2, **dev))
    for call in (lambda: opt.step(good, lr=float("nan")), lambda: opt.step(good, torch.ones(6, **dev)[1:5]), lambda: opt.grad_norm(good, torch.ones(6, **dev)[1:5]),
                 lambda: opt.grad_norm(good, grad_scale=float("inf")), lambda: opt.grad_norm(good, max_norm=float("nan")),
                 lambda: b.AdamW([p], state_bits=32).state_values(), lambda: opt.set_steps(-1)):
        with pytest.raises(b.Co3Error) as e:
            call()
        assert e.value.code == b.EINVAL
    with pytest.raises(ValueError):
        b.AdamW([])
    with pytest.raises(TypeError):
        b.AdamW([p.double()])
    with pytest.raises(ValueError, match="weight_decay"):
        b.AdamW([p], weight_decay=[0.1, 0.1])
    with pytest.raises(ValueError, match="m:"):
        b.AdamW([p], state=dict(m=torch.zeros(256, **dev), v=torch.zeros(512, **dev)))
    with pytest.raises(b.Co3Error):
        b.AdamW([p], state_bits=16)
    assert opt.steps() == 0 and opt.status() == (0, 0, 0) and torch.equal(p, torch.ones_like(p))
    L, null = b.lib(), None
    two = (C.c_void_p * 2)(g.data_ptr(), good[1].data_ptr())
    odd = (C.c_void_p * 2)(g.data_ptr() + 2, good[1].data_ptr())
    none = (C.c_void_p * 2)(None, good[1].data_ptr())
    w = opt.params.pointers
    info = torch.ones(4, **dev)
    for args in ((w, odd, null), (w, none, null), (odd, two, null), (none, two, null), (w, two, two)):
        assert L.co3_adamw_step(opt.handle, args[0], args[1], args[2], opt._state_p, 1e-3, null, null, null) == b.EINVAL
    empty = b.AdamwState(opt.m.data_ptr() + 4, opt.v.data_ptr(), opt.m_exp.data_ptr(), opt.v_exp.data_ptr())
    assert L.co3_adamw_step(opt.handle, w, two, null, C.byref(empty), 1e-3, null, null, null) == b.EINVAL
    assert L.co3_grad_norm(opt.handle, none, 1.0, 0.0, null, info.data_ptr(), null) == b.EINVAL
    assert L.co3_grad_norm(opt.handle, two, 1.0, 0.0, null, null, null) == b.EINVAL
    torch.cuda.synchronize()
    assert opt.steps() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_no_elements_at_all(binding, bits):
    p = torch.empty(0, device="cuda")
    opt = binding.AdamW([p, p], state_bits=bits)
    info = opt.grad_norm([p, p], max_norm=1.0)
    assert info[:2].tolist() == [1.0, 0.0]
    opt.step([p, p], info)
    assert opt.steps() == 1 and opt.n_blocks == 0


@pytest.mark.gpu
def test_bound_gradients_of_another_optimizer_are_checked_again(binding):
    b = binding
    p, q = [torch.ones(300, device="cuda")], [torch.ones(5000, device="cuda")]
    small, large = b.AdamW(p), b.AdamW(q)
    bound = small.bind_grads([torch.ones(300, device="cuda")])
    small.step(bound)
    with pytest.raises(ValueError, match="5000 elements"):
        large.step(bound)
    with pytest.raises(ValueError, match="bfloat16"):
        b.AdamW(p, grad_dtype=torch.bfloat16).grad_norm(bound)
    b.AdamW([torch.ones(300, device="cuda")]).step(bound)          # fits: used as it is
    assert large.steps() == 0


# ---- mixtures, neighbours in memory, calls in a row ---------------------------------------------------------------------------------
def _mixture(n, top, seed):
    rng = np.random.default_rng(seed)
    return [int(x) for x in np.exp(rng.uniform(0.0, math.log(top), n)).astype(np.int64)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,top,off", [(3000, 40_000, 0), (500, 300_000, 1), (40, 4_000_000, 0), (385, 2000, 0), (384, 2000, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_mixtures(binding, n, top, off, dtype):
    """Tensors of very different sizes: pieces that all warps of a thread block share, that one takes, that several thread blocks have."""
    sizes = _mixture(n, top, n + off)
    gen = torch.Generator(device="cuda").manual_seed(n)
    row = (torch.randn(sum(sizes) + off, generator=gen, device="cuda") * 0.01).to(DT[dtype])[off:]
    grads = list(row.split(sizes))
    opt = binding.GradNorm(sizes, DT[dtype])
    norms = torch.empty(n, device="cuda")
    info = opt.grad_norm(grads, max_norm=0.5, tensor_norms=norms)
    want = torch.stack([g.double().pow(2).sum().sqrt() for g in grads])
    assert ((norms.double() - want).abs() <= 2.0 ** -23 * want).all()
    total = row.double().pow(2).sum().sqrt().item()
    assert abs(info[1].item() - total) <= 2.0 ** -23 * total
    for _ in range(3):
        again = opt.grad_norm(grads, max_norm=0.5)
        assert torch.equal(again.view(torch.int32), info.view(torch.int32))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("off", [0, 1, 2])
@pytest.mark.parametrize("weight,grad,copy", [("f32", "bf16", "bf16"), ("bf16", "bf16", None), ("f32", "f32", None)])
def test_places_between_tensors_are_left_alone(binding, bits, off, weight, grad, copy):
    sizes = [1, 700, 256, 5, 1024, 3000]
    gaps = [3, 2, 8, 1, 16, 5]

    def spread(dtype, fill):
        buf = torch.full((off + sum(sizes) + sum(gaps) + 64,), fill, device="cuda", dtype=dtype)
        at, views = off, []
        mask = torch.ones_like(buf, dtype=torch.bool)
        for n, gap in zip(sizes, gaps):
            views.append(buf[at:at + n])
            mask[at:at + n] = False
            at += n + gap
        return buf, views, mask
    w, ws, w_mask = spread(DT[weight], 0.375)
    g, gs, _ = spread(DT[grad], float("nan"))
    for x in gs:
        x.copy_(torch.randn(x.numel(), device="cuda"))
    c, cs, c_mask = spread(DT[copy], 0.625) if copy else (None, None, None)
    opt = binding.AdamW(ws, grad_dtype=DT[grad], copies=cs, state_bits=bits, lr=0.1)
    used = torch.zeros(opt.n_blocks * 256, dtype=torch.bool, device="cuda")
    for i in range(len(sizes)):
        a = opt.moments_of(i)[0]
        start = (a.data_ptr() - opt.m.data_ptr()) // a.element_size()
        used[start:start + sizes[i]] = True
    sentinel = 77 if bits == 8 else 77.0
    opt.m.view(-1)[~used] = sentinel
    opt.v.view(-1)[~used] = sentinel
    info = opt.grad_norm(gs)                                  # the NaN between the gradients are not counted
    assert info[2:].view(torch.int64).item() == 0
    opt.step(gs, info)
    opt.step(gs)
    assert (w[w_mask] == 0.375).all() and all((x != 0.375).all() for x in ws)
    assert c is None or (c[c_mask] == 0.625).all()
    assert (opt.m.view(-1)[~used] == sentinel).all() and (opt.v.view(-1)[~used] == sentinel).all()
    assert opt.status() == (0, 0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n,top", [(2, 5000), (300, 3000), (30, 200_000)])
def test_calls_in_a_row_wait_for_one_another(binding, bits, n, top):
    """Each kernel may start before the one ahead of it has ended.  Gradients that change between the calls, norm, step and values one
    after the other without a pause give the bits of the same calls with a wait after each."""
    sizes = _mixture(n, top, n)

    def loop(wait):
        gen = torch.Generator(device="cuda").manual_seed(5)
        row = torch.randn(sum(sizes), generator=gen, device="cuda")
        base = torch.randn(sum(sizes), generator=gen, device="cuda") * 1e-3
        grad = torch.empty_like(base)
        opt = binding.AdamW(list(row.split(sizes)), state_bits=bits, seed=4)
        bound, info = opt.bind_grads(list(grad.split(sizes))), torch.zeros(4, device="cuda")
        norms = torch.empty(n, device="cuda")
        kept = torch.zeros((), dtype=torch.float64, device="cuda")
        sync = torch.cuda.synchronize if wait else (lambda: None)
        for t in range(60):
            torch.mul(base, 1.0 + 0.1 * t, out=grad)
            sync()
            opt.grad_norm(bound, info, max_norm=0.5, tensor_norms=norms)
            sync()
            opt.step(bound, info)
            sync()
            if bits == 8:
                m, v = opt.state_values()
                sync()
                kept += m.double().abs().sum() + norms.double().sum()
            opt.step(bound, info)
            sync()
            opt.grad_norm(bound, info)
            sync()
            kept += info[1].double()
        return row, opt.m.clone(), opt.v.clone(), kept
    a, b = loop(True), loop(False)
    assert all(torch.equal(x, y) for x, y in zip(a[:3], b[:3])) and abs(a[3].item() / b[3].item() - 1) < 1e-12


@pytest.mark.gpu
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("bits", [32, 8])
def test_weights_that_are_not_finite_change_no_others(binding, bits, off):
    """An infinite weight times its decay, taken from itself, is no number by the formula; stochastic rounding must not make one of it."""
    for dtype in (torch.float32, torch.bfloat16):
        w = torch.randn(2000 + off, device="cuda").to(dtype)[off:]
        bad = [0, 255, 256, 700, 1999]
        w[bad] = torch.tensor([float("nan"), float("inf"), -float("inf"), float("nan"), float("inf")], device="cuda", dtype=dtype)
        opt = binding.AdamW([w], grad_dtype=torch.float32, state_bits=bits, weight_decay=0.1, lr=1e-3)
        for _ in range(3):
            opt.step([torch.randn(2000, device="cuda")])
        fine = torch.isfinite(w)
        assert not fine[bad].any() and int(fine.sum()) == 1995 and opt.status() == (0, 0, 0)


@pytest.mark.gpu
def test_against_torch_s_optimizer_in_64_bits(binding):
    """torch.optim.AdamW on 64-bit copies of the same weights and gradients, 20 steps with two decays."""
    gen = torch.Generator().manual_seed(11)
    sizes = [3000, 17, 512]
    p = make(sizes, torch.float32, gen)
    q = [x.double().clone().requires_grad_() for x in p]
    theirs = torch.optim.AdamW([{"params": q[:2], "weight_decay": 0.1}, {"params": q[2:], "weight_decay": 0.0}], lr=1e-2, betas=(0.9, 0.99))
    ours = binding.AdamW(p, lr=1e-2, betas=(0.9, 0.99), weight_decay=[0.1, 0.1, 0.0])
    for t in range(1, 21):
        g = make(sizes, torch.float32, gen)
        for x, y in zip(q, g):
            x.grad = y.double()
        theirs.step()
        ours.step(g)
        for x, y in zip(p, q):
            # one step's bound (updates below 10 lr) for each step so far
            assert (x.double() - y.detach()).abs().max() <= t * (2.0 ** -23 * y.detach().abs().max() + 2.0 ** -19 * 0.1)


@pytest.mark.gpu
def test_training_loop_learns_with_either_kind_of_moments(binding):
    from paper_2203_09044_b200 import train_step
    l32 = train_step.run(iterations=80, n_users=3, d=60_000, state_bits=32)
    l8 = train_step.run(iterations=80, n_users=3, d=60_000, state_bits=8)
    assert l32[0] == l8[0] and l32[-1] < 0.2 * l32[0] and l8[-1] < 0.2 * l8[0]


@pytest.mark.gpu
@pytest.mark.parametrize("off", [0, 1])
def test_every_code_is_read_by_the_formula(binding, off):
    """Moments of 8 bits that no step of this library has made: all 256 codes in each block, with exponents from the least to the
    largest, values and a step on from them."""
    n, seed = 256 * 12, 5
    tops_m = np.array([17, 18, 100, 120, 127, 139, 140, 141, 150, 17, 30, 113], np.uint8)
    tops_v = np.array([33, 34, 90, 120, 127, 155, 156, 157, 170, 33, 40, 100], np.uint8)
    rng = np.random.default_rng(1)
    code_m = np.stack([rng.permutation(256) for _ in range(12)]).astype(np.uint8)
    code_v = np.stack([rng.permutation(256) for _ in range(12)]).astype(np.uint8)
    state = dict(m=torch.from_numpy(code_m).cuda(), v=torch.from_numpy(code_v).cuda(), m_exp=torch.from_numpy(tops_m).cuda(), v_exp=torch.from_numpy(tops_v).cuda())
    gen = torch.Generator().manual_seed(3)
    p, g = make([n], torch.float32, gen, off), make([n], torch.float32, gen, off)
    opt = binding.AdamW(p, state_bits=8, seed=seed, state=state, weight_decay=0.0, lr=0.0)
    ref = Reference(as_f32(p), np.zeros(1), 8, 0.0, (0.9, 0.999), 1e-8, seed, False)
    ref.mc, ref.mt, ref.vc, ref.vt = code_m.copy(), tops_m.copy(), code_v.copy(), tops_v.copy()
    m, v = (x.double().cpu().numpy() for x in opt.state_values(*(torch.empty((12, 256), device="cuda") for _ in range(2))))
    assert np.array_equal(m, decode_ref(code_m, tops_m, M_FIELD, True)) and np.array_equal(v, decode_ref(code_v, tops_v, V_FIELD, False))
    opt.step(g)
    ref.step(as_f32(g))
    assert ref.kept == 0 and opt.status() == (0, 0, 0)
    for got, want in ((opt.m_exp, ref.mt), (opt.v_exp, ref.vt), (opt.m, ref.mc), (opt.v, ref.vc)):
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_negative_zeros_leave_fresh_moments_at_zero(binding, bits):
    """In whole blocks and in a part of one the same bits: a sum of +0 and -0 is +0."""
    p, g = torch.randn(600, device="cuda"), torch.full((600,), -0.0, device="cuda")
    before = p.clone()
    opt = binding.AdamW([p], state_bits=bits, weight_decay=0.0)
    for _ in range(2):
        opt.step([g])
    assert not opt.m.view(torch.int32 if bits == 32 else torch.uint8).any() and not opt.v.view(torch.int32 if bits == 32 else torch.uint8).any()
    assert torch.equal(p, before)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_on_a_side_stream_sees_steps_that_were_just_set(binding, bits):
    """set_steps and status(clear=True), each followed at once by a step on a stream that does not wait for the null stream."""
    gen = torch.Generator().manual_seed(12)
    w, g = make([3000], torch.bfloat16, gen), make([3000], torch.bfloat16, gen)
    side, out = torch.cuda.Stream(), []
    for wait in (True, False):
        p = [w[0].clone()]
        opt = binding.AdamW(p, state_bits=bits, seed=6)
        bound = opt.bind_grads(g)
        torch.cuda.synchronize()
        for t in (0, 10, 1000, 50_000):
            opt.set_steps(t)
            if wait:
                torch.cuda.synchronize()
            opt.step(bound, stream=side)
            assert opt.status(clear=True) == (0, 0, 0)
            if wait:
                torch.cuda.synchronize()
            opt.step(bound, stream=side)
            assert opt.steps() == t + 2
        out.append((p[0], opt.m, opt.v))
    assert all(torch.equal(x, y) for x, y in zip(*out))


@pytest.mark.gpu
def test_outputs_for_another_stream_take_no_memory_that_is_still_in_use(binding):
    """Tensors of the size of the outputs are given back while work that reads them still waits on the current stream."""
    opt = binding.AdamW([torch.ones(1 << 20, device="cuda")], state_bits=8)
    g = opt.bind_grads([torch.ones(1 << 20, device="cuda")])
    opt.step(g)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    used = [torch.full((opt.n_blocks, 256), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)] + [torch.full((4,), 3.0, device="cuda")]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)                       # about 10 ms
    copies = [x.clone() for x in used]
    used.clear()
    info = opt.grad_norm(g, stream=side)
    m, v = opt.state_values(stream=side)
    torch.cuda.synchronize()
    assert all((x == 3.0).all() for x in copies)
    assert info[1].item() == 1024.0 and (m > 0.09).all() and (v > 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_weights_that_are_given_other_storage(binding, bits):
    """`p.data = x` between two steps: the second one updates x, and the old storage is left alone."""
    p = [torch.nn.Parameter(torch.ones(700, device="cuda")), torch.nn.Parameter(torch.ones(9, device="cuda"))]
    g = [torch.full((700,), 0.5, device="cuda"), torch.full((9,), -0.5, device="cuda")]
    opt = binding.AdamW(p, lr=0.1, weight_decay=0.0, state_bits=bits)
    bound = opt.bind_grads(g)
    opt.step(bound)
    old, kept, m = p[0].detach(), p[0].detach().clone(), opt.m
    p[0].data = torch.full((700,), 5.0, device="cuda")
    opt.m = m.clone()
    before = m.clone()
    opt.step(bound)
    assert torch.equal(old, kept) and torch.equal(m, before) and not torch.equal(opt.m, before)
    # gradients that do not change: an update of lr, but for the rounding of 8-bit moments (a first moment's by an eighth, a root's by 15 %)
    for x, want in ((p[0], 4.9), (p[1], 1.2)):
        assert ((x.detach() - want).abs() < (0.05 if bits == 8 else 1e-5)).all()


# ---- sets large enough that each warp takes several blocks ----------------------------------------------------------------------
# A thread block has 8 warps and one block of 256 for each at least; what comes after it (the loads one block ahead, the two stages in
# turn, a tensor's border inside a thread block's blocks, their exponents) needs more: 2 to 16 blocks a warp here, fewer in the least.
LARGE = {
    "1.6M": [700_000, 255, 700, 130_007, 2048, 1, 513, 377_781, 4096, 65_537, 0, 300_000, 7, 3000, 20_003],
    "7.6M": [2_700_000, 255, 700, 430_007, 2048, 1, 513, 1_377_781, 4096, 65_537, 0, 1_900_000, 7, 3000, 1_120_003],
    "19.2M": [6_000_000, 255, 700, 1_300_007, 2048, 1, 513, 3_777_781, 4096, 65_537, 0, 4_500_000, 7, 3000, 3_500_003],
}


class LargeReference:
    """The formula on the device, elementary operations only: the moments' products and sums one by one in 32 bits, all else in 64."""

    def __init__(self, sizes, bits, betas, eps, seed):
        self.sizes, self.bits, self.betas, self.eps, self.seed, self.t = sizes, bits, betas, eps, seed, 0
        nb = [(n + 255) // 256 for n in sizes]
        self.owner = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor(nb, device="cuda"))
        begin = np.concatenate([[0], np.cumsum(nb)])[:-1] * 256
        self.at = [slice(int(b), int(b) + n) for b, n in zip(begin, sizes)]
        self.m, self.v = (torch.zeros(sum(nb), 256, device="cuda") for _ in range(2))
        self.codes = None

    def blocks(self, tensors):
        out = torch.zeros(self.m.numel(), device="cuda")
        for at, x in zip(self.at, tensors):
            out[at] = x.float()
        return out.view(-1, 256)

    @staticmethod
    def value(code, top, field, signed):
        c = code.long()
        mag = c & 127 if signed else c
        e = mag >> 3
        n = torch.where(e > 0, 8 + (mag & 7), mag & 7).double()
        x = n * torch.exp2((e.clamp(min=1) - 1 + top.long()[:, None] - 127 - field - 2).double())
        return torch.where(c > 127, -x, x) if signed else x

    @staticmethod
    def code(x, rand, field, signed):
        a = x.abs().double()
        top = (x.abs().amax(1).view(torch.int32) >> 23).clamp(min=field + 3).long()
        least = (top - 127 - field + 1)[:, None]
        octave = torch.maximum(torch.frexp(torch.where(a > 0, a, 1e-300))[1].long() - 1, least)
        steps = (a * torch.exp2((23 - octave).double())).round().long()
        code = (octave - least) * 8 + ((steps + rand) >> 20)
        code = torch.where(x < 0, code + 128, code) if signed else torch.maximum(code, (x > 0).long())
        return code.to(torch.uint8), top.to(torch.uint8)

    def step(self, weights, grads, factor, lr, decay):
        """New weights in 64 bits, their tolerance, the random bits; blocks each."""
        self.t += 1
        b1, b2 = self.betas
        if self.bits == 8 and self.codes is not None:
            self.m, self.v = (self.value(c, t, f, s).float() for c, t, f, s in ((*self.codes[:2], M_FIELD, True), (*self.codes[2:], V_FIELD, False)))
        g = self.blocks(grads) * torch.tensor(factor, device="cuda")
        self.m = self.m * float(f32(b1)) + g * float(f32(1.0 - b1))
        self.v = self.v * float(f32(b2)) + (g * g) * float(f32(1.0 - b2))
        w, d = self.blocks(weights).double(), lr * torch.tensor(decay, device="cuda", dtype=torch.float64)[self.owner][:, None]
        upd = lr * (self.m.double() / (1 - b1 ** self.t)) / (torch.sqrt(self.v.double() / (1 - b2 ** self.t)) + self.eps)
        new = w - (d * w + upd)
        tol = 2.0 ** -23 * new.abs() + 2.0 ** -20 * (upd.abs() + (d * w).abs()) + 1e-44
        p = torch.arange(self.m.numel(), device="cuda").view(-1, 256)
        s = (mix32((mix32(self.seed) + self.t) & 0xFFFFFFFF) + p * 0x9E3779B9) & 0xFFFFFFFF
        rand = ((s ^ (s >> 15)) * 0x2C1B3C6D) & 0xFFFFFFFF
        if self.bits == 8:
            self.codes = (*self.code(self.m, rand & 0xFFFFF, M_FIELD, True), *self.code(self.v, rand >> 12, V_FIELD, False))
        return new, tol, rand


def spread(sizes, dtype, gen, apart, scale):
    """Tensors each at a multiple of 256 elements, or back to back from an odd one."""
    at, out = 0 if apart else 1, []
    buf = torch.randn(sum(n + 255 for n in sizes) + 64, generator=gen, device="cuda").mul_(scale).to(dtype)
    for n in sizes:
        out.append(buf[at:at + n])
        at += (n + 255) // 256 * 256 if apart else n
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("apart", [True, False])
@pytest.mark.parametrize("weight,grad,copy", [("f32", "f32", None), ("bf16", "bf16", None), ("f32", "bf16", "bf16"), ("f32", "f16", "f16"), ("bf16", "f32", None)])
@pytest.mark.parametrize("name", list(LARGE))
def test_step_over_large_sets(binding, name, weight, grad, copy, apart, bits):
    sizes, lr, seed = LARGE[name], 1e-2, 21
    gen = torch.Generator(device="cuda").manual_seed(len(name) + bits)
    params = spread(sizes, DT[weight], gen, apart, 0.05)
    copies = None if copy is None else spread(sizes, DT[copy], gen, apart, 1.0)
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    opt = binding.AdamW(params, grad_dtype=DT[grad], copies=copies, lr=lr, weight_decay=decay, state_bits=bits, seed=seed)
    ref = LargeReference(sizes, bits, (0.9, 0.999), 1e-8, seed)
    inside = ref.blocks([torch.ones(n, device="cuda") for n in sizes]) > 0
    info = torch.tensor([0.5, 0, 0, 0], device="cuda")
    for t in range(3):
        grads = spread(sizes, DT[grad], gen, apart, 10.0 ** -t)
        before = [p.clone() for p in params]
        opt.step(grads, info)
        new, tol, rand = ref.step(before, grads, 0.5, lr, np.array(decay, f32).astype(np.float64))
        if bits == 8:
            for got, want, what in zip((opt.m, opt.m_exp, opt.v, opt.v_exp), ref.codes, ("m", "m_exp", "v", "v_exp")):
                assert torch.equal(got, want), f"t={t} {what}"
        else:
            assert torch.equal(opt.m.view(torch.int32), ref.m.view(torch.int32)) and torch.equal(opt.v.view(torch.int32), ref.v.view(torch.int32)), f"t={t}"
        got = ref.blocks(params)
        if weight == "bf16":                              # as in run_steps
            r = (rand >> 10 & 0xFFFF).int()
            a, b = (((x.float().view(torch.int32) + r) & -65536).view(torch.float32) for x in (new - tol, new + tol))
            ok = (got >= torch.minimum(a, b)) & (got <= torch.maximum(a, b))
        else:
            ok = (got.double() - new).abs() <= tol
        assert (ok | ~inside).all(), f"t={t} weights"
        if copies is not None:
            assert all(torch.equal(c, p.to(DT[copy])) for c, p in zip(copies, params)), f"t={t} copies"
    assert opt.status() == (0, 0, 0) and opt.steps() == 3


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [5, 256, 261])
@pytest.mark.parametrize("factor", [float("inf"), float("nan")])
def test_elements_left_out_are_counted_within_the_tensors(binding, bits, n, factor):
    """A factor that is not finite leaves every element out, and no place past a tensor's end counts (0 times infinity is no number)."""
    p, g = torch.ones(n, device="cuda"), torch.full((n,), 0.5, device="cuda")
    opt = binding.AdamW([p], state_bits=bits)
    opt.step([g], torch.tensor([factor, 0, 0, 0], device="cuda"))
    assert opt.status() == (binding.FLAG_NONFINITE, n, 0)
    assert (p == 1).all() and not opt.m.any() and not opt.v.any()


@pytest.mark.gpu
def test_elements_left_out_of_a_step_share_their_block_s_exponents(binding):
    """8-bit moments of an element that a step leaves out: the same values where its block's largest did not grow, and where it did, one
    of the two neighbours on the coarser grid."""
    n, bad = 512, [3, 300]
    p, g = torch.ones(n, device="cuda"), torch.linspace(0.5, 1.0, n, device="cuda")
    opt = binding.AdamW([p], state_bits=8, lr=0.1)
    opt.step([g])
    w, (m, v) = p.clone(), opt.state_values()
    quiet = torch.zeros(n, device="cuda")
    quiet[bad] = float("inf")
    opt.step([quiet])
    m1, v1 = opt.state_values()
    for x, y in ((w, p), (m.view(-1), m1.view(-1)), (v.view(-1), v1.view(-1))):
        assert torch.equal(x[bad], y[bad])
    assert not torch.equal(m, m1)
    loud = quiet.clone()
    loud[[100, 400]] = 3e4
    opt.step([loud])
    m2, v2 = opt.state_values()
    assert torch.equal(w[bad], p[bad])
    # first moments of 0.05 to 0.1 beside one of 3000: the top is 2^11, the smallest steps 2^(11-16); second ones of 3e-4 to 1e-3 beside
    # 9e5: the top is 2^19, the smallest steps 2^(19-32), and none goes to zero
    for x, y, step in ((m1, m2, 2.0 ** -5), (v1, v2, 2.0 ** -13)):
        x, y = x.view(-1)[bad].double(), y.view(-1)[bad].double()
        assert ((x - y).abs() <= step).all() and (y % step == 0).all()
    assert m1.view(-1)[3] != m2.view(-1)[3] and (v2.view(-1)[bad] > 0).all()
    assert opt.status()[1] == 4


@pytest.mark.gpu
def test_an_infinite_bound_clips_nothing(binding):
    g = [torch.full((100,), 3.0, device="cuda")]
    info = binding.GradNorm([100]).grad_norm(g, max_norm=float("inf"), grad_scale=0.5)
    assert info[:2].tolist() == [0.5, 15.0]
    for bad in (float("nan"), -float("nan")):
        with pytest.raises(binding.Co3Error):
            binding.GradNorm([100]).grad_norm(g, max_norm=bad)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,whole", [("bf16", 8), ("f16", 8), ("f32", 8)])
def test_norm_at_other_addresses(binding, dtype, whole):
    """The same bits at addresses alike to the header's rule.  At others: pairs of squares with one rounding of 2^-24 each, which the
    root halves, and the norm's own rounding of 2^-24, on either side: 3 * 2^-24 between them."""
    sizes = [256, 700, 2048, 5000] * 80
    gen = torch.Generator(device="cuda").manual_seed(17)
    data = [torch.randn(n, generator=gen, device="cuda").to(DT[dtype]) for n in sizes]
    opt = binding.GradNorm(sizes, DT[dtype])

    def norms(places):                                    # of each tensor in turn, in elements past a multiple of `whole`
        buf = torch.zeros(sum(n + 4 * whole for n in sizes), dtype=DT[dtype], device="cuda")
        at, grads = 0, []
        for i, x in enumerate(data):
            at = -(-at // whole) * whole + places[i % len(places)]
            grads.append(buf[at:at + x.numel()])
            grads[-1].copy_(x)
            at += x.numel()
        out = torch.empty(len(sizes), device="cuda")
        info = opt.grad_norm(grads, max_norm=1.0, tensor_norms=out)
        return torch.cat([out, info[:2]])
    on, off = norms([0]), norms([1])
    assert torch.equal(norms([whole, 0, 2 * whole]), on) and torch.equal(norms([3, 5, whole + 1, 2]), off)
    assert ((on.double() - off.double()).abs() <= 3 * 2.0 ** -24 * on.double()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [63, 64, 65, 159, 160, 161])
def test_pointers_with_the_launch_and_by_way_of_the_table(binding, bits, n):
    run_steps(binding, [1 + 37 * i % 300 for i in range(n)], bits, factor=0.5, steps=2)
