"""The operators at a language model's two ends: embedding and its gradient, layer norm, losses over a vocabulary without the logits.

The reference is the formula in 64 bits.  Tolerances count roundings: half a step is u(type) = finfo.eps / 2 of the value; a sum of n
numbers in 32 bits, in whatever order, is off by at most n 2^-24 of the sum of their magnitudes; the tensor cores cut off what lies
below the last place of a 32-bit sum at each 16 of depth, 2^-23 of the sum of the magnitudes so far, and sums over more than 1024 are
added in 32 bits.  No input was chosen by its outcome."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2203_09044_b200 import binding as b                                     # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U32 = 2.0 ** -24
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def u(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half a step among the smallest numbers."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def within(got, want, bound, dtype=F32):
    """|got - want| <= bound and the rounding of the output, everywhere; NaN where the reference has it."""
    got, want = got.double(), want.double()
    assert torch.equal(got.isnan(), want.isnan())
    off = (got - want).abs().nan_to_num(0.0)
    room = bound + u(dtype) * (want.abs() + bound) + tiny(dtype)
    worst = (off - room).nan_to_num(0.0).max() if off.numel() else torch.zeros(())
    assert worst <= 0, f"off by {off.flatten()[(off - room).argmax()].item():.3g}, {room.flatten()[(off - room).argmax()].item() if room.dim() else room:.3g} allowed"


def strided(g, users, tokens, dim, dtype, how):
    """[users][tokens][dim] of random numbers: dense, with gaps at aligned places, or beginning at odd elements with gaps; a
    user outermost or a token."""
    if how == "dense":
        return normal(g, users, tokens, dim, dtype=dtype)
    if how == "gaps":
        return normal(g, users, tokens + 1, (dim + 15) // 8 * 8, dtype=dtype)[:, :tokens, :dim]
    if how == "odd":
        return normal(g, users, tokens, dim + 3, dtype=dtype)[:, :, 1:dim + 1]
    return normal(g, tokens, users, dim, dtype=dtype).transpose(0, 1)                # "tokens first"


def rows_for(users, n, at, dtype, fill=7.0):
    """Gradient rows, the part of n elements that begins at element `at`, and a check that the rest stayed as it was."""
    rows = torch.full((users, (at + n + 9) // 4 * 4), fill, dtype=dtype, device="cuda")
    return rows, rows[:, at:at + n], lambda: bool((rows[:, :at] == fill).all() and (rows[:, at + n:] == fill).all())


# ---- embedding ----------------------------------------------------------------------------------------------------------------
def some_tokens(g, users, tokens, vocab, kind=torch.int64, none=0.2, skew=1.0):
    x = (torch.rand((users, tokens), generator=g, device="cuda").double() ** skew * vocab).long().clamp(max=vocab - 1)
    return torch.where(torch.rand((users, tokens), generator=g, device="cuda") < none, -1 - x, x).to(kind)


@pytest.mark.parametrize("table_type,out_type", [(F32, F32), (F32, BF16), (BF16, BF16), (F16, F32), (BF16, F16), (F16, F16)])
@pytest.mark.parametrize("dim,how", [(1, "dense"), (7, "dense"), (8, "odd"), (64, "tokens first"), (1000, "gaps"), (1024, "dense"), (2056, "odd"), (2056, "dense")])
def test_lookup(table_type, out_type, dim, how):
    g = gen(dim)
    users, tokens, vocab = 3, 37, 501
    e = b.Embedding(vocab, dim, n_users=users, tokens=40)
    table = normal(g, vocab, dim, dtype=table_type)
    k = some_tokens(g, users, tokens, vocab, torch.int32 if dim % 2 else torch.int64)
    out = strided(g, users, tokens, dim, out_type, how)
    around = out._base.clone() if out._is_view() else None
    e.forward(k, table, scale=1.7, out=out)
    want = (table.float()[k.clamp(min=0).long()] * torch.tensor(1.7)).to(out_type)     # one product in 32 bits, one rounding
    want = torch.where((k < 0)[..., None], torch.zeros((), dtype=out_type, device="cuda"), want)
    assert torch.equal(out, want)
    if around is not None:
        out.copy_(torch.zeros_like(out))
        base, copy = out._base.clone(), around.as_strided(out.size(), out.stride(), out.storage_offset())
        copy.zero_()
        assert torch.equal(base, around)
    assert e.status() == (0, 0)


def test_lookup_of_tokens_that_the_vocabulary_does_not_have():
    e = b.Embedding(10, 16, tokens=4)
    table = torch.ones((10, 16), device="cuda")
    k = torch.tensor([9, 10, 2 ** 40, -(2 ** 40)], device="cuda")
    out = e.forward(k, table, scale=3.0)
    assert out.sum(1).tolist() == [48.0, 0.0, 0.0, 0.0]
    assert e.status(clear=True) == (b.FLAG_TOKEN, 2) and e.status() == (0, 0)
    d = torch.full((10, 16), 5.0, device="cuda")
    e.backward(torch.full((4, 16), NAN, device="cuda").index_fill_(0, torch.tensor([0], device="cuda"), 2.0), k, d)
    want = torch.zeros((10, 16), device="cuda")
    want[9] = 2.0
    assert torch.equal(d, want) and e.status() == (b.FLAG_TOKEN, 2)


def embed_reference(dout, k, vocab, scale):
    """The table's gradient in 64 bits, sum of magnitudes, and the number of terms."""
    users, tokens, dim = dout.shape
    out = torch.zeros((users, vocab, dim), dtype=torch.float64, device="cuda")
    mag, n = torch.zeros_like(out), torch.zeros((users, vocab, 1), dtype=torch.float64, device="cuda")
    for i in range(users):
        here = (k[i] >= 0).nonzero().view(-1)
        at = k[i][here].long()
        x = dout[i][here].double() * scale
        out[i].index_put_((at,), x, accumulate=True)
        mag[i].index_put_((at,), x.abs(), accumulate=True)
        n[i].index_put_((at,), torch.ones_like(at, dtype=torch.float64)[:, None], accumulate=True)
    return out, mag, n


@pytest.mark.parametrize("tokens", [1, 31, 32, 33, 257, 4096, 4097, 20001])
@pytest.mark.parametrize("vocab,dim,skew", [(1, 8, 1.0), (2, 5, 1.0), (255, 40, 3.0), (256, 264, 1.0), (257, 8, 6.0), (70000, 16, 2.0)])
def test_embedding_gradient(tokens, vocab, dim, skew):
    g = gen(tokens * 7 + vocab)
    users = 2 if tokens < 20000 else 1
    act, kind = [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16)][(tokens + vocab) % 4]
    at = [0, 1, 8][(tokens + dim) % 3]
    e = b.Embedding(vocab, dim, n_users=users, tokens=tokens + 5)
    k = some_tokens(g, users, tokens, vocab, torch.int32 if tokens % 2 else torch.int64, skew=skew)
    dout = strided(g, users, tokens, dim, act, ["dense", "odd", "gaps", "tokens first"][(tokens + vocab + dim) % 4])
    dout.masked_fill_((k < 0)[..., None], NAN)              # what lies in places without a token
    want, mag, n = embed_reference(dout, k, vocab, 0.3)
    rows, part, untouched = rows_for(users, vocab * dim, at, kind)
    e.backward(dout, k, part, scale=0.3)
    # n terms, the product with the scale, and that scale itself
    within(part.view(users, vocab, dim), want, (n + 2) * U32 * mag, kind)
    assert untouched() and e.status() == (0, 0)
    first = part.clone()
    e.backward(dout, k, part, scale=0.3)
    assert torch.equal(first, part), "the same inputs give the same bits"
    e.backward(dout, k, part, scale=0.3, accumulate=True)
    within(part.view(users, vocab, dim), first.view(users, vocab, dim).double() + want, (n + 2) * U32 * mag + U32 * (first.view(users, vocab, dim).double().abs() + mag), kind)
    assert untouched()


@pytest.mark.parametrize("tokens", [40, 5000, 70000])
def test_embedding_gradient_of_one_token_alone(tokens):
    """A run over all places: sums by chunk, joined."""
    e = b.Embedding(5, 24, tokens=tokens)
    g = gen(1)
    dout = normal(g, tokens, 24)
    d = torch.empty((5, 24), device="cuda")
    e.backward(dout, torch.full((tokens,), 3, device="cuda"), d)
    within(d[3], dout.double().sum(0), tokens * U32 * dout.double().abs().sum(0))
    assert not d[[0, 1, 2, 4]].any()


def test_embedding_of_no_tokens():
    e = b.Embedding(6, 8, n_users=2, tokens=4)
    k = torch.empty((2, 0), dtype=torch.int64, device="cuda")
    assert e.forward(k, torch.ones((6, 8), device="cuda")).shape == (2, 0, 8)
    d = torch.ones((2, 48), device="cuda")
    e.backward(torch.empty((2, 0, 8), device="cuda"), k, d, accumulate=True)
    assert bool((d == 1).all())
    e.backward(torch.empty((2, 0, 8), device="cuda"), k, d)
    assert not d.any()
    k = torch.full((2, 3), -1, device="cuda")
    d.fill_(2.0)
    e.backward(torch.full((2, 3, 8), NAN, device="cuda"), k, d)
    assert not d.any()


def test_embedding_whose_table_passes_32_bits():
    vocab, dim = 70_001, 65_536                           # 4.6e9 elements
    e = b.Embedding(vocab, dim, tokens=3)
    table = torch.zeros((vocab, dim), dtype=BF16, device="cuda")
    table[vocab - 1] = 3.0
    k = torch.tensor([vocab - 1, 5, vocab - 2], device="cuda")
    out = e.forward(k, table)
    assert bool((out[0] == 3).all()) and not out[1:].any()
    table.fill_(1.0)
    e.backward(torch.ones((3, dim), device="cuda"), k, table, scale=2.0)
    assert bool((table[vocab - 1] == 2).all()) and bool((table[vocab - 2] == 2).all()) and bool((table[5] == 2).all())
    table[[5, vocab - 2, vocab - 1]] = 0.0
    assert not any(bool(part.any()) for part in table.split(10_000))


@pytest.mark.parametrize("dim,at,act,kind", [(1024, 0, BF16, BF16), (1024, 4, F32, F32), (1032, 8, F16, F32), (1032, 1, BF16, F32), (1028, 0, F32, BF16), (1028, 3, F16, F16), (1026, 0, BF16, BF16)])
@pytest.mark.parametrize("users,skew", [(1, 1.0), (2, 4.0)])
def test_embedding_gradient_of_many_wide_rows(dim, at, act, kind, users, skew):
    """Eight, four and two columns a lane: the wider ones are taken from 2368 parts of 32 tokens and 256 (128) columns on, of a device of 148 SMs."""
    g = gen(dim + at)
    tokens, vocab = 20001 // users, 3001
    e = b.Embedding(vocab, dim, n_users=users, tokens=tokens)
    k = some_tokens(g, users, tokens, vocab, skew=skew)
    dout = normal(g, users, tokens, dim, dtype=act)
    dout.masked_fill_((k < 0)[..., None], NAN)
    want, mag, n = embed_reference(dout, k, vocab, 0.3)
    rows, part, untouched = rows_for(users, vocab * dim, at, kind)
    got = part.view(users, vocab, dim) if users == 1 else part.unflatten(1, (vocab, dim))
    e.backward(dout, k, part, scale=0.3)
    within(got, want, (n + 2) * U32 * mag, kind)
    first = part.clone()
    e.backward(dout, k, part, scale=0.3, accumulate=True)
    old = first.unflatten(1, (vocab, dim)).double()
    within(got, old + want, (n + 2) * U32 * mag + U32 * (old.abs() + mag), kind)
    assert untouched() and e.status() == (0, 0)


@pytest.mark.parametrize("tokens,vocab,skew", [(70_001, 100_003, 3.0), (131_077, 700, 1.0), (200_000, 600_011, 2.0)])
def test_embedding_gradient_of_long_batches(tokens, vocab, skew):
    """Above 65536 tokens a warp of the sort has more keys than it holds and ranks them twice; two and three passes."""
    g = gen(tokens)
    e = b.Embedding(vocab, 8, tokens=tokens)
    k = some_tokens(g, 1, tokens, vocab, skew=skew)
    dout = normal(g, 1, tokens, 8)
    want, mag, n = embed_reference(dout, k, vocab, 1.5)
    d = torch.full((1, vocab, 8), NAN, device="cuda")
    e.backward(dout, k, d, scale=1.5)
    within(d, want, (n + 2) * U32 * mag)


@pytest.mark.parametrize("tokens", [3, 300, 4098, 12_000, 70_002, 150_000])
def test_equal_tokens_are_added_in_their_order(tokens):
    """Each token stands three times: the sums, to the last bit, are those of the rows one after the other."""
    g = gen(tokens)
    vocab = tokens // 3
    e = b.Embedding(vocab, 6, tokens=tokens)
    k = torch.randperm(tokens, generator=g, device="cuda") // 3
    dout = normal(g, tokens, 6) * 10.0 ** torch.randint(-3, 4, (tokens, 1), generator=g, device="cuda")
    d = torch.empty((vocab, 6), device="cuda")
    e.backward(dout, k, d)
    x = dout[k.argsort(stable=True)].view(vocab, 3, 6)
    assert torch.equal(d, (x[:, 0] + x[:, 1]) + x[:, 2])


# ---- layer norm ---------------------------------------------------------------------------------------------------------------
DIMS = [1, 2, 7, 8, 64, 255, 256, 257, 512, 768, 1000, 1024, 1025, 2048, 3000, 4096, 5000, 8192, 8200, 16384]


def norm_reference(x, w, bias, eps):
    x = x.double()
    mean = x.mean(-1)
    var = ((x - mean[..., None]) ** 2).mean(-1)
    rstd = (var + eps) ** -0.5
    xhat = (x - mean[..., None]) * rstd[..., None]
    return mean, rstd, xhat, xhat * (1.0 if w is None else w.double()) + (0.0 if bias is None else bias.double())


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("dtype,how,weights", [(F32, "dense", F32), (BF16, "dense", F32), (F16, "odd", F16), (BF16, "gaps", None), (F32, "tokens first", BF16)])
def test_layer_norm(dim, dtype, how, weights):
    g = gen(dim)
    users, tokens = (3, 41) if dim < 5000 else (2, 5)
    n = b.LayerNorm(dim, n_users=users)
    x = strided(g, users, tokens, dim, dtype, how)
    x.mul_(torch.rand((users, tokens, 1), generator=g, device="cuda").to(dtype) * 3).add_(normal(g, users, tokens, 1, dtype=dtype))
    w = None if weights is None else (1 + 0.3 * normal(g, dim)).to(weights)
    bias = None if weights is None else normal(g, dim, dtype=weights)
    y, mean, rstd = n.forward(x, w, bias)
    m, r, xhat, want = norm_reference(x, w, bias, 1e-5)
    mag = x.double().abs().mean(-1)
    e_mean = (dim + 2) * U32 * mag                        # a sum, its quotient, whose divisor is rounded too
    within(mean, m, e_mean)
    # the differences are off by the mean's error and a rounding; their squares' sum and quotient by dim + 2 roundings; a root and a quotient more.
    # An error of d in every difference shifts the mean of squares by d^2 (the differences' own sum is 0 up to the same error).
    shift = e_mean + U32 * (m.abs() + mag)
    e_var = 2 * shift * (shift + (r ** -2).sqrt() * 2 * U32) + (dim + 6) * U32 * r ** -2
    e_r = 0.5 * r ** 3 * e_var + 4 * U32 * r
    within(rstd, r, e_r)
    gain = 1.0 if w is None else w.double().abs()
    e_x = (x.double() - m[..., None]).abs()
    bound = gain * (r[..., None] * (shift + U32 * e_x.amax(-1))[..., None] + (e_r + 2 * U32 * r)[..., None] * e_x) + 2 * U32 * (want.abs() + (0.0 if bias is None else bias.double().abs()))
    within(y, want, bound, dtype)


@pytest.mark.parametrize("dim", [64, 1000, 4096])
def test_layer_norm_far_from_zero(dim):
    """A mean 10^4 times the deviation: the variance is that of differences (the difference of squares would have no digit left)."""
    g = gen(3)
    x = 1e4 + normal(g, 9, dim)
    y, mean, rstd = b.LayerNorm(dim).forward(x)
    m, r, _, want = norm_reference(x, None, None, 1e-5)
    # the mean of numbers near 1e4 in 32 bits is off by at most (dim + 2) 2^-24 of it, in any order; in sums of 32 or fewer terms a thread joined
    # by tree, and the variance by the square of that
    off = (dim + 2) * U32 * 1e4 * 1.01
    assert (mean.double() - m).abs().max() <= off
    assert ((rstd.double() / r) - 1).abs().max() <= off ** 2 + 2 * off * 1e-3 + (dim + 8) * U32
    assert (y.double() - want).abs().max() <= 2 * off + 5 * (off ** 2 + 2 * off * 1e-3 + (dim + 8) * U32)


def test_layer_norm_of_equal_elements_and_in_place():
    n = b.LayerNorm(48)
    x = torch.full((2, 48), 2.5, device="cuda")
    w, bias = torch.full((48,), 3.0, device="cuda"), torch.arange(48.0, device="cuda")
    y, mean, rstd = n.forward(x, w, bias, y=x)
    assert y is x and torch.equal(x, bias.expand(2, 48)) and mean.tolist() == [2.5, 2.5]
    assert (rstd.double() / 1e-5 ** -0.5 - 1).abs().max() <= 4 * U32


def grad_reference(dy, x, w, mean, rstd):
    dy, x, r = dy.double(), x.double(), rstd.double()[..., None]
    xhat = (x - mean.double()[..., None]) * r
    gain = dy * (1.0 if w is None else w.double())
    c1, c2 = gain.mean(-1, keepdim=True), (gain * xhat).mean(-1, keepdim=True)
    return xhat, gain, c1, c2, r * (gain - c1 - xhat * c2)


def test_the_gradient_formula_of_layer_norm_against_differences():
    g = gen(11)
    x, w, bias, dy = (normal(g, *s, dtype=torch.float64) for s in ((3, 17), (17,), (17,), (3, 17)))

    def value(x, w, bias):
        return (norm_reference(x, w, bias, 1e-5)[3] * dy).sum()

    mean, rstd, xhat, _ = norm_reference(x, w, bias, 1e-5)
    dx = grad_reference(dy, x, w, mean, rstd)[4]
    h = 1e-6                                              # central differences: h^2 and 1e-16 / h
    for t, grad in ((x, dx), (w, (dy * xhat).sum(0)), (bias, dy.sum(0))):
        for i in range(0, t.numel(), 5):
            step = torch.zeros_like(t).view(-1)
            step[i] = h
            step = step.view(t.shape)
            args = [(x, w, bias), (x, w, bias)]
            args = [tuple(a + s * step if a is t else a for a in (x, w, bias)) for s in (1, -1)]
            assert abs((value(*args[0]) - value(*args[1])).item() / (2 * h) - grad.view(-1)[i].item()) < 1e-7


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("dtype,how,weights,kind,at", [(F32, "dense", F32, F32, 0), (BF16, "dense", F32, F32, 3), (F16, "odd", F16, F16, 1), (BF16, "gaps", None, BF16, 0),
                                                       (F32, "tokens first", BF16, F32, 5)])
def test_layer_norm_gradient(dim, dtype, how, weights, kind, at):
    g = gen(dim + 1)
    users, tokens = (3, 43) if dim < 5000 else (2, 5)
    if dim in (64, 2048):
        users, tokens = 1, 1500                           # several thread blocks a user
    n = b.LayerNorm(dim, n_users=users)
    x, dy = strided(g, users, tokens, dim, dtype, how), strided(g, users, tokens, dim, dtype, how)
    w = None if weights is None else (1 + 0.3 * normal(g, dim)).to(weights)
    _, mean, rstd = n.forward(x, w)
    xhat, gain, c1, c2, want = grad_reference(dy, x, w, mean, rstd)
    rows, part, untouched = rows_for(users, 2 * dim, at, kind)
    dx = n.backward(dy, x, w, mean, rstd, dweight=part[:, :dim], dbias=part[:, dim:])
    e_hat = 2 * U32 * rstd.double()[..., None] * (x.double().abs() + mean.double().abs()[..., None])        # difference and product
    g1, gx = gain.abs().mean(-1, keepdim=True), (gain * xhat).abs().mean(-1, keepdim=True)
    e_c1, e_c2 = (dim + 3) * U32 * g1, (dim + 4) * U32 * gx + (gain.abs() * e_hat).mean(-1, keepdim=True)
    bound = rstd.double()[..., None] * (3 * U32 * (gain.abs() + c1.abs() + (xhat * c2).abs()) + e_c1 + xhat.abs() * e_c2 + e_hat * c2.abs())
    within(dx, want, bound, dtype)
    terms, d = dy.double() * xhat, dy.double()
    e_terms = (d.abs() * e_hat).sum(1)
    within(part[:, :dim], terms.sum(1), (tokens + 2) * U32 * terms.abs().sum(1) + e_terms, kind)
    within(part[:, dim:], d.sum(1), (tokens + 2) * U32 * d.abs().sum(1), kind)
    assert untouched()
    before = part.clone()
    assert n.backward(dy, x, w, mean, rstd, dweight=part[:, :dim], accumulate=True, want_dx=False) is None
    assert torch.equal(part[:, dim:], before[:, dim:])
    old = before[:, :dim].double()
    within(part[:, :dim], old + terms.sum(1), (tokens + 3) * U32 * terms.abs().sum(1) + e_terms + U32 * old.abs(), kind)
    other = n.backward(dy, x, w, mean, rstd, dx=dy)        # in place of dy
    assert other is dy and torch.equal(dy, dx)


def test_layer_norm_of_no_rows():
    n = b.LayerNorm(8, n_users=2)
    x = torch.empty((2, 0, 8), device="cuda")
    y, mean, rstd = n.forward(x)
    assert y.shape == (2, 0, 8) and mean.shape == rstd.shape == (2, 0)
    d = torch.ones((2, 8), device="cuda")
    n.backward(x, x, None, mean, rstd, dweight=d, accumulate=True)
    assert bool((d == 1).all())
    n.backward(x, x, None, mean, rstd, dweight=d)
    assert not d.any()


# (tokens, dim, type): several rows, and more than are on their way at a time, for each group of threads that the device holds; three users, of whose rows
# a group's next one may be the next user's
LONG = [(20_011, 64, BF16), (20_011, 200, F32), (12_007, 768, BF16), (7001, 1001, F32), (7001, 1001, BF16), (7001, 1024, F16), (2503, 4096, BF16), (2503, 4096, F32), (1201, 8192, BF16),
        (701, 16_384, BF16), (701, 16_384, F32), (701, 16_383, F32)]


@pytest.mark.parametrize("tokens,dim,dtype", LONG)
@pytest.mark.parametrize("how", ["dense", "gaps", "tokens first"])
def test_layer_norm_of_many_rows(tokens, dim, dtype, how):
    g = gen(dim)
    users = 3
    n = b.LayerNorm(dim, n_users=users)
    x = strided(g, users, tokens, dim, dtype, how)
    x.mul_(torch.rand((users, tokens, 1), generator=g, device="cuda").to(dtype) * 3).add_(normal(g, users, tokens, 1, dtype=dtype))
    w, bias = 1 + 0.3 * normal(g, dim), normal(g, dim)
    y, mean, rstd = n.forward(x, w, bias)
    for i in range(users):
        for at in range(0, tokens, 2000):                 # bounds as in test_layer_norm
            part = x[i, at:at + 2000].double()
            m, r, xhat, want = norm_reference(part, w, bias, 1e-5)
            mag = part.abs().mean(-1)
            e_mean = (dim + 2) * U32 * mag
            within(mean[i, at:at + 2000], m, e_mean)
            shift = e_mean + U32 * (m.abs() + mag)
            e_var = 2 * shift * (shift + (r ** -2).sqrt() * 2 * U32) + (dim + 6) * U32 * r ** -2
            e_r = 0.5 * r ** 3 * e_var + 4 * U32 * r
            within(rstd[i, at:at + 2000], r, e_r)
            e_x = (part - m[..., None]).abs()
            bound = w.double().abs() * (r[..., None] * (shift + U32 * e_x.amax(-1))[..., None] + (e_r + 2 * U32 * r)[..., None] * e_x) + 2 * U32 * (want.abs() + bias.double().abs())
            within(y[i, at:at + 2000], want, bound, dtype)
    dy, dw, db = normal(g, users, tokens, dim, dtype=dtype), torch.empty((users, dim), device="cuda"), torch.empty((users, dim), device="cuda")
    dx = n.backward(dy, x, w, mean, rstd, dweight=dw, dbias=db)
    for i in range(users):
        sums = [torch.zeros(dim, dtype=torch.float64, device="cuda") for _ in range(5)]
        for at in range(0, tokens, 2000):                 # bounds as in test_layer_norm_gradient
            g2, x2, m2, r2 = dy[i, at:at + 2000], x[i, at:at + 2000], mean[i, at:at + 2000], rstd[i, at:at + 2000]
            xhat, gain, c1, c2, want = grad_reference(g2, x2, w, m2, r2)
            e_hat = 2 * U32 * r2.double()[..., None] * (x2.double().abs() + m2.double().abs()[..., None])
            g1, gx = gain.abs().mean(-1, keepdim=True), (gain * xhat).abs().mean(-1, keepdim=True)
            e_c1, e_c2 = (dim + 3) * U32 * g1, (dim + 4) * U32 * gx + (gain.abs() * e_hat).mean(-1, keepdim=True)
            bound = r2.double()[..., None] * (3 * U32 * (gain.abs() + c1.abs() + (xhat * c2).abs()) + e_c1 + xhat.abs() * e_c2 + e_hat * c2.abs())
            within(dx[i, at:at + 2000], want, bound, dtype)
            d = g2.double()
            for s, more in zip(sums, ((d * xhat).sum(0), (d * xhat).abs().sum(0), (d.abs() * e_hat).sum(0), d.sum(0), d.abs().sum(0))):
                s.add_(more)
        within(dw[i], sums[0], (tokens + 2) * U32 * sums[1] + sums[2])
        within(db[i], sums[3], (tokens + 2) * U32 * sums[4])
    # in place, with rows of it on their way
    assert torch.equal(n.backward(dy, x, w, mean, rstd, dx=dy), dx)
    other, m, r = n.forward(x, w, bias, y=x)
    assert other is x and torch.equal(x, y) and torch.equal(m, mean) and torch.equal(r, rstd)


# ---- losses -------------------------------------------------------------------------------------------------------------------
def loss_reference(hidden, weight, index, q, tau):
    """Everything in 64 bits for one user's tokens that count.  index [n][k] with shares q [n][k]; (loss, lse, dz / c, error of a logit)."""
    h, w = hidden.double(), weight.double()
    z = h @ w.T / tau
    lse = torch.logsumexp(z, 1)
    dense = torch.zeros_like(z).scatter_add_(1, index, q)
    about = torch.where(q > 0, q * q.clamp(min=1e-300).log(), 0.0).sum(1)
    loss = about + lse * q.sum(1) - (dense * z).sum(1)
    dim = h.shape[1]
    steps = (min(dim, 1024) + 15) // 16 + 3 + (dim + 1023) // 1024
    e_z = steps * 2 * U32 * (h.abs() @ w.abs().T) / tau + 2 * U32 * z.abs()
    return loss, lse, (z - lse[:, None]).exp() - dense, e_z, dense, z


def check_losses(op, hidden, weight, there, index, q, tau, loss, lse, c=None, dhidden=None, dweight=None, kind=F32, old=None):
    """Compare a call's results, user by user.  c [users][tokens]: factor of each token's gradient."""
    dtype = hidden.dtype
    low = 2.0 ** -16 if dtype == BF16 else 2.0 ** -22     # dz in two numbers of 16 bits
    for i in range(hidden.shape[0]):
        on = there[i].nonzero().view(-1)
        off = (~there[i]).nonzero().view(-1)
        assert not loss[i][off].any() and not lse[i][off].any()
        want_loss, want_lse, dz, e_z, dense, z = loss_reference(hidden[i][on], weight, index[i][on], q[i][on], tau)
        n = on.numel()
        e_lse = e_z.amax(1) + 8 * U32 * (want_lse.abs() + z.abs().amax(1)) + (weight.shape[0] // 64 + 80) * U32 if n else want_lse
        within(lse[i][on], want_lse, e_lse)
        # shares from 32-bit exponentials, the entries' logits, the sum over entries
        qk = q[i][on]
        e_q = (16 + qk.shape[1]) * U32
        within(loss[i][on], want_loss, e_lse + (dense * e_z).sum(1) + 4 * e_q * (dense * (z.abs() + want_lse.abs()[:, None] + 100)).sum(1) + 4 * U32 * (want_lse.abs() + want_loss.abs()))
        if c is None:
            continue
        cc = c[i][on].double()[:, None] / tau
        # exponents in powers of two: their roundings are part of e; the exponential itself 2^-22
        e = e_z + e_lse[:, None] + 4 * U32 * (z.abs() + want_lse.abs()[:, None]) + 8 * U32
        e_dz = cc.abs() * ((dz + dense) * e * 1.01 + e_q * dense + 6 * U32 * dz.abs())
        # an exponential below 2^-126, the smallest normal number, is 0, and so is its product with c; nothing smaller is carried into a sum
        e_dz = e_dz + (cc.abs() + 1) * 2.0 ** -126
        g = cc * dz
        if dtype == F16:                                  # below 2^-24 of the user's largest factor's 2^14th part
            e_dz = e_dz + cc.abs().amax() * 2.0 ** -36 if n else e_dz
        hh, ww = hidden[i][on].double(), weight.double()
        if dhidden is not None:
            assert not dhidden[i][off].any()
            e16 = e_dz + u(dtype) * (g.abs() + e_dz)
            bound = e16 @ ww.abs() + (weight.shape[0] / 16 + 40) * 2 * U32 * (g.abs() @ ww.abs())
            within(dhidden[i][on], g @ ww, bound, dtype)
        if dweight is not None:
            e16 = e_dz + (low if kind == F32 else u(dtype)) * (g.abs() + e_dz)
            bound = e16.T @ hh.abs() + (64 + 4 + n / 512) * 2 * 2 * U32 * (g.abs().T @ hh.abs())
            want = g.T @ hh
            if old is not None:
                bound = bound + 2 * U32 * (old[i].double().abs() + want.abs())
                want = want + old[i].double()
            within(dweight[i], want, bound, kind)


SHAPES = [  # users, tokens, vocab, dim
    (1, 1, 1, 8), (1, 1, 2, 16), (2, 3, 100, 64), (1, 64, 127, 72), (3, 65, 128, 128), (1, 130, 129, 200), (2, 257, 255, 136), (1, 300, 256, 264),
    (2, 40, 257, 1032), (1, 700, 1000, 96), (3, 200, 5003, 64), (1, 33, 700, 2056), (5, 9, 513, 40),
]


def some_targets(g, users, tokens, vocab, none=0.25):
    k = torch.randint(0, vocab, (users, tokens), generator=g, device="cuda")
    k = torch.where(torch.rand((users, tokens), generator=g, device="cuda") < none, -1 - k, k)
    if users > 2:
        k[1] = -5                                         # a user without a target
    return k


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape", SHAPES)
def test_cross_entropy(shape, dtype):
    users, tokens, vocab, dim = shape
    g = gen(sum(shape))
    i = SHAPES.index(shape)
    kind = F32 if (i + (dtype == F16)) % 2 else dtype
    at = [0, 8, 1][i % 3]
    t = b.TokenLoss(vocab, dim, n_users=users, tokens=tokens + (i % 2) * 70, dtype=dtype, grad_dtype=kind)
    hidden = strided(g, users, tokens, dim, dtype, ["dense", "gaps", "odd", "tokens first"][i % 4])
    weight = normal(g, vocab, dim + 8 * (i % 2), dtype=dtype)[:, :dim]
    weight.mul_(2.0 / math.sqrt(dim))
    k = some_targets(g, users, tokens, vocab)
    there = k >= 0
    hidden.masked_fill_(~there[..., None], [NAN, math.inf][i % 2])
    targets = k.int() if i % 2 else k
    index, q = k.clamp(min=0)[..., None], torch.ones((users, tokens, 1), dtype=torch.float64, device="cuda")
    loss, lse = t.loss(hidden, weight, targets)
    rows, part, untouched = rows_for(users, vocab * dim, at, kind)
    if i % 2:                                             # the mean of each user
        c = (1.0 / there.sum(1, keepdim=True).clamp(min=1)).expand(users, tokens)
        dhidden = t.loss_grad(hidden, weight, targets, lse, dweight=part)
    else:
        given = normal(g, users, tokens)
        given.masked_fill_(~there, NAN)
        c = given.double() * 0.7
        dhidden = t.loss_grad(hidden, weight, targets, lse, given, scale=0.7, dweight=part)
    d = part.view(users, vocab, dim) if at == 0 and users == 1 else part.reshape(users, vocab, dim)
    check_losses(t, hidden, weight, there, index, q, 1.0, loss, lse, c, dhidden, d, kind)
    assert untouched() and t.status() == (0, 0)
    first, h1 = part.clone(), dhidden.clone()
    args = (hidden, weight, targets, lse) + (() if i % 2 else (given,))
    more = {} if i % 2 else {"scale": 0.7}
    assert torch.equal(t.loss_grad(*args, **more), h1), "without dweight"
    assert t.loss_grad(*args, **more, dweight=part, want_dhidden=False) is None and torch.equal(part, first)
    t.loss_grad(*args, **more, dweight=part, accumulate=True)
    check_losses(t, hidden, weight, there, index, q, 1.0, loss, lse, c, None, part.reshape(users, vocab, dim), kind, old=first.reshape(users, vocab, dim))
    assert untouched() and t.status() == (0, 0)


def shares(logits, index, tau):
    x = torch.where(index >= 0, logits.double() / tau, -math.inf)
    m = x.amax(-1, keepdim=True)
    e = torch.where(m == -math.inf, 0.0, (x - torch.where(m == -math.inf, 0.0, m)).exp())
    total = e.sum(-1, keepdim=True)
    return torch.where(total > 0, e / total.clamp(min=1e-300), 0.0)


@pytest.mark.parametrize("dtype,teacher", [(BF16, F32), (F16, F16), (BF16, BF16)])
@pytest.mark.parametrize("top,tau", [(1, 1.0), (2, 3.0), (33, 0.7), (64, 1.5), (128, 2.0)])
@pytest.mark.parametrize("shape", [(1, 5, 40, 64), (3, 70, 1000, 136), (2, 140, 129, 72)])
def test_distillation(shape, top, tau, dtype, teacher):
    users, tokens, vocab, dim = shape
    g = gen(sum(shape) + top)
    kind = F32 if top % 2 else dtype
    t = b.TokenLoss(vocab, dim, n_users=users, tokens=tokens, dtype=dtype, grad_dtype=kind, top=top)
    hidden, weight = normal(g, users, tokens, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype).mul_(2.0 / math.sqrt(dim))
    index = torch.randint(0, vocab, (users, tokens, top), generator=g, device="cuda")        # some stand twice
    index = torch.where(torch.rand(index.shape, generator=g, device="cuda") < 0.2, -1, index)
    logits = (3 * normal(g, users, tokens, top)).to(teacher)
    logits = torch.where(torch.rand(index.shape, generator=g, device="cuda") < 0.1, -math.inf, logits)
    logits = torch.where(index < 0, torch.tensor([NAN, math.inf, -math.inf], device="cuda").to(teacher)[torch.randint(0, 3, index.shape, generator=g, device="cuda")], logits)
    index[0, 0] = -3                                      # a token without any entry, and one whose entries have no mass
    if tokens > 2:
        logits[0, 2] = -math.inf
    q = shares(logits, index, tau)
    there = q.sum(-1) > 0
    hidden.masked_fill_(~there[..., None], NAN)
    loss, lse = t.distill(hidden, weight, index, logits, tau)
    given = torch.rand((users, tokens), generator=g, device="cuda")
    rows, part, untouched = rows_for(users, vocab * dim, 8 * (top % 3), kind)
    dhidden = t.distill_grad(hidden, weight, index.int(), logits, lse, given, tau, scale=2.0, dweight=part)
    check_losses(t, hidden, weight, there, index.clamp(min=0), q, tau, loss, lse, 2.0 * given.double(), dhidden, part.reshape(users, vocab, dim), kind)
    assert untouched() and t.status() == (0, 0)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("users,tokens", [(1, 8192), (1, 8193), (32, 256), (33, 249), (256, 32), (256, 1), (257, 3), (300, 40), (2100, 5)])
def test_losses_of_many_tokens_and_users(users, tokens, dtype):
    """Both sides of the limits of 8192 tokens and 256 users, above which the tokens with a target are packed in another way; beyond 1024 users that one keeps its counts elsewhere."""
    g = gen(users + tokens)
    vocab, dim = 24, 8
    t = b.TokenLoss(vocab, dim, n_users=users, tokens=tokens, dtype=dtype, grad_dtype=F32, top=3)
    hidden, weight = normal(g, users, tokens, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype)
    k = some_targets(g, users, tokens, vocab)
    there = k >= 0
    loss, lse = t.loss(hidden, weight, k)
    c = torch.rand((users, tokens), generator=g, device="cuda")
    d = torch.empty((users, vocab, dim), device="cuda")
    dhidden = t.loss_grad(hidden, weight, k, lse, c, dweight=d)
    check_losses(t, hidden, weight, there, k.clamp(min=0)[..., None], torch.ones((users, tokens, 1), dtype=torch.float64, device="cuda"), 1.0, loss, lse, c, dhidden, d)
    # no token's loss depends on the others, nor on the user it is of
    alone = b.TokenLoss(vocab, dim, tokens=tokens, dtype=dtype, top=3)
    index = torch.stack([k, torch.randint(-2, vocab, k.shape, generator=g, device="cuda"), (k + 1).clamp(min=-1, max=vocab - 1)], -1)
    logits = normal(g, users, tokens, 3)
    soft = t.distill(hidden, weight, index, logits, 2.0)
    for i in {0, users // 2, users - 1}:
        assert all(torch.equal(x[i], y) for x, y in zip((loss, lse), alone.loss(hidden[i], weight, k[i])))
        assert all(torch.equal(x[i], y) for x, y in zip(soft, alone.distill(hidden[i], weight, index[i], logits[i], 2.0)))
    assert t.status() == (0, 0) and alone.status() == (0, 0)


@pytest.mark.parametrize("teacher", [F32, BF16, F16])
@pytest.mark.parametrize("tau", [0.25, 1.0])
def test_teacher_logits_at_their_type_s_ends(teacher, tau):
    """Masked with the type's lowest value, or as large as it goes: over the temperature they pass 32 bits, their differences from the largest tell the shares."""
    low, high, inf = torch.finfo(teacher).min, torch.finfo(teacher).max, math.inf
    logits = torch.tensor([[low, low, low], [high, high, 0.0], [low, 1.0, 0.0], [high, low, high], [low, low, -inf], [-inf, low, 0.0], [-inf, -inf, -inf], [-inf, low, -inf]],
                          dtype=teacher, device="cuda")[None]
    g = gen(7)
    vocab, dim, n = 40, 64, logits.shape[1]
    t = b.TokenLoss(vocab, dim, tokens=n, dtype=BF16, top=3)
    hidden, weight = normal(g, 1, n, dim, dtype=BF16), normal(g, vocab, dim, dtype=BF16) * 0.25
    index = torch.tensor([[5, 0, 39]], device="cuda").expand(1, n, 3).contiguous()
    q = shares(logits, index, tau)
    there = q.sum(-1) > 0
    assert there.tolist() == [[True] * 6 + [False, True]]
    loss, lse = t.distill(hidden, weight, index, logits, tau)
    c, d = torch.ones((1, n), device="cuda"), torch.empty((1, vocab, dim), device="cuda")
    dhidden = t.distill_grad(hidden, weight, index, logits, lse, c, tau, dweight=d[0])
    check_losses(t, hidden, weight, there, index, q, tau, loss, lse, c, dhidden, d)


def test_the_gradient_formula_of_distillation_against_differences():
    g = gen(2)
    n, vocab, dim, tau = 3, 7, 8, 1.7
    h, w = normal(g, n, dim, dtype=torch.float64), normal(g, vocab, dim, dtype=torch.float64)
    index = torch.tensor([[0, 3], [3, 3], [6, 1]], device="cuda")
    q = torch.tensor([[0.7, 0.3], [0.6, 0.4], [1.0, 0.0]], dtype=torch.float64, device="cuda")
    dz = loss_reference(h, w, index, q, tau)[2] / tau
    step = 1e-6
    for t, grad in ((h, dz @ w), (w, dz.T @ h)):
        for i in range(0, t.numel(), 5):
            e = torch.zeros_like(t).view(-1)
            e[i] = step
            e = e.view(t.shape)
            up, down = (loss_reference(*(x + s * e if x is t else x for x in (h, w)), index, q, tau)[0].sum() for s in (1, -1))
            assert abs((up - down).item() / (2 * step) - grad.reshape(-1)[i].item()) < 1e-7


def test_a_vocabulary_in_several_pieces():
    """256 rows of dz over 600001 entries pass the 2^27 elements that are held at a time."""
    vocab, dim, tokens = 600_001, 8, 60
    g = gen(8)
    for dtype, kind in ((BF16, F32), (F16, F16)):
        t = b.TokenLoss(vocab, dim, tokens=tokens, dtype=dtype, grad_dtype=kind)
        hidden, weight = normal(g, 1, tokens, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype)
        k = torch.randint(0, vocab, (1, tokens), generator=g, device="cuda")
        k[0, :4] = torch.tensor([0, vocab - 1, -1, 300_032], device="cuda")
        there = k >= 0
        loss, lse = t.loss(hidden[0], weight, k[0])
        d = torch.empty((vocab, dim), dtype=kind, device="cuda")
        dhidden = t.loss_grad(hidden[0], weight, k[0], lse, dweight=d)
        c = torch.full((1, tokens), 1.0 / there.sum().item(), device="cuda")
        check_losses(t, hidden, weight, there, k.clamp(min=0)[..., None], torch.ones((1, tokens, 1), dtype=torch.float64, device="cuda"), 1.0, loss[None], lse[None],
                     c, dhidden[None], d[None], kind)


@pytest.mark.parametrize("at", [0, 3])
def test_a_weight_that_passes_32_bits(at):
    """4.6e9 elements.  Of a weight of zeros all logits are 0: dz is 1 / vocab, less 1 at the target, and dhidden is 0."""
    vocab, dim = 70_001, 65_536
    t = b.TokenLoss(vocab, dim, tokens=2, dtype=BF16, grad_dtype=BF16)
    weight = torch.zeros((vocab, dim), dtype=BF16, device="cuda")
    hidden = torch.ones((2, dim), dtype=BF16, device="cuda")
    k = torch.tensor([vocab - 1, -1], device="cuda")
    loss, lse = t.loss(hidden, weight, k)
    assert abs(loss[0].item() - math.log(vocab)) <= 1e-5 and loss[1].item() == 0
    memory = torch.full((vocab * dim + 8,), 7.0, dtype=BF16, device="cuda")
    d = memory[at:at + vocab * dim]
    dhidden = t.loss_grad(hidden, weight, k, lse, dweight=d)
    assert not dhidden.any()
    p, d = 1.0 / vocab, d.view(vocab, dim)
    for rows, want in ((d[:9], p), (d[65_530:65_540], p), (d[vocab - 9:vocab - 1], p), (d[vocab - 1:], p - 1.0)):
        assert ((rows.double() - want).abs() <= abs(want) * (2 * u(BF16) + 1e-5)).all()
    assert bool((memory[:at] == 7).all()) and bool((memory[at + vocab * dim:] == 7).all())


@pytest.mark.parametrize("dtype,kind", [(BF16, F32), (BF16, BF16), (F16, F32), (F16, F16)])
@pytest.mark.parametrize("tokens,vocab,dim", [(300, 20_011, 2056), (2500, 2603, 1032)])
def test_losses_of_many_deep_tiles(tokens, vocab, dim, dtype, kind):
    """More tiles than pairs of SMs, and a depth that accumulators take in an odd number of parts: of the logits (33 stages of 64), and of the weight's gradient
    (users of different lengths, the longer of over 1024 tokens)."""
    g = gen(tokens)
    users = 2
    t = b.TokenLoss(vocab, dim, n_users=users, tokens=tokens, dtype=dtype, grad_dtype=kind)
    hidden, weight = normal(g, users, tokens, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype).mul_(2.0 / math.sqrt(dim))
    k = some_targets(g, users, tokens, vocab, none=0.1)
    k[1, tokens // 2:] = -1
    there = k >= 0
    hidden.masked_fill_(~there[..., None], NAN)
    loss, lse = t.loss(hidden, weight, k)
    c = 0.1 + torch.rand((users, tokens), generator=g, device="cuda")
    for at in (0, 1):                                     # by TMA, and through shared memory
        rows, part, untouched = rows_for(users, vocab * dim, at, kind)
        dhidden = t.loss_grad(hidden, weight, k, lse, c, dweight=part)
        check_losses(t, hidden, weight, there, k.clamp(min=0)[..., None], torch.ones((users, tokens, 1), dtype=torch.float64, device="cuda"), 1.0, loss, lse, c, dhidden,
                     part.unflatten(1, (vocab, dim)), kind)
        assert untouched() and t.status() == (0, 0)


def test_rows_of_a_weight_that_passes_32_bits():
    """Of 4.6e9 elements three rows are not zero, the first, one in the middle and the last: their logits are whole numbers."""
    vocab, dim = 70_001, 65_536
    t = b.TokenLoss(vocab, dim, tokens=3, dtype=BF16, grad_dtype=BF16)
    weight, hidden = torch.zeros((vocab, dim), dtype=BF16, device="cuda"), torch.ones((3, dim), dtype=BF16, device="cuda")
    rows = {0: 1.0, 35_003: -2.0, vocab - 1: 3.0}
    for v, z in rows.items():
        weight[v] = z / dim
    k = torch.tensor([vocab - 1, 35_003, 17], device="cuda")
    loss, lse = t.loss(hidden, weight, k)
    want = math.log(vocab - 3 + sum(math.exp(z) for z in rows.values()))
    # sums of 65536 equal products: each cut off at 16 of depth, 64 parts of 1024 added in 32 bits
    e = (64 + 67) * 2 * U32 * 3.0 + 40 * U32 * want
    assert (lse.double() - want).abs().max() <= e
    assert (loss.double() - (want - torch.tensor([3.0, -2.0, 0.0], device="cuda").double())).abs().max() <= 2 * e
    d = torch.empty((vocab, dim), dtype=BF16, device="cuda")
    dhidden = t.loss_grad(hidden, weight, k, lse, torch.ones(3, device="cuda"), dweight=d)
    # logits of the gradient call are one sum: 4096 parts of 16 of depth
    e = 4096 * 2 * U32 * 3.0 + e
    at = torch.tensor([0, 1, 17, 35_002, 35_003, 35_004, vocab - 2, vocab - 1], device="cuda")
    p = torch.tensor([math.exp(rows.get(int(v), 0.0) - want) for v in at], device="cuda").double()
    dz = p - (at == k[:, None]).double()                  # [3][8]
    e_dz = p * e + u(BF16) * (dz.abs() + p * e) + 2.0 ** -20 * p
    got = d[at].double()
    assert bool((got == got[:, :1]).all())                # all hidden states are 1
    assert ((got[:, 0] - dz.sum(0)).abs() <= e_dz.sum(0) * 1.01 + u(BF16) * dz.sum(0).abs() * 1.01).all()
    some = [0, 4, 7]                                      # the rows that are not zero
    w = torch.tensor(list(rows.values()), device="cuda").double() / dim
    h = (dz[:, some] * w).sum(1, keepdim=True)
    room = (e_dz[:, some] * w.abs()).sum(1, keepdim=True) * 1.01 + (vocab / 16) * 2 * U32 * (dz[:, some] * w).abs().sum(1, keepdim=True) + u(BF16) * h.abs() * 1.01
    assert ((dhidden.double() - h).abs() <= room).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape", SHAPES + [(2, 300, 20_011, 2056)])
def test_cross_entropy_to_a_few_roundings(shape, dtype):
    """One exact entry: the loss is off by what lse and the target's logit are, and the difference's rounding."""
    users, tokens, vocab, dim = shape
    g = gen(sum(shape) + 1)
    t = b.TokenLoss(vocab, dim, n_users=users, tokens=tokens, dtype=dtype)
    hidden, weight = normal(g, users, tokens, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype).mul_(2.0 / math.sqrt(dim))
    k = torch.randint(0, vocab, (users, tokens), generator=g, device="cuda")
    loss, lse = t.loss(hidden, weight, k)
    for i in range(users):
        want, want_lse, _, e_z, dense, z = loss_reference(hidden[i], weight, k[i][:, None], torch.ones((tokens, 1), dtype=torch.float64, device="cuda"), 1.0)
        # the largest logit over the logarithm's and the exponents' conversion to powers of two and back; a tile's 64 and the tiles' sums
        e_lse = e_z.amax(1) + 8 * U32 * (want_lse.abs() + z.abs().amax(1)) + (vocab // 64 + 80) * U32
        within(lse[i], want_lse, e_lse)
        within(loss[i], want, e_lse + (dense * e_z).sum(1) + U32 * want.abs())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_logits_far_apart(dtype):
    """Logits of hundreds: exponentials of differences only, losses of 0 and of hundreds."""
    g = gen(4)
    hidden, weight = 20 * normal(g, 1, 50, 64, dtype=dtype), normal(g, 300, 64, dtype=dtype)
    t = b.TokenLoss(300, 64, tokens=50, dtype=dtype)
    k = (hidden[0].double() @ weight.double().T).argmax(1)[None]
    k[0, ::2] = 7
    loss, lse = t.loss(hidden, weight, k)
    d = torch.empty((300, 64), device="cuda")
    dhidden = t.loss_grad(hidden, weight, k, lse, dweight=d)
    check_losses(t, hidden, weight, k >= 0, k[..., None], torch.ones((1, 50, 1), dtype=torch.float64, device="cuda"), 1.0, loss, lse, torch.full((1, 50), 0.02, device="cuda"), dhidden, d[None])


@pytest.mark.parametrize("size", [1e-9, 1e5])
def test_small_and_large_gradients_in_half_precision(size):
    """dz is scaled by a power of two of the user's own: neither lost below 6e-8 nor beyond 65504."""
    g = gen(5)
    users, tokens, vocab, dim = 2, 30, 200, 64
    t = b.TokenLoss(vocab, dim, n_users=users, tokens=tokens, dtype=F16, grad_dtype=F32)
    hidden, weight = normal(g, users, tokens, dim, dtype=F16), normal(g, vocab, dim, dtype=F16) * 0.25
    k = some_targets(g, users, tokens, vocab)
    loss, lse = t.loss(hidden, weight, k)
    c = torch.rand((users, tokens), generator=g, device="cuda") * size
    c[1] *= 1e-6
    d = torch.empty((users, vocab, dim), device="cuda")
    dhidden = t.loss_grad(hidden, weight, k, lse, c, dweight=d, want_dhidden=False)
    check_losses(t, hidden, weight, k >= 0, k.clamp(min=0)[..., None], torch.ones((users, tokens, 1), dtype=torch.float64, device="cuda"), 1.0, loss, lse, c, dhidden, d)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("at,dim", [(0, 72), (1, 136), (2, 8)])
def test_a_weight_gradient_in_16_bits_that_is_added_to_is_rounded_once(dtype, at, dim):
    """A weight of zeros: dz is 1/64, or -63/64 at the target, exactly in 16 bits, and sums of whole hidden states up to 255 and of whole numbers up to
    2000 have 20 bits at most.  So nothing is rounded but what is stored."""
    g = gen(at)
    users, tokens, vocab = 2, 60, 64
    t = b.TokenLoss(vocab, dim, n_users=users, tokens=tokens, dtype=dtype, grad_dtype=dtype)
    hidden = torch.randint(-255, 256, (users, tokens, dim), generator=g, device="cuda").to(dtype)
    weight = torch.zeros((vocab, dim), dtype=dtype, device="cuda")
    k = torch.randint(0, vocab, (users, tokens), generator=g, device="cuda")
    _, lse = t.loss(hidden, weight, k)
    rows, part, untouched = rows_for(users, vocab * dim, at, dtype)
    part.copy_(torch.randint(-2000, 2001, part.shape, generator=g, device="cuda"))
    dz = 1 / 64 - torch.nn.functional.one_hot(k, vocab).double()
    want = part.double() + (dz.transpose(1, 2) @ hidden.double()).reshape(users, -1)
    t.loss_grad(hidden, weight, k, lse, torch.ones((users, tokens), device="cuda"), dweight=part, accumulate=True)
    assert torch.equal(part, want.float().to(dtype)) and untouched()


def test_targets_that_the_vocabulary_does_not_have():
    g = gen(6)
    t = b.TokenLoss(100, 64, tokens=6, top=2)
    hidden, weight = normal(g, 6, 64, dtype=BF16), normal(g, 100, 64, dtype=BF16)
    k = torch.tensor([0, 100, 99, 2 ** 40, -1, 5], device="cuda")
    loss, lse = t.loss(hidden, weight, k)
    assert (loss == 0).tolist() == [False, True, False, True, True, False]
    assert t.status(clear=True) == (b.FLAG_TOKEN, 2) and t.status() == (0, 0)
    index = torch.stack([k, torch.full_like(k, 3)], 1)
    loss, _ = t.distill(hidden, weight, index, torch.zeros((6, 2), device="cuda"))
    alone, _ = t.distill(hidden, weight, torch.where(index > 99, -1, index), torch.zeros((6, 2), device="cuda"))
    assert torch.equal(loss, alone) and t.status() == (b.FLAG_TOKEN, 2)


def test_not_a_number_where_it_counts():
    """In a token that has a target it reaches that token's loss, and the gradient of its user's weight, not other users'."""
    g = gen(7)
    t = b.TokenLoss(40, 64, n_users=2, tokens=5, grad_dtype=F32)
    hidden, weight, k = normal(g, 2, 5, 64, dtype=BF16), normal(g, 40, 64, dtype=BF16), torch.zeros((2, 5), dtype=torch.int64, device="cuda")
    hidden[1, 2, 7] = NAN
    loss, lse = t.loss(hidden, weight, k)
    assert loss.isnan().nonzero().tolist() == [[1, 2]]
    d = torch.empty((2, 40, 64), device="cuda")
    dhidden = t.loss_grad(hidden, weight, k, lse, dweight=d)
    assert not d[0].isnan().any() and d[1].isnan().all()
    assert dhidden.isnan().all(2).nonzero().tolist() == [[1, 2]] and dhidden.isnan().sum() == 64
    # a token whose gradient is not wanted has none, whatever it holds
    d.zero_()
    t.loss_grad(hidden, weight, k, lse, torch.tensor([[1.0] * 5, [1.0, 1.0, 0.0, 1.0, 1.0]], device="cuda"), dweight=d[:, :, :].view(2, -1))
    assert d[0].isfinite().all()


@pytest.mark.parametrize("dtype,kind", [(BF16, F32), (BF16, BF16), (F16, F32)])
@pytest.mark.parametrize("users,tokens", [(2, 90), (257, 5)])         # both ways of packing
def test_tokens_whose_gradient_is_not_wanted(users, tokens, dtype, kind):
    """A token with dloss 0 has no gradient, whatever it holds: the same bits as if it had no target."""
    g = gen(users)
    vocab, dim, top = 300, 72, 3
    t = b.TokenLoss(vocab, dim, n_users=users, tokens=tokens, dtype=dtype, grad_dtype=kind, top=top)
    hidden, weight = normal(g, users, tokens, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype) * 0.2
    k = torch.randint(0, vocab, (users, tokens), generator=g, device="cuda")
    out = torch.rand((users, tokens), generator=g, device="cuda") < 0.3
    out[1], out[0, 0] = True, True                        # a user of whose tokens none counts
    hidden = torch.where(out[..., None], torch.tensor([NAN, math.inf], dtype=dtype, device="cuda")[k % 2][..., None], hidden)
    c = torch.where(out, torch.tensor([0.0, -0.0], device="cuda")[k % 2], 0.1 + torch.rand((users, tokens), generator=g, device="cuda"))
    index, logits = torch.stack([k, (k + 1) % vocab, (k + 7) % vocab], -1), normal(g, users, tokens, top)
    d, e = torch.empty((users, vocab * dim), dtype=kind, device="cuda"), torch.empty((users, vocab * dim), dtype=kind, device="cuda")
    _, lse = t.loss(hidden, weight, k)
    got, want = t.loss_grad(hidden, weight, k, lse, c, dweight=d), t.loss_grad(hidden, weight, k.masked_fill(out, -1), lse, c, dweight=e)
    assert torch.equal(got, want) and not got[out].any() and torch.equal(d, e) and d.isfinite().all() and not d[1].any() and d[0].any()
    _, lse = t.distill(hidden, weight, index, logits, 2.0)
    got = t.distill_grad(hidden, weight, index, logits, lse, c, 2.0, dweight=d)
    want = t.distill_grad(hidden, weight, index.masked_fill(out[..., None], -1), logits, lse, c, 2.0, dweight=e)
    assert torch.equal(got, want) and not got[out].any() and torch.equal(d, e) and d.isfinite().all() and not d[1].any() and d[0].any()
    assert t.status() == (0, 0)


def test_losses_of_no_tokens():
    t = b.TokenLoss(40, 64, n_users=2, tokens=5, grad_dtype=F32)
    weight, none = torch.ones((40, 64), dtype=BF16, device="cuda"), torch.empty((2, 0, 64), dtype=BF16, device="cuda")
    k = torch.empty((2, 0), dtype=torch.int64, device="cuda")
    loss, lse = t.loss(none, weight, k)
    assert loss.shape == lse.shape == (2, 0)
    d = torch.ones((2, 40 * 64), device="cuda")
    assert t.loss_grad(none, weight, k, lse, dweight=d, accumulate=True).shape == (2, 0, 64) and bool((d == 1).all())
    t.loss_grad(none, weight, k, lse, dweight=d)
    assert not d.any()
    k = torch.full((2, 5), -1, device="cuda")
    hidden = torch.full((2, 5, 64), NAN, dtype=BF16, device="cuda")
    loss, lse = t.loss(hidden, weight, k)
    d.fill_(3.0)
    dhidden = t.loss_grad(hidden, weight, k, lse, dweight=d)
    assert not loss.any() and not lse.any() and not d.any() and not dhidden.any()


# ---- together, streams, graphs ----------------------------------------------------------------------------------------------------
class Chain:
    """Embedding, layer norm, loss and back, for three users, into gradient rows."""

    def __init__(self, seed, top=1):
        g = gen(seed)
        self.users, self.tokens, self.vocab, self.dim = 3, 50, 300, 72
        U, T, V, D = self.users, self.tokens, self.vocab, self.dim
        self.e, self.n = b.Embedding(V, D, n_users=U, tokens=T), b.LayerNorm(D, n_users=U)
        self.t = b.TokenLoss(V, D, n_users=U, tokens=T, dtype=BF16, grad_dtype=F32, top=top)
        self.table, self.w, self.bias, self.head = normal(g, V, D), 1 + 0.1 * normal(g, D), normal(g, D), normal(g, V, D, dtype=BF16) * 0.2
        self.inputs, self.targets = some_tokens(g, U, T, V), some_targets(g, U, T, V)
        self.rows = torch.zeros((U, (2 * V * D + 2 * D + 3) // 4 * 4 + 4), device="cuda")
        at = [1, 1 + V * D, 1 + V * D + D, 1 + V * D + 2 * D, 1 + 2 * V * D + 2 * D]
        self.parts = [self.rows[:, i:j] for i, j in zip(at, at[1:])]

    def run(self, stream=None):
        x = self.e.forward(self.inputs, self.table, scale=2.0, stream=stream)
        y, mean, rstd = self.n.forward(x, self.w, self.bias, stream=stream)
        if stream is None:
            h = y.bfloat16()
        else:
            with torch.cuda.stream(stream):
                h = y.bfloat16()
        loss, lse = self.t.loss(h, self.head, self.targets, stream=stream)
        dh = self.t.loss_grad(h, self.head, self.targets, lse, dweight=self.parts[3], stream=stream)
        if stream is None:
            dy = dh.float()
        else:
            with torch.cuda.stream(stream):
                dy = dh.float()
        dx = self.n.backward(dy, x, self.w, mean, rstd, dweight=self.parts[1], dbias=self.parts[2], stream=stream)
        self.e.backward(dx, self.inputs, self.parts[0], scale=2.0, stream=stream)
        return loss, dh, dx


def test_the_chain_against_autograd():
    c = Chain(1)
    loss, _, _ = c.run()
    for i in range(c.users):
        table, w, bias, head = (x.double().requires_grad_() for x in (c.table, c.w, c.bias, c.head))
        here = c.inputs[i] >= 0
        x = torch.where(here[:, None], table[c.inputs[i].clamp(min=0)] * 2.0, 0.0)
        y = torch.nn.functional.layer_norm(x, (c.dim,), w, bias, 1e-5)
        on = c.targets[i] >= 0
        each = torch.nn.functional.cross_entropy(y @ head.T, c.targets[i].clamp(min=0), reduction="none")
        # hidden states are rounded to 8 bits before the head: 2^-8 of |y|, times a row of the head
        room = u(BF16) * (y.abs() @ head.abs().T).amax(1) * 2 + 1e-5
        assert ((loss[i].double() - each).abs() <= room)[on].all() and not loss[i][~on].any()
        if not on.any():
            assert not c.rows[i].any()
            continue
        (each[on].mean()).backward()
        for part, grad in zip(c.parts, (table.grad, w.grad, bias.grad, head.grad)):
            got, want = part[i].double(), grad.reshape(-1)
            # four roundings to 8 bits along the way (hidden, dz, dhidden, and the head's product with the first), 2^-8 each at most, in the norm of the whole
            assert (got - want).norm() <= 5 * u(BF16) * want.norm()


def test_the_chain_on_other_streams_and_replayed():
    c, d = Chain(2), Chain(2)
    want = [x.clone() for x in c.run()] + [c.rows.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.rows.fill_(NAN)
    got = c.run(stream=side)
    d.rows.fill_(NAN)
    again = d.run()                                       # another set of handles at the same time
    torch.cuda.synchronize()
    for part, other in zip(c.parts, d.parts):
        assert torch.equal(part, other)
    for x, y, z in zip(want, got, again):
        assert torch.equal(x, y) and torch.equal(x, z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.run()
    for seed in (2, 9, 2):
        fresh = Chain(seed)
        for name in ("table", "w", "bias", "head", "inputs", "targets"):
            getattr(c, name).copy_(getattr(fresh, name))
        c.rows.fill_(NAN)
        graph.replay()
        expect = fresh.run()
        torch.cuda.synchronize()
        for x, y in zip(expect, out):
            assert torch.equal(x, y)
        for x, y in zip(fresh.parts, c.parts):
            assert torch.equal(x, y)
    assert c.t.status() == c.e.status() == (0, 0)


def test_a_chain_on_another_stream_whose_rows_were_filled_before():
    """The fill is ordered before the side stream's work, and the rows are those of the first run."""
    c = Chain(4)
    want = [x.clone() for x in c.run()]
    rows = [part.clone() for part in c.parts]
    for fill in (NAN, 3.0):
        c.rows.fill_(fill)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = c.run(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(x, y) for x, y in zip(want, got)) and all(torch.equal(x, y) for x, y in zip(rows, c.parts))


def test_outputs_are_marked_as_changed():
    c = Chain(3)
    before = c.rows._version
    c.run()
    assert c.rows._version > before
    loss, lse = torch.empty((3, 50), device="cuda"), torch.empty((3, 50), device="cuda")
    v = loss._version
    c.t.loss(normal(gen(1), 3, 50, 72, dtype=BF16), c.head, c.targets, loss=loss, lse=lse)
    assert loss._version > v


@pytest.mark.parametrize("teacher", [0, 3])
def test_the_training_loop_of_tokens(teacher):
    """It runs, encodes and decodes, and its rows hold the users' gradients."""
    from paper_2203_09044_b200 import train_step
    losses = train_step.run_tokens(iterations=4, n_users=3, vocab=300, dim=64, tokens=40, teacher=teacher)
    assert len(losses) == 4 and all(math.isfinite(x) for x in losses)
    g = gen(5)
    model = train_step.TokenModel(300, 64, 3, 40, top=max(1, teacher), seed=1)
    inputs, targets = train_step.token_batch(torch.randint(0, 300, (300, 4), generator=g, device="cuda"), 3, 40, g)
    rows = torch.full((3, model.d + 3), NAN, device="cuda")
    entries = None
    if teacher:
        index = torch.randint(0, 300, (3, 40, teacher), generator=g, device="cuda").masked_fill((inputs < 0)[..., None], -1)
        entries = index, normal(g, 3, 40, teacher)
    loss = model.gradients(inputs, targets, rows, entries)
    for i in range(3):
        on = inputs[i] >= 0
        table, scale, shift, head = (c.double().requires_grad_() for c in model.copies)
        y = torch.nn.functional.layer_norm(table[inputs[i][on]], (64,), scale, shift, 1e-5)
        logp = torch.log_softmax(y @ head.T, 1)
        if teacher:
            q = shares(entries[1][i][on], index[i][on], 1.0)
            each = (q * (q.log() - logp.gather(1, index[i][on]))).sum(1)
        else:
            each = -logp.gather(1, targets[i][on][:, None])[:, 0]
        assert not loss[i][~on].any()
        # hidden states in 8 bits: 2^-8 of |y|, times a row of the head, for the target and the mean over the others
        assert ((loss[i][on].double() - each).abs() <= 2 * u(BF16) * (y.abs() @ head.abs().T).amax(1) + 1e-5).all()
        each.mean().backward()
        for part, grad in zip(model.segments(rows), (table.grad, scale.grad, shift.grad, head.grad)):
            # roundings to 8 bits on the way: hidden, dz, dhidden, dx
            assert (part[i].double() - grad.reshape(-1)).norm() <= 5 * u(BF16) * grad.norm()
    assert rows[:, model.d:].isnan().all()


def test_the_training_loop_of_one_token():
    """A user's only token is always there: no mean over no tokens."""
    from paper_2203_09044_b200 import train_step
    for seed in range(3):
        assert all(math.isfinite(x) for x in train_step.run_tokens(iterations=8, n_users=1, vocab=50, dim=64, tokens=1, seed=seed))


# ---- refusals -----------------------------------------------------------------------------------------------------------------
def refused(call, *errors):
    with pytest.raises(errors or (ValueError, TypeError, b.Co3Error)):
        call()


def test_refusals():
    for make in (lambda: b.Embedding(0, 8, tokens=1), lambda: b.Embedding(8, 0, tokens=1), lambda: b.Embedding(8, 8, n_users=0, tokens=1), lambda: b.Embedding(8, 8, tokens=-1),
                 lambda: b.Embedding(1 << 31, 8, tokens=1),
                 lambda: b.LayerNorm(0), lambda: b.LayerNorm(16385), lambda: b.LayerNorm(8, eps=-1.0), lambda: b.LayerNorm(8, eps=NAN), lambda: b.LayerNorm(8, n_users=0),
                 lambda: b.TokenLoss(0, 8, tokens=1), lambda: b.TokenLoss(8, 12, tokens=1), lambda: b.TokenLoss(8, 8, tokens=1, top=129), lambda: b.TokenLoss(8, 8, tokens=1, top=0),
                 lambda: b.TokenLoss(8, 8, tokens=1, dtype=F32), lambda: b.TokenLoss(8, 8, tokens=1, dtype=BF16, grad_dtype=F16), lambda: b.TokenLoss(8, 8, n_users=0, tokens=1)):
        refused(make, b.Co3Error)
    cuda = dict(device="cuda")
    e = b.Embedding(10, 8, n_users=2, tokens=4)
    k, table = torch.zeros((2, 4), dtype=torch.int64, **cuda), torch.zeros((10, 8), **cuda)
    d, dout = torch.zeros((2, 80), **cuda), torch.zeros((2, 4, 8), **cuda)
    refused(lambda: e.forward(k.float(), table))
    refused(lambda: e.forward(k.cpu(), table))
    refused(lambda: e.forward(k[0], table))
    refused(lambda: e.forward(torch.zeros((2, 5), dtype=torch.int64, **cuda), table), b.Co3Error)       # more than the handle was made for
    refused(lambda: e.forward(k, table.cpu()))
    refused(lambda: e.forward(k, table[:, :7]))
    refused(lambda: e.forward(k, table.double()))
    refused(lambda: e.forward(k, table, out=torch.zeros((2, 3, 8), **cuda)))
    refused(lambda: e.forward(k, table, out=torch.zeros((2, 1, 8), **cuda).expand(2, 4, 8)), b.Co3Error)
    refused(lambda: e.forward(k, table, out=torch.zeros((2, 4, 8), **cuda), out_dtype=BF16))
    refused(lambda: e.forward(k, table, scale=NAN), b.Co3Error)
    refused(lambda: e.backward(dout, k, d[:, :79]))
    refused(lambda: e.backward(dout, k, d[:1].expand(2, 80)), b.Co3Error)
    refused(lambda: e.backward(dout, k, torch.zeros((80, 2), **cuda).t()))
    refused(lambda: e.backward(dout[:, :3], k, d))
    refused(lambda: e.backward(dout.transpose(1, 2).contiguous().transpose(1, 2), k, d))
    n = b.LayerNorm(8, n_users=2)
    x, m = torch.zeros((2, 4, 8), **cuda), torch.zeros((2, 4), **cuda)
    refused(lambda: n.forward(x[:, :, :7]))
    refused(lambda: n.forward(x, torch.ones(7, **cuda)))
    refused(lambda: n.forward(x, torch.ones(8, **cuda), torch.ones(8, dtype=BF16, **cuda)))
    refused(lambda: n.forward(x, y=torch.zeros((2, 4, 8), dtype=BF16, **cuda)), b.Co3Error)
    refused(lambda: n.forward(x, mean=m.double()))
    refused(lambda: n.backward(x.bfloat16(), x, None, m, m), b.Co3Error)
    refused(lambda: n.backward(x, x, None, m[:, :3], m))
    refused(lambda: n.backward(x, x, None, m, m, dweight=torch.zeros((2, 9), **cuda)))
    t = b.TokenLoss(10, 8, n_users=2, tokens=4, top=3)
    h, w, lse = torch.zeros((2, 4, 8), dtype=BF16, **cuda), torch.zeros((10, 8), dtype=BF16, **cuda), torch.zeros((2, 4), **cuda)
    refused(lambda: t.loss(h.float(), w, k))
    refused(lambda: t.loss(h, w.half(), k))
    refused(lambda: t.loss(h, w[:9], k))
    refused(lambda: t.loss(h, torch.zeros(89, dtype=BF16, **cuda)[1:81].view(10, 8), k), b.Co3Error)      # not at a multiple of 16 bytes
    refused(lambda: t.loss(h, torch.zeros((10, 12), dtype=BF16, **cuda)[:, :8], k), b.Co3Error)
    refused(lambda: t.loss(h, w, k[:, :3]))
    refused(lambda: t.loss(h, w, k, lse=lse.double()))
    refused(lambda: t.loss_grad(h, w, k, lse[:1]))
    refused(lambda: t.loss_grad(h, w, k, lse, dweight=torch.zeros((2, 80), dtype=BF16, **cuda)), b.Co3Error)
    refused(lambda: t.loss_grad(h, w, k, lse, dhidden=torch.zeros((2, 4, 8), **cuda)), b.Co3Error)
    refused(lambda: t.loss_grad(h, w, k, lse, scale=math.inf), b.Co3Error)
    index, logits = torch.zeros((2, 4, 4), dtype=torch.int64, **cuda), torch.zeros((2, 4, 4), **cuda)
    refused(lambda: t.distill(h, w, index, logits), b.Co3Error)                                          # more entries than the handle was made for
    refused(lambda: t.distill(h, w, index[..., :3], logits))
    for tau in (0.0, -1.0, NAN, math.inf):
        refused(lambda: t.distill(h, w, index[..., :3].contiguous(), logits[..., :3].contiguous(), tau), b.Co3Error)
    torch.cuda.synchronize()
    assert t.status() == e.status() == (0, 0) and not d.any()
