"""The host side of the language-model operators, without a GPU: their files linked with a runtime of host memory that writes launches down
(fake_cudart_lm.c).  What is refused, that a refused call launches nothing, and that launches and scratch fit what is asked for."""
import concurrent.futures
import ctypes as C
import os
import subprocess

import pytest

from paper_2203_09044_b200 import binding as b, build

TESTS = os.path.dirname(os.path.abspath(__file__))
NAMES = ("embed", "layernorm", "token_loss")


class Launch(C.Structure):
    _fields_ = [("grid", C.c_uint * 3), ("block", C.c_uint * 3), ("shared", C.c_ulonglong), ("arg", C.c_ubyte * 512)]


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    d = tmp_path_factory.mktemp("fake_lm")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")

    def compile_one(name):
        # for the host alone: the kernels stay virtual code
        subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O0", "-fmad=false", "-Xcompiler", "-fPIC", "-I", build.INCLUDE, "-I", build.CSRC,
                        "-c", os.path.join(build.CSRC, f"co3_{name}.cu"), "-o", str(d / f"{name}.o")], check=True)

    with concurrent.futures.ThreadPoolExecutor(3) as pool:
        list(pool.map(compile_one, NAMES))
    subprocess.run(["gcc", "-O1", "-fPIC", "-w", "-I", TESTS, "-c", os.path.join(TESTS, "fake_cudart_lm.c"), "-o", str(d / "fake.o")], check=True)
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", *[str(d / f"{n}.o") for n in NAMES], str(d / "fake.o"), "-o", str(d / "fake.so")], check=True)
    L = C.CDLL(str(d / "fake.so"))
    real = b.lib()
    for name in b.EXPORTS:
        if any(f"co3_{n}_" in name for n in NAMES):
            f = getattr(L, name)
            f.argtypes, f.restype = getattr(real, name).argtypes, getattr(real, name).restype
    L.fake_launch.restype = C.POINTER(Launch)
    L.fake_allocated_bytes.restype = C.c_ulonglong
    L.fake_allocated.restype = C.c_void_p
    return L


@pytest.fixture(autouse=True)
def clean(fake):
    fake.fake_forget()
    fake.fake_set_device(0)
    fake.fake_fail_malloc(0)
    yield
    fake.fake_set_device(0)


A = 1 << 20                                               # an address that nothing is read from


def array(type_=b.F32, us=0, ts=0, data=A):
    return b.Array(data, type_, 0, us, ts)


def tokens(n=0, top=1, type_=b.I64, data=A):
    return b.Tokens(data, type_, top, n * top, top)


def grad(type_=b.F32, stride=0, accumulate=0, data=A):
    return b.ParamGrad(data, type_, accumulate, stride)


def launches(fake):
    out = [fake.fake_launch(i).contents for i in range(fake.fake_seen())]
    for x in out:
        assert all(1 <= v for v in [*x.grid, *x.block]) and x.grid[0] < 2 ** 31 and x.grid[1] < 2 ** 16 and x.grid[2] < 2 ** 16
        assert x.block[0] * x.block[1] * x.block[2] <= 1024 and x.shared <= 232448
    fake.fake_forget()
    return out


class Made:
    def __init__(self, fake, name, *args, expect=b.OK):
        self.fake, self.name, self.h = fake, name, C.c_void_p()
        assert getattr(fake, f"co3_{name}_create")(C.byref(self.h), *args) == expect

    def __enter__(self):
        return self

    def __exit__(self, *_):
        self.fake.fake_set_device(0)
        getattr(self.fake, f"co3_{self.name}_destroy")(self.h)

    def __call__(self, what, *args, expect=b.OK):
        rc = getattr(self.fake, f"co3_{self.name}_{what}")(self.h, *args)
        assert rc == expect, (what, rc)
        seen = launches(self.fake)
        if expect != b.OK:
            assert not seen, "a refused call launches nothing"
        return seen


# ---- embedding ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("args", [(0, 8, 1, 1), (8, 0, 1, 1), (8, 8, 0, 1), (8, 8, 1, -1), (1 << 31, 8, 1, 1), (8, 1 << 31, 1, 1), (8, 8, 1 << 16, 1), (8, 8, 4, 1 << 30),
                                  (1 << 30, 1 << 20, 1, 1)])
def test_embedding_shapes_that_are_refused(fake, args):
    Made(fake, "embed", *args, expect=b.EINVAL)


@pytest.mark.parametrize("users,n,vocab,dim", [(1, 1, 1, 1), (3, 5, 7, 9), (2, 4097, 50257, 768), (8, 2000, 32000, 768), (1, 1 << 20, 131072, 4096), (65535, 2, 100, 8), (1, 100, (1 << 31) - 1, 1)])
def test_embedding_launches(fake, users, n, vocab, dim):
    with Made(fake, "embed", vocab, dim, users, n) as e:
        for kind in (b.F32, b.BF16, b.F16):
            assert len(e("forward", tokens(n), n, A, kind, 1.0, array(b.BF16, n * dim, dim), None)) == 1
            for stride in (vocab * dim, vocab * dim + 3):
                for accumulate in (0, 1):
                    if users * vocab * dim < 1 << 40:
                        seen = e("backward", array(kind, n * dim, dim), tokens(n), n, 1.0, grad(kind, stride, accumulate), None)
                        assert 2 <= len(seen) <= 3
        assert not e("forward", tokens(0, data=None), 0, A, b.F32, 1.0, array(data=None), None)
        assert len(e("backward", array(data=None), tokens(0, data=None), 0, 1.0, grad(b.F32, vocab * dim), None)) == 1          # zeros
        assert not e("backward", array(data=None), tokens(0, data=None), 0, 1.0, grad(b.F32, vocab * dim, 1), None)


@pytest.mark.parametrize("users,n,dim,kind,at,grad_kind,columns", [
    (1, 20001, 1024, b.BF16, 0, b.BF16, 256), (1, 20001, 1024, b.F32, 4, b.F32, 256), (2, 10000, 1032, b.F16, 8, b.F32, 256),       # eight neighbours a lane
    (1, 20001, 1032, b.BF16, 1, b.F32, 128), (2, 10000, 1028, b.F32, 0, b.BF16, 128), (1, 20001, 1028, b.F16, 3, b.F16, 128),       # four
    (1, 20001, 1026, b.BF16, 0, b.BF16, 64), (1, 2000, 1024, b.BF16, 0, b.BF16, 64), (1, 20001, 264, b.BF16, 0, b.BF16, 64),        # two
    (1, 20001, 1027, b.BF16, 0, b.BF16, 64)])                                                                                       # one and one
def test_columns_that_a_warp_of_the_embedding_gradient_takes(fake, users, n, dim, kind, at, grad_kind, columns):
    """The wider ways are taken where rows begin at their multiples and 2368 warps are left: the sizes of the tests that compare their results."""
    vocab, width = 3001, 4 if grad_kind == b.F32 else 2
    with Made(fake, "embed", vocab, dim, users, n) as e:
        seen = e("backward", array(kind, n * dim, dim), tokens(n), n, 1.0, grad(grad_kind, (at + vocab * dim + 9) // 4 * 4, data=A + at * width), None)
        assert len(seen) == 3 and seen[1].grid[0] == (users * ((n + 31) // 32) * ((dim + columns - 1) // columns) + 7) // 8


def test_embedding_calls_that_are_refused(fake):
    with Made(fake, "embed", 100, 16, 2, 10) as e:
        good = [tokens(10), 10, A, b.F32, 1.0, array(b.F32, 160, 16), None]

        def bad(at, value):
            e("forward", *[value if i == at else x for i, x in enumerate(good)], expect=b.EINVAL)
        assert e("forward", *good)
        for at, value in [(0, None), (0, tokens(10, data=None)), (0, tokens(10, data=A + 4)), (0, tokens(10, type_=b.F32)), (0, tokens(10, top=2)), (1, -1), (1, 11), (2, None), (2, A + 2), (3, 7),
                          (4, float("nan")), (4, float("inf")), (5, None), (5, array(b.F32, 160, 15)), (5, array(b.F32, 16, 16)), (5, array(b.F32, 160, 16, A + 1)), (5, array(9, 160, 16)),
                          (5, array(b.F32, -160, 16))]:
            bad(at, value)
        back = [array(b.BF16, 160, 16), tokens(10), 10, 1.0, grad(b.F32, 1600), None]
        assert e("backward", *back)
        for at, value in [(0, None), (0, array(b.BF16, 160, 16, None)), (1, None), (2, 11), (3, float("nan")), (4, None), (4, grad(b.F32, 1599)), (4, grad(b.F32, 1600, data=A + 2)), (4, grad(5, 1600))]:
            e("backward", *[value if i == at else x for i, x in enumerate(back)], expect=b.EINVAL)
        fake.fake_set_device(1)
        e("forward", *good, expect=b.EINVAL)
        e("backward", *back, expect=b.EINVAL)
        assert fake.co3_embed_status(e.h, None, None, 0) == b.EINVAL
    fake.fake_fail_malloc(1)
    Made(fake, "embed", 100, 16, 2, 10, expect=b.ENOMEM)


# ---- layer norm ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("args", [(0, 1, 1e-5), (16385, 1, 1e-5), (8, 0, 1e-5), (8, 1 << 16, 1e-5), (8, 1, -1e-9), (8, 1, float("nan")), (8, 1, float("inf"))])
def test_layer_norm_shapes_that_are_refused(fake, args):
    Made(fake, "layernorm", *args, expect=b.EINVAL)


@pytest.mark.parametrize("dim", [1, 255, 256, 257, 768, 1000, 1024, 2048, 4096, 8192, 16384])
@pytest.mark.parametrize("users,n", [(1, 1), (1, 100_000), (3, 50), (1000, 7), (65535, 3)])
def test_layer_norm_launches_and_scratch(fake, dim, users, n):
    with Made(fake, "layernorm", dim, users, 1e-5) as h:
        scratch = fake.fake_allocated_bytes()
        for kind in (b.F32, b.BF16, b.F16):
            for stride in (dim, dim + 1):
                x = array(kind, n * stride, stride)
                assert len(h("forward", x, A, A, b.F32, n, x, A, A, None)) == 1
                seen = h("backward", x, x, A, b.F32, A, A, n, x, grad(b.F32, dim), None, None)
                slices = seen[0].grid[0]
                assert len(seen) == (1 if slices == 1 else 2) and seen[0].grid[1] == users
                if slices > 1:
                    assert users * slices * 2 * dim * 4 <= scratch
                assert len(h("backward", x, x, A, b.F32, A, A, n, x, None, None, None)) == 1
                assert not h("backward", x, x, A, b.F32, A, A, n, None, None, None, None)


def test_layer_norm_calls_that_are_refused(fake):
    with Made(fake, "layernorm", 16, 2, 1e-5) as h:
        x = array(b.F32, 160, 16)
        good = [x, A, A, b.F32, 10, x, A, A, None]
        assert h("forward", *good)
        for at, value in [(0, None), (0, array(b.F32, 160, 16, None)), (1, A + 2), (3, 7), (4, -1), (4, 1 << 31), (5, None), (5, array(b.BF16, 160, 16)), (5, array(b.F32, 0, 16)), (6, None), (7, A + 1)]:
            h("forward", *[value if i == at else v for i, v in enumerate(good)], expect=b.EINVAL)
        back = [x, x, A, b.F32, A, A, 10, x, grad(b.F32, 16), grad(b.F32, 16), None]
        assert h("backward", *back)
        for at, value in [(0, None), (0, array(b.BF16, 160, 16)), (1, None), (2, A + 1), (3, 9), (4, None), (5, A + 2), (6, -1), (7, array(b.F32, 160, 15)), (8, grad(b.F32, 15)), (9, grad(b.F32, 16, data=A + 1))]:
            h("backward", *[value if i == at else v for i, v in enumerate(back)], expect=b.EINVAL)
        fake.fake_set_device(1)
        h("forward", *good, expect=b.EINVAL)
        h("backward", *back, expect=b.EINVAL)
    fake.fake_fail_malloc(1)
    Made(fake, "layernorm", 16, 2, 1e-5, expect=b.ENOMEM)


def test_layer_norm_of_more_rows_than_a_product_of_64_bits_holds(fake):
    """n_tokens times 4 users is 4, or 0, in 64 bits."""
    x = array(b.F32, 16, 16)
    with Made(fake, "layernorm", 16, 4, 1e-5) as h:
        for n in ((1 << 62) + 1, 1 << 62):
            h("backward", x, x, A, b.F32, A, A, n, x, grad(b.F32, 16), None, None, expect=b.EINVAL)
            h("forward", x, A, A, b.F32, n, x, A, A, None, expect=b.EINVAL)


@pytest.mark.parametrize("what", ["x", "y", "dy", "dx", "dweight", "hidden", "targets", "teacher", "dhidden"])
def test_strides_whose_last_element_has_no_address(fake, what):
    """Strides of up to 2^46 elements were taken whatever their number: 2^18 of 2^45 wrap to a negative number of 64 bits, under which an array
    whose users all lie in one place looked like one whose users lie apart."""
    n, far = (1 << 18) + 1, 1 << 45
    with Made(fake, "layernorm", 16, 2, 1e-5) as h:
        x, wide = array(b.F32, 16 * n, 16), array(b.F32, 0, far)
        pick = lambda name, good=x: wide if name == what else good                                             # noqa: E731
        refused = b.EINVAL if what in ("x", "y", "dy", "dx") else b.OK
        if what in ("x", "y") or refused == b.OK:
            h("forward", pick("x"), A, A, b.F32, n, pick("y"), A, A, None, expect=refused)
        if what != "y":
            h("backward", pick("dy"), pick("x"), A, b.F32, A, A, n, pick("dx"), None, None, None, expect=refused)
    with Made(fake, "layernorm", 16, 65535, 1e-5) as h:
        x, far = array(b.F32, 16, 16), (1 << 46) // 65534 + 1
        h("backward", x, x, A, b.F32, A, A, 1, x, grad(b.F32, far if what == "dweight" else 16), None, None, expect=b.EINVAL if what == "dweight" else b.OK)
    with Made(fake, "token_loss", C.byref(config(n=3, users=2, top=2))) as h:
        far = (1 << 45) + 8
        x, t, lg = array(b.BF16, 3 * 64, 64), tokens(3, 2), array(b.F32, 6, 2)
        bad = {"hidden": array(b.BF16, 64, far), "targets": b.Tokens(A, b.I64, 2, 2, far), "teacher": array(b.F32, 2, far), "dhidden": array(b.BF16, 64, far)}
        args = {"hidden": x, "targets": t, "teacher": lg, "dhidden": x} | ({what: bad[what]} if what in bad else {})
        refused = b.EINVAL if what in bad else b.OK
        h("backward", args["hidden"], A, 64, args["targets"], args["teacher"], 2.0, 3, A, A, 1.0, args["dhidden"], grad(b.F32, 64000), None, expect=refused)
    with Made(fake, "embed", 100, 16, 2, 3) as e:
        x, t = array(b.F32, 48, 16), b.Tokens(A, b.I64, 1, 1, far) if what == "targets" else tokens(3)
        e("forward", t, 3, A, b.F32, 1.0, x, None, expect=b.EINVAL if what == "targets" else b.OK)
        e("backward", x, t, 3, 1.0, grad(b.F32, 1600), None, expect=b.EINVAL if what == "targets" else b.OK)


def test_a_gradient_of_2_to_64_elements(fake):
    with Made(fake, "token_loss", C.byref(config(vocab=1 << 30, dim=1 << 20, n=0, users=1 << 14))) as h:
        h("backward", array(b.BF16, data=None), A, 1 << 20, tokens(0, data=None), None, 1.0, 0, None, None, 1.0, None, grad(b.F32, data=None), None, expect=b.EINVAL)


# ---- losses -------------------------------------------------------------------------------------------------------------------
def config(vocab=1000, dim=64, n=100, users=2, type_=b.BF16, grad_type=b.F32, top=1):
    return b.TokenLossConfig(vocab, dim, n, users, type_, grad_type, top)


@pytest.mark.parametrize("change", [dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(dim=0), dict(dim=12), dict(dim=4), dict(n=-1), dict(n=1 << 26), dict(users=0), dict(users=1 << 16), dict(type_=b.F32),
                                    dict(grad_type=b.F16), dict(grad_type=b.NONE), dict(top=0), dict(top=129)])
def test_loss_shapes_that_are_refused(fake, change):
    Made(fake, "token_loss", C.byref(config(**change)), expect=b.EINVAL)


class Entry(C.Structure):
    """What the kernel of the teacher's entries is given (EntryArgs)."""
    _fields_ = [("data", C.c_void_p), ("us", C.c_int64), ("ts", C.c_int64), ("wide", C.c_int), ("top", C.c_int), ("teacher", C.c_void_p), ("tu", C.c_int64), ("tt", C.c_int64), ("type", C.c_int),
                ("n_all", C.c_int64), ("tokens", C.c_uint32), ("vocab", C.c_int), ("tiles", C.c_int), ("inv_t", C.c_float),
                ("entry", C.c_void_p), ("q", C.c_void_p), ("constant", C.c_void_p), ("first", C.c_void_p), ("mass", C.c_void_p), ("status", C.c_void_p)]


@pytest.mark.parametrize("users,n,vocab,dim,top", [(1, 1, 1, 8, 1), (2, 100, 1000, 64, 1), (3, 65, 50257, 768, 64), (1, 8192, 131072, 4096, 128), (65535, 3, 100, 8, 2), (1, 60, 600_001, 8, 5)])
@pytest.mark.parametrize("type_,grad_type", [(b.BF16, b.F32), (b.F16, b.F16)])
def test_loss_launches_and_scratch(fake, users, n, vocab, dim, top, type_, grad_type):
    with Made(fake, "token_loss", C.byref(config(vocab, dim, n, users, type_, grad_type, top))) as h:
        base, size = fake.fake_allocated(), fake.fake_allocated_bytes()
        x, t = array(type_, n * dim, dim), tokens(n)
        first = 1 if users * n <= 8192 and users <= 256 else 2                  # launches that pack the tokens with a target
        assert len(h("forward", x, A, dim, t, None, 1.0, n, A, A, None)) == 2 + first
        for stride in (vocab * dim, vocab * dim + 1):
            seen = h("backward", x, A, dim, t, None, 1.0, n, A, A, 1.0, x, grad(grad_type, stride), None)
            other = 1 + first
            assert (len(seen) - other) % 3 == 0 and len(seen) >= other + 3
            assert len(h("backward", x, A, dim, t, None, 1.0, n, A, None, 1.0, x, None, None)) == other + 2 * (len(seen) - other) // 3
        kt, lg = tokens(n, top), array(b.F32, n * top, top)
        seen = h("forward", x, A, dim, kt, lg, 2.0, n, A, A, None)
        assert len(seen) == 3 + first
        e = Entry.from_buffer_copy(bytes(seen[0].arg))
        assert e.n_all == users * n and e.tiles == (vocab + 255) // 256 and e.top == top
        # each array ends before the next begins, and the last with the allocation
        ends = [(e.entry, 4 * e.n_all * top), (e.q, 4 * e.n_all * top), (e.constant, 4 * e.n_all), (e.first, e.n_all * e.tiles), (e.mass, e.n_all)]
        for (at, length), (following, _) in zip(ends, ends[1:] + [(base + size, 0)]):
            assert base <= at and at + length <= following
        assert not h("forward", array(type_, data=None), A, dim, tokens(0, data=None), None, 1.0, 0, None, None, None)
        assert h("backward", array(type_, data=None), A, dim, tokens(0, data=None), None, 1.0, 0, None, None, 1.0, None, grad(grad_type, vocab * dim), None)


def test_loss_calls_that_are_refused(fake):
    nan = float("nan")
    with Made(fake, "token_loss", C.byref(config(top=3))) as h:
        x = array(b.BF16, 6400, 64)
        good = [x, A, 64, tokens(100), None, 1.0, 100, A, A, None]
        assert h("forward", *good)
        for at, value in [(0, None), (0, array(b.F16, 6400, 64)), (0, array(b.BF16, 6400, 64, None)), (1, None), (1, A + 8), (2, 63), (2, 68), (3, None), (3, tokens(100, data=None)), (3, tokens(100, 2)),
                          (3, tokens(100, type_=0)), (5, 2.0), (6, -1), (6, 101), (7, None), (8, A + 2)]:
            h("forward", *[value if i == at else v for i, v in enumerate(good)], expect=b.EINVAL)
        soft = [x, A, 64, tokens(100, 3), array(b.F32, 300, 3), 2.0, 100, A, A, None]
        assert h("forward", *soft)
        for at, value in [(3, tokens(100, 4)), (3, tokens(100, 0)), (4, array(b.F32, 300, 3, None)), (4, array(8, 300, 3)), (5, 0.0), (5, -1.0), (5, nan), (5, float("inf")), (5, 1e-38)]:
            h("forward", *[value if i == at else v for i, v in enumerate(soft)], expect=b.EINVAL)
        back = [x, A, 64, tokens(100), None, 1.0, 100, A, A, 1.0, x, grad(b.F32, 64000), None]
        assert h("backward", *back)
        for at, value in [(0, None), (1, A + 2), (7, None), (7, A + 1), (8, A + 2), (9, nan), (9, float("inf")), (10, array(b.F32, 6400, 64)), (10, array(b.BF16, 6400, 63)), (11, grad(b.BF16, 64000)),
                          (11, grad(b.F32, 63999)), (11, grad(b.F32, 64000, data=None))]:
            h("backward", *[value if i == at else v for i, v in enumerate(back)], expect=b.EINVAL)
        assert not h("backward", *[None if i in (10, 11) else v for i, v in enumerate(back)])
        fake.fake_set_device(1)
        h("forward", *good, expect=b.EINVAL)
        h("backward", *back, expect=b.EINVAL)
        assert fake.co3_token_loss_status(h.h, None, None, 1) == b.EINVAL
    fake.fake_fail_malloc(1)
    Made(fake, "token_loss", C.byref(config()), expect=b.ENOMEM)


def test_a_scale_that_the_temperature_makes_infinite(fake):
    """c / tau of every token would be infinite or not a number, although scale and temperature are numbers that are taken."""
    with Made(fake, "token_loss", C.byref(config(top=3))) as h:
        x, g = array(b.BF16, 6400, 64), grad(b.F32, 64000)
        back = lambda tau, scale, rc: h("backward", x, A, 64, tokens(100, 3), array(b.F32, 300, 3), tau, 100, A, A, scale, x, g, None, expect=rc)     # noqa: E731
        for tau, scale, rc in ((1e-30, 1e9, b.EINVAL), (0.5, -3e38, b.EINVAL), (1e-30, 1e8, b.OK), (0.5, 1e38, b.OK), (1e30, -3e38, b.OK), (2.0, 0.0, b.OK)):
            back(tau, scale, rc)


def test_null_handles(fake):
    x, t, g = array(), tokens(1), grad()
    assert fake.co3_embed_forward(None, t, 1, A, 0, 1.0, x, None) == b.EINVAL and fake.co3_embed_backward(None, x, t, 1, 1.0, g, None) == b.EINVAL
    assert fake.co3_layernorm_forward(None, x, A, A, 0, 1, x, A, A, None) == b.EINVAL and fake.co3_layernorm_backward(None, x, x, A, 0, A, A, 1, x, g, g, None) == b.EINVAL
    assert fake.co3_token_loss_forward(None, x, A, 8, t, None, 1.0, 1, A, A, None) == b.EINVAL
    assert fake.co3_token_loss_backward(None, x, A, 8, t, None, 1.0, 1, A, A, 1.0, x, g, None) == b.EINVAL
    for n in NAMES:
        getattr(fake, f"co3_{n}_destroy")(None)
        assert getattr(fake, f"co3_{n}_launch_count")(None) == 0
    for n in ("embed", "token_loss"):
        assert getattr(fake, f"co3_{n}_status")(None, None, None, 0) == b.EINVAL
    for n, args in (("embed", (8, 8, 1, 1)), ("layernorm", (8, 1, 1e-5)), ("token_loss", (C.byref(config()),))):
        assert getattr(fake, f"co3_{n}_create")(None, *args) == b.EINVAL
