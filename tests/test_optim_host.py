"""The host side of the optimizer calls, without a GPU: csrc/co3_optim.cu linked with a runtime of host memory (fake_cudart.c), in
which copies and fills are late as the real one may have them."""
import contextlib
import ctypes as C
import os
import subprocess
import time
import types

import numpy as np
import pytest
import torch

from paper_2203_09044_b200 import binding as b, build

TESTS = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    d = tmp_path_factory.mktemp("fake_cudart")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-fmad=false", "-Xcompiler", "-fPIC", "-I", build.INCLUDE,
                    "-I", build.CSRC, "-c", os.path.join(build.CSRC, "co3_optim.cu"), "-o", str(d / "optim.o")], check=True)
    subprocess.run(["gcc", "-O1", "-fPIC", "-c", os.path.join(TESTS, "fake_cudart.c"), "-o", str(d / "fake.o")], check=True)
    # symbolic: this process may hold the real runtime already
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", str(d / "optim.o"), str(d / "fake.o"), "-o", str(d / "fake.so")], check=True)
    L = C.CDLL(str(d / "fake.so"))
    L.co3_adamw_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(b.AdamwConfig)]
    L.co3_adamw_destroy.argtypes = [C.c_void_p]
    L.co3_adamw_status.argtypes = [C.c_void_p, C.POINTER(C.c_uint32), C.POINTER(C.c_uint64), C.POINTER(C.c_uint64), C.c_int32]
    L.co3_adamw_steps_export.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
    L.co3_adamw_steps_import.argtypes = [C.c_void_p, C.c_int64]
    L.fake_written.restype = C.c_long
    L.fake_allocated.restype = C.c_void_p
    return L


class Handle:
    """A handle of the library with the fake runtime."""

    def __init__(self, L, sizes=(1000, 5), betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, expect=b.OK):
        n = np.array(sizes, np.int64)
        cfg = b.AdamwConfig(len(n), n.ctypes.data_as(C.POINTER(C.c_int64)), None, b.F32, b.F32, b.NONE, 32, betas[0], betas[1], eps, weight_decay, 0, 0)
        self.L, self.h = L, C.c_void_p()
        assert L.co3_adamw_create(C.byref(self.h), C.byref(cfg)) == expect

    def __enter__(self):
        return self

    def __exit__(self, *_):
        self.L.fake_set_device(0)
        self.L.co3_adamw_destroy(self.h)

    def status(self, clear):
        f, e, s = C.c_uint32(), C.c_uint64(), C.c_uint64()
        return self.L.co3_adamw_status(self.h, C.byref(f), C.byref(e), C.byref(s), clear), (f.value, e.value, s.value)

    def steps(self):
        n = C.c_int64(-1)
        return self.L.co3_adamw_steps_export(self.h, C.byref(n)), n.value

    def set_steps(self, n):
        return self.L.co3_adamw_steps_import(self.h, n)


@pytest.mark.parametrize("sizes", [(1000, 5), (0,)])
def test_nothing_is_left_to_be_copied_when_a_call_returns(fake, sizes):
    """A step on a stream that does not wait for the null stream may follow at once."""
    with Handle(fake, sizes) as h:
        assert fake.fake_waiting() == 0
        assert h.set_steps(7) == b.OK and fake.fake_waiting() == 0
        assert h.status(clear=1) == (b.OK, (0, 0, 0)) and fake.fake_waiting() == 0
        assert h.steps() == (b.OK, 7)


def test_with_another_device_current_every_call_is_refused(fake):
    """As the norm and the step refuse it; a wait would be for the wrong device."""
    with Handle(fake) as h:
        assert h.set_steps(3) == b.OK
        fake.fake_set_device(1)
        before = fake.fake_calls()
        assert h.steps() == (b.EINVAL, -1) and h.set_steps(9) == b.EINVAL
        assert h.status(clear=0)[0] == b.EINVAL and h.status(clear=1)[0] == b.EINVAL
        assert fake.fake_calls() == before
        fake.fake_set_device(0)
        assert h.steps() == (b.OK, 3)


def test_clearing_the_status_writes_nothing_else(fake):
    """Not the step count, which another thread's step may have moved on since it was read."""
    with Handle(fake) as h:
        assert h.set_steps(3) == b.OK
        fake.fake_advance()
        assert h.status(clear=1) == (b.OK, (0, 0, 0))
        assert h.steps() == (b.OK, 4)


def test_setting_the_steps_leaves_the_status(fake):
    """... and the tickets, which a step that another thread has begun may hold."""
    with Handle(fake) as h:
        fake.fake_written()
        assert h.set_steps(3) == b.OK
        assert fake.fake_written() <= 40                # count, two powers, two corrections, key


@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.5, 0.75), (0.0, 0.3), (0.99, 0.0), (1.0 - 2.0 ** -53, 0.9999)])
def test_set_steps_leaves_the_powers_that_the_steps_would_have(fake, betas):
    """Products of 64 bits one after the other, to the last subnormal one and beyond."""
    with Handle(fake, betas=betas) as h:
        at = fake.fake_allocated()                        # count, then the two powers
        powers, t = [1.0, 1.0], 0
        for stop in (0, 1, 7, 60, 1074, 1080, 7200, 760_000, 1_000_001):
            while t < stop:
                powers = [powers[0] * betas[0], powers[1] * betas[1]]
                t += 1
            assert h.set_steps(stop) == b.OK
            assert C.c_int64.from_address(at).value == stop
            assert [x.hex() for x in (C.c_double * 2).from_address(at + 8)] == [x.hex() for x in powers], stop


def test_set_steps_far_into_a_run_is_quick(fake):
    """The powers of usual betas stop at a subnormal number that a product no longer changes: 6 s of products of such for 2^26 steps if
    one goes on, 2 ms until then."""
    with Handle(fake) as h:
        begin = time.process_time()
        assert h.set_steps(1 << 26) == b.OK
        assert time.process_time() - begin < 1.0


def test_numbers_that_32_bits_cannot_hold_are_refused(fake):
    """An eps that would be zero there makes 0 / 0 of an element without a gradient, a learning rate or decay that would be infinite no
    numbers of all weights."""
    least = 2.0 ** -126
    for kw in (dict(eps=1e-50), dict(eps=1e39), dict(eps=2.0 ** 126 * 1.001), dict(eps=least / 1.001, betas=(0.9, 0.0)), dict(eps=least * 9.9, betas=(0.9, 0.99)),
               dict(weight_decay=1e39)):
        Handle(fake, expect=b.EINVAL, **kw)
    for kw in (dict(eps=0.0), dict(eps=least, betas=(0.9, 0.0)), dict(eps=least * 10.1, betas=(0.9, 0.99)), dict(eps=1e-30), dict(eps=2.0 ** 126), dict(weight_decay=1e38)):
        with Handle(fake, **kw):
            pass


# ---- the Python binding, with tensors of the host in the place of the device's ----------------------------------------------
STREAM = types.SimpleNamespace(cuda_stream=0)


class Library:
    """The library with the fake runtime; `steps` has the arguments of each co3_adamw_step."""

    def __init__(self, L):
        self.L, self.steps, self.co3_strerror = L, [], b.lib().co3_strerror
        for name in b.EXPORTS:
            if "adamw" in name or name == "co3_grad_norm":
                getattr(L, name).restype, getattr(L, name).argtypes = getattr(b.lib(), name).restype, getattr(b.lib(), name).argtypes

    def __getattr__(self, name):
        return getattr(self.L, name)

    def co3_adamw_step(self, handle, weights, grads, copies, state, *rest):
        self.steps.append((weights, grads, copies, state))
        return self.L.co3_adamw_step(handle, weights, grads, copies, state, *rest)


@pytest.fixture
def host(fake, monkeypatch):
    """A place to run the binding in: `library`, `inside` (whether torch.cuda.stream is in force), `events`."""
    place = types.SimpleNamespace(library=Library(fake), inside=False, events=[])
    create = b.GradNorm._create

    def create_here(self, *a, **k):
        create(self, *a, **k)
        self.device, self._current_stream = torch.device("cpu"), lambda: 0

    @contextlib.contextmanager
    def in_stream(stream):
        assert stream is STREAM
        place.inside = True
        yield
        place.inside = False
    monkeypatch.setattr(b, "_lib", place.library)
    monkeypatch.setattr(b.GradNorm, "_create", create_here)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "stream", in_stream)
    current = types.SimpleNamespace(cuda_stream=0, synchronize=lambda: place.events.append("synchronize"))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: place.events.append(("record", t.data_ptr(), s)))
    place.current = current
    return place


def test_outputs_that_a_call_makes_for_a_stream_come_from_its_memory(host, monkeypatch):
    """Memory of the current stream may still be in use by work that waits there; and what was made for the other stream may be in use
    on the current one when it is given back."""
    opt = b.AdamW([torch.ones(300)], state_bits=8)
    made, empty_of = [], torch.empty

    def empty(*a, **k):
        made.append((empty_of(*a, **k), host.inside))
        return made[-1][0]
    monkeypatch.setattr(torch, "empty", empty)
    g = [torch.ones(300)]
    info = opt.grad_norm(g, stream=STREAM)
    assert [i for _, i in made] == [True] and info is made[0][0]
    assert ("record", info.data_ptr(), host.current) in host.events and ("record", info.data_ptr(), STREAM) in host.events
    made.clear()
    values = opt.state_values(stream=STREAM)
    assert [i for _, i in made] == [True, True]
    for v, (m, _) in zip(values, made):
        assert v is m and ("record", v.data_ptr(), host.current) in host.events and ("record", v.data_ptr(), STREAM) in host.events
    made.clear()
    opt.grad_norm(g)
    opt.state_values()
    assert [i for _, i in made] == [False] * 3


def test_a_new_optimizer_s_moments_are_zero_for_every_stream(host):
    """The fill is waited for, as what co3_adamw_create copies is: the first step may be on another stream."""
    opt = b.AdamW([torch.ones(300)])
    assert host.events == ["synchronize"]
    host.events.clear()
    b.AdamW([torch.ones(300)], state=dict(m=opt.m, v=opt.v))
    assert host.events == []


def pointers(address, n):
    return list((C.c_void_p * n).from_address(address))


def test_weights_copies_and_moments_that_are_given_other_storage(host):
    """Each step takes them where they are then, not where they were when the optimizer was made."""
    p, q = torch.nn.Parameter(torch.ones(300)), torch.nn.Parameter(torch.ones(5))
    copies = [torch.zeros(300, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.bfloat16)]
    opt = b.AdamW([p, q], copies=copies)
    grads = opt.bind_grads([torch.ones(300), torch.ones(5)])
    seen = host.library.steps
    kept = []                                            # so that no storage can come back at its old place

    def step():
        opt.step(grads)
        weights, _, c, state = seen[-1]
        m, v = (C.c_void_p * 2).from_address(state)
        assert pointers(weights, 2) == [p.data_ptr(), q.data_ptr()] and pointers(c, 2) == [c.data_ptr() for c in copies]
        assert (m, v) == (opt.m.data_ptr(), opt.v.data_ptr())
    step()
    for change in (lambda: setattr(p, "data", torch.zeros(300)), lambda: setattr(copies[1], "data", torch.ones(5, dtype=torch.bfloat16)),
                   lambda: setattr(opt, "m", torch.ones(3, 256)), lambda: setattr(opt, "v", torch.ones(3, 256))):
        before = [t.data_ptr() for t in (p, q, *copies, opt.m, opt.v)]
        kept.append([t.detach() for t in (p, q, *copies, opt.m, opt.v)])
        change()
        assert before != [t.data_ptr() for t in (p, q, *copies, opt.m, opt.v)]
        step()
    n = len(seen)
    for word, change, back in (("300 elements", lambda: setattr(p, "data", torch.zeros(299)), lambda: setattr(p, "data", torch.zeros(300))),
                               ("one piece", lambda: setattr(q, "data", torch.zeros(10)[::2]), lambda: setattr(q, "data", torch.zeros(5)))):
        change()
        with pytest.raises(ValueError, match=word):
            opt.step(grads)
        assert len(seen) == n
        back()
    step()
    with pytest.raises(ValueError, match="v: 768"):
        opt.v = torch.zeros(2, 256)
    step()
    with pytest.raises(AttributeError):
        opt.m_exp
    before = opt.m.data_ptr(), opt.v.data_ptr()          # what one reads is not the optimizer's own object
    opt.m.set_(torch.ones(3, 256))
    opt.v.data = torch.ones(3, 256)
    assert (opt.m.data_ptr(), opt.v.data_ptr()) == before
    step()
    given = dict(m=torch.ones(3, 256), v=torch.ones(3, 256))
    kept.append([t.detach() for t in given.values()])
    opt = b.AdamW([p, q], copies=copies, state=given)
    grads = opt.bind_grads([torch.ones(300), torch.ones(5)])
    given["m"].set_(torch.ones(3, 256))
    assert opt.m.data_ptr() == kept[-1][0].data_ptr() and opt.v.data_ptr() == given["v"].data_ptr()
    step()


def test_views_of_a_row_that_is_given_other_memory(host):
    """One of them is looked at, for all have the row's storage."""
    row, other = torch.ones(1000), torch.nn.Parameter(torch.ones(4))
    opt = b.AdamW([row[:300], other, row[300:900], row[900:]])
    grads = opt.bind_grads([torch.ones(n) for n in (300, 4, 600, 100)])
    seen, kept = host.library.steps, []
    assert len(opt._written) == 2                        # the row and the other one
    for change in (lambda: None, lambda: row.untyped_storage().resize_(1 << 20), lambda: setattr(other, "data", torch.zeros(4))):
        kept.append((row.clone(), other.detach()))
        change()
        opt.step(grads)
        assert pointers(seen[-1][0], 4) == [row.data_ptr(), other.data_ptr(), row[300:].data_ptr(), row[900:].data_ptr()]
    version = row._version
    opt.step(grads)
    assert row._version == version + 1


def test_gradients_bound_before_weights_took_another_order_are_looked_at_again(host):
    p = torch.nn.Parameter(torch.ones(4, 3, 2, 2))
    opt = b.AdamW([p])
    g = torch.ones(4, 3, 2, 2)
    bound = opt.bind_grads([g])
    opt.step(bound)
    p.data = torch.ones(4, 3, 2, 2).contiguous(memory_format=torch.channels_last)
    with pytest.raises(ValueError, match="another order"):
        opt.step(bound)
    bound = opt.bind_grads([g.contiguous(memory_format=torch.channels_last)])
    opt.step(bound)
    assert len(host.library.steps) == 2


def test_values_of_moments_that_are_given_other_storage(host, monkeypatch):
    opt = b.AdamW([torch.ones(300)], state_bits=8)
    seen = []
    monkeypatch.setattr(Library, "co3_adamw_values", lambda self, h, state, *rest: seen.append(pointers(state, 4)) or b.OK, raising=False)
    for name in ("m", "v", "m_exp", "v_exp"):
        setattr(opt, name, getattr(opt, name).clone())
        opt.state_values()
        assert seen[-1] == [getattr(opt, k).data_ptr() for k in ("m", "v", "m_exp", "v_exp")]
    opt.m.set_(opt.m.clone())
    opt.state_values()
    assert seen[-1][0] == opt.m.data_ptr() == seen[-2][0]


def test_tensors_that_share_memory_are_refused(host):
    """Two warps would write the same elements."""
    row = torch.ones(1000)
    half = torch.zeros(1000, dtype=torch.bfloat16)
    for params, copies, word in (([row, row], None, "weights 0 and weights 1"), ([row[:600], row[500:]], None, "weights 0 and weights 1"),
                                 ([row[500:], torch.ones(3), row[:501]], None, "weights 2 and weights 0"),
                                 ([row[:500], row[500:]], [half[:500], half[499:999]], "copies 0 and copies 1"),
                                 ([row[:500]], [row[250:500].view(torch.bfloat16)], "weights 0 and copies 0")):
        with pytest.raises(ValueError, match=word):
            b.AdamW(params, copies=copies)
    m, e = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, dtype=torch.uint8)
    for state, word in ((dict(m=m, v=m, m_exp=e, v_exp=e.clone()), "m and v"), (dict(m=m, v=m.clone(), m_exp=e, v_exp=e), "m_exp and v_exp")):
        with pytest.raises(ValueError, match=word):
            b.AdamW([row], state_bits=8, state=state)
    with pytest.raises(ValueError, match="weights 0 and m"):
        big = torch.zeros(4, 256)
        b.AdamW([big.view(-1)[:1000]], state=dict(m=big, v=torch.zeros(4, 256)))
    # neighbours, empty tensors anywhere, and gradients that share memory with one another are fine
    opt = b.AdamW([row[:500], row[500:], row[200:200], row[0:0]])
    opt.step([row.clone()[:500]] * 2 + [row[0:0]] * 2)
    with pytest.raises(ValueError, match="m and v"):
        opt.v = opt.m
    p = [torch.nn.Parameter(torch.ones(500)) for _ in range(2)]
    opt = b.AdamW(p)
    p[1].data = p[0].data
    with pytest.raises(ValueError, match="weights 0 and weights 1"):
        opt.step([row[:500]] * 2)


def test_autograd_sees_that_a_step_changed_weights_and_copies(host):
    p, row = torch.nn.Parameter(torch.ones(300)), torch.ones(600)
    copies = [torch.ones(300, dtype=torch.bfloat16), torch.ones(300, dtype=torch.bfloat16), torch.ones(300, dtype=torch.bfloat16)]
    opt = b.AdamW([p, row[:300], row[300:]], copies=copies)
    bound = opt.bind_grads([torch.ones(300)] * 3)
    x = torch.ones(300, requires_grad=True)
    losses = [(x * p).sum(), (x * row[:300]).sum(), (x * copies[2].float()).sum(), (x.bfloat16() * copies[2]).sum()]
    before = [p._version, row._version, copies[0]._version]
    opt.step(bound)
    assert all(now > then for now, then in zip([p._version, row._version, copies[0]._version], before))
    for loss, stale in zip(losses, (True, True, False, True)):
        if stale:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
        else:
            loss.backward()
    p.data = torch.ones(300)
    before = p._version
    opt.step(bound)
    assert p._version > before
    with pytest.raises(b.Co3Error):
        opt.step(bound, lr=float("nan"))
    assert p._version == before + 1
    with torch.inference_mode():                         # has no counter
        w = torch.ones(5)
    b.AdamW([w]).step([torch.ones(5)])


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_values_go_to_the_one_output_that_is_given(host, monkeypatch, kind):
    """... and the other is made to match it."""
    opt = b.AdamW([torch.ones(300)], state_bits=8)
    seen = []
    monkeypatch.setattr(Library, "co3_adamw_values", lambda self, h, state, m, v, code, s: seen.append((m, v, code)) or b.OK, raising=False)
    mine = torch.zeros(opt.n_blocks, 256, dtype=kind)
    for which in (0, 1):
        out = opt.state_values(**{("m_out", "v_out")[which]: mine})
        assert out[which] is mine and out[1 - which] is not mine and out[1 - which].dtype == kind and out[1 - which].shape == mine.shape
        assert seen[-1] == (out[0].data_ptr(), out[1].data_ptr(), b._type_code(kind))
    assert [t.dtype for t in opt.state_values()] == [torch.bfloat16] * 2
    with pytest.raises(ValueError, match="v_out"):
        opt.state_values(mine, mine.view(torch.int16 if kind == torch.bfloat16 else torch.int32))


def test_a_learning_rate_that_32_bits_cannot_hold_is_refused(host):
    opt = b.AdamW([torch.ones(300)])
    for lr in (1e39, -1e39, float("inf"), float("nan")):
        with pytest.raises(b.Co3Error) as e:
            opt.step([torch.ones(300)], lr=lr)
        assert e.value.code == b.EINVAL
    for lr in (1e38, -1e38, 0.0):
        opt.step([torch.ones(300)], lr=lr)
