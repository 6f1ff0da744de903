"""The host code of a network and of an AdamW list on a CUDA runtime in host memory (fake_runtime.cpp): allocations that fail
part of the way (a call that fails leaves the network as it was, its captured step included: nothing that a later step
launches or replays names memory that is gone), copies that land late, and two devices."""
import ctypes as C
import os
import subprocess

import pytest

from paper_1712_04432_b200 import build, mbd

HERE = os.path.dirname(os.path.abspath(__file__))
CUDA = os.path.dirname(os.path.dirname(build._nvcc())) or "/usr/local/cuda"
ETA = 0.01


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    """net.cu and adamw.cu over the fake runtime."""
    out = tmp_path_factory.mktemp("fake")
    std = ["-std=c++17", "-fPIC", "-fvisibility=hidden", "-I", os.path.join(CUDA, "include"), "-I", build.CSRC]
    run = lambda *cmd: subprocess.run(cmd, check=True, capture_output=True, text=True, timeout=300)  # noqa: E731
    run("g++", *std, "-x", "c++", "-c", os.path.join(build.CSRC, "net.cu"), "-o", str(out / "net.o"))
    run("g++", *std, "-c", os.path.join(HERE, "fake_runtime.cpp"), "-o", str(out / "fake.o"))
    run(build._nvcc(), "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-Xcompiler", "-fPIC,-fvisibility=hidden",
        "-c", os.path.join(build.CSRC, "adamw.cu"), "-o", str(out / "adamw.o"))
    run("g++", "-shared", "-Wl,-Bsymbolic", "-o", str(out / "libfake.so"), *(str(out / o) for o in ("net.o", "adamw.o", "fake.o")))
    lib = C.CDLL(str(out / "libfake.so"))
    vp, i32, i64 = C.c_void_p, C.c_int, C.c_int64
    for name in ("mbd_net_create", "mbd_net_destroy", "mbd_train_step", "mbd_forward", "mbd_backward", "mbd_sgd_step", "mbd_enable_adamw",
                 "mbd_enable_master_weights", "mbd_enable_momentum", "mbd_get_tensor", "mbd_adamw_create", "mbd_adamw_destroy", "mbd_adamw_step"):
        getattr(lib, name).argtypes = getattr(mbd.lib(), name).argtypes
    lib.mbd_enable_master_weights.argtypes = [vp]
    lib.mbd_enable_momentum.argtypes = [vp, C.c_float]
    lib.mbd_adamw_get_steps.argtypes, lib.mbd_adamw_set_steps.argtypes = [vp, C.POINTER(i64)], [vp, i64]
    lib.fake_violations.restype = lib.fake_adamw_launches.restype = i64
    lib.fake_malloc.restype, lib.fake_malloc.argtypes, lib.fake_free.argtypes = vp, [C.c_size_t], [vp]
    lib.fake_fail_in.argtypes, lib.fake_set_device.argtypes = [i32], [i32]
    yield lib
    assert lib.fake_blocks() == 0 and lib.fake_violations() == 0


class Net:
    """Two fully connected layers with biases on a stream that can be captured, and a batch."""

    def __init__(self, L, dtype=mbd.F32):
        self.L, self.h = L, C.c_void_p()
        layers = (mbd.Layer * 2)(*mbd.fc_layers((16, 24, 8), bias=True))
        assert L.mbd_net_create(layers, 2, 8, 1, 1, dtype, mbd.LOSS_SOFTMAX_CE, 0, 0x5000, C.byref(self.h)) == mbd.OK
        self.X, self.labels = C.create_string_buffer(8 * 16 * 4), C.create_string_buffer(8 * 4)

    def step(self):
        """One captured step; returns how many AdamW launches it made."""
        before = self.L.fake_adamw_launches()
        assert self.L.mbd_train_step(self.h, C.addressof(self.X), C.addressof(self.labels), ETA, None) == mbd.OK
        return self.L.fake_adamw_launches() - before

    def adamw(self, bits=32):
        return self.L.mbd_enable_adamw(self.h, 0.9, 0.999, 1e-8, 0.0, bits)

    def moments(self):
        """Whether the moments of the first layer can be read (those in 32 bits can)."""
        got = C.create_string_buffer(16 * 24 * 4)
        return self.L.mbd_get_tensor(self.h, mbd.T_ADAM_M, 0, C.addressof(got), len(got)) == mbd.OK

    def masters(self):
        """How many of the layers have a master that can be read."""
        got = C.create_string_buffer(16 * 24 * 4)
        return sum(self.L.mbd_get_tensor(self.h, mbd.T_MASTER, i, C.addressof(got), n * 4) == mbd.OK for i, n in enumerate((16 * 24, 24 * 8)))

    def close(self):
        assert self.L.mbd_net_destroy(self.h) == mbd.OK


def failing(L, call, most=64):
    """`call` with its first, second, .. allocation failing, until it needs no more; yields after each failure."""
    for n in range(most):
        L.fake_fail_in(n)
        status = call()
        L.fake_fail_in(-1)
        if status == mbd.OK:
            assert n > 0                                         # it did allocate
            return
        assert status == mbd.E_ALLOC
        yield n
    raise AssertionError("never enough memory")


@pytest.mark.parametrize("old,new", [(32, 8), (8, 32), (32, 32), (8, 8)])
def test_adamw_with_other_moments_that_do_not_fit(L, old, new):
    net = Net(L)
    assert net.adamw(old) == mbd.OK and net.step() == 1 and net.step() == 1
    held, bad = L.fake_blocks(), L.fake_violations()
    for _ in failing(L, lambda: net.adamw(new)):
        # as it was: the method, its moments, the captured step
        assert net.step() == 1 and net.step() == 1
        assert L.fake_violations() == bad and L.fake_blocks() == held
        assert net.moments() == (old == 32)
    assert net.step() == 1 and net.step() == 1 and L.fake_violations() == bad and net.moments() == (new == 32)
    net.close()


def test_adamw_that_does_not_fit_after_momentum(L):
    net = Net(L)
    assert L.mbd_enable_momentum(net.h, 0.9) == mbd.OK and net.step() == 0
    held, bad = L.fake_blocks(), L.fake_violations()
    for _ in failing(L, lambda: net.adamw(8)):
        assert net.step() == 0 and L.fake_violations() == bad and L.fake_blocks() == held
    assert net.step() == 1
    net.close()


@pytest.mark.parametrize("method", ["none", "adamw32", "adamw8", "momentum"])
def test_masters_that_do_not_fit(L, method):
    net = Net(L, mbd.BF16)
    if method == "momentum":
        assert L.mbd_enable_momentum(net.h, 0.9) == mbd.OK
    if method.startswith("adamw"):
        assert net.adamw(int(method[5:])) == mbd.OK
    launches = int(method.startswith("adamw"))
    named = lambda: L.fake_adamw_masters() if launches else None  # noqa: E731
    assert net.step() == launches and net.masters() == 0 and not named()
    held, bad = L.fake_blocks(), L.fake_violations()
    for _ in failing(L, lambda: L.mbd_enable_master_weights(net.h)):
        assert net.step() == launches and net.masters() == 0 and not named()
        assert L.fake_violations() == bad and L.fake_blocks() == held
    # now there are masters, and they are what is updated
    assert net.masters() == 2 and L.mbd_enable_master_weights(net.h) == mbd.OK
    assert net.step() == launches and named() in (2, None) and L.fake_violations() == bad
    net.close()


@pytest.mark.parametrize("before", ["none", "adamw"])
def test_velocities_that_do_not_fit(L, before):
    net = Net(L)
    if before == "adamw":
        assert net.adamw() == mbd.OK
    launches = int(before == "adamw")
    assert net.step() == launches
    held, bad = L.fake_blocks(), L.fake_violations()
    for _ in failing(L, lambda: L.mbd_enable_momentum(net.h, 0.9)):
        assert net.step() == launches and L.fake_violations() == bad and L.fake_blocks() == held
    # weights and biases of every layer have a velocity
    assert net.step() == 0 and L.fake_violations() == bad
    assert L.mbd_enable_momentum(net.h, 0.5) == mbd.OK and net.step() == 0 and L.fake_violations() == bad
    net.close()


def adamw_list(L, n=300, steps=0):
    """A list of one tensor, and its buffers."""
    at = [L.fake_malloc(n * 4) for _ in range(4)]
    table = (mbd.AdamWTensor * 1)(mbd.AdamWTensor(at[0], None, at[1], at[2], at[3], None, None, n, 0.0, 0, 0, 0))
    h = C.c_void_p()
    assert L.mbd_adamw_create(table, 1, 32, 0.9, 0.999, 1e-8, steps, C.byref(h)) == mbd.OK
    return h, at


def gone(L, h, buffers):
    assert L.mbd_adamw_destroy(h) == mbd.OK
    for p in buffers:
        L.fake_free(p)


def test_a_step_on_any_stream_may_follow_creation_and_set_steps(L):
    # a copy from pageable host memory may return before it has landed, and only the stream it went through waits for that: what a list
    # puts on the device has to be there when the call returns, since the step goes to a stream of the caller's
    L.fake_late_copies(1)
    try:
        h, buffers = adamw_list(L, steps=5)
        assert L.fake_copies_under_way() == 0
        assert L.mbd_adamw_set_steps(h, 7) == mbd.OK and L.fake_copies_under_way() == 0
        steps = C.c_int64()
        assert L.mbd_adamw_get_steps(h, C.byref(steps)) == mbd.OK and steps.value == 7
        gone(L, h, buffers)
    finally:
        L.fake_late_copies(0)


def test_the_step_count_from_another_current_device(L):
    # steps under way are waited for on the list's device, whichever is current, and that stays current
    h, buffers = adamw_list(L)
    steps = C.c_int64()
    for _ in range(3):
        assert L.mbd_adamw_step(h, 0.1, 1.0, 0x5000) == mbd.OK
    L.fake_set_device(1)
    try:
        assert L.mbd_adamw_step(h, 0.1, 1.0, 0x5000) == mbd.E_STATE
        assert L.mbd_adamw_get_steps(h, C.byref(steps)) == mbd.OK and steps.value == 3 and L.fake_device() == 1
        L.fake_set_device(0)
        assert L.mbd_adamw_step(h, 0.1, 1.0, 0x5000) == mbd.OK
        L.fake_set_device(1)
        assert L.mbd_adamw_set_steps(h, 10) == mbd.OK and L.fake_device() == 1      # after the step under way, not before it
        assert L.mbd_adamw_get_steps(h, C.byref(steps)) == mbd.OK and steps.value == 10
    finally:
        L.fake_set_device(0)
    gone(L, h, buffers)
