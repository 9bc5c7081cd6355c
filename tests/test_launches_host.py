"""The launches of mixtures and of the clipped training step, from the host's side: the library runs on a HIP runtime without a GPU
(fake_launches.cpp), each test in a process of its own."""
import ctypes
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)

from test_host_memory import Library  # noqa: E402

OK, ARGUMENT, SHAPE, WORKSPACE, HIP = 0, -1, -2, -4, -5
P = 1 << 20   # an address that is aligned and never read


def library(fake):
    L = Library(fake)
    for name in ("expert_placement_bytes", "expert_combine_workspace_bytes", "mlp_clipped_workspace_bytes"):
        getattr(L.lib, name).restype = ctypes.c_size_t
    return L


def refused_or_launched(L, call, refused):
    before = L.hip.fake_launches()
    rc = call()
    launched = L.hip.fake_launches() - before
    assert L.hip.fake_too_large() == 0, "a launch of more threads than there may be"
    if refused:
        assert rc == SHAPE and launched == 0, (rc, launched, L.lib.nerva_last_error())
        assert b"columns" in L.lib.nerva_last_error()
    else:
        assert rc == OK and launched > 0, (rc, L.lib.nerva_last_error())


def a_call_that_no_launch_holds_is_refused_before_the_first(L):
    """Columns and choices that the documented ranges allow, to both sides of 2^32 threads."""
    p = ctypes.c_void_p(P)
    f = ctypes.c_float

    def route(batch, experts, k, groups, top, flags=0, bias=False):
        return lambda: L.lib.expert_route(p, batch, p if bias else None, experts, batch, k, groups, top, flags, f(1), p, p, batch, None)

    def route_backward(batch, experts, k, flags):
        return lambda: L.lib.expert_route_backward(p, batch, p, p, batch, experts, batch, k, flags, f(1), p, batch, None)

    # a wave per column, 32 threads a column; a few experts more, 64
    refused_or_launched(L, route(1 << 27, 32, 1, 32, 1), True)
    refused_or_launched(L, route((1 << 27) - 32, 32, 1, 32, 1), False)
    refused_or_launched(L, route((1 << 27) - 31, 32, 1, 32, 1), True)
    refused_or_launched(L, route(1 << 26, 64 * 9, 1, 64, 1, bias=True), True)
    refused_or_launched(L, route((1 << 26) - 16, 64 * 9, 1, 64, 1, bias=True), False)
    # a lane per column, 16 threads a column
    for flags in (0, 1, 2):
        refused_or_launched(L, route(1 << 28, 128, 2, 1, 1, flags), True)
        refused_or_launched(L, route((1 << 28) - 64, 128, 2, 1, 1, flags), False)
    refused_or_launched(L, route((1 << 29) - 1, 8, 1, 1, 1), False)      # (few lists)
    for flags in (0, 1, 2):
        refused_or_launched(L, route_backward(1 << 28, 128, 1, flags), True)
        refused_or_launched(L, route_backward((1 << 28) - 64, 128, 1, flags), False)
        refused_or_launched(L, route_backward((1 << 30) - 64, 8, 1, flags), False)      # (four threads a column)

    def place(batch, experts, k, capacity):
        n = L.lib.expert_placement_bytes(experts, batch, k)
        assert n > 0
        return lambda: L.lib.expert_place(p, batch, experts, batch, k, capacity, p, p, p, ctypes.c_size_t(n), None)

    for batch, experts, k in (((1 << 30) - 1, 1, 1), ((1 << 30) - 1, 1024, 1), ((1 << 25) - 1, 1024, 32), ((1 << 25) - 1, 2, 32), ((1 << 30) // 3 - 1, 4, 3)):
        refused_or_launched(L, place(batch, experts, k, 1000), False)

    def exchange(which, batch, experts, k, features, capacity=1000, weights=True, dye=True, dw=True):
        n = L.lib.expert_placement_bytes(experts, batch, k)
        room = L.lib.expert_combine_workspace_bytes(features, batch, k)
        w = p if weights else None
        n, room = ctypes.c_size_t(n), ctypes.c_size_t(room)
        if which == "dispatch":
            return lambda: L.lib.expert_dispatch(p, batch, p, n, features, experts, batch, k, capacity, p, capacity, None)
        if which == "combine":
            return lambda: L.lib.expert_combine(p, capacity, p, n, w, batch, features, experts, batch, k, capacity, p, batch, None)
        return lambda: L.lib.expert_combine_backward(p, capacity, p, batch, p, n, w, batch, features, experts, batch, k, capacity, p if dye else None, p if dw else None,
                                                     p, room, None)

    # gradients of the weights: 8 threads a choice, behind a launch that writes the blocks
    for dye in (True, False):
        refused_or_launched(L, exchange("backward", 1 << 29, 2, 1, 1, dye=dye), True)
        refused_or_launched(L, exchange("backward", (1 << 29) - 64, 2, 1, 1, dye=dye), False)
    refused_or_launched(L, exchange("backward", 1 << 29, 2, 1, 1, dw=False), False)
    refused_or_launched(L, exchange("backward", (1 << 24) - 2, 8, 32, 4, dye=False), False)
    # rows of columns to blocks and back: 4 entries a thread at least, where tiles and groups of rows are full
    for batch, experts, k, features in ((1 << 20, 8, 8, 4096), (1 << 20, 64, 8, 8191), (1 << 21, 8, 8, 4095), (1 << 19, 8, 32, 16383), (257, 8, 32, (1 << 24) - 1),
                                        (511, 64, 8, (1 << 24) - 1), ((1 << 25) + 1, 8, 1, 255), ((1 << 26) - 1, 8, 7, 127)):
        assert features * batch < 1 << 33 and batch * k < 1 << 29
        for which in ("dispatch", "combine", "backward"):
            refused_or_launched(L, exchange(which, batch, experts, k, features), False)
    refused_or_launched(L, exchange("dispatch", 1 << 22, 8, 4, 4096), True)
    refused_or_launched(L, exchange("dispatch", (1 << 22) - 2048, 8, 4, 4096), False)
    refused_or_launched(L, exchange("backward", 1 << 22, 8, 4, 4096), True)
    refused_or_launched(L, exchange("combine", 1 << 22, 8, 4, 4096), False)
    for weights in (True, False):
        refused_or_launched(L, exchange("combine", 1 << 22, 8, 4, 1 << 14, weights=weights), True)
        refused_or_launched(L, exchange("combine", (1 << 22) - 256, 8, 4, 1 << 14, weights=weights), False)


def a_workspace_is_given_for_sizes_that_the_call_takes(L):
    """expert_combine_workspace_bytes: 0 where no call of these sizes forms gradients of weights, and what it needs to both sides."""
    p = ctypes.c_void_p(P)
    top = (1 << 31) - 1

    def call(features, batch, k, room):
        n = ctypes.c_size_t(1 << 62)   # (placements of any size)
        return L.lib.expert_combine_backward(p, 8, p, batch, p, n, p, batch, features, 1024, batch, k, 8, p, p, p, ctypes.c_size_t(room), None)

    def rows(features, batch):   # of features in one sum, at least
        rows = 16
        while rows > 4 and -(-features // rows) * -(-batch // 1024) < 512:
            rows //= 2
        return rows

    for features, batch, k in ((1, 1 << 29, 1), (1, 1 << 28, 2), (100, (1 << 30) - 1, 2), (1, top, 32), (1, 1 << 30, 1), (top, 100, 1), (top - 14, 1, 1), (top, top, 1), (1 << 30, 1, 1),
                               (1 << 20, 1 << 22, 1), (0, 5, 1), (5, 0, 1), (-1, 5, 1), (5, -1, 1), (5, 5, 0), (5, 5, 33)):
        assert L.lib.expert_combine_workspace_bytes(features, batch, k) == 0, (features, batch, k)
        assert L.lib.nerva_last_error() != b""
        assert call(features, batch, k, 1 << 62) in (ARGUMENT, SHAPE), (features, batch, k)
    for features, batch, k in ((1, (1 << 29) - 64, 1), (1, (1 << 24) - 2, 32), (4096, 8192, 4), (1501, 777, 4), (1, 1, 1), (2047, 4096, 28), (1 << 20, 100, 1)):
        need = L.lib.expert_combine_workspace_bytes(features, batch, k)
        assert need == -(-features // rows(features, batch)) * batch * k * 4
        assert call(features, batch, k, need) == OK and call(features, batch, k, need - 4) == WORKSPACE, (features, batch, k, L.lib.nerva_last_error())


class Network:
    """A chain of layers on the runtime without a GPU, with a workspace."""

    def __init__(self, L, sizes, batch, flags=0):
        self.L, self.batch, self.layers, self.handle = L, batch, [], ctypes.c_void_p()
        a = [ctypes.c_void_p(ctypes.addressof(h)) for h in L.host]
        for n, (cols, rows) in enumerate(zip(sizes[:-1], sizes[1:])):
            for side in (0, 1):
                L.counts(side, n_blocks=8, longest_row=cols)
            layer = ctypes.c_void_p()
            assert L.lib.sparse_linear_create(ctypes.byref(layer), rows, cols, rows * cols // 8, a[0], a[1], a[2], None, 1 if n + 2 < len(sizes) else 0, batch, None) == OK
            self.layers.append(layer)
        n = len(self.layers)
        arrays = (ctypes.c_void_p * n)(*[x.value for x in self.layers])
        velocities = (ctypes.c_void_p * n)(*[a[3].value] * n)
        assert L.lib.mlp_create(ctypes.byref(self.handle), n, arrays, velocities, (ctypes.c_void_p * n)(), batch, flags) == OK, L.lib.nerva_last_error()
        self.room = L.lib.mlp_clipped_workspace_bytes(self.handle, batch)
        self.workspace = ctypes.create_string_buffer(self.room + 256)
        self.at = ctypes.c_void_p((ctypes.addressof(self.workspace) + 255) // 256 * 256)

    def step(self, clipped=False):
        p, f = ctypes.c_void_p(ctypes.addressof(self.L.host[3])), ctypes.c_float
        common = (self.handle, p, self.batch, p, self.batch, f(0.1), f(0.9))
        if clipped:
            return self.L.lib.mlp_train_step_clipped(*common, f(1.0), self.at, ctypes.c_size_t(self.room), None, p, None)
        return self.L.lib.mlp_train_step(*common, self.at, ctypes.c_size_t(self.room), None, None)

    def profile(self, steps):
        assert self.L.lib.mlp_profile_enable(self.handle, steps) == OK

    def slots(self):
        n, steps, ms = ctypes.c_int32(), ctypes.c_int32(), (ctypes.c_double * 256)()
        self.L.lib.mlp_profile_slot_name.restype = ctypes.c_char_p
        assert self.L.lib.mlp_profile_read(self.handle, 256, ctypes.byref(n), ms, ctypes.byref(steps)) == OK, self.L.lib.nerva_last_error()
        return steps.value, [self.L.lib.mlp_profile_slot_name(self.handle, i).decode() for i in range(n.value)]


def a_profile_is_of_one_kind_of_step(L):
    """The slots' names are those of the first step that is recorded: the other kind, which launches something else, is refused until as many
    steps as were asked for have been recorded."""
    for flags in (0, 1):   # (fused and not)
        N = Network(L, (64, 48, 32, 10), 20, flags)
        for clipped in (True, False):
            N.profile(3)
            assert N.step(clipped) == OK and N.step(clipped) == OK
            before = L.hip.fake_launches()
            assert N.step(not clipped) == ARGUMENT and L.hip.fake_launches() == before
            assert b"clipped" in L.lib.nerva_last_error()
            assert N.slots()[0] == 2 and N.step(clipped) == OK
            steps, names = N.slots()
            assert steps == 3 and ("norm+momentum[0]" in names) == clipped
            if clipped:
                assert names[-3:] == ["norm+momentum[0]", "mirror_refresh[2]", "mirror_refresh[1]"] and names.count("norm+momentum[0]") == 1
            assert N.step(not clipped) == OK and N.step(clipped) == OK     # (no longer recorded)
            assert N.slots() == (3, names)
        N.profile(0)
        assert N.step(True) == OK and N.step(False) == OK and N.slots() == (0, [])


CASES = [a_call_that_no_launch_holds_is_refused_before_the_first, a_workspace_is_given_for_sizes_that_the_call_takes, a_profile_is_of_one_kind_of_step]


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("hip") / "fake_launches.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__=1", "-isystem", "/opt/rocm/include",
                    os.path.join(HERE, "fake_launches.cpp"), "-o", out], check=True)
    return out


@pytest.mark.parametrize("case", [c.__name__ for c in CASES])
def test_launches(fake, case):
    run = subprocess.run([sys.executable, os.path.abspath(__file__), fake, case], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout + run.stderr


if __name__ == "__main__":
    globals()[sys.argv[2]](library(sys.argv[1]))
