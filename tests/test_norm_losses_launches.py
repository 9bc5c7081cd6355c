"""The launches of group norm, dropout and the losses of labels, from the host's side: the library runs on a HIP runtime without a GPU
(fake_launches.cpp), each test in a process of its own."""
import ctypes
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)

from test_launches_host import OK, SHAPE, WORKSPACE, P, fake, library, refused_or_launched  # noqa: E402,F401

F, SZ, V = ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p


def sizes(L):
    for name in ("group_norm_workspace_bytes", "label_loss_workspace_bytes"):
        getattr(L.lib, name).restype = SZ
    return L.lib


def norm(lib, features, groups, batch, room=None, forward=True):
    p, q, n = V(P), V(2 * P), SZ(lib.group_norm_workspace_bytes(features, groups, batch) if room is None else room)
    if forward:
        return lib.group_norm_forward(p, batch, p, p, features, groups, batch, F(1e-5), 2, F(0.5), 0, p, q, batch, p, p, batch, p, n, None)
    return lib.group_norm_backward(p, batch, p, p, p, p, batch, p, batch, features, groups, batch, 2, F(0.5), 0, p, q, batch, p, p, p, n, None)


def losses(lib, classes, batch, sequences, room=None):
    p, q = V(P), V(2 * P)

    def n(sequences):
        return SZ(lib.label_loss_workspace_bytes(classes, batch, sequences) if room is None else room)
    yield lambda: lib.label_log_probs(p, batch, p, classes, batch, p, sequences, p, p, p, n(sequences), None)
    yield lambda: lib.policy_loss(p, batch, p, p, p, p, p, classes, batch, F(0.2), F(0.2), F(0.1), q, batch, p, p, p, n(0), None)
    yield lambda: lib.preference_loss(p, batch, p, p, p, classes, batch, sequences // 2, F(0.1), F(0), q, batch, p, p, p, p, n(sequences), None)


def every_size_is_launched_with_its_workspace_and_refused_without(L):
    lib = sizes(L)
    around = [1, 2, 3, 7, 16, 63, 64, 65, 255, 256, 257, 1023, 1024, 1025, 2048, 2049, 4096, 8191, 8193, 40000, 1 << 20]
    for m in around:
        for groups in (1, 3, 64, 4096):
            if m * groups >= 1 << 30:
                continue
            for batch in around:
                if m * groups * batch > 1 << 31:     # (what the header promises)
                    continue
                n = lib.group_norm_workspace_bytes(m * groups, groups, batch)
                for forward in (True, False):
                    refused_or_launched(L, lambda: norm(lib, m * groups, groups, batch, forward=forward), False)
                if n:
                    before = L.hip.fake_launches()
                    assert norm(lib, m * groups, groups, batch, n - 4) == WORKSPACE and norm(lib, m * groups, groups, batch, n - 4, False) == WORKSPACE
                    assert L.hip.fake_launches() == before
    for classes in around:
        for batch in around + [1 << 24]:
            for sequences in (2, 64):
                for call in losses(lib, classes, batch, sequences):
                    refused_or_launched(L, call, False)
                before = L.hip.fake_launches()
                for call in losses(lib, classes, batch, sequences, lib.label_loss_workspace_bytes(classes, batch, 0) - 4):
                    assert call() == WORKSPACE
                assert L.hip.fake_launches() == before


def a_call_that_no_launch_holds_is_refused_before_the_first(L):
    lib = sizes(L)
    p, q = V(P), V(2 * P)

    def dropout(features, batch):
        return lambda: lib.dropout(p, batch, features, batch, F(0.5), 0, p, q, batch, None)
    # eight entries a thread, and as many again of them where tiles are full
    refused_or_launched(L, dropout(1 << 15, 1 << 21), True)
    refused_or_launched(L, dropout((1 << 15) - 1024, 1 << 20), False)
    refused_or_launched(L, dropout((1 << 30) - 1, 1), False)
    refused_or_launched(L, dropout(1, (1 << 30) - 1), False)
    for forward in (True, False):
        refused_or_launched(L, lambda: norm(lib, (1 << 30) - 1, 1, 1, forward=forward), False)
        refused_or_launched(L, lambda: norm(lib, 1, 1, (1 << 30) - 1, forward=forward), False)
        refused_or_launched(L, lambda: norm(lib, 1 << 29, 1 << 29, 1 << 20, 1 << 62, forward=forward), True)
        refused_or_launched(L, lambda: norm(lib, 1 << 15, 1 << 5, 1 << 18, forward=forward), False)
        for m, batch in ((64, 33), (64, 1 << 20), (65, 33), (65, 1 << 22), (66, 5), (129, 129), (513, 33), (515, 8191), (1025, 33), (1027, 40000), (2049, 33), (2051, 1 << 21), (5000, 1)):
            groups = min(1 << 25, ((1 << 30) - 1) // m, (1 << 34) // (m * batch))
            refused_or_launched(L, lambda: norm(lib, m * groups, groups, batch, forward=forward), False)
        for features, groups, batch in ((1 << 25, 1 << 25, 1), (1 << 25, 1 << 25, 64), (1 << 25, 1 << 24, 63), (3 << 23, 1 << 23, 85), (5 << 20, 5 << 20, 409), (1 << 21, 1 << 21, 1023),
                                        (1 << 21, 1 << 20, 257 * 3), (7 << 10, 1 << 10, 299593), (1, 1, (1 << 30) - 1), (2, 1, (1 << 30) - 1), (9 << 4, 1 << 4, 14913080), (3, 3, 715827882)):
            assert features * batch <= 1 << 31
            refused_or_launched(L, lambda: norm(lib, features, groups, batch, forward=forward), False)
        refused_or_launched(L, lambda: norm(lib, 1 << 20, 1, 1 << 20, 1 << 62, forward=forward), True)     # (in chunks)
    for classes, batch in ((1, (1 << 30) - 1), ((1 << 30) - 1, 1), (1 << 20, 1 << 20), (10, 1 << 28)):
        for call in losses(lib, classes, batch, 2):
            before = L.hip.fake_launches()
            rc = call()
            assert L.hip.fake_too_large() == 0
            assert rc == OK and L.hip.fake_launches() > before or rc == SHAPE and L.hip.fake_launches() == before and b"columns" in lib.nerva_last_error()
    for classes in (1, 2, 5, 60, 64, 100, 1000, 1024, 1025, 5000, 1 << 20, 1 << 25):
        for call in losses(lib, classes, 1 << 26, (1 << 22) - 2 if classes < 100 else 1 << 10):
            refused_or_launched(L, call, False)
    label, policy, preference = losses(lib, 10, 1000, 1 << 23)
    refused_or_launched(L, label, True)
    refused_or_launched(L, policy, False)
    refused_or_launched(L, preference, True)


CASES = [every_size_is_launched_with_its_workspace_and_refused_without, a_call_that_no_launch_holds_is_refused_before_the_first]


@pytest.mark.parametrize("case", [c.__name__ for c in CASES])
def test_launches(fake, case):  # noqa: F811
    run = subprocess.run([sys.executable, os.path.abspath(__file__), fake, case], capture_output=True, text=True, timeout=240)
    assert run.returncode == 0, run.stdout + run.stderr


if __name__ == "__main__":
    globals()[sys.argv[2]](library(sys.argv[1]))
