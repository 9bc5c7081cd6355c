"""How the losses of labels are laid out, seen by their launches from the host's side: the library runs on a HIP runtime without a GPU (fake_launches.cpp), in a
process of its own."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)

from test_launches_host import OK, fake, library  # noqa: E402,F401
from test_norm_losses_launches import losses, sizes  # noqa: E402

# launches of log-probabilities with their sums, policy loss, preference loss: all in one; columns held by work-groups of several tiles; columns cut into chunks
ONE, HELD, CHUNKS = [1, 1, 1], [2, 2, 3], [3, 3, 4]
PLANS = [
    # one tile of 8 to 128 columns holds 4096 quads, its neighbours are held in narrow tiles, or cut where a narrow tile is too long as well
    (65, 128, ONE), (128, 128, ONE), (129, 128, HELD), (128, 100, ONE), (129, 100, HELD), (256, 64, ONE), (257, 64, HELD), (512, 32, ONE), (513, 32, HELD), (1000, 16, ONE),
    (1024, 16, ONE), (1025, 16, HELD), (1025, 8, ONE), (2048, 8, ONE), (2048, 5, ONE), (2049, 8, CHUNKS), (10, 100, ONE),
    # of 256 columns, or four and fewer, 2048
    (32, 256, ONE), (33, 256, HELD), (64, 256, HELD), (65, 256, HELD), (32, 129, ONE), (33, 129, HELD), (2048, 4, ONE), (2049, 4, CHUNKS), (2048, 1, ONE), (2049, 1, CHUNKS),
    # several tiles
    (64, 257, HELD), (1024, 8192, HELD), (1025, 8192, CHUNKS),
]


def limits(L):
    lib = sizes(L)
    for classes, batch, want in PLANS:
        got = []
        for call in losses(lib, classes, batch, 2):
            before = L.hip.fake_launches()
            assert call() == OK
            got.append(L.hip.fake_launches() - before)
        # (the sums of sixteen columns or fewer are the last part of the launch before)
        if want is CHUNKS and batch <= 16:
            got[0] += 1
        assert got == want, (classes, batch, got, want)


def test_columns_are_held_up_to_one_limit(fake):  # noqa: F811
    run = subprocess.run([sys.executable, os.path.abspath(__file__), fake], capture_output=True, text=True, timeout=240)
    assert run.returncode == 0, run.stdout + run.stderr


if __name__ == "__main__":
    limits(library(sys.argv[1]))
