"""The two layers that make the library's calls, compiled and through ctypes: numbers and strides that the C calls do not hold are refused by both."""
import pytest


@pytest.fixture(scope="module")
def layers():
    from paper_2407_17437_amd import binding as nb
    from paper_2407_17437_amd.calls import Calls
    return nb._fastcall, Calls(nb.lib, nb._stream)


def test_numbers_beyond_32_bits(layers):
    import torch
    f, i = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.int32)
    b = f.view(2, 2, 8)
    for n in (2 ** 31, 2 ** 32 + 1, -2 ** 31 - 1):
        for calls in layers:
            for name, args, at in (("route", [f, None, 4, 8, 2, 1, 1, 0, 1.0, i, f, 0], range(2, 8)), ("route_backward", [f, i, f, 4, 8, 2, 0, 1.0, f, 0], range(3, 7)),
                                   ("place", [i, 4, 8, 2, 3, None, None, i, 0], range(1, 5)), ("dispatch", [f, i, 4, 2, 8, 2, 8, b, 0], range(2, 7)),
                                   ("combine", [b, i, f, 2, 2, 8, 2, 8, f, 0], range(3, 8)), ("combine_backward", [b, f, i, f, 2, 2, 8, 2, 8, None, f, f, 0], range(4, 9))):
                for k in at:
                    with pytest.raises(OverflowError):
                        getattr(calls, name)(*args[:k], n, *args[k + 1:])


@pytest.mark.gpu
def test_rows_beyond_32_bits_apart(layers):
    """Rows 2^32 + 64 entries apart: 64 in 32 bits."""
    import torch
    memory = torch.empty(2 ** 32 + 64 + 32 * 3, device="cuda")
    far, far_i = memory.as_strided((2, 32), (2 ** 32 + 64, 1)), memory.view(torch.int32).as_strided((2, 32), (2 ** 32 + 64, 1))
    far_blocks = memory.as_strided((1, 2, 32), (1, 2 ** 32 + 64, 1))
    f, i, b = torch.zeros(2, 32, device="cuda"), torch.zeros(2, 32, dtype=torch.int32, device="cuda"), torch.zeros(1, 2, 32, device="cuda")
    p = torch.zeros(4096, dtype=torch.int32, device="cuda")
    for calls in layers:
        for call in (lambda: calls.route(far, None, 2, 32, 2, 1, 1, 0, 1.0, i, f, None), lambda: calls.route(f, None, 2, 32, 2, 1, 1, 0, 1.0, far_i, far, None),
                     lambda: calls.route_backward(far, i, f, 2, 32, 2, 0, 1.0, f, None), lambda: calls.place(far_i, 1, 32, 2, 8, None, None, p, None),
                     lambda: calls.dispatch(far, p, 2, 1, 32, 2, 32, b, None), lambda: calls.dispatch(f, p, 2, 1, 32, 2, 32, far_blocks, None),
                     lambda: calls.combine(far_blocks, p, None, 2, 1, 32, 2, 32, f, None), lambda: calls.combine_backward(b, far, p, f, 2, 1, 32, 2, 32, b, None, None, None)):
            with pytest.raises(AssertionError):
                call()
