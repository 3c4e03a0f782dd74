"""What the entry points of ocean_experts.h refuse and what they take, where nothing is launched yet: without a GPU."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def ex():
    from paper_2604_19004_amd import build, experts
    if not os.path.exists(build.lib_path()):
        build.build()
    experts.load()
    return experts


def test_refused_sizes_name_their_header(ex):
    """What one launch does not take is refused with the header that has the sizes: that of the operator that was called."""
    lib, b = ex.load(), ctypes.byref
    n = 1 << 23
    groups = ex.ocean_groups(n, 1, 0x1000, None, n)
    tall, rows = ex.ocean_mx4(1, n, 64, 0x1000, 32, 0, 0x1000, 16, 0), ex.ocean_mx4(1, n, 64, 0x1000, 32, 0, 0x1000, 16, 0)
    for call, header in ((lambda: lib.ocean_grouped_matmul_mx4(b(groups), 1, 0x1000, 64, b(tall), 0, 0x1000, n, None), "ocean_experts.h"),
                         (lambda: lib.ocean_grouped_matmul_mx4_mx4(b(groups), b(rows), b(tall), 2, 0x1000, n, None), "ocean_experts.h"),
                         (lambda: lib.ocean_grouped_matmul(b(groups), 1, 64, n, 0x1000, 64, 0x1000, 64, 64 * n, 0, 0x1000, n, None), "ocean_routed.h")):
        assert call() == 1 and header in lib.ocean_last_error().decode(), (header, lib.ocean_last_error())


def test_rows_of_all_matrices_up_to_the_limit(ex):
    """Conversions take fewer than 2^31 - 4096 rows in all, whatever the number of matrices divides (rows of no numbers: nothing is launched)."""
    lib, b = ex.load(), ctypes.byref
    most = 2 ** 31 - 4096 - 1
    for count in (1, 2, 3, 7, 16384):
        rows = most // count
        fits, beyond = (ex.ocean_mx4(count, r, 0, None, 0, 0, None, 0, 0) for r in (rows, rows + 1))
        for convert in (lambda q: lib.ocean_mx4_quantize(None, 1, 0, 0, b(q), None), lambda q: lib.ocean_mx4_dequantize(b(q), 1, None, 0, 0, None)):
            assert convert(fits) == 0, (count, rows, lib.ocean_last_error())
            assert convert(beyond) == 1 and "2^31" in lib.ocean_last_error().decode() or count == 1


def test_the_balance_asks_for_what_it_reads(ex):
    """ocean_route_balance reads tokens, experts and expert_ptr of the routing, its gradient without dval tokens and experts: the other members may hold anything.  (Each call
    is refused for its workspace or its dlogits, the last arguments that are looked at.)"""
    lib, b = ex.load(), ctypes.byref
    out = ex.ocean_balance(0x1000, 0x1000, 0x1000, 0x1000)
    for k, row_ptr in ((2, None), (0, 0x1000), (-1, None), (70, 0x1000), (1 << 30, None)):
        r = ex.ocean_routing(1 << 20, 4, k, 0, row_ptr, None, None, 0x1000, None, None)
        assert lib.ocean_route_balance(b(r), 0x1000, 1, 4, b(out), None, 0, None) == 1 and "workspace" in lib.ocean_last_error().decode(), (k, lib.ocean_last_error())
        assert lib.ocean_route_balance_backward(b(out), b(r), 0x1000, 1, 4, 0x1000, None, 1, None, 4, None) == 1 and "a matrix is null" in lib.ocean_last_error().decode(), (k, lib.ocean_last_error())
        # with the gradient of the weights all of it is read
        assert lib.ocean_route_balance_backward(b(out), b(r), 0x1000, 1, 4, 0x1000, 0x1000, 1, None, 4, None) == 1 and "a matrix is null" not in lib.ocean_last_error().decode()
    for bad in (ex.ocean_routing(-1, 4, 2, 0, 0x1000, None, None, 0x1000, None, None), ex.ocean_routing((1 << 28) + 1, 4, 2, 0, 0x1000, None, None, 0x1000, None, None),
                ex.ocean_routing(10, 1025, 2, 0, 0x1000, None, None, 0x1000, None, None), ex.ocean_routing(10, 0, 2, 0, 0x1000, None, None, 0x1000, None, None)):
        assert lib.ocean_route_balance(b(bad), 0x1000, 1, 1025, b(out), None, 0, None) == 1 and "tokens" in lib.ocean_last_error().decode()
        assert lib.ocean_route_balance_backward(b(out), b(bad), 0x1000, 1, 1025, 0x1000, None, 1, None, 1025, None) == 1 and "tokens" in lib.ocean_last_error().decode()
