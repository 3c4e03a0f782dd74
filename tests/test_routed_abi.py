"""ocean_routed.h without a GPU: every function is exported, the structs have the header's layout, arguments are refused before anything
is launched, and calls on CPU tensors raise."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rt():
    from paper_2604_19004_amd import build, routed
    if not os.path.exists(build.lib_path()):
        build.build()
    routed.load()
    return routed


def test_every_declared_symbol_is_exported(rt):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ocean_routed.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(ocean_[a-z0-9_]+)\s*\(", text))
    assert len(names) == 9
    for n in names:
        assert hasattr(rt.load(), n), f"{n} is declared in include/ocean_routed.h but not exported"


def test_struct_layouts_match_the_header(rt, tmp_path):
    src = tmp_path / "sz.c"
    src.write_text('#include "ocean_routed.h"\n#include <stdio.h>\n#include <stddef.h>\n'
                   'int main(){printf("%zu %zu %zu %zu %zu %zu %d %d\\n", sizeof(ocean_routing), sizeof(ocean_groups), sizeof(ocean_adapters), '
                   'offsetof(ocean_routing, slot), offsetof(ocean_groups, x_rows), offsetof(ocean_adapters, scale), OCEAN_BF16, OCEAN_F16);}')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(rt.ocean_routing), ctypes.sizeof(rt.ocean_groups), ctypes.sizeof(rt.ocean_adapters), rt.ocean_routing.slot.offset,
                   rt.ocean_groups.x_rows.offset, rt.ocean_adapters.scale.offset, rt.BF16, rt.F16]


def test_refusals_before_any_launch(rt):
    lib = rt.load()
    none = rt.ocean_routing(-1, 4, 2)
    far = rt.ocean_routing(1 << 28, 1024, 64)
    groups = rt.ocean_groups(10, -1, 8, None, 10)
    wide = rt.ocean_groups(1 << 31, 2, 8, None, 1 << 31)
    lora = rt.ocean_adapters(2, 8, 0x1000, 16, 128, 0x1000, 8, 64, None, None)
    b = ctypes.byref
    for rc, word in ((lambda: lib.ocean_route(0x1000, 1, 4, 1, b(none), 0x1000, 1 << 30, None), "tokens"),
                     (lambda: lib.ocean_route(0x1000, 1, 1024, 1, b(far), 0x1000, 1 << 30, None), "2^31"),
                     (lambda: lib.ocean_route(0x1000, 1, 4, 1, None, 0x1000, 1 << 30, None), "null"),
                     (lambda: lib.ocean_route_backward(None, None, None, 1, 4, 1, None, 4, None), "null"),
                     (lambda: lib.ocean_combine_backward(None, None, 4, None, 4, 1, 4, None, 4, None, None), "null"),
                     (lambda: lib.ocean_grouped_matmul(b(groups), 1, 4, 4, 0x1000, 4, 0x1000, 4, 16, 0, 0x1000, 4, None), "range"),
                     (lambda: lib.ocean_grouped_matmul(b(wide), 1, 4, 4, 0x1000, 4, 0x1000, 4, 16, 0, 0x1000, 4, None), "range"),
                     (lambda: lib.ocean_grouped_weight_grad(None, 2, 4, 4, 0x1000, 4, 0x1000, 4, 0x1000, 4, 16, 0, None), "null"),
                     (lambda: lib.ocean_adapter_matmul(b(lora), 0x1000, 9, 4, 16, 8, 0x1000, 16, 0x1000, 16, 0x1000, 8, 0x1000, 1 << 30, None), "dtype"),
                     (lambda: lib.ocean_adapter_matmul(b(lora), None, 2, 4, 16, 8, 0x1000, 16, 0x1000, 16, 0x1000, 8, 0x1000, 1 << 30, None), "ids"),
                     (lambda: lib.ocean_adapter_matmul(b(lora), 0x1000, 2, 4, 16, 8, 0x1000, 16, 0x1000, 16, 0x1000, 8, 0x1080, 1 << 30, None), "workspace"),
                     (lambda: lib.ocean_adapter_matmul(None, 0x1000, 2, 4, 16, 8, 0x1000, 16, 0x1000, 16, 0x1000, 8, 0x1000, 1 << 30, None), "null")):
        assert rc() == 1 and word in lib.ocean_last_error().decode(), word
    assert lib.ocean_route_workspace(64, 1024, 8) == 0 and lib.ocean_route_workspace(65, 1024, 8) > 0
    assert lib.ocean_route_workspace(10, 1025, 8) == 0 and lib.ocean_adapter_workspace(8, 8, 8, 9000, 8, 2) == 0


def test_sizes_of_workspaces_cover_what_they_hold(rt):
    lib = rt.load()
    for T, E, k in ((65, 1, 1), (1000, 60, 8), (1 << 20, 256, 8)):
        assert lib.ocean_route_workspace(T, E, k) >= 8 * T * k + 4 * E * ((T + 63) // 64 + 1)
    for M, K, N, L, R in ((1, 4096, 4096, 8, 16), (5000, 4096, 4096, 32, 64), (300, 100, 50, 3, 13)):
        assert lib.ocean_adapter_workspace(M, K, N, L, R, 2) >= M * (4 + 4 + 4 + 4 * R + 4 * R) + 8 * (L + 1)


def test_calls_on_the_cpu_raise(rt):
    import torch
    x = torch.zeros(4, 8)
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises((RuntimeError, ValueError)):
        rt.route(x, 2)
    with pytest.raises((RuntimeError, ValueError)):
        rt.grouped_matmul(x, torch.zeros(2, 8, 8), torch.zeros(3, dtype=torch.int64))


def test_refusals_of_sizes(rt):
    lib = rt.load()
    b = ctypes.byref
    many = rt.ocean_groups(10, 16385, 0x1000, None, 10)
    two = rt.ocean_groups(10, 2, 0x1000, None, 10)
    for rc, word in ((lambda: lib.ocean_grouped_matmul(b(many), 1, 4, 4, 0x1000, 4, 0x1000, 4, 16, 0, 0x1000, 4, None), "OCEAN_GROUPS_MAX"),
                     (lambda: lib.ocean_grouped_matmul(b(two), 1, 4, 4, 0x1000, 3, 0x1000, 4, 16, 0, 0x1000, 4, None), "row stride"),
                     (lambda: lib.ocean_grouped_matmul(b(two), 1, 4, 4, 0x1000, 1 << 45, 0x1000, 4, 16, 0, 0x1000, 4, None), "2^46"),
                     (lambda: lib.ocean_grouped_matmul(b(two), 1, 4, 4, 0x1002, 4, 0x1000, 4, 16, 0, 0x1000, 4, None), "aligned"),
                     (lambda: lib.ocean_grouped_matmul(b(two), 1, 4, 4, 0x1000, 4, 0x1000, 4, -16, 0, 0x1000, 4, None), "stride"),
                     (lambda: lib.ocean_grouped_weight_grad(b(two), 1, 4, 4, 0x1000, 4, 0x1000, 4, 0x1000, 4, 15, 0, None), "overlap"),
                     (lambda: lib.ocean_grouped_weight_grad(b(two), 1, 4, 4, 0x1000, 4, 0x1000, 4, 0x1000, 1 << 39, 16, 0, None), "overlap")):
        assert rc() == 1 and word in lib.ocean_last_error().decode(), word


def test_results_of_more_tiles_than_a_launch_takes_are_refused(rt):
    """Before anything is launched (the pointers name nothing)."""
    lib = rt.load()
    b = ctypes.byref
    n = 1 << 23
    groups, one = rt.ocean_groups(n, 3, 0x1000, None, n), rt.ocean_groups(100, 1, 0x1000, None, 100)
    lora = rt.ocean_adapters(2, 8, 0x1000, 8, 64, 0x1000, 8, n * 8, None, None)
    for dtype in (1, 2, 3):
        for inner in (8, 7):
            for rc in (lambda: lib.ocean_grouped_matmul(b(groups), dtype, inner, n, 0x1000, 8, 0x1000, 8, 8 * n, 0, 0x1000, n, None),
                       lambda: lib.ocean_grouped_matmul(b(groups), dtype, inner, n, 0x1000, 8, 0x1000, n, 8 * n, 1, 0x1000, n, None),
                       lambda: lib.ocean_grouped_weight_grad(b(one), dtype, n - 8 + inner, n, 0x1000, n, 0x1000, n, 0x1000, n, 0, 0, None),
                       lambda: lib.ocean_adapter_matmul(b(lora), 0x1000, dtype, n, inner, n, 0x1000, 8, 0x1000, 8, 0x1000, n, 0x1000, 1 << 60, None)):
                assert rc() == 1 and "tiles" in lib.ocean_last_error().decode(), (dtype, inner, lib.ocean_last_error())


def _small_routing(rt, weights=True):
    import torch
    i32 = torch.int32
    return rt.Routing(3, 4, 2, torch.tensor([0, 2, 2, 3]), torch.tensor([0, 3, 1, -1, -1, -1], dtype=i32),
                      torch.tensor([0.25, 0.75, 1, 0, 0, 0]) if weights else None, torch.tensor([0, 1, 2, 2, 3]),
                      torch.tensor([0, 2, 0, -1, -1, -1], dtype=i32), torch.tensor([0, 2, 1, -1, -1, -1], dtype=i32))


def test_a_routing_as_an_operand_of_the_sparse_product(rt):
    """Without weights every one is 1."""
    for weights, val in ((True, [0.25, 0.75, 1]), (False, [1, 1, 1])):
        R = _small_routing(rt, weights).csr()
        assert (R.rows, R.cols, R.nnz) == (3, 4, 3) and R.col_idx.tolist() == [0, 3, 1] and R.row_ptr.tolist() == [0, 2, 2, 3]
        assert R.val.tolist() == val and str(R.val.dtype) == "torch.float32"


def test_copies_of_a_routing_hold_their_own_lists(rt):
    import copy
    import dataclasses
    import pickle
    for weights in (True, False):
        r = _small_routing(rt, weights)
        for c in (copy.deepcopy(r), pickle.loads(pickle.dumps(r)), dataclasses.replace(r, slot=r.slot.clone()), copy.copy(r)):
            assert (c.tokens, c.experts, c.k) == (3, 4, 2)
            for weighted in (False, weights):
                s = c._struct(weighted)
                for name in ("row_ptr", "col_idx", "expert_ptr", "token", "slot"):
                    assert getattr(c, name).tolist() == getattr(r, name).tolist() and getattr(s, name) == getattr(c, name).data_ptr(), name
                assert s.val == (c.val.data_ptr() if weighted else None)
        assert copy.deepcopy(r).slot.data_ptr() != r.slot.data_ptr()
