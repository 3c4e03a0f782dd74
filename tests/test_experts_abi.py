"""ocean_experts.h without a GPU: every function is exported, the structs have the header's layout, arguments are refused before anything is
launched, and calls on CPU tensors raise."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    from paper_2604_19004_amd import build, experts
    if not os.path.exists(build.lib_path()):
        build.build()
    experts.load()
    return experts


def test_every_declared_symbol_is_exported(ex):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ocean_experts.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(ocean_[a-z0-9_]+)\s*\(", text))
    assert len(names) == 7
    for n in names:
        assert hasattr(ex.load(), n), f"{n} is declared in include/ocean_experts.h but not exported"


def test_struct_layouts_match_the_header(ex, tmp_path):
    src = tmp_path / "sz.c"
    src.write_text('#include "ocean_experts.h"\n#include <stdio.h>\n#include <stddef.h>\n'
                   'int main(){printf("%zu %zu %zu %zu %zu\\n", sizeof(ocean_balance), sizeof(ocean_mx4), offsetof(ocean_balance, rows), '
                   'offsetof(ocean_mx4, codes), offsetof(ocean_mx4, stride_scales));}')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(ex.ocean_balance), ctypes.sizeof(ex.ocean_mx4), ex.ocean_balance.rows.offset, ex.ocean_mx4.codes.offset, ex.ocean_mx4.stride_scales.offset]


def _four(ex, **change):
    q = ex.ocean_mx4(2, 8, 64, 0x1000, 32, 256, 0x1000, 16, 128)
    for name, v in change.items():
        setattr(q, name, v)
    return q


def test_refusals_of_matrices_in_four_bits(ex):
    lib, b = ex.load(), ctypes.byref
    groups = ex.ocean_groups(10, 2, 0x1000, None, 10)
    calls = (lambda q: lib.ocean_mx4_quantize(0x1000, 1, 64, 512, q, None), lambda q: lib.ocean_mx4_dequantize(q, 1, 0x1000, 64, 512, None),
             lambda q: lib.ocean_grouped_matmul_mx4(b(groups), 1, 0x1000, 64, q, 0, 0x1000, 8, None))
    for call in calls:
        for q, word in ((None, "null"), (_four(ex, count=-1), "range"), (_four(ex, count=16385), "OCEAN_GROUPS_MAX"), (_four(ex, rows=1 << 31), "range"),
                        (_four(ex, inner=-3), "range"), (_four(ex, codes=0x1008), "aligned"), (_four(ex, ld_codes=40), "aligned"), (_four(ex, stride_codes=264), "aligned"),
                        (_four(ex, scales=0x1008), "aligned"), (_four(ex, ld_scales=24), "aligned"), (_four(ex, stride_scales=132), "aligned"), (_four(ex, ld_codes=16), "stride"),
                        (_four(ex, ld_scales=0), "stride"), (_four(ex, ld_codes=1 << 45), "2^46"), (_four(ex, ld_scales=1 << 45), "2^46"), (_four(ex, stride_codes=-16), "stride"),
                        (_four(ex, stride_scales=1 << 50), "stride"), (_four(ex, codes=None), "null"), (_four(ex, scales=None), "null")):
            assert call(b(q) if q else None) == 1 and word in lib.ocean_last_error().decode(), (word, lib.ocean_last_error())
    for q in (_four(ex, stride_codes=240), _four(ex, stride_scales=112)):   # (read they may overlap)
        assert calls[0](b(q)) == 1 and "overlap" in lib.ocean_last_error().decode()
    q = _four(ex)
    for rc, word in ((lambda: lib.ocean_mx4_quantize(0x1000, 0, 64, 512, b(q), None), "dtype"), (lambda: lib.ocean_mx4_quantize(0x1000, 1, 63, 512, b(q), None), "stride"),
                     (lambda: lib.ocean_mx4_quantize(0x1001, 1, 64, 512, b(q), None), "aligned"), (lambda: lib.ocean_mx4_quantize(None, 1, 64, 512, b(q), None), "null"),
                     (lambda: lib.ocean_mx4_dequantize(b(q), 1, 0x1000, 64, 500, None), "overlap"),
                     (lambda: lib.ocean_mx4_quantize(0x1000, 1, 64, 512, b(_four(ex, rows=1 << 30, stride_codes=1 << 35, stride_scales=1 << 34)), None), "2^31")):
        assert rc() == 1 and word in lib.ocean_last_error().decode(), (word, lib.ocean_last_error())


def test_refusals_of_products(ex):
    lib, b = ex.load(), ctypes.byref
    g, q, x = ex.ocean_groups(10, 2, 0x1000, None, 10), _four(ex), _four(ex, count=1, rows=10)
    product, both = lib.ocean_grouped_matmul_mx4, lib.ocean_grouped_matmul_mx4_mx4
    for rc, word in ((lambda: product(b(g), 0, 0x1000, 64, b(q), 0, 0x1000, 8, None), "dtype"), (lambda: product(None, 1, 0x1000, 64, b(q), 0, 0x1000, 8, None), "null"),
                     (lambda: product(b(ex.ocean_groups(10, 3, 0x1000, None, 10)), 1, 0x1000, 64, b(q), 0, 0x1000, 8, None), "as many"),
                     (lambda: product(b(g), 1, 0x1000, 63, b(q), 0, 0x1000, 8, None), "stride"), (lambda: product(b(g), 1, 0x1000, 64, b(q), 0, 0x1000, 7, None), "stride"),
                     (lambda: product(b(g), 1, 0x1000, 7, b(q), 1, 0x1000, 64, None), "stride"), (lambda: product(b(g), 1, 0x1000, 8, b(q), 1, 0x1000, 63, None), "stride"),
                     (lambda: product(b(g), 1, None, 64, b(q), 0, 0x1000, 8, None), "null"), (lambda: product(b(g), 2, 0x1001, 64, b(q), 0, 0x1000, 8, None), "aligned"),
                     (lambda: product(b(g), 1, 0x1000, 64, b(_four(ex, ld_codes=1 << 23)), 0, 0x1000, 8, None), "2^23"),
                     (lambda: both(b(g), b(x), b(_four(ex, ld_scales=1 << 23)), 2, 0x1000, 8, None), "2^23"),
                     (lambda: both(b(g), None, b(q), 2, 0x1000, 8, None), "null"), (lambda: both(b(g), b(x), None, 2, 0x1000, 8, None), "null"),
                     (lambda: both(b(g), b(_four(ex, count=1, rows=9)), b(q), 2, 0x1000, 8, None), "x_rows"),
                     (lambda: both(b(g), b(_four(ex, count=1, rows=10, inner=63)), b(q), 2, 0x1000, 8, None), "inner"),
                     (lambda: both(b(g), b(_four(ex, rows=10)), b(q), 2, 0x1000, 8, None), "one matrix"), (lambda: both(b(g), b(x), b(q), 7, 0x1000, 8, None), "dtype"),
                     (lambda: both(b(g), b(x), b(q), 2, 0x1000, 7, None), "stride")):
        assert rc() == 1 and word in lib.ocean_last_error().decode(), (word, lib.ocean_last_error())
    n = 1 << 23   # more tiles than a launch takes
    wide = ex.ocean_groups(n, 1, 0x1000, None, n)
    tall = ex.ocean_mx4(1, n, 64, 0x1000, 32, 0, 0x1000, 16, 0)
    rows = ex.ocean_mx4(1, n, 64, 0x1000, 32, 0, 0x1000, 16, 0)
    for rc in (lambda d: product(b(wide), d, 0x1000, 64, b(tall), 0, 0x1000, n, None), lambda d: both(b(wide), b(rows), b(tall), d, 0x1000, n, None)):
        for dtype in (1, 2, 3):
            assert rc(dtype) == 1 and "tiles" in lib.ocean_last_error().decode()


def test_refusals_of_the_balance(ex):
    lib, b = ex.load(), ctypes.byref
    r = ex.ocean_routing(10, 4, 2, 0, 0x1000, 0x1000, 0x1000, 0x1000, 0x1000, 0x1000)
    out = ex.ocean_balance(0x1000, 0x1000, 0x1000, 0x1000)
    assert lib.ocean_route_balance_workspace(10, 1025) == 0 and lib.ocean_route_balance_workspace(-1, 4) == 0
    for T, E in ((1, 1), (100000, 1024)):
        assert lib.ocean_route_balance_workspace(T, E) >= 256 * (4 * E + 12)
    need = 1 << 20
    forward, backward = lib.ocean_route_balance, lib.ocean_route_balance_backward
    none = ex.ocean_routing(10, 4, 2, 0, 0x1000, 0x1000, 0x1000, None, 0x1000, 0x1000)
    bare = ex.ocean_routing(10, 4, 2, 0, 0x1000, 0x1000, None, 0x1000, 0x1000, 0x1000)
    for rc, word in ((lambda: forward(b(r), 0x1000, 1, 1 << 23, b(out), 0x1000, need, None), "2^23"),
                     (lambda: backward(b(out), b(r), 0x1000, 1, 4, 0x1000, None, 1, 0x1000, 1 << 23, None), "2^23"),
                     (lambda: forward(None, 0x1000, 1, 4, b(out), 0x1000, need, None), "null"), (lambda: forward(b(r), 0x1000, 0, 4, b(out), 0x1000, need, None), "dtype"),
                     (lambda: forward(b(none), 0x1000, 1, 4, b(out), 0x1000, need, None), "expert_ptr"), (lambda: forward(b(r), 0x1000, 1, 3, b(out), 0x1000, need, None), "stride"),
                     (lambda: forward(b(r), None, 1, 4, b(out), 0x1000, need, None), "null"), (lambda: forward(b(r), 0x1000, 1, 4, None, 0x1000, need, None), "balance"),
                     (lambda: forward(b(r), 0x1000, 1, 4, b(ex.ocean_balance(0x1000, None, 0x1000, 0x1000)), 0x1000, need, None), "balance"),
                     (lambda: forward(b(r), 0x1000, 1, 4, b(out), 0x1000, 100, None), "workspace"), (lambda: forward(b(r), 0x1000, 1, 4, b(out), 0x1080, need, None), "workspace"),
                     (lambda: backward(None, b(r), 0x1000, 1, 4, 0x1000, None, 1, 0x1000, 4, None), "balance"),
                     (lambda: backward(b(out), b(r), 0x1000, 1, 4, None, None, 1, 0x1000, 4, None), "dloss"),
                     (lambda: backward(b(out), b(bare), 0x1000, 1, 4, 0x1000, 0x1000, 1, 0x1000, 4, None), "val"),
                     (lambda: backward(b(out), b(r), 0x1000, 1, 4, 0x1000, None, 1, 0x1000, 3, None), "stride")):
        assert rc() == 1 and word in lib.ocean_last_error().decode(), (word, lib.ocean_last_error())


def test_matrices_in_four_bits_without_a_gpu(ex):
    """Shapes and layouts are checked where they are made."""
    import copy
    import pickle
    import torch
    u8 = torch.uint8
    codes, scales = torch.zeros(3, 10, 48, dtype=u8), torch.zeros(3, 10, 16, dtype=u8)
    q = ex.Mx4(codes, scales, 70)
    assert q.shape == (3, 10, 70) and ex.Mx4(codes[0], scales[0], 96).shape == (10, 96)
    for c in (copy.deepcopy(q), pickle.loads(pickle.dumps(q))):
        assert c.shape == q.shape and c._struct.codes == c.codes.data_ptr() != q.codes.data_ptr()
    s = ex.Mx4(codes[1:, 2:], scales[1:, 2:], 70)._struct
    assert (s.count, s.rows, s.inner, s.ld_codes, s.stride_codes, s.ld_scales, s.stride_scales) == (2, 8, 70, 48, 480, 16, 160)
    assert s.codes == codes.data_ptr() + 480 + 96 and s.scales == scales.data_ptr() + 160 + 32
    for bad in (lambda: ex.Mx4(codes, scales, 64), lambda: ex.Mx4(codes, scales, 97), lambda: ex.Mx4(codes, scales[..., :3], 70), lambda: ex.Mx4(codes.int(), scales, 70),
                lambda: ex.Mx4(codes, scales[:2], 70), lambda: ex.Mx4(codes[0, 0], scales[0, 0], 70), lambda: ex.Mx4(codes[..., 8:40], scales, 64),
                lambda: ex.Mx4(torch.zeros(3, 10, 49, dtype=u8)[..., :48], scales, 70),
                lambda: ex.Mx4(codes, torch.zeros(3, 10, 32, dtype=u8)[..., 8:24], 70)):
        with pytest.raises(ValueError):
            bad()
    p = ex.Mx4.laid_out(torch.zeros(3, 10, 49, dtype=u8)[..., :48], torch.ones(3, 10, 3, dtype=u8), 70)
    assert p.shape == (3, 10, 70) and bool((p.scales[..., :3] == 1).all())
    with pytest.raises(ValueError):
        ex.Mx4.laid_out(codes, scales, 70)


def test_calls_on_the_cpu_raise(ex):
    import torch
    from paper_2604_19004_amd import routed
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    x = torch.zeros(4, 64)
    q = ex.Mx4(torch.zeros(2, 8, 32, dtype=torch.uint8), torch.zeros(2, 8, 16, dtype=torch.uint8), 64)
    for call in (lambda: ex.mx4_quantize(x), lambda: ex.mx4_dequantize(q), lambda: ex.grouped_matmul_mx4(x, q, torch.zeros(3, dtype=torch.int64))):
        with pytest.raises((RuntimeError, ValueError)):
            call()


def test_the_oracle_of_four_bits():
    """Its rounding against the nearest of all numbers, and the reading back of what it packs."""
    from oracle import experts as X
    rng = np.random.default_rng(1)
    x = rng.standard_normal((20, 70)) * np.exp(rng.standard_normal((20, 1)) * 4)
    codes, scales = X.quantize(x)
    assert np.array_equal(X.unpack(X.pack(codes)), codes)
    got = X.values(codes, scales, 70)
    for i in range(20):
        for j in range(70):
            grid = np.concatenate([X.E2M1, -X.E2M1]) * 2.0 ** (scales[i, j // 32] - 127)
            assert abs(got[i, j] - x[i, j]) == np.abs(grid - x[i, j]).min()
