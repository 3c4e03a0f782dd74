"""Products with matrices in four bits at the ends of the scales: infinite numbers of the matrix, subnormal numbers on either side, the largest finite ones.

Tolerance as in test_gpu_mx4_products.py; a part of a single precision number that is below 2^-133 is not kept, which is less than 2^-133 for each number of x, so results may be
off by that much of the matrix's numbers' magnitudes besides."""
import numpy as np
import pytest

from oracle import experts as X

pytestmark = pytest.mark.gpu
EPS = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -25}
TERMS = {"float32": 3, "bfloat16": 1, "float16": 2}
# few rows; tiles of 64; of 128 and 256.  (groups' rows, K, N)
SIZES = [([5, 12], 96, 40), ([3], 8192, 33), ([40, 23], 200, 70), ([200, 130], 200, 150), ([700, 900], 264, 2000)]


@pytest.fixture(scope="module")
def ex():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2604_19004_amd import experts
    experts.load()
    return experts


def _np(t):
    return t.detach().cpu().double().numpy()


def _ptr(sizes):
    import torch
    return torch.tensor(np.cumsum([0] + list(sizes)), dtype=torch.int64)


def _made(ex, codes, scales, inner):
    """The matrices of codes [.., rows, 32 * blocks] (a number each) and scales [.., rows, blocks], and their numbers."""
    import torch
    blocks = scales.shape[-1]
    up = np.zeros((*scales.shape[:-1], (blocks + 15) // 16 * 16), dtype=np.uint8)
    up[..., :blocks] = scales
    return ex.Mx4(torch.from_numpy(X.pack(codes)).cuda(), torch.from_numpy(up).cuda(), inner), X.values(codes, scales, inner)


def _random(ex, rng, shape, low, high):
    """Every code, scales from low to high by block."""
    blocks = (shape[-1] + 31) // 32
    return _made(ex, rng.integers(0, 16, (*shape[:-1], blocks * 32)), rng.integers(low, high + 1, (*shape[:-1], blocks)), shape[-1])


def _rows(rng, shape, dtype, exponent):
    import torch
    return torch.from_numpy(rng.standard_normal(shape) * 2.0 ** exponent).to(getattr(torch, dtype))


def _wanted(sizes, x, w):
    """x @ w[e].T by groups in 64 bits, the sums of the magnitudes, and of the matrix's."""
    lo, want, mag, size = 0, [], [], []
    for e, n in enumerate(sizes):
        with np.errstate(invalid="ignore", over="ignore"):
            want.append(x[lo:lo + n] @ w[e].T)
            mag.append(np.abs(x[lo:lo + n]) @ np.abs(w[e].T))
        size.append(np.broadcast_to(np.abs(w[e]).sum(1), want[-1].shape))
        lo += n
    return np.concatenate(want), np.concatenate(mag), np.concatenate(size)


def _same_ends(got, want):
    got = _np(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN elsewhere"
    at = np.isinf(got) | np.isinf(want)
    assert np.array_equal(got[at], want[at]), "infinities elsewhere"
    return got, ~at & ~np.isnan(want)


@pytest.mark.parametrize("sizes,K,N", SIZES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_infinite_numbers_of_the_matrix(ex, sizes, K, N, dtype):
    """4 * 2^126, 6 * 2^126 and 2 to 6 * 2^127 are beyond bfloat16, and infinite: times x an infinity of its sign, times 0 NaN, whatever parts x has.  Each of them is alone in
    its block; some lines have two, of one sign or both, some a largest finite number (3 * 2^126, 1.5 * 2^127) or a zero at such a scale, most nothing of the kind."""
    import torch
    rng = np.random.default_rng(sum(sizes) + K + N)
    E, blocks = len(sizes), (K + 31) // 32
    for across in (False, True):
        codes, scales = rng.integers(0, 16, (E, N, blocks * 32)), rng.integers(124, 131, (E, N, blocks))
        special = []   # (matrix, line, place)
        for i in range(24):
            e, n, k = int(rng.integers(E)), int(rng.integers(N)), int(rng.integers(K))
            if i < 3:
                e, n, k = E - 1, N - 1 if i < 2 else 0, (K - 1, 0, K - 1)[i]   # (the last of the last, the first)
            b, s = k // 32, int(rng.integers(253, 255))
            if scales[e, n, b] >= 253:
                continue
            codes[e, n, b * 32:b * 32 + 32], scales[e, n, b] = 0, s
            codes[e, n, k] = (6, 7, 14, 15, 5 if s == 253 else 3, 8)[int(rng.integers(6))]
            special.append((e, n, k))
        w, value = _made(ex, codes, scales, K)
        value[np.abs(value) >= 2.0 ** 128] *= np.inf
        assert np.isinf(value).sum() >= 8
        S, inner = sum(sizes), N if across else K
        x = _rows(rng, (S, inner), dtype, 0)
        x[x == 0] = 1.0
        for e, n, k in special:   # (what meets them: numbers of one part, of several, 0, and the least that keep the largest finite ones within the type)
            c = n if across else k
            for i in range(min(S, 12)):
                x[(i * 5) % S, c] = (1.0, -1.0, 0.0, 1.0 + 2.0 ** -9, -1.5, 2.0 ** -14, -2.0 ** -12)[i % 7]
            if abs(value[e, n, k]) < np.inf and value[e, n, k] != 0:   # (finite: the rows that meet it are small enough for their results)
                x[:, c] = 0.0 if dtype == "float16" else 2.0 ** -100
        x[1, (special[0][1] if across else special[0][2])] = float("inf")
        matrix = value.transpose(0, 2, 1) if across else value
        want, mag, _ = _wanted(sizes, _np(x), matrix)
        want[np.abs(want) > float(torch.finfo(x.dtype).max)] *= np.inf   # (a result beyond its type is infinite in it: float16 has no 2^-12 * 3 * 2^126)
        got, ok = _same_ends(ex.grouped_matmul_mx4(x.cuda(), w, _ptr(sizes).cuda(), transposed=across), want)
        assert ok.any() and np.isinf(want).any() and np.isnan(want).any()
        assert np.all(np.abs(got[ok] - want[ok]) <= (TERMS[dtype] * (inner + 2) * 2.0 ** -24 * mag[ok] + EPS[dtype] * np.abs(want[ok]) + TINY[dtype]))


@pytest.mark.parametrize("sizes,K,N", SIZES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("low,high,exponent", [(0, 8, 100), (0, 0, 120), (1, 30, 90), (245, 250, -118), (248, 252, -126), (252, 252, -130), (236, 244, -118), (250, 252, -30)])
def test_products_at_the_ends_of_the_scales(ex, sizes, K, N, dtype, low, high, exponent):
    """Scales 0 and the next (subnormal numbers of the matrix) with large rows, 236 to 252 with rows whose last parts, or which themselves, are subnormal."""
    import torch
    rng = np.random.default_rng(low * 1000 + high + K)
    w, value = _random(ex, rng, (len(sizes), N, K), low, high)
    ptr, S = _ptr(sizes).cuda(), sum(sizes)
    lost = 2.0 ** -133 if dtype == "float32" else 0.0
    for x, across in ((_rows(rng, (S, K), dtype, exponent), False), (_rows(rng, (S, N), dtype, exponent), True)):
        want, mag, size = _wanted(sizes, _np(x), value.transpose(0, 2, 1) if across else value)
        got = _np(ex.grouped_matmul_mx4(x.cuda(), w, ptr, transposed=across))
        assert np.abs(want).max() < 2.0 ** 127 and np.abs(want).max() > 2.0 ** -60
        assert np.all(np.abs(got - want) <= TERMS[dtype] * (x.shape[1] + 2) * 2.0 ** -24 * mag + lost * size + EPS[dtype] * np.abs(want) + TINY[dtype])


@pytest.mark.parametrize("sizes,K,N", SIZES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,matrix", [((0, 0), (250, 250)), ((254, 254), (0, 0)), ((0, 4), (246, 254)), ((246, 254), (0, 4)), ((127, 127), (0, 2)), ((1, 1), (127, 127)),
                                         ((100, 150), (100, 150))])
def test_rows_in_four_bits_at_the_ends_of_the_scales(ex, sizes, K, N, dtype, rows, matrix):
    """Both sides' scales go into the matrix instruction as they are: numbers that no type has meet others that bring them back."""
    import torch
    rng = np.random.default_rng(rows[0] * 7 + matrix[0] + K)
    w, value = _random(ex, rng, (len(sizes), N, K), *matrix)
    q, rows_value = _random(ex, rng, (sum(sizes), K), *rows)
    want, mag, _ = _wanted(sizes, rows_value, value)
    got = _np(ex.grouped_matmul_mx4(q, w, _ptr(sizes).cuda(), dtype=getattr(torch, dtype)))
    most = float(torch.finfo(getattr(torch, dtype)).max)
    off = (K + 2) * 2.0 ** -24 * mag
    ok = np.abs(want) < most / 2
    assert np.all(np.abs(got[ok] - want[ok]) <= off[ok] + EPS[dtype] * np.abs(want[ok]) + TINY[dtype])
    # (a sum that is off by less than its size has its sign; one whose terms all but cancel need not)
    sure = ~ok & (np.abs(want) > off)
    assert np.array_equal(np.sign(got[sure]), np.sign(want[sure]))


def test_float16_rows_at_the_least_scales(ex):
    """Numbers of scales up to 51 may count as 0 beside float16 rows; from 52 on an infinite row makes infinities of them, and finite ones less than half float16's least number."""
    import torch
    rng = np.random.default_rng(5)
    for sizes, K, N in SIZES:
        for low in (0, 51, 52):
            codes, scales = rng.integers(1, 8, (len(sizes), N, (K + 31) // 32 * 32)), np.full((len(sizes), N, (K + 31) // 32), low)
            w, _ = _made(ex, codes, scales, K)
            x = _rows(rng, (sum(sizes), K), "float16", 10)
            x[2, K // 2] = float("-inf")
            y = _np(ex.grouped_matmul_mx4(x.cuda(), w, _ptr(sizes).cuda()))
            rest = np.delete(y, 2, 0)
            assert np.all(np.abs(rest) == 0) and (np.all(y[2] == -np.inf) if low == 52 else np.all(np.isnan(y[2]) | (y[2] == -np.inf)))
