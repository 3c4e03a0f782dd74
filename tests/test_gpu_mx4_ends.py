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
