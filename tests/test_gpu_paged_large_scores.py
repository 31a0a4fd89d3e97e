"""Attention over the paged cache where scores are so large that a float32 near them is coarse.

Q and K are chosen so that every score, and every partial sum of its products, is a whole number below
2^24 times a power of two: float32 holds it exactly, in any order of summation. So a probability's
error is what the softmax adds, and the tolerance is that of _cache_ref with e = 0.
"""

import pytest
import torch

from tests import _cache_ref as R
from tests.test_gpu_paged_attn import BF, F, run

pytestmark = pytest.mark.gpu


def expect(bt, O, lse, scale, causal=True):
    for b in range(bt.B):
        n, N, o = bt.new[b], bt.kv[b], int(bt.new_off[b])
        v, _ = bt.seq(bt.V, b)
        for h, (x, _) in enumerate(R.scores(bt, b, scale, causal)):
            p = torch.softmax(x, 1)
            vv = v[h // (bt.Hq // bt.H)]
            r = 2.0 ** -8 if bt.dtype == BF else 0.0
            tol = (p @ vv.abs()) * (r + 2 * (N + 64) * R.U + 2.0 ** -18)
            want = p @ vv
            R.close(O[h, o:o + n], want, tol + R.HALF[O.dtype] * want.abs(), f"O {b} {h}")
            l = torch.logsumexp(x, 1)
            R.close(lse[h, o:o + n], l, (N + 64) * R.U + 2.0 ** -19 + 4 * R.U * l.abs(), f"lse {b} {h}")


def fill(bt, q_of, k_of):
    """q_of(token), k_of(sequence, cached token): the channels of a row, the same for every head."""
    for c in range(int(bt.new_off[-1])):
        bt.Q[:, c] = q_of(c)
    for b, t, p, r in bt.places():
        bt.K[p, :, r] = k_of(b, t)


# dtype, Hq, H, d, page, new, kv: few rows and many, whole and in parts, an odd last part
SHAPES = [
    (BF, 4, 1, 128, 64, (1, 2), (77, 2900)),
    (BF, 2, 2, 64, 16, (9, 1), (4100, 20)),
    (BF, 4, 2, 64, 16, (20, 3), (600, 130)),
    (BF, 3, 3, 128, 64, (150, 90), (150, 3001)),
    (BF, 2, 1, 96, 32, (200,), (1111,)),
    (BF, 6, 2, 64, 128, (170, 33), (2700, 33)),
    (F, 4, 2, 64, 16, (1, 3), (1601, 50)),
    (F, 2, 2, 128, 32, (70,), (1300,)),
]


POWERS = [22, 33, 90]


def equal_scores(dtype, Hq, H, d, page, new, kv, power, sign, workspace):
    """Scores of d 2^power (over 8 for a third of the rows) or none: the average of V's rows over the
    tokens of the largest, whose number differs from part to part."""
    bt = R.Batch(61, dtype, Hq, H, d, page, new, kv, tail=1)
    g = torch.Generator().manual_seed(62)
    big = [torch.rand(k, generator=g) < 0.3 for k in kv]
    for x in big:
        x[: len(x) // 2] &= torch.rand(len(x) // 2, generator=g) < 0.1
    half = power // 2
    fill(bt, lambda c: torch.full((d,), 2.0 ** (half - (3 if c % 3 == 1 else 0))),
         lambda b, t: torch.full((d,), sign * 2.0 ** (power - half) * float(big[b][t])))
    expect(bt, *run(bt, "token", workspace, softmax_scale=1.0), 1.0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("power", POWERS)
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_equal_scores(gpu, shape, power, sign):
    equal_scores(*shape, power, sign, workspace=False)


def close_scores(dtype, Hq, H, d, page, new, kv, start, workspace):
    """Scores of 11,629,080 and some units around it, 2^24 in log2 units: an ordinary softmax."""
    bt = R.Batch(63, dtype, Hq, H, d, page, new, kv, tail=1)
    g = torch.Generator().manual_seed(64)
    extra = [torch.randint(-6, 7, (k,), generator=g) for k in kv]
    for x in extra:  # the largest of a row come late
        x[: len(x) // 2] -= 3
    rest = start - 4096 * 2838  # of 2,838 = 2,832 + 6
    assert 0 <= rest < 16 * 320

    def k_of(b, t):
        row = torch.zeros(d)
        row[:5] = torch.tensor([2832.0, 6.0, rest // 16 // 4 * 4, rest - rest // 16 // 4 * 64,
                                float(extra[b][t])])
        return row

    q = torch.zeros(d)
    q[:5] = torch.tensor([4096.0, 4096.0, 16.0, 1.0, 1.0])
    fill(bt, lambda c: q, k_of)
    x = bt.seq(bt.K, 0)[0][0] @ q.double()
    assert int(x.min()) >= start - 9 and int(x.max()) <= start + 6  # (bf16 holds every entry)
    expect(bt, *run(bt, "head", workspace, softmax_scale=1.0), 1.0)


STARTS = [11629080, 11629080 - 300]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("start", STARTS)
def test_close_scores_near_2_to_the_24(gpu, shape, start):
    close_scores(*shape, start, workspace=False)


def scaled_scores(dtype, scale, workspace):
    """Whole numbers as scores and a scale that makes one unit everything, or nothing."""
    for Hq, H, d, new, kv in ((4, 1, 64, (2,), (2000,)), (2, 2, 128, (140,), (900,))):
        bt = R.Batch(65, dtype, Hq, H, d, 16, new, kv)
        g = torch.Generator().manual_seed(66)
        k = torch.randint(-4, 5, (max(kv), d), generator=g).float()
        q = torch.randint(-4, 5, (max(new), d), generator=g).float()
        fill(bt, lambda c: q[c], lambda b, t: k[t])
        expect(bt, *run(bt, "head", workspace, softmax_scale=scale), scale)


SCALES = [2.0 ** 60, 2.0 ** 99, 2.0 ** -60]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("scale", SCALES)
def test_large_and_small_scales(gpu, dtype, scale):
    scaled_scores(dtype, scale, workspace=False)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("power", POWERS)
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_equal_scores_in_parts(gpu, shape, power, sign):
    equal_scores(*shape, power, sign, workspace=True)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("start", STARTS)
def test_close_scores_in_parts(gpu, shape, start):
    close_scores(*shape, start, workspace=True)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("scale", SCALES)
def test_scales_in_parts(gpu, dtype, scale):
    scaled_scores(dtype, scale, workspace=True)
