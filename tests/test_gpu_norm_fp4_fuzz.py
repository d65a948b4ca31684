"""Random sizes, types, alignments and options of the norms and the 4-bit operators against the 64-bit definitions."""
import random

import pytest
import torch

import test_gpu_fp4_linear
import test_gpu_fp4_quantize
import test_gpu_norm
from feed_forward_util import ACTS, gen
from fp4_util import MX, NV

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def size(r, most, step=None):
    """Small ones often, and as often multiples of eight as not."""
    v = int(round(2 ** r.uniform(0, torch.tensor(float(most)).log2().item())))
    step = r.choice([1, 8, 32]) if step is None else step
    return max(1, min(most, (v + step - 1) // step * step))


@pytest.mark.parametrize("seed", range(60))
def test_norm(seed):
    r = random.Random(seed)
    n = size(r, 20000)
    m = size(r, max(1, min(6000, 4000000 // n)), 1)
    rms, kind = r.random() < 0.5, r.choice([BF, F32])
    test_gpu_norm.test_forward(m, n, rms, kind)
    test_gpu_norm.test_backward(m, n, rms, kind)
    if r.random() < 0.3:
        test_gpu_norm.test_unaligned_tensors(m, n, kind)


@pytest.mark.parametrize("seed", range(60))
def test_quantize(seed):
    r = random.Random(1000 + seed)
    parts = r.choice([1, 1, 2, 3])
    rows, k = parts * size(r, 700, 1), size(r, 3000)
    kind, fmt = r.choice([BF, F32]), r.choice([MX, NV])
    test_gpu_fp4_quantize.test_quantize_and_read_back(rows, parts, k, fmt, kind, r.random() < 0.5, r.random() < 0.5)


@pytest.mark.parametrize("seed", range(80))
def test_linear(seed):
    r = random.Random(2000 + seed)
    flag = lambda: r.random() < 0.5  # noqa: E731
    m, k, n = size(r, 1500, 1), size(r, 4000), size(r, 2000)
    test_gpu_fp4_linear.run(m, k, n, r.choice([MX, NV]), r.choice(list(ACTS)), flag(), flag(), flag(), flag(), True, seed,
                            r.random() < 0.25)


@pytest.mark.parametrize("seed", range(6))
def test_pairs_of_blocks(seed):
    # sizes that fill the device: the tile kernel's pairs, several tiles to each
    r = random.Random(3000 + seed)
    m, k, n = r.randint(1500, 4000), size(r, 1500, 1) + 700, r.randint(2000, 5000)
    test_gpu_fp4_linear.run(m, k, n, r.choice([MX, NV]), r.choice(list(ACTS)), seed % 2 == 0, True, seed % 3 == 0, seed % 3 == 1, True, seed)
