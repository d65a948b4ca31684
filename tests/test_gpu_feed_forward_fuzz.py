"""Random sizes, layouts, types and alignments of the feed-forward operators against the 64-bit definitions."""
import random

import pytest
import torch

import test_gpu_expert_padding
import test_gpu_experts
import test_gpu_linear
from feed_forward_util import ACTS

pytestmark = pytest.mark.gpu


def size(r, most, step=None):
    """Small ones often, and as often multiples of eight as not."""
    v = int(round(2 ** r.uniform(0, torch.tensor(float(most)).log2().item())))
    step = r.choice([1, 8, 64]) if step is None else step
    return max(1, min(most, (v + step - 1) // step * step))


@pytest.mark.parametrize("seed", range(60))
def test_linear(seed):
    r = random.Random(seed)
    flag = lambda: r.random() < 0.5  # noqa: E731
    m, k, n = size(r, 2500, 1), size(r, 1500), size(r, 1500)
    test_gpu_linear.run_linear(m, k, n, r.choice(list(ACTS)), flag(), flag(), flag(), flag(), flag(), flag(), seed, r.random() < 0.25)


@pytest.mark.parametrize("seed", range(60))
def test_linear_backward(seed):
    r = random.Random(1000 + seed)
    flag = lambda: r.random() < 0.5  # noqa: E731
    m, k, n, f32 = size(r, 2500, 1), size(r, 1000), size(r, 1000), flag()
    test_gpu_linear.run_backward(m, k, n, r.choice(list(ACTS)), flag(), flag(), flag(), f32, f32 and flag(), seed, r.random() < 0.25)


def experts_of(r):
    e = r.choice([1, 2, 5, 16, 64, 300])
    return size(r, 1200, 1), r.choice([k for k in (1, 2, 4, 7) if k <= e]), e, size(r, 400), size(r, 400)


@pytest.mark.parametrize("seed", range(40))
def test_experts(seed):
    r = random.Random(2000 + seed)
    flag = lambda: r.random() < 0.5  # noqa: E731
    t, topk, e, k, n = experts_of(r)
    test_gpu_experts.test_forward(t, topk, e, k, n, flag(), flag(), flag(), r.choice(["spread", "dropped", "one"]))


@pytest.mark.parametrize("seed", range(60))
def test_experts_backward(seed):
    r = random.Random(3000 + seed)
    flag = lambda: r.random() < 0.5  # noqa: E731
    t, topk, e, k, n = experts_of(r)
    how, gated, colmajor, gather = r.choice(["spread", "dropped", "one"]), flag(), flag(), flag()
    if flag():
        test_gpu_experts.run_backward(t, topk, e, k, n, gated, colmajor, gather, how, r.choice(list(ACTS)), flag())
    else:
        test_gpu_expert_padding.run(t, topk, e, k, n, r.choice(list(ACTS)), gated, colmajor, gather,
                                    [s for s in ("x", "dy") if flag()], flag(), how)
