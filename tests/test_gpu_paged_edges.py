"""Numbers at the ends of their ranges through each of the paged cache's attention kernels: decode, and prefill's two."""
import numpy as np
import pytest
import torch

import paper_2504_03661_amd as pq
from tests.paged_inputs import TORCH
from tests.test_gpu_paged_tiles import DIM, HEADS, Prompt

pytestmark = pytest.mark.gpu

PATHS = ["decode", "prefill of few rows", "prefill of many rows"]


def prompt(rng, path, dtype, length):
    return Prompt(rng, dtype, length, {"decode": 1, "prefill of few rows": 5, "prefill of many rows": None}[path])


def attend(p, path, scale):
    if path != "decode":
        return p(scale)
    out = torch.full((1, HEADS, DIM), 7.0, dtype=TORCH[p.dtype], device="cuda")
    pq.pq_paged_decode(p.ctx.handle, 1, p.q.cuda(), HEADS * DIM, *p.c.args(), scale, out)
    return out


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_below_the_normal_numbers(path, dtype):
    """Rows whose elements are all subnormal, under a scale that makes scores of ordinary size of them."""
    rng = np.random.default_rng(40)
    p = prompt(rng, path, dtype, 700)
    p.q = torch.from_numpy(p.values * 1e-39).to(torch.float32).to(TORCH[dtype])
    p.values = p.q.double().numpy()
    assert 0.0 < np.abs(p.values).max() < 2.0 ** -126
    scale = float(np.float32(1e38))
    p.check(attend(p, path, scale), scale)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_queries_of_zeros_under_a_large_scale(path, dtype):
    """Scores are 0 whatever the scale is, also where its product with that of the keys is beyond fp32."""
    p = prompt(np.random.default_rng(41), path, dtype, 700)
    p.values[:] = 0.0
    p.q = torch.zeros_like(p.q)
    p.c.model["k"].scale *= np.float32(2.0 ** 13)
    p.put("k")
    scale = float(np.float32(1e38))
    p.check(attend(p, path, scale), scale)


@pytest.mark.parametrize("path", PATHS)
def test_scales_that_have_no_logarithm_to_two(path):
    """scale * log2(e) has to be a number: what is not is refused, what just is gives the mean for queries of zeros."""
    p = prompt(np.random.default_rng(43), path, "f32", 700)
    p.q, p.values[:] = torch.zeros_like(p.q), 0.0
    for scale in (2.37e38, -3e38, 3.4e38):
        with pytest.raises(pq.PQAttnError) as e:
            attend(p, path, scale)
        assert e.value.status == -2
    scale = float(np.float32(-2.35e38))
    p.check(attend(p, path, scale), scale)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_far_larger_than_those_beside_them(path, dtype):
    """Values up to 2^64 in every second block, zeros in the others.  Their scales are 2^97 apart, which leaves 2^-29 of 2^-126 for the
    smallest softmax weight that counts (scores here spread over some 8: 2^-12)."""
    p = prompt(np.random.default_rng(42), path, dtype, 700)
    m = p.c.model["v"]
    m.scale *= np.float32(2.0 ** 62)
    zero = p.c.table[0][1::2]
    m.codes[zero], m.scale[zero] = 0, np.float32(2.0 ** -40)
    p.put("v")
    p.check(attend(p, path, 0.1), 0.1)
