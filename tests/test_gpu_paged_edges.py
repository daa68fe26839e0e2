"""Numbers at the ends of their ranges through each of the paged cache's attention kernels: decode, and prefill's two."""
import math

import numpy as np
import pytest
import torch

import paper_2504_03661_amd as pq
from tests.paged_inputs import HALF_STEP, TORCH, Filled, check, context, dev, rounded
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


CLAIMS = {       # rows claimed by each sequence: first, number; rows of the tensors; whether they are more in all
    "apart": ([(0, 30), (30, 10)], 40, False),
    "apart, cut off by the tensors' end": ([(0, 30), (30, 2 ** 31 - 1)], 40, False),
    "outside the tensors": ([(0, 40), (40, 5), (-3, 9), (2 ** 31 - 1, 1)], 40, False),
    "twice, and others by nobody": ([(0, 10), (0, 10), (20, 10)], 40, False),
    "one row twice": ([(0, 30), (29, 11)], 40, True),
    "all by sixty": ([(0, 40)] * 60, 40, True),
    "as many as numbers reach": ([(0, 2 ** 31 - 1)] * 300, 50, True),
}


@pytest.mark.parametrize("what", CLAIMS)
@pytest.mark.parametrize("heads", [2, 128], ids=["few rows", "many rows"])
def test_rows_claimed_twice_are_reported(what, heads):
    """Bit 2 where the claims are more than there are rows; else a sequence whose rows nobody else claims gets what is right."""
    claims, tokens, more = CLAIMS[what]
    more_rows = 1 if heads == 2 else 30                      # 128 heads: 300 and more rows a sequence, enough for tiles of 256
    claims = [(first * more_rows if 0 <= first < 2 ** 20 else first, min(n * more_rows, 2 ** 31 - 1)) for first, n in claims]
    tokens *= more_rows
    rng = np.random.default_rng(44)
    c = Filled(rng, np.array([500] * 3), heads, DIM, 16)
    c.table, c.lengths = c.table[np.arange(len(claims)) % 3], np.full(len(claims), 500)     # (sequences that share their blocks)
    c.block_table, c.seq_len = dev(c.table), dev(c.lengths)
    ctx = context("f16", heads, heads, DIM, 16, c.n_blocks, c.width, len(claims), tokens)
    q, values = rounded(rng.standard_normal((tokens, heads, DIM)), "f16")
    room = torch.full((tokens + 8, heads, DIM), 7.0, dtype=torch.float16, device="cuda")
    out = room[4:-4]
    first, n = (dev([x[i] for x in claims] + [0]) for i in (0, 1))
    pq.pq_paged_prefill(ctx.handle, len(claims), tokens, q.cuda(), heads * DIM, *c.args(), first, n, 0.1, out)
    assert pq.pq_paged_device_error(ctx.handle) == (4 if more else 0)
    assert (room[:4] == 7.0).all() and (room[-4:] == 7.0).all()
    if more:
        return
    claimed = np.zeros(tokens, int)
    ends = [min(first + n, tokens) if 0 <= first < tokens else first for first, n in claims]
    for (first, _), end in zip(claims, ends):
        claimed[first:max(first, end)] += 1 if 0 <= first < tokens else 0
    assert (out[claimed == 0] == 7.0).all()
    for b, ((first, n), end) in enumerate(zip(claims, ends)):
        if 0 <= first < tokens and (claimed[first:end] == 1).all():
            i = np.arange(end - first)[::-57][::-1]
            check(out[first + i], *c.attention(values[first + i], b, 0.1, 500 - n + i + 1), "f16", DIM, f"sequence {b}")


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("power", [12, 23, 40, 120])
def test_scores_far_beyond_the_numbers_below_one(path, dtype, power):
    """Where a row's largest score is further above the next than both can be off, its answer is that token's value: off by the rounding of
    its weight (fp32: in two parts), 2^-19 for the sum and half a step of the output."""
    p = prompt(np.random.default_rng(45), path, dtype, 700)
    out = attend(p, path, 2.0 ** power).double().cpu().numpy()
    assert np.isfinite(out).all()
    k, v = (p.c.model[kind].rows(p.c.table[0], 700)[0] for kind in "kv")
    decided = 0
    rows = np.arange(p.new)[::-37]
    for r in rows:
        for h in range(HEADS):
            t = k[h, :p.sees(r)] @ p.values[r, h]
            off = (DIM + 16) * 2.0 ** -24 * (np.abs(k[h]) @ np.abs(p.values[r, h])).max()
            best = int(t.argmax())
            gap = t[best] - np.delete(t, best).max()
            if gap > 4 * off and gap * 2.0 ** power > 60:
                decided += 1
                want = v[h, best]
                allowed = np.abs(want) * (HALF_STEP[dtype] * 1.01 + (2.0 ** -21 if dtype == "f32" else 2.0 ** -11) + 2.0 ** -19) + 2.0 ** -25
                assert (np.abs(out[r, h] - want) <= allowed).all(), (r, h)
    assert decided > 0.9 * HEADS * len(rows)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("at", [-3.3e38, 3.3e38, 2.0 ** 22, -2.0 ** 22 + 3.0, 2.0 ** 26 + 24.0, -2.0 ** 27])
def test_scores_all_alike_far_from_zero(path, at):
    """Every token has the score `at` (in base two), or nearly, so every row's answer is the mean of the values it sees: whatever a score's
    rounding is it is the same for all, 2^-11 for the weights, 2^-19 for sums and half a step of the output are left."""
    p = prompt(np.random.default_rng(46), path, "f16", 700)
    m = p.c.model["k"]
    m.codes[:], m.scale[:] = 64, np.float32(2.0 ** -6)
    p.put("k")
    m = p.c.model["v"]
    m.scale[:] = np.float32(2.0 ** -6)
    p.put("v")
    p.q, p.values[:] = torch.ones_like(p.q), 1.0
    out = attend(p, path, at / math.log2(math.e) / DIM).double().cpu().numpy()
    v = p.c.model["v"].rows(p.c.table[0], 700)[0]
    for r in np.arange(p.new)[::-37]:
        n = p.sees(r)
        want, spread = v[:, :n].mean(1), np.abs(v[:, :n]).mean(1)
        allowed = spread * (2.0 ** -11 + 2.0 ** -19) + np.abs(want) * 2.0 ** -11 * 1.01 + 2.0 ** -25
        assert (np.abs(out[r] - want) <= allowed).all(), r
