"""pq_paged_prefill's kernel for tiles of 256 rows, which takes calls that fill the chip, on inputs that it could get wrong, against the
plain model in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2504_03661_amd as pq
from oracle import paged_oracle as O
from tests.paged_inputs import TORCH, Filled, check, context, dev, rounded

pytestmark = pytest.mark.gpu

HEADS, DIM, BLOCK, SCALE = 128, 64, 16, 0.1
ZERO = np.float32(2.0 ** -40)     # the scale of a block of zeros


def many_rows():
    """Tokens of one sequence that fill three quarters of the chip in tiles of 256 rows (a row is a token and query head), which
    is when a sequence of more than 256 rows goes through them."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    return max(-(-3 * 256 * cus // (4 * HEADS)), 257) + 17


class Prompt:
    """One sequence of `length` tokens, the last `new` of which are asked about by HEADS query heads."""

    def __init__(self, rng, dtype, length, new=None, kv_heads=HEADS, dim=DIM, block=BLOCK):
        self.dtype, self.dim, self.block = dtype, dim, block
        self.new = many_rows() if new is None else new
        self.c = Filled(rng, np.array([length]), kv_heads, dim, block)
        self.ctx = context(dtype, HEADS, kv_heads, dim, block, self.c.n_blocks, self.c.width, 1, self.new)
        self.q, self.values = rounded(rng.standard_normal((self.new, HEADS, dim)), dtype)

    def put(self, kind):
        """What the model holds, onto the device"""
        m = self.c.model[kind]
        self.c.data[kind].copy_(torch.from_numpy(m.bytes(kind == "v")))
        self.c.scale[kind].copy_(torch.from_numpy(m.scale))

    def __call__(self, scale=SCALE, out=None):
        out = torch.full((self.new, HEADS, self.dim), 7.0, dtype=TORCH[self.dtype], device="cuda") if out is None else out
        pq.pq_paged_prefill(self.ctx.handle, 1, self.new, self.q.cuda(), HEADS * self.dim, *self.c.args(), dev([0, self.new]),
                            dev([self.new]), scale, out)
        return out

    def sees(self, rows):
        return int(self.c.lengths[0]) - self.new + rows + 1

    def check(self, out, scale=SCALE, every=37, heads=None, rows=None):
        rows = np.arange(self.new)[::-every][::-1] if rows is None else rows
        want = self.c.attention(self.values[rows], 0, scale, self.sees(rows))
        got = out[rows]
        if heads is not None:
            got, want = got[:, heads], [w[:, heads] for w in want]
        check(got, *want, self.dtype, self.dim)


WHERE = {
    "every second block": lambda n: np.arange(n) % 2 == 1,
    "the second half": lambda n: np.arange(n) >= n // 2,
    "one block in sixteen": lambda n: np.arange(n) % 16 == 5,
    "all but one block in sixteen": lambda n: np.arange(n) % 16 != 5,
}


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("larger", [0, 5, 8])
def test_values_of_zero_count_in_the_sum_of_weights(dtype, where, larger):
    """Blocks whose values are zeros have the scale 2^-40, next to ones of 2^-7 .. 2^-5 times 2^larger.  What such a token adds to the
    sum of the weights counts as much as any other's: paged_inputs.bound, whose terms for the sum are the score's error and 2^-19,
    holds for them as for others."""
    p = Prompt(np.random.default_rng(larger), dtype, 1201)
    blocks = p.c.table[0][WHERE[where](p.c.width)]
    m = p.c.model["v"]
    m.scale *= np.float32(2.0 ** larger)
    m.codes[blocks], m.scale[blocks] = 0, ZERO
    p.put("v")
    p.check(p())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, 0.1, -0.4])
def test_scales_of_all_sizes(dtype, scale):
    """Values' scales spread over 2^30, keys' over 2^14: weights far below the largest, and maxima that move often."""
    rng = np.random.default_rng(30)
    p = Prompt(rng, dtype, 1000)
    for kind, low, high in (("k", -11, 3), ("v", -25, 5)):
        p.c.model[kind].scale *= np.exp2(rng.integers(low, high + 1, p.c.model[kind].scale.shape)).astype(np.float32)
        p.put(kind)
    p.check(p(scale), float(np.float32(scale)))
