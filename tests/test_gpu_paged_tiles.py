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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_of_extreme_sizes(dtype):
    """Rows of one call that are 2^100 apart, rows of zeros, one large element."""
    rng = np.random.default_rng(31)
    p = Prompt(rng, dtype, 600)
    p.values *= np.exp2(rng.integers(-100, 101, (p.new, HEADS, 1)))
    p.values[:, 5] = 0.0
    p.values[:, 6] = 0.0
    p.values[:, 6, 9] = 2.0 ** 97
    p.q, p.values = rounded(p.values, dtype)
    for scale in (2.0 ** -100, 2.0 ** -60):
        every = p(scale)
        rows = np.arange(p.new)[::-37][::-1]
        # rows whose scores stay where exp has an answer
        small = np.abs(p.values[rows]).max(-1) * scale < 2.0 ** 3
        got = torch.where(torch.from_numpy(small).cuda()[..., None], every[rows], 0.0)
        want = p.c.attention(p.values[rows], 0, scale, p.sees(rows))
        want = [np.where(small[..., None] if w.ndim == 3 else small, w, 0.0) for w in want]
        check(got, *want, dtype, DIM, f"{scale}")
        assert every.isfinite().all()
        assert small[:, 5].all() and (scale != 2.0 ** -100 or small[:, 6].all())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_not_finite_blocks_reach_their_readers_only(dtype):
    p = Prompt(np.random.default_rng(32), dtype, many_rows() + 200)
    k_head, v_head, both = 3, 77, 120
    sees = {}
    for kind, head, block in (("k", k_head, 20), ("v", v_head, 30), ("k", both, 0), ("v", both, 1)):
        p.c.scale[kind][p.c.table[0, block], head] = float("nan")
        sees[head] = min(sees.get(head, 10 ** 9), block * BLOCK)
    out = p()
    poisoned = torch.zeros((p.new, HEADS), dtype=torch.bool)
    for head, first in sees.items():
        poisoned[:, head] = torch.arange(p.new) + 200 + 1 > first
    assert poisoned[:, both].all() and not poisoned[:, k_head].all() and poisoned[-1, v_head]
    assert (out.isnan().all(-1).cpu() == poisoned).all() and (out.isnan().any(-1).cpu() == poisoned).all()
    clean = np.setdiff1d(np.arange(HEADS), list(sees))
    p.check(out, heads=clean)
    for head, first in sees.items():
        rows = np.arange(0, max(0, first - 200), 11)
        if len(rows):
            p.check(out, heads=[head], rows=rows)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_blocks_outside_the_cache_are_left_out(dtype):
    """Missing ones at the start, in the middle, as the only ones that a row sees, and a whole batch of 64."""
    p = Prompt(np.random.default_rng(33), dtype, 2400, dim=128)
    bad = [0, 1, 7, *range(64, 128), 140]
    p.c.table[0, bad] = np.resize([-1, p.c.n_blocks, 2 ** 31 - 1, -2 ** 31], len(bad))
    p.c.block_table = dev(p.c.table)
    p.check(p())
    assert pq.pq_paged_device_error(p.ctx.handle) == 2
    p = Prompt(np.random.default_rng(34), dtype, many_rows())
    p.c.table[0, :3] = -1                                   # the first 48 rows see nothing at all
    p.c.block_table = dev(p.c.table)
    out = p()
    assert (out[:48] == 0).all()
    p.check(out, rows=np.arange(40, p.new, 29))
    assert pq.pq_paged_device_error(p.ctx.handle) == 2


@pytest.mark.parametrize("length", [0, 1, 50, 300, 383])
def test_rows_before_the_first_token_get_zeros(length):
    """More rows than tokens: whole tiles, whole wavefronts and single rows that see nothing."""
    p = Prompt(np.random.default_rng(35), "f16", max(length, 1))
    p.c.lengths[0] = length
    p.c.seq_len = dev([length])
    out = p()
    assert (out[:p.new - length] == 0).all()
    p.check(out, rows=np.arange(max(0, p.new - length - 1), p.new, 17))
    assert pq.pq_paged_device_error(p.ctx.handle) == 0


def test_answers_repeat_bit_for_bit():
    for dtype in ("f16", "f32"):
        p = Prompt(np.random.default_rng(36), dtype, 1500)
        first = p()
        for _ in range(3):
            assert torch.equal(p(), first)


def test_replays_from_a_graph():
    """Lengths, tables and inputs change between replays, with eager calls in between."""
    rng = np.random.default_rng(37)
    p = Prompt(rng, "f16", 1800)
    other = [Prompt(rng, "f16", n) for n in (many_rows(), 1750, 900)]
    q, out = p.q.cuda(), torch.zeros((p.new, HEADS, DIM), dtype=torch.float16, device="cuda")
    table, length = p.c.block_table, p.c.seq_len
    start, n = dev([0, p.new]), dev([p.new])
    view = (p.c.data["k"], p.c.data["v"], p.c.scale["k"], p.c.scale["v"])

    def call():
        pq.pq_paged_prefill(p.ctx.handle, 1, p.new, q, HEADS * DIM, *view, table, length, start, n, SCALE, out)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call()
    for step, x in enumerate([*other, *other]):
        rows = x.c.n_blocks
        for kind in "kv":
            p.c.data[kind][:rows].copy_(x.c.data[kind])
            p.c.scale[kind][:rows].copy_(x.c.scale[kind])
        table.fill_(-1)
        table[0, :x.c.width].copy_(x.c.block_table[0])
        length.copy_(x.c.seq_len)
        q.copy_(x.q)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        x.check(out, every=97)
        again = out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(again, out), step
    assert pq.pq_paged_device_error(p.ctx.handle) == 0
