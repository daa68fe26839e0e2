"""pq_paged_plan, pq_paged_append and pq_paged_read against the plain model: every number of a plan, every code and scale."""
import numpy as np
import pytest
import torch

import paper_2504_03661_amd as pq
from oracle import paged_oracle as O
from tests.paged_inputs import HALF_STEP, TORCH, Filled, context, dev, rounded

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------- plan

class Plan:
    def __init__(self, n_blocks, width, block, seqs, tokens):
        self.n_blocks, self.width, self.block = n_blocks, width, block
        self.ctx = context("f16", 1, 1, 64, block, n_blocks, width, seqs, tokens)

    def __call__(self, n_new, seq_len, free, count, table, n_tokens, in_place=False):
        n = len(n_new)
        d = {"seq_len": dev(seq_len), "free_list": dev(free), "free_count": dev([count]), "block_table": dev(table),
             "tok_start": dev(np.full(n + 1, -7)), "tok_len": dev(np.full(n, -7)), "slot_map": dev(np.full(n_tokens, -7))}
        d["new_seq_len"] = d["seq_len"] if in_place else dev(np.full(n, -7))
        d["new_free_count"] = d["free_count"] if in_place else dev([-7])
        pq.pq_paged_plan(self.ctx.handle, n, n_tokens, dev(n_new), d["seq_len"], d["free_list"], d["free_count"],
                         d["block_table"], d["new_seq_len"], d["new_free_count"], d["tok_start"], d["tok_len"], d["slot_map"])
        got = {k: v.cpu().numpy() for k, v in d.items()}
        got["refused"] = pq.pq_paged_device_error(self.ctx.handle) & 1
        return got


def same_plan(got, want, what=""):
    for name, value in want.items():
        np.testing.assert_array_equal(got[name], value, err_msg=f"{what} {name}")


@pytest.mark.parametrize("seqs,block,width,n_blocks,most", [(1, 16, 4, 5, 40), (7, 32, 6, 23, 70), (64, 16, 20, 700, 50),
                                                           (65, 64, 3, 90, 130)])
def test_plan_over_many_steps(seqs, block, width, n_blocks, most):
    """A server's life: every step's outputs go into the next."""
    rng = np.random.default_rng(seqs)
    plan = Plan(n_blocks, width, block, seqs, seqs * most)
    table, length, free, count = np.full((seqs, width), -1), np.zeros(seqs, int), np.arange(n_blocks)[::-1], n_blocks
    for step in range(25):
        n_new = np.where(rng.random(seqs) < 0.15, -1, rng.integers(0, most, seqs))
        n_tokens = max(0, int(np.maximum(n_new, 0).sum()) + int(rng.integers(-3, 4)))
        n_tokens = min(n_tokens, seqs * most)
        want = O.plan(n_new, length, free, count, table, block, n_tokens)
        same_plan(plan(n_new, length, free, count, table, n_tokens, in_place=step % 2 == 0), want, f"step {step}")
        table, length, free, count = want["block_table"], want["new_seq_len"], want["free_list"], int(want["new_free_count"][0])


@pytest.mark.parametrize("seqs,most,short", [(1024, 8, False), (1025, 3, True), (2100, 40, False), (4096, 2, True), (3, 20000, False), (2000, 60, True)])
def test_plan_of_many_requests_and_tokens(seqs, most, short):
    rng = np.random.default_rng(seqs + most)
    block, width = 16, max(8, -(-(100 + most) // 16))
    length = rng.integers(0, 100, seqs)
    used = -(-length // block)
    n_new = np.where(rng.random(seqs) < 0.2, -1, rng.integers(0, most + 1, seqs))
    need = (-(-(length + np.maximum(n_new, 0)) // block) - used).sum()
    spare = max(1, int(need) // 3) if short else int(need) + 5
    n_blocks = int(used.sum()) + spare
    order = rng.permutation(n_blocks)
    table = np.full((seqs, width), -1)
    table[np.arange(width)[None, :] < used[:, None]] = order[:used.sum()]
    free = np.full(n_blocks, -1)
    free[:spare] = order[used.sum():]
    n_tokens = int(np.maximum(n_new, 0).sum())
    plan = Plan(n_blocks, width, block, seqs, max(1, n_tokens))
    want = O.plan(n_new, length, free, spare, table, block, n_tokens)
    assert want["refused"] or not short or most < 60        # (with few tokens the ended requests' blocks are enough)
    same_plan(plan(n_new, length, free, spare, table, n_tokens), want)
    same_plan(plan(n_new, length, free, spare, table, n_tokens, in_place=True), want)


def test_plan_keeps_to_its_bounds():
    """Lengths, counts and block numbers that nobody should hand over: clamped, passed over, reported."""
    plan = Plan(6, 2, 16, 4, 64)
    table = np.array([[0, 99], [-5, 1], [2, 3], [-1, -1]])
    n_new, length, free, count = [2, 3, 2 ** 31 - 1, -2 ** 31], [20, 5, 0, -9], [4, 5, 0, 0, 0, 0], 2
    want = O.plan(n_new, length, free, count, table, 16, 64)
    got = plan(n_new, length, free, count, table, 64)
    same_plan(got, want)
    assert got["slot_map"].max() < 96
    want = O.plan([-1, -1, -1, 5], [32, 32, 32, 0], free, 5, table, 16, 64)      # more given back than there are blocks
    same_plan(plan([-1, -1, -1, 5], [32, 32, 32, 0], free, 5, table, 64), want)
    got = plan([1, 1, 1, 1], [0, 0, 0, 0], free, 77, table, 4)                    # a count beyond the list
    same_plan(got, O.plan([1, 1, 1, 1], [0, 0, 0, 0], free, 77, table, 16, 4))


# --------------------------------------------------------------------------------------------------- append and read

class Store:
    """A cache on the device and its model, appended to side by side."""

    def __init__(self, dtype, Hkv, dim, block, n_blocks, width=1, seqs=1, tokens=4096):
        self.dtype, self.Hkv, self.dim, self.block, self.n_blocks = dtype, Hkv, dim, block, n_blocks
        self.ctx = context(dtype, Hkv, Hkv, dim, block, n_blocks, width, seqs, tokens)
        assert pq.pq_paged_cache_bytes(self.ctx.cfg) == n_blocks * Hkv * block * dim
        self.data = [torch.full((n_blocks, Hkv, block * dim), 128, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.scale = [torch.zeros((n_blocks, Hkv), device="cuda") for _ in range(2)]
        self.model = [O.Cache(n_blocks, Hkv, block, dim) for _ in range(2)]

    def append(self, xs, slots, gap=0):
        """xs: k and v [tokens, Hkv, d]; gap: elements between the rows of the tensors that hold them."""
        rows, values = [], []
        for x in xs:
            t, v = rounded(x, self.dtype)
            flat = t.reshape(len(slots), -1).cuda()
            wide = torch.full((len(slots), flat.shape[1] + gap), float("nan"), dtype=flat.dtype, device="cuda")
            wide[:, :flat.shape[1]] = flat
            rows.append(wide)
            values.append(v)
        pq.pq_paged_append(self.ctx.handle, len(slots), rows[0], rows[1], rows[0].shape[1], dev(slots), *self.data, *self.scale)
        for model, v in zip(self.model, values):
            model.append(v, slots)

    def check(self, what=""):
        for i in range(2):
            scale = self.scale[i].cpu().numpy()
            np.testing.assert_array_equal(scale, self.model[i].scale, err_msg=f"{what} scale {'kv'[i]}")
            np.testing.assert_array_equal(self.data[i].cpu().numpy(), self.model[i].bytes(i == 1), err_msg=f"{what} codes {'kv'[i]}")


def draw(rng, n, Hkv, dim):
    return [rng.standard_normal((n, Hkv, dim)) * np.exp2(rng.uniform(-3, 2, (Hkv, dim))) for _ in range(2)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim,block", [(128, 16), (128, 32), (128, 64), (64, 16), (64, 32), (64, 64)])
def test_append_in_pieces_of_all_lengths(dtype, dim, block):
    """One sequence through blocks in shuffled order, in appends of 1 to many tokens that begin anywhere in a block."""
    rng = np.random.default_rng(dim + block)
    store = Store(dtype, 3, dim, block, 12)
    order = rng.permutation(12)
    at, sizes = 0, [1, 1, block - 2, 3, 2 * block + 5, 1, 7, 1, block, 1, 3 * block - 1]
    for n in sizes:
        p = np.arange(at, at + n)
        store.append(draw(rng, n, 3, dim), order[p // block] * block + p % block, gap=8 * (n % 3))
        at += n
        store.check(f"after {at}")


@pytest.mark.parametrize("Hkv,seqs", [(1, 40), (8, 33), (32, 5)])
def test_append_of_a_step_and_of_a_ragged_batch(Hkv, seqs):
    rng = np.random.default_rng(Hkv)
    block, width = 16, 12
    store = Store("f16", Hkv, 128, block, seqs * width)
    table = rng.permutation(seqs * width).reshape(seqs, width)
    length = np.zeros(seqs, int)
    for step, new in enumerate([rng.integers(0, 60, seqs), np.ones(seqs, int), rng.integers(0, 3, seqs), np.ones(seqs, int)]):
        owner = np.repeat(np.arange(seqs), new)
        p = np.concatenate([np.arange(a, a + n) for a, n in zip(length, new)]).astype(int)
        slots = table[owner, p // block] * block + p % block
        if step == 0:
            slots[len(slots) // 2:] = -1             # requests that have got no place
            new = np.array([(slots[owner == b] >= 0).sum() for b in range(seqs)])
        store.append(draw(rng, len(slots), Hkv, 128), slots)
        length = length + new
        store.check(f"step {step}")
    assert pq.pq_paged_device_error(store.ctx.handle) == 0


def test_append_of_a_long_prompt():
    """Enough rows that a wavefront looks through a block's worth of the slot map."""
    rng = np.random.default_rng(4)
    for block in (16, 64):
        store = Store("bf16", 8, 64, block, 160)
        order = rng.permutation(160)
        p = np.arange(5, 5 + 2311)
        store.append(draw(rng, len(p), 8, 64), order[p // block] * block + p % block)
        store.check(str(block))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim,block", [(128, 16), (128, 32), (128, 64), (64, 16), (64, 32), (64, 64)])
def test_append_of_a_ragged_batch_of_many_rows(dtype, dim, block):
    """More rows times heads than get a unit each: several sequences' tokens lie in the rows that a unit looks through, their blocks
    begin and end there, and older tokens stand in front of some."""
    rng = np.random.default_rng(dim + block + 1)
    seqs, Hkv, width = 44, 32, 6
    store = Store(dtype, Hkv, dim, block, seqs * width)
    table = rng.permutation(seqs * width).reshape(seqs, width)
    length = np.zeros(seqs, int)
    for step in range(2):
        new = np.where(rng.random(seqs) < 0.4, rng.integers(1, 4, seqs), rng.integers(0, 2 * block + 10, seqs))
        owner = np.repeat(np.arange(seqs), new)
        assert len(owner) * 2 * Hkv > 64 * 256           # (256 compute units)
        p = np.concatenate([np.arange(a, a + n) for a, n in zip(length, new)]).astype(int)
        slots = table[owner, p // block] * block + p % block
        slots[owner == 3 + step] = -1
        store.append(draw(rng, len(slots), Hkv, dim), slots, gap=8)
        length = length + new
        length[3 + step] -= new[3 + step]
        store.check(f"step {step}")
    assert pq.pq_paged_device_error(store.ctx.handle) == 0


def test_append_of_ties_small_numbers_and_what_is_not_finite():
    store = Store("f32", 6, 64, 16, 2)
    x = np.zeros((3, 6, 64), np.float32)
    x[:, 0, 0], x[0, 0, 1:7] = 127.0, [0.5, -0.5, 1.5, 63.5, np.nextafter(np.float32(63.5), np.float32(0)), -126.5]
    x[0, 1, :4] = [2.0 ** -41, 2.0 ** -40, -1e-38, 1e-45]
    x[1, 2, 3], x[1, 3, 3], x[0, 4, 0] = np.inf, np.nan, 3.0e38
    x[0, 4, 1:3] = [1.2e36, -3.0e38]
    x[1, 5, 7] = 1e-3
    store.append([x, -x], [0, 1, 2])
    store.check("anew")
    y = np.zeros((1, 6, 64), np.float32)
    y[0, :, 5] = [300.0, 2.0 ** -39, 1.0, 1.0, 3.3e38, -77.0]
    store.append([y, y], [3])
    store.check("raised")
    store.append([x, y.repeat(3, 0)], [16, 17, 18])
    store.append([y, y], [0])                       # begun anew: NaN and old scales are gone
    for model in store.model:
        model.codes[0, :, 1:] = 0                   # (what follows a new beginning is nobody's)
    for i in range(2):
        got = O.Cache.from_bytes(store.data[i].cpu().numpy(), store.scale[i].cpu().numpy(), 16, 64, i == 1)
        np.testing.assert_array_equal(got.scale, store.model[i].scale)
        np.testing.assert_array_equal(got.codes[0, :, 0], store.model[i].codes[0, :, 0])
        np.testing.assert_array_equal(got.codes[1, :, :3], store.model[i].codes[1, :, :3])


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim,block", [(128, 16), (128, 32), (128, 64), (64, 32), (64, 64)])
def test_one_value_that_is_not_finite_anywhere_in_a_block(dtype, dim, block):
    """In every piece of the block, first and last, with larger and smaller numbers in the others."""
    rng = np.random.default_rng(dim + block)
    places = [0, 1, block // 2 - 1, block // 2, block - 1] + [16 * i + 5 for i in range(block // 16)]
    store = Store(dtype, len(places), dim, block, 2)
    xs = draw(rng, block, len(places), dim)
    for h, r in enumerate(places):
        xs[0][r, h, rng.integers(dim)] = [np.nan, np.inf, -np.inf][h % 3]
        xs[1][r, h, rng.integers(dim)] = [-np.inf, np.nan, np.nan][h % 3]
    store.append(xs, np.arange(block) + block)
    store.check()
    assert np.isnan(store.model[0].scale[1]).all()


def test_append_outside_the_cache_writes_nothing():
    rng = np.random.default_rng(6)
    store = Store("f16", 2, 128, 16, 3)
    store.append(draw(rng, 6, 2, 128), [0, -1, 48, 49, 2 ** 31 - 1, 47])
    store.check()
    assert pq.pq_paged_device_error(store.ctx.handle) == 2
    assert pq.pq_paged_device_error(store.ctx.handle) == 0
    before = [t.clone() for t in store.data + store.scale]
    pq.pq_paged_append(store.ctx.handle, 0, None, None, 256, None, *store.data, *store.scale)
    assert all(torch.equal(a, b) for a, b in zip(before, store.data + store.scale))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim,block,Hkv", [(128, 16, 3), (64, 32, 1), (128, 64, 8)])
def test_read_any_rows(dtype, dim, block, Hkv):
    rng = np.random.default_rng(dim)
    lengths = np.array([0, 1, block, 3 * block + 5, 2 * block - 1])
    c = Filled(rng, lengths, Hkv, dim, block)
    ctx = context(dtype, Hkv, Hkv, dim, block, c.n_blocks, c.width, len(lengths))
    for rows, first in ((1, [0, 0, 3, 7, 2 * block - 2]), (2 * block + 3, [0, 1, 0, 5, 3]), (block, None), (7, [4, 9, block - 3, block, 1])):
        out = [torch.full((len(lengths), Hkv, rows, dim), -5.0, dtype=TORCH[dtype], device="cuda") for _ in range(2)]
        pq.pq_paged_read(ctx.handle, len(lengths), rows, *c.args(), None if first is None else dev(first), *out)
        for got, kind in zip(out, "kv"):
            got = got.to(torch.float64).cpu().numpy()
            for b, n in enumerate(lengths):
                f = 0 if first is None else first[b]
                want, _ = c.model[kind].rows(c.table[b], int(n))
                want = want[:, f:f + rows]
                assert (got[b, :, want.shape[1]:] == -5.0).all()                 # rows behind the last: as they were
                # one product, rounded once (fp16 numbers below its smallest normal one by steps of 2^-24)
                far = np.abs(got[b, :, :want.shape[1]] - want) - np.abs(want) * HALF_STEP[dtype] * 1.0001 - 2.0 ** -25
                assert far.max(initial=-1) <= 0


def test_read_passes_over_blocks_that_are_none():
    c = Filled(np.random.default_rng(8), np.array([40, 40]), 2, 64, 16)
    c.table[0, 1], c.table[1, 2] = -1, c.n_blocks
    ctx = context("f32", 2, 2, 64, 16, c.n_blocks, c.width, 2)
    out = [torch.full((2, 2, 40, 64), 9.0, device="cuda") for _ in range(2)]
    pq.pq_paged_read(ctx.handle, 2, 40, *c.args()[:4], dev(c.table), c.seq_len, None, *out)
    for got, kind in zip(out, "kv"):
        for b in range(2):
            want, there = c.model[kind].rows(c.table[b], 40)
            np.testing.assert_array_equal(got[b].cpu().numpy(), np.where(there[:, None], want, 9.0).astype(np.float32))
    assert pq.pq_paged_device_error(ctx.handle) == 2
