"""pq_paged_decode and pq_paged_prefill against the plain model in 64 bits, within bounds derived in paged_inputs.bound."""
import math

import numpy as np
import pytest
import torch

import paper_2504_03661_amd as pq
from tests.paged_inputs import TORCH, Filled, check, context, dev, rounded

pytestmark = pytest.mark.gpu


def queries(rng, rows, Hq, dim, dtype, gap=0):
    t, values = rounded(rng.standard_normal((rows, Hq, dim)), dtype)
    wide = torch.full((rows, Hq * dim + gap), float("nan"), dtype=t.dtype)
    wide[:, :Hq * dim] = t.reshape(rows, -1)
    return wide.cuda(), values


def decode(c, ctx, q, out, scale, n=None):
    pq.pq_paged_decode(ctx.handle, len(c.lengths) if n is None else n, q, q.shape[1], *c.args(), scale, out)
    return out


def expected_decode(c, values, scale):
    parts = [c.attention(values[b:b + 1], b, scale, [c.lengths[b]]) for b in range(len(c.lengths))]
    return [np.concatenate(x) for x in zip(*parts)]


HEADS = [(1, 1), (4, 4), (8, 2), (7, 1), (32, 8), (28, 4), (16, 1), (17, 1), (40, 1)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_decode_heads_and_types(dtype, Hq, Hkv):
    rng = np.random.default_rng(Hq * 100 + Hkv)
    for dim, block in ((128, 16), (64, 32)):
        c = Filled(rng, np.array([37, 300, 0, 1]), Hkv, dim, block)
        ctx = context(dtype, Hq, Hkv, dim, block, c.n_blocks, c.width, 4)
        q, values = queries(rng, 4, Hq, dim, dtype, gap=8 * (Hq % 3))
        scale = 1.0 / math.sqrt(dim)
        out = decode(c, ctx, q, torch.full((4, Hq, dim), float("nan"), dtype=TORCH[dtype], device="cuda"), scale)
        check(out, *expected_decode(c, values, scale), dtype, dim, f"{dim}")
        assert (out[2] == 0).all()
        assert pq.pq_paged_device_error(ctx.handle) == 0


@pytest.mark.parametrize("dtype,block,dim", [("f16", 16, 128), ("bf16", 64, 128), ("f32", 32, 64), ("f16", 32, 64)])
def test_decode_lengths_around_every_border(dtype, block, dim):
    """One batch of all the lengths at which a tile, a block, a wavefront's share or a split may end."""
    rng = np.random.default_rng(block)
    lengths = sorted({max(0, m + e) for m in (0, 16, 32, 48, 64, 128, 256, 512, 1024, 1500, 2048) for e in (-1, 0, 1)})
    c = Filled(rng, np.array(lengths), 2, dim, block)
    ctx = context(dtype, 6, 2, dim, block, c.n_blocks, c.width, len(lengths))
    q, values = queries(rng, len(lengths), 6, dim, dtype)
    out = decode(c, ctx, q, torch.empty((len(lengths), 6, dim), dtype=TORCH[dtype], device="cuda"), 0.11)
    check(out, *expected_decode(c, values, 0.11), dtype, dim)


@pytest.mark.parametrize("lengths", [[9000], [20000, 3, 0, 17], [5000] * 3, [1] * 70, [33000, 100, 100, 8000, 64, 1]])
def test_decode_split_over_long_lengths(lengths):
    rng = np.random.default_rng(len(lengths))
    for dtype, Hq, Hkv in (("f16", 4, 4), ("bf16", 8, 1), ("f32", 4, 2)):
        c = Filled(rng, np.array(lengths), Hkv, 128, 16)
        ctx = context(dtype, Hq, Hkv, 128, 16, c.n_blocks, c.width, len(lengths))
        q, values = queries(rng, len(lengths), Hq, 128, dtype)
        want = expected_decode(c, values, 0.09)
        for again in range(3):                       # what one call leaves behind must not reach the next
            out = decode(c, ctx, q, torch.empty((len(lengths), Hq, 128), dtype=TORCH[dtype], device="cuda"), 0.09)
            check(out, *want, dtype, 128, f"{dtype} call {again}")


def test_fewer_sequences_than_the_context_allows():
    rng = np.random.default_rng(9)
    c = Filled(rng, np.array([700, 40, 3000]), 2, 128, 32)
    ctx = context("f16", 4, 2, 128, 32, c.n_blocks, c.width, 64)
    q, values = queries(rng, 3, 4, 128, "f16")
    want = expected_decode(c, values, 0.09)
    out = torch.full((3, 4, 128), 7.0, dtype=torch.float16, device="cuda")
    decode(c, ctx, q, out, 0.09, n=2)
    assert (out[2] == 7.0).all()
    check(out[:2], *(x[:2] for x in want), "f16", 128)


@pytest.mark.parametrize("scale", [0.0, -0.2, 4.0])
def test_scores_of_all_sizes(scale):
    """No weight but one, all weights alike, scores far below and above the others; blocks of very different scales."""
    rng = np.random.default_rng(10)
    for dtype in ("f16", "bf16", "f32"):
        c = Filled(rng, np.array([500, 2500]), 1, 128, 16)
        for kind in "kv":
            factor = np.exp2(rng.integers(-12, 6, c.model[kind].scale.shape)).astype(np.float32)
            c.model[kind].scale *= factor
            c.scale[kind].copy_(torch.from_numpy(c.model[kind].scale))
        ctx = context(dtype, 2, 1, 128, 16, c.n_blocks, c.width, 2)
        q, values = queries(rng, 2, 2, 128, dtype)
        out = decode(c, ctx, q, torch.empty((2, 2, 128), dtype=TORCH[dtype], device="cuda"), scale)
        check(out, *expected_decode(c, values, scale), dtype, 128, dtype)


def test_queries_of_extreme_sizes():
    """bf16 and fp32 reach where fp16 does not: very large and very small queries, rows of zeros, one large element."""
    rng = np.random.default_rng(11)
    for dtype in ("bf16", "f32"):
        c = Filled(rng, np.array([300] * 5), 1, 64, 16)
        ctx = context(dtype, 1, 1, 64, 16, c.n_blocks, c.width, 5)
        x = rng.standard_normal((5, 1, 64))
        x[0] *= 1e30
        x[1] *= 1e-30
        x[2] = 0.0
        x[3, 0, 5] = 3e4
        x[4] *= 1e-3
        t, values = rounded(x, dtype)
        for scale, rows in ((1e-31, [0, 2]), (1.0, [1, 2, 4]), (1e29, [1, 2]), (0.01, [3])):
            out = torch.empty((5, 1, 64), dtype=TORCH[dtype], device="cuda")
            pq.pq_paged_decode(ctx.handle, 5, t.cuda(), 64, *c.args(), scale, out)
            want = expected_decode(c, values, float(np.float32(scale)))
            check(out[rows], *(w[rows] for w in want), dtype, 64, f"{dtype} {scale}")


def test_not_finite_blocks_reach_their_readers_only():
    rng = np.random.default_rng(12)
    c = Filled(rng, np.array([100, 100, 100]), 2, 128, 16)
    c.scale["k"][c.table[0, 2], 0] = float("nan")
    c.scale["v"][c.table[1, 6], 1] = float("nan")
    ctx = context("f16", 4, 2, 128, 16, c.n_blocks, c.width, 3)
    q, values = queries(rng, 3, 4, 128, "f16")
    out = decode(c, ctx, q, torch.zeros((3, 4, 128), dtype=torch.float16, device="cuda"), 0.09)
    poisoned = torch.zeros((3, 4), dtype=torch.bool)
    poisoned[0, :2] = poisoned[1, 2:] = True
    assert (out.cpu().isnan().all(-1) == poisoned).all()
    want = expected_decode(c, values, 0.09)
    clean = ~poisoned.numpy()
    check(out[~poisoned.cuda()], *(w[clean] for w in want), "f16", 128)
    # a prompt whose first rows do not see the block
    q, values = queries(rng, 100, 4, 128, "f16")
    out = torch.zeros((100, 4, 128), dtype=torch.float16, device="cuda")
    ctx = context("f16", 4, 2, 128, 16, c.n_blocks, c.width, 3, 100)
    pq.pq_paged_prefill(ctx.handle, 1, 100, q, q.shape[1], *c.args(), dev([0, 100]), dev([100]),
                        0.09, out)
    assert not out[:32].isnan().any() and out[32:, :2].isnan().all() and not out[:, 2:].isnan().any()
    args = list(c.args())
    args[4], args[5] = args[4][1:], args[5][1:]
    pq.pq_paged_prefill(ctx.handle, 1, 100, q, q.shape[1], *args, dev([0, 100]), dev([100]), 0.09, out)
    assert not out[:96].isnan().any() and out[96:, 2:].isnan().all() and not out[:, :2].isnan().any()


def test_blocks_outside_the_cache_are_left_out():
    rng = np.random.default_rng(13)
    c = Filled(rng, np.array([90, 90, 20]), 1, 128, 16)
    c.table[0, 3], c.table[1, 0], c.table[1, 5] = -1, c.n_blocks, 2 ** 31 - 1
    c.table[2] = -2 ** 31
    c.block_table = dev(c.table)
    for dtype in ("f16", "f32"):
        ctx = context(dtype, 3, 1, 128, 16, c.n_blocks, c.width, 3, 30)
        q, values = queries(rng, 3, 3, 128, dtype)
        out = decode(c, ctx, q, torch.empty((3, 3, 128), dtype=TORCH[dtype], device="cuda"), 0.09)
        check(out, *expected_decode(c, values, 0.09), dtype, 128)
        assert (out[2] == 0).all()
        assert pq.pq_paged_device_error(ctx.handle) == 2
        q, values = queries(rng, 30, 3, 128, dtype)
        out = torch.empty((30, 3, 128), dtype=TORCH[dtype], device="cuda")
        pq.pq_paged_prefill(ctx.handle, 3, 30, q, q.shape[1], *c.args(), dev([0, 10, 20, 30]), dev([10, 10, 10]), 0.09, out)
        for b in range(3):
            check(out[10 * b:10 * b + 10], *c.attention(values[10 * b:10 * b + 10], b, 0.09, c.lengths[b] - 9 + np.arange(10)), dtype, 128)
        assert pq.pq_paged_device_error(ctx.handle) == 2


def test_lengths_outside_the_table_are_clamped():
    rng = np.random.default_rng(14)
    c = Filled(rng, np.array([48, 48]), 1, 64, 16, width=3)
    ctx = context("f16", 1, 1, 64, 16, c.n_blocks, c.width, 2)
    q, values = queries(rng, 2, 1, 64, "f16")
    want = expected_decode(c, values, 0.1)
    c.seq_len = dev([2 ** 31 - 1, -2 ** 31])
    out = decode(c, ctx, q, torch.empty((2, 1, 64), dtype=torch.float16, device="cuda"), 0.1)
    check(out[:1], *(w[:1] for w in want), "f16", 64)
    assert (out[1] == 0).all()


def prefill_case(rng, dtype, Hq, Hkv, dim, block, lengths, new, scale=0.1, gap=0, lead=0, tail=0, every=1):
    """`lead` and `tail`: rows before the first and behind the last sequence's, that belong to nobody.  `every`: of a
    sequence's rows the last and every such one before it are compared, the others are to be finite."""
    lengths, new = np.asarray(lengths), np.asarray(new)
    c = Filled(rng, lengths, Hkv, dim, block)
    start = lead + np.concatenate([[0], np.cumsum(new)])
    rows = int(start[-1]) + tail
    ctx = context(dtype, Hq, Hkv, dim, block, c.n_blocks, c.width, len(lengths), rows)
    q, values = queries(rng, rows, Hq, dim, dtype, gap)
    out = torch.full((rows, Hq, dim), 7.0, dtype=TORCH[dtype], device="cuda")
    pq.pq_paged_prefill(ctx.handle, len(lengths), rows, q, q.shape[1], *c.args(), dev(start), dev(new), scale, out)
    assert (out[:lead] == 7.0).all() and (out[rows - tail:] == 7.0).all()
    for b in range(len(lengths)):
        i = np.arange(new[b])[::-every][::-1]
        if len(i):
            part = int(start[b]) + i
            check(out[part], *c.attention(values[part], b, scale, lengths[b] - new[b] + i + 1), dtype, dim, f"sequence {b}")
            assert out[int(start[b]):int(start[b]) + int(new[b])].isfinite().all()
    assert pq.pq_paged_device_error(ctx.handle) == 0
    return c, ctx, q, out, start


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_prefill_heads_and_types(dtype, Hq, Hkv):
    rng = np.random.default_rng(Hq + 50)
    for dim, block in ((128, 16), (64, 64)):
        prefill_case(rng, dtype, Hq, Hkv, dim, block, [70, 20, 0, 33], [70, 5, 0, 1], gap=8 * (Hq % 2), lead=2, tail=3)


@pytest.mark.parametrize("dtype,dim,block", [("f16", 128, 32), ("bf16", 64, 16), ("f32", 128, 64)])
@pytest.mark.parametrize("lengths,new", [([1], [1]), ([257], [257]), ([2], [2]), ([129, 64, 65, 1], [129, 64, 65, 1]),
                                         ([1000, 31, 400], [3, 31, 128]), ([2500], [17]), ([600] * 9, [1, 2, 3, 0, 5, 0, 7, 8, 64])])
def test_prefill_lengths(dtype, dim, block, lengths, new):
    prefill_case(np.random.default_rng(sum(lengths)), dtype, 4, 2, dim, block, lengths, new)


def test_prefill_of_few_rows_over_a_long_cache():
    for dtype in ("f16", "f32"):
        prefill_case(np.random.default_rng(20), dtype, 4, 1, 128, 16, [12000, 300, 5003], [5, 20, 33])


LONG = [("f16", 128, 64), ("bf16", 128, 32), ("f32", 128, 16), ("f32", 128, 64), ("bf16", 64, 64), ("f16", 64, 16)]


@pytest.mark.parametrize("dtype,dim,block", LONG)
@pytest.mark.parametrize("heads,lengths,new", [
    ((4, 2), [140, 130], [151, 3]),
    ((4, 1), [140], [300]),
    ((64, 64), [75], [400]),
    ((128, 128), [70], [257]),
    ((128, 128), [70, 3], [401, 2]),    # from here on more than a chip of 256 compute units takes in tiles of 32 rows
    ((128, 64), [67], [521]),
])
def test_prefill_of_many_rows_over_a_long_cache(dtype, dim, block, heads, lengths, new):
    """More than 256 rows of a KV head, over more than one batch of 64 blocks (lengths in blocks): tiles of all kinds, cut along the
    keys and whole."""
    prefill_case(np.random.default_rng(26), dtype, *heads, dim, block, [n * block - 9 for n in lengths], new, every=37)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("heads,seqs,longest", [
    ((7, 1), 140, 900),
    ((28, 4), 100, 700),
    ((56, 8), 100, 700),                # the longer ones in tiles of 256 rows
    ((4, 2), 70, 6000),                 # few tiles of very different lengths
])
def test_prefill_of_many_ragged_sequences(dtype, heads, seqs, longest):
    """More sequences than a wavefront looks at in one go, of which some bring many rows, most a few and some none."""
    rng = np.random.default_rng(seqs)
    lengths = rng.integers(0, longest, seqs)
    lengths[[3, seqs - 2]] = 3 * longest
    new = np.minimum(lengths, np.where(rng.random(seqs) < 0.2, rng.integers(20, 120, seqs), rng.integers(0, 5, seqs)))
    prefill_case(rng, dtype, *heads, 64, 16, lengths, new, gap=8, lead=1, tail=2, every=11)


def test_prefill_of_one_token_is_decode():
    rng = np.random.default_rng(21)
    lengths = [1, 40, 3001]
    for dtype in ("f16", "bf16", "f32"):
        c, ctx, q, out, _ = prefill_case(rng, dtype, 8, 2, 128, 16, lengths, [1, 1, 1])
        got = decode(c, ctx, q, torch.empty_like(out), 0.1)
        off = (got.double() - out.double()).abs().max().item()
        assert off <= {"f16": 2e-3, "bf16": 1.6e-2, "f32": 1e-5}[dtype] * float(out.double().abs().max()), off


def test_prefill_rows_before_the_first_token_get_zeros():
    """More rows than tokens: the first of them attend over nothing.  Rows beyond the tensors are left out."""
    rng = np.random.default_rng(22)
    c = Filled(rng, np.array([5, 60]), 2, 128, 16)
    ctx = context("f16", 4, 2, 128, 16, c.n_blocks, c.width, 2, 40)
    q, values = queries(rng, 40, 4, 128, "f16")
    out = torch.full((40, 4, 128), 7.0, dtype=torch.float16, device="cuda")
    pq.pq_paged_prefill(ctx.handle, 2, 40, q, q.shape[1], *c.args(), dev([0, 8, 60]), dev([8, 52]), 0.1, out)
    assert (out[:3] == 0).all()
    check(out[:8], *c.attention(values[:8], 0, 0.1, np.arange(8) - 2), "f16", 128)
    check(out[8:], *c.attention(values[8:], 1, 0.1, 60 - 52 + 1 + np.arange(32)), "f16", 128)


@pytest.mark.parametrize("start,count", [([-5, 2], [4, 3]), ([39, 2], [5, 0]), ([2 ** 31 - 1, 0], [2 ** 31 - 1, 2]), ([0, 0], [-3, 2]),
                                         ([-2 ** 31, 4], [2 ** 31 - 1, 2])])
def test_prefill_keeps_to_the_rows_it_has(start, count):
    rng = np.random.default_rng(23)
    c = Filled(rng, np.array([64, 64]), 1, 64, 16)
    ctx = context("f16", 1, 1, 64, 16, c.n_blocks, c.width, 2, 40)
    q, values = queries(rng, 40, 1, 64, "f16")
    room = torch.full((48, 1, 64), 7.0, dtype=torch.float16, device="cuda")
    out = room[4:44]
    pq.pq_paged_prefill(ctx.handle, 2, 40, q, q.shape[1], *c.args(), dev(start + [0]), dev(count), 0.1, out)
    torch.cuda.synchronize()
    assert (room[:4] == 7.0).all() and (room[44:] == 7.0).all()
    for b in (1,):
        if count[b] > 0:
            part = slice(start[b], start[b] + count[b])
            check(out[part], *c.attention(values[part], b, 0.1, 64 - count[b] + 1 + np.arange(count[b])), "f16", 64)


def test_sequences_whose_rows_overlap_stay_within_memory():
    """What comes out is nobody's, but no row outside is written and the next call is right."""
    rng = np.random.default_rng(25)
    c = Filled(rng, np.array([3000] * 60), 2, 64, 16)
    ctx = context("f16", 4, 2, 64, 16, c.n_blocks, c.width, 60, 40)
    q, values = queries(rng, 40, 4, 64, "f16")
    room = torch.full((48, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    pq.pq_paged_prefill(ctx.handle, 60, 40, q, q.shape[1], *c.args(), dev([0] * 61), dev([40] * 60), 0.1, room[4:44])
    torch.cuda.synchronize()
    assert (room[:4] == 7.0).all() and (room[44:] == 7.0).all()
    pq.pq_paged_prefill(ctx.handle, 1, 40, q, q.shape[1], *c.args(), dev([0, 40]), dev([40]), 0.1, room[4:44])
    check(room[4:44], *c.attention(values, 0, 0.1, 2961 + np.arange(40)), "f16", 64)


def test_a_cache_of_more_than_4_gib():
    """Offsets beyond 32 bits: blocks at the far end of a cache of 4.5 GiB a tensor."""
    Hkv, dim, block = 32, 128, 64
    per_block = Hkv * dim * block
    n_blocks = (9 << 29) // per_block
    table = np.array([[n_blocks - 1, 0, n_blocks - 7]])
    ctx = context("f16", Hkv, Hkv, dim, block, n_blocks, 3, 1, 150)
    data = [torch.full((n_blocks, Hkv, block * dim), 128, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.full((n_blocks, Hkv), float("nan"), device="cuda") for _ in range(2)]
    rng = np.random.default_rng(24)
    x = [rounded(rng.standard_normal((150, Hkv, dim)), "f16") for _ in range(2)]
    slots = table[0, np.arange(150) // block] * block + np.arange(150) % block
    pq.pq_paged_append(ctx.handle, 150, x[0][0].cuda(), x[1][0].cuda(), Hkv * dim, dev(slots), *data, *scale)
    view = (*data, *scale, dev(table), dev([150]))
    rows = [torch.zeros((1, Hkv, 150, dim), dtype=torch.float16, device="cuda") for _ in range(2)]
    pq.pq_paged_read(ctx.handle, 1, 150, *view, None, *rows)
    held = [r[0].double().cpu().numpy() for r in rows]
    for h, (_, values) in zip(held, x):
        assert np.abs(h - values.transpose(1, 0, 2)).max() <= 0.51 * np.abs(values).max() / 127 + 2.0 ** -9
    q, values = queries(rng, 150, Hkv, dim, "f16")
    out = torch.empty((150, Hkv, dim), dtype=torch.float16, device="cuda")
    pq.pq_paged_prefill(ctx.handle, 1, 150, q, q.shape[1], *view, dev([0, 150]), dev([150]), 0.09, out)
    last = torch.empty((1, Hkv, dim), dtype=torch.float16, device="cuda")
    pq.pq_paged_decode(ctx.handle, 1, q[149:], q.shape[1], *view, 0.09, last)
    for h in range(Hkv):                             # against what was read back: half a step of each value more
        t = held[0][h] @ values[149, h] * 0.09
        p = np.exp(t - t.max())
        want = (p / p.sum()) @ held[1][h]
        for got in (out[149, h], last[0, h]):
            assert np.abs(got.double().cpu().numpy() - want).max() <= 0.01
