"""pq_paged_fork, pq_paged_free, pq_paged_compact and pq_paged_copy against the plain model: whole numbers and bytes, all equal."""
import numpy as np
import pytest
import torch

import paper_2504_03661_amd as pq
from oracle import paged_oracle as O
from tests.paged_inputs import context, dev

pytestmark = pytest.mark.gpu


def requests(rng, lengths, block, spare, width=None, shared=0):
    """Tables of requests of these lengths, the first `shared` tokens (whole blocks) of every second one the same; the free
    blocks, and the counts of holders."""
    lengths = np.asarray(lengths)
    used = -(-lengths // block)
    width = int(max(1, used.max())) if width is None else width
    n_shared = shared // block
    joins = (np.arange(len(lengths)) % 2 == 0) & (used >= n_shared) & (n_shared > 0)
    own = used - np.where(joins, n_shared, 0)
    n_held = int(own.sum()) + (n_shared if joins.any() else 0)
    n_blocks = n_held + spare
    order = rng.permutation(n_blocks)
    table, holders, at = np.full((len(lengths), width), -1), np.zeros(n_blocks, int), n_shared if joins.any() else 0
    if joins.any():
        holders[order[:n_shared]] = joins.sum() - 1
    for b in range(len(lengths)):
        first = n_shared if joins[b] else 0
        table[b, :first] = order[:first]
        table[b, first:used[b]] = order[at:at + own[b]]
        at += own[b]
    free = np.full(n_blocks, -7)
    free[:spare] = order[at:]
    return table, free, holders


class State:
    """Arrays of a call on the device; new lengths and counts in arrays of their own, or in the same."""

    def __init__(self, lengths, table, free, count, holders, block, same):
        self.seqs, self.block, self.n_blocks = len(lengths), block, len(free)
        self.seq_len, self.table, self.free, self.count, self.holders = dev(lengths), dev(table), dev(free), dev([count]), dev(holders)
        self.new_len = self.seq_len if same else torch.full_like(self.seq_len, 77)
        self.new_count = self.count if same else torch.full_like(self.count, 77)
        self.ctx = context("f16", 1, 1, 64, block, self.n_blocks, np.shape(table)[1], self.seqs)

    def equal(self, want, **got):
        got = {"new_seq_len": self.new_len, "new_free_count": self.new_count, **got}
        for name, t in got.items():
            np.testing.assert_array_equal(t.cpu().numpy(), want[name], err_msg=name)

    def reported(self):
        return pq.pq_paged_device_error(self.ctx.handle)


def do_fork(s, parent, keep=None):
    src, dst = (torch.full((s.seqs,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    pq.pq_paged_fork(s.ctx.handle, s.seqs, dev(parent), None if keep is None else dev(keep), s.seq_len, s.free, s.count, s.table,
                     s.holders, s.new_len, s.new_count, src, dst)
    return src, dst


def check_fork(rng, parent, keep, lengths, block, spare, same=False, width=None, count=None, spoil=0):
    table, free, holders = requests(rng, lengths, block, spare, width)
    for _ in range(spoil):                                    # numbers outside the cache, in tables and in the list
        b = int(rng.choice(np.nonzero(np.asarray(lengths) > 0)[0]))
        table[b, rng.integers(-(-lengths[b] // block))] = rng.choice([-1, len(free), 2 ** 31 - 1, -2 ** 31])
    count = spare if count is None else count
    s = State(lengths, table, free, count, holders, block, same)
    want = O.fork(parent, keep, lengths, free, count, table, holders, block)
    src, dst = do_fork(s, parent, keep)
    s.equal(want, block_table=s.table, holders=s.holders, copy_src=src, copy_dst=dst)
    np.testing.assert_array_equal(s.free.cpu().numpy(), free)
    assert s.reported() == (1 if want["refused"] else 0) | (2 if want["outside"] else 0)
    return want


@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("same", [False, True])
def test_fork_lengths_around_a_block(block, same):
    rng = np.random.default_rng(block)
    lengths = [0, 1, block - 1, block, block + 1, 5 * block, 5 * block + 3] + [0] * 14
    parent = [-1] * 7 + [0, 1, 2, 3, 4, 5, 6, 6, 6, -5, 16, 3, 5, 4]           # (request 16 is none of the forks of another)
    want = check_fork(rng, parent, None, lengths, block, 12, same)
    assert (want["new_seq_len"][7:14] == lengths[:7]).all()
    keep = rng.integers(-1, 6 * block, len(lengths))
    check_fork(rng, parent, keep, lengths, block, 12, same)
    check_fork(rng, parent, [2 ** 31 - 1] * 20 + [-2 ** 31], lengths, block, 12, same)


@pytest.mark.parametrize("count", [0, 1, 3, 8, -4, 100])
def test_fork_refuses_what_finds_no_block(count):
    """Also: requests that are not empty, parents that are none, a fork's fork."""
    rng = np.random.default_rng(1)
    lengths = [20, 16, 40, 0, 0, 0, 0, 0, 0, 0, 0]
    parent = [-1, 0, -1, 2, 1, 0, 3, 11, 2 ** 31 - 1, 2, 9]
    want = check_fork(rng, parent, None, lengths, 16, 8, count=count)
    assert want["refused"] and want["new_seq_len"][1] == 16 and want["new_seq_len"][4] == 16 and want["new_seq_len"][6] == 0


def test_fork_follows_no_number_outside_the_cache():
    rng = np.random.default_rng(2)
    for spoil in (1, 5, 30):
        lengths = list(rng.integers(1, 200, 10)) + [0] * 30
        check_fork(rng, [-1] * 10 + list(rng.integers(0, 10, 30)), None, lengths, 16, 50, spoil=spoil)


@pytest.mark.parametrize("seqs", [1, 2, 63, 64, 65, 1023, 1024, 1025, 4096])
def test_fork_any_number_of_requests(seqs):
    rng = np.random.default_rng(seqs)
    lengths = np.where(rng.random(seqs) < 0.3, rng.integers(1, 300, seqs), 0)
    lengths[0] = 100
    parent = rng.integers(-1, seqs, seqs)
    check_fork(rng, parent, np.where(rng.random(seqs) < 0.5, 2 ** 20, rng.integers(0, 300, seqs)), lengths, 16, max(1, seqs // 3), same=seqs % 2 == 0)


def test_fork_of_a_long_request_into_wide_tables():
    rng = np.random.default_rng(3)
    lengths = [300_000, 0, 7, 0, 0]
    check_fork(rng, [-1, 0, -1, 0, 2], None, lengths, 16, 5, width=40_000)


def check_free(rng, n_new, lengths, block, spare, shared=0, same=False, change=None, count=None, width=None):
    table, free, holders = requests(rng, lengths, block, spare, width, shared)
    if change is not None:
        change(table, holders)
    count = spare if count is None else count
    s = State(lengths, table, free, count, holders, block, same)
    want = O.free(n_new, lengths, free, count, table, holders, block)
    pq.pq_paged_free(s.ctx.handle, s.seqs, dev(n_new), s.seq_len, s.free, s.count, s.table, s.holders, s.new_len, s.new_count)
    s.equal(want, free_list=s.free, holders=s.holders)
    np.testing.assert_array_equal(s.table.cpu().numpy(), table)
    assert s.reported() == (8 if want["over"] else 0) | (2 if want["outside"] else 0)
    return want


@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("same", [False, True])
def test_free_gives_back_what_nobody_holds(block, same):
    rng = np.random.default_rng(block)
    lengths = [0, 1, 7 * block, 3 * block, 9 * block + 1, 100, 2000, 0, 640, 641]
    for n_new in ([-1] * 10, [1] * 10, [-1, 5, -1, 0, -3, 1, 1, -1, -2 ** 31, 1], [1, -1] * 5, [-1, 1] * 5):
        check_free(rng, n_new, lengths, block, 5, shared=3 * block, same=same)


@pytest.mark.parametrize("seqs,most,spare", [(1, 1, 1), (1, 100_000, 3), (70, 3000, 1), (1024, 200, 100), (4096, 40, 7), (300, 20_000, 270_000)])
def test_free_any_number_of_blocks(seqs, most, spare):
    """One block up to hundreds of thousands, of which each workgroup of the second half has a part."""
    rng = np.random.default_rng(seqs)
    lengths = rng.integers(0, most + 1, seqs)
    lengths[0] = most
    check_free(rng, np.where(rng.random(seqs) < 0.6, -1, 1), lengths, 16, spare, shared=most // 32 * 16)


def test_free_of_counts_and_tables_that_do_not_fit():
    """Given back more often than held, by several or by one; numbers outside; a list that is full already."""
    rng = np.random.default_rng(4)
    lengths = [160, 160, 48, 320]

    def held_once_too_few(table, holders):
        holders[holders > 0] -= 1

    def twice_in_a_table(table, holders):
        table[3, 5] = table[3, 9] = table[3, 2]
        table[1, 1] = table[2, 1]

    def outside(table, holders):
        table[0, 3], table[2, 2], table[3, 0] = -1, len(holders), 2 ** 31 - 1

    for change in (held_once_too_few, twice_in_a_table, outside):
        want = check_free(rng, [-1] * 4, lengths, 16, 4, shared=32, change=change)
        assert want["over"] or want["outside"]
    for count in (-1, 0, 30, 1000):
        check_free(rng, [-1] * 4, lengths, 16, 4, shared=64, count=count)


def test_plan_behind_free_gives_nothing_back_twice():
    rng = np.random.default_rng(5)
    lengths, n_new = [100, 100, 30, 64], [-1, 3, -1, 1]
    table, free, holders = requests(rng, lengths, 16, 9, 12, shared=48)
    s = State(lengths, table, free, 9, holders, 16, True)
    s.ctx = context("f16", 1, 1, 64, 16, s.n_blocks, 12, 4, 8)
    first = O.free(n_new, lengths, free, 9, table, holders, 16)
    then = O.plan(n_new, first["new_seq_len"], first["free_list"], first["new_free_count"][0], table, 16, 8)
    start, got, slots = dev([0] * 5), dev([0] * 4), dev([0] * 8)
    pq.pq_paged_free(s.ctx.handle, 4, dev(n_new), s.seq_len, s.free, s.count, s.table, s.holders, s.new_len, s.new_count)
    pq.pq_paged_plan(s.ctx.handle, 4, 8, dev(n_new), s.seq_len, s.free, s.count, s.table, s.new_len, s.new_count, start, got, slots)
    s.equal(then, free_list=s.free, block_table=s.table, tok_len=got, slot_map=slots)
    assert (s.holders[torch.tensor(table[1, :3]).cuda()] == 0).all() and (s.holders >= 0).all()


def check_compact(rng, lengths, block, spare, shared=0, same=False, change=None, count=None, width=None):
    table, free, holders = requests(rng, lengths, block, spare, width, shared)
    if change is not None:
        change(table, free)
    count = spare if count is None else count
    s = State(lengths, table, free, count, holders, block, same)
    want = O.compact(lengths, free, count, table, holders, block)
    fill = lambda t: t if same else torch.full_like(t, 77)
    new_free, new_table, new_holders = fill(s.free), fill(s.table), fill(s.holders)
    moved, src, dst = (torch.full((s.n_blocks,), 77, dtype=torch.int32, device="cuda") for _ in range(3))
    n = dev([77])
    pq.pq_paged_compact(s.ctx.handle, s.seqs, s.seq_len, s.free, s.count, s.table, s.holders, new_free, s.new_count, new_table,
                        new_holders, moved, src, dst, n)
    m, n_free = int(want["n_copies"][0]), int(want["new_free_count"][0])
    assert n.item() == m and s.new_count.item() == n_free
    for name, t, upto in (("copy_src", src, m), ("copy_dst", dst, m), ("new_free_list", new_free, n_free)):
        np.testing.assert_array_equal(t[:upto].cpu().numpy(), want[name], err_msg=name)
        assert (t[upto:].cpu().numpy() == (free[upto:] if same and name == "new_free_list" else 77)).all(), name
    np.testing.assert_array_equal(new_holders.cpu().numpy(), want["new_holders"])
    np.testing.assert_array_equal(moved.cpu().numpy(), want["moved_to"])
    used = -(-np.clip(np.asarray(lengths), 0, table.shape[1] * block) // block)
    mine = np.arange(table.shape[1])[None, :] < used[:, None]
    np.testing.assert_array_equal(new_table.cpu().numpy(), np.where(mine, want["new_block_table"], table if same else 77))
    assert s.reported() == (2 if want["outside"] else 0)
    return want


@pytest.mark.parametrize("same", [False, True])
@pytest.mark.parametrize("lengths,spare", [([1], 1), ([0], 1), ([0, 0], 1500), ([100, 0, 33, 1000], 3), ([5000, 16, 20_000], 900), ([64] * 70, 200)])
def test_compact_moves_the_highest_to_the_lowest(lengths, spare, same):
    rng = np.random.default_rng(len(lengths) + spare)
    for block in (16, 64):
        want = check_compact(rng, lengths, block, spare, shared=3 * block, same=same)
        assert sorted(want["moved_to"][want["moved_to"] >= 0]) == list(range(len(want["moved_to"]) - want["new_free_count"][0]))


@pytest.mark.parametrize("seqs,most,spare,count", [(4096, 50, 4000, None), (300, 30_000, 100_000, None), (64, 2000, 300, 0), (64, 2000, 300, -1),
                                                  (1, 400_000, 1, None), (3, 70, 5, 10 ** 6)])
def test_compact_any_number_of_blocks(seqs, most, spare, count):
    """Also: nothing free by the count, and a count larger than the list."""
    rng = np.random.default_rng(seqs + spare)
    lengths = rng.integers(0, most + 1, seqs)
    lengths[0] = most

    def list_of_all(table, free):
        if count is not None and count > len(free):
            free[spare:] = free[0]

    check_compact(rng, lengths, 16, spare, shared=most // 32 * 16, count=count, change=list_of_all)


@pytest.mark.parametrize("n_blocks", [1, 31, 32, 33, 1023, 1024, 4096, 16383, 16384, 16385, 65535, 65536, 65537, 262145])
def test_caches_around_what_one_workgroup_does(n_blocks):
    """free and compact of caches that are about as large as their variants take, all kinds of last words and segments."""
    rng = np.random.default_rng(n_blocks)
    for spare in sorted({n_blocks, n_blocks // 2, 1, 0}):
        lengths = [0, (n_blocks - spare) // 3 * 16, 0, 0]
        lengths[2] = (n_blocks - spare) * 16 - lengths[1]
        if max(lengths) > 2 ** 24:
            continue
        check_compact(rng, lengths, 16, spare, same=spare % 2 == 0)
        check_free(rng, [1, -1, -1, -1], lengths, 16, spare, same=spare % 2 == 0)
        check_free(rng, [1, 1, -1, -1], lengths, 16, spare)


@pytest.mark.parametrize("n_blocks", [64, 4097, 32768, 65535, 65536, 65537])
def test_few_requests_of_a_large_cache_end(n_blocks):
    """Small tables, of blocks anywhere among many, the last ones too."""
    rng = np.random.default_rng(n_blocks)
    lengths = [400, 100, 0, 33, 300]
    for n_new in ([-1, -1, -1, -1, -1], [0, -1, -1, 1, -1], [5, 5, 5, 5, 5]):
        for same in (False, True):
            check_free(rng, n_new, lengths, 16, n_blocks - 52, shared=32, same=same)


@pytest.mark.parametrize("seqs,width", [(1, 4095), (1, 4096), (1, 4097), (64, 64), (64, 65), (4096, 1), (4095, 2), (1, 7168), (1, 7169),
                                        (64, 112), (64, 113), (1024, 7)])
def test_tables_around_what_one_workgroup_does(seqs, width):
    rng = np.random.default_rng(seqs)
    lengths = np.where(rng.random(seqs) < 0.5, rng.integers(1, width * 16 + 1, seqs), 0)
    lengths[0] = width * 16
    check_free(rng, np.where(rng.random(seqs) < 0.6, -1, 1), lengths, 16, 5, shared=min(width, 3) * 16)
    check_fork(rng, rng.integers(-1, seqs, seqs), rng.integers(0, width * 16 + 1, seqs), lengths, 16, max(1, seqs // 3), width=width)


def test_compact_of_lists_and_tables_that_do_not_fit():
    rng = np.random.default_rng(6)

    def listed_twice(table, free):
        free[3] = free[7] = free[0]

    def listed_and_held(table, free):
        free[2] = table[1, 1]

    def outside(table, free):
        free[1], table[0, 2], table[1, 0] = -5, 2 ** 31 - 1, len(free)

    for change in (listed_twice, listed_and_held, outside):
        for same in (False, True):
            check_compact(rng, [300, 200, 10], 16, 40, change=change, same=same)


def caches(gen, n, heads, block, dim):
    data = [torch.randint(0, 256, (n, heads, block * dim), generator=gen, device="cuda", dtype=torch.uint8) for _ in range(2)]
    return data + [torch.randn((n, heads), generator=gen, device="cuda") for _ in range(2)]


@pytest.mark.parametrize("heads,dim,block", [(1, 64, 16), (3, 64, 32), (8, 128, 16), (5, 128, 64), (32, 128, 16), (300, 64, 16)])
def test_copy_of_blocks(heads, dim, block):
    """From a cache into another of another size, and within one; pairs passed over, numbers outside, a count."""
    gen = torch.Generator(device="cuda").manual_seed(heads)
    rng = np.random.default_rng(heads)
    ctx = context("bf16", heads, heads, dim, block, 40, 4, 2)
    for n_from, n_to, n_pairs in ((40, 40, 12), (23, 70, 20), (1, 1, 1), (200, 90, 61)):
        inside = n_from == n_to and n_from > 1
        source = caches(gen, n_from, heads, block, dim)
        target = source if inside else caches(gen, n_to, heads, block, dim)
        src = rng.permutation(n_from)[:n_pairs] if n_from >= n_pairs else rng.integers(0, n_from, n_pairs)
        dst = np.setdiff1d(np.arange(n_to), src)[:n_pairs] if inside else rng.permutation(n_to)[:n_pairs]
        n_pairs = len(dst)
        src = src[:n_pairs].copy()
        wrong = n_pairs > 8
        if wrong:
            src[3], src[5], dst[6], dst[7] = -1, n_from, n_to, -1
        for count in (None, n_pairs, 9, 1, 0, -3, n_pairs + 5):
            limit = n_pairs if count is None else min(max(count, 0), n_pairs)
            want = [t.clone() for t in target]
            for i, j in zip(src[:limit], dst[:limit]):
                if 0 <= i < n_from and 0 <= j < n_to:
                    for t, w in zip(source, want):
                        w[j] = t[i]
            pq.pq_paged_copy(ctx.handle, n_pairs, dev(src), dev(dst), None if count is None else dev([count]), n_from, *source, n_to, *target)
            for t, w in zip(target, want):
                assert torch.equal(t, w)
            assert pq.pq_paged_device_error(ctx.handle) == (2 if wrong and limit > 5 else 0)


def test_copy_of_nothing_of_all_and_to_host_memory():
    gen = torch.Generator(device="cuda").manual_seed(9)
    ctx = context("f16", 4, 4, 128, 16, 3000, 4, 2)
    source = caches(gen, 3000, 4, 16, 128)
    before = [t.clone() for t in source]
    pq.pq_paged_copy(ctx.handle, 0, None, None, None, 3000, *source, 3000, *source)
    order = torch.randperm(3000, generator=gen, device="cuda").int()
    out = [torch.empty(t.shape, dtype=t.dtype, pin_memory=True) for t in source]       # swapped out ..
    pq.pq_paged_copy(ctx.handle, 3000, order, torch.arange(3000, device="cuda").int(), None, 3000, *source, 3000, *out)
    torch.cuda.synchronize()
    for t, w in zip(out, source):
        assert torch.equal(t, w[order.long()].cpu())
    for t in source:
        t.zero_()
    pq.pq_paged_copy(ctx.handle, 3000, torch.arange(3000, device="cuda").int(), order, None, 3000, *out, 3000, *source)   # .. and in again
    assert all(torch.equal(a, b) for a, b in zip(source, before))


def test_copy_within_caches_of_more_than_4_gib():
    heads, dim, block, n = 32, 128, 64, 18_000                       # 256 KiB a block and tensor
    ctx = context("f16", heads, heads, dim, block, n, 4, 1)
    data = [torch.zeros((n, heads, block * dim), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.zeros((n, heads), device="cuda") for _ in range(2)]
    for i, t in enumerate(data + scale):
        t[n - 1], t[n - 2], t[0] = 3 + i, 5 + i, 7 + i
    pq.pq_paged_copy(ctx.handle, 3, dev([n - 1, n - 2, 0]), dev([1, n - 3, n // 2 + 1]), None, n, *data, *scale, n, *data, *scale)
    for i, t in enumerate(data + scale):
        assert (t[1] == 3 + i).all() and (t[n - 3] == 5 + i).all() and (t[n // 2 + 1] == 7 + i).all()
        assert sum(int((row != 0).sum()) for row in (t[2], t[n - 4], t[n // 2], t[n // 2 + 2])) == 0


def refused(status, call, *args):
    with pytest.raises(pq.PQAttnError) as e:
        call(*args)
    assert e.value.status == status


def test_refusals_launch_nothing():
    NULL, SHAPE, CAPACITY = -1, -2, -4
    rng = np.random.default_rng(7)
    lengths = [40, 0, 20]
    table, free, holders = requests(rng, lengths, 16, 6)
    s = State(lengths, table, free, 6, holders, 16, True)
    h = s.ctx.handle
    extra = [dev(np.full(s.n_blocks, 5)) for _ in range(5)]
    data = torch.zeros((s.n_blocks, 1, 16 * 64), dtype=torch.uint8, device="cuda")
    scale, off = torch.zeros((s.n_blocks, 1), device="cuda"), data.flatten()[2:]
    tensors = [s.seq_len, s.table, s.free, s.count, s.holders, *extra, data, scale]
    before = [t.clone() for t in tensors]
    calls = {pq.pq_paged_fork: ([dev([-1, 0, -1]), None, s.seq_len, s.free, s.count, s.table, s.holders, s.new_len, s.new_count, *extra[:2]], [1]),
             pq.pq_paged_free: ([dev([-1, -1, -1]), s.seq_len, s.free, s.count, s.table, s.holders, s.new_len, s.new_count], []),
             pq.pq_paged_compact: ([s.seq_len, s.free, s.count, s.table, s.holders, s.free, s.new_count, s.table, s.holders, *extra[:3], s.new_count], [])}
    for call, (args, may_be_null) in calls.items():
        for i in range(len(args)):
            if i not in may_be_null:
                refused(NULL, call, h, 3, *args[:i], None, *args[i + 1:])
        refused(NULL, call, None, 3, *args)
        for n, status in ((0, SHAPE), (-1, SHAPE), (4, CAPACITY)):
            refused(status, call, h, n, *args)
    cache = [data, data, scale, scale]
    copy = [dev([0]), dev([1]), None, 4, *cache, 4, *cache]
    for i in (0, 1, 4, 5, 6, 7, 9, 10, 11, 12):
        refused(NULL, pq.pq_paged_copy, h, 1, *copy[:i], None, *copy[i + 1:])
    refused(NULL, pq.pq_paged_copy, None, 1, *copy)
    refused(SHAPE, pq.pq_paged_copy, h, -1, *copy)
    refused(CAPACITY, pq.pq_paged_copy, h, 2 ** 27, *copy)
    for i, bad, status in ((3, 0, SHAPE), (8, 0, SHAPE), (3, -1, SHAPE), (3, 2 ** 27, CAPACITY), (8, 2 ** 27, CAPACITY), (4, off, SHAPE),
                           (5, off, SHAPE), (9, off, SHAPE), (10, off, SHAPE)):
        refused(status, pq.pq_paged_copy, h, 1, *copy[:i], bad, *copy[i + 1:])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, tensors))
    assert s.reported() == 0
