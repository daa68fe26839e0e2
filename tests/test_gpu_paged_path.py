"""The paged cache as a program uses it: the calls one after another, from a graph, on other streams, into the product-quantized
cache, and what they refuse."""
import math

import numpy as np
import pytest
import torch

import paper_2504_03661_amd as pq
from oracle import paged_oracle as O
from oracle import pq_oracle
from tests.paged_inputs import TORCH, check, context, dev, rounded

pytestmark = pytest.mark.gpu


class Server:
    """Device state of a few requests, and the plain model of all of it."""

    def __init__(self, dtype, Hq, Hkv, dim, block, n_blocks, width, seqs, tokens, seed=0):
        self.dtype, self.Hq, self.Hkv, self.dim, self.block, self.seqs, self.tokens = dtype, Hq, Hkv, dim, block, seqs, tokens
        self.rng = np.random.default_rng(seed)
        self.scale = float(np.float32(1 / math.sqrt(dim)))
        self.ctx = context(dtype, Hq, Hkv, dim, block, n_blocks, width, seqs, tokens)
        self.cache = [torch.full((n_blocks, Hkv, block * dim), 128, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.scales = [torch.full((n_blocks, Hkv), float("nan"), device="cuda") for _ in range(2)]
        self.table, self.free = dev(np.full((seqs, width), -1)), dev(np.arange(n_blocks))
        self.length, self.count = dev(np.zeros(seqs)), dev([n_blocks])
        self.start, self.got, self.slots = dev(np.zeros(seqs + 1)), dev(np.zeros(seqs)), dev(np.zeros(tokens))
        self.n_new = dev(np.zeros(seqs))
        kind = TORCH[dtype]
        self.qkv = torch.zeros((tokens, (Hq + 2 * Hkv) * dim), dtype=kind, device="cuda")     # as one product gives them
        self.out = torch.zeros((tokens, Hq, dim), dtype=kind, device="cuda")
        self.out1 = torch.zeros((seqs, Hq, dim), dtype=kind, device="cuda")
        self.model = [O.Cache(n_blocks, Hkv, block, dim) for _ in range(2)]
        self.state = {"block_table": np.full((seqs, width), -1), "new_seq_len": np.zeros(seqs, int),
                      "free_list": np.arange(n_blocks), "new_free_count": [n_blocks]}

    def view(self):
        return (*self.cache, *self.scales, self.table, self.length)

    def parts(self):
        q, k, v = self.qkv.split([self.Hq * self.dim, self.Hkv * self.dim, self.Hkv * self.dim], 1)
        return q, k, v, self.qkv.shape[1]

    def plan(self, tokens):
        pq.pq_paged_plan(self.ctx.handle, self.seqs, tokens, self.n_new, self.length, self.free, self.count, self.table,
                         self.length, self.count, self.start, self.got, self.slots)

    def append(self, tokens):
        _, k, v, stride = self.parts()
        pq.pq_paged_append(self.ctx.handle, tokens, k, v, stride, self.slots, *self.cache, *self.scales)

    def prefill(self, tokens):
        q, _, _, stride = self.parts()
        pq.pq_paged_prefill(self.ctx.handle, self.seqs, tokens, q, stride, *self.view(), self.start, self.got, self.scale, self.out)

    def decode(self):
        q, _, _, stride = self.parts()
        pq.pq_paged_decode(self.ctx.handle, self.seqs, q, stride, *self.view(), self.scale, self.out1)

    def step(self, tokens):
        self.plan(tokens)
        self.append(tokens)
        self.prefill(tokens)

    def inputs(self, n_new):
        """Draws the step's rows; returns their values as the model takes them."""
        self.n_new.copy_(dev(n_new))
        tokens = int(np.maximum(n_new, 0).sum())
        t, values = rounded(self.rng.standard_normal((self.tokens, self.qkv.shape[1])), self.dtype)
        self.qkv.copy_(t)
        q = values[:, :self.Hq * self.dim].reshape(self.tokens, self.Hq, self.dim)
        kv = values[:, self.Hq * self.dim:].reshape(self.tokens, 2, self.Hkv, self.dim)
        return tokens, q, kv

    def follow(self, n_new, tokens, kv):
        s = self.state
        self.state = s = O.plan(n_new, s["new_seq_len"], s["free_list"], s["new_free_count"][0], s["block_table"], self.block, tokens)
        for i in range(2):
            self.model[i].append(kv[:tokens, i], s["slot_map"])
        return s

    def rows(self, b):
        n = int(self.state["new_seq_len"][b])
        (k, there), (v, _) = (m.rows(self.state["block_table"][b], n) for m in self.model)
        return k, v, there

    def check_plan(self, tokens):
        s = self.state
        for name, t in (("new_seq_len", self.length), ("new_free_count", self.count), ("block_table", self.table),
                        ("tok_start", self.start), ("tok_len", self.got), ("free_list", self.free)):
            np.testing.assert_array_equal(t.cpu().numpy(), s[name], err_msg=name)
        np.testing.assert_array_equal(self.slots[:tokens].cpu().numpy(), s["slot_map"])

    def check_cache(self):
        for i in range(2):
            for b in range(self.seqs):
                n = int(self.state["new_seq_len"][b])
                held = self.state["block_table"][b][:-(-n // self.block)]
                got = O.Cache.from_bytes(self.cache[i][held.tolist()].cpu().numpy(), self.scales[i][held.tolist()].cpu().numpy(),
                                         self.block, self.dim, i == 1)
                np.testing.assert_array_equal(got.scale, self.model[i].scale[held])
                x = got.codes.transpose(1, 0, 2, 3).reshape(self.Hkv, -1, self.dim)[:, :n]
                y = self.model[i].codes[held].transpose(1, 0, 2, 3).reshape(self.Hkv, -1, self.dim)[:, :n]
                np.testing.assert_array_equal(x, y)

    def check_prefill(self, q, out):
        s = self.state
        for b in range(self.seqs):
            n = int(s["tok_len"][b])
            if n:
                part = slice(int(s["tok_start"][b]), int(s["tok_start"][b]) + n)
                k, v, there = self.rows(b)
                check(out[part], *O.attention(q[part], k, v, there, self.scale, k.shape[1] - n + 1 + np.arange(n)), self.dtype, self.dim, f"sequence {b}")

    def check_decode(self, q, out):
        for b in range(self.seqs):
            k, v, there = self.rows(b)
            check(out[b:b + 1], *O.attention(q[b:b + 1], k, v, there, self.scale, [k.shape[1]]), self.dtype, self.dim, f"sequence {b}")


@pytest.mark.parametrize("dtype,dim,block", [("f16", 128, 16), ("bf16", 64, 32), ("f32", 128, 64)])
def test_requests_come_grow_and_end(dtype, dim, block):
    """Prompts, chunks, single steps, refusals, ends and blocks that change hands."""
    s = Server(dtype, 6, 2, dim, block, 19 * 32 // block, 640 // block, 5, 700, seed=dim)
    steps = [[100, 0, 7, 33, 1], [1, 64, 1, 1, 1], [1, 1, -1, 40, 1], [-1, 1, 90, 1, -1], [130, 1, 1, 1, 20], [600, -1, 1, 60, 5],
             [1, 12, 1, 1, -1], [1, 1, 1, 1, 33]]
    for n_new in steps:
        n_new = np.array(n_new)
        tokens, q, kv = s.inputs(n_new)
        s.out.fill_(7.0)
        s.step(tokens)
        s.follow(n_new, tokens, kv)
        s.check_plan(tokens)
        s.check_cache()
        s.check_prefill(q, s.out)
        for b in range(s.seqs):                               # rows of refused requests: as they were
            if s.state["tok_len"][b] == 0:
                assert (s.out[int(s.state["tok_start"][b]):int(s.state["tok_start"][b + 1])] == 7.0).all()
        s.decode()
        s.check_decode(q, s.out1)


def graph_of(call):
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    return graph


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_step_replays_from_a_graph(dtype):
    """plan, append, prefill and decode recorded once; every replay on other lengths and inputs, with eager work between."""
    s = Server(dtype, 8, 2, 128, 16, 400, 160, 4, 4 * 90, seed=3)
    n_new = np.array([90, 5, 0, 17])
    tokens, q, kv = s.inputs(n_new)
    s.step(360)                                               # rows behind the last request's belong to nobody
    s.follow(n_new, 360, kv)
    graph = graph_of(lambda: (s.step(360), s.decode()))
    for step, n_new in enumerate([[1, 1, 1, 1], [90, 90, 90, 90], [1, 0, 1, -1], [2, 3, 4, 5], [1, 1, 1, 1], [0, 0, 0, 0], [90, -1, 1, 90], [1, 7, 1, 1]]):
        n_new = np.array(n_new)
        _, q, kv = s.inputs(n_new)
        s.out.fill_(7.0)
        s.out1.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        s.follow(n_new, 360, kv)
        s.check_plan(360)
        s.check_cache()
        s.check_prefill(q, s.out)
        s.check_decode(q, s.out1)
        again = s.out1.clone()
        s.decode()                                            # eager, on the same context
        torch.cuda.synchronize()
        off = (again.double() - s.out1.double()).abs().max().item()
        assert off <= (1e-6 if dtype == "f32" else 2.0 ** -9), (step, off)


def test_long_caches_replay_from_a_graph():
    """Splits of decode, pieces and merges of prefill, and how many there are change between replays."""
    s = Server("f16", 4, 1, 64, 64, 900, 800, 3, 3 * 64, seed=4)
    graph = None
    for step, length in enumerate([[20000, 40, 0], [300, 30000, 7], [64, 64, 64], [50000, 1, 900], [1000, 0, 0]]):
        s.length.copy_(dev(length))
        rng = np.random.default_rng(step)
        held = rng.permutation(900)
        table, at = np.full((3, 800), -1), 0
        for b, n in enumerate(length):
            used = -(-n // 64)
            table[b, :used] = held[at:at + used]
            at += used
        s.table.copy_(dev(table))
        data = rng.integers(1, 256, (2, 900, 1, 64 * 64), dtype=np.uint8)
        scale = np.exp2(rng.uniform(-7, -5, (2, 900, 1))).astype(np.float32)
        for i in range(2):
            s.cache[i].copy_(torch.from_numpy(data[i]))
            s.scales[i].copy_(torch.from_numpy(scale[i]))
            s.model[i] = O.Cache.from_bytes(data[i], scale[i], 64, 64, i == 1)
        new = np.minimum(length, [3, 64, 40][step % 3])
        s.start.copy_(dev(np.concatenate([[0], np.cumsum(new)])))
        s.got.copy_(dev(new))
        s.state = {"tok_start": np.concatenate([[0], np.cumsum(new)]), "tok_len": new, "new_seq_len": np.array(length), "block_table": table}
        _, q, _ = s.inputs(np.zeros(3))
        call = lambda: (s.prefill(192), s.decode())
        if graph is None:
            call()
            graph = graph_of(call)
        for again in range(3):
            s.out.fill_(7.0)
            s.out1.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            s.check_prefill(q, s.out)
            s.check_decode(q, s.out1)


def test_another_stream_than_the_tensors_own():
    s = Server("bf16", 4, 2, 128, 32, 60, 20, 3, 200, seed=5)
    n_new = np.array([70, 100, 30])
    tokens, q, kv = s.inputs(n_new)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(tokens)
        s.decode()
    torch.cuda.current_stream().wait_stream(side)
    s.follow(n_new, tokens, kv)
    s.check_cache()
    s.check_prefill(q, s.out)
    s.check_decode(q, s.out1)


def test_two_contexts_on_two_streams_at_once():
    """Each has its own scratch: long decodes that run side by side do not meet."""
    servers = []
    for seed in (6, 7):
        s = Server("f16", 8, 2, 128, 16, 1300, 1300, 1, 16, seed=seed)
        rng = np.random.default_rng(seed)
        data, scale = rng.integers(1, 256, (2, 1300, 2, 16 * 128), dtype=np.uint8), np.exp2(rng.uniform(-7, -5, (2, 1300, 2))).astype(np.float32)
        for i in range(2):
            s.cache[i].copy_(torch.from_numpy(data[i]))
            s.scales[i].copy_(torch.from_numpy(scale[i]))
            s.model[i] = O.Cache.from_bytes(data[i], scale[i], 16, 128, i == 1)
        table = rng.permutation(1300)[None]
        s.table.copy_(dev(table))
        s.length.copy_(dev([20000]))
        s.start.copy_(dev([0, 16]))
        s.got.copy_(dev([16]))
        s.state = {"tok_start": [0, 16], "tok_len": [16], "new_seq_len": [20000], "block_table": table}
        servers.append((s, s.inputs(np.zeros(1))[1], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for s, _, stream in servers:
            with torch.cuda.stream(stream):
                s.decode()
                s.prefill(16)
    torch.cuda.synchronize()
    for s, q, _ in servers:
        s.check_decode(q, s.out1)
        s.check_prefill(q, s.out)


def test_tokens_read_back_go_into_the_product_quantized_cache():
    """A prompt is attended and kept in 8 bits, then its tokens become product-quantized codes and are attended there."""
    Hkv, dim, n = 4, 128, 300
    s = Server("f16", Hkv, Hkv, dim, 16, 40, 20, 2, 2 * n, seed=8)
    n_new = np.array([n, n])
    tokens, q, kv = s.inputs(n_new)
    s.step(tokens)
    s.follow(n_new, tokens, kv)
    k, v = (torch.empty((2, Hkv, n, dim), dtype=torch.float16, device="cuda") for _ in range(2))
    pq.pq_paged_read(s.ctx.handle, 2, n, *s.view(), None, k, v)
    cfg = pq.PQAttnConfig(batch=2, n_q_heads=Hkv, n_kv_heads=Hkv, max_context=512)
    ctx = pq.pq_attn_create(cfg)
    try:
        codebooks = [s.rng.standard_normal((Hkv, 64, 256, 2)).astype(np.float16) for _ in range(2)]
        codes = [torch.zeros(pq.pq_attn_codes_bytes(cfg), dtype=torch.uint8, device="cuda") for _ in range(2)]
        length = dev([0, 0])
        pq.pq_attn_set_codebooks(ctx, *(torch.from_numpy(c).cuda() for c in codebooks))
        pq.pq_encode_append(ctx, k, v, n, None, None, *codes, length)
        query = torch.from_numpy(s.rng.standard_normal((2, Hkv, dim)).astype(np.float16)).cuda()
        out = torch.empty((2, Hkv, dim), device="cuda")
        pq.pq_attn_decode(ctx, query, *codes, length, None, None, None, None, None, s.scale, out)
        got = out.cpu().numpy()
    finally:
        torch.cuda.synchronize()
        pq.pq_attn_destroy(ctx)
    encoded = [pq_oracle.encode(x.cpu().numpy(), c) for x, c in zip((k, v), codebooks)]
    ref = pq_oracle.decode(query.cpu().numpy(), *encoded, np.full(2, n, np.int32), *codebooks, None, None, np.zeros(2, np.int32), scale=s.scale)
    assert np.abs(got - ref).max() <= 2e-3
    for i, x in enumerate((k, v)):                            # and what was read is what the model holds
        for b in range(2):
            want = s.model[i].rows(s.state["block_table"][b], n)[0]
            assert np.abs(x[b].double().cpu().numpy() - want).max() <= np.abs(want).max() * 2.0 ** -11


# --------------------------------------------------------------------------------------------------------- refusals

def refused(status, call, *args):
    with pytest.raises(pq.PQAttnError) as e:
        call(*args)
    assert e.value.status == status


def test_refusals_launch_nothing():
    s = Server("f16", 4, 2, 64, 16, 10, 4, 3, 32, seed=9)
    tensors = [*s.cache, s.table, s.free, s.length, s.count, s.start, s.got, s.slots, s.out, s.out1]
    before = [t.clone() for t in tensors]
    q, k, v, stride = s.parts()
    h, off = s.ctx.handle, s.qkv.view(torch.uint8).flatten()[2:]       # an address that 16 does not divide
    state = (s.n_new, s.length, s.free, s.count, s.table, s.length, s.count, s.start, s.got, s.slots)
    NULL, SHAPE, CAPACITY = -1, -2, -4
    for i in range(10):
        refused(NULL, pq.pq_paged_plan, h, 3, 8, *state[:i], None, *state[i + 1:])
    refused(NULL, pq.pq_paged_plan, None, 3, 8, *state)
    for n, tokens, status in ((0, 8, SHAPE), (-1, 8, SHAPE), (4, 8, CAPACITY), (3, -1, SHAPE), (3, 33, CAPACITY)):
        refused(status, pq.pq_paged_plan, h, n, tokens, *state)

    append = (k, v, stride, s.slots, *s.cache, *s.scales)
    for i in (0, 1, 3, 4, 5, 6, 7):
        refused(NULL, pq.pq_paged_append, h, 8, *append[:i], None, *append[i + 1:])
    refused(SHAPE, pq.pq_paged_append, h, -1, *append)
    refused(CAPACITY, pq.pq_paged_append, h, 33, *append)
    for i, bad in ((0, off), (1, off), (2, 127), (2, 132), (2, -stride), (2, 2 ** 31), (4, off), (5, off)):
        refused(SHAPE, pq.pq_paged_append, h, 8, *append[:i], bad, *append[i + 1:])

    out = torch.zeros((3, 2, 4, 64), dtype=torch.float16, device="cuda")
    read = (*s.view(), None, out, out)
    for i in (0, 1, 2, 3, 4, 5, 7, 8):
        refused(NULL, pq.pq_paged_read, h, 3, 4, *read[:i], None, *read[i + 1:])
    for n, rows, status in ((0, 4, SHAPE), (4, 4, CAPACITY), (3, -1, SHAPE), (3, 2 ** 24 + 1, CAPACITY)):
        refused(status, pq.pq_paged_read, h, n, rows, *read)
    for i in (0, 1, 7, 8):
        refused(SHAPE, pq.pq_paged_read, h, 3, 4, *read[:i], off, *read[i + 1:])
    pq.pq_paged_read(h, 3, 0, *s.view(), None, None, None)             # no rows: nothing to do

    decode = (q, stride, *s.view(), 0.1, s.out1)
    for i in (0, 2, 3, 4, 5, 6, 7, 9):
        refused(NULL, pq.pq_paged_decode, h, 3, *decode[:i], None, *decode[i + 1:])
    refused(SHAPE, pq.pq_paged_decode, h, 0, *decode)
    refused(CAPACITY, pq.pq_paged_decode, h, 4, *decode)
    for i, bad in ((0, off), (1, 255), (1, 260), (2, off), (3, off), (8, float("nan")), (8, float("inf")), (9, off)):
        refused(SHAPE, pq.pq_paged_decode, h, 3, *decode[:i], bad, *decode[i + 1:])

    prefill = (q, stride, *s.view(), s.start, s.got, 0.1, s.out)
    for i in (0, 2, 3, 4, 5, 6, 7, 8, 9, 11):
        refused(NULL, pq.pq_paged_prefill, h, 3, 8, *prefill[:i], None, *prefill[i + 1:])
    for n, tokens, status in ((0, 8, SHAPE), (4, 8, CAPACITY), (3, -1, SHAPE), (3, 33, CAPACITY)):
        refused(status, pq.pq_paged_prefill, h, n, tokens, *prefill)
    for i, bad in ((0, off), (1, 255), (2, off), (3, off), (10, float("nan")), (11, off)):
        refused(SHAPE, pq.pq_paged_prefill, h, 3, 8, *prefill[:i], bad, *prefill[i + 1:])
    pq.pq_paged_prefill(h, 3, 0, None, stride, *s.view(), s.start, s.got, 0.1, None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, tensors))
    assert torch.stack(s.scales).isnan().all()
    assert pq.pq_paged_device_error(h) == 0


def test_read_refuses_more_than_a_launch_has_threads():
    ctx = context("f16", 8, 8, 64, 16, 4, 2, 64)
    length, table = dev([20] * 64), dev([[0, 1]] * 64)
    data, scale = torch.zeros(4 * 8 * 16 * 64, dtype=torch.uint8, device="cuda"), torch.zeros((4, 8), device="cuda")
    out = torch.full((16,), 3.0, dtype=torch.float16, device="cuda")
    for rows in (2 ** 21 - 7, 2 ** 24):                                 # 64 x 8 x (rows + 8) x 64 against 2^36
        refused(-4, pq.pq_paged_read, ctx.handle, 64, rows, data, data, scale, scale, table, length, None, out, out)
    torch.cuda.synchronize()
    assert (out == 3.0).all()


def test_a_context_ends_with_its_object():
    c = context("f16", 2, 1, 64, 16, 4, 2, 1)
    assert c.handle
    c.close()
    c.close()
    assert c.handle is None
    refused(-1, pq.pq_paged_destroy, None)
    with pq.PQPaged(c.cfg) as again:
        assert pq.pq_paged_device_error(again.handle) == 0
    assert again.handle is None
