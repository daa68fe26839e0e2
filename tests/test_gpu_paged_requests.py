"""Requests that share blocks as a program uses them: prompts, samples, beams, ends, a cache that is tidied up and made smaller —
fork, copy, plan, append, shared_decode, free and compact one after another, eagerly, from graphs and on other streams."""
import numpy as np
import pytest
import torch

import paper_2504_03661_amd as pq
from oracle import paged_oracle as O
from tests.paged_inputs import check, dev
from tests.test_gpu_paged_path import Server, graph_of
from tests.test_gpu_paged_shared import work

pytestmark = pytest.mark.gpu


class Sampler(Server):
    """A server whose requests share blocks, and the plain model of that."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        n_blocks = self.free.shape[0]
        self.holders, self.parent, self.keep = dev(np.zeros(n_blocks)), dev(np.full(self.seqs, -1)), dev(np.zeros(self.seqs))
        self.src, self.dst = dev(np.full(n_blocks, -1)), dev(np.full(n_blocks, -1))
        self.moved, self.n_copies = dev(np.zeros(n_blocks)), dev([0])
        self.members, self.group_start, self.shared = dev(np.arange(self.seqs)), dev(np.zeros(self.seqs + 1)), dev(np.zeros(self.seqs))
        self.workspace = work(self.ctx, self.seqs, self.seqs)
        self.state["holders"] = np.zeros(n_blocks, int)

    def copy(self, n, count=None):
        cache, n_blocks = [*self.cache, *self.scales], self.free.shape[0]
        pq.pq_paged_copy(self.ctx.handle, n, self.src, self.dst, count, n_blocks, *cache, n_blocks, *cache)

    def fork(self):
        pq.pq_paged_fork(self.ctx.handle, self.seqs, self.parent, self.keep, self.length, self.free, self.count, self.table, self.holders,
                         self.length, self.count, self.src, self.dst)
        self.copy(self.seqs)

    def end(self):
        pq.pq_paged_free(self.ctx.handle, self.seqs, self.n_new, self.length, self.free, self.count, self.table, self.holders,
                         self.length, self.count)

    def compact(self):
        pq.pq_paged_compact(self.ctx.handle, self.seqs, self.length, self.free, self.count, self.table, self.holders, self.free,
                            self.count, self.table, self.holders, self.moved, self.src, self.dst, self.n_copies)
        self.copy(self.free.shape[0], self.n_copies)

    def shared_decode(self, n_groups):
        q, _, _, stride = self.parts()
        pq.pq_paged_shared_decode(self.ctx.handle, self.seqs, n_groups, q, stride, *self.view(), self.members, self.group_start,
                                  self.shared, self.scale, self.workspace, self.workspace.numel(), self.out1)

    # the model's side of each

    def follow_copies(self, src, dst):
        for m in self.model:
            for i, j in zip(src, dst):
                if i >= 0:
                    m.codes[j], m.scale[j] = m.codes[i], m.scale[i]

    def take(self, got):
        for name, value in got.items():
            self.state["block_table" if name == "new_block_table" else name] = value

    def follow_fork(self, parent, keep):
        s = self.state
        got = O.fork(parent, keep, s["new_seq_len"], s["free_list"], s["new_free_count"][0], s["block_table"], s["holders"], self.block)
        self.follow_copies(got["copy_src"], got["copy_dst"])
        self.take(got)
        return got

    def follow_free(self, n_new):
        s = self.state
        got = O.free(n_new, s["new_seq_len"], s["free_list"], s["new_free_count"][0], s["block_table"], s["holders"], self.block)
        assert not got["over"]
        self.take(got)

    def follow_compact(self):
        s = self.state
        got = O.compact(s["new_seq_len"], s["free_list"], s["new_free_count"][0], s["block_table"], s["holders"], self.block)
        self.follow_copies(got["copy_src"], got["copy_dst"])
        listed = np.array(s["free_list"])
        listed[:len(got["new_free_list"])] = got["new_free_list"]
        self.take({**got, "free_list": listed, "holders": got["new_holders"]})

    def follow_step(self, n_new, tokens, kv):
        held = self.state["holders"]
        self.follow(n_new, tokens, kv)
        self.state["holders"] = held

    def groups_of(self):
        """Requests whose tables begin with the same block, and how many blocks all of such a group share; set on the device."""
        s, groups = self.state, {}
        for b in range(self.seqs):
            if s["new_seq_len"][b] > 0:
                groups.setdefault(int(s["block_table"][b, 0]), []).append(b)
        groups = list(groups.values())
        shared = []
        for g in groups:
            n = min(int(s["new_seq_len"][b]) for b in g) // self.block
            rows = s["block_table"][g, :n]
            same = (rows == rows[0]).all(0)
            shared.append((n if same.all() else int(same.argmin())) * self.block)
        order = [b for g in groups for b in g]
        self.members.copy_(dev(order + [0] * (self.seqs - len(order))))
        start = np.cumsum([0] + [len(g) for g in groups])
        self.group_start.copy_(dev(np.concatenate([start, np.full(self.seqs - len(groups), start[-1])])))
        self.shared.copy_(dev(shared + [0] * (self.seqs - len(groups))))
        return len(groups), max(shared, default=0)

    def check_all(self):
        s = self.state
        for name, t in (("new_seq_len", self.length), ("new_free_count", self.count), ("holders", self.holders)):
            np.testing.assert_array_equal(t.cpu().numpy(), s[name], err_msg=name)
        n = int(s["new_free_count"][0])
        np.testing.assert_array_equal(self.free[:n].cpu().numpy(), s["free_list"][:n])
        for b in range(self.seqs):
            used = -(-int(s["new_seq_len"][b]) // self.block)
            np.testing.assert_array_equal(self.table[b, :used].cpu().numpy(), s["block_table"][b, :used])
        self.check_cache()

    def check_shared(self, q, n_groups):
        self.out1.fill_(7.0)
        self.shared_decode(n_groups)
        alive = [b for b in range(self.seqs) if self.state["new_seq_len"][b] > 0]
        for b in alive:
            k, v, there = self.rows(b)
            check(self.out1[b:b + 1], *O.attention(q[b:b + 1], k, v, there, self.scale, [k.shape[1]]), self.dtype, self.dim, f"sequence {b}")
        for b in set(range(self.seqs)) - set(alive):
            assert (self.out1[b] == 7.0).all()


def one_each(s):
    return np.where(s.state["new_seq_len"] > 0, 1, 0)


@pytest.mark.parametrize("dtype,dim,block,Hq,Hkv", [("f16", 128, 16, 6, 2), ("bf16", 64, 32, 4, 4), ("f32", 128, 64, 17, 1)])
def test_prompts_samples_beams_and_ends(dtype, dim, block, Hq, Hkv):
    s = Sampler(dtype, Hq, Hkv, dim, block, 60 * 32 // block, 1024 // block, 9, 700, seed=dim)
    n_new = np.array([300, 0, 0, 0, 161, 0, 0, 0, 5])
    tokens, q, kv = s.inputs(n_new)
    s.step(tokens)
    s.follow_step(n_new, tokens, kv)
    forks = [[-1, 0, 0, -1, -1, 4, 4, 0, -1], [-1, -1, -1, 8, -1, -1, -1, -1, -1], [-1, 1, 1, -1, 1, -1, -1, 7, -1],
             [0, -1, 0, -1, -1, 4, 2, 4, 1], [-1] * 9]
    keeps = [[999, 999, 999, 999, 999, 999, 100, 64, 0], [2] * 9, [999] * 9, [999, 999, 70, 999, 999, 30, 999, 999, 999], [0] * 9]
    ends = [[], [0, 2], [8, 3, 5], [6, 1], [0, 1, 2, 4, 5, 6, 7, 8]]
    saw_shared = 0
    for round_, (parent, keep, gone) in enumerate(zip(forks, keeps, ends)):
        s.parent.copy_(dev(parent))
        s.keep.copy_(dev(keep))
        s.fork()
        s.follow_fork(parent, keep)
        s.check_all()
        for _ in range(3):
            n_new = one_each(s)
            tokens, q, kv = s.inputs(n_new)
            s.plan(tokens)
            s.append(tokens)
            s.follow_step(n_new, tokens, kv)
            s.check_plan(tokens)
            n_groups, shared = s.groups_of()
            saw_shared = max(saw_shared, shared)
            s.check_shared(q, n_groups)
        if round_ % 2 == 1:
            s.compact()
            s.follow_compact()
            s.check_all()
            s.check_shared(q, s.groups_of()[0])
        n_new = np.array([-1 if b in gone else 0 for b in range(9)])
        s.n_new.copy_(dev(n_new))
        s.end()
        s.follow_free(n_new)
        s.check_all()
    assert saw_shared >= 64
    n_new = np.full(9, -1)
    s.n_new.copy_(dev(n_new))
    s.end()
    s.follow_free(n_new)
    s.compact()
    s.follow_compact()
    s.check_all()
    assert s.count.item() == s.free.shape[0] and (s.holders == 0).all()
    assert pq.pq_paged_device_error(s.ctx.handle) == 1         # (the refused forks of requests that were not empty)


def test_steps_forks_and_ends_replay_from_graphs():
    """One graph of fork and copy, one of a step with shared_decode, one of ends and compact: replayed in turn on other lengths, with
    eager calls and synchronizations between them."""
    s = Sampler("f16", 8, 2, 128, 16, 300, 64, 6, 6 * 8, seed=11)
    n_new = np.array([8, 0, 0, 7, 0, 0])
    for _ in range(12):
        tokens, q, kv = s.inputs(n_new)
        s.plan(48)
        s.append(48)
        s.follow_step(n_new, 48, kv)
    s.groups_of()
    s.shared_decode(6)
    graphs = {"fork": graph_of(s.fork), "step": graph_of(lambda: (s.plan(48), s.append(48), s.shared_decode(6))),
              "end": graph_of(lambda: (s.end(), s.compact()))}
    torch.cuda.synchronize()
    for parent, gone in (([-1, 0, 0, -1, 3, -1], []), ([-1, -1, -1, -1, -1, 4], [0, 2]), ([1, -1, 5, -1, -1, -1], [3, 4, 1])):
        s.parent.copy_(dev(parent))
        s.keep.copy_(dev([1000, 1000, 50, 1000, 33, 1000]))
        graphs["fork"].replay()
        torch.cuda.synchronize()
        s.follow_fork(parent, [1000, 1000, 50, 1000, 33, 1000])
        s.check_all()
        for n in (1, 3, 1):
            n_new = one_each(s) * n
            _, q, kv = s.inputs(n_new)
            s.follow_step(n_new, 48, kv)
            s.groups_of()
            s.out1.fill_(7.0)
            graphs["step"].replay()
            torch.cuda.synchronize()
            s.check_all()
            first = s.out1.clone()
            s.check_shared(q, 6)                              # eager, on the same state
            assert torch.equal(first, s.out1)
        n_new = np.array([-1 if b in gone else 0 for b in range(6)])
        s.n_new.copy_(dev(n_new))
        graphs["end"].replay()
        torch.cuda.synchronize()
        s.follow_free(n_new)
        s.follow_compact()
        s.check_all()


def test_all_of_it_on_another_stream():
    s = Sampler("bf16", 4, 2, 128, 32, 60, 20, 4, 300, seed=12)
    n_new = np.array([200, 0, 0, 70])
    tokens, q, kv = s.inputs(n_new)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(tokens)
        s.follow_step(n_new, tokens, kv)
        s.parent.copy_(dev([-1, 0, 0, -1]))
        s.keep.copy_(dev([0, 150, 200, 0]))
        s.fork()
        s.follow_fork([-1, 0, 0, -1], [0, 150, 200, 0])
        n_groups, shared = s.groups_of()
        s.shared_decode(n_groups)
        first = s.out1.clone()
        s.compact()
        s.follow_compact()
        s.shared_decode(n_groups)
        s.n_new.copy_(dev([0, -1, 0, -1]))
        s.end()
        s.follow_free([0, -1, 0, -1])
    torch.cuda.current_stream().wait_stream(side)
    assert shared == 128
    assert torch.equal(first, s.out1)                         # the same blocks elsewhere
    s.check_all()


def test_a_smaller_cache_takes_the_place_of_one_that_was_compacted():
    s = Sampler("f16", 4, 2, 128, 16, 200, 40, 5, 400, seed=13)
    n_new = np.array([150, 60, 170, 0, 0])
    tokens, q, kv = s.inputs(n_new)
    s.step(tokens)
    s.follow_step(n_new, tokens, kv)
    s.parent.copy_(dev([-1, -1, -1, 2, 2]))
    s.keep.copy_(dev([999] * 5))
    s.fork()
    s.follow_fork([-1, -1, -1, 2, 2], [999] * 5)
    n_new = np.array([0, -1, 0, 0, -1])
    s.n_new.copy_(dev(n_new))
    s.end()
    s.follow_free(n_new)
    s.compact()
    s.follow_compact()
    n_live = 200 - s.count.item()
    small = Sampler("f16", 4, 2, 128, 16, n_live, 40, 5, 400, seed=14)
    every = dev(np.arange(n_live))
    pq.pq_paged_copy(small.ctx.handle, n_live, every, every, None, 200, *s.cache, *s.scales, n_live, *small.cache, *small.scales)
    small.table.copy_(s.table)
    small.length.copy_(s.length)
    small.qkv.copy_(s.qkv)
    small.state, small.model = s.state, s.model
    n_groups, shared = small.groups_of()
    assert shared == 160
    small.check_shared(q, n_groups)
    assert pq.pq_paged_device_error(small.ctx.handle) == 0
