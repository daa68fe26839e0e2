"""The largest shapes that a context takes."""
import numpy as np
import pytest
import torch

import paper_2504_03661_amd as pq
from tests.paged_inputs import TORCH, Filled, bound, check, context, dev, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(1024, 1), (1024, 1024), (1022, 2)])
def test_a_thousand_query_heads(dtype, Hq, Hkv):
    """All of one KV head, one each, and groups that nothing divides; a token, a few and a hundred."""
    rng = np.random.default_rng(Hkv)
    for new in (1, 3, 100):
        c = Filled(rng, np.array([150]), Hkv, 64, 16)
        ctx = context(dtype, Hq, Hkv, 64, 16, c.n_blocks, c.width, 1, new)
        q, values = rounded(rng.standard_normal((new, Hq, 64)), dtype)
        out = torch.full((new, Hq, 64), 7.0, dtype=TORCH[dtype], device="cuda")
        rows = np.unique([0, new // 2, new - 1])
        want = c.attention(values[rows], 0, 0.1, 150 - new + 1 + rows)
        pq.pq_paged_prefill(ctx.handle, 1, new, q.cuda(), Hq * 64, *c.args(), dev([0, new]), dev([new]), 0.1, out)
        check(out[rows], *want, dtype, 64, f"prefill {new}")
        assert out.isfinite().all()
        if new == 1:
            out.fill_(7.0)
            pq.pq_paged_decode(ctx.handle, 1, q.cuda(), Hq * 64, *c.args(), 0.1, out)
            check(out, *want, dtype, 64, "decode")


def test_four_thousand_sequences():
    """Lengths from 0 on, of which some need several chunks; as decode, and as prefill of 0 to 3 tokens."""
    rng = np.random.default_rng(50)
    lengths = rng.integers(0, 40, 4096)
    lengths[[0, 63, 64, 4095]] = 3000, 0, 1500, 2000
    c = Filled(rng, lengths, 2, 64, 16)
    new = np.minimum(lengths, rng.integers(0, 4, 4096))
    rows = int(new.sum())
    ctx = context("f16", 4, 2, 64, 16, c.n_blocks, c.width, 4096, rows)
    q, values = rounded(rng.standard_normal((4096, 4, 64)), "f16")
    out = torch.full((4096, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    pq.pq_paged_decode(ctx.handle, 4096, q.cuda(), 256, *c.args(), 0.1, out)
    for b in [*range(0, 4096, 41), 63, 64, 4095]:
        check(out[b:b + 1], *c.attention(values[b:b + 1], b, 0.1, [lengths[b]]), "f16", 64, f"sequence {b}")
    start = np.concatenate([[0], np.cumsum(new)])
    q, values = rounded(rng.standard_normal((rows, 4, 64)), "f16")
    out = torch.full((rows, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    pq.pq_paged_prefill(ctx.handle, 4096, rows, q.cuda(), 256, *c.args(), dev(start), dev(new), 0.1, out)
    for b in [*range(0, 4096, 41), 63, 64, 4095]:
        i = np.arange(new[b])
        if len(i):
            check(out[start[b] + i], *c.attention(values[start[b] + i], b, 0.1, lengths[b] - new[b] + i + 1), "f16", 64, f"sequence {b}")
    assert pq.pq_paged_device_error(ctx.handle) == 0


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("heads,new,length", [(1, 1, 1 << 24), (1, 3, 1 << 24), (128, 401, 1 << 19)])
def test_sequences_as_long_as_a_table_can_say(dtype, heads, new, length):
    """A table that names the same four blocks over and over: all rounds but the last, which a row may see in part, have the same weights.

    Beside what paged_inputs.bound has, sums of a wavefront over a share of the keys are added up 16 keys at a time, each time to
    half a unit in the last place: (share / 16) 2^-24 of the numerator's size and as much of the denominator.  One KV head's keys are cut
    into 64 pieces for four wavefronts each; in tiles of 256 rows they are not cut."""
    rng = np.random.default_rng(51)
    c = Filled(rng, np.array([64]), heads, 64, 16)
    table = np.resize(c.table[0], (1, length // 16))
    ctx = context(dtype, heads, heads, 64, 16, c.n_blocks, length // 16, 1, new)
    q, values = rounded(rng.standard_normal((new, heads, 64)), dtype)
    view = (*c.args()[:4], dev(table), dev([length]))
    rows = np.arange(new)[::-37][::-1]
    k, v = (c.model[kind].rows(c.table[0], 64)[0] for kind in "kv")
    want, spread, size, peak = (np.zeros((len(rows), heads, 64)), np.zeros((len(rows), heads, 64)), np.zeros((len(rows), heads)),
                                np.zeros((len(rows), heads)))
    for i, r in enumerate(rows):
        sees = length - new + r + 1
        times = sees // 64 + (np.arange(64) < sees % 64)      # how often the row sees each of the 64
        for h in range(heads):
            t = k[h] @ values[r, h] * 0.1
            p = times * np.exp(t - t.max())
            p /= p.sum()
            want[i, h], spread[i, h] = p @ v[h], p @ np.abs(v[h])
            size[i, h] = (np.abs(k[h]) @ np.abs(values[r, h])).max() * 0.1
            peak[i, h] = (p / times * np.abs(v[h]).max(-1)).max() * sees
    share = length / (64 * 4) if heads == 1 else length
    allowed = bound(dtype, want, spread, size, peak, 64) + 2.0 * share / 16 * 2.0 ** -24 * spread
    calls = {"prefill": lambda out: pq.pq_paged_prefill(ctx.handle, 1, new, q.cuda(), heads * 64, *view, dev([0, new]), dev([new]), 0.1, out)}
    if new == 1:
        calls["decode"] = lambda out: pq.pq_paged_decode(ctx.handle, 1, q.cuda(), heads * 64, *view, 0.1, out)
    for name, call in calls.items():
        out = torch.full((new, heads, 64), 7.0, dtype=TORCH[dtype], device="cuda")
        call(out)
        assert out.isfinite().all()
        off = np.abs(out[rows].double().cpu().numpy() - want)
        assert (off <= allowed).all(), (name, (off / allowed).max())
    assert pq.pq_paged_device_error(ctx.handle) == 0
