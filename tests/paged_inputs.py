"""Inputs and bounds that the tests of the paged 8-bit cache share."""
import numpy as np
import torch

import paper_2504_03661_amd as pq
from oracle import paged_oracle as O

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
PQ = {"f16": pq.PQ_F16, "bf16": pq.PQ_BF16, "f32": pq.PQ_F32}
#: half a step of a rounding to the type, relative
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).cuda()


def rounded(a, dtype):
    """As the storage type holds it: a CPU tensor of that type and its values in double."""
    t = torch.as_tensor(np.asarray(a, np.float32)).to(TORCH[dtype])
    return t, t.to(torch.float64).numpy()


def context(dtype, Hq, Hkv, dim, block, n_blocks, width, seqs, tokens=1):
    return pq.PQPaged(pq.PQPagedConfig(max_seqs=seqs, max_tokens=max(1, tokens), n_q_heads=Hq, n_kv_heads=Hkv, head_dim=dim,
                                       block_tokens=block, n_blocks=n_blocks, max_blocks=width, dtype=PQ[dtype]))


class Filled:
    """A cache of random codes and scales with block tables for the given lengths, on the device and as the oracle has it.
    Blocks that no sequence holds have NaN scales: whoever reads one shows it."""

    def __init__(self, rng, lengths, Hkv, dim, block, spare=3, width=None):
        lengths = np.asarray(lengths)
        used = -(-lengths // block)
        self.width = int(max(1, used.max())) if width is None else width
        self.n_blocks, self.block, self.dim = int(used.sum()) + spare, block, dim
        order = rng.permutation(self.n_blocks)
        self.table = np.full((len(lengths), self.width), -1)
        self.table[np.arange(self.width)[None, :] < used[:, None]] = order[:used.sum()]
        self.lengths = lengths
        self.data, self.scale, self.model = {}, {}, {}
        for kind in "kv":
            scale = np.exp2(rng.uniform(-7.0, -5.0, (self.n_blocks, Hkv))).astype(np.float32)
            scale[order[used.sum():]] = np.nan
            data = rng.integers(1, 256, (self.n_blocks, Hkv, block * dim), dtype=np.uint8)
            self.model[kind] = O.Cache.from_bytes(data, scale, block, dim, kind == "v")
            self.data[kind], self.scale[kind] = dev(data, torch.uint8), dev(scale, torch.float32)
        self.seq_len, self.block_table = dev(lengths), dev(self.table)

    def args(self):
        return self.data["k"], self.data["v"], self.scale["k"], self.scale["v"], self.block_table, self.seq_len

    def attention(self, q, b, scale, sees):
        n = int(self.lengths[b])
        k, there = self.model["k"].rows(self.table[b], n)
        v, _ = self.model["v"].rows(self.table[b], n)
        return O.attention(q, k, v, there, scale, sees)


def bound(dtype, out, spread, size, peak, dim):
    """How far an output may be off.  A score is a sum of `dim` products in fp32 and a few fp32 operations on it (scale, block
    scale, the maximum, the exponent's base): its error is at most (dim + 16) 2^-24 times the sum of the products' sizes, the
    same number is the weight's relative error, and numerator and denominator both have it.  Weights are rounded to 11 bits
    (fp32 outputs: to 21) before they meet V, those below 2^-27 of the largest to a step of 2^-38 of it (the largest of these
    caches' codes in a row is at least half of what codes can be: 2^-37 of a token's largest value), and sums of them are
    fp32.  Then half a step of the output's type, which for fp16 is never less than 2^-25."""
    weights = 2.0 ** -11 if dtype != "f32" else 2.0 ** -21
    per_score = (dim + 16) * 2.0 ** -24 * (size[..., None] + 1.0)
    smallest = 2.0 ** -25 if dtype == "f16" else 1e-30
    return spread * (2.0 * per_score + weights + 2.0 ** -19) + peak[..., None] * 2.0 ** -37 + HALF_STEP[dtype] * np.abs(out) * 1.01 + smallest


def check(got, out, spread, size, peak, dtype, dim, what=""):
    got = got.to(torch.float64).cpu().numpy()
    far = np.abs(got - out) - bound(dtype, out, spread, size, peak, dim)
    assert np.isfinite(got).all(), what
    assert far.max(initial=-1.0) <= 0.0, f"{what}: {far.max():.3e} over the bound at {np.unravel_index(far.argmax(), far.shape)}"
