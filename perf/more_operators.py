"""Requests that share blocks of the paged 8-bit cache, as cases that can be timed and checked.

Many answers are drawn from one prompt, many chats begin with the same instructions: their requests can hold the same blocks of
a paged cache.  Five operators serve that:

    fork           requests that begin as copies of others: their full blocks are held together and counted, a block
                   that is not full is copied
    free           requests that end: a block goes back when its last holder has ended
    compact        live blocks moved to the lowest numbers, so that a cache can be made smaller
    copy           blocks copied within a cache, or into another one
    shared_decode  attention of one query token per request, where the blocks that a group of requests begins with are
                   read once for the group

fork and compact say which blocks are to be copied (block tables are the same for all layers of a model, the caches are not);
their cases copy those of one layer as well.

`own` says which side runs: the plain forms below, or the library's kernels through its public binding.

A case is a dict of plain values: "op", "dtype" of queries ("f16" | "bf16" | "f32"), "groups" of requests that share a prompt,
"members" of a group at most, "q_heads", "kv_heads", "dim", "block" (tokens), "prompt" (the longest shared length), "ctx"
(the longest length behind it), "ragged" (sizes spread, or all equal to the largest), "spare" (blocks that no request
holds, as a share of those held), "pairs" (blocks copied; 0: within the cache, else into one of so many blocks: "to"), and
"shape", a number that the sizes are drawn from, so that the work of a case does not depend on the seed of its values.

A cache is bytes (code + 128) [block][KV head][block * dim] and fp32 scales [block][KV head], for K and for V.  K's bytes are
[token][dim]; V's, for every 16 tokens, [dim / 64][token / 4][dim % 16][dim / 16 % 4][token % 4].  They are copied as they are.
holders[block] is the number of requests that hold a block besides the first.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _case(op, dtype="f16", groups=1, members=4, q_heads=32, kv_heads=8, dim=128, block=16, prompt=1000, ctx=0, ragged=False,
          spare=0.25, pairs=0, to=0, shape=0):
    return {"op": op, "dtype": dtype, "groups": groups, "members": members, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "block": block, "prompt": prompt, "ctx": ctx, "ragged": ragged, "spare": spare, "pairs": pairs, "to": to,
            "shape": shape}


def listed():
    cases = {
        # four answers to one question of a chat
        "fork_4_of_1k": _case("fork", shape=1),
        # a batch of 64 prompts of all lengths up to 8K, each sampled eight times, some from a part of the prompt only
        "fork_512_of_64": _case("fork", groups=64, members=8, prompt=8192, ragged=True, shape=2),
        # the end of a round of sampling: most of eight answers have come
        "free_8x1k": _case("free", members=8, ctx=100, shape=3),
        # a busy server's step: half of a thousand requests end, in groups that share prompts of up to 8K
        "free_1000x8k": _case("free", groups=125, members=8, prompt=8192, ctx=2048, ragged=True, shape=4),
        # the blocks that 64 samples cannot share
        "copy_64": _case("copy", pairs=64, shape=5),
        # long requests swapped out to make room: 8192 blocks of 32 heads into a cache of their own
        "copy_swap_8k": _case("copy", kv_heads=32, pairs=8192, to=9000, prompt=8192 * 16, ragged=True, shape=6),
        # a small cache tidied up
        "compact_2k": _case("compact", groups=6, members=4, prompt=2000, ctx=800, ragged=True, shape=7),
        # a large one, a quarter of its blocks free
        "compact_64k": _case("compact", groups=64, members=4, prompt=8000, ctx=2000, spare=0.3, shape=8),
        # four samples of a short prompt, where latency is the time
        "shared_4x1k": _case("shared_decode", prompt=1008, ctx=64, shape=9),
        # 32 samples of a long prompt
        "shared_32x8k": _case("shared_decode", members=32, prompt=8192, ctx=512, ragged=True, shape=10),
        # 256 chats that begin with the same instructions, and go on for up to 4K tokens
        "shared_256x2k": _case("shared_decode", "bf16", members=256, prompt=2048, ctx=4096, ragged=True, shape=11),
        # a full-precision program's beams over several documents, heads of 64 dims
        "shared_beams_f32": _case("shared_decode", "f32", groups=9, members=8, q_heads=28, kv_heads=4, dim=64, block=32,
                                  prompt=6000, ctx=300, ragged=True, shape=12),
    }
    return [{"name": name, **case} for name, case in cases.items()]


def _log(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["fork", "free", "compact", "copy", "shared_decode", "shared_decode"])
    kv = rng.choice([1, 2, 3, 4, 8, 8, 32])
    group = 1 if kv == 32 else rng.choice([1, 2, 4, 4, 7, 8, 16])
    dim = rng.choice([64, 128, 128])
    block = rng.choice([16, 32, 64])
    case = _case(op, rng.choice(["f16", "bf16", "f32"]), q_heads=kv * group, kv_heads=kv, dim=dim, block=block,
                 ragged=rng.random() < 0.7, spare=rng.uniform(0.1, 0.5), shape=rng.randrange(1 << 30))
    groups = _log(rng, 1, 64)
    members = _log(rng, 1, max(1, min(256, 1000 // groups)))
    row = kv * dim
    if op == "fork":
        most = min(16384, 64 * 8192 * 1024 // (groups * row))
        case |= {"groups": groups, "members": min(members, 16), "prompt": _log(rng, 1, most)}
    elif op == "free":
        case |= {"groups": groups, "members": members, "prompt": _log(rng, 1, 8192), "ctx": _log(rng, 1, 2048)}
    elif op == "compact":
        groups = min(groups, 16)
        members = min(members, 8)
        most = 64 * 16000 * 1024 // (row * groups)
        case |= {"groups": groups, "members": members, "prompt": _log(rng, 1, max(1, min(8000, most // 2))),
                 "ctx": _log(rng, 1, max(1, min(2000, most // (2 * members))))}
    elif op == "copy":
        pairs = _log(rng, 1, min(8192, 8192 * 65536 // (row * block)))
        case |= {"pairs": pairs, "prompt": pairs * block, "to": rng.choice([0, pairs + _log(rng, 1, 1000)])}
    else:
        most = 256 * 4096 * 1024 // (row * groups)                     # values of a group
        prompt = _log(rng, 1, max(1, min(32768, most // 4)))
        ctx = _log(rng, 1, max(1, min(4096, most // (2 * members))))
        # (the plain form lays out every member's tokens by themselves)
        while groups * members * (prompt + ctx) * max(row, 4 * kv * group * dim // 16) > 256 * 6144 * 1024:
            prompt, members = max(1, prompt // 2), max(1, members * 3 // 4)
        case |= {"groups": groups, "members": members, "prompt": prompt, "ctx": ctx}
    return case


def _sizes(case):
    """Members, shared tokens and (a list of) own tokens of each group, from the case alone."""
    r = np.random.RandomState(case["shape"] % (1 << 32))
    groups, members, prompt, ctx, block = case["groups"], case["members"], case["prompt"], case["ctx"], case["block"]
    count = r.randint(1, members + 1, groups) if case["ragged"] else np.full(groups, members)
    count[r.randint(groups)] = members
    shared = np.exp(r.uniform(0, np.log(prompt + 1), groups)).astype(np.int64) if case["ragged"] else np.full(groups, prompt)
    shared[r.randint(groups)] = prompt
    shared = np.minimum(np.maximum(shared, 1), prompt)
    if case["op"] != "fork":
        shared = shared // block * block                                      # what is shared are whole blocks
    rest = [r.randint(1, ctx + 1, n) if case["ragged"] and ctx else np.full(n, ctx) for n in count]
    return count, shared, rest, r


def _ints(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device=DEVICE)


def _context(case, seqs, n_blocks, width):
    import paper_2504_03661_amd as pq
    dtype = {"f16": pq.PQ_F16, "bf16": pq.PQ_BF16, "f32": pq.PQ_F32}[case["dtype"]]
    return pq.PQPaged(pq.PQPagedConfig(
        max_seqs=seqs, max_tokens=seqs, n_q_heads=case["q_heads"], n_kv_heads=case["kv_heads"], head_dim=case["dim"],
        block_tokens=case["block"], n_blocks=n_blocks, max_blocks=width, dtype=dtype, device=0))


def _cache(case, n_blocks, gen, name):
    kv, size = case["kv_heads"], case["block"] * case["dim"]
    made = {}
    for kind in "kv":
        made[name + kind + "_cache"] = torch.randint(1, 256, (n_blocks, kv, size), generator=gen, device=DEVICE, dtype=torch.uint8)
        made[name + kind + "_scale"] = torch.exp2(torch.rand((n_blocks, kv), generator=gen, device=DEVICE) * 1.5 - 6.0)
    return made


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    host = np.random.RandomState(seed % (1 << 32))
    op, block = case["op"], case["block"]
    s = {"case": case}
    if op == "copy":
        n_from = case["pairs"] * (1 if case["to"] else 2) + 7
        n_to = case["to"] or n_from
        src, order = host.permutation(n_from)[:case["pairs"]], host.permutation(n_to)
        # (within a cache the copies go where no pair copies from)
        dst = order[:case["pairs"]] if case["to"] else host.permutation(np.setdiff1d(np.arange(n_from), src))[:case["pairs"]]
        if case["ragged"]:                                                     # pairs that say nothing, and a count
            src[host.rand(src.size) < 1 / 16] = -1
        s |= _cache(case, n_from, gen, "from_" if case["to"] else "")
        if case["to"]:
            s |= _cache(case, n_to, gen, "")
        s |= {"src": _ints(src), "dst": _ints(dst), "count": _ints([case["pairs"] * 15 // 16]) if case["ragged"] else None,
              "n_from": n_from, "n_to": n_to, "ctx": _context(case, 1, n_to, 1) if own else None}
        return s

    count, shared, rest, r = _sizes(case)
    forks = op == "fork"
    if forks:                                                                  # the parents, and empty rows for the children
        seqs = int(count.sum()) + case["groups"]
        group = np.concatenate([np.arange(case["groups"]), np.repeat(np.arange(case["groups"]), count)])
        length = np.concatenate([shared, np.zeros(int(count.sum()), np.int64)])
        begin = np.zeros(seqs, np.int64)
    else:
        seqs = int(count.sum())
        group = np.repeat(np.arange(case["groups"]), count)
        begin = shared[group]
        length = begin + np.concatenate(rest)
    rows = host.permutation(seqs)                                              # request i is row rows[i] of the tables
    used = -(-length // block)
    own_blocks = used - begin // block
    most = max(1, int(used.max()))
    held = int(own_blocks.sum() + (0 if forks else (shared // block).sum()))
    spare = max(1, int(held * case["spare"])) if not forks else max(1, int(count.sum() * (0.9 if case["ragged"] else 1.0)) + 5)
    n_blocks = held + spare
    order = host.permutation(n_blocks)
    table = np.full((seqs, most), -1)
    holders = np.zeros(n_blocks, np.int64)
    at = 0
    prompts = []
    for g in range(case["groups"]):
        n = 0 if forks else int(shared[g] // block)
        prompts.append(order[at:at + n])
        holders[order[at:at + n]] = count[g] - 1
        at += n
    for i in range(seqs):
        first = begin[i] // block
        table[i, :first] = prompts[group[i]]
        table[i, first:used[i]] = order[at:at + own_blocks[i]]
        at += own_blocks[i]
    free = np.full(n_blocks, -1)
    free[:spare] = order[at:]

    def by_row(x, fill=0):
        got = np.full((seqs,) + np.shape(x)[1:], fill, np.int64)
        got[rows] = x
        return got

    s |= {"seqs": seqs, "n_blocks": n_blocks, "width": most, "seq_len": _ints(by_row(length)), "block_table": _ints(by_row(table)),
          "free_list": _ints(free), "free_count": _ints([spare]), "holders": _ints(holders),
          "ctx": _context(case, seqs, n_blocks, most) if own else None}
    if op in ("fork", "free"):
        s |= {"new_seq_len": torch.zeros_like(s["seq_len"]), "new_free_count": torch.zeros_like(s["free_count"])}
    if forks:
        parent = np.where(length > 0, -1, rows[group])
        s |= {"parent": _ints(by_row(parent)), "copy_src": _ints(np.zeros(seqs)), "copy_dst": _ints(np.zeros(seqs)), "keep": None}
        if case["ragged"]:
            part = np.where(r.rand(seqs) < 0.3, (r.rand(seqs) * (shared[group] + 1)).astype(np.int64), case["prompt"])
            s["keep"] = _ints(by_row(part))
    if op == "free":
        ends = r.rand(seqs) < (0.5 if case["ragged"] else 0.75)
        ends |= (r.rand(case["groups"]) < 0.2)[group] if case["ragged"] else False      # some groups as a whole
        ends[r.randint(seqs)] = True
        s |= {"n_new": _ints(by_row(np.where(ends, -1, 1))), "holders_before": s["holders"].clone()}
    if op == "compact":
        s |= {name: torch.full((n_blocks,), -1, dtype=torch.int32, device=DEVICE) for name in ("new_free_list", "copy_src", "copy_dst", "moved_to")}
        s |= {"new_free_count": torch.zeros_like(s["free_count"]), "new_table": s["block_table"].clone(),
              "new_holders": torch.zeros_like(s["holders"]), "n_copies": torch.zeros_like(s["free_count"])}
    if op == "shared_decode":
        s |= {"members": _ints(rows), "group_start": _ints(np.concatenate([[0], np.cumsum(count)])), "shared_len": _ints(shared)}
        s["scale"] = float(np.float32(1.0 / math.sqrt(case["dim"])))
        q = torch.randn((seqs, case["q_heads"], case["dim"]), generator=gen, device=DEVICE, dtype=torch.float32)
        s["q"] = q.to(DTYPES[case["dtype"]])
        s["out"] = torch.empty_like(s["q"])
    if op != "free":
        s |= _cache(case, n_blocks, gen, "")
    if own and op == "shared_decode":
        import paper_2504_03661_amd as pq
        size = pq.pq_paged_shared_workspace_bytes(s["ctx"].handle, seqs, case["groups"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEVICE)
    return s


# -------------------------------------------------------------------------------------------------- plain forms

def _plain_copy(s, src, dst, source, target):
    """Blocks src[i] of the cache `source` to dst[i] of `target`, where src[i] is not negative."""
    says = src >= 0
    src, dst = src[says], dst[says]
    for kind in "kv":
        for what in ("_cache", "_scale"):
            s[target + kind + what][dst] = s[source + kind + what][src]


def _caches(s):
    return {kind + what: s[kind + what] for kind in "kv" for what in ("_cache", "_scale")}


def _plain_fork(s):
    block, seqs, n_blocks, width = s["case"]["block"], s["seqs"], s["n_blocks"], s["width"]
    table, length, parent, free = s["block_table"].long(), s["seq_len"].long(), s["parent"].long(), s["free_list"].long()
    row = torch.arange(seqs, device=DEVICE)
    asks = (parent >= 0) & (parent != row)
    fits = asks & (parent < seqs) & (length == 0)
    of = torch.where(fits, parent, 0)
    takes = length[of] if s["keep"] is None else torch.minimum(length[of], s["keep"].long().clamp(min=0))
    takes = torch.where(fits, takes, 0)
    full, part = takes // block, takes % block > 0
    # blocks come from the top of the free ones, in the order of the rows
    count = s["free_count"].long()
    upto = part.long().cumsum(0)
    granted = fits & (~part | (upto <= count))
    new = free[(count - upto).clamp(0, n_blocks - 1)]
    column = torch.arange(width, device=DEVICE)
    theirs = table[of]
    shares = granted[:, None] & (column < full[:, None])
    copies = granted & part
    last = theirs.gather(1, full.clamp(max=width - 1)[:, None])[:, 0]
    got = torch.where(shares, theirs, table)
    got = torch.where(copies[:, None] & (column == full[:, None]), new[:, None], got)
    held = torch.zeros(n_blocks + 1, dtype=torch.long, device=DEVICE)
    held.scatter_add_(0, torch.where(shares, theirs, n_blocks).reshape(-1), torch.ones(shares.numel(), dtype=torch.long, device=DEVICE))
    s["holders"] += held[:-1].int()
    s["block_table"].copy_(got)
    src, dst = torch.where(copies, last, -1), torch.where(copies, new, -1)
    _plain_copy(s, src, dst, "", "")
    return {"new_seq_len": torch.where(granted, takes, length).int(),
            "new_free_count": (count - torch.where(copies, upto, 0).amax()).int(), "block_table": s["block_table"],
            "holders": s["holders"], "copy_src": src.int(), "copy_dst": dst.int(), **_caches(s)}


def _plain_free(s):
    block, n_blocks = s["case"]["block"], s["n_blocks"]
    table, length, ends = s["block_table"].long(), s["seq_len"].long(), s["n_new"] < 0
    column = torch.arange(s["width"], device=DEVICE)
    gives = ends[:, None] & (column < ((length + block - 1) // block)[:, None])
    given = torch.zeros(n_blocks + 1, dtype=torch.long, device=DEVICE)
    given.scatter_add_(0, torch.where(gives, table, n_blocks).reshape(-1), torch.ones(gives.numel(), dtype=torch.long, device=DEVICE))
    left = s["holders"].long() - given[:-1]
    goes = (given[:-1] > 0) & (left < 0)
    # onto the free ones from the highest number down: the lowest lies on top
    count = s["free_count"].long()
    above = goes.flip(0).long().cumsum(0).flip(0)
    place = torch.where(goes & (count + above <= n_blocks), count + above - 1, n_blocks)
    free = torch.cat([s["free_list"], s["free_list"][:1]])
    free[place] = torch.arange(n_blocks, device=DEVICE, dtype=torch.int32)
    s["free_list"].copy_(free[:-1])
    s["holders"].copy_(torch.where(goes, 0, left))
    return {"new_seq_len": torch.where(ends, 0, length).int(), "new_free_count": (count + above[:1]).clamp(max=n_blocks).int(),
            "free_list": s["free_list"], "holders": s["holders"]}


def _plain_compact(s):
    block, n_blocks = s["case"]["block"], s["n_blocks"]
    number = torch.arange(n_blocks, device=DEVICE)
    on_list = torch.where(number < s["free_count"], s["free_list"].long(), n_blocks)
    is_free = torch.zeros(n_blocks + 1, dtype=torch.bool, device=DEVICE)
    is_free[on_list] = True
    is_free = is_free[:-1]
    n_free = is_free.sum()
    n_live = n_blocks - n_free
    # the k-th lowest free number below n_live takes the k-th highest live block
    low, high = is_free & (number < n_live), ~is_free & (number >= n_live)
    from_bottom, from_top = low.long().cumsum(0) - 1, high.flip(0).long().cumsum(0).flip(0) - 1
    spare = torch.full((1,), -1, device=DEVICE)
    lows = torch.cat([spare.expand(n_blocks), spare])
    highs = lows.clone()
    lows[torch.where(low, from_bottom, n_blocks)] = number
    highs[torch.where(high, from_top, n_blocks)] = number
    lows, highs = lows[:-1], highs[:-1]
    moves = number < low.sum()
    moved = torch.where(is_free, -1, torch.where(high, lows[from_top.clamp(min=0)], number))
    used = (s["seq_len"].long() + block - 1) // block
    holds = torch.arange(s["width"], device=DEVICE) < used[:, None]
    table = torch.where(holds, moved[s["block_table"].long().clamp(min=0)], s["new_table"].long())
    came = highs[from_bottom.clamp(min=0)]
    holders = torch.where(number >= n_live, 0, s["holders"].long()[torch.where(low, came, number)])
    free = torch.where(number < n_free, n_blocks - 1 - number, s["new_free_list"].long())
    src, dst = torch.where(moves, highs, s["copy_src"].long()), torch.where(moves, lows, s["copy_dst"].long())
    _plain_copy(s, torch.where(moves, highs, -1), dst, "", "")
    return {"new_free_list": free.int(), "new_free_count": n_free.int().reshape(1), "new_table": table.int(),
            "new_holders": holders.int(), "copy_src": src.int(), "copy_dst": dst.int(), "n_copies": low.sum().int().reshape(1),
            "moved_to": moved.int(), **_caches(s)}


def _plain_values(s, kind):
    """All tokens that the block tables name: [request, KV head, token, dim] in fp32."""
    block, dim, kv = s["case"]["block"], s["case"]["dim"], s["case"]["kv_heads"]
    blocks = s["block_table"].long().clamp(min=0)
    x = s[kind + "_cache"][blocks]
    if kind == "v":
        # tile, dim / 64, token / 4, dim % 16, dim / 16 % 4, token % 4
        x = x.reshape(*x.shape[:3], block // 16, dim // 64, 4, 16, 4, 4).permute(0, 1, 2, 3, 5, 8, 4, 7, 6)
    x = x.reshape(s["seqs"], s["width"], kv, block, dim).transpose(1, 2).to(torch.float32)
    scale = s[kind + "_scale"][blocks].transpose(1, 2)[..., None, None]
    return x.sub_(128.0).mul_(scale).reshape(s["seqs"], kv, s["width"] * block, dim)


def _plain_shared_decode(s):
    case, seqs = s["case"], s["seqs"]
    kv, dim = case["kv_heads"], case["dim"]
    q = s["q"].to(torch.float32).reshape(seqs, kv, -1, dim)
    k = _plain_values(s, "k")
    t = torch.matmul(q, k.transpose(-1, -2)) * s["scale"]
    del k
    there = torch.arange(t.shape[-1], device=DEVICE) < s["seq_len"][:, None, None, None]
    t = t.masked_fill(~there, -math.inf)
    e = torch.exp(t - t.amax(-1, keepdim=True).clamp(min=-3.0e38))
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e, _plain_values(s, "v")) / torch.where(total > 0, total, 1.0)
    return out.reshape(seqs, -1, dim).to(s["q"].dtype)


# -------------------------------------------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if op == "free":
        # a pass begins with the counts that a program has in front of the call
        s["holders"].copy_(s["holders_before"])
    if own:
        return _run_own(s, op)
    if op == "fork":
        return _plain_fork(s)
    if op == "free":
        return _plain_free(s)
    if op == "compact":
        return _plain_compact(s)
    if op == "copy":
        src = s["src"].long()
        if s["count"] is not None:
            src = torch.where(torch.arange(src.shape[0], device=DEVICE) < s["count"], src, -1)
        _plain_copy(s, src, s["dst"].long(), "from_" if s["case"]["to"] else "", "")
        return _caches(s)
    return _plain_shared_decode(s)


def _run_own(s, op):
    import paper_2504_03661_amd as pq
    case, ctx = s["case"], s["ctx"].handle
    if op == "free":
        pq.pq_paged_free(ctx, s["seqs"], s["n_new"], s["seq_len"], s["free_list"], s["free_count"], s["block_table"],
                         s["holders"], s["new_seq_len"], s["new_free_count"])
        return {name: s[name] for name in ("new_seq_len", "new_free_count", "free_list", "holders")}
    if op == "shared_decode":
        pq.pq_paged_shared_decode(ctx, s["seqs"], case["groups"], s["q"], case["q_heads"] * case["dim"], s["k_cache"],
                                  s["v_cache"], s["k_scale"], s["v_scale"], s["block_table"], s["seq_len"], s["members"],
                                  s["group_start"], s["shared_len"], s["scale"], s["workspace"], s["workspace"].numel(), s["out"])
        return s["out"]
    cache = [s[name] for name in ("k_cache", "v_cache", "k_scale", "v_scale")]
    if op == "copy":
        source = [s["from_" + name] for name in ("k_cache", "v_cache", "k_scale", "v_scale")] if case["to"] else cache
        pq.pq_paged_copy(ctx, case["pairs"], s["src"], s["dst"], s["count"], s["n_from"], *source, s["n_to"], *cache)
        return _caches(s)
    n_blocks = s["n_blocks"]
    if op == "fork":
        pq.pq_paged_fork(ctx, s["seqs"], s["parent"], s["keep"], s["seq_len"], s["free_list"], s["free_count"],
                         s["block_table"], s["holders"], s["new_seq_len"], s["new_free_count"], s["copy_src"], s["copy_dst"])
        pq.pq_paged_copy(ctx, s["seqs"], s["copy_src"], s["copy_dst"], None, n_blocks, *cache, n_blocks, *cache)
        names = ("new_seq_len", "new_free_count", "block_table", "holders", "copy_src", "copy_dst")
    else:
        pq.pq_paged_compact(ctx, s["seqs"], s["seq_len"], s["free_list"], s["free_count"], s["block_table"], s["holders"],
                            s["new_free_list"], s["new_free_count"], s["new_table"], s["new_holders"], s["moved_to"],
                            s["copy_src"], s["copy_dst"], s["n_copies"])
        pq.pq_paged_copy(ctx, n_blocks, s["copy_src"], s["copy_dst"], s["n_copies"], n_blocks, *cache, n_blocks, *cache)
        names = ("new_free_list", "new_free_count", "new_table", "new_holders", "moved_to", "copy_src", "copy_dst", "n_copies")
    return {**{name: s[name] for name in names}, **_caches(s)}


def work(case):
    size = DTYPES[case["dtype"]].itemsize
    block, kv, dim, heads = case["block"], case["kv_heads"], case["dim"], case["q_heads"]
    of_block = 2 * kv * (block * dim + 4)                                       # bytes of K and V and their scales
    if case["op"] == "copy":
        return {"bytes": float(2 * of_block * case["pairs"]), "flops": 0.0}
    count, shared, rest, r = _sizes(case)
    own_tokens = np.concatenate(rest)
    begin = np.repeat(shared, count)
    if case["op"] == "fork":
        full = (shared // block * count).sum()                                  # entries: read, written, a count raised
        copied = (count * (shared % block > 0)).sum()
        return {"bytes": float(4 * (4 * full + 6 * count.sum()) + 2 * of_block * copied), "flops": 0.0}
    if case["op"] == "free":
        entries = (-(-(begin + own_tokens) // block)).sum() * (0.5 if case["ragged"] else 0.75)
        return {"bytes": float(4 * (3 * entries + 4 * count.sum() + entries // 2)), "flops": 0.0}
    if case["op"] == "compact":
        entries = (-(-(begin + own_tokens) // block)).sum()
        held = (-(-own_tokens // block)).sum() + (shared // block).sum()
        n_blocks = held * (1.0 + case["spare"])
        moved = held * (n_blocks - held) / n_blocks
        return {"bytes": float(4 * (2 * entries + 6 * n_blocks) + 2 * of_block * moved), "flops": 0.0}
    blocks = (shared // block).sum() + (-(-own_tokens // block)).sum()
    tokens = (shared.sum() + own_tokens.sum())                                  # read once
    return {"bytes": float(2 * tokens * kv * dim + 8 * blocks * kv + 2 * count.sum() * heads * dim * size),
            "flops": float(4 * (begin + own_tokens).sum() * heads * dim)}


# -------------------------------------------------------------------------------------------------- in 64 bits

def _exact_rows(s, kind, b, upto):
    """Values of the first `upto` tokens of request b, [KV head, token, dim], token by token from the layout's definition."""
    case = s["case"]
    block, kv, dim = case["block"], case["kv_heads"], case["dim"]
    t = torch.arange(upto, device=DEVICE)
    number = s["block_table"][b].long()[t // block]
    d = torch.arange(dim, device=DEVICE)
    r = (t % block)[:, None]
    if kind == "k":
        place = r * dim + d
    else:
        place = r // 16 * (16 * dim) + d // 64 * 1024 + r % 16 // 4 * 256 + d % 16 * 16 + d // 16 % 4 * 4 + r % 4
    flat = s[kind + "_cache"].reshape(-1)
    rows = [flat[(number[:, None] * kv + h) * (block * dim) + place].double() - 128.0 for h in range(kv)]
    return torch.stack([x * s[kind + "_scale"][number, h].double()[:, None] for h, x in enumerate(rows)])


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "shared_decode":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
        for b, n in enumerate(s["seq_len"].tolist()):
            if n:
                k, v = _exact_rows(s, "k", b, n), _exact_rows(s, "v", b, n)
                q = s["q"][b].double().reshape(k.shape[0], -1, k.shape[2])
                for h in range(k.shape[0]):
                    p = torch.softmax(q[h] @ k[h].T.contiguous() * s["scale"], -1)
                    out[b].reshape(k.shape[0], -1, k.shape[2])[h] = p @ v[h]
        return out
    if case["op"] == "copy":
        pairs = list(zip(s["src"].tolist(), s["dst"].tolist()))[:None if s["count"] is None else s["count"].item()]
        got = {}
        for name in ("k_scale", "v_scale"):
            source = s[("from_" if case["to"] else "") + name].double().cpu().numpy()
            to = s[name].double().cpu().numpy()
            for i, j in pairs:
                if i >= 0:
                    to[j] = source[i]
            got[name] = torch.from_numpy(to)
        return {"k_cache": None, "v_cache": None, **got}
    return None                                                                 # whole numbers, and scales that are copied
