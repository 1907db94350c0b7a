"""The operators of a worker's step, as a serving loop calls them.

A router sends a worker the requests whose longest cached prefix it holds.
What the worker then does with the batch, in four operators:

groups   requests that share a prompt prefix are found from their block-hash
         chains, and the batch is ordered group by group
tables   block tables and slot maps from the requests' lengths: which cache
         block holds which part of a sequence (a group's prefix once), and
         where each new token's key and value go
write    the new tokens' keys and values go into the block cache
attend   attention of the new tokens over the block cache, a group's shared
         prefix read once for all its members

Blocks are 16 tokens, as the router counts them.  Lengths are drawn from the
case alone; hashes, block numbers, queries, keys and values from the seed.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _batch_case(name, kind, B, groups, prefix, tail, new, **more):
    """B requests in `groups` groups (0: nothing is shared); a group's prefix, a request's tokens after it and how
    many of those are new are each (lowest, highest)."""
    c = dict(name=name, kind=kind, B=B, groups=groups, prefix_lo=prefix[0], prefix_hi=prefix[1], tail_lo=tail[0],
             tail_hi=tail[1], new_lo=new[0], new_hi=new[1])
    c.update(more)
    return c


def listed():
    return [
        # the requests that arrived together at a router, and a large waiting queue
        dict(name="groups_arrivals", kind="groups", B=32, groups=8, len_lo=8, len_hi=512, min_blocks=2),
        dict(name="groups_queue", kind="groups", B=4096, groups=256, len_lo=16, len_hi=512, min_blocks=8),
        # one more token for every running request; and a step that admits many prompts
        _batch_case("tables_decode", "tables", 64, 8, (1024, 8192), (17, 2000), (1, 1), fresh=False),
        _batch_case("tables_prompts", "tables", 1024, 64, (128, 8192), (1, 8192), (1, 8192), fresh=True),
        # the same two steps' keys and values, on a quarter of eight key heads and on all of them
        dict(name="write_decode", kind="write", T=64, Hkv=2, D=128, blocks=4096, dtype="bf16", heads_first=False),
        dict(name="write_prompts", kind="write", T=16384, Hkv=8, D=128, blocks=2048, dtype="bf16", heads_first=True),
        # one user alone, a short answer so far: all latency
        _batch_case("attend_one", "attend", 1, 0, (0, 0), (100, 100), (1, 1), Hq=16, Hkv=2, D=128, dtype="bf16",
                    heads_first=False, lse=False),
        # a system prompt that the whole batch shares, one token each
        _batch_case("attend_prompt_shared", "attend", 128, 1, (8192, 8192), (16, 512), (1, 1), Hq=64, Hkv=8, D=128,
                    dtype="bf16", heads_first=False, lse=False),
        # requests of several groups and lengths, and of none
        _batch_case("attend_groups", "attend", 200, 24, (512, 16384), (1, 4000), (1, 1), Hq=16, Hkv=2, D=128,
                    dtype="fp16", heads_first=True, lse=True),
        # few long conversations, nothing in common: the cache is read at its full rate or not
        _batch_case("attend_long", "attend", 5, 0, (0, 0), (60000, 131072), (1, 1), Hq=16, Hkv=4, D=128,
                    dtype="bf16", heads_first=False, lse=False),
        # pieces of long prompts beside decoding requests, heads of 192
        _batch_case("attend_pieces", "attend", 12, 3, (2000, 8000), (1, 3000), (1, 700), Hq=12, Hkv=1, D=192,
                    dtype="bf16", heads_first=False, lse=True),
        # whole prompts
        _batch_case("attend_prompts", "attend", 3, 0, (0, 0), (2500, 6000), (6000, 6000), Hq=64, Hkv=8, D=128,
                    dtype="bf16", heads_first=False, lse=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("groups", "tables", "write", "attend", "attend", "attend"))
    if kind == "groups":
        least = _log(rng, 1, 16)
        B = _log(rng, 20, 4096)
        lo = rng.randint(1, 4 * least + 8)
        return dict(kind=kind, B=B, groups=rng.randint(2, max(3, min(B // 8, 300))), len_lo=lo,
                    len_hi=4 * least + lo + _log(rng, 1, 440), min_blocks=least)
    if kind == "tables":
        fresh = rng.random() < 0.5
        B = _log(rng, 1, 1024)
        hi = _log(rng, 40, 8000)
        c = _batch_case("", kind, B, rng.choice((0, 1, max(1, B // 9))), (16, _log(rng, 17, 8000)), (1, hi),
                        (1, hi if fresh else rng.choice((1, 1, 5, min(hi, 600)))), fresh=fresh)
        del c["name"]
        return c
    heads = dict(Hkv=rng.choice((1, 2, 3, 4, 5, 8)), D=rng.choice((64, 128, 128, 128, 192, 256, 80, 96)),
                 dtype=rng.choice(("bf16", "fp16")), heads_first=rng.random() < 0.5)
    if kind == "write":
        T = _log(rng, 1, 12000)
        return dict(kind=kind, T=T, blocks=T // BLOCK + _log(rng, 8, 1000), **heads)
    heads.update(Hq=heads["Hkv"] * rng.choice((1, 2, 4, 5, 7, 8, 12)), lse=rng.random() < 0.5)
    shape = rng.choice(("decode", "decode", "pieces", "prompts"))
    B = {"decode": _log(rng, 1, 200), "pieces": _log(rng, 2, 16), "prompts": _log(rng, 1, 5)}[shape]
    tail = _log(rng, 20, {"decode": 60000, "pieces": 6000, "prompts": 5000}[shape])
    prefix = _log(rng, 17, 8000)
    new = {"decode": rng.choice((1, 1, 1, 2, 4)), "pieces": _log(rng, 2, 900), "prompts": tail}[shape]
    while B > 1 and B * (prefix + tail) * heads["Hkv"] > 3_000_000:
        B = B * 3 // 4
    while B > 1 and B * (prefix + tail) * min(new, tail) * heads["Hq"] > 3_000_000_000:
        B = B * 3 // 4
    c = _batch_case("", kind, B, rng.choice((0, 1, max(1, B // 6))), (16, prefix), (1 if B > 1 else tail, tail),
                    (1 if shape == "pieces" else new, new), **heads)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs

def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _spread(rng, lo, hi, n):
    """n lengths between lo and hi, even over their logarithm, both ends among them."""
    v = np.rint(np.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1)), n))).astype(np.int64)
    if n > 1:
        v[int(rng.integers(0, n))] = lo
    v[int(rng.integers(0, n))] = hi
    return np.clip(v, lo, hi)


def _zipf_sizes(rng, n_groups, n):
    """n requests over groups of falling popularity, by group."""
    p = 1.0 / np.arange(1, n_groups + 1)
    return np.sort(rng.choice(n_groups, n, p=p / p.sum()))


def _lengths(case):
    """Of each request, group by group: first request of its group, blocks it shares with that one (by group too), tokens in
    all, tokens new.  The case alone decides."""
    rng = np.random.Generator(np.random.PCG64([case["B"], case["groups"], case["tail_hi"], case["prefix_hi"]]))
    B, G = case["B"], case["groups"]
    tail = _spread(rng, case["tail_lo"], case["tail_hi"], B)
    if G == 0:
        first, group_off, shared = np.arange(B), np.arange(B + 1), np.zeros(B, np.int64)
        prefix = np.zeros(B, np.int64)
    else:
        _, group = np.unique(_zipf_sizes(rng, G, B), return_inverse=True)
        n = int(group.max()) + 1
        count = np.bincount(group, minlength=n)
        group_off = np.full(B + 1, B, np.int64)
        group_off[:n] = np.cumsum(count) - count
        blocks = _spread(rng, case["prefix_lo"], case["prefix_hi"], n) // BLOCK
        shared = np.zeros(B, np.int64)
        shared[:n] = np.where(count > 1, blocks, 0)
        first, prefix = group_off[group], BLOCK * blocks[group]
    kv = prefix + tail
    if case.get("fresh"):         # nothing is in the cache yet: the first of a group brings the prefix
        new = np.where((first == np.arange(B)) | (prefix == 0), kv, tail)
    else:
        new = np.minimum(_spread(rng, case["new_lo"], case["new_hi"], B), tail)
    return first, group_off, shared, kv, new


def _offsets(n):
    off = np.zeros(n.size + 1, np.int64)
    np.cumsum(n, out=off[1:])
    return off


def _prepare_groups(case, seed):
    rng = np.random.Generator(np.random.PCG64([case["B"], case["len_hi"], 3]))
    B = case["B"]
    L = _spread(rng, case["len_lo"], case["len_hi"], B)
    g = np.random.Generator(np.random.PCG64([seed, 5])).permutation(_zipf_sizes(rng, case["groups"], B))
    # a group's prompts have 25-75% of their blocks in common with its longest one
    common = np.rint(L * rng.uniform(0.25, 0.75, B)).astype(np.int64)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    off = _offsets(L)
    hashes = lambda *n: torch.randint(1, 1 << 62, n, generator=gen, device="cuda")  # noqa: E731
    base, private = hashes(case["groups"], case["len_hi"]), hashes(int(off[-1]))
    owner = torch.repeat_interleave(torch.arange(B, device="cuda"), _up(L))
    pos = torch.arange(int(off[-1]), device="cuda") - _up(off)[owner]
    is_common = pos < _up(common)[owner]
    chains = torch.where(is_common, base[_up(g)[owner], torch.where(is_common, pos, 0)], private)
    return dict(case=case, chains=chains, chain_off=_up(off), longest=int(L.max()))


def _shuffled(n, gen, offset=0):
    return (torch.randperm(n, generator=gen, device="cuda") + offset).to(torch.int32)


def _prepare_tables(case, seed):
    first, group_off, shared, kv, new = _lengths(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    need = -(-kv // BLOCK)
    have = np.zeros_like(kv) if case["fresh"] else -(-(kv - new) // BLOCK)
    total, stride = int(need.sum()), int(need.max()) + 8
    ids = _shuffled(2 * total + 64, gen)
    tables = torch.full((case["B"], stride), -1, dtype=torch.int32, device="cuda")
    p = torch.arange(stride, device="cuda")
    # what the rows hold from earlier steps
    held = p[None, :] < _up(have)[:, None]
    old = (_up(np.cumsum(have) - have)[:, None] + p).clamp_(max=total - 1)
    tables = torch.where(held, ids[old], tables)
    return dict(case=case, tables=tables, kv_len=_up(kv.astype(np.int32)), new_len=_up(new.astype(np.int32)),
                have=_up(have.astype(np.int32)), free=ids[total:].contiguous(), n_slots=int(new.sum()) + 5,
                group_off=_up(group_off), shared=_up(shared.astype(np.int32)))


def _cache(case, blocks, gen):
    """Block cache of keys or of values, [block, token, head, D]; heads_first: with a block's heads before its tokens."""
    H, D = case["Hkv"], case["D"]
    shape = (blocks, H, BLOCK, D) if case["heads_first"] else (blocks, BLOCK, H, D)
    x = torch.randn(shape, generator=gen, device="cuda", dtype=TYPES[case["dtype"]])
    return x.transpose(1, 2) if case["heads_first"] else x


def _prepare_write(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, H, D = case["T"], case["Hkv"], case["D"]
    new = torch.randn((T, H, 2, D), generator=gen, device="cuda", dtype=TYPES[case["dtype"]])
    slots = torch.randperm(BLOCK * case["blocks"], generator=gen, device="cuda")[:T]
    slots = torch.where(torch.rand(T, generator=gen, device="cuda") < 0.02, -1, slots)    # tokens that another request writes
    # the last block is nobody's
    return dict(case=case, k=new[:, :, 0], v=new[:, :, 1], slots=slots, k_cache=_cache(case, case["blocks"] + 1, gen),
                v_cache=_cache(case, case["blocks"] + 1, gen))


def _prepare_attend(case, seed):
    first, group_off, shared, kv, new = _lengths(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, Hq, D = case["B"], case["Hq"], case["D"]
    group = np.searchsorted(group_off, np.arange(B), side="right") - 1
    need = -(-kv // BLOCK)
    lead = np.where(first == np.arange(B), 0, shared[group])
    own_blocks = need - lead
    start = np.cumsum(own_blocks) - own_blocks
    blocks, stride = int(own_blocks.sum()) + 3, int(need.max())
    p = torch.arange(stride, device="cuda")
    row = torch.where(p[None, :] < _up(lead)[:, None], _up(start[first])[:, None] + p, _up(start - lead)[:, None] + p)
    tables = torch.where(p[None, :] < _up(need)[:, None], _shuffled(blocks, gen)[row.clamp_(0, blocks - 1)], 0)
    q_off = _offsets(new)
    q = torch.randn((int(q_off[-1]), Hq, D), generator=gen, device="cuda", dtype=TYPES[case["dtype"]])
    return dict(case=case, q=q, k_cache=_cache(case, blocks, gen), v_cache=_cache(case, blocks, gen), tables=tables,
                kv_len=_up(kv.astype(np.int32)), q_off=_up(q_off), group_off=_up(group_off),
                shared=_up(shared.astype(np.int32)), most_new=int(new.max()))


def prepare(case, seed):
    return {"groups": _prepare_groups, "tables": _prepare_tables, "write": _prepare_write,
            "attend": _prepare_attend}[case["kind"]](case, seed)


# ------------------------------------------------------------------ plain forms

def _plain_groups(st):
    """Requests whose first min_blocks blocks are alike form a group; a chained hash names its whole prefix, so
    one hash of each tells.  A group is numbered by its first request, and shares what all its members have in common
    with that one."""
    chains, off, least = st["chains"], st["chain_off"], st["case"]["min_blocks"]
    B = off.numel() - 1
    i = torch.arange(B, device=chains.device)
    L = off[1:] - off[:-1]
    long = L >= least
    key = chains[torch.where(long, off[:-1] + least - 1, 0)]
    alike = ((key[:, None] == key[None, :]) & long[:, None] & long[None, :]) | (i[:, None] == i[None, :])
    first = torch.where(alike, i[None, :], B).amin(1)
    order = torch.argsort(first, stable=True)
    leads = first == i
    count = torch.zeros(B, dtype=torch.int64, device=chains.device).index_add_(0, first, torch.ones_like(first))
    rank = leads.cumsum(0) - 1
    n = leads.sum()
    group = rank[first]
    sizes = torch.zeros(B, dtype=torch.int64, device=chains.device).index_add_(0, group, torch.ones_like(group))
    group_off = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)])
    p = torch.arange(st["longest"], device=chains.device)
    both = torch.minimum(L, L[first])
    inside = p[None, :] < both[:, None]
    mine = chains[torch.where(inside, off[:-1, None] + p, 0)]
    its = chains[torch.where(inside, off[:-1][first][:, None] + p, 0)]
    common = ((mine == its) & inside).to(torch.int32).cumprod(1).sum(1)
    shared = torch.full((B,), 1 << 30, dtype=torch.int64, device=chains.device).scatter_reduce_(0, group, common, "amin")
    shared = torch.where(sizes > 1, shared, 0)
    return order.to(torch.int32), group_off, shared.to(torch.int32), n.to(torch.int32).reshape(1)


def _plain_tables(st):
    """Row i has ceil(kv_len / 16) blocks: those it had, those of the group's shared prefix from the group's first
    row, and the rest from the free list, in the order of the rows."""
    tables, free = st["tables"], st["free"].long()
    kv, new, have = st["kv_len"].long(), st["new_len"].long(), st["have"].long()
    B, stride = tables.shape
    i = torch.arange(B, device=tables.device)
    group = torch.searchsorted(st["group_off"], i, right=True) - 1
    first = st["group_off"][group]
    need = (kv + BLOCK - 1) // BLOCK
    lead = torch.where(first == i, 0, torch.minimum(st["shared"].long()[group], kv[first] // BLOCK))
    start = torch.maximum(have, lead)
    count = (need - start).clamp(min=0)
    base = count.cumsum(0) - count
    p = torch.arange(stride, device=tables.device)[None, :]
    theirs = torch.where(p < have[first][:, None], tables[first].long(),
                         free[(base[first][:, None] + p - have[first][:, None]).clamp(0, free.numel() - 1)])
    mine = free[(base[:, None] + p - start[:, None]).clamp(0, free.numel() - 1)]
    held, after = p < have[:, None], p >= need[:, None]
    out = torch.where(held | after, tables.long(), torch.where(p < lead[:, None], theirs, mine))
    q_off = torch.cat([new.new_zeros(1), new.cumsum(0)])
    t = torch.arange(st["n_slots"], device=tables.device)
    r = (torch.searchsorted(q_off, t, right=True) - 1).clamp(max=B - 1)
    pos = kv[r] - new[r] + t - q_off[r]
    block = (pos // BLOCK).clamp(0, stride - 1)
    written = (t < q_off[-1]) & ~((block >= have[r]) & (block < lead[r]))
    slots = torch.where(written, out[r, block] * BLOCK + pos % BLOCK, -1)
    return out.to(torch.int32), slots, q_off, count.sum().to(torch.int32).reshape(1)


def _plain_write(st):
    n = st["case"]["blocks"]
    for new, cache in ((st["k"], st["k_cache"]), (st["v"], st["v_cache"])):
        slot = torch.where(st["slots"] < 0, BLOCK * n, st["slots"])       # into nobody's block
        cache[slot // BLOCK, slot % BLOCK] = new
    return st["k_cache"][:n], st["v_cache"][:n]


def _plain_attend(st):
    """softmax(q k / sqrt(D)) v of each new token over its sequence up to itself, on rows padded to the longest."""
    q, tables, kv, off = st["q"], st["tables"].long(), st["kv_len"].long(), st["q_off"]
    T, Hq, D = q.shape
    H, B, n, dev = st["case"]["Hkv"], kv.numel(), st["most_new"], q.device
    new = off[1:] - off[:-1]
    t = torch.arange(n, device=dev)
    pos = (kv - new)[:, None] + t                                         # [B, n]
    qs = q[(off[:-1, None] + t).clamp(max=T - 1)].float() / math.sqrt(D)  # [B, n, Hq, D]
    qs = qs.view(B, n, H, Hq // H, D).permute(0, 2, 3, 1, 4).reshape(B * H, -1, D)
    there = torch.arange(BLOCK * tables.shape[1], device=dev)
    k = st["k_cache"][tables].float().flatten(1, 2).permute(0, 2, 3, 1).reshape(B * H, D, -1)
    s = torch.bmm(qs, k).view(B, H, Hq // H, n, -1)
    del k
    s.masked_fill_(there > pos[:, None, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = s.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    v = st["v_cache"][tables].float().flatten(1, 2)
    v = v.masked_fill_((there >= kv[:, None])[:, :, None, None], 0).transpose(1, 2).reshape(B * H, -1, D)
    o = torch.bmm(e.view(B * H, -1, there.numel()), v).view(B, H, Hq // H, n, D) / total
    tok = torch.arange(T, device=dev)
    r = torch.searchsorted(off, tok, right=True) - 1
    at = tok - off[r]
    out = o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)[r, at].to(q.dtype)
    if not st["case"]["lse"]:
        return (out,)
    lse = (m + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, n, Hq)[r, at]
    return out, lse


# ------------------------------------------------------------------ one pass

def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"groups": _plain_groups, "tables": _plain_tables, "write": _plain_write,
                "attend": _plain_attend}[kind](st)
    from paper_2606_17081_amd import rkroute as rk
    if kind == "groups":
        return rk.prefix_groups(st["chains"], st["chain_off"], st["case"]["min_blocks"])
    if kind == "tables":
        return rk.block_tables(st["tables"], st["kv_len"], st["new_len"], st["have"], st["free"], st["n_slots"],
                               group_off=st["group_off"], shared=st["shared"])
    if kind == "write":
        n = st["case"]["blocks"]
        k, v = st["k_cache"][:n], st["v_cache"][:n]
        rk.kv_write(st["k"], st["v"], k, v, st["slots"])
        return k, v
    out, lse = rk.prefix_attention(st["q"], st["k_cache"], st["v_cache"], st["tables"], st["kv_len"], st["q_off"],
                                   group_off=st["group_off"], shared=st["shared"], want_lse=st["case"]["lse"])
    return (out, lse) if st["case"]["lse"] else (out,)


def work(case):
    kind = case["kind"]
    if kind == "groups":
        # of each request its offset, the hash that names its group and the two at either side of where it leaves
        # its group's first request, and those of that one; an order, an offset and a count come back
        B = case["B"]
        return {"bytes": B * (8 + 5 * 8) + B * (4 + 8 + 4) + 12, "flops": 0}
    if kind == "write":
        return {"bytes": 2 * 2 * 2 * case["T"] * case["Hkv"] * case["D"] + 8 * case["T"], "flops": 0}
    first, group_off, shared, kv, new = _lengths(case)
    B = case["B"]
    group = np.searchsorted(group_off, np.arange(B), side="right") - 1
    lead = np.where(first == np.arange(B), 0, shared[group])
    need = -(-kv // BLOCK)
    if kind == "tables":
        have = np.zeros_like(kv) if case["fresh"] else -(-(kv - new) // BLOCK)
        put = np.maximum(need - have, 0)
        taken = np.maximum(need - np.maximum(have, lead), 0)
        # lengths and groups, the blocks taken from the list, and table entries, slots and offsets written
        return {"bytes": int(24 * B + 4 * taken.sum() + 4 * put.sum() + 8 * new.sum() + 8 * B + 52), "flops": 0}
    Hq, H, D = case["Hq"], case["Hkv"], case["D"]
    keys = int((kv - BLOCK * lead).sum())                 # a group's prefix once
    pairs = int((new * kv - new * (new - 1) // 2).sum())  # each new token and what it sees
    return {"bytes": 2 * 2 * keys * H * D + 2 * 2 * int(new.sum()) * Hq * D + (4 * int(new.sum()) * Hq if case["lse"] else 0)
            + 4 * int((need - lead).sum()) + 28 * B, "flops": 4 * pairs * Hq * D}


def exact(case, seed):
    """Attention request by request in 64 bits; the other operators' outputs are whole numbers and copies."""
    if case["kind"] != "attend":
        return None
    st = prepare(case, seed)
    off, kv = st["q_off"].tolist(), st["kv_len"].tolist()
    H, G, D = case["Hkv"], case["Hq"] // case["Hkv"], case["D"]
    outs, lses = [], []
    for i in range(case["B"]):
        n, L = off[i + 1] - off[i], kv[i]
        rows = st["tables"][i, : -(-L // BLOCK)].long()
        k, v = (st[c][rows].reshape(-1, H, D)[:L].double() for c in ("k_cache", "v_cache"))
        q = st["q"][off[i]: off[i + 1]].double().view(n, H, G, D)
        hidden = torch.ones((n, L), dtype=torch.bool, device="cuda").triu(L - n + 1)
        for h in range(H):
            s = (q[:, h].reshape(n * G, D) @ k[:, h].t().contiguous()).view(n, G, L) * D ** -0.5
            s.masked_fill_(hidden[:, None, :], -math.inf)
            lse = torch.logsumexp(s, -1, keepdim=True)
            outs.append((s.sub_(lse).exp_().view(n * G, L) @ v[:, h]).view(n, G, D))
            lses.append(lse.squeeze(-1))
    # pieces come request by request, head by head
    parts = lambda x: torch.cat([torch.cat(x[i * H:(i + 1) * H], 1) for i in range(case["B"])])  # noqa: E731
    return (parts(outs), parts(lses)) if case["lse"] else (parts(outs),)
