"""A worker's cache held in 4 bits, as a serving loop calls it.

The blocks that a worker can keep bound the prefixes that a router can send it.
In this cache 32 neighbouring values of a head share a power of two and each is
a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6: 4.25 bits a value.  Three
operators:

write    the new tokens' keys and values are put into the cache; they are then
         read back as the cache holds them, so that whoever uses them in this
         step sees what the next steps will see
read     tokens of the cache as 16-bit values again: a prefix that is handed to
         a worker with a 16-bit cache
attend   attention of the new tokens over the cache, a group's shared prefix
         read once for all its members

Blocks are 16 tokens.  Lengths are drawn from the case alone; block numbers,
slots, queries, keys and values from the seed.
"""
import math

import numpy as np
import torch

own = False

BLOCK, SHARE = 16, 32
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EXPONENTS = {"bf16": (-125, 125), "fp16": (-23, 13)}   # of the shared powers of two, so that the type holds every value


def _batch_case(name, B, groups, prefix, tail, new, **more):
    """B requests in `groups` groups (0: nothing is shared); a group's prefix, a request's tokens after it and how
    many of those are new are each (lowest, highest)."""
    c = dict(name=name, kind="attend", B=B, groups=groups, prefix_lo=prefix[0], prefix_hi=prefix[1], tail_lo=tail[0],
             tail_hi=tail[1], new_lo=new[0], new_hi=new[1])
    c.update(more)
    return c


def listed():
    return [
        # a decoding batch's new tokens, on a quarter of eight key heads; and a step's prompts on all of them
        dict(name="write_decode", kind="write", T=64, Hkv=2, D=128, blocks=4096, dtype="bf16", heads_first=False),
        dict(name="write_prompts", kind="write", T=16384, Hkv=8, D=128, blocks=2048, dtype="bf16", heads_first=True),
        # a short prefix and a long conversation, handed on
        dict(name="read_prefix", kind="read", T=500, Hkv=5, D=80, blocks=700, dtype="fp16", heads_first=False),
        dict(name="read_long", kind="read", T=65536, Hkv=8, D=128, blocks=6000, dtype="bf16", heads_first=True),
        # one user alone, a short answer so far: all latency
        _batch_case("attend_one", 1, 0, (0, 0), (100, 100), (1, 1), Hq=16, Hkv=2, D=128, dtype="bf16", heads_first=False,
                    lse=False),
        # a decoding batch with nothing in common, and few long conversations: the cache is read at its full rate or not
        _batch_case("attend_decode", 96, 0, (0, 0), (500, 12000), (1, 1), Hq=64, Hkv=8, D=128, dtype="bf16",
                    heads_first=True, lse=False),
        _batch_case("attend_long", 5, 0, (0, 0), (60000, 200000), (1, 1), Hq=16, Hkv=4, D=128, dtype="bf16",
                    heads_first=True, lse=False),
        # a system prompt that the whole batch shares, one token each
        _batch_case("attend_prompt_shared", 128, 1, (8192, 8192), (16, 512), (1, 1), Hq=64, Hkv=8, D=128, dtype="bf16",
                    heads_first=True, lse=False),
        # requests of several groups and lengths, and of none
        _batch_case("attend_groups", 200, 24, (512, 16384), (1, 4000), (1, 1), Hq=16, Hkv=2, D=128, dtype="fp16",
                    heads_first=False, lse=True),
        # pieces of long prompts beside decoding requests, heads of 192
        _batch_case("attend_pieces", 12, 3, (2000, 8000), (1, 3000), (1, 700), Hq=12, Hkv=1, D=192, dtype="bf16",
                    heads_first=False, lse=True),
        # a few drafted tokens for each request, heads that fill no whole share
        _batch_case("attend_drafts", 40, 0, (0, 0), (33, 9000), (2, 5), Hq=20, Hkv=5, D=80, dtype="fp16",
                    heads_first=True, lse=False),
        # whole prompts
        _batch_case("attend_prompts", 3, 0, (0, 0), (2500, 6000), (6000, 6000), Hq=64, Hkv=8, D=128, dtype="bf16",
                    heads_first=True, lse=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("write", "read", "attend", "attend", "attend", "attend"))
    heads = dict(Hkv=rng.choice((1, 2, 3, 4, 5, 8)), D=rng.choice((64, 128, 128, 128, 192, 256, 80, 96, 40)),
                 dtype=rng.choice(("bf16", "fp16")), heads_first=rng.random() < 0.5)
    if kind != "attend":
        T = _log(rng, 1, 12000 if kind == "write" else 40000)
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
    c = _batch_case("", B, rng.choice((0, 1, max(1, B // 6))), (16, prefix), (1 if B > 1 else tail, tail),
                    (1 if shape == "pieces" else new, new), **heads)
    del c["name"]
    return c


# ------------------------------------------------------------------ the format

def _shares(D):
    return -(-D // SHARE)


def _encode(x, dtype):
    """Codes [..., 16 shares] and scales [..., shares] of values [..., D]; whole shares, the missing values 0."""
    D = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, SHARE * _shares(D) - D)).unflatten(-1, (-1, SHARE))
    top = x.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(x).all(-1, keepdim=True)
    m, e = torch.frexp(torch.where(finite, top, 0))          # top = m 2^e, m in [0.5, 1): the least power with top <= 7 2^e
    e = e - 3 + (m > 0.875).to(e.dtype)
    e = torch.where(top > 0, e, -1000).clamp(*EXPONENTS[dtype])
    y = torch.ldexp(torch.ldexp(x.abs(), -e // 2), -e - (-e // 2))      # (2^-e alone might not be a number)
    # the nearest of the eight magnitudes, ties to the even code
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)).to(torch.uint8)
    code = torch.where(finite, code + 8 * torch.signbit(x).to(torch.uint8), 0).flatten(-2)
    scale = torch.where(finite, e + 127, 255).squeeze(-1).to(torch.uint8)
    return code[..., ::2] + 16 * code[..., 1::2], scale


def _tables(dev):
    """The two values that a byte of codes stands for, and what a scale does."""
    one = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=dev)
    one = torch.cat([one, -one])
    pair = torch.stack([one.repeat(16), one.repeat_interleave(16)], 1)
    power = torch.ldexp(torch.ones(256, device=dev, dtype=torch.float64), torch.arange(256, device=dev) - 127).float()
    power[255] = math.nan
    return pair, power


def _decode(codes, scales, D):
    """The values [..., D] held, in 32 bits."""
    pair, power = _tables(codes.device)
    x = pair[codes.int()].flatten(-2).unflatten(-1, (-1, SHARE)) * power[scales.int()].unsqueeze(-1)
    return x.flatten(-2)[..., :D]


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
    return first, group_off, shared, prefix + tail, np.minimum(_spread(rng, case["new_lo"], case["new_hi"], B), tail)


def _cache(case, blocks, gen):
    """Codes and scales of keys or of values, [block, token, head, bytes]; heads_first: with a block's heads before its
    tokens.  The keys and values are normal."""
    H, D, dtype = case["Hkv"], case["D"], case["dtype"]
    shape = (blocks, H, BLOCK) if case["heads_first"] else (blocks, BLOCK, H)
    codes, scales = _encode(torch.randn(shape + (D,), generator=gen, device="cuda", dtype=TYPES[dtype]), dtype)
    return (codes.transpose(1, 2), scales.transpose(1, 2)) if case["heads_first"] else (codes, scales)


def _caches(case, blocks, gen):
    k, ks = _cache(case, blocks, gen)
    v, vs = _cache(case, blocks, gen)
    return dict(k_cache=k, v_cache=v, k_scales=ks, v_scales=vs)


def _prepare_tokens(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, H, D = case["T"], case["Hkv"], case["D"]
    slots = torch.randperm(BLOCK * case["blocks"], generator=gen, device="cuda")[:T]
    st = dict(case=case, slots=slots, **_caches(case, case["blocks"] + 1, gen))        # the last block is nobody's
    if case["kind"] == "write":
        new = torch.randn((T, H, 2, D), generator=gen, device="cuda", dtype=TYPES[case["dtype"]])
        elsewhere = torch.rand(T, generator=gen, device="cuda") < 0.02                 # tokens that another request writes
        st.update(k=new[:, :, 0], v=new[:, :, 1], slots=torch.where(elsewhere, -1, slots))
    return st


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
    ids = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    tables = torch.where(p[None, :] < _up(need)[:, None], ids[row.clamp_(0, blocks - 1)], 0)
    q_off = np.zeros(B + 1, np.int64)
    np.cumsum(new, out=q_off[1:])
    q = torch.randn((int(q_off[-1]), Hq, D), generator=gen, device="cuda", dtype=TYPES[case["dtype"]])
    return dict(case=case, q=q, tables=tables, kv_len=_up(kv.astype(np.int32)), q_off=_up(q_off), group_off=_up(group_off),
                shared=_up(shared.astype(np.int32)), most_new=int(new.max()), **_caches(case, blocks, gen))


def prepare(case, seed):
    return _prepare_attend(case, seed) if case["kind"] == "attend" else _prepare_tokens(case, seed)


# ------------------------------------------------------------------ plain forms

def _plain_read(st):
    D, dtype, slots = st["case"]["D"], TYPES[st["case"]["dtype"]], st["slots"]
    there = (slots >= 0)[:, None, None]
    at = slots.clamp(min=0)
    b, t = at // BLOCK, at % BLOCK
    k = _decode(st["k_cache"][b, t], st["k_scales"][b, t], D)
    v = _decode(st["v_cache"][b, t], st["v_scales"][b, t], D)
    return torch.where(there, k, 0).to(dtype), torch.where(there, v, 0).to(dtype)


def _plain_write(st):
    n = st["case"]["blocks"]
    slot = torch.where(st["slots"] < 0, BLOCK * n, st["slots"])           # into nobody's block
    b, t = slot // BLOCK, slot % BLOCK
    st["k_cache"][b, t], st["k_scales"][b, t] = _encode(st["k"], st["case"]["dtype"])
    st["v_cache"][b, t], st["v_scales"][b, t] = _encode(st["v"], st["case"]["dtype"])
    return _plain_read(st)


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
    k = _decode(st["k_cache"][tables], st["k_scales"][tables], D).flatten(1, 2).permute(0, 2, 3, 1).reshape(B * H, D, -1)
    s = torch.bmm(qs, k).view(B, H, Hq // H, n, -1)
    del k
    s.masked_fill_(there > pos[:, None, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = s.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    v = _decode(st["v_cache"][tables], st["v_scales"][tables], D).flatten(1, 2)
    v = v.masked_fill((there >= kv[:, None])[:, :, None, None], 0).transpose(1, 2).reshape(B * H, -1, D)
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
    case = st["case"]
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[case["kind"]](st)
    from paper_2606_17081_amd import rkroute as rk
    if case["kind"] == "attend":
        out, lse = rk.prefix_attention_fp4(st["q"], st["k_cache"], st["v_cache"], st["k_scales"], st["v_scales"],
                                           st["tables"], st["kv_len"], st["q_off"], group_off=st["group_off"],
                                           shared=st["shared"], want_lse=case["lse"])
        return (out, lse) if case["lse"] else (out,)
    caches = st["k_cache"], st["v_cache"], st["k_scales"], st["v_scales"]
    if case["kind"] == "write":
        rk.kv_write_fp4(st["k"], st["v"], *caches, st["slots"])
    return rk.kv_read_fp4(*caches, st["slots"], D=case["D"], dtype=TYPES[case["dtype"]])


def work(case):
    H, D = case["Hkv"], case["D"]
    row = 16 * _shares(D) + _shares(D)                    # bytes of a token's head in a cache
    if case["kind"] != "attend":
        # values in (of a write), rows of the cache in or out, values out
        wide = 2 * D * (2 if case["kind"] == "write" else 1)
        return {"bytes": 2 * case["T"] * H * (row + wide) + 8 * case["T"], "flops": 0}
    first, group_off, shared, kv, new = _lengths(case)
    B, Hq = case["B"], case["Hq"]
    group = np.searchsorted(group_off, np.arange(B), side="right") - 1
    lead = np.where(first == np.arange(B), 0, shared[group])
    keys = int((kv - BLOCK * lead).sum())                 # a group's prefix once
    pairs = int((new * kv - new * (new - 1) // 2).sum())  # each new token and what it sees
    tokens = int(new.sum())
    return {"bytes": 2 * keys * H * row + 2 * 2 * tokens * Hq * D + (4 * tokens * Hq if case["lse"] else 0)
            + 4 * int((-(-kv // BLOCK) - lead).sum()) + 28 * B, "flops": 4 * pairs * Hq * D}


# ------------------------------------------------------------------ in 64 bits

def _held(codes, scales, D):
    """The values held, bit by bit: e2m1 is 0 or 0.5 where its two exponent bits are 0, else (1 + m / 2) 2^(e - 1)."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)[..., :D].double()
    sign, rest = torch.div(c, 8, rounding_mode="floor"), c % 8
    e, m = torch.div(rest, 2, rounding_mode="floor"), rest % 2
    x = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e - 1)) * (1 - 2 * sign)
    s = scales.double().repeat_interleave(SHARE, -1)[..., :D]
    return torch.where(s == 255, math.nan, x * torch.exp2(s - 127))


def _rounded(x, dtype):
    """What the cache holds in the place of values [T, H, D]: each group of 32 on the grid of its power of two."""
    lo, hi = EXPONENTS[dtype]
    D = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, SHARE * _shares(D) - D)).unflatten(-1, (-1, SHARE))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 7)).clamp(lo, hi)
    e = torch.where(top > 7 * torch.exp2(e), e + 1, e)                                 # (the logarithm's rounding)
    e = torch.where(top <= 7 * torch.exp2(e - 1), e - 1, e).clamp(lo, hi)
    y = x.abs() / torch.exp2(e)
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    held = torch.clamp(torch.round(y / step) * step, max=6) * torch.exp2(e)            # (halves to even)
    return torch.copysign(held, x).flatten(-2)[..., :D]


def exact(case, seed):
    """The definitions in 64 bits: attention request by request, writes value by value."""
    st = prepare(case, seed)
    D = case["D"]
    if case["kind"] == "write":
        there = (st["slots"] >= 0)[:, None, None]
        return tuple(torch.where(there, _rounded(st[x], case["dtype"]), 0) for x in ("k", "v"))
    if case["kind"] == "read":
        b, t = st["slots"] // BLOCK, st["slots"] % BLOCK
        return tuple(_held(st[x + "_cache"][b, t], st[x + "_scales"][b, t], D) for x in ("k", "v"))
    off, kv = st["q_off"].tolist(), st["kv_len"].tolist()
    H, G = case["Hkv"], case["Hq"] // case["Hkv"]
    outs, lses = [], []
    for i in range(case["B"]):
        n, L = off[i + 1] - off[i], kv[i]
        rows = st["tables"][i, : -(-L // BLOCK)].long()
        k, v = (_held(st[x + "_cache"][rows], st[x + "_scales"][rows], D).reshape(-1, H, D)[:L] for x in ("k", "v"))
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
