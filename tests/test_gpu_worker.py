"""A worker's step on the GPU against the numpy oracle: prefix groups, block
tables, cache writes (equal), attention (within the roundings that its
definition allows), alone and together, captured and on other streams."""
import zlib

import numpy as np
import pytest

from oracle import worker as ow

pytestmark = pytest.mark.gpu

BLOCK = 16
STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}       # half a step of the type, relative


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2606_17081_amd import rkroute as rk
    rk.lib()
    assert rk.device_status(reset=True) == 0
    return torch, rk


def rng_of(*what):
    return np.random.default_rng(zlib.crc32(repr(what).encode()))


def offsets(n):
    return np.concatenate([[0], np.cumsum(np.asarray(n, np.int64))]).astype(np.int64)


def dtype_of(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float16


def host(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


# ------------------------------------------------------------------ groups

def chains_of(rng, B, groups, longest, shortest=1):
    base = rng.integers(1, 2 ** 62, (groups, longest)).astype(np.uint64)
    L = rng.integers(shortest, longest + 1, B)
    rows = []
    for i in range(B):
        c = int(rng.integers(0, L[i] + 1))
        rows.append(np.concatenate([base[rng.integers(0, groups), :c], rng.integers(1, 2 ** 62, L[i] - c).astype(np.uint64)]))
    return np.concatenate(rows + [np.zeros(0, np.uint64)]), offsets(L)


def check_groups(gpu, chains, off, least):
    torch, rk = gpu
    got = rk.prefix_groups(rk.to_device(chains if chains.size else np.zeros(1, np.uint64)), rk.to_device(off), least)
    want = ow.prefix_groups(chains, off, least)
    for g, w in zip(got, want):
        assert np.array_equal(host(g), np.atleast_1d(w))


@pytest.mark.parametrize("B,groups,longest,least", [
    (0, 1, 4, 1), (1, 1, 5, 1), (2, 1, 1, 1), (3, 1, 40, 2), (63, 5, 30, 1), (64, 1, 300, 3), (65, 64, 9, 1),
    (127, 3, 17, 18), (200, 66, 33, 1), (1000, 7, 64, 2), (1025, 300, 20, 1), (4095, 1000, 12, 1), (4096, 1, 70, 1),
    (4096, 4000, 3, 1)])
def test_groups(gpu, B, groups, longest, least):
    rng = rng_of(B, groups, longest)
    chains, off = chains_of(rng, B, groups, longest, 0 if B > 4 else 1)
    check_groups(gpu, chains, off, least)
    assert gpu[1].device_status(reset=True) == 0


def test_groups_whole_prefixes_and_one_block(gpu):
    """Chains that are prefixes of each other, all equal, or differ at either end only."""
    base = rng_of("whole").integers(1, 2 ** 62, 2000).astype(np.uint64)
    for lengths in ([2000, 1999, 1, 1000, 16, 17], [17] * 5, [2000] * 3, [16, 32, 15, 33, 64]):
        check_groups(gpu, np.concatenate([base[:n] for n in lengths]), offsets(lengths), 1)
    rows = [base.copy() for _ in range(40)]
    for i, r in enumerate(rows[1:]):
        r[1999 - 50 * i:] += np.uint64(1)
    check_groups(gpu, np.concatenate(rows), offsets([2000] * 40), 20)
    assert gpu[1].device_status(reset=True) == 0


def test_groups_same_low_bits(gpu):
    """Keys that all want the same slot."""
    rng = rng_of("low")
    keys = (rng.permutation(3000)[:1500].astype(np.uint64) + np.uint64(1)) << np.uint64(32)
    chains = keys[rng.integers(0, 1500, 4000)]
    check_groups(gpu, chains, np.arange(4001, dtype=np.int64), 1)


def test_groups_zero_hash_and_bad_offsets(gpu):
    torch, rk = gpu
    chains = np.array([0, 0, 5, 5], np.uint64)
    check_groups(gpu, chains, np.arange(5, dtype=np.int64), 1)
    assert rk.device_status(reset=True) == 0x4
    order, off, shared, n = rk.prefix_groups(rk.to_device(chains), rk.to_device(np.array([0, 3, 2, 4])), 1)
    assert sorted(host(order).tolist()) == [0, 1, 2] and rk.device_status(reset=True) & 0x1


@pytest.mark.parametrize("B", [2, 5, 64, 128, 129, 700])
@pytest.mark.parametrize("longest", [6, 7, 33, 300])
def test_groups_chains_left_short(gpu, B, longest):
    """Chains whose last hashes are missing (0), agreeing with the group's first chain up to there or less far, and the first
    chain itself left short: missing hashes are in common with none."""
    rng = rng_of("short", B, longest)
    base = rng.integers(1, 2 ** 62, longest).astype(np.uint64)
    for first_missing in (0, 1, longest // 2):
        rows = []
        for i in range(B):
            r = base.copy()
            agree = int(rng.integers(1, longest + 1))
            r[agree:] = rng.integers(1, 2 ** 62, longest - agree).astype(np.uint64)
            missing = first_missing if i == 0 else int(rng.integers(0, longest))
            r[longest - missing:] = 0
            rows.append(r)
        check_groups(gpu, np.concatenate(rows), offsets([longest] * B), 1)
        # two blocks, of which one agrees, and nothing else
        short = np.zeros((B, longest), np.uint64)
        short[:, 0] = base[0]
        short[:, 1] = base[1] + np.arange(B, dtype=np.uint64)
        check_groups(gpu, short.reshape(-1), offsets([longest] * B), 1)
    assert gpu[1].device_status(reset=True) == 0


# ------------------------------------------------------------------ tables

def lengths_of(rng, B, groups, shared_most, tail_most, new_most, fresh):
    """Groups side by side, lengths, and what each row holds already."""
    if groups:
        cut = np.sort(rng.integers(0, B + 1, groups - 1)) if B else np.zeros(groups - 1, np.int64)
        goff = np.concatenate([[0], cut, np.full(B + 1 - groups, B)]).astype(np.int64) if groups <= B else \
            np.concatenate([[0], np.full(B, B)]).astype(np.int64)
        shared = rng.integers(0, shared_most + 1, B).astype(np.int32)
    else:
        goff, shared = None, None
    kv = rng.integers(0, tail_most + 1, B)
    if groups:
        for g in range(B):
            for i in range(goff[g], goff[g + 1]):
                kv[i] += BLOCK * shared[g] if rng.random() < 0.9 else 0
    new = np.minimum(rng.integers(0, new_most + 1, B), kv) if B else kv
    have = np.zeros(B, np.int64) if fresh else -(-(kv - new) // BLOCK)
    return goff, shared, kv.astype(np.int32), new.astype(np.int32), have.astype(np.int32)


def run_tables(gpu, tables, kv, new, have, free, n_slots, goff, shared):
    torch, rk = gpu
    up = rk.to_device
    t = up(tables)
    got = rk.block_tables(t, up(kv), up(new), up(have), up(free), n_slots, None if goff is None else up(goff),
                          None if shared is None else up(shared))
    assert got[0] is t
    return [host(x) for x in got]


@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("B,groups,shared_most,tail_most,new_most", [
    (0, 0, 0, 0, 0), (1, 0, 0, 1, 1), (1, 1, 3, 40, 40), (2, 1, 5, 17, 1), (7, 3, 9, 100, 60), (64, 0, 0, 300, 1),
    (65, 9, 20, 33, 5), (300, 300, 4, 50, 50), (1025, 40, 6, 70, 64), (4096, 100, 3, 40, 3), (3, 1, 300, 9000, 9000)])
def test_tables(gpu, B, groups, shared_most, tail_most, new_most, fresh):
    rng = rng_of(B, groups, shared_most, fresh)
    goff, shared, kv, new, have = lengths_of(rng, B, groups, shared_most, tail_most, new_most, fresh)
    stride = int(-(-kv.max(initial=1) // BLOCK)) + 2
    tables = rng.integers(1000, 2000, (max(B, 1), stride)).astype(np.int32)
    need = int((-(-kv.astype(np.int64) // BLOCK)).sum())
    free = rng.permutation(need + 7).astype(np.int32) + 5000
    for n_slots in (int(new.sum()), int(new.sum()) + 70):
        got = run_tables(gpu, tables, kv, new, have, free, n_slots, goff, shared)
        want = ow.block_tables(tables, kv, new, have, free, n_slots, goff, shared)
        for g, w in zip(got, want):
            assert np.array_equal(g, np.atleast_1d(w))
    assert gpu[1].device_status(reset=True) == 0


def test_tables_free_list_ends(gpu):
    rng = rng_of("ends")
    goff, shared, kv, new, have = lengths_of(rng, 40, 4, 6, 90, 60, True)
    tables = np.full((40, 30), 7, np.int32)
    for n_free in (0, 1, 33):
        got = run_tables(gpu, tables, kv, new, have, np.arange(n_free, dtype=np.int32), int(new.sum()), goff, shared)
        want = ow.block_tables(tables, kv, new, have, np.arange(n_free), int(new.sum()), goff, shared)
        for g, w in zip(got, want):
            assert np.array_equal(g, np.atleast_1d(w))
        assert gpu[1].device_status(reset=True) == 0x8


def test_tables_bad_lengths_and_groups(gpu):
    """A request out of bounds counts as empty, offsets that are no partition as none; nothing else changes."""
    kv = np.array([20, 300, 20, -5, 20, 20], np.int32)
    new = np.array([5, 5, 30, 0, -1, 20], np.int32)
    have = np.array([1, 0, 0, 0, 0, 0], np.int32)
    tables, free = np.full((6, 16), 3, np.int32), np.arange(100, 120, dtype=np.int32)
    ok = np.array([True, False, False, False, False, True])
    want = ow.block_tables(tables, kv * ok, new * ok, have, free, 30)
    for goff in (None, np.array([0, 4, 3, 6, 6, 6, 6]), np.array([1, 6, 6, 6, 6, 6, 6]), np.array([0, 2, 5, 5, 5, 5, 5]),
                 np.array([0, 7, 7, 7, 7, 7, 7])):
        got = run_tables(gpu, tables, kv, new, have, free, 30, goff, None if goff is None else np.full(6, 4, np.int32))
        for g, w in zip(got, want):
            assert np.array_equal(g, np.atleast_1d(w))
        assert gpu[1].device_status(reset=True) == 0x1 | 0x10
    got = run_tables(gpu, tables, kv * ok, new * ok, have, free, 10, None, None)
    assert np.array_equal(got[1], want[1][:10]) and gpu[1].device_status(reset=True) == 0x2


# ------------------------------------------------------------------ cache writes

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,Hkv,D,blocks,heads_first", [
    (0, 1, 8, 1, False), (1, 1, 8, 1, False), (1, 2, 128, 3, True), (17, 3, 72, 9, False), (100, 8, 64, 40, True),
    (33, 1, 256, 2, False), (1000, 5, 96, 70, True), (7000, 2, 128, 600, False)])
def test_write(gpu, T, Hkv, D, blocks, heads_first, dtype):
    torch, rk = gpu
    rng = rng_of(T, Hkv, D)
    bits = lambda *n: torch.from_numpy(rng.integers(-2 ** 15, 2 ** 15, n).astype(np.int16)).cuda()  # noqa: E731
    new = bits(T, Hkv + 2, 2, D).view(dtype_of(torch, dtype))[:, 1:1 + Hkv]            # every bit pattern, NaN too
    caches = [bits(*((blocks, Hkv, BLOCK, D) if heads_first else (blocks, BLOCK, Hkv, D))) for _ in range(2)]
    views = [c.view(dtype_of(torch, dtype)).transpose(1, 2) if heads_first else c.view(dtype_of(torch, dtype)) for c in caches]
    slots = rng.permutation(BLOCK * blocks)[:T]
    slots = np.where(rng.random(slots.size) < 0.2, -1, slots)
    slots = np.concatenate([slots, np.full(T - slots.size, -3)]).astype(np.int64)
    want = [v.clone() for v in views]
    for w, n in zip(want, (new[:, :, 0], new[:, :, 1])):
        for t in np.nonzero(slots >= 0)[0]:
            w[slots[t] // BLOCK, slots[t] % BLOCK] = n[int(t)]
    rk.kv_write(new[:, :, 0], new[:, :, 1], views[0], views[1], rk.to_device(slots) if T else torch.zeros(0, dtype=torch.int64, device="cuda"))
    for w, v in zip(want, views):
        assert torch.equal(w.contiguous().view(torch.int16), v.contiguous().view(torch.int16))
    assert rk.device_status(reset=True) == 0


def test_write_slot_behind_the_cache(gpu):
    torch, rk = gpu
    c = torch.zeros((3, BLOCK, 1, 8), dtype=torch.bfloat16, device="cuda")
    ones = torch.ones((4, 1, 8), dtype=torch.bfloat16, device="cuda")
    rk.kv_write(ones, ones, c[:2], c[:2].clone(), torch.tensor([31, 32, 1 << 40, -1], device="cuda"))
    assert float(c.sum()) == 8 and float(c[1, 15].sum()) == 8
    assert rk.device_status(reset=True) == 0x80


# ------------------------------------------------------------------ attention

class Batch:
    """Requests over a block cache: `kv` and `new` by request, `goff` and `shared` by group; garbage everywhere that
    belongs to no sequence."""

    def __init__(self, torch, rng, kv, new, Hq, Hkv, D, dtype="bf16", goff=None, shared=None, heads_first=False,
                 together=False, rows_behind=0, garbage=float("nan"), spread=1.0, extra_blocks=3):
        self.torch, self.dtype = torch, dtype
        kv, new = np.asarray(kv, np.int64), np.asarray(new, np.int64)
        B, ty = kv.size, dtype_of(torch, dtype)
        first, lead = ow.leads(kv, goff, shared)
        need = -(-kv // BLOCK)
        lead = np.minimum(lead, need)
        blocks = int((need - lead).sum()) + extra_blocks
        ids = rng.permutation(blocks).astype(np.int32)
        self.tables = np.full((max(B, 1), int(need.max(initial=0)) + 1), -1, np.int32)
        at = 0
        for i in range(B):
            self.tables[i, :lead[i]] = self.tables[first[i], :lead[i]]
            self.tables[i, lead[i]:need[i]] = ids[at:at + need[i] - lead[i]]
            at += need[i] - lead[i]
        shape = (blocks, Hkv, BLOCK, D) if heads_first else (blocks, BLOCK, Hkv, D)
        caches = [torch.from_numpy(rng.normal(size=shape).astype(np.float32) * spread).cuda().to(ty) for _ in range(2)]
        if together:                 # one tensor of keys and values
            caches = list(torch.stack(caches, 1).unbind(1))
        self.caches = [c.transpose(1, 2) if heads_first else c for c in caches]
        owned = torch.zeros((blocks, BLOCK), dtype=torch.bool)
        for i in range(B):
            p = np.arange(kv[i])
            owned[self.tables[i][p // BLOCK].astype(np.int64), p % BLOCK] = True
        for c in self.caches:
            c[~owned.cuda()] = garbage
        self.kv, self.new, self.goff, self.shared = kv.astype(np.int32), new, goff, shared
        self.q_off = offsets(new)
        T = int(self.q_off[-1]) + rows_behind
        self.q = torch.from_numpy(rng.normal(size=(T, Hq + 1, D)).astype(np.float32) * spread).cuda().to(ty)[:, :Hq]
        self.Hq, self.Hkv, self.D = Hq, Hkv, D

    def args(self, rk):
        up = rk.to_device
        more = {} if self.goff is None else dict(group_off=up(self.goff), shared=up(self.shared.astype(np.int32)))
        return [self.q, *self.caches, up(self.tables), up(self.kv), up(self.q_off)], more

    def want(self, **kw):
        return ow.attention(host(self.q), host(self.caches[0]), host(self.caches[1]), self.tables, self.kv, self.q_off, **kw)

    def check(self, out, lse, scale=None, want=None):
        """Half a step of the type for the result, one for each weight (relative, so as much of the mean of |v|), and
        the fp32 sums: a score is off by at most (D + 2) steps of sum |q k|, a weight by twice that with its maximum,
        the sums over n keys by (n + 2) steps of the mean of |v|, the exponentials by a few."""
        o, l, mean, most = self.want(scale=scale) if want is None else want
        u, e = STEP[self.dtype], 2.0 ** -24
        rows = int(self.q_off[-1])
        out, lse = host(out)[:rows], host(lse)[:rows]
        o, l, mean, most = o[:rows], l[:rows], mean[:rows], most[:rows]
        n = float(self.kv.max(initial=0))
        weight = (2 * (self.D + 2) * most + 2 * n + 64) * e
        bound = u * np.abs(o) + (1 + u) * (u + weight[..., None]) * mean + (2.0 ** -24 if self.dtype == "fp16" else 1e-38)
        fine = np.isfinite(o)
        assert np.array_equal(fine, np.isfinite(out))
        assert np.array_equal(np.isnan(o), np.isnan(out)) and np.array_equal(o[~fine & ~np.isnan(o)], out[~fine & ~np.isnan(o)])
        over = (np.abs(out - np.where(fine, o, 0)) > bound) & fine
        assert not over.any(), (np.argwhere(over)[:5], out[over][:5], o[over][:5], bound[over][:5])
        fine = np.isfinite(l)
        assert np.array_equal(np.isfinite(lse), fine) and np.array_equal(np.isnan(l), np.isnan(lse))
        assert np.array_equal(l[~fine & ~np.isnan(l)], lse[~fine & ~np.isnan(l)])
        assert (np.abs(lse[fine] - l[fine]) <= weight[fine] + 4 * e * np.abs(l[fine])).all()


def attend(gpu, b, scale=None, **kw):
    torch, rk = gpu
    a, more = b.args(rk)
    out, lse = rk.prefix_attention(*a, **more, scale=scale, want_lse=True, **kw)
    b.check(out, lse, scale)
    return out, lse


@pytest.mark.parametrize("kv", [1, 2, 15, 16, 17, 31, 33, 100, 127, 128, 129, 255, 500, 1025, 5000])
def test_attend_single_token(gpu, kv):
    b = Batch(gpu[0], rng_of(kv), [kv], [1], 16, 2, 128)
    attend(gpu, b)
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("Hq,Hkv,D", [(1, 1, 8), (2, 1, 64), (8, 1, 128), (12, 1, 192), (16, 2, 256), (7, 1, 80), (5, 5, 96),
                                      (40, 8, 128), (128, 1, 64), (34, 1, 128), (10, 2, 136), (33, 11, 72), (17, 1, 248),
                                      (24, 8, 16)])
def test_attend_head_layouts(gpu, Hq, Hkv, D, dtype):
    rng = rng_of(Hq, Hkv, D, dtype)
    kv = rng.integers(1, 400, 9)
    new = np.minimum(rng.integers(0, 40, 9), kv)
    new[:3] = np.minimum([1, 130, 0], kv[:3])
    b = Batch(gpu[0], rng, kv, new, Hq, Hkv, D, dtype, heads_first=bool(Hq % 2), rows_behind=3)
    attend(gpu, b)
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("heads_first,together", [(False, False), (True, False), (False, True), (True, True)])
def test_attend_cache_strides(gpu, heads_first, together):
    rng = rng_of("strides", heads_first, together)
    b = Batch(gpu[0], rng, [70, 1, 300, 16], [3, 1, 300, 16], 8, 4, 64, heads_first=heads_first, together=together)
    attend(gpu, b)


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (16, 2, 64), (12, 1, 192), (3, 3, 256)])
@pytest.mark.parametrize("kv,new", [([300], [300]), ([129, 700, 1], [129, 500, 1]), ([1000, 64, 63, 65], [1, 64, 63, 65]),
                                    ([2000], [33]), ([513, 514], [257, 129])])
def test_attend_many_new_tokens(gpu, kv, new, Hq, Hkv, D):
    """Prompts and pieces of prompts: each token sees up to itself."""
    b = Batch(gpu[0], rng_of(kv, new, Hq), kv, new, Hq, Hkv, D)
    attend(gpu, b)
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("sizes,shared,tail,new", [
    ([2], [1], 20, 1), ([40], [30], 50, 1), ([1, 5, 1, 9], [3, 8, 100, 1], 200, 1), ([3, 3], [64, 0], 33, 4),
    ([70, 2], [9, 130], 40, 1), ([6], [20], 300, 150), ([200], [5], 3, 2), ([3, 4], [7, 40], 0, 0)])
def test_attend_groups(gpu, sizes, shared, tail, new, dtype):
    rng = rng_of(sizes, shared, tail)
    B = sum(sizes)
    goff = np.concatenate([offsets(sizes), np.full(B + 1 - len(sizes) - 1, B)]).astype(np.int64)
    sh = np.zeros(B, np.int32)
    sh[:len(sizes)] = shared
    prefix = BLOCK * np.repeat(shared, sizes)
    own = rng.integers(0, tail + 1, B)
    kv = prefix + np.maximum(own, 1 if new else 0)
    n = np.minimum(rng.integers(1 if new else 0, new + 1, B) if new else np.zeros(B, np.int64), np.maximum(own, 1))
    b = Batch(gpu[0], rng, kv, n, 8, 2, 128, dtype, goff=goff, shared=sh, rows_behind=2)
    attend(gpu, b)
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("sizes,shared,tail,new,Hq,Hkv,D,dtype,apart", [
    ([30], [100], 20, 1, 8, 2, 128, "bf16", ()), ([2], [300], 100, 1, 4, 4, 64, "fp16", ()), ([3], [90], 700, 1, 12, 1, 192, "bf16", ()),
    ([40, 2, 50], [60, 200, 33], 40, 3, 7, 1, 80, "bf16", (1,)), ([64, 70], [70, 50], 1, 1, 16, 1, 256, "fp16", ()),
    ([9, 200, 7], [25, 40, 31], 30, 1, 8, 8, 64, "bf16", ()), ([5], [120], 60, 12, 16, 2, 128, "bf16", ()),
    ([20], [4000], 30, 1, 8, 1, 128, "bf16", ()), ([300], [20], 16, 1, 1, 1, 128, "fp16", ())])
def test_attend_prefix_read_once(gpu, sizes, shared, tail, new, Hq, Hkv, D, dtype, apart):
    """Prefixes long enough that a group attends to them together: through one row, the others' entries are not read.
    apart: groups of the case whose members do it each for themselves all the same.  (In the fourth case two members of 200
    shared blocks have up to 42 rows: one wide tile of 50 steps, 4 (12 + 2 * 50) + 4 * 2 * 2 = 464 quarters of the cost
    unit, against 2 * 200 = 400 for the members' own steps.)"""
    torch, rk = gpu
    rng = rng_of("once", sizes, shared)
    B = sum(sizes)
    goff = np.concatenate([offsets(sizes), np.full(B - len(sizes), B)]).astype(np.int64)
    sh = np.zeros(B, np.int32)
    sh[:len(sizes)] = shared
    own = rng.integers(1, tail + 1, B)
    n = np.minimum(rng.integers(1, new + 1, B), own)
    b = Batch(torch, rng, BLOCK * np.repeat(shared, sizes) + own, n, Hq, Hkv, D, dtype, goff=goff, shared=sh,
              heads_first=Hq == 8)
    want = b.want()
    attend(gpu, b)
    for i in range(B):
        g = int(np.searchsorted(goff, i, side="right")) - 1
        if i != goff[g] and g not in apart:
            b.tables[i, :sh[g]] = -1
    a, more = b.args(rk)
    out, lse = rk.prefix_attention(*a, **more, want_lse=True)
    b.check(out, lse, want=want)
    assert rk.device_status(reset=True) == 0


def test_attend_groups_over_several_launches(gpu):
    """More requests than a launch takes: a group that spans two of them is attended to in parts."""
    rng = rng_of("spans")
    sizes, sh = [700, 900, 3, 497], [40, 30, 200, 60]
    B = sum(sizes)
    goff = np.concatenate([offsets(sizes), np.full(B - 4, B)]).astype(np.int64)
    shared = np.zeros(B, np.int32)
    shared[:4] = sh
    kv = BLOCK * np.repeat(sh, sizes) + rng.integers(1, 30, B)
    attend(gpu, Batch(gpu[0], rng, kv, np.ones(B, np.int64), 2, 1, 64, goff=goff, shared=shared))
    assert gpu[1].device_status(reset=True) == 0


def test_attend_group_brings_its_prefix(gpu):
    """The step in which a group arrives: the first request's new tokens are the prefix that the others share; and one
    member whose own new tokens lie in the prefix too."""
    rng = rng_of("brings")
    for kv, new, most in (([200, 180, 170, 165, 161], [200, 20, 170, 5, 1], 10),
                          ([1700, 1620, 1700, 1605, 1601], [1700, 20, 3, 5, 1], 100),
                          ([1700, 1620, 1700, 1605, 1601], [1, 1, 300, 1, 1], 100),
                          ([1700, 1620, 1700, 1605, 1601], [1, 30, 1, 0, 1], 100)):
        for shared in (most, most - 1, most + 2, 1, 1000):
            goff, sh = np.array([0, 5, 5, 5, 5, 5]), np.array([shared, 0, 0, 0, 0], np.int32)
            b = Batch(gpu[0], rng, kv, new, 4, 2, 64, goff=goff, shared=sh)
            attend(gpu, b)
    # members shorter than what they share
    b = Batch(gpu[0], rng, [200, 30, 16, 0, 200], [1, 1, 1, 0, 2], 4, 2, 64, goff=goff,
              shared=np.array([12, 0, 0, 0, 0], np.int32))
    attend(gpu, b)
    assert gpu[1].device_status(reset=True) == 0


def test_attend_group_whose_next_member_waits(gpu):
    """The first request brings the prefix, and the next has neither new tokens nor the prefix's length: its row, which
    names other blocks there, is not the one that the others' prefix is read through.  The same where it is the first
    of a group's rest in another launch."""
    rng = rng_of("waits")
    kv, new = [1700, 10, 1620, 1605, 1601, 1630, 1640], [1700, 0, 1, 1, 1, 1, 1]
    b = Batch(gpu[0], rng, kv, new, 4, 2, 64, goff=np.array([0] + [7] * 7), shared=np.array([100] + [0] * 6, np.int32))
    b.tables[1, 1:100] = b.tables[2, 100]
    attend(gpu, b)
    B = 1100
    kv = 16 * 40 + rng.integers(1, 60, B)
    new = np.ones(B, np.int64)
    kv[1024], new[1024] = 20, 0
    b = Batch(gpu[0], rng, kv, new, 2, 1, 64, goff=np.array([0] + [B] * B), shared=np.array([40] + [0] * (B - 1), np.int32))
    b.tables[1024, 2:40] = b.tables[0, 40]
    attend(gpu, b)
    assert gpu[1].device_status(reset=True) == 0


def test_attend_many_requests(gpu):
    rng = rng_of("many")
    kv = rng.integers(1, 60, 4096)
    b = Batch(gpu[0], rng, kv, np.ones(4096, np.int64), 2, 1, 64)
    attend(gpu, b)
    sizes = [1500, 1, 2000, 595]
    goff = np.concatenate([offsets(sizes), np.full(4092, 4096)]).astype(np.int64)
    sh = np.zeros(4096, np.int32)
    sh[:4] = 5, 7, 3, 1
    kv = BLOCK * np.repeat(sh[:4], sizes) + rng.integers(1, 40, 4096)
    b = Batch(gpu[0], rng, kv, np.ones(4096, np.int64), 2, 1, 64, goff=goff, shared=sh)
    attend(gpu, b)
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("B,Hq,Hkv,D,dtype", [
    (512, 4, 1, 128, "bf16"), (513, 4, 1, 128, "bf16"), (513, 2, 2, 72, "fp16"), (1024, 2, 1, 128, "fp16"), (1024, 2, 1, 192, "bf16"),
    (1024, 1, 1, 256, "fp16"), (1025, 2, 1, 256, "bf16"), (700, 3, 1, 200, "bf16")])
def test_attend_many_requests_of_wide_heads(gpu, B, Hq, Hkv, D, dtype):
    """On both sides of where what is kept of the requests leaves room for one workgroup a CU, and of a launch's most requests;
    prompts, single tokens and empty requests, with a group and without."""
    rng = rng_of("wide heads", B, D)
    kv = rng.integers(1, 70, B)
    new = np.where(rng.random(B) < 0.1, kv, np.minimum(1, kv))
    new[rng.random(B) < 0.05] = 0
    kv[5] = new[5] = 300
    attend(gpu, Batch(gpu[0], rng, kv, new, Hq, Hkv, D, dtype))
    sizes = [B // 2, 3, B - B // 2 - 3]
    goff = np.concatenate([offsets(sizes), np.full(B - 3, B)]).astype(np.int64)
    sh = np.zeros(B, np.int32)
    sh[:3] = 30, 5, 2
    kv = BLOCK * np.repeat(sh[:3], sizes) + rng.integers(1, 20, B)
    attend(gpu, Batch(gpu[0], rng, kv, np.ones(B, np.int64), Hq, Hkv, D, dtype, goff=goff, shared=sh))
    assert gpu[1].device_status(reset=True) == 0


def test_attend_long(gpu):
    """Long sequences, cut over many workgroups."""
    rng = rng_of("long")
    attend(gpu, Batch(gpu[0], rng, [40000, 33000], [1, 2], 4, 1, 64))
    attend(gpu, Batch(gpu[0], rng, [20000], [70], 8, 1, 128))
    goff, sh = np.array([0, 3, 3, 3]), np.array([1500, 0, 0], np.int32)
    attend(gpu, Batch(gpu[0], rng, [24100, 24001, 30000], [1, 1, 3], 8, 1, 128, goff=goff, shared=sh))
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("garbage", [float("nan"), float("inf"), -3.3e38])
def test_attend_garbage_where_nothing_lies(gpu, garbage):
    """Slots behind a sequence, and blocks of nobody, hold anything."""
    b = Batch(gpu[0], rng_of("garbage"), [5, 17, 40, 130, 33], [5, 1, 3, 130, 20], 8, 2, 128, garbage=garbage)
    attend(gpu, b)


@pytest.mark.parametrize("Hq,new", [(1, 40), (8, 40), (4, 200), (16, 3)])
def test_attend_not_finite_in_later_tokens(gpu, Hq, new):
    """A key or value that is not finite shows in the tokens that see it and in no earlier one."""
    torch, rk = gpu
    rng = rng_of("later", Hq, new)
    for value in (float("nan"), float("inf"), float("-inf")):
        for which in (0, 1):
            b = Batch(torch, rng, [new + 30, 64], [new, 2], Hq, 1, 128)
            at = new + 30 - max(2, new // 2)
            b.caches[which][int(b.tables[0, at // BLOCK]), at % BLOCK, 0, 3 if which else slice(None)] = value
            a, more = b.args(rk)
            out, lse = rk.prefix_attention(*a, want_lse=True)
            o, l, mean, most = b.want()
            seen = new - max(2, new // 2)                            # new tokens before the one at `at`
            rows = np.r_[0:seen, new:new + 2]
            sub = (o[rows], l[rows], mean[rows], most[rows])
            assert np.isfinite(host(out)[rows]).all() and np.isfinite(host(lse)[rows]).all()
            assert np.abs(host(out)[rows] - sub[0]).max() < 0.05
            if which:                                                # values: the weights stay what they are
                assert np.array_equal(np.isnan(o[:new]), np.isnan(host(out)[:new]))
                assert np.array_equal(np.isinf(o[:new]), np.isinf(host(out)[:new]))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 80, 128, 192, 256])
@pytest.mark.parametrize("Hq,new", [(1, 12), (3, 9), (8, 40), (5, 70)])
def test_attend_not_finite_at_every_head_size(gpu, Hq, new, D, dtype):
    """Keys and values that are not finite, in several tokens, heads' places and signs, on narrow tiles of one and two row
    blocks and wide ones: every row within check()'s bounds, its infinities of the right sign, its log-sum-exp too."""
    torch, rk = gpu
    rng = rng_of("not finite", Hq, new, D)
    kv = [new + 100, 90]
    for which in (0, 1):
        b = Batch(torch, rng, kv, [new, 1], Hq, 1, D, dtype, garbage=float("nan"))
        for value in (float("inf"), float("-inf"), float("nan")):
            for at in rng.integers(100, 100 + new, 3):              # a new token's own
                piece = int(rng.integers(0, D // 8)), int(rng.integers(0, 8))
                slot = int(b.tables[0, at // BLOCK]), int(at % BLOCK)
                if which:
                    b.caches[1][slot[0], slot[1], 0, 8 * piece[0] + piece[1]] = value
                elif at >= 100 + new // 2:                          # so that there are rows without
                    b.caches[0][slot[0], slot[1], 0, 8 * piece[0] + piece[1]] = value
        a, _ = b.args(rk)
        out, lse = rk.prefix_attention(*a, want_lse=True)
        b.check(out, lse)
    assert rk.device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [8, 64, 72, 80, 96, 128, 136, 192, 200, 248])
@pytest.mark.parametrize("kv,new,Hq", [(60, 1, 2), (3000, 1, 5), (700, 40, 2), (700, 300, 8)])
def test_attend_infinite_keys(gpu, kv, new, Hq, D, dtype):
    """A key with an infinity among its last 8 values, at every head size: where the query's value is of the other sign the
    score is -infinity, and the key has no weight; where it is of the same one, the row is no number."""
    torch, rk = gpu
    b = Batch(torch, rng_of("infinite", kv, D), [kv, 40], [new, 1], Hq, 1, D, dtype)
    last = D - 1 - 3 * (D > 8)
    b.q[..., last] = b.q[..., last].abs() + 0.5
    b.q[-1, 0, last] *= -1
    for at in (3, 30):                          # in front of every new token of the first request
        b.caches[0][int(b.tables[0, at // BLOCK]), at % BLOCK, 0, last] = float("-inf")
    b.caches[0][int(b.tables[1, 0]), 5, 0, last] = float("-inf")
    a, more = b.args(rk)
    out, lse = rk.prefix_attention(*a, want_lse=True)
    o, l, mean, _ = b.want()
    b.caches[0][b.caches[0].isinf()] = 0        # (the roundings of the other scores)
    b.check(out, lse, want=(o, l, mean, b.want()[3]))
    got = host(out)
    assert np.isfinite(got[:new]).all() and np.isnan(got[-1, 0]).all() and np.isfinite(got[-1, 1:]).all()
    assert rk.device_status(reset=True) == 0


@pytest.mark.parametrize("kv,new,Hq", [(60, 1, 2), (9000, 1, 4), (700, 300, 8), (9000, 2, 64)])
def test_attend_scores_that_are_no_numbers(gpu, kv, new, Hq):
    """A query that is NaN gives NaN, also where its parts are joined; a key that is NaN, to the tokens that see it."""
    torch, rk = gpu
    b = Batch(torch, rng_of("nan", kv, new), [kv, 50], [new, 1], Hq, 1, 64)
    b.q[0, Hq - 1, 5] = float("nan")
    a, more = b.args(rk)
    out, lse = rk.prefix_attention(*a, want_lse=True)
    b.check(out, lse)
    assert np.isnan(host(out)[0, Hq - 1]).all() and np.isfinite(host(out)[1:]).all()
    b.caches[0][int(b.tables[0, 1]), 2, 0, 3] = float("nan")           # position 18
    out, lse = rk.prefix_attention(*a, want_lse=True)
    b.check(out, lse)
    assert np.isnan(host(out)[:new]).all() and np.isnan(host(lse)[:new]).all() and np.isfinite(host(out)[new:]).all()


def test_attend_large_scores(gpu):
    """Scores in the thousands: one key takes all, none overflows."""
    rng = rng_of("large")
    for dtype in ("bf16", "fp16"):
        b = Batch(gpu[0], rng, [300, 20, 1], [1, 20, 1], 4, 2, 64, dtype, spread=16.0)
        attend(gpu, b)
        attend(gpu, b, scale=1.0)
        attend(gpu, b, scale=0.0)
        attend(gpu, b, scale=-0.5)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("kv,new,Hq", [(70, 1, 2), (3000, 1, 4), (500, 300, 4), (8100, 2, 64)])
def test_attend_scores_in_the_millions(gpu, kv, new, Hq, dtype):
    """Scores up to the documented 2^23, thousands apart: each row is the value of its largest."""
    torch, rk = gpu
    rng = rng_of("millions", kv, new)
    b = Batch(torch, rng, [kv], [new], Hq, 1, 64, dtype)
    b.q.zero_()
    b.q[..., 0] = 2048.0
    k, v = b.caches
    score = np.concatenate([rng.permutation(kv - new), np.arange(kv - new, kv)])      # a new token's own is its largest
    at = np.arange(kv)
    block = torch.from_numpy(b.tables[0][at // BLOCK].astype(np.int64)).cuda()
    coarse, fine = score // 64, score % 64                      # scores are 2^16 * coarse + 2^10 * fine, exactly
    k[block, at % BLOCK] = 0.0
    b.q[..., 1] = 32.0
    k[block, at % BLOCK, 0, 0] = torch.from_numpy(coarse * 32.0).to(k.dtype).cuda()
    k[block, at % BLOCK, 0, 1] = torch.from_numpy(fine * 32.0).to(k.dtype).cuda()
    a, _ = b.args(rk)
    assert score.max() * 2 ** 10 < 2 ** 23
    out, lse = rk.prefix_attention(*a, scale=1.0, want_lse=True)
    want = host(v[block, at % BLOCK, 0])[kv - new:]
    assert np.abs(host(out) - want[:, None]).max() <= 2 * STEP[dtype] * np.abs(want).max()
    top = score[kv - new:] * 2.0 ** 10
    assert np.abs(host(lse) - top[:, None]).max() <= 4 * 2.0 ** -24 * top.max()
    assert rk.device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("others", ["equal", "spread"])
@pytest.mark.parametrize("kv,new,Hq,Hkv,D,shared", [
    ([3000], [1], 4, 1, 128, 0), ([2500, 40], [4, 1], 8, 1, 80, 0), ([300] * 40, [1] * 40, 8, 8, 64, 0),
    ([700, 900], [300, 900], 8, 2, 64, 0), ([1000], [400], 4, 1, 192, 0), ([1700] * 30, [1] * 30, 8, 2, 128, 100),
    ([100000], [1], 2, 1, 64, 0)])
def test_attend_one_key_far_above(gpu, kv, new, Hq, Hkv, D, shared, others, dtype):
    """A key of value 0 (at the front, in the middle, or the token's own) that stands far above the others: what is left of
    these is the result, to the same relative roundings, down to what the type holds at all."""
    torch, rk = gpu
    rng = rng_of("far above", kv, new, others)
    B = len(kv)
    goff, sh = (np.array([0] + [B] * B), np.array([shared] + [0] * (B - 1), np.int32)) if shared else (None, None)
    b = Batch(torch, rng, kv, new, Hq, Hkv, D, dtype, goff=goff, shared=sh)
    b.q.zero_()
    b.q[..., 0] = 1.0                                       # a key's first value is its score
    k, v = b.caches
    k[..., 0] = torch.from_numpy(rng.normal(size=tuple(k.shape[:3]))).to(k.dtype).cuda() if others == "spread" else 0.0
    v[:] = v * 0.3 + 1.0
    was = k.clone(), v.clone()
    a, more = b.args(rk)
    for gap in (8, 10.5, 12, 14, 15, 16, 17.5, 18, 20, 25, 33, 60):
        for place in ("front", "middle", "own"):
            for i in range(B):
                at = {"front": 0, "middle": kv[i] // 2, "own": kv[i] - 1}[place]
                slot = int(b.tables[i, at // BLOCK]), at % BLOCK
                k[slot[0], slot[1], :, 0] = gap
                v[slot[0], slot[1]] = 0.0
            out, lse = rk.prefix_attention(*a, **more, scale=1.0, want_lse=True)
            if gap in (8, 16, 18, 25) or kv[0] < 100000 and B == 1:       # (the oracle takes its time)
                b.check(out, lse, scale=1.0)
            k.copy_(was[0])
            v.copy_(was[1])
    assert rk.device_status(reset=True) == 0


def test_attend_rows_behind_and_empty_requests(gpu):
    torch, rk = gpu
    b = Batch(torch, rng_of("behind"), [0, 9, 40, 0], [0, 2, 0, 0], 4, 2, 64, rows_behind=50)
    a, more = b.args(rk)
    out = torch.full((52, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((52, 4), 7.0, device="cuda")
    rk.prefix_attention(*a, out=out, lse=lse)
    b.check(out, lse)
    assert (out[2:] == 7).all() and (lse[2:] == 7).all()
    strided = torch.full((52, 4, 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    rk.prefix_attention(*a, out=strided[:, :, 1], lse=lse)
    assert torch.equal(strided[:, :, 1], out) and (strided[:, :, 0] == 7).all() and (strided[:, :, 2] == 7).all()
    rk.prefix_attention(b.q[:0], *a[1:3], *[x[:0] for x in a[3:5]], a[5][:1])
    assert rk.device_status(reset=True) == 0


def test_attend_bad_blocks(gpu):
    """Blocks outside the cache are left out; a token that sees nothing else gets 0 and -infinity."""
    torch, rk = gpu
    rng = rng_of("bad blocks")
    for Hq in (2, 16, 64):
        b = Batch(torch, rng, [100, 30, 200, 90], [1, 2, 60, 90], Hq, 2, 128)
        b.tables[0, 2], b.tables[1, :2] = -1, [1 << 30, -7]
        b.tables[2, 3], b.tables[3, 0] = b.caches[0].shape[0], -2 ** 31
        attend(gpu, b)
        assert rk.device_status(reset=True) == 0x80


def test_attend_bad_lengths(gpu):
    """Requests that do not fit are skipped, their rows left alone, the others done."""
    torch, rk = gpu
    b = Batch(torch, rng_of("bad"), [100, 30, 50, 20], [1, 2, 3, 20], 8, 2, 64)
    a, more = b.args(rk)
    good = rk.prefix_attention(*a)[0]
    for kv, bits in (([100, 1, 50, 20], 0x1), ([100, 16 * b.tables.shape[1] + 1, 50, 20], 0x10), ([100, -1, 50, 20], 0x1)):
        out = torch.full_like(good, 7.0)
        rk.prefix_attention(*a[:4], rk.to_device(np.array(kv, np.int32)), a[5], out=out)
        assert torch.equal(out[:1], good[:1]) and torch.equal(out[3:], good[3:]) and (out[1:3] == 7).all()
        assert rk.device_status(reset=True) == bits
    for q_off in ([0, 1, 0, 6, 26], [0, 1, 3, 6, 27], [-1, 1, 3, 6, 26]):
        out = torch.full_like(good, 7.0)
        rk.prefix_attention(*a[:5], rk.to_device(np.array(q_off)), out=out)
        assert rk.device_status(reset=True) == 0x1
    for goff in ([0, 3, 2, 4, 4], [0, 5, 5, 5, 5], [1, 4, 4, 4, 4], [0, 3, 3, 3, 3]):
        out = rk.prefix_attention(*a, group_off=rk.to_device(np.array(goff)), shared=rk.to_device(np.full(4, 1, np.int32)))[0]
        assert torch.equal(out, good) and rk.device_status(reset=True) == 0x1


@pytest.mark.parametrize("B,G", [(12, 1), (600, 4)])
def test_attend_offsets_that_go_back(gpu, B, G):
    """Offsets with steps back between good ones, so that groups claim the same two tokens again and again, more of them
    than there are: each request attends for itself, in the workspace of two tokens and not behind it."""
    torch, rk = gpu
    one = Batch(torch, rng_of("back", B), [1640, 1640, 1640], [1, 1, 0], G, 1, 64)
    one.tables[1] = one.tables[0]
    one.q[1] = one.q[0]
    a, _ = one.args(rk)
    want = rk.prefix_attention(*a)[0]
    n = B // 3
    q_off = np.concatenate([np.tile([0, 1, 2], n), [0]])
    goff = np.concatenate([(3 * np.arange(n)[:, None] + [0, 2]).reshape(-1), np.full(B + 1 - 2 * n, B)])
    up = rk.to_device
    need = rk.prefix_attention_workspace_size(2, B, G, 1, 64)
    ws = torch.full((need + 2 ** 22,), 77, dtype=torch.uint8, device="cuda")
    got = rk.prefix_attention(one.q, *one.caches, up(np.tile(one.tables[0], (B, 1))), up(np.full(B, 1640, np.int32)), up(q_off),
                              group_off=up(goff), shared=up(np.full(B, 100, np.int32)), workspace=ws)[0]
    assert rk.device_status(reset=True) == 0x1
    assert torch.allclose(got.float(), want.float(), rtol=4 * STEP["bf16"], atol=4 * STEP["bf16"])
    assert (ws[need:] == 77).all()


def test_attend_past_32_bits(gpu):
    """Blocks whose elements lie past 2^32 in the cache."""
    torch, rk = gpu
    rng = rng_of("far")
    b = Batch(torch, rng, [40, 300, 700], [1, 300, 1], 8, 1, 128, extra_blocks=3)
    far, n = 2_200_000, b.caches[0].shape[0]             # 2.2 M blocks of 2,048 elements: 9 GB a cache
    stretched = []
    for c in b.caches:
        big = torch.empty((far, BLOCK, 1, 128), dtype=torch.bfloat16, device="cuda")
        big[far - n:] = c
        stretched.append(big)
    a, more = b.args(rk)
    near = rk.prefix_attention(*a, want_lse=True)
    got = rk.prefix_attention(a[0], *stretched, torch.where(a[3] >= 0, a[3] + far - n, a[3]), *a[4:], want_lse=True)
    assert torch.equal(near[0], got[0]) and torch.equal(near[1], got[1])
    slots = torch.tensor([BLOCK * (far - 1) + 3, 5], device="cuda")
    x = torch.ones((2, 1, 128), dtype=torch.bfloat16, device="cuda")
    rk.kv_write(x, x, *stretched, slots)
    for c in stretched:
        assert float(c[far - 1, 3].sum()) == 128 and float(c[0, 5].sum()) == 128
    assert rk.device_status(reset=True) == 0


def test_attend_same_bits_each_time(gpu):
    torch, rk = gpu
    rng = rng_of("bits")
    goff, sh = np.array([0, 30, 30] + [40] * 38), np.array([60, 0, 9] + [0] * 37, np.int32)
    kv = BLOCK * np.repeat([60, 9], [30, 10]) + rng.integers(1, 300, 40)
    b = Batch(torch, rng, kv, np.minimum(rng.integers(1, 4, 40), 1 + 0 * kv), 16, 2, 128, goff=goff, shared=sh)
    a, more = b.args(rk)
    first = rk.prefix_attention(*a, **more, want_lse=True)
    for fill in (0, 255, 127):
        n = rk.prefix_attention_workspace_size(b.q.shape[0], 40, 16, 2, 128)
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")        # a workspace of any content
        again = rk.prefix_attention(*a, **more, want_lse=True, workspace=ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("B,new,Hq,Hkv,D", [(3, 500, 8, 2, 128), (600, 1, 4, 1, 64), (700, 5, 2, 1, 80)])
def test_attend_without_groups_in_a_small_workspace(gpu, B, new, Hq, Hkv, D):
    """A call without groups keeps to the workspace that T = 0 gives."""
    torch, rk = gpu
    rng = rng_of("small", B)
    kv = new + rng.integers(0, 900, B)
    b = Batch(torch, rng, kv, [new] * B, Hq, Hkv, D)
    a, _ = b.args(rk)
    n = rk.prefix_attention_workspace_size(0, B, Hq, Hkv, D)
    assert n < rk.prefix_attention_workspace_size(B * new, B, Hq, Hkv, D)
    ws = torch.full((n + 2 ** 22,), 77, dtype=torch.uint8, device="cuda")
    out, lse = rk.prefix_attention(*a, want_lse=True, workspace=ws[:n])
    b.check(out, lse)
    assert (ws[n:] == 77).all()
    with pytest.raises(rk.RkError, match="workspace"):
        rk.prefix_attention(*a, workspace=ws[:n - 1])
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    rk.prefix_attention(*a, out=out)
    assert torch.cuda.max_memory_allocated() - before < n + 2 ** 21
    assert rk.device_status(reset=True) == 0


def test_attend_two_streams_at_once(gpu):
    torch, rk = gpu
    rng = rng_of("streams")
    batches = [Batch(torch, rng, rng.integers(500, 4000, 20), np.ones(20, np.int64), 16, 2, 128) for _ in range(2)]
    calls = [b.args(rk) for b in batches]
    want = [rk.prefix_attention(*a, **m)[0] for a, m in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for k in range(2):
            got[k].append(rk.prefix_attention(*calls[k][0], **calls[k][1], stream=streams[k])[0])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(want[k], g) for g in got[k])


def test_attend_captured_by_a_fresh_process(gpu):
    """The process's first calls of the library may be captured ones."""
    import subprocess
    import sys
    code = """
import numpy as np, torch
from paper_2606_17081_amd import rkroute as rk
B, D = 5, 64
t = torch.arange(40, dtype=torch.int32, device="cuda").view(B, 8)
k, v = (torch.randn(40, 16, 2, D, device="cuda", dtype=torch.float16) for _ in range(2))
q = torch.randn(B, 4, D, device="cuda", dtype=torch.float16)
kv = torch.tensor([3, 128, 17, 60, 99], dtype=torch.int32, device="cuda")
off = torch.arange(B + 1, device="cuda")
one, have = torch.ones_like(kv), torch.full_like(kv, 8)
chains = torch.arange(1, 11, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    groups = rk.prefix_groups(chains, 2 * off, 1)
    _, slots, q_off, _ = rk.block_tables(t, kv, one, have, t.view(-1), B)
    rk.kv_write(k[0, :B], v[0, :B], k, v, slots)
    out, _ = rk.prefix_attention(q, k, v, t, kv, q_off)
for _ in range(3):
    q.normal_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, rk.prefix_attention(q, k, v, t, kv, off)[0])
assert int(groups[3]) == 5 and rk.device_status() == 0
print("replayed")
"""
    import os
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and "replayed" in r.stdout, r.stderr[-2000:]


def test_binding_refuses_gradients_and_empty_heads(gpu):
    """What would go wrong without a word: results that a backward pass would take for constants; and heads of no values."""
    torch, rk = gpu
    b = Batch(torch, rng_of("grad"), [40], [3], 4, 2, 64)
    a, _ = b.args(rk)
    q, k = a[0].clone().requires_grad_(), a[1].clone().requires_grad_()
    slots = torch.arange(3, device="cuda")
    new = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: rk.prefix_attention(q, *a[1:]), lambda: rk.prefix_attention(a[0], k, *a[2:]),
                 lambda: rk.kv_write(new.clone().requires_grad_(), new, a[1].clone(), a[2].clone(), slots)):
        with pytest.raises(rk.RkError, match="gradient"):
            call()
    with torch.no_grad():
        assert torch.equal(rk.prefix_attention(q, *a[1:])[0], rk.prefix_attention(*a)[0])
    with pytest.raises(rk.RkError, match="multiple of 8"):
        rk.prefix_attention(a[0][..., :0], a[1][..., :0], a[2][..., :0], *a[3:])
    assert rk.device_status(reset=True) == 0


def test_binding_refuses_tangents_and_outputs_that_want_a_gradient(gpu):
    torch, rk = gpu
    import torch.autograd.forward_ad as fw
    b = Batch(torch, rng_of("tangent"), [40], [3], 4, 2, 64)
    a, _ = b.args(rk)
    slots = torch.arange(3, device="cuda")
    new = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    k, v = a[1].clone(), a[2].clone()
    want = rk.prefix_attention(*a)[0]
    with fw.dual_level():
        dual = lambda t: fw.make_dual(t, torch.ones_like(t))  # noqa: E731
        for call in (lambda: rk.prefix_attention(dual(a[0]), *a[1:]), lambda: rk.prefix_attention(a[0], dual(k), *a[2:]),
                     lambda: rk.prefix_attention(*a[:2], dual(v), *a[3:]), lambda: rk.kv_write(dual(new), new, k, v, slots),
                     lambda: rk.kv_write(new, dual(new), k, v, slots), lambda: rk.kv_write(new, new, dual(k), v, slots)):
            with pytest.raises(rk.RkError, match="forward-mode"):
                call()
            with torch.no_grad(), pytest.raises(rk.RkError, match="forward-mode"):
                call()
        assert torch.equal(rk.prefix_attention(*a)[0], want)
        assert torch.equal(rk.prefix_attention(fw.unpack_dual(dual(a[0])).primal, *a[1:])[0], want)
    out, lse = torch.zeros_like(want), torch.zeros(want.shape[:2], device="cuda")
    for kw in (dict(out=out.clone().requires_grad_()), dict(lse=lse.clone().requires_grad_())):
        with pytest.raises(rk.RkError, match="gradient"):
            rk.prefix_attention(*a, **kw)
        with torch.no_grad():
            assert torch.equal(rk.prefix_attention(*a, **kw)[0], want)


def test_binding_counts_its_writes(gpu):
    """A backward pass that saved what a call then wrote to says so, as for any write in place."""
    torch, rk = gpu
    b = Batch(torch, rng_of("counts"), [40, 20], [3, 1], 4, 2, 64)
    a, _ = b.args(rk)
    new = torch.ones((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    k, v = a[1].nan_to_num(), a[2].nan_to_num()
    x = torch.ones_like(k, requires_grad=True)
    y = (x * k).sum()
    rk.kv_write(new, new, k, v, torch.arange(4, device="cuda"))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    out, lse = torch.empty_like(b.q), torch.empty((4, 4), device="cuda")
    chains, off = torch.arange(1, 5, device="cuda"), torch.tensor([0, 2, 4], device="cuda")
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    i64 = lambda n: torch.zeros(n, dtype=torch.int64, device="cuda")  # noqa: E731
    groups, tables = (i32(2), i64(3), i32(2), i32(1)), (i32(2, 4), i64(4), i64(3), i32(1))
    written = [k, v, out, lse, *groups, *tables]
    was = [t._version for t in written]
    rk.kv_write(new, new, k, v, torch.arange(4, device="cuda"))
    rk.prefix_attention(b.q, k, v, *a[3:], out=out, lse=lse)
    rk.prefix_groups(chains, off, 1, *groups)
    rk.block_tables(tables[0], a[4], i32(2), i32(2), i32(8), 4, None, None, *tables[1:])
    assert [t._version for t in written] == [x + 1 for x in was]
    with torch.inference_mode():
        c = torch.zeros_like(k)
        rk.kv_write(new, new, c, c.clone(), torch.arange(4, device="cuda"))
        rk.prefix_attention(b.q, k, v, *a[3:], out=torch.empty_like(out))
    assert rk.device_status(reset=True) == 0


# ------------------------------------------------------------------ together

def test_whole_steps_together(gpu):
    """Prompts hashed, grouped, given blocks, written and attended to; then two more tokens each, a graph replayed for the
    second of them: as plain attention of each request over its own keys and values."""
    torch, rk = gpu
    rng = rng_of("whole")
    Hq, Hkv, D, B = 8, 2, 64, 23
    group = rng.integers(0, 4, B)
    prefixes = rng.integers(0, 32000, (4, 640)).astype(np.int32)
    prompts = [np.concatenate([prefixes[g], rng.integers(0, 32000, rng.integers(1, 90)).astype(np.int32)]) for g in group]
    n_tok = np.array([len(p) for p in prompts])
    chains = rk.hash_chains(rk.to_device(np.concatenate(prompts)), rk.to_device(offsets(n_tok)), rk.to_device(offsets(n_tok // 16)))
    order, goff, shared, n_groups = rk.prefix_groups(chains, rk.to_device(offsets(n_tok // 16)), 4)
    o = host(order)
    assert int(n_groups) == len(set(group.tolist())) and (host(shared)[:int(n_groups)] >= 40).all()
    n_tok = n_tok[o]
    first, lead = ow.leads(n_tok, host(goff), host(shared))

    class Sequence:                  # of a request: what it would hold without sharing, in the cache's type
        pass

    emb = torch.randn((32000, 2, Hkv, D), device="cuda", dtype=torch.bfloat16)

    stride, blocks = 52, 23 * 52
    tables = torch.zeros((B, stride), dtype=torch.int32, device="cuda")
    k_cache = torch.full((blocks, BLOCK, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    v_cache = torch.full_like(k_cache, float("nan"))
    free = torch.from_numpy(rng.permutation(blocks).astype(np.int32)).cuda()
    tokens = [prompts[i].tolist() for i in o]
    kv = rk.to_device(n_tok.astype(np.int32))
    new = rk.to_device((n_tok - BLOCK * lead).astype(np.int32))
    have = torch.zeros(B, dtype=torch.int32, device="cuda")
    T = int(new.sum())
    static = {}

    def step(q, ids, kv, new, have, free, T):
        _, slots, q_off, taken = rk.block_tables(tables, kv, new, have, free, T, goff, shared)
        x = emb[ids]
        rk.kv_write(x[:, 0], x[:, 1], k_cache, v_cache, slots)
        return rk.prefix_attention(q, k_cache, v_cache, tables, kv, q_off, goff, shared, want_lse=True), taken, q_off

    def check(out, lse, q, n_new):
        at = 0
        for i in range(B):
            x = host(emb[torch.tensor(tokens[i], device="cuda")])
            L, n = len(tokens[i]), n_new[i]
            pad = -L % BLOCK
            kc, vc = (np.concatenate([x[:, c], np.zeros((pad, Hkv, D))]).reshape(-1, BLOCK, Hkv, D) for c in (0, 1))
            want = ow.attention(host(q[at:at + n]), kc, vc, np.arange(len(kc))[None], [L], [0, n])
            assert np.abs(host(out[at:at + n]) - want[0]).max() < 2 * STEP["bf16"] * 6        # |v| < 6
            assert np.abs(host(lse[at:at + n]) - want[1]).max() < 1e-3
            at += n

    q = torch.randn((T, Hq, D), device="cuda", dtype=torch.bfloat16)
    n_new = (n_tok - BLOCK * lead).tolist()
    ids = torch.tensor([t for s, n in zip(tokens, n_new) for t in s[-n:]], device="cuda")
    (out, lse), taken, _ = step(q, ids, kv, new, have, free, T)
    check(out, lse, q, n_new)
    need = -(-n_tok // BLOCK)
    assert int(taken) == int((need - lead).sum())

    # one token each, as a graph over fixed arrays
    static = dict(q=torch.zeros((B, Hq, D), device="cuda", dtype=torch.bfloat16), ids=torch.zeros(B, dtype=torch.int64, device="cuda"),
                  kv=kv.clone(), new=torch.ones_like(kv), have=have.clone(), free=free.clone())

    def fill(used):
        for s in tokens:
            s.append(int(rng.integers(0, 32000)))
        L = np.array([len(s) for s in tokens])
        static["q"].copy_(torch.randn((B, Hq, D), device="cuda", dtype=torch.bfloat16))
        static["ids"].copy_(torch.tensor([s[-1] for s in tokens], device="cuda"))
        static["kv"].copy_(torch.from_numpy(L.astype(np.int32)))
        static["have"].copy_(torch.from_numpy((-(-(L - 1) // BLOCK)).astype(np.int32)))
        static["free"].copy_(torch.roll(free, -used))

    used = int(taken)
    fill(used)
    (out, lse), taken, _ = step(**static, T=B)
    check(out, lse, static["q"], [1] * B)
    used += int(taken)
    fill(used)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            (out, lse), taken, _ = step(**static, T=B)
    torch.cuda.synchronize()
    for replay in range(20):
        if replay:
            used += int(taken)
            fill(used)
        graph.replay()
        torch.cuda.synchronize()
        check(out, lse, static["q"], [1] * B)
        assert torch.equal(rk.prefix_attention(static["q"], k_cache, v_cache, tables, static["kv"],
                                               torch.arange(B + 1, device="cuda"), goff, shared)[0], out)
    assert rk.device_status(reset=True) == 0
