"""A worker's cache in 4 bits on the GPU against the numpy oracle: writes and reads (equal), attention (within the roundings that
its definition allows: the values held are the type's own, so they are those of attention over a 16-bit cache that
holds the same), alone and together, captured and on other streams."""
import numpy as np
import pytest

from oracle import worker as ow
from test_gpu_worker import BLOCK, STEP, Batch, dtype_of, gpu, host, offsets, rng_of  # noqa: F401

pytestmark = pytest.mark.gpu


def equal(a, b):
    a, b = np.asarray(a), np.asarray(b)
    assert a.shape == b.shape
    bad = np.argwhere((a != b) & ~((a != a) & (b != b)))
    assert not len(bad), (len(bad), bad[:5].tolist(), [(a[tuple(i)], b[tuple(i)]) for i in bad[:5]])
    return True


def shares(D):
    return -(-D // 32)


def fill(torch, rng, blocks, Hkv, D, heads_first=False, scales=None):
    """Codes and scales of random bytes."""
    shape = (blocks, Hkv, BLOCK) if heads_first else (blocks, BLOCK, Hkv)
    made = [torch.from_numpy(rng.integers(0, 256, (*shape, 16 * shares(D))).astype(np.uint8)).cuda(),
            torch.from_numpy(rng.integers(*(scales or (0, 256)), (*shape, shares(D))).astype(np.uint8)).cuda()]
    return [c.transpose(1, 2) if heads_first else c for c in made]


def bits16(torch, rng, shape, dtype):
    """Every bit pattern but few that are not finite: exponents of all ones are made smaller in 49 of 50 groups."""
    x = rng.integers(0, 1 << 16, shape).astype(np.uint16)
    top = 0x7f80 if dtype == "bf16" else 0x7c00
    near = np.where(rng.random(shape[:-1]) < 0.5, 0, 1)[..., None]       # half of the rows have exponents near each other
    x = np.where(near & ((x & top) != 0), (x & ~np.uint16(top >> 1 & top)) | (top >> 1 & top), x).astype(np.uint16)
    odd = (x & top) == top
    keep = rng.random(shape[:-1])[..., None] < 0.02
    x = np.where(odd & ~keep, x ^ np.uint16(top ^ (top >> 1) & top), x)
    return torch.from_numpy(x.view(np.int16)).cuda().view(dtype_of(torch, dtype))


# ------------------------------------------------------------------ writes

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,Hkv,D,blocks,heads_first", [
    (0, 1, 8, 1, False), (1, 1, 8, 1, False), (1, 2, 128, 3, True), (17, 3, 72, 9, False), (100, 8, 64, 40, True),
    (33, 1, 256, 3, False), (1000, 5, 96, 70, True), (3000, 2, 128, 300, False), (40, 3, 200, 5, True), (50, 1, 40, 4, False)])
def test_write(gpu, T, Hkv, D, blocks, heads_first, dtype):
    torch, rk = gpu
    rng = rng_of("write4", T, Hkv, D)
    new = bits16(torch, rng, (T, Hkv + 2, 2, D), dtype)[:, 1:1 + Hkv]
    caches = [fill(torch, rng, blocks, Hkv, D, heads_first) for _ in range(2)]
    slots = rng.permutation(BLOCK * blocks)[:T]
    slots = np.where(rng.random(slots.size) < 0.2, -1, slots)
    slots = np.concatenate([slots, np.full(T - slots.size, -3)]).astype(np.int64)
    want = [[host(x).copy() for x in c] for c in caches]
    at = np.nonzero(slots >= 0)[0]
    for w, n in zip(want, (new[:, :, 0], new[:, :, 1])):
        codes, scales = ow.fp4_encode(host(n)[at], dtype)
        w[0][slots[at] // BLOCK, slots[at] % BLOCK] = codes
        w[1][slots[at] // BLOCK, slots[at] % BLOCK] = scales
    was = [x._version for c in caches for x in c]
    rk.kv_write_fp4(new[:, :, 0], new[:, :, 1], caches[0][0], caches[1][0], caches[0][1], caches[1][1],
                    torch.from_numpy(slots).cuda())
    assert [x._version for c in caches for x in c] == [x + 1 for x in was]
    for w, c in zip(want, caches):
        assert equal(w[0], host(c[0])) and equal(w[1], host(c[1]))
    assert rk.device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_write_every_value_beside_every_power(gpu, dtype):
    """All 2^16 bit patterns, in groups whose largest is a power of two, at each power that the type has; with its neighbours where the
    scale changes."""
    torch, rk = gpu
    top = 255 if dtype == "bf16" else 31
    patterns = np.arange(1 << 16).astype(np.uint16)
    rows = []
    man = 7 if dtype == "bf16" else 10
    for e in range(top):
        for m in ((0,) if e % 5 else (0, 3 << (man - 2), (3 << (man - 2)) + 1, (1 << man) - 1)):
            largest = np.uint16(e << man | m)
            part = patterns[(patterns & 0x7fff) <= largest]
            near = part[(part & 0x7fff) + (6 << man) >= largest]                # within 2^6 or so: all that does not become 0
            pick = near[rng_of(e, m).integers(0, near.size, (12, 32))] if near.size > 400 else np.resize(near, (12, 32))
            pick = pick.copy()
            pick[:, 5] = largest
            rows.append(pick)
    x = np.concatenate(rows).reshape(-1, 1, 32)
    new = torch.from_numpy(x.view(np.int16)).cuda().view(dtype_of(torch, dtype))
    blocks = -(-len(x) // BLOCK)
    c = fill(torch, rng_of("c"), blocks, 1, 32)
    v = fill(torch, rng_of("v"), blocks, 1, 32)
    slots = torch.arange(len(x), device="cuda")
    rk.kv_write_fp4(new, -new, c[0], v[0], c[1], v[1], slots)
    for got, y in ((c, new), (v, -new)):
        codes, scales = ow.fp4_encode(host(y), dtype)
        assert equal(host(got[1]).reshape(-1, 1, 1)[:len(x)], scales)
        assert equal(host(got[0]).reshape(-1, 1, 16)[:len(x)], codes)
    # what was written is read without a rounding
    k, w = rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots, dtype=new.dtype)
    want = ow.fp4_decode(*ow.fp4_encode(host(new), dtype), 32)
    assert equal(host(k), want) and equal(host(w), -want)
    assert rk.device_status(reset=True) == 0


def test_write_slot_behind_the_cache(gpu):
    torch, rk = gpu
    c = torch.zeros((3, BLOCK, 1, 16), dtype=torch.uint8, device="cuda")
    s = torch.zeros((3, BLOCK, 1, 1), dtype=torch.uint8, device="cuda")
    ones = torch.ones((4, 1, 32), dtype=torch.bfloat16, device="cuda")
    rk.kv_write_fp4(ones, ones, c[:2], c[:2].clone(), s[:2], s[:2].clone(), torch.tensor([31, 32, 1 << 40, -1], device="cuda"))
    assert int(c.sum()) == int(c[1, 15].sum()) == 16 * 0x66 and int(s.sum()) == int(s[1, 15, 0, 0]) == 125
    assert rk.device_status(reset=True) == 0x80


# ------------------------------------------------------------------ reads

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_read_every_code_beside_every_scale(gpu, dtype):
    torch, rk = gpu
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(256).view(256, 16, 1, 16)
    scales = torch.arange(256, dtype=torch.uint8, device="cuda").view(256, 1, 1, 1).repeat(1, 16, 1, 1)
    slots = torch.arange(4096, device="cuda")
    k, v = rk.kv_read_fp4(codes, codes, scales, scales, slots, dtype=dtype_of(torch, dtype))
    want = torch.from_numpy(ow.fp4_decode(host(codes), host(scales), 32)).reshape(4096, 1, 32).to(dtype_of(torch, dtype))
    for got in (k, v):
        assert equal(host(got), host(want))
    assert rk.device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,Hkv,D,blocks,heads_first", [
    (0, 1, 8, 1, False), (1, 1, 8, 1, False), (1, 2, 128, 3, True), (17, 3, 72, 9, False), (400, 8, 64, 4, True),
    (33, 1, 256, 3, False), (1000, 5, 96, 70, True), (3000, 2, 128, 300, False), (40, 3, 200, 5, True), (9, 1, 40, 4, False)])
def test_read(gpu, T, Hkv, D, blocks, heads_first, dtype):
    """Slots in any order, twice too, negative ones and some behind the cache; outputs of any strides, what lies between their
    rows as it was."""
    torch, rk = gpu
    rng = rng_of("read4", T, Hkv, D)
    caches = [fill(torch, rng, blocks, Hkv, D, heads_first, scales=(115, 135)) for _ in range(2)]
    slots = rng.integers(-3, BLOCK * blocks, T)
    bad = rng.random(T) < 0.05
    slots = np.where(bad, BLOCK * blocks + rng.integers(0, 1 << 40, T), slots).astype(np.int64)
    behind = slots >= BLOCK * blocks
    there = (slots >= 0) & ~behind
    at = np.where(there, slots, 0)
    want = []
    for codes, scales in caches:
        x = ow.fp4_decode(host(codes)[at // BLOCK, at % BLOCK], host(scales)[at // BLOCK, at % BLOCK], D)
        want.append(np.where(there[:, None, None], x, 0))
    ty = dtype_of(torch, dtype)
    args = caches[0][0], caches[1][0], caches[0][1], caches[1][1], torch.from_numpy(slots).cuda()
    got = rk.kv_read_fp4(*args, D=D, dtype=ty)
    both = torch.full((Hkv, T, 3, D), 7.0, dtype=ty, device="cuda").transpose(0, 1)
    again = rk.kv_read_fp4(*args, k=both[:, :, 0], v=both[:, :, 2])
    for g, a, w in zip(got, again, want):
        assert g.dtype == ty and g.shape == (T, Hkv, D) and equal(host(g), w) and torch.equal(g, a)
    assert (both[:, :, 1] == 7).all() and both._version == 2
    assert rk.device_status(reset=True) == (0x80 if behind.any() else 0)


def test_binding_of_reads_and_writes(gpu):
    """Defaults, what does not fit, gradients."""
    torch, rk = gpu
    rng = rng_of("binding")
    c, v = fill(torch, rng, 4, 2, 64, scales=(120, 130)), fill(torch, rng, 4, 2, 64, scales=(120, 130))
    slots = torch.arange(5, device="cuda")
    k, w = rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots)
    assert k.shape == w.shape == (5, 2, 64) and k.dtype == torch.bfloat16
    short = rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots, D=40)[0]
    assert torch.equal(short, k[..., :40])
    half = rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots, k=torch.empty_like(k, dtype=torch.float16))
    assert half[0].dtype == half[1].dtype == torch.float16 and torch.equal(half[1].float(), w.float())
    refused = [
        lambda: rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots, D=72), lambda: rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots.int()),
        lambda: rk.kv_read_fp4(c[0], v[0], c[1], v[1][:, :, :1], slots), lambda: rk.kv_read_fp4(c[0], v[0][:3], c[1], v[1], slots),
        lambda: rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots, dtype=torch.float32),
        lambda: rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots, k=k[:4]), lambda: rk.kv_read_fp4(c[0], v[0].cpu(), c[1], v[1], slots),
        lambda: rk.kv_write_fp4(k, w, c[0].view(torch.int8), v[0], c[1], v[1], slots),
        lambda: rk.kv_write_fp4(k, w.half(), c[0], v[0], c[1], v[1], slots), lambda: rk.kv_write_fp4(k, w, c[0], v[0], c[1], v[1], slots[:4]),
        lambda: rk.kv_write_fp4(k[..., :32], w[..., :32], c[0], v[0], c[1], v[1], slots),
        lambda: rk.kv_write_fp4(k, w, c[0][..., ::2], v[0], c[1], v[1], slots),
        lambda: rk.kv_write_fp4(k.requires_grad_(), w, c[0], v[0], c[1], v[1], slots)]
    for call in refused:
        with pytest.raises(rk.RkError):
            call()
    rk.kv_write_fp4(k.detach(), w, c[0], v[0], c[1], v[1], slots)
    assert torch.equal(rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots)[1], w)           # (what was held stays)
    assert rk.device_status(reset=True) == 0


# ------------------------------------------------------------------ attention

class Batch4(Batch):
    """A Batch whose caches are held in 4 bits: `caches` are the values held."""

    def __init__(self, torch, rng, *what, **how):
        super().__init__(torch, rng, *what, **how)
        self.heads_first = how.get("heads_first", False)
        self.hold()

    def hold(self):
        torch, self.held = self.torch, []
        for i, c in enumerate(self.caches):
            parts = ow.fp4_encode(host(c), self.dtype)
            put = []
            for x in parts:
                x = np.ascontiguousarray(x.transpose(0, 2, 1, 3)) if self.heads_first else x
                x = torch.from_numpy(x).cuda()
                put.append(x.transpose(1, 2) if self.heads_first else x)
            self.held.append(put)
            self.caches[i] = torch.from_numpy(ow.fp4_decode(*parts, self.D)).cuda().to(dtype_of(torch, self.dtype))

    def check(self, out, lse, scale=None, want=None):
        """As Batch.check, with two more terms.  A weight below 2^-126 of its row's largest is held as 0 in 32 bits, so n of them
        may take n 2^-126 max |v| from a result (values held are often 0 themselves, and then such weights are all that is left).
        And a query may be multiplied as a sum of 8-bit floating values, exact but for values below 2^-14 of the group's
        largest, which are off by at most 2^-22 of that: a score by 2^-22 max |q| sum |k|."""
        o, l, mean, most = self.want(scale=scale) if want is None else want
        u, e = STEP[self.dtype], 2.0 ** -24
        rows = int(self.q_off[-1])
        out, lse = host(out)[:rows], host(lse)[:rows]
        o, l, mean, most = o[:rows], l[:rows], mean[:rows], most[:rows]
        n = float(self.kv.max(initial=0))
        k, v, q = (np.nan_to_num(host(x), posinf=0, neginf=0) for x in (*self.caches, self.q[:rows]))
        split = 2.0 ** -22 * abs(self.D ** -0.5 if scale is None else scale) * np.abs(q).max(-1, initial=0) * np.abs(k).sum(-1).max(initial=0)
        weight = (2 * (self.D + 2) * most + 2 * n + 64) * e + 2 * split
        bound = u * np.abs(o) + (1 + u) * (u + weight[..., None]) * mean + (2.0 ** -24 if self.dtype == "fp16" else 1e-38)
        bound += n * 2.0 ** -126 * np.abs(v).max(initial=0)
        fine = np.isfinite(o)
        equal(np.where(fine, 0, o), np.where(np.isfinite(out), 0, out))
        over = (np.abs(out - np.where(fine, o, 0)) > bound) & fine
        assert not over.any(), (len(over), np.argwhere(over)[:5], out[over][:5], o[over][:5], bound[over][:5])
        fine = np.isfinite(l)
        equal(np.where(fine, 0, l), np.where(np.isfinite(lse), 0, lse))
        over = (np.abs(lse - np.where(fine, l, 0)) > weight + 4 * e * np.abs(l)) & fine
        assert not over.any(), (np.argwhere(over)[:5], lse[over][:5], l[over][:5])

    def args(self, rk):
        a, more = super().args(rk)
        (kc, ks), (vc, vs) = self.held
        return [self.q, kc, vc, ks, vs, *a[3:]], more


def attend(gpu, b, scale=None, **kw):
    torch, rk = gpu
    a, more = b.args(rk)
    out, lse = rk.prefix_attention_fp4(*a, **more, scale=scale, want_lse=True, **kw)
    b.check(out, lse, scale)
    return out, lse


@pytest.mark.parametrize("kv", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 257, 500, 1025, 5000])
def test_attend_single_token(gpu, kv):
    attend(gpu, Batch4(gpu[0], rng_of("4", kv), [kv], [1], 16, 2, 128))
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("Hq,new,D", [(17, 1, 256), (31, 1, 200), (10, 2, 256), (11, 2, 248), (9, 3, 136), (25, 1, 128), (6, 3, 64)])
def test_attend_rows_that_are_not_there(gpu, Hq, new, D, dtype):
    """17 to 31 rows of a key head, the others of 32 not there, with blocks in the cache and outside it."""
    torch, rk = gpu
    for bad in (False, True):
        b = Batch4(torch, rng_of("not there", Hq, D), [700, 50, 2000], [new, new, new], Hq, 1, D, dtype)
        if bad:
            b.tables[0, 3], b.tables[2, 100] = -5, 1 << 30
        attend(gpu, b)
        assert rk.device_status(reset=True) == (0x80 if bad else 0)


@pytest.mark.parametrize("Hq,kv,new", [(4, [700, 50], [1, 2]), (1, [30] * 300, [1] * 300), (8, [300, 90], [300, 33])])
def test_attend_smallest_values(gpu, Hq, kv, new):
    """fp16 keys and values below 2^-14, which the type holds with fewer bits."""
    torch, rk = gpu
    b = Batch4(torch, rng_of("small", Hq, len(kv)), kv, new, Hq, 1, 128, "fp16", garbage=0.0)
    power = torch.tensor([2.0 ** -17, 2.0 ** -20], device="cuda").repeat(64)
    for c in b.caches:
        c.copy_((c.float() * power).half())
    b.hold()
    assert float(b.caches[0].abs().max()) < 2.0 ** -13 and float(b.caches[0].abs().max()) > 0
    attend(gpu, b, scale=2.0 ** 14)
    assert rk.device_status(reset=True) == 0


@pytest.mark.parametrize("singles,pieces,Hq,Hkv,D,dtype", [
    (40, [(6000, 128)], 2, 2, 128, "bf16"), (60, [(5000, 64), (300, 300)], 4, 2, 64, "fp16"), (30, [(4000, 128)], 8, 1, 72, "bf16"),
    (5, [(6000, 1)], 1, 1, 128, "fp16"), (0, [(7000, 4)], 4, 1, 64, "bf16"), (2, [(5000, 20)], 1, 1, 192, "bf16"), (9, [(3000, 40)], 3, 1, 256, "fp16")])
def test_attend_pieces_beside_single_tokens(gpu, singles, pieces, Hq, Hkv, D, dtype):
    """Tiles of many rows, cut over workgroups, in batches whose average request has few."""
    rng = rng_of("beside 4", singles, pieces, Hq)
    kv = np.concatenate([rng.integers(1, 1500, singles), [k for k, _ in pieces]])
    new = np.concatenate([np.ones(singles, np.int64), [n for _, n in pieces]])
    order = rng.permutation(len(kv))
    attend(gpu, Batch4(gpu[0], rng, kv[order], new[order], Hq, Hkv, D, dtype, rows_behind=2))
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("Hq,Hkv,D", [(1, 1, 8), (2, 1, 64), (8, 1, 128), (12, 1, 192), (16, 2, 256), (7, 1, 80), (5, 5, 96),
                                      (40, 8, 128), (128, 1, 64), (34, 1, 128), (10, 2, 136), (33, 11, 72), (17, 1, 248),
                                      (24, 8, 16), (6, 3, 32), (20, 5, 40), (4, 1, 224)])
def test_attend_head_layouts(gpu, Hq, Hkv, D, dtype):
    rng = rng_of("4", Hq, Hkv, D, dtype)
    kv = rng.integers(1, 400, 9)
    new = np.minimum(rng.integers(0, 40, 9), kv)
    new[:3] = np.minimum([1, 130, 0], kv[:3])
    attend(gpu, Batch4(gpu[0], rng, kv, new, Hq, Hkv, D, dtype, heads_first=bool(Hq % 2), rows_behind=3))
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (16, 2, 64), (12, 1, 192), (3, 3, 256)])
@pytest.mark.parametrize("kv,new", [([300], [300]), ([129, 700, 1], [129, 500, 1]), ([1000, 64, 63, 65], [1, 64, 63, 65]),
                                    ([2000], [33]), ([513, 514], [257, 129])])
def test_attend_many_new_tokens(gpu, kv, new, Hq, Hkv, D):
    """Prompts and pieces of prompts: each token sees up to itself."""
    for dtype in ("bf16", "fp16"):
        attend(gpu, Batch4(gpu[0], rng_of("4", kv, new, Hq), kv, new, Hq, Hkv, D, dtype, heads_first=Hq == 4))
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("sizes,shared,tail,new,Hq,Hkv,D", [
    ([2], [1], 20, 1, 8, 2, 128), ([40], [30], 50, 1, 8, 2, 128), ([1, 5, 1, 9], [3, 8, 100, 1], 200, 1, 8, 2, 128),
    ([3, 3], [64, 0], 33, 4, 8, 2, 128), ([70, 2], [9, 130], 40, 1, 8, 2, 128), ([6], [20], 300, 150, 8, 2, 128),
    ([200], [5], 3, 2, 8, 2, 128), ([3, 4], [7, 40], 0, 0, 8, 2, 128), ([3], [90], 700, 1, 12, 1, 192),
    ([40, 2, 50], [60, 200, 33], 40, 3, 7, 1, 80), ([64, 70], [70, 50], 1, 1, 16, 1, 256), ([20], [2000], 30, 1, 8, 1, 128),
    ([9, 200, 7], [25, 40, 31], 30, 1, 8, 8, 64)])
def test_attend_groups(gpu, sizes, shared, tail, new, Hq, Hkv, D, dtype):
    rng = rng_of("4", sizes, shared, tail)
    B = sum(sizes)
    goff = np.concatenate([offsets(sizes), np.full(B + 1 - len(sizes) - 1, B)]).astype(np.int64)
    sh = np.zeros(B, np.int32)
    sh[:len(sizes)] = shared
    own = rng.integers(0, tail + 1, B)
    kv = BLOCK * np.repeat(shared, sizes) + np.maximum(own, 1 if new else 0)
    n = np.minimum(rng.integers(1 if new else 0, new + 1, B) if new else np.zeros(B, np.int64), np.maximum(own, 1))
    attend(gpu, Batch4(gpu[0], rng, kv, n, Hq, Hkv, D, dtype, goff=goff, shared=sh, rows_behind=2, heads_first=Hq == 7))
    assert gpu[1].device_status(reset=True) == 0


def test_attend_many_requests(gpu):
    rng = rng_of("many4")
    attend(gpu, Batch4(gpu[0], rng, rng.integers(1, 60, 4096), np.ones(4096, np.int64), 2, 1, 64))
    sizes = [700, 900, 3, 497]
    B = sum(sizes)
    goff = np.concatenate([offsets(sizes), np.full(B - 4, B)]).astype(np.int64)
    shared = np.zeros(B, np.int32)
    shared[:4] = 40, 30, 200, 60
    kv = BLOCK * np.repeat(shared[:4], sizes) + rng.integers(1, 30, B)
    attend(gpu, Batch4(gpu[0], rng, kv, np.ones(B, np.int64), 2, 1, 64, goff=goff, shared=shared))
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("B,Hq,Hkv,D,dtype", [(512, 4, 1, 128, "bf16"), (513, 4, 1, 128, "bf16"), (513, 2, 2, 72, "fp16"),
                                              (1024, 2, 1, 192, "bf16"), (1025, 2, 1, 256, "fp16")])
def test_attend_many_requests_of_wide_heads(gpu, B, Hq, Hkv, D, dtype):
    rng = rng_of("wide heads 4", B, D)
    kv = rng.integers(1, 70, B)
    new = np.where(rng.random(B) < 0.1, kv, np.minimum(1, kv))
    new[rng.random(B) < 0.05] = 0
    kv[5] = new[5] = 300
    attend(gpu, Batch4(gpu[0], rng, kv, new, Hq, Hkv, D, dtype))
    assert gpu[1].device_status(reset=True) == 0


class Batch4As16(Batch4):
    """Held to what attention over a 16-bit cache of the same values is held to."""
    check = Batch.check


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kv,new,Hq,Hkv,D", [
    ([1], [1], 16, 2, 128), ([5000], [1], 16, 2, 128), ([300, 17, 2000], [1, 1, 4], 8, 1, 64), ([700, 64], [300, 64], 4, 1, 128),
    ([40] * 270, [1] * 270, 4, 1, 128), ([900, 33], [5, 33], 6, 2, 192), ([2000, 300], [70, 1], 3, 1, 256), ([129, 1025], [3, 200], 7, 1, 80),
    ([3000], [33], 2, 2, 40), ([20000, 9000], [1, 2], 4, 1, 64)])
def test_attend_as_close_as_16_bits(gpu, kv, new, Hq, Hkv, D, dtype):
    attend(gpu, Batch4As16(gpu[0], rng_of("as 16", kv[0], Hq, D), kv, new, Hq, Hkv, D, dtype, heads_first=Hq % 2 == 0))
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("sizes,shared,tail,new,Hq,Hkv,D", [([40], [30], 50, 1, 8, 2, 128), ([70, 2], [9, 130], 40, 1, 8, 2, 128),
                                                            ([6], [20], 300, 150, 8, 2, 128), ([20], [1000], 30, 1, 8, 1, 64)])
def test_attend_groups_as_close_as_16_bits(gpu, sizes, shared, tail, new, Hq, Hkv, D, dtype):
    rng = rng_of("groups as 16", sizes, shared, tail)
    B = sum(sizes)
    goff = np.concatenate([offsets(sizes), np.full(B + 1 - len(sizes) - 1, B)]).astype(np.int64)
    sh = np.zeros(B, np.int32)
    sh[:len(sizes)] = shared
    own = rng.integers(1, tail + 1, B)
    kv = BLOCK * np.repeat(shared, sizes) + own
    n = np.minimum(rng.integers(1, new + 1, B), own)
    attend(gpu, Batch4As16(gpu[0], rng, kv, n, Hq, Hkv, D, dtype, goff=goff, shared=sh))
    assert gpu[1].device_status(reset=True) == 0


def test_attend_long(gpu):
    """Long sequences, cut over many workgroups."""
    rng = rng_of("long4")
    attend(gpu, Batch4(gpu[0], rng, [40000, 33000], [1, 2], 4, 1, 64, "fp16"))
    attend(gpu, Batch4(gpu[0], rng, [20000], [70], 8, 1, 128))
    goff, sh = np.array([0, 3, 3, 3]), np.array([1500, 0, 0], np.int32)
    attend(gpu, Batch4(gpu[0], rng, [24100, 24001, 30000], [1, 1, 3], 8, 1, 128, goff=goff, shared=sh))
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("spread", [1e-3, 16.0, 300.0])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attend_spreads_of_values(gpu, spread, dtype):
    """Scores from nearly equal to thousands, queries and values from small to large."""
    rng = rng_of("spread4")
    b = Batch4(gpu[0], rng, [300, 20, 1, 900], [1, 20, 1, 60], 4, 2, 64, dtype, spread=spread)
    for scale in (None, 0.0, -0.5, 1.0):
        if spread < 300 or scale in (None, 0.0):
            attend(gpu, b, scale=scale)
    # queries whose values differ by many powers of two, the large ones beside small keys
    b = Batch4(gpu[0], rng, [400, 70], [1, 70], 4, 2, 128, dtype)
    power = gpu[0].from_numpy(rng.integers(-12, 3, (1, 1, 128)).astype(np.float32)).cuda().exp2()
    b.q = (b.q.float() * power).to(b.q.dtype)
    attend(gpu, b, scale=1.0)
    b.q[..., 5] = 0.0
    b.q[0] = 0.0
    attend(gpu, b)
    assert gpu[1].device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 80, 128, 192, 256])
@pytest.mark.parametrize("Hq,new", [(1, 12), (3, 9), (8, 40), (5, 70)])
def test_attend_not_finite(gpu, Hq, new, D, dtype):
    """Groups of keys and values that are no numbers, in new tokens of which some rows see them and some do not; behind the
    sequences and in blocks of nobody everything is such."""
    torch, rk = gpu
    rng = rng_of("not finite 4", Hq, new, D)
    for which in (0, 1):
        b = Batch4(torch, rng, [new + 100, 90], [new, 1], Hq, 1, D, dtype, garbage=float("nan"))
        for at in rng.integers(100, 100 + new, 3):
            if which == 0 and at < 100 + new // 2:                       # so that there are rows without
                continue
            share = int(rng.integers(0, shares(D)))
            slot = int(b.tables[0, at // BLOCK]), int(at % BLOCK)
            b.held[which][1][slot[0], slot[1], 0, share] = 255
            b.caches[which][slot[0], slot[1], 0, 32 * share:32 * share + 32] = float("nan")
        attend(gpu, b)
    assert rk.device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [8, 16, 40, 56, 72, 80, 120, 136, 152, 184, 200, 240, 248])
@pytest.mark.parametrize("kv,new,Hq,Hkv", [([40] * 300, [1] * 300, 1, 1), ([3000, 90], [1, 3], 4, 2), ([700, 40], [3, 2], 8, 1),
                                           ([500, 129], [300, 129], 4, 1)])
def test_attend_codes_behind_the_head(gpu, kv, new, Hq, Hkv, D, dtype):
    """Codes behind D beside a scale with which the largest of them are past the type's range, while what lies before D is not: they
    have no effect.  (Keys before D up to 3 * 2^14 or 3 * 2^126, with queries and a scale that make usual scores of them.)"""
    torch, rk = gpu
    b = Batch4(torch, rng_of("behind D", D, kv[0]), kv, new, Hq, Hkv, D, dtype)
    if dtype == "bf16":
        b.q = (b.q.float() * 2.0 ** -110).to(b.q.dtype)
    large = 141 if dtype == "fp16" else 253
    owned = ~torch.from_numpy((host(b.held[0][1]) == 255).any(-1)).cuda()
    C, left = shares(D), D % 32 // 2                                    # (the last share's bytes before D)
    for i, (codes, scales) in enumerate(b.held):
        last = codes[..., 16 * C - 16:]
        if i == 0:
            nibble = torch.randint(0, 6, (2, *last.shape), device="cuda") + 8 * torch.randint(0, 2, (2, *last.shape), device="cuda")
            last.copy_((nibble[0] | nibble[1] << 4).to(torch.uint8))
        else:
            last.zero_()
        last[..., left:] = torch.tensor([0x77, 0x7f, 0xf7, 0x6e], dtype=torch.uint8, device="cuda").repeat(4)[:16 - left]
        scales[..., C - 1][owned] = large
        b.caches[i] = torch.from_numpy(ow.fp4_decode(host(codes), host(scales), D)).cuda().to(b.q.dtype)
    slots = torch.arange(BLOCK * len(b.caches[0]), device="cuda")
    read = rk.kv_read_fp4(b.held[0][0], b.held[1][0], b.held[0][1], b.held[1][1], slots, D=D, dtype=b.q.dtype)
    for x, want in zip(read, b.caches):
        assert equal(host(x), host(want).reshape(x.shape)) and torch.isfinite(want[owned]).all()
    attend(gpu, b, scale=2.0 ** (-15 if dtype == "fp16" else -17))
    assert rk.device_status(reset=True) == 0


@pytest.mark.parametrize("kv,new,Hq", [(60, 1, 2), (9000, 1, 4), (700, 300, 8), (9000, 2, 64)])
def test_attend_queries_that_are_no_numbers(gpu, kv, new, Hq):
    """A query with a NaN gives NaN, also where its parts are joined; and one with an infinity where its scores are none."""
    torch, rk = gpu
    for value in (float("nan"), float("inf")):
        b = Batch4(torch, rng_of("nan4", kv, new), [kv, 50], [new, 1], Hq, 1, 64)
        b.q[0, Hq - 1, 5] = value
        a, more = b.args(rk)
        out, lse = rk.prefix_attention_fp4(*a, want_lse=True)
        assert np.isnan(host(out)[0, Hq - 1]).all()
        sane = np.ones(host(out).shape[:2], bool)
        sane[0, Hq - 1] = False
        assert np.isfinite(host(out)[sane]).all() and np.isfinite(host(lse)[sane]).all()
        if np.isnan(value):
            b.check(out, lse)
    assert rk.device_status(reset=True) == 0


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("kv,new,Hq,Hkv,D,shared", [
    ([3000], [1], 4, 1, 128, 0), ([2500, 40], [4, 1], 8, 1, 80, 0), ([700, 900], [300, 900], 8, 2, 64, 0),
    ([1700] * 30, [1] * 30, 8, 2, 128, 100)])
def test_attend_one_key_far_above(gpu, kv, new, Hq, Hkv, D, shared, dtype):
    """A key of value 0 far above the others takes no bits from what is left of them."""
    torch, rk = gpu
    rng = rng_of("far above 4", kv, new)
    B = len(kv)
    goff, sh = (np.array([0] + [B] * B), np.array([shared] + [0] * (B - 1), np.int32)) if shared else (None, None)
    b = Batch4(torch, rng, kv, new, Hq, Hkv, D, dtype, goff=goff, shared=sh)
    b.q.zero_()
    b.q[..., 0] = 1.0                                       # a key's first value is its score
    k, v = b.caches
    for gap in (8, 12, 16, 24, 48):
        for place in ("front", "middle", "own"):
            k[..., :32] = 0.0
            v[:] = 1.0 + (torch.arange(D, device="cuda") % 5).to(v.dtype)
            for i in range(B):
                at = {"front": 0, "middle": kv[i] // 2, "own": kv[i] - 1}[place]
                slot = int(b.tables[i, at // BLOCK]), at % BLOCK
                k[slot[0], slot[1], :, 0] = gap
                v[slot[0], slot[1]] = 0.0
            b.hold()
            k, v = b.caches
            attend(gpu, b, scale=1.0)
    assert rk.device_status(reset=True) == 0


def test_attend_cache_strides(gpu):
    """Keys, values and scales in one tensor, rows with space between them at odd places of scales."""
    torch, rk = gpu
    rng = rng_of("strides 4")
    for D in (64, 72, 128):
        b = Batch4(torch, rng, [70, 1, 300, 16], [3, 1, 300, 16], 8, 4, D)
        want = attend(gpu, b)
        blocks, C = b.held[0][0].shape[0], shares(D)
        row = 16 * C + 16
        both = torch.full((blocks, 4, BLOCK, 2, row), 255, dtype=torch.uint8, device="cuda")
        odd = torch.full((blocks * BLOCK * 4 * (2 * C + 1) + 1,), 255, dtype=torch.uint8, device="cuda")[1:]
        odd = odd.view(BLOCK, blocks, 4, 2 * C + 1).transpose(0, 1)
        codes = [both[:, :, :, x, :16 * C].transpose(1, 2) for x in (0, 1)]
        scales = [odd[..., x * C:(x + 1) * C] for x in (0, 1)]
        for x in (0, 1):
            codes[x].copy_(b.held[x][0])
            scales[x].copy_(b.held[x][1])
        a, _ = b.args(rk)
        got = rk.prefix_attention_fp4(a[0], *codes, *scales, *a[5:], want_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        slots = torch.arange(0, BLOCK * blocks, 3, device="cuda")
        near = rk.kv_read_fp4(b.held[0][0], b.held[1][0], b.held[0][1], b.held[1][1], slots, D=D)
        far = rk.kv_read_fp4(*codes, *scales, slots, D=D)
        assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(near, far))
        was = both.clone(), odd.clone()
        rk.kv_write_fp4(*near, *codes, *scales, slots)
        for x in (0, 1):
            was[0][:, :, :, x, :16 * C].transpose(1, 2).copy_(codes[x])
            was[1][..., x * C:(x + 1) * C].copy_(scales[x])
        assert torch.equal(was[0], both) and torch.equal(was[1], odd)
    assert rk.device_status(reset=True) == 0


def test_attend_rows_behind_and_empty_requests(gpu):
    torch, rk = gpu
    b = Batch4(torch, rng_of("behind4"), [0, 9, 40, 0], [0, 2, 0, 0], 4, 2, 64, rows_behind=50)
    a, more = b.args(rk)
    out = torch.full((52, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((52, 4), 7.0, device="cuda")
    rk.prefix_attention_fp4(*a, out=out, lse=lse)
    b.check(out, lse)
    assert (out[2:] == 7).all() and (lse[2:] == 7).all()
    strided = torch.full((52, 4, 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    rk.prefix_attention_fp4(*a, out=strided[:, :, 1], lse=lse)
    assert torch.equal(strided[:, :, 1], out) and (strided[:, :, 0] == 7).all() and (strided[:, :, 2] == 7).all()
    rk.prefix_attention_fp4(b.q[:0], *a[1:5], *[x[:0] for x in a[5:7]], a[7][:1])
    with pytest.raises(rk.RkError, match="gradient"):
        rk.prefix_attention_fp4(b.q.clone().requires_grad_(), *a[1:])
    with pytest.raises(rk.RkError, match="uint8"):
        rk.prefix_attention_fp4(*b.args(rk)[0][:1], *b.caches, *a[3:])
    assert rk.device_status(reset=True) == 0


def test_attend_bad_blocks_and_lengths(gpu):
    """Blocks outside the cache are left out; requests that do not fit are skipped, the others done."""
    torch, rk = gpu
    rng = rng_of("bad blocks 4")
    for Hq in (2, 16, 64):
        b = Batch4(torch, rng, [100, 30, 200, 90], [1, 2, 60, 90], Hq, 2, 128)
        b.tables[0, 2], b.tables[1, :2] = -1, [1 << 30, -7]
        b.tables[2, 3], b.tables[3, 0] = b.caches[0].shape[0], -2 ** 31
        attend(gpu, b)
        assert rk.device_status(reset=True) == 0x80
    b = Batch4(torch, rng, [100, 30, 50, 20], [1, 2, 3, 20], 8, 2, 64)
    a, more = b.args(rk)
    good = rk.prefix_attention_fp4(*a)[0]
    for kv, bits in (([100, 1, 50, 20], 0x1), ([100, 16 * b.tables.shape[1] + 1, 50, 20], 0x10)):
        out = torch.full_like(good, 7.0)
        rk.prefix_attention_fp4(*a[:6], rk.to_device(np.array(kv, np.int32)), a[7], out=out)
        assert torch.equal(out[:1], good[:1]) and torch.equal(out[3:], good[3:]) and (out[1:3] == 7).all()
        assert rk.device_status(reset=True) == bits


def test_past_32_bits(gpu):
    """Blocks whose codes, and whose scales, lie past 2^32 bytes in the cache."""
    torch, rk = gpu
    rng = rng_of("far4")
    b = Batch4(torch, rng, [40, 300, 700], [1, 300, 1], 8, 1, 128, extra_blocks=3)
    n = b.held[0][0].shape[0]
    far = 4_400_000 + n                                  # 4.4 M blocks of 1,024 bytes of codes: 4.5 GB a cache
    codes, scales = [], []
    for c, s in b.held:
        big = torch.empty((far, BLOCK, 1, 64), dtype=torch.uint8, device="cuda")
        big[far - n:] = c
        wide = torch.empty((far, 1024), dtype=torch.uint8, device="cuda")[:, 960:].view(far, BLOCK, 1, 4)
        wide[far - n:] = s
        codes.append(big)
        scales.append(wide)
    a, more = b.args(rk)
    near = rk.prefix_attention_fp4(*a, want_lse=True)
    tables = torch.where(a[5] >= 0, a[5] + far - n, a[5])
    got = rk.prefix_attention_fp4(a[0], *codes, *scales, tables, *a[6:], want_lse=True)
    assert torch.equal(near[0], got[0]) and torch.equal(near[1], got[1])
    slots = torch.tensor([BLOCK * (far - 1) + 3, 5], device="cuda")
    x = torch.full((2, 1, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    rk.kv_write_fp4(x, -x, *codes, *scales, slots)
    k, v = rk.kv_read_fp4(*codes, *scales, slots)
    assert torch.equal(k, x) and torch.equal(v, -x)
    for c, s in zip(codes, scales):
        assert int(scales[0][far - 1, 3].sum()) == 4 * 126 and int(s[0, 5].sum()) == 4 * 126
    assert rk.device_status(reset=True) == 0


def test_past_32_bits_of_each_cache(gpu):
    """What is written past 2^32 bytes of codes and of scales lies there, in the keys' cache and in the values', and is read from there."""
    torch, rk = gpu
    far = 4_400_000                                      # blocks of 1,024 bytes of codes
    codes = [torch.empty((far, BLOCK, 1, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty((far, 1024), dtype=torch.uint8, device="cuda")[:, 960:].view(far, BLOCK, 1, 4) for _ in range(2)]
    places = [(far - 1, 3), (0, 5), ((1 << 32) // 1024 - 1, 15), ((1 << 32) // 1024, 0)]
    low = [(int(b * 1024 + t * 64) % (1 << 32)) // 64 for b, t in places]                # (where an address of 32 bits would lead)
    assert len(set(low)) == len(low)
    for x in (*codes, *scales):
        x.fill_(9)
    slots = torch.tensor([BLOCK * b + t for b, t in places], device="cuda")
    x = torch.tensor([3.0, -1.5, 0.75, 12.0], dtype=torch.bfloat16, device="cuda").view(4, 1, 1).expand(4, 1, 128).contiguous()
    rk.kv_write_fp4(x, -x, *codes, *scales, slots)
    for c, s, sign in zip(codes, scales, (1, -1)):
        for (b, t), value in zip(places, (3.0, -1.5, 0.75, 12.0)):
            want = ow.fp4_encode(np.full((1, 128), sign * value), "bf16")
            assert equal(host(c[b, t]), want[0]) and equal(host(s[b, t]), want[1])
            c[b, t], s[b, t] = 9, 9
        assert all(bool((x[k:k + 100_000] == 9).all()) for x in (c, s) for k in range(0, far, 100_000))
    # and read: other bytes in each cache
    for k, (c, s) in enumerate(zip(codes, scales)):
        for n, (b, t) in enumerate(places):
            c[b, t], s[b, t] = 0x22 + 0x11 * n, 127 + k
    for k, got in enumerate(rk.kv_read_fp4(*codes, *scales, slots)):
        assert equal(host(got), np.array([1.0, 1.5, 2.0, 3.0]).reshape(4, 1, 1) * 2 ** k * np.ones((4, 1, 128)))
    assert rk.device_status(reset=True) == 0


def test_attend_same_bits_each_time(gpu):
    torch, rk = gpu
    rng = rng_of("bits4")
    goff, sh = np.array([0, 30, 30] + [40] * 38), np.array([60, 0, 9] + [0] * 37, np.int32)
    kv = BLOCK * np.repeat([60, 9], [30, 10]) + rng.integers(1, 300, 40)
    b = Batch4(torch, rng, kv, np.minimum(rng.integers(1, 4, 40), 1 + 0 * kv), 16, 2, 128, goff=goff, shared=sh)
    a, more = b.args(rk)
    first = rk.prefix_attention_fp4(*a, **more, want_lse=True)
    n = rk.prefix_attention_fp4_workspace_size(b.q.shape[0], 40, 16, 2, 128)
    for value in (0, 255, 127):
        ws = torch.full((n + 2 ** 20,), value, dtype=torch.uint8, device="cuda")        # a workspace of any content
        again = rk.prefix_attention_fp4(*a, **more, want_lse=True, workspace=ws[:n])
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1]) and (ws[n:] == value).all()
    with pytest.raises(rk.RkError, match="workspace"):
        rk.prefix_attention_fp4(*a, **more, workspace=ws[:n - 1])


def test_attend_two_streams_at_once(gpu):
    torch, rk = gpu
    rng = rng_of("streams4")
    batches = [Batch4(torch, rng, rng.integers(500, 4000, 20), np.ones(20, np.int64), 16, 2, 128) for _ in range(2)]
    calls = [b.args(rk) for b in batches]
    want = [rk.prefix_attention_fp4(*a, **m)[0] for a, m in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for k in range(2):
            got[k].append(rk.prefix_attention_fp4(*calls[k][0], **calls[k][1], stream=streams[k])[0])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(want[k], g) for g in got[k])


def test_same_as_attention_over_what_is_read_back(gpu):
    """Reading the cache into a 16-bit one and attending there gives the same to the type's roundings."""
    torch, rk = gpu
    rng = rng_of("as read")
    for dtype, D in (("bf16", 128), ("fp16", 80)):
        b = Batch4(torch, rng, [700, 33, 256], [1, 33, 5], 8, 2, D, dtype)
        a, _ = b.args(rk)
        blocks = b.held[0][0].shape[0]
        k, v = rk.kv_read_fp4(*a[1:5], torch.arange(BLOCK * blocks, device="cuda"), D=D, dtype=b.q.dtype)
        out4, lse4 = rk.prefix_attention_fp4(*a, want_lse=True)
        out, lse = rk.prefix_attention(b.q, k.view(blocks, BLOCK, 2, D), v.view(blocks, BLOCK, 2, D), *a[5:], want_lse=True)
        want = b.want()
        b.check(out4, lse4, want=want)
        b.check(out, lse, want=want)


def test_attend_a_cache_of_no_blocks(gpu):
    """Every block is outside it: results of 0, and no read."""
    torch, rk = gpu
    q = torch.randn((3, 8, 80), device="cuda", dtype=torch.float16)
    codes, scales = (torch.empty((0, BLOCK, 2, n), dtype=torch.uint8, device="cuda") for n in (48, 3))
    up = rk.to_device
    for new, kv in (([1, 2], [40, 700]), ([3, 0], [3, 9])):
        out, lse = rk.prefix_attention_fp4(q, codes, codes, scales, scales, torch.zeros((2, 50), dtype=torch.int32, device="cuda"),
                                           up(np.array(kv, np.int32)), up(offsets(new)), want_lse=True)
        assert (out == 0).all() and (lse == -np.inf).all() and rk.device_status(reset=True) == 0x80
    slots = torch.tensor([-1, 5], device="cuda")
    k, v = rk.kv_read_fp4(codes, codes, scales, scales, slots, D=80, dtype=torch.float16)
    assert (k == 0).all() and (v == 0).all() and rk.device_status(reset=True) == 0x80
    rk.kv_write_fp4(k, v, codes, codes, scales, scales, slots)
    assert rk.device_status(reset=True) == 0x80


@pytest.mark.parametrize("dtype,B,kv,new,Hq,Hkv,D,shared,bad", [
    ("bf16", 64, 20000, 1, 8, 8, 128, 0, 0), ("fp16", 2, 9000, 9000, 16, 2, 128, 0, 0), ("bf16", 3, 7000, 2500, 8, 1, 192, 0, 0),
    ("fp16", 40, 9000, 2, 40, 8, 64, 500, 0), ("bf16", 20, 70000, 3, 16, 8, 40, 0, 0), ("fp16", 64, 20000, 1, 8, 8, 128, 0, 1100),
    ("bf16", 2, 9000, 4000, 16, 2, 128, 0, 300), ("bf16", 20, 70000, 3, 16, 8, 64, 0, 4200)])
def test_attend_at_size(gpu, dtype, B, kv, new, Hq, Hkv, D, shared, bad):
    """Tiles of more steps than a wavefront's block numbers are read for at once, narrow and wide, with blocks outside the cache or
    without: as attention over a 16-bit cache that holds the same.  Each is off by at most half a step for the result and one for the
    weights, of the mean of |v| (from the same attention over |v|), and by the fp32 sums' errors, with |score| <= scale sum |q| |k|
    <= scale D max |q| max |k|."""
    torch, rk = gpu
    rng = rng_of("size", B, kv, new)
    ty, u = dtype_of(torch, dtype), STEP[dtype]
    per = -(-kv // BLOCK)
    own = per - shared
    blocks = shared + B * own
    caches = [fill(torch, rng, blocks, Hkv, D, heads_first=True, scales=(125, 128)) for _ in range(2)]
    first = np.arange(shared)[None, :].repeat(B, 0)
    tables = np.concatenate([first, shared + np.arange(B * own).reshape(B, own)], 1)
    tables = torch.from_numpy(rng.permutation(blocks)[tables].astype(np.int32)).cuda()
    lengths = np.full(B, kv) - (np.arange(B) % 13)          # fewer than its new tokens: that request is skipped
    q = torch.randn((B * new, Hq, D), device="cuda", dtype=ty)
    more = dict(group_off=torch.tensor([0] + [B] * B, device="cuda"),
                shared=torch.tensor([shared] + [0] * (B - 1), dtype=torch.int32, device="cuda")) if shared else {}
    if bad:                                                 # blocks outside the cache, from entry `bad` on
        outside = rng.random(tables.shape) < 0.03
        outside[:, :bad] = False
        tables = torch.where(torch.from_numpy(outside).cuda(), torch.tensor([-1, blocks] * tables.shape[1], dtype=torch.int32, device="cuda")
                             [:tables.shape[1]], tables)
    rest = [tables, rk.to_device(lengths.astype(np.int32)), rk.to_device(offsets([new] * B))]

    def results():
        return dict(out=torch.full_like(q, 9), lse=torch.full((B * new, Hq), 7.0, device="cuda"))

    out, lse = rk.prefix_attention_fp4(q, caches[0][0], caches[1][0], caches[0][1], caches[1][1], *rest, **more, **results())
    k, v = (x.view(blocks, BLOCK, Hkv, D) for x in rk.kv_read_fp4(
        caches[0][0], caches[1][0], caches[0][1], caches[1][1], torch.arange(BLOCK * blocks, device="cuda"), D=D, dtype=ty))
    want, want_lse = rk.prefix_attention(q, k, v, *rest, **more, **results())
    mean = rk.prefix_attention(q, k, v.abs(), *rest, **more, **results())[0].float() * (1 + 4 * u)
    most = D ** -0.5 * D * float(q.abs().max()) * float(k.abs().max())
    weight = (2 * (D + 2) * most + 2 * kv + 64) * 2.0 ** -24
    bound = 2 * (u * want.float().abs() * (1 + u) + (1 + u) * (u + weight) * mean)
    assert ((out.float() - want.float()).abs() <= bound).all()
    assert ((lse - want_lse).abs() <= 2 * (weight + 4 * 2.0 ** -24 * want_lse.abs())).all()
    skipped = torch.from_numpy(np.repeat(lengths < new, new)).cuda()
    assert (out[skipped] == 9).all() and (lse[skipped] == 7).all() and bool(skipped.any()) == (kv == new)
    assert rk.device_status(reset=True) == (0x01 if kv == new else 0x80 if bad else 0)


def test_read_of_many_tokens(gpu):
    """More tokens than workgroups, outputs past 2^32 bytes, on a stream of the caller's."""
    torch, rk = gpu
    rng = rng_of("many tokens")
    T, Hkv, D = (1 << 20) + 77, 128, 64
    c, v = (fill(torch, rng, 3, Hkv, D, scales=(120, 130)) for _ in range(2))
    slots = torch.randint(-1, 3 * BLOCK, (T,), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    k, w = rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for at in (slice(0, 500), slice(1 << 19, (1 << 19) + 500), slice(T - 500, T)):
        kk, ww = rk.kv_read_fp4(c[0], v[0], c[1], v[1], slots[at].contiguous())
        assert torch.equal(k[at], kk) and torch.equal(w[at], ww)
    where = (slots == 7).nonzero()[:, 0]
    assert torch.equal(k[where], k[where[:1]].expand(len(where), -1, -1))
    del w
    # and written to a cache of as many blocks, of which every other token's rows stay
    blocks = T // BLOCK + 1
    codes = torch.full((blocks, BLOCK, Hkv, 32), 17, dtype=torch.uint8, device="cuda")
    scales = torch.full((blocks, BLOCK, Hkv, 2), 99, dtype=torch.uint8, device="cuda")
    other = codes[:1].expand(1, -1, -1, -1).clone(), scales[:1].clone()
    to = torch.arange(T, device="cuda")
    to = torch.where(to % 2 == 0, to, -1)
    rk.kv_write_fp4(k, k, codes, codes.clone(), scales, scales.clone(), to)
    back = rk.kv_read_fp4(codes, codes, scales, scales, to)[0]
    assert torch.equal(back[::2], k[::2]) and not back[1::2].any()
    flat = codes.view(-1, Hkv, 32)
    assert (flat[1:T:2] == 17).all() and (flat[T:] == 17).all() and (scales.view(-1, Hkv, 2)[1:T:2] == 99).all()
    assert torch.equal(other[0][0, 1], codes[0, 1]) and rk.device_status(reset=True) == 0


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 72)])
def test_whole_steps_together(gpu, dtype, D):
    """Prompts hashed, grouped, given blocks, written and attended to over a cache in 4 bits; then a token each, eagerly and as a
    graph that is replayed with the program's own work between: against the oracle on each request's own tokens."""
    torch, rk = gpu
    rng = rng_of("whole4", D)
    ty = dtype_of(torch, dtype)
    Hq, Hkv, B = 8, 2, 11
    group = rng.integers(0, 3, B)
    prefixes = rng.integers(0, 3000, (3, 640)).astype(np.int32)
    prompts = [np.concatenate([prefixes[g], rng.integers(0, 3000, rng.integers(1, 90)).astype(np.int32)]) for g in group]
    n_tok = np.array([len(p) for p in prompts])
    chains = rk.hash_chains(rk.to_device(np.concatenate(prompts)), rk.to_device(offsets(n_tok)), rk.to_device(offsets(n_tok // 16)))
    order, goff, shared, _ = rk.prefix_groups(chains, rk.to_device(offsets(n_tok // 16)), 4)
    o = host(order)
    n_tok = n_tok[o]
    _, lead = ow.leads(n_tok, host(goff), host(shared))
    emb = torch.randn((3000, 2, Hkv, D), device="cuda", dtype=ty)
    held = ow.fp4_decode(*ow.fp4_encode(host(emb), dtype), D)
    stride, blocks = 52, B * 52
    tables = torch.zeros((B, stride), dtype=torch.int32, device="cuda")
    codes = [torch.full((blocks, Hkv, BLOCK, 16 * shares(D)), 255, dtype=torch.uint8, device="cuda").transpose(1, 2) for _ in range(2)]
    scales = [torch.full((blocks, Hkv, BLOCK, shares(D)), 255, dtype=torch.uint8, device="cuda").transpose(1, 2) for _ in range(2)]
    free = torch.from_numpy(rng.permutation(blocks).astype(np.int32)).cuda()
    tokens = [prompts[i].tolist() for i in o]

    def step(q, ids, kv, new, have, free, T):
        _, slots, q_off, taken = rk.block_tables(tables, kv, new, have, free, T, goff, shared)
        x = emb[ids]
        rk.kv_write_fp4(x[:, 0], x[:, 1], *codes, *scales, slots)
        back = rk.kv_read_fp4(*codes, *scales, slots, D=D, dtype=ty)
        return rk.prefix_attention_fp4(q, *codes, *scales, tables, kv, q_off, goff, shared, want_lse=True), taken, back, slots

    def check(out, lse, q, n_new, back, slots, ids):
        there = (host(slots) >= 0)[:, None, None]
        for x in (0, 1):
            assert equal(host(back[x]), np.where(there, held[host(ids)][:, x], 0))
        at = 0
        for i in range(B):
            x = held[tokens[i]]
            L, n = len(tokens[i]), n_new[i]
            pad = -L % BLOCK
            kc, vc = (np.concatenate([x[:, c], np.zeros((pad, Hkv, D))]).reshape(-1, BLOCK, Hkv, D) for c in (0, 1))
            want = ow.attention(host(q[at:at + n]), kc, vc, np.arange(len(kc))[None], [L], [0, n])
            assert np.abs(host(out[at:at + n]) - want[0]).max() < 2 * STEP[dtype] * 6        # |v| < 6
            assert np.abs(host(lse[at:at + n]) - want[1]).max() < 1e-3
            at += n

    n_new = (n_tok - BLOCK * lead).tolist()
    T = sum(n_new)
    q = torch.randn((T, Hq, D), device="cuda", dtype=ty)
    ids = torch.tensor([t for s, n in zip(tokens, n_new) for t in s[-n:]], device="cuda")
    kv, new = rk.to_device(n_tok.astype(np.int32)), rk.to_device(np.array(n_new, np.int32))
    (out, lse), taken, back, slots = step(q, ids, kv, new, torch.zeros(B, dtype=torch.int32, device="cuda"), free, T)
    check(out, lse, q, n_new, back, slots, ids)
    used = int(taken)
    static = dict(q=torch.zeros((B, Hq, D), device="cuda", dtype=ty), ids=torch.zeros(B, dtype=torch.int64, device="cuda"),
                  kv=kv.clone(), new=torch.ones_like(kv), have=torch.zeros_like(kv), free=free.clone())

    def one_more():
        for s in tokens:
            s.append(int(rng.integers(0, 3000)))
        L = np.array([len(s) for s in tokens])
        static["q"].copy_(torch.randn((B, Hq, D), device="cuda", dtype=ty))
        static["ids"].copy_(torch.tensor([s[-1] for s in tokens], device="cuda"))
        static["kv"].copy_(torch.from_numpy(L.astype(np.int32)))
        static["have"].copy_(torch.from_numpy((-(-(L - 1) // BLOCK)).astype(np.int32)))
        static["free"].copy_(torch.roll(free, -used))

    one_more()
    (out, lse), taken, back, slots = step(**static, T=B)
    check(out, lse, static["q"], [1] * B, back, slots, static["ids"])
    used += int(taken)
    one_more()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            (out, lse), taken, back, slots = step(**static, T=B)
    torch.cuda.synchronize()
    for replay in range(12):
        if replay:
            used += int(taken)
            one_more()
        graph.replay()
        torch.cuda.synchronize()
        check(out, lse, static["q"], [1] * B, back, slots, static["ids"])
        assert torch.equal(rk.prefix_attention_fp4(static["q"], *codes, *scales, tables, static["kv"],
                                                   torch.arange(B + 1, device="cuda"), goff, shared)[0], out)
    assert rk.device_status(reset=True) == 0
