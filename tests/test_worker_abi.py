"""A worker's step: what the C ABI refuses on the host, before any launch, and what the binding refuses."""
import ctypes as C

import pytest

from paper_2606_17081_amd import rkroute as rk

P = C.c_void_p(4096)


@pytest.fixture(scope="module")
def L():
    if not rk.library_available():
        pytest.skip("librkroute.so not built")
    return rk.lib()


def test_groups_refusals(L):
    f = L.rk_prefix_groups
    assert f(-1, P, P, 1, P, P, P, P, None) == rk.RK_EINVAL
    assert f(rk.RK_MAX_BATCH + 1, P, P, 1, P, P, P, P, None) == rk.RK_EUNSUPPORTED
    assert f(4, P, P, 0, P, P, P, P, None) == rk.RK_EINVAL and b"min_blocks" in L.rk_last_error()
    for k in (1, 2, 4, 5, 6, 7):
        a = [4, P, P, 1, P, P, P, P, None]
        a[k] = None
        assert f(*a) == rk.RK_EINVAL


def test_tables_refusals(L):
    f = L.rk_block_tables
    good = [4, P, P, P, P, P, P, 9, P, 8, P, 5, P, P, None]

    def rc(**at):
        a = list(good)
        for k, v in at.items():
            a[int(k[1:])] = v
        return f(*a)

    for k in ("_0", "_7", "_9", "_11"):
        assert rc(**{k: -1}) == rk.RK_EINVAL and b"negative" in L.rk_last_error()
    assert rc(_0=rk.RK_MAX_BATCH + 1) == rk.RK_EUNSUPPORTED
    assert rc(_9=1 << 20) == rk.RK_EUNSUPPORTED and b"stride" in L.rk_last_error()
    for k in (1, 2, 3, 4, 5, 6, 8, 10, 12, 13):
        assert rc(**{f"_{k}": None}) == rk.RK_EINVAL


def test_write_refusals(L):
    f = L.rk_kv_write
    s = rk.CacheStrides(16 * 64, 64, 64)
    good = [3, 1, 64, P, 64, 64, P, 64, 64, P, s, P, s, 7, P, None]

    def rc(**at):
        a = list(good)
        for k, v in at.items():
            a[int(k[1:])] = v
        return f(*a)

    assert rc(_0=-1) == rk.RK_EINVAL and rc(_13=-1) == rk.RK_EINVAL
    assert rc(_0=0) == rk.RK_OK
    assert rc(_1=0) == rc(_1=1025) == rk.RK_EUNSUPPORTED
    assert rc(_2=0) == rc(_2=60) == rc(_2=264) == rk.RK_EUNSUPPORTED
    for k in (4, 5, 7, 8):
        assert rc(**{f"_{k}": 4}) == rc(**{f"_{k}": -8}) == rk.RK_EINVAL and b"stride" in L.rk_last_error()
    for k in (10, 12):
        for bad in (rk.CacheStrides(1, 64, 64), rk.CacheStrides(1024, -64, 64), rk.CacheStrides(1024, 64, 3)):
            assert rc(**{f"_{k}": bad}) == rk.RK_EINVAL
    for k in (3, 6, 9, 11, 14):
        assert rc(**{f"_{k}": None}) == rk.RK_EINVAL
    for k in (3, 6, 9, 11):
        assert rc(**{f"_{k}": C.c_void_p(4104)}) == rk.RK_EINVAL and b"aligned" in L.rk_last_error()


def test_write_refuses_caches_that_overlap_themselves(L):
    def rc(s, t=None, n_blocks=7, Hkv=2, D=64):
        # a NULL slot map is refused, but not before the strides
        rc = L.rk_kv_write(3, Hkv, D, P, 128, 64, P, 128, 64, P, rk.CacheStrides(*s), P, rk.CacheStrides(*(t or s)), n_blocks, None, None)
        assert rc == rk.RK_EINVAL
        return b"over each other" in L.rk_last_error()

    good = [(2048, 128, 64), (2048, 64, 1024), (4096, 128, 64), (4096, 256, 128), (1024, 64, 7 * 1024), (64, 2 * 7 * 64, 7 * 64)]
    for s in good:
        assert not rc(s)
    for s in ((2048, 56, 64), (2048, 128, 56), (2048, 64, 64), (2040, 128, 64), (0, 128, 64), (2048, 0, 64), (2048, 128, 0),
              (1024, 64, 1024), (64, 64, 64), (2048, 64, 1016)):
        assert rc(s) and rc(good[0], s) and rc(s, good[0])
    # of one block or one head, that stride does not matter; of no block, none does
    assert not rc((0, 128, 64), n_blocks=1) and not rc((1024, 64, 0), Hkv=1) and not rc((0, 0, 0), n_blocks=0)
    assert rc((0, 56, 0), n_blocks=1, Hkv=1)
    assert not rc((1 << 62, 1 << 58, 64)) and rc((1 << 62, 1 << 59, 64))


def test_attention_refuses_an_output_that_overlaps_itself(L):
    def rc(token, head, **change):
        rc = L.rk_prefix_attention(C.byref(_attention(out_token=token, out_head=head, q=None, **change)), P, 1 << 40, None)
        assert rc == rk.RK_EINVAL                       # the NULL query, if nothing before it
        return b"over each other" in L.rk_last_error()

    assert not rc(512, 64) and not rc(64, 640) and not rc(1024, 128) and not rc(1 << 60, 64)
    for token, head in ((0, 64), (512, 0), (504, 64), (512, 56), (64, 64), (64, 632)):
        assert rc(token, head)
    assert not rc(0, 64, T=1) and not rc(64, 0, Hq=1, Hkv=1)


def _attention(**change):
    s = rk.CacheStrides(16 * 2 * 64, 2 * 64, 64)
    v = P.value
    a = rk.Attention(4, 8, 2, 64, rk.RK_BF16, 50, 9, 0.125, 10, v, 8 * 64, 64, v, s, v, s, v, v, v, v, v, v, 8 * 64, 64, v)
    for k, x in change.items():
        setattr(a, k, x)
    return a


def test_attention_refusals(L):
    def rc(ws=P, size=1 << 40, **change):
        return L.rk_prefix_attention(C.byref(_attention(**change)), ws, size, None)

    assert L.rk_prefix_attention(None, P, 1 << 30, None) == rk.RK_EINVAL
    for k in ("B", "T", "n_blocks", "table_stride"):
        assert rc(**{k: -1}) == rk.RK_EINVAL
    assert rc(B=0) == rc(T=0) == rk.RK_OK
    assert rc(Hq=7) == rc(Hq=0) == rc(Hkv=0) == rk.RK_EINVAL
    assert rc(B=rk.RK_MAX_BATCH + 1) == rc(Hq=2 * 129) == rc(D=12) == rc(D=264) == rc(D=0) == rk.RK_EUNSUPPORTED
    assert rc(T=1 << 40) == rc(dtype=2) == rc(dtype=-1) == rk.RK_EUNSUPPORTED
    assert rc(scale=float("nan")) == rc(scale=float("inf")) == rc(scale=-2e18) == rk.RK_EINVAL
    assert rc(table_stride=(1 << 26) + 1) == rk.RK_EUNSUPPORTED
    for k in ("q_token", "q_head", "out_token", "out_head"):
        assert rc(**{k: 4}) == rc(**{k: -8}) == rk.RK_EINVAL
    for k in ("ks", "vs"):
        for s in (rk.CacheStrides(7, 128, 64), rk.CacheStrides(2048, 56, 64), rk.CacheStrides(2048, 1 << 26, 64),
                  rk.CacheStrides(2048, 128, -64)):
            assert rc(**{k: s}) == rk.RK_EINVAL
    for k in ("q", "k_cache", "v_cache", "tables", "kv_len", "q_off", "group_off", "shared", "out"):
        assert rc(**{k: None}) == rk.RK_EINVAL
    for k in ("q", "k_cache", "v_cache", "out"):
        assert rc(**{k: 4104}) == rk.RK_EINVAL and b"aligned" in L.rk_last_error()


def test_attention_refuses_a_workspace_too_small(L):
    need = rk.prefix_attention_workspace_size(10, 4, 8, 2, 64)
    assert need > 0
    a = _attention()
    assert L.rk_prefix_attention(C.byref(a), P, need - 1, None) == rk.RK_ENOMEM
    assert L.rk_prefix_attention(C.byref(a), None, need, None) == rk.RK_ENOMEM
    assert L.rk_prefix_attention(C.byref(a), C.c_void_p(4096 + 16), need, None) == rk.RK_EINVAL


def test_a_call_without_groups_needs_no_room_for_shared_rows(L):
    size = rk.prefix_attention_workspace_size
    least, most = size(0, 1024, 64, 8, 128), size(16384, 1024, 64, 8, 128)
    assert 0 < least < 1 << 27 and most > 1 << 30
    a = _attention(T=16384, B=1024, Hq=64, Hkv=8, D=128, q_head=128, out_head=128, q_token=8192, out_token=8192,
                   ks=rk.CacheStrides(16 * 1024, 1024, 128), vs=rk.CacheStrides(16 * 1024, 1024, 128))
    odd = C.c_void_p(4096 + 16)                           # refused for its address, but for its size before that
    assert L.rk_prefix_attention(C.byref(a), odd, most - 1, None) == rk.RK_ENOMEM
    assert L.rk_prefix_attention(C.byref(a), odd, most, None) == rk.RK_EINVAL
    a.group_off = a.shared = None
    assert L.rk_prefix_attention(C.byref(a), odd, least - 1, None) == rk.RK_ENOMEM
    assert L.rk_prefix_attention(C.byref(a), odd, least, None) == rk.RK_EINVAL


def test_workspace_sizes(L):
    size = rk.prefix_attention_workspace_size
    assert size(1, 4097, 8, 2, 64) == size(1, 1, 7, 2, 64) == size(1, 1, 8, 2, 60) == size(-1, 1, 8, 2, 64) == 0
    assert 0 < size(1, 1, 8, 2, 64) <= size(100, 50, 8, 2, 64) <= size(5000, 50, 8, 2, 64)


def test_binding_needs_a_gpu_tensor():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("a GPU is there")
    with pytest.raises(rk.RkError, match="no GPU"):
        rk.kv_write(torch.zeros(1, 1, 8), torch.zeros(1, 1, 8), torch.zeros(1, 16, 1, 8), torch.zeros(1, 16, 1, 8), None)
