"""A cache in 4 bits: what the C ABI refuses on the host, before any launch, and what the binding refuses."""
import ctypes as C

import pytest

from paper_2606_17081_amd import rkroute as rk

P = C.c_void_p(4096)


@pytest.fixture(scope="module")
def L():
    if not rk.library_available():
        pytest.skip("librkroute.so not built")
    return rk.lib()


def _cache(**change):
    """Of 7 blocks of 2 heads of 80: rows of 48 bytes of codes and 3 of scales."""
    c = rk.Fp4Cache(4096, rk.CacheStrides(16 * 96, 96, 48), 4096, rk.CacheStrides(16 * 6, 6, 3))
    for k, x in change.items():
        setattr(c, k, x)
    return c


def _strides_refused(rc):
    """Strides that no entry point takes, as changes of _cache."""
    S = rk.CacheStrides
    return [c for c in (dict(cs=S(1544, 96, 48)), dict(cs=S(1536, 104, 48)), dict(cs=S(1536, 96, 56)), dict(cs=S(-16, 96, 48)),
                        dict(cs=S(1536, -96, 48)), dict(cs=S(1536, 96, -48)), dict(ss=S(-1, 6, 3)), dict(ss=S(96, -6, 3)),
                        dict(ss=S(96, 6, -3))) if rc(c) != rk.RK_EINVAL or b"stride" not in rk.lib().rk_last_error()]


def _write(L, k=None, v=None, **at):
    a = [3, 2, 80, rk.RK_BF16, P, 160, 80, P, 160, 80, C.byref(k or _cache()), C.byref(v or _cache()), 7, P, None]
    for i, x in at.items():
        a[int(i[1:])] = x
    return L.rk_kv_write_fp4(*a)


def _read(L, k=None, v=None, **at):
    a = [3, 2, 80, rk.RK_F16, C.byref(k or _cache()), C.byref(v or _cache()), 7, P, P, 160, 80, P, 160, 80, None]
    for i, x in at.items():
        a[int(i[1:])] = x
    return L.rk_kv_read_fp4(*a)


def test_write_refusals(L):
    rc = lambda **at: _write(L, **at)  # noqa: E731
    assert rc(_0=-1) == rc(_12=-1) == rk.RK_EINVAL
    assert rc(_0=0) == rk.RK_OK
    assert rc(_1=0) == rc(_1=1025) == rc(_2=0) == rc(_2=60) == rc(_2=264) == rc(_3=2) == rc(_3=-1) == rk.RK_EUNSUPPORTED
    for i in (5, 6, 8, 9):
        assert rc(**{f"_{i}": 4}) == rc(**{f"_{i}": -8}) == rk.RK_EINVAL and b"stride" in L.rk_last_error()
    for i in (4, 7, 10, 11, 13):
        assert rc(**{f"_{i}": None}) == rk.RK_EINVAL
    for which in "kv":
        assert not _strides_refused(lambda c: rc(**{which: _cache(**c)}))
        for what in ("codes", "scales"):
            assert rc(**{which: _cache(**{what: None})}) == rk.RK_EINVAL and b"NULL" in L.rk_last_error()
        assert rc(**{which: _cache(codes=4104)}) == rk.RK_EINVAL and b"aligned" in L.rk_last_error()
    for i in (4, 7):
        assert rc(**{f"_{i}": C.c_void_p(4104)}) == rk.RK_EINVAL and b"aligned" in L.rk_last_error()


def test_read_refusals(L):
    rc = lambda **at: _read(L, **at)  # noqa: E731
    assert rc(_0=-1) == rc(_6=-1) == rk.RK_EINVAL
    assert rc(_0=0) == rk.RK_OK
    assert rc(_1=0) == rc(_1=1025) == rc(_2=0) == rc(_2=60) == rc(_2=264) == rc(_3=2) == rc(_3=-1) == rk.RK_EUNSUPPORTED
    for i in (9, 10, 12, 13):
        assert rc(**{f"_{i}": 4}) == rc(**{f"_{i}": -8}) == rk.RK_EINVAL and b"stride" in L.rk_last_error()
    for i in (4, 5, 7, 8, 11):
        assert rc(**{f"_{i}": None}) == rk.RK_EINVAL
    for which in "kv":
        assert not _strides_refused(lambda c: rc(**{which: _cache(**c)}))
        for what in ("codes", "scales"):
            assert rc(**{which: _cache(**{what: None})}) == rk.RK_EINVAL and b"NULL" in L.rk_last_error()
    for i in (8, 11):
        assert rc(**{f"_{i}": C.c_void_p(4104)}) == rk.RK_EINVAL and b"aligned" in L.rk_last_error()
    for token, head in ((80, 80), (0, 80), (160, 0), (152, 80), (160, 72)):
        assert rc(_9=token, _10=head) == rc(_12=token, _13=head) == rk.RK_EINVAL and b"over each other" in L.rk_last_error()


def test_write_refuses_caches_that_overlap_themselves(L):
    S = rk.CacheStrides
    for c in (dict(cs=S(1536, 96, 32)), dict(cs=S(1536, 80, 48)), dict(cs=S(1520, 96, 48)), dict(cs=S(0, 96, 48)),
              dict(cs=S(1536, 0, 48)), dict(cs=S(1536, 96, 0)), dict(ss=S(96, 6, 2)), dict(ss=S(96, 5, 3)), dict(ss=S(95, 6, 3)),
              dict(ss=S(0, 6, 3)), dict(ss=S(96, 0, 3)), dict(ss=S(96, 6, 0))):
        for which in "kv":
            assert _write(L, **{which: _cache(**c)}) == rk.RK_EINVAL and b"over each other" in L.rk_last_error()


def _attention(k=None, v=None, **change):
    x = P.value
    a = rk.Attention(4, 8, 2, 80, rk.RK_BF16, 7, 9, 0.125, 10, x, 8 * 80, 80, 0, rk.CacheStrides(3, -1, 5), 0, rk.CacheStrides(0, 0, 0),
                     x, x, x, x, x, x, 8 * 80, 80, x)
    for name, y in change.items():
        setattr(a, name, y)
    return rk.AttentionFp4(a, k or _cache(), v or _cache())


def test_attention_refusals(L):
    def rc(ws=P, size=1 << 40, **change):
        return L.rk_prefix_attention_fp4(C.byref(_attention(**change)), ws, size, None)

    assert L.rk_prefix_attention_fp4(None, P, 1 << 30, None) == rk.RK_EINVAL
    for k in ("B", "T", "n_blocks", "table_stride"):
        assert rc(**{k: -1}) == rk.RK_EINVAL
    assert rc(B=0) == rc(T=0) == rk.RK_OK                   # (the strides of 16-bit caches are not looked at)
    assert rc(Hq=7) == rc(Hq=0) == rc(Hkv=0) == rk.RK_EINVAL
    assert rc(B=rk.RK_MAX_BATCH + 1) == rc(Hq=2 * 129) == rc(D=12) == rc(D=264) == rc(D=0) == rk.RK_EUNSUPPORTED
    assert rc(T=1 << 40) == rc(dtype=2) == rc(dtype=-1) == rc(table_stride=(1 << 26) + 1) == rk.RK_EUNSUPPORTED
    assert rc(scale=float("nan")) == rc(scale=float("inf")) == rc(scale=-2e18) == rk.RK_EINVAL
    for k in ("q_token", "q_head", "out_token", "out_head"):
        assert rc(**{k: 4}) == rc(**{k: -8}) == rk.RK_EINVAL
    assert rc(out_token=560) == rk.RK_EINVAL and b"over each other" in L.rk_last_error()
    S = rk.CacheStrides
    for which in "kv":
        assert not _strides_refused(lambda c: rc(**{which: _cache(**c)}))
        for c in (dict(cs=S(1536, 32, 48)), dict(cs=S(1536, 1 << 26, 48)), dict(ss=S(96, 2, 3)), dict(ss=S(96, 1 << 26, 3))):
            assert rc(**{which: _cache(**c)}) == rk.RK_EINVAL and b"token stride" in L.rk_last_error()
        for c in (dict(cs=S(1 << 32, 96, 48)), dict(ss=S(1 << 32, 6, 3))):
            assert rc(**{which: _cache(**c)}) == rk.RK_EUNSUPPORTED and b"block stride" in L.rk_last_error()
            assert rc(**{which: _cache(**c)}, n_blocks=1, q=None) == rk.RK_EINVAL       # of one block it does not matter
        for what in ("codes", "scales"):
            assert rc(**{which: _cache(**{what: None})}) == rk.RK_EINVAL and b"NULL" in L.rk_last_error()
        assert rc(**{which: _cache(codes=4104)}) == rk.RK_EINVAL and b"aligned" in L.rk_last_error()
    for k in ("q", "tables", "kv_len", "q_off", "group_off", "shared", "out"):
        assert rc(**{k: None}) == rk.RK_EINVAL
    for k in ("q", "out"):
        assert rc(**{k: 4104}) == rk.RK_EINVAL and b"aligned" in L.rk_last_error()


def test_attention_refuses_a_workspace_too_small(L):
    size = rk.prefix_attention_fp4_workspace_size
    need = size(10, 4, 8, 2, 80)
    assert need > 0
    a = _attention()
    assert L.rk_prefix_attention_fp4(C.byref(a), P, need - 1, None) == rk.RK_ENOMEM
    assert L.rk_prefix_attention_fp4(C.byref(a), None, need, None) == rk.RK_ENOMEM
    assert L.rk_prefix_attention_fp4(C.byref(a), C.c_void_p(4096 + 16), need, None) == rk.RK_EINVAL
    assert size(1, 4097, 8, 2, 64) == size(1, 1, 7, 2, 64) == size(1, 1, 8, 2, 60) == size(-1, 1, 8, 2, 64) == 0
    assert 0 < size(0, 1, 8, 2, 64) <= size(1, 1, 8, 2, 64) <= size(100, 50, 8, 2, 64) <= size(5000, 50, 8, 2, 64)


def test_binding_needs_a_gpu_tensor():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("a GPU is there")
    u8 = lambda *n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    c = u8(1, 16, 1, 16), u8(1, 16, 1, 16), u8(1, 16, 1, 1), u8(1, 16, 1, 1)
    x = torch.zeros(1, 1, 8, dtype=torch.bfloat16)
    for call in (lambda: rk.kv_write_fp4(x, x, *c, None), lambda: rk.kv_read_fp4(*c, None),
                 lambda: rk.prefix_attention_fp4(x, *c, None, None, None)):
        with pytest.raises(rk.RkError, match="no GPU"):
            call()
