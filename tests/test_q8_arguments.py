"""What the 8-bit operators refuse, as codes and before any device work: no GPU needed."""
import ctypes as C

import numpy as np
import pytest


@pytest.fixture(scope="module")
def L():
    import paper_2410_17375_amd as A
    return A.lib


P, NULL = 4096, None          # an address that nothing reads: every call here is refused


def _refused(rc, L):
    assert rc == -1, rc
    assert L.amusd_last_error()


def test_rows(L):
    good = dict(x=P, dtype=1, ldx=32, rows=4, n=30, q=P, ldq=32, scale=P)
    order = ("x", "dtype", "ldx", "rows", "n", "q", "ldq", "scale")
    for change in (dict(x=NULL), dict(q=NULL), dict(scale=NULL), dict(dtype=2), dict(dtype=-1), dict(ldx=29), dict(rows=-1), dict(n=0), dict(ldq=24),
                   dict(ldq=40), dict(ldq=16), dict(q=P + 8), dict(x=P + 1), dict(dtype=0, x=P + 2)):
        a = {**good, **change}
        _refused(L.amusd_q8_quantize(*[a[k] for k in order], None), L)
    assert L.amusd_q8_quantize(*[{**good, "rows": 0}[k] for k in order], None) == 0


def test_rmsnorm(L):
    good = dict(x=P, dtype=1, ldx=32, add=P, add_dtype=0, ldadd=30, gain=P, eps=1e-5, rows=4, n=30, sum=P + 8192, ldsum=30, q=P, ldq=32, scale=P)
    for change in (dict(x=NULL), dict(gain=NULL), dict(gain=P + 2), dict(dtype=3), dict(add_dtype=2), dict(ldadd=29), dict(add=P + 2), dict(eps=-1.0),
                   dict(eps=float("nan")), dict(ldsum=29), dict(sum=P + 1), dict(q=NULL), dict(ldq=30), dict(scale=NULL), dict(n=-3), dict(ldx=1),
                   dict(sum=P, ldsum=40), dict(sum=P, n=16385, ldx=16400, ldadd=16400, ldsum=16400, ldq=16400)):
        _refused(L.amusd_q8_rmsnorm(*{**good, **change}.values(), None), L)
    for change in (dict(rows=0), dict(rows=0, add=NULL, add_dtype=9), dict(rows=0, sum=NULL, ldsum=0)):
        assert L.amusd_q8_rmsnorm(*{**good, **change}.values(), None) == 0


def test_rmsnorm_sum_over_the_addend(L):
    """add is read a second time where rows are longer than the registers: its place cannot take the sum, whatever its type."""
    good = dict(x=P, dtype=0, ldx=32, add=P + 8192, add_dtype=0, ldadd=32, gain=P, eps=1e-5, rows=0, n=30, sum=NULL, ldsum=32, q=P, ldq=32, scale=P)
    assert L.amusd_q8_rmsnorm(*good.values(), None) == 0
    for change in (dict(), dict(add_dtype=1), dict(dtype=1, add_dtype=1), dict(n=20000, ldx=20000, ldadd=20000, ldsum=20000, ldq=20000)):
        a = {**good, **change}
        _refused(L.amusd_q8_rmsnorm(*{**a, "sum": a["add"]}.values(), None), L)
        assert L.amusd_q8_rmsnorm(*{**a, "sum": P if a["dtype"] == 0 else P + 4}.values(), None) == 0


def test_matrix_and_product(L):
    w = np.zeros((4, 64), np.float32).ctypes.data
    good = dict(w=w, dtype=0, scale=NULL, n=4, k=64, ld=64, gated=0, on_device=0, stream=NULL)
    h = C.c_void_p()
    for change in (dict(w=NULL), dict(dtype=3), dict(dtype=2), dict(scale=w), dict(n=0), dict(k=0), dict(ld=63), dict(gated=1, n=3), dict(k=131073, ld=131073)):
        _refused(L.amusd_q8_matrix_create(*{**good, **change}.values(), C.byref(h)), L)
        assert not h
    _refused(L.amusd_q8_matrix_create(*good.values(), None), L)
    assert L.amusd_q8_matrix_free(None) == 0
    assert L.amusd_q8_gemm_workspace_bytes(None, 1) == -1
    assert L.amusd_q8_gemm(None, P, 64, P, 1, P, 0, 4, None, 0, None) == -1


def test_sizes_past_64_bits(L):
    """Products of sizes, each of which is allowed, that do not fit the type of an allocation's size."""
    h = C.c_void_p()
    for layers, seqs, heads, capacity in ((1 << 30, 4096, 2, 1 << 24), (1 << 20, 4096, 1 << 13, 1 << 24), (2 ** 31 - 1, 4096, 65535, 1 << 24), (1 << 17, 4096, 4096, 1 << 23)):
        _refused(L.amusd_q8_cache_create(layers, seqs, heads, heads, 128, capacity, 1, None, C.byref(h)), L)
        assert not h
    for on_device in (0, 1):
        for n, ld in ((1 << 20, 1 << 44), (3, 1 << 62), (2, 2 ** 63 - 1)):
            _refused(L.amusd_q8_matrix_create(P, 0, None, n, 64, ld, 0, on_device, None, C.byref(h)), L)
            assert not h


def test_matrix_of_more_features_than_a_launch(L):
    h = C.c_void_p()
    _refused(L.amusd_q8_matrix_create(P, 0, None, 1 << 28, 1, 1, 0, 1, None, C.byref(h)), L)      # two tiles a workgroup of 512: 2^32 threads
    assert not h


def test_matrix_of_a_host_array(L):
    """The binding hands over no array that is shorter than what the call reads, nor one whose rows lie otherwise."""
    import paper_2410_17375_amd as A
    w, s = np.zeros((4, 64), np.float32), np.ones(4, np.float32)
    for bad in (dict(n=5), dict(k=65), dict(n=4, k=60, ld=66), dict(dtype=A.DTYPE_BF16), dict(w=w.astype(np.float64)), dict(w=w[:, :60], k=60, ld=60),
                dict(w=w[:, ::2], k=32, ld=64), dict(w=w.T, n=64, k=4, ld=64), dict(w=w.astype(np.int8), dtype=A.DTYPE_INT8, scale=s[:3]), dict(w=w[:3]),
                dict(w=w[0], n=2, k=33)):
        with pytest.raises(ValueError):
            A.Q8Matrix(**{**dict(w=w, dtype=A.DTYPE_FP32, n=4, k=64), **bad})
    # these get past the binding: refused for want of a device (here), or for what the call itself refuses
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        return
    for good in (dict(), dict(n=3), dict(w=w[:, :60], k=60, ld=64), dict(w=w[:, :60], k=60), dict(w=w.T, n=64, k=4), dict(w=w.reshape(-1), ld=64), dict(n=0), dict(dtype=7),
                 dict(w=w.astype(np.int8), dtype=A.DTYPE_INT8, scale=s)):
        with pytest.raises(A.AmusdError):
            A.Q8Matrix(**{**dict(w=w, dtype=A.DTYPE_FP32, n=4, k=64), **good})


def test_cache(L):
    good = dict(n_layers=1, n_seqs=1, n_q_heads=8, n_kv_heads=2, head_dim=64, capacity=64, block=1, stream=NULL)
    h = C.c_void_p()
    for change in (dict(n_layers=0), dict(n_seqs=0), dict(n_seqs=5000), dict(n_q_heads=6), dict(n_kv_heads=0), dict(n_q_heads=32), dict(head_dim=96), dict(capacity=0), dict(capacity=(1 << 24) + 1),
                   dict(block=0), dict(block=8), dict(block=128)):
        _refused(L.amusd_q8_cache_create(*{**good, **change}.values(), C.byref(h)), L)
        assert not h
    _refused(L.amusd_q8_cache_create(*good.values(), None), L)
    assert L.amusd_q8_cache_free(None) == 0
    one = (C.c_int32 * 1)(0)
    assert L.amusd_q8_cache_append(None, 0, 1, one, one, one, P, P, 128, None, None, None) == -1
    assert L.amusd_q8_cache_read(None, 0, 1, one, one, one, P, P, 0, 128, None) == -1
    assert L.amusd_q8_attention(None, 0, 1, one, one, one, P, 512, 0.125, None, None, P, 512, None) == -1


def test_models(L):
    import paper_2410_17375_amd as A
    good = dict(n_layers=1, d_model=64, n_q_heads=1, n_kv_heads=1, head_dim=64, d_ffn=64, vocab=64, max_ctx=64, max_k=8, dtype=A.DTYPE_INT8, rope_theta=1e4,
                rms_eps=1e-5, max_seqs=1)
    h = C.c_void_p()
    for change in (dict(d_ffn=131072 + 64), dict(d_model=131072 + 64), dict(max_ctx=(1 << 24) + 1), dict(dtype=3), dict(d_ffn=48)):
        cfg = A.Config(*{**good, **change}.values())
        _refused(L.amusd_model_create(C.byref(cfg), None, C.byref(h)), L)
        assert not h


def test_model_of_a_vocabulary_that_no_product_takes(L):
    import paper_2410_17375_amd as A
    cfg = A.Config(*dict(n_layers=1, d_model=64, n_q_heads=1, n_kv_heads=1, head_dim=64, d_ffn=64, vocab=1 << 28, max_ctx=64, max_k=8, dtype=A.DTYPE_INT8,
                         rope_theta=1e4, rms_eps=1e-5, max_seqs=1).values())
    h = C.c_void_p()
    _refused(L.amusd_model_create(C.byref(cfg), None, C.byref(h)), L)
    assert not h


def test_calls_need_a_device(L):
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("has one")
    h = C.c_void_p()
    assert L.amusd_q8_cache_create(1, 1, 8, 2, 64, 64, 1, None, C.byref(h)) == -6 and not h
    w = np.zeros((4, 64), np.float32)
    assert L.amusd_q8_matrix_create(w.ctypes.data, 0, None, 4, 64, 64, 0, 0, None, C.byref(h)) == -6 and not h
