"""The 8-bit operators on the GPU against their plain form in float64 (oracle/q8.py).

Tolerances are counted in roundings: u32 = 2^-24 and u16 = 2^-8 are the largest relative errors of a rounding to fp32 and
to bf16, 2^-11 that of one to half."""
import numpy as np
import pytest

from oracle import q8 as O

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_17375_amd as A
    return torch, A


def _code(A, torch, t):
    return A.DTYPE_BF16 if t.dtype == torch.bfloat16 else A.DTYPE_FP32


def _np(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _strided(torch, a, dtype, ld, offset=0, fill=7.0):
    """The rows of a at a distance of ld elements, beginning `offset` elements into an allocation."""
    n = a.shape[0]
    buf = torch.full((offset + max(n, 1) * ld,), fill, dtype=dtype, device="cuda")
    view = torch.as_strided(buf, a.shape, (ld, 1), offset)
    view.copy_(torch.from_numpy(np.ascontiguousarray(a)).to(dtype))
    return view


def _up16(n):
    return -(-n // 16) * 16


# ---------------------------------------------------------------- rows to 8 bits
ROWS = [(1, 1), (1, 64), (3, 2048), (2, 2055), (5, 7), (9, 1023), (1, 14336), (2, 16384), (2, 16385), (1, 40001), (70, 130)]


def _check_q8(q, scale, want, u):
    """q, scale of the GPU against rows `want` (float64), whose elements are known up to a relative error u."""
    ref, s, border = O.quantize(want)
    assert np.array_equal(np.isnan(scale), np.isnan(s))
    fine = ~np.isnan(s)
    # the scale: one rounding of a quotient of values that are known up to u, where those are results (u > 0) rounded to fp32 first; s itself
    # is a rounded one
    more = U32 if u else 0
    assert (np.abs(scale[fine].astype(np.float64) - s[fine]) <= (2 * U32 + more + u) * s[fine] + 1e-45).all()
    # an integer may be its neighbour only where the quotient is within its own error of the border between them
    off = q != ref
    assert (np.abs(q - ref)[off] == 1).all()
    assert (border[off] <= 127 * (2 * U32 + 2 * more + 2 * u)).all() if u else not off.any()      # (the element's rounding, and the scale's)


@pytest.mark.parametrize("rows,n", ROWS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_quantize(gpu, rows, n, dtype):
    torch, A = gpu
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    rng = np.random.default_rng([rows, n])
    a = rng.standard_normal((rows, n)) * np.exp(3 * rng.standard_normal((rows, 1)))
    x = _strided(torch, a, dt, n + 3, offset=1)
    q = torch.full((rows, _up16(n) + 16), 99, dtype=torch.int8, device="cuda")
    s = torch.empty(rows, device="cuda")
    A.q8_quantize(x.data_ptr(), _code(A, torch, x), n + 3, rows, n, q.data_ptr(), q.shape[1], s.data_ptr())
    got = _np(q)
    _check_q8(got[:, :n].astype(np.int64), _np(s), _np(x).astype(np.float64), 0)
    assert (got[:, n:] == 99).all()


@pytest.mark.parametrize("n", [8200, 14336, 20001])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize_many_rows_as_few(gpu, n, dtype):
    """Rows are laid over threads otherwise where they are many and long."""
    torch, A = gpu
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(1100, n, generator=gen, device="cuda").to(getattr(torch, dtype))
    got = []
    for step in (1100, 100):
        q, s = torch.zeros((1100, _up16(n)), dtype=torch.int8, device="cuda"), torch.empty(1100, device="cuda")
        for r in range(0, 1100, step):
            A.q8_quantize(x[r].data_ptr(), _code(A, torch, x), n, step, n, q[r].data_ptr(), q.shape[1], s[r:].data_ptr())
        got.append((q, s))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_quantize_special_rows(gpu):
    torch, A = gpu
    n = 50
    rows = np.zeros((9, n), np.float32)
    rows[1, 3] = np.inf
    rows[2, 49] = np.nan
    rows[3] = 1e-44                                    # max / 127 is 0 in fp32
    rows[4] = 3.4e38
    rows[5, ::2] = -5
    rows[6] = (np.arange(n) - 25) * 0.5 * 3            # scale 3 * 0.5 * 25 / 127 ..
    rows[6, 0] = 127 * 3
    rows[6, 1:5] = [7.5, -7.5, 4.5, 10.5]              # .. 3: quotients 2.5, -2.5, 1.5, 3.5 lie on the border: to even
    rows[7, 0] = -np.inf
    x = torch.from_numpy(rows).cuda()
    q, s = torch.empty((9, 64), dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    A.q8_quantize(x.data_ptr(), A.DTYPE_FP32, n, 9, n, q.data_ptr(), 64, s.data_ptr())
    q, s = _np(q)[:, :n], _np(s)
    assert s[0] == 0 and s[3] == 0 and (q[[0, 1, 2, 3, 7]] == 0).all()
    assert np.isnan(s[[1, 2, 7]]).all()
    assert (q[4] == 127).all() and s[4] == np.float32(np.float64(np.float32(3.4e38)) / 127)
    assert (q[5, ::2] == -127).all() and (q[5, 1::2] == 0).all()
    assert s[6] == 3 and list(q[6, 1:5]) == [2, -2, 2, 4]


@pytest.mark.parametrize("rows,n", ROWS)
@pytest.mark.parametrize("dtype,add,inplace", [("fp32", None, False), ("fp32", "bf16", True), ("bf16", "fp32", False), ("bf16", "bf16", True),
                                               ("fp32", "fp32", True)])
def test_rmsnorm(gpu, rows, n, dtype, add, inplace):
    torch, A = gpu
    if inplace and dtype == "bf16" and n > 16384:
        pytest.skip("refused (test_q8_arguments.py)")
    kind = {"fp32": torch.float32, "bf16": torch.bfloat16}
    rng = np.random.default_rng([rows, n, 5])
    x = _strided(torch, rng.standard_normal((rows, n)) * np.exp(rng.standard_normal((rows, 1))), kind[dtype], n + 1)
    d = None if add is None else _strided(torch, rng.standard_normal((rows, n)) * 0.3, kind[add], n + 5, offset=1)
    gain = torch.from_numpy((1 + 0.1 * rng.standard_normal(n)).astype(np.float32)).cuda()
    want_sum, y = O.rmsnorm(_np(x), None if d is None else _np(d), _np(gain), 1e-5)
    out = x if inplace else _strided(torch, np.zeros((rows, n)), kind[dtype], n + 1)
    q, s = torch.empty((rows, _up16(n)), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    A.q8_rmsnorm(x.data_ptr(), _code(A, torch, x), n + 1, 0 if d is None else d.data_ptr(), 0 if d is None else _code(A, torch, d), n + 5,
                 gain.data_ptr(), 1e-5, rows, n, out.data_ptr(), n + 1, q.data_ptr(), q.shape[1], s.data_ptr())
    assert np.array_equal(_np(out), torch.from_numpy(want_sum).to(kind[dtype]).float().numpy())
    # sums of n squares and a root in 64 bits: n + 4 roundings of 2^-53; eps is a float32
    _check_q8(_np(q)[:, :n].astype(np.int64), _np(s), O.rmsnorm(want_sum, None, _np(gain), float(np.float32(1e-5)))[1], (n + 8) * 2.0 ** -53)


@pytest.mark.parametrize("n", [512, 1030, 2048, 4096, 5120, 14336, 16384])
def test_rmsnorm_rows_keep_their_bits(gpu, n):
    torch, A = gpu
    rows = 1500
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, gain = torch.randn(rows, n, generator=gen, device="cuda"), torch.rand(n, generator=gen, device="cuda") + 0.5

    def norm(first, count):
        q, s = torch.zeros((count, _up16(n)), dtype=torch.int8, device="cuda"), torch.empty(count, device="cuda")
        A.q8_rmsnorm(x[first].data_ptr(), 0, n, 0, 0, 0, gain.data_ptr(), 1e-5, count, n, 0, 0, q.data_ptr(), q.shape[1], s.data_ptr())
        return q, s

    q, s = norm(0, rows)
    for first, count in ((0, 1), (1, 8), (9, 128), (137, 129), (266, 1024), (1290, 210)):
        a, b = norm(first, count)
        assert torch.equal(a, q[first:first + count]) and torch.equal(b, s[first:first + count])


def test_rmsnorm_of_huge_and_of_nonfinite_rows(gpu):
    torch, A = gpu
    n = 96
    rng = np.random.default_rng(3)
    rows = rng.standard_normal((4, n)).astype(np.float32)
    rows[0] *= 1e30                                     # squares are past fp32
    rows[1] = 0
    rows[2, 5] = np.nan
    x, gain = torch.from_numpy(rows).cuda(), torch.ones(n, device="cuda")
    q, s = torch.empty((4, n), dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    A.q8_rmsnorm(x.data_ptr(), 0, n, 0, 0, 0, gain.data_ptr(), 0.0, 4, n, 0, 0, q.data_ptr(), n, s.data_ptr())
    with np.errstate(all="ignore"):
        want = O.rmsnorm(rows, None, np.ones(n), 0.0)[1]
    assert np.isnan(_np(s)[1:3]).all()                  # 0 / sqrt(0), and a NaN
    _check_q8(_np(q).astype(np.int64)[[0, 3]], _np(s)[[0, 3]], want[[0, 3]], (n + 8) * 2.0 ** -53)


# ---------------------------------------------------------------- the product
def _matrix(gpu, n, k, gated=False, seed=0):
    torch, A = gpu
    rng = np.random.default_rng([n, k, seed])
    w = rng.integers(-127, 128, (n, k)).astype(np.int8)
    sw = (rng.random(n).astype(np.float32) + 0.5) * np.float32(0.01)
    return w, sw, A.Q8Matrix(w, A.DTYPE_INT8, n, k, scale=sw, gated=gated)


_SPACE = []


def _workspace(torch, need):
    """One for all products: each leaves it fit for the next, of any matrix."""
    if not _SPACE or _SPACE[0].numel() < need:
        _SPACE[:] = [torch.zeros(max(need, 1 << 24), dtype=torch.uint8, device="cuda")]
    return _SPACE[0]


def _product(gpu, m, x, sx, n, dtype, ldo=None, work=True, ldx=None):
    torch, A = gpu
    rows, k = x.shape
    xd = _strided(torch, x, torch.int8, ldx or _up16(k), fill=77)
    s = torch.from_numpy(sx).cuda()
    out = torch.full((rows, ldo or n), 5.0, dtype=dtype, device="cuda")
    need = m.workspace_bytes(rows)
    w = _workspace(torch, need)
    A.q8_gemm(m, xd.data_ptr(), ldx or _up16(k), s.data_ptr(), rows, out.data_ptr(), _code(A, torch, out), out.shape[1],
              w.data_ptr() if work else 0, w.numel() if work else 0)
    assert (out[:, n:] == 5).all().item()
    return out[:, :n]


GEMMS = [(1, 1, 1), (1, 16, 64), (3, 17, 65), (16, 100, 1000), (8, 4096, 512), (5, 300, 14336), (16, 2000, 576), (17, 129, 320), (32, 64, 4096),
         (33, 257, 129), (64, 80, 640), (100, 1040, 256), (129, 4112, 192), (200, 300, 2048), (256, 512, 1024), (300, 1000, 333), (1030, 520, 130),
         (513, 2304, 512)]


@pytest.mark.parametrize("rows,n,k", GEMMS)
def test_gemm(gpu, rows, n, k):
    torch, A = gpu
    w, sw, m = _matrix(gpu, n, k)
    rng = np.random.default_rng([rows, n, k])
    x = rng.integers(-127, 128, (rows, k)).astype(np.int8)
    sx = (rng.random(rows).astype(np.float32) + 0.5) * np.float32(0.02)
    want = O.gemm(x, sx, w, sw)
    got = _np(_product(gpu, m, x, sx, n, torch.float32, ldo=n + 3))
    assert (np.abs(got - want) <= 3.01 * U32 * np.abs(want)).all()            # an exact sum, rounded, times two scales
    half = _np(_product(gpu, m, x, sx, n, torch.bfloat16, ldo=n + 1, work=False, ldx=_up16(k) + 16))
    assert np.array_equal(half, O.bf16(got).astype(np.float32))               # the same bits without a workspace, rounded once more


# sizes whose contractions workgroups share where there is a workspace: every form that can
SHARED = [(20, 256, 8192), (32, 1000, 4099), (33, 2048, 8192), (60, 300, 14336), (100, 1024, 6000), (130, 2048, 8200), (250, 4096, 14336), (300, 1040, 8256),
          (500, 2048, 14330), (700, 500, 9000), (17, 2176, 4096), (40, 2176, 8192), (17, 4224, 5632), (17, 8320, 4608), (70, 8064, 6144), (1024, 4096, 14336)]


@pytest.mark.parametrize("rows,n,k", SHARED)
@pytest.mark.parametrize("gated", [False, True])
def test_gemm_shared(gpu, rows, n, k, gated):
    torch, A = gpu
    w, sw, m = _matrix(gpu, n - n % 2 if gated else n, k, gated=gated)
    no = n // 2 if gated else n
    rng = np.random.default_rng([rows, n, k])
    x = rng.integers(-127, 128, (rows, k)).astype(np.int8)
    sx = ((rng.random(rows) + 0.5) * 3 / (0.01 * 73 * 73 * np.sqrt(k))).astype(np.float32)
    assert m.workspace_bytes(rows + 16) >= m.workspace_bytes(rows) > 0 == m.workspace_bytes(16)
    alone = _product(gpu, m, x, sx, no, torch.float32, work=False)
    if not gated:
        # the sums in 64 bits are exact, float64 products of integers below 2^53
        sums = torch.from_numpy(x).cuda().double() @ torch.from_numpy(w).cuda().double().T
        want = sums.float() * torch.from_numpy(sx).cuda()[:, None] * torch.from_numpy(sw).cuda()
        assert torch.equal(alone, want)
    for _ in range(3):
        assert torch.equal(_product(gpu, m, x, sx, no, torch.float32), alone)
    s = torch.cuda.Stream()
    xd, sd = torch.from_numpy(np.pad(x, ((0, 0), (0, _up16(k) - k)))).cuda(), torch.from_numpy(sx).cuda()
    out, space = torch.zeros(rows, no, dtype=torch.float32, device="cuda"), torch.zeros(m.workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        for _ in range(2):
            A.q8_gemm(m, xd.data_ptr(), _up16(k), sd.data_ptr(), rows, out.data_ptr(), A.DTYPE_FP32, no, space.data_ptr(), space.numel(),
                      torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, alone)


@pytest.mark.parametrize("rows,n,k", [(1, 8, 64), (1, 500, 70), (16, 1000, 512), (40, 129, 300), (129, 100, 512), (300, 1024, 256), (520, 1100, 128)])
def test_gemm_gated(gpu, rows, n, k):
    torch, A = gpu
    w, sw, m = _matrix(gpu, 2 * n, k, gated=True)
    rng = np.random.default_rng([rows, n, k])
    x = rng.integers(-127, 128, (rows, k)).astype(np.int8)
    sx = ((rng.random(rows) + 0.5) * 3 / (0.01 * 73 * 73 * np.sqrt(k))).astype(np.float32)      # products of a few units
    y = O.gemm(x, sx, w, sw)
    want = O.swiglu(y)
    g = np.abs(y[:, :n])
    # the gate's error (3 roundings) moves silu by at most (1 + |g|) of it; the exponential's argument and result, sum, quotient and
    # product add |g| + 6 roundings, the up half 3
    rel = (3 * (1 + g) + g + 9) * U32
    got = _np(_product(gpu, m, x, sx, n, torch.float32))
    assert (np.abs(got - want) <= rel * np.abs(want) + 1e-37).all()
    assert np.array_equal(_np(_product(gpu, m, x, sx, n, torch.bfloat16)), O.bf16(got).astype(np.float32))


def test_gemm_extremes(gpu):
    """The longest contraction of the largest values; scales that are 0, NaN and infinite; no rows."""
    torch, A = gpu
    n, k = 20, 131072
    w = np.full((n, k), 127, np.int8)
    w[1::2] = -127
    m = A.Q8Matrix(w, A.DTYPE_INT8, n, k, scale=np.ones(n, np.float32))
    x = np.full((4, k), 127, np.int8)
    sx = np.array([1, 0, np.nan, np.inf], np.float32)
    got = _np(_product(gpu, m, x, sx, n, torch.float32))
    big = np.float32(127 * 127 * k)
    assert (got[0, ::2] == big).all() and (got[0, 1::2] == -big).all()
    assert (got[1] == 0).all() and np.isnan(got[2]).all() and np.isinf(got[3]).all()
    out = torch.full((1, n), 3.0, device="cuda")
    A.q8_gemm(m, out.data_ptr(), k, out.data_ptr(), 0, out.data_ptr(), A.DTYPE_FP32, n)
    assert (out == 3).all().item()


def test_gemm_rows_keep_their_bits(gpu):
    torch, A = gpu
    n, k = 1300, 2112
    w, sw, m = _matrix(gpu, n, k)
    rng = np.random.default_rng(1)
    x = rng.integers(-127, 128, (700, k)).astype(np.int8)
    sx = (rng.random(700).astype(np.float32) + 0.5) * np.float32(0.02)
    whole = _product(gpu, m, x, sx, n, torch.bfloat16)
    for lo, hi in ((0, 1), (5, 13), (100, 116), (0, 17), (3, 50), (10, 138), (200, 500)):
        assert torch.equal(_product(gpu, m, x[lo:hi], sx[lo:hi], n, torch.bfloat16), whole[lo:hi]), (lo, hi)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_matrix_from_floats(gpu, dtype):
    """A matrix that is rounded here has the integers and scales of its rows; read off through unit vectors."""
    torch, A = gpu
    n, k = 70, 45
    rng = np.random.default_rng(8)
    w = rng.standard_normal((n, k)).astype(np.float32)
    w[3] = 0
    w[4, 2] = np.inf
    t = torch.from_numpy(w).to(torch.float32 if dtype == "fp32" else torch.bfloat16).cuda()
    wide = torch.zeros((n, k + 6), dtype=t.dtype, device="cuda")
    wide[:, :k] = t
    m = A.Q8Matrix(wide.data_ptr(), _code(A, torch, t), n, k, ld=k + 6, on_device=True)
    got = _np(_product(gpu, m, np.eye(k, dtype=np.int8), np.ones(k, np.float32), n, torch.float32)).T
    q, s, _ = O.quantize(_np(t))
    assert np.isnan(got[4]).all()
    fine = np.arange(n) != 4
    assert np.array_equal(got[fine], (q.astype(np.float32) * s[:, None])[fine])
    host = A.Q8Matrix(w if dtype == "fp32" else t.cpu().view(torch.int16).numpy(), _code(A, torch, t), n, k)
    again = _np(_product(gpu, host, np.eye(k, dtype=np.int8), np.ones(k, np.float32), n, torch.float32)).T
    assert np.array_equal(again[fine], got[fine])


# ---------------------------------------------------------------- the cache
def _rope(torch, positions, hd):
    ang = np.arange(positions)[:, None] * 10000.0 ** (-2.0 * np.arange(hd // 2) / hd)
    c, s = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    return c, s, torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()


def _append(gpu, cache, seqs, pos0, k, v, rope=(0, 0), layer=0, ld_more=0):
    """k, v: one [n, heads, hd] bf16 tensor a sequence."""
    torch, A = gpu
    flat = [torch.cat([a.reshape(a.shape[0], -1) for a in x]) for x in (k, v)]
    width = flat[0].shape[1]
    pads = []
    for f in flat:
        p = torch.full((f.shape[0], width + ld_more), float("nan"), dtype=torch.bfloat16, device="cuda")
        p[:, :width] = f
        pads.append(p)
    cache.append(layer, seqs, pos0, [a.shape[0] for a in k], pads[0].data_ptr(), pads[1].data_ptr(), width + ld_more, *rope)
    torch.cuda.synchronize()


def _read(gpu, cache, seq, pos0, n, heads, hd, layer=0):
    torch, A = gpu
    k, v = (torch.empty((n, heads, hd), device="cuda") for _ in range(2))
    cache.read(layer, [seq], [pos0], [n], k.data_ptr(), v.data_ptr(), A.DTYPE_FP32, heads * hd)
    return _np(k), _np(v)


def _rand(torch, rng, *shape, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("block", [1, 16, 32, 64])
@pytest.mark.parametrize("hd,heads", [(64, 3), (128, 2)])
def test_append_in_pieces(gpu, block, hd, heads):
    """Pieces of odd lengths, growing so that blocks are rounded again; then a piece behind a truncation."""
    torch, A = gpu
    cache = A.Q8Cache(n_layers=2, n_seqs=2, n_q_heads=heads, n_kv_heads=heads, head_dim=hd, capacity=400, block=block)
    ref = [O.Cache(heads, hd, 448, block) for _ in range(2)]
    rng = np.random.default_rng([block, hd])
    at = 0
    for i, n in enumerate((1, 2, 5, 31, 32, 64, 1, 65, 7, 100)):
        k, v = _rand(torch, rng, n, heads, hd, std=1 + i % 4), _rand(torch, rng, n, heads, hd, std=1 + (i * 3) % 5)
        _append(gpu, cache, [1], [at], [k], [v], layer=1, ld_more=3)
        ref[0].append(at, _np(k))
        ref[1].append(at, _np(v))
        at += n
    kk, vv = _read(gpu, cache, 1, 0, at, heads, hd, layer=1)
    assert np.array_equal(kk, ref[0].values(at).astype(np.float32)) and np.array_equal(vv, ref[1].values(at).astype(np.float32))
    k, v = _rand(torch, rng, 40, heads, hd, std=0.1), _rand(torch, rng, 40, heads, hd, std=30)
    _append(gpu, cache, [1], [100], [k], [v], layer=1)
    ref[0].append(100, _np(k))
    ref[1].append(100, _np(v))
    kk, vv = _read(gpu, cache, 1, 0, 140, heads, hd, layer=1)
    assert np.array_equal(kk, ref[0].values(140).astype(np.float32)) and np.array_equal(vv, ref[1].values(140).astype(np.float32))
    other = _read(gpu, cache, 0, 0, 400, heads, hd, layer=1)
    first = _read(gpu, cache, 1, 0, 400, heads, hd, layer=0)
    assert not any(a.any() for a in other + first)                # nothing of another sequence or layer was touched


def test_append_turns_keys(gpu):
    torch, A = gpu
    for hd in (64, 128):
        cache = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=4, n_kv_heads=2, head_dim=hd, capacity=300)
        c, s, dc, ds = _rope(torch, 300, hd)
        rng = np.random.default_rng(hd)
        k, v = _rand(torch, rng, 150, 2, hd), _rand(torch, rng, 150, 2, hd)
        _append(gpu, cache, [0], [129], [k], [v], rope=(dc.data_ptr(), ds.data_ptr()))
        kk, vv = _read(gpu, cache, 0, 129, 150, 2, hd)
        want = O.rotate(_np(k), c[129:279], s[129:279])
        most = np.abs(want).max(-1, keepdims=True)
        # half a step of the scale, and the three roundings of a turned component (of at most sqrt(2) * the largest)
        assert (np.abs(kk - want) <= most / 254 * (1 + 1e-5) + 8 * U32 * np.abs(_np(k)).max(-1, keepdims=True)).all()
        ref = O.Cache(2, hd, 320, 1)
        ref.append(129, _np(v))
        assert np.array_equal(vv, ref.values(279)[129:].astype(np.float32))


def test_append_of_several_sequences_and_of_zeros_and_nans(gpu):
    torch, A = gpu
    rng = np.random.default_rng(0)
    for block in (1, 32):
        cache = A.Q8Cache(n_layers=1, n_seqs=5, n_q_heads=2, n_kv_heads=2, head_dim=64, capacity=128, block=block)
        ref = {}
        seqs, pos0, ks, vs = [4, 0, 2], [0, 61, 30], [], []
        for s, p, n in zip(seqs, pos0, (70, 5, 1)):
            k, v = _rand(torch, rng, n, 2, 64), _rand(torch, rng, n, 2, 64)
            if s == 0:
                k[1], v[2] = 0, 0
                k[3, 1, 7] = float("nan")
                v[4, 0, 9] = float("-inf")
            ks.append(k)
            vs.append(v)
            ref[s] = (O.Cache(2, 64, 128, block), O.Cache(2, 64, 128, block))
            with np.errstate(invalid="ignore"):
                ref[s][0].append(p, _np(k))
                ref[s][1].append(p, _np(v))
        _append(gpu, cache, seqs, pos0, ks, vs)
        for s, p, n in zip(seqs, pos0, (70, 5, 1)):
            got = _read(gpu, cache, s, p, n, 2, 64)
            for a, r in zip(got, ref[s]):
                assert np.array_equal(a, r.values(p + n)[p:].astype(np.float32), equal_nan=True), (block, s)


# ---------------------------------------------------------------- attention
def _attend(gpu, cache, seqs, pos0, q, scale, rope=(0, 0), layer=0, more=0):
    """q: one [n, Hq, hd] bf16 tensor a sequence; rows at a distance that is `more` longer than they are."""
    torch, A = gpu
    flat = torch.cat([a.reshape(a.shape[0], -1) for a in q])
    width = flat.shape[1]
    qq = torch.full((flat.shape[0], width + more), float("nan"), dtype=torch.bfloat16, device="cuda")
    qq[:, :width] = flat
    out = torch.full((flat.shape[0], width + more), 9.0, dtype=torch.bfloat16, device="cuda")
    cache.attention(layer, seqs, pos0, [a.shape[0] for a in q], qq.data_ptr(), width + more, scale, *rope, out.data_ptr(), width + more)
    torch.cuda.synchronize()
    assert (out[:, width:] == 9).all().item()
    return list(torch.split(out[:, :width].reshape(-1, *q[0].shape[1:]), [a.shape[0] for a in q]))


def _tolerance(q, k, v, pos0, scale, out, weighted, s, turned):
    """How far a result may be off, element by element:
    its own rounding to bf16; the weights' to half (2^-11) and the instruction's for 2^x (2^-22), of the weighted mean |v|; and what
    the scores are off, twice (numerator and denominator): the query's 16 bits (half of largest / 32512 in every component, times the
    key's magnitudes), a turn's roundings, and the fp32 chain from the integer product to the exponent (five roundings of the score,
    one of its distance from the reference), as exp(d) - 1 <= 1.1 d.  Sums of n fp32 terms: n roundings of the weighted mean; within a
    chunk, of at most 512 keys, the terms are 1152 + v for integers v of up to 127 steps."""
    group = q.shape[1] // k.shape[1]
    kabs = np.repeat(np.abs(k).sum(-1), group, 1).T[None]                        # [1, Hq, positions]
    qmost = np.abs(q).max(-1)[:, :, None]                                        # [rows, Hq, 1]
    d = scale * kabs * qmost * (0.5 / 32512 + 2 * U32 + (8 * U32 if turned else 0))
    seen = np.isfinite(s)
    size = np.where(seen, np.abs(np.where(seen, s, 0)), 0).max(-1, keepdims=True)
    d = np.where(seen, d + 7 * U32 * 2 * size, 0).max(-1)[..., None]
    assert d.max() < 0.1
    n = k.shape[0]
    return U16 * np.abs(out) + weighted * (2.0 ** -11 + 2.0 ** -21 + 2 * 1.1 * d + 2 * n * U32) + 520 * U32 * 1280 / 127 * np.abs(v).max() + 1e-30


def _case(gpu, heads, block, lens, rows, rope=True, seed=0, std=1.0, cap=None):
    """Sequences of lens[i] held positions and rows[i] new ones, appended and asked about."""
    torch, A = gpu
    hq, hkv, hd = heads
    cap = cap or max(a + b for a, b in zip(lens, rows)) + 3
    cache = A.Q8Cache(n_layers=1, n_seqs=len(lens), n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, capacity=cap, block=block)
    rng = np.random.default_rng([seed, hq, hd, block])
    c, s, dc, ds = _rope(torch, cap, hd)
    ptr = (dc.data_ptr(), ds.data_ptr()) if rope else (0, 0)
    qs = []
    for i, (held, n) in enumerate(zip(lens, rows)):
        k, v = _rand(torch, rng, held + n, hkv, hd, std=std), _rand(torch, rng, held + n, hkv, hd, std=std)
        _append(gpu, cache, [i], [0], [k], [v], rope=ptr)
        qs.append(_rand(torch, rng, n, hq, hd, std=std))
    return cache, qs, (c, s), ptr, (dc, ds)


def _check(gpu, cache, qs, tables, lens, heads, outs, scale, rope):
    hq, hkv, hd = heads
    for i, (q, held, out) in enumerate(zip(qs, lens, outs)):
        n = q.shape[0]
        k, v = (a.astype(np.float64) for a in _read(gpu, cache, i, 0, held + n, hkv, hd))
        qn = _np(q).astype(np.float64)
        if rope:
            qn = O.rotate(qn, tables[0][held:held + n], tables[1][held:held + n])
        for lo in range(0, n, 64):                      # a few rows at a time
            hi = min(n, lo + 64)
            want, weighted, s = O.attention(qn[lo:hi], k, v, held + lo, scale)
            tol = _tolerance(qn[lo:hi], k, v, held + lo, scale, want, weighted, s, rope)
            err = np.abs(_np(out)[lo:hi].astype(np.float64) - want)
            assert (err <= tol).all(), (i, lo, float((err / tol).max()))


_A = [((4, 4, 64), 1, [0], [1]), ((4, 2, 128), 1, [0], [1]), ((8, 2, 64), 1, [1], [1]), ((8, 1, 128), 1, [30], [3]),
      ((8, 2, 128), 1, [31], [2]), ((8, 2, 64), 16, [63], [5]), ((4, 4, 128), 32, [64], [16]), ((16, 2, 64), 64, [127], [9]),
      ((8, 2, 128), 1, [255], [16]), ((2, 1, 64), 1, [511], [1]), ((32, 8, 64), 1, [700], [5]), ((8, 2, 64), 1, [0, 100, 5], [4, 1, 9]),
      ((8, 1, 64), 32, [33, 300], [1, 15]), ((4, 4, 64), 1, [3] * 16, [1] * 16), ((8, 2, 128), 1, [40], [17]), ((4, 2, 64), 1, [0], [300]),
      ((8, 2, 128), 64, [100], [333]), ((16, 2, 128), 1, [70, 0], [150, 90]), ((4, 4, 128), 16, [500], [129]), ((8, 8, 64), 1, [10], [700]),
      ((8, 1, 64), 1, [2000], [40])]


@pytest.mark.parametrize("heads,block,lens,rows", _A)
@pytest.mark.parametrize("rope", [False, True])
def test_attention(gpu, heads, block, lens, rows, rope):
    scale = heads[2] ** -0.5
    cache, qs, tables, ptr, _keep = _case(gpu, heads, block, lens, rows, rope)
    outs = _attend(gpu, cache, list(range(len(lens))), lens, qs, scale, ptr, more=5)
    _check(gpu, cache, qs, tables, lens, heads, outs, scale, rope)


@pytest.mark.parametrize("heads,block,length", [((8, 2, 64), 1, 600), ((8, 2, 128), 1, 900), ((4, 4, 128), 1, 300), ((8, 1, 64), 32, 500),
                                                ((32, 8, 128), 1, 1000)])
def test_attention_rows_keep_their_bits(gpu, heads, block, length):
    """A row's result from one row at a time, from windows and from all rows at once, and beside other sequences.  What the cache holds
    is fixed first: with blocks of several positions that depends on how it was filled."""
    torch, A = gpu
    scale = heads[2] ** -0.5
    cache, (q,), _, ptr, _keep = _case(gpu, heads, block, [0], [length], cap=4096 if length == 1000 else None)
    whole, = _attend(gpu, cache, [0], [0], [q], scale, ptr)
    for lo, n in ((0, 1), (1, 3), (length - 1, 1), (length - 16, 16), (77, 8), (250, 13), (200, 64), (30, 200)):
        part, = _attend(gpu, cache, [0], [lo], [q[lo:lo + n]], scale, ptr)
        assert torch.equal(part, whole[lo:lo + n]), (lo, n)


def test_cache_of_single_positions_does_not_depend_on_how_it_was_filled(gpu):
    torch, A = gpu
    rng = np.random.default_rng(2)
    k, v = _rand(torch, rng, 150, 2, 64), _rand(torch, rng, 150, 2, 64)
    c, s, dc, ds = _rope(torch, 256, 64)
    got = []
    for cuts in ([0, 150], list(range(0, 151, 10)), [0, 1, 64, 65, 100, 150]):
        cache = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=8, n_kv_heads=2, head_dim=64, capacity=256)
        _append(gpu, cache, [0], [0], [_rand(torch, rng, 200, 2, 64)], [_rand(torch, rng, 200, 2, 64, std=1e4)])     # truncated to nothing
        for lo, hi in zip(cuts, cuts[1:]):
            _append(gpu, cache, [0], [lo], [k[lo:hi]], [v[lo:hi]], rope=(dc.data_ptr(), ds.data_ptr()))
        got.append(_read(gpu, cache, 0, 0, 150, 2, 64))
    for g in got[1:]:
        assert np.array_equal(g[0], got[0][0]) and np.array_equal(g[1], got[0][1])


def test_attention_sees_nothing_behind_a_row(gpu):
    """Positions behind the row that hold NaN, infinities or huge values, in its tile and chunk, change no bit of it."""
    torch, A = gpu
    heads = (8, 2, 64)
    rng = np.random.default_rng(4)
    for n, lo in ((3, 40), (200, 20)):
        cache, (q,), _, ptr, _keep = _case(gpu, heads, 1, [lo], [n], cap=512, seed=n)
        clean, = _attend(gpu, cache, [0], [lo], [q], 0.125, ptr)
        bad = _rand(torch, rng, 130, 2, 64, std=1e30)
        bad[0, 0, 3], bad[1, 1, 5], bad[2] = float("nan"), float("inf"), 0
        _append(gpu, cache, [0], [lo + n], [bad], [bad])
        again, = _attend(gpu, cache, [0], [lo], [q], 0.125, ptr)
        assert torch.equal(clean, again)
        seen, = _attend(gpu, cache, [0], [lo], [torch.cat([q, q[:2]])], 0.125, ptr)           # the row that stands on the NaN sees it
        assert torch.equal(seen[:n], clean)
        assert torch.isnan(seen[n, :4]).all().item()


def test_attention_of_unlike_scales(gpu):
    """Values whose scales lie 2^60 apart, all-zero values and keys, a query of zeros, scores far from 0."""
    torch, A = gpu
    heads = (4, 2, 64)
    rng = np.random.default_rng(6)
    k, v = _rand(torch, rng, 300, 2, 64), _rand(torch, rng, 300, 2, 64)
    v[::3] *= 2.0 ** -30
    v[1::7] *= 2.0 ** 30
    v[5:9], k[20:22] = 0, 0
    cache = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=4, n_kv_heads=2, head_dim=64, capacity=300)
    _append(gpu, cache, [0], [0], [k], [v])
    q = _rand(torch, rng, 300, 4, 64, std=6)
    q[7] = 0
    for lo, n in ((290, 10), (0, 300)):
        out, = _attend(gpu, cache, [0], [lo], [q[lo:lo + n]], 0.125)
        _check_rows(gpu, cache, q[lo:lo + n], lo, heads, out, 0.125)
    zero = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=4, n_kv_heads=2, head_dim=64, capacity=300)
    _append(gpu, zero, [0], [0], [k], [torch.zeros_like(v)])
    assert not _attend(gpu, zero, [0], [100], [q[100:110]], 0.125)[0].any().item()


def _check_rows(gpu, cache, q, pos0, heads, out, scale):
    hq, hkv, hd = heads
    k, v = (a.astype(np.float64) for a in _read(gpu, cache, 0, 0, pos0 + q.shape[0], hkv, hd))
    qn = _np(q).astype(np.float64)
    want, weighted, s = O.attention(qn, k, v, pos0, scale)
    tol = _tolerance(qn, k, v, pos0, scale, want, weighted, s, False)
    # Weights times scales that half holds with less than 11 bits: half a step of its smallest numbers is 2^-25, and the chunk's largest
    # scale is brought to at least 2^10, so each key is off by at most 2^-35 of the largest value; denominators are 1 or more
    tol = tol + k.shape[0] * 2.0 ** -35 * np.abs(v).max()
    assert (np.abs(_np(out).astype(np.float64) - want) <= tol).all()


def test_attention_of_nonfinite_queries(gpu):
    torch, A = gpu
    cache, (q,), _, ptr, _keep = _case(gpu, (4, 2, 64), 1, [50], [6])
    clean, = _attend(gpu, cache, [0], [50], [q], 0.125, ptr)
    q[2, 1, 5], q[4, 3, 0] = float("nan"), float("inf")
    got, = _attend(gpu, cache, [0], [50], [q], 0.125, ptr)
    bad = torch.zeros(6, 4, dtype=torch.bool)
    bad[2, 1] = bad[4, 3] = True
    assert torch.isnan(got[bad.cuda()]).all().item()
    assert torch.equal(got[~bad.cuda()], clean[~bad.cuda()])


# ---------------------------------------------------------------- together
def _layer(gpu, t, stream=0):
    """A decoder layer's way through the operators: norm, QKV, append, attention, rows to 8 bits, O, norm, gate/up, down."""
    torch, A = gpu
    p = lambda name: t[name].data_ptr()   # noqa: E731
    rows, d, hq, hkv, hd, F = t["dims"]
    qd, kvd, nqkv = hq * hd, hkv * hd, (hq + 2 * hkv) * hd
    w = (p("work"), t["work"].numel())
    A.q8_rmsnorm(p("x"), A.DTYPE_FP32, d, 0, 0, 0, p("gain"), 1e-5, rows, d, 0, 0, p("xq"), d, p("xs"), stream)
    A.q8_gemm(t["wqkv"], p("xq"), d, p("xs"), rows, p("qkv"), A.DTYPE_BF16, nqkv, *w, stream)
    t["cache"].append(0, t["ids"], t["pos"], t["n"], p("qkv") + 2 * qd, p("qkv") + 2 * (qd + kvd), nqkv, p("cos"), p("sin"), stream)
    t["cache"].attention(0, t["ids"], t["pos"], t["n"], p("qkv"), nqkv, hd ** -0.5, p("cos"), p("sin"), p("att"), qd, stream)
    A.q8_quantize(p("att"), A.DTYPE_BF16, qd, rows, qd, p("aq"), qd, p("as_"), stream)
    A.q8_gemm(t["wo"], p("aq"), qd, p("as_"), rows, p("delta"), A.DTYPE_BF16, d, *w, stream)
    A.q8_rmsnorm(p("x"), A.DTYPE_FP32, d, p("delta"), A.DTYPE_BF16, d, p("gain"), 1e-5, rows, d, p("mid"), d, p("xq"), d, p("xs"), stream)
    A.q8_gemm(t["wgu"], p("xq"), d, p("xs"), rows, p("h"), A.DTYPE_BF16, F, *w, stream)
    A.q8_quantize(p("h"), A.DTYPE_BF16, F, rows, F, p("hq"), F, p("hs"), stream)
    A.q8_gemm(t["wd"], p("hq"), F, p("hs"), rows, p("out"), A.DTYPE_FP32, d, *w, stream)


def _layer_state(gpu, ids, pos, n, seed=0, dims=(128, 4, 2, 64, 320)):
    torch, A = gpu
    d, hq, hkv, hd, F = dims
    rows = sum(n)
    rng = np.random.default_rng(seed)
    t = {"dims": (rows, d, hq, hkv, hd, F), "ids": ids, "pos": pos, "n": n}
    mat = lambda a, b: (rng.standard_normal((a, b)) * b ** -0.5).astype(np.float32)   # noqa: E731
    t["w"] = {"wqkv": mat((hq + 2 * hkv) * hd, d), "wo": mat(d, hq * hd), "wgu": mat(2 * F, d), "wd": mat(d, F)}
    for name, w in t["w"].items():
        t[name] = A.Q8Matrix(w, A.DTYPE_FP32, w.shape[0], w.shape[1], gated=name == "wgu")
    t["work"] = torch.zeros(max(16, max(t[m].workspace_bytes(rows) for m in t["w"])), dtype=torch.uint8, device="cuda")
    t["cache"] = A.Q8Cache(n_layers=1, n_seqs=max(ids) + 1, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, capacity=256)
    t["ctab"], t["stab"], t["cos"], t["sin"] = _rope(torch, 256, hd)
    t["x"] = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).cuda()
    t["gain"] = torch.from_numpy((1 + 0.1 * rng.standard_normal(d)).astype(np.float32)).cuda()
    i8, f32, b16 = torch.int8, torch.float32, torch.bfloat16
    for name, width, dt in (("xq", d, i8), ("qkv", (hq + 2 * hkv) * hd, b16), ("att", hq * hd, b16), ("aq", hq * hd, i8), ("delta", d, b16),
                            ("mid", d, f32), ("h", F, b16), ("hq", F, i8), ("out", d, f32)):
        t[name] = torch.zeros((rows, width), dtype=dt, device="cuda")
    for name in ("xs", "as_", "hs"):
        t[name] = torch.zeros(rows, device="cuda")
    return t


@pytest.mark.parametrize("n", [1, 8, 100])
def test_a_layer(gpu, n):
    """The operators one after the other, as a decoder layer has them.  Each step is checked against its plain form on what the
    step before left."""
    torch, A = gpu
    t = _layer_state(gpu, [0], [0], [n])
    _layer(gpu, t)
    torch.cuda.synchronize()
    rows, d, hq, hkv, hd, F = t["dims"]
    W = {m: O.quantize(w)[:2] for m, w in t["w"].items()}
    eps = float(np.float32(1e-5))
    s, y = O.rmsnorm(_np(t["x"]), _np(t["delta"]), _np(t["gain"]), eps)
    assert np.array_equal(_np(t["mid"]), s)
    _check_q8(_np(t["xq"]).astype(np.int64), _np(t["xs"]), y, (d + 8) * 2.0 ** -53)
    _check_q8(_np(t["aq"]).astype(np.int64), _np(t["as_"]), _np(t["att"]).astype(np.float64), 0)
    _check_q8(_np(t["hq"]).astype(np.int64), _np(t["hs"]), _np(t["h"]).astype(np.float64), 0)
    want = O.gemm(_np(t["hq"]), _np(t["hs"]), *W["wd"])
    assert (np.abs(_np(t["out"]) - want) <= 3.01 * U32 * np.abs(want)).all()
    want = O.gemm(_np(t["aq"]), _np(t["as_"]), *W["wo"])
    assert (np.abs(_np(t["delta"]) - want) <= (U16 + 4 * U32) * np.abs(want)).all()
    q = _np(t["qkv"])[:, :hq * hd].reshape(rows, hq, hd)
    _check(gpu, t["cache"], [torch.from_numpy(q)], (t["ctab"], t["stab"]), [0], (hq, hkv, hd), [t["att"].view(rows, hq, hd)], hd ** -0.5, True)


def test_on_another_stream(gpu):
    torch, A = gpu
    t = _layer_state(gpu, [0], [0], [5])
    _layer(gpu, t)
    torch.cuda.synchronize()
    want = t["out"].clone()
    t["out"].zero_()
    t["x"].mul_(1.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _layer(gpu, t, s.cuda_stream)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(t["out"], want)


def test_in_a_graph(gpu):
    """Captured once, replayed on changed rows with eager work in between; two graphs side by side."""
    torch, A = gpu
    graphs = []
    for seed, n in ((0, [3, 1]), (1, [60, 40])):
        t = _layer_state(gpu, [0, 1], [0, 7], n, seed=seed)
        _layer(gpu, t)                                 # (a kernel is loaded at its first launch)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _layer(gpu, t, torch.cuda.current_stream().cuda_stream)
        graphs.append((g, t))
    for i in range(4):
        wants = []
        for g, t in graphs:
            t["x"].copy_(torch.from_numpy(np.random.default_rng([i, 9]).standard_normal(tuple(t["x"].shape)).astype(np.float32)))
            _layer(gpu, t)
            torch.cuda.synchronize()
            wants.append(t["out"].clone())
            t["out"].zero_()
        torch.cuda.synchronize()
        for g, t in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (g, t), want in zip(graphs, wants):
            assert torch.equal(t["out"], want)


# ---------------------------------------------------------------- far apart, side by side, refused
def test_gemm_rows_far_apart(gpu):
    torch, A = gpu
    rows, n, k = 300, 512, 200
    w, sw, m = _matrix(gpu, n, k)
    rng = np.random.default_rng(5)
    x, sx = rng.integers(-127, 128, (rows, k)).astype(np.int8), rng.random(rows).astype(np.float32)
    want = _product(gpu, m, x, sx, n, torch.float32)
    for ld in (1 << 22, (1 << 24) + 16):               # row 255 of a tile at 2^30 and past 2^32
        xd = torch.empty((rows - 1) * ld + 256, dtype=torch.int8, device="cuda")
        xd.as_strided((rows, k), (ld, 1)).copy_(torch.from_numpy(x))
        s, out = torch.from_numpy(sx).cuda(), torch.empty(rows, n, dtype=torch.float32, device="cuda")
        A.q8_gemm(m, xd.data_ptr(), ld, s.data_ptr(), rows, out.data_ptr(), A.DTYPE_FP32, n)
        assert torch.equal(out, want), ld


def test_products_side_by_side(gpu):
    """Two streams, one matrix, a workspace each."""
    torch, A = gpu
    rows, n, k = 200, 1024, 8192
    w, sw, m = _matrix(gpu, n, k)
    rng = np.random.default_rng(6)
    jobs = []
    for i in range(2):
        x, sx = rng.integers(-127, 128, (rows, k)).astype(np.int8), rng.random(rows).astype(np.float32)
        want = _product(gpu, m, x, sx, n, torch.float32, work=False)
        jobs.append((torch.from_numpy(x).cuda(), torch.from_numpy(sx).cuda(), torch.zeros(m.workspace_bytes(rows), dtype=torch.uint8, device="cuda"),
                     torch.zeros(20, rows, n, dtype=torch.float32, device="cuda"), torch.cuda.Stream(), want))
    torch.cuda.synchronize()
    for r in range(20):
        for x, s, space, out, stream, _ in jobs:
            A.q8_gemm(m, x.data_ptr(), k, s.data_ptr(), rows, out[r].data_ptr(), A.DTYPE_FP32, n, space.data_ptr(), space.numel(), stream.cuda_stream)
    torch.cuda.synchronize()
    for *_, out, _, want in jobs:
        assert (out == want).all().item()


@pytest.mark.parametrize("hd", [64, 128])
def test_a_cache_past_32_bits(gpu, hd):
    """The last sequences of a large cache hold and give what the first ones do."""
    torch, A = gpu
    seqs, cap, heads = (1 << 33) // (8 * (1 << 16) * hd) + 2, 1 << 16, (16, 8, hd)
    cache = A.Q8Cache(n_layers=1, n_seqs=seqs, n_q_heads=16, n_kv_heads=8, head_dim=hd, capacity=cap, block=16)
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, base = 70, cap - 400
    k, v = (torch.randn(n, 8 * hd, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(n, 16, hd, generator=gen, device="cuda").to(torch.bfloat16)
    got = []
    for s in (0, seqs - 1):
        for pos in (0, base):                           # an early stretch and a late one; what lies between are zeros
            cache.append(0, [s], [pos], [n], k.data_ptr(), v.data_ptr(), 8 * hd)
        kk, vv = (torch.empty(n, 8 * hd, dtype=torch.float32, device="cuda") for _ in range(2))
        cache.read(0, [s], [base], [n], kk.data_ptr(), vv.data_ptr(), A.DTYPE_FP32, 8 * hd)
        got.append((kk, vv, _attend(gpu, cache, [s], [base], [q], hd ** -0.5)[0], _attend(gpu, cache, [s], [base + n - 1], [q[:1]], hd ** -0.5)[0]))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert (got[1][0].view(n, -1) - k.float()).abs().max().item() <= k.float().abs().max().item() / 127 * 0.501
    assert got[1][2].float().abs().max().item() > 0


def test_refusals_with_handles(gpu):
    torch, A = gpu
    E = A.AmusdError
    w, sw, m = _matrix(gpu, 8, 64)
    x, s, out = (torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda"), torch.full((4, 8), 3.0, device="cuda"))
    good = dict(w=m, x=x.data_ptr(), ldx=64, scale=s.data_ptr(), rows=4, out=out.data_ptr(), dtype=A.DTYPE_FP32, ldo=8, workspace=0, workspace_bytes=0)
    for bad in (dict(x=0), dict(x=x.data_ptr() + 8), dict(ldx=48), dict(ldx=72), dict(scale=0), dict(rows=-1), dict(out=0), dict(out=out.data_ptr() + 2), dict(dtype=2),
                dict(ldo=7), dict(workspace=x.data_ptr() + 4, workspace_bytes=64), dict(workspace=x.data_ptr(), workspace_bytes=-1)):
        with pytest.raises(E):
            A.q8_gemm(*{**good, **bad}.values())
    A.q8_gemm(*{**good, "rows": 0}.values())
    with pytest.raises(E):
        m.workspace_bytes(-1)
    c = A.Q8Cache(n_layers=2, n_seqs=3, n_q_heads=8, n_kv_heads=2, head_dim=64, capacity=100, block=16)              # room for 128: whole tiles of 64
    kv, q, o = (torch.zeros(4, d, dtype=torch.bfloat16, device="cuda") for d in (128, 512, 512))
    o += 3
    f = torch.full((4, 128), 3.0, device="cuda")
    for layer, seqs, pos, n in ((2, [0], [0], [1]), (-1, [0], [0], [1]), (0, [3], [0], [1]), (0, [-1], [0], [1]), (0, [0, 0], [0, 1], [1, 1]), (0, [0], [-1], [2]),
                                (0, [0], [127], [2]), (0, [0], [2 ** 31 - 1], [4]), (0, [0], [0], [0]), (0, [], [], []), (0, list(range(17)), [0] * 17, [1] * 17)):
        with pytest.raises(E):
            c.append(layer, seqs, pos, n, kv.data_ptr(), kv.data_ptr(), 128)
        with pytest.raises(E):
            c.read(layer, seqs, pos, n, f.data_ptr(), f.data_ptr(), A.DTYPE_FP32, 128)
        with pytest.raises(E):
            c.attention(layer, seqs, pos, n, q.data_ptr(), 512, 0.125, 0, 0, o.data_ptr(), 512)
    one = (0, [0], [0], [1])
    for bad in ((0, kv.data_ptr(), 128), (kv.data_ptr(), 0, 128), (kv.data_ptr(), kv.data_ptr(), 127), (kv.data_ptr() + 1, kv.data_ptr(), 128)):
        with pytest.raises(E):
            c.append(*one, *bad)
    with pytest.raises(E):
        c.append(*one, kv.data_ptr(), kv.data_ptr(), 128, f.data_ptr(), 0)
    for bad in ((f.data_ptr(), 0, 0, 128), (f.data_ptr(), f.data_ptr(), 2, 128), (f.data_ptr() + 2, f.data_ptr(), 0, 128), (f.data_ptr(), f.data_ptr(), 0, 100)):
        with pytest.raises(E):
            c.read(*one, *bad)
    for bad in ((0, 512, 0.125, 0, 0, o.data_ptr(), 512), (q.data_ptr(), 511, 0.125, 0, 0, o.data_ptr(), 512), (q.data_ptr(), 512, 0.0, 0, 0, o.data_ptr(), 512),
                (q.data_ptr(), 512, float("inf"), 0, 0, o.data_ptr(), 512), (q.data_ptr(), 512, float("nan"), 0, 0, o.data_ptr(), 512),
                (q.data_ptr(), 512, 0.125, f.data_ptr(), 0, o.data_ptr(), 512), (q.data_ptr(), 512, 0.125, 0, 0, o.data_ptr(), 500)):
        with pytest.raises(E):
            c.attention(*one, *bad)
    with pytest.raises(E):
        A.Q8Cache(n_layers=64, n_seqs=64, n_q_heads=8, n_kv_heads=8, head_dim=128, capacity=1 << 24, block=64)       # more memory than there is; nothing is left behind for the next call
    long = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=8, n_kv_heads=1, head_dim=64, capacity=1 << 17, block=64)
    with pytest.raises(E):
        long.attention(0, [0], [0], [(1 << 16) + 1], q.data_ptr(), 512, 0.125, 0, 0, o.data_ptr(), 512)
    c.append(*one, kv.data_ptr(), kv.data_ptr(), 128)
    torch.cuda.synchronize()
    assert (out == 3).all().item() and (o == 3).all().item() and (f == 3).all().item()
