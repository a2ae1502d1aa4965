"""The 8-bit operators at the ends of the number range: scales that are subnormal, values and keys near the largest float32, queries near
the smallest.  Tolerances are counted in roundings as in test_gpu_q8.py."""
import numpy as np
import pytest

from oracle import q8 as O
from test_gpu_q8 import U16, U32, _append, _attend, _check_q8, _np, _product, _rand, _read, _strided, _tolerance, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _rows_of(rng, most, n):
    """A row for each magnitude: random values up to it, and the magnitude itself."""
    a = rng.uniform(-1, 1, (len(most), n))
    a[:, ::7] *= 2.0 ** -5
    a[:, n // 2] = np.where(np.arange(len(most)) % 2, -1, 1)
    return (a * np.asarray(most, dtype=np.float64)[:, None]).astype(np.float32)


# magnitudes around those whose scale (a 127th) has no finite reciprocal in float32 (below 3.7e-37), and around subnormal ones
SMALL = [4e-37, 3.8e-37, 3.6e-37, 3e-37, 1e-37, 1.2e-38, 1e-38, 3e-39, 1e-40, 3e-41]


# ---------------------------------------------------------------- scales without a reciprocal
@pytest.mark.parametrize("n", [50, 2055, 20001])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize_small_rows(gpu, n, dtype):
    torch, A = gpu
    x = torch.from_numpy(_rows_of(np.random.default_rng(n), SMALL, n)).to(getattr(torch, dtype)).cuda()
    ld = -(-n // 16) * 16
    q, s = torch.empty((len(SMALL), ld), dtype=torch.int8, device="cuda"), torch.empty(len(SMALL), device="cuda")
    A.q8_quantize(x.data_ptr(), A.DTYPE_FP32 if dtype == "float32" else A.DTYPE_BF16, n, len(SMALL), n, q.data_ptr(), ld, s.data_ptr())
    want, scale, _ = O.quantize(_np(x))
    assert np.array_equal(_np(s), scale)
    assert np.array_equal(_np(q)[:, :n], want)
    live = _np(x).any(1)                                  # (3e-41 is below half of bf16's smallest: a row of zeros)
    assert live[:-1].all() and (np.abs(_np(q)[live, :n]).max(1) == 127).all()


@pytest.mark.parametrize("n", [96, 1030, 17000])
def test_rmsnorm_small_gains(gpu, n):
    torch, A = gpu
    rng = np.random.default_rng(n)
    x = torch.from_numpy(rng.standard_normal((3, n)).astype(np.float32)).cuda()
    for size in (2e-37, 1e-38):
        gain = torch.from_numpy(((1 + 0.1 * rng.standard_normal(n)) * size / 4).astype(np.float32)).cuda()
        ld = -(-n // 16) * 16
        q, s = torch.empty((3, ld), dtype=torch.int8, device="cuda"), torch.empty(3, device="cuda")
        A.q8_rmsnorm(x.data_ptr(), 0, n, 0, 0, 0, gain.data_ptr(), 1e-5, 3, n, 0, 0, q.data_ptr(), ld, s.data_ptr())
        y = O.rmsnorm(_np(x), None, _np(gain), float(np.float32(1e-5)))[1]
        _check_q8(_np(q)[:, :n].astype(np.int64), _np(s), y, (n + 8) * 2.0 ** -53)
        assert (np.abs(_np(q)[:, :n]).max(1) == 127).all()


@pytest.mark.parametrize("block", [1, 32])
@pytest.mark.parametrize("hd", [64, 128])
def test_append_small_rows(gpu, block, hd):
    """Pieces that grow from magnitudes whose scale has no reciprocal; blocks that hold them are rounded again."""
    torch, A = gpu
    cache = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=2, n_kv_heads=2, head_dim=hd, capacity=256, block=block)
    ref = [O.Cache(2, hd, 256, block) for _ in range(2)]
    rng, at = np.random.default_rng(hd), 0
    for n, size in ((5, 1e-39), (9, 5e-38), (40, 1e-37), (30, 3e-37), (64, 2e-37), (3, 1e-36), (20, 1.0)):
        k, v = (torch.from_numpy(_rows_of(rng, [size] * (n * 2), hd).reshape(n, 2, hd)).to(torch.bfloat16).cuda() for _ in range(2))
        _append(gpu, cache, [0], [at], [k], [v])
        ref[0].append(at, _np(k))
        ref[1].append(at, _np(v))
        at += n
    for got, want in zip(_read(gpu, cache, 0, 0, at, 2, hd), ref):
        assert np.array_equal(got, want.values(at).astype(np.float32))
        assert got[:5].any() and got[54:84].any()


# ---------------------------------------------------------------- scales of a few units of the smallest number: quotients past 127
UNIT = 2.0 ** -149
FEW = [64 * UNIT, 100 * UNIT, 143 * UNIT, 190 * UNIT, 191 * UNIT, 260 * UNIT, 317 * UNIT, 1000 * UNIT, 3.3e-42, 2e-41]


def test_quotients_past_127(gpu):
    torch, A = gpu
    n = 70
    rows = _rows_of(np.random.default_rng(1), FEW, n)
    assert (np.abs(rows[3] / (np.abs(rows[3]).max() / np.float32(127))) > 128).any()
    x = torch.from_numpy(rows).cuda()
    q, s = torch.empty((len(FEW), 80), dtype=torch.int8, device="cuda"), torch.empty(len(FEW), device="cuda")
    A.q8_quantize(x.data_ptr(), A.DTYPE_FP32, n, len(FEW), n, q.data_ptr(), 80, s.data_ptr())
    want, scale, _ = O.quantize(rows)
    assert np.array_equal(_np(s), scale)
    assert np.array_equal(_np(q)[:, :n], want)
    # a matrix's rows, read off through unit vectors
    for w in (rows, _rows_of(np.random.default_rng(2), SMALL, n)):
        m = A.Q8Matrix(w, A.DTYPE_FP32, len(w), n)
        got = _np(_product(gpu, m, np.eye(n, dtype=np.int8), np.ones(n, np.float32), len(w), torch.float32)).T
        want, scale, _ = O.quantize(w)
        assert np.array_equal(got, (want * scale[:, None].astype(np.float64)).astype(np.float32))


@pytest.mark.parametrize("block", [1, 16])
def test_quotients_past_127_in_the_cache(gpu, block):
    """Rotary turns keys to magnitudes that bf16 itself does not have: a few units of the smallest float32."""
    torch, A = gpu
    hd, n = 64, 40
    cache = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=2, n_kv_heads=2, head_dim=hd, capacity=64, block=block)
    rng = np.random.default_rng(5)
    k = torch.from_numpy(_rows_of(rng, [1.0] * (n * 2), hd).reshape(n, 2, hd)).to(torch.bfloat16).cuda()
    size = np.asarray(FEW * 4, dtype=np.float32)[:, None]
    if block > 1:
        size[:] = 190 * UNIT
    cos, sin = torch.from_numpy(np.repeat(size, hd // 2, 1)).cuda(), torch.zeros((n, hd // 2), device="cuda")
    _append(gpu, cache, [0], [0], [k], [k], rope=(cos.data_ptr(), sin.data_ptr()))
    ref = O.Cache(2, hd, 64, block)
    ref.append(0, _np(k) * np.repeat(size, 1, 1)[:, :, None])
    kk, _ = _read(gpu, cache, 0, 0, n, 2, hd)
    assert np.array_equal(kk, ref.values(n).astype(np.float32))


# ---------------------------------------------------------------- attention
def _filled(gpu, heads, n, k_std, v_std, seed=0, block=1, cap=None, k_edit=None, v_edit=None):
    torch, A = gpu
    hq, hkv, hd = heads
    rng = np.random.default_rng([seed, hd, n])
    k, v = (np.clip(rng.standard_normal((n, hkv, hd)) * std, -3.3e38, 3.3e38).astype(np.float32) for std in (k_std, v_std))
    for a, edit in ((k, k_edit), (v, v_edit)):
        if edit:
            edit(a)
    cache = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, capacity=cap or n, block=block)
    bf = lambda a: torch.from_numpy(a).to(torch.bfloat16).cuda()   # noqa: E731
    _append(gpu, cache, [0], [0], [bf(k)], [bf(v)])
    return cache, rng


def _held(gpu, cache, heads, n):
    return (a.astype(np.float64) for a in _read(gpu, cache, 0, 0, n, heads[1], heads[2]))


def _check_seen(gpu, cache, heads, q, pos0, scale, parts=True):
    """All rows against float64, and a few of them in calls of their own: the same bits, whichever form takes them."""
    torch, A = gpu
    n = q.shape[0]
    out, = _attend(gpu, cache, [0], [pos0], [q], scale)
    k, v = _held(gpu, cache, heads, pos0 + n)
    for lo in range(0, n, 64):
        hi = min(n, lo + 64)
        qn = _np(q)[lo:hi].astype(np.float64)
        want, weighted, s = O.attention(qn, k, v, pos0 + lo, scale)
        # (without the absolute 1e-30 of ordinary sizes; half a step of the smallest bf16 instead, which is four of float32's)
        tol = _tolerance(qn, k, v, pos0 + lo, scale, want, weighted, s, False) - 1e-30 + 1.01 * 2.0 ** -134
        err = np.abs(_np(out)[lo:hi].astype(np.float64) - want)
        assert (err <= tol).all(), (lo, float((err / tol).max()))
    if parts:
        for lo, m in ((0, 1), (n - 1, 1), (n // 3, min(5, n - n // 3))):
            part, = _attend(gpu, cache, [0], [pos0 + lo], [q[lo:lo + m]], scale)
            assert torch.equal(part, out[lo:lo + m]), (lo, m)


SHAPES = [((4, 2, 64), 300, 10, 1), ((8, 2, 128), 300, 4, 1), ((8, 2, 64), 600, 600, 1), ((8, 2, 128), 500, 500, 1), ((8, 1, 64), 400, 9, 32), ((8, 8, 128), 330, 330, 64),
          ((4, 1, 64), 4500, 3, 1)]


@pytest.mark.parametrize("heads,n,rows,block", SHAPES)
@pytest.mark.parametrize("size", [1e31, 1e34, 1e35, 1e37, 3e38])
def test_attention_of_large_values(gpu, heads, n, rows, block, size):
    """3e38: of one sign as well, where the weighted sum before the division is past float32."""
    torch, A = gpu

    def edit(v):
        if size == 3e38:
            v[:] = np.abs(v)
            v[..., ::5] = size
        v[n // 2:n // 2 + 3] = 0
    cache, rng = _filled(gpu, heads, n, 1.0, size / (8 if size == 3e38 else 1), block=block, v_edit=edit)
    _check_seen(gpu, cache, heads, _rand(torch, rng, rows, heads[0], heads[2]), n - rows, heads[2] ** -0.5)


@pytest.mark.parametrize("heads,n,rows,block", SHAPES)
@pytest.mark.parametrize("first", [True, False])
def test_attention_of_large_values_in_some_chunks(gpu, heads, n, rows, block, first):
    """A stretch of large values behind, or in front of, ordinary ones."""
    torch, A = gpu

    def edit(v):
        v[:n // 2 if first else n] *= 1e30
        if not first:
            v[:n // 2] *= 1e-30
        v *= 1e6
    cache, rng = _filled(gpu, heads, n, 1.0, 1.0, seed=1, block=block, v_edit=edit)
    _check_seen(gpu, cache, heads, _rand(torch, rng, rows, heads[0], heads[2]), n - rows, heads[2] ** -0.5)


@pytest.mark.parametrize("heads,n,rows,block", SHAPES)
@pytest.mark.parametrize("size", [1e-28, 1e-33, 1e-36, 2e-38])
def test_attention_of_small_values(gpu, heads, n, rows, block, size):
    torch, A = gpu
    cache, rng = _filled(gpu, heads, n, 1.0, size, seed=2, block=block)
    _check_seen(gpu, cache, heads, _rand(torch, rng, rows, heads[0], heads[2]), n - rows, heads[2] ** -0.5)


def test_attention_large_values_behind_a_row_change_nothing(gpu):
    """What a row does not see moves neither its power of two nor its sums' scale, however large."""
    torch, A = gpu
    heads = (8, 2, 64)
    for n, rows in ((40, 3), (220, 200)):
        cache, rng = _filled(gpu, heads, n, 1.0, 1.0, seed=3, cap=512)
        q = _rand(torch, rng, rows, 8, 64)
        clean, = _attend(gpu, cache, [0], [n - rows], [q], 0.125)
        bad = torch.full((100, 2, 64), 3e38, dtype=torch.bfloat16, device="cuda")
        _append(gpu, cache, [0], [n], [bad], [bad])
        again, = _attend(gpu, cache, [0], [n - rows], [q], 0.125)
        assert torch.equal(clean, again)


@pytest.mark.parametrize("heads,n,rows,block", SHAPES)
@pytest.mark.parametrize("qs,ks", [(1e-30, 1e30), (1e-32, 1e32), (1e-33, 1e34), (1e33, 1e-33), (1e36, 1e-37)])
def test_attention_of_large_keys(gpu, heads, n, rows, block, qs, ks):
    """Scores of ordinary size whose factors are not."""
    torch, A = gpu
    cache, rng = _filled(gpu, heads, n, ks, 1.0, seed=4, block=block)
    _check_seen(gpu, cache, heads, _rand(torch, rng, rows, heads[0], heads[2], std=qs), n - rows, heads[2] ** -0.5)


# ---------------------------------------------------------------- small queries
@pytest.mark.parametrize("heads,n,rows,block", SHAPES)
@pytest.mark.parametrize("qs,ks", [(1e-34, 1e34), (1e-36, 1e37), (1e-37, 1e36), (1e-38, 1e38)])
def test_attention_of_small_queries(gpu, heads, n, rows, block, qs, ks):
    """Queries whose 16 bits have no finite reciprocal in float32, against keys that give scores of ordinary size."""
    torch, A = gpu
    cache, rng = _filled(gpu, heads, n, ks, 1.0, seed=4, block=block)
    _check_seen(gpu, cache, heads, _rand(torch, rng, rows, heads[0], heads[2], std=qs), n - rows, heads[2] ** -0.5)


# ---------------------------------------------------------------- large scores
@pytest.mark.parametrize("heads,n,rows,block", SHAPES)
@pytest.mark.parametrize("size", [300.0, 3e3, 1e4, 1e5, 1e8, 1e13, 1e17])
def test_attention_of_large_scores(gpu, heads, n, rows, block, size):
    """Scores up to float32's range, of either sign: a row whose largest is far above the others has its value."""
    torch, A = gpu
    hq, hkv, hd = heads
    for sign in (0, -1):
        def edit(k):
            if sign:
                k[:] = -np.abs(k) - size

        cache, rng = _filled(gpu, heads, n, size, 1.0, seed=6, block=block, k_edit=edit)
        q = _rand(torch, rng, rows, hq, hd, std=size)
        q = torch.abs(q) if sign else q
        out, = _attend(gpu, cache, [0], [n - rows], [q], hd ** -0.5)
        k, v = _held(gpu, cache, heads, n)
        qn = _np(q).astype(np.float64)
        want, _, s = O.attention(qn, k, v, n - rows, hd ** -0.5)
        # a score is off by the query's 16 bits and five roundings of float32 at most, of the sum of its terms' magnitudes
        off = hd ** -0.5 * np.repeat(np.abs(k).sum(-1), hq // hkv, 1).T[None] * np.abs(qn).max(-1)[:, :, None] * (0.5 / 32512 + 7 * U32)
        off = np.where(np.isfinite(s), off, 0).max(-1)
        two = np.sort(s, -1)[..., -2:]                                       # (one row may see a single key: -inf below it)
        clear = two[..., 1] - two[..., 0] > 2 * off + 30
        assert clear.mean() > 0.5
        err = np.abs(_np(out).astype(np.float64) - want)[clear]
        # one weight; the others' are below e^-30.  Its value's half step in bf16; the weight times its value's scale to half (2^-11), where the
        # denominator has the weight as it is; and the sums' with 1152 + v
        assert (err <= ((U16 + 1.01 * 2.0 ** -11) * np.abs(want) + (8 * U32 * 1280 / 127 + n * np.exp(-30.0)) * np.abs(v).max())[clear]).all()
        for lo, m in ((0, 1), (rows - 1, 1), (rows // 3, min(5, rows - rows // 3))):
            part, = _attend(gpu, cache, [0], [n - rows + lo], [q[lo:lo + m]], hd ** -0.5)
            assert torch.equal(part, out[lo:lo + m]), (lo, m)


@pytest.mark.parametrize("heads,n,rows", [((4, 2, 64), 300, 10), ((8, 2, 128), 500, 500)])
def test_attention_of_a_far_largest_score(gpu, heads, n, rows):
    """Scores near 1e36: finite, and so far apart that the largest has all the weight."""
    torch, A = gpu
    hq, hkv, hd = heads

    def edit(k):
        k[3] = 1e36                                   # every row sees it
    cache, rng = _filled(gpu, heads, n, 1.0, 1.0, seed=5, k_edit=edit)
    q = torch.abs(_rand(torch, rng, rows, hq, hd)) + 0.5
    if rows == n:
        q[:3] = 0
    out, = _attend(gpu, cache, [0], [n - rows], [q], hd ** -0.5)
    _, v = _held(gpu, cache, heads, n)
    want = np.repeat(v[3], hq // hkv, 0)
    got = _np(out)[3 if rows == n else 0:].astype(np.float64)
    # one weight: its value's half step in bf16; the weight times its value's scale to half (2^-11), where the denominator has the weight as
    # it is; and the step that the chain of fp32 sums with 1152 + v leaves
    assert (np.abs(got - want) <= (U16 + 1.01 * 2.0 ** -11) * np.abs(want) + 4 * U32 * 1280 / 127 * np.abs(v).max()).all()


# ---------------------------------------------------------------- products of rows with large scales
@pytest.mark.parametrize("rows,n,k", [(1, 100, 600), (8, 512, 4096), (40, 300, 1000), (200, 512, 2048), (600, 1040, 640)])
@pytest.mark.parametrize("gated", [False, True])
def test_gemm_of_large_row_scales(gpu, rows, n, k, gated):
    """The sum times the row's scale is past float32, the result is not: rows of magnitudes around 1e34, weights around 1e-4."""
    torch, A = gpu
    rng = np.random.default_rng([rows, n, k])
    w = rng.integers(-127, 128, (n, k)).astype(np.int8)
    w[:, 0] = 127
    sw = ((rng.random(n) + 0.5) * 1e-6).astype(np.float32)
    if gated:
        sw[n // 2:] *= np.float32(1e-28)                      # (both halves are large otherwise)
    x = rng.integers(100, 128, (rows, k)).astype(np.int8)
    x[:, 1::2] *= -1
    sx = (2.0 ** rng.uniform(60, 121, rows)).astype(np.float32)
    sx[0] = 2.0 ** 115
    sx[1::3] = (rng.random(len(sx[1::3])) + 0.5) * 0.01      # ordinary ones beside them
    m = A.Q8Matrix(w, A.DTYPE_INT8, n, k, scale=sw, gated=gated)
    y = O.gemm(x, sx, w, sw)
    got = _np(_product(gpu, m, x, sx, n // 2 if gated else n, torch.float32))
    if not gated:
        fine = np.abs(y) < 3.3e38
        assert (np.abs(got - y) <= 3.01 * U32 * np.abs(y))[fine].all()
        assert fine.mean() > 0.9 and (np.abs(y) > 1e30).any()
        alone = _np(_product(gpu, m, x, sx, n, torch.float32, work=False))
        assert np.array_equal(got, alone)
        for r in (0, rows - 1):
            assert np.array_equal(_np(_product(gpu, m, x[r:r + 1], sx[r:r + 1], n, torch.float32))[0], got[r])
        return
    gate = y[:, :n // 2]
    with np.errstate(over="ignore"):
        want = np.where(gate < -700, 0, O.swiglu(y))
    # beyond a score of units silu is the gate itself or 0; errors as in test_gpu_q8.py, where the exponential's are within a unit's range
    sure = (np.abs(want) < 3.3e38) & ((gate > 100) | (gate < -200))
    assert sure.any()
    assert (np.abs(got - want) <= 9 * U32 * np.abs(want) + 1e-37)[sure].all()


@pytest.mark.parametrize("rows", [1, 70])
def test_attention_of_large_scores_a_step_apart(gpu, rows):
    """Scores of about 2^26.5 (in units of log2) that grow from one step of 64 keys to the next by the distance of neighbouring float32 numbers, 8 there:
    more than a reference may be exceeded by, less than half a step of the sum of the two."""
    torch, A = gpu
    hd, n = 64, 512 + rows
    for first in range(3):
        k = np.zeros((n, 8, hd), np.float32)
        k[..., :16] = 254                                     # 127 steps of 2
        k[..., 16] = 2 * np.minimum(np.arange(n) // 64 + first, 126)[:, None]
        v = np.random.default_rng(first).standard_normal((n, 8, hd)).astype(np.float32)
        q = np.zeros((rows, 8, hd), np.float32)
        q[..., :16], q[..., 16] = 131072, 16.125              # 32512 and 4 of the query's 16 bits
        cache = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=8, n_kv_heads=8, head_dim=hd, capacity=8192)     # chunks of 512
        bf = lambda a: torch.from_numpy(a).to(torch.bfloat16).cuda()   # noqa: E731
        _append(gpu, cache, [0], [0], [bf(k)], [bf(v)])
        out, = _attend(gpu, cache, [0], [n - rows], [bf(q)], 0.125)
        held = np.abs(_read(gpu, cache, 0, 0, n, 8, hd)[1]).max()
        assert (np.abs(_np(out)) <= held * (1 + 2.0 ** -7)).all()          # a mean of values: no NaN, none past the largest
