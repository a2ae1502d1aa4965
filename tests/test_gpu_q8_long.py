"""The 8-bit cache and its attention at long capacities: the memory that it takes beside keys and values, and calls whose chunk sums go through that
memory a part at a time."""
import numpy as np
import pytest

from test_gpu_q8 import _attend, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _long_cache(gpu, heads, capacity, n_seqs, base, rows, block=1, seed=0):
    """Sequences with 300 early positions and `rows` behind `base`; what lies between are zeros."""
    torch, A = gpu
    hq, hkv, hd = heads
    cache = A.Q8Cache(n_layers=1, n_seqs=n_seqs, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, capacity=capacity, block=block)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)   # noqa: E731
    qs = []
    for i in range(n_seqs):
        for at, n in ((0, 300), (base - 50, 50 + rows)):
            k, v = normal(n, hkv * hd), normal(n, hkv * hd)
            cache.append(0, [i], [at], [n], k.data_ptr(), v.data_ptr(), hkv * hd)
        qs.append(normal(rows, hq, hd))
    torch.cuda.synchronize()
    return cache, qs


@pytest.mark.parametrize("n_seqs", [1, 3])
def test_memory_beside_keys_and_values(gpu, n_seqs):
    torch, A = gpu
    capacity, heads, hd = 1 << 17, 8, 128
    _long_cache(gpu, (4, 2, 64), 512, 1, 400, 3)[0].free()          # (the first calls of a process take memory for its programs)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    cache = A.Q8Cache(n_layers=1, n_seqs=n_seqs, n_q_heads=4 * heads, n_kv_heads=heads, head_dim=hd, capacity=capacity)
    taken = free - torch.cuda.mem_get_info()[0]
    cache.free()
    held = 2 * n_seqs * heads * capacity * (hd + 4)
    # Room for sums: 128 MB or a 32nd, or what 16 rows have.  Chunks of 512 keys, a tile's sums (hd + 2) * 16 floats each: 16 rows of 4 heads are 4 tiles, and a part of one more for each sequence
    sums = (64 + 15 * n_seqs) // 16 * heads * (capacity // 512) * (hd + 2) * 64
    assert held <= taken <= held + max(sums, 128 << 20, held // 32) + (16 << 20)


@pytest.mark.parametrize("heads,capacities", [((8, 2, 64), (700, 2048, 4096)), ((8, 2, 128), (4160, 8192)), ((4, 4, 64), (4352, 8192)), ((16, 8, 128), (4608, 70000))])
def test_capacities_with_one_chunk_give_one_result(gpu, heads, capacities):
    """Bits follow from the chunks, and these from the capacity times the kv heads (on 256 compute units: up to 8192, 16384, 32768, more)."""
    torch, A = gpu
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the capacities are those of 256 compute units")
    hq, hkv, hd = heads
    gen = torch.Generator(device="cuda").manual_seed(7)
    k, v = (torch.randn(690, hkv * hd, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(300, hq, hd, generator=gen, device="cuda").to(torch.bfloat16)
    got = []
    for capacity in capacities:
        cache = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, capacity=capacity)
        cache.append(0, [0], [0], [690], k.data_ptr(), v.data_ptr(), hkv * hd)
        got.append([_attend(gpu, cache, [0], [690 - n], [q[:n]], hd ** -0.5)[0] for n in (1, 9, 300)])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("heads,n_seqs,rows", [((32, 8, 128), 1, 80), ((8, 1, 64), 3, 90), ((16, 8, 64), 2, 65)])
def test_sums_a_part_at_a_time(gpu, heads, n_seqs, rows):
    """Rows whose sums do not fit the room together, against the same rows 7 at a time."""
    torch, A = gpu
    capacity, base = 1 << 17, (1 << 17) - 200
    cache, qs = _long_cache(gpu, heads, capacity, n_seqs, base, rows)
    whole = _attend(gpu, cache, list(range(n_seqs)), [base] * n_seqs, qs, heads[2] ** -0.5)
    for i, q in enumerate(qs):
        for lo in range(0, rows, 7):
            part, = _attend(gpu, cache, [i], [base + lo], [q[lo:lo + 7]], heads[2] ** -0.5)
            assert torch.equal(part, whole[i][lo:lo + 7]), (i, lo)


def test_rows_of_2_31_columns(gpu):
    """The longest rows that a call takes: positions behind the last one are past 31 bits."""
    torch, A = gpu
    n, part = 2 ** 31 - 1, 1 << 27
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, n, part):
        x[lo:lo + part] = torch.randn(min(part, n - lo), generator=gen, device="cuda")
    q = torch.full((n + 17,), 99, dtype=torch.int8, device="cuda")
    s = torch.empty(1, device="cuda")
    A.q8_quantize(x.data_ptr(), A.DTYPE_BF16, n, 1, n, q.data_ptr(), n + 1, s.data_ptr())
    torch.cuda.synchronize()
    most = max(x[lo:lo + part].abs().max().item() for lo in range(0, n, part))
    assert s.item() == np.float32(np.float64(most) / 127)
    for lo in range(0, n, part):
        assert torch.equal(q[lo:lo + part][:n - lo].float(), torch.round(x[lo:lo + part].float() / s)), lo
    assert (q[n:] == 99).all().item()
    gain = torch.ones(n, device="cuda")
    A.q8_rmsnorm(x.data_ptr(), A.DTYPE_BF16, n, 0, 0, 0, gain.data_ptr(), 0.0, 1, n, 0, 0, q.data_ptr(), n + 1, s.data_ptr())
    torch.cuda.synchronize()
    mean = sum((x[lo:lo + part].double() ** 2).sum().item() for lo in range(0, n, part)) / n
    # the element's rounding and the scale's, 2^-24 each, and 2^31 sums of 2^-53
    assert abs(s.item() / (most / mean ** 0.5 / 127) - 1) <= 2 * 2.0 ** -24 + 2 * 2.0 ** -22
    assert (q[n:] == 99).all().item()


def test_more_rows_than_a_launch_takes(gpu):
    """2^26 rows of a wave each are 2^32 threads."""
    torch, A = gpu
    rows = (1 << 26) + 37
    x = torch.arange(rows, dtype=torch.int32, device="cuda").remainder_(1013).float() - 500
    q, s = torch.full((rows, 16), 99, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    A.q8_quantize(x.data_ptr(), A.DTYPE_FP32, 1, rows, 1, q.data_ptr(), 16, s.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(q[:, 0].float(), 127 * torch.sign(x)) and (q[:, 1:] == 99).all().item()
    assert torch.equal(s, torch.abs(x) / torch.full_like(x, 127))
    gain = torch.ones(1, device="cuda")
    y = torch.empty(rows, device="cuda")
    A.q8_rmsnorm(x.data_ptr(), A.DTYPE_FP32, 1, x.data_ptr(), A.DTYPE_FP32, 1, gain.data_ptr(), 1e-5, rows, 1, y.data_ptr(), 1, q.data_ptr(), 16, s.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(y, 2 * x) and torch.equal(q[:, 0].float(), 127 * torch.sign(x))


def test_read_of_2_26_positions(gpu):
    """As many positions of several sequences at once as a launch of a workgroup for each four has no threads for."""
    torch, A = gpu
    capacity, seqs = 1 << 24, 5
    cache = A.Q8Cache(n_layers=1, n_seqs=seqs, n_q_heads=1, n_kv_heads=1, head_dim=64, capacity=capacity, block=64)
    gen = torch.Generator(device="cuda").manual_seed(9)
    n = (1 << 26) // seqs + 100
    for i in range(seqs):
        k, v = (torch.randn(100, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        cache.append(0, [i], [n - 100], [100], k.data_ptr(), v.data_ptr(), 64)
    back = [torch.full((seqs * n, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache.read(0, list(range(seqs)), [0] * seqs, [n] * seqs, back[0].data_ptr(), back[1].data_ptr(), A.DTYPE_BF16, 64)
    one = [torch.empty(100, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for i in range(seqs):
        cache.read(0, [i], [n - 100], [100], one[0].data_ptr(), one[1].data_ptr(), A.DTYPE_BF16, 64)
        for a, b in zip(back, one):
            assert b.any().item() and torch.equal(a[(i + 1) * n - 100:(i + 1) * n], b)
            assert not a[i * n:(i + 1) * n - 200].any().item()          # (its last block of zeros ends there)


@pytest.mark.parametrize("n,gated,dtype", [(1, False, "bfloat16"), (4, True, "bfloat16")])
def test_product_of_2_30_rows(gpu, n, gated, dtype):
    torch, A = gpu
    rows, k = (1 << 30) + 77, 16
    w = (np.arange(n * k).reshape(n, k) % 7 - 3).astype(np.int8)
    w[:, 0] = 5 + np.arange(n)
    m = A.Q8Matrix(w, A.DTYPE_INT8, n, k, scale=np.full(n, 0.5, np.float32), gated=gated)
    x = torch.zeros(rows, k, dtype=torch.int8, device="cuda")
    pattern = (torch.arange(1000, device="cuda") % 250 - 125).to(torch.int8)
    x[:, 0] = pattern.repeat(rows // 1000 + 1)[:rows]
    s = torch.ones(rows, device="cuda")
    cols = n // 2 if gated else n
    out, few = torch.full((rows, cols), 99.0, dtype=torch.bfloat16, device="cuda"), torch.empty(1000, cols, dtype=torch.bfloat16, device="cuda")
    A.q8_gemm(m, x.data_ptr(), k, s.data_ptr(), 1000, few.data_ptr(), A.DTYPE_BF16, cols)
    A.q8_gemm(m, x.data_ptr(), k, s.data_ptr(), rows, out.data_ptr(), A.DTYPE_BF16, cols)
    torch.cuda.synchronize()
    whole = rows // 1000 * 1000
    assert (out[:whole].view(-1, 1000, cols) == few).all().item() and torch.equal(out[whole:], few[:rows - whole])


def test_matrix_of_2_26_features(gpu):
    """A wave rounds a feature: more features than a launch has waves."""
    torch, A = gpu
    n = (1 << 26) + 53
    w = torch.arange(n, dtype=torch.int32, device="cuda").remainder_(1013).float() - 500
    torch.cuda.synchronize()
    m = A.Q8Matrix(w.data_ptr(), A.DTYPE_FP32, n, 1, on_device=True)
    x, s = torch.ones(1, 16, dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda")
    out = torch.empty(n, device="cuda")
    A.q8_gemm(m, x.data_ptr(), 16, s.data_ptr(), 1, out.data_ptr(), A.DTYPE_FP32, n)
    assert torch.equal(out, 127 * (torch.abs(w) / torch.full_like(w, 127)) * torch.sign(w))


@pytest.mark.parametrize("rows,n", [(2048, 10240), (2100, 10300), (4000, 6144), (1700, 14336), (700, 32000), (700, 32768), (700, 32769)])
def test_quantize_many_long_rows_as_few(gpu, rows, n):
    """bf16 rows are laid over threads otherwise where they are many and long: on either side of that, and of what registers hold."""
    torch, A = gpu
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(rows, n, generator=gen, device="cuda").to(torch.bfloat16)
    ld, got = -(-n // 16) * 16, []
    for step in (rows, 90):
        q, s = torch.zeros((rows, ld), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
        for r in range(0, rows, step):
            A.q8_quantize(x[r].data_ptr(), A.DTYPE_BF16, n, min(step, rows - r), n, q[r].data_ptr(), ld, s[r:].data_ptr())
        got.append((q, s))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert (got[0][0].abs().amax(1) == 127).all().item()


@pytest.mark.parametrize("hd,block", [(64, 1), (128, 64)])
def test_attention_at_the_last_of_2_24_positions(gpu, hd, block):
    """The longest cache: a window at its end, over zeros and a few keys there and at its beginning that outweigh them."""
    torch, A = gpu
    capacity, rows = 1 << 24, 3
    cache = A.Q8Cache(n_layers=1, n_seqs=1, n_q_heads=2, n_kv_heads=1, head_dim=hd, capacity=capacity, block=block)
    rng = np.random.default_rng(hd)
    bf = lambda a: torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16).cuda()   # noqa: E731
    held = []
    for at, n in ((0, 64), (capacity - 64, 64)):
        k, v = bf(rng.standard_normal((n, hd)) * 1.5), bf(rng.standard_normal((n, hd)))
        cache.append(0, [0], [at], [n], k.data_ptr(), v.data_ptr(), hd)
        kk, vv = (torch.empty(n, hd, device="cuda") for _ in range(2))
        cache.read(0, [0], [at], [n], kk.data_ptr(), vv.data_ptr(), A.DTYPE_FP32, hd)
        held.append((kk.cpu().numpy().astype(np.float64), vv.cpu().numpy().astype(np.float64)))
    q = bf(rng.standard_normal((rows, 2, hd)) * 12)
    out, = _attend(gpu, cache, [0], [capacity - rows], [q], hd ** -0.5)
    qn, got = q.float().cpu().numpy().astype(np.float64), out.float().cpu().numpy()
    for r in range(rows):
        k = np.concatenate([held[0][0], held[1][0][:64 - rows + r + 1]])
        v = np.concatenate([held[0][1], held[1][1][:64 - rows + r + 1]])
        s = qn[r] @ k.T * hd ** -0.5                                         # [2, keys]; all others are 0
        top = np.maximum(s.max(1, keepdims=True), 0)
        p = np.exp(s - top)
        den = p.sum(1, keepdims=True) + (capacity - rows + r + 1 - len(k)) * np.exp(-top)
        want, weighted = p @ v / den, p @ np.abs(v) / den
        assert np.abs(want).max() > 0.1
        # the scores' rounding (a query's 16 bits and seven of float32, twice), the weights' to half, 32768 chunks' sums one after the other
        off = hd ** -0.5 * np.abs(k).sum(1).max() * np.abs(qn[r]).max() * (0.5 / 32512 + 7 * 2.0 ** -24)
        assert off < 0.1
        tol = 2.0 ** -8 * np.abs(want) + weighted * (2.0 ** -11 + 2 * 1.1 * off + 2 * 33300 * 2.0 ** -24) + 520 * 2.0 ** -24 * 1280 / 127 * np.abs(v).max()
        assert (np.abs(got[r] - want) <= tol).all(), r
