"""Models in 8 bits: a pass is the public 8-bit operators one after the other, bit for bit; and it keeps what the other models' passes
promise (a row's bits depend on its sequence alone)."""
import numpy as np
import pytest

from workload import SHAPES, WeightStore, prompt_tokens

pytestmark = pytest.mark.gpu

NAMES = ["tiny_gqa_bf16", "tiny_gqa128_bf16", "tiny_g8_bf16", "tiny_wide_bf16"]


def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_17375_amd as A
    from paper_2410_17375_amd.harness import load_model
    return torch, A, load_model


def _model(name, max_ctx=256, **kw):
    torch, A, load_model = _gpu()
    shape = SHAPES[name]
    g = load_model(shape, max_ctx, int8=True, **kw)
    g.set_option(A.OPT_KEEP_LOGITS, 1)
    return A, shape, g


class Chain:
    """A decoder of the public operators."""

    def __init__(self, shape, max_ctx):
        self.torch, self.A, _ = _gpu()
        torch, A, s = self.torch, self.A, shape
        self.s, store = s, WeightStore(s)
        dev = lambda name, l=None: torch.from_numpy(store.bits(name, l).view(np.int16)).cuda().view(torch.bfloat16)   # noqa: E731
        cat = lambda l, *names: torch.cat([dev(n, l).reshape(-1, s.d_ffn if names == ("wd",) else s.q_dim if names == ("wo",) else s.d_model) for n in names])   # noqa: E731

        def mat(w, gated=False):
            torch.cuda.synchronize()
            return A.Q8Matrix(w.data_ptr(), A.DTYPE_BF16, w.shape[0], w.shape[1], gated=gated, on_device=True)
        self.layers = [(mat(cat(l, "wq", "wk", "wv")), mat(cat(l, "wo")), mat(cat(l, "wg", "wu"), True), mat(cat(l, "wd")),
                        dev("norm_attn", l).float().reshape(-1), dev("norm_mlp", l).float().reshape(-1)) for l in range(s.n_layers)]
        self.lm, self.embed, self.final = mat(dev("lm_head").reshape(s.vocab, s.d_model)), dev("embed").reshape(s.vocab, s.d_model), dev("final_norm").float().reshape(-1)
        self.cache = A.Q8Cache(n_layers=s.n_layers, n_seqs=1, n_q_heads=s.n_q_heads, n_kv_heads=s.n_kv_heads, head_dim=s.head_dim, capacity=max_ctx)
        inv = np.float64(np.float32(s.rope_theta)) ** (-2.0 * np.arange(s.head_dim // 2) / s.head_dim)
        ang = np.arange(max_ctx)[:, None] * inv
        self.cos, self.sin = (torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin))

    def __call__(self, tokens, pos0):
        torch, A, s = self.torch, self.A, self.s
        n, d, F, qd, kvd, hd = len(tokens), s.d_model, s.d_ffn, s.q_dim, s.kv_dim, s.head_dim
        nqkv = qd + 2 * kvd
        empty = lambda w, dt: torch.empty((n, w), dtype=dt, device="cuda")   # noqa: E731
        x, b16 = self.embed[torch.from_numpy(np.asarray(tokens, dtype=np.int64)).cuda()].float(), torch.bfloat16
        q, sc = empty(max(d, F, qd), torch.int8), torch.empty(n, device="cuda")
        qkv, att, delta, h, z = empty(nqkv, b16), empty(qd, b16), empty(d, b16), empty(F, b16), empty(s.vocab, torch.float32)
        p = lambda t: t.data_ptr()   # noqa: E731

        def norm(add, gain):
            A.q8_rmsnorm(p(x), A.DTYPE_FP32, d, p(delta) if add else 0, A.DTYPE_BF16, d, p(gain), s.rms_eps, n, d, p(x) if add else 0, d, p(q), d, p(sc))

        def rows(t, w):
            A.q8_quantize(p(t), A.DTYPE_BF16, w, n, w, p(q), w, p(sc))

        def product(m, k, out, w, dt=None):
            A.q8_gemm(m, p(q), k, p(sc), n, p(out), A.DTYPE_BF16 if dt is None else dt, w)
        tables = (p(self.cos), p(self.sin))
        for l, (wqkv, wo, wgu, wd, g_attn, g_mlp) in enumerate(self.layers):
            norm(l > 0, g_attn)
            product(wqkv, d, qkv, nqkv)
            self.cache.append(l, [0], [pos0], [n], p(qkv) + 2 * qd, p(qkv) + 2 * (qd + kvd), nqkv, *tables)
            self.cache.attention(l, [0], [pos0], [n], p(qkv), nqkv, float(1 / np.sqrt(np.float32(hd))), *tables, p(att), qd)
            rows(att, qd)
            product(wo, qd, delta, d)
            norm(True, g_mlp)
            product(wgu, d, h, F)
            rows(h, F)
            product(wd, F, delta, d)
        norm(True, self.final)
        product(self.lm, d, z, s.vocab, A.DTYPE_FP32)
        torch.cuda.synchronize()
        return z.cpu().numpy()


@pytest.mark.parametrize("name", NAMES)
def test_a_pass_is_the_operators_one_after_the_other(name):
    A, shape, g = _model(name)
    chain = Chain(shape, 256)
    toks = prompt_tokens(3, 100, shape.vocab)
    g.prefill(toks[:16])
    assert np.array_equal(g.get_logits(16), chain(toks[:16], 0))
    g.prefill(toks[16:90])                          # 74 rows: a prompt's pass
    z = chain(toks[16:90], 16)
    rows = (74 - 1) % 16 + 1
    assert np.array_equal(g.get_logits(rows), z[-rows:])
    assert np.array_equal(g.get_greedy(rows), z[-rows:].argmax(1))
    g.set_next(int(toks[90]))
    g.verify(90, toks[90:97])
    z = chain(toks[90:97], 90)
    assert np.array_equal(g.get_logits(7), z)
    for l in range(shape.n_layers):
        kk, vv = (chain.torch.empty((97, shape.n_kv_heads, shape.head_dim), device="cuda") for _ in range(2))
        chain.cache.read(l, [0], [0], [97], kk.data_ptr(), vv.data_ptr(), A.DTYPE_FP32, shape.kv_dim)
        for which, t in ((0, kk), (1, vv)):
            assert np.array_equal(g.get_kv(l, which, 0, 97), t.cpu().numpy().transpose(1, 0, 2))


@pytest.mark.parametrize("name", NAMES)
def test_rows_keep_their_bits(name):
    """A prompt at once, in pieces, token by token, in verify passes without the prefill workspace; a window after a rollback."""
    A, shape, g = _model(name)
    toks = prompt_tokens(5, 150, shape.vocab)
    logits = {}
    for cuts in ([0, 150], [0, 1, 40, 149, 150], [0, 100, 133, 150], list(range(0, 151))):
        g.kv_rollback(0)
        for lo, hi in zip(cuts, cuts[1:]):
            g.prefill(toks[lo:hi])
        logits[len(cuts)] = (g.get_logits(1) if cuts[-1] - cuts[-2] == 1 else g.get_logits((cuts[-1] - cuts[-2] - 1) % 16 + 1)[-1:], g.get_kv(1, 0, 0, 150), g.get_kv(1, 1, 0, 150))
    first = logits.pop(2)
    for other in logits.values():
        assert all(np.array_equal(a, b) for a, b in zip(first, other))
    g.set_option(A.OPT_PREFILL_WORKSPACE, 0)
    assert g.prefill_workspace_bytes() == 0
    g.kv_rollback(0)
    g.prefill(toks)
    assert np.array_equal(g.get_kv(1, 1, 0, 150), first[2])
    # a window behind a rollback, against its rows one at a time
    g.kv_rollback(100)
    g.set_next(int(toks[100]))
    g.verify(100, toks[100:113])
    window = g.get_logits(13)
    g.kv_rollback(100)
    for j in range(13):
        g.set_next(int(toks[100 + j]))
        g.draft_step()
        assert np.array_equal(g.get_logits(1)[0], window[j])
    g.kv_rollback(100)
    g.set_next(int(toks[100]))
    assert g.verify_static(100, toks[100:113]) is not None
    assert np.array_equal(g.get_logits(13), window)


def test_sequences_that_share_a_pass():
    A, shape, g = _model("tiny_gqa_bf16", max_seqs=5)
    toks = [prompt_tokens(10 + i, 60 + 13 * i, shape.vocab) for i in range(5)]
    alone = {}
    for i, t in enumerate(toks):
        g.seq_prefill(i, t[:-4])
    for i, t in enumerate(toks):
        g.seq_set_next(i, int(t[-4]))
        g.verify_batch([i], [len(t) - 4], [t[-4:-1 - i % 3]])
        alone[i] = g.get_logits(len(t[-4:-1 - i % 3]))
        g.seq_rollback(i, len(t) - 4)
        g.seq_set_next(i, int(t[-4]))
    order = [3, 0, 4, 1, 2]
    windows = [toks[i][-4:-1 - i % 3] for i in order]
    g.verify_batch(order, [len(toks[i]) - 4 for i in order], windows)
    z, at = g.get_logits(sum(len(w) for w in windows)), 0
    for i, w in zip(order, windows):
        assert np.array_equal(z[at:at + len(w)], alone[i])
        at += len(w)


def test_loops_give_the_greedy_sequence():
    """An 8-bit draft of a bf16 model, and an 8-bit model verified by itself: both loops reproduce plain greedy decoding."""
    torch, A, load_model = _gpu()
    shape = SHAPES["tiny_gqa_bf16"]
    streams = [torch.cuda.Stream() for _ in range(3)]
    big = load_model(shape, 256, stream=streams[0].cuda_stream)
    small = load_model(shape, 256, stream=streams[1].cuda_stream, int8=True)
    twin = load_model(shape, 256, stream=streams[2].cuda_stream, int8=True)
    prompt = prompt_tokens(1, 30, shape.vocab)
    want, _ = A.generate_greedy(big, prompt, 60)
    for loop in (A.generate_sync, A.generate_async):
        got, stats = loop(small, big, prompt, 60, 6)
        assert np.array_equal(got, want)
        assert stats["accepted_total"] > 0
    own, _ = A.generate_greedy(small, prompt, 60)
    for loop in (A.generate_sync, A.generate_async):
        assert np.array_equal(loop(twin, small, prompt, 60, 6)[0], own)


def test_what_an_8_bit_model_reports():
    torch, A, load_model = _gpu()
    s = SHAPES["tiny_gqa_bf16"]
    full, small = load_model(s, 128), load_model(s, 128, int8=True)
    features = s.n_layers * (s.q_dim + 2 * s.kv_dim + 2 * s.d_model + 2 * s.d_ffn) + s.vocab
    gains = (2 * s.n_layers + 1) * s.d_model * 2
    assert small.weight_bytes_per_pass() == (full.weight_bytes_per_pass() - gains) // 2 + 4 * features + gains
    assert small.kv_bytes_per_pass(100, 4) == s.n_layers * 2 * s.n_kv_heads * (s.head_dim + 4) * 104
    toks = prompt_tokens(2, 20, s.vocab)
    for stage, launches in (("embed", 1), ("qkv", s.n_layers), ("attention", s.n_layers), ("attn_merge", 0), ("gateup", s.n_layers), ("lmhead", 1), ("accept", 1)):
        small.kv_rollback(0)
        small.set_option(A.OPT_TIME_STAGE, A.STAGES[stage])
        small.prefill(toks[:16])
        ms, n, nbytes = small.stage_time()
        assert n == launches and (ms > 0) == (launches > 0)
        if stage == "gateup":
            assert nbytes == 2 * s.d_ffn * (s.d_model + 4)
    small.set_option(A.OPT_TIME_STAGE, -1)
    # arguments are checked as for the other models, and change nothing
    for call, code in ((lambda: small.verify(17, toks[:2]), -2), (lambda: small.prefill(prompt_tokens(0, 200, s.vocab)), -3),
                       (lambda: small.verify(3, [s.vocab]), -4), (lambda: small.get_kv(0, 0, 120, 9), -1)):
        with pytest.raises(A.AmusdError) as e:
            call()
        assert e.value.code == code
    assert small.kv_len() == 16


def test_prefill_workspace_declined_and_taken_again():
    """The prefill workspace of an 8-bit model can be declined, returned and taken again, and prompts keep their bits."""
    A, shape, g = _model("tiny_gqa_bf16")
    toks = prompt_tokens(9, 70, shape.vocab)
    g.prefill(toks)
    want = g.get_logits(6)
    assert g.prefill_workspace_bytes() > 0
    g.set_option(A.OPT_PREFILL_WORKSPACE, 0)
    g.kv_rollback(0)
    g.prefill(toks)
    assert np.array_equal(g.get_logits(6), want)
    g.set_option(A.OPT_PREFILL_WORKSPACE, 1)
    assert g.prefill_workspace_bytes() > 0
    g.kv_rollback(0)
    g.prefill(toks)
    assert np.array_equal(g.get_logits(6), want)


def test_weights_have_to_be_bf16_and_complete():
    torch, A, load_model = _gpu()
    with pytest.raises(ValueError):
        load_model(SHAPES["tiny_verify"], 64, int8=True)
    m = A.Model(n_layers=1, d_model=64, n_q_heads=2, n_kv_heads=1, head_dim=64, d_ffn=128, vocab=64, max_ctx=8, dtype=A.DTYPE_INT8)
    with pytest.raises(A.AmusdError) as e:
        m.finalize()
    assert e.value.code == -5
    m.free()
