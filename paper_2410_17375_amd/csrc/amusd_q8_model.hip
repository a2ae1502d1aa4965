// Models in 8 bits: matrices and cache in 8 bits, a pass is the 8-bit operators one after the other.  Residual stream and
// logits are fp32, what goes from operator to operator bf16 or 8-bit rows.  Every operator gives a row the same bits whatever
// rows are beside it, so passes keep what the other models' promise: k rows at once are k passes of one row, and a prompt is the
// passes of its tokens.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "amusd_math.h"
#include "amusd_q8.h"

#pragma clang fp contract(off)

namespace amusd {

struct Q8Model {
    struct Layer {
        amusd_q8_matrix qkv, o, gu, down;
    };
    std::vector<Layer> layers;
    amusd_q8_matrix lm;
    amusd_q8_cache cache;
};

namespace {

// Rows of the embedding table as the residual stream.
struct Q8Tokens {
    int t[kRows];
    const int* many;       // pinned host memory, or null
};
__global__ void __launch_bounds__(256) k_q8_embed(float* __restrict__ X, const uint16_t* __restrict__ table, int d, Q8Tokens T) {
    const int row = blockIdx.x;
    const uint16_t* src = table + (size_t)(T.many ? T.many[row] : T.t[row & (kRows - 1)]) * d;
    for (int c = threadIdx.x * 8; c < d; c += 2048) {
        const uint4 v = *reinterpret_cast<const uint4*>(src + c);
        float* out = X + (size_t)row * d + c;
        *reinterpret_cast<v4f*>(out) = v4f{bf16_to_f32(v.x & 0xFFFF), bf16_to_f32(v.x >> 16), bf16_to_f32(v.y & 0xFFFF), bf16_to_f32(v.y >> 16)};
        *reinterpret_cast<v4f*>(out + 4) = v4f{bf16_to_f32(v.z & 0xFFFF), bf16_to_f32(v.z >> 16), bf16_to_f32(v.w & 0xFFFF), bf16_to_f32(v.w >> 16)};
    }
}

// The best of columns [c0, c1) of a row in every thread 0 (lowest column on ties; none among values that are not numbers).
__device__ __forceinline__ void row_best(const float* z, int c0, int c1, float& bv, int& bi) {
    __shared__ float vals[16];
    __shared__ int ids[16];
    bv = -INFINITY;
    bi = 0x7fffffff;
    for (int c = c0 + threadIdx.x * 4; c < c1; c += blockDim.x * 4) {
        const v4f v = *reinterpret_cast<const v4f*>(z + c);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (better(v[e], c + e, bv, bi)) { bv = v[e]; bi = c + e; }
    }
    keep_better_xor<32>(bv, bi);
    keep_better_xor<16>(bv, bi);
    keep_better_xor<8>(bv, bi);
    keep_better_xor<4>(bv, bi);
    keep_better_xor<2>(bv, bi);
    keep_better_xor<1>(bv, bi);
    if ((threadIdx.x & 63) == 0) {
        vals[threadIdx.x >> 6] = bv;
        ids[threadIdx.x >> 6] = bi;
    }
    __syncthreads();
    for (int w = 0; w < (int)blockDim.x >> 6; ++w)
        if (better(vals[w], ids[w], bv, bi)) { bv = vals[w]; bi = ids[w]; }
}

// (the vocabulary is a multiple of 16)
__global__ void __launch_bounds__(256) k_q8_argmax(const float* __restrict__ logits, int V, float* __restrict__ best_val, int* __restrict__ best_idx) {
    const int part = blockIdx.x, row = blockIdx.y;
    const int per = (V / 16 + kQ8LmParts - 1) / kQ8LmParts * 16;
    float bv;
    int bi;
    row_best(logits + (size_t)row * V, min(V, part * per), min(V, (part + 1) * per), bv, bi);
    if (threadIdx.x == 0) {
        best_val[part * kRows + row] = bv;
        best_idx[part * kRows + row] = bi;
    }
}
__global__ void __launch_bounds__(1024) k_q8_greedy(const float* __restrict__ logits, int V, int* __restrict__ greedy) {
    float bv;
    int bi;
    row_best(logits + (size_t)blockIdx.x * V, 0, V, bv, bi);
    if (threadIdx.x == 0) greedy[blockIdx.x] = bi;
}
__global__ void __launch_bounds__(256) k_q8_export(DevModel M, int bytes) { export_logits(M, bytes, blockIdx.x); }

struct Stage {                     // events around the launches of the stage that is timed
    StageTimer* tm;
    hipStream_t stream;
    template <class F>
    hipError_t operator()(int id, F f) const {
        const bool timed = tm && tm->stage == id;
        hipError_t e = hipSuccess;
        if (timed) e = hipEventRecord(tm->begin[tm->used], stream);
        if (e == hipSuccess) e = f();
        if (e == hipSuccess && timed) e = hipEventRecord(tm->end[tm->used++], stream);
        return e;
    }
};

#define TRY(expr)                            \
    do {                                     \
        const hipError_t e_ = (expr);        \
        if (e_ != hipSuccess) return e_;     \
    } while (0)

// Embedding and all layers; leaves the normalised last rows in B.q, B.s.
hipError_t layers_of(const Q8Model& Q, const DevModel& D, const DevLayer* Ls, const Q8Bufs& B, Q8Segs& S, const Q8Tokens& T, hipStream_t s, Stage stage) {
    const int n = S.rows, d = D.d, F = D.F, q = D.qdim;
    const float scale = 1.f / std::sqrt((float)D.hd);
    TRY(stage(AMUSD_STAGE_EMBED, [&] {
        hipLaunchKernelGGL(k_q8_embed, dim3(n), dim3(256), 0, s, B.X, static_cast<const uint16_t*>(D.embed), d, T);
        return hipGetLastError();
    }));
    auto norm = [&](bool add, const float* gain) {
        return launch_q8_rows(B.X, AMUSD_DTYPE_FP32, d, add ? B.delta : nullptr, AMUSD_DTYPE_BF16, d, gain, D.eps, n, d, add ? B.X : nullptr, d, B.q, d, B.s, s);
    };
    auto rows = [&](const uint16_t* x, int w) {
        return launch_q8_rows(x, AMUSD_DTYPE_BF16, w, nullptr, AMUSD_DTYPE_BF16, 0, nullptr, 0.f, n, w, nullptr, 0, B.q, w, B.s, s);
    };
    auto product = [&](const amusd_q8_matrix& w, uint16_t* out, int stage_id) {
        return stage(stage_id, [&] { return launch_q8_gemm(w, B.q, w.k, B.s, n, out, AMUSD_DTYPE_BF16, w.n, B.work, B.work_bytes, s); });
    };
    for (int l = 0; l < D.n_layers; ++l) {
        const Q8Model::Layer& W = Q.layers[l];
        TRY(norm(l > 0, Ls[l].g_attn));
        TRY(product(W.qkv, B.qkv, AMUSD_STAGE_QKV));
        q8_append_units(S);
        TRY(launch_q8_append(Q.cache, l, S, B.qkv + q, B.qkv + q + D.kvdim, D.nqkv, D.rope_cos, D.rope_sin, s));
        TRY(stage(AMUSD_STAGE_ATTENTION, [&] { return launch_q8_attention(Q.cache, l, S, B.qkv, D.nqkv, scale, D.rope_cos, D.rope_sin, B.att, q, s); }));
        TRY(rows(B.att, q));
        TRY(product(W.o, B.delta, AMUSD_STAGE_OPROJ));
        TRY(norm(true, Ls[l].g_mlp));
        TRY(product(W.gu, B.h, AMUSD_STAGE_GATEUP));
        TRY(rows(B.h, F));
        TRY(product(W.down, B.delta, AMUSD_STAGE_DOWN));
    }
    return norm(true, D.g_final);
}

}  // namespace

int q8_model_create(const DevModel& D, int, Q8Alloc alloc, hipStream_t stream, Q8Model** out) {
    Q8Model* q = new (std::nothrow) Q8Model();
    if (!q) return report(AMUSD_E_NOMEM, "8-bit model");
    hipError_t e = hipSuccess;
    try {
        q->layers.resize(D.n_layers);
    } catch (const std::bad_alloc&) {
        delete q;
        return report(AMUSD_E_NOMEM, "8-bit model");
    }
    auto take = [&](amusd_q8_matrix& m, int n, int k, bool gated) {
        if (e == hipSuccess) e = q8_matrix_take(m, n, k, gated, alloc, stream);
    };
    for (Q8Model::Layer& L : q->layers) {
        take(L.qkv, D.nqkv, D.d, false);
        take(L.o, D.d, D.qdim, false);
        take(L.gu, 2 * D.F, D.d, true);
        take(L.down, D.d, D.F, false);
    }
    take(q->lm, D.V, D.d, false);
    // A scale for every position: what a row sees then never depends on the rows behind it, and a cache that was rolled back and
    // extended again is the cache that was extended once.
    if (e == hipSuccess) e = q8_cache_take(q->cache, D.n_layers, D.n_slots, D.Hq, D.Hkv, D.hd, D.max_ctx, 1, alloc, stream);
    if (e != hipSuccess) {
        (void)hipGetLastError();          // reported here, not by the next launch
        q8_model_free(q);
        return report(AMUSD_E_HIP, "8-bit model", hipGetErrorString(e));
    }
    *out = q;
    return AMUSD_OK;
}

void q8_model_free(Q8Model* q) {
    if (!q) return;
    for (Q8Model::Layer& L : q->layers)
        for (amusd_q8_matrix* m : {&L.qkv, &L.o, &L.gu, &L.down}) q8_matrix_drop(*m);
    q8_matrix_drop(q->lm);
    q8_cache_drop(q->cache);
    delete q;
}

int q8_model_set(Q8Model* q, int id, int layer, const void* src, hipStream_t stream) {
    const int qdim = q->cache.Hq * q->cache.hd, kvdim = q->cache.Hkv * q->cache.hd;
    const bool global = id == AMUSD_T_LM_HEAD;
    amusd_q8_matrix* m = global ? &q->lm : nullptr;
    int rows = global ? q->lm.n : 0, first = 0, part = 0;
    if (!global) {
        Q8Model::Layer& L = q->layers[layer];
        switch (id) {
            case AMUSD_T_WQ: m = &L.qkv; rows = qdim; break;
            case AMUSD_T_WK: m = &L.qkv; rows = kvdim; first = qdim; break;
            case AMUSD_T_WV: m = &L.qkv; rows = kvdim; first = qdim + kvdim; break;
            case AMUSD_T_WO: m = &L.o; rows = L.o.n; break;
            case AMUSD_T_WG: m = &L.gu; rows = L.gu.n; part = 1; break;
            case AMUSD_T_WU: m = &L.gu; rows = L.gu.n; part = 2; break;
            case AMUSD_T_WD: m = &L.down; rows = L.down.n; break;
            default: return report(AMUSD_E_ARG, "unknown tensor id");
        }
    }
    hipError_t e = launch_q8_matrix(*m, src, AMUSD_DTYPE_BF16, m->k, nullptr, rows, first, part, stream);
    if (e == hipSuccess) e = hipStreamSynchronize(stream);
    return e == hipSuccess ? AMUSD_OK : report(AMUSD_E_HIP, "tensor to 8 bits", hipGetErrorString(e));
}

size_t q8_model_bufs(const Q8Model* q, const DevModel& D, int cap, uintptr_t base, Q8Bufs& B) {
    size_t off = 0;
    auto place = [&](size_t bytes) {
        void* p = reinterpret_cast<void*>(base + off);
        off += (bytes + 255) & ~(size_t)255;
        return p;
    };
    const size_t n = cap;
    B.cap = cap;
    B.X = static_cast<float*>(place(n * D.d * 4));
    B.q = static_cast<int8_t*>(place(n * std::max({D.d, D.qdim, D.F})));
    B.s = static_cast<float*>(place(n * 4));
    B.qkv = static_cast<uint16_t*>(place(n * D.nqkv * 2));
    B.att = static_cast<uint16_t*>(place(n * D.qdim * 2));
    B.delta = static_cast<uint16_t*>(place(n * D.d * 2));
    B.h = static_cast<uint16_t*>(place(n * D.F * 2));
    B.work_bytes = 0;
    for (const amusd_q8_matrix* m : {&q->layers[0].qkv, &q->layers[0].o, &q->layers[0].gu, &q->layers[0].down, &q->lm})
        B.work_bytes = std::max(B.work_bytes, q8_gemm_workspace(*m, cap));
    B.work = place(B.work_bytes);
    B.logits = static_cast<float*>(place(cap > kRows ? (size_t)std::min(cap, kQ8LmRows) * D.V * 4 : 0));
    return off;
}

hipError_t q8_model_pass(const Q8Model* Q, const DevModel& D, const DevLayer* Ls, const Q8Bufs& B, const PassArgs& P, hipStream_t s, StageTimer* tm) {
    if (tm) tm->used = 0;
    const Stage stage{tm, s};
    Q8Segs S{};
    S.n_seg = P.n_seg;
    S.rows = P.k;
    for (int i = 0; i < P.n_seg; ++i) {
        S.s[i] = Q8Seg{P.seg[i].slot, P.seg[i].L, P.seg[i].k, P.seg[i].row0, 0};
        S.max_len = std::max(S.max_len, P.seg[i].L + P.seg[i].k);
    }
    Q8Tokens T{};
    for (int i = 0; i < P.k; ++i) T.t[i] = P.tokens[i];
    TRY(layers_of(*Q, D, Ls, B, S, T, s, stage));
    TRY(stage(AMUSD_STAGE_LMHEAD, [&] { return launch_q8_gemm(Q->lm, B.q, D.d, B.s, P.k, D.logits, AMUSD_DTYPE_FP32, D.V, B.work, B.work_bytes, s); }));
    return stage(AMUSD_STAGE_ACCEPT, [&] {
        hipLaunchKernelGGL(k_q8_argmax, dim3(kQ8LmParts, P.k), dim3(256), 0, s, D.logits, D.V, D.best_val, D.best_idx);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? launch_accept(D, P, s) : e;
    });
}

hipError_t q8_model_prefill(const Q8Model* Q, const DevModel& D, const DevLayer* Ls, const Q8Bufs& B, const PrefillBufs& T, const PrefillArgs& P, int tail,
                            hipStream_t s) {
    Q8Segs S{};
    S.n_seg = 1;
    S.rows = P.n;
    S.s[0] = Q8Seg{P.slot, P.L0, P.n, 0, 0};
    S.max_len = P.L0 + P.n;
    Q8Tokens tokens{};
    tokens.many = T.tokens;
    TRY(layers_of(*Q, D, Ls, B, S, tokens, s, Stage{nullptr, s}));
    // The last `tail` rows' logits can be asked for; of the others only the arg-max is kept.
    for (int r = 0; r < P.n;) {
        const int rows = r < P.n - tail ? std::min(P.n - tail - r, kQ8LmRows) : tail;
        float* z = r < P.n - tail ? B.logits : D.logits;
        TRY(launch_q8_gemm(Q->lm, B.q + (size_t)r * D.d, D.d, B.s + r, rows, z, AMUSD_DTYPE_FP32, D.V, B.work, B.work_bytes, s));
        hipLaunchKernelGGL(k_q8_greedy, dim3(rows), dim3(1024), 0, s, z, D.V, T.greedy + r);
        TRY(hipGetLastError());
        r += rows;
    }
    if (P.export_bytes) {
        hipLaunchKernelGGL(k_q8_export, dim3(export_wgs(P.export_bytes, 256)), dim3(256), 0, s, D, P.export_bytes);
        TRY(hipGetLastError());
    }
    return hipSuccess;
}

hipError_t q8_model_read(const Q8Model* q, int layer, int seq, int pos0, int n, float* k, float* v, hipStream_t stream) {
    Q8Segs S{};
    S.n_seg = 1;
    S.rows = n;
    S.s[0] = Q8Seg{seq, pos0, n, 0, 0};
    return launch_q8_read(q->cache, layer, S, k, v, AMUSD_DTYPE_FP32, (int64_t)q->cache.Hkv * q->cache.hd, stream);
}

}  // namespace amusd
