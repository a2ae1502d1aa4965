// Rows to 8 bits, appending to and reading an 8-bit cache, and the C entry points of the 8-bit operators.
#include "amusd_q8.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <string>

#include "amusd_math.h"

#pragma clang fp contract(off)

namespace amusd {

// ---------------------------------------------------------------- rows to 8 bits
// A workgroup a row, the row in registers: it is read once and written once, so the bytes bound it (and its launch, where
// there are few rows).  Squares are summed and rows divided in 64 bits: a square of a large element stays finite, and an
// element is rounded to the wrong one of two neighbours only if it is nearer than 2^-50 to their middle.
// Loads and stores take any alignment (one instruction of 16 bytes all the same).
template <class T>
__device__ __forceinline__ void q8_load(const T* p, int n, float (&v)[8]) {       // n: elements there are, 1..8
    T e[8];
    if (n >= 8) {
        __builtin_memcpy(e, p, 8 * sizeof(T));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : T(0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 2) v[i] = bf16_to_f32(e[i]);
        else v[i] = __uint_as_float(e[i]);
    }
}
template <class T>
__device__ __forceinline__ void q8_store(T* p, int n, const float (&v)[8]) {
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 2) {
            const uint32_t b = bf16_rne(v[i]);
            e[i] = (T)(v[i] == v[i] ? b : 0x7FC0u);                              // the rounding's carry could end a NaN
        } else {
            e[i] = __float_as_uint(v[i]);
        }
    }
    if (n >= 8) {
        __builtin_memcpy(p, e, 8 * sizeof(T));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = e[i];
    }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}
__device__ __forceinline__ double wave_max(double v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmax(v, __shfl_xor(v, off, 64));
    return v;
}
// Over a workgroup; every thread gets the result.
template <class F>
__device__ __forceinline__ double group_reduce(double v, double* lds, F wave_op, bool is_max) {
    const int waves = blockDim.x >> 6;
    v = wave_op(v);
    if (waves == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double r = lds[0];
    for (int w = 1; w < waves; ++w) r = is_max ? fmax(r, lds[w]) : r + lds[w];
    return r;
}

// X, A: bits of the input's and the addend's elements.  kHeld: vectors of 8 that a thread keeps (0: rows too long for that are read
// again).  NORM: with an RMS norm in front.
template <class X, class A, bool NORM, int kHeld>
__global__ void __launch_bounds__(1024) k_q8_rows(const X* x, int64_t ldx, const A* __restrict__ add, int64_t ldadd,
                                                  const float* __restrict__ gain, float eps, int n, X* sum, int64_t ldsum, int8_t* __restrict__ q,
                                                  int64_t ldq, float* __restrict__ scale) {
    __shared__ double lds[16];
    const int64_t row = blockIdx.x;
    x += row * ldx;
    q += row * ldq;
    if (add) add += row * ldadd;
    if (sum) sum += row * ldsum;
    const int stride = blockDim.x * 8, first = threadIdx.x * 8;
    constexpr int kKeep = kHeld ? kHeld : 1;
    float held[kKeep][8];
    auto fetch = [&](int i, int at, float (&v)[8], bool from_memory) {    // x + add of the thread's i-th vector
        if (!from_memory) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = held[kHeld ? i : 0][e];
            return;
        }
        q8_load(x + at, n - at, v);
        if (NORM && add) {
            float a[8];
            q8_load(add + at, n - at, a);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += a[e];
        }
    };
    double squares = 0.;
    double most = 0.;
    bool bad = false;
    auto first_pass = [&](int i, int at) {
        float v[8];
        fetch(i, at, v, true);
        if (NORM && sum) q8_store(sum + at, n - at, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (kHeld) held[kHeld ? i : 0][e] = v[e];
            bad |= !(fabsf(v[e]) <= 3.402823466e38f);
            if (NORM) squares += (double)v[e] * (double)v[e];
            else most = fmax(most, (double)fabsf(v[e]));
        }
    };
    if constexpr (kHeld > 0) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (first + i * stride < n) first_pass(i, first + i * stride);
    } else {
        for (int at = first; at < n; at += stride) first_pass(0, at);
    }
    // Rows longer than the registers are read again, from `sum` if it took the place of x (in full precision only where sum is fp32,
    // so the host has no bf16 row of that length written over itself).
    const bool over = !kHeld && NORM && sum == x;
    double rstd = 1.;
    if (NORM) rstd = 1. / sqrt(group_reduce(squares, lds, wave_sum, false) / n + (double)eps);
    auto normed = [&](int i, int at, double (&y)[8]) {
        float v[8];
        if (over) q8_load(x + at, n - at, v);
        else fetch(i, at, v, !kHeld);
        float g[8];
        if (NORM) q8_load(reinterpret_cast<const uint32_t*>(gain) + at, n - at, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = NORM ? (double)v[e] * rstd * (double)g[e] : (double)v[e];
    };
    if (NORM) {
        auto second_pass = [&](int i, int at) {
            double y[8];
            normed(i, at, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                most = fmax(most, fabs(y[e]));
                bad |= !(fabs(y[e]) <= 3.402823466e38);
            }
        };
        if constexpr (kHeld > 0) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (first + i * stride < n) second_pass(i, first + i * stride);
        } else {
            for (int at = first; at < n; at += stride) second_pass(0, at);
        }
    }
    most = group_reduce(bad ? INFINITY : most, lds, wave_max, true);
    const bool finite = most <= 3.402823466e38;
    const float s = finite ? (float)(most / 127.) : __uint_as_float(0x7FC00000u);
    const double inv = finite && s > 0.f ? 1. / (double)s : 0.;
    if (threadIdx.x == 0) scale[row] = s;
    auto last_pass = [&](int i, int at) {
        double y[8];
        normed(i, at, y);
        int8_t b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            double t = y[e] * inv;
            if (fabs(fabs(t - rint(t)) - 0.5) < 1e-9) t = y[e] / (double)s;      // (the product may be off a tie that the quotient hits)
            b[e] = finite && s > 0.f ? (int8_t)(int)fmin(fmax(rint(t), -127.), 127.) : (int8_t)0;
        }
        if (n - at >= 8) {
            __builtin_memcpy(q + at, b, 8);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n - at) q[at + e] = b[e];
        }
    };
    if constexpr (kHeld > 0) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (first + i * stride < n) last_pass(i, first + i * stride);
    } else {
        for (int at = first; at < n; at += stride) last_pass(0, at);
    }
}

template <class X, class A, bool NORM>
static void q8_rows(const void* x, int64_t ldx, const void* add, int64_t ldadd, const float* gain, float eps, int rows, int n, void* sum, int64_t ldsum,
                    int8_t* q, int64_t ldq, float* scale, hipStream_t stream) {
    const int threads = std::min(1024, std::max(64, (n + 16 * 64 - 1) / (16 * 64) * 64));     // two vectors of 8 a thread
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(rows), dim3(threads), 0, stream, static_cast<const X*>(x), ldx, static_cast<const A*>(add), ldadd, gain, eps, n,
                           static_cast<X*>(sum), ldsum, q, ldq, scale);
    };
    if (n <= 2 * 8 * threads) launch(k_q8_rows<X, A, NORM, 2>);
    else launch(k_q8_rows<X, A, NORM, 0>);
}

hipError_t launch_q8_rows(const void* x, int dtype, int64_t ldx, const void* add, int add_dtype, int64_t ldadd, const float* gain, float eps, int rows,
                          int n, void* sum, int64_t ldsum, int8_t* q, int64_t ldq, float* scale, hipStream_t stream) {
    const bool half = dtype == AMUSD_DTYPE_BF16, add_half = add_dtype == AMUSD_DTYPE_BF16;
    auto go = [&](auto f) { f(x, ldx, add, ldadd, gain, eps, rows, n, sum, ldsum, q, ldq, scale, stream); };
    if (!gain) {
        if (half) go(q8_rows<uint16_t, uint16_t, false>);
        else go(q8_rows<uint32_t, uint16_t, false>);
    } else if (half) {
        if (add_half) go(q8_rows<uint16_t, uint16_t, true>);
        else go(q8_rows<uint16_t, uint32_t, true>);
    } else {
        if (add_half) go(q8_rows<uint32_t, uint16_t, true>);
        else go(q8_rows<uint32_t, uint32_t, true>);
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------- into the cache
// A workgroup owns 64 positions of one kv head's keys or values (blocks do not reach over that), so nothing is shared between
// workgroups.  16 lanes hold a row (its rotary pairs in one lane), so its largest element needs four lane exchanges; the rows then
// lie in LDS for the store in the cache's order.  Blocks that held tokens before keep their scale unless a new value outgrows it;
// then what they hold is rounded once more, to the new scale.
__device__ __forceinline__ const Q8Seg& q8_find(const Q8Segs& S, int unit) {
    int i = 0;
    while (i + 1 < S.n_seg && unit >= S.s[i + 1].unit0) ++i;
    return S.s[i];
}

template <int HD>
__global__ void __launch_bounds__(256) k_q8_append(amusd_q8_cache C, int layer, Q8Segs S, const uint16_t* __restrict__ krows,
                                                   const uint16_t* __restrict__ vrows, int64_t ld, const float* __restrict__ cos,
                                                   const float* __restrict__ sin) {
    constexpr int kPer = HD / 32;                    // elements a lane has of each half of a row
    __shared__ float rows[kQ8Group][HD + 4];
    __shared__ uint32_t most[kQ8Group];              // bits of a row's largest magnitude: those of a NaN are above all others
    __shared__ float new_scale[kQ8Group], ratio[kQ8Group];
    const int head = blockIdx.y, t = threadIdx.x;
    const bool values = blockIdx.z;
    const Q8Seg seg = q8_find(S, blockIdx.x);
    const int p0 = (seg.pos0 / kQ8Group + (int)blockIdx.x - seg.unit0) * kQ8Group;      // first position of the group
    const int from = max(seg.pos0, p0), to = min(seg.pos0 + seg.n, p0 + kQ8Group);      // new ones among them
    const uint16_t* src = (values ? vrows : krows) + (int64_t)(seg.row0 - seg.pos0) * ld + (int64_t)head * HD;
    for (int r = t >> 4; r < kQ8Group; r += 16) {
        const int pos = p0 + r, l = t & 15;
        uint32_t m = 0;
        if (pos >= from && pos < to) {
            const uint16_t* p = src + (int64_t)pos * ld + l * kPer;
            uint16_t a[kPer], b[kPer];
            __builtin_memcpy(a, p, sizeof a);
            __builtin_memcpy(b, p + HD / 2, sizeof b);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                float x = bf16_to_f32(a[i]), y = bf16_to_f32(b[i]);
                if (!values && cos) {
                    const float c = cos[(int64_t)pos * (HD / 2) + l * kPer + i], s = sin[(int64_t)pos * (HD / 2) + l * kPer + i];
                    rotate_pair(x, y, c, s, x, y);
                }
                rows[r][l * kPer + i] = x;
                rows[r][l * kPer + i + HD / 2] = y;
                m = max(m, max(__float_as_uint(x) & 0x7FFFFFFFu, __float_as_uint(y) & 0x7FFFFFFFu));
            }
        }
        m = max(m, lane_xor_u<1>(m));
        m = max(m, lane_xor_u<2>(m));
        m = max(m, lane_xor_u<4>(m));
        m = max(m, lane_xor_u<8>(m));
        if (l == 0) most[r] = m;
    }
    __syncthreads();
    const size_t kvh = ((size_t)layer * C.n_seqs + seg.seq) * C.Hkv + head;
    const int B = C.block;
    if (t < kQ8Group / B) {
        const int b0 = p0 + t * B;                                   // the block's first position
        float* scales = (values ? C.vs : C.ks) + kvh * (C.cap / B);
        float s = 0.f, r = 1.f;
        if (b0 < to && b0 + B > from) {
            uint32_t m = 0;
            for (int i = 0; i < B; ++i) m = max(m, most[t * B + i]);
            const float was = b0 < seg.pos0 ? scales[b0 / B] : 0.f;
            s = m >= 0x7F800000u || was != was ? __uint_as_float(0x7FC00000u) : fmaxf(was, __uint_as_float(m) / 127.f);
            r = s > 0.f ? was / s : s == s ? 1.f : 0.f;
            scales[b0 / B] = s;
        }
        new_scale[t] = s;
        ratio[t] = r;
    }
    __syncthreads();
    // 4 bytes a thread: keys 4 columns of a position, values 4 positions of a column
    int8_t* out = (values ? C.v : C.k) + kvh * ((size_t)C.cap * HD);
    // (values are kept as q + 128: amusd_q8_attention.hip)
    const uint8_t bias = values ? 0x80 : 0;
    auto eight = [&](int r, int c, bool& write, int8_t old) {        // position p0 + r, column c
        const int pos = p0 + r, b = r / B;
        const float s = new_scale[b];
        if (pos >= from && pos < to) {
            write = true;
            return (int8_t)((s > 0.f ? (int)fminf(fmaxf(rintf(rows[r][c] / s), -127.f), 127.f) : 0) ^ bias);
        }
        // held before, in a block whose scale has grown (from a block that this call does not touch `ratio` is 1)
        write = pos < from && pos < seg.pos0 && ratio[b] != 1.f;
        return write ? (int8_t)((int)rintf((float)(int8_t)(old ^ bias) * ratio[b]) ^ bias) : old;
    };
    const int first_row = max(0, from / B * B - p0), last_row = to - p0;          // rows that can change
    if (!values) {
        for (int i = t; i < (last_row - first_row) * (HD / 4); i += 256) {
            const int r = first_row + i / (HD / 4), c = i % (HD / 4) * 4;
            int8_t* p = out + q8_k_index(HD, p0 + r, c);
            const char4 old = *reinterpret_cast<const char4*>(p);
            bool w = false;
            char4 b;
            b.x = eight(r, c, w, old.x);
            b.y = eight(r, c + 1, w, old.y);
            b.z = eight(r, c + 2, w, old.z);
            b.w = eight(r, c + 3, w, old.w);
            if (w) *reinterpret_cast<char4*>(p) = b;
        }
    } else {
        const int q0 = first_row / 4, quads = (last_row + 3) / 4 - q0;
        for (int i = t; i < quads * HD; i += 256) {
            const int r = (q0 + i / HD) * 4, c = i % HD;
            int8_t* p = out + q8_v_index(HD, p0 + r, c);
            const char4 old = *reinterpret_cast<const char4*>(p);
            const int8_t o[4] = {old.x, old.y, old.z, old.w};
            int8_t b[4];
            bool any = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bool w = false;
                b[e] = eight(r + e, c, w, o[e]);
                any |= w;
            }
            if (any) *reinterpret_cast<char4*>(p) = char4{b[0], b[1], b[2], b[3]};
        }
    }
}

hipError_t launch_q8_append(const amusd_q8_cache& c, int layer, const Q8Segs& S, const void* k, const void* v, int64_t ld, const float* cos,
                            const float* sin, hipStream_t stream) {
    const dim3 grid(S.units, c.Hkv, 2);
    const uint16_t *kr = static_cast<const uint16_t*>(k), *vr = static_cast<const uint16_t*>(v);
    if (c.hd == 64) hipLaunchKernelGGL(k_q8_append<64>, grid, dim3(256), 0, stream, c, layer, S, kr, vr, ld, cos, sin);
    else hipLaunchKernelGGL(k_q8_append<128>, grid, dim3(256), 0, stream, c, layer, S, kr, vr, ld, cos, sin);
    return hipGetLastError();
}

// ---------------------------------------------------------------- out of the cache
// The values that rows of the cache stand for, four columns of a position a thread.
template <class T>
__global__ void __launch_bounds__(256) k_q8_read(amusd_q8_cache C, int layer, Q8Segs S, T* __restrict__ kout, T* __restrict__ vout, int64_t ld) {
    const int row = blockIdx.x, quads = C.Hkv * C.hd / 4;
    int i = 0;
    while (i + 1 < S.n_seg && row >= S.s[i + 1].row0) ++i;
    const int pos = S.s[i].pos0 + row - S.s[i].row0;
    const bool values = blockIdx.y;
    T* out = (values ? vout : kout) + (int64_t)row * ld;
    for (int x = threadIdx.x; x < quads; x += blockDim.x) {
        const int head = x * 4 / C.hd, c = x * 4 % C.hd;
        const size_t kvh = ((size_t)layer * C.n_seqs + S.s[i].seq) * C.Hkv + head;
        const float s = (values ? C.vs : C.ks)[kvh * (C.cap / C.block) + pos / C.block];
        const int8_t* p = (values ? C.v : C.k) + kvh * ((size_t)C.cap * C.hd);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float y = (float)(values ? (int8_t)(p[q8_v_index(C.hd, pos, c + e)] ^ 0x80) : p[q8_k_index(C.hd, pos, c + e)]) * s;
            if constexpr (sizeof(T) == 2) out[x * 4 + e] = (T)(y == y ? bf16_rne(y) : 0x7FC0u);
            else out[x * 4 + e] = __float_as_uint(y);
        }
    }
}

hipError_t launch_q8_read(const amusd_q8_cache& c, int layer, const Q8Segs& S, void* k, void* v, int dtype, int64_t ld, hipStream_t stream) {
    const dim3 grid(S.rows, 2);
    if (dtype == AMUSD_DTYPE_BF16)
        hipLaunchKernelGGL(k_q8_read<uint16_t>, grid, dim3(256), 0, stream, c, layer, S, static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), ld);
    else
        hipLaunchKernelGGL(k_q8_read<uint32_t>, grid, dim3(256), 0, stream, c, layer, S, static_cast<uint32_t*>(k), static_cast<uint32_t*>(v), ld);
    return hipGetLastError();
}

// ---------------------------------------------------------------- weights to 8 bits, in operand order
// One wave a row of the source: finds its scale (unless it is given), then writes the feature's bytes.  Row i is feature first + i
// of the matrix or, in a gated one, its gate's or up projection's (part 1, 2) feature i.
template <class T>
__global__ void __launch_bounds__(64) k_q8_matrix(uint4* __restrict__ frag, float* __restrict__ scale, const T* __restrict__ w, int64_t ld,
                                                  const float* __restrict__ given, int k, int first, int part) {
    const int i = blockIdx.x, lane = threadIdx.x;
    const int tile = part ? (i >> 4) * 2 + part - 1 : (first + i) >> 4, r = part ? i & 15 : (first + i) & 15;
    w += i * ld;
    double s = 0.;
    auto value = [&](int c) {
        if constexpr (sizeof(T) == 2) return bf16_to_f32(w[c]);
        else return __uint_as_float(w[c]);
    };
    if constexpr (sizeof(T) > 1) {
        float most = 0.f;
        bool bad = false;
        for (int c = lane; c < k; c += 64) {
            const float x = value(c);
            bad |= !(fabsf(x) <= 3.402823466e38f);
            most = fmaxf(most, fabsf(x));
        }
        const double m = wave_max(bad ? INFINITY : (double)most);
        bad = !(m <= 3.402823466e38);
        s = bad ? 0. : (double)(float)(m / 127.);
        if (lane == 0) scale[tile * 16 + r] = bad ? __uint_as_float(0x7FC00000u) : (float)s;
    } else if (lane == 0) {
        scale[tile * 16 + r] = given[i];
    }
    const int kblocks = (k + 63) / 64;
    int8_t* out = reinterpret_cast<int8_t*>(frag);
    for (int kb = 0; kb < kblocks; ++kb) {
        const int c = kb * 64 + lane;
        int8_t b = 0;
        if (c < k) {
            if constexpr (sizeof(T) == 1) b = (int8_t)w[c];
            else b = s > 0. ? (int8_t)(int)fmin(fmax(rint((double)value(c) / s), -127.), 127.) : (int8_t)0;
        }
        out[(((size_t)tile * kblocks + kb) * 64 + (lane >> 4) * 16 + r) * 16 + (lane & 15)] = b;
    }
}

hipError_t launch_q8_matrix(const amusd_q8_matrix& m, const void* w, int dtype, int64_t ld, const float* scale, int rows, int first, int part,
                            hipStream_t stream) {
    auto go = [&](auto kernel, auto* src) {
        hipLaunchKernelGGL(kernel, dim3(rows), dim3(64), 0, stream, const_cast<uint4*>(m.frag), const_cast<float*>(m.scale), src, ld, scale, m.k, first, part);
    };
    if (dtype == AMUSD_DTYPE_FP32) go(k_q8_matrix<uint32_t>, static_cast<const uint32_t*>(w));
    else if (dtype == AMUSD_DTYPE_BF16) go(k_q8_matrix<uint16_t>, static_cast<const uint16_t*>(w));
    else go(k_q8_matrix<int8_t>, static_cast<const int8_t*>(w));
    return hipGetLastError();
}

// ---------------------------------------------------------------- handles
hipError_t q8_device(int& device, int& cus) {
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device);
    return e;
}

hipError_t q8_matrix_take(amusd_q8_matrix& m, int n, int k, bool gated, Q8Alloc alloc, hipStream_t stream) {
    m.gated = gated;
    m.n = gated ? n / 2 : n;
    m.k = k;
    m.kblocks = (k + 63) / 64;
    m.tiles = (m.n + 15) / 16 * (gated ? 2 : 1);
    void *frag = nullptr, *scale = nullptr;
    const size_t bytes = (size_t)m.tiles * m.kblocks * 1024, scales = (size_t)m.tiles * 16 * 4;
    hipError_t e = q8_device(m.device, m.cus);
    if (e == hipSuccess) e = alloc(m.device, &frag, bytes);
    m.frag = static_cast<const uint4*>(frag);
    if (e == hipSuccess) e = alloc(m.device, &scale, scales);
    m.scale = static_cast<const float*>(scale);
    // (zeros are what pads features and columns)
    if (e == hipSuccess) e = hipMemsetAsync(frag, 0, bytes, stream);
    if (e == hipSuccess) e = hipMemsetAsync(scale, 0, scales, stream);
    return e;
}
void q8_matrix_drop(amusd_q8_matrix& m) {
    if (m.frag) (void)hipFree(const_cast<uint4*>(m.frag));
    if (m.scale) (void)hipFree(const_cast<float*>(m.scale));
    m.frag = nullptr;
    m.scale = nullptr;
}

hipError_t q8_cache_take(amusd_q8_cache& c, int n_layers, int n_seqs, int n_q_heads, int n_kv_heads, int head_dim, int capacity, int block, Q8Alloc alloc,
                         hipStream_t stream) {
    c.n_layers = n_layers;
    c.n_seqs = n_seqs;
    c.Hq = n_q_heads;
    c.Hkv = n_kv_heads;
    c.hd = head_dim;
    c.G = n_q_heads / n_kv_heads;
    c.block = block;
    c.cap = (capacity + kQ8Group - 1) / kQ8Group * kQ8Group;
    hipError_t e = q8_device(c.device, c.cus);
    q8_attention_plan(c);
    const size_t heads = (size_t)n_layers * n_seqs * n_kv_heads, bytes = heads * c.cap * head_dim, scales = heads * (c.cap / block) * 4;
    auto take = [&](auto& p, size_t n, bool zero) {
        if (e != hipSuccess) return;
        void* got = nullptr;
        e = alloc(c.device, &got, n);
        p = static_cast<std::remove_reference_t<decltype(p)>>(got);
        if (e == hipSuccess && zero) e = hipMemsetAsync(got, 0, n, stream);
    };
    // zeros: positions that were never written take part in tiles, with weight 0
    take(c.k, bytes, true);
    take(c.v, bytes, true);
    take(c.ks, scales, true);
    take(c.vs, scales, true);
    take(c.part, (size_t)c.part_tiles * c.max_chunks * (head_dim + 2) * 16 * 4, false);
    return e;
}
void q8_cache_drop(amusd_q8_cache& c) {
    for (void* p : {(void*)c.k, (void*)c.v, (void*)c.ks, (void*)c.vs, (void*)c.part})
        if (p) (void)hipFree(p);
    c.k = c.v = nullptr;
    c.ks = c.vs = c.part = nullptr;
}

void q8_append_units(Q8Segs& S) {
    S.units = 0;
    for (int i = 0; i < S.n_seg; ++i) {
        S.s[i].unit0 = S.units;
        S.units += (S.s[i].pos0 + S.s[i].n - 1) / kQ8Group - S.s[i].pos0 / kQ8Group + 1;
    }
}

}  // namespace amusd

using namespace amusd;

namespace {

#define Q8_TRY(expr)                                                                                    \
    do {                                                                                                \
        hipError_t e_ = (expr);                                                                         \
        if (e_ != hipSuccess) return report(AMUSD_E_HIP, #expr, hipGetErrorString(e_));                 \
    } while (0)

hipError_t q8_malloc(int, void** p, size_t bytes) { return hipMalloc(p, bytes); }

bool float_dtype(int dtype) { return dtype == AMUSD_DTYPE_FP32 || dtype == AMUSD_DTYPE_BF16; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int on_device(int device) {
    int now = -1;
    Q8_TRY(hipGetDevice(&now));
    return now == device ? AMUSD_OK : report(AMUSD_E_ARG, "the handle belongs to another device than the current one");
}

int rows_args(int32_t rows, int32_t n, const int8_t* q, int64_t ldq, const float* scale) {
    if (!q || !scale) return report(AMUSD_E_ARG, "q8 rows: null argument");
    if (rows < 0 || n < 1) return report(AMUSD_E_ARG, "q8 rows: rows < 0 or n < 1");
    if (ldq < n || ldq % 16 || !aligned(q, 16)) return report(AMUSD_E_ARG, "q8 rows: 8-bit rows have to begin at multiples of 16 bytes");
    return AMUSD_OK;
}

// Segments of a call; `group`: positions of a unit of work.
int segments(const amusd_q8_cache* c, int32_t layer, int32_t n_seq, const int32_t* seq_ids, const int32_t* pos0, const int32_t* n, Q8Segs& S) {
    if (!c || !seq_ids || !pos0 || !n) return report(AMUSD_E_ARG, "q8 cache: null argument");
    if (layer < 0 || layer >= c->n_layers) return report(AMUSD_E_ARG, "q8 cache: layer out of range");
    if (n_seq < 1 || n_seq > kMaxSegs) return report(AMUSD_E_ARG, "q8 cache: n_seq outside [1, 16]");
    S.n_seg = n_seq;
    int64_t rows = 0;
    S.max_len = 0;
    for (int i = 0; i < n_seq; ++i) {
        if (seq_ids[i] < 0 || seq_ids[i] >= c->n_seqs) return report(AMUSD_E_ARG, "q8 cache: sequence id outside [0, n_seqs)");
        for (int j = 0; j < i; ++j)
            if (seq_ids[j] == seq_ids[i]) return report(AMUSD_E_ARG, "q8 cache: a sequence appears twice");
        if (n[i] < 1) return report(AMUSD_E_ARG, "q8 cache: a sequence without rows");
        if (pos0[i] < 0) return report(AMUSD_E_RANGE, "q8 cache: position below 0");
        if ((int64_t)pos0[i] + n[i] > c->cap) return report(AMUSD_E_CAPACITY, "q8 cache: capacity exceeded");
        S.s[i] = Q8Seg{seq_ids[i], pos0[i], n[i], (int)rows, 0};
        rows += n[i];
        S.max_len = std::max(S.max_len, pos0[i] + n[i]);
    }
    if (rows > INT32_MAX) return report(AMUSD_E_ARG, "q8 cache: too many rows");
    S.rows = (int)rows;
    const int rc = on_device(c->device);
    return rc;
}

int rope_args(const float* cos, const float* sin) {
    return !cos == !sin ? AMUSD_OK : report(AMUSD_E_ARG, "q8 cache: one rotary table without the other");
}

}  // namespace

extern "C" {

int amusd_q8_quantize(const void* x, int32_t dtype, int64_t ldx, int32_t rows, int32_t n, int8_t* q, int64_t ldq, float* scale, void* hip_stream) {
    const int rc = rows_args(rows, n, q, ldq, scale);
    if (rc) return rc;
    if (!x || !float_dtype(dtype) || ldx < n || !aligned(x, dtype == AMUSD_DTYPE_BF16 ? 2 : 4)) return report(AMUSD_E_ARG, "q8_quantize: bad input rows");
    if (!rows) return AMUSD_OK;
    Q8_TRY(launch_q8_rows(x, dtype, ldx, nullptr, AMUSD_DTYPE_BF16, 0, nullptr, 0.f, rows, n, nullptr, 0, q, ldq, scale, static_cast<hipStream_t>(hip_stream)));
    return AMUSD_OK;
}

int amusd_q8_rmsnorm(const void* x, int32_t dtype, int64_t ldx, const void* add, int32_t add_dtype, int64_t ldadd, const float* gain, float eps,
                     int32_t rows, int32_t n, void* sum, int64_t ldsum, int8_t* q, int64_t ldq, float* scale, void* hip_stream) {
    const int rc = rows_args(rows, n, q, ldq, scale);
    if (rc) return rc;
    if (!x || !gain || !float_dtype(dtype) || ldx < n || !aligned(x, dtype == AMUSD_DTYPE_BF16 ? 2 : 4) || !aligned(gain, 4) || !(eps >= 0.f))
        return report(AMUSD_E_ARG, "q8_rmsnorm: bad input rows, gain or eps");
    if (add && (!float_dtype(add_dtype) || ldadd < n || !aligned(add, add_dtype == AMUSD_DTYPE_BF16 ? 2 : 4)))
        return report(AMUSD_E_ARG, "q8_rmsnorm: bad rows to add");
    if (sum && (ldsum < n || !aligned(sum, dtype == AMUSD_DTYPE_BF16 ? 2 : 4))) return report(AMUSD_E_ARG, "q8_rmsnorm: bad rows for the sum");
    if (sum == x && sum && ldsum != ldx) return report(AMUSD_E_ARG, "q8_rmsnorm: the sum takes the place of x at another distance of rows");
    if (n > kQ8MaxRow && sum == x && dtype == AMUSD_DTYPE_BF16 && sum)
        return report(AMUSD_E_ARG, "q8_rmsnorm: a bf16 row of more than 16384 columns cannot be written over itself");
    if (!rows) return AMUSD_OK;
    Q8_TRY(launch_q8_rows(x, dtype, ldx, add, add_dtype, ldadd, gain, eps, rows, n, sum, ldsum, q, ldq, scale, static_cast<hipStream_t>(hip_stream)));
    return AMUSD_OK;
}

int amusd_q8_matrix_create(const void* w, int32_t dtype, const float* scale, int32_t n, int32_t k, int64_t ld, int32_t gated, int32_t on_device_,
                           void* hip_stream, amusd_q8_matrix** out) {
    if (!w || !out) return report(AMUSD_E_ARG, "q8_matrix: null argument");
    if (!float_dtype(dtype) && dtype != AMUSD_DTYPE_INT8) return report(AMUSD_E_ARG, "q8_matrix: unknown dtype");
    if ((dtype == AMUSD_DTYPE_INT8) != (scale != nullptr)) return report(AMUSD_E_ARG, "q8_matrix: scales go with 8-bit weights, and only with them");
    if (n < 1 || k < 1 || ld < k || (gated && n % 2) || n > (1 << 28) || k > kQ8MaxK) return report(AMUSD_E_ARG, "q8_matrix: bad sizes");
    amusd_q8_matrix* m = new (std::nothrow) amusd_q8_matrix();
    if (!m) return report(AMUSD_E_NOMEM, "q8_matrix: handle");
    const size_t esz = dtype == AMUSD_DTYPE_FP32 ? 4 : dtype == AMUSD_DTYPE_BF16 ? 2 : 1;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t e = q8_matrix_take(*m, n, k, gated, q8_malloc, stream);
    void *tmp = nullptr, *tmp_scale = nullptr;
    if (!on_device_) {
        const size_t bytes = ((size_t)(n - 1) * ld + k) * esz;
        if (e == hipSuccess) e = hipMalloc(&tmp, bytes);
        if (e == hipSuccess) e = hipMemcpy(tmp, w, bytes, hipMemcpyHostToDevice);
        w = tmp;
        if (scale) {
            if (e == hipSuccess) e = hipMalloc(&tmp_scale, (size_t)n * 4);
            if (e == hipSuccess) e = hipMemcpy(tmp_scale, scale, (size_t)n * 4, hipMemcpyHostToDevice);
            scale = static_cast<const float*>(tmp_scale);
        }
    }
    if (e == hipSuccess) e = launch_q8_matrix(*m, w, dtype, ld, scale, m->n, 0, gated ? 1 : 0, stream);
    if (e == hipSuccess && gated)
        e = launch_q8_matrix(*m, static_cast<const char*>(w) + (size_t)m->n * ld * esz, dtype, ld, scale ? scale + m->n : nullptr, m->n, 0, 2, stream);
    if (e == hipSuccess) e = hipStreamSynchronize(stream);
    if (tmp) (void)hipFree(tmp);
    if (tmp_scale) (void)hipFree(tmp_scale);
    if (e != hipSuccess) {
        amusd_q8_matrix_free(m);
        return report(AMUSD_E_HIP, "q8_matrix", hipGetErrorString(e));
    }
    *out = m;
    return AMUSD_OK;
}

int amusd_q8_matrix_free(amusd_q8_matrix* m) {
    if (!m) return AMUSD_OK;
    q8_matrix_drop(*m);
    delete m;
    return AMUSD_OK;
}

int64_t amusd_q8_gemm_workspace_bytes(const amusd_q8_matrix* m, int32_t rows) {
    if (!m || rows < 0) return report(AMUSD_E_ARG, "q8_gemm_workspace_bytes: bad argument");
    return q8_gemm_workspace(*m, rows);
}

int amusd_q8_gemm(const amusd_q8_matrix* w, const int8_t* x, int64_t ldx, const float* scale, int32_t rows, void* out, int32_t dtype, int64_t ldo,
                  void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!w || !x || !scale || !out) return report(AMUSD_E_ARG, "q8_gemm: null argument");
    if (rows < 0 || !float_dtype(dtype) || ldo < w->n || !aligned(out, dtype == AMUSD_DTYPE_BF16 ? 2 : 4)) return report(AMUSD_E_ARG, "q8_gemm: bad output");
    if (ldx < w->k || ldx % 16 || !aligned(x, 16)) return report(AMUSD_E_ARG, "q8_gemm: 8-bit rows have to begin at multiples of 16 bytes");
    if (workspace && (workspace_bytes < 0 || !aligned(workspace, 16))) return report(AMUSD_E_ARG, "q8_gemm: bad workspace");
    const int rc = on_device(w->device);
    if (rc) return rc;
    if (!rows) return AMUSD_OK;
    Q8_TRY(launch_q8_gemm(*w, x, ldx, scale, rows, out, dtype, ldo, workspace, workspace ? workspace_bytes : 0, static_cast<hipStream_t>(hip_stream)));
    return AMUSD_OK;
}

int amusd_q8_cache_create(int32_t n_layers, int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t capacity, int32_t block,
                          void* hip_stream, amusd_q8_cache** out) {
    if (!out) return report(AMUSD_E_ARG, "q8_cache: null argument");
    if (n_layers < 1 || n_seqs < 1 || n_seqs > AMUSD_MAX_SEQS || n_q_heads < 1 || n_kv_heads < 1 || n_kv_heads > 65535 || capacity < 1 ||
        capacity > (1 << 30))
        return report(AMUSD_E_ARG, "q8_cache: bad sizes");
    if (head_dim != 64 && head_dim != 128) return report(AMUSD_E_ARG, "q8_cache: head_dim must be 64 or 128");
    if (block != 1 && block != 16 && block != 32 && block != 64) return report(AMUSD_E_ARG, "q8_cache: block must be 1, 16, 32 or 64");
    const int G = n_q_heads / n_kv_heads;
    if (n_q_heads % n_kv_heads || (G != 1 && G != 2 && G != 4 && G != 8)) return report(AMUSD_E_ARG, "q8_cache: n_q_heads / n_kv_heads must be 1, 2, 4 or 8");
    amusd_q8_cache* c = new (std::nothrow) amusd_q8_cache();
    if (!c) return report(AMUSD_E_NOMEM, "q8_cache: handle");
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t e = q8_cache_take(*c, n_layers, n_seqs, n_q_heads, n_kv_heads, head_dim, capacity, block, q8_malloc, stream);
    if (e == hipSuccess) e = hipStreamSynchronize(stream);
    if (e != hipSuccess) {
        amusd_q8_cache_free(c);
        return report(AMUSD_E_HIP, "q8_cache", hipGetErrorString(e));
    }
    *out = c;
    return AMUSD_OK;
}

int amusd_q8_cache_free(amusd_q8_cache* c) {
    if (!c) return AMUSD_OK;
    q8_cache_drop(*c);
    delete c;
    return AMUSD_OK;
}

int amusd_q8_cache_append(amusd_q8_cache* c, int32_t layer, int32_t n_seq, const int32_t* seq_ids, const int32_t* pos0, const int32_t* n, const void* k,
                          const void* v, int64_t ld, const float* rope_cos, const float* rope_sin, void* hip_stream) {
    Q8Segs S;
    int rc = segments(c, layer, n_seq, seq_ids, pos0, n, S);
    if (rc || (rc = rope_args(rope_cos, rope_sin))) return rc;
    if (!k || !v || ld < (int64_t)c->Hkv * c->hd || !aligned(k, 2) || !aligned(v, 2)) return report(AMUSD_E_ARG, "q8_cache_append: bad rows");
    q8_append_units(S);
    Q8_TRY(launch_q8_append(*c, layer, S, k, v, ld, rope_cos, rope_sin, static_cast<hipStream_t>(hip_stream)));
    return AMUSD_OK;
}

int amusd_q8_cache_read(const amusd_q8_cache* c, int32_t layer, int32_t n_seq, const int32_t* seq_ids, const int32_t* pos0, const int32_t* n, void* k,
                        void* v, int32_t dtype, int64_t ld, void* hip_stream) {
    Q8Segs S;
    const int rc = segments(c, layer, n_seq, seq_ids, pos0, n, S);
    if (rc) return rc;
    const size_t esz = dtype == AMUSD_DTYPE_BF16 ? 2 : 4;
    if (!k || !v || !float_dtype(dtype) || ld < (int64_t)c->Hkv * c->hd || !aligned(k, esz) || !aligned(v, esz))
        return report(AMUSD_E_ARG, "q8_cache_read: bad rows");
    Q8_TRY(launch_q8_read(*c, layer, S, k, v, dtype, ld, static_cast<hipStream_t>(hip_stream)));
    return AMUSD_OK;
}

int amusd_q8_attention(amusd_q8_cache* c, int32_t layer, int32_t n_seq, const int32_t* seq_ids, const int32_t* pos0, const int32_t* n, const void* q,
                       int64_t ldq, float scale, const float* rope_cos, const float* rope_sin, void* out, int64_t ldo, void* hip_stream) {
    Q8Segs S;
    int rc = segments(c, layer, n_seq, seq_ids, pos0, n, S);
    if (rc || (rc = rope_args(rope_cos, rope_sin))) return rc;
    const int64_t width = (int64_t)c->Hq * c->hd;
    if (!q || !out || ldq < width || ldo < width || !aligned(q, 2) || !aligned(out, 2)) return report(AMUSD_E_ARG, "q8_attention: bad rows");
    if (!(scale > 0.f) || !(scale < INFINITY)) return report(AMUSD_E_ARG, "q8_attention: scale must be positive and finite");
    Q8_TRY(launch_q8_attention(*c, layer, S, q, ldq, scale, rope_cos, rope_sin, out, ldo, static_cast<hipStream_t>(hip_stream)));
    return AMUSD_OK;
}

}  // extern "C"
