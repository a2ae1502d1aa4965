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
// A workgroup a row, the row in registers: it is read once and written once.  Bound by its launch where there are few rows; with many by the
// way through a row, whose loads, reduction and stores come one after the other: waves wait 58 to 68 % of their cycles, vector instructions
// take 72 % of those in which a compute unit is busy (2048 x 14336: 19 an element) or 32 % (1531 x 2055 with norm).  Loads and stores take any alignment (one instruction of 16 bytes all the same).  Sums of squares, their root and the normalised
// element are in 64 bits, the element then rounded to 32: a square of a large element stays finite.
// The quotient is taken as the product with the scale's reciprocal, and divided in full only where that is too near the middle between
// two integers to tell (half the largest value stands on one); adding 1.5 * 2^23 leaves the nearest integer, ties to even, in the low bits.
// Measured (MI355X): 2048 x 14336 bf16 26 us (3.4 TB/s; a division for each element 53), 2048 x 4096 fp32 + bf16 with norm and sum 25 (3.7 TB/s),
// 1531 x 2055 14.5-15 (a third of its vectors of 8 are empty), 8 x 4096 with norm 5.8, 1 x 2048 2.3.
template <class T>
__device__ __forceinline__ void q8_load(const T* p, int n, float (&v)[8]) {       // n: elements there are, 1 or more
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
        if constexpr (sizeof(T) == 2) e[i] = __builtin_bit_cast(uint16_t, (__bf16)v[i]);
        else e[i] = __float_as_uint(v[i]);
    }
    if (n >= 8) {
        __builtin_memcpy(p, e, 8 * sizeof(T));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = e[i];
    }
}

template <int OFF>
__device__ __forceinline__ double lane_xor(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    return __longlong_as_double((long long)((uint64_t)lane_xor_u<OFF>((uint32_t)(b >> 32)) << 32 | lane_xor_u<OFF>((uint32_t)b)));
}
__device__ __forceinline__ double wave_sum(double v) {
    v += lane_xor<1>(v);
    v += lane_xor<2>(v);
    v += lane_xor<4>(v);
    v += lane_xor<8>(v);
    v += lane_xor<16>(v);
    return v + lane_xor<32>(v);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, lane_xor_u<1>(v));
    v = max(v, lane_xor_u<2>(v));
    v = max(v, lane_xor_u<4>(v));
    v = max(v, lane_xor_u<8>(v));
    v = max(v, lane_xor_u<16>(v));
    return max(v, lane_xor_u<32>(v));
}

// The scale of values whose largest magnitude has these bits (those of a NaN are above all others), and its reciprocal, 0 where there is none.
__device__ __forceinline__ float q8_scale(uint32_t bits, float& inv) {
    if (bits >= 0x7F800000u) {
        inv = 0.f;
        return __uint_as_float(0x7FC00000u);
    }
    const float s = (float)((double)__uint_as_float(bits) / 127.);
    inv = s > 0.f ? (float)(1. / (double)s) : 0.f;
    return s;
}
// The nearest integer to v / s.  A scale of a few units of the smallest number is rounded so far that the quotient can be past 127.
__device__ __forceinline__ int q8_quotient(float v, float s) { return (int)rintf(fminf(fmaxf(v / s, -127.f), 127.f)); }
// Low bytes: the float32 quotients v[i] / s rounded to the nearest integer (0 where there is no scale).
template <int N>
__device__ __forceinline__ void q8_round(const float (&v)[N], float s, float inv, uint32_t (&b)[N]) {
    float far = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = v[i] * inv, r = t + 12582912.f;
        far = fmaxf(far, fabsf(t - (r - 12582912.f)));
        b[i] = inv > 0.f ? __float_as_uint(r) : 0u;
    }
    // (t is off by at most 127 * 2^-23.  A scale below 2^-128 has no finite reciprocal: t then says nothing.)
    if ((far > 0.49998f || inv > 3.4028235e38f) && inv > 0.f)
#pragma unroll
        for (int i = 0; i < N; ++i) b[i] = (uint32_t)q8_quotient(v[i], s);
}
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
}

// X, A: bits of the input's and the addend's elements.  kHeld: vectors of 8 that a thread keeps (0: rows too long for that are read
// again).  NORM: with an RMS norm in front.
template <class X, class A, bool NORM, int kHeld>
__global__ void __launch_bounds__(1024) k_q8_rows(const X* x, int64_t ldx, const A* __restrict__ add, int64_t ldadd, const float* __restrict__ gain, float eps,
                                                  int n, X* sum, int64_t ldsum, int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale) {
    __shared__ double sums[16];
    __shared__ uint32_t tops[16];
    const int64_t row = blockIdx.x;
    x += row * ldx;
    q += row * ldq;
    if (add) add += row * ldadd;
    if (sum) sum += row * ldsum;
    const int stride = blockDim.x * 8, first = threadIdx.x * 8, waves = blockDim.x >> 6;
    float held[kHeld ? kHeld : 1][8], gains[kHeld ? kHeld : 1][8];
    // f(i, at, v) for each of the thread's vectors
    auto vectors = [&](auto f) {
        if constexpr (kHeld > 0) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (first + i * stride < n) f(i, first + i * stride);
        } else {
            for (unsigned at = first; at < (unsigned)n; at += stride) f(0, (int)at);       // (past the end of a longest row: 2^31 and more)
        }
    };
    auto fetch = [&](int i, int at, bool summed) {                   // summed: what is in x's place is the sum already
        q8_load(x + at, n - at, held[i]);
        if (NORM && add && !summed) {
            float a[8];
            q8_load(add + at, n - at, a);
#pragma unroll
            for (int e = 0; e < 8; ++e) held[i][e] += a[e];
        }
    };
    // Rows longer than the registers are read again, from `sum` if it took the place of x (the host has no bf16 row of that length written
    // over itself, as its sum would be a rounded one).
    const bool over = NORM && sum == x;
    double rstd = 1.;
    if constexpr (NORM) {
        double squares = 0.;
        vectors([&](int i, int at) {
            fetch(i, at, false);
            if (kHeld) q8_load(reinterpret_cast<const uint32_t*>(gain) + at, n - at, gains[i]);
            if (sum) q8_store(sum + at, n - at, held[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) squares = fma((double)held[i][e], (double)held[i][e], squares);
        });
        squares = wave_sum(squares);
        if (waves > 1) {
            if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = squares;
            __syncthreads();
            squares = sums[0];
            for (int w = 1; w < waves; ++w) squares += sums[w];
        }
        rstd = 1. / sqrt(squares / n + (double)eps);
    }
    auto normed = [&](int i, int at) {                               // held[i] from x + add to what is rounded
        if constexpr (NORM) {
            if (!kHeld) q8_load(reinterpret_cast<const uint32_t*>(gain) + at, n - at, gains[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) held[i][e] = (float)((double)held[i][e] * rstd * (double)gains[i][e]);
        }
    };
    uint32_t top = 0;
    vectors([&](int i, int at) {
        if (!NORM || !kHeld) fetch(i, at, over);
        normed(i, at);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(held[i][e]) & 0x7FFFFFFFu);
    });
    top = wave_max(top);
    if (waves > 1) {
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
        __syncthreads();
        top = tops[0];
        for (int w = 1; w < waves; ++w) top = max(top, tops[w]);
    }
    float inv;
    const float s = q8_scale(top, inv);
    if (threadIdx.x == 0) scale[row] = s;
    vectors([&](int i, int at) {
        if (!kHeld) {
            fetch(i, at, over);
            normed(i, at);
        }
        uint32_t b[8];
        q8_round(held[i], s, inv, b);
        const uint32_t w[2] = {pack4(b[0], b[1], b[2], b[3]), pack4(b[4], b[5], b[6], b[7])};
        if (n - at >= 8) {
            __builtin_memcpy(q + at, w, 8);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n - at) q[at + e] = (int8_t)b[e];
        }
    });
}

template <class X, class A, bool NORM>
static void q8_rows(const void* x, int64_t ldx, const void* add, int64_t ldadd, const float* gain, float eps, int rows, int n, void* sum, int64_t ldsum,
                    int8_t* q, int64_t ldq, float* scale, hipStream_t stream) {
    // Vectors of 8 elements a thread, where only the largest is sought: one for few rows, as then the way through one row counts (8 x 14336 5.8 us for
    // 6.2); four for many long ones in bf16, for more workgroups a compute unit, in different phases.  us with four / two, inputs from memory: 2048 x
    // 10240 21.2 / 22.5, x 12288 24.7 / 24.3, x 14336 26.1 / 29.7, 4096 x 6144 22.6 / 23.5, x 8192 28.0 / 28.3, 8192 x 16384 89 / 101; below either bound
    // 4096 x 4096 17.1 / 15.8, 1100 x 8208 13.4 / 12.3, 2048 x 9216 19.7 / 19.0; fp32 2048 x 10240 23.7 / 23.6, 4096 x 14336 56.6 / 55.4,
    // 8192 x 16384 125 / 118.  A norm has two whatever the number of rows: its sum of squares has its order from that.
    const bool many_long = sizeof(X) == 2 && n >= 6144 && (int64_t)rows * n >= 20 << 20;
    const int vectors = NORM ? 2 : rows <= 128 ? 1 : many_long ? 4 : 2;
    const int threads = (int)std::min<int64_t>(1024, ((int64_t)n + vectors * 512 - 1) / (vectors * 512) * 64);
    // (a launch of 2^32 threads and more ends without an error and without its last workgroups)
    const int most = (int)(0xFFFFFFFFu / threads);
    auto launch = [&](auto kernel) {
        for (int64_t r = 0; r < rows; r += most)
            hipLaunchKernelGGL(kernel, dim3(std::min<int64_t>(most, rows - r)), dim3(threads), 0, stream, static_cast<const X*>(x) + r * ldx, ldx,
                               add ? static_cast<const A*>(add) + r * ldadd : nullptr, ldadd, gain, eps, n, sum ? static_cast<X*>(sum) + r * ldsum : nullptr,
                               ldsum, q + r * ldq, ldq, scale + r);
    };
    if (n <= 8 * threads) launch(k_q8_rows<X, A, NORM, 1>);
    else if (n <= 2 * 8 * threads) launch(k_q8_rows<X, A, NORM, 2>);
    else if (!NORM && n <= 4 * 8 * threads) launch(k_q8_rows<X, A, NORM, NORM ? 2 : 4>);
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
// then what they hold is rounded once more, to the new scale.  Bound by its phases, one after the other between barriers, of eight waves a compute
// unit (they wait 49 % of their cycles; vector instructions take 30 % of the busy ones) with stores of 4 bytes at a distance of 16 for
// values: 2048 rows of 8 heads of 128 in blocks of 32 12-13 us (1.0 TB/s), 5 rows of 8 heads of 64 4.8.
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
    __shared__ uint32_t most[kQ8Group];              // bits of a block's largest new magnitude: those of a NaN are above all others
    __shared__ float new_scale[kQ8Group], inverse[kQ8Group], ratio[kQ8Group];
    const int head = blockIdx.y, t = threadIdx.x, B = C.block, sh = __builtin_ctz(B);
    const bool values = blockIdx.z, turn = !values && cos;
    const Q8Seg seg = q8_find(S, blockIdx.x);
    const int p0 = (seg.pos0 / kQ8Group + (int)blockIdx.x - seg.unit0) * kQ8Group;      // first position of the group
    const int from = max(seg.pos0, p0), to = min(seg.pos0 + seg.n, p0 + kQ8Group);      // new ones among them
    const uint16_t* src = (values ? vrows : krows) + (int64_t)(seg.row0 - seg.pos0) * ld + (int64_t)head * HD;
    const int l = t & 15;
    uint16_t a[4][kPer], b[4][kPer];
    float cs[4][kPer], sn[4][kPer];
    if (t < kQ8Group) most[t] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int pos = p0 + i * 16 + (t >> 4);
        if (pos < from || pos >= to) continue;
        const uint16_t* p = src + (int64_t)pos * ld + l * kPer;
        __builtin_memcpy(a[i], p, sizeof a[i]);
        __builtin_memcpy(b[i], p + HD / 2, sizeof b[i]);
        if (turn) {
            __builtin_memcpy(cs[i], cos + (int64_t)pos * (HD / 2) + l * kPer, sizeof cs[i]);
            __builtin_memcpy(sn[i], sin + (int64_t)pos * (HD / 2) + l * kPer, sizeof sn[i]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 16 + (t >> 4), pos = p0 + r;
        uint32_t m = 0;
        if (pos >= from && pos < to) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                float x = bf16_to_f32(a[i][e]), y = bf16_to_f32(b[i][e]);
                if (turn) rotate_pair(x, y, cs[i][e], sn[i][e], x, y);
                rows[r][l * kPer + e] = x;
                rows[r][l * kPer + e + HD / 2] = y;
                m = max(m, max(__float_as_uint(x) & 0x7FFFFFFFu, __float_as_uint(y) & 0x7FFFFFFFu));
            }
        }
        m = max(m, lane_xor_u<1>(m));
        m = max(m, lane_xor_u<2>(m));
        m = max(m, lane_xor_u<4>(m));
        m = max(m, lane_xor_u<8>(m));
        if (l == 0 && m) atomicMax(&most[r >> sh], m);
    }
    __syncthreads();
    const size_t kvh = ((size_t)layer * C.n_seqs + seg.seq) * C.Hkv + head;
    if (t < kQ8Group >> sh) {
        const int b0 = p0 + t * B;                                   // the block's first position
        float* scales = (values ? C.vs : C.ks) + kvh * (C.cap >> sh);
        float s = 0.f, r = 1.f;
        if (b0 < to && b0 + B > from) {
            const uint32_t m = most[t];
            const float was = b0 < seg.pos0 ? scales[b0 >> sh] : 0.f;
            s = m >= 0x7F800000u || was != was ? __uint_as_float(0x7FC00000u) : fmaxf(was, __uint_as_float(m) / 127.f);
            r = s > 0.f ? was / s : s == s ? 1.f : 0.f;
            scales[b0 >> sh] = s;
        }
        new_scale[t] = s;
        inverse[t] = s > 0.f ? (float)(1. / (double)s) : 0.f;
        ratio[t] = r;
    }
    __syncthreads();
    // Keys: 16 columns of a position a thread; values: 4 positions of columns c and c + 16 (kept as q + 128: amusd_q8_attention.hip).
    // What a block that this call reaches held before is rounded again where its scale has grown.
    int8_t* out = (values ? C.v : C.k) + kvh * ((size_t)C.cap * HD);
    const int first_row = max(0, (from & -B) - p0), last_row = to - p0;           // rows that can change
    auto fresh = [&](int r) { return p0 + r >= from && p0 + r < to; };
    auto grown = [&](int r) { return p0 + r < from && ratio[r >> sh] != 1.f; };   // (1 in blocks that this call does not reach)
    auto again = [&](int old, int r) { return (uint32_t)(int)rintf((float)old * ratio[r >> sh]); };
    if (!values) {
        for (int i = first_row * (HD / 16) + t; i < last_row * (HD / 16); i += 256) {
            const int r = i / (HD / 16), c = i % (HD / 16) * 16;
            uint4* p = reinterpret_cast<uint4*>(out + q8_k_index(HD, p0 + r, c));
            uint32_t b[16];
            if (fresh(r)) {
                float v[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = rows[r][c + e];
                q8_round(v, new_scale[r >> sh], inverse[r >> sh], b);
            } else if (grown(r)) {
                const uint4 old = *p;
                const uint32_t o[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                for (int e = 0; e < 16; ++e) b[e] = again((int8_t)(o[e / 4] >> (e % 4 * 8)), r);
            } else {
                continue;
            }
            *p = uint4{pack4(b[0], b[1], b[2], b[3]), pack4(b[4], b[5], b[6], b[7]), pack4(b[8], b[9], b[10], b[11]), pack4(b[12], b[13], b[14], b[15])};
        }
    } else {
        // 4 rows of columns c and c + 16: two words of a lane's piece
        for (int i = t; i < (kQ8Group / 4) * (HD / 2); i += 256) {
            const int c = i % (HD / 2) / 16 * 32 + (i & 15), r = i / (HD / 2) * 4;
            if (r >= last_row || r + 4 <= first_row) continue;
            uint32_t* p = reinterpret_cast<uint32_t*>(out + q8_v_index(HD, p0 + r, c));
            uint32_t b[2][4] = {};
            const bool whole = fresh(r) && fresh(r + 3);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!whole) {
                    const uint32_t o = p[2 * h] ^ 0x80808080u;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        b[h][e] = o >> (8 * e);
                        if (grown(r + e)) b[h][e] = again((int8_t)b[h][e], r + e);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!fresh(r + e)) continue;
                    const int k = (r + e) >> sh;
                    const float v[1] = {rows[r + e][c + 16 * h]};
                    uint32_t q[1];
                    q8_round(v, new_scale[k], inverse[k], q);
                    b[h][e] = q[0];
                }
                p[2 * h] = pack4(b[h][0], b[h][1], b[h][2], b[h][3]) ^ 0x80808080u;
            }
        }
    }
    wait_vm<0>();          // a wave does not end with loads under way
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
// The values that rows of the cache stand for: 4 positions x 4 columns a thread, in words of 4 bytes (keys: of a position, values: of a
// column).  2048 positions of 8 heads of 128 6 us, 5 of heads of 64 3.5.
template <class T>
__global__ void __launch_bounds__(256) k_q8_read(amusd_q8_cache C, int layer, Q8Segs S, T* __restrict__ kout, T* __restrict__ vout, int64_t ld) {
    const int unit = blockIdx.z * gridDim.x + blockIdx.x;
    if (unit >= S.units) return;
    const Q8Seg& seg = q8_find(S, unit);
    const int p0 = (seg.pos0 / 4 + unit - seg.unit0) * 4, quads = C.Hkv * C.hd / 4;
    const bool values = blockIdx.y;
    T* out = (values ? vout : kout) + (int64_t)(seg.row0 - seg.pos0) * ld;
    for (int x = threadIdx.x; x < quads; x += blockDim.x) {
        const int head = x * 4 / C.hd, c = x * 4 % C.hd;
        const size_t kvh = ((size_t)layer * C.n_seqs + seg.seq) * C.Hkv + head;
        const float* scales = (values ? C.vs : C.ks) + kvh * (C.cap / C.block);
        const int8_t* p = (values ? C.v : C.k) + kvh * ((size_t)C.cap * C.hd);
        uint32_t w[4];                                       // keys: of position i; values: of column i
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = values ? *reinterpret_cast<const uint32_t*>(p + q8_v_index(C.hd, p0, c + i)) ^ 0x80808080u
                          : *reinterpret_cast<const uint32_t*>(p + q8_k_index(C.hd, p0 + i, c));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int pos = p0 + i;
            if (pos < seg.pos0 || pos >= seg.pos0 + seg.n) continue;
            const float s = scales[pos / C.block];
            T v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = (float)(int8_t)(values ? w[e] >> (8 * i) : w[i] >> (8 * e)) * s;
                if constexpr (sizeof(T) == 2) v[e] = __builtin_bit_cast(uint16_t, (__bf16)y);
                else v[e] = __float_as_uint(y);
            }
            __builtin_memcpy(out + (int64_t)pos * ld + x * 4, v, sizeof v);
        }
    }
    wait_vm<0>();
}

hipError_t launch_q8_read(const amusd_q8_cache& c, int layer, const Q8Segs& segs, void* k, void* v, int dtype, int64_t ld, hipStream_t stream) {
    Q8Segs S = segs;
    S.units = 0;                                             // groups of 4 positions
    for (int i = 0; i < S.n_seg; ++i) {
        S.s[i].unit0 = S.units;
        S.units += (S.s[i].pos0 + S.s[i].n - 1) / 4 - S.s[i].pos0 / 4 + 1;
    }
    constexpr int kMost = 1 << 22;                           // (2^32 threads along one side of a grid and more are cut off without an error)
    const dim3 grid(std::min(S.units, kMost), 2, (S.units + kMost - 1) / kMost);
    if (dtype == AMUSD_DTYPE_BF16)
        hipLaunchKernelGGL(k_q8_read<uint16_t>, grid, dim3(256), 0, stream, c, layer, S, static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), ld);
    else
        hipLaunchKernelGGL(k_q8_read<uint32_t>, grid, dim3(256), 0, stream, c, layer, S, static_cast<uint32_t*>(k), static_cast<uint32_t*>(v), ld);
    return hipGetLastError();
}

// ---------------------------------------------------------------- weights to 8 bits, in operand order
// One wave a row of the source: finds its scale (unless it is given), then writes the feature's bytes.  Row i is feature first + i
// of the matrix or, in a gated one, of its gate or up projection (part 1, 2).
template <class T>
__global__ void __launch_bounds__(64) k_q8_matrix(uint4* __restrict__ frag, float* __restrict__ scale, const T* __restrict__ w, int64_t ld,
                                                  const float* __restrict__ given, int k, int first, int part) {
    const int i = blockIdx.x, f = first + i, lane = threadIdx.x;
    const int tile = part ? (f >> 4) * 2 + part - 1 : f >> 4, r = f & 15;
    w += i * ld;
    float s = 0.f, inv = 0.f;
    auto value = [&](int c) {
        if constexpr (sizeof(T) == 2) return bf16_to_f32(w[c]);
        else return __uint_as_float(w[c]);
    };
    if constexpr (sizeof(T) > 1) {
        uint32_t top = 0;
        for (int c = lane; c < k; c += 64) top = max(top, __float_as_uint(value(c)) & 0x7FFFFFFFu);
        s = q8_scale(wave_max(top), inv);
        if (lane == 0) scale[tile * 16 + r] = s;
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
            else b = inv > 0.f ? (int8_t)q8_quotient(value(c), s) : (int8_t)0;
        }
        out[(((size_t)tile * kblocks + kb) * 64 + (lane >> 4) * 16 + r) * 16 + (lane & 15)] = b;
    }
}

hipError_t launch_q8_matrix(const amusd_q8_matrix& m, const void* w, int dtype, int64_t ld, const float* scale, int rows, int first, int part,
                            hipStream_t stream) {
    auto go = [&](auto kernel, auto* src) {
        constexpr int kMost = 1 << 25;                       // (2^32 threads and more are cut off without an error)
        for (int r = 0; r < rows; r += kMost)
            hipLaunchKernelGGL(kernel, dim3(std::min(kMost, rows - r)), dim3(64), 0, stream, const_cast<uint4*>(m.frag), const_cast<float*>(m.scale),
                               src + r * ld, ld, scale ? scale + r : nullptr, m.k, first + r, part);
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

// (in floating point: the product need not fit 64 bits)
static double q8_cache_bytes(int n_layers, int n_seqs, int n_kv_heads, int head_dim, int capacity) {
    return 2. * n_layers * n_seqs * n_kv_heads * head_dim * capacity;
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
    if (q8_cache_bytes(n_layers, n_seqs, n_kv_heads, head_dim, capacity) > kQ8MaxBytes) return hipErrorOutOfMemory;
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
    // (rows longer than the registers read add a second time, after their sum was stored)
    if (sum && sum == add) return report(AMUSD_E_ARG, "q8_rmsnorm: the sum takes the place of x or of neither");
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
    if (n < 1 || k < 1 || ld < k || (gated && n % 2) || n >= kQ8MaxFeatures || k > kQ8MaxK || (double)(n - 1) * (double)ld > kQ8MaxBytes)
        return report(AMUSD_E_ARG, "q8_matrix: bad sizes");
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
        (void)hipGetLastError();          // reported here, not by the next launch
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
        capacity > kQ8MaxPositions || q8_cache_bytes(n_layers, n_seqs, n_kv_heads, head_dim, capacity) > kQ8MaxBytes)
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
        (void)hipGetLastError();
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
    if ((int64_t)S.rows * c->G > 1 << 19) return report(AMUSD_E_ARG, "q8_attention: too many rows");      // a grid's second side ends at 65535
    Q8_TRY(launch_q8_attention(*c, layer, S, q, ldq, scale, rope_cos, rope_sin, out, ldo, static_cast<hipStream_t>(hip_stream)));
    return AMUSD_OK;
}

}  // extern "C"
