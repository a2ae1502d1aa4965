// Attention of rows over the cache in 8 bits.
//
// A tile is 16 (row, head) pairs of one sequence and kv head: they share its keys.  Queries are rotated and held in 16 bits
// relative to their largest component, as two planes of 8-bit integers: their products with the keys are then exact integers,
// half as many matrix instructions as half precision would take, and no key is converted.  The rounding of a query moves a score
// by at most 2^-16 of (its largest component times the sum of the key's magnitudes).  Softmax weights carry the scales of their
// values, are brought below 2^15 by a power of two and rounded to half (11 bits); values are exact in half.  Maxima, sums and
// results are fp32.  One half a weight, where two would take twice the products of weights and values: the result is rounded to bf16, an
// eighth as fine, and lies as far from 64 bits as one whose weights are fp32 (0.0017 to 0.0018 of its norm for 0.0016 to 0.0017).
//
// Keys are taken in chunks at absolute positions, whose sums start anew and are merged in order, whoever does it: with few rows a
// wave takes one chunk and a second launch merges (k_q8_att_part, k_q8_att_merge), with many a wave walks all of them
// (k_q8_att_whole).  What a chunk's sums depend on is only what the row may see.  So a row's bits depend neither on how many
// rows a call has nor on the form; they do on the chunks (q8_attention_plan).
//
// Bound by the instructions between the two products (vector instructions take 76 to 96 % of the cycles in which a compute unit is busy: scales,
// 2^x, maxima, roundings, bytes to halves).  Measured (MI355X; part + merge, or whole), 8B heads: 16 rows behind 16384 keys 22 + 8 us (34 MB of cache),
// 8 rows behind 2048 13 in all, 1111 rows behind 1024 in blocks of 64 87 after a pause, 77 in a long run of them (the clock rises), 2048 rows of
// a prompt 84-86; 1B heads: 1 row behind 512 5.6 + 4.
#include <algorithm>

#include "amusd_math.h"
#include "amusd_q8.h"

#pragma clang fp contract(off)

namespace amusd {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

constexpr int kPlane = 32512;                    // 127 * 256: a query's largest component in its 16 bits

// Products of integers are below 2^29, so with a key's scale of 2^99 they are past float32, whatever the query's factor; and a factor below
// float32's normal numbers, which is held at the smallest of them, matters from a scale of 2^90 on.  Scales of a chunk that holds one from kHugeKey on
// (seen or not: powers of two change no bits, but for keys 2^150 times smaller) are then taken down by kLowKey and the factor up, or the
// sums up again where the factor is so large that the score itself is past float32.
constexpr float kHugeKey = 0x1p64f, kLowKey = 0x1p-32f, kLargeQs = 0x1p60f;

struct Q8Query {                                 // a launch's constants
    const uint16_t* q;
    int64_t ldq;
    uint16_t* out;
    int64_t ldo;
    const float *cos, *sin;
    float scale2;                                // scores in units of log2
};

// One tile's queries, the way the score product takes them: lane l has pair l % 16 and columns 16 * (l / 16) .. of each 64.
template <int HD>
struct Tile {
    uint4 hi[HD / 64], lo[HD / 64];
    float qs;                                    // score (in units of log2) per unit of the integer product, without the key's scale; positive
    float low_qs;                                // .. for keys' scales that were taken down by kLowKey, where that is smaller than kLargeQs
    int pos;                                     // the pair's row's position (the last key that it sees); -1: no pair
};

template <int HD>
__device__ __forceinline__ Tile<HD> load_tile(const amusd_q8_cache& C, const Q8Query& Q, const Q8Seg& seg, int kvh, int tile) {
    Tile<HD> T;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int p = tile * 16 + (lane & 15), pairs = seg.n * C.G;
    const int pc = min(p, pairs - 1);
    const int row = pc / C.G, pos = seg.pos0 + row;
    T.pos = p < pairs ? pos : -1;
    const uint16_t* src = Q.q + (int64_t)(seg.row0 + row) * Q.ldq + (int64_t)(kvh * C.G + pc % C.G) * HD;
    float x[HD / 64][16];
#pragma unroll
    for (int f = 0; f < HD / 64; ++f) {
        uint16_t b[16];
        __builtin_memcpy(b, src + f * 64 + g * 16, 32);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[f][i] = bf16_to_f32(b[i]);
    }
    if (Q.cos) {
        if constexpr (HD == 128) {               // pairs (i, i + 64) are in one lane
            float c[16], s[16];
            __builtin_memcpy(c, Q.cos + (int64_t)pos * 64 + g * 16, 64);
            __builtin_memcpy(s, Q.sin + (int64_t)pos * 64 + g * 16, 64);
#pragma unroll
            for (int i = 0; i < 16; ++i) rotate_pair(x[0][i], x[1][i], c[i], s[i], x[0][i], x[1][i]);
        } else {                                 // (i, i + 32): in the lanes 32 apart
            float c[16], s[16];
            __builtin_memcpy(c, Q.cos + (int64_t)pos * 32 + (g & 1) * 16, 64);
            __builtin_memcpy(s, Q.sin + (int64_t)pos * 32 + (g & 1) * 16, 64);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float other = lane_xor<32>(x[0][i]);
                float a, b;
                if (g < 2) rotate_pair(x[0][i], other, c[i], s[i], a, b);
                else rotate_pair(other, x[0][i], c[i], s[i], b, a);
                x[0][i] = a;
            }
        }
    }
    uint32_t most = 0;
#pragma unroll
    for (int f = 0; f < HD / 64; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(x[f][i]) & 0x7FFFFFFFu);
    most = max(most, lane_xor_u<16>(most));
    most = max(most, lane_xor_u<32>(most));
    const bool bad = most >= 0x7F800000u;
    const float m = bad ? 0.f : __uint_as_float(most);
    // A largest component below 1e-34 has no finite reciprocal (kPlane times it): such queries are taken up first, by a power of two.
    const float up = m < 0x1p-64f ? 0x1p64f : 1.f, step = m * up / (float)kPlane;
    const float inv = m > 0.f ? (float)kPlane / (m * up) : 0.f;
    // (the factors are not 0: 0 times -infinity)
    T.qs = bad ? __uint_as_float(0x7FC00000u) : fmaxf(step * Q.scale2 / up, 1.17549435e-38f);
    T.low_qs = bad ? T.qs : fmaxf(step * (Q.scale2 * (1.f / kLowKey / up)), 1.17549435e-38f);
#pragma unroll
    for (int f = 0; f < HD / 64; ++f) {
        uint32_t hi[4] = {}, lo[4] = {};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int v = bad ? 0 : min(max((int)rintf(x[f][i] * up * inv), -kPlane), kPlane);
            const int h = (v + 128) >> 8;
            hi[i / 4] |= (uint32_t)(h & 255) << (i % 4 * 8);
            lo[i / 4] |= (uint32_t)((v - h * 256) & 255) << (i % 4 * 8);
        }
        T.hi[f] = uint4{hi[0], hi[1], hi[2], hi[3]};
        T.lo[f] = uint4{lo[0], lo[1], lo[2], lo[3]};
    }
    return T;
}

__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

// Four bytes of values, which are kept as v + 128, as the halves 1152 + v: 1024 + u is the half whose low byte is u.  What the 1152 add
// to the sums is taken off again at a chunk's end, with the sum of the weights that one more matrix instruction gives: a
// third of the instructions of a subtraction for every value, and the sums, ten times larger so, are rounded a thousand times finer than
// the values themselves were.
__device__ __forceinline__ void bytes_to_half(uint32_t u, uint32_t& lo, uint32_t& hi) {
    lo = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u);
    hi = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
}

// A chunk's sums for 16 pairs: lane l has columns dt * 16 + 4 * (l / 16) + e of pair l % 16.
template <int HD>
struct Sums {
    v4f acc[HD / 16], weights;                   // weights: their sum (as scaled for the product), the same in all four
    float ref, den;
};

// Scales of a chunk's keys and values, 8 keys a lane: two loads of the wave have those of a longest chunk.
constexpr int kMaxChunk = 512;
enum { kPost, kBack, kQs, kLowQs, kRare };            // what each lane keeps apart, as it is rarely read
constexpr int kWalkLds = 2 * kMaxChunk + kRare * 64;     // floats: a chunk's scales, and that
struct Scales {
    v4f k[2], v[2];
};
template <bool PER_TOKEN>
__device__ __forceinline__ Scales load_scales(const amusd_q8_cache& C, size_t kvh, int c0) {
    Scales s;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int pos = c0 + i * 256 + (threadIdx.x & 63) * 4;
        s.k[i] = s.v[i] = v4f{0.f, 0.f, 0.f, 0.f};
        if (pos < C.cap && pos < c0 + C.chunk) {
            const size_t at = kvh * (C.cap / C.block);
            if constexpr (PER_TOKEN) {
                s.k[i] = *reinterpret_cast<const v4f*>(C.ks + at + pos);
                s.v[i] = *reinterpret_cast<const v4f*>(C.vs + at + pos);
            } else {
                const int b = pos >> __builtin_ctz(C.block);
                const float k = C.ks[at + b], v = C.vs[at + b];
                s.k[i] = v4f{k, k, k, k};
                s.v[i] = v4f{v, v, v, v};
            }
        }
    }
    return s;
}

// A step takes 64 keys: two blocks of 32, the values' unit.  (A wave issues an instruction every 4 to 12 clocks, dependent ones
// the more slowly: one block a step took 0.82 us for a wave alone on its SIMD, two take 1.06.)
constexpr int kStep = 64;
template <int HD>
struct Keys {
    uint4 k[4][HD / 64];
};
template <int HD>
struct Values {
    uint4 v[2][HD / 32];
};
template <int HD>
__device__ __forceinline__ Keys<HD> load_keys(const amusd_q8_cache& C, size_t kvh, int b) {
    const uint4* K = reinterpret_cast<const uint4*>(C.k + kvh * ((size_t)C.cap * HD)) + (size_t)(b >> 4) * (HD / 64) * 64 + (threadIdx.x & 63);
    Keys<HD> B;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int f = 0; f < HD / 64; ++f) B.k[t][f] = K[(t * (HD / 64) + f) * 64];
    return B;
}
template <int HD>
__device__ __forceinline__ Values<HD> load_values(const amusd_q8_cache& C, size_t kvh, int b) {
    const uint4* V = reinterpret_cast<const uint4*>(C.v + kvh * ((size_t)C.cap * HD)) + (size_t)(b >> 5) * (HD / 32) * 64 + (threadIdx.x & 63);
    Values<HD> B;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) B.v[h][d] = V[(h * (HD / 32) + d) * 64];
    return B;
}

// Weights are lifted by at most 2^60 with their own exponent, as 2^x has to leave small ones; where the values' scales want more (below 2^-50, or
// from 2^71 on) the rest goes with the scale.  Numerators of such large values would be past float32 before they are divided: they are
// kept kDown times what they are, which a denominator below 0 says.
constexpr int kMaxLift = 60;
constexpr float kDown = 0x1p-40f;

constexpr float kSlack = 4.f;                    // a maximum may exceed its reference by 2^4 before the sums are rescaled

// A step's scores, without the query's factor.
template <int HD>
__device__ __forceinline__ void step_scores(const Keys<HD>& K, const Tile<HD>& T, const v4f* ks, float (&sc)[4][4]) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        v4i hi = {}, lo = {};
#pragma unroll
        for (int f = 0; f < HD / 64; ++f) {
            hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, K.k[t][f]), __builtin_bit_cast(v4i, T.hi[f]), hi, 0, 0, 0);
            lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, K.k[t][f]), __builtin_bit_cast(v4i, T.lo[f]), lo, 0, 0, 0);
        }
        const v4f scale = ks[t * 4];
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[t][e] = (float)(hi[e] * 256 + lo[e]) * scale[e];
    }
}

// The lane, such that addresses made of it are found where they are used, once a chunk, and not kept in registers through its steps.
__device__ __forceinline__ int lane_anew() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}
// The reference is the largest product of a score and the factor, rounded; what the exponents are taken from is the product as it is (one
// instruction).  From 2^24 on the two differ by 1 and more, from 2^30 by what a half cannot hold: such pairs' products are rounded too.
__device__ __forceinline__ bool large_score(float ref) { return fabsf(ref) >= 0x1p23f && ref != -INFINITY; }

__device__ __forceinline__ float& rare_of(float* lds, int what) { return lds[2 * kMaxChunk + what * 64 + lane_anew()]; }

// .. and its weights, as the values' product takes them, 2^lift (RARE: and post) times what they are.  MASK: some pair does not see all of
// its keys.  left: keys from the step's first one up to the last that the lane's pair sees.
template <int HD, bool MASK, bool RARE>
__device__ __forceinline__ void step_exps(const float (&sc)[4][4], float qs, const v4f* vs, float lift, float post, int left, Sums<HD>& S, uint4 (&out)[2]) {
    const int g4 = (threadIdx.x & 48) >> 2;
    const float at = S.ref == -INFINITY ? 0.f : S.ref - lift;
    const bool far = RARE && large_score(S.ref);
    float sum[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        v4f scale = vs[t * 4];
        if (RARE) scale *= post;
        float p[4], w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = fmaf(sc[t][e], qs, -at);
            p[e] = pow2(far ? (sc[t][e] * qs - S.ref) + lift : x);
            w[e] = p[e] * scale[e];
            if (MASK && t * 16 + g4 + e > left) w[e] = 0.f;          // (whatever its value's scale is)
        }
        sum[t] = (p[0] + p[1]) + (p[2] + p[3]);
        auto two = [](float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, h2)); };
        (t & 1 ? out[t >> 1].z : out[t >> 1].x) = two(w[0], w[1]);
        (t & 1 ? out[t >> 1].w : out[t >> 1].y) = two(w[2], w[3]);
    }
    S.den += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}
template <int HD, bool MASK>
__device__ __forceinline__ void step_weights(float (&sc)[4][4], float qs, const v4f* vs, float lift, bool& rare, float* lds, int left, Sums<HD>& S,
                                             uint4 (&out)[2]) {
    const int g4 = (threadIdx.x & 48) >> 2;
    float top[4];
    if (MASK && __builtin_expect(rare, 0)) {
        const float back = rare_of(lds, kBack);
        qs = rare_of(lds, kQs);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[t][e] *= back;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (MASK && t * 16 + g4 + e > left) sc[t][e] = -INFINITY;
        top[t] = fmaxf(fmaxf(sc[t][0], sc[t][1]), fmaxf(sc[t][2], sc[t][3]));
    }
    float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    most = fmaxf(most, lane_xor<16>(most));
    most = fmaxf(most, lane_xor<32>(most)) * qs;
    const bool grow = most - S.ref > kSlack;                 // (the difference: their sum would be rounded, up as well)
    if (__any(grow)) {
        const float ref = grow ? most : S.ref, shrink = pow2(S.ref - (ref == -INFINITY ? 0.f : ref));    // (1 where nothing grows, or 0 * 0)
        S.ref = ref;
        S.den *= shrink;
        S.weights *= shrink;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) S.acc[d] *= shrink;
        if (__builtin_expect(!rare && __any(large_score(ref)), 0)) {         // from here on the chunk's steps are of the rare kind
            rare = true;
            rare_of(lds, kPost) = rare_of(lds, kBack) = 1.f;
            rare_of(lds, kQs) = qs;
            return step_exps<HD, true, true>(sc, qs, vs, lift, 1.f, left, S, out);
        }
    }
    if (!MASK || __builtin_expect(!rare, 1)) step_exps<HD, MASK, false>(sc, qs, vs, lift, 1.f, left, S, out);
    else step_exps<HD, MASK, true>(sc, qs, vs, lift, rare_of(lds, kPost), left, S, out);
}

// sums so far and a chunk's: how both are weighed.  down: whether the numerators so far are kDown times what they are.
__device__ __forceinline__ void merge_weights(float& ref, float& den, bool& down, float cref, float cden, float& a, float& b) {
    const float to = fmaxf(ref, cref), at = to == -INFINITY ? 0.f : to;
    a = pow2(ref - at);
    b = pow2(cref - at);
    den = fmaf(den, a, fabsf(cden) * b);
    ref = to;
    if (cden < 0.f) {
        if (!down) a *= kDown;
        down = true;
    } else if (down) {
        b *= kDown;
    }
}

// Walks the keys [begin, end) (multiples of a step; begin a chunk's) and calls done(chunk's first key, its sums) at the end of each chunk.
// The next step's keys are fetched as soon as a step's scores are found, its values behind the values' product: into the registers that
// those leave free.  least: the last key that all pairs see.
template <int HD, bool PER_TOKEN, class Done>
__device__ __forceinline__ void walk(const amusd_q8_cache& C, size_t kvh, const Tile<HD>& T, int least, int begin, int end, Keys<HD> K, Scales sc,
                                     float* lds, Done&& done) {
    const int g = (threadIdx.x & 63) >> 4;
    v4f* const kl = reinterpret_cast<v4f*>(lds);
    v4f* const vl = reinterpret_cast<v4f*>(lds + kMaxChunk);
    rare_of(lds, kLowQs) = T.low_qs;
    Sums<HD> S;
    float lift = 0.f;
    bool far = false;                            // the chunk's steps are of the rare kind
    int c0 = begin;
    auto chunk_begin = [&](int b) {
        c0 = b;
        const int lane = lane_anew(), g = lane >> 4;
        __builtin_amdgcn_wave_barrier();
        float all = 0.f, keys = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            keys = fmaxf(keys, fmaxf(fmaxf(sc.k[i][0], sc.k[i][1]), fmaxf(sc.k[i][2], sc.k[i][3])));
            vl[i * 64 + lane] = sc.v[i];
            all = fmaxf(all, fmaxf(fmaxf(sc.v[i][0], sc.v[i][1]), fmaxf(sc.v[i][2], sc.v[i][3])));
        }
        __builtin_amdgcn_wave_barrier();
        // The power of two that brings each pair's weights below 2^15: the largest scale among the values that it sees here to [2^10, 2^11).
        float most = 0.f;
        if (least >= c0 + C.chunk - 1) {                    // (the same in all lanes)
            most = fmaxf(all, lane_xor<1>(all));
            most = fmaxf(most, lane_xor<2>(most));
            most = fmaxf(most, lane_xor<4>(most));
            most = fmaxf(most, lane_xor<8>(most));
        } else {
            for (int k = g * 4; k < min(C.chunk, end - c0); k += 16) {
                const v4f s = vl[k >> 2];
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, c0 + k + e <= T.pos ? s[e] : 0.f);
            }
        }
        most = fmaxf(most, lane_xor<16>(most));
        most = fmaxf(most, lane_xor<32>(most));
        const int all_of_it = most > 0.f ? 137 - (int)(__float_as_uint(most) >> 23) : 0, here = min(max(all_of_it, -kMaxLift), kMaxLift);
        lift = (float)here;
        far = __any(keys >= kHugeKey || all_of_it != here);
        if (__builtin_expect(far, 0)) {
            const bool huge = __any(keys >= kHugeKey), low = T.qs < kLargeQs;
            rare_of(lds, kPost) = __uint_as_float((uint32_t)(127 + all_of_it - here) << 23);
            rare_of(lds, kBack) = huge && !low ? 1.f / kLowKey : 1.f;
            rare_of(lds, kQs) = huge && low ? rare_of(lds, kLowQs) : T.qs;
#pragma unroll
            for (int i = 0; i < 2; ++i) sc.k[i] *= huge ? kLowKey : 1.f;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) kl[i * 64 + lane] = sc.k[i];
        __builtin_amdgcn_wave_barrier();
        S.ref = -INFINITY;
        S.den = 0.f;
        S.weights = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) S.acc[d] = v4f{0.f, 0.f, 0.f, 0.f};
    };
    Values<HD> V = load_values<HD>(C, kvh, begin);
    for (int b = begin; b < end; b += kStep) {
        if (!(b & (C.chunk - 1))) chunk_begin(b);
        const bool more = b + kStep < end, ends = !((b + kStep) & (C.chunk - 1)) || !more;
        const v4f* const ks = kl + ((b - c0) >> 2) + g;
        const v4f* const vs = vl + ((b - c0) >> 2) + g;
        float sc4[4][4];
        step_scores<HD>(K, T, ks, sc4);
        if (more) K = load_keys<HD>(C, kvh, b + kStep);
        if (ends && more) sc = load_scales<PER_TOKEN>(C, kvh, b + kStep);
        uint4 w[2];
        if (!far && b + kStep - 1 <= least) step_weights<HD, false>(sc4, T.qs, vs, lift, far, lds, kStep, S, w);
        else step_weights<HD, true>(sc4, T.qs, vs, lift, far, lds, T.pos - b, S, w);
        const uint4 ones{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            S.weights = BF16::mfma_att(ones, w[h], S.weights);
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) {
                uint4 a, c;
                bytes_to_half(V.v[h][d].x, a.x, a.y);
                bytes_to_half(V.v[h][d].y, a.z, a.w);
                bytes_to_half(V.v[h][d].z, c.x, c.y);
                bytes_to_half(V.v[h][d].w, c.z, c.w);
                S.acc[2 * d] = BF16::mfma_att(a, w[h], S.acc[2 * d]);
                S.acc[2 * d + 1] = BF16::mfma_att(c, w[h], S.acc[2 * d + 1]);
                __builtin_amdgcn_sched_barrier(0);           // (all values converted first would take 64 registers)
            }
        }
        if (more) V = load_values<HD>(C, kvh, b + kStep);
        if (ends) {
            const float down = __uint_as_float((uint32_t)(127 - (int)lift) << 23);
            S.den += lane_xor<16>(S.den);
            S.den += lane_xor<32>(S.den);
            S.den *= down;
#pragma unroll
            for (int d = 0; d < HD / 16; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) S.acc[d][e] = fmaf(-1152.f, S.weights[e], S.acc[d][e]) * down;
            if (__builtin_expect(far, 0)) {
                const float more = rare_of(lds, kPost);
                const float rest = more < 1.f ? kDown / more : 1.f / more;          // (powers of two)
                if (more < 1.f) S.den = -S.den;
#pragma unroll
                for (int d = 0; d < HD / 16; ++d) S.acc[d] *= rest;
            }
            done(c0, S);
        }
    }
}

__device__ __forceinline__ int find_seg(const Q8Segs& S, int unit) {
    int i = 0;
    while (i + 1 < S.n_seg && unit >= S.s[i + 1].unit0) ++i;
    return i;
}

// What a wave works on: tile `tile` of all sequences' tiles.
struct Work {
    const Q8Seg* seg;
    int local, least, last;                     // the sequence's tile; the last key that its first pair sees, and that any does
    size_t head;
};
__device__ __forceinline__ Work find_work(const amusd_q8_cache& C, const Q8Segs& S, int layer, int tile, int kvh) {
    Work w;
    w.seg = &S.s[find_seg(S, tile)];
    w.local = tile - w.seg->unit0;
    w.least = w.seg->pos0 + w.local * 16 / C.G;
    w.last = w.seg->pos0 + min((w.local * 16 + 15) / C.G, w.seg->n - 1);
    w.head = ((size_t)layer * C.n_seqs + w.seg->seq) * C.Hkv + kvh;
    return w;
}

// A wave: a tile, one chunk.  Its sums go to memory.
template <int HD, bool PER_TOKEN>
__global__ void __launch_bounds__(64, HD == 64 ? 3 : 1) k_q8_att_part(amusd_q8_cache C, int layer, Q8Segs S, Q8Query Q, int tile0) {
    __shared__ float lds[kWalkLds];
    const int kvh = blockIdx.x, tile = tile0 + blockIdx.y, chunk = blockIdx.z, c0 = chunk * C.chunk;       // a kv head's waves on one XCD
    const Work W = find_work(C, S, layer, tile, kvh);
    if (c0 > W.last) return;
    const size_t head = W.head;
    const Keys<HD> keys = load_keys<HD>(C, head, c0);
    const Scales sc = load_scales<PER_TOKEN>(C, head, c0);
    const Tile<HD> T = load_tile<HD>(C, Q, *W.seg, kvh, W.local);
    walk<HD, PER_TOKEN>(C, head, T, W.least, c0, min(c0 + C.chunk, (W.last + kStep) / kStep * kStep), keys, sc, lds, [&](int, const Sums<HD>& sums) {
        const int lane = lane_anew(), g = lane >> 4, pair = lane & 15;
        float* out = C.part + (((size_t)blockIdx.y * C.Hkv + kvh) * C.max_chunks + chunk) * ((HD + 2) * 16);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) out[(d * 16 + g * 4 + e) * 16 + pair] = sums.acc[d][e];
        if (g == 0) {
            out[HD * 16 + pair] = sums.ref;
            out[(HD + 1) * 16 + pair] = sums.den;
        }
    });
    wait_vm<0>();          // a wave does not end with loads under way
}

__device__ __forceinline__ uint16_t q8_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

// A workgroup merges HD / 8 columns of a tile: thread (column, pair).  How each chunk is weighed follows from the references alone: found
// for up to 64 chunks at a time by as many threads, while the sums are on their way; those are then added up in order.
template <int HD>
__global__ void __launch_bounds__(HD * 2) k_q8_att_merge(amusd_q8_cache C, Q8Segs S, Q8Query Q, int tile0) {
    constexpr int kAtOnce = 16, kRound = 64, kPart = (HD + 2) * 16, kThreadsOf = HD * 2;
    __shared__ float refs[kRound][16], dens[kRound][16], upto[kRound + 1][16];
    __shared__ v4f how[kRound][16];                          // what is done with a chunk: the sums before it times [0], its own times [1]; [2] its denominator
    __shared__ int big[kThreadsOf / 64];                     // pairs (a bit each) with numerators that are kDown times what they are, of a wave's chunks
    const int kvh = blockIdx.x, tile = tile0 + blockIdx.y, t = threadIdx.x;
    const Q8Seg& seg = S.s[find_seg(S, tile)];
    const int first = (tile - seg.unit0) * 16, pairs = min(16, seg.n * C.G - first);
    const int pair = t & 15, col = blockIdx.z * (HD / 8) + (t >> 4);
    auto chunks_of = [&](int p) { return (seg.pos0 + (first + p) / C.G) / C.chunk + 1; };
    const int mine = chunks_of(min(pair, pairs - 1)), most = chunks_of(pairs - 1);
    const float* const part = C.part + ((size_t)blockIdx.y * C.Hkv + kvh) * C.max_chunks * kPart;
    float ref = -INFINITY, den = 0.f, acc = 0.f;             // ref: the largest of the rounds before (threads 0 to 15)
    bool down = false;
    for (int c0 = 0; c0 < most; c0 += kRound) {
        const int n = min(kRound, most - c0);
        float x[kAtOnce];
        auto fetch = [&](int from) {
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) x[i] = part[(size_t)min(from + i, most - 1) * kPart + col * 16 + pair];
        };
        unsigned long long here = 0;
        for (int i = t; i < n * 32; i += kThreadsOf) {       // (references and denominators lie together)
            const float v = part[(size_t)(c0 + (i >> 5)) * kPart + HD * 16 + (i & 31)];
            (i & 16 ? dens : refs)[i >> 5][pair] = v;
            here |= __ballot((i & 16) && v < 0.f && c0 + (i >> 5) < mine);
        }
        if ((t & 63) == 0) big[t >> 6] = (int)((here >> 16 | here >> 48) & 0xFFFF);
        fetch(c0);
        __syncthreads();
        if (t < 16) {
            upto[0][t] = ref;
            for (int c = 0; c < n; c += 16) {
                float r[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) r[i] = refs[min(c + i, n - 1)][t];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    ref = fmaxf(ref, r[i]);
                    if (c + i < n) upto[c + i + 1][t] = ref;
                }
            }
        }
        __syncthreads();
        int all_big = 0;
#pragma unroll
        for (int w = 0; w < kThreadsOf / 64; ++w) all_big |= big[w];
        if (!down && (all_big >> pair & 1)) {
            down = true;
            acc *= kDown;
        }
        for (int i = t; i < n * 16; i += kThreadsOf) {
            const int c = i >> 4;
            const float to = upto[c + 1][pair], at = to == -INFINITY ? 0.f : to;
            const float b = pow2(refs[c][pair] - at);
            const float d = dens[c][pair];
            how[c][pair] = v4f{pow2(upto[c][pair] - at), down && !(d < 0.f) ? b * kDown : b, fabsf(d) * b, 0.f};
        }
        __syncthreads();
        for (int c = 0; c < n; c += kAtOnce) {
            if (c) fetch(c0 + c);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const v4f h = how[min(c + i, n - 1)][pair];
                const float d = fmaf(den, h[0], h[2]), s = fmaf(acc, h[0], x[i] * h[1]);
                const bool sees = c0 + c + i < mine && c + i < n;       // (a chunk that the pair sees nothing of is not merged)
                den = sees ? d : den;
                acc = sees ? s : acc;
            }
        }
        if (c0 + kRound < most) __syncthreads();
    }
    wait_vm<0>();
    if (pair >= pairs) return;
    const int row = (first + pair) / C.G, head = kvh * C.G + (first + pair) % C.G;
    Q.out[(int64_t)(seg.row0 + row) * Q.ldo + (int64_t)head * HD + col] = q8_bf16(acc / den * (down ? 1.f / kDown : 1.f));
}

// A wave: a tile, all chunks.  The sums over the chunks so far wait in LDS, where they are touched once a chunk.
template <int HD, bool PER_TOKEN>
__global__ void __launch_bounds__(64, HD == 64 ? 3 : 2) k_q8_att_whole(amusd_q8_cache C, int layer, Q8Segs S, Q8Query Q) {
    __shared__ float lds[kWalkLds];
    __shared__ v4f all[HD / 16][64];
    const int kvh = blockIdx.x, lane = threadIdx.x;                             // a kv head's waves on one XCD, the longest first
    const Work W = find_work(C, S, layer, gridDim.y - 1 - blockIdx.y, kvh);
    const Tile<HD> T = load_tile<HD>(C, Q, *W.seg, kvh, W.local);
    __builtin_amdgcn_sched_barrier(0);
    const Keys<HD> keys = load_keys<HD>(C, W.head, 0);
    const Scales sc = load_scales<PER_TOKEN>(C, W.head, 0);
    float ref = -INFINITY, den = 0.f;
    bool down = false;
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) all[d][lane] = v4f{0.f, 0.f, 0.f, 0.f};
    walk<HD, PER_TOKEN>(C, W.head, T, W.least, 0, (W.last + kStep) / kStep * kStep, keys, sc, lds, [&](int c0, const Sums<HD>& part) {
        if (c0 > T.pos) return;                             // a chunk that the pair sees nothing of is not merged
        const int lane = lane_anew();
        float a, b;
        merge_weights(ref, den, down, part.ref, part.den, a, b);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) {
            v4f v = all[d][lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(v[e], a, part.acc[d][e] * b);
            all[d][lane] = v;
        }
    });
    wait_vm<0>();
    if (T.pos < 0) return;
    const int own = lane_anew(), pair = W.local * 16 + (own & 15);
    uint16_t* out = Q.out + (int64_t)(W.seg->row0 + pair / C.G) * Q.ldo + (int64_t)(kvh * C.G + pair % C.G) * HD + (own >> 4) * 4;
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) {
        uint16_t b[4];
        const v4f v = all[d][own];
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = q8_bf16(v[e] / den * (down ? 1.f / kDown : 1.f));
        __builtin_memcpy(out + d * 16, b, 8);
    }
}

void q8_attention_plan(amusd_q8_cache& c) {
    // A chunk is a wave's work where there are few rows.  Short, for a wave on every other compute unit from one tile's full cache; no
    // shorter, as a chunk costs a wave its beginning and end (64 keys of 64 a step: 450 instructions a step, of 512: 300) and has
    // sums to write and to merge.  us, chunks of 64 / 128 / 256 / 512: 1B shape, 1 row, 512 keys 8.6 / 8.9 / 10.3 / 13.3, 4000 keys - /
    // 11.0 / 10.8 / 14.1; 8B shape, 8 rows, 2048 keys 12.9 / 12.8 / 13.0 / 16.6; 2048 rows 102 / 88 / 82 / 78.
    int chunk = kStep;
    while (chunk < kMaxChunk && (int64_t)c.cap / chunk * c.Hkv > c.cus / 2) chunk *= 2;
    c.chunk = chunk;
    c.max_chunks = (c.cap + chunk - 1) / chunk;
    c.part_tiles = q8_part_tiles(c.n_seqs, c.G, c.Hkv, c.cus, (int64_t)c.max_chunks * (c.hd + 2) * 16 * 4,
                                 (int64_t)c.n_layers * c.n_seqs * c.Hkv * c.cap * 2 * c.hd);
}

hipError_t launch_q8_attention(const amusd_q8_cache& c, int layer, const Q8Segs& segs, const void* q, int64_t ldq, float scale, const float* cos,
                               const float* sin, void* out, int64_t ldo, hipStream_t stream) {
    Q8Segs S = segs;
    const Q8Query Q{static_cast<const uint16_t*>(q), ldq, static_cast<uint16_t*>(out), ldo, cos, sin, scale * 1.44269504088896340736f};
    int64_t tiles = 0;
    for (int i = 0; i < S.n_seg; ++i) {
        S.s[i].unit0 = (int)tiles;
        tiles += ((int64_t)S.s[i].n * c.G + 15) / 16;
    }
    auto go = [&](auto hd, auto per_token) {
        constexpr int HD = decltype(hd)::value;
        constexpr bool PT = decltype(per_token)::value;
        // Chunks are split over waves while there are fewer than five tiles for four compute units (8B shape, 100 rows behind 1000 keys, 200
        // tiles: 21 us against 29 for a wave a tile; 250 rows, 504 tiles: 43 against 34), or what 16 rows have; as many at a time as there is room for.
        if (tiles * c.Hkv <= std::max(c.part_tiles, q8_split_tiles(c.cus))) {
            const int chunks = (S.max_len + c.chunk - 1) / c.chunk, most = c.part_tiles / c.Hkv, turns = ((int)tiles + most - 1) / most;
            const int per = ((int)tiles + turns - 1) / turns;
            for (int at = 0; at < tiles; at += per) {
                const unsigned n = (unsigned)std::min(per, (int)tiles - at);
                hipLaunchKernelGGL((k_q8_att_part<HD, PT>), dim3(c.Hkv, n, chunks), dim3(64), 0, stream, c, layer, S, Q, at);
                hipLaunchKernelGGL((k_q8_att_merge<HD>), dim3(c.Hkv, n, 8), dim3(HD * 2), 0, stream, c, S, Q, at);
            }
        } else {
            hipLaunchKernelGGL((k_q8_att_whole<HD, PT>), dim3(c.Hkv, (unsigned)tiles), dim3(64), 0, stream, c, layer, S, Q);
        }
    };
    auto by_block = [&](auto hd) {
        if (c.block == 1) go(hd, std::true_type{});
        else go(hd, std::false_type{});
    };
    if (c.hd == 64) by_block(std::integral_constant<int, 64>{});
    else by_block(std::integral_constant<int, 128>{});
    return hipGetLastError();
}

}  // namespace amusd
