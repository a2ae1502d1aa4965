// Attention of rows over the cache in 8 bits.
//
// A tile is 16 (row, head) pairs of one sequence and kv head: they share its keys.  Queries are rotated and held in 16 bits
// relative to their largest component, as two planes of 8-bit integers: their products with the keys are then exact integers,
// half as many matrix instructions as half precision would take, and no key is converted.  The rounding of a query moves a score
// by at most 2^-16 of (its largest component times the sum of the key's magnitudes).  Softmax weights carry the scales of their
// values, are brought below 2^15 by a power of two and rounded to half (11 bits); values are exact in half.  Maxima, sums and
// results are fp32.
//
// Keys are taken in chunks at absolute positions, whose sums start anew and are merged in order, whoever does it: with few rows a
// wave takes one chunk and a second launch merges (k_q8_att_part, k_q8_att_merge), with many a wave walks all of them
// (k_q8_att_whole).  What a chunk's sums depend on is only what the row may see.  So a row's bits depend neither on how many
// rows a call has nor on the form.
#include <algorithm>

#include "amusd_math.h"
#include "amusd_q8.h"

#pragma clang fp contract(off)

namespace amusd {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

constexpr int kPlane = 32512;                    // 127 * 256: a query's largest component in its 16 bits

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
    float qs;                                    // score per unit of the integer product, without the key's scale
    int pos;                                     // the pair's row's position (the last key that it sees); -1: no pair
    int row, head;
};

template <int HD>
__device__ __forceinline__ Tile<HD> load_tile(const amusd_q8_cache& C, const Q8Query& Q, const Q8Seg& seg, int kvh, int tile) {
    Tile<HD> T;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int p = tile * 16 + (lane & 15), pairs = seg.n * C.G;
    const int pc = min(p, pairs - 1);
    T.row = pc / C.G;
    T.head = kvh * C.G + pc % C.G;
    const int pos = seg.pos0 + T.row;
    T.pos = p < pairs ? pos : -1;
    const uint16_t* src = Q.q + (int64_t)(seg.row0 + T.row) * Q.ldq + (int64_t)T.head * HD;
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
    const float inv = m > 0.f ? (float)kPlane / m : 0.f;
    T.qs = bad ? __uint_as_float(0x7FC00000u) : m / (float)kPlane * Q.scale2;
#pragma unroll
    for (int f = 0; f < HD / 64; ++f) {
        uint32_t hi[4] = {}, lo[4] = {};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int v = bad ? 0 : min(max((int)rintf(x[f][i] * inv), -kPlane), kPlane);
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

// Four signed bytes as half values: 1024 + (b + 128) is the half whose low byte is b + 128.
__device__ __forceinline__ void bytes_to_half(uint32_t b, uint32_t& lo, uint32_t& hi) {
    const uint32_t u = b ^ 0x80808080u;
    const h2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off);
}

// A chunk's sums for 16 pairs: lane l has columns dt * 16 + 4 * (l / 16) + e of pair l % 16.
template <int HD>
struct Sums {
    v4f acc[HD / 16];
    float ref, den;
};

// Scales of the 4 keys pos .. pos + 3 (pos a multiple of 4).
template <bool PER_TOKEN>
__device__ __forceinline__ v4f key_scales(const float* s, int pos, int shift) {
    if constexpr (PER_TOKEN) return *reinterpret_cast<const v4f*>(s + pos);
    const float v = s[pos >> shift];
    return v4f{v, v, v, v};
}

template <int HD, bool PER_TOKEN, int NT>
__device__ __forceinline__ void chunk_sums(const amusd_q8_cache& C, size_t kvh, const Tile<HD> (&T)[NT], int c0, int c1, Sums<HD> (&S)[NT]) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int8_t* K = C.k + kvh * ((size_t)C.cap * HD) + (size_t)(lane & 15) * HD + g * 16;
    const uint4* V = reinterpret_cast<const uint4*>(C.v + kvh * ((size_t)C.cap * HD)) + lane;
    const float *ks = C.ks + kvh * (C.cap / C.block), *vs = C.vs + kvh * (C.cap / C.block);
    const int shift = __builtin_ctz(C.block);
    // The power of two that brings each pair's weights below 2^15 (of the values that it sees in this chunk).
    float up[NT], down[NT];
    {
        float most[NT] = {};
        for (int pos = c0 + g * 4; pos < c1; pos += 16) {
            const v4f s = key_scales<PER_TOKEN>(vs, pos, shift);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) most[n] = fmaxf(most[n], pos + e <= T[n].pos ? s[e] : 0.f);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            most[n] = fmaxf(most[n], lane_xor<16>(most[n]));
            most[n] = fmaxf(most[n], lane_xor<32>(most[n]));
            const int e = min(max((int)(__float_as_uint(most[n]) >> 23) - 127, -110), 126);
            up[n] = __uint_as_float((uint32_t)(127 + 14 - e) << 23);       // most * up in [2^14, 2^15)
            down[n] = __uint_as_float((uint32_t)(127 - 14 + e) << 23);
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        S[n].ref = -INFINITY;
        S[n].den = 0.f;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) S[n].acc[d] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    for (int b = c0; b < c1; b += 32) {
        uint4 kf[2][HD / 64], vf[HD / 32];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int f = 0; f < HD / 64; ++f) kf[t][f] = *reinterpret_cast<const uint4*>(K + (size_t)(b + t * 16) * HD + f * 64);
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) vf[d] = V[((size_t)(b >> 5) * (HD / 32) + d) * 64];
        v4f kscale[2], vscale[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            kscale[t] = key_scales<PER_TOKEN>(ks, b + t * 16 + g * 4, shift);
            vscale[t] = key_scales<PER_TOKEN>(vs, b + t * 16 + g * 4, shift);
        }
        uint4 w[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float sc[2][4], top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                v4i hi = {}, lo = {};
#pragma unroll
                for (int f = 0; f < HD / 64; ++f) {
                    hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, kf[t][f]), __builtin_bit_cast(v4i, T[n].hi[f]), hi, 0, 0, 0);
                    lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, kf[t][f]), __builtin_bit_cast(v4i, T[n].lo[f]), lo, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float s = (float)(hi[e] * 256 + lo[e]) * (T[n].qs * kscale[t][e]);
                    sc[t][e] = b + t * 16 + g * 4 + e <= T[n].pos ? s : -INFINITY;
                    top = fmaxf(top, sc[t][e]);
                }
            }
            top = fmaxf(top, lane_xor<16>(top));
            top = fmaxf(top, lane_xor<32>(top));
            const float ref = fmaxf(S[n].ref, top), at = ref == -INFINITY ? 0.f : ref;
            const float shrink = pow2(S[n].ref - at);
            float sum = 0.f, p[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[t][e] = pow2(sc[t][e] - at);
                    sum += p[t][e];
                    // (a key that is not seen has weight 0 whatever its value's scale is)
                    p[t][e] *= b + t * 16 + g * 4 + e <= T[n].pos ? vscale[t][e] * up[n] : 0.f;
                }
            S[n].den = fmaf(S[n].den, shrink, sum);
            S[n].ref = ref;
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) S[n].acc[d] *= shrink;
            auto two = [](float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, h2)); };
            w[n] = uint4{two(p[0][0], p[0][1]), two(p[0][2], p[0][3]), two(p[1][0], p[1][1]), two(p[1][2], p[1][3])};
        }
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) {
            uint4 a, c;
            bytes_to_half(vf[d].x, a.x, a.y);
            bytes_to_half(vf[d].y, a.z, a.w);
            bytes_to_half(vf[d].z, c.x, c.y);
            bytes_to_half(vf[d].w, c.z, c.w);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                S[n].acc[2 * d] = BF16::mfma_att(a, w[n], S[n].acc[2 * d]);
                S[n].acc[2 * d + 1] = BF16::mfma_att(c, w[n], S[n].acc[2 * d + 1]);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        S[n].den += lane_xor<16>(S[n].den);
        S[n].den += lane_xor<32>(S[n].den);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) S[n].acc[d] *= down[n];
    }
}

// sums so far and a chunk's: how both are weighed
__device__ __forceinline__ void merge_weights(float& ref, float& den, float cref, float cden, float& a, float& b) {
    const float to = fmaxf(ref, cref), at = to == -INFINITY ? 0.f : to;
    a = pow2(ref - at);
    b = pow2(cref - at);
    den = fmaf(den, a, cden * b);
    ref = to;
}

__device__ __forceinline__ int find_seg(const Q8Segs& S, int unit) {
    int i = 0;
    while (i + 1 < S.n_seg && unit >= S.s[i + 1].unit0) ++i;
    return i;
}

// A wave: one tile, one chunk.  Its sums go to memory.
template <int HD, bool PER_TOKEN>
__global__ void __launch_bounds__(64) k_q8_att_part(amusd_q8_cache C, int layer, Q8Segs S, Q8Query Q) {
    const int chunk = blockIdx.x, tile = blockIdx.y, kvh = blockIdx.z;
    const Q8Seg& seg = S.s[find_seg(S, tile)];
    const int local = tile - seg.unit0;
    const int last = seg.pos0 + min((local * 16 + 15) / C.G, seg.n - 1);        // the last key that a pair of the tile sees
    const int c0 = chunk * C.chunk;
    if (c0 > last) return;
    Tile<HD> T[1] = {load_tile<HD>(C, Q, seg, kvh, local)};
    Sums<HD> sums[1];
    const size_t head = ((size_t)layer * C.n_seqs + seg.seq) * C.Hkv + kvh;
    chunk_sums<HD, PER_TOKEN, 1>(C, head, T, c0, min(c0 + C.chunk, (last + 32) / 32 * 32), sums);
    const int lane = threadIdx.x, g = lane >> 4, pair = lane & 15;
    float* out = C.part + (((size_t)tile * C.Hkv + kvh) * C.max_chunks + chunk) * ((HD + 2) * 16);
#pragma unroll
    for (int d = 0; d < HD / 16; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) out[(d * 16 + g * 4 + e) * 16 + pair] = sums[0].acc[d][e];
    if (g == 0) {
        out[HD * 16 + pair] = sums[0].ref;
        out[(HD + 1) * 16 + pair] = sums[0].den;
    }
}

__device__ __forceinline__ uint16_t q8_bf16(float v) { return (uint16_t)(v == v ? bf16_rne(v) : 0x7FC0u); }

// A workgroup merges a tile's chunks: thread (column, pair).
template <int HD>
__global__ void __launch_bounds__(HD * 4) k_q8_att_merge(amusd_q8_cache C, Q8Segs S, Q8Query Q) {
    const int tile = blockIdx.x, kvh = blockIdx.y, part = blockIdx.z;           // a quarter of the columns a workgroup
    const Q8Seg& seg = S.s[find_seg(S, tile)];
    const int pair = threadIdx.x & 15, col = part * (HD / 4) + (threadIdx.x >> 4);
    const int p = (tile - seg.unit0) * 16 + pair;
    if (p >= seg.n * C.G) return;
    const int row = p / C.G, head = kvh * C.G + p % C.G;
    const int chunks = (seg.pos0 + row) / C.chunk + 1;
    const float* in = C.part + ((size_t)tile * C.Hkv + kvh) * C.max_chunks * ((HD + 2) * 16) + pair;
    float ref = -INFINITY, den = 0.f, acc = 0.f;
    for (int c = 0; c < chunks; ++c, in += (HD + 2) * 16) {
        float a, b;
        merge_weights(ref, den, in[HD * 16], in[(HD + 1) * 16], a, b);
        acc = fmaf(acc, a, in[col * 16] * b);
    }
    Q.out[(int64_t)(seg.row0 + row) * Q.ldo + (int64_t)head * HD + col] = q8_bf16(acc / den);
}

// A wave: NT neighbouring tiles, all chunks, merged in registers.
template <int HD, bool PER_TOKEN, int NT>
__global__ void __launch_bounds__(64) k_q8_att_whole(amusd_q8_cache C, int layer, Q8Segs S, Q8Query Q) {
    const int unit = gridDim.x - 1 - blockIdx.x, kvh = blockIdx.y;              // the longest first
    const Q8Seg& seg = S.s[find_seg(S, unit)];
    const int local = (unit - seg.unit0) * NT, tiles = (seg.n * C.G + 15) / 16;
    Tile<HD> T[NT];
    Sums<HD> all[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        T[n] = load_tile<HD>(C, Q, seg, kvh, min(local + n, tiles - 1));
        if (local + n >= tiles) T[n].pos = -1;
        all[n].ref = -INFINITY;
        all[n].den = 0.f;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) all[n].acc[d] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    const int last = seg.pos0 + min((local * 16 + NT * 16 - 1) / C.G, seg.n - 1);
    const size_t head = ((size_t)layer * C.n_seqs + seg.seq) * C.Hkv + kvh;
    for (int c0 = 0; c0 <= last; c0 += C.chunk) {
        Sums<HD> part[NT];
        chunk_sums<HD, PER_TOKEN, NT>(C, head, T, c0, min(c0 + C.chunk, (last + 32) / 32 * 32), part);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (c0 > T[n].pos) continue;                    // a chunk that the pair sees nothing of is not merged
            float a, b;
            merge_weights(all[n].ref, all[n].den, part[n].ref, part[n].den, a, b);
#pragma unroll
            for (int d = 0; d < HD / 16; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) all[n].acc[d][e] = fmaf(all[n].acc[d][e], a, part[n].acc[d][e] * b);
        }
    }
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (T[n].pos < 0) continue;
        uint16_t* out = Q.out + (int64_t)(seg.row0 + T[n].row) * Q.ldo + (int64_t)T[n].head * HD + g * 4;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) {
            uint16_t b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] = q8_bf16(all[n].acc[d][e] / all[n].den);
            __builtin_memcpy(out + d * 16, b, 8);
        }
    }
}

void q8_attention_plan(amusd_q8_cache& c) {
    // A chunk is a wave's work where there are few rows: with a full cache there should be a few waves a compute unit.
    int chunk = 64;
    while (chunk < 256 && (int64_t)c.cap / chunk * c.Hkv > 2 * c.cus) chunk *= 2;
    c.chunk = chunk;
    c.max_chunks = (c.cap + chunk - 1) / chunk;
    c.part_tiles = (kMaxSegs * c.G + 15) / 16 + kMaxSegs;       // 16 rows in up to 16 sequences, and each sequence's last tile
    c.part_tiles *= c.Hkv;
}

hipError_t launch_q8_attention(const amusd_q8_cache& c, int layer, const Q8Segs& segs, const void* q, int64_t ldq, float scale, const float* cos,
                               const float* sin, void* out, int64_t ldo, hipStream_t stream) {
    Q8Segs S = segs;
    const Q8Query Q{static_cast<const uint16_t*>(q), ldq, static_cast<uint16_t*>(out), ldo, cos, sin, scale * 1.44269504088896340736f};
    auto units = [&](int per) {
        int n = 0;
        for (int i = 0; i < S.n_seg; ++i) {
            S.s[i].unit0 = n;
            n += ((S.s[i].n * c.G + 15) / 16 + per - 1) / per;
        }
        return n;
    };
    auto go = [&](auto hd, auto per_token) {
        constexpr int HD = decltype(hd)::value;
        constexpr bool PT = decltype(per_token)::value;
        const int tiles = units(1);
        if (tiles * c.Hkv <= c.part_tiles) {
            const int chunks = (S.max_len + c.chunk - 1) / c.chunk;
            hipLaunchKernelGGL((k_q8_att_part<HD, PT>), dim3(chunks, tiles, c.Hkv), dim3(64), 0, stream, c, layer, S, Q);
            hipLaunchKernelGGL((k_q8_att_merge<HD>), dim3(tiles, c.Hkv, 4), dim3(HD * 4), 0, stream, c, S, Q);
        } else {
            const int u = units(2);
            hipLaunchKernelGGL((k_q8_att_whole<HD, PT, 2>), dim3(u, c.Hkv), dim3(64), 0, stream, c, layer, S, Q);
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
