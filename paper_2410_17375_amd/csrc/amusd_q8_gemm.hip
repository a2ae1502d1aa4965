// Products of 8-bit integers: out[r][c] = sx[r] * sw[c] * sum_k x[r][k] * w[c][k], sums exact in 32 bits.
#include <algorithm>

#include "amusd_math.h"
#include "amusd_q8.h"

#pragma clang fp contract(off)

namespace amusd {

typedef int v4i __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4i mfma_i8(uint4 a, uint4 b, v4i c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, a), __builtin_bit_cast(v4i, b), c, 0, 0, 0);
}

// What every form of the product makes of a sum, in this order: a row's bits do not depend on the form.  A large row scale (rows of 1e21 and more) is
// taken down by a power of two, which the result is given back: the sum times it could be past float32 where the result is not.
struct Q8RowScale {
    float s, back;
};
__device__ __forceinline__ Q8RowScale q8_row_scale(float s) {
    const bool large = s >= 0x1p64f;
    return {large ? s * 0x1p-40f : s, large ? 0x1p40f : 1.f};
}
__device__ __forceinline__ float q8_value(int sum, Q8RowScale sx, float sw) { return (float)sum * sx.s * sw * sx.back; }
__device__ __forceinline__ void q8_put(float* p, float v) { *p = v; }
__device__ __forceinline__ void q8_put(uint16_t* p, float v) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }
// silu(gate) * up.  With the instructions for 2^x and 1/x (an error of one unit in the last place each; the rounding of 2^x's argument adds |gate|
// half units): a division in full is ten instructions more for each of the outputs, which wait for nothing else.
__device__ __forceinline__ float q8_swiglu(float gate, float up) {
    return gate * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(gate * -1.44269504f)) * up;
}

// Few rows: the weights are read once and their bytes bound it.  A workgroup owns NT tiles of 16 features, its waves every
// eighth block of 64 columns, and each wave keeps D blocks under way; the sums meet in LDS.  MT: tiles of 16 rows.  Where
// workgroups share a contraction (blockIdx.z: which part), their sums meet in `work`: kQ8Tickets counts, then the sums.
// Measured (MI355X), 8 rows: 28672 x 4096 gated 19.8 us (5.9 TB/s), 4096 x 14336 11.5 (5.1), 4096 x 4096 5.3 (3.2), 128256 x 4096 75 (7.0).
template <class OUT, bool GATED, int MT, int NT, int D>
__global__ void __launch_bounds__(512) k_q8_gemm_rows(const uint4* __restrict__ frag, const float* __restrict__ wscale, int kblocks, int k, int tiles, int n,
                                                      const int8_t* __restrict__ x, int64_t ldx, const float* __restrict__ xscale, int rows,
                                                      OUT* __restrict__ out, int64_t ldo, int* __restrict__ work) {
    extern __shared__ int lds[];                     // [8 waves][MT][NT][16 rows][16 features]
    __shared__ int last;
    // (the wave's number as a scalar: matrix instructions take no notice of masked lanes, so what is around them has to be a branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
    const int tile0 = blockIdx.x * NT, row0 = blockIdx.y * (MT * 16);
    const uint4* wp[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) wp[t] = frag + (size_t)min(tile0 + t, tiles - 1) * kblocks * 64 + lane;
    const int8_t* xp[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) xp[m] = x + (int64_t)min(row0 + m * 16 + r, rows - 1) * ldx;
    const int ways = gridDim.z, per = (kblocks + ways - 1) / ways, first = blockIdx.z * per;
    const int S = (min(kblocks - first, per) - wave + 7) / 8;        // this wave's blocks: first + wave, first + wave + 8, ..
    v4i acc[MT][NT] = {};
    uint4 wf[D][NT], xf[D][MT];
    auto load = [&](int slot, int i) {
        const int kb = first + wave + 8 * min(i, S - 1);     // (S is no multiple of D: the last block once more, unused)
        const int at = kb * 64 + g * 16;
#pragma unroll
        for (int t = 0; t < NT; ++t) wf[slot][t] = load_stream(wp[t] + (size_t)kb * 64);
        // (columns past k meet weights that are zero; their own address could be past the end of the row)
#pragma unroll
        for (int m = 0; m < MT; ++m) xf[slot][m] = *reinterpret_cast<const uint4*>(xp[m] + (at < k ? at : 0));
    };
    auto use = [&](int slot) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[m][t] = mfma_i8(xf[slot][m], wf[slot][t], acc[m][t]);
    };
    if (S > 0) {
#pragma unroll
        for (int d = 0; d < D; ++d) load(d, d);
        int i = 0;
        for (; i + D < S; i += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                use(d);
                load(d, i + d + D);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (i + d < S) use(d);
        wait_vm<0>();          // a wave does not end with loads under way
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) lds[(((wave * MT + m) * NT + t) * 16 + g * 4 + e) * 16 + r] = acc[m][t][e];
    __syncthreads();
    constexpr int kSums = MT * NT * 256;
    auto of_waves = [&](int i) {
        int s = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += lds[w * kSums + i];
        return s;
    };
    if (ways > 1) {
        // Each workgroup of the `ways` writes its sums and counts itself; the one that counts last adds them up (integers: the order does
        // not show) and goes on.  Nobody waits for anybody.  What another die has written or is to read passes its L2: atomics.
        const int group = blockIdx.y * gridDim.x + blockIdx.x;
        int* const all = work + kQ8Tickets + (size_t)group * ways * kSums;
        for (int i = threadIdx.x; i < kSums; i += 512)
            __hip_atomic_store(all + blockIdx.z * kSums + i, of_waves(i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
            const int seen = __hip_atomic_fetch_add(work + group, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (seen == ways - 1) __hip_atomic_store(work + group, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next call
            last = seen == ways - 1;
        }
        __syncthreads();
        if (!last) return;
        auto from = [&](int p, int i) { return __hip_atomic_load(all + p * kSums + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
#pragma unroll
        for (int j = 0; j < (kSums + 511) / 512; ++j) {
            const int i = j * 512 + threadIdx.x;
            if (kSums % 512 && i >= kSums) break;
            int s = from(0, i) + from(1, i);
            if (ways == 4) s += from(2, i) + from(3, i);
            lds[i] = s;
        }
        __syncthreads();
    }
    auto sum = [&](int m, int t, int at) {
        const int i = (m * NT + t) * 256 + at;
        return ways > 1 ? lds[i] : of_waves(i);
    };
    constexpr int kOut = GATED ? NT / 2 : NT;        // tiles of output columns
    for (int i = threadIdx.x; i < MT * kOut * 256; i += 512) {
        const int f = i % (kOut * 16), row = i / (kOut * 16);               // features fastest: whole lines of a row
        const int t = f >> 4, m = row >> 4, at = (row & 15) * 16 + (f & 15);
        const int gr = row0 + row, gc = (GATED ? tile0 / 2 : tile0) * 16 + f;
        if (gr >= rows || gc >= n) continue;
        const Q8RowScale sx = q8_row_scale(xscale[gr]);
        float v;
        if constexpr (GATED) {
            const float* s = wscale + (tile0 + 2 * t) * 16 + (f & 15);
            v = q8_swiglu(q8_value(sum(m, 2 * t, at), sx, s[0]), q8_value(sum(m, 2 * t + 1, at), sx, s[16]));
        } else {
            v = q8_value(sum(m, t, at), sx, wscale[gc]);
        }
        q8_put(out + (int64_t)gr * ldo + gc, v);
    }
}

// Many rows: the matrix instructions bound it.  A workgroup of WN x WM waves has WN * A tiles of 16 features x WM * B tiles of 16 rows,
// a wave A x B of them.  Both operands go through rings in LDS, filled by loads that deliver straight into it:
//   weights a block of 64 columns at a time, as they lie in memory (4 slots);
//   rows two blocks at a time (3 slots), a load fetching 8 whole lines of 128 bytes: with 16 half lines a load, a block of 256 x 256 took
//   0.75 us instead of 0.56.  The eight 16-byte pieces of a line lie in an order that depends on the row, so that the 16
//   lanes that read a column of pieces find them in different banks.
// Measured (MI355X), 2048 rows: 28672 x 4096 gated 208-217 us, 230 after a pause (2.2-2.3 POP/s; with every compute unit multiplying a block of 256 x 256 takes 0.70
// us, at the clock that their power leaves), 6144 x 4096 53, 4096 x 4096 38, 4096 x 14336 118-124; 8192 x 8192 of 8192 rows 2.47 POP/s.
template <int WN_, int WM_, int A_, int B_, int WAVES_>
struct Q8Shape {
    static constexpr int WN = WN_, WM = WM_, A = A_, B = B_, kMinWaves = WAVES_;
    static constexpr int kWavesOf = WN * WM, kThreads = kWavesOf * 64;
    static constexpr int kColTiles = WN * A, kRowTiles = WM * B;
    static constexpr int NW = kColTiles / kWavesOf, NX = kRowTiles / kWavesOf;      // loads of a wave and block
    static constexpr int kWSlots = 4, kXSlots = 3, kWBytes = kColTiles * 1024, kXBytes = kRowTiles * 2048;
    static constexpr int kLds = kWSlots * kWBytes + kXSlots * kXBytes;
    static_assert(kColTiles % kWavesOf == 0 && kRowTiles % kWavesOf == 0 && A % 2 == 0, "");
};

template <class Sh, class OUT, bool GATED>
__global__ void __launch_bounds__(Sh::kThreads, Sh::kMinWaves) k_q8_gemm_tile(const uint4* __restrict__ frag, const float* __restrict__ wscale, int kblocks,
                                                                             int k, int tiles, int n, const int8_t* __restrict__ x, int64_t ldx,
                                                                             const float* __restrict__ xscale, int rows, OUT* __restrict__ out, int64_t ldo,
                                                                             int row_wgs, int wgs, int* __restrict__ work) {
    constexpr int WN = Sh::WN, A = Sh::A, B = Sh::B, NW = Sh::NW, NX = Sh::NX, NPW = NW + NX, MID = A / 2, WR = A >= 4 ? 4 : 2, WD = WR / 2;
    static_assert(MID + WD <= A && A % WR == 0, "");
    extern __shared__ char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
    const int wn = wave % WN, wm = wave / WN;
    // Workgroups are dealt to the 8 XCDs in turn: each gets a run of neighbouring tiles, rows fastest, so that the weights that its
    // workgroups want at a time are few and in its L2.
    const int xcd = blockIdx.x & 7, per = wgs >> 3, more = wgs & 7;
    const int at = xcd * per + min(xcd, more) + (blockIdx.x >> 3);
    const int row0 = at % row_wgs * (Sh::kRowTiles * 16), tile0 = at / row_wgs * Sh::kColTiles;
    const int ways = gridDim.y, share = ((kblocks + 1) / 2 + ways - 1) / ways * 2, first = blockIdx.y * share, blocks = min(kblocks - first, share);
    const char* wsrc[NW];
#pragma unroll
    for (int q = 0; q < NW; ++q) wsrc[q] = reinterpret_cast<const char*>(frag + ((size_t)min(tile0 + wave * NW + q, tiles - 1) * kblocks + first) * 64);
    // rows: load q of half h of a pair of blocks is of the 8 rows from 8 * (h * kRowTiles + wave * NX + q)
    const char* xsrc = reinterpret_cast<const char*>(x + (int64_t)row0 * ldx + first * 64);
    unsigned xoff[2][NX], xcol[2][NX];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < NX; ++q) {
            const int piece = h * Sh::kRowTiles + wave * NX + q;
            xoff[h][q] = (unsigned)(min(piece * 8 + (lane >> 3), rows - 1 - row0) * ldx);
            xcol[h][q] = ((lane & 7) ^ (lane >> 3) ^ (piece & 1)) * 16;
        }
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)smem;
    const unsigned ldsx = lds0 + Sh::kWSlots * Sh::kWBytes;
    const int pairs = (blocks + 1) / 2, columns = k - first * 64;
    // Issues load q of NPW with block `b` of weights and half h of pair `p` of rows (past the end: the last once more, unused).
    int wslot = 0, xslot = 0;
    unsigned wdst = 0, wat = 0;
    auto begin_w = [&](int b) {
        wdst = lds0 + wslot * Sh::kWBytes + wave * (NW * 1024);
        wat = (unsigned)min(b, blocks - 1) * 1024u + lane * 16;
        wslot = (wslot + 1) & 3;
    };
    auto load_w = [&](int q) { load_to_lds(wsrc[q], wat, wdst + q * 1024); };
    auto load_x = [&](int q, int p, int h) {
        const unsigned c = (unsigned)min(p, pairs - 1) * 128u + xcol[h][q];
        load_to_lds(xsrc, xoff[h][q] + (c < (unsigned)columns ? c : 0u), ldsx + xslot * Sh::kXBytes + (h * Sh::kRowTiles + wave * NX + q) * 1024);   // columns past k meet zeros
    };
    auto next_x = [&] { xslot = xslot == 2 ? 0 : xslot + 1; };
    auto w_frag = [&](const char* slot, int f) { return *reinterpret_cast<const uint4*>(slot + f * 1024 + lane * 16); };
    const int xread = (r >> 3) * 1024 + (r & 7) * 128 + ((g ^ (r & 7) ^ (r >> 3)) * 16);
    auto x_frag = [&](const char* slot, int half, int f) { return *reinterpret_cast<const uint4*>(slot + f * 2048 + (half ? xread ^ 64 : xread)); };
    const char* const wring = smem;
    const char* const xring = smem + Sh::kWSlots * Sh::kWBytes;
    v4i acc[A][B] = {};
    uint4 wf[WR], xf[2][B];
    // Before the loop: blocks 0 to 2 of the weights, pairs 0 and 1 of the rows; what the loop's first half block issues is left out.
    constexpr int kFirst = NPW * (A - MID) / A;
    begin_w(0);
#pragma unroll
    for (int q = 0; q < NW; ++q) load_w(q);
#pragma unroll
    for (int q = 0; q < 2 * NX; ++q) load_x(q % NX, 0, q / NX);
    next_x();
    begin_w(1);
#pragma unroll
    for (int q = 0; q < NW; ++q) load_w(q);
#pragma unroll
    for (int q = 0; q < NX; ++q) load_x(q, 1, 0);
    begin_w(2);
#pragma unroll
    for (int q = 0; q < kFirst; ++q) {
        if (q < NW) load_w(q);
        else load_x(q - NW, 1, 1);
    }
    wait_vm<NPW + kFirst>();
    __builtin_amdgcn_s_waitcnt(0xC07F);                  // lgkmcnt(0): no scalar load is pending in the loop
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < WD; ++i) wf[i] = w_frag(wring, wn * A + i);
#pragma unroll
    for (int j = 0; j < B; ++j) xf[0][j] = x_frag(xring, 0, wm * B + j);
    int cw = 0, cx = 0, kb = 0;
    // One block, its rows' fragments in xf[P] (P: which of its pair).  The next block is in LDS after the barrier in the middle, and the loads
    // of what is three blocks ahead begin, into slots that every wave is past, a few with each tile's products.  Fragments are
    // read from LDS well before their use: weights WD tiles ahead, rows half a block.
    auto block = [&](auto parity) {
        constexpr int P = decltype(parity)::value;
        const char* cur = wring + cw * Sh::kWBytes;
        cw = (cw + 1) & 3;
        const char* nxt = wring + cw * Sh::kWBytes;
        if (P) cx = cx == 2 ? 0 : cx + 1;
        const char* nx = xring + cx * Sh::kXBytes;       // where the next block's rows are
#pragma unroll
        for (int i = 0; i < A; ++i) {
            if (i == MID) {
                wait_vm<NPW>();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                begin_w(kb + 3);
                if (!P) next_x();
            }
            // steps from the middle on fetch for (kb + 3, half P of pair kb / 2 + 2), those before it what the block before began
            const int step = (i - MID + A) % A;
#pragma unroll
            for (int q = step * NPW / A; q < (step + 1) * NPW / A; ++q) {
                if (q < NW) load_w(q);
                else if (i >= MID) load_x(q - NW, (kb >> 1) + 2, P);
                else load_x(q - NW, ((kb - 1) >> 1) + 2, 1 - P);
            }
            wf[(i + WD) % WR] = i + WD < A ? w_frag(cur, wn * A + i + WD) : w_frag(nxt, wn * A + i + WD - A);
            if (i >= MID)
#pragma unroll
                for (int j = (i - MID) * B / (A - MID); j < (i - MID + 1) * B / (A - MID); ++j) xf[1 - P][j] = x_frag(nx, 1 - P, wm * B + j);
#pragma unroll
            for (int j = 0; j < B; ++j) acc[i][j] = mfma_i8(wf[i % WR], xf[P][j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        ++kb;
    };
#pragma unroll 1
    while (kb + 2 <= blocks) {
        block(std::integral_constant<int, 0>{});
        block(std::integral_constant<int, 1>{});
    }
    if (kb < blocks) block(std::integral_constant<int, 0>{});
    wait_vm<0>();                                        // what was loaded past the end
    // Lane: row r of a row tile, features 4 g .. 4 g + 3 of a feature tile.  Through LDS, so that whole lines are stored: a wave's rows
    // at a distance of W elements, a little more than they have (banks).
    __syncthreads();
    if (ways > 1) {
        // As with few rows, but each wave by itself: of the waves that have a part of the same sums, the one that counts last goes on.
        typedef unsigned long long u64;
        constexpr int kPairs = A * B * 2;
        const int place = at * Sh::kWavesOf + wave;
        u64* const all = reinterpret_cast<u64*>(work + kQ8Tickets) + (size_t)place * ways * (kPairs * 64) + lane;
        u64* const mine = all + blockIdx.y * (kPairs * 64);
#pragma unroll
        for (int q = 0; q < kPairs; ++q) {
            const v4i a = acc[q / 2 / B][q / 2 % B];
            const u64 v = (u64)(unsigned)a[q % 2 * 2 + 1] << 32 | (unsigned)a[q % 2 * 2];
            __hip_atomic_store(mine + q * 64, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        int seen = 0;
        if (lane == 0) {
            seen = __hip_atomic_fetch_add(work + place, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (seen == ways - 1) __hip_atomic_store(work + place, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (__builtin_amdgcn_readfirstlane(seen) != ways - 1) return;
#pragma unroll 1
        for (int p = 1; p < ways; ++p) {
            const u64* from = all + (blockIdx.y + p) % ways * (kPairs * 64);
            u64 v[kPairs];
#pragma unroll
            for (int q = 0; q < kPairs; ++q) v[q] = __hip_atomic_load(from + q * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int q = 0; q < kPairs; ++q) {
                acc[q / 2 / B][q / 2 % B][q % 2 * 2] += (int)v[q];
                acc[q / 2 / B][q / 2 % B][q % 2 * 2 + 1] += (int)(v[q] >> 32);
            }
        }
    }
    constexpr int kOutTiles = GATED ? A / 2 : A, W = kOutTiles * 16 + 16 / (int)sizeof(OUT);
    constexpr int kSpan = kOutTiles * 16 * (int)sizeof(OUT) / 16;             // 16-byte pieces of a row
    OUT* const stage = reinterpret_cast<OUT*>(smem) + wave * (16 * W);
    static_assert(Sh::kWavesOf * 16 * W * (int)sizeof(OUT) <= Sh::kLds, "");
    const int col0 = (GATED ? (tile0 + wn * A) / 2 : tile0 + wn * A) * 16;
    v4f sw[A];
#pragma unroll
    for (int i = 0; i < A; ++i) sw[i] = *reinterpret_cast<const v4f*>(wscale + min(tile0 + wn * A + i, tiles - 1) * 16 + g * 4);
#pragma unroll
    for (int j = 0; j < B; ++j) {
        const int jrow = row0 + (wm * B + j) * 16;
        const Q8RowScale sx = q8_row_scale(xscale[min(jrow + r, rows - 1)]);
#pragma unroll
        for (int i = 0; i < A; i += GATED ? 2 : 1) {
            OUT v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (GATED) q8_put(&v[e], q8_swiglu(q8_value(acc[i][j][e], sx, sw[i][e]), q8_value(acc[i + 1][j][e], sx, sw[i + 1][e])));
                else q8_put(&v[e], q8_value(acc[i][j][e], sx, sw[i][e]));
            }
            __builtin_memcpy(stage + r * W + (GATED ? i / 2 : i) * 16 + g * 4, v, sizeof v);
        }
        __builtin_amdgcn_wave_barrier();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int c = lane; c < 16 * kSpan; c += 64) {
            constexpr int kPiece = 16 / (int)sizeof(OUT);
            const int row = jrow + c / kSpan, col = col0 + c % kSpan * kPiece;
            OUT v[kPiece];
            __builtin_memcpy(v, stage + c / kSpan * W + c % kSpan * kPiece, 16);
            if (row >= rows || col >= n) continue;
            OUT* o = out + (int64_t)row * ldo + col;
            if (col + kPiece <= n) {
                __builtin_memcpy(o, v, 16);
            } else {
#pragma unroll
                for (int e = 0; e < kPiece; ++e)
                    if (col + e < n) o[e] = v[e];
            }
        }
        __builtin_amdgcn_wave_barrier();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

template <class OUT, bool GATED>
static void gemm(const amusd_q8_matrix& w, const int8_t* x, int64_t ldx, const float* scale, int rows, OUT* out, int64_t ldo, const Q8Plan& plan, int* work,
                 hipStream_t stream) {
    auto few = [&](auto kernel, int mt, int nt) {
        const int lds = 8 * mt * nt * 256 * 4;
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        hipLaunchKernelGGL(kernel, dim3((w.tiles + nt - 1) / nt, (rows + mt * 16 - 1) / (mt * 16), plan.ways), dim3(512), lds, stream, w.frag, w.scale,
                           w.kblocks, w.k, w.tiles, w.n, x, ldx, scale, rows, out, ldo, work);
    };
    auto many = [&](auto shape) {
        using Sh = decltype(shape);
        const auto kernel = k_q8_gemm_tile<Sh, OUT, GATED>;
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, Sh::kLds);
        // (a launch of 2^32 threads and more is cut off without an error: at most 2^31, so many rows at a time)
        const int col_wgs = (w.tiles + Sh::kColTiles - 1) / Sh::kColTiles;
        const int64_t most = std::max(1, (1 << 22) / col_wgs) * (int64_t)(Sh::kRowTiles * 16);
        for (int64_t r = 0; r < rows; r += most) {
            const int n = (int)std::min(most, rows - r), row_wgs = (int)(((int64_t)n + Sh::kRowTiles * 16 - 1) / (Sh::kRowTiles * 16)), wgs = row_wgs * col_wgs;
            hipLaunchKernelGGL(kernel, dim3(wgs, plan.ways), dim3(Sh::kThreads), Sh::kLds, stream, w.frag, w.scale, w.kblocks, w.k, w.tiles, w.n,
                               x + r * ldx, ldx, scale + r, n, out + r * ldo, ldo, row_wgs, wgs, work);
        }
    };
    switch (plan.form) {
        case kQ8Few1x1: if constexpr (!GATED) return few(k_q8_gemm_rows<OUT, GATED, 1, 1, 4>, 1, 1); else return;
        case kQ8Few1x2: return few(k_q8_gemm_rows<OUT, GATED, 1, 2, 4>, 1, 2);
        case kQ8Few2x2: return few(k_q8_gemm_rows<OUT, GATED, 2, 2, 4>, 2, 2);
        case kQ8Few2x4: return few(k_q8_gemm_rows<OUT, GATED, 2, 4, 4>, 2, 4);
        case kQ8Few4x4: return few(k_q8_gemm_rows<OUT, GATED, 4, 4, 2>, 4, 4);
        case kQ8Tile64: return many(Q8Shape<2, 2, 2, 2, 4>{});
        case kQ8Tile128x64: return many(Q8Shape<2, 2, 4, 2, 2>{});
        case kQ8Tile128: return many(Q8Shape<2, 2, 4, 4, 2>{});
        case kQ8Tile256: return many(Q8Shape<2, 4, 8, 4, 2>{});
    }
}

constexpr int64_t kMaxLd = 1 << 22;      // the forms for many rows have 32-bit offsets into a tile's rows

static int64_t work_of(const amusd_q8_matrix& w, int rows, const Q8Plan& p) {
    if (p.ways == 1) return 0;
    const int mt = q8_form_rows(p.form), nt = q8_form_tiles(p.form);
    const int64_t groups = (int64_t)((w.tiles + nt - 1) / nt) * ((rows + 16 * mt - 1) / (16 * mt));
    return (kQ8Tickets + groups * p.ways * mt * nt * 256) * 4;
}
// .. of up to `rows` rows: what is chosen depends on the tiles of 16 rows, and past so many nobody shares.
int64_t q8_gemm_workspace(const amusd_q8_matrix& w, int rows) {
    int64_t most = 0;
    const int end = std::min(rows, (kQ8Tickets / 4 + 1) * 128);
    for (int r = 17; r <= end; r = (r & ~15) + 17) most = std::max(most, work_of(w, r, q8_gemm_plan(w.tiles, w.kblocks, w.gated, r, w.cus, true)));
    return most;
}

hipError_t launch_q8_gemm(const amusd_q8_matrix& w, const int8_t* x, int64_t ldx, const float* scale, int rows, void* out, int dtype, int64_t ldo,
                          void* work, int64_t work_bytes, hipStream_t stream) {
    Q8Plan plan = q8_gemm_plan(w.tiles, w.kblocks, w.gated, rows, w.cus, true);
    if (work_of(w, rows, plan) > work_bytes) plan = q8_gemm_plan(w.tiles, w.kblocks, w.gated, rows, w.cus, false);
    if (ldx > kMaxLd) plan = {kQ8Few4x4, 1};
    auto go = [&](auto* o) {
        if (w.gated) gemm<std::remove_pointer_t<decltype(o)>, true>(w, x, ldx, scale, rows, o, ldo, plan, static_cast<int*>(work), stream);
        else gemm<std::remove_pointer_t<decltype(o)>, false>(w, x, ldx, scale, rows, o, ldo, plan, static_cast<int*>(work), stream);
    };
    if (dtype == AMUSD_DTYPE_BF16) go(static_cast<uint16_t*>(out));
    else go(static_cast<float*>(out));
    return hipGetLastError();
}

}  // namespace amusd
