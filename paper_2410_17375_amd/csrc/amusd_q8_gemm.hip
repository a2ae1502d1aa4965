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

// What every form of the product makes of a sum, in this order: a row's bits do not depend on the form.
__device__ __forceinline__ float q8_value(int sum, float sx, float sw) { return (float)sum * sx * sw; }
__device__ __forceinline__ void q8_put(float* p, float v) { *p = v; }
__device__ __forceinline__ void q8_put(uint16_t* p, float v) { *p = (uint16_t)(v == v ? bf16_rne(v) : 0x7FC0u); }

// Few rows: the weights are read once and their bytes bound it.  A workgroup owns NT tiles of 16 features, its waves every
// eighth block of 64 columns, and each wave keeps D blocks under way; the sums meet in LDS.  MT: tiles of 16 rows.
template <class OUT, bool GATED, int MT, int NT, int D>
__global__ void __launch_bounds__(512) k_q8_gemm_rows(const uint4* __restrict__ frag, const float* __restrict__ wscale, int kblocks, int k, int tiles, int n,
                                                      const int8_t* __restrict__ x, int64_t ldx, const float* __restrict__ xscale, int rows,
                                                      OUT* __restrict__ out, int64_t ldo) {
    extern __shared__ int lds[];                     // [8 waves][MT][NT][16 rows][16 features]
    // (the wave's number as a scalar: matrix instructions take no notice of masked lanes, so what is around them has to be a branch)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
    const int tile0 = blockIdx.x * NT, row0 = blockIdx.y * (MT * 16);
    const uint4* wp[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) wp[t] = frag + (size_t)min(tile0 + t, tiles - 1) * kblocks * 64 + lane;
    const int8_t* xp[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) xp[m] = x + (int64_t)min(row0 + m * 16 + r, rows - 1) * ldx;
    const int S = (kblocks - wave + 7) / 8;          // this wave's blocks: wave, wave + 8, ..
    v4i acc[MT][NT] = {};
    uint4 wf[D][NT], xf[D][MT];
    auto load = [&](int slot, int i) {
        const int kb = wave + 8 * min(i, S - 1);     // (S is no multiple of D: the last block once more, unused)
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
        for (int d = 0; d < D; ++d) {
            asm volatile("" ::"v"(wf[d][0].x), "v"(xf[d][0].x));     // a wave does not end with loads under way
            if (i + d < S) use(d);
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) lds[(((wave * MT + m) * NT + t) * 16 + g * 4 + e) * 16 + r] = acc[m][t][e];
    __syncthreads();
    auto sum = [&](int m, int t, int at) {
        int s = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += lds[((w * MT + m) * NT + t) * 256 + at];
        return s;
    };
    constexpr int kOut = GATED ? NT / 2 : NT;        // tiles of output columns
    for (int i = threadIdx.x; i < MT * kOut * 256; i += 512) {
        const int f = i % (kOut * 16), row = i / (kOut * 16);               // features fastest: whole lines of a row
        const int t = f >> 4, m = row >> 4, at = (row & 15) * 16 + (f & 15);
        const int gr = row0 + row, gc = (GATED ? tile0 / 2 : tile0) * 16 + f;
        if (gr >= rows || gc >= n) continue;
        const float sx = xscale[gr];
        float v;
        if constexpr (GATED) {
            const float* s = wscale + (tile0 + 2 * t) * 16 + (f & 15);
            v = swiglu(q8_value(sum(m, 2 * t, at), sx, s[0]), q8_value(sum(m, 2 * t + 1, at), sx, s[16]));
        } else {
            v = q8_value(sum(m, t, at), sx, wscale[gc]);
        }
        q8_put(out + (int64_t)gr * ldo + gc, v);
    }
}

int64_t q8_gemm_workspace(const amusd_q8_matrix&, int) { return 0; }

template <class OUT, bool GATED>
static void gemm(const amusd_q8_matrix& w, const int8_t* x, int64_t ldx, const float* scale, int rows, OUT* out, int64_t ldo, hipStream_t stream) {
    auto go = [&](auto kernel, int mt, int nt) {
        const int lds = 8 * mt * nt * 256 * 4;
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        hipLaunchKernelGGL(kernel, dim3((w.tiles + nt - 1) / nt, (rows + mt * 16 - 1) / (mt * 16)), dim3(512), lds, stream, w.frag, w.scale, w.kblocks, w.k,
                           w.tiles, w.n, x, ldx, scale, rows, out, ldo);
    };
    if (rows <= 16) {
        if constexpr (!GATED) {
            if (w.tiles <= w.cus) return go(k_q8_gemm_rows<OUT, GATED, 1, 1, 8>, 1, 1);
        }
        if (w.tiles <= 4 * w.cus) return go(k_q8_gemm_rows<OUT, GATED, 1, 2, 4>, 1, 2);
        return go(k_q8_gemm_rows<OUT, GATED, 1, 4, 4>, 1, 4);
    }
    if (rows <= 32) return go(k_q8_gemm_rows<OUT, GATED, 2, 2, 4>, 2, 2);
    go(k_q8_gemm_rows<OUT, GATED, 4, 2, 4>, 4, 2);
}

hipError_t launch_q8_gemm(const amusd_q8_matrix& w, const int8_t* x, int64_t ldx, const float* scale, int rows, void* out, int dtype, int64_t ldo,
                          void* work, int64_t work_bytes, hipStream_t stream) {
    (void)work;
    (void)work_bytes;
    auto go = [&](auto* o) {
        if (w.gated) gemm<std::remove_pointer_t<decltype(o)>, true>(w, x, ldx, scale, rows, o, ldo, stream);
        else gemm<std::remove_pointer_t<decltype(o)>, false>(w, x, ldx, scale, rows, o, ldo, stream);
    };
    if (dtype == AMUSD_DTYPE_BF16) go(static_cast<uint16_t*>(out));
    else go(static_cast<float*>(out));
    return hipGetLastError();
}

}  // namespace amusd
