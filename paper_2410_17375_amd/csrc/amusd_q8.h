// The operators of 8-bit models: rows to 8 bits (with or without an RMS norm), products of 8-bit integers, a key-value cache in
// 8 bits and its attention.  Types shared by their kernels and host code, and the host-callable launchers.
//
// 8 bits here: symmetric signed integers and an fp32 scale, x ~ q * s with s = max|x| / 127 over what shares the scale and
// q = x / s rounded to nearest even.  s = 0 stands for zeros; values that are not finite make s NaN (and q 0), so that whatever
// reads them is NaN as well.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/amusd.h"
#include "amusd_launch.h"
#include "amusd_plan.h"

// Opaque handles of the C interface.
struct amusd_q8_matrix {
    const uint4* frag = nullptr;   // [tile of 16 features][K / 64][64 lanes] x 16 B: lane l holds feature l%16, K bytes (l/16)*16 ..
                                   // of the block; features past n and columns past k are zeros.  Gated: tile 2t gate, 2t+1 up
    const float* scale = nullptr;  // [tiles * 16], same order
    int n = 0, k = 0;              // output columns (gated: half the features), contraction
    int tiles = 0, kblocks = 0, gated = 0, device = 0, cus = 0;
};

struct amusd_q8_cache {
    int n_layers = 0, n_seqs = 0, Hq = 0, Hkv = 0, hd = 0, G = 0, cap = 0, block = 1, device = 0, cus = 0;
    int chunk = 0;                 // keys of a chunk: its sums are complete before they are merged
    int max_chunks = 0, part_tiles = 0;
    int8_t* k = nullptr;           // [layer][seq][kv head][cap/16][hd/64][64 lanes][16]: operand order (q8_k_index)
    int8_t* v = nullptr;           // [layer][seq][kv head][cap/32][hd/32][64 lanes][16]: q + 128 in operand order (q8_v_index)
    float* ks = nullptr;           // [layer][seq][kv head][cap/block]
    float* vs = nullptr;
    float* part = nullptr;         // [part_tiles][max_chunks][hd + 2][16]: numerators, reference, denominator of 16 pairs (part_tiles: q8_part_tiles)
};

namespace amusd {

// Keeps a message for amusd_last_error and returns the code.
int report(int code, const char* what, const char* detail = nullptr);

constexpr int kQ8MaxK = 1 << 17;     // columns of a contraction: its sum of products of 127 * 127 stays inside 32 bits
constexpr int kQ8MaxFeatures = 1 << 28;      // of a matrix (fewer): two tiles of 16 a workgroup of 512 are then fewer than 2^32 threads
constexpr int kQ8MaxPositions = 1 << 24;     // of a sequence: chunks of 512 keys are a grid's third side
constexpr double kQ8MaxBytes = 0x1p48;     // of an allocation: sizes that come to more are refused before their product is taken in 64 bits
constexpr int kQ8MaxRow = 2 * 8 * 1024;   // columns of a row that a workgroup keeps in registers
constexpr int kQ8Group = 64;       // positions an append workgroup owns; the cache's capacity is a multiple of it

// A sequence's share of a call: rows row0 .. row0+n-1 are its positions pos0 .. pos0+n-1.
struct Q8Seg {
    int seq, pos0, n, row0;
    int unit0;                     // its first unit of work (append: groups of 64 positions; attention: tiles of pairs)
};
struct Q8Segs {
    int n_seg, rows, units, max_len;
    Q8Seg s[kMaxSegs];
};

// Byte of (position, column) in a kv head's keys.
__host__ __device__ inline size_t q8_k_index(int hd, int pos, int c) {
    return (((size_t)(pos >> 4) * (hd >> 6) + (c >> 6)) * 64 + ((c & 63) >> 4) * 16 + (pos & 15)) * 16 + (c & 15);
}
// .. in its values.  The 8 keys of a lane are those whose scores the lane holds: the weights then
// are the matrix instruction's operand as they come.
__host__ __device__ inline size_t q8_v_index(int hd, int pos, int c) {
    return (((size_t)(pos >> 5) * (hd >> 5) + (c >> 5)) * 64 + ((pos & 15) >> 2) * 16 + (c & 15)) * 16 + ((c >> 4) & 1) * 8 + ((pos >> 4) & 1) * 4 +
           (pos & 3);
}

hipError_t launch_q8_rows(const void* x, int dtype, int64_t ldx, const void* add, int add_dtype, int64_t ldadd, const float* gain, float eps, int rows,
                          int n, void* sum, int64_t ldsum, int8_t* q, int64_t ldq, float* scale, hipStream_t stream);
hipError_t launch_q8_gemm(const amusd_q8_matrix& w, const int8_t* x, int64_t ldx, const float* scale, int rows, void* out, int dtype, int64_t ldo,
                          void* work, int64_t work_bytes, hipStream_t stream);
int64_t q8_gemm_workspace(const amusd_q8_matrix& w, int rows);
// Memory of the handles; the caller waits for the stream before it uses them.
typedef hipError_t (*Q8Alloc)(int device, void** p, size_t bytes);
hipError_t q8_matrix_take(amusd_q8_matrix& m, int n, int k, bool gated, Q8Alloc alloc, hipStream_t stream);
hipError_t launch_q8_matrix(const amusd_q8_matrix& m, const void* w, int dtype, int64_t ld, const float* scale, int rows, int first, int part,
                            hipStream_t stream);
void q8_matrix_drop(amusd_q8_matrix& m);
hipError_t q8_cache_take(amusd_q8_cache& c, int n_layers, int n_seqs, int n_q_heads, int n_kv_heads, int head_dim, int capacity, int block, Q8Alloc alloc,
                         hipStream_t stream);
void q8_cache_drop(amusd_q8_cache& c);
void q8_append_units(Q8Segs& S);
void q8_attention_plan(amusd_q8_cache& c);        // chunk, max_chunks and part_tiles from the sizes
hipError_t launch_q8_append(const amusd_q8_cache& c, int layer, const Q8Segs& S, const void* k, const void* v, int64_t ld, const float* cos,
                            const float* sin, hipStream_t stream);
hipError_t launch_q8_read(const amusd_q8_cache& c, int layer, const Q8Segs& S, void* k, void* v, int dtype, int64_t ld, hipStream_t stream);
hipError_t launch_q8_attention(const amusd_q8_cache& c, int layer, const Q8Segs& S, const void* q, int64_t ldq, float scale, const float* cos,
                               const float* sin, void* out, int64_t ldo, hipStream_t stream);

// ---- models in 8 bits (AMUSD_DTYPE_INT8): a pass is the operators above one after the other.  Weak: the host side links
// without them where it is tested on its own, on a CPU.
struct Q8Model;

constexpr int kQ8LmRows = 256;     // rows of a prompt whose logits are there at a time (a prompt of 2048 through 4 layers and 128256 tokens: 4.07 ms; 128 rows: 4.78)

// Buffers of a pass of up to `cap` rows.
struct Q8Bufs {
    int cap = 0;
    float* X;              // residual stream [cap][d]
    int8_t* q;             // 8-bit rows on their way into a product
    float* s;              // their scales
    uint16_t* qkv;         // [cap][nqkv]
    uint16_t* att;         // [cap][qdim]
    uint16_t* delta;       // what a block adds to the residual stream [cap][d]
    uint16_t* h;           // [cap][F]
    void* work;            // of the products; zeros between passes
    int64_t work_bytes;
    float* logits;         // [min(cap, kQ8LmRows)][V], rows of a prompt whose arg-max alone is wanted; not in a pass of 16 rows
};

__attribute__((weak)) int q8_model_create(const DevModel& D, int device, Q8Alloc alloc, hipStream_t stream, Q8Model** out);
__attribute__((weak)) void q8_model_free(Q8Model* q);
// One tensor in bf16, on the device.
__attribute__((weak)) int q8_model_set(Q8Model* q, int id, int layer, const void* src, hipStream_t stream);
// Lays the buffers out from `base`; bytes.
__attribute__((weak)) size_t q8_model_bufs(const Q8Model* q, const DevModel& D, int cap, uintptr_t base, Q8Bufs& B);
__attribute__((weak)) hipError_t q8_model_pass(const Q8Model* q, const DevModel& D, const DevLayer* layers, const Q8Bufs& B, const PassArgs& P,
                                               hipStream_t stream, StageTimer* timer);
__attribute__((weak)) hipError_t q8_model_prefill(const Q8Model* q, const DevModel& D, const DevLayer* layers, const Q8Bufs& B, const PrefillBufs& T,
                                                  const PrefillArgs& P, int tail, hipStream_t stream);
// Rows of a layer's cache as fp32 rows on the device.
__attribute__((weak)) hipError_t q8_model_read(const Q8Model* q, int layer, int seq, int pos0, int n, float* k, float* v, hipStream_t stream);
constexpr int kQ8LmParts = 64;     // stretches of the vocabulary whose arg-max is found apart

}  // namespace amusd
