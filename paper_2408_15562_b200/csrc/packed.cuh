// The cache held in 4 bits: layout, and the arithmetic between bf16 rows and what is kept of them.
//
// A row of 128 elements is kept as 8 blocks of 16: an e4m3 scale a block and an e2m1 code (sign, magnitude 0, 0.5, 1, 1.5, 2, 3, 4, 6) an
// element, together 72 bytes against 256.  Rows lie in blocks of 128 (a page of one sequence):
//   codes  [layers][2][n_blocks][Hkv][128][64] bytes: element 2i in the low, 2i + 1 in the high half of byte i
//   scales [layers][2][n_blocks][Hkv][128][8] bytes
// A kept value is code * scale.  It has at most six significant bits and lies in [2^-10, 2688], so that fp16 and bf16 hold it exactly.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

#define FSPAD_PACKED_CODE_BYTES 64      /* codes of a row */
#define FSPAD_PACKED_SCALE_BYTES 8      /* scales of a row */
#define FSPAD_PLAN_MAX_BATCH 1024       /* sequences of one plan: a thread each */

// Frequencies of the rotary pairs in turns a position (theta^(-2i/d) / 2 pi), and the pairs' axes: [0, split0) the first, [split0, split1)
// the second, the rest the third.
struct FspadRopeTable {
    double turns[FSPAD_HEAD_DIM / 2];
    int split0, split1;
};

cudaError_t fspad_launch_rope_qkv(fspad_ctx *ctx, const fspad_bf16 *qkv, long long row_stride, const int *positions, const int *start,
                                  const int *parent, int N, int B, const FspadRopeTable &table, bool adjacent, fspad_bf16 *q,
                                  fspad_bf16 *k, fspad_bf16 *v, cudaStream_t st);
cudaError_t fspad_launch_block_plan(fspad_ctx *ctx, const int *len, const int *add, const int *drop, int B, int bps, int n_blocks,
                                    int *table, int *held, int *free_blocks, int *n_free, int max_rows, int *row_start,
                                    long long *slots, int *row_seq, int *row_pos, cudaStream_t st);
cudaError_t fspad_launch_kv_write_packed(fspad_ctx *ctx, const fspad_bf16 *k, const fspad_bf16 *v, const long long *slots, int rows,
                                         int layer, uint8_t *codes, uint8_t *scales, int n_blocks, fspad_bf16 *k_rounded,
                                         fspad_bf16 *v_rounded, cudaStream_t st);
cudaError_t fspad_launch_kv_append_packed(fspad_ctx *ctx, uint8_t *codes, uint8_t *scales, FspadPaged paged, const fspad_bf16 *tree_kv,
                                          const int *path, const int *n_acc, const int *prefix_len, int N, int B,
                                          fspad_bf16 *rounded, int *new_len, cudaStream_t st);
size_t fspad_attn_packed_workspace(const fspad_ctx *ctx, int N, int B);
bool fspad_attn_packed_fits(const fspad_ctx *ctx, int N, int B, int bps);
cudaError_t fspad_launch_tree_attn_packed(fspad_ctx *ctx, const fspad_bf16 *q, const uint8_t *k_codes, const uint8_t *k_scales,
                                          const uint8_t *v_codes, const uint8_t *v_scales, FspadPaged paged, const fspad_bf16 *tk,
                                          const fspad_bf16 *tv, const int *parent, const int *prefix_len, int N, int B,
                                          fspad_bf16 *out, void *workspace, cudaStream_t st);

namespace packed {
// A kernel's dynamic shared memory, once a context: to the most that any call needs, for the limit is the kernel's, whoever launches it.  (Its static memory counts against the
// 48 KB that need no such call.)
static inline cudaError_t raise_shared(fspad_ctx *ctx, int bit, const void *kernel, int bytes)
{
    if ((ctx->packed_attr_done >> bit) & 1) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) ctx->packed_attr_done |= 1 << bit;
    return e;
}
}  // namespace packed

#ifdef __CUDACC__
// Eight codes (a 32-bit word) as four pairs of fp16 values, the pair of byte i in r[i].
__device__ __forceinline__ void fspad_e2m1_to_f16(uint32_t w, uint32_t (&r)[4])
{
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
}
// Two e4m3 scales as a pair of fp16 values.
__device__ __forceinline__ uint32_t fspad_e4m3_to_f16(uint32_t two_bytes)
{
    uint32_t r;
    asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}\n" : "=r"(r) : "r"(two_bytes));
    return r;
}
// Larger magnitudes of two pairs of bf16 (an infinity or a NaN stays one); what comes out has no signs.
__device__ __forceinline__ uint32_t fspad_most2(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 m = __hmax2_nan(__habs2(*reinterpret_cast<const __nv_bfloat162 *>(&a)), __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&b)));
    return *reinterpret_cast<const uint32_t *>(&m);
}
__device__ __forceinline__ uint32_t fspad_hmul2(uint32_t a, uint32_t b)
{
    const __half2 h = __hmul2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&h);
}
#endif
