// The cache held in 8 bits: layout, and the arithmetic between bf16 rows and what is kept of them.
//
// A row of 128 elements is kept as 128 e4m3 codes; 32 rows of a head (a group: a quarter of a block of 128 rows) share a single-precision scale:
//   codes  [layers][2][n_blocks][Hkv][128][128] bytes
//   scales [layers][2][n_blocks][Hkv][4] float
// A kept value is code * scale.  The scales that the writes leave are powers of two, 2^e with e from -64 to 64: products with them and with their
// reciprocals are exact, and a group whose scale rises loses nothing but what falls below its least codes.
#pragma once
#include "packed.cuh"

#define FSPAD_FP8_GROUP 32                              /* rows that share a scale */
#define FSPAD_FP8_GROUPS (128 / FSPAD_FP8_GROUP)        /* of a block */
#define FSPAD_PAGES_MAX_BLOCKS (1 << 19)                /* blocks of a pool that is forked, freed or compacted: a bit each in shared memory, and more */

struct FspadPool {                       // what the calls on blocks keep of a pool (device)
    int *table;                          // [B][bps]
    int *held;                           // [B]
    int *shares;                         // [n_blocks]: holders of a block beyond the first
    int *free_blocks, *n_free;           // a stack
    int B, bps, n_blocks;
};

cudaError_t fspad_launch_kv_write_fp8(fspad_ctx *ctx, const fspad_bf16 *k, const fspad_bf16 *v, const long long *slots, int rows, int layer,
                                      uint8_t *codes, float *scales, int n_blocks, fspad_bf16 *k_rounded, fspad_bf16 *v_rounded, cudaStream_t st);
cudaError_t fspad_launch_kv_append_fp8(fspad_ctx *ctx, uint8_t *codes, float *scales, FspadPaged paged, const fspad_bf16 *tree_kv, const int *path,
                                       const int *n_acc, const int *prefix_len, int N, int B, fspad_bf16 *rounded, int *new_len, cudaStream_t st);
size_t fspad_attn_fp8_workspace(const fspad_ctx *ctx);
bool fspad_attn_fp8_fits(const fspad_ctx *ctx, int N, int B, int bps, int n_blocks);
cudaError_t fspad_launch_tree_attn_fp8(fspad_ctx *ctx, const fspad_bf16 *q, const uint8_t *k_codes, const float *k_scales, const uint8_t *v_codes,
                                       const float *v_scales, FspadPaged paged, const fspad_bf16 *tk, const fspad_bf16 *tv, const int *parent,
                                       const int *prefix_len, int N, int B, fspad_bf16 *out, void *workspace, cudaStream_t st);
cudaError_t fspad_launch_block_fork(fspad_ctx *ctx, const FspadPool &pool, const int *src, const int *dst, int n, int *len, int *pairs, cudaStream_t st);
cudaError_t fspad_launch_block_free(fspad_ctx *ctx, const FspadPool &pool, const int *drop, cudaStream_t st);
cudaError_t fspad_launch_block_compact(fspad_ctx *ctx, const FspadPool &pool, int *pairs, int max_pairs, cudaStream_t st);
cudaError_t fspad_launch_block_copy(fspad_ctx *ctx, void *pool0, long long bytes0, void *pool1, long long bytes1, int planes, int n_blocks,
                                    const int *pairs, int n_pairs, cudaStream_t st);

#ifdef __CUDACC__
// Exponent fields of the least and the largest scale that the writes leave.
constexpr int kFp8LeastField = 127 - 64, kFp8MostField = 127 + 64;
constexpr float kFp8Least = 0x1p-64f, kFp8Most = 0x1p64f;
constexpr float kMost = 0x1.fffffep127f;                         // (single precision's)

// Exponent field of the least power of two 2^e with which a finite bf16 magnitude (its bits) is at most 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int fspad_fp8_field(uint32_t magnitude)
{
    const int f = (int)((magnitude + 0x1fu) >> 7) - 8;           // (a mantissa above 1.75 carries)
    return min(max(f, kFp8LeastField), kFp8MostField);
}
__device__ __forceinline__ float fspad_field_float(int field) { return __uint_as_float((uint32_t)field << 23); }
// Two codes from two values, to the nearest, ties to the even one, beyond 448 to 448; the first in the low byte.
__device__ __forceinline__ uint32_t fspad_f32_to_e4m3(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
#endif
