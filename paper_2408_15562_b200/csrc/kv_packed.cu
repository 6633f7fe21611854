// Rows into the cache held in 4 bits: a prompt's rows by slots, and the accepted path's rows of every layer ("Preliminaries": the accepted
// tokens continue the sequence, the others and their descendants are discarded).
//
// Of every 16 elements: scale s = e4m3(max |x| / 6), codes e2m1(x / s), both to the nearest value, ties to the even code, a larger
// magnitude than the type has to its largest.  A division here is a product with a reciprocal that is 2^-20 too large, cut to 12 significant bits: a quotient
// that is a tie of the type (three bits, of a scale five) comes out a little above it and is met again, and nothing else can come to look like one, because
// x has 8 significant bits, s four and a tie three, so that a quotient that is no tie lies at least 1/256 of its value away from one.  (Divisions, and
// quotients rounded by an addition and given their sign back, took half as many instructions again, and the instructions bounded the kernels: 16K rows
// of 8 heads 33.0 us.)
// A block with an infinity or a NaN gets a scale that is no number and codes of zero: it reads as NaN.
//
// Bound by memory in the end, 256 bytes read and 72 written a row (256 more where the caller asks for the values that are kept), and by the issue of
// instructions nearly as much (some 80 for eight elements; 84 % of the slots taken when they were 130).  Half a warp
// takes a row, 16 bytes a lane, so that two lanes share a scale; four pairs of rows are in flight (two: 30.7 us against 29.4 on 16K rows of 8 heads, eight:
// 33.7 against 33.1 when both were slower).  With the values kept, by the bytes of the rows that are: 16411 rows of 8 heads 29.8 us, 5.15 TB/s (a seventh of
// them left out 29.2 us, 4.8 TB/s); 64 paths of up to 24 nodes in 16 layers 45.1 us, 5.0 TB/s.  Without, where nothing but the instructions is left: 23.6 us and 33.2 us, 3.7 and 3.8 TB/s.
#include "packed.cuh"

namespace {

constexpr int kWarpsPerCta = 8;
constexpr int kInFlight = 4;             // row pairs

// See above: what reciprocals are too large by, and a quotient's first 12 bits.
constexpr float kUp = 1.0f + 0x1p-20f;
__device__ __forceinline__ float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xfffff000u); }

// Eight elements of a row (two bf16 a word) -> their codes; `scale` is the block's, which the neighbouring lane (lane ^ 1) shares.
// With `rounded` the kept values come back in x.
__device__ __forceinline__ uint32_t quantise(uint4 &x, uint32_t &scale, bool rounded)
{
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t m = fspad_most2(fspad_most2(w[0], w[1]), fspad_most2(w[2], w[3]));
    m = max(m & 0xffffu, m >> 16);       // (magnitudes of bf16 order like whole numbers, infinities and NaN on top)
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    const bool finite = m < 0x7f80u;
    const float most = cut(__uint_as_float(m << 16) * (kUp / 6.0f));
    uint16_t two;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(two) : "f"(0.0f), "f"(finite ? most : 0.0f));
    const uint32_t f16 = fspad_e4m3_to_f16(two);
    const float s = __half2float(__ushort_as_half((unsigned short)f16));
    const float r = s > 0.0f ? __fdividef(kUp, s) : 0.0f;
    scale = finite ? (two & 0xffu) : 0x7fu;
    float q[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        q[2 * i] = cut(__uint_as_float(w[i] << 16) * r);
        q[2 * i + 1] = cut(__uint_as_float(w[i] & 0xffff0000u) * r);
    }
    uint32_t codes;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}\n"
        : "=r"(codes) : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    if (!finite) codes = 0;
    if (rounded) {
        uint32_t h[4];
        fspad_e2m1_to_f16(codes, h);
        const uint32_t sc = finite ? (f16 & 0xffffu) * 0x10001u : 0x7e007e00u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = fspad_hmul2(h[i], sc);
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&v));
            const __nv_bfloat162 o = __floats2bfloat162_rn(f.x, f.y);
            w[i] = *reinterpret_cast<const uint32_t *>(&o);
        }
        x = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return codes;
}

// Rows [2][Hkv][rows] of a prompt to the slots slots[rows] (block * 128 + row of it) of one layer; a warp takes eight consecutive rows.
__global__ void __launch_bounds__(kWarpsPerCta * 32)
kv_write_packed_kernel(const uint4 *k, const uint4 *v, const long long *__restrict__ slots, int rows, int Hkv,
                       uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, int n_blocks, uint4 *k_rounded, uint4 *v_rounded,
                       int *__restrict__ status)
{
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int lane = threadIdx.x & 31, piece = lane & 15, half = lane >> 4;
    // (32 bits are enough for the number, and a division of 64 takes a hundred instructions)
    const unsigned groups = (unsigned)(rows + 2 * kInFlight - 1) / (2 * kInFlight), job = blockIdx.x * kWarpsPerCta + (threadIdx.x >> 5);
    const unsigned of_head = job / groups;
    if (of_head >= 2u * Hkv) return;
    const int group = (int)(job - of_head * groups), plane = of_head >= (unsigned)Hkv ? 1 : 0, head = (int)of_head - plane * Hkv;
    const long long first = ((long long)plane * n_blocks * Hkv + head) * 128;        // the head's rows of a block: 128 Hkv to the next block's
    const uint4 *src = (plane ? v : k) + (long long)head * rows * 16;
    uint4 *back = plane ? v_rounded : k_rounded;
    uint4 x[kInFlight];
    long long slot[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
        const int r = group * 2 * kInFlight + 2 * u + half;
        slot[u] = -1;
        x[u] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows) {
            slot[u] = slots[r];
            x[u] = src[(long long)r * 16 + piece];
        }
        if (slot[u] < -1 || slot[u] >= (long long)n_blocks * 128) {
            fspad_report(status, FSPAD_ERR_RANGE);
            slot[u] = -1;
        }
    }
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
        const int r = group * 2 * kInFlight + 2 * u + half;
        uint32_t scale;
        const uint32_t c = quantise(x[u], scale, back != nullptr);
        if (slot[u] < 0) continue;
        const long long to = first + (long long)(int)(slot[u] >> 7) * (Hkv * 128) + (slot[u] & 127);
        reinterpret_cast<uint32_t *>(codes)[to * 16 + piece] = c;
        if (!(piece & 1)) scales[to * 8 + (piece >> 1)] = (uint8_t)scale;
        if (back) back[((long long)head * rows + r) * 16 + piece] = x[u];
    }
}

// cache row L_b + j <- tree row path[b][j] of the slice, j < n_acc[b]; one warp per (layer, K/V, sequence, head).
__global__ void __launch_bounds__(kWarpsPerCta * 32)
kv_append_packed_kernel(uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, const int *__restrict__ table, int table_stride,
                        int n_blocks, const uint4 *tree_kv, const int *__restrict__ path, const int *__restrict__ n_acc,
                        const int *__restrict__ prefix_len, int n_layers, int B, int Hkv, int N, int path_stride, uint4 *rounded,
                        int *__restrict__ new_len, int *__restrict__ status)
{
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int lane = threadIdx.x & 31, piece = lane & 15, half = lane >> 4;
    // (a slice has 256 bytes of tree_kv at least: 32 bits are enough for the number)
    const unsigned number = blockIdx.x * kWarpsPerCta + (threadIdx.x >> 5), of_seq = number / (unsigned)Hkv, lk = of_seq / (unsigned)B;  // lk: layer * 2 + (K or V)
    if (lk >= 2u * n_layers) return;
    const int h = (int)(number - of_seq * Hkv), b = (int)(of_seq - lk * B);
    const long long slice = number, first = ((long long)lk * n_blocks * Hkv + h) * 128;      // the head's rows of a block: 128 Hkv to the next block's
    int L = prefix_len[b], n = n_acc[b];
    const int *pth = path + (size_t)b * path_stride;
    bool bad = false;
    if (n < 0 || n > path_stride || n > N) { bad = true; n = 0; }
    if (L < 0 || (long long)L + n > (long long)table_stride * 128) { bad = true; n = 0; }
    if (new_len && lane == 0 && lk == 0 && h == 0) new_len[b] = L + n;
    const uint4 *src = tree_kv + slice * N * 16;
    for (int j0 = 0; j0 < n; j0 += 32) {
        // nodes and blocks of 32 rows at once, a lane each: a trip to memory for every few rows was a third of the time
        int node_of = -1, block_of = -1;
        if (j0 + lane < n) {
            node_of = pth[j0 + lane];
            block_of = table[(size_t)b * table_stride + ((L + j0 + lane) >> 7)];
            if (node_of < 0 || node_of >= N || block_of < 0 || block_of >= n_blocks) { bad = true; node_of = -1; }
        }
#pragma unroll 1
        for (int j1 = 0; j1 < min(32, n - j0); j1 += 2 * kInFlight) {
            uint4 x[kInFlight];
            int node[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                node[u] = __shfl_sync(0xffffffffu, node_of, j1 + 2 * u + half);
                x[u] = make_uint4(0u, 0u, 0u, 0u);
                if (node[u] >= 0) x[u] = src[(long long)node[u] * 16 + piece];
            }
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                const int block = __shfl_sync(0xffffffffu, block_of, j1 + 2 * u + half);
                uint32_t scale;
                const uint32_t c = quantise(x[u], scale, rounded != nullptr);
                if (node[u] < 0) continue;
                const long long to = first + (long long)block * (Hkv * 128) + ((L + j0 + j1 + 2 * u + half) & 127);
                reinterpret_cast<uint32_t *>(codes)[to * 16 + piece] = c;
                if (!(piece & 1)) scales[to * 8 + (piece >> 1)] = (uint8_t)scale;
                if (rounded) rounded[(slice * N + node[u]) * 16 + piece] = x[u];
            }
        }
    }
    if (bad) fspad_report(status, FSPAD_ERR_RANGE);
}

}  // namespace

cudaError_t fspad_launch_kv_write_packed(fspad_ctx *ctx, const fspad_bf16 *k, const fspad_bf16 *v, const long long *slots, int rows,
                                         int layer, uint8_t *codes, uint8_t *scales, int n_blocks, fspad_bf16 *k_rounded,
                                         fspad_bf16 *v_rounded, cudaStream_t st)
{
    const int Hkv = ctx->cfg.n_kv_heads;
    const size_t plane_rows = (size_t)layer * 2 * n_blocks * Hkv * 128;
    const long long jobs = (long long)((rows + 2 * kInFlight - 1) / (2 * kInFlight)) * Hkv * 2;
    ctx->launches++;
    return fspad_launch(kv_write_packed_kernel, dim3((unsigned)((jobs + kWarpsPerCta - 1) / kWarpsPerCta)), dim3(kWarpsPerCta * 32), 0, st, 0,
                        reinterpret_cast<const uint4 *>(k), reinterpret_cast<const uint4 *>(v), slots, rows, Hkv,
                        codes + plane_rows * FSPAD_PACKED_CODE_BYTES, scales + plane_rows * FSPAD_PACKED_SCALE_BYTES, n_blocks,
                        reinterpret_cast<uint4 *>(k_rounded), reinterpret_cast<uint4 *>(v_rounded), ctx->d_status);
}

cudaError_t fspad_launch_kv_append_packed(fspad_ctx *ctx, uint8_t *codes, uint8_t *scales, FspadPaged paged, const fspad_bf16 *tree_kv,
                                          const int *path, const int *n_acc, const int *prefix_len, int N, int B,
                                          fspad_bf16 *rounded, int *new_len, cudaStream_t st)
{
    const fspad_config &c = ctx->cfg;
    const long long slices = (long long)c.n_layers * 2 * B * c.n_kv_heads;
    ctx->launches++;
    return fspad_launch(kv_append_packed_kernel, dim3((unsigned)((slices + kWarpsPerCta - 1) / kWarpsPerCta)), dim3(kWarpsPerCta * 32), 0, st, 0,
                        codes, scales, paged.table, paged.stride, paged.n_blocks, reinterpret_cast<const uint4 *>(tree_kv), path, n_acc,
                        prefix_len, c.n_layers, B, c.n_kv_heads, N, c.max_nodes, reinterpret_cast<uint4 *>(rounded), new_len, ctx->d_status);
}
