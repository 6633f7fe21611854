// Rows into the cache held in 8 bits: a prompt's rows, or a step's, by slots, and the accepted path's rows of every layer ("Preliminaries": the accepted
// tokens continue the sequence, the others and their descendants are discarded).
//
// Of a group of 32 rows of a head: s = the least power of two with max |x| <= 448 s, codes e4m3(x / s), to the nearest, ties to the even one.  Rows of one
// call that fall into a group are taken together by one warp: asynchronous copies bring them into 8 KB of shared memory, where every lane looks at what it has asked for, 16 bytes of a row, once for the group's maximum and again for the
// codes.  (Kept in registers, all 32 of them, an SM had 16 warps, not 24: 64 paths of up to 24 nodes in 16 layers 62 us.)
// A group that was begun before (its row 0 is not among them) keeps its scale or, where the new rows need a larger one, is
// rounded again by it: with powers of two that changes only what falls below the least codes.
// An element that is not finite has no part in the maximum and is kept as NaN.
//
// Bound by memory: 256 bytes read and 128 written a row (256 more where the caller asks for the values that are kept), and 4 KB read and written of a group that is rounded again.  Captured in a
// graph and repeated, so that no scale rises any more, prompts of four requests, 16400 rows of 8 heads with the kept values, take 32 us (161 MB: 5.0 TB/s; 33 called one after another) and those paths 55
// (252 MB with the kept values: 4.6 TB/s; by the counters 99 MB are read, so no group is, and 93 written, the rest of it later).  One row of each of 256 sequences takes 6.0 us, of one sequence in 32 layers
// 4.0 (5.3 called one after another): a launch, and loads that depend on one another (slot, row and scale, group).  Where the scales of the begun groups rise, nearly all of them, the paths read 163 MB and
// write 126: one call alone with nothing in L2 takes 76 us against 61, the prompts 39 against 37, the rows of 256 sequences 16.4 against 12.3, of one sequence 8 to 9 either way.
#include "fp8.cuh"
#include "umma_common.cuh"

namespace {

constexpr int kWarps = 4;                // of a CTA
constexpr int kRows = FSPAD_FP8_GROUP;
constexpr int kCtas = 6;                 // of an SM: 32 KB each, and 1 KB of the system's
constexpr int kStage = kRows * FSPAD_HEAD_DIM * 2;   // bytes of a warp's rows

// Larger finite magnitude among two pairs of bf16 that may hold infinities and NaN: what is none counts as 0.
__device__ __forceinline__ uint32_t finite_most(uint32_t w)
{
    uint32_t lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
    lo = lo < 0x7f80u ? lo : 0u;
    hi = hi < 0x7f80u ? hi : 0u;
    return max(lo, hi);
}

// All lanes: row `from` of lane t of src into the warp's row t, where bit t of `there` says so.
__device__ __forceinline__ void fetch(uint32_t rows, const uint4 *src, uint32_t there, long long from)
{
    const int lane = threadIdx.x & 31, piece = lane & 15, half = lane >> 4;
#pragma unroll 8
    for (int u = 0; u < kRows / 2; ++u) {
        const long long at = __shfl_sync(0xffffffffu, from, 2 * u + half);
        if ((there >> (2 * u + half)) & 1u) umma::cp_async16(rows + (uint32_t)((2 * u + half) * 256 + piece * 16), src + at * 16 + piece, true);
    }
    umma::cp_async_commit();
}

// Rows of a group that have been asked for: lane t has row t's place in src and its row of the group; bit t of `there` says whether there is one (there != 0).
// codes: row 0 of the group; scale: the group's; begun: its rows before the new ones stay.  `back`, if not NULL, receives the values that are kept, at src's places.
__device__ __forceinline__ void put_group(uint32_t rows, uint4 *back, uint8_t *codes, float *scale, uint32_t there, long long from, int to, bool begun)
{
    const int lane = threadIdx.x & 31, piece = lane & 15, half = lane >> 4;
    const float old = begun ? *scale : 0.f;          // (asked for while the rows are on their way)
    umma::cp_async_wait<0>();
    const uint32_t at0 = rows + (uint32_t)(half * 256 + piece * 16);
    uint32_t most = 0;
#pragma unroll 4
    for (int u = 0; u < kRows / 2; ++u) {
        if (!((there >> (2 * u)) & 3u)) continue;
        if ((there >> (2 * u + half)) & 1u) {
            const uint4 x = umma::ld_shared16(at0 + 512u * u);
            const uint32_t m = fspad_most2(fspad_most2(x.x, x.y), fspad_most2(x.z, x.w));
            uint32_t top = max(m & 0xffffu, m >> 16);
            if (top >= 0x7f80u) top = max(max(finite_most(x.x), finite_most(x.y)), max(finite_most(x.z), finite_most(x.w)));     // (rare)
            most = max(most, top);
        }
    }
    most = __reduce_max_sync(0xffffffffu, most);
    int field = fspad_fp8_field(most);
    bool again = false;
    float ratio = 1.f;
    if (begun) {
        const float is = fminf(fmaxf(old, kFp8Least), kFp8Most);         // (what the attention takes it for)
        field = max(field, (int)((__float_as_uint(is) + 0x7fffffu) >> 23));
        ratio = is * fspad_field_float(254 - field);             // (a reciprocal's field; exact)
        again = ratio != 1.f;
    }
    const float s = fspad_field_float(field), inv = fspad_field_float(254 - field);
    if (again) {
        // 32 rows of 128 codes: 16 codes a lane at a time
#pragma unroll 4
        for (int i = 0; i < 8; ++i) {
            uint4 *at = reinterpret_cast<uint4 *>(codes) + i * 32 + lane;
            uint4 c = *at;
            uint32_t *w = &c.x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t h[2] = {fspad_e4m3_to_f16(w[j]), fspad_e4m3_to_f16(w[j] >> 16)}, r[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[y]));
                    r[y] = fspad_f32_to_e4m3(f.x * ratio, f.y * ratio);
                }
                w[j] = r[0] | (r[1] << 16);
            }
            *at = c;
        }
    }
    __syncwarp();                                    // (the new rows' codes come after)
    if (lane == 0 && !(begun && !again && s == old)) *scale = s;
#pragma unroll 2
    for (int u = 0; u < kRows / 2; ++u) {
        if (!((there >> (2 * u)) & 3u)) continue;
        const long long at = __shfl_sync(0xffffffffu, from, 2 * u + half);
        const int row = __shfl_sync(0xffffffffu, to, 2 * u + half);
        if (!((there >> (2 * u + half)) & 1u)) continue;
        const uint4 x = umma::ld_shared16(at0 + 512u * u);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        uint32_t c[4], m = fspad_most2(fspad_most2(x.x, x.y), fspad_most2(x.z, x.w));
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = fspad_f32_to_e4m3(__uint_as_float(w[j] << 16) * inv, __uint_as_float(w[j] & 0xffff0000u) * inv);
        if (max(m & 0xffffu, m >> 16) >= 0x7f80u) {  // (an infinity, which would be cut to 448)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if ((w[j] & 0x7fffu) >= 0x7f80u) c[j] = (c[j] & 0xff00u) | 0x7fu;
                if (((w[j] >> 16) & 0x7fffu) >= 0x7f80u) c[j] = (c[j] & 0xffu) | 0x7f00u;
            }
        }
        reinterpret_cast<uint2 *>(codes)[row * 16 + piece] = make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
        if (back) {
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t h = fspad_e4m3_to_f16(c[j]);
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
                const __nv_bfloat162 v = __floats2bfloat162_rn(f.x * s, f.y * s);
                o[j] = *reinterpret_cast<const uint32_t *>(&v);
            }
            back[at * 16 + piece] = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

// Rows [2][Hkv][rows] to the slots slots[rows] of one layer.  A warp looks at `each` entries (a power of two, at most 32) of a head's K or V and takes the groups that have their first row there;
// the rows of a group stand within 32 entries.
__global__ void __launch_bounds__(kWarps * 32, kCtas)
kv_write_fp8_kernel(const uint4 *k, const uint4 *v, const long long *__restrict__ slots, int rows, int Hkv, int each, uint8_t *codes, float *scales,
                    int n_blocks, uint4 *k_rounded, uint4 *v_rounded, int *__restrict__ status)
{
    __shared__ __align__(128) unsigned char s_rows[kWarps * kStage];
    const uint32_t st = umma::smem_u32(s_rows) + (threadIdx.x >> 5) * kStage;
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int lane = threadIdx.x & 31;
    const unsigned jobs = ((unsigned)rows + each - 1) / each, job = blockIdx.x * kWarps + (threadIdx.x >> 5), of_head = job / jobs;
    if (of_head >= 2u * Hkv) return;
    const int first = (int)(job - of_head * jobs) * each, plane = of_head >= (unsigned)Hkv ? 1 : 0, head = (int)of_head - plane * Hkv;
    // entries first - 32 .. first + 63
    long long s[3];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const long long at = (long long)first + 32 * (i - 1) + lane;
        s[i] = at >= 0 && at < rows ? slots[at] : -1;
        if (s[i] < 0 || s[i] >= (long long)n_blocks * 128) {
            bad |= s[i] != -1;
            s[i] = -1;
        }
    }
    if (bad) fspad_report(status, FSPAD_ERR_RANGE);
    const long long group0 = s[0] >> 5, group1 = s[1] >> 5, group2 = s[2] >> 5;      // (-1: none)
    const long long ahead = __shfl_up_sync(0xffffffffu, group1, 1), last = __shfl_sync(0xffffffffu, group0, 31);
    // an entry whose predecessor is of the same group is not its first; of the others that is looked up
    uint32_t firsts = __ballot_sync(0xffffffffu, lane < each && group1 >= 0 && group1 != (lane > 0 ? ahead : last));
    while (firsts) {
        const int i = __ffs(firsts) - 1;
        firsts &= firsts - 1;
        const long long group = __shfl_sync(0xffffffffu, group1, i);
        const uint32_t before = __ballot_sync(0xffffffffu, group0 == group), now = __ballot_sync(0xffffffffu, group1 == group),
                       after = __ballot_sync(0xffffffffu, group2 == group);
        if ((before & (i < 31 ? ~0u << (i + 1) : 0u)) | (now & ((1u << i) - 1u))) continue;
        const uint32_t there = (now >> i) | (i > 0 ? after << (32 - i) : 0u);
        const long long sl1 = __shfl_sync(0xffffffffu, s[1], (i + lane) & 31), sl2 = __shfl_sync(0xffffffffu, s[2], (i + lane) & 31);
        const long long slot = i + lane < 32 ? sl1 : sl2;
        const long long from = (long long)head * rows + first + i + lane;
        fetch(st, plane ? v : k, there, from);
        const bool begun = !__any_sync(0xffffffffu, ((there >> lane) & 1u) && (slot & 31) == 0);
        const long long block = group >> 2, g = ((long long)plane * n_blocks + block) * Hkv + head;
        put_group(st, plane ? v_rounded : k_rounded, codes + (g * 128 + (group & 3) * kRows) * 128, scales + g * FSPAD_FP8_GROUPS + (group & 3), there, from,
                       (int)(slot & 31), begun);
    }
}

// cache row L_b + j <- tree row path[b][j] of the slice, j < n_acc[b]; a warp per (layer, K/V, sequence, head) and group of 32 rows (as many as a path of all nodes can touch).
__global__ void __launch_bounds__(kWarps * 32, kCtas)
kv_append_fp8_kernel(uint8_t *codes, float *scales, const int *__restrict__ table, int table_stride, int n_blocks, const uint4 *tree_kv,
                     const int *__restrict__ path, const int *__restrict__ n_acc, const int *__restrict__ prefix_len, int n_layers, int B, int Hkv, int N,
                     int path_stride, int groups, uint4 *rounded, int *__restrict__ new_len, int *__restrict__ status)
{
    __shared__ __align__(128) unsigned char s_rows[kWarps * kStage];
    const uint32_t st = umma::smem_u32(s_rows) + (threadIdx.x >> 5) * kStage;
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long job = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
    // (a slice has 256 bytes of tree_kv at least: 32 bits are enough for its number)
    const long long slices = (long long)n_layers * 2 * B * Hkv;
    const int group = (int)(job / slices);           // (the last ones, which few paths reach, at the end)
    const unsigned number = (unsigned)(job - group * slices), of_seq = number / (unsigned)Hkv, lk = of_seq / (unsigned)B;        // lk: layer * 2 + (K or V)
    if (group >= groups) return;
    const int h = (int)(number - of_seq * Hkv), b = (int)(of_seq - lk * B);
    const int *pth = path + (size_t)b * path_stride;
    // entries 32 (group - 1) .. of the path, before it is known which the group's are
    const int e0 = 32 * (group - 1) + lane, e1 = e0 + 32;
    const int p0 = e0 >= 0 && e0 < path_stride ? pth[e0] : -1, p1 = e1 < path_stride ? pth[e1] : -1;
    int L = prefix_len[b], n = n_acc[b];
    bool bad = false;
    if (n < 0 || n > path_stride || n > N) { bad = true; n = 0; }
    if (L < 0 || (long long)L + n > (long long)table_stride * 128) { bad = true; n = 0; }
    if (new_len && lane == 0 && lk == 0 && h == 0 && group == 0) new_len[b] = L + n;
    const int end = L + n, begin = L & ~(kRows - 1);
    if (n > 0 && group * kRows < end - begin) {      // (looked at before it is added: a row's number may be as large as 32 bits hold)
        const int r0 = begin + group * kRows;
        // row r0 + lane is entry 32 group + lane - (L % 32)
        const int back = L & (kRows - 1), from_lane = (lane - back) & 31, q0 = __shfl_sync(0xffffffffu, p0, from_lane), q1 = __shfl_sync(0xffffffffu, p1, from_lane), r = r0 + lane;
        int node = lane >= back ? q1 : q0;
        const int block = table[(size_t)b * table_stride + (r0 >> 7)];
        if (r < L || r >= end) {
            node = -1;
        } else if (node < 0 || node >= N) {
            bad = true;
            node = -1;
        }
        uint32_t there = __ballot_sync(0xffffffffu, node >= 0);
        const long long from = (long long)number * N + node;
        if (there) fetch(st, tree_kv, there, from);
        const bool inside = block >= 0 && block < n_blocks;
        if (!inside) bad = true;
        if (there && inside) {
            const long long g = ((long long)lk * n_blocks + block) * Hkv + h;
            put_group(st, rounded, codes + (g * 128 + (r0 & 127)) * 128, scales + g * FSPAD_FP8_GROUPS + ((r0 & 127) / kRows), there, from, lane, r0 < L);
        } else {
            umma::cp_async_wait<0>();                // (rows that nobody takes: they land before the CTA's memory goes)
        }
    }
    if (bad) fspad_report(status, FSPAD_ERR_RANGE);
}

}  // namespace

cudaError_t fspad_launch_kv_write_fp8(fspad_ctx *ctx, const fspad_bf16 *k, const fspad_bf16 *v, const long long *slots, int rows, int layer,
                                      uint8_t *codes, float *scales, int n_blocks, fspad_bf16 *k_rounded, fspad_bf16 *v_rounded, cudaStream_t st)
{
    const int Hkv = ctx->cfg.n_kv_heads;
    const size_t plane_blocks = (size_t)layer * 2 * n_blocks * Hkv;
    int each = 32;
    while (each > 1 && (long long)((rows + each - 1) / each) * Hkv * 2 < 16ll * ctx->sm_count) each /= 2;
    const long long jobs = (long long)((rows + each - 1) / each) * Hkv * 2;
    ctx->launches++;
    return fspad_launch(kv_write_fp8_kernel, dim3((unsigned)((jobs + kWarps - 1) / kWarps)), dim3(kWarps * 32), 0, st, 0, reinterpret_cast<const uint4 *>(k),
                        reinterpret_cast<const uint4 *>(v), slots, rows, Hkv, each, codes + plane_blocks * 128 * 128, scales + plane_blocks * FSPAD_FP8_GROUPS,
                        n_blocks, reinterpret_cast<uint4 *>(k_rounded), reinterpret_cast<uint4 *>(v_rounded), ctx->d_status);
}

cudaError_t fspad_launch_kv_append_fp8(fspad_ctx *ctx, uint8_t *codes, float *scales, FspadPaged paged, const fspad_bf16 *tree_kv, const int *path,
                                       const int *n_acc, const int *prefix_len, int N, int B, fspad_bf16 *rounded, int *new_len, cudaStream_t st)
{
    const fspad_config &c = ctx->cfg;
    const int groups = (N + 2 * kRows - 2) / kRows;              // (that N rows, from anywhere in a group on, touch)
    const long long jobs = (long long)c.n_layers * 2 * B * c.n_kv_heads * groups;
    if (jobs > 0x7fffffffll * kWarps) return cudaErrorInvalidConfiguration;
    ctx->launches++;
    return fspad_launch(kv_append_fp8_kernel, dim3((unsigned)((jobs + kWarps - 1) / kWarps)), dim3(kWarps * 32), 0, st, 0, codes, scales, paged.table,
                        paged.stride, paged.n_blocks, reinterpret_cast<const uint4 *>(tree_kv), path, n_acc, prefix_len, c.n_layers, B, c.n_kv_heads, N,
                        c.max_nodes, groups, reinterpret_cast<uint4 *>(rounded), new_len, ctx->d_status);
}
