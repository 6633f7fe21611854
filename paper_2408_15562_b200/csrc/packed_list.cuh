// What the two kernels of the attention over the 4-bit cache share: their arguments, the list of work that its CTAs cut into equal parts, and the merge of
// the runs that were cut.
//
// For every sequence, kv head and tile of BM query rows the list holds a run of units of UNIT keys: the tree's first, then the cache's.  Every CTA (or warp) takes an
// equal part of the list wherever the cuts fall, so that ragged lengths and any number of sequences fill the SMs alike, and nothing about the lengths has to be
// known on the host.  A run that was cut leaves a partial (maximum, sum, unnormalised row) for each piece.
#pragma once
#include "packed.cuh"
#include "umma_common.cuh"

namespace packed {

constexpr int D = FSPAD_HEAD_DIM;
// (With a lag of 4 the accumulators are rescaled so often that one tree of 60 nodes and 64 heads over 8, 32700 keys, takes 90.5 us, not 87.5; a longer one leaves kDown no exact form.)
constexpr float kLazyLog2 = 7.f;         // a row's reference maximum may lag its true maximum by this much (log2)
// Weights are 2^(score - reference + 7), at most 2^14 with the lag: as fp16 operands they keep their 11 bits down to 2^-21 of the reference's own.
constexpr float kBiasLog2 = 7.f;
// What is added up is a row of V times 2^-14 of its weight, so at most the row itself: V of the tree may be of any size, and 2^14 times it beyond 32 bits.  The
// cache's V goes into its products times 2^-14, which is exact (it is a multiple of 2^-10, and fp16's least value is 2^-24); of the tree's keys the weights do.
constexpr float kDown = 0x1p-14f, kUp = 0x1p14f;
constexpr uint32_t kDown2 = 0x04000400u, kOne2 = 0x3c003c00u;        // 2^-14 and 1, a pair in fp16
static_assert(kLazyLog2 + kBiasLog2 == 14.f && kDown * kUp == 1.f, "of the tree's keys the weights are 2^(score - reference - kLazyLog2)");
constexpr float kLog2e = 1.4426950408889634f;

// Division by a number that the host knows: x / d = (x * mul) >> 32 >> shift for 0 <= x < 2^31 (d of s bits: mul = 2^(31 + s) / d rounded up, which is off
// by less than d / 2^(31 + s) <= 2^-31 of it).
struct Divisor {
    unsigned d, mul, shift;
    void set(unsigned by)
    {
        d = by;
        shift = 0;
        while (shift < 31 && (1ull << shift) < by) ++shift;
        mul = by <= 1 ? 0u : (unsigned)(((1ull << (31 + shift)) + by - 1) / by);
    }
#ifdef __CUDACC__
    __device__ __forceinline__ int of(int x) const { return d <= 1u ? x : (int)(__umulhi((unsigned)x, mul) >> (shift - 1)); }
#endif
};

struct Args {
    const fspad_bf16 *q;
    const uint8_t *kc, *ks, *vc, *vs;    // codes and scales of one layer's K and V planes
    const int *table;
    int table_stride, n_blocks;
    const fspad_bf16 *tk, *tv;
    const int *parent, *prefix_len;
    int N, B, Hq, Hkv, G, M, mtiles;     // M = N * G query rows of a kv head, in mtiles tiles
    Divisor by_G, by_tiles;              // G and mtiles again
    float scale_log2;
    fspad_bf16 *out;
    float *part_o;                       // [parts][2][BM][D]: of the run that began before the part, of the one that goes on behind it.  Of 256 rows:
                                         // [..][2 row tiles][4 quarters of the columns][128][32], a row's 16-byte pieces in the order piece ^ (row & 7)
    float2 *part_ml;                     // [parts][2][BM]
    int *cuts;                           // [parts][8]: runs that were cut (see tell)
    int entry_runs;                      // no more runs than parts there can be: an entry for every run
    int *status;
};

// Where a sequence's units lie in the list.
__device__ __forceinline__ int prefix_of(const Args &a, int b, bool report)
{
    const int L = a.prefix_len[b];
    const long long most = (long long)a.table_stride * 128;
    if (L >= 0 && L <= most) return L;
    if (report) fspad_report(a.status, FSPAD_ERR_RANGE);
    return L < 0 ? 0 : (int)most;
}
template <int UNIT> __device__ __forceinline__ int tree_units(const Args &a) { return (a.N + UNIT - 1) / UNIT; }
template <int UNIT> __device__ __forceinline__ int run_units(const Args &a, int L) { return tree_units<UNIT>(a) + (int)(((long long)L + UNIT - 1) / UNIT); }
template <int UNIT> constexpr int kStretch = UNIT == 128 ? 4 : 2;

// How many parts the list may be cut into.  With chunks of 128 keys for 256 rows a part of a cut run leaves 128 KB, which cost about a hundredth of what a chunk
// takes to write and read again: of few chunks, then, fewer parts than SMs (12 sqrt(total); with 5 sqrt(total) 60 nodes over 2K keys took 25.2 us, not 20.4).
template <int UNIT> __device__ __forceinline__ int parts_of(int total, int ctas)
{
    if (UNIT == 128 && total < (ctas * ctas) / 150) ctas = max(1, (int)sqrtf((float)(total * 150)));
    return min(total, ctas);
}

// The list is cut in one of two ways.  With no more runs than parts (and no more than 32 sequences) every run is cut into equal pieces, one to a part; or the list
// into equal parts, wherever the cuts fall.  Equal parts are the shorter ones, but have stretches of two runs in them, and what a stretch costs besides
// its units (queries, the rows' way out) is worth kStretch units: the first way is taken where its longest piece is not longer by more.  (Units are counted in 32 bits: the host has seen to it that they fit.)
struct Parts {
    int n, q, r;                         // parts, units / parts, units % parts
    __device__ __forceinline__ int start(int i) const { return i * q + min(i, r); }
    __device__ __forceinline__ int owner(int x) const { const int b = r * (q + 1); return x < b ? x / (q + 1) : r + (x - b) / q; }
};

// A part: it begins at unit u of run `run` (kv head and tile) of sequence b and is `left` units long, over further runs and sequences as they come.
struct Part {
    int b, run, u, left;
    int i0, i1;                          // pieces of the run that the part begins in: the parts that hold the first and the last of them
    bool by_run;                         // cut in the first way: i0 and i1 hold
};

// All T threads of the CTA call it, and there is a CTA barrier in it; scratch holds T / 32 + 2 W values.  W: how many parts a CTA takes: one, which all its
// threads ask for, or one for each of its W = T / 32 warps: part0 + w * gridDim.x, so that few parts are on as many SMs.  slots: how many there may be.
template <int T, int UNIT, int W>
__device__ __forceinline__ Part cut_list(const Args &a, int part0, int slots, Parts &p, int *scratch, bool report)
{
    const int part = part0 + (W > 1 ? (int)(threadIdx.x >> 5) * (int)gridDim.x : 0), ctas = slots;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, runs = a.Hkv * a.mtiles;
    Part s = {0, 0, 0, 0, 0, 0, false};
    if (a.B <= 32) {                     // every warp for itself
        const int n = lane < a.B ? run_units<UNIT>(a, prefix_of(a, lane, report)) : 0;
        int inc = runs * n;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, inc, off);
            if (lane >= off) inc += o;
        }
        const int total = __shfl_sync(0xffffffffu, inc, 31);
        p.n = parts_of<UNIT>(total, ctas);
        p.q = total / p.n;
        p.r = total - p.q * p.n;
        const int want = part < p.n ? p.start(part) : total, most = p.q + kStretch<UNIT>;
        if (a.B * runs <= p.n) {
            // the smallest piece with which there are no more pieces than parts, from below, within a step or two
            int k = 0, sum = 0, q = max(1, (total + p.n - 1) / p.n), by_run = 0;
            while (q <= most) {
                k = lane < a.B ? (n + q - 1) / q : 0;
                inc = runs * k;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const int o = __shfl_up_sync(0xffffffffu, inc, off);
                    if (lane >= off) inc += o;
                }
                sum = __shfl_sync(0xffffffffu, inc, 31);
                if (sum <= p.n) { by_run = 1; break; }
                q += max(1, (int)((float)q * (float)(sum - p.n) / (float)(2 * sum)));
            }
            if (by_run) {
                s.by_run = true;
                p.n = sum;
                if (part < sum) {
                    s.b = __popc(__ballot_sync(0xffffffffu, inc <= part));
                    k = __shfl_sync(0xffffffffu, k, s.b);
                    const int nb = __shfl_sync(0xffffffffu, n, s.b), x = part - (s.b > 0 ? __shfl_sync(0xffffffffu, inc, s.b - 1) : 0);
                    s.run = x / k;
                    const int piece = x - s.run * k, w = nb / k, more = nb - w * k;          // the first `more` pieces are of w + 1 units
                    s.u = piece * w + min(piece, more);
                    s.left = w + (piece < more ? 1 : 0);
                    s.i0 = part - piece;
                    s.i1 = s.i0 + k - 1;
                }
                __syncthreads();
                return s;
            }
            inc = runs * n;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, inc, off);
                if (lane >= off) inc += o;
            }
        }
        if (part < p.n) {
            s.b = __popc(__ballot_sync(0xffffffffu, inc <= want));
            const int nb = __shfl_sync(0xffffffffu, n, s.b), x = want - (s.b > 0 ? __shfl_sync(0xffffffffu, inc, s.b - 1) : 0);
            s.run = x / nb;
            s.u = x - s.run * nb;
            s.left = p.start(part + 1) - want;
        }
        __syncthreads();
        return s;
    }
    const int per = (a.B + T - 1) / T;
    const int b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
    int mine = 0;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) mine += runs * run_units<UNIT>(a, prefix_of(a, b, report));
    int inc = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, inc, off);
        if (lane >= off) inc += o;
    }
    if (lane == 31) scratch[warp] = inc;
    __syncthreads();
    int total = 0;
#pragma unroll 4
    for (int w = 0; w < T / 32; ++w) {
        if (w < warp) inc += scratch[w];
        total += scratch[w];
    }
    p.n = parts_of<UNIT>(total, ctas);
    p.q = total / p.n;
    p.r = total - p.q * p.n;
    int x = inc - mine;
#pragma unroll 1
    for (int w = 0; w < W; ++w) {
        const int its = part0 + w * (int)gridDim.x, want = its < p.n ? p.start(its) : total;
        if (x <= want && want < inc) {
            int b = b0, y = x;
#pragma unroll 1
            for (; b < b1; ++b) {
                const int n = runs * run_units<UNIT>(a, prefix_of(a, b, false));
                if (want < y + n) break;
                y += n;
            }
            scratch[T / 32 + 2 * w] = b;
            scratch[T / 32 + 2 * w + 1] = want - y;
        }
    }
    __syncthreads();
    if (part < p.n) {
        const int at = T / 32 + (W > 1 ? 2 * warp : 0);
        s.b = scratch[at];
        const int nb = run_units<UNIT>(a, prefix_of(a, s.b, false));
        s.run = scratch[at + 1] / nb;
        s.u = scratch[at + 1] - s.run * nb;
        s.left = p.start(part + 1) - p.start(part);
    }
    return s;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// shared -> global; the thread that issued copies waits until their source may be written again, and until they are done
__device__ __forceinline__ void bulk_store(void *dst, uint32_t src, uint32_t bytes)
{
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n\tcp.async.bulk.commit_group;\n" :: "l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_store_read() { asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory"); }
__device__ __forceinline__ void bulk_store_read_but_one() { asm volatile("cp.async.bulk.wait_group.read 1;\n" ::: "memory"); }
__device__ __forceinline__ void bulk_store_wait() { asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory"); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// Whether one of the two bf16 of a word is an infinity or a NaN.
__device__ __forceinline__ bool odd_value(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

// Word of the runs that were cut, for the merge: sequence (-1: nothing to merge), kv head, tile, and the parts that hold the first and the last piece.
// Where there is an entry for every run (a.entry_runs), the n-th is the n-th run's, and the part that holds the run's beginning, as its unit 0 comes, writes it; otherwise
// the n-th is the n-th part's, of the run that the part begins inside of, if it holds the second piece.
__device__ __forceinline__ void tell(const Args &a, int n, int b, int run, int i0, int i1)
{
    const int h = a.by_tiles.of(run);
    reinterpret_cast<int4 *>(a.cuts)[2 * n] = make_int4(i1 > i0 ? b : -1, h, run - h * a.mtiles, i0);
    a.cuts[8 * n + 4] = i1;
}
// One thread for every part, before anything of it is taken.
template <int UNIT> __device__ __forceinline__ void tell_part(const Args &a, const Parts &p, const Part &s, int part)
{
    if (a.entry_runs) return;
    int i0 = 0, i1 = 0;
    if (s.left > 0 && s.u > 0) {
        const int start = p.start(part) - s.u;
        i0 = p.owner(start);
        i1 = i0 == part - 1 ? p.owner(start + run_units<UNIT>(a, prefix_of(a, s.b, false)) - 1) : i0;
    }
    tell(a, part, s.b, s.run, i0, i1);
}
// One thread, when the part comes to the beginning of a run (s.u = 0): `done` units of the part lie before it.
__device__ __forceinline__ void tell_run(const Args &a, const Parts &p, const Part &s, int part, int done, int n_run)
{
    if (!a.entry_runs) return;
    tell(a, (s.b * a.Hkv * a.mtiles) + s.run, s.b, s.run, part, s.by_run ? s.i1 : p.owner(p.start(part) + done + n_run - 1));
}

// The pieces of the runs that were cut, merged.  A CTA takes `rows` rows (a power of two, at most WARPS) of a run at a time, each by WARPS / rows warps that take its
// pieces in turn, four elements a lane.
template <int BM, int WARPS, int U>           // U: pieces of a row under way
__global__ void __launch_bounds__(WARPS * 32, WARPS > 8 ? 1 : U > 2 ? 3 : 6)
tree_attn_packed_merge_kernel(const Args a, int rows, int parts)
{
    __shared__ float4 s_acc[WARPS][32];
    __shared__ float2 s_ml[WARPS];
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wpr = WARPS / rows;
    const int4 run = __ldcg(reinterpret_cast<const int4 *>(a.cuts) + 2 * blockIdx.x);
    const int i0 = run.w, i1 = __ldcg(a.cuts + 8 * blockIdx.x + 4);
    // (-1: nothing to merge; and should a part have given up, its runs were never told of, and what is read is no run)
    if ((unsigned)run.x >= (unsigned)a.B || (unsigned)run.y >= (unsigned)a.Hkv || (unsigned)run.z >= (unsigned)a.mtiles || i0 < 0 || i1 < i0 || i1 >= parts) return;
#pragma unroll 1
    for (int row0 = blockIdx.y * rows; row0 < BM && run.z * BM + row0 < a.M; row0 += gridDim.y * rows) {
        const int row = row0 + warp % rows, gr = run.z * BM + row;
        const bool there = gr < a.M;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        float l = 0.f, m = -INFINITY;
        auto add = [&](float2 ml, float4 v, float m_new) {   // (without a maximum a piece's sum and row are zero, or NaN)
            const float w = ml.x == -INFINITY ? 1.f : umma::ex2f(ml.x - m_new);
            l += w * ml.y;
            acc.x += w * v.x; acc.y += w * v.y; acc.z += w * v.z; acc.w += w * v.w;
        };
        auto move = [&](float m_new) {
            const float w = m == -INFINITY ? 1.f : umma::ex2f(m - m_new);
            l *= w;
            acc.x *= w; acc.y *= w; acc.z *= w; acc.w *= w;
            m = m_new;
        };
        if (there) {
#pragma unroll 1
            for (int i = i0 + warp / rows; i <= i1; i += U * wpr) {
                float2 ml[U];
                float4 v[U];
                float top = m;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int at = i + u * wpr;
                    ml[u] = make_float2(-INFINITY, 0.f);
                    v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (at <= i1) {
                        const size_t slot = ((size_t)at * 2 + (at == i0 ? 1 : 0)) * BM + row;
                        ml[u] = __ldcg(&a.part_ml[slot]);
                        v[u] = __ldcg(reinterpret_cast<const float4 *>(a.part_o) + (BM == 256 ? (slot >> 7) * 4096 + (lane >> 3) * 1024 + (row & 127) * 8 + ((lane & 7) ^ (row & 7))
                                                                                              : slot * (D / 4) + lane));
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) top = fmaxf(top, ml[u].x);
                move(top);
#pragma unroll
                for (int u = 0; u < U; ++u) add(ml[u], v[u], top);
            }
        }
        if (wpr > 1) {
            __syncthreads();
            s_acc[warp][lane] = acc;
            if (lane == 0) s_ml[warp] = make_float2(m, l);
            __syncthreads();
            if (warp < rows) {
                float top = -INFINITY;
                for (int w = warp; w < WARPS; w += rows) top = fmaxf(top, s_ml[w].x);
                move(top);
                for (int w = warp + rows; w < WARPS; w += rows) add(s_ml[w], s_acc[w][lane], top);
            }
        }
        if (warp < rows && there) {
            const float inv = kUp / l;
            const int node = a.by_G.of(gr);
            *reinterpret_cast<uint2 *>(a.out + (((size_t)run.x * a.N + node) * a.Hq + run.y * a.G + (gr - node * a.G)) * D + 4 * lane) =
                make_uint2(umma::pack_bf16(acc.x * inv, acc.y * inv), umma::pack_bf16(acc.z * inv, acc.w * inv));
        }
    }
}

// The scratch of a call of so many parts: partial rows, their maxima and sums, the cuts.
template <int BM> static inline size_t scratch_bytes(int parts)
{
    return (size_t)parts * (2 * BM * (D * sizeof(float) + sizeof(float2)) + 8 * sizeof(int));
}
template <int BM> static inline void scratch_in(Args &a, int parts, void *workspace)
{
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<float2 *>(a.part_o + (size_t)parts * 2 * BM * D);
    a.cuts = reinterpret_cast<int *>(a.part_ml + (size_t)parts * 2 * BM);
}

// A kernel's dynamic shared memory, once a context.
static inline cudaError_t raise_shared(fspad_ctx *ctx, int bit, const void *kernel, int bytes)
{
    if ((ctx->packed_attr_done >> bit) & 1) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) ctx->packed_attr_done |= 1 << bit;
    return e;
}

// Parts there can be -> how the runs that were cut are told of; and the merge's launch: entries x groups of so many rows, so that they are all there at once (three CTAs an SM).
static inline int merge_entries(Args &a, int parts)
{
    const long long runs = (long long)a.B * a.Hkv * a.mtiles;
    a.entry_runs = runs <= parts ? 1 : 0;
    return a.entry_runs ? (int)runs : parts;
}
template <int BM> static inline cudaError_t launch_merge(fspad_ctx *ctx, const Args &a, int entries, int parts, cudaStream_t st)
{
    const int m = a.M < BM ? a.M : BM;
    ctx->launches++;
    // a row a CTA, with twice the warps, where that is no more than a CTA an SM (long runs in many pieces: 21.6 us against 24.9 on one token over 32K keys)
    if ((long long)entries * m <= ctx->sm_count)
        return fspad_launch(tree_attn_packed_merge_kernel<BM, 16, 8>, dim3((unsigned)entries, (unsigned)m), dim3(512), 0, st, 0, a, 1, parts);
    int rows = 1;
    while (rows < 8 && rows < m && (long long)entries * ((m + rows - 1) / rows) > 3 * ctx->sm_count) rows *= 2;
    const dim3 grid((unsigned)entries, (unsigned)((m + rows - 1) / rows));
    // runs in two pieces or three: fewer loads a row and twice the rows on an SM (16 trees of 60 nodes, 32 heads over 8, 512 to 4096 keys 95.6 -> 87.7 us, but
    // one tree over 2K keys, in 19 pieces a run, 19.6 -> 23.9)
    if ((long long)a.B * a.Hkv * a.mtiles * 2 >= parts) return fspad_launch(tree_attn_packed_merge_kernel<BM, 8, 2>, grid, dim3(256), 0, st, 0, a, rows, parts);
    return fspad_launch(tree_attn_packed_merge_kernel<BM, 8, 8>, grid, dim3(256), 0, st, 0, a, rows, parts);
}

// Whether the units of a call, at most, can be counted in 32 bits (and 25 times as many as are cut into fewer parts than there are CTAs).
template <int UNIT> static inline bool units_fit(const Args &a)
{
    const long long run = ((long long)a.N + UNIT - 1) / UNIT + ((long long)a.table_stride * 128 + UNIT - 1) / UNIT;
    return (double)run * a.B * a.Hkv * a.mtiles < 2147483647.0 - 1e6;
}

}  // namespace packed

size_t fspad_attn_packed_umma_workspace(const fspad_ctx *ctx);
cudaError_t fspad_launch_attn_packed_umma(fspad_ctx *ctx, packed::Args a, void *workspace, cudaStream_t st);
