// Blocks of a paged cache between requests: sequences that go on from another one's rows, blocks given back, the blocks in use moved together (the paper touches
// deployment only in its remark on practical frameworks, "Performance on Fewer Candidate Tokens"; serving systems keep the cache in fixed-size blocks).
//
// The state is whole numbers in device memory: tables, how many blocks a sequence holds, how many holders a block has beyond the first, a stack of free blocks.  One
// CTA changes it, in phases that barriers separate, and looks at everything first: what does not fit changes nothing.  Sets of blocks are bits in shared
// memory, so that lists come out in the order of the blocks' numbers whatever the order of the threads.  What bounds these is latency: dependent loads, barriers.
// The contents move in one kernel for any cache: bulk copies through shared memory, six on the way in and up to six on the way out of an SM, 16 KB each.
//
// Measured, captured in a graph (in brackets called one after another): 64 answers to four prompts of 5001 rows in 32 layers, the fork and the copy of 60 and more blocks a plane, 114 to 120 us, by the
// board (117; 537 MB written, which alone take 91 us; a source that several pairs name comes from L2, and keeping its piece in shared memory for the next pair did not help: 119.8 against 116.6);
// 88 moves of 400 blocks in bf16 74 us (76; 5.0 TB/s).  Two answers to 300 rows take 8.7 to 11.0 us (17.6), and a pool of 48 blocks with 7 moves 9.1 to 9.8 (14.2): two or three launches and their
// dependent loads.
#include "fp8.cuh"
#include "umma_common.cuh"

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;

// Exclusive sum over the CTA's threads; all of them call it.
__device__ __forceinline__ int scan(int x, int *s_warp, int &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = x;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, inc, off);
        if (lane >= off) inc += o;
    }
    __syncthreads();                     // (s_warp may still be read)
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    const int w = s_warp[lane];
    int before = lane < warp ? w : 0;
    before = __reduce_add_sync(0xffffffffu, before);
    total = __reduce_add_sync(0xffffffffu, w);
    return before + inc - x;
}

__global__ void __launch_bounds__(kThreads, 1)
block_fork_kernel(const FspadPool p, const int *__restrict__ src, const int *__restrict__ dst, int n, int *len, int *__restrict__ pairs, int *__restrict__ status)
{
    __shared__ int s_src[FSPAD_PLAN_MAX_BATCH], s_dst[FSPAD_PLAN_MAX_BATCH], s_len[FSPAD_PLAN_MAX_BATCH], s_to[FSPAD_PLAN_MAX_BATCH];
    __shared__ int s_warp[kWarps], s_bad;
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) s_bad = 0;
    s_to[tid] = 0;
    __syncthreads();
    const int free0 = *p.n_free;
    bool bad = free0 < 0 || free0 > p.n_blocks;
    int s = 0, d = 0, L = 0, part = 0;
    if (tid < n) {
        s = src[tid];
        d = dst[tid];
        if (s < 0 || s >= p.B || d < 0 || d >= p.B) {
            bad = true;
        } else {
            L = len[s];
            const int hs = p.held[s];
            if (hs < 0 || hs > p.bps || L < 0 || (long long)L > (long long)hs * 128 || p.held[d] != 0) bad = true;
            else part = (L & 127) != 0;
            if (atomicAdd(&s_to[d], 1) != 0) bad = true;         // (twice)
        }
        s_src[tid] = bad ? 0 : s;
        s_dst[tid] = d;
        s_len[tid] = bad ? 0 : L;
    }
    __syncthreads();
    if (tid < n && !bad && s_to[s] != 0) bad = true;             // (what is read is written)
    int taken;
    const int at = scan(part, s_warp, taken);
    if (taken > free0) bad = true;
    if (part && !bad) {
        const int blk = p.free_blocks[free0 - 1 - at];
        if (blk < 0 || blk >= p.n_blocks) bad = true;
    }
    if (bad) s_bad = 1;
    for (int i = warp; i < n; i += kWarps) {         // (of a thread that has found something wrong the length is 0)
        const int *row = p.table + (size_t)s_src[i] * p.bps;
        for (int j = lane; (long long)j * 128 < s_len[i]; j += 32)
            if (row[j] < 0 || row[j] >= p.n_blocks) s_bad = 1;
    }
    __syncthreads();
    if (s_bad != 0) {
        if (tid == 0) fspad_report(status, FSPAD_ERR_RANGE);
        for (int i = tid; i < 2 * n; i += kThreads) pairs[i] = -1;
        return;
    }
    for (int i = warp; i < n; i += kWarps) {
        const int *row = p.table + (size_t)s_src[i] * p.bps;
        int *to = p.table + (size_t)s_dst[i] * p.bps;
        for (int j = lane; (long long)j * 128 + 127 < s_len[i]; j += 32) {
            atomicAdd(p.shares + row[j], 1);
            to[j] = row[j];
        }
    }
    if (tid < n) {
        const int full = L >> 7;
        if (part) {
            const int blk = p.free_blocks[free0 - 1 - at];
            pairs[2 * at] = p.table[(size_t)s * p.bps + full];
            pairs[2 * at + 1] = blk;
            p.table[(size_t)d * p.bps + full] = blk;
        }
        p.held[d] = full + part;
        len[d] = L;
    }
    for (int i = 2 * taken + tid; i < 2 * n; i += kThreads) pairs[i] = -1;
    if (tid == 0) *p.n_free = free0 - taken;
}

__global__ void __launch_bounds__(kThreads, 1)
block_free_kernel(const FspadPool p, const int *__restrict__ drop, int *__restrict__ status)
{
    extern __shared__ uint32_t s_freed[];            // a bit a block
    __shared__ int s_warp[kWarps], s_bad;
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, words = (p.n_blocks + 31) / 32;
    for (int i = tid; i < words; i += kThreads) s_freed[i] = 0u;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    const int free0 = *p.n_free;
    if (free0 < 0 || free0 > p.n_blocks) s_bad = 1;
    for (int b = warp; b < p.B; b += kWarps) {
        if (drop[b] == 0) continue;
        const int h = p.held[b];
        if (h < 0 || h > p.bps) { s_bad = 1; continue; }
        for (int j = lane; j < h; j += 32) {
            const int blk = p.table[(size_t)b * p.bps + j];
            if (blk < 0 || blk >= p.n_blocks) s_bad = 1;
        }
    }
    __syncthreads();
    const bool fits = s_bad == 0;
    __syncthreads();                                 // (before anybody finds something else wrong)
    // one holder less of each; whoever takes away the last one finds 0 (every holder of a block takes one away: which of them that is does not matter)
    auto each = [&](auto f) {
        for (int b = warp; b < p.B; b += kWarps)
            if (drop[b] != 0)
                for (int j = lane; j < p.held[b]; j += 32) f(p.table[(size_t)b * p.bps + j]);
    };
    int total = 0, first = 0;
    const int per = (words + kThreads - 1) / kThreads, w0 = min(words, tid * per), w1 = min(words, w0 + per);
    if (fits) {
        each([&](int blk) {
            const int was = atomicSub(p.shares + blk, 1);
            if (was == 0) atomicOr(&s_freed[blk >> 5], 1u << (blk & 31));
            if (was < 0) s_bad = 1;                  // held more often than its count says
        });
        __syncthreads();
        int mine = 0;
        for (int i = w0; i < w1; ++i) mine += __popc(s_freed[i]);
        first = scan(mine, s_warp, total);
        if (tid == 0 && free0 + total > p.n_blocks) s_bad = 1;
        __syncthreads();
        if (s_bad != 0) {
            each([&](int blk) { atomicAdd(p.shares + blk, 1); });
        }
    }
    if (s_bad != 0) {
        if (tid == 0) fspad_report(status, FSPAD_ERR_RANGE);
        return;
    }
    // onto the stack, the highest number first: the lowest is taken next
    int at = free0 + total - 1 - first;
    for (int i = w0; i < w1; ++i)
        for (uint32_t w = s_freed[i]; w; w &= w - 1) {
            const int blk = i * 32 + __ffs(w) - 1;
            p.free_blocks[at--] = blk;
            p.shares[blk] = 0;
        }
    for (int b = tid; b < p.B; b += kThreads)
        if (drop[b] != 0) p.held[b] = 0;
    if (tid == 0) *p.n_free = free0 + total;
}

__global__ void __launch_bounds__(kThreads, 1)
block_compact_kernel(const FspadPool p, int *pairs, int max_pairs, int *__restrict__ status)
{
    extern __shared__ uint32_t s_words[];            // blocks in use | free ones, a bit each | moved ones before a word
    __shared__ int s_warp[kWarps], s_bad;
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, words = (p.n_blocks + 31) / 32;
    uint32_t *live = s_words, *idle = s_words + words;
    int *before = reinterpret_cast<int *>(s_words + 2 * words);
    for (int i = tid; i < 2 * words; i += kThreads) s_words[i] = 0u;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    const int n_free = *p.n_free;
    if (n_free < 0 || n_free > p.n_blocks) {
        s_bad = 1;
    } else {
        for (int i = tid; i < n_free; i += kThreads) {
            const int blk = p.free_blocks[i];
            if (blk < 0 || blk >= p.n_blocks || ((atomicOr(&idle[blk >> 5], 1u << (blk & 31)) >> (blk & 31)) & 1u)) s_bad = 1;
        }
    }
    for (int b = warp; b < p.B; b += kWarps) {
        const int h = p.held[b];
        if (h < 0 || h > p.bps) { s_bad = 1; continue; }
        for (int j = lane; j < h; j += 32) {
            const int blk = p.table[(size_t)b * p.bps + j];
            if (blk < 0 || blk >= p.n_blocks) s_bad = 1;
            else atomicOr(&live[blk >> 5], 1u << (blk & 31));
        }
    }
    __syncthreads();
    // the blocks that are in use or free, in order: the first of them, as many as are in use, are to be in use
    const int per = (words + kThreads - 1) / kThreads, w0 = min(words, tid * per), w1 = min(words, w0 + per);
    int mine = 0, used = 0;
    for (int i = w0; i < w1; ++i) {
        if (live[i] & idle[i]) s_bad = 1;
        mine += __popc(live[i] | idle[i]);
        used += __popc(live[i]);
    }
    int n_live, n_all, moves;
    scan(used, s_warp, n_live);
    const int rank0 = scan(mine, s_warp, n_all);
    // bits of word i that come to lie among the first n_live, the word's first having rank r
    auto low = [&](int i, int r) -> uint32_t {
        const uint32_t all = live[i] | idle[i];
        const int n = __popc(all);
        if (r + n <= n_live) return all;
        if (r >= n_live) return 0u;
        uint32_t w = all;
        for (int k = n_live - r; k > 0; --k) w &= w - 1;
        return all & ~w;
    };
    int out = 0, holes = 0;
    for (int i = w0, r = rank0; i < w1; ++i) {
        const uint32_t l = low(i, r);
        out += __popc(live[i] & ~l);
        holes += __popc(idle[i] & l);
        r += __popc(live[i] | idle[i]);
    }
    int from = scan(out, s_warp, moves);
    int into = scan(holes, s_warp, n_all);           // (as many)
    if (tid == 0 && moves > max_pairs) s_bad = 1;
    __syncthreads();
    if (s_bad != 0) {
        if (tid == 0) fspad_report(status, FSPAD_ERR_RANGE);
        for (int i = tid; i < 2 * max_pairs; i += kThreads) pairs[i] = -1;
        return;
    }
    for (int i = w0, r = rank0; i < w1; ++i) {
        const uint32_t l = low(i, r), all = live[i] | idle[i];
        before[i] = from;
        for (uint32_t w = live[i] & ~l; w; w &= w - 1) pairs[2 * from++] = i * 32 + __ffs(w) - 1;
        for (uint32_t w = idle[i] & l; w; w &= w - 1) pairs[2 * into++ + 1] = i * 32 + __ffs(w) - 1;
        // the stack, the highest number first
        int at = n_free - 1 - (r + __popc(l) - n_live);
        for (uint32_t w = all & ~l; w; w &= w - 1) p.free_blocks[at--] = i * 32 + __ffs(w) - 1;
        r += __popc(all);
        live[i] &= ~l;                               // the moved ones
    }
    __syncthreads();
    for (int i = 2 * moves + tid; i < 2 * max_pairs; i += kThreads) pairs[i] = -1;
    for (int i = tid; i < moves; i += kThreads) {
        const int x = __ldcg(pairs + 2 * i), y = __ldcg(pairs + 2 * i + 1);
        p.shares[y] = p.shares[x];
        p.shares[x] = 0;
    }
    if (moves > 0)
        for (int b = warp; b < p.B; b += kWarps)
            for (int j = lane; j < p.held[b]; j += 32) {
                int *at = p.table + (size_t)b * p.bps + j;
                const int blk = *at;
                const uint32_t w = live[blk >> 5], bit = 1u << (blk & 31);
                if (w & bit) *at = __ldcg(pairs + 2 * (before[blk >> 5] + __popc(w & (bit - 1u))) + 1);
            }
}

constexpr int kPiece = 16384, kSlots = 12, kAhead = 6;

// Blocks of one pool or two (their bytes: a multiple of 16) from pairs[i][0] to pairs[i][1] in every plane; pairs of -1 stand at the list's end.
__global__ void __launch_bounds__(32)
block_copy_kernel(unsigned char *pool0, long long bytes0, unsigned char *pool1, long long bytes1, int planes, int n_blocks, const int2 *__restrict__ pairs, int n_pairs,
                  int *__restrict__ status)
{
    extern __shared__ __align__(128) unsigned char s_ring[];
    __shared__ __align__(8) unsigned long long s_bar[kSlots];
    __shared__ unsigned char *s_to[kSlots];          // where a slot's piece goes, and how large it is
    __shared__ uint32_t s_size[kSlots];
    const int lane = threadIdx.x;
    const uint32_t ring = umma::smem_u32(s_ring), bar0 = umma::smem_u32(s_bar);
    if (lane < kSlots) umma::mbar_init(bar0 + 8u * lane, 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    __syncwarp();
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const long long pieces0 = (bytes0 + kPiece - 1) / kPiece, pieces = pieces0 + (bytes1 + kPiece - 1) / kPiece, per = pieces * planes, all = per * n_pairs;
    long long n = 0;                                 // pieces asked for so far
    bool failed = false;
    // the piece that was asked for `kAhead` ago goes out
    auto send = [&](long long i) {
        const uint32_t s = (uint32_t)(i % kSlots);
        if (!umma::mbar_wait_thread(bar0 + 8u * s, (uint32_t)(i / kSlots) & 1u)) { failed = true; return; }
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n\tcp.async.bulk.commit_group;\n"
                     :: "l"(s_to[s]), "r"(ring + s * kPiece), "r"(s_size[s]) : "memory");
    };
    for (long long x0 = blockIdx.x; x0 < all; x0 += 32ll * gridDim.x) {
        // 32 pieces at a time: which they are, a lane each
        const long long x = x0 + (long long)lane * gridDim.x;
        unsigned char *a = nullptr, *b = nullptr;
        uint32_t bytes = 0;
        bool end = x >= all;
        if (!end) {
            const long long i = x / per, y = x - i * per, plane = y / pieces, piece = y - plane * pieces;
            const int2 pr = pairs[i];
            end = pr.x < 0 && pr.y < 0;
            if (!end && (pr.x < 0 || pr.x >= n_blocks || pr.y < 0 || pr.y >= n_blocks)) {
                fspad_report(status, FSPAD_ERR_RANGE);
            } else if (!end) {
                const bool one = piece >= pieces0;
                const long long size_of = one ? bytes1 : bytes0, at = (one ? piece - pieces0 : piece) * kPiece;
                unsigned char *pool = (one ? pool1 : pool0) + plane * n_blocks * size_of + at;
                a = pool + pr.x * size_of;
                b = pool + pr.y * size_of;
                bytes = (uint32_t)min((long long)kPiece, size_of - at);
            }
        }
        const uint32_t work = __ballot_sync(0xffffffffu, bytes > 0), ends = __ballot_sync(0xffffffffu, end);
        for (uint32_t w = work; w; w &= w - 1) {
            const int l = __ffs(w) - 1;
            unsigned char *from = reinterpret_cast<unsigned char *>(__shfl_sync(0xffffffffu, (unsigned long long)a, l));
            unsigned char *dest = reinterpret_cast<unsigned char *>(__shfl_sync(0xffffffffu, (unsigned long long)b, l));
            const uint32_t count = __shfl_sync(0xffffffffu, bytes, l);
            if (lane == 0 && !failed) {
                const uint32_t s = (uint32_t)(n % kSlots);
                if (n >= kAhead) send(n - kAhead);
                // the slot's last copy out has been read: of those since it at most kSlots - kAhead are under way
                asm volatile("cp.async.bulk.wait_group.read %0;\n" ::"n"(kSlots - kAhead) : "memory");
                if (!failed) {
                    umma::mbar_expect_tx(bar0 + 8u * s, count);
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n"
                                 :: "r"(ring + s * kPiece), "l"(from), "r"(count), "r"(bar0 + 8u * s) : "memory");
                    s_to[s] = dest;
                    s_size[s] = count;
                    ++n;
                }
            }
            __syncwarp();
        }
        if (ends) break;
    }
    if (lane == 0) {
        for (long long i = n > kAhead ? n - kAhead : 0; i < n && !failed; ++i) send(i);
        if (failed) {
            fspad_report(status, FSPAD_ERR_TIMEOUT);
            // what is under way gets another bounded time to land before its memory goes
            for (long long i = n > kSlots ? n - kSlots : 0; i < n; ++i) (void)umma::mbar_wait_thread(bar0 + 8u * (uint32_t)(i % kSlots), (uint32_t)(i / kSlots) & 1u);
        }
        asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory");
    }
}

// Dynamic shared memory of the calls that keep sets of blocks.
constexpr int free_bytes(int n_blocks) { return (n_blocks + 31) / 32 * 4; }
constexpr int compact_bytes(int n_blocks) { return (n_blocks + 31) / 32 * 12; }

}  // namespace

cudaError_t fspad_launch_block_fork(fspad_ctx *ctx, const FspadPool &pool, const int *src, const int *dst, int n, int *len, int *pairs, cudaStream_t st)
{
    ctx->launches++;
    return fspad_launch(block_fork_kernel, dim3(1), dim3(kThreads), 0, st, 0, pool, src, dst, n, len, pairs, ctx->d_status);
}

cudaError_t fspad_launch_block_free(fspad_ctx *ctx, const FspadPool &pool, const int *drop, cudaStream_t st)
{
    const int smem = free_bytes(pool.n_blocks);
    const cudaError_t e = packed::raise_shared(ctx, 6, reinterpret_cast<const void *>(&block_free_kernel), free_bytes(FSPAD_PAGES_MAX_BLOCKS));
    if (e != cudaSuccess) return e;
    ctx->launches++;
    return fspad_launch(block_free_kernel, dim3(1), dim3(kThreads), smem, st, 0, pool, drop, ctx->d_status);
}

cudaError_t fspad_launch_block_compact(fspad_ctx *ctx, const FspadPool &pool, int *pairs, int max_pairs, cudaStream_t st)
{
    const int smem = compact_bytes(pool.n_blocks);
    const cudaError_t e = packed::raise_shared(ctx, 7, reinterpret_cast<const void *>(&block_compact_kernel), compact_bytes(FSPAD_PAGES_MAX_BLOCKS));
    if (e != cudaSuccess) return e;
    ctx->launches++;
    return fspad_launch(block_compact_kernel, dim3(1), dim3(kThreads), smem, st, 0, pool, pairs, max_pairs, ctx->d_status);
}

cudaError_t fspad_launch_block_copy(fspad_ctx *ctx, void *pool0, long long bytes0, void *pool1, long long bytes1, int planes, int n_blocks,
                                    const int *pairs, int n_pairs, cudaStream_t st)
{
    const int smem = kSlots * kPiece;
    const cudaError_t e = packed::raise_shared(ctx, 8, reinterpret_cast<const void *>(&block_copy_kernel), smem);
    if (e != cudaSuccess) return e;
    const long long pieces = (bytes0 + kPiece - 1) / kPiece + (bytes1 + kPiece - 1) / kPiece, all = pieces * planes * n_pairs;
    ctx->launches++;
    return fspad_launch(block_copy_kernel, dim3((unsigned)(all < ctx->sm_count ? all : ctx->sm_count)), dim3(32), smem, st, 0, static_cast<unsigned char *>(pool0), bytes0,
                        static_cast<unsigned char *>(pool1), bytes1, planes, n_blocks, reinterpret_cast<const int2 *>(pairs), n_pairs, ctx->d_status);
}
