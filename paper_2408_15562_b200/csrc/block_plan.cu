// Block tables and slots of a paged cache from the lengths of the requests (the paper touches deployment only in its remark on practical
// frameworks, "Performance on Fewer Candidate Tokens"; serving systems keep the cache in fixed-size blocks).
//
// One cluster does it all, in phases that a cluster barrier separates, so that no host round trip and no second launch is needed: every CTA
// scans the (at most 1024) sequences for itself, a thread each; blocks of dropped sequences are pushed onto the free stack; blocks are popped
// into the tables; then the rows' slots are written.  What bounds it is latency: for a step of a batch (16 sequences 4.0 us) the barriers and dependent
// loads; for prompts the instructions of eight SMs besides (200 requests of up to 600 rows, 61000 in all, 11.1 us, 1 MB written; 16000 rows 5.6 us): a
// second launch for the rows alone, on all SMs, where max_rows is large, is what would shorten those.
#include "packed.cuh"

namespace {

constexpr int kPlanThreads = 1024;

struct PlanArgs {
    const int *len, *add, *drop;
    int B, bps, n_blocks, max_rows;
    int *table, *held, *free_blocks, *n_free;
    int *row_start;
    long long *slots;
    int *row_seq, *row_pos;
    int *status;
};

__device__ __forceinline__ void cluster_barrier()
{
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}

// Of n runs with ascending starts s[0] = 0 .. s[n], the one that x < s[n] falls into (empty ones are passed over): s[i] <= x < s[i + 1].
__device__ __forceinline__ int run_of(const long long *s, int n, long long x)
{
    int lo = 0, hi = n;                  // s[lo] <= x < s[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kPlanThreads, 1)
block_plan_kernel(const PlanArgs a)
{
    __shared__ long long s_row[FSPAD_PLAN_MAX_BATCH + 1], s_take[FSPAD_PLAN_MAX_BATCH + 1], s_back[FSPAD_PLAN_MAX_BATCH + 1];
    __shared__ int s_len[FSPAD_PLAN_MAX_BATCH], s_have[FSPAD_PLAN_MAX_BATCH];
    __shared__ long long s_warp[3][32];
    __shared__ int s_bad;
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int cta = blockIdx.x, n_cta = gridDim.x;
    if (tid == 0) s_bad = 0;
    // ---- every CTA: what each sequence gives back, takes and adds, as exclusive sums ----
    int L = 0, have = 0;
    long long val[3] = {0, 0, 0};        // rows, blocks taken, blocks given back
    bool bad = false;
    if (tid < a.B) {
        L = a.len[tid];
        const int A = a.add[tid], h = a.held[tid];
        const bool gone = a.drop != nullptr && a.drop[tid] != 0;
        bad = L < 0 || A < 0 || h < 0 || h > a.bps || (long long)L + A > (long long)a.bps * 128;
        if (!bad) {
            have = gone ? 0 : h;
            const int need = (int)(((long long)L + A + 127) >> 7);
            val[0] = A;
            val[1] = need > have ? need - have : 0;
            val[2] = gone ? h : 0;
        }
        s_len[tid] = L;
        s_have[tid] = have;
    }
    const int free0 = *a.n_free;
    long long inc[3];
#pragma unroll
    for (int x = 0; x < 3; ++x) {
        inc[x] = val[x];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long o = __shfl_up_sync(0xffffffffu, inc[x], off);
            if (lane >= off) inc[x] += o;
        }
        if (lane == 31) s_warp[x][warp] = inc[x];
    }
    __syncthreads();
    if (bad) s_bad = 1;
    if (warp < 3) {
        long long w = s_warp[warp][lane];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long o = __shfl_up_sync(0xffffffffu, w, off);
            if (lane >= off) w += o;
        }
        s_warp[warp][lane] = w;
    }
    __syncthreads();
    long long total[3];
#pragma unroll
    for (int x = 0; x < 3; ++x) {
        total[x] = s_warp[x][31];
        inc[x] += warp > 0 ? s_warp[x][warp - 1] : 0;
    }
    if (tid < a.B) {
        if (tid == 0) s_row[0] = s_take[0] = s_back[0] = 0;
        s_row[tid + 1] = inc[0];
        s_take[tid + 1] = inc[1];
        s_back[tid + 1] = inc[2];
    }
    const bool fits = s_bad == 0 && free0 >= 0 && free0 + total[2] <= a.n_blocks && total[1] <= free0 + total[2] && total[0] <= a.max_rows;
    __syncthreads();
    const int step = n_cta * kPlanThreads, first = cta * kPlanThreads + tid;
    if (!fits) {                         // the same answer in every CTA: nothing is changed, no row has a slot
        if (first == 0) fspad_report(a.status, FSPAD_ERR_RANGE);
        for (int b = first; b <= a.B; b += step) a.row_start[b] = 0;
        for (long long r = first; r < a.max_rows; r += step) {
            a.slots[r] = -1;
            if (a.row_seq) a.row_seq[r] = -1;
            if (a.row_pos) a.row_pos[r] = -1;
        }
        return;
    }
    // ---- dropped sequences' blocks onto the stack ----
    for (long long x = first; x < total[2]; x += step) {
        const int b = run_of(s_back, a.B, x);
        a.free_blocks[free0 + x] = a.table[(size_t)b * a.bps + (x - s_back[b])];
    }
    cluster_barrier();                   // (and nobody reads the old state any more)
    // ---- new blocks from the top of it ----
    const long long top = free0 + total[2] - 1;
    for (long long x = first; x < total[1]; x += step) {
        const int b = run_of(s_take, a.B, x);
        a.table[(size_t)b * a.bps + s_have[b] + (x - s_take[b])] = __ldcg(a.free_blocks + (top - x));
    }
    if (cta == 0) {
        if (tid < a.B) {
            a.held[tid] = have + (int)val[1];
            a.row_start[tid + 1] = (int)inc[0];
        }
        if (tid == 0) {
            a.row_start[0] = 0;
            *a.n_free = (int)(free0 + total[2] - total[1]);
        }
    }
    cluster_barrier();
    // ---- the rows: a warp looks for the run of its first one, 32 starts at a time, and most of its others are in it, too (each looking for itself took 200
    // instructions a row: 12.5 us for 200 requests of up to 600 rows) ----
    const unsigned n_row = (unsigned)total[0], most = (unsigned)a.max_rows;      // (the first at most the second)
    for (unsigned r0 = (unsigned)(first - lane); r0 < most; r0 += (unsigned)step) {
        const unsigned r = r0 + lane;
        long long slot = -1;
        int b = -1, p = -1;
        if (r0 < n_row) {
            int at = 32 * (__popc(__ballot_sync(0xffffffffu, 32 * lane < a.B && s_row[min(32 * lane, a.B)] <= r0)) - 1);
            at += __popc(__ballot_sync(0xffffffffu, at + lane < a.B && s_row[min(at + lane, a.B)] <= r0)) - 1;
            if (r < n_row) {
                b = r < s_row[at + 1] ? at : run_of(s_row, a.B, r);
                p = s_len[b] + (int)((long long)r - s_row[b]);
                slot = (long long)__ldcg(a.table + (size_t)b * a.bps + (p >> 7)) * 128 + (p & 127);
            }
        }
        if (r >= most) continue;
        a.slots[r] = slot;
        if (a.row_seq) a.row_seq[r] = b;
        if (a.row_pos) a.row_pos[r] = p;
    }
}

}  // namespace

cudaError_t fspad_launch_block_plan(fspad_ctx *ctx, const int *len, const int *add, const int *drop, int B, int bps, int n_blocks,
                                    int *table, int *held, int *free_blocks, int *n_free, int max_rows, int *row_start,
                                    long long *slots, int *row_seq, int *row_pos, cudaStream_t st)
{
    PlanArgs a;
    a.len = len; a.add = add; a.drop = drop; a.B = B; a.bps = bps; a.n_blocks = n_blocks; a.max_rows = max_rows;
    a.table = table; a.held = held; a.free_blocks = free_blocks; a.n_free = n_free; a.row_start = row_start; a.slots = slots;
    a.row_seq = row_seq; a.row_pos = row_pos; a.status = ctx->d_status;
    const unsigned ctas = 8u;            // (of one CTA a plan for 2048 rows took 5.7 us, of eight 5.0; for 256 rows both 5.1)
    ctx->launches++;
    return fspad_launch(block_plan_kernel, dim3(ctas), dim3(kPlanThreads), 0, st, ctas, a);
}
