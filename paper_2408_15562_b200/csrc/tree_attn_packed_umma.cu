// Attention over the cache held in 4 bits for many query rows a kv head (a tree's verification), on the 5th-generation tensor cores.  (What is
// computed, and the kernel for few rows: tree_attn_packed.cu; the list of work and its cutting: packed_list.cuh.)
//
// A CTA takes 256 query rows of a kv head and chunks of 128 keys.  Its sixteen warps have four jobs and meet only on mbarriers:
//   warps 0-7   softmax, in two groups of 128 threads, a query row a thread
//   warp 8      copies: codes and scales of the chunks into a ring of stages, by bulk copies
//   warp 9      tensor cores: one lane issues every product; the warp owns the tensor memory
//   warps 12-15 codes -> fp16 values (code * scale, exact), into K and V tiles as the tensor cores read them (two of each); the tree's bf16 rows too
// Per chunk and group: S = Q K^T (128 x 128 x 128) into tensor memory, weights in registers, P back over the scores, O += P V with P read from tensor
// memory.  With more than 128 rows group g has rows 128 g .. and every chunk; with fewer both have the same rows and take the
// chunks in turn, each with an accumulator of its own, and are merged at the end.  Either way the groups' products alternate: while one
// group is at its exponentials the tensor cores work for the other.
//
// Queries are fp16 too, each row scaled by a power of two (exact for elements of at least 2^-31 of the row's largest); but against the tree's rows, which are
// bf16 of any size, they are taken as they are: the tree's chunks come first, with bf16 operands (one product's operands have one type), and the query tile is then written
// again.  With one row tile its two forms lie in the two tiles' places.
//
// What bounds it: with two row tiles a chunk takes 4450 cycles, in which the products take 2900 (128 x 128 x 16 with both operands in shared memory 108 cycles, with
// one in tensor memory 75) and each group goes through a chain: exponentials 2050, its product with V 600, the next scores 860, the handing over between
// the warps the rest.  One tree of 60 nodes, 64 heads over 8, over 32700 keys: 87.7 us (64 GFLOP, 730 TFLOP/s).  With one row tile the codes' warps are the
// slowest, 3150 cycles a chunk.  What a stretch takes besides (queries, the tree's rows in bf16, the rows' way out, code that is fetched cold: 15000 to 20000 cycles) bounds
// short runs: 16 trees of 60 nodes, 32 heads over 8, 512 to 4096 keys 87.7 us, with the merge (16 by itself, from a cold cache).  Not kept: weights handed over in halves (91.4 us for the first of
// these), the products told of behind the next scores (one row tile 10 % longer).
//
// Every wait is bounded; on expiry the CTA records FSPAD_ERR_TIMEOUT, lets what is under way land and frees its tensor memory.
#include "packed_list.cuh"

namespace {

using namespace packed;
using namespace umma;

constexpr int UNIT = 128;                // keys of a chunk
constexpr int BM = 256;                  // query rows of a CTA: two tiles
constexpr int NT = 512;
constexpr int HALF = 128 * 128;          // bytes of one [128 rows][64 elements] half tile (128-byte swizzle)
constexpr int TILE = 2 * HALF;
constexpr int KCODES = UNIT * FSPAD_PACKED_CODE_BYTES, KSCALES = UNIT * FSPAD_PACKED_SCALE_BYTES;
constexpr int STAGE = KCODES + KSCALES;  // one plane of a chunk
constexpr int STAGES = 3;
constexpr int SMEM = 6 * TILE + STAGES * STAGE + 1024;      // Q[2] | K[2] | V[2] | stages, and alignment slack
constexpr uint32_t TMEM_COLS = 512;      // S, then P, of group g: columns 128 g ..; O of group g: 256 + 128 g ..
constexpr uint32_t IDESC = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);      // 128 x 128, fp32 accumulator, fp16 operands
constexpr uint32_t IDESC_BF = (1u << 7) | (1u << 10), IDESC_MN = 1u << 16;             // bf16 operands; B (= V) MN-major

// byte offset of 16-byte piece c (0..15) of row r of a tile
__device__ __forceinline__ uint32_t tile_off(int r, int c) { return (uint32_t)((c >> 3) * HALF + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }
__device__ __forceinline__ void st_shared(uint32_t at, uint4 v) { st_shared16(at, v.x, v.y, v.z, v.w); }

// A stretch of a run that a CTA takes.
struct Segment {
    int b, h, row0, rows, L;             // sequence, kv head, first query row of the tile and how many, keys in the cache
    int u0, n_ch, n_tree, n_run;         // first chunk, chunks, how many of them the tree's (they come first), chunks of the run
    bool two;                            // two row tiles
};

// 16 columns of a row of an accumulator times alpha.
__device__ __forceinline__ void tmem_scale16(uint32_t at, float alpha)
{
    uint32_t r[16];
    __syncwarp();
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;\n"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
#pragma unroll
    for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * alpha);
    tmem_st16(at, r);
}

// One group's turn at a chunk: scores -> weights.  All 128 scores of a row are in registers after one trip to tensor memory (every further
// wait for it costs 250 cycles: by quarters, read twice, a turn took 2650); the weights, packed in pairs, go to columns 64 .. 127, over scores.
__device__ __forceinline__ void softmax_chunk(bool tree, uint32_t tS, uint32_t tO, const uint32_t (&see)[4], bool masked, float cs, bool row_ok, bool first,
                                              float &m_run, float &l_run)
{
    uint32_t r[4][32];
    __syncwarp();
#pragma unroll
    for (int x = 0; x < 4; ++x) tmem_ld32_issue(tS + 32u * x, r[x]);
    tmem_ld_wait(r[0]);
    tmem_ld_pin(r[1]);
    tmem_ld_pin(r[2]);
    tmem_ld_pin(r[3]);
    if (masked) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (!((see[x] >> j) & 1u)) r[x][j] = 0xff800000u;
    }
    float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < 32; j += 2)
#pragma unroll
        for (int x = 0; x < 4; ++x) mx4[x] = fmaxf(fmaxf(mx4[x], __uint_as_float(r[x][j])), __uint_as_float(r[x][j + 1]));
    const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * cs;
    // the reference follows the row's maximum when some row of the warp would see a weight too large otherwise (a warp moves as one:
    // its accesses to tensor memory are collective); a row that does not exist has no say
    const float m_cand = fmaxf(m_run, mx);
    const bool move = !__all_sync(0xffffffffu, !row_ok || m_cand - m_run <= kLazyLog2);
    const float m_new = move ? m_cand : m_run;
    const float m_safe = m_new == -INFINITY ? 0.f : m_new;
    if (move) {
        const float alpha = ex2f(m_run - m_safe);
        l_run *= alpha;
        if (!first) {                    // the group's products so far are complete: the scores that were waited for come behind them
#pragma unroll 1
            for (int blk = 0; blk < 8; ++blk) tmem_scale16(tO + (uint32_t)blk * 16u, alpha);
        }
    }
    m_run = m_new;
    const float shift = (tree ? -kLazyLog2 : kBiasLog2) - m_safe;        // (of the tree's keys times kDown)
    const uint64_t scale2 = f32x2(cs, cs), neg = f32x2(shift, shift);
    uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float x0, x1;
            f32x2_split(f32x2_fma(f32x2(__uint_as_float(r[x][2 * e]), __uint_as_float(r[x][2 * e + 1])), scale2, neg), x0, x1);
            const float p0 = ex2f(x0), p1 = ex2f(x1);
            acc[e & 3] = f32x2_add(acc[e & 3], f32x2(p0, p1));
            if (tree) w[e] = pack_bf16(p0, p1);
            else w[e] = pack_f16(p0, p1);
        }
        tmem_st16(tS + 64u + 16u * x, w);
    }
    float lo, hi;
    f32x2_split(f32x2_add(f32x2_add(acc[0], acc[1]), f32x2_add(acc[2], acc[3])), lo, hi);
    l_run += (lo + hi) * (tree ? kUp : 1.f);
}

__global__ void __launch_bounds__(NT, 1)
tree_attn_packed_umma_kernel(const Args a)
{
    extern __shared__ unsigned char smem_raw[];
    enum { ST_FULL = 0, ST_FREE = STAGES, K_FULL = 2 * STAGES, K_FREE = K_FULL + 2, V_FULL = K_FREE + 2, V_FREE = V_FULL + 2, S_FULL = V_FREE + 2,
           P_FULL = S_FULL + 2, O_DONE = P_FULL + 2, Q_FULL = O_DONE + 4, DRAIN = Q_FULL + 2, N_BAR };
    __shared__ __align__(8) unsigned long long s_bar[N_BAR];
    __shared__ int s_scan[NT / 32 + 2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_fail, s_soft_fail;              // (the second: written and read by the softmax warps alone, around their barriers)
    __shared__ short s_par[FSPAD_MAX_NODES_WIDE];
    __shared__ uint32_t s_odd[2][4];                 // which V rows of a tree's chunk have an infinity or a NaN in them
    __shared__ float2 s_ml[2][128];
    __shared__ int s_to[2][128];                     // where a staged row goes

    const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp();
    const uint32_t bar0 = smem_u32(&s_bar[0]);
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
    if (tid == 0) {
        for (int i = 0; i < N_BAR; ++i) {
            int count = 1;
            if ((i >= ST_FREE && i < K_FULL) || (i >= K_FULL && i < K_FREE) || (i >= V_FULL && i < V_FREE) || (i >= P_FULL && i < O_DONE) ||
                (i >= Q_FULL && i < DRAIN))
                count = 4;                           // the four warps of a group, or of the dequantising ones
            mbar_init(bar(i), count);
        }
        s_fail = s_soft_fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 9) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" :: "r"(smem_u32(&s_tmem)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    fspad_pdl_trigger();
    fspad_pdl_wait();
    tc_fence_before();
    const int cta = blockIdx.x;
    Parts parts;
    Part part = cut_list<NT, UNIT, 1>(a, cta, gridDim.x, parts, s_scan, cta == 0);      // (with a barrier in it)
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    const int nt = tree_units<UNIT>(a), runs = a.Hkv * a.mtiles;

    if (warp == 11 && lane == 0) tell_part<UNIT>(a, parts, part, cta);       // (a warp without another job)

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t sQ = base, sK = base + 2 * TILE, sV = base + 4 * TILE, sStage = base + 6 * TILE;

    // Every warp goes through the CTA's stretches by itself.
    auto next = [&](Segment &s) -> bool {
        if (part.left <= 0) return false;
        s.b = part.b;
        s.L = prefix_of(a, part.b, false);
        s.n_run = run_units<UNIT>(a, s.L);
        s.u0 = part.u;
        s.n_ch = min(s.n_run - s.u0, part.left);
        s.n_tree = max(0, min(nt - s.u0, s.n_ch));
        s.h = a.by_tiles.of(part.run);
        s.row0 = (part.run - s.h * a.mtiles) * BM;
        s.rows = min(BM, a.M - s.row0);
        s.two = s.rows > 128;
        part.left -= s.n_ch;
        part.u = 0;
        if (++part.run == runs) { part.run = 0; ++part.b; }
        return true;
    };
    bool failed = false;
    Segment s;

    if (warp < 8) {
        // ================= softmax =================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");    // 2 x 176 + 64 + 96 a lane of each warpgroup: the launch's 4 x 128
        const int grp = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lanes + 128u * grp, tO = tmem + lanes + 256u + 128u * grp;
        uint32_t ph_s = 0, n_done = 0, tree_chunks = 0;      // phase of S_FULL; products of the group so far; tree chunks of the CTA so far
        while (next(s)) {
            const int gr = s.row0 + (s.two ? grp * 128 : 0) + row;           // row of the kv head
            const bool row_ok = gr < a.M;
            const bool live = s.row0 + (s.two ? grp * 128 : 0) + (warp & 3) * 32 < a.M;
            const int node = row_ok ? a.by_G.of(gr) : -1, head = s.h * a.G + gr - node * a.G;        // (the head of a row that exists)
            float cs = 0.f;
            // The group's rows of queries into tile t, half a warp a row (a thread taking its own row met 32 lines an instruction); code that runs once
            // a stretch is kept short, for it is fetched cold: unrolled it took 12000 cycles.
            auto fetch_q = [&](int t) {
                const uint32_t to = sQ + (uint32_t)t * TILE;
                const long long mine = row_ok ? (((long long)s.b * a.N + node) * a.Hq + head) * D : -1;
                const int piece = lane & 15, r0 = (warp & 3) * 32;
#pragma unroll 2
                for (int k = 0; k < 16; ++k) {
                    const int r = 2 * k + (lane >> 4);
                    const long long at = __shfl_sync(0xffffffffu, mine, r);
                    cp_async16(to + tile_off(r0 + r, piece), a.q + (at < 0 ? 0 : at) + piece * 8, at >= 0);
                }
                cp_async_commit();
                cp_async_wait<0>();
                __syncwarp();
            };
            // The rows of tile t as fp16, each with its largest magnitude in [2^14, 2^15) (change: false for the factors alone, which stay with the rows' threads).
            auto scale_q = [&](int t, bool change) {
                const uint32_t to = sQ + (uint32_t)t * TILE;
                const int piece = lane & 15, r0 = (warp & 3) * 32;
#pragma unroll 1
                for (int k0 = 0; k0 < 16; k0 += 4) {
                    uint4 w[4];                              // (all of them under way before the first is used)
#pragma unroll
                    for (int y = 0; y < 4; ++y) w[y] = ld_shared16(to + tile_off(r0 + 2 * (k0 + y) + (lane >> 4), piece));
                    uint32_t m[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) m[y] = fspad_most2(fspad_most2(w[y].x, w[y].y), fspad_most2(w[y].z, w[y].w));
#pragma unroll
                    for (int off = 8; off > 0; off >>= 1)
#pragma unroll
                        for (int y = 0; y < 4; ++y) m[y] = fspad_most2(m[y], __shfl_xor_sync(0xffffffffu, m[y], off));
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const uint32_t top = max(m[y] & 0xffffu, m[y] >> 16);
                        const int e = top == 0u || top >= 0x7f80u ? 14 : max((int)(top >> 7) - 127, -100);
                        const int mine = __shfl_sync(0xffffffffu, e, (lane & 1) * 16);       // of row 2 (k0 + y) + (lane & 1)
                        if (lane >> 1 == k0 + y) cs = a.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + mine) << 23);
                        const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
                        auto half2 = [&](uint32_t x) { return pack_f16(__uint_as_float(x << 16) * up, __uint_as_float(x & 0xffff0000u) * up); };
                        w[y] = make_uint4(half2(w[y].x), half2(w[y].y), half2(w[y].z), half2(w[y].w));
                    }
                    if (change)
#pragma unroll
                        for (int y = 0; y < 4; ++y) st_shared(to + tile_off(r0 + 2 * (k0 + y) + (lane >> 4), piece), w[y]);
                }
            };
            auto tell_q = [&](int t) {
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(Q_FULL + t));
            };
            // one row tile: group 0's as it is, for the tree, group 1's as fp16; two: fp16, or first as they are for the tree
            fetch_q(grp);
            const bool raw = s.two ? s.n_tree > 0 : grp == 0;
            if (!raw) scale_q(grp, true);
            tell_q(grp);
            // (group 0's own chunks of the cache, if there are any, need the factors all the same)
            if (raw && !s.two && s.n_ch > s.n_tree + (s.n_tree & 1)) scale_q(grp, false);
            if (s.n_tree > 0) {
                for (int i = tid; i < a.N; i += 256) {
                    int p = a.parent[(size_t)s.b * a.N + i];
                    if (i == 0 ? p != -1 : (p < 0 || p >= i)) { fspad_report(a.status, FSPAD_ERR_BAD_TREE); p = -1; }
                    s_par[i] = (short)p;
                }
                asm volatile("bar.sync 1, 256;\n" ::: "memory");
            }
            float m_run = -INFINITY, l_run = 0.f;
            const int n_items = s.two ? 2 * s.n_ch : s.n_ch;
            bool first = true;
            for (int i = grp; i < n_items; i += 2) {
                const int c = s.two ? i >> 1 : i, u = s.u0 + c;
                const bool tree = c < s.n_tree;
                const int key0 = tree ? u * UNIT : (u - nt) * UNIT;
                const bool masked = tree || key0 + UNIT > s.L;
                uint32_t see[4] = {~0u, ~0u, ~0u, ~0u};
                if (tree) {
                    // from the node up, word by word, for an ancestor comes before its descendants (with two words of 64 bits a step took three times as long:
                    // 22 chains of 156 nodes, 32 heads, 186 us against 117; trees of ten nodes' depth 54 and 51)
                    int at = node;
                    while (at >= key0 + 128) at = s_par[at];
#pragma unroll
                    for (int x = 3; x >= 0; --x) {
                        see[x] = 0u;
                        while (at >= key0 + 32 * x) {
                            see[x] |= 1u << (at & 31);
                            at = s_par[at];
                        }
                    }
                } else if (masked) {
                    const int left = s.L - key0;             // 1 .. 127
#pragma unroll
                    for (int x = 0; x < 4; ++x) see[x] = left >= 32 * x + 32 ? ~0u : left > 32 * x ? (1u << (left - 32 * x)) - 1u : 0u;
                }
                if (!failed && !mbar_wait(bar(S_FULL + grp), ph_s)) failed = true;
                ph_s ^= 1u;
                tc_fence_after();
                if (live) {
                    softmax_chunk(tree, tS, tO, see, masked, tree ? a.scale_log2 : cs, row_ok, first, m_run, l_run);
                    if (tree) {
                        const uint32_t *odd = s_odd[(tree_chunks + c) & 1];
                        if ((see[0] & odd[0]) | (see[1] & odd[1]) | (see[2] & odd[2]) | (see[3] & odd[3])) l_run = NAN;
                    }
                    asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
                }
                first = false;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_light(bar(P_FULL + grp));
                ++n_done;
                if (s.two && c == s.n_tree - 1 && s.n_ch > s.n_tree) {       // (the tile's last reader's scores are here)
                    scale_q(grp, true);
                    tell_q(grp);
                }
            }
            tree_chunks += s.n_tree;
            // ---- the group's last product, then the rows ----
            if (!first && !failed && !mbar_wait(bar(O_DONE + 2 * grp + (int)((n_done - 1) & 1u)), ((n_done - 1) >> 1) & 1u)) failed = true;
            tc_fence_after();
            const bool whole = s.n_ch == s.n_run;
            const int slot = cta * 2 + (s.u0 == 0 ? 1 : 0);
            s_to[grp][row] = !row_ok ? -1 : (s.b * a.N + node) * a.Hq + head;
            float f0 = 1.f, f1 = 0.f;                        // factors of the accumulators that make up the row: the group's own, or group 0's and group 1's
            float m_fin = m_run, l_fin = l_run;
            if (!s.two) {
                if (failed) s_soft_fail = s_fail = 1;
                s_ml[grp][row] = make_float2(m_run, l_run);
                tc_fence_before();
                asm volatile("bar.sync 1, 256;\n" ::: "memory");
                tc_fence_after();
                if (s_soft_fail != 0) failed = true;
                const float2 o = s_ml[grp ^ 1][row];
                m_fin = fmaxf(m_run, o.x);
                const float ref = m_fin == -INFINITY ? 0.f : m_fin;
                const float own = ex2f(m_run - ref), other = ex2f(o.x - ref);
                l_fin = (m_run == -INFINITY ? l_run : l_run * own) + (o.x == -INFINITY ? o.y : o.y * other);     // (without a maximum: zero, or a NaN)
                f0 = grp == 0 ? own : other;
                f1 = grp == 0 ? other : own;
            }
            __syncwarp();
            if (whole) {
                const float inv = kUp / l_fin;
                f0 *= inv;
                f1 *= inv;
            }
            if (!whole && row_ok && (s.two || grp == 0)) a.part_ml[(size_t)slot * BM + (gr - s.row0)] = make_float2(m_fin, l_fin);
            const bool both = !s.two && s.n_ch > 1;          // group 1 has had a chunk
            const uint32_t stage = sQ + (uint32_t)grp * TILE + (uint32_t)((warp & 3) * 8192);        // 8 KB a warp (the query tiles are read)
            if (live && !failed) {
#pragma unroll 1
                for (int x = s.two ? 0 : 2 * grp; x < (s.two ? 4 : 2 * grp + 2); ++x) {
                    // columns 32 x ..: a row's pieces of 16 bytes lie in an order that depends on the row, so that neither side's accesses collide
                    uint32_t r[32];
                    const uint32_t own = tmem + lanes + 256u + 32u * x + (s.two ? 128u * grp : 0u);
                    __syncwarp();
                    tmem_ld32_issue(own, r);
                    tmem_ld_wait(r);
#pragma unroll
                    for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * f0);
                    if (both) {
                        uint32_t r1[32];
                        __syncwarp();
                        tmem_ld32_issue(own + 128u, r1);
                        tmem_ld_wait(r1);
#pragma unroll
                        for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(fmaf(__uint_as_float(r1[j]), f1, __uint_as_float(r[j])));
                    }
                    auto val = [&](int j) { return __uint_as_float(r[j]); };
                    if (whole) {
                        // two quarters side by side, then whole pieces of 128 bytes: 4 rows at a time
#pragma unroll
                        for (int j = 0; j < 32; j += 8)
                            st_shared16(stage + (uint32_t)(lane * 128 + ((((x & 1) * 4 + j / 8) ^ (lane & 7)) << 4)), pack_bf16(val(j), val(j + 1)),
                                        pack_bf16(val(j + 2), val(j + 3)), pack_bf16(val(j + 4), val(j + 5)), pack_bf16(val(j + 6), val(j + 7)));
                        if (x & 1) {
                            __syncwarp();
#pragma unroll 2
                            for (int k = 0; k < 8; ++k) {
                                const int r4 = 4 * k + (lane >> 3), to = s_to[grp][(warp & 3) * 32 + r4];
                                if (to >= 0)
                                    reinterpret_cast<uint4 *>(a.out + (size_t)to * D + (x >> 1) * 64)[lane & 7] =
                                        ld_shared16(stage + (uint32_t)(r4 * 128 + (((lane & 7) ^ (r4 & 7)) << 4)));
                            }
                            __syncwarp();
                        }
                    } else {
                        // the warp's 32 rows as they lie, 4 KB in one copy, from one of two places in turn (rows that do not exist among them: nobody looks at those)
                        const uint32_t at = stage + (uint32_t)((x & 1) * 4096);
                        if (lane == 0) bulk_store_read_but_one();
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 32; j += 4) st_shared16(at + (uint32_t)(lane * 128 + (((j / 4) ^ (lane & 7)) << 4)), r[j], r[j + 1], r[j + 2], r[j + 3]);
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0)
                            bulk_store(a.part_o + (((size_t)slot * 2 + (s.two ? grp : 0)) * 4 + x) * (128 * 32) + (warp & 3) * (32 * 32), at, 4096);
                    }
                }
            }
            if (failed) s_fail = 1;
            // nobody goes on to the next stretch (whose queries, products, parents and exchange use the same places) before all have read
            if (part.left > 0) {
                if (lane == 0) bulk_store_read();
                tc_fence_before();
                asm volatile("bar.sync 1, 256;\n" ::: "memory");
                tc_fence_after();
            }
        }
        if (lane == 0) bulk_store_wait();                    // (the copies' memory is this CTA's)
    } else if (warp < 12) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
      if (warp == 8) {
        // ================= copies =================
        int n = 0, done = 0;                                 // stages filled, chunks taken so far
        for (;; done += s.n_ch) {
            const Part at = part;
            if (failed || !next(s)) break;
            if (s.u0 == 0 && lane == 0) tell_run(a, parts, at, cta, done, s.n_run);
            const int *blocks = a.table + (size_t)s.b * a.table_stride;
            const int kv0 = s.u0 + s.n_tree - nt, n_kv = s.n_ch - s.n_tree;  // chunks of the cache
            int mine = 0;
            for (int i = 0; i < n_kv && !failed; ++i) {
                if ((i & 31) == 0) {
                    if (i + lane < n_kv) {
                        mine = __ldg(blocks + kv0 + i + lane);
                        if (mine < 0 || mine >= a.n_blocks) { fspad_report(a.status, FSPAD_ERR_RANGE); mine = 0; }
                    }
                }
                const int blk = __shfl_sync(0xffffffffu, mine, i & 31);
                const size_t r0 = ((size_t)blk * a.Hkv + s.h) * 128;
                for (int plane = 0; plane < 2 && !failed; ++plane, ++n) {
                    const int st = n % STAGES;
                    if (n >= STAGES && !mbar_wait(bar(ST_FREE + st), (uint32_t)(n / STAGES - 1) & 1u)) { failed = true; break; }
                    if (lane == 0) {
                        const uint32_t to = sStage + (uint32_t)(st * STAGE), full = bar(ST_FULL + st);
                        mbar_expect_tx(full, STAGE);
                        bulk_load(to, (plane ? a.vc : a.kc) + r0 * FSPAD_PACKED_CODE_BYTES, KCODES, full);
                        bulk_load(to + KCODES, (plane ? a.vs : a.ks) + r0 * FSPAD_PACKED_SCALE_BYTES, KSCALES, full);
                    }
                    __syncwarp();
                }
            }
        }
        if (failed) s_fail = 1;
        // a CTA that gives up: what has been asked for gets a bounded time to land
        if (failed)
            for (int x = n > STAGES ? n - STAGES : 0; x < n; ++x) (void)mbar_wait(bar(ST_FULL + x % STAGES), (uint32_t)(x / STAGES) & 1u);
      } else if (warp == 9) {
        // ================= tensor cores =================
        // (A warp for each group kept the groups in step, both at their exponentials or both waiting for products: 5600 cycles a chunk against 4300.)
        const bool issuer = elect_one();
        const uint32_t hi = (uint32_t)(make_desc(0, 16) >> 32);
        const uint32_t q_lo = (uint32_t)make_desc(sQ, 16), k_lo = (uint32_t)make_desc(sK, 16), v_lo = (uint32_t)make_desc(sV, HALF);
        uint32_t cc = 0;                                     // chunks of the stretches before (slot: modulo 2)
        uint32_t ph_q[2] = {0u, 0u}, n_p[2] = {0u, 0u};      // phases of Q_FULL; products of each group so far
        while (!failed && next(s)) {
            // (through a shuffle they are values that the compiler knows to be the same in every lane, as an instruction's operands have to be)
            s.n_ch = __shfl_sync(0xffffffffu, s.n_ch, 0);
            s.n_tree = __shfl_sync(0xffffffffu, s.n_tree, 0);
            s.two = __shfl_sync(0xffffffffu, (int)s.two, 0) != 0;
            const int n_items = s.two ? 2 * s.n_ch : s.n_ch;
            auto wait_q = [&](int t) {
                if (!failed && !mbar_wait(bar(Q_FULL + t), ph_q[t])) failed = true;
                ph_q[t] ^= 1u;
            };
            bool have_q[2] = {false, false};                 // of one row tile: its two forms
            // item i: group i & 1, chunk i / 2 or, of one row tile, i
            auto issue_s = [&](int i) {
                const int g = i & 1, c = s.two ? i >> 1 : i;
                const bool tree = c < s.n_tree;
                if (s.two && c == s.n_tree && c > 0) wait_q(g);              // the tile again, as fp16
                const uint32_t at = cc + (uint32_t)c, slot = at & 1u;
                const int t = s.two ? g : tree ? 0 : 1;
                if (!s.two && !have_q[t]) {
                    wait_q(t);
                    have_q[t] = true;
                }
                if ((!s.two || g == 0) && !failed && !mbar_wait(bar(K_FULL + slot), (at >> 1) & 1u)) failed = true;
                if (!failed && issuer) {
                    tc_fence_after();
                    const uint32_t kb = k_lo + slot * (TILE >> 4), qb = q_lo + (uint32_t)t * (TILE >> 4), d = tmem + 128u * g;
                    const uint32_t idesc = IDESC | (tree ? IDESC_BF : 0u);
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        const uint32_t off = ((ks >> 2) * HALF + (ks & 3) * 32) >> 4;
                        mma_f16_ss(d, qb + off, kb + off, hi, idesc, ks > 0);
                    }
                    mma_commit(bar(S_FULL + g));
                    if (!s.two || g == 1) mma_commit(bar(K_FREE + slot));
                }
                __syncwarp();
            };
            if (s.two) wait_q(0);
#pragma unroll 1
            for (int i = -2; i < n_items; ++i) {
                if (i >= 0) {
                    const int g = i & 1, c = s.two ? i >> 1 : i;
                    const bool tree = c < s.n_tree;
                    const uint32_t at = cc + (uint32_t)c, slot = at & 1u;
                    // (a form that no chunk needs is written all the same; its phase is over before the stretch can be)
                    if (!s.two && i == n_items - 1) {
                        if (!have_q[0]) wait_q(0);
                        if (!have_q[1]) wait_q(1);
                    }
                    if ((!s.two || g == 0) && !failed && !mbar_wait(bar(V_FULL + slot), (at >> 1) & 1u)) failed = true;
                    if (!failed && !mbar_wait(bar(P_FULL + g), n_p[g] & 1u)) failed = true;
                    if (!failed && issuer) {
                        tc_fence_after();
                        const uint32_t vb = v_lo + slot * (TILE >> 4), idesc = IDESC | IDESC_MN | (tree ? IDESC_BF : 0u);
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)       // 16 keys an instruction: 8 columns of packed pairs
                            mma_f16_ts(tmem + 256u + 128u * g, tmem + 128u * g + 64u + (uint32_t)ks * 8u, vb + (uint32_t)(ks * 16 * 128 >> 4), hi,
                                       idesc, i > 1 || ks > 0);
                        mma_commit(bar(O_DONE + 2 * g + (int)(n_p[g] & 1u)));
                        if (!s.two || g == 1) mma_commit(bar(V_FREE + slot));
                    }
                    __syncwarp();
                    ++n_p[g];
                }
                if (i == -1 && s.two) wait_q(1);
                if (i + 2 < n_items) issue_s(i + 2);         // (products complete in order: the scores may replace P)
            }
            cc += (uint32_t)s.n_ch;
        }
        if (failed) {
            s_fail = 1;
            if (lane == 0) mma_commit(bar(DRAIN));
            (void)mbar_wait(bar(DRAIN), 0u);
        }
      }
    } else {
        // ================= values =================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
        const int w4 = warp - 12;
        uint32_t n = 0, cc = 0, tree_chunks = 0;             // stages read, chunks filled, the tree's chunks so far
        while (!failed && next(s)) {
            for (int c = 0; c < s.n_ch && !failed; ++c, ++cc) {
                const uint32_t slot = cc & 1u;
                const int u = s.u0 + c;
                if (c < s.n_tree) {
                    // a chunk of the tree: V before K, so that whoever sees its scores sees which of its V rows are odd
                    const int key0 = u * UNIT;
                    uint32_t *odd = s_odd[tree_chunks & 1];
                    ++tree_chunks;
                    const int piece = lane & 15, rows = min(a.N - key0, UNIT);
                    const size_t first = (((size_t)s.b * a.Hkv + s.h) * a.N + key0) * D + piece * 8;
                    if (cc >= 2 && !mbar_wait(bar(V_FREE + slot), ((cc >> 1) - 1u) & 1u)) { failed = true; break; }
                    if (cc >= 2 && !mbar_wait(bar(K_FREE + slot), ((cc >> 1) - 1u) & 1u)) { failed = true; break; }
                    if (lane == 0) odd[w4] = 0u;             // (a warp's 32 rows are a word)
#pragma unroll 4
                    for (int r = w4 * 32 + (lane >> 4); r < w4 * 32 + 32; r += 2) {
                        const size_t at = r < rows ? first + (size_t)r * D : 0;
                        cp_async16(sV + slot * TILE + tile_off(r, piece), a.tv + at, r < rows);
                        cp_async16(sK + slot * TILE + tile_off(r, piece), a.tk + at, r < rows);
                    }
                    cp_async_commit();
                    cp_async_wait<0>();
                    __syncwarp();                            // (the word is zero)
#pragma unroll 1
                    for (int r8 = 0; r8 < 32; r8 += 16) {    // V, as this lane has copied it
                        uint4 x[8];
#pragma unroll
                        for (int y = 0; y < 8; ++y) x[y] = ld_shared16(sV + slot * TILE + tile_off(w4 * 32 + r8 + 2 * y + (lane >> 4), piece));
#pragma unroll
                        for (int y = 0; y < 8; ++y)
                            if (odd_value(x[y].x) || odd_value(x[y].y) || odd_value(x[y].z) || odd_value(x[y].w)) {
                                const int r = r8 + 2 * y + (lane >> 4);
                                atomicOr(&odd[w4], 1u << r);         // out of the product: see softmax
                                st_shared(sV + slot * TILE + tile_off(w4 * 32 + r, piece), make_uint4(0u, 0u, 0u, 0u));
                            }
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(bar(V_FULL + slot));
                        mbar_arrive(bar(K_FULL + slot));
                    }
                } else {
                    const int left = s.L - (u - nt) * UNIT;  // keys of the chunk that exist
#pragma unroll 1
                    for (int plane = 0; plane < 2; ++plane, ++n) {
                        const uint32_t st = n % STAGES;
                        if (cc >= 2 && !mbar_wait(bar((plane ? V_FREE : K_FREE) + slot), ((cc >> 1) - 1u) & 1u)) { failed = true; break; }
                        if (!mbar_wait(bar(ST_FULL + st), (n / STAGES) & 1u)) { failed = true; break; }
                        const uint32_t from = sStage + st * STAGE, to = (plane ? sV : sK) + slot * TILE, down = plane ? kDown2 : kOne2;
                        // a lane takes a block of 16: blocks 4 x + (lane & 3) of eight rows at a time, so that the stores do not collide
                        uint32_t w0[8], w1[8], sc[8];        // (all of them under way before the first is used)
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int r = w4 * 32 + (k >> 1) * 8 + (lane >> 2), blk = 4 * (k & 1) + (lane & 3);
                            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];\n" : "=r"(w0[k]), "=r"(w1[k]) : "r"(from + (uint32_t)(r * 64 + blk * 8)));
                            asm volatile("ld.shared.u8 %0, [%1];\n" : "=r"(sc[k]) : "r"(from + KCODES + (uint32_t)(r * 8 + blk)));
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int r = w4 * 32 + (k >> 1) * 8 + (lane >> 2), blk = 4 * (k & 1) + (lane & 3);
                            if (r >= left) sc[k] = 0u;       // what lies behind the end may be anything: zeros
                            const uint32_t s2 = fspad_hmul2(fspad_e4m3_to_f16(sc[k] * 0x101u), down);
                            uint32_t f0[4], f1[4];
                            fspad_e2m1_to_f16(w0[k], f0);
                            fspad_e2m1_to_f16(w1[k], f1);
#pragma unroll
                            for (int j = 0; j < 4; ++j) { f0[j] = fspad_hmul2(f0[j], s2); f1[j] = fspad_hmul2(f1[j], s2); }
                            st_shared16(to + tile_off(r, 2 * blk), f0[0], f0[1], f0[2], f0[3]);
                            st_shared16(to + tile_off(r, 2 * blk + 1), f1[0], f1[1], f1[2], f1[3]);
                        }
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(bar(ST_FREE + st));
                            mbar_arrive(bar((plane ? V_FULL : K_FULL) + slot));
                        }
                    }
                }
            }
        }
        if (failed) s_fail = 1;
    }
    // ---- everybody has done: the tensor memory goes back ----
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (tid == 0 && s_fail != 0) fspad_report(a.status, FSPAD_ERR_TIMEOUT);
    if (warp == 9) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" :: "r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

}  // namespace

size_t fspad_attn_packed_umma_workspace(const fspad_ctx *ctx)
{
    return scratch_bytes<BM>(ctx->sm_count);
}

cudaError_t fspad_launch_attn_packed_umma(fspad_ctx *ctx, packed::Args a, void *workspace, cudaStream_t st)
{
    const int ctas = ctx->sm_count;
    a.mtiles = (a.M + BM - 1) / BM;
    a.by_tiles.set((unsigned)a.mtiles);
    scratch_in<BM>(a, ctas, workspace);
    cudaError_t e = raise_shared(ctx, 0, reinterpret_cast<const void *>(&tree_attn_packed_umma_kernel), SMEM);
    if (e != cudaSuccess) return e;
    const int entries = merge_entries(a, ctas);
    ctx->launches++;
    e = fspad_launch(tree_attn_packed_umma_kernel, dim3((unsigned)ctas), dim3(NT), SMEM, st, 0, a);
    return e == cudaSuccess ? launch_merge<BM>(ctx, a, entries, ctas, st) : e;
}
