// Attention over the cache held in 8 bits for many query rows a kv head (a tree's verification), on the 5th-generation tensor cores.  (What is computed, and
// the kernel for few rows: tree_attn_fp8.cu; the list of work and its cutting: packed_list.cuh.)
//
// A CTA takes 256 query rows of a kv head and chunks of 128 keys.  Its sixteen warps have five jobs and meet only on mbarriers:
//   warps 0-7   softmax, in two groups of 128 threads, a query row a thread
//   warp 8      copies: K and V codes of a chunk into one of three buffers, K's by TMA as the tensor cores read them, V's as they lie
//   warps 9, 11 tensor cores: a warp for each group, one lane of which issues its products; warp 9 owns the tensor memory
//   warp 10     scales of a chunk, as the softmax takes them
//   warps 12-15 V codes -> fp16 values, into V tiles as the tensor cores read them (two of them); the tree's bf16 rows too
// Per chunk and group, 64 keys at a time: S = Q K^T (128 x 64 x 128) into tensor memory, weights in registers, P back over the scores, O += P V with P read from tensor
// memory; while one half of a chunk is at its exponentials, the products around the other go on.  With more than 128 rows group g has rows 128 g .. and every chunk; with fewer both have the
// same rows and take the chunks in turn, each with an accumulator of its own, and are merged at the end.
//
// K is never touched outside the tensor cores: its e4m3 codes are an operand as they are, and a query is the sum of two e4m3 numbers, the nearest one and what is
// left, which is exact for elements of at least 2^-9 of the row's largest (a bf16 number has 8 significant bits, the two have 4 each, whole multiples of 2^-9 where the largest lies in
// [2^7, 2^8)); smaller ones are off by at most 2^-17 of the largest.  32 keys' scale is a factor of 32 columns of the scores.  V's scale goes into the weights, as an addend of the
// exponent: the reference that a row's weights are relative to follows the maximum of score + log2(scale), and the sum of the weights takes each
// group's part times 1 / scale.  Against the tree's rows, which are bf16 of any size, the queries are taken as they are: its chunks come first, and the query
// tile is then written again.  With one row tile its two forms lie in the two tiles' places.
//
// Measured, captured in a graph: 16 trees of 60 nodes, 32 heads over 8, 512 to 4096 keys 73.7 us (75 called one after another; floor 21.5: 36 GFLOP at the measured bf16 rate); one tree of 60 over 32700
// keys with 64 heads over 8 86.4 us (91; 38.5).  A chunk of 256 rows costs some 4900 cycles, of which the products take 2560 (scores of 64 keys: 32 instructions of 48 cycles; the others 16 of 64) and the
// exponentials, on their unit, 2100: each is a third busy over a call, and what bounds it is the chain of a half chunk, wait, load, maximum, vote, exponentials, store, with two warps a scheduler.  Not kept,
// on these two: scores of halves ahead from one issuing warp 110 and 110, whole chunks with a warp a group 97 and 103, those with the groups' exponentials in turn 92 and 92, beginnings of
// runs not counted in the cut 94.5 and 86.
//
// Every wait is bounded; on expiry the CTA records FSPAD_ERR_TIMEOUT, lets what is under way land and frees its tensor memory.
#include "fp8.cuh"
#include "packed_list.cuh"

#include <type_traits>

namespace {

using namespace packed;
using namespace umma;

constexpr int UNIT = 128;                // keys of a chunk
constexpr int BM = 256;                  // query rows of a CTA: two tiles
constexpr int NT = 512;
constexpr int HALF = 128 * 128;          // bytes of one [128 rows][64 elements] half tile (128-byte swizzle)
constexpr int TILE = 2 * HALF;
constexpr int BUFS = 3;                  // K codes | V codes of a chunk; of the tree's chunks the K tile
constexpr int SMEM = (4 + BUFS) * TILE;  // Q[2] | buffers | V[2]
constexpr uint32_t TMEM_COLS = 512;      // S, then P, of group g: columns 128 g ..; O of group g: 256 + 128 g ..
constexpr uint32_t IDESC = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);      // 128 x 128, fp32 accumulator, fp16 operands (kind::f8f6f4: e4m3 ones)
constexpr uint32_t IDESC64 = (1u << 4) | ((64u >> 3) << 17) | ((128u >> 4) << 24);       // 128 x 64
constexpr uint32_t IDESC_BF = (1u << 7) | (1u << 10), IDESC_MN = 1u << 16;             // bf16 operands; B (= V) MN-major

// byte offset of 16-byte piece c (0..15) of row r of a tile
__device__ __forceinline__ uint32_t tile_off(int r, int c) { return (uint32_t)((c >> 3) * HALF + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }
__device__ __forceinline__ void st_shared(uint32_t at, uint4 v) { st_shared16(at, v.x, v.y, v.z, v.w); }

// Products issued by the one lane whose `e` is not 0, while the whole warp goes through the loop, so that descriptors and addresses are values that are the same in
// every lane: in a branch of one lane a product took 100 cycles to issue, which bounded the kernel.
// D[tmem] (+)= A[smem] * B[smem], e4m3 operands, 32 elements deep
__device__ __forceinline__ void mma_f8_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate, uint32_t e)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
                 "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, p;\n\t}\n"
                 :: "r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(e) : "memory");
}
// the same with A from tensor memory, 16-bit operands
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate, uint32_t e)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
                 "mov.b64 db, {%2, %3};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}\n"
                 :: "r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(e) : "memory");
}

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

// A query's factor times 32 keys' scale; not less than the least normal number (masked scores are -infinity, and must stay it), and no infinity (scores of 0 must stay that).
__device__ __forceinline__ float factor(float cs, float scale)
{
    return fminf(fmaxf(cs * scale, 0x1p-126f), kMost);
}

// One group's turn at half a chunk: 64 scores of a row -> weights, over the scores' first 32 columns, packed in pairs.
// `of_keys`: of each 32 keys of the chunk the scale of K, log2 of V's scale, and its reciprocal (four of each); the tree's have none.  `wait_o`: until the group's product before the last
// one (which the scores are known to come behind) is complete too.
template <bool plain, typename F>
__device__ __forceinline__ void softmax_half(bool tree, uint32_t tS, uint32_t tO, const uint32_t (&see)[2], float cs, const float *of_keys, bool row_ok, bool first,
                                             float &m_run, float &l_run, F wait_o)
{
    uint32_t r[2][32];
    __syncwarp();
#pragma unroll
    for (int x = 0; x < 2; ++x) tmem_ld32_issue(tS + 32u * x, r[x]);
    tmem_ld_wait(r[0]);
    tmem_ld_pin(r[1]);
    if (!plain) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (!((see[x] >> j) & 1u)) r[x][j] = 0xff800000u;
    }
    float mx4[2][2] = {{-INFINITY, -INFINITY}, {-INFINITY, -INFINITY}};
#pragma unroll
    for (int j = 0; j < 32; j += 4)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) mx4[x][y] = fmaxf(fmaxf(mx4[x][y], __uint_as_float(r[x][j + 2 * y])), __uint_as_float(r[x][j + 2 * y + 1]));
    float mul[2], log_v[2], mx = -INFINITY;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        mul[x] = factor(cs, !plain && tree ? 1.f : of_keys[x]);
        log_v[x] = !plain && tree ? 0.f : of_keys[4 + x];
        mx = fmaxf(mx, fmaf(fmaxf(mx4[x][0], mx4[x][1]), mul[x], log_v[x]));
    }
    // the reference follows the row's maximum when some row of the warp would see a weight too large otherwise (a warp moves as one:
    // its accesses to tensor memory are collective); a row that does not exist has no say
    const float m_cand = fmaxf(m_run, mx);
    const bool move = !__all_sync(0xffffffffu, !row_ok || m_cand - m_run <= kLazyLog2);
    const float m_new = move ? m_cand : m_run;
    const float m_safe = m_new == -INFINITY ? 0.f : m_new;
    if (move) {
        const float alpha = ex2f_wide(m_run - m_safe);
        l_run *= alpha;
        if (!first) {
            wait_o();
#pragma unroll 1
            for (int blk = 0; blk < 8; ++blk) tmem_scale16(tO + (uint32_t)blk * 16u, alpha);
        }
    }
    m_run = m_new;
    const float shift = (!plain && tree ? -kLazyLog2 : kBiasLog2) - m_safe;        // (of the tree's keys times kDown)
    float sum = 0.f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const float add = shift + log_v[x];
        const uint64_t scale2 = f32x2(mul[x], mul[x]), neg = f32x2(add, add);
        uint64_t acc[2] = {0ull, 0ull};
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float x0, x1;
            f32x2_split(f32x2_fma(f32x2(__uint_as_float(r[x][2 * e]), __uint_as_float(r[x][2 * e + 1])), scale2, neg), x0, x1);
            const float p0 = ex2f(x0), p1 = ex2f(x1);
            acc[e & 1] = f32x2_add(acc[e & 1], f32x2(p0, p1));
            if (!plain && tree) w[e] = pack_bf16(p0, p1);
            else w[e] = pack_f16(p0, p1);
        }
        tmem_st16(tS + 16u * x, w);
        float lo, hi;
        f32x2_split(f32x2_add(acc[0], acc[1]), lo, hi);
        sum = fmaf(lo + hi, !plain && tree ? 1.f : of_keys[8 + x], sum);
    }
    l_run += sum * (!plain && tree ? kUp : 1.f);
}

constexpr int SCALES = 6;                // (a chunk's are written once the one 6 before it has been through the products)
// Places for the flags of a tree's chunk.  The softmax reads them after its last word on chunk c, which lets the product go that frees the chunk's V tile, so that flags of chunks c + 2 and c + 3
// may be written while a warp has yet to read c's (of one row tile, c + 1 is the other group's; a tree of more than 128 nodes has two chunks in a stretch, its last row tile may be the
// only one).  Those of chunk c + 4 and later wait for the product of c + 2: in the same stretch that warp has a hand in it, with one row tile or two, and a later stretch lies behind the barrier
// at this one's end.  (With two places, and the flags read ahead of that word, 16 trees of 60 nodes over 512 to 4096 keys took 0.7 us longer.)
constexpr uint32_t ODDS = 4;
struct Small {
    static constexpr int BARS = 34;
    unsigned long long bar[BARS];
    union {
        float2 ml[2][128];
        int scan[NT / 32 + 4];           // (before anything else)
    };
    alignas(16) float raw[BUFS][8];      // scales of K and V as they come (bulk copies' destination)
    float scale[SCALES][12];             // of a chunk of the cache, by its number: of each 32 keys K's scale, log2 of V's, 1 / V's
    unsigned char par[FSPAD_MAX_NODES_WIDE];         // parents plus one
    uint32_t odd[ODDS][4];               // which V rows of a tree's chunk have an infinity or a NaN in them
    uint32_t tmem;
    int fail, soft_fail;                 // (the second: written and read by the softmax warps alone, around their barriers)
};
static_assert(SMEM + sizeof(Small) <= 232448, "shared memory of an SM");
static_assert(SMEM % 16 == 0 && alignof(Small) >= 16 && offsetof(Small, raw) % 16 == 0, "bulk copies' destination");

__global__ void __launch_bounds__(NT, 1)
tree_attn_fp8_umma_kernel(const Args a, const __grid_constant__ CUtensorMap k_map)
{
    extern __shared__ __align__(1024) unsigned char smem_raw[];      // (nothing else is in shared memory, so it starts on such a boundary: looked at below)
    enum { B_FULL = 0, B_FREE = BUFS, K_FULL = 2 * BUFS, T_FULL = 3 * BUFS, V_FULL = 4 * BUFS, V_FREE = V_FULL + 2, S_FULL = V_FREE + 2,
           P_FULL = S_FULL + 4, O_DONE = P_FULL + 4, Q_FULL = O_DONE + 4, E_FULL = Q_FULL + 2, DRAIN = E_FULL + 2, N_BAR = DRAIN + 2 };
    Small &sm = *reinterpret_cast<Small *>(smem_raw + SMEM);
    static_assert(N_BAR <= Small::BARS, "barriers");
    auto &s_bar = sm.bar;
    auto &s_scan = sm.scan;
    auto &s_tmem = sm.tmem;
    auto &s_fail = sm.fail;
    auto &s_soft_fail = sm.soft_fail;
    auto &s_par = sm.par;
    auto &s_odd = sm.odd;
    auto &s_ml = sm.ml;
    auto &s_raw = sm.raw;
    auto &s_scale = sm.scale;

    if (smem_u32(smem_raw) & 1023u) {                // (tiles are addressed by it)
        if (threadIdx.x == 0) fspad_report(a.status, FSPAD_ERR_ALIGN);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp();
    const uint32_t bar0 = smem_u32(&s_bar[0]);
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
    if (tid == 0) {
        for (int i = 0; i < N_BAR; ++i) {
            int count = 1;
            if (i >= V_FREE && i < S_FULL) count = 2;        // both groups' products
            if ((i >= T_FULL && i < V_FREE) || (i >= P_FULL && i < O_DONE) || (i >= Q_FULL && i < DRAIN))
                count = 4;                           // the four warps of a group, or of those that make values
            if (i >= B_FREE && i < K_FULL) count = 7;        // those, the one for the scales, and both groups' products
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
    Part part = cut_list<NT, UNIT, 1, kManyRows>(a, cta, gridDim.x, parts, s_scan, cta == 0);      // (with a barrier in it)
    __syncthreads();                                 // (what it has used serves for something else)
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    const int nt = tree_units<UNIT>(a), runs = a.Hkv * a.mtiles;

    if (warp == 10 && lane == 0) tell_part<UNIT, kManyRows>(a, parts, part, cta);

    const uint32_t base = smem_u32(smem_raw);
    const uint32_t sQ = base, sK = base + 2 * TILE, sV = base + (2 + BUFS) * TILE;

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
        part.v += s.n_run + kExtra<kManyRows>;
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
        uint32_t n_done = 0, tree_chunks = 0, chunks = 0;    // products of the group so far; the tree's chunks and all of the CTA so far
        auto told = [&](int y) {                             // half y of the weights is there, and what was read of shared memory before may be written again
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(P_FULL + 2 * grp + y));
        };
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
            // The rows of tile t as pairs of e4m3 numbers, each row with its largest magnitude in [2^7, 2^8): the nearest ones in the tile's first half, what is left
            // in its second (change: false for the factors alone, which stay with the rows' threads).  A row that is not finite reads as NaN.
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
                        const int e = top == 0u || top >= 0x7f80u ? 7 : max((int)(top >> 7) - 127, -100);
                        const int mine = __shfl_sync(0xffffffffu, e, (lane & 1) * 16);       // of row 2 (k0 + y) + (lane & 1)
                        if (lane >> 1 == k0 + y) cs = a.scale_log2 * __uint_as_float((uint32_t)(127 - 7 + mine) << 23);
                        if (!change) continue;
                        const float up = __uint_as_float((uint32_t)(127 + 7 - e) << 23);
                        const uint32_t in[4] = {w[y].x, w[y].y, w[y].z, w[y].w};
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float x0 = __uint_as_float(in[j] << 16) * up, x1 = __uint_as_float(in[j] & 0xffff0000u) * up;
                            hi[j] = fspad_f32_to_e4m3(x0, x1);
                            const uint32_t h = fspad_e4m3_to_f16(hi[j]);
                            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
                            lo[j] = fspad_f32_to_e4m3(x0 - f.x, x1 - f.y);
                            if (top >= 0x7f80u) hi[j] = 0x7f7fu;
                        }
                        w[y] = make_uint4(hi[0] | (hi[1] << 16), hi[2] | (hi[3] << 16), lo[0] | (lo[1] << 16), lo[2] | (lo[3] << 16));
                    }
                    __syncwarp();                            // (the rows are read before others write them)
                    if (change)
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const int r = r0 + 2 * (k0 + y) + (lane >> 4);
                            const uint32_t at = to + (uint32_t)(r * 128 + (((piece >> 1) ^ (r & 7)) << 4) + (piece & 1) * 8);
                            asm volatile("st.shared.v2.b32 [%0], {%1, %2};\n" :: "r"(at), "r"(w[y].x), "r"(w[y].y) : "memory");
                            asm volatile("st.shared.v2.b32 [%0], {%1, %2};\n" :: "r"(at + HALF), "r"(w[y].z), "r"(w[y].w) : "memory");
                        }
                }
            };
            // two row tiles: the group's own warp of the tensor cores is told; one: both are, of either form
            auto tell_q = [&] {
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    const int b = s.two || grp == 0 ? Q_FULL : E_FULL;
                    if (!s.two || grp == 0) mbar_arrive(bar(b));
                    if (!s.two || grp == 1) mbar_arrive(bar(b + 1));
                }
            };
            // one row tile: group 0's as it is, for the tree, group 1's as e4m3; two: e4m3, or first as they are for the tree
            fetch_q(grp);
            const bool raw = s.two ? s.n_tree > 0 : grp == 0;
            if (!raw) scale_q(grp, true);
            tell_q();
            // (group 0's own chunks of the cache, if there are any, need the factors all the same)
            if (raw && !s.two && s.n_ch > s.n_tree + (s.n_tree & 1)) scale_q(grp, false);
            if (s.n_tree > 0) {
                for (int i = tid; i < a.N; i += 256) {
                    int p = a.parent[(size_t)s.b * a.N + i];
                    if (i == 0 ? p != -1 : (p < 0 || p >= i)) { fspad_report(a.status, FSPAD_ERR_BAD_TREE); p = -1; }
                    s_par[i] = (unsigned char)(p + 1);
                }
                asm volatile("bar.sync 1, 256;\n" ::: "memory");
            }
            float m_run = -INFINITY, l_run = 0.f;
            bool first = true;
            // Chunks of the cache that exist as a whole have a loop of their own, so that its code is short: jumps over the rest of it cost 600 cycles a turn.
            const int step = s.two ? 1 : 2, whole_end = s.n_ch - (s.L % UNIT != 0 && s.u0 + s.n_ch == s.n_run ? 1 : 0);
            int c = s.two ? 0 : grp;
            auto turn = [&](auto plain_, bool tree, const uint32_t (&see)[4]) {
                constexpr bool plain = decltype(plain_)::value;
                const float *of_keys = s_scale[(chunks + (uint32_t)c) % SCALES];
#pragma unroll 1
                for (int y = 0; y < 2; ++y) {                // 64 keys at a time
                    if (!failed && !mbar_wait(bar(S_FULL + 2 * grp + y), n_done & 1u)) failed = true;
                    tc_fence_after();
                    if (live) {
                        const uint32_t see2[2] = {y ? see[2] : see[0], y ? see[3] : see[1]};
                        softmax_half<plain>(tree, tS + 64u * y, tO, see2, !plain && tree ? a.scale_log2 : cs, of_keys + 2 * y, row_ok, first, m_run, l_run, [&] {
                            // the other half's product before this one
                            if (!failed && !mbar_wait(bar(O_DONE + 2 * grp + (y ^ 1)), (n_done + (uint32_t)y - 1u) & 1u)) failed = true;
                            tc_fence_after();
                        });
                        asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
                    }
                    told(y);
                    first = false;
                }
                ++n_done;
            };
#pragma unroll 1
            while (c < s.n_ch) {
                if (c >= s.n_tree && c < whole_end) {
                    const uint32_t all[4] = {~0u, ~0u, ~0u, ~0u};
#pragma unroll 1
                    for (; c < whole_end; c += step) turn(std::true_type(), false, all);
                    continue;
                }
                const int u = s.u0 + c;
                const bool tree = c < s.n_tree;
                uint32_t see[4];
                if (tree) {
                    // from the node up, word by word, for an ancestor comes before its descendants (with two words of 64 bits a step took three times as long:
                    // 22 chains of 156 nodes, 32 heads, 186 us against 117; trees of ten nodes' depth 54 and 51)
                    const int key0 = u * UNIT;
                    int at = node;
                    while (at >= key0 + 128) at = (int)s_par[at] - 1;
#pragma unroll
                    for (int x = 3; x >= 0; --x) {
                        see[x] = 0u;
                        while (at >= key0 + 32 * x) {
                            see[x] |= 1u << (at & 31);
                            at = (int)s_par[at] - 1;
                        }
                    }
                } else {
                    const int left = s.L - (u - nt) * UNIT;  // 1 .. 127
#pragma unroll
                    for (int x = 0; x < 4; ++x) see[x] = left >= 32 * x + 32 ? ~0u : left > 32 * x ? (1u << (left - 32 * x)) - 1u : 0u;
                }
                turn(std::false_type(), tree, see);
                if (tree) {
                    const uint32_t *odd = s_odd[(tree_chunks + (uint32_t)c) % ODDS];
                    if ((see[0] & odd[0]) | (see[1] & odd[1]) | (see[2] & odd[2]) | (see[3] & odd[3])) l_run = NAN;
                    if (s.two && c == s.n_tree - 1 && s.n_ch > s.n_tree) {   // (the tile's last reader's scores are here)
                        scale_q(grp, true);
                        tell_q();
                    }
                }
                c += step;
            }
            tree_chunks += s.n_tree;
            chunks += (uint32_t)s.n_ch;
            // ---- the group's last product, then the rows ----
            if (!first) {
                if (!failed && !mbar_wait(bar(O_DONE + 2 * grp + 1), (n_done - 1u) & 1u)) failed = true;
            }
            tc_fence_after();
            const bool whole = s.n_ch == s.n_run;
            const int slot = cta * 2 + (s.u0 == 0 ? 1 : 0);
            const long long to_row = !row_ok ? -1 : ((long long)s.b * a.N + node) * a.Hq + head;
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
                const float own = ex2f_wide(m_run - ref), other = ex2f_wide(o.x - ref);
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
                                const int r4 = 4 * k + (lane >> 3);
                                const long long to = __shfl_sync(0xffffffffu, to_row, r4);
                                if (to >= 0)
                                    reinterpret_cast<uint4 *>(a.out + to * D + (x >> 1) * 64)[lane & 7] =
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
        int n = 0, done = 0;                                 // buffers filled, chunks taken so far
        for (;; done += s.n_ch) {
            const Part at = part;
            if (failed || !next(s)) break;
            if (s.u0 == 0 && lane == 0) tell_run<kManyRows>(a, parts, at, cta, done, s.n_run);
            const int *blocks = a.table + (size_t)s.b * a.table_stride;
            const int kv0 = s.u0 + s.n_tree - nt, n_kv = s.n_ch - s.n_tree;  // chunks of the cache
            int mine = 0;
            for (int i = -s.n_tree; i < n_kv && !failed; ++i, ++n) {
                if (i >= 0 && (i & 31) == 0) {
                    if (i + lane < n_kv) {
                        mine = __ldg(blocks + kv0 + i + lane);
                        if (mine < 0 || mine >= a.n_blocks) { fspad_report(a.status, FSPAD_ERR_RANGE); mine = 0; }
                    }
                }
                const int blk = __shfl_sync(0xffffffffu, mine, i & 31);
                const long long at_head = (long long)blk * a.Hkv + s.h;
                const int buf = n % BUFS;
                if (n >= BUFS && !mbar_wait(bar(B_FREE + buf), (uint32_t)(n / BUFS - 1) & 1u)) { failed = true; break; }
                if (lane == 0) {
                    const uint32_t to = sK + (uint32_t)(buf * TILE), full = bar(B_FULL + buf);
                    if (i < 0) {
                        mbar_arrive(full);                   // (the tree's rows are for others to fetch)
                    } else {
                        mbar_expect_tx(full, 2 * HALF + 32);
                        tma_load_2d(to, &k_map, 0, (int)(at_head * 128), full);
                        bulk_load(to + HALF, a.vc + at_head * HALF, HALF, full);
                        bulk_load(smem_u32(&s_raw[buf][0]), a.ks + at_head * 16, 16, full);
                        bulk_load(smem_u32(&s_raw[buf][4]), a.vs + at_head * 16, 16, full);
                    }
                }
                __syncwarp();
            }
        }
        if (failed) s_fail = 1;
        // a CTA that gives up: what has been asked for gets a bounded time to land
        if (failed)
            for (int x = n > BUFS ? n - BUFS : 0; x < n; ++x) (void)mbar_wait(bar(B_FULL + x % BUFS), (uint32_t)(x / BUFS) & 1u);
      } else if (warp != 10) {
        // ================= tensor cores =================
        // A warp for each group.  (One for both took 3000 cycles for what the tensor cores do in 1300: a wait for a phase that is long over costs 170 cycles, a product 50, and
        // nothing in a warp overlaps them.)
        const int g = warp == 9 ? 0 : 1;
        const uint32_t issuer = elect_one() ? 1u : 0u;
        const uint32_t hi = (uint32_t)(make_desc(0, 16) >> 32);
        const uint32_t q_lo = (uint32_t)make_desc(sQ, 16), k_lo = (uint32_t)make_desc(sK, 16), v_lo = (uint32_t)make_desc(sV, HALF);
        const uint32_t tS = tmem + 128u * g, tO = tmem + 256u + 128u * g;
        uint32_t cc = 0;                                     // chunks of the stretches before (slot: modulo 2)
        uint32_t ph_q = 0u, ph_e = 0u, ph_t = 0u, n_p = 0u;  // phases of Q_FULL, E_FULL and (by buffers) T_FULL; products of the group so far
        while (!failed && next(s)) {
            // (through a shuffle they are values that the compiler knows to be the same in every lane, as an instruction's operands have to be)
            s.n_ch = __shfl_sync(0xffffffffu, s.n_ch, 0);
            s.n_tree = __shfl_sync(0xffffffffu, s.n_tree, 0);
            s.two = __shfl_sync(0xffffffffu, (int)s.two, 0) != 0;
            const int turns = s.two ? s.n_ch : (s.n_ch - g + 1) >> 1;
            auto wait_q = [&] {
                if (!failed && !mbar_wait(bar(Q_FULL + g), ph_q)) failed = true;
                ph_q ^= 1u;
            };
            wait_q();
            if (!s.two) {                                    // both forms, whichever the group's chunks need: no phase may be missed
                if (!failed && !mbar_wait(bar(E_FULL + g), ph_e)) failed = true;
                ph_e ^= 1u;
            }
            // the j-th chunk or, of one row tile, the j-th of every other one
            auto wait_k = [&](int j) {
                const int c = s.two ? j : 2 * j + g;
                const uint32_t at = cc + (uint32_t)c, buf = at % BUFS;
                if (!failed && !mbar_wait(bar(K_FULL + buf), (at / BUFS) & 1u)) failed = true;
                if (c < s.n_tree && !failed && !mbar_wait(bar(T_FULL + buf), (ph_t >> buf) & 1u)) failed = true;
            };
            auto issue_s = [&](int j, int y) {               // half y of its keys
                const int c = s.two ? j : 2 * j + g;
                const bool tree = c < s.n_tree;
                const uint32_t buf = (cc + (uint32_t)c) % BUFS;
                if (y == 0 && s.two && c == s.n_tree && c > 0) wait_q();     // the tile again, as e4m3
                if (failed) return;
                tc_fence_after();
                const uint32_t kb = k_lo + buf * (TILE >> 4) + (uint32_t)y * (8192u >> 4), qb = q_lo + (s.two ? (uint32_t)g : tree ? 0u : 1u) * (TILE >> 4), d = tS + 64u * y;
                if (tree) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        const uint32_t off = ((ks >> 2) * HALF + (ks & 3) * 32) >> 4;
                        mma_f16_lo(d, qb + off, hi, kb + off, hi, IDESC64 | IDESC_BF, ks > 0, issuer);
                    }
                } else {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)           // (the queries' second halves against the same codes)
                        mma_f8_ss(d, qb + (uint32_t)(((ks >> 2) * HALF + (ks & 3) * 32) >> 4), kb + (uint32_t)((ks & 3) * 32 >> 4), hi, IDESC64, ks > 0, issuer);
                }
                mma_commit_if(bar(S_FULL + 2 * g + y), issuer);
                if (y == 1) {                                // (two groups' products with two tiles, one group's twice with one)
                    mma_commit_if(bar(B_FREE + buf), issuer);
                    if (!s.two) mma_commit_if(bar(B_FREE + buf), issuer);
                }
            };
            if (turns > 0) {
                wait_k(0);
                issue_s(0, 0);
                issue_s(0, 1);
            }
#pragma unroll 1
            for (int j = 0; j < turns; ++j) {
                const int c = s.two ? j : 2 * j + g;
                const bool tree = c < s.n_tree;
                const uint32_t at = cc + (uint32_t)c, slot = at & 1u;
                // (what the next scores and this product need besides the weights is waited for ahead of them: a wait for a phase that is long over costs 170 cycles)
                if (j + 1 < turns) wait_k(j + 1);
                if (!failed && !mbar_wait(bar(V_FULL + slot), (at >> 1) & 1u)) failed = true;
#pragma unroll 1
                for (int y = 0; y < 2; ++y) {
                    const uint32_t vb = v_lo + slot * (TILE >> 4) + (uint32_t)y * (8192u >> 4), idesc = IDESC | IDESC_MN | (tree ? IDESC_BF : 0u);
                    if (!failed && !mbar_wait(bar(P_FULL + 2 * g + y), n_p & 1u)) failed = true;
                    if (failed) continue;
                    tc_fence_after();
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)           // 16 keys an instruction: 8 columns of packed pairs
                        mma_f16_ts(tO, tS + 64u * y + (uint32_t)ks * 8u, vb + (uint32_t)(ks * 16 * 128 >> 4), hi, idesc, j + y + ks > 0, issuer);
                    mma_commit_if(bar(O_DONE + 2 * g + y), issuer);
                    if (j + 1 < turns) issue_s(j + 1, y);    // (a thread's products complete in order: the scores may replace the weights)
                    if (y == 1) {
                        mma_commit_if(bar(V_FREE + slot), issuer);
                        if (!s.two) mma_commit_if(bar(V_FREE + slot), issuer);
                    }
                }
                ++n_p;
            }
            for (int c = 0; c < s.n_tree; ++c) ph_t ^= 1u << ((cc + (uint32_t)c) % BUFS);
            cc += (uint32_t)s.n_ch;
        }
        if (failed) {
            s_fail = 1;
            if (lane == 0) mma_commit(bar(DRAIN + g));
            (void)mbar_wait(bar(DRAIN + g), 0u);
        }
      } else {
        // ================= scales =================
        uint32_t cc = 0;
        while (!failed && next(s)) {
            for (int c = 0; c < s.n_ch && !failed; ++c, ++cc) {
                const uint32_t buf = cc % BUFS;
                if (!mbar_wait(bar(B_FULL + buf), (cc / BUFS) & 1u)) { failed = true; break; }
                // K's, log2 of V's, its reciprocal, kept in the range that the cache's may have (behind the end there may be anything)
                if (c >= s.n_tree && lane < 4) {
                    const float v = fminf(fmaxf(s_raw[buf][4 + lane], kFp8Least), kFp8Most);
                    float *to = s_scale[cc % SCALES];
                    to[lane] = fminf(fmaxf(s_raw[buf][lane], kFp8Least), kFp8Most);
                    to[4 + lane] = __log2f(v);
                    to[8 + lane] = __frcp_rn(v);
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(bar(K_FULL + buf));
                    mbar_arrive(bar(B_FREE + buf));
                }
            }
        }
        if (failed) s_fail = 1;
      }
    } else {
        // ================= values =================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
        const int w4 = warp - 12;
        uint32_t cc = 0, tree_chunks = 0;                    // chunks so far, the tree's among them
        while (!failed && next(s)) {
            for (int c = 0; c < s.n_ch && !failed; ++c, ++cc) {
                const uint32_t slot = cc & 1u, buf = cc % BUFS, sKb = sK + buf * TILE;
                const int u = s.u0 + c;
                if (!mbar_wait(bar(B_FULL + buf), (cc / BUFS) & 1u)) { failed = true; break; }
                if (c < s.n_tree) {
                    // a chunk of the tree: V before K, so that whoever sees its scores sees which of its V rows are odd
                    const int key0 = u * UNIT;
                    uint32_t *odd = s_odd[tree_chunks % ODDS];
                    ++tree_chunks;
                    const int piece = lane & 15, rows = min(a.N - key0, UNIT);
                    const size_t first = (((size_t)s.b * a.Hkv + s.h) * a.N + key0) * D + piece * 8;
                    if (cc >= 2 && !mbar_wait(bar(V_FREE + slot), ((cc >> 1) - 1u) & 1u)) { failed = true; break; }
                    if (lane == 0) odd[w4] = 0u;             // (a warp's 32 rows are a word)
#pragma unroll 4
                    for (int r = w4 * 32 + (lane >> 4); r < w4 * 32 + 32; r += 2) {
                        const size_t at = r < rows ? first + (size_t)r * D : 0;
                        cp_async16(sV + slot * TILE + tile_off(r, piece), a.tv + at, r < rows);
                        cp_async16(sKb + tile_off(r, piece), a.tk + at, r < rows);
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
                        mbar_arrive(bar(T_FULL + buf));
                        mbar_arrive(bar(B_FREE + buf));
                    }
                } else {
                    const int left = s.L - (u - nt) * UNIT;  // keys of the chunk that exist
                    if (cc >= 2 && !mbar_wait(bar(V_FREE + slot), ((cc >> 1) - 1u) & 1u)) { failed = true; break; }
                    const uint32_t from = sKb + HALF, to = sV + slot * TILE;
                    // a lane takes 16 codes of a row, four rows an instruction; of the 16-byte pieces that they become, lanes of a row's second half store the later
                    // one first, so that the eight of a row lie in eight places of the 128-byte line
                    const int piece = lane & 7, late = piece >> 2;
#pragma unroll 1
                    for (int r8 = 0; r8 < 32; r8 += 16) {
                        uint4 w[4];                          // (all of them under way before the first is used)
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[k] = ld_shared16(from + (uint32_t)((w4 * 32 + r8 + 4 * k + (lane >> 3)) * 128 + piece * 16));
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int r = w4 * 32 + r8 + 4 * k + (lane >> 3);
                            if (r >= left) w[k] = make_uint4(0u, 0u, 0u, 0u);        // what lies behind the end may be anything: zeros
                            const uint32_t in[4] = {late ? w[k].z : w[k].x, late ? w[k].w : w[k].y, late ? w[k].x : w[k].z, late ? w[k].y : w[k].w};
                            uint32_t f[8];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                f[2 * j] = fspad_hmul2(fspad_e4m3_to_f16(in[j]), kDown2);
                                f[2 * j + 1] = fspad_hmul2(fspad_e4m3_to_f16(in[j] >> 16), kDown2);
                            }
                            st_shared16(to + tile_off(r, 2 * piece + late), f[0], f[1], f[2], f[3]);
                            st_shared16(to + tile_off(r, 2 * piece + 1 - late), f[4], f[5], f[6], f[7]);
                        }
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(bar(V_FULL + slot));
                        mbar_arrive(bar(B_FREE + buf));
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

size_t fspad_attn_fp8_umma_workspace(const fspad_ctx *ctx)
{
    return scratch_bytes<BM>(ctx->sm_count);
}

// k_map: rows of the plane's K codes as boxes of 128 rows.
cudaError_t fspad_launch_attn_fp8_umma(fspad_ctx *ctx, packed::Args a, const CUtensorMap &k_map, void *workspace, cudaStream_t st)
{
    const int ctas = ctx->sm_count, smem = SMEM + (int)sizeof(Small);
    a.mtiles = (a.M + BM - 1) / BM;
    a.by_tiles.set((unsigned)a.mtiles);
    scratch_in<BM>(a, ctas, workspace);
    cudaError_t e = raise_shared(ctx, 3, reinterpret_cast<const void *>(&tree_attn_fp8_umma_kernel), smem);
    if (e != cudaSuccess) return e;
    const int entries = merge_entries(a, ctas);
    ctx->launches++;
    e = fspad_launch(tree_attn_fp8_umma_kernel, dim3((unsigned)ctas), dim3(NT), smem, st, 0, a, k_map);
    return e == cudaSuccess ? launch_merge<BM, true>(ctx, a, entries, ctas, st) : e;
}
