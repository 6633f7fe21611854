// Tree-masked attention over a cache held in 8 bits ("Preliminaries": the flattened token tree is the target's input and the attention mask
// built from the tree introduces the dependencies between its tokens; one node is the plain single-token step).
//
// For query row i (tree node x head of the group) of sequence b and kv head h:
//   s_j = c q_i . k_j,   out_i = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
// over the L_b cached keys, whose rows are code * scale, and over the node itself and its ancestors among the bf16 tree rows.
//
// Few query rows a kv head (up to 16, in tiles of 8 or 16; more: tree_attn_fp8_umma.cu).  Nothing but the tensor cores reads a code: K and V come by TMA and are
// operands as they are.  The products stand on their heads, so that the cache is the operand with 128 rows: S^T [128 keys][rows] = K Q^T, then
// O^T [128 elements][rows] += V^T P^T, with V's tile taken as its own transpose.  What the other operand holds is 16 bits wide by nature, and is written as a sum of 8-bit numbers, in
// columns of their own that are added up afterwards:
//   a query  = hi + lo / 16, e4m3, the row scaled by a power of two to a largest magnitude in [2^7, 2^8): exact from 2^-6 on, at most 2^-13 of the largest, and off by at most 2^-14 below, 2^-21 of it
//   a weight = hi + mid + lo, e5m2, each the nearest number to what is left: 3 significant bits each, off by at most 2^-9 of the weight and 2^-17 (2^11 stands for the largest)
// V's scale goes into the weights, as an addend of the exponent: the reference that weights are relative to follows the maximum of score + log2(scale).
//
// A CTA's warps: 0 copies, 1 and 2 the tensor cores' products of the two groups, 4-7 and 8-11 the groups that take the chunks of 128 keys in turn, a key a thread, each with a
// reference, sums and an accumulator of its own; 12-15 make the queries' two forms and deal with the tree's keys (16 at most) in single precision, up to two stretches ahead.
//
// Bound by reading the cache where sequences are long: 32 single tokens (8 heads a kv head) over 4 to 32 thousand keys take 184 us captured in a graph (196 called one after another), 95 percent of what the codes and scales take at
// the measured copy bandwidth (captured, as all that follows: 199 with one warp for both groups' products, 190 without warps of their own for queries and trees); with 16 rows, 32 sequences of 4 to 12 thousand keys
// take 97.  Short sequences are bound by a stretch's chain, some 7000 cycles with three chunks: a turn 1700 to 2000 (the first moves the references), the sums 700, the last product 1100, the
// rows 700; 64 single tokens over 100 to 600 keys take 23.1 us (32.6 with queries and tree in the groups' own way).  A short call is its latencies: one token over 2000 keys
// takes 9.3 us (9.8 called one after another), the list 2400 cycles of it, the part 7000, and the merge behind it; its copies take 0.6.
#include "fp8.cuh"
#include "packed_list.cuh"

namespace {

using namespace packed;
using namespace umma;

constexpr int UNIT = 128;                // keys of a chunk
constexpr int NT = 512;
constexpr int SLOT = 128 * 128;          // codes of a chunk's K or V
constexpr uint32_t TMEM = 256;           // columns
constexpr float kLag = 4.f, kBias = 11.f;            // weights are 2^(score - reference + 11), the largest at most 2^15
constexpr float kOwnDown = 0x1p-11f;                 // ... of which the accumulators and sums are rid at the end

__host__ __device__ constexpr int slots_of(int R) { return R == 8 ? 12 : 11; }                // (what shared memory holds)
__host__ __device__ constexpr int columns_of(int R) { return R == 8 ? 32 : 3 * R; }          // of weights: a multiple of 16

template <int R> struct Small {
    unsigned long long full[slots_of(R)], free[slots_of(R)], s_full[2][2], p_full[2][2], o_done[2][2], ready[2], tree_done[2], over[2], drain[2];
    alignas(16) float raw[8][8];         // (bulk copies' destination) scales of a chunk's K and V, by its number
    alignas(16) float tree_w[R * R];     // [nodes][R]: scores, then weights of the tree's keys
    float cs[2][R];                      // a query's scores -> log2 units (of two stretches in turn, as whatever the front's warps make)
    float ref[2][R], lim[2][R], m[2][R], alpha[2][R];        // of each group's rows: kBias - reference; what a score may reach; the reference; the accumulator's factor
    float top[2][4][R], sum[2][4][R];    // by warps
    float tree_m[2][R], tree_l[2][R];
    float end[2][4][R];                  // by groups: the factors of a row's three parts, and of what they add up to
    uint32_t odd;
    int scan[NT / 32 + 4];
    uint32_t tmem;
    int fail;
};
template <int R> constexpr int bytes_of() { return slots_of(R) * SLOT + 4 * R * 128 + 4 * columns_of(R) * 128 + (int)sizeof(Small<R>); }

struct Maps { CUtensorMap k, v; };

// (Issued by the one lane whose e is not 0.)
__device__ __forceinline__ void mma_f8(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate, uint32_t e)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
                 "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %5, p;\n\t}\n"
                 :: "r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate), "r"(e) : "memory");
}
// N columns of a lane, from tensor memory; all that were asked for are there behind ld_wait.
__device__ __forceinline__ void ld_issue(uint32_t at, uint32_t (&r)[4])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ld_issue(uint32_t at, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ld_issue(uint32_t at, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
// (no use of them can be scheduled ahead of the wait)
template <int N> __device__ __forceinline__ void pin(uint32_t (&r)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]) :: "memory");
}
__device__ __forceinline__ void st8(uint32_t at, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// The largest of a warp's values (NaN have no part in it).
__device__ __forceinline__ float warp_max(float x)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;\n" : "=f"(r) : "f"(x));     // (volatile: of the whole warp, whoever uses it)
    return r;
}
__device__ __forceinline__ void group_sync(int g) { asm volatile("bar.sync %0, 128;\n" :: "r"(1 + g) : "memory"); }
__device__ __forceinline__ bool group_any(int g, bool x)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %2, 0;\n\tbarrier.cta.red.or.pred q, %1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}\n" : "=r"(r) : "r"(1 + g), "r"((uint32_t)x) : "memory");
    return r != 0;
}
__device__ __forceinline__ void front_sync() { asm volatile("bar.sync 4, 128;\n" ::: "memory"); }
__device__ __forceinline__ void both_sync() { asm volatile("bar.sync 3, 256;\n" ::: "memory"); }

// Two weights as three pairs of e5m2 numbers (an e5m2 number is a half's upper byte): hi, mid and lo in the low 16 bits of what comes back.
__device__ __forceinline__ void split_weights(float w0, float w1, uint32_t &hi, uint32_t &mid, uint32_t &lo)
{
    __half2 x = __floats2half2_rn(w0, w1);
    auto piece = [](__half2 y) {
        uint16_t r;
        asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;\n" : "=h"(r) : "r"(*reinterpret_cast<const uint32_t *>(&y)));
        return (uint32_t)r;
    };
    auto back = [](uint32_t two) {
        const uint32_t h = __byte_perm(two, 0u, 0x1404);          // byte 0 and byte 1, each above a zero byte
        return *reinterpret_cast<const __half2 *>(&h);
    };
    hi = piece(x);
    x = __hsub2(x, back(hi));
    mid = piece(x);
    x = __hsub2(x, back(mid));
    lo = piece(x);
}

template <int R>
__global__ void __launch_bounds__(NT, 1)
tree_attn_fp8_kernel(const Args a, const __grid_constant__ Maps maps)
{
    constexpr int SLOTS = slots_of(R), NP = columns_of(R), H = R / 2;
    static_assert(alignof(Small<R>) == 16 && offsetof(Small<R>, raw) % 16 == 0, "bulk copies' destination");
    constexpr uint32_t O_AT = 8 * R, TREE_AT = O_AT + 2 * NP;     // S of group g, one of two in turn: 4 R g + 2 R (0, 1) ..; O: O_AT + NP g ..; tree: TREE_AT + R (0, 1) ..
    static_assert(TREE_AT + 2 * R <= TMEM, "tensor memory");
    constexpr uint32_t IDESC = (1u << 4) | ((128u >> 4) << 24);
    constexpr uint32_t IDESC_S = IDESC | ((2u * R >> 3) << 17);                      // e4m3 x e4m3
    constexpr uint32_t IDESC_O = IDESC | ((uint32_t)(NP >> 3) << 17) | (1u << 10) | (1u << 15) | (1u << 16);     // e4m3 x e5m2, both with their rows running fastest
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    if (smem_u32(smem_raw) & 1023u) {                // (tiles are addressed by it)
        if (threadIdx.x == 0) fspad_report(a.status, FSPAD_ERR_ALIGN);
        return;
    }
    constexpr int Q_OFF = SLOTS * SLOT, P_OFF = Q_OFF + 4 * R * 128, END = P_OFF + 4 * NP * 128;      // (weights of group g: P_OFF + 2 NP 128 g, one of two in turn)
    Small<R> &sm = *reinterpret_cast<Small<R> *>(smem_raw + END);
    const uint32_t ring = smem_u32(smem_raw), sQ = ring + Q_OFF, sP = ring + P_OFF;
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp();
    auto bar = [&](const unsigned long long &b) { return smem_u32(&b); };
    if (tid == 0) {
        for (int i = 0; i < SLOTS; ++i) { mbar_init(bar(sm.full[i]), 1); mbar_init(bar(sm.free[i]), 1); }
        for (int g = 0; g < 2; ++g) {
            for (int y = 0; y < 2; ++y) { mbar_init(bar(sm.s_full[g][y]), 1); mbar_init(bar(sm.p_full[g][y]), 4); mbar_init(bar(sm.o_done[g][y]), 1); }
            mbar_init(bar(sm.drain[g]), 1);
            mbar_init(bar(sm.ready[g]), 4);
            mbar_init(bar(sm.tree_done[g]), 4);
            mbar_init(bar(sm.over[g]), 10);
        }
        sm.fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" :: "r"(smem_u32(&sm.tmem)), "r"(TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    fspad_pdl_trigger();
    fspad_pdl_wait();
    tc_fence_before();
    const int cta = blockIdx.x;
    Parts parts;
    Part part = cut_list<NT, UNIT, 1, kFewRows>(a, cta, gridDim.x, parts, sm.scan, cta == 0);        // (with a barrier in it)
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sm.tmem, 0);
    const int runs = a.Hkv * a.mtiles;               // (the tree is one unit: it has 16 nodes at most)
    if (warp == 3 && lane == 0) tell_part<UNIT, kFewRows>(a, parts, part, cta);

    // Every warp goes through the CTA's stretches by itself: of run (b, h, tile) the tree, if it is among the units, and n_kv chunks of the cache from kv0 on.
    struct Stretch { int b, h, row0, L, n_run, units, kv0, n_kv; bool tree, whole; };
    auto next = [&](Stretch &s) -> bool {
        if (part.left <= 0) return false;
        if (s.b != part.b) s.L = prefix_of(a, part.b, false);
        s.b = part.b;
        s.n_run = run_units<UNIT>(a, s.L);
        s.units = min(s.n_run - part.u, part.left);
        s.tree = part.u == 0;
        s.whole = s.units == s.n_run;
        s.kv0 = part.u - (s.tree ? 0 : 1);
        s.n_kv = s.units - (s.tree ? 1 : 0);
        s.h = a.by_tiles.of(part.run);
        s.row0 = (part.run - s.h * a.mtiles) * R;
        part.left -= s.units;
        part.u = 0;
        part.v += s.n_run + kExtra<kFewRows>;
        if (++part.run == runs) { part.run = 0; ++part.b; }
        return true;
    };
    bool failed = false;
    Stretch s;
    s.b = -1;

    if (warp == 0) {
        // ================= copies =================
        uint32_t n = 0, chunk = 0;                   // slots filled, chunks so far
        for (int done = 0;; done += s.units) {
            const Part at = part;
            if (failed || !next(s)) break;
            if (s.tree && lane == 0) tell_run<kFewRows>(a, parts, at, cta, done, s.n_run);
            const int *blocks = a.table + (size_t)s.b * a.table_stride;
            int mine = 0;
            for (int i = 0; i < s.n_kv && !failed; ++i, ++chunk) {
                if ((i & 31) == 0 && i + lane < s.n_kv) {
                    mine = __ldg(blocks + s.kv0 + i + lane);
                    if (mine < 0 || mine >= a.n_blocks) { fspad_report(a.status, FSPAD_ERR_RANGE); mine = 0; }
                }
                const long long at_head = (long long)__shfl_sync(0xffffffffu, mine, i & 31) * a.Hkv + s.h;
                for (int plane = 0; plane < 2; ++plane, ++n) {
                    const uint32_t slot = n % SLOTS;
                    if (n >= SLOTS && !mbar_wait(bar(sm.free[slot]), (n / SLOTS - 1u) & 1u)) { failed = true; break; }
                    if (lane == 0) {
                        const uint32_t full = bar(sm.full[slot]);
                        mbar_expect_tx(full, plane ? SLOT + 32 : SLOT);
                        tma_load_2d(ring + slot * SLOT, plane ? &maps.v : &maps.k, 0, (int)(at_head * 128), full);
                        if (plane) {                 // (both scales: this slot cannot be filled again before they have been read)
                            bulk_load(smem_u32(&sm.raw[chunk & 7u][0]), a.ks + at_head * 16, 16, full);
                            bulk_load(smem_u32(&sm.raw[chunk & 7u][4]), a.vs + at_head * 16, 16, full);
                        }
                    }
                    __syncwarp();
                }
            }
        }
        if (failed) {                                // what has been asked for gets a bounded time to land
            sm.fail = 1;
            for (uint32_t x = n > SLOTS ? n - SLOTS : 0u; x < n; ++x) (void)mbar_wait(bar(sm.full[x % SLOTS]), (x / SLOTS) & 1u);
        }
    } else if (warp < 3) {
        // ================= tensor cores =================
        // A warp for each group: a wait for a phase that is long over costs 200 cycles, a product 50 to 100, and nothing in a warp overlaps them (one warp for both took
        // up to 1650 cycles a chunk).  The scores of a group's next turn are made ahead.
        const int g = warp - 1;
        const uint32_t issuer = elect_one() ? 1u : 0u;
        const uint32_t hi = (uint32_t)(make_desc(0, 16) >> 32);                      // 128-byte swizzle, 8 rows 1024 bytes apart
        const uint32_t q_lo = (uint32_t)make_desc(sQ, 16), r_lo = (uint32_t)make_desc(ring, 16);
        // weights: 16 columns of a key side by side, keys one behind the other, eight of them 128 bytes, the next 16 columns 2048 bytes further
        const uint32_t p_hi = (1u << 14) | (2048u >> 4), p_lo = (((sP + (uint32_t)(2 * NP * 128 * g)) >> 4) & 0x3fffu) | ((128u >> 4) << 16);
        const uint32_t tS = tmem + 4u * R * g, tO = tmem + O_AT + (uint32_t)(NP * g);
        uint32_t n = 0, n_p = 0, number = 0;         // chunks of the stretches before, turns of the group, stretches
        for (; !failed && next(s); ++number) {
            s.n_kv = __shfl_sync(0xffffffffu, s.n_kv, 0);
            // (of every stretch, whether there is something to do in it or not: a parity tells a phase from the next only)
            if (!mbar_wait(bar(sm.ready[number & 1u]), (number >> 1) & 1u)) failed = true;
            const uint32_t q_at = q_lo + (number & 1u) * (uint32_t)(2 * R * 128 >> 4);
            const int turns = (s.n_kv - g + 1) >> 1;
            auto wait_k = [&](int t) {
                const uint32_t at = 2u * (n + (uint32_t)(2 * t + g));
                if (!failed && !mbar_wait(bar(sm.full[at % SLOTS]), (at / SLOTS) & 1u)) failed = true;
            };
            auto scores = [&](int t) {
                const uint32_t slot = 2u * (n + (uint32_t)(2 * t + g)) % SLOTS, y = (n_p + (uint32_t)t) & 1u;
                if (failed) return;
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) mma_f8(tS + 2u * R * y, r_lo + slot * (SLOT >> 4) + ks * 2u, hi, q_at + ks * 2u, hi, IDESC_S, ks > 0, issuer);
                mma_commit_if(bar(sm.s_full[g][y]), issuer);
                mma_commit_if(bar(sm.free[slot]), issuer);
            };
#pragma unroll 1
            for (int t = 0; t < 2 && t < turns; ++t) {
                wait_k(t);
                scores(t);
            }
#pragma unroll 1
            for (int t = 0; t < turns; ++t) {
                const uint32_t at = 2u * (n + (uint32_t)(2 * t + g)) + 1u, slot = at % SLOTS, k = n_p + (uint32_t)t, y = k & 1u;
                if (t + 2 < turns) wait_k(t + 2);
                if (!failed && !mbar_wait(bar(sm.full[slot]), (at / SLOTS) & 1u)) failed = true;
                if (!failed && !mbar_wait(bar(sm.p_full[g][y]), (k >> 1) & 1u)) failed = true;
                if (!failed) {
                    tc_fence_after();
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)   // 32 keys an instruction
                        mma_f8(tO, r_lo + slot * (SLOT >> 4) + ks * 256u, hi, p_lo + y * (uint32_t)(NP * 128 >> 4) + ks * 32u, p_hi, IDESC_O, t + ks > 0, issuer);
                    mma_commit_if(bar(sm.o_done[g][y]), issuer);
                    mma_commit_if(bar(sm.free[slot]), issuer);
                }
                if (t + 2 < turns) scores(t + 2);    // (the group has read the ones in their place)
            }
            n_p += (uint32_t)turns;
            n += (uint32_t)s.n_kv;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.over[number & 1u]));
        }
        if (failed) {
            sm.fail = 1;
            if (lane == 0) mma_commit(bar(sm.drain[g]));
            (void)mbar_wait(bar(sm.drain[g]), 0u);
        }
    } else if (warp >= 12) {
        // ================= queries and the tree's keys, a stretch or two ahead of the groups =================
        const int w4 = warp & 3, t = tid & 127;      // t: element of a row
        const uint32_t tT = tmem + ((uint32_t)(w4 * 32) << 16) + TREE_AT;
        for (uint32_t number = 0; next(s); ++number) {
            const uint32_t y2 = number & 1u;
            // what is needed first is asked for at once: the half warp's query rows (8 x + 2 w4 + lane / 16, 16 bytes a lane), parents, the first node's K and V
            const int half = 2 * w4 + (lane >> 4), piece = lane & 15;
            const size_t first = ((size_t)s.b * a.Hkv + s.h) * a.N * D;
            const unsigned short *const v_at = reinterpret_cast<const unsigned short *>(a.tv + first) + t;
            const uint4 *const k_at = reinterpret_cast<const uint4 *>(a.tk + first) + piece;
            uint4 qw[R / 8], k0 = make_uint4(0u, 0u, 0u, 0u);
            uint32_t v0 = 0u;
            int up = -1;
#pragma unroll
            for (int x = 0; x < R / 8; ++x) {
                const int gr = s.row0 + 8 * x + half, node = a.by_G.of(gr);
                qw[x] = make_uint4(0u, 0u, 0u, 0u);
                if (gr < a.M) qw[x] = __ldg(reinterpret_cast<const uint4 *>(a.q + ((size_t)(s.b * a.N + node) * a.Hq + s.h * a.G + (gr - node * a.G)) * D) + piece);
            }
            if (s.tree) {
                k0 = __ldg(k_at);
                v0 = __ldg(v_at);
                if (w4 == 0 && lane < a.N) up = __ldg(a.parent + (size_t)s.b * a.N + lane);
            }
            // (what the stretch before the last used is free again)
            if (number >= 2 && !failed && !mbar_wait(bar(sm.over[y2]), ((number >> 1) - 1u) & 1u)) failed = true;
            tc_fence_after();
            if (s.n_kv > 0) {
                // ---- queries: half a warp a row ----
#pragma unroll
                for (int x = 0; x < R / 8; ++x) {
                    const int r = 8 * x + half;
                    const uint4 w = qw[x];
                    uint32_t m = fspad_most2(fspad_most2(w.x, w.y), fspad_most2(w.z, w.w));
#pragma unroll
                    for (int off = 8; off > 0; off >>= 1) m = fspad_most2(m, __shfl_xor_sync(0xffffffffu, m, off));
                    const uint32_t top = max(m & 0xffffu, m >> 16);
                    const int e = top == 0u || top >= 0x7f80u ? 7 : max((int)(top >> 7) - 127, -100);
                    const float up = __uint_as_float((uint32_t)(127 + 7 - e) << 23);
                    if (piece == 0) sm.cs[y2][r] = a.scale_log2 * __uint_as_float((uint32_t)(127 - 7 + e) << 23);
                    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
                    uint32_t q_hi[4], q_lo[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float x0 = __uint_as_float(in[j] << 16) * up, x1 = __uint_as_float(in[j] & 0xffff0000u) * up;
                        q_hi[j] = fspad_f32_to_e4m3(x0, x1);
                        const uint32_t h = fspad_e4m3_to_f16(q_hi[j]);
                        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
                        q_lo[j] = fspad_f32_to_e4m3((x0 - f.x) * 16.f, (x1 - f.y) * 16.f);
                        if (top >= 0x7f80u) q_hi[j] = 0x7f7fu;       // a row that is not finite reads as NaN
                    }
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int row = r + y * R;
                        const uint32_t at = sQ + y2 * (uint32_t)(2 * R * 128) + (uint32_t)(row * 128 + (((piece >> 1) ^ (row & 7)) << 4) + (piece & 1) * 8);
                        const uint32_t *c = y ? q_lo : q_hi;
                        asm volatile("st.shared.v2.b32 [%0], {%1, %2};\n" :: "r"(at), "r"(c[0] | (c[1] << 16)), "r"(c[2] | (c[3] << 16)) : "memory");
                    }
                }
                fence_async_smem();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.ready[y2]));
            if (s.tree) {
                // ---- the tree's keys, in single precision ----
                float *const w_at = sm.tree_w;
                // (which of them a row sees is looked at behind the products; a row's 16 lanes have 8 elements each)
#pragma unroll 2
                for (int j = 0; j < a.N; ++j) {
                    const uint4 k = j == 0 ? k0 : __ldg(k_at + (size_t)j * 16);
#pragma unroll
                    for (int x = 0; x < R / 8; ++x) {
                        float d = 0.f;
                        auto two = [&](uint32_t p, uint32_t q) {
                            d = fmaf(__uint_as_float(p << 16), __uint_as_float(q << 16), d);
                            d = fmaf(__uint_as_float(p & 0xffff0000u), __uint_as_float(q & 0xffff0000u), d);
                        };
                        two(qw[x].x, k.x); two(qw[x].y, k.y); two(qw[x].z, k.z); two(qw[x].w, k.w);
#pragma unroll
                        for (int off = 8; off > 0; off >>= 1) d += __shfl_xor_sync(0xffffffffu, d, off);
                        if (piece == 0) w_at[j * R + 8 * x + half] = d * a.scale_log2;
                    }
                }
                uint32_t see = 0u;                   // of row `lane`, in the first warp
                if (w4 == 0) {
                    // each node's ancestors and itself, a node a lane, by doubling: after a round a lane has those up to 2^r above, and the node that far up
                    uint32_t above = 1u << lane;
                    if (lane < a.N && (lane == 0 ? up != -1 : (up < 0 || up >= lane))) { fspad_report(a.status, FSPAD_ERR_BAD_TREE); up = -1; }
#pragma unroll 1
                    for (int reach = 1; reach < a.N; reach <<= 1) {
                        const uint32_t m = __shfl_sync(0xffffffffu, above, up & 31);
                        const int nx = __shfl_sync(0xffffffffu, up, up & 31);
                        if (up >= 0) { above |= m; up = nx; }
                    }
                    const int gr = s.row0 + lane;
                    see = __shfl_sync(0xffffffffu, above, a.by_G.of(min(gr, a.M - 1)) & 31);
                    if (gr >= a.M) see = 0u;
                    if (lane == 0) sm.odd = 0u;
                }
                front_sync();
                if (t < R) {
                    float m = -INFINITY, l = 0.f;
                    for (int j = 0; j < a.N; ++j) m = fmaxf(m, (see >> j) & 1u ? w_at[j * R + t] : -INFINITY);
                    const float safe = m == -INFINITY ? 0.f : m;
                    for (int j = 0; j < a.N; ++j) {
                        const float w = (see >> j) & 1u ? ex2f(w_at[j * R + t] - safe) : 0.f;
                        w_at[j * R + t] = w;
                        l += w;
                    }
                    sm.tree_m[y2][t] = m;
                    sm.tree_l[y2][t] = l;
                }
                front_sync();
                float acc[R];
#pragma unroll
                for (int r = 0; r < R; ++r) acc[r] = 0.f;
                uint32_t odd = 0u;
#pragma unroll 2
                for (int j = 0; j < a.N; ++j) {
                    const uint32_t v16 = j == 0 ? v0 : __ldg(v_at + (size_t)j * D);
                    // (an infinity or a NaN must not reach the rows that do not see it: it is taken out, and those that do get NaN)
                    const bool is_odd = (v16 & 0x7f80u) == 0x7f80u;
                    if (is_odd) odd |= 1u << j;
                    const float v = is_odd ? 0.f : __uint_as_float(v16 << 16) * kDown;
#pragma unroll
                    for (int r = 0; r < R; r += 4) {
                        const float4 w = *reinterpret_cast<const float4 *>(w_at + j * R + r);
                        acc[r] = fmaf(w.x, v, acc[r]); acc[r + 1] = fmaf(w.y, v, acc[r + 1]); acc[r + 2] = fmaf(w.z, v, acc[r + 2]); acc[r + 3] = fmaf(w.w, v, acc[r + 3]);
                    }
                }
                odd = __reduce_or_sync(0xffffffffu, odd);
                if (lane == 0 && odd) atomicOr(&sm.odd, odd);
#pragma unroll
                for (int r = 0; r < R; r += 8) {
                    uint32_t v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = __float_as_uint(acc[r + j]);
                    __syncwarp();
                    st8(tT + y2 * (uint32_t)R + (uint32_t)r, v);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
                tc_fence_before();
                front_sync();
                if (t < R && (see & sm.odd)) sm.tree_l[y2][t] = NAN;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.tree_done[y2]));
        }
        if (failed) sm.fail = 1;
    } else if (warp >= 4) {
        // ================= weights, rows =================
        const int g = (warp - 4) >> 2, w4 = warp & 3, t = (tid - 128) & 127;         // t: key of a chunk, and element of a row
        const uint32_t lanes = (uint32_t)(w4 * 32) << 16, tS = tmem + lanes + 4u * R * g, tO = tmem + lanes + O_AT, tT = tmem + lanes + TREE_AT;
        unsigned char *const p_at = smem_raw + P_OFF + 2 * NP * 128 * g;
        uint32_t chunks = 0, n_s = 0, n_o[2] = {0u, 0u}, stretch = 0;        // chunks of the stretches before; scores of the group, products of both so far; stretches
        for (; next(s); ++stretch) {
            const uint32_t at2 = stretch & 1u;
            if (t < R) {
                sm.m[g][t] = sm.lim[g][t] = -INFINITY;
                sm.ref[g][t] = kBias;
            }
            group_sync(g);
            if (s.n_kv > g && !failed && !mbar_wait(bar(sm.ready[at2]), (stretch >> 1) & 1u)) failed = true;
            float l[R];
#pragma unroll
            for (int r = 0; r < R; ++r) l[r] = 0.f;
            bool first = true;
#pragma unroll 1
            for (int i = g; i < s.n_kv; i += 2) {
                const uint32_t k = n_s++, buf = k & 1u;      // (the group's turns so far)
                if (!failed && !mbar_wait(bar(sm.s_full[g][buf]), (k >> 1) & 1u)) failed = true;
                tc_fence_after();
                float x[R];
                {
                    uint32_t u[R], v[R];
                    __syncwarp();
                    ld_issue(tS + 2u * R * buf, u);
                    ld_issue(tS + 2u * R * buf + R, v);
                    ld_wait();
                    pin(u);
                    pin(v);
#pragma unroll
                    for (int r = 0; r < R; ++r) x[r] = fmaf(__uint_as_float(v[r]), 0.0625f, __uint_as_float(u[r]));
                }
                const uint32_t number = chunks + (uint32_t)i, v_slot = (2u * number + 1u) % SLOTS;
                if (!failed && !mbar_wait(bar(sm.full[v_slot]), ((2u * number + 1u) / SLOTS) & 1u)) failed = true;
                // the warp's 32 keys' scales (kept in the range that the cache's may have: behind the end there may be anything)
                const float ks = fminf(fmaxf(sm.raw[number & 7u][w4], kFp8Least), kFp8Most), vs = fminf(fmaxf(sm.raw[number & 7u][4 + w4], kFp8Least), kFp8Most);
                const float lv = __log2f(vs), iv = __frcp_rn(vs);
                const int left = s.L - (s.kv0 + i) * UNIT;       // keys of the chunk that exist
                const bool there = t < left;
                bool above = false;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    x[r] = there ? fmaf(x[r], fminf(fmaxf(sm.cs[at2][r] * ks, 0x1p-126f), kMost), lv) : -INFINITY;       // (scores of 0 stay that)
                    above |= x[r] > sm.lim[g][r];
                }
                if (group_any(g, above)) {
                    // ---- the references move to the rows' maxima ----
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float m = warp_max(x[r]);
                        if (lane == r) sm.top[g][w4][r] = m;
                    }
                    group_sync(g);
                    if (t < R) {
                        const float was = sm.m[g][t], m = fmaxf(fmaxf(fmaxf(sm.top[g][0][t], sm.top[g][1][t]), fmaxf(sm.top[g][2][t], sm.top[g][3][t])), was);
                        sm.alpha[g][t] = m == -INFINITY ? 1.f : ex2f_wide(was - m);
                        sm.m[g][t] = m;
                        sm.lim[g][t] = m + kLag;
                        sm.ref[g][t] = m == -INFINITY ? kBias : kBias - m;
                    }
                    group_sync(g);
#pragma unroll
                    for (int r = 0; r < R; ++r) l[r] *= sm.alpha[g][r];
                    if (!first) {                    // the product of the turn before (those before that are known to be complete: the scores came behind them)
                        if (!failed && !mbar_wait(bar(sm.o_done[g][buf ^ 1u]), ((k - 1u) >> 1) & 1u)) failed = true;
                        tc_fence_after();
#pragma unroll 1
                        for (int z = 0; z < 3; ++z) {
                            uint32_t u[R];
                            __syncwarp();
                            ld_issue(tO + (uint32_t)(NP * g + z * R), u);
                            ld_wait();
                            pin(u);
#pragma unroll
                            for (int j = 0; j < R; ++j) u[j] = __float_as_uint(__uint_as_float(u[j]) * sm.alpha[g][j]);
#pragma unroll
                            for (int j = 0; j < R; j += 8) {
                                const uint32_t v[8] = {u[j], u[j + 1], u[j + 2], u[j + 3], u[j + 4], u[j + 5], u[j + 6], u[j + 7]};
                                st8(tO + (uint32_t)(NP * g + z * R + j), v);
                            }
                        }
                        asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
                    }
                }
                first = false;
                uint32_t words[3][R / 4];
#pragma unroll
                for (int r = 0; r < R; r += 4) {
                    uint32_t c[3][2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float w0 = ex2f(x[r + 2 * y] + sm.ref[g][r + 2 * y]), w1 = ex2f(x[r + 2 * y + 1] + sm.ref[g][r + 2 * y + 1]);
                        l[r + 2 * y] = fmaf(w0, iv, l[r + 2 * y]);
                        l[r + 2 * y + 1] = fmaf(w1, iv, l[r + 2 * y + 1]);
                        split_weights(w0, w1, c[0][y], c[1][y], c[2][y]);
                    }
#pragma unroll
                    for (int z = 0; z < 3; ++z) words[z][r / 4] = __byte_perm(c[z][0], c[z][1], 0x5410);
                }
                auto word = [&](int i4) { return i4 < 3 * R / 4 ? words[i4 / (R / 4)][i4 % (R / 4)] : 0u; };
#pragma unroll
                for (int c = 0; c < NP / 16; ++c)
                    *reinterpret_cast<uint4 *>(p_at + buf * (NP * 128) + c * 2048 + t * 16) = make_uint4(word(4 * c), word(4 * c + 1), word(4 * c + 2), word(4 * c + 3));
                if (left < UNIT) {
                    // what lies behind the end may be anything, and 0 times a NaN is one: rows of zeros
                    if (!there)
#pragma unroll
                        for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4 *>(smem_raw + v_slot * SLOT + t * 128 + c * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                fence_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sm.p_full[g][buf]));
            }
            chunks += (uint32_t)s.n_kv;
            // ---- sums over the keys, then the rows: each group the half of them ----
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float v = l[r];
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
                if (lane == r) sm.sum[g][w4][r] = v;
            }
            const int mine[2] = {(s.n_kv + 1) / 2, s.n_kv / 2};      // chunks of each group
            n_o[0] += (uint32_t)mine[0];
            n_o[1] += (uint32_t)mine[1];
            tc_fence_before();
            both_sync();
            if (s.tree && !failed && !mbar_wait(bar(sm.tree_done[at2]), (stretch >> 1) & 1u)) failed = true;
            const int rows = min(R, a.M - s.row0), r0 = g * ((rows + 1) >> 1), r1 = g ? rows : (rows + 1) >> 1, slot = cta * 2 + (s.tree ? 1 : 0);
            if (t >= r0 && t < r1) {                 // (while the last products are under way)
                float m[3], lr[3];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    m[y] = mine[y] > 0 ? sm.m[y][t] : -INFINITY;
                    lr[y] = mine[y] > 0 ? ((sm.sum[y][0][t] + sm.sum[y][1][t]) + (sm.sum[y][2][t] + sm.sum[y][3][t])) * kOwnDown : 0.f;
                }
                m[2] = s.tree ? sm.tree_m[at2][t] : -INFINITY;
                lr[2] = s.tree ? sm.tree_l[at2][t] : 0.f;
                const float top = fmaxf(fmaxf(m[0], m[1]), m[2]);
                float sum = 0.f;
#pragma unroll
                for (int y = 0; y < 3; ++y) {
                    const float f = m[y] == -INFINITY ? 1.f : ex2f_wide(m[y] - top);      // (without a maximum a part is zero, or NaN)
                    sm.end[g][y][t] = f;
                    sum = fmaf(f, lr[y], sum);
                }
                sm.end[g][3][t] = kUp / sum;
                if (!s.whole) a.part_ml[(size_t)slot * R + t] = make_float2(top, sum);
            }
            group_sync(g);
#pragma unroll
            for (int y = 0; y < 2; ++y)
                if (mine[y] > 0 && !failed && !mbar_wait(bar(sm.o_done[y][(n_o[y] - 1u) & 1u]), ((n_o[y] - 1u) >> 1) & 1u)) failed = true;
            tc_fence_after();
            if (failed) sm.fail = 1;
            uint32_t o[2][3][H], tr[H];
            __syncwarp();
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int z = 0; z < 3; ++z) ld_issue(tO + (uint32_t)(NP * y + z * R + r0), o[y][z]);
            ld_issue(tT + at2 * (uint32_t)R + (uint32_t)r0, tr);
            ld_wait();
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int z = 0; z < 3; ++z) pin(o[y][z]);
            pin(tr);
#pragma unroll
            for (int x = 0; x < H; ++x) {
                const int r = r0 + x, gr = s.row0 + r;
                if (r >= r1) break;
                float v[3], acc = 0.f;
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    v[y] = mine[y] > 0 ? ((__uint_as_float(o[y][0][x]) + __uint_as_float(o[y][1][x])) + __uint_as_float(o[y][2][x])) * (kOwnDown * kDown) : 0.f;
                v[2] = s.tree ? __uint_as_float(tr[x]) : 0.f;
#pragma unroll
                for (int y = 0; y < 3; ++y) acc = fmaf(sm.end[g][y][r], v[y], acc);
                if (s.whole) {
                    const int node = a.by_G.of(gr);
                    const __nv_bfloat16 b = __float2bfloat16_rn(acc * sm.end[g][3][r]);
                    reinterpret_cast<__nv_bfloat16 *>(a.out)[((size_t)(s.b * a.N + node) * a.Hq + s.h * a.G + (gr - node * a.G)) * D + t] = b;
                } else {
                    a.part_o[((size_t)slot * R + r) * D + t] = acc;
                }
            }
            // nobody goes on to the next stretch (whose scores, weights and sums use the same places) before all have read
            tc_fence_before();
            if (lane == 0) mbar_arrive(bar(sm.over[at2]));
            both_sync();
            tc_fence_after();
        }
        if (failed) sm.fail = 1;
    }
    // ---- everybody has done: the tensor memory goes back ----
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (tid == 0 && sm.fail != 0) fspad_report(a.status, FSPAD_ERR_TIMEOUT);
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" :: "r"(tmem), "r"(TMEM) : "memory");
    }
}

template <int R> cudaError_t launch_few(fspad_ctx *ctx, Args &a, const Maps &maps, void *workspace, cudaStream_t st)
{
    static_assert(bytes_of<R>() <= 232448, "shared memory of an SM");
    const int ctas = ctx->sm_count;
    a.mtiles = (a.M + R - 1) / R;
    a.by_tiles.set((unsigned)a.mtiles);
    scratch_in<R>(a, ctas, workspace);
    cudaError_t e = raise_shared(ctx, R == 8 ? 4 : 5, reinterpret_cast<const void *>(&tree_attn_fp8_kernel<R>), bytes_of<R>());
    if (e != cudaSuccess) return e;
    const int entries = merge_entries(a, ctas);
    ctx->launches++;
    e = fspad_launch(tree_attn_fp8_kernel<R>, dim3((unsigned)ctas), dim3(NT), bytes_of<R>(), st, 0, a, maps);
    return e == cudaSuccess ? launch_merge<R, true>(ctx, a, entries, ctas, st) : e;
}

}  // namespace

size_t fspad_attn_fp8_umma_workspace(const fspad_ctx *ctx);
cudaError_t fspad_launch_attn_fp8_umma(fspad_ctx *ctx, packed::Args a, const CUtensorMap &k_map, void *workspace, cudaStream_t st);

// (of either kernel, so that a workspace made for one call serves every other: the one with 256 rows a CTA needs the most)
size_t fspad_attn_fp8_workspace(const fspad_ctx *ctx) { return fspad_attn_fp8_umma_workspace(ctx); }

// Whether a call's list (what the beginnings of runs count among it) can be counted in 32 bits, and the rows of a plane of codes in a TMA coordinate.
bool fspad_attn_fp8_fits(const fspad_ctx *ctx, int N, int B, int bps, int n_blocks)
{
    const fspad_config &c = ctx->cfg;
    const long long tiles = ((long long)N * (c.n_q_heads / c.n_kv_heads) + 7) / 8, run = (N + 127) / 128 + (long long)bps + max(kExtra<kManyRows>, kExtra<kFewRows>);
    return (double)run * B * c.n_kv_heads * tiles < 2147483647.0 - 1e6 && (long long)n_blocks * c.n_kv_heads * 128 <= 0x7fffffffll;
}

cudaError_t fspad_launch_tree_attn_fp8(fspad_ctx *ctx, const fspad_bf16 *q, const uint8_t *k_codes, const float *k_scales, const uint8_t *v_codes,
                                       const float *v_scales, FspadPaged paged, const fspad_bf16 *tk, const fspad_bf16 *tv, const int *parent,
                                       const int *prefix_len, int N, int B, fspad_bf16 *out, void *workspace, cudaStream_t st)
{
    const fspad_config &c = ctx->cfg;
    Args a;
    a.q = q; a.kc = k_codes; a.ks = reinterpret_cast<const uint8_t *>(k_scales); a.vc = v_codes; a.vs = reinterpret_cast<const uint8_t *>(v_scales);
    a.table = paged.table; a.table_stride = paged.stride; a.n_blocks = paged.n_blocks;
    a.tk = tk; a.tv = tv; a.parent = parent; a.prefix_len = prefix_len;
    a.N = N; a.B = B; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads;
    a.M = N * a.G;
    a.by_G.set((unsigned)a.G);
    a.scale_log2 = ctx->scale * kLog2e;
    a.out = out; a.status = ctx->d_status;
    Maps maps;
    const size_t rows = (size_t)paged.n_blocks * c.n_kv_heads * 128;
    if (!fspad_make_tmap_u8_2d(&maps.k, k_codes, rows, 128u)) return cudaErrorInvalidValue;
    // Measured on both sides, 8 kv heads, us: 16 rows here and there, 32 sequences of 4 to 12 thousand keys 97 and 160, 16 of 512 to 4096 24 and 46, 64 of 100 to 600 32 and 74.
    // A tile of 32 rows here (192 columns of weights a chunk) took from 17 rows on 157 against 163, but 60 against 47 and 90 against 74: not kept.
    if (a.M > 16) return fspad_launch_attn_fp8_umma(ctx, a, maps.k, workspace, st);
    if (!fspad_make_tmap_u8_2d(&maps.v, v_codes, rows, 128u)) return cudaErrorInvalidValue;
    return a.M <= 8 ? launch_few<8>(ctx, a, maps, workspace, st) : launch_few<16>(ctx, a, maps, workspace, st);
}
