// Tree-masked attention over a cache held in 4 bits ("Preliminaries": the flattened token tree is the target's input and the attention mask
// built from the tree introduces the dependencies between its tokens; one node is the plain single-token step).
//
// For query row i (tree node x head of the group) of sequence b and kv head h:
//   s_j = c q_i . k_j,   out_i = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
// over the L_b cached keys, whose rows are code * scale, and over the node itself and its ancestors among the bf16 tree rows.
//
// Few query rows a kv head (up to 32, in tiles of 16; more: tree_attn_packed_umma.cu).  Every warp takes a part of the list of work (packed_list.cuh) by itself, in units of 32 keys,
// with its own maximum, sum and accumulators; nothing in a CTA waits for anything else of it.
//
// A warp keeps its queries in registers as tensor-core operands (fp16, each row scaled by a power of two, which is exact).  A unit's codes and
// scales come by bulk copies into a ring of the warp's own; they go from shared memory straight into the registers of the operands (no
// second trip through shared memory): the order of the elements within a product and of the keys within a unit is chosen so
// that every lane reads 16 bytes of a row of K, and 8 of a row of V, and finds its operands in them.  The tree's rows are taken as bf16.
//
// What bounds it.  Long contexts: 32 tokens of 64 heads over 8, 4000 to 32000 keys, 139 us with the merge (139 to 153 from one board to another), 645 MB read at
// 4.65 TB/s (72 % of the measured copy rate).  The integer pipe is 59 % busy and 65 % of the issue slots are taken: a unit of 32 keys takes some 660 instructions,
// 140 of them conversions of codes and scales, which each element needs once however few rows there are; 16 warps an SM, with all registers taken, do not hide the
// rest.  Short ones: one token over 2000 keys 8.7 us, of which the two launches, the list and the first trips to memory in turn are the most.
#include <type_traits>

#include "packed_list.cuh"

namespace {

using namespace packed;
using umma::ex2f;
using umma::mbar_expect_tx;
using umma::mbar_init;
using umma::mbar_wait;
using umma::smem_u32;

constexpr int UNIT = 32;                 // keys of a unit
constexpr int BM = 16;                   // query rows of a tile, at most
constexpr int CODES = UNIT * FSPAD_PACKED_CODE_BYTES, SCALES = UNIT * FSPAD_PACKED_SCALE_BYTES;
constexpr int STAGE = 2 * (CODES + SCALES);          // K codes | V codes | K scales | V scales
// With 8 rows a warp does with 128 registers.
__host__ __device__ constexpr int warps_of(int nt) { return nt == 1 ? 16 : 12; }
__host__ __device__ constexpr int stages_of(int nt) { return nt == 1 ? 3 : 4; }
constexpr int MAX_WARPS = 16;

__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16_bf(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Shared loads at a register plus a constant (as operands of the instruction, no additions).
template <int AT> __device__ __forceinline__ uint4 ld16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4 + %5];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at), "n"(AT));
    return v;
}
template <int AT> __device__ __forceinline__ uint2 ld8(uint32_t at)
{
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2 + %3];\n" : "=r"(v.x), "=r"(v.y) : "r"(at), "n"(AT));
    return v;
}
template <int AT> __device__ __forceinline__ uint32_t ld2(uint32_t at)
{
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1 + %2];\n" : "=h"(v) : "r"(at), "n"(AT));
    return v;
}
template <int AT> __device__ __forceinline__ uint32_t ld1(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1 + %2];\n" : "=r"(v) : "r"(at), "n"(AT));
    return v;
}

// f(0), f(1), ... f(N - 1), each with its number as a constant
template <int N, typename F> __device__ __forceinline__ void each(F &&f)
{
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(std::integral_constant<int, N - 1>());
    }
}

// Eight by eight 16-bit values, a row's two in each lane, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
    return y;
}

// Rows 2c and 2c + 1 of eight keys of a product are keys c and 4 + (c ^ 1): rows that the lanes read side by side then begin in
// different halves of the shared memory's 128-byte line.
__device__ __forceinline__ int key_of(int column) { return (column & 1) ? 4 + ((column >> 1) ^ 1) : column >> 1; }

// NT: eights of query rows.  The products stand on their heads: scores S^T [keys][rows] = K Q^T, then O^T [elements][rows] += V^T P^T, so that K and V are the
// operands with 16 rows and no half of an instruction goes to rows that do not exist.
template <int NT>
__global__ void __launch_bounds__(warps_of(NT) * 32, 1)
tree_attn_packed_kernel(const Args a)
{
    constexpr int WARPS = warps_of(NT), STAGES = stages_of(NT);
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) unsigned long long s_bar[WARPS * STAGES];
    __shared__ int s_scan[WARPS + 2 * WARPS];

    const int tid = threadIdx.x, lane = tid & 31, warp = umma::uniform_warp();
    const int g = lane >> 2, c = lane & 3;           // tensor-core operand rows / columns
    const uint32_t bar0 = smem_u32(&s_bar[warp * STAGES]);
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * STAGES * STAGE);
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < STAGES; ++s) mbar_init(bar0 + 8u * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    __syncwarp();
    fspad_pdl_trigger();
    fspad_pdl_wait();

    const int slot0 = warp * gridDim.x + blockIdx.x;
    Parts parts;
    Part part = cut_list<WARPS * 32, UNIT, WARPS>(a, blockIdx.x, gridDim.x * WARPS, parts, s_scan, blockIdx.x == 0);
    if (lane == 0) tell_part<UNIT>(a, parts, part, slot0);
    const int nt = tree_units<UNIT>(a), runs = a.Hkv * a.mtiles;
    // what lanes 0 .. 3 copy of a unit: from which array, of how many bytes a row, to where in the stage
    const uint8_t *part_src = lane == 0 ? a.kc : lane == 1 ? a.vc : lane == 2 ? a.ks : a.vs;
    const uint32_t part_row = lane < 2 ? FSPAD_PACKED_CODE_BYTES : FSPAD_PACKED_SCALE_BYTES;
    const uint32_t part_at = lane < 2 ? lane * CODES : 2 * CODES + (lane - 2) * SCALES;
    const uint32_t lane_k = key_of(g) * 64 + c * 16, lane_ks = 2 * CODES + key_of(g) * 8 + c * 2;
    const uint32_t lane_va = CODES + key_of(2 * c) * 64 + g * 8, lane_vb = CODES + key_of(2 * c + 1) * 64 + g * 8;
    const uint32_t lane_sa = 2 * CODES + SCALES + key_of(2 * c) * 8 + g, lane_sb = 2 * CODES + SCALES + key_of(2 * c + 1) * 8 + g;
    int done = 0;                                    // units of the part so far
    uint32_t n_fill = 0, n_use = 0;                  // stages filled and used so far

#pragma unroll 1
    while (part.left > 0) {
        const int b = part.b, L = prefix_of(a, b, false), n_run = run_units<UNIT>(a, L);
        const int u0 = part.u, u1 = min(n_run, u0 + part.left);
        const int h = a.by_tiles.of(part.run), row0 = (part.run - h * a.mtiles) * BM;
        const int *blocks = a.table + (size_t)b * a.table_stride;

        // ---- the first fills: lanes 0 .. 3 copy K codes, V codes, K scales, V scales; blocks are looked up 32 at a time ----
        const int kv0 = max(u0, nt) - nt, n_kv = max(0, u1 - nt - kv0);      // units of the cache
        int block = 0, looked = -32;                 // of this lane, and lane 0's place in the table
        auto fill = [&](int i) {
            const int key0 = (kv0 + i) * UNIT, page = key0 >> 7;
            if (page >= looked + 32) {
                looked = page;
                block = 0;
                if ((long long)(page + lane) * 128 < L) {
                    block = __ldg(blocks + page + lane);
                    if (block < 0 || block >= a.n_blocks) { fspad_report(a.status, FSPAD_ERR_RANGE); block = 0; }
                }
            }
            const int blk = __shfl_sync(0xffffffffu, block, page - looked);
            const uint32_t st = n_fill % STAGES, bar = bar0 + 8u * st;
            if (lane == 0) mbar_expect_tx(bar, STAGE);
            __syncwarp();
            if (lane < 4) bulk_load(ring + st * STAGE + part_at, part_src + ((size_t)(blk * a.Hkv + h) * 128 + (key0 & 127)) * part_row, part_row * UNIT, bar);
            ++n_fill;
        };
#pragma unroll 1
        for (int i = 0; i < STAGES && i < n_kv; ++i) fill(i);
        if (u0 == 0 && lane == 0) tell_run(a, parts, part, slot0, done, n_run);

        // ---- queries: row g of each eight, elements 32 c .. 32 c + 31, as they are ----
        uint32_t qf[NT][8][2];                       // [eight][product][elements 4 s, 4 s + 1 / 4 s + 2, 4 s + 3 of the lane's 32]
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const int gr = row0 + g + 8 * x, node = a.by_G.of(gr);
            const fspad_bf16 *q = a.q + ((size_t)(b * a.N + node) * a.Hq + h * a.G + (gr - node * a.G)) * D + 32 * c;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 w = gr < a.M ? __ldg(reinterpret_cast<const uint4 *>(q) + i) : make_uint4(0u, 0u, 0u, 0u);
                qf[x][2 * i][0] = w.x; qf[x][2 * i][1] = w.y; qf[x][2 * i + 1][0] = w.z; qf[x][2 * i + 1][1] = w.w;
            }
        }
        float o[NT][8][4];                           // elements 16 g + 2 j (0, 1) and 16 g + 2 j + 1 (2, 3) of rows 2 c and 2 c + 1
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int y = 0; y < 4; ++y) o[x][j][y] = 0.f;
        float m_run[NT][2], l_run[NT][2];            // of rows 2 c, 2 c + 1; the sums of the lane's own keys alone
#pragma unroll
        for (int x = 0; x < NT; ++x) m_run[x][0] = m_run[x][1] = -INFINITY, l_run[x][0] = l_run[x][1] = 0.f;

        // scores (masked; `to_log2` of each row's makes log2 units of them) of 16 T keys -> weights, of the tree's times kDown; the row's reference follows its maximum
        // where that is far ahead of it
        auto softmax = [&](auto &s, const float (&to_log2)[NT][2], auto tiles, auto tree) {
            constexpr int T = decltype(tiles)::value;
            constexpr bool of_tree = decltype(tree)::value;
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int t = 0; t < T; ++t)
#pragma unroll
                    for (int y = 0; y < 2; ++y) mx[y] = fmaxf(fmaxf(mx[y], s[t][x][y]), s[t][x][y + 2]);
#pragma unroll
                for (int off = 4; off < 32; off <<= 1)
#pragma unroll
                    for (int y = 0; y < 2; ++y) mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xffffffffu, mx[y], off));
#pragma unroll
                for (int y = 0; y < 2; ++y) mx[y] *= to_log2[x][y];
                bool move[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) move[y] = mx[y] > m_run[x][y] + kLazyLog2 || (m_run[x][y] == -INFINITY && mx[y] > -INFINITY);
                if (__any_sync(0xffffffffu, move[0] || move[1])) {
                    float alpha[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float m_new = move[y] ? mx[y] : m_run[x][y];
                        alpha[y] = move[y] ? ex2f(m_run[x][y] - m_new) : 1.f;
                        m_run[x][y] = m_new;
                        l_run[x][y] *= alpha[y];
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int y = 0; y < 4; ++y) o[x][j][y] *= alpha[y & 1];
                }
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float bias = of_tree ? -kLazyLog2 : kBiasLog2, ref = m_run[x][y] == -INFINITY ? 0.f : bias - m_run[x][y];
#pragma unroll
                    for (int t = 0; t < T; ++t)
#pragma unroll
                        for (int z = 0; z < 4; z += 2) {
                            const float p = ex2f(fmaf(s[t][x][y + z], to_log2[x][y], ref));
                            s[t][x][y + z] = p;
                            l_run[x][y] = of_tree ? fmaf(p, kUp, l_run[x][y]) : l_run[x][y] + p;
                        }
                }
            }
        };

        // ---- the tree's keys, 16 at a time: bf16 ----
        // Each node's ancestors and itself, a node a lane (no more nodes than rows come here, and those are at most 32), by doubling: after a round a lane has
        // those up to 2^r above, and the node that far up.  (14 nodes, 8 sequences of 32 heads 13.2 -> 11.8 us; with 8 rows, and so nodes, at most, the
        // registers it takes cost more than the walk from node to node: a token over 2000 keys 8.9 us against 8.7.)
        uint32_t above = 1u << lane;
        if (NT > 1 && u0 < nt) {
            int up = -1;
            if (lane < a.N) {
                up = __ldg(a.parent + (size_t)b * a.N + lane);
                if (lane == 0 ? up != -1 : (up < 0 || up >= lane)) { fspad_report(a.status, FSPAD_ERR_BAD_TREE); up = -1; }
            }
#pragma unroll 1
            for (int reach = 1; reach < a.N; reach <<= 1) {
                const uint32_t m = __shfl_sync(0xffffffffu, above, up & 31);
                const int next = __shfl_sync(0xffffffffu, up, up & 31);
                if (up >= 0) { above |= m; up = next; }
            }
        }
        const int t_end = min(a.N, u1 * UNIT);
#pragma unroll 1
        for (int t0 = u0 * UNIT; t0 < t_end; t0 += 16) {
            const size_t first = (((size_t)b * a.Hkv + h) * a.N + t0) * D;
            uint4 kw[2][4], vw[4][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int key = 8 * t + key_of(g);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    kw[t][i] = t0 + key < a.N ? __ldg(reinterpret_cast<const uint4 *>(a.tk + first + key * D + 32 * c) + i) : make_uint4(0u, 0u, 0u, 0u);
            }
            float s[1][NT][4];
#pragma unroll
            for (int x = 0; x < NT; ++x) {
#pragma unroll
                for (int y = 0; y < 4; ++y) s[0][x][y] = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t lo[4] = {kw[0][i].x, kw[1][i].x, kw[0][i].y, kw[1][i].y}, hi[4] = {kw[0][i].z, kw[1][i].z, kw[0][i].w, kw[1][i].w};
                    mma16_bf(s[0][x], lo, qf[x][2 * i][0], qf[x][2 * i][1]);
                    mma16_bf(s[0][x], hi, qf[x][2 * i + 1][0], qf[x][2 * i + 1][1]);
                }
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {            // keys of columns 2c, 2c + 1, 2c + 8, 2c + 9: elements 16 g .. 16 g + 15
                const int key = 8 * (y >> 1) + key_of(2 * c + (y & 1));
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    vw[y][i] = t0 + key < a.N ? __ldg(reinterpret_cast<const uint4 *>(a.tv + first + key * D + 16 * g) + i) : make_uint4(0u, 0u, 0u, 0u);
            }
            uint32_t see[NT][2];                     // which of the 16 keys rows 2 c, 2 c + 1 see
#pragma unroll
            for (int x = 0; x < NT; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int gr = row0 + 8 * x + 2 * c + y;
                    if constexpr (NT > 1) {
                        const uint32_t all = __shfl_sync(0xffffffffu, above, a.by_G.of(gr) & 31);
                        see[x][y] = gr < a.M ? (all >> t0) & 0xffffu : 0u;
                    } else {                         // (t0 = 0)
                        see[x][y] = 0u;
                        int at = gr < a.M ? a.by_G.of(gr) : -1;
                        while (at >= 0) {
                            see[x][y] |= 1u << at;
                            const int up = __ldg(a.parent + (size_t)b * a.N + at);
                            if (at == 0 ? up != -1 : (up < 0 || up >= at)) { fspad_report(a.status, FSPAD_ERR_BAD_TREE); break; }
                            at = up;
                        }
                    }
#pragma unroll
                    for (int z = 0; z < 4; z += 2) s[0][x][y + z] = (see[x][y] >> (4 * z + key_of(g))) & 1u ? s[0][x][y + z] : -INFINITY;
                }
            float plain[NT][2];
#pragma unroll
            for (int x = 0; x < NT; ++x) plain[x][0] = plain[x][1] = a.scale_log2;
            softmax(s, plain, std::integral_constant<int, 1>(), std::true_type());
            // A row of V with an infinity or a NaN in it must not reach the queries that do not see it (0 times it is a NaN): it is taken
            // out of the product, and the queries that do see it get NaN.
            uint32_t keys = 0;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const uint4 w0 = vw[y][0], w1 = vw[y][1];
                if (odd_value(w0.x) || odd_value(w0.y) || odd_value(w0.z) || odd_value(w0.w) || odd_value(w1.x) || odd_value(w1.y) || odd_value(w1.z) || odd_value(w1.w)) {
                    keys |= 1u << (8 * (y >> 1) + key_of(2 * c + (y & 1)));
                    vw[y][0] = vw[y][1] = make_uint4(0u, 0u, 0u, 0u);
                }
            }
            keys = __reduce_or_sync(0xffffffffu, keys);
#pragma unroll
            for (int x = 0; x < NT; ++x) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    if (see[x][y] & keys) l_run[x][y] = NAN;
                const uint32_t p0 = transpose8(umma::pack_bf16(s[0][x][0], s[0][x][1])), p1 = transpose8(umma::pack_bf16(s[0][x][2], s[0][x][3]));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    auto word = [&](int y) {
                        const uint4 w = vw[y][j >> 2];
                        return (j & 3) == 0 ? w.x : (j & 3) == 1 ? w.y : (j & 3) == 2 ? w.z : w.w;
                    };
                    const uint32_t v[4] = {__byte_perm(word(0), word(1), 0x5410), __byte_perm(word(0), word(1), 0x7632),
                                           __byte_perm(word(2), word(3), 0x5410), __byte_perm(word(2), word(3), 0x7632)};
                    mma16_bf(o[x][j], v, p0, p1);
                }
            }
        }

        // ---- queries as fp16, scaled by a power of two so that the row's largest magnitude lies in [2^14, 2^15): 8 significant bits
        // stay exact down to 2^-31 of the largest ----
        float cs[NT][2];                             // scores -> log2 units, of rows 2 c, 2 c + 1
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fspad_most2(m, fspad_most2(qf[x][i][0], qf[x][i][1]));
            m = fspad_most2(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fspad_most2(m, __shfl_xor_sync(0xffffffffu, m, 2));
            m = max(m & 0xffffu, m >> 16);
            // the largest magnitude is in [2^e, 2^(e+1)); of zeros, and of rows that are not finite (whose result is not either), as it is
            const int e = m == 0u || m >= 0x7f80u ? 14 : max((int)(m >> 7) - 127, -100);
            const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
#pragma unroll
            for (int y = 0; y < 2; ++y) cs[x][y] = a.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + __shfl_sync(0xffffffffu, e, 4 * (2 * c + y))) << 23);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    qf[x][i][y] = pack_f16(__uint_as_float(qf[x][i][y] << 16) * up, __uint_as_float(qf[x][i][y] & 0xffff0000u) * up);
        }

        // ---- units of the cache ----
        bool failed = false;
#pragma unroll 1
        for (int i = 0; i < n_kv; ++i) {
            const uint32_t st = n_use % STAGES, at = ring + st * STAGE;
            if (!mbar_wait(bar0 + 8u * st, (n_use / STAGES) & 1u)) {
                failed = true;
                break;
            }
            ++n_use;
            const int left = L - (kv0 + i) * UNIT;   // keys of the unit that exist
            // the lane's places: its row of K, its scales; the rows of V of columns 2 c and 2 c + 1, their scales
            const uint32_t at_k = at + lane_k, at_ks = at + lane_ks, at_va = at + lane_va, at_vb = at + lane_vb, at_sa = at + lane_sa, at_sb = at + lane_sb;
            float s[2][NT][4];
            each<2>([&](auto t_) {
                constexpr int t = decltype(t_)::value;
                uint4 w[2] = {ld16<t * 1024>(at_k), ld16<t * 1024 + 512>(at_k)};
                uint32_t sc[2] = {fspad_e4m3_to_f16(ld2<t * 128>(at_ks)), fspad_e4m3_to_f16(ld2<t * 128 + 64>(at_ks))};
#pragma unroll
                for (int x = 0; x < NT; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) s[t][x][y] = 0.f;
#pragma unroll
                for (int i2 = 0; i2 < 4; ++i2) {
                    uint32_t f[2][4];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint32_t word = i2 == 0 ? w[y].x : i2 == 1 ? w[y].y : i2 == 2 ? w[y].z : w[y].w, s2 = __byte_perm(sc[y], sc[y], i2 < 2 ? 0x1010 : 0x3232);
                        fspad_e2m1_to_f16(word, f[y]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) f[y][j] = fspad_hmul2(f[y][j], s2);
                    }
                    const uint32_t lo[4] = {f[0][0], f[1][0], f[0][1], f[1][1]}, hi[4] = {f[0][2], f[1][2], f[0][3], f[1][3]};
#pragma unroll
                    for (int x = 0; x < NT; ++x) {
                        mma16(s[t][x], lo, qf[x][2 * i2][0], qf[x][2 * i2][1]);
                        mma16(s[t][x], hi, qf[x][2 * i2 + 1][0], qf[x][2 * i2 + 1][1]);
                    }
                }
            });
            if (left < UNIT) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (16 * t + 4 * (y & 2) + key_of(g) >= left)
#pragma unroll
                            for (int x = 0; x < NT; ++x) s[t][x][y] = -INFINITY;
            }
            uint32_t scv[2][2];                      // scales of V, times kDown, of columns 2c.. and 2c + 8.. of the two sixteens of keys
            auto scales_v = [&](auto t_) {
                constexpr int t = decltype(t_)::value;
                uint32_t sa[2] = {ld1<t * 128>(at_sa), ld1<t * 128 + 64>(at_sa)}, sb[2] = {ld1<t * 128>(at_sb), ld1<t * 128 + 64>(at_sb)};
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    // what lies behind the sequence's end may be anything, and 0 times a NaN is one: its scale is zero
                    if (left < UNIT) {
                        if (16 * t + 8 * y + key_of(2 * c) >= left) sa[y] = 0u;
                        if (16 * t + 8 * y + key_of(2 * c + 1) >= left) sb[y] = 0u;
                    }
                    scv[t][y] = fspad_hmul2(fspad_e4m3_to_f16(sb[y] * 256u + sa[y]), kDown2);
                }
            };
            // (of two eights of rows ahead of the exponentials: 24 rows, 32 sequences of 12000 keys 8 kv heads 271 -> 266 us; of one eight there they cost 1.5 %)
            if constexpr (NT > 1) each<2>(scales_v);
            softmax(s, cs, std::integral_constant<int, 2>(), std::false_type());
            each<2>([&](auto t_) {
                constexpr int t = decltype(t_)::value;
                uint32_t p[NT][2];
#pragma unroll
                for (int x = 0; x < NT; ++x) {
                    p[x][0] = transpose8(pack_f16(s[t][x][0], s[t][x][1]));
                    p[x][1] = transpose8(pack_f16(s[t][x][2], s[t][x][3]));
                }
                const uint2 w[4] = {ld8<t * 1024>(at_va), ld8<t * 1024>(at_vb), ld8<t * 1024 + 512>(at_va), ld8<t * 1024 + 512>(at_vb)};
                if constexpr (NT == 1) scales_v(t_);
#pragma unroll
                for (int i2 = 0; i2 < 2; ++i2) {     // elements 16 g + 8 i2 ..
                    uint32_t f[2][2][4];             // [columns 2c.. / 2c + 8..][even / odd elements][pair of keys of element 2 j (+ 1)]
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint32_t wa = i2 ? w[2 * y].y : w[2 * y].x, wb = i2 ? w[2 * y + 1].y : w[2 * y + 1].x;
                        fspad_e2m1_to_f16((wa & 0x0f0f0f0fu) | ((wb << 4) & 0xf0f0f0f0u), f[y][0]);
                        fspad_e2m1_to_f16(((wa >> 4) & 0x0f0f0f0fu) | (wb & 0xf0f0f0f0u), f[y][1]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            f[y][0][j] = fspad_hmul2(f[y][0][j], scv[t][y]);
                            f[y][1][j] = fspad_hmul2(f[y][1][j], scv[t][y]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t v[4] = {f[0][0][j], f[0][1][j], f[1][0][j], f[1][1][j]};
#pragma unroll
                        for (int x = 0; x < NT; ++x) mma16(o[x][4 * i2 + j], v, p[x][0], p[x][1]);
                    }
                }
            });
            __syncwarp();                            // every lane has read the stage
            if (i + STAGES < n_kv) fill(i + STAGES);
        }
        if (failed) {
            // what is under way gets another bounded time to land before the warp leaves
            for (; n_use < n_fill; ++n_use) (void)mbar_wait(bar0 + 8u * (n_use % STAGES), (n_use / STAGES) & 1u);
            if (lane == 0) fspad_report(a.status, FSPAD_ERR_TIMEOUT);
            return;
        }

        // ---- the rows: of rows 2 c and 2 c + 1 the lane has elements 16 g .. 16 g + 15 ----
        const bool whole = u0 == 0 && u1 == n_run;
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float l = l_run[x][y];
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
                const int r = 8 * x + 2 * c + y, gr = row0 + r;
                if (gr >= a.M) continue;
                if (whole) {
                    const int node = a.by_G.of(gr);
                    const float inv = kUp / l;
                    uint4 *dst = reinterpret_cast<uint4 *>(a.out + ((size_t)(b * a.N + node) * a.Hq + h * a.G + (gr - node * a.G)) * D + 16 * g);
#pragma unroll
                    for (int j = 0; j < 8; j += 4)
                        dst[j / 4] = make_uint4(umma::pack_bf16(o[x][j][y] * inv, o[x][j][y + 2] * inv), umma::pack_bf16(o[x][j + 1][y] * inv, o[x][j + 1][y + 2] * inv),
                                                umma::pack_bf16(o[x][j + 2][y] * inv, o[x][j + 2][y + 2] * inv), umma::pack_bf16(o[x][j + 3][y] * inv, o[x][j + 3][y + 2] * inv));
                } else {
                    const size_t slot = ((size_t)slot0 * 2 + (u0 == 0 ? 1 : 0)) * BM + r;
                    float4 *dst = reinterpret_cast<float4 *>(a.part_o + slot * D + 16 * g);
#pragma unroll
                    for (int j = 0; j < 8; j += 2) dst[j / 2] = make_float4(o[x][j][y], o[x][j][y + 2], o[x][j + 1][y], o[x][j + 1][y + 2]);
                    if (g == 0) a.part_ml[slot] = make_float2(m_run[x][y], l);
                }
            }
        done += u1 - u0;
        part.left -= u1 - u0;
        part.u = 0;
        if (++part.run == runs) { part.run = 0; ++part.b; }
    }
}

template <int NT> cudaError_t launch_few(fspad_ctx *ctx, Args &a, cudaStream_t st)
{
    const int ctas = ctx->sm_count, smem = warps_of(NT) * stages_of(NT) * STAGE;
    cudaError_t e = raise_shared(ctx, NT, reinterpret_cast<const void *>(&tree_attn_packed_kernel<NT>), smem);
    if (e != cudaSuccess) return e;
    const int entries = merge_entries(a, ctas * warps_of(NT));
    ctx->launches++;
    e = fspad_launch(tree_attn_packed_kernel<NT>, dim3((unsigned)ctas), dim3(warps_of(NT) * 32), smem, st, 0, a);
    return e == cudaSuccess ? launch_merge<BM>(ctx, a, entries, ctas * warps_of(NT), st) : e;
}

}  // namespace

// Which of the two kernels takes a call.  Up to 32 query rows a kv head this one does (above 16 in two tiles, each of which takes the cache's codes apart for itself):
// the other's fixed costs are for 128 rows, and paid for every (sequence, kv head).  us, this kernel and the other, 20 to 32 rows: one sequence of 8 kv heads, 300 to
// 4000 keys 11 - 15 and 13 - 16, thirty-two of 1500 54 - 56 and 65, twenty nodes of sixteen sequences, 32 heads and 300 keys 42 and 62; but sixteen of 8 heads
// and 1500 keys 30 - 32 and 29, thirty-two of 4000 to 12000 186 and 182, of 12000 265 - 268 and 245.  A tree of more than 24 nodes without shared heads has keys of
// its own besides: 32 nodes, 8 heads, one sequence of 300 keys 12.2 and 13.8, of 4000 16.5 and 16.3, four 13.4 and 14.3, 27.1 and 26.2, but thirty-two 26 and 37, 111 and
// 110: the line by the number of runs gives a long cache's few per cent for a short one's.  48 rows: 32 heads, sixteen of 1500 keys 120 and 103, of 300 61 and 63.
static bool many_rows(const fspad_ctx *ctx, int N, int B)
{
    const fspad_config &c = ctx->cfg;
    const long long M = (long long)N * (c.n_q_heads / c.n_kv_heads);
    return M > 32 || (M > 16 && N > 24 && (long long)B * c.n_kv_heads <= ctx->sm_count);
}

size_t fspad_attn_packed_workspace(const fspad_ctx *ctx, int N, int B)
{
    // of either kernel, so that a workspace made for one call serves every other
    (void)N; (void)B;
    const size_t few = scratch_bytes<BM>(ctx->sm_count * MAX_WARPS), many = fspad_attn_packed_umma_workspace(ctx);
    return few > many ? few : many;
}

// Whether a call's list can be counted in 32 bits.
bool fspad_attn_packed_fits(const fspad_ctx *ctx, int N, int B, int bps)
{
    const fspad_config &c = ctx->cfg;
    Args a;
    a.N = N; a.B = B; a.Hkv = c.n_kv_heads; a.M = N * (c.n_q_heads / c.n_kv_heads); a.mtiles = (a.M + BM - 1) / BM; a.table_stride = bps;
    return units_fit<UNIT>(a);
}

cudaError_t fspad_launch_tree_attn_packed(fspad_ctx *ctx, const fspad_bf16 *q, const uint8_t *k_codes, const uint8_t *k_scales,
                                          const uint8_t *v_codes, const uint8_t *v_scales, FspadPaged paged, const fspad_bf16 *tk,
                                          const fspad_bf16 *tv, const int *parent, const int *prefix_len, int N, int B,
                                          fspad_bf16 *out, void *workspace, cudaStream_t st)
{
    const fspad_config &c = ctx->cfg;
    Args a;
    a.q = q; a.kc = k_codes; a.ks = k_scales; a.vc = v_codes; a.vs = v_scales;
    a.table = paged.table; a.table_stride = paged.stride; a.n_blocks = paged.n_blocks;
    a.tk = tk; a.tv = tv; a.parent = parent; a.prefix_len = prefix_len;
    a.N = N; a.B = B; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads;
    a.M = N * a.G; a.mtiles = (a.M + BM - 1) / BM;
    a.by_G.set((unsigned)a.G); a.by_tiles.set((unsigned)a.mtiles);
    a.scale_log2 = ctx->scale * kLog2e;
    a.out = out; a.status = ctx->d_status;
    if (many_rows(ctx, N, B)) return fspad_launch_attn_packed_umma(ctx, a, workspace, st);
    scratch_in<BM>(a, ctx->sm_count * MAX_WARPS, workspace);
    return a.M <= 8 ? launch_few<1>(ctx, a, st) : launch_few<2>(ctx, a, st);
}
