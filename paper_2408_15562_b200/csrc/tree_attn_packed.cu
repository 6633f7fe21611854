// Tree-masked attention over a cache held in 4 bits ("Preliminaries": the flattened token tree is the target's input and the attention mask
// built from the tree introduces the dependencies between its tokens; one node is the plain single-token step).
//
// For query row i (tree node x head of the group) of sequence b and kv head h:
//   s_j = c q_i . k_j,   out_i = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
// over the L_b cached keys, whose rows are code * scale, and over the node itself and its ancestors among the bf16 tree rows.
//
// Few query rows a kv head (up to 16; more: tree_attn_packed_umma.cu).  Every warp takes a part of the list of work (packed_list.cuh) by itself, in units of 32 keys,
// with its own maximum, sum and accumulators; nothing in a CTA waits for anything else of it.
//
// A warp keeps its queries in registers as tensor-core operands (fp16, each row scaled by a power of two, which is exact).  A unit's codes and
// scales come by bulk copies into a ring of the warp's own; they go from shared memory straight into the registers of the operands (no
// second trip through shared memory): the order of the elements within a product and of the keys within a unit is chosen so
// that every lane reads 16 bytes of a row of K, and 8 of a row of V, and finds its operands in them.  The tree's rows are taken as bf16.
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
constexpr int BM = 16;                   // query rows of a tile
constexpr int WARPS = 12;
constexpr int STAGES = 4;
constexpr int CODES = UNIT * FSPAD_PACKED_CODE_BYTES, SCALES = UNIT * FSPAD_PACKED_SCALE_BYTES;
constexpr int STAGE = 2 * (CODES + SCALES);          // K codes | V codes | K scales | V scales
constexpr int SMEM = WARPS * STAGES * STAGE;

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
__device__ __forceinline__ uint4 ld16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 ld8(uint32_t at)
{
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];\n" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
__device__ __forceinline__ uint32_t ld2(uint32_t at)
{
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ uint32_t ld1(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];\n" : "=r"(v) : "r"(at));
    return v;
}
// Columns 2c and 2c + 1 of a product's tile of eight keys are keys c and 4 + (c ^ 1): rows that the lanes read side by side then begin in
// different halves of the shared memory's 128-byte line.
__device__ __forceinline__ int key_of(int column) { return (column & 1) ? 4 + ((column >> 1) ^ 1) : column >> 1; }

// WIDE: tiles may have more than 8 rows.
template <bool WIDE>
__global__ void __launch_bounds__(WARPS * 32, 1)
tree_attn_packed_kernel(const Args a)
{
    constexpr int NX = WIDE ? 2 : 1;
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

    const int slot0 = blockIdx.x * WARPS + warp;
    Parts parts;
    Part part = cut_list<WARPS * 32, UNIT, WARPS>(a, blockIdx.x * WARPS, gridDim.x * WARPS, parts, s_scan, blockIdx.x == 0);
    if (lane == 0) tell_cut<UNIT>(a, parts, part, slot0);
    const int nt = tree_units<UNIT>(a), runs = a.Hkv * a.mtiles;
    uint32_t n_fill = 0, n_use = 0;                  // stages filled and used so far

#pragma unroll 1
    while (part.left > 0) {
        const int b = part.b, L = prefix_of(a, b, false), n_run = run_units<UNIT>(a, L);
        const int u0 = part.u, u1 = min(n_run, u0 + part.left);
        const int h = a.by_tiles.of(part.run), row0 = (part.run - h * a.mtiles) * BM;
        const int *blocks = a.table + (size_t)b * a.table_stride;

        // ---- the first fills ----
        const int kv0 = max(u0, nt) - nt, n_kv = max(0, u1 - nt - kv0);      // units of the cache
        auto fill = [&](int i) {                     // lane 0
            const int key0 = (kv0 + i) * UNIT;
            int blk = __ldg(blocks + (key0 >> 7));
            if (blk < 0 || blk >= a.n_blocks) { fspad_report(a.status, FSPAD_ERR_RANGE); blk = 0; }
            const size_t row = ((size_t)blk * a.Hkv + h) * 128 + (key0 & 127);
            const uint32_t st = n_fill % STAGES, to = ring + st * STAGE, bar = bar0 + 8u * st;
            mbar_expect_tx(bar, STAGE);
            bulk_load(to, a.kc + row * FSPAD_PACKED_CODE_BYTES, CODES, bar);
            bulk_load(to + 2 * CODES, a.ks + row * FSPAD_PACKED_SCALE_BYTES, SCALES, bar);
            bulk_load(to + CODES, a.vc + row * FSPAD_PACKED_CODE_BYTES, CODES, bar);
            bulk_load(to + 2 * CODES + SCALES, a.vs + row * FSPAD_PACKED_SCALE_BYTES, SCALES, bar);
        };
#pragma unroll 1
        for (int i = 0; i < STAGES && i < n_kv; ++i) {
            if (lane == 0) fill(i);
            ++n_fill;
        }

        // ---- queries: rows g and g + 8 of the tile, elements 32 c .. 32 c + 31, as they are ----
        uint32_t qf[8][4];                           // [product][a0, a1 (row + 8), a2 (column + 8), a3]
        int node[2], to_row[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int gr = row0 + g + 8 * x;
            const bool there = (WIDE || x == 0) && gr < a.M;
            node[x] = there ? a.by_G.of(gr) : -1;
            to_row[x] = there ? (b * a.N + node[x]) * a.Hq + h * a.G + (gr - node[x] * a.G) : -1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {            // pair 4 i + j of 16: product 2 i + j / 2, its columns 2c (j even) or 2c + 8
                const uint4 w = there ? __ldg(reinterpret_cast<const uint4 *>(a.q + (size_t)to_row[x] * D + 32 * c) + i) : make_uint4(0u, 0u, 0u, 0u);
                qf[2 * i][x] = w.x; qf[2 * i][x + 2] = w.y; qf[2 * i + 1][x] = w.z; qf[2 * i + 1][x + 2] = w.w;
            }
        }
        float o[16][4];
#pragma unroll
        for (int j = 0; j < 16; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[j][x] = 0.f;
        float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};

        // scores (log2 units, masked) of 8 T keys -> weights; the row's reference follows its maximum where that is far ahead of it
        auto softmax = [&](auto &s, auto tiles) {
            constexpr int T = decltype(tiles)::value;
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                float mx = -INFINITY;
#pragma unroll
                for (int t = 0; t < T; ++t) mx = fmaxf(fmaxf(mx, s[t][2 * x]), s[t][2 * x + 1]);
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                const bool move = mx > m_run[x] + kLazyLog2 || (m_run[x] == -INFINITY && mx > -INFINITY);
                if (__any_sync(0xffffffffu, move)) {
                    const float m_new = move ? mx : m_run[x];
                    const float alpha = move ? ex2f(m_run[x] - m_new) : 1.f;
                    m_run[x] = m_new;
                    l_run[x] *= alpha;
#pragma unroll
                    for (int j = 0; j < 16; ++j) { o[j][2 * x] *= alpha; o[j][2 * x + 1] *= alpha; }
                }
                const float ref = m_run[x] == -INFINITY ? 0.f : m_run[x] - kBiasLog2;
#pragma unroll
                for (int t = 0; t < T; ++t)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float p = ex2f(s[t][2 * x + y] - ref);
                        s[t][2 * x + y] = p;
                        l_run[x] += p;
                    }
            }
        };

        // ---- the tree's keys, 16 at a time: bf16 ----
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
#pragma unroll
            for (int y = 0; y < 4; ++y) {            // keys of columns 2c, 2c + 1, 2c + 8, 2c + 9: elements 16 g .. 16 g + 15
                const int key = 8 * (y >> 1) + key_of(2 * c + (y & 1));
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    vw[y][i] = t0 + key < a.N ? __ldg(reinterpret_cast<const uint4 *>(a.tv + first + key * D + 16 * g) + i) : make_uint4(0u, 0u, 0u, 0u);
            }
            uint32_t see[2] = {0u, 0u};              // which of the 16 keys a row sees
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                int at = node[x];
                while (at >= t0) {
                    if (at < t0 + 16) see[x] |= 1u << (at - t0);
                    const int up = __ldg(a.parent + (size_t)b * a.N + at);
                    if (at == 0 ? up != -1 : (up < 0 || up >= at)) { fspad_report(a.status, FSPAD_ERR_BAD_TREE); break; }
                    at = up;
                }
            }
            float s[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int x = 0; x < 4; ++x) s[t][x] = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mma16_bf(s[t], qf[2 * i], kw[t][i].x, kw[t][i].y);
                    mma16_bf(s[t], qf[2 * i + 1], kw[t][i].z, kw[t][i].w);
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) s[t][x] = (see[x >> 1] >> (8 * t + key_of(2 * c + (x & 1)))) & 1u ? s[t][x] * a.scale_log2 : -INFINITY;
            }
            softmax(s, std::integral_constant<int, 2>());
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
            for (int x = 0; x < NX; ++x)
                if (see[x] & keys) l_run[x] = NAN;
            const uint32_t p[4] = {umma::pack_bf16(s[0][0], s[0][1]), WIDE ? umma::pack_bf16(s[0][2], s[0][3]) : 0u,
                                   umma::pack_bf16(s[1][0], s[1][1]), WIDE ? umma::pack_bf16(s[1][2], s[1][3]) : 0u};
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
                auto word = [&](int y) {
                    const uint4 w = vw[y][j >> 3];
                    return ((j >> 1) & 3) == 0 ? w.x : ((j >> 1) & 3) == 1 ? w.y : ((j >> 1) & 3) == 2 ? w.z : w.w;
                };
                mma16_bf(o[j], p, __byte_perm(word(0), word(1), sel), __byte_perm(word(2), word(3), sel));
            }
        }

        // ---- queries as fp16, scaled by a power of two so that the row's largest magnitude lies in [2^14, 2^15): 8 significant bits
        // stay exact down to 2^-31 of the largest ----
        float cs[2] = {0.f, 0.f};                    // scores -> log2 units
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fspad_most2(m, fspad_most2(qf[i][x], qf[i][x + 2]));
            m = fspad_most2(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fspad_most2(m, __shfl_xor_sync(0xffffffffu, m, 2));
            m = max(m & 0xffffu, m >> 16);
            // the largest magnitude is in [2^e, 2^(e+1)); of zeros, and of rows that are not finite (whose result is not either), as it is
            const int e = m == 0u || m >= 0x7f80u ? 14 : max((int)(m >> 7) - 127, -100);
            const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
            cs[x] = a.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int y = 0; y < 4; y += 2)
                    qf[i][x + y] = pack_f16(__uint_as_float(qf[i][x + y] << 16) * up, __uint_as_float(qf[i][x + y] & 0xffff0000u) * up);
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
            float s[4][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int key = 8 * t + key_of(g);
                const uint4 w = ld16(at + (uint32_t)(key * 64 + c * 16));
                const uint32_t sc = fspad_e4m3_to_f16(ld2(at + 2 * CODES + (uint32_t)(key * 8 + c * 2)));
                const uint32_t s0 = __byte_perm(sc, sc, 0x1010), s1 = __byte_perm(sc, sc, 0x3232);
                const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) s[t][x] = 0.f;
#pragma unroll
                for (int i2 = 0; i2 < 4; ++i2) {
                    uint32_t f[4];
                    fspad_e2m1_to_f16(ws[i2], f);
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = fspad_hmul2(f[j], i2 < 2 ? s0 : s1);
                    mma16(s[t], qf[2 * i2], f[0], f[1]);
                    mma16(s[t], qf[2 * i2 + 1], f[2], f[3]);
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int x = 0; x < 2 * NX; ++x) s[t][x] *= cs[x >> 1];
            if (left < UNIT) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (8 * t + key_of(2 * c + (x & 1)) >= left) s[t][x] = -INFINITY;
            }
            softmax(s, std::integral_constant<int, 4>());
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2) {
                const uint32_t p[4] = {pack_f16(s[2 * k2][0], s[2 * k2][1]), WIDE ? pack_f16(s[2 * k2][2], s[2 * k2][3]) : 0u,
                                       pack_f16(s[2 * k2 + 1][0], s[2 * k2 + 1][1]), WIDE ? pack_f16(s[2 * k2 + 1][2], s[2 * k2 + 1][3]) : 0u};
                uint2 w[4];
                uint32_t sc[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int ka = 16 * k2 + 8 * y + key_of(2 * c), kb = 16 * k2 + 8 * y + key_of(2 * c + 1);
                    w[2 * y] = ld8(at + CODES + (uint32_t)(ka * 64 + g * 8));
                    w[2 * y + 1] = ld8(at + CODES + (uint32_t)(kb * 64 + g * 8));
                    uint32_t sa = ld1(at + 2 * CODES + SCALES + (uint32_t)(ka * 8 + g)), sb = ld1(at + 2 * CODES + SCALES + (uint32_t)(kb * 8 + g));
                    // what lies behind the sequence's end may be anything, and 0 times a NaN is one: its scale is zero
                    if (ka >= left) sa = 0u;
                    if (kb >= left) sb = 0u;
                    sc[y] = fspad_e4m3_to_f16(sa | (sb << 8));
                }
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
                            f[y][0][j] = fspad_hmul2(f[y][0][j], sc[y]);
                            f[y][1][j] = fspad_hmul2(f[y][1][j], sc[y]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        mma16(o[8 * i2 + 2 * j], p, f[0][0][j], f[1][0][j]);
                        mma16(o[8 * i2 + 2 * j + 1], p, f[0][1][j], f[1][1][j]);
                    }
                }
            }
            __syncwarp();                            // every lane has read the stage
            if (i + STAGES < n_kv) {
                if (lane == 0) fill(i + STAGES);
                ++n_fill;
            }
        }
        if (failed) {
            // what is under way gets another bounded time to land before the warp leaves
            for (; n_use < n_fill; ++n_use) (void)mbar_wait(bar0 + 8u * (n_use % STAGES), (n_use / STAGES) & 1u);
            if (lane == 0) fspad_report(a.status, FSPAD_ERR_TIMEOUT);
            return;
        }

        // ---- the rows: lane (g, c) has elements 32 c + j in o[j][2 x], 32 c + 16 + j in o[j][2 x + 1] ----
        const bool whole = u0 == 0 && u1 == n_run;
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            l_run[x] += __shfl_xor_sync(0xffffffffu, l_run[x], 1);
            l_run[x] += __shfl_xor_sync(0xffffffffu, l_run[x], 2);
            if (node[x] < 0) continue;
            if (whole) {
                const float inv = 1.f / l_run[x];
                uint4 *dst = reinterpret_cast<uint4 *>(a.out + (size_t)to_row[x] * D + 32 * c);
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int j = 0; j < 16; j += 8)
                        dst[2 * y + j / 8] = make_uint4(umma::pack_bf16(o[j][2 * x + y] * inv, o[j + 1][2 * x + y] * inv), umma::pack_bf16(o[j + 2][2 * x + y] * inv, o[j + 3][2 * x + y] * inv),
                                                        umma::pack_bf16(o[j + 4][2 * x + y] * inv, o[j + 5][2 * x + y] * inv), umma::pack_bf16(o[j + 6][2 * x + y] * inv, o[j + 7][2 * x + y] * inv));
            } else {
                const size_t slot = ((size_t)slot0 * 2 + (u0 == 0 ? 1 : 0)) * BM + g + 8 * x;
                float4 *dst = reinterpret_cast<float4 *>(a.part_o + slot * D + 32 * c);
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int j = 0; j < 16; j += 4) dst[4 * y + j / 4] = make_float4(o[j][2 * x + y], o[j + 1][2 * x + y], o[j + 2][2 * x + y], o[j + 3][2 * x + y]);
                if (c == 0) a.part_ml[slot] = make_float2(m_run[x], l_run[x]);
            }
        }
        part.left -= u1 - u0;
        part.u = 0;
        if (++part.run == runs) { part.run = 0; ++part.b; }
    }
}

}  // namespace

// Which of the two kernels takes a call, by the query rows of a kv head.
static bool many_rows(const fspad_ctx *ctx, int N) { return (long long)N * (ctx->cfg.n_q_heads / ctx->cfg.n_kv_heads) > BM; }

size_t fspad_attn_packed_workspace(const fspad_ctx *ctx, int N, int B)
{
    (void)B;
    if (many_rows(ctx, N)) return fspad_attn_packed_umma_workspace(ctx);
    return scratch_bytes<BM>(ctx->sm_count * WARPS);
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
    if (many_rows(ctx, N)) return fspad_launch_attn_packed_umma(ctx, a, workspace, st);
    const int ctas = ctx->sm_count;
    scratch_in<BM>(a, ctas * WARPS, workspace);
    auto kernel = a.M > 8 ? tree_attn_packed_kernel<true> : tree_attn_packed_kernel<false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    ctx->launches += 2;
    e = fspad_launch(kernel, dim3((unsigned)ctas), dim3(WARPS * 32), SMEM, st, 0, a);
    if (e != cudaSuccess) return e;
    int rows = 1;
    while (rows < a.M && rows < BM) rows *= 2;
    return fspad_launch(tree_attn_packed_merge_kernel<BM, 16>, dim3((unsigned)(ctas * WARPS)), dim3(512), 0, st, 0, a, rows);
}
