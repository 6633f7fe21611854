// Tree-masked attention over a cache held in 4 bits ("Preliminaries": the flattened token tree is the target's input and the attention mask
// built from the tree introduces the dependencies between its tokens; one node is the plain single-token step).
//
// For query row i (tree node x head of the group) of sequence b and kv head h:
//   s_j = c q_i . k_j,   out_i = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
// over the L_b cached keys, whose rows are code * scale, and over the node itself and its ancestors among the bf16 tree rows.
//
// The work is one list: for every sequence, kv head and tile of 16 query rows a run of units of 32 keys, the tree's first.  Every CTA takes an
// equal part of the list wherever the cuts fall, so that ragged lengths and any number of sequences fill the SMs alike; a run that
// was cut leaves a partial (maximum, sum, unnormalised row) for each piece, which a second kernel merges.  A CTA's eight warps take the units of a
// run in turn, each with its own maximum, sum and accumulators, and meet at the run's end.
//
// A warp keeps its queries in registers as tensor-core operands (fp16, each row scaled by a power of two, which is exact).  A unit's codes and
// scales come by bulk copies into a ring of the warp's own; they go from shared memory straight into the registers of the operands (no
// second trip through shared memory): the order of the elements within a product and of the keys within a unit is chosen so
// that every lane reads 16 bytes of a row of K, and 8 of a row of V, and finds its operands in them.  The tree's rows are taken as bf16.
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
constexpr int WARPS = 8;
constexpr int STAGES = 3;
constexpr int CODES = UNIT * FSPAD_PACKED_CODE_BYTES, SCALES = UNIT * FSPAD_PACKED_SCALE_BYTES;
constexpr int STAGE = 2 * (CODES + SCALES);          // K codes | V codes | K scales | V scales
constexpr int OROW = 4 * 36;             // floats of a staged row of 128: runs of 32 with a gap of 4, so that 16-byte stores do not collide
constexpr int SMEM = WARPS * STAGES * STAGE + WARPS * BM * OROW * 4;

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

__global__ void __launch_bounds__(WARPS * 32, 1)
tree_attn_packed_kernel(const Args a)
{
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) unsigned long long s_bar[WARPS * STAGES];
    __shared__ int s_scan[WARPS + 2];
    __shared__ short s_par[FSPAD_MAX_NODES_WIDE];
    __shared__ float2 s_ml[WARPS][BM];
    __shared__ int s_fail;

    const int tid = threadIdx.x, lane = tid & 31, warp = umma::uniform_warp();
    const int g = lane >> 2, c = lane & 3;           // tensor-core operand rows / columns
    const uint32_t bar0 = smem_u32(&s_bar[warp * STAGES]);
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * STAGES * STAGE);
    float *s_o = reinterpret_cast<float *>(smem + WARPS * STAGES * STAGE);
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < STAGES; ++s) mbar_init(bar0 + 8u * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (tid == 0) s_fail = 0;
    __syncwarp();
    fspad_pdl_trigger();
    fspad_pdl_wait();

    const int ctas = gridDim.x, cta = blockIdx.x;
    Parts parts;
    Part part = cut_list<WARPS * 32, UNIT>(a, cta, ctas, parts, s_scan, cta == 0);
    if (tid == 0) tell_cut<UNIT>(a, parts, part, cta);
    const int nt = tree_units<UNIT>(a), runs = a.Hkv * a.mtiles;
    uint32_t phase = 0;                              // of the ring's barriers, a bit a stage
    bool failed = false;

    while (part.left > 0) {
        const int b = part.b, L = prefix_of(a, b, false), n_run = run_units<UNIT>(a, L);
        const int run = part.run, u0 = part.u, u1 = min(n_run, u0 + part.left);
        const int h = a.by_tiles.of(run), row0 = (run - h * a.mtiles) * BM;
        const int *blocks = a.table + (size_t)b * a.table_stride;

        // ---- the warp's first fills: units u0 + warp, u0 + warp + WARPS, ... that lie in the cache ----
        const int first = u0 + warp;
        const int first_kv = first >= nt ? first : first + ((nt - first + WARPS - 1) / WARPS) * WARPS;
        const int n_kv = first_kv < u1 ? (u1 - first_kv + WARPS - 1) / WARPS : 0;
        auto fill = [&](int i) {                     // lane 0: the warp's i-th unit of the cache
            const int key0 = (first_kv + i * WARPS - nt) * UNIT, s = i % STAGES;
            int blk = __ldg(blocks + (key0 >> 7));
            if (blk < 0 || blk >= a.n_blocks) { fspad_report(a.status, FSPAD_ERR_RANGE); blk = 0; }
            const size_t row = ((size_t)blk * a.Hkv + h) * 128 + (key0 & 127);
            const uint32_t to = ring + (uint32_t)(s * STAGE), bar = bar0 + 8u * s;
            mbar_expect_tx(bar, STAGE);
            bulk_load(to, a.kc + row * FSPAD_PACKED_CODE_BYTES, CODES, bar);
            bulk_load(to + 2 * CODES, a.ks + row * FSPAD_PACKED_SCALE_BYTES, SCALES, bar);
            bulk_load(to + CODES, a.vc + row * FSPAD_PACKED_CODE_BYTES, CODES, bar);
            bulk_load(to + 2 * CODES + SCALES, a.vs + row * FSPAD_PACKED_SCALE_BYTES, SCALES, bar);
        };
        if (lane == 0)
            for (int i = 0; i < STAGES && i < n_kv; ++i) fill(i);

        // ---- queries: rows g and g + 8 of the tile, elements 32 c .. 32 c + 31, scaled by a power of two so that the row's largest
        // magnitude lies in [2^14, 2^15): 8 significant bits stay exact down to 2^-31 of the largest ----
        const fspad_bf16 *qrow[2];
        float cs[2];                                 // scores -> log2 units
        uint32_t qf[8][4];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int gr = row0 + g + 8 * x;
            const bool there = gr < a.M;
            qrow[x] = there ? a.q + (((size_t)b * a.N + gr / a.G) * a.Hq + h * a.G + gr % a.G) * D + 32 * c : nullptr;
            uint4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = there ? __ldg(reinterpret_cast<const uint4 *>(qrow[x]) + i) : make_uint4(0u, 0u, 0u, 0u);
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m = fspad_most2(m, fspad_most2(fspad_most2(w[i].x, w[i].y), fspad_most2(w[i].z, w[i].w)));
            }
            m = max(m & 0xffffu, m >> 16);
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
            // the largest magnitude is in [2^e, 2^(e+1)); of zeros, and of rows that are not finite (whose result is not either), as it is
            const int e = m == 0u || m >= 0x7f80u ? 14 : max((int)(m >> 7) - 127, -100);
            const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
            cs[x] = a.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {        // pair 4 i + j of 16: product 2 i + j / 2, its columns 2c (j even) or 2c + 8
                    const uint32_t f = pack_f16(__uint_as_float(v[j] << 16) * up, __uint_as_float(v[j] & 0xffff0000u) * up);
                    qf[2 * i + (j >> 1)][x + 2 * (j & 1)] = f;
                }
            }
        }
        float o[16][4];
#pragma unroll
        for (int j = 0; j < 16; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[j][x] = 0.f;
        float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};

        // scores (log2 units, masked) of 32 keys -> weights; the row's reference follows its maximum where that is far ahead of it
        auto softmax = [&](float (&s)[4][4]) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                float mx = -INFINITY;
#pragma unroll
                for (int t = 0; t < 4; ++t) mx = fmaxf(mx, fmaxf(s[t][2 * x], s[t][2 * x + 1]));
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
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float p = ex2f(s[t][2 * x + y] - ref);
                        s[t][2 * x + y] = p;
                        l_run[x] += p;
                    }
            }
        };

        if (u0 < nt) {
            __syncthreads();                         // (nobody still walks another sequence's tree)
            for (int i = tid; i < a.N; i += WARPS * 32) {
                int p = a.parent[(size_t)b * a.N + i];
                if (i == 0 ? p != -1 : (p < 0 || p >= i)) { fspad_report(a.status, FSPAD_ERR_BAD_TREE); p = -1; }
                s_par[i] = (short)p;
            }
            __syncthreads();
        }
        // ---- units of the tree: bf16 ----
        for (int u = first; u < min(u1, nt); u += WARPS) {
            const int t0 = u * UNIT;
            const fspad_bf16 *tk = a.tk + ((size_t)b * a.Hkv + h) * a.N * D, *tv = a.tv + ((size_t)b * a.Hkv + h) * a.N * D;
            uint32_t see[2] = {0u, 0u};              // which of the unit's keys a row sees
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int gr = row0 + g + 8 * x;
                for (int at = gr < a.M ? gr / a.G : -1; at >= t0; at = s_par[at])
                    if (at < t0 + 32) see[x] |= 1u << (at - t0);
            }
            float s[4][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int x = 0; x < 4; ++x) s[t][x] = 0.f;
                const int key = t0 + 8 * t + key_of(g);
                uint4 kw[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    kw[i] = key < a.N ? __ldg(reinterpret_cast<const uint4 *>(tk + (size_t)key * D + 32 * c) + i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint4 q0 = make_uint4(0u, 0u, 0u, 0u), q1 = q0;
                    if (qrow[0]) q0 = __ldg(reinterpret_cast<const uint4 *>(qrow[0]) + i);
                    if (qrow[1]) q1 = __ldg(reinterpret_cast<const uint4 *>(qrow[1]) + i);
                    const uint32_t lo[4] = {q0.x, q1.x, q0.y, q1.y}, hi[4] = {q0.z, q1.z, q0.w, q1.w};
                    mma16_bf(s[t], lo, kw[i].x, kw[i].y);
                    mma16_bf(s[t], hi, kw[i].z, kw[i].w);
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int k = 8 * t + key_of(2 * c + (x & 1));
                    s[t][x] = (see[x >> 1] >> k) & 1u ? s[t][x] * a.scale_log2 : -INFINITY;
                }
            }
            softmax(s);
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                uint32_t vw[4][8];                   // keys of columns 2c, 2c + 1, 2c + 8, 2c + 9: elements 16 g .. 16 g + 15
                bool odd = false;
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int key = t0 + 16 * st + 8 * (y >> 1) + key_of(2 * c + (y & 1));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint4 w = key < a.N ? __ldg(reinterpret_cast<const uint4 *>(tv + (size_t)key * D + 16 * g) + i) : make_uint4(0u, 0u, 0u, 0u);
                        vw[y][4 * i] = w.x; vw[y][4 * i + 1] = w.y; vw[y][4 * i + 2] = w.z; vw[y][4 * i + 3] = w.w;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) odd |= odd_value(vw[y][i]);
                }
                // A row with an infinity or a NaN in it must not reach the queries that do not see it (0 times it is a NaN): it is taken
                // out of the product, and the queries that do see it get NaN.
                if (__any_sync(0xffffffffu, odd)) {
                    uint32_t keys = 0;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        bool bad = false;
#pragma unroll
                        for (int i = 0; i < 8; ++i) bad |= odd_value(vw[y][i]);
                        if (bad) keys |= 1u << (16 * st + 8 * (y >> 1) + key_of(2 * c + (y & 1)));
                    }
                    keys = __reduce_or_sync(0xffffffffu, keys);
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if ((keys >> (16 * st + 8 * (y >> 1) + key_of(2 * c + (y & 1)))) & 1u)
#pragma unroll
                            for (int i = 0; i < 8; ++i) vw[y][i] = 0u;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (see[x] & keys) l_run[x] = NAN;
                }
                const uint32_t p[4] = {umma::pack_bf16(s[2 * st][0], s[2 * st][1]), umma::pack_bf16(s[2 * st][2], s[2 * st][3]),
                                       umma::pack_bf16(s[2 * st + 1][0], s[2 * st + 1][1]), umma::pack_bf16(s[2 * st + 1][2], s[2 * st + 1][3])};
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
                    mma16_bf(o[j], p, __byte_perm(vw[0][j >> 1], vw[1][j >> 1], sel), __byte_perm(vw[2][j >> 1], vw[3][j >> 1], sel));
                }
            }
        }

        // ---- units of the cache ----
        for (int i = 0; i < n_kv; ++i) {
            const int key0 = (first_kv + i * WARPS - nt) * UNIT, st = i % STAGES;
            const uint32_t at = ring + (uint32_t)(st * STAGE);
            if (!mbar_wait(bar0 + 8u * st, (phase >> st) & 1u)) {
                failed = true;                       // what is under way gets another bounded time to land before the CTA leaves
                for (int y = i; y < n_kv && y < i + STAGES; ++y) (void)mbar_wait(bar0 + 8u * (y % STAGES), (phase >> (y % STAGES)) & 1u);
                break;
            }
            phase ^= 1u << st;
            const int left = L - key0;               // keys of the unit that exist
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
                for (int x = 0; x < 4; ++x) s[t][x] *= cs[x >> 1];
            if (left < UNIT) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (8 * t + key_of(2 * c + (x & 1)) >= left) s[t][x] = -INFINITY;
            }
            softmax(s);
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2) {
                const uint32_t p[4] = {pack_f16(s[2 * k2][0], s[2 * k2][1]), pack_f16(s[2 * k2][2], s[2 * k2][3]),
                                       pack_f16(s[2 * k2 + 1][0], s[2 * k2 + 1][1]), pack_f16(s[2 * k2 + 1][2], s[2 * k2 + 1][3])};
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
            if (lane == 0 && i + STAGES < n_kv) fill(i + STAGES);
        }
        if (failed && lane == 0) s_fail = 1;

        // ---- the warps' results together ----
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            l_run[x] += __shfl_xor_sync(0xffffffffu, l_run[x], 1);
            l_run[x] += __shfl_xor_sync(0xffffffffu, l_run[x], 2);
            if (c == 0) s_ml[warp][g + 8 * x] = make_float2(m_run[x], l_run[x]);
        }
        __syncthreads();
        const bool any_fail = s_fail != 0;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) m = fmaxf(m, s_ml[w][g + 8 * x].x);
            const float f = m_run[x] == -INFINITY ? 0.f : ex2f(m_run[x] - m);
            // lane (g, c): elements 32 c + j in o[j][2 x], 32 c + 16 + j in o[j][2 x + 1]
            float4 *dst = reinterpret_cast<float4 *>(s_o + ((size_t)warp * BM + g + 8 * x) * OROW + c * 36);
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int j = 0; j < 16; j += 4)
                    dst[y * 4 + j / 4] = make_float4(o[j][2 * x + y] * f, o[j + 1][2 * x + y] * f, o[j + 2][2 * x + y] * f, o[j + 3][2 * x + y] * f);
        }
        __syncthreads();
        {
            // thread: row tid / 16, elements 8 (tid % 16) ..
            const int row = tid >> 4, d0 = (tid & 15) * 8;
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) m = fmaxf(m, s_ml[w][row].x);
            float acc[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) acc[x] = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float2 ml = s_ml[w][row];
                l += ml.x == -INFINITY ? ml.y : ml.y * ex2f(ml.x - m);       // (a sum without a maximum is zero, or a NaN)
                const float4 *src = reinterpret_cast<const float4 *>(s_o + ((size_t)w * BM + row) * OROW + (d0 >> 5) * 36 + (d0 & 31));
                const float4 lo = src[0], hi = src[1];
                acc[0] += lo.x; acc[1] += lo.y; acc[2] += lo.z; acc[3] += lo.w;
                acc[4] += hi.x; acc[5] += hi.y; acc[6] += hi.z; acc[7] += hi.w;
            }
            const int gr = row0 + row;
            if (gr < a.M && !any_fail) {
                if (u0 == 0 && u1 == n_run) {
                    const float inv = 1.f / l;
                    uint4 pk;
                    pk.x = umma::pack_bf16(acc[0] * inv, acc[1] * inv); pk.y = umma::pack_bf16(acc[2] * inv, acc[3] * inv);
                    pk.z = umma::pack_bf16(acc[4] * inv, acc[5] * inv); pk.w = umma::pack_bf16(acc[6] * inv, acc[7] * inv);
                    *reinterpret_cast<uint4 *>(a.out + (((size_t)b * a.N + gr / a.G) * a.Hq + h * a.G + gr % a.G) * D + d0) = pk;
                } else {
                    const size_t slot = ((size_t)cta * 2 + (u0 == 0 ? 1 : 0)) * BM + row;
                    float4 *dst = reinterpret_cast<float4 *>(a.part_o + slot * D + d0);
                    dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
                    dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
                    if (d0 == 0) a.part_ml[slot] = make_float2(m, l);
                }
            }
        }
        if (any_fail) break;
        __syncthreads();                             // the staged rows are read
        part.left -= u1 - u0;
        part.u = 0;
        if (++part.run == runs) { part.run = 0; ++part.b; }
    }
    if (s_fail != 0 && tid == 0) fspad_report(a.status, FSPAD_ERR_TIMEOUT);
}

}  // namespace

// Which of the two kernels takes a call, by the query rows of a kv head.
static bool many_rows(const fspad_ctx *ctx, int N) { return (long long)N * (ctx->cfg.n_q_heads / ctx->cfg.n_kv_heads) > BM; }

size_t fspad_attn_packed_workspace(const fspad_ctx *ctx, int N, int B)
{
    (void)B;
    if (many_rows(ctx, N)) return fspad_attn_packed_umma_workspace(ctx);
    return scratch_bytes<BM>(ctx->sm_count);
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
    scratch_in<BM>(a, ctas, workspace);
    cudaError_t e = cudaFuncSetAttribute(tree_attn_packed_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    ctx->launches += 2;
    e = fspad_launch(tree_attn_packed_kernel, dim3((unsigned)ctas), dim3(WARPS * 32), SMEM, st, 0, a);
    if (e != cudaSuccess) return e;
    return fspad_launch(tree_attn_packed_merge_kernel<BM, 2, 4>, dim3((unsigned)ctas, (unsigned)((a.M < BM ? a.M : BM) + 1) / 2), dim3(256), 0, st, 0, a);
}
