// Rotary positions of several axes on the rows of the QKV product ("Preliminaries": the flattened tree goes through the target in one
// forward; a node's position is its depth behind the prefix, whatever its place in the flattened order).
//
// Pair i of a head of 128 turns by angle a_i = p[axis(i)] * theta^(-2i/128): y1 = x1 cos a - x2 sin a, y2 = x2 cos a + x1 sin a.  The
// pairs' axes are three consecutive runs (time, height, width).  Angles are taken in turns in double precision and reduced there, so that
// a position of any size costs no accuracy: what reaches the sine is a fraction of a turn rounded once to 32 bits.
//
// Bound by memory: a row is read and written once, Q in place order, K and V into the head-major layout of the tree arrays.  A
// thread keeps the sines of eight pairs of one row in registers and takes those pairs of one head after the other, 32 bytes each way; how
// many heads fall to a thread follows from how many rows there are, so that few rows still reach every SM.  What a thread needs of the first four heads
// is asked for before positions and sines, which take as long as the loads.  8201 rows of 48 heads, three axes: 32.9 us, 6.1 TB/s, 95 % of the copy rate (with
// the loads behind the sines 36.0); 60 nodes 3.9 us, a launch and three trips to memory in turn; 64 trees of 60 nodes 19.6 us, 4.8 TB/s: each CTA takes its
// tree's depths for itself.
#include "packed.cuh"

namespace {

constexpr int kThreads = 128;
constexpr int kRows = kThreads / 8;      // rows of a CTA: eight threads a row

struct RopeArgs {
    const fspad_bf16 *qkv;
    long long row_stride;
    const int *positions, *start, *parent;
    int N, B, Hq, Hkv;
    int heads_per;                       // heads a thread takes
    fspad_bf16 *q, *k, *v;
    int *status;
    FspadRopeTable table;
};

__device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
}

// TREE: rows are the nodes of tree blockIdx.z, positions start + depth.  Otherwise rows of all sequences in one run, positions given.
template <bool TREE, bool ADJACENT>
__global__ void __launch_bounds__(kThreads)
rope_qkv_kernel(const __grid_constant__ RopeArgs a)
{
    __shared__ short s_up[2][FSPAD_MAX_NODES_WIDE], s_depth[2][FSPAD_MAX_NODES_WIDE];
    fspad_pdl_trigger();
    fspad_pdl_wait();
    const int c = threadIdx.x & 7;
    const long long r = (long long)blockIdx.x * kRows + (threadIdx.x >> 3);
    long long row;                       // of all rows
    int b, i;
    if (TREE) {
        b = blockIdx.z;
        i = (int)r;
        row = (long long)b * a.N + i;
    } else {
        row = r;
        b = (int)((unsigned)r / (unsigned)a.N);      // (at most 2^31 rows, and the last CTA's)
        i = (int)((unsigned)r - (unsigned)b * (unsigned)a.N);
    }
    const bool ok = TREE ? i < a.N : r < (long long)a.B * a.N;
    const int heads = a.Hq + 2 * a.Hkv;
    const int h0 = blockIdx.y * a.heads_per, h1 = min(heads, h0 + a.heads_per);
    const uint4 *src = reinterpret_cast<const uint4 *>(a.qkv + row * a.row_stride);
    // the thread's 16-byte pieces of a head: elements 8c .. and 64 + 8c .. (pairs across the halves), or 16c .. (neighbours)
    const int p0 = ADJACENT ? 2 * c : c, p1 = ADJACENT ? 2 * c + 1 : c + 8;
    constexpr int U = 4;                 // heads under way: the first are asked for before the positions and their sines are taken
    uint4 first[U], second[U];
    auto fetch = [&](int h) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (ok && h + u < h1) {
                first[u] = __ldg(src + (h + u) * 16 + p0);
                second[u] = __ldg(src + (h + u) * 16 + p1);
            }
    };
    fetch(h0);
    double pos[3] = {0.0, 0.0, 0.0};
    if (TREE) {
        // depth by doubling: after round t every node knows its ancestor 2^t up and how far that is
        for (int n = threadIdx.x; n < a.N; n += kThreads) {
            int p = a.parent[(size_t)b * a.N + n];
            if (n == 0 ? p != -1 : (p < 0 || p >= n)) { fspad_report(a.status, FSPAD_ERR_BAD_TREE); p = n - 1; }
            s_up[0][n] = (short)(n == 0 ? 0 : p);
            s_depth[0][n] = n == 0 ? 0 : 1;
        }
        int at = 0;
        for (int reach = 1; reach < a.N; reach <<= 1) {
            __syncthreads();
            for (int n = threadIdx.x; n < a.N; n += kThreads) {
                const int u = s_up[at][n];
                s_depth[at ^ 1][n] = s_depth[at][n] + s_depth[at][u];
                s_up[at ^ 1][n] = s_up[at][u];
            }
            at ^= 1;
        }
        __syncthreads();
        if (ok) {
            const int d = s_depth[at][i];
#pragma unroll
            for (int x = 0; x < 3; ++x) pos[x] = (double)a.start[b * 3 + x] + (double)d;
        }
    } else if (ok) {
#pragma unroll
        for (int x = 0; x < 3; ++x) pos[x] = (double)a.positions[row * 3 + x];
    }
    if (!ok) return;
    float co[8], si[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int p = 8 * c + j;
        const double t = (p < a.table.split0 ? pos[0] : p < a.table.split1 ? pos[1] : pos[2]) * a.table.turns[p];
        sincospif(2.0f * (float)(t - rint(t)), &si[j], &co[j]);
    }
#pragma unroll 1
    for (int h4 = h0; h4 < h1; h4 += U) {
      if (h4 > h0) fetch(h4);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h4 + u;
        if (h >= h1) break;
        const uint4 lo = first[u], hi = second[u];
        uint4 o0, o1;
        fspad_bf16 *to;
        if (h < a.Hq) to = a.q + (row * a.Hq + h) * FSPAD_HEAD_DIM;
        else if (h < a.Hq + a.Hkv) to = a.k + (((long long)b * a.Hkv + (h - a.Hq)) * a.N + i) * FSPAD_HEAD_DIM;
        else to = a.v + (((long long)b * a.Hkv + (h - a.Hq - a.Hkv)) * a.N + i) * FSPAD_HEAD_DIM;
        if (h >= a.Hq + a.Hkv) {
            o0 = lo;
            o1 = hi;
        } else {
            const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
            uint32_t y0[4], y1[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 x = unpack(wl[j]), z = unpack(wh[j]);
                if (ADJACENT) {          // (x.x, x.y) is pair j, (z.x, z.y) pair 4 + j
                    y0[j] = pack(x.x * co[j] - x.y * si[j], x.y * co[j] + x.x * si[j]);
                    y1[j] = pack(z.x * co[4 + j] - z.y * si[4 + j], z.y * co[4 + j] + z.x * si[4 + j]);
                } else {                 // (x.x, z.x) is pair 2j, (x.y, z.y) pair 2j + 1
                    y0[j] = pack(x.x * co[2 * j] - z.x * si[2 * j], x.y * co[2 * j + 1] - z.y * si[2 * j + 1]);
                    y1[j] = pack(z.x * co[2 * j] + x.x * si[2 * j], z.y * co[2 * j + 1] + x.y * si[2 * j + 1]);
                }
            }
            o0 = make_uint4(y0[0], y0[1], y0[2], y0[3]);
            o1 = make_uint4(y1[0], y1[1], y1[2], y1[3]);
        }
        reinterpret_cast<uint4 *>(to)[p0] = o0;
        reinterpret_cast<uint4 *>(to)[p1] = o1;
      }
    }
}

}  // namespace

cudaError_t fspad_launch_rope_qkv(fspad_ctx *ctx, const fspad_bf16 *qkv, long long row_stride, const int *positions, const int *start,
                                  const int *parent, int N, int B, const FspadRopeTable &table, bool adjacent, fspad_bf16 *q,
                                  fspad_bf16 *k, fspad_bf16 *v, cudaStream_t st)
{
    const fspad_config &c = ctx->cfg;
    RopeArgs a;
    a.qkv = qkv; a.row_stride = row_stride; a.positions = positions; a.start = start; a.parent = parent;
    a.N = N; a.B = B; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.q = q; a.k = k; a.v = v; a.status = ctx->d_status;
    a.table = table;
    const bool tree = positions == nullptr;
    const int heads = c.n_q_heads + 2 * c.n_kv_heads;
    const long long tiles = tree ? (N + kRows - 1) / kRows : ((long long)B * N + kRows - 1) / kRows;
    const long long seqs = tree ? B : 1;
    // eight CTAs an SM where there are rows enough; else as few heads a thread as reach that (their sines are taken again in each)
    long long groups = ((long long)ctx->sm_count * 8 + tiles * seqs - 1) / (tiles * seqs);
    if (groups > heads) groups = heads;
    if (groups > 65535) groups = 65535;
    a.heads_per = (int)((heads + groups - 1) / groups);
    // many rows: shorter CTAs, for the last ones leave SMs idle (8201 rows of 48 heads: 39.9 us with 16 heads a thread, 36.0 with 4 and 40.4 with 3, before the
    // loads went ahead of the sines; trees, whose CTAs all take the depths again, did not gain: 64 of 60 nodes 21.8 us with 10 heads and 23.3 with 5)
    if (!tree && a.heads_per > 4) a.heads_per = 4;
    const dim3 grid((unsigned)tiles, (unsigned)((heads + a.heads_per - 1) / a.heads_per), (unsigned)seqs);
    auto kernel = tree ? (adjacent ? rope_qkv_kernel<true, true> : rope_qkv_kernel<true, false>)
                       : (adjacent ? rope_qkv_kernel<false, true> : rope_qkv_kernel<false, false>);
    ctx->launches++;
    return fspad_launch(kernel, grid, dim3(kThreads), 0, st, 0, a);
}
