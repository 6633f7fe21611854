// C ABI of the operators around the cache held in 8 bits, and of the calls on blocks: argument validation.
#include <climits>

#include "fp8.cuh"

namespace {

inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// Kernels are launched on the current device, and the context's scratch and status word lie on its own.
int check_device(const fspad_ctx *ctx)
{
    if (!ctx) return FSPAD_ERR_NULL;
    int d = -1;
    if (cudaGetDevice(&d) != cudaSuccess) return FSPAD_ERR_CUDA;
    return d == ctx->device ? FSPAD_OK : FSPAD_ERR_DEVICE;
}
// Whether two arrays of so many bytes share any.
bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na > 0 && nb > 0 && (x < y ? y - x < na : x - y < nb);
}
int result(cudaError_t e) { return e == cudaSuccess ? FSPAD_OK : FSPAD_ERR_CUDA; }

int check_tree(const fspad_ctx *ctx, int n_nodes, int batch)
{
    if (n_nodes > FSPAD_MAX_NODES_WIDE || n_nodes > ctx->cfg.max_nodes) return FSPAD_ERR_TREE_TOO_LARGE;
    if (n_nodes < 1 || batch < 0 || batch > ctx->cfg.max_batch) return FSPAD_ERR_SHAPE;
    return FSPAD_OK;
}
// A table of blocks: rows are counted in 32 bits.
int check_blocks(int blocks_per_seq, int n_blocks)
{
    if (blocks_per_seq < 1 || n_blocks < 1) return FSPAD_ERR_SHAPE;
    return blocks_per_seq > INT_MAX / 128 ? FSPAD_ERR_TOO_LARGE : FSPAD_OK;
}
// The state of a pool.
int check_pool(const fspad_ctx *ctx, const FspadPool &p)
{
    if (!p.table || !p.held || !p.shares || !p.free_blocks || !p.n_free) return FSPAD_ERR_NULL;
    if (p.B < 0 || p.B > ctx->cfg.max_batch) return FSPAD_ERR_SHAPE;
    const int rc = check_blocks(p.bps, p.n_blocks);
    if (rc) return rc;
    if (p.B > FSPAD_PLAN_MAX_BATCH || p.n_blocks > FSPAD_PAGES_MAX_BLOCKS) return FSPAD_ERR_TOO_LARGE;
    const struct { const void *at; size_t n; } part[] = {{p.table, (size_t)p.B * p.bps}, {p.held, (size_t)p.B}, {p.shares, (size_t)p.n_blocks},
                                                          {p.free_blocks, (size_t)p.n_blocks}, {p.n_free, 1}};
    for (int i = 0; i < 5; ++i)
        for (int j = 0; j < i; ++j)
            if (overlap(part[i].at, part[i].n * sizeof(int), part[j].at, part[j].n * sizeof(int))) return FSPAD_ERR_RANGE;
    return FSPAD_OK;
}
// Whether an array of n numbers shares any with the pool's state.
bool in_pool(const FspadPool &p, const void *a, size_t n)
{
    n *= sizeof(int);
    return overlap(a, n, p.table, sizeof(int) * (size_t)p.B * p.bps) || overlap(a, n, p.held, sizeof(int) * (size_t)p.B) ||
           overlap(a, n, p.shares, sizeof(int) * (size_t)p.n_blocks) || overlap(a, n, p.free_blocks, sizeof(int) * (size_t)p.n_blocks) ||
           overlap(a, n, p.n_free, sizeof(int));
}

}  // namespace

extern "C" {

int fspad_kv_write_fp8(fspad_ctx *ctx, const fspad_bf16 *k, const fspad_bf16 *v, const int64_t *slots, int rows, int layer,
                       uint8_t *codes, float *scales, int n_blocks, fspad_bf16 *k_rounded, fspad_bf16 *v_rounded, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    if (!k || !v || !slots || !codes || !scales) return FSPAD_ERR_NULL;
    if ((k_rounded == nullptr) != (v_rounded == nullptr)) return FSPAD_ERR_NULL;
    if (misaligned(k) || misaligned(v) || misaligned(codes) || misaligned(scales) || misaligned(k_rounded) || misaligned(v_rounded))
        return FSPAD_ERR_ALIGN;
    if (rows < 0 || layer < 0 || layer >= ctx->cfg.n_layers || n_blocks < 1) return FSPAD_ERR_SHAPE;
    if ((int64_t)rows * ctx->cfg.n_kv_heads > INT_MAX / 2) return FSPAD_ERR_TOO_LARGE;
    if (rows == 0) return FSPAD_OK;
    const size_t n = (size_t)rows * ctx->cfg.n_kv_heads * FSPAD_HEAD_DIM * sizeof(fspad_bf16);
    if (k_rounded && (overlap(k_rounded, n, v, n) || overlap(v_rounded, n, k, n) || overlap(k_rounded, n, v_rounded, n) ||       // (K and V go at the same time)
                      (k_rounded != k && overlap(k_rounded, n, k, n)) || (v_rounded != v && overlap(v_rounded, n, v, n))))
        return FSPAD_ERR_RANGE;
    static_assert(sizeof(long long) == sizeof(int64_t), "slots");
    return result(fspad_launch_kv_write_fp8(ctx, k, v, reinterpret_cast<const long long *>(slots), rows, layer, codes, scales, n_blocks,
                                            k_rounded, v_rounded, fspad_stream(stream)));
}

int fspad_kv_append_fp8(fspad_ctx *ctx, uint8_t *codes, float *scales, const int32_t *block_table, int blocks_per_seq, int n_blocks,
                        const fspad_bf16 *tree_kv, const int32_t *accepted_path, const int32_t *n_accepted, const int32_t *prefix_len,
                        int n_nodes, int batch, fspad_bf16 *rounded, int32_t *new_len, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    if ((rc = check_tree(ctx, n_nodes, batch)) != 0) return rc;
    if (!codes || !scales || !block_table || !tree_kv || !accepted_path || !n_accepted || !prefix_len) return FSPAD_ERR_NULL;
    if (misaligned(codes) || misaligned(scales) || misaligned(tree_kv) || misaligned(rounded)) return FSPAD_ERR_ALIGN;
    if ((rc = check_blocks(blocks_per_seq, n_blocks)) != 0) return rc;
    if (batch == 0) return FSPAD_OK;
    const size_t word = sizeof(int32_t), seqs = word * batch;
    if (new_len && (overlap(new_len, seqs, prefix_len, seqs) || overlap(new_len, seqs, n_accepted, seqs) ||         // (other warps still read them)
                    overlap(new_len, seqs, accepted_path, seqs * ctx->cfg.max_nodes) || overlap(new_len, seqs, block_table, seqs * blocks_per_seq)))
        return FSPAD_ERR_RANGE;
    const size_t tree = (size_t)ctx->cfg.n_layers * 2 * batch * ctx->cfg.n_kv_heads * n_nodes * FSPAD_HEAD_DIM * sizeof(fspad_bf16);
    if (rounded && rounded != tree_kv && overlap(rounded, tree, tree_kv, tree)) return FSPAD_ERR_RANGE;
    const FspadPaged pg{block_table, blocks_per_seq, n_blocks};
    return result(fspad_launch_kv_append_fp8(ctx, codes, scales, pg, tree_kv, accepted_path, n_accepted, prefix_len, n_nodes, batch,
                                             rounded, new_len, fspad_stream(stream)));
}

size_t fspad_tree_attn_fp8_workspace_bytes(const fspad_ctx *ctx) { return ctx ? fspad_attn_fp8_workspace(ctx) : 0; }

int fspad_tree_attn_fp8(fspad_ctx *ctx, const fspad_bf16 *q, const uint8_t *codes, const float *scales, int layer,
                        const int32_t *block_table, int blocks_per_seq, int n_blocks, const fspad_bf16 *tree_k,
                        const fspad_bf16 *tree_v, const int32_t *parent, const int32_t *prefix_len, int n_nodes, int batch,
                        fspad_bf16 *out, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    if ((rc = check_tree(ctx, n_nodes, batch)) != 0) return rc;
    if (!q || !codes || !scales || !block_table || !tree_k || !tree_v || !parent || !prefix_len || !out || !workspace) return FSPAD_ERR_NULL;
    if (misaligned(q) || misaligned(codes) || misaligned(scales) || misaligned(tree_k) || misaligned(tree_v) || misaligned(out) ||
        misaligned(workspace))
        return FSPAD_ERR_ALIGN;
    if (layer < 0 || layer >= ctx->cfg.n_layers) return FSPAD_ERR_SHAPE;
    if ((rc = check_blocks(blocks_per_seq, n_blocks)) != 0) return rc;
    if (batch == 0) return FSPAD_OK;
    if (out == q || out == tree_k || out == tree_v) return FSPAD_ERR_RANGE;
    if (workspace_bytes < fspad_attn_fp8_workspace(ctx)) return FSPAD_ERR_RANGE;
    if (!fspad_attn_fp8_fits(ctx, n_nodes, batch, blocks_per_seq, n_blocks)) return FSPAD_ERR_TOO_LARGE;
    const size_t heads = (size_t)n_blocks * ctx->cfg.n_kv_heads, first = (size_t)layer * 2 * heads;
    const uint8_t *kc = codes + first * 128 * FSPAD_HEAD_DIM;
    const float *ks = scales + first * FSPAD_FP8_GROUPS;
    const FspadPaged pg{block_table, blocks_per_seq, n_blocks};
    return result(fspad_launch_tree_attn_fp8(ctx, q, kc, ks, kc + heads * 128 * FSPAD_HEAD_DIM, ks + heads * FSPAD_FP8_GROUPS, pg, tree_k, tree_v, parent,
                                             prefix_len, n_nodes, batch, out, workspace, fspad_stream(stream)));
}

int fspad_block_fork(fspad_ctx *ctx, const int32_t *src, const int32_t *dst, int n, int32_t *len, int batch, int blocks_per_seq, int n_blocks,
                     int32_t *block_table, int32_t *held, int32_t *shares, int32_t *free_blocks, int32_t *n_free, int32_t *pairs, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    const FspadPool p{block_table, held, shares, free_blocks, n_free, batch, blocks_per_seq, n_blocks};
    if (!src || !dst || !len || !pairs) return FSPAD_ERR_NULL;
    if ((rc = check_pool(ctx, p)) != 0) return rc;
    if (n < 0 || n > batch) return FSPAD_ERR_SHAPE;
    if (n == 0) return FSPAD_OK;
    const size_t w = sizeof(int32_t);
    if (in_pool(p, src, n) || in_pool(p, dst, n) || in_pool(p, len, batch) || in_pool(p, pairs, 2 * (size_t)n) || overlap(pairs, 2 * w * n, src, w * n) ||
        overlap(pairs, 2 * w * n, dst, w * n) || overlap(pairs, 2 * w * n, len, w * batch) || overlap(len, w * batch, src, w * n) || overlap(len, w * batch, dst, w * n))
        return FSPAD_ERR_RANGE;
    return result(fspad_launch_block_fork(ctx, p, src, dst, n, len, pairs, fspad_stream(stream)));
}

int fspad_block_free(fspad_ctx *ctx, const int32_t *drop, int batch, int blocks_per_seq, int n_blocks, int32_t *block_table, int32_t *held,
                     int32_t *shares, int32_t *free_blocks, int32_t *n_free, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    const FspadPool p{block_table, held, shares, free_blocks, n_free, batch, blocks_per_seq, n_blocks};
    if (!drop) return FSPAD_ERR_NULL;
    if ((rc = check_pool(ctx, p)) != 0) return rc;
    if (batch == 0) return FSPAD_OK;
    if (in_pool(p, drop, batch)) return FSPAD_ERR_RANGE;
    return result(fspad_launch_block_free(ctx, p, drop, fspad_stream(stream)));
}

int fspad_block_compact(fspad_ctx *ctx, int batch, int blocks_per_seq, int n_blocks, int32_t *block_table, int32_t *held, int32_t *shares,
                        int32_t *free_blocks, int32_t *n_free, int32_t *pairs, int max_pairs, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    const FspadPool p{block_table, held, shares, free_blocks, n_free, batch, blocks_per_seq, n_blocks};
    if (!pairs) return FSPAD_ERR_NULL;
    if ((rc = check_pool(ctx, p)) != 0) return rc;
    if (max_pairs < 0 || max_pairs > n_blocks) return FSPAD_ERR_SHAPE;
    if (in_pool(p, pairs, 2 * (size_t)max_pairs)) return FSPAD_ERR_RANGE;
    return result(fspad_launch_block_compact(ctx, p, pairs, max_pairs, fspad_stream(stream)));
}

int fspad_block_copy(fspad_ctx *ctx, void *pool, int64_t block_bytes, void *pool2, int64_t block_bytes2, int planes, int n_blocks,
                     const int32_t *pairs, int n_pairs, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    if (!pool || !pairs || (pool2 == nullptr) != (block_bytes2 == 0)) return FSPAD_ERR_NULL;
    if (misaligned(pool) || misaligned(pool2) || (reinterpret_cast<uintptr_t>(pairs) & 7u)) return FSPAD_ERR_ALIGN;
    if (block_bytes < 16 || block_bytes % 16 || block_bytes2 < 0 || block_bytes2 % 16 || planes < 1 || n_blocks < 1 || n_pairs < 0) return FSPAD_ERR_SHAPE;
    // (a plane, and the number of pieces of a call, in 64 bits with room)
    if (block_bytes > (1ll << 40) || block_bytes2 > (1ll << 40)) return FSPAD_ERR_TOO_LARGE;
    if ((double)(block_bytes + block_bytes2) * planes * n_blocks > 1e15 || (double)(block_bytes + block_bytes2) * planes * n_pairs > 1e18) return FSPAD_ERR_TOO_LARGE;
    if (n_pairs == 0) return FSPAD_OK;
    return result(fspad_launch_block_copy(ctx, pool, block_bytes, pool2, block_bytes2, planes, n_blocks, pairs, n_pairs, fspad_stream(stream)));
}

}  // extern "C"
