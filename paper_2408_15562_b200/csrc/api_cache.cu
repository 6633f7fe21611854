// C ABI of the operators around the cache held in 4 bits: argument validation.  (The calls of the verify step: api.cu.)
#include <climits>
#include <cmath>
#include <cstring>

#include "packed.cuh"

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
// Frequencies of the rotary pairs in turns a position.  Each host thread keeps those of its last theta (64 powers take 3 us): kept in the context, calls of two
// threads with a theta each got a mixture.
void rope_turns(double theta, double (&to)[FSPAD_HEAD_DIM / 2])
{
    thread_local double last = 0.0, turns[FSPAD_HEAD_DIM / 2];       // (no theta is 0)
    if (last != theta) {
        for (int i = 0; i < FSPAD_HEAD_DIM / 2; ++i) turns[i] = std::pow(theta, -2.0 * i / FSPAD_HEAD_DIM) / (2.0 * 3.14159265358979323846);
        last = theta;
    }
    std::memcpy(to, turns, sizeof turns);
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

}  // namespace

extern "C" {

int fspad_device(const fspad_ctx *ctx) { return ctx ? ctx->device : -1; }

int fspad_rope_qkv(fspad_ctx *ctx, const fspad_bf16 *qkv, int64_t row_stride, const int32_t *positions, const int32_t *start,
                   const int32_t *parent, int n_nodes, int batch, double theta, int sec_t, int sec_h, int sec_w, int adjacent,
                   fspad_bf16 *q, fspad_bf16 *k, fspad_bf16 *v, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    const fspad_config &c = ctx->cfg;
    if (!qkv || !q || !k || !v) return FSPAD_ERR_NULL;
    if (positions ? start != nullptr || parent != nullptr : !start || !parent) return FSPAD_ERR_NULL;
    if (misaligned(qkv) || misaligned(q) || misaligned(k) || misaligned(v)) return FSPAD_ERR_ALIGN;
    if (positions) {
        if (n_nodes < 1 || batch < 0 || batch > c.max_batch) return FSPAD_ERR_SHAPE;
    } else if ((rc = check_tree(ctx, n_nodes, batch)) != 0) {
        return rc;
    }
    const int half = FSPAD_HEAD_DIM / 2;
    const int64_t width = ((int64_t)c.n_q_heads + 2 * (int64_t)c.n_kv_heads) * FSPAD_HEAD_DIM;
    if (sec_t < 0 || sec_h < 0 || sec_w < 0 || sec_t > half || sec_h > half || sec_w > half || sec_t + sec_h + sec_w != half) return FSPAD_ERR_SHAPE;
    if (row_stride < width || row_stride % 8 != 0) return FSPAD_ERR_SHAPE;
    if (!(theta > 0.0) || std::isinf(theta) || std::isinf(std::pow(theta, -2.0 * (half - 1) / FSPAD_HEAD_DIM))) return FSPAD_ERR_RANGE;
    if ((int64_t)n_nodes * batch > INT_MAX || batch > 65535) return FSPAD_ERR_TOO_LARGE;
    if (batch == 0) return FSPAD_OK;
    if (q == qkv || k == qkv || v == qkv || q == k || q == v || k == v) return FSPAD_ERR_RANGE;
    FspadRopeTable t;
    rope_turns(theta, t.turns);
    t.split0 = sec_t;
    t.split1 = sec_t + sec_h;
    return result(fspad_launch_rope_qkv(ctx, qkv, row_stride, positions, start, parent, n_nodes, batch, t, adjacent != 0, q, k, v,
                                        fspad_stream(stream)));
}

int fspad_block_plan(fspad_ctx *ctx, const int32_t *len, const int32_t *add, const int32_t *drop, int batch, int blocks_per_seq,
                     int n_blocks, int32_t *block_table, int32_t *held, int32_t *free_blocks, int32_t *n_free, int max_rows,
                     int32_t *row_start, int64_t *slots, int32_t *row_seq, int32_t *row_pos, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    if (!len || !add || !block_table || !held || !free_blocks || !n_free || !row_start || !slots) return FSPAD_ERR_NULL;
    if (batch < 0 || batch > ctx->cfg.max_batch || max_rows < 0) return FSPAD_ERR_SHAPE;
    if ((rc = check_blocks(blocks_per_seq, n_blocks)) != 0) return rc;
    if (batch > FSPAD_PLAN_MAX_BATCH) return FSPAD_ERR_TOO_LARGE;      // (no sequences: row_start[0] and the slots are written all the same)
    static_assert(sizeof(long long) == sizeof(int64_t), "slots");
    return result(fspad_launch_block_plan(ctx, len, add, drop, batch, blocks_per_seq, n_blocks, block_table, held, free_blocks, n_free,
                                          max_rows, row_start, reinterpret_cast<long long *>(slots), row_seq, row_pos, fspad_stream(stream)));
}

int fspad_kv_write_packed(fspad_ctx *ctx, const fspad_bf16 *k, const fspad_bf16 *v, const int64_t *slots, int rows, int layer,
                          uint8_t *codes, uint8_t *scales, int n_blocks, fspad_bf16 *k_rounded, fspad_bf16 *v_rounded, void *stream)
{
    int rc = check_device(ctx);
    if (rc) return rc;
    if (!k || !v || !slots || !codes || !scales) return FSPAD_ERR_NULL;
    if ((k_rounded == nullptr) != (v_rounded == nullptr)) return FSPAD_ERR_NULL;
    if (misaligned(k) || misaligned(v) || misaligned(codes) || misaligned(scales) || misaligned(k_rounded) || misaligned(v_rounded))
        return FSPAD_ERR_ALIGN;
    if (rows < 0 || layer < 0 || layer >= ctx->cfg.n_layers || n_blocks < 1) return FSPAD_ERR_SHAPE;
    if ((int64_t)rows * ctx->cfg.n_kv_heads > INT_MAX) return FSPAD_ERR_TOO_LARGE;
    if (rows == 0) return FSPAD_OK;
    const size_t n = (size_t)rows * ctx->cfg.n_kv_heads * FSPAD_HEAD_DIM * sizeof(fspad_bf16);
    if (k_rounded && (overlap(k_rounded, n, v, n) || overlap(v_rounded, n, k, n) || overlap(k_rounded, n, v_rounded, n) ||       // (K and V go at the same time)
                      (k_rounded != k && overlap(k_rounded, n, k, n)) || (v_rounded != v && overlap(v_rounded, n, v, n))))
        return FSPAD_ERR_RANGE;
    return result(fspad_launch_kv_write_packed(ctx, k, v, reinterpret_cast<const long long *>(slots), rows, layer, codes, scales, n_blocks,
                                               k_rounded, v_rounded, fspad_stream(stream)));
}

int fspad_kv_append_packed(fspad_ctx *ctx, uint8_t *codes, uint8_t *scales, const int32_t *block_table, int blocks_per_seq, int n_blocks,
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
    return result(fspad_launch_kv_append_packed(ctx, codes, scales, pg, tree_kv, accepted_path, n_accepted, prefix_len, n_nodes, batch,
                                                rounded, new_len, fspad_stream(stream)));
}

size_t fspad_tree_attn_packed_workspace_bytes(const fspad_ctx *ctx, int n_nodes, int batch)
{
    if (!ctx || check_tree(ctx, n_nodes, batch) != 0) return 0;
    return fspad_attn_packed_workspace(ctx, n_nodes, batch);
}

int fspad_tree_attn_packed(fspad_ctx *ctx, const fspad_bf16 *q, const uint8_t *codes, const uint8_t *scales, int layer,
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
    if (workspace_bytes < fspad_attn_packed_workspace(ctx, n_nodes, batch)) return FSPAD_ERR_RANGE;
    if (!fspad_attn_packed_fits(ctx, n_nodes, batch, blocks_per_seq)) return FSPAD_ERR_TOO_LARGE;
    const size_t rows = (size_t)n_blocks * ctx->cfg.n_kv_heads * 128, first = (size_t)layer * 2 * rows;
    const uint8_t *kc = codes + first * FSPAD_PACKED_CODE_BYTES, *ks = scales + first * FSPAD_PACKED_SCALE_BYTES;
    const FspadPaged pg{block_table, blocks_per_seq, n_blocks};
    return result(fspad_launch_tree_attn_packed(ctx, q, kc, ks, kc + rows * FSPAD_PACKED_CODE_BYTES, ks + rows * FSPAD_PACKED_SCALE_BYTES, pg,
                                                tree_k, tree_v, parent, prefix_len, n_nodes, batch, out, workspace, fspad_stream(stream)));
}

}  // extern "C"
