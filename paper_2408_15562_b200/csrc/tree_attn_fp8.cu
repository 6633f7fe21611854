// Tree-masked attention over a cache held in 8 bits ("Preliminaries": the flattened token tree is the target's input and the attention mask
// built from the tree introduces the dependencies between its tokens; one node is the plain single-token step).
//
// For query row i (tree node x head of the group) of sequence b and kv head h:
//   s_j = c q_i . k_j,   out_i = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
// over the L_b cached keys, whose rows are code * scale, and over the node itself and its ancestors among the bf16 tree rows.
#include "fp8.cuh"
#include "packed_list.cuh"

size_t fspad_attn_fp8_umma_workspace(const fspad_ctx *ctx);
cudaError_t fspad_launch_attn_fp8_umma(fspad_ctx *ctx, packed::Args a, const CUtensorMap &k_map, int k_row0, void *workspace, cudaStream_t st);

size_t fspad_attn_fp8_workspace(const fspad_ctx *ctx) { return fspad_attn_fp8_umma_workspace(ctx); }

// Whether a call's list can be counted in 32 bits, and the rows of a plane of codes in a TMA coordinate.
bool fspad_attn_fp8_fits(const fspad_ctx *ctx, int N, int B, int bps, int n_blocks)
{
    const fspad_config &c = ctx->cfg;
    packed::Args a;
    a.N = N; a.B = B; a.Hkv = c.n_kv_heads; a.M = N * (c.n_q_heads / c.n_kv_heads); a.mtiles = (a.M + 7) / 8; a.table_stride = bps;
    return packed::units_fit<128>(a) && (long long)n_blocks * c.n_kv_heads * 128 <= 0x7fffffffll;
}

cudaError_t fspad_launch_tree_attn_fp8(fspad_ctx *ctx, const fspad_bf16 *q, const uint8_t *k_codes, const float *k_scales, const uint8_t *v_codes,
                                       const float *v_scales, FspadPaged paged, const fspad_bf16 *tk, const fspad_bf16 *tv, const int *parent,
                                       const int *prefix_len, int N, int B, fspad_bf16 *out, void *workspace, cudaStream_t st)
{
    const fspad_config &c = ctx->cfg;
    packed::Args a;
    a.q = q; a.kc = k_codes; a.ks = reinterpret_cast<const uint8_t *>(k_scales); a.vc = v_codes; a.vs = reinterpret_cast<const uint8_t *>(v_scales);
    a.table = paged.table; a.table_stride = paged.stride; a.n_blocks = paged.n_blocks;
    a.tk = tk; a.tv = tv; a.parent = parent; a.prefix_len = prefix_len;
    a.N = N; a.B = B; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads;
    a.M = N * a.G;
    a.by_G.set((unsigned)a.G);
    a.scale_log2 = ctx->scale * packed::kLog2e;
    a.out = out; a.status = ctx->d_status;
    CUtensorMap k_map;
    if (!fspad_make_tmap_u8_2d(&k_map, k_codes, (size_t)paged.n_blocks * c.n_kv_heads * 128, 128u)) return cudaErrorInvalidValue;
    return fspad_launch_attn_fp8_umma(ctx, a, k_map, 0, workspace, st);
}
