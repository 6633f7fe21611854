// Stand-ins for the device and the launchers of the operators around the 4-bit cache, so that the checks of api_cache.cu run without a device:
// each launch is written to a log and can be made to fail.
#include <cstdio>
#include <cstring>
#include <string>

#include "packed.cuh"

namespace {

std::string g_log;
int g_device = 0;
cudaError_t g_answer = cudaSuccess;
bool g_fits = true;
FspadRopeTable g_table;

cudaError_t call(const std::string &what)
{
    g_log += what + "\n";
    return g_answer;
}
unsigned long long at(const void *p) { return (unsigned long long)(uintptr_t)p; }

}  // namespace

extern "C" {

void *fake_context(int hq, int hkv, int max_nodes, int layers, int max_batch)
{
    auto *c = new fspad_ctx();
    c->cfg.n_q_heads = hq; c->cfg.n_kv_heads = hkv; c->cfg.head_dim = 128; c->cfg.max_nodes = max_nodes; c->cfg.n_layers = layers;
    c->cfg.max_batch = max_batch;
    return c;
}
void fake_context_free(void *c) { delete static_cast<fspad_ctx *>(c); }
const char *fake_log() { return g_log.c_str(); }
void fake_set(int device, int fails, int fits)
{
    g_log.clear();
    g_device = device;
    g_answer = fails ? cudaErrorUnknown : cudaSuccess;
    g_fits = fits != 0;
}
double fake_turns(int i) { return g_table.turns[i]; }
cudaError_t cudaGetDevice(int *d) { *d = g_device; return g_device < 0 ? cudaErrorNoDevice : cudaSuccess; }

}  // extern "C"

cudaError_t fspad_launch_rope_qkv(fspad_ctx *, const fspad_bf16 *, long long row_stride, const int *positions, const int *, const int *, int N,
                                  int B, const FspadRopeTable &t, bool adjacent, fspad_bf16 *, fspad_bf16 *, fspad_bf16 *, cudaStream_t st)
{
    g_table = t;
    return call("rope " + std::to_string(row_stride) + (positions ? " given" : " tree") + " " + std::to_string(N) + " " + std::to_string(B) + " " +
                std::to_string(t.split0) + " " + std::to_string(t.split1) + (adjacent ? " adjacent" : " halves") + " " + std::to_string(at(st)));
}
cudaError_t fspad_launch_block_plan(fspad_ctx *, const int *, const int *, const int *, int B, int bps, int n_blocks, int *, int *, int *, int *,
                                    int max_rows, int *, long long *, int *, int *, cudaStream_t)
{
    return call("plan " + std::to_string(B) + " " + std::to_string(bps) + " " + std::to_string(n_blocks) + " " + std::to_string(max_rows));
}
cudaError_t fspad_launch_kv_write_packed(fspad_ctx *, const fspad_bf16 *, const fspad_bf16 *, const long long *, int rows, int layer, uint8_t *,
                                         uint8_t *, int n_blocks, fspad_bf16 *, fspad_bf16 *, cudaStream_t)
{
    return call("write " + std::to_string(rows) + " " + std::to_string(layer) + " " + std::to_string(n_blocks));
}
cudaError_t fspad_launch_kv_append_packed(fspad_ctx *, uint8_t *, uint8_t *, FspadPaged p, const fspad_bf16 *, const int *, const int *, const int *,
                                          int N, int B, fspad_bf16 *, int *, cudaStream_t)
{
    return call("append " + std::to_string(p.stride) + " " + std::to_string(N) + " " + std::to_string(B));
}
size_t fspad_attn_packed_workspace(const fspad_ctx *, int N, int B) { return (size_t)N * B * 1000; }
bool fspad_attn_packed_fits(const fspad_ctx *, int, int, int) { return g_fits; }
cudaError_t fspad_launch_tree_attn_packed(fspad_ctx *, const fspad_bf16 *, const uint8_t *kc, const uint8_t *ks, const uint8_t *vc, const uint8_t *vs,
                                          FspadPaged, const fspad_bf16 *, const fspad_bf16 *, const int *, const int *, int N, int B, fspad_bf16 *,
                                          void *, cudaStream_t)
{
    return call("attention " + std::to_string(at(kc)) + " " + std::to_string(at(ks)) + " " + std::to_string(at(vc)) + " " + std::to_string(at(vs)) +
                " " + std::to_string(N) + " " + std::to_string(B));
}
