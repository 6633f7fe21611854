// Stand-ins for the device and the launchers of the operators around the 8-bit cache and on blocks, so that the checks of api_fp8.cu run without a device:
// each launch is written to a log and can be made to fail.
#include <string>

#include "fp8.cuh"

namespace {

std::string g_log;
int g_device = 0;
cudaError_t g_answer = cudaSuccess;
bool g_fits = true;

template <typename... T> cudaError_t call(const char *what, T... x)
{
    g_log += what;
    (void)std::initializer_list<int>{(g_log += " " + std::to_string(x), 0)...};
    g_log += "\n";
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
cudaError_t cudaGetDevice(int *d) { *d = g_device; return g_device < 0 ? cudaErrorNoDevice : cudaSuccess; }

}  // extern "C"

cudaError_t fspad_launch_kv_write_fp8(fspad_ctx *, const fspad_bf16 *, const fspad_bf16 *, const long long *, int rows, int layer, uint8_t *, float *, int n_blocks,
                                      fspad_bf16 *, fspad_bf16 *, cudaStream_t st) { return call("write", rows, layer, n_blocks, at(st)); }
cudaError_t fspad_launch_kv_append_fp8(fspad_ctx *, uint8_t *, float *, FspadPaged p, const fspad_bf16 *, const int *, const int *, const int *, int N, int B,
                                       fspad_bf16 *, int *, cudaStream_t st) { return call("append", p.stride, p.n_blocks, N, B, at(st)); }
size_t fspad_attn_fp8_workspace(const fspad_ctx *) { return 128000; }
bool fspad_attn_fp8_fits(const fspad_ctx *, int, int, int, int) { return g_fits; }
cudaError_t fspad_launch_tree_attn_fp8(fspad_ctx *, const fspad_bf16 *, const uint8_t *kc, const float *ks, const uint8_t *vc, const float *vs, FspadPaged,
                                       const fspad_bf16 *, const fspad_bf16 *, const int *, const int *, int N, int B, fspad_bf16 *, void *, cudaStream_t st)
{
    return call("attention", at(kc), at(ks), at(vc), at(vs), N, B, at(st));
}
cudaError_t fspad_launch_block_fork(fspad_ctx *, const FspadPool &p, const int *, const int *, int n, int *, int *, cudaStream_t st) { return call("fork", p.B, p.bps, p.n_blocks, n, at(st)); }
cudaError_t fspad_launch_block_free(fspad_ctx *, const FspadPool &p, const int *, cudaStream_t st) { return call("free", p.B, p.bps, p.n_blocks, at(st)); }
cudaError_t fspad_launch_block_compact(fspad_ctx *, const FspadPool &p, int *, int max_pairs, cudaStream_t st) { return call("compact", p.B, p.bps, p.n_blocks, max_pairs, at(st)); }
cudaError_t fspad_launch_block_copy(fspad_ctx *, void *, long long b0, void *, long long b1, int planes, int n_blocks, const int *, int n, cudaStream_t st)
{
    return call("copy", b0, b1, planes, n_blocks, n, at(st));
}
