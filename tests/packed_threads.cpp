// Rotary calls of one context from several host threads, each with a theta of its own: stand-ins for the launchers, of which the rotary one looks at the
// frequencies that it is given.
#include <atomic>
#include <cmath>
#include <cstdlib>
#include <thread>
#include <vector>

#include "packed.cuh"

namespace {

std::atomic<long> g_wrong{0};
double theta_of(int thread) { return 1e4 * (1 + thread); }

}  // namespace

extern "C" {

// How many of the calls got other frequencies than their theta's (or were refused): `calls` each by `threads` threads.
long rotary_calls_at_once(int threads, int calls)
{
    fspad_ctx ctx{};
    ctx.cfg.n_q_heads = ctx.cfg.n_kv_heads = 1; ctx.cfg.head_dim = 128; ctx.cfg.max_nodes = ctx.cfg.n_layers = ctx.cfg.max_batch = 1;
    g_wrong = 0;
    std::vector<std::thread> all;
    for (int t = 0; t < threads; ++t)
        all.emplace_back([&ctx, t, calls] {
            auto at = [](int i) { return reinterpret_cast<fspad_bf16 *>((uintptr_t)(0x100000 * (i + 1))); };
            int32_t word = 0;
            for (int i = 0; i < calls; ++i)
                if (fspad_rope_qkv(&ctx, at(0), 3 * 128, nullptr, &word, &word, 1, 1, theta_of(t), 64, 0, 0, 0, at(1), at(2), at(3), reinterpret_cast<void *>((uintptr_t)t)) != 0) ++g_wrong;
        });
    for (auto &t : all) t.join();
    return g_wrong;
}
cudaError_t cudaGetDevice(int *d) { *d = 0; return cudaSuccess; }

}  // extern "C"

cudaError_t fspad_launch_rope_qkv(fspad_ctx *, const fspad_bf16 *, long long, const int *, const int *, const int *, int, int, const FspadRopeTable &t, bool, fspad_bf16 *, fspad_bf16 *,
                                  fspad_bf16 *, cudaStream_t st)
{
    const double theta = theta_of((int)reinterpret_cast<uintptr_t>(st));
    for (int i = 0; i < FSPAD_HEAD_DIM / 2; ++i) {
        const double want = std::pow(theta, -2.0 * i / FSPAD_HEAD_DIM) / (2.0 * 3.14159265358979323846);
        if (std::fabs(t.turns[i] - want) > 1e-14 * want) { ++g_wrong; break; }
    }
    return cudaSuccess;
}
cudaError_t fspad_launch_block_plan(fspad_ctx *, const int *, const int *, const int *, int, int, int, int *, int *, int *, int *, int, int *, long long *, int *, int *, cudaStream_t) { return cudaSuccess; }
cudaError_t fspad_launch_kv_write_packed(fspad_ctx *, const fspad_bf16 *, const fspad_bf16 *, const long long *, int, int, uint8_t *, uint8_t *, int, fspad_bf16 *, fspad_bf16 *, cudaStream_t) { return cudaSuccess; }
cudaError_t fspad_launch_kv_append_packed(fspad_ctx *, uint8_t *, uint8_t *, FspadPaged, const fspad_bf16 *, const int *, const int *, const int *, int, int, fspad_bf16 *, int *, cudaStream_t) { return cudaSuccess; }
size_t fspad_attn_packed_workspace(const fspad_ctx *, int, int) { return 0; }
bool fspad_attn_packed_fits(const fspad_ctx *, int, int, int) { return true; }
cudaError_t fspad_launch_tree_attn_packed(fspad_ctx *, const fspad_bf16 *, const uint8_t *, const uint8_t *, const uint8_t *, const uint8_t *, FspadPaged, const fspad_bf16 *, const fspad_bf16 *, const int *,
                                          const int *, int, int, fspad_bf16 *, void *, cudaStream_t) { return cudaSuccess; }
