// Internal declarations of the query/key preparation and the window cache kernels.
#pragma once
#include <stdint.h>

#include <atomic>

#include "sh_internal.h"

// Kernel-side forms of the public structs: byte strides, resolved options.
struct WinRows {
    char *p;
    long long ts, hs;             // bytes between tokens, between heads
};

struct RopeParams {
    WinRows q, k, qo, ko;
    const int32_t *positions;     // [axes] rows, axis_stride apart
    long long axis_stride;
    const float *inv_freq;
    const void *qw, *kw;
    int tokens, q_heads, k_heads;
    int rot, axes, sec0, sec01;   // pairs [0, sec0) turn with axis 0, [sec0, sec01) with axis 1, the rest with axis 2
    int spread_h, spread_w;       // spread: 3 * sections[1], 3 * sections[2] (else 0 and `spread` false)
    int spread, adjacent;
    float eps;
    int hpw;                      // set by the launcher: head groups a warp walks through
};

struct WindowParams {
    WinRows q, k, v, out;
    char *kc, *vc;                // caches, or NULL
    long long css, chs, cls;      // bytes between sequences, heads, slots
    const int32_t *starts, *lengths;
    int tokens, sequences;
    int hq, hk, g;                // query heads, key heads, query heads per key head
    int window, sinks;
    float scale_log2e;
    RopeParams rope;              // decode only: how the step's q and k are prepared
    bool with_rope;
    float *part;                  // scratch of sh_window_decode_scratch or sh_window_prefill_scratch bytes, or NULL
};

// SMs of the current device, and that a kernel may use `smem` bytes of shared memory there.  Both are facts of the device, asked once
// (two threads that come first together both ask, and write the same).
struct ShKernelSetup {
    static constexpr int DEVICES = 64;
    std::atomic<bool> done[DEVICES];
};
cudaError_t sh_device_sms(int *dev, int *sms);
template <typename K>
cudaError_t sh_setup_kernel(ShKernelSetup &setup, K kern, size_t smem, int *sms) {
    int dev = 0;
    cudaError_t e = sh_device_sms(&dev, sms);
    if (e != cudaSuccess || (dev < ShKernelSetup::DEVICES && setup.done[dev].load(std::memory_order_relaxed))) return e;
    if (smem > 48 * 1024) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess && dev < ShKernelSetup::DEVICES) setup.done[dev].store(true, std::memory_order_relaxed);
    return e;
}

cudaError_t sh_launch_qk_norm_rope(RopeParams p, int dtype, int D, cudaStream_t s);
cudaError_t sh_launch_window_prefill_f32(const WindowParams &p, int D, cudaStream_t s);
// tensor cores: f16 and bf16
cudaError_t sh_launch_window_prefill_umma(const WindowParams &p, int dtype, int D, cudaStream_t s);
size_t sh_window_prefill_scratch(int tokens, int sequences, int hk, int g, int window, int sinks, bool with_cache, int dtype, int D);
// code of the first bounded wait that gave up in a window kernel of the current device since the last call (0: none); synchronises
cudaError_t sh_window_error_take(int *code, cudaStream_t s);
cudaError_t sh_launch_window_append(const WindowParams &p, int es, int D, cudaStream_t s);
size_t sh_window_decode_scratch(int sequences, int hk, int g, int dtype, int D);
cudaError_t sh_launch_window_decode(const WindowParams &p, int dtype, int D, cudaStream_t s);
