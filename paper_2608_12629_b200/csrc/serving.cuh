// What the serving operators share: bf16 / e4m3 conversions, workspace header, host-side checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <limits.h>

#include <atomic>

#include "../../include/cake_serving.h"
#include "internal.h"
#include "ptx.cuh"

namespace cake {
namespace serving {

constexpr float kE4M3Max = 448.0f;
constexpr float kScaleMin = 7.888609052210118e-31f;   // 2^-100: the scale of a group of zeros; its reciprocal is finite

// Workspace header: 64 status words (word 0 is the sticky status), then arrival counters, one per CTA that can be the first
// of several to work on one output.  They are zero between calls, whatever sizes the calls have.
constexpr int kMaxCtas = 4096;
constexpr size_t kHeaderBytes = 256 + kMaxCtas * 4;
static_assert(kHeaderBytes == CAKE_SERVING_HEADER_BYTES, "header and ABI constant agree");

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// A number about a kernel on a device, asked for by the first launch there and kept.  Host threads that launch for the first time at once all ask,
// and get the same answer; an answer of 0 (the query failed) is not kept.
class PerDevice {
public:
    template <class Ask>
    int get(int device, Ask&& ask) {
        if (device < 0 || device >= kDevices) return ask();
        int v = known_[device].load(std::memory_order_acquire);
        if (v == 0 && (v = ask()) != 0) known_[device].store(v, std::memory_order_release);
        return v;
    }

private:
    static constexpr int kDevices = 64;
    std::atomic<int> known_[kDevices] = {};
};
// Room in shared memory for a kernel: 1, or 0 where the device refuses it.
template <class Kernel>
int allow_smem(Kernel kernel, size_t bytes) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)) == cudaSuccess) return 1;
    cudaGetLastError();
    return 0;
}

// Launch that may begin while the kernel ahead of it in the stream drains: the kernel waits for that one itself (ptx::grid_dep_wait,
// before its first access to global memory).  In a stream of short kernels this hides their launch.  Such a kernel runs while its
// inputs are still written, so it reads them by plain loads: none of them is constant for the kernel's whole life.  (Letting the
// next kernel go ahead from a kernel's first instruction on gains nothing more: norm and append of 16 rows 2.5 -> 3.2 us, decode of long 8-bit contexts
// 142 -> 159 us, whose next call's CTAs then take the SMs' places unevenly; the product alone keeps it, 17.8 -> 16.8 us for 517 rows.)
template <class... P, class... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, A&&... args) {
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
    if (e != cudaSuccess) cudaGetLastError();
    note_launches(1);
    return e;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float bf16_f(cake_bf16 v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {   // round to nearest even
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ cake_bf16 to_bf16(float v) { return static_cast<cake_bf16>(pack_bf16(v, 0.f) & 0xffffu); }
// two floats to e4m3, nearest even, values beyond 448 become 448, NaN stays NaN
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint32_t pack4_e4m3(float a, float b, float c, float d) {
    return pack_e4m3(a, b) | (pack_e4m3(c, d) << 16);
}
__device__ __forceinline__ void raise_bad_index(int* status) { atomicCAS(status, CAKE_OK, CAKE_ERR_BAD_INDEX); }

}  // namespace serving
}  // namespace cake
