// Keys and values of a paged cache read back by slots, 8-bit ones widened by their scales.
//
//   out[n][h] = bf16(cache[slot n][h] * scale[h])
//
// Bound by memory: a token's heads are read once and written once.  A thread moves runs of 8 (bf16) or 16 (e4m3) elements, 16 bytes a
// load, four loads in flight.
#include "serving.cuh"

namespace cake {
namespace serving {

int check_cache(const cake_paged_cache* c);   // kv_append.cu

namespace {

constexpr int READ_THREADS = 256, READ_BATCH = 4;

struct ReadArgs {
    cake_paged_cache c;
    const long long* slots;
    cake_bf16 *out_k, *out_v;
    i64 N, stride, head_stride, units;      // units: of all tokens, in both matrices
    int per_head, per_token;                // units of a head, of a token in one matrix
    int* status;
};

template <bool E4M3>
__global__ void __launch_bounds__(READ_THREADS)
kv_read_kernel(const ReadArgs a) {
    constexpr int RUN = E4M3 ? 16 : 8, ELEM = E4M3 ? 1 : 2;
    ptx::grid_dep_wait();
    // unit i of a block's stretch: (token, matrix, head, run), the runs of a token's head in one matrix next to each other
    const i64 first = static_cast<i64>(blockIdx.x) * (READ_THREADS * READ_BATCH) + threadIdx.x;
    const int both = a.out_v && a.out_k ? 2 : 1;
    uint4 got[READ_BATCH];
    cake_bf16* to[READ_BATCH];
    const float* scale[READ_BATCH];
#pragma unroll
    for (int b = 0; b < READ_BATCH; ++b) {
        const i64 i = first + b * READ_THREADS;
        to[b] = nullptr, scale[b] = nullptr;
        got[b] = make_uint4(0u, 0u, 0u, 0u);
        if (i >= a.units) continue;
        const int per = a.per_token * both;
        const i64 n = (static_cast<unsigned long long>(i) >> 32) == 0 ? static_cast<unsigned>(i) / static_cast<unsigned>(per) : i / per;
        int rest = static_cast<int>(i - n * per);
        const bool is_v = both == 2 ? rest >= a.per_token : a.out_v != nullptr;
        if (both == 2 && is_v) rest -= a.per_token;
        const int h = rest / a.per_head, d = (rest - h * a.per_head) * RUN;
        const i64 slot = a.slots[n];
        const i64 page = (static_cast<unsigned long long>(slot) >> 32) == 0 ? static_cast<unsigned>(slot) / static_cast<unsigned>(a.c.page_size)
                                                                            : slot / a.c.page_size;
        to[b] = (is_v ? a.out_v : a.out_k) + n * a.stride + h * a.head_stride + d;
        if (slot >= 0 && page < a.c.num_pages) {
            const i64 off = slot - page * a.c.page_size;
            const i64 at = is_v ? page * a.c.v_page_stride + off * a.c.v_token_stride + h * a.c.v_head_stride
                                : page * a.c.k_page_stride + off * a.c.k_token_stride + h * a.c.k_head_stride;
            got[b] = *reinterpret_cast<const uint4*>(static_cast<const char*>(is_v ? a.c.v : a.c.k) + (at + d) * ELEM);
            if (E4M3) {
                const float* s = is_v ? a.c.v_scale : a.c.k_scale;
                if (s) scale[b] = s + h;
            }
        } else if (slot >= 0) {
            raise_bad_index(a.status);
        }
    }
#pragma unroll
    for (int b = 0; b < READ_BATCH; ++b) {
        if (!to[b]) continue;
        if (E4M3) {
            const float s = scale[b] ? *scale[b] : 1.f;
            const uint32_t w[4] = {got[b].x, got[b].y, got[b].z, got[b].w};
            uint32_t p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint16_t pair = static_cast<uint16_t>(w[j >> 1] >> (16 * (j & 1)));
                uint32_t f16;
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(f16) : "h"(pair));
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&f16));
                p[j] = pack_bf16(f.x * s, f.y * s);
            }
            reinterpret_cast<uint4*>(to[b])[0] = make_uint4(p[0], p[1], p[2], p[3]);
            reinterpret_cast<uint4*>(to[b])[1] = make_uint4(p[4], p[5], p[6], p[7]);
        } else {
            *reinterpret_cast<uint4*>(to[b]) = got[b];
        }
    }
}

}  // namespace
}  // namespace serving
}  // namespace cake

using namespace cake;
using namespace cake::serving;

extern "C" int cake_kv_read(const cake_paged_cache* cache, const long long* slots, long long N, cake_bf16* out_k, cake_bf16* out_v,
                            long long out_stride, long long out_head_stride, void* ws, size_t ws_bytes, cake_stream_t stream) {
    int rc = check_cache(cache);
    if (rc != CAKE_OK) return rc;
    if (N < 0 || N > INT_MAX || (N > 1 && out_stride < cache->D) || (cache->Hkv > 1 && out_head_stride < cache->D)) return CAKE_ERR_SHAPE;
    if (!ws) return CAKE_ERR_NULL;
    if (!aligned(ws, 256)) return CAKE_ERR_ALIGN;
    if (ws_bytes < kHeaderBytes) return CAKE_ERR_WORKSPACE;
    if (N == 0 || (!out_k && !out_v)) return CAKE_OK;
    if (!slots) return CAKE_ERR_NULL;
    if (!aligned(slots, 8) || !aligned(out_k, 16) || !aligned(out_v, 16)) return CAKE_ERR_ALIGN;
    if ((N > 1 && out_stride % 8 != 0) || (cache->Hkv > 1 && out_head_stride % 8 != 0)) return CAKE_ERR_ALIGN;
    DeviceInfo di;
    rc = current_device_info(&di);
    if (rc != CAKE_OK) return rc;
    if (di.cc_major != 10) return CAKE_ERR_DEVICE;
    const bool e4m3 = cache->type == CAKE_KV_E4M3;
    ReadArgs a;
    a.c = *cache, a.slots = slots, a.out_k = out_k, a.out_v = out_v, a.N = N, a.stride = out_stride, a.head_stride = out_head_stride;
    a.per_head = cache->D / (e4m3 ? 16 : 8);
    if (a.per_head > INT_MAX / 2 / cache->Hkv) return CAKE_ERR_SHAPE;
    a.per_token = a.per_head * cache->Hkv;
    a.units = N * a.per_token * (out_k && out_v ? 2 : 1);
    a.status = static_cast<int*>(ws);
    const i64 blocks = (a.units + READ_THREADS * READ_BATCH - 1) / (READ_THREADS * READ_BATCH);
    if (blocks > INT_MAX) return CAKE_ERR_SHAPE;
    return launch_early(e4m3 ? kv_read_kernel<true> : kv_read_kernel<false>, dim3(static_cast<unsigned>(blocks)), dim3(READ_THREADS), 0,
                        reinterpret_cast<cudaStream_t>(stream), a) == cudaSuccess ? CAKE_OK : CAKE_ERR_CUDA;
}
