// Keys and values of a paged cache read back by slots, 8-bit ones widened by their scales.
//
//   out[n][h] = bf16(cache[slot n][h] * scale[h])
//
// Bound by memory: a token's heads are read once and written once.  A thread has one place in a token's row, 16 elements of a head (8 where the outputs'
// alignment asks for it), and walks over tokens, several loads in flight.  It stores its 32 bytes at once: half as many instructions as for two stores of neighbouring threads,
// and whole sectors, which two stores of one thread are not.
//
// Measured (one B200): 100,001 8-bit tokens of 8 heads of 128 96 us = 6.4 TB/s, 98 % of a copy's rate (8 elements a thread 119 us, 16 in two stores 128); of a bf16 cache
// 124 us = 6.6 TB/s.  One sequence's 777 tokens 3.0 us, a launch's latency.
#include "serving.cuh"

namespace cake {
namespace serving {

int check_cache(const cake_paged_cache* c);   // kv_append.cu

namespace {

constexpr int READ_THREADS = 256;

struct ReadArgs {
    cake_paged_cache c;
    const long long* slots;
    cake_bf16 *out_k, *out_v;
    i64 N, stride, head_stride;
    int per_head, units, tokens;            // runs of a head, of a token in both matrices; tokens of a block's step
    int* status;
};

template <bool E4M3, int RUN, int BATCH>
__global__ void __launch_bounds__(READ_THREADS)
kv_read_kernel(const ReadArgs a) {
    constexpr int ELEM = E4M3 ? 1 : 2, WORDS = RUN * ELEM / 4;      // of the cache
    // the thread's place: (matrix, head, run)
    const int t = threadIdx.x / a.units, u = blockIdx.y * READ_THREADS + threadIdx.x - t * a.units;
    if (u >= a.units || t >= a.tokens) return;
    const int heads = u / a.per_head, d = (u - heads * a.per_head) * RUN;
    const bool is_v = a.out_k == nullptr || heads >= a.c.Hkv;
    const int h = a.out_k != nullptr && is_v ? heads - a.c.Hkv : heads;
    const i64 page_stride = is_v ? a.c.v_page_stride : a.c.k_page_stride, token_stride = is_v ? a.c.v_token_stride : a.c.k_token_stride;
    const char* const from = static_cast<const char*>(is_v ? a.c.v : a.c.k) + (h * (is_v ? a.c.v_head_stride : a.c.k_head_stride) + d) * ELEM;
    cake_bf16* const to = (is_v ? a.out_v : a.out_k) + h * a.head_stride + d;
    const float* const scales = E4M3 ? (is_v ? a.c.v_scale : a.c.k_scale) : nullptr;
    ptx::grid_dep_wait();
    const float scale = scales ? scales[h] : 1.f;
    const i64 first = static_cast<i64>(blockIdx.x) * a.tokens * BATCH + t;
    i64 slot[BATCH];
    uint32_t got[BATCH][WORDS];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
        const i64 n = first + b * a.tokens;
        slot[b] = n < a.N ? a.slots[n] : -1;
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
#pragma unroll
        for (int j = 0; j < WORDS; ++j) got[b][j] = 0u;
        // (32-bit division where it will do: the 64-bit one is a hundred instructions)
        const i64 page = (static_cast<unsigned long long>(slot[b]) >> 32) == 0 ? static_cast<unsigned>(slot[b]) / static_cast<unsigned>(a.c.page_size)
                                                                               : slot[b] / a.c.page_size;
        if (slot[b] >= 0 && page < a.c.num_pages) {
            const char* const at = from + (page * page_stride + (slot[b] - page * a.c.page_size) * token_stride) * ELEM;
            if (WORDS == 2) {
                const uint2 w = *reinterpret_cast<const uint2*>(at);
                got[b][0] = w.x, got[b][1] = w.y;
            } else {
#pragma unroll
                for (int j = 0; j < WORDS; j += 4) {
                    const uint4 w = *reinterpret_cast<const uint4*>(at + 4 * j);
                    got[b][j] = w.x, got[b][j + 1] = w.y, got[b][j + 2] = w.z, got[b][j + 3] = w.w;
                }
            }
        } else if (slot[b] >= 0) {
            raise_bad_index(a.status);
        }
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
        const i64 n = first + b * a.tokens;
        if (n >= a.N) break;
        uint32_t p[RUN / 2];
#pragma unroll
        for (int j = 0; j < RUN / 2; ++j) {
            if (E4M3) {
                const uint16_t pair = static_cast<uint16_t>(got[b][j >> 1] >> (16 * (j & 1)));
                uint32_t f16;
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(f16) : "h"(pair));
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&f16));
                p[j] = pack_bf16(f.x * scale, f.y * scale);
            } else {
                p[j] = got[b][j];
            }
        }
        cake_bf16* const dst = to + n * a.stride;
        if constexpr (RUN == 16)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"(dst), "r"(p[0]), "r"(p[1]), "r"(p[2]), "r"(p[3]), "r"(p[4]), "r"(p[5]), "r"(p[6]), "r"(p[7]) : "memory");
        else
            *reinterpret_cast<uint4*>(dst) = make_uint4(p[0], p[1], p[2], p[3]);
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
    // 16 elements a thread where it may store 32 bytes at once
    const bool wide = aligned(out_k, 32) && aligned(out_v, 32) && (N == 1 || out_stride % 16 == 0) && (cache->Hkv == 1 || out_head_stride % 16 == 0);
    a.per_head = cache->D / (wide ? 16 : 8);
    if (a.per_head > INT_MAX / 4 / cache->Hkv) return CAKE_ERR_SHAPE;
    a.units = a.per_head * cache->Hkv * (out_k && out_v ? 2 : 1);
    a.status = static_cast<int*>(ws);
    const unsigned parts = static_cast<unsigned>((a.units + READ_THREADS - 1) / READ_THREADS);
    if (parts > 65535) return CAKE_ERR_SHAPE;
    a.tokens = a.units < READ_THREADS ? READ_THREADS / a.units : 1;
    // Tokens to a thread: one while that leaves the SMs less than a few blocks each (latency: 777 tokens 3.4 us), else several, whose loads overlap: eight, or four of 64
    // bytes (100,001 8-bit tokens with four 98 us, with eight 96; bf16 ones 124 and 130)
    const i64 steps = (N + a.tokens - 1) / a.tokens;
    const bool few = steps * parts < 8 * di.sm_count;
    const int batch = few ? 1 : wide && !e4m3 ? 4 : 8;
    const i64 blocks = (steps + batch - 1) / batch;
    void (*const kernel)(const ReadArgs) =
        e4m3 ? (wide ? (few ? kv_read_kernel<true, 16, 1> : kv_read_kernel<true, 16, 8>) : (few ? kv_read_kernel<true, 8, 1> : kv_read_kernel<true, 8, 8>))
             : (wide ? (few ? kv_read_kernel<false, 16, 1> : kv_read_kernel<false, 16, 4>) : (few ? kv_read_kernel<false, 8, 1> : kv_read_kernel<false, 8, 8>));
    return launch_early(kernel, dim3(static_cast<unsigned>(blocks), parts), dim3(READ_THREADS), 0, reinterpret_cast<cudaStream_t>(stream), a) == cudaSuccess
               ? CAKE_OK : CAKE_ERR_CUDA;
}
