// Norms of each query and key head, rotation by position, and the write to a paged cache, in one pass.
//
//   y = x rsqrt(mean_d x_d^2 + eps) w;   (a, b) -> (a cos - b sin, b cos + a sin) for the pairs (i, i + rot/2) or (2i, 2i+1), i < rot/2
//
// Bound by memory: q, k, v are read once and written once (keys twice where they are asked for beside the cache).  A head lies in the
// registers of D/16 neighbouring lanes, 16 elements each: two runs of 8 that rotate into each other, so that the only exchange
// between lanes is the sum of squares (2 to 4 shuffles).  A thread keeps its place's cosines, sines and norm weights and walks over heads, four
// at a time.  Sums, norm and rotation in 32 bits, one rounding at the store.
//
// Measured (one B200): 16 tokens of 32 + 2 x 8 heads of 128 3.1 us, a launch's latency; 16,001 tokens 83 us = 5.25 TB/s, 80 % of a copy's rate; 5,000 tokens of
// 16 + 2 x 4 heads of 256 into an 8-bit cache 33 us.  Blocks of one warp: what a token needs before its heads (slot, position, angles, weights) is a chain
// of loads, and many short blocks hide it better than few long ones (16,001 tokens: 81 us by one warp, 95 by two, 107 by four).
#include "serving.cuh"

namespace cake {
namespace serving {

int check_cache(const cake_paged_cache* c);   // kv_append.cu

namespace {

struct NormArgs {
    cake_paged_cache c;
    const cake_bf16 *q, *k, *v, *q_weight, *k_weight;
    cake_bf16 *out_q, *out_k;
    const long long* slots;
    const int* positions;
    const float* cos_sin;
    i64 q_stride, k_stride, v_stride, max_positions, T;
    int Hq, rot;
    float eps;
    int* status;
};

// where a token's keys and values go
struct Place {
    bool rotate_ok, kv;
    i64 page;
    int off, pos;
};
__device__ __forceinline__ Place place_of(const NormArgs& a, i64 t, bool report) {
    Place p;
    p.pos = a.rot ? a.positions[t] : 0;
    p.rotate_ok = !a.rot || (p.pos >= 0 && p.pos < a.max_positions);
    const i64 slot = a.slots[t];
    // (32-bit division where it will do: the 64-bit one is a hundred instructions)
    const i64 page = (static_cast<unsigned long long>(slot) >> 32) == 0 ? static_cast<unsigned>(slot) / static_cast<unsigned>(a.c.page_size)
                                                                        : slot / a.c.page_size;
    p.kv = p.rotate_ok && slot >= 0 && page < a.c.num_pages;
    p.page = page;
    p.off = static_cast<int>(slot - page * a.c.page_size);
    if (report && (!p.rotate_ok || (slot >= 0 && page >= a.c.num_pages))) raise_bad_index(a.status);
    return p;
}

__device__ __forceinline__ void unpack8(const uint4& u, float (&f)[16], int at) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[at + 2 * j] = bf16_lo(w[j]), f[at + 2 * j + 1] = bf16_hi(w[j]);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[16], int at) {
    return make_uint4(pack_bf16(f[at], f[at + 1]), pack_bf16(f[at + 2], f[at + 3]), pack_bf16(f[at + 4], f[at + 5]), pack_bf16(f[at + 6], f[at + 7]));
}
template <bool E4M3>
__device__ __forceinline__ void store8(void* base, i64 to, const float (&f)[16], int at, float inv) {      // inv: 1 / scale
    if (E4M3) {
        *reinterpret_cast<uint2*>(static_cast<cake_e4m3*>(base) + to) =
            make_uint2(pack4_e4m3(f[at] * inv, f[at + 1] * inv, f[at + 2] * inv, f[at + 3] * inv),
                       pack4_e4m3(f[at + 4] * inv, f[at + 5] * inv, f[at + 6] * inv, f[at + 7] * inv));
    } else {
        *reinterpret_cast<uint4*>(static_cast<cake_bf16*>(base) + to) = pack8(f, at);
    }
}
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
    const float t = fmaf(a, c, __fmul_rn(b, -s));
    b = fmaf(b, c, __fmul_rn(a, s));
    a = t;
}

// Block (lanes of a head, heads in parallel, tokens).  L: lanes of a head, a power of two; D / 16 of them have elements.
template <bool E4M3, bool PAIRS, int L>
__global__ void __launch_bounds__(512)
qk_norm_kernel(const NormArgs a) {
    ptx::grid_dep_wait();
    const i64 t = static_cast<i64>(blockIdx.x) * blockDim.z + threadIdx.z;
    if (t >= a.T) return;
    const int u = threadIdx.x, D = a.c.D;
    const Place p = place_of(a, t, threadIdx.x == 0 && threadIdx.y == 0);
    if (!p.rotate_ok) return;
    const bool live = 16 * u < D;
    const int half = a.rot >> 1;
    // The two runs of 8 elements, neighbours in neighbouring lanes (runs of a lane beside each other would be loaded and stored in half sectors).
    // Pairs (i, i + rot/2): the first rot/16 lanes have those that rotate into each other
    const bool opposite = !PAIRS && 16 * u < a.rot;
    const int rest = PAIRS || opposite ? 0 : a.rot, v = u - (rest >> 4);
    const int d0 = rest + 8 * v, d1 = d0 + (opposite ? half : (D - rest) >> 1);
    const bool turn0 = live && (PAIRS ? d0 < a.rot : opposite), turn1 = live && PAIRS && d1 < a.rot;
    float cs[8], sn[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) cs[j] = 1.f, sn[j] = 0.f;
    const float* const angles = a.cos_sin + static_cast<i64>(p.pos) * a.rot;
    auto angle4 = [&](int at, int j) {
        const float4 c = *reinterpret_cast<const float4*>(angles + at), w = *reinterpret_cast<const float4*>(angles + half + at);
        cs[j] = c.x, cs[j + 1] = c.y, cs[j + 2] = c.z, cs[j + 3] = c.w;
        sn[j] = w.x, sn[j + 1] = w.y, sn[j + 2] = w.z, sn[j + 3] = w.w;
    };
    if (turn0) angle4(PAIRS ? d0 >> 1 : d0, 0);
    if (PAIRS ? turn1 : turn0) angle4(PAIRS ? d1 >> 1 : d0 + 4, 4);
    constexpr uint32_t kOnes = 0x3f803f80u;
    uint4 wq[2], wk[2];
    wq[0] = wq[1] = wk[0] = wk[1] = make_uint4(kOnes, kOnes, kOnes, kOnes);
    if (live && a.q_weight) wq[0] = *reinterpret_cast<const uint4*>(a.q_weight + d0), wq[1] = *reinterpret_cast<const uint4*>(a.q_weight + d1);
    if (live && a.k_weight) wk[0] = *reinterpret_cast<const uint4*>(a.k_weight + d0), wk[1] = *reinterpret_cast<const uint4*>(a.k_weight + d1);
    const int linear = threadIdx.x + L * (threadIdx.y + blockDim.y * threadIdx.z);
    const unsigned group = (L == 32 ? ~0u : (1u << L) - 1) << (linear & 31 & ~(L - 1));      // the lanes of the head: one path through the code
    const int Hkv = a.c.Hkv, heads = a.Hq + (p.kv ? 2 : a.out_k ? 1 : 0) * Hkv;
    constexpr int BATCH = 4;
    for (int h0 = threadIdx.y; h0 < heads; h0 += BATCH * blockDim.y) {
        uint4 x0[BATCH], x1[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int h = h0 + b * blockDim.y;
            x0[b] = x1[b] = make_uint4(0u, 0u, 0u, 0u);
            if (h >= heads || !live) continue;
            const cake_bf16* src = h < a.Hq ? a.q + t * a.q_stride + static_cast<i64>(h) * D
                                 : h < a.Hq + Hkv ? a.k + t * a.k_stride + static_cast<i64>(h - a.Hq) * D
                                                  : a.v + t * a.v_stride + static_cast<i64>(h - a.Hq - Hkv) * D;
            x0[b] = *reinterpret_cast<const uint4*>(src + d0);
            x1[b] = *reinterpret_cast<const uint4*>(src + d1);
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int h = h0 + b * blockDim.y;
            if (h >= heads) break;
            const bool is_q = h < a.Hq, is_v = h >= a.Hq + Hkv;
            const int g = h - a.Hq - (is_v ? Hkv : 0);
            float f[16];
            unpack8(x0[b], f, 0);
            unpack8(x1[b], f, 8);
            if (!is_v) {
                float sum = 0.f, sum1 = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = fmaf(f[j], f[j], sum), sum1 = fmaf(f[8 + j], f[8 + j], sum1);
                sum += sum1;
#pragma unroll
                for (int o = 1; o < L; o <<= 1) sum += __shfl_xor_sync(group, sum, o);
                const float r = rsqrtf(sum / static_cast<float>(D) + a.eps);
                float w[16];
                unpack8(is_q ? wq[0] : wk[0], w, 0);
                unpack8(is_q ? wq[1] : wk[1], w, 8);
#pragma unroll
                for (int j = 0; j < 16; ++j) f[j] *= r * w[j];
                if (PAIRS) {
                    if (turn0)
#pragma unroll
                        for (int j = 0; j < 8; ++j) turn(f[2 * j], f[2 * j + 1], cs[j], sn[j]);      // (an angle of 0 where the second run does not turn)
                } else if (turn0) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) turn(f[j], f[8 + j], cs[j], sn[j]);
                }
            }
            if (!live) continue;
            if (is_q) {
                cake_bf16* dst = a.out_q + (t * a.Hq + h) * static_cast<i64>(D);
                *reinterpret_cast<uint4*>(dst + d0) = pack8(f, 0);
                *reinterpret_cast<uint4*>(dst + d1) = pack8(f, 8);
                continue;
            }
            if (!is_v && a.out_k) {
                cake_bf16* dst = a.out_k + (t * Hkv + g) * static_cast<i64>(D);
                *reinterpret_cast<uint4*>(dst + d0) = pack8(f, 0);
                *reinterpret_cast<uint4*>(dst + d1) = pack8(f, 8);
            }
            if (!p.kv) continue;
            const i64 at = is_v ? p.page * a.c.v_page_stride + p.off * a.c.v_token_stride + g * a.c.v_head_stride
                                : p.page * a.c.k_page_stride + p.off * a.c.k_token_stride + g * a.c.k_head_stride;
            const float* scale = is_v ? a.c.v_scale : a.c.k_scale;
            const float inv = E4M3 && scale ? 1.f / scale[g] : 1.f;
            void* const base = is_v ? a.c.v : a.c.k;
            store8<E4M3>(base, at + d0, f, 0, inv);
            store8<E4M3>(base, at + d1, f, 8, inv);
        }
    }
}

// Any rot, any alignment: a warp to a head, one pair of elements (or one element that does not rotate) per lane and step.
template <bool E4M3>
__global__ void __launch_bounds__(256)
qk_norm_scalar_kernel(const NormArgs a, bool pairs) {
    ptx::grid_dep_wait();
    const i64 t = blockIdx.x;
    const int lane = threadIdx.x & 31;
    const Place p = place_of(a, t, threadIdx.x == 0);
    if (!p.rotate_ok) return;
    const int D = a.c.D, half = a.rot >> 1, Hkv = a.c.Hkv;
    const int units = half + (D - a.rot);
    auto put = [&](void* base, i64 at, float f, float inv) {      // inv: 1 / scale
        if (E4M3) static_cast<cake_e4m3*>(base)[at] = static_cast<cake_e4m3>(pack_e4m3(f * inv, 0.f) & 0xff);
        else static_cast<cake_bf16*>(base)[at] = to_bf16(f);
    };
    const int heads = a.Hq + (p.kv ? 2 : a.out_k ? 1 : 0) * Hkv;
    for (int h = threadIdx.x >> 5; h < heads; h += blockDim.x >> 5) {
        const bool is_q = h < a.Hq, is_v = h >= a.Hq + Hkv;
        const int g = h - a.Hq - (is_v ? Hkv : 0);
        const cake_bf16* src = is_q ? a.q + t * a.q_stride + static_cast<i64>(h) * D
                             : is_v ? a.v + t * a.v_stride + static_cast<i64>(g) * D : a.k + t * a.k_stride + static_cast<i64>(g) * D;
        if (is_v) {
            const i64 at = p.page * a.c.v_page_stride + p.off * a.c.v_token_stride + g * a.c.v_head_stride;
            const float inv = E4M3 && a.c.v_scale ? 1.f / a.c.v_scale[g] : 1.f;
            for (int d = lane; d < D; d += 32) put(a.c.v, at + d, bf16_f(src[d]), inv);
            continue;
        }
        float sum = 0.f;
        for (int d = lane; d < D; d += 32) sum = fmaf(bf16_f(src[d]), bf16_f(src[d]), sum);
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float r = rsqrtf(sum / static_cast<float>(D) + a.eps);
        const cake_bf16* w = is_q ? a.q_weight : a.k_weight;
        const i64 at = p.page * a.c.k_page_stride + p.off * a.c.k_token_stride + g * a.c.k_head_stride;
        const float inv = E4M3 && a.c.k_scale && !is_q ? 1.f / a.c.k_scale[g] : 1.f;
        cake_bf16* const dense = is_q ? a.out_q + (t * a.Hq + h) * static_cast<i64>(D) : a.out_k ? a.out_k + (t * Hkv + g) * static_cast<i64>(D) : nullptr;
        for (int u = lane; u < units; u += 32) {
            const bool turns = u < half;
            const int d = turns ? (pairs ? 2 * u : u) : a.rot + (u - half);
            const int e = pairs ? d + 1 : d + half;
            float x = bf16_f(src[d]) * (r * (w ? bf16_f(w[d]) : 1.f)), y = 0.f;
            if (turns) {
                const float* row = a.cos_sin + static_cast<i64>(p.pos) * a.rot;
                y = bf16_f(src[e]) * (r * (w ? bf16_f(w[e]) : 1.f));
                turn(x, y, row[u], row[half + u]);
            }
            if (dense) {
                dense[d] = to_bf16(x);
                if (turns) dense[e] = to_bf16(y);
            }
            if (!is_q && p.kv) {
                put(a.c.k, at + d, x, inv);
                if (turns) put(a.c.k, at + e, y, inv);
            }
        }
    }
}

template <bool E4M3, bool PAIRS>
void (*kernel_of(int D))(const NormArgs) {
    switch (D) {
        case 64: return qk_norm_kernel<E4M3, PAIRS, 4>;
        case 256: return qk_norm_kernel<E4M3, PAIRS, 16>;
        default: return qk_norm_kernel<E4M3, PAIRS, 8>;      // 96: six of the eight lanes
    }
}

}  // namespace
}  // namespace serving
}  // namespace cake

using namespace cake;
using namespace cake::serving;

extern "C" int cake_qk_norm_append(const cake_paged_cache* cache, const cake_bf16* q, long long q_stride, int Hq, const cake_bf16* k,
                                   long long k_stride, const cake_bf16* v, long long v_stride, const cake_bf16* q_weight,
                                   const cake_bf16* k_weight, float eps, cake_bf16* out_q, cake_bf16* out_k, const long long* slots,
                                   const int* positions, const float* cos_sin, long long max_positions, int rot, long long T, void* ws,
                                   size_t ws_bytes, cake_stream_t stream, unsigned flags) {
    int rc = check_cache(cache);
    if (rc != CAKE_OK) return rc;
    const int D = cache->D;
    const i64 kv_row = static_cast<i64>(cache->Hkv) * D;
    if (T < 0 || T > INT_MAX || rot < 0 || rot % 2 != 0 || rot > D || Hq < 1) return CAKE_ERR_SHAPE;
    if (k_stride < kv_row || v_stride < kv_row || q_stride < static_cast<i64>(Hq) * D) return CAKE_ERR_SHAPE;
    if (rot && max_positions < 1) return CAKE_ERR_SHAPE;
    if ((flags & ~CAKE_APPEND_INTERLEAVED) != 0) return CAKE_ERR_UNSUPPORTED;
    if (!ws) return CAKE_ERR_NULL;
    if (!aligned(ws, 256)) return CAKE_ERR_ALIGN;
    if (ws_bytes < kHeaderBytes) return CAKE_ERR_WORKSPACE;
    if (T == 0) return CAKE_OK;
    if (!q || !k || !v || !slots || !out_q || (rot && (!positions || !cos_sin))) return CAKE_ERR_NULL;
    for (const void* p : {static_cast<const void*>(q), static_cast<const void*>(k), static_cast<const void*>(v), static_cast<const void*>(q_weight),
                          static_cast<const void*>(k_weight), static_cast<const void*>(out_q), static_cast<const void*>(out_k)})
        if (!aligned(p, 2)) return CAKE_ERR_ALIGN;
    if (!aligned(slots, 8) || !aligned(positions, 4) || !aligned(cos_sin, 4)) return CAKE_ERR_ALIGN;
    DeviceInfo di;
    rc = current_device_info(&di);
    if (rc != CAKE_OK) return rc;
    if (di.cc_major != 10) return CAKE_ERR_DEVICE;
    NormArgs a;
    a.c = *cache, a.q = q, a.k = k, a.v = v, a.q_weight = q_weight, a.k_weight = k_weight, a.out_q = out_q, a.out_k = out_k;
    a.slots = slots, a.positions = positions, a.cos_sin = cos_sin, a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
    a.max_positions = max_positions, a.T = T, a.Hq = Hq, a.rot = rot, a.eps = eps, a.status = static_cast<int*>(ws);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool pairs = flags & CAKE_APPEND_INTERLEAVED, e4m3 = cache->type == CAKE_KV_E4M3;
    bool wide = (pairs ? rot % 8 == 0 : rot % 16 == 0) && q_stride % 8 == 0 && k_stride % 8 == 0 && v_stride % 8 == 0 && aligned(cos_sin, 16);
    for (const void* p : {static_cast<const void*>(q), static_cast<const void*>(k), static_cast<const void*>(v), static_cast<const void*>(q_weight),
                          static_cast<const void*>(k_weight), static_cast<const void*>(out_q), static_cast<const void*>(out_k)})
        wide = wide && aligned(p, 16);
    const unsigned blocks = static_cast<unsigned>(T);
    cudaError_t e;
    if (wide) {
        const int lanes = D == 64 ? 4 : D == 256 ? 16 : 8;
        const int heads = Hq + 2 * cache->Hkv;
        // Few tokens: a head to a group of lanes (latency).  More: four heads to a group, whose loads overlap and share the token's angles and weights, in blocks of
        // 128 threads and, where those are plenty, of a single warp.  32 + 2 * 8 heads of 128, bf16 cache, us by a head to a group, 128 threads and a warp: 128 tokens 2.7,
        // 3.5 and 6.8; 192 4.4, 3.7 and 6.7; 512 12, 5.6 and 9.1; 1,024 22, 10.6 and 10.4; 1,500 32, 13.2 and 11.7; 2,048 42, 16.4 and 13.1; 4,096 82, 30 and 24; 16,001 310,
        // 104 and 80 (16 + 2 * 4 heads of 256 and 64 + 2 * 8 of 128 into 8-bit caches change places at the same sizes).  8 + 2 * 2 heads of 64: 512 2.5, 3.7 and 3.7;
        // 1,500 4.6, 3.9 and 4.0; 16,001 40, 17.8 and 20.7
        int par, tokens = 1;
        if (T <= 128) {
            par = heads * lanes <= 512 ? heads : 512 / lanes;
            while (par * lanes % 32 != 0 && par * lanes < 512) ++par;      // (whole warps: shuffles name lanes of the head alone, but the rest is idle)
        } else {
            const int target = T >= 2048 ? 32 : 128, most = target / lanes;
            par = (heads + 3) / 4 <= most ? (heads + 3) / 4 : most;
            tokens = target / (lanes * par) > 0 ? target / (lanes * par) : 1;
        }
        void (*const kernel)(const NormArgs) = e4m3 ? (pairs ? kernel_of<true, true>(D) : kernel_of<true, false>(D))
                                                    : (pairs ? kernel_of<false, true>(D) : kernel_of<false, false>(D));
        e = launch_early(kernel, dim3((blocks + tokens - 1) / tokens), dim3(lanes, par, tokens), 0, s, a);
    } else {
        e = launch_early(e4m3 ? qk_norm_scalar_kernel<true> : qk_norm_scalar_kernel<false>, dim3(blocks), dim3(256), 0, s, a, pairs);
    }
    return e == cudaSuccess ? CAKE_OK : CAKE_ERR_CUDA;
}
