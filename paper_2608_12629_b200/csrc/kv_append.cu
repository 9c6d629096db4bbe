// Keys and values of new tokens into a paged cache, keys and queries rotated by their positions on the way.
//
//   (a, b) -> (a cos - b sin, b cos + a sin) for the pairs (i, i + rot/2) or (2i, 2i+1) of a head's first `rot` elements
//
// Bound by memory: q, k, v are read once and written once.  A thread keeps the cosines and sines of its place in a head
// and walks over heads, four at a time, so the table is read once per token and group of threads, not once per head.
// Measured: 16,001 tokens of 32 + 2 * 8 heads of 128, half of each rotated, into an 8-bit cache 63 us, 5.82 TB/s, 89 % of the copy
// rate; 16,384 tokens into a bf16 cache 69 us, 91 %; 16 tokens 2.5 us.  A value goes into an 8-bit cache as x * (1 / scale): a rounding of 2^-24 more than
// x / scale, far below the format's 2^-4, and one division for eight elements.
#include "serving.cuh"

namespace cake {
namespace serving {
namespace {

struct AppendArgs {
    cake_paged_cache c;
    const cake_bf16* k;
    const cake_bf16* v;
    const cake_bf16* q;
    cake_bf16* out_q;
    const long long* slots;
    const int* positions;
    const float* cos_sin;
    i64 k_stride, v_stride, q_stride, max_positions, T;
    int Hq, rot;
    int* status;
};

// where a token's keys and values go; false: nowhere
struct Place {
    bool rotate_ok, kv;
    i64 page;
    int off, pos;
};
__device__ __forceinline__ Place place_of(const AppendArgs& a, i64 t, bool report) {
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

__device__ __forceinline__ void unpack8(const uint4& u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[2 * j] = bf16_lo(w[j]), f[2 * j + 1] = bf16_hi(w[j]);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
template <bool E4M3>
__device__ __forceinline__ void store8(void* base, i64 at, const float (&f)[8], float inv) {      // inv: 1 / scale
    if (E4M3) {
        *reinterpret_cast<uint2*>(static_cast<cake_e4m3*>(base) + at) =
            make_uint2(pack4_e4m3(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv),
                       pack4_e4m3(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
    } else {
        *reinterpret_cast<uint4*>(static_cast<cake_bf16*>(base) + at) = pack8(f);
    }
}

// (a, b) -> (a c - b s, b c + a s): the roundings of turn2, so that a token's bits do not depend on the alignment of its sources
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
    const float t = fmaf(a, c, __fmul_rn(b, -s));
    b = fmaf(b, c, __fmul_rn(a, s));
    a = t;
}
// the same for two pairs at a time (packed instructions: issue is half of what bounds the kernel)
__device__ __forceinline__ void turn2(float& a0, float& a1, float& b0, float& b1, float c0, float c1, float s0, float s1) {
    asm("{\n\t.reg .b64 a, b, c, s, t, u, n;\n\t"
        "mov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\tmov.b64 c, {%4, %5};\n\tmov.b64 s, {%6, %7};\n\tmov.b64 n, {%8, %9};\n\t"
        "mul.rn.f32x2 t, b, n;\n\tfma.rn.f32x2 t, a, c, t;\n\t"
        "mul.rn.f32x2 u, a, s;\n\tfma.rn.f32x2 u, b, c, u;\n\t"
        "mov.b64 {%0, %1}, t;\n\tmov.b64 {%2, %3}, u;\n\t}"
        : "+f"(a0), "+f"(a1), "+f"(b0), "+f"(b1) : "f"(c0), "f"(c1), "f"(s0), "f"(s1), "f"(-s0), "f"(-s1));
}

// Block (units, heads in parallel, tokens): thread (u, y, z) takes of token z unit u of the heads y, y + blockDim.y, ... of the token's
// Hq query, Hkv key and Hkv value heads, four heads' loads in flight.  A unit is 8 neighbouring elements, or two such runs rot/2
// apart that rotate into each other (PAIRS false, the first rot/16 units of a head).
template <bool E4M3, bool PAIRS>
__global__ void __launch_bounds__(288)
kv_append_kernel(const AppendArgs a) {
    const i64 t = static_cast<i64>(blockIdx.x) * blockDim.z + threadIdx.z;
    if (t >= a.T) return;
    const int u = threadIdx.x;
    ptx::grid_dep_wait();
    const Place p = place_of(a, t, threadIdx.x == 0 && threadIdx.y == 0);
    if (!p.rotate_ok) return;
    const int D = a.c.D, half = a.rot >> 1;
    const int turning = PAIRS ? a.rot >> 3 : a.rot >> 4;              // units that rotate
    const bool turns = u < turning;
    const int d0 = (PAIRS || turns) ? 8 * u : a.rot + 8 * (u - turning);
    const bool two = !PAIRS && turns;
    float cs[8], sn[8];
    if (turns) {
        const float* row = a.cos_sin + static_cast<i64>(p.pos) * a.rot;
        constexpr int N = PAIRS ? 4 : 8;
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const float4 c = *reinterpret_cast<const float4*>(row + N * u + j), w = *reinterpret_cast<const float4*>(row + half + N * u + j);
            cs[j] = c.x, cs[j + 1] = c.y, cs[j + 2] = c.z, cs[j + 3] = c.w;
            sn[j] = w.x, sn[j + 1] = w.y, sn[j + 2] = w.z, sn[j + 3] = w.w;
        }
    }
    const int hq = a.q ? a.Hq : 0;
    const int heads = hq + (p.kv ? 2 * a.c.Hkv : 0);
    constexpr int BATCH = 4;
    for (int h0 = threadIdx.y; h0 < heads; h0 += BATCH * blockDim.y) {
        uint4 lo[BATCH], hi[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int h = h0 + k * blockDim.y;
            if (h >= heads) break;
            const cake_bf16* src = h < hq ? a.q + t * a.q_stride + static_cast<i64>(h) * D
                                 : h < hq + a.c.Hkv ? a.k + t * a.k_stride + static_cast<i64>(h - hq) * D
                                                    : a.v + t * a.v_stride + static_cast<i64>(h - hq - a.c.Hkv) * D;
            lo[k] = *reinterpret_cast<const uint4*>(src + d0);
            if (two) hi[k] = *reinterpret_cast<const uint4*>(src + d0 + half);
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int h = h0 + k * blockDim.y;
            if (h >= heads) break;
            const bool is_q = h < hq, is_v = h >= hq + a.c.Hkv;
            const int g = h - hq - (is_v ? a.c.Hkv : 0);
            float x[8], y[8];
            unpack8(lo[k], x);
            if (two) unpack8(hi[k], y);
            if (turns && !is_v) {
                if (!PAIRS) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) turn2(x[j], x[j + 1], y[j], y[j + 1], cs[j], cs[j + 1], sn[j], sn[j + 1]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) turn(x[2 * j], x[2 * j + 1], cs[j], sn[j]);
                }
            }
            if (is_q) {
                cake_bf16* dst = a.out_q + (t * a.Hq + h) * static_cast<i64>(D) + d0;
                *reinterpret_cast<uint4*>(dst) = pack8(x);
                if (two) *reinterpret_cast<uint4*>(dst + half) = pack8(y);
            } else {
                const i64 at = is_v ? p.page * a.c.v_page_stride + p.off * a.c.v_token_stride + g * a.c.v_head_stride + d0
                                    : p.page * a.c.k_page_stride + p.off * a.c.k_token_stride + g * a.c.k_head_stride + d0;
                const float* scale = is_v ? a.c.v_scale : a.c.k_scale;
                const float inv = E4M3 && scale ? 1.f / scale[g] : 1.f;
                void* const base = is_v ? a.c.v : a.c.k;
                store8<E4M3>(base, at, x, inv);
                if (two) store8<E4M3>(base, at + half, y, inv);
            }
        }
    }
}

// Any rot, any alignment of q, k, v: one pair of elements (or one element that does not rotate) per thread and step.
template <bool E4M3>
__global__ void __launch_bounds__(256)
kv_append_scalar_kernel(const AppendArgs a, bool pairs) {
    const i64 t = blockIdx.x;
    ptx::grid_dep_wait();
    const Place p = place_of(a, t, threadIdx.x == 0);
    if (!p.rotate_ok) return;
    const int D = a.c.D, half = a.rot >> 1;
    const int units = half + (D - a.rot);
    const int hq = a.q ? a.Hq : 0;
    auto put = [&](void* base, i64 at, float f, float inv) {      // inv: 1 / scale
        if (E4M3) static_cast<cake_e4m3*>(base)[at] = static_cast<cake_e4m3>(pack_e4m3(f * inv, 0.f) & 0xff);
        else static_cast<cake_bf16*>(base)[at] = to_bf16(f);
    };
    for (int i = threadIdx.x; i < (hq + a.c.Hkv) * units; i += blockDim.x) {
        const int h = i / units, u = i - h * units, g = h - hq;
        const bool is_q = h < hq, turns = u < half;
        if (!is_q && !p.kv) continue;
        const cake_bf16* src = is_q ? a.q + t * a.q_stride + static_cast<i64>(h) * D : a.k + t * a.k_stride + static_cast<i64>(g) * D;
        const int d = turns ? (pairs ? 2 * u : u) : a.rot + (u - half);
        const int e = pairs ? d + 1 : d + half;
        float x = bf16_f(src[d]), y = 0.f;
        if (turns) {
            const float* row = a.cos_sin + static_cast<i64>(p.pos) * a.rot;
            y = bf16_f(src[e]);
            turn(x, y, row[u], row[half + u]);
        }
        if (is_q) {
            cake_bf16* dst = a.out_q + (t * a.Hq + h) * static_cast<i64>(D);
            dst[d] = to_bf16(x);
            if (turns) dst[e] = to_bf16(y);
        } else {
            const i64 at = p.page * a.c.k_page_stride + p.off * a.c.k_token_stride + g * a.c.k_head_stride;
            const float inv = E4M3 && a.c.k_scale ? 1.f / a.c.k_scale[g] : 1.f;
            put(a.c.k, at + d, x, inv);
            if (turns) put(a.c.k, at + e, y, inv);
        }
    }
    if (!p.kv) return;
    for (int i = threadIdx.x; i < a.c.Hkv * D; i += blockDim.x) {
        const int g = i / D, d = i - g * D;
        const i64 at = p.page * a.c.v_page_stride + p.off * a.c.v_token_stride + g * a.c.v_head_stride + d;
        put(a.c.v, at, bf16_f(a.v[t * a.v_stride + static_cast<i64>(g) * D + d]), E4M3 && a.c.v_scale ? 1.f / a.c.v_scale[g] : 1.f);
    }
}

}  // namespace

int check_cache(const cake_paged_cache* c) {
    if (!c || !c->k || !c->v) return CAKE_ERR_NULL;
    if (c->num_pages < 1 || c->page_size < 1 || c->Hkv < 1 || c->D < 1) return CAKE_ERR_SHAPE;
    if (c->num_pages > INT_MAX || c->num_pages > LLONG_MAX / 2 / c->page_size) return CAKE_ERR_SHAPE;
    if (c->type != CAKE_KV_BF16 && c->type != CAKE_KV_E4M3) return CAKE_ERR_UNSUPPORTED;
    if (c->D != 64 && c->D != 96 && c->D != 128 && c->D != 256) return CAKE_ERR_UNSUPPORTED;
    const i64 per16 = c->type == CAKE_KV_BF16 ? 8 : 16;
    const i64 st[6] = {c->k_page_stride, c->k_token_stride, c->k_head_stride, c->v_page_stride, c->v_token_stride, c->v_head_stride};
    for (i64 s : st) {
        if (s < 0) return CAKE_ERR_SHAPE;
        if (s % per16 != 0) return CAKE_ERR_ALIGN;
    }
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return CAKE_ERR_ALIGN;
    return CAKE_OK;
}

}  // namespace serving
}  // namespace cake

using namespace cake;
using namespace cake::serving;

extern "C" int cake_kv_append(const cake_paged_cache* cache, const cake_bf16* k, long long k_stride, const cake_bf16* v,
                              long long v_stride, const cake_bf16* q, long long q_stride, int Hq, cake_bf16* out_q,
                              const long long* slots, const int* positions, const float* cos_sin, long long max_positions, int rot,
                              long long T, void* ws, size_t ws_bytes, cake_stream_t stream, unsigned flags) {
    int rc = check_cache(cache);
    if (rc != CAKE_OK) return rc;
    const i64 kv_row = static_cast<i64>(cache->Hkv) * cache->D;
    if (T < 0 || T > INT_MAX || rot < 0 || rot % 2 != 0 || rot > cache->D || k_stride < kv_row || v_stride < kv_row) return CAKE_ERR_SHAPE;
    if (q && (Hq < 1 || q_stride < static_cast<i64>(Hq) * cache->D)) return CAKE_ERR_SHAPE;
    if (rot && max_positions < 1) return CAKE_ERR_SHAPE;
    if ((flags & ~CAKE_APPEND_INTERLEAVED) != 0) return CAKE_ERR_UNSUPPORTED;
    if (!ws) return CAKE_ERR_NULL;
    if (!aligned(ws, 256)) return CAKE_ERR_ALIGN;
    if (ws_bytes < kHeaderBytes) return CAKE_ERR_WORKSPACE;
    if (T == 0) return CAKE_OK;
    if (!k || !v || !slots || (q && !out_q) || (rot && (!positions || !cos_sin))) return CAKE_ERR_NULL;
    if (!aligned(k, 2) || !aligned(v, 2) || !aligned(q, 2) || !aligned(out_q, 2) || !aligned(slots, 8) || !aligned(positions, 4) || !aligned(cos_sin, 4))
        return CAKE_ERR_ALIGN;
    DeviceInfo di;
    rc = current_device_info(&di);
    if (rc != CAKE_OK) return rc;
    if (di.cc_major != 10) return CAKE_ERR_DEVICE;
    AppendArgs a;
    a.c = *cache, a.k = k, a.v = v, a.q = q, a.out_q = out_q, a.slots = slots, a.positions = positions, a.cos_sin = cos_sin;
    a.k_stride = k_stride, a.v_stride = v_stride, a.q_stride = q_stride, a.max_positions = max_positions, a.T = T, a.Hq = Hq, a.rot = rot;
    a.status = static_cast<int*>(ws);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool pairs = flags & CAKE_APPEND_INTERLEAVED;
    const bool e4m3 = cache->type == CAKE_KV_E4M3;
    const int D = cache->D;
    const bool wide = (pairs ? rot % 8 == 0 : rot % 16 == 0) && aligned(cos_sin, 16) && k_stride % 8 == 0 && v_stride % 8 == 0 && aligned(k, 16) && aligned(v, 16) &&
                      (!q || (q_stride % 8 == 0 && aligned(q, 16) && aligned(out_q, 16)));
    const unsigned blocks = static_cast<unsigned>(T);
    cudaError_t e;
    if (wide) {
        const int units = pairs ? D / 8 : rot / 16 + (D - rot) / 8;
        const int heads = (q ? Hq : 0) + 2 * cache->Hkv;
        // Few tokens: a head to a thread (latency).  More: four heads to a thread, whose loads overlap and share the token's row of the
        // table, in blocks of 128 threads (one or more tokens) and, where those are plenty, of a single warp: 32 + 2 * 8 heads, half rotated in
        // pairs, into an 8-bit cache, 128 threads and 32: 500 tokens 3.9 and 7.7 us, 1,000 5.4 and 9.6, 2,048 12.6 and 13.6, 4,096 22.7 and 18.6, 16,001
        // 78 and 63; all rotated into a bf16 cache, 1,000 tokens 6.2 and 6.4 us, 2,048 14.1 and 11.2, 4,096 25.2 and 20.2; 8 + 2 heads, 8,192 14.2 and 16.1
        int par, tokens = 1;
        if (T <= 128) {
            par = heads * units <= 256 ? heads : (256 + units - 1) / units;
        } else {
            const int target = T >= 2048 ? 32 : 128;
            const int most = target / units > 0 ? target / units : 1;
            par = (heads + 3) / 4 <= most ? (heads + 3) / 4 : most;
            tokens = target / (units * par) > 0 ? target / (units * par) : 1;
        }
        void (*const kernel)(const AppendArgs) = e4m3 ? (pairs ? kv_append_kernel<true, true> : kv_append_kernel<true, false>)
                                                      : (pairs ? kv_append_kernel<false, true> : kv_append_kernel<false, false>);
        e = launch_early(kernel, dim3((blocks + tokens - 1) / tokens), dim3(units, par, tokens), 0, s, a);
    } else {
        e = launch_early(e4m3 ? kv_append_scalar_kernel<true> : kv_append_scalar_kernel<false>, dim3(blocks), dim3(256), 0, s, a, pairs);
    }
    return e == cudaSuccess ? CAKE_OK : CAKE_ERR_CUDA;
}
