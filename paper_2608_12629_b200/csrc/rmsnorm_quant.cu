// Residual addition + root-mean-square norm + 8-bit output with scales, one pass over memory.
//
//   s = x + r;   y = s * rsqrt(sum(s^2) / H + eps) * w;   scale_g = max(max_g|y| / 448, 2^-100);   q = e4m3(y / scale_g)
//
// Bound by memory: x and r are read once (4 bytes an element), s and q written once (3 bytes).  A row lives in the
// registers of the threads that read it, so nothing is read twice.
#include "serving.cuh"

namespace cake {
namespace serving {
namespace {

constexpr int kMaxH = 32768;

struct NormArgs {
    const cake_bf16* x;
    const cake_bf16* r;
    const cake_bf16* w;
    cake_bf16* out_r;
    cake_bf16* out_y;
    cake_e4m3* out_q;
    float* out_scale;
    i64 x_stride, r_stride, T;
    int H, n_scales;
    float eps;
    bool by_row, norm;
};

// sum (or maximum) over the threads of a row: shuffles inside a warp, then one word per warp through shared memory.  The
// row's warps write `part` and read it after one barrier; callers alternate between two such arrays.
template <bool MAX>
__device__ __forceinline__ float row_reduce(float v, float* part, int warp, int first_warp, int warps) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? fmaxf(v, u) : v + u;
    }
    if (warps == 1) return v;
    const int lane = threadIdx.x & 31;
    if (lane == 0) part[warp] = v;
    __syncthreads();
    v = lane < warps ? part[first_warp + lane] : 0.f;       // (maxima are of absolute values)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? fmaxf(v, u) : v + u;
    }
    return v;
}
// 1 / scale, one unit in the last place
__device__ __forceinline__ float recip(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// WIDE: a lane holds 8 neighbouring elements of a 256-element chunk (two groups of 128 = half a warp each); otherwise 4
// elements 32 apart of a 128-element chunk (one group), loaded one by one: rows of any length and alignment.
// NV: chunks per warp.  `tpr` threads (whole warps) share a row; a block holds blockDim.x / tpr rows.
template <bool WIDE, int NV, int MOST_THREADS>
__global__ void __launch_bounds__(MOST_THREADS)
rmsnorm_quant_kernel(const NormArgs a, int tpr) {
    constexpr int E = WIDE ? 8 : 4;
    constexpr int CHUNK = 32 * E;
    __shared__ float part[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int warps = tpr >> 5;
    const int sub = warp / warps, w_in_row = warp - sub * warps;
    const i64 row = static_cast<i64>(blockIdx.x) * (blockDim.x / tpr) + sub;
    const bool live = row < a.T;
    float s[NV][E];
    float ss = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int base = (v * warps + w_in_row) * CHUNK;
        if (WIDE) {
            const int c = base + lane * 8;
            uint4 u = make_uint4(0, 0, 0, 0), t = u;
            if (live && c < a.H) {
                u = *reinterpret_cast<const uint4*>(a.x + row * a.x_stride + c);
                if (a.r) t = *reinterpret_cast<const uint4*>(a.r + row * a.r_stride + c);
            }
            const uint32_t uw[4] = {u.x, u.y, u.z, u.w}, tw[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[v][2 * j] = bf16_lo(uw[j]) + bf16_lo(tw[j]);
                s[v][2 * j + 1] = bf16_hi(uw[j]) + bf16_hi(tw[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int c = base + j * 32 + lane;
                float f = 0.f;
                if (live && c < a.H) {
                    f = bf16_f(a.x[row * a.x_stride + c]);
                    if (a.r) f += bf16_f(a.r[row * a.r_stride + c]);
                }
                s[v][j] = f;
            }
        }
#pragma unroll
        for (int j = 0; j < E; ++j) ss = fmaf(s[v][j], s[v][j], ss);
    }
    float rs = 1.f;
    if (a.norm) {
        ss = row_reduce<false>(ss, part[0], warp, sub * warps, warps);
        rs = rsqrtf(ss / static_cast<float>(a.H) + a.eps);
    }
    if (a.out_r && live) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int base = (v * warps + w_in_row) * CHUNK;
            if (WIDE) {
                const int c = base + lane * 8;
                if (c < a.H)
                    *reinterpret_cast<uint4*>(a.out_r + row * a.H + c) =
                        make_uint4(pack_bf16(s[v][0], s[v][1]), pack_bf16(s[v][2], s[v][3]), pack_bf16(s[v][4], s[v][5]),
                                   pack_bf16(s[v][6], s[v][7]));
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const int c = base + j * 32 + lane;
                    if (c < a.H) a.out_r[row * a.H + c] = to_bf16(s[v][j]);
                }
            }
        }
    }
    float most = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int base = (v * warps + w_in_row) * CHUNK;
        float y[E];
        if (WIDE) {
            const int c = base + lane * 8;
            uint4 wv = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
            if (a.w && c < a.H) wv = __ldg(reinterpret_cast<const uint4*>(a.w + c));
            const uint32_t ww[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[2 * j] = s[v][2 * j] * rs * bf16_lo(ww[j]);
                y[2 * j + 1] = s[v][2 * j + 1] * rs * bf16_hi(ww[j]);
            }
            if (a.out_y && live && c < a.H)
                *reinterpret_cast<uint4*>(a.out_y + row * a.H + c) =
                    make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int c = base + j * 32 + lane;
                const float wf = (a.w && c < a.H) ? bf16_f(__ldg(a.w + c)) : 1.f;
                y[j] = s[v][j] * rs * wf;
                if (a.out_y && live && c < a.H) a.out_y[row * a.H + c] = to_bf16(y[j]);
            }
        }
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            m = fmaxf(m, fabsf(y[j]));
            s[v][j] = y[j];
        }
        most = fmaxf(most, m);
        if (!a.out_q || a.by_row) continue;
        // one scale per 128 columns: half a warp (WIDE) or the warp
#pragma unroll
        for (int o = WIDE ? 8 : 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float sc = fmaxf(m * (1.f / kE4M3Max), kScaleMin);
        const float inv = recip(sc);
        if (WIDE) {
            const int c = base + lane * 8;
            if (live && c < a.H) {
                *reinterpret_cast<uint2*>(a.out_q + row * a.H + c) =
                    make_uint2(pack4_e4m3(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                               pack4_e4m3(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
                if ((lane & 15) == 0) a.out_scale[row * a.n_scales + (c >> 7)] = sc;
            }
        } else if (live && base < a.H) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int c = base + j * 32 + lane;
                if (c < a.H) a.out_q[row * a.H + c] = static_cast<cake_e4m3>(pack_e4m3(y[j] * inv, 0.f) & 0xff);
            }
            if (lane == 0) a.out_scale[row * a.n_scales + (base >> 7)] = sc;
        }
    }
    if (!a.out_q || !a.by_row) return;
    most = row_reduce<true>(most, part[1], warp, sub * warps, warps);
    const float sc = fmaxf(most * (1.f / kE4M3Max), kScaleMin);
    const float inv = recip(sc);
    if (!live) return;
    if (lane == 0 && w_in_row == 0) a.out_scale[row] = sc;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int base = (v * warps + w_in_row) * CHUNK;
        if (WIDE) {
            const int c = base + lane * 8;
            if (c < a.H)
                *reinterpret_cast<uint2*>(a.out_q + row * a.H + c) =
                    make_uint2(pack4_e4m3(s[v][0] * inv, s[v][1] * inv, s[v][2] * inv, s[v][3] * inv),
                               pack4_e4m3(s[v][4] * inv, s[v][5] * inv, s[v][6] * inv, s[v][7] * inv));
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int c = base + j * 32 + lane;
                if (c < a.H) a.out_q[row * a.H + c] = static_cast<cake_e4m3>(pack_e4m3(s[v][j] * inv, 0.f) & 0xff);
            }
        }
    }
}

template <bool WIDE, int NV, int MOST_THREADS>
cudaError_t launch_nv(const NormArgs& a, cudaStream_t s) {
    constexpr int CHUNK = WIDE ? 256 : 128;
    const int chunks = (a.H + CHUNK - 1) / CHUNK;
    const int warps = (chunks + NV - 1) / NV;
    const int rows = warps >= 4 ? 1 : 4 / warps;      // blocks of at least about 128 threads
    const i64 blocks = (a.T + rows - 1) / rows;
    rmsnorm_quant_kernel<WIDE, NV, MOST_THREADS><<<static_cast<unsigned>(blocks), rows * warps * 32, 0, s>>>(a, warps * 32);
    note_launches(1);
    return cudaGetLastError();
}

}  // namespace
}  // namespace serving
}  // namespace cake

using namespace cake;
using namespace cake::serving;

extern "C" int cake_rmsnorm_quant(const cake_bf16* x, long long x_stride, const cake_bf16* residual, long long residual_stride,
                                  const cake_bf16* weight, long long T, int H, float eps, int group, cake_bf16* out_residual,
                                  cake_bf16* out_y, cake_e4m3* out_q, float* out_scale, cake_stream_t stream, unsigned flags) {
    if (T < 0 || T > INT_MAX || H < 1 || x_stride < H || (residual && residual_stride < H)) return CAKE_ERR_SHAPE;
    if (group != 0 && group != 128) return CAKE_ERR_UNSUPPORTED;
    if (H > kMaxH || (flags & ~CAKE_RMSNORM_NONE) != 0) return CAKE_ERR_UNSUPPORTED;
    if (T == 0) return CAKE_OK;
    if (!x || (!out_y && !out_q) || ((out_q != nullptr) != (out_scale != nullptr))) return CAKE_ERR_NULL;
    if (!aligned(x, 2) || !aligned(residual, 2) || !aligned(weight, 2) || !aligned(out_residual, 2) || !aligned(out_y, 2) ||
        !aligned(out_scale, 4))
        return CAKE_ERR_ALIGN;
    DeviceInfo di;
    const int rc = current_device_info(&di);
    if (rc != CAKE_OK) return rc;
    if (di.cc_major != 10) return CAKE_ERR_DEVICE;
    NormArgs a;
    a.x = x, a.r = residual, a.w = weight, a.out_r = out_residual, a.out_y = out_y, a.out_q = out_q, a.out_scale = out_scale;
    a.x_stride = x_stride, a.r_stride = residual_stride, a.T = T, a.H = H, a.eps = eps;
    a.by_row = group == 0, a.norm = !(flags & CAKE_RMSNORM_NONE);
    a.n_scales = a.by_row ? 1 : (H + 127) / 128;
    const bool wide = H % 8 == 0 && x_stride % 8 == 0 && aligned(x, 16) && (!residual || (residual_stride % 8 == 0 && aligned(residual, 16))) &&
                      aligned(weight, 16) && aligned(out_residual, 16) && aligned(out_y, 16) && aligned(out_q, 8);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (wide)
        e = H <= 2048 ? launch_nv<true, 1, 256>(a, s) : H <= 4096 ? launch_nv<true, 2, 256>(a, s)
          : H <= 8192 ? launch_nv<true, 4, 256>(a, s) : H <= 16384 ? launch_nv<true, 4, 512>(a, s) : launch_nv<true, 4, 1024>(a, s);
    else
        e = H <= 1024 ? launch_nv<false, 1, 256>(a, s) : H <= 8192 ? launch_nv<false, 4, 512>(a, s) : launch_nv<false, 8, 1024>(a, s);
    return e == cudaSuccess ? CAKE_OK : CAKE_ERR_CUDA;
}
