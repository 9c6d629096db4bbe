// Residual addition + root-mean-square norm + 8-bit output with scales, one pass over memory.
//
//   s = x + r;   y = s * rsqrt(sum(s^2) / H + eps) * w;   scale_g = max(max_g|y| / 448, 2^-100);   q = e4m3(y / scale_g)
//
// Bound by memory, and nearly as much by issue: x and r are read once (4 bytes an element), s and q written once (3 bytes).  A row lives
// in the registers of the threads that read it, so nothing is read twice; blocks walk over the rows with the next rows' loads in
// flight, so a row's reductions (one or two barriers) cost no bandwidth; the arithmetic is packed, two floats to an instruction.  Rows of
// more than 1,024 columns have 64 registers and 1,024 threads an SM: blocks of one row without the loads ahead took 25 % longer, half the threads with twice
// the registers 14 %.  (Shorter rows: 38 to 46 registers, 1,280 or 1,536 threads.)
// Measured: 8192 x 8192 with residual and scales per 128 columns 83.5 us, 5.65 TB/s, 86 % of the copy rate; 16,384 x 1024 83 %; 16 x 4096
// 2.5 us.  Above 16,384 columns four chunks and their successors do not fit 64 registers (492 bytes of spills): 2,048 x 32,768 140 us, 52 %.  Rows
// of even length that is no multiple of 8 are loaded by pairs (4,096 x 5,122 46 us, 49 %), of odd length element by element (4,096 x 5,121
// 112 us, 20 %).
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

// two floats at a time (one instruction): the kernel is bound by issue as much as by memory
__device__ __forceinline__ void mul2(float& a, float& b, float x, float y) {
    asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tmul.rn.f32x2 u, u, v;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}
__device__ __forceinline__ void add2(float& a, float& b, float x, float y) {
    asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tadd.rn.f32x2 u, u, v;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}
// (a, b) += (x^2, y^2)
__device__ __forceinline__ void square2(float& a, float& b, float x, float y) {
    asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tfma.rn.f32x2 u, v, v, u;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}

// LOADS says how a lane's elements lie in a chunk: WIDE, 8 neighbours of a 256-element chunk (two groups of 128 = half a warp each) in one 16-byte
// load; PAIRS, two pairs 64 apart of a 128-element chunk (one group); SINGLE, four elements 32 apart of one: rows of any length
// and alignment.
// NV: chunks per warp.  `tpr` threads (whole warps) share a row; a block holds blockDim.x / tpr rows and walks over
// the matrix, the next rows' loads in flight while a row is reduced and written.
enum { SINGLE, PAIRS, WIDE_LOADS };
template <int LOADS, int NV, int MOST_THREADS, int PER_SM>
__global__ void __launch_bounds__(MOST_THREADS, PER_SM)
rmsnorm_quant_kernel(const NormArgs a, int tpr) {
    constexpr bool WIDE = LOADS == WIDE_LOADS, PAIR = LOADS == PAIRS;
    constexpr int E = WIDE ? 8 : 4;
    constexpr int CHUNK = 32 * E;
    __shared__ float part[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int warps = tpr >> 5;
    const int sub = warp / warps, w_in_row = warp - sub * warps;
    const int per_block = blockDim.x / tpr;
    const int col0 = w_in_row * CHUNK + lane * (WIDE ? 8 : PAIR ? 2 : 1);       // of the first chunk
    const int step = warps * CHUNK;                                   // to the next chunk of this warp
    uint32_t raw[NV][E];              // WIDE: x in words 0-3, r in 4-7; PAIRS: x in 0-1, r in 2-3; SINGLE: x and r of an element side by side
    auto load = [&](i64 row) {
        const bool live = row < a.T;
        const cake_bf16* x = a.x + (live ? row : 0) * a.x_stride;
        const cake_bf16* r = a.r ? a.r + (live ? row : 0) * a.r_stride : nullptr;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = col0 + v * step;
            if (WIDE) {
                uint4 u = make_uint4(0, 0, 0, 0), t = u;
                if (live && c < a.H) {
                    u = *reinterpret_cast<const uint4*>(x + c);
                    if (r) t = *reinterpret_cast<const uint4*>(r + c);
                }
                raw[v][0] = u.x, raw[v][1] = u.y, raw[v][2] = u.z, raw[v][3] = u.w;
                raw[v][E - 4] = t.x, raw[v][E - 3] = t.y, raw[v][E - 2] = t.z, raw[v][E - 1] = t.w;
            } else if (PAIR) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bool in = live && c + 64 * j < a.H;
                    raw[v][j] = in ? *reinterpret_cast<const uint32_t*>(x + c + 64 * j) : 0u;
                    raw[v][2 + j] = in && r ? *reinterpret_cast<const uint32_t*>(r + c + 64 * j) : 0u;
                }
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const bool in = live && c + 32 * j < a.H;
                    raw[v][j] = (in ? x[c + 32 * j] : 0u) | ((in && r ? static_cast<uint32_t>(r[c + 32 * j]) : 0u) << 16);
                }
            }
        }
    };
    i64 row = static_cast<i64>(blockIdx.x) * per_block + sub;
    ptx::grid_dep_wait();
    if (WIDE) load(row);
    // a thread has the same columns in every row: where the registers allow, its weights stay in them
    constexpr bool KEEP = NV <= 2;
    uint32_t wr[NV][4];
    auto weights = [&]() {
        if (!a.w) return;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = col0 + v * step;
            if (WIDE) {
                const uint4 u = c < a.H ? *reinterpret_cast<const uint4*>(a.w + c) : make_uint4(0, 0, 0, 0);
                wr[v][0] = u.x, wr[v][1] = u.y, wr[v][2] = u.z, wr[v][3] = u.w;
            } else if (PAIR) {
#pragma unroll
                for (int j = 0; j < 2; ++j) wr[v][j] = c + 64 * j < a.H ? *reinterpret_cast<const uint32_t*>(a.w + c + 64 * j) : 0u;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) wr[v][j] = c + 32 * j < a.H ? a.w[c + 32 * j] : 0u;
            }
        }
    };
    if (KEEP) weights();
    // (the rows of a block leave the loop together: its barriers are for all threads)
    for (i64 first = static_cast<i64>(blockIdx.x) * per_block; first < a.T; first += static_cast<i64>(gridDim.x) * per_block) {
        const bool live = row < a.T;
        if (!WIDE) load(row);
        float s[NV][E];
        float ss = 0.f, ss_odd = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (WIDE) {
#pragma unroll
                for (int j = 0; j < E; j += 2) {
                    s[v][j] = bf16_lo(raw[v][j / 2]), s[v][j + 1] = bf16_hi(raw[v][j / 2]);
                    add2(s[v][j], s[v][j + 1], bf16_lo(raw[v][E - 4 + j / 2]), bf16_hi(raw[v][E - 4 + j / 2]));
                    square2(ss, ss_odd, s[v][j], s[v][j + 1]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (PAIR) s[v][j] = (j & 1) ? bf16_hi(raw[v][j / 2]) + bf16_hi(raw[v][2 + j / 2]) : bf16_lo(raw[v][j / 2]) + bf16_lo(raw[v][2 + j / 2]);
                    else s[v][j] = bf16_lo(raw[v][j]) + bf16_hi(raw[v][j]);
                    ss = fmaf(s[v][j], s[v][j], ss);
                }
            }
        }
        ss += ss_odd;
        const i64 now = row;
        row += static_cast<i64>(gridDim.x) * per_block;
        if (WIDE && first + static_cast<i64>(gridDim.x) * per_block < a.T) load(row);
        if (a.out_r && live) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = col0 + v * step;
                if (WIDE) {
                    if (c < a.H)
                        *reinterpret_cast<uint4*>(a.out_r + now * a.H + c) =
                            make_uint4(pack_bf16(s[v][0], s[v][1]), pack_bf16(s[v][2], s[v][3]), pack_bf16(s[v][E - 4], s[v][E - 3]),
                                       pack_bf16(s[v][E - 2], s[v][E - 1]));
                } else if (PAIR) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (c + 64 * j < a.H) *reinterpret_cast<uint32_t*>(a.out_r + now * a.H + c + 64 * j) = pack_bf16(s[v][2 * j], s[v][2 * j + 1]);
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j)
                        if (c + 32 * j < a.H) a.out_r[now * a.H + c + 32 * j] = to_bf16(s[v][j]);
                }
            }
        }
        // s becomes s * w; y is that times rs, which is applied to the group's maximum and with the scale instead of element by element
        if (!KEEP) weights();
        if (a.w) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (WIDE) {
                        if (!(j & 1)) mul2(s[v][j], s[v][(j + 1) % E], bf16_lo(wr[v][j / 2]), bf16_hi(wr[v][j / 2]));
                    } else s[v][j] *= (WIDE || PAIR) ? ((j & 1) ? bf16_hi(wr[v][j / 2]) : bf16_lo(wr[v][j / 2])) : bf16_lo(wr[v][j % 4]);
        }
        float rs = 1.f;
        if (a.norm) {
            ss = row_reduce<false>(ss, part[0], warp, sub * warps, warps);
            rs = rsqrtf(ss / static_cast<float>(a.H) + a.eps);
            // rs / scale stays finite up to here (the smallest scale is 2^-100).  Beyond, for rows of next to nothing under an eps as small, the
            // elements take rs themselves; else the zeros of such a row would become 0 * infinity
            if (rs > 0x1p27f && rs < INFINITY) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < E; ++j) s[v][j] *= rs;
                rs = 1.f;
            }
        }
        float most = 0.f;
        auto write_q = [&](int v, float f) {           // f: rs / scale
            const int c = col0 + v * step;
            if (WIDE) {
#pragma unroll
                for (int j = 0; j < E; j += 2) mul2(s[v][j], s[v][(j + 1) % E], f, f);
                if (c < a.H)
                    *reinterpret_cast<uint2*>(a.out_q + now * a.H + c) =
                        make_uint2(pack4_e4m3(s[v][0], s[v][1], s[v][2], s[v][3]), pack4_e4m3(s[v][E - 4], s[v][E - 3], s[v][E - 2], s[v][E - 1]));
            } else if (PAIR) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (c + 64 * j < a.H)
                        *reinterpret_cast<uint16_t*>(a.out_q + now * a.H + c + 64 * j) = static_cast<uint16_t>(pack_e4m3(s[v][2 * j] * f, s[v][2 * j + 1] * f));
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (c + 32 * j < a.H) a.out_q[now * a.H + c + 32 * j] = static_cast<cake_e4m3>(pack_e4m3(s[v][j] * f, 0.f) & 0xff);
            }
        };
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = col0 + v * step;
            if (a.out_y && live) {
                if (WIDE) {
                    if (c < a.H)
                        *reinterpret_cast<uint4*>(a.out_y + now * a.H + c) =
                            make_uint4(pack_bf16(s[v][0] * rs, s[v][1] * rs), pack_bf16(s[v][2] * rs, s[v][3] * rs),
                                       pack_bf16(s[v][E - 4] * rs, s[v][E - 3] * rs), pack_bf16(s[v][E - 2] * rs, s[v][E - 1] * rs));
                } else if (PAIR) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (c + 64 * j < a.H)
                            *reinterpret_cast<uint32_t*>(a.out_y + now * a.H + c + 64 * j) = pack_bf16(s[v][2 * j] * rs, s[v][2 * j + 1] * rs);
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j)
                        if (c + 32 * j < a.H) a.out_y[now * a.H + c + 32 * j] = to_bf16(s[v][j] * rs);
                }
            }
            if (!a.out_q) continue;
            float m = 0.f;
#pragma unroll
            for (int j = 0; j < E; ++j) m = fmaxf(m, fabsf(s[v][j]));
            if (a.by_row) {
                most = fmaxf(most, m);
                continue;
            }
            // one scale per 128 columns: half a warp (WIDE) or the warp
#pragma unroll
            for (int o = WIDE ? 8 : 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float sc = fmaxf(m * rs * (1.f / kE4M3Max), kScaleMin);
            if (live) {
                write_q(v, rs * recip(sc));
                if (WIDE ? ((lane & 15) == 0 && c < a.H) : (lane == 0 && c < a.H)) a.out_scale[now * a.n_scales + (c >> 7)] = sc;
            }
        }
        if (a.out_q && a.by_row) {
            most = row_reduce<true>(most, part[1], warp, sub * warps, warps);
            const float sc = fmaxf(most * rs * (1.f / kE4M3Max), kScaleMin);
            if (live) {
                const float f = rs * recip(sc);
                if (lane == 0 && w_in_row == 0) a.out_scale[now] = sc;
#pragma unroll
                for (int v = 0; v < NV; ++v) write_q(v, f);
            }
        }
        // a row's second barrier (by_row) or the next row's first one separates the reads of `part` from its next writes only if there
        // are two per row; with one, the rows would race
        if (warps > 1 && !(a.norm && a.out_q && a.by_row)) __syncthreads();
    }
}

template <int LOADS, int NV, int MOST_THREADS, int PER_SM>
cudaError_t launch_nv(const NormArgs& a, const DeviceInfo& di, cudaStream_t s) {
    constexpr int CHUNK = LOADS == WIDE_LOADS ? 256 : 128;
    const int chunks = (a.H + CHUNK - 1) / CHUNK;
    const int warps = (chunks + NV - 1) / NV;
    const int rows = warps >= 4 ? 1 : 4 / warps;      // blocks of at least about 128 threads
    const i64 blocks = (a.T + rows - 1) / rows;
    // no more blocks than are resident, the rows spread evenly over their rounds
    const i64 resident = static_cast<i64>(di.sm_count) * (PER_SM * MOST_THREADS / (rows * warps * 32));
    const i64 rounds = (blocks + resident - 1) / resident;
    return launch_early(rmsnorm_quant_kernel<LOADS, NV, MOST_THREADS, PER_SM>, dim3(static_cast<unsigned>((blocks + rounds - 1) / rounds)),
                        dim3(rows * warps * 32), 0, s, a, warps * 32);
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
    const bool pairs = H % 2 == 0 && x_stride % 2 == 0 && aligned(x, 4) && (!residual || (residual_stride % 2 == 0 && aligned(residual, 4))) &&
                       aligned(weight, 4) && aligned(out_residual, 4) && aligned(out_y, 4) && aligned(out_q, 2);
    cudaError_t e;
    // 1,024 threads an SM with 64 registers: two chunks of a row per warp and their successors
    if (wide)
        e = H <= 1024 ? launch_nv<WIDE_LOADS, 1, 128, 10>(a, di, s) : H <= 4096 ? launch_nv<WIDE_LOADS, 2, 256, 4>(a, di, s)
          : H <= 8192 ? launch_nv<WIDE_LOADS, 2, 512, 2>(a, di, s) : H <= 16384 ? launch_nv<WIDE_LOADS, 2, 1024, 1>(a, di, s)
                                                                                : launch_nv<WIDE_LOADS, 4, 1024, 1>(a, di, s);
    else if (pairs)
        e = H <= 1024 ? launch_nv<PAIRS, 1, 256, 6>(a, di, s) : H <= 4096 ? launch_nv<PAIRS, 4, 256, 4>(a, di, s)
          : H <= 8192 ? launch_nv<PAIRS, 4, 512, 2>(a, di, s) : launch_nv<PAIRS, 8, 1024, 1>(a, di, s);
    else
        e = H <= 1024 ? launch_nv<SINGLE, 1, 256, 6>(a, di, s) : H <= 4096 ? launch_nv<SINGLE, 4, 256, 4>(a, di, s)
          : H <= 8192 ? launch_nv<SINGLE, 4, 512, 2>(a, di, s) : launch_nv<SINGLE, 8, 1024, 1>(a, di, s);
    return e == cudaSuccess ? CAKE_OK : CAKE_ERR_CUDA;
}
