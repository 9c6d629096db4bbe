// Product of two e4m3 matrices with a scale for each block of 128 columns:
//
//   out[m][n] = sum_kb xs[m][kb] ws[n/128][kb] (sum_{k in kb} X[m][k] W[n][k])
//
// A block of 128 columns is 128 bytes: one swizzled row of a shared-memory tile and four k-steps of tcgen05.mma
// (kind::f8f6f4).  The tensor core starts every block from zero in one of a ring of tensor-memory buffers; the epilogue
// warps fetch a finished block, scale it and add it to 32-bit sums in their registers, while the next blocks run.
//
// The weights are the M side of the instruction (128 rows of W = 128 lanes of tensor memory), the rows of X its columns:
// a few rows of X (a decode step) then cost a narrow tile instead of a mostly empty one, a tile of W lies in one row of the
// weights' scales, and 32 lanes store 32 neighbouring outputs.  The scale of an element depends on its column alone
// (xs * ws, multiplied once per block by a warp of its own and read as a broadcast), so the addition is one FMA.
#include "ptx.cuh"
#include "serving.cuh"

namespace cake {
namespace serving {
namespace {

constexpr int TM = 128;                        // rows of W per tile
constexpr int KB = 128;                        // columns of a block
constexpr int EPI_WARPS = 8;                   // two warpgroups, half of the tile's columns each
constexpr int WARP_TMA = 8, WARP_MMA = 9, WARP_SCALE = 10;
constexpr int THREADS = 11 * 32;
constexpr int SCALE_BUFS = 8;                  // blocks of scales ahead
constexpr uint32_t W_BYTES = TM * KB;
constexpr uint64_t WAIT_LIMIT_NS = 2000000000ull;

struct GemmArgs {
    const float* xs;
    const float* ws;
    void* out;
    float* parts;
    int* counters;
    int* status;
    i64 M, out_stride;
    int N, nkb, tiles_m, tiles_n, splits;      // tiles_m: of X's rows
    bool fp32;
};

struct __align__(16) Ctrl {
    uint64_t full[16], empty[16], tfull[4], tempty[4], sfull[SCALE_BUFS], sempty[SCALE_BUFS];
    uint32_t tmem;
    int abort_flag;
    int last;
};

__device__ __forceinline__ void wait_bar(uint64_t* bar, uint32_t parity, Ctrl* ctrl, int* status) {
    const uint32_t addr = ptx::smem_u32(bar);
    if (ptx::mbar_try_wait(addr, parity)) return;
    const uint64_t t0 = ptx::globaltimer_ns();
    while (!ptx::mbar_try_wait_hint(addr, parity, 20000)) {
        if (*reinterpret_cast<volatile int*>(&ctrl->abort_flag)) return;
        if (ptx::globaltimer_ns() - t0 > WAIT_LIMIT_NS) {
            *reinterpret_cast<volatile int*>(&ctrl->abort_flag) = 1;
            atomicCAS(status, CAKE_OK, CAKE_ERR_TIMEOUT);
            return;
        }
    }
}
__device__ __forceinline__ bool aborted(Ctrl* ctrl) { return *reinterpret_cast<volatile int*>(&ctrl->abort_flag) != 0; }

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y)
        : "memory");
}
template <bool ACC>
__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "n"(ACC ? 1 : 0)
        : "memory");
}
// fp32 accumulator, e4m3 x e4m3, both K-major, M x N tile
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N) {
    return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[N]) {
    static_assert(N == 8 || N == 16 || N == 32, "");
    if constexpr (N == 32) {
        ptx::tmem_ld_x32(addr, r);
        ptx::tmem_ld_wait(r);
    } else if constexpr (N == 16) {
        ptx::tmem_ld_x16(addr, r);
    } else {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
                     "tcgen05.wait::ld.sync.aligned;"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(addr) : "memory");
    }
}

template <int TN>
struct Tile {
    static constexpr int COLS = TN / 2;                              // columns of an epilogue thread
    static constexpr int LD = COLS < 32 ? COLS : 32;
    static constexpr uint32_t STAGE = W_BYTES + TN * KB;
    static constexpr int STAGES = TN == 256 ? 4 : TN == 128 ? 6 : TN == 64 ? 8 : TN == 32 ? 10 : 11;
    static constexpr int BUFS = TN == 256 ? 2 : 4;
    static constexpr uint32_t TMEM_COLS = BUFS * TN < 32 ? 32 : BUFS * TN;
    static constexpr uint32_t SMEM = 1024 + STAGES * STAGE + SCALE_BUFS * TN * 4 + sizeof(Ctrl);
    static_assert(SMEM <= 227 * 1024, "");
};

struct Item {
    int m0, n0, kb0, kb1, split, tile;
};
// items in the order (tile of W, tile of X, split); CTA c takes items c, c + n, ...
__device__ __forceinline__ Item item_of(const GemmArgs& a, int i, int tn) {
    Item it;
    it.split = i % a.splits;
    it.tile = i / a.splits;
    const int nt = it.tile % a.tiles_n;
    it.n0 = nt * TM;
    it.m0 = (it.tile / a.tiles_n) * tn;
    it.kb0 = static_cast<int>(static_cast<i64>(it.split) * a.nkb / a.splits);
    it.kb1 = static_cast<int>(static_cast<i64>(it.split + 1) * a.nkb / a.splits);
    return it;
}

template <int TN>
__global__ void __launch_bounds__(THREADS, 1)
gemm_fp8_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const GemmArgs a) {
    using T = Tile<TN>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* const tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    float* const scales = reinterpret_cast<float*>(tiles + T::STAGES * T::STAGE);
    Ctrl* const ctrl = reinterpret_cast<Ctrl*>(scales + SCALE_BUFS * TN);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int items = a.tiles_m * a.tiles_n * a.splits;

    if (threadIdx.x == 0) {
        for (int i = 0; i < T::STAGES; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctrl->full[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctrl->empty[i]), 1);
        }
        for (int i = 0; i < T::BUFS; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctrl->tfull[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctrl->tempty[i]), EPI_WARPS);
        }
        for (int i = 0; i < SCALE_BUFS; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctrl->sfull[i]), 32);
            ptx::mbar_init(ptx::smem_u32(&ctrl->sempty[i]), EPI_WARPS);
        }
        ctrl->abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&map_w);
        ptx::prefetch_tensormap(&map_x);
    }
    if (warp == WARP_MMA) {
        ptx::tmem_alloc(ptx::smem_u32(&ctrl->tmem), T::TMEM_COLS);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ctrl->tmem;

    if (warp == WARP_TMA) {
        if (ptx::elect_one()) {
            uint32_t n = 0;      // blocks so far
            for (int i = blockIdx.x; i < items && !aborted(ctrl); i += gridDim.x) {
                const Item it = item_of(a, i, TN);
                for (int kb = it.kb0; kb < it.kb1; ++kb, ++n) {
                    const uint32_t s = n % T::STAGES, round = n / T::STAGES;
                    wait_bar(&ctrl->empty[s], (round & 1) ^ 1, ctrl, a.status);
                    if (aborted(ctrl)) break;
                    const uint32_t bar = ptx::smem_u32(&ctrl->full[s]), dst = ptx::smem_u32(tiles + s * T::STAGE);
                    ptx::mbar_arrive_expect_tx(bar, T::STAGE);
                    tma_load_2d(dst, &map_w, bar, kb * KB, it.n0);
                    tma_load_2d(dst + W_BYTES, &map_x, bar, kb * KB, it.m0);
                }
            }
            // copies in flight land before the CTA gives up its shared memory (they have, unless a wait has expired)
            if (aborted(ctrl)) {
                const uint64_t t0 = ptx::globaltimer_ns();
                for (uint32_t j = n > T::STAGES ? n - T::STAGES : 0; j < n; ++j)
                    while (!ptx::mbar_try_wait(ptx::smem_u32(&ctrl->full[j % T::STAGES]), (j / T::STAGES) & 1) &&
                           ptx::globaltimer_ns() - t0 < WAIT_LIMIT_NS / 4) {}
            }
        }
        __syncwarp();
    } else if (warp == WARP_MMA) {
        if (ptx::elect_one()) {
            uint32_t n = 0;
            constexpr uint32_t idesc = idesc_e4m3(TM, TN);
            for (int i = blockIdx.x; i < items && !aborted(ctrl); i += gridDim.x) {
                const Item it = item_of(a, i, TN);
                for (int kb = it.kb0; kb < it.kb1; ++kb, ++n) {
                    const uint32_t s = n % T::STAGES, b = n % T::BUFS;
                    wait_bar(&ctrl->tempty[b], ((n / T::BUFS) & 1) ^ 1, ctrl, a.status);
                    wait_bar(&ctrl->full[s], (n / T::STAGES) & 1, ctrl, a.status);
                    if (aborted(ctrl)) break;
                    ptx::tc_fence_after();
                    const uint32_t base = ptx::smem_u32(tiles + s * T::STAGE);
                    const uint64_t da = ptx::umma_desc_sw128(base), db = ptx::umma_desc_sw128(base + W_BYTES);
                    const uint32_t d = tmem + b * TN;
                    umma_e4m3<false>(d, da, db, idesc);          // 32 columns (32 bytes) a step
                    umma_e4m3<true>(d, da + 2, db + 2, idesc);
                    umma_e4m3<true>(d, da + 4, db + 4, idesc);
                    umma_e4m3<true>(d, da + 6, db + 6, idesc);
                    ptx::umma_commit(ptx::smem_u32(&ctrl->empty[s]));
                    ptx::umma_commit(ptx::smem_u32(&ctrl->tfull[b]));
                }
            }
        }
        __syncwarp();
    } else if (warp == WARP_SCALE) {
        // one product xs * ws per column and block; the loads of four blocks run together, ahead of the waits
        constexpr int PER = (TN + 31) / 32;
        constexpr int AHEAD = 4;
        uint32_t n = 0;
        for (int i = blockIdx.x; i < items; i += gridDim.x) {
            const Item it = item_of(a, i, TN);
            const float* wrow = a.ws + static_cast<i64>(it.n0 / TM) * a.nkb;
            float next[AHEAD][PER];
            auto fetch = [&](int kb) {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
                        const i64 m = static_cast<i64>(it.m0) + j * 32 + lane;
                        next[u][j] = (kb + u < it.kb1 && m < a.M) ? __ldg(a.xs + m * a.nkb + kb + u) * __ldg(wrow + kb + u) : 0.f;
                    }
            };
            fetch(it.kb0);
            for (int kb = it.kb0; kb < it.kb1; kb += AHEAD) {
                float cur[AHEAD][PER];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                    for (int j = 0; j < PER; ++j) cur[u][j] = next[u][j];
                if (kb + AHEAD < it.kb1) fetch(kb + AHEAD);
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    if (kb + u >= it.kb1) break;
                    const uint32_t b = n % SCALE_BUFS;
                    wait_bar(&ctrl->sempty[b], ((n / SCALE_BUFS) & 1) ^ 1, ctrl, a.status);
#pragma unroll
                    for (int j = 0; j < PER; ++j)
                        if (j * 32 + lane < TN) scales[b * TN + j * 32 + lane] = cur[u][j];
                    ptx::mbar_arrive(ptx::smem_u32(&ctrl->sfull[b]));
                    ++n;
                }
            }
        }
    } else {
        const int half = warp >> 2, quad = warp & 3;      // a warp reads the 32 lanes of its place in its warpgroup
        const uint32_t t_lane = tmem + (static_cast<uint32_t>(quad * 32) << 16) + half * T::COLS;
        uint32_t n = 0;
        // (after an expired wait this loop and the scales' run on with waits that return at once: its warps meet at a
        // barrier below, so all of them have to take every step)
        for (int i = blockIdx.x; i < items; i += gridDim.x) {
            const Item it = item_of(a, i, TN);
            float acc[T::COLS];
#pragma unroll
            for (int c = 0; c < T::COLS; ++c) acc[c] = 0.f;
            for (int kb = it.kb0; kb < it.kb1; ++kb, ++n) {
                const uint32_t b = n % T::BUFS, sb = n % SCALE_BUFS;
                wait_bar(&ctrl->sfull[sb], (n / SCALE_BUFS) & 1, ctrl, a.status);
                wait_bar(&ctrl->tfull[b], (n / T::BUFS) & 1, ctrl, a.status);
                ptx::tc_fence_after();
                const float* sc = scales + sb * TN + half * T::COLS;
#pragma unroll
                for (int c0 = 0; c0 < T::COLS; c0 += T::LD) {
                    uint32_t r[T::LD];
                    tmem_load<T::LD>(t_lane + b * TN + c0, r);
#pragma unroll
                    for (int c = 0; c < T::LD; c += 4) {
                        const float4 f = *reinterpret_cast<const float4*>(sc + c0 + c);
                        acc[c0 + c] = fmaf(__uint_as_float(r[c]), f.x, acc[c0 + c]);
                        acc[c0 + c + 1] = fmaf(__uint_as_float(r[c + 1]), f.y, acc[c0 + c + 1]);
                        acc[c0 + c + 2] = fmaf(__uint_as_float(r[c + 2]), f.z, acc[c0 + c + 2]);
                        acc[c0 + c + 3] = fmaf(__uint_as_float(r[c + 3]), f.w, acc[c0 + c + 3]);
                    }
                }
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(ptx::smem_u32(&ctrl->tempty[b]));
                    ptx::mbar_arrive(ptx::smem_u32(&ctrl->sempty[sb]));
                }
            }
            const int col = it.n0 + quad * 32 + lane;              // column of the output
            const i64 row0 = static_cast<i64>(it.m0) + half * T::COLS;
            auto store = [&](int c, float v) {
                const i64 row = row0 + c;
                if (row >= a.M || col >= a.N) return;
                if (a.fp32) static_cast<float*>(a.out)[row * a.out_stride + col] = v;
                else static_cast<cake_bf16*>(a.out)[row * a.out_stride + col] = to_bf16(v);
            };
            if (a.splits == 1) {
#pragma unroll
                for (int c = 0; c < T::COLS; ++c) store(c, acc[c]);
                continue;
            }
            // ---- parts of the contraction: the last of the tile's CTAs adds them up in order
            float* const mine = a.parts + static_cast<i64>(i) * (TM * TN) + (half * T::COLS) * TM + quad * 32 + lane;
#pragma unroll
            for (int c = 0; c < T::COLS; ++c) __stcg(mine + c * TM, acc[c]);
            asm volatile("bar.sync 1, %0;" ::"n"(EPI_WARPS * 32) : "memory");
            if (threadIdx.x == 0) {
                __threadfence();
                const int seen = atomicAdd(a.counters + it.tile, 1);
                ctrl->last = seen == a.splits - 1;
                if (ctrl->last) a.counters[it.tile] = 0;
                __threadfence();
            }
            asm volatile("bar.sync 1, %0;" ::"n"(EPI_WARPS * 32) : "memory");
            if (ctrl->last) {
#pragma unroll
                for (int c = 0; c < T::COLS; ++c) acc[c] = 0.f;
                for (int s = 0; s < a.splits; ++s) {
                    const float* from = mine + static_cast<i64>(s - it.split) * (TM * TN);
#pragma unroll
                    for (int c = 0; c < T::COLS; ++c) acc[c] += __ldcg(from + c * TM);
                }
#pragma unroll
                for (int c = 0; c < T::COLS; ++c) store(c, acc[c]);
            }
            asm volatile("bar.sync 1, %0;" ::"n"(EPI_WARPS * 32) : "memory");     // ctrl->last is read by all before the next item
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == WARP_MMA) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, T::TMEM_COLS);
    }
}

// ---------------------------------------------------------------------------------------------------------------- host
struct Plan {
    int tn, tiles_m, tiles_n, splits, nkb;
    size_t part_bytes;
};
Plan plan_of(i64 M, int N, int K, int sms) {
    Plan p;
    p.nkb = (K + KB - 1) / KB;
    p.tiles_n = (N + TM - 1) / TM;
    p.tn = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : M <= 128 ? 128 : 256;
    if (p.tn == 256) {      // 128 columns where they need less time for the last, partly filled round of CTAs
        const i64 t256 = (M + 255) / 256 * p.tiles_n, t128 = (M + 127) / 128 * p.tiles_n;
        if ((t128 + sms - 1) / sms < 2 * ((t256 + sms - 1) / sms)) p.tn = 128;
    }
    p.tiles_m = static_cast<int>((M + p.tn - 1) / p.tn);
    const i64 tiles = static_cast<i64>(p.tiles_m) * p.tiles_n;
    p.splits = 1;
    if (tiles > 0 && tiles < sms) {
        p.splits = static_cast<int>(sms / tiles);
        if (p.splits > p.nkb / 4) p.splits = p.nkb / 4;
        if (p.splits < 1) p.splits = 1;
    }
    p.part_bytes = p.splits > 1 ? static_cast<size_t>(tiles) * p.splits * TM * p.tn * 4 : 0;
    return p;
}

template <int TN>
int launch(const GemmArgs& a, const CUtensorMap& mw, const CUtensorMap& mx, const DeviceInfo& di, cudaStream_t s) {
    using T = Tile<TN>;
    static bool set[64] = {};
    if (di.device < 0 || di.device >= 64 || !set[di.device]) {
        if (cudaFuncSetAttribute(gemm_fp8_kernel<TN>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::SMEM) != cudaSuccess) return CAKE_ERR_CUDA;
        if (di.device >= 0 && di.device < 64) set[di.device] = true;
    }
    const i64 items = static_cast<i64>(a.tiles_m) * a.tiles_n * a.splits;
    const int ctas = static_cast<int>(items < di.sm_count ? items : di.sm_count);
    gemm_fp8_kernel<TN><<<ctas, THREADS, T::SMEM, s>>>(mw, mx, a);
    note_launches(1);
    return cudaGetLastError() == cudaSuccess ? CAKE_OK : CAKE_ERR_CUDA;
}

int check_shape(i64 M, int N, int K) {
    if (M < 0 || N < 1 || K < 1 || M > INT_MAX - 1024 || N > INT_MAX - 1024 || K > INT_MAX - 1024) return CAKE_ERR_SHAPE;
    if (((M + 127) / 128) * ((static_cast<i64>(N) + TM - 1) / TM) > INT_MAX / 2) return CAKE_ERR_SHAPE;
    return CAKE_OK;
}
constexpr int kMaxSms = 148;      // the plan that sizes the workspace touches no device: that of a B200

}  // namespace
}  // namespace serving
}  // namespace cake

using namespace cake;
using namespace cake::serving;

extern "C" {

int cake_gemm_fp8_workspace_bytes(long long M, int N, int K, size_t* out_bytes) {
    if (!out_bytes) return CAKE_ERR_NULL;
    const int rc = check_shape(M, N, K);
    if (rc != CAKE_OK) return rc;
    *out_bytes = kHeaderBytes + plan_of(M, N, K, kMaxSms).part_bytes;
    return CAKE_OK;
}

int cake_gemm_fp8(const cake_e4m3* X, long long x_stride, const float* x_scale, const cake_e4m3* W, long long w_stride,
                  const float* w_scale, long long M, int N, int K, void* out, long long out_stride, void* ws, size_t ws_bytes,
                  cake_stream_t stream, unsigned flags) {
    int rc = check_shape(M, N, K);
    if (rc != CAKE_OK) return rc;
    if (x_stride < K || w_stride < K || out_stride < N) return CAKE_ERR_SHAPE;
    if ((flags & ~CAKE_GEMM_OUT_FP32) != 0) return CAKE_ERR_UNSUPPORTED;
    if (!ws) return CAKE_ERR_NULL;
    if (!aligned(ws, 256)) return CAKE_ERR_ALIGN;
    if (M == 0) return CAKE_OK;
    if (!X || !W || !x_scale || !w_scale || !out) return CAKE_ERR_NULL;
    if (K % 16 != 0 || x_stride % 16 != 0 || w_stride % 16 != 0 || !aligned(X, 16) || !aligned(W, 16)) return CAKE_ERR_ALIGN;
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(out, (flags & CAKE_GEMM_OUT_FP32) ? 4 : 2)) return CAKE_ERR_ALIGN;
    const Plan p = plan_of(M, N, K, kMaxSms);
    if (ws_bytes < kHeaderBytes + p.part_bytes) return CAKE_ERR_WORKSPACE;
    DeviceInfo di;
    rc = current_device_info(&di);
    if (rc != CAKE_OK) return rc;
    if (di.cc_major != 10) return CAKE_ERR_DEVICE;
    CUtensorMap mw, mx;
    rc = make_tmap_bytes(&mw, W, K, N, w_stride, TM);
    if (rc != CAKE_OK) return rc;
    rc = make_tmap_bytes(&mx, X, K, M, x_stride, p.tn);
    if (rc != CAKE_OK) return rc;
    GemmArgs a;
    a.xs = x_scale, a.ws = w_scale, a.out = out, a.status = static_cast<int*>(ws), a.counters = static_cast<int*>(ws) + 64;
    a.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + kHeaderBytes);
    a.M = M, a.out_stride = out_stride, a.N = N, a.nkb = p.nkb, a.tiles_m = p.tiles_m, a.tiles_n = p.tiles_n, a.splits = p.splits;
    a.fp32 = flags & CAKE_GEMM_OUT_FP32;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    switch (p.tn) {
        case 16: return launch<16>(a, mw, mx, di, s);
        case 32: return launch<32>(a, mw, mx, di, s);
        case 64: return launch<64>(a, mw, mx, di, s);
        case 128: return launch<128>(a, mw, mx, di, s);
        default: return launch<256>(a, mw, mx, di, s);
    }
}

}  // extern "C"
