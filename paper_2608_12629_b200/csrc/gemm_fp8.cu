// Product of two e4m3 matrices with a scale for each block of 128 columns:
//
//   out[m][n] = sum_kb xs[m][kb] ws[n/128][kb] (sum_{k in kb} X[m][k] W[n][k])
//
// A block of 128 columns is 128 bytes: one swizzled row of a shared-memory tile and four k-steps of tcgen05.mma
// (kind::f8f6f4).  The tensor core starts every block from zero in one of a ring of tensor-memory buffers; the epilogue
// warps fetch a finished block, scale it and add it to 32-bit sums in their registers, while the next blocks run.
//
// Two kernels, chosen by the rows of X:
//   up to 64 rows   The weights are the M side of the instruction (128 rows of W = 128 lanes of tensor memory), the rows of X its
//                   columns: a few rows then cost a narrow tile instead of a mostly empty one.  Bound by reading W.  The scale of an
//                   element depends on its column (xs * ws, multiplied once per block by a warp of its own, read as a broadcast).
//   more            X is the M side, two SMs to a 256 x 256 tile (cta_group::2: each loads half of both operands, 32 KiB a block instead
//                   of the 48 of a 128 x 256 tile of one SM, whose demand of 94 bytes a clock the L2 does not meet).  The scale of an
//                   element depends on its lane and on its half of the columns: one factor per thread and block, packed FMAs.
// Measured: 8192 x 8192 x 8192 526 - 556 us repeated (1.98 - 2.09 PFLOP/s, 60 - 63 % of twice the bf16 burst rate; under the power cap, clocks of 1.4 to
// 1.9 GHz), 504 in short bursts, 478 in a single launch at full clock (tensor pipe 65 % busy): an accumulator's round trip (product, signal, 128 columns added by the epilogue, signal) is what bounds
// a block, and the operands' 96 KiB of shared-memory traffic is close behind.  16 x 6144 x 4096 9.1 us with weights from memory (2.8 TB/s, 43 % of the copy
// rate; 6.8 - 7.6 us where they lie in the L2), 64 x 8192 x 8192 16.8 - 21.5 us (3.2 - 4.1 TB/s, 49 - 63 %, from one device to the next; 13.9 in the
// L2): start, first loads and join are about 4 us of each.
// Where a product has too few tiles for the SMs its contraction is split; the parts of a narrow tile are added up
// through the shared memory of a cluster, those of the pairs by a second kernel.
#include "ptx.cuh"
#include "serving.cuh"

namespace cake {
namespace serving {
namespace {

constexpr int TM = 128;                        // rows of W per tile
constexpr int KB = 128;                        // columns of a block
constexpr int EPI_WARPS = 8;                   // two warpgroups, half of the tile's columns each
constexpr int WARP_TMA = 8, WARP_MMA = 9, WARP_SCALE = 10, WARP_MMA1 = 11;
constexpr int THREADS = 12 * 32;
constexpr int BUFS = 4;                        // steps whose accumulators, and whose scales, are in flight
// Blocks of a step.  A block of a narrow tile is less work (64 to 256 clocks) than its barriers: about 100 clocks to issue an instruction, 120
// for a commit, 200 for a wait.  So two blocks share them, and two threads issue every other step
constexpr int PER_STEP = 2;
constexpr uint32_t W_BYTES = TM * KB;
constexpr uint64_t WAIT_LIMIT_NS = 2000000000ull;
// The plan of a product, its workspace and the order of its sums follow from the sizes alone: it asks no device, but has a B200's figures
constexpr int SMS = 148;
// Rows of X up to which the narrow kernel is taken: 64 rows against 8192 x 8192, 16.8 us there and 20.8 us by pairs (same device); 40 against 5000 x 5120,
// 9.4 and 14.2; beyond 64 the narrow tile would read W more than once
constexpr int NARROW_M = 64;

struct GemmArgs {
    const float* xs;
    const float* ws;
    void* out;
    float* parts;
    int* status;
    i64 M, out_stride;
    int N, nkb, tiles_m, tiles_n, splits;      // tiles_m: of X's rows
    bool fp32, out_wide, xs_wide;              // 16-byte stores of out, loads of xs and ws
};

struct __align__(16) Ctrl {
    uint64_t full[8], empty[8], tfull[BUFS], tempty[BUFS], sfull[BUFS], sempty[BUFS];
    uint32_t tmem;
    int abort_flag;
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
    static constexpr int LD = COLS;
    static_assert(COLS == 8 || COLS == 16 || COLS == 32, "one load of tensor memory");
    static constexpr uint32_t BLOCK = W_BYTES + TN * KB;
    static constexpr uint32_t STAGE = PER_STEP * BLOCK;
    static constexpr int STAGES = TN == 64 ? 4 : TN == 32 ? 5 : 6;
    static constexpr uint32_t TMEM_COLS = BUFS * PER_STEP * TN;
    static constexpr uint32_t SMEM = 1024 + STAGES * STAGE + BUFS * PER_STEP * TN * 4 + sizeof(Ctrl);
    static_assert(SMEM <= 227 * 1024 && TMEM_COLS <= 512, "");
};

__device__ __forceinline__ void store_one(const GemmArgs& a, i64 row, int col, float v) {
    if (row >= a.M || col >= a.N) return;
    if (a.fp32) static_cast<float*>(a.out)[row * a.out_stride + col] = v;
    else static_cast<cake_bf16*>(a.out)[row * a.out_stride + col] = to_bf16(v);
}

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
    float* const part = reinterpret_cast<float*>(tiles);      // [TN][TM], after the loop
    float* const scales = reinterpret_cast<float*>(tiles + T::STAGES * T::STAGE);
    Ctrl* const ctrl = reinterpret_cast<Ctrl*>(scales + BUFS * PER_STEP * TN);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int items = a.tiles_m * a.tiles_n * a.splits;

    if (threadIdx.x == 0) {
        for (int i = 0; i < T::STAGES; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctrl->full[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctrl->empty[i]), 1);
        }
        for (int i = 0; i < BUFS; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctrl->tfull[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctrl->tempty[i]), EPI_WARPS);
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
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();

    if (warp == WARP_TMA) {
        if (ptx::elect_one()) {
            uint32_t n = 0;      // steps so far
            for (int i = blockIdx.x; i < items && !aborted(ctrl); i += gridDim.x) {
                const Item it = item_of(a, i, TN);
                for (int kb = it.kb0; kb < it.kb1; kb += PER_STEP, ++n) {
                    const uint32_t s = n % T::STAGES, round = n / T::STAGES;
                    wait_bar(&ctrl->empty[s], (round & 1) ^ 1, ctrl, a.status);
                    if (aborted(ctrl)) break;
                    const int blocks = min(PER_STEP, it.kb1 - kb);
                    const uint32_t bar = ptx::smem_u32(&ctrl->full[s]);
                    ptx::mbar_arrive_expect_tx(bar, blocks * T::BLOCK);
                    for (int j = 0; j < blocks; ++j) {
                        const uint32_t dst = ptx::smem_u32(tiles + s * T::STAGE + j * T::BLOCK);
                        tma_load_2d(dst, &map_w, bar, (kb + j) * KB, it.n0);
                        tma_load_2d(dst + W_BYTES, &map_x, bar, (kb + j) * KB, it.m0);
                    }
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
    } else if (warp == WARP_MMA || warp == WARP_MMA1) {
        if (ptx::elect_one()) {
            const uint32_t who = warp == WARP_MMA ? 0 : 1;
            uint32_t n = 0;
            constexpr uint32_t idesc = idesc_e4m3(TM, TN);
            for (int i = blockIdx.x; i < items && !aborted(ctrl); i += gridDim.x) {
                const Item it = item_of(a, i, TN);
                for (int kb = it.kb0; kb < it.kb1; kb += PER_STEP, ++n) {
                    if ((n & 1) != who) continue;
                    const uint32_t s = n % T::STAGES, b = n % BUFS;
                    wait_bar(&ctrl->tempty[b], ((n / BUFS) & 1) ^ 1, ctrl, a.status);
                    wait_bar(&ctrl->full[s], (n / T::STAGES) & 1, ctrl, a.status);
                    if (aborted(ctrl)) break;
                    ptx::tc_fence_after();
                    const int blocks = min(PER_STEP, it.kb1 - kb);
                    for (int j = 0; j < blocks; ++j) {
                        const uint32_t base = ptx::smem_u32(tiles + s * T::STAGE + j * T::BLOCK);
                        const uint64_t da = ptx::umma_desc_sw128(base), db = ptx::umma_desc_sw128(base + W_BYTES);
                        const uint32_t d = tmem + (b * PER_STEP + j) * TN;
                        umma_e4m3<false>(d, da, db, idesc);          // 32 columns (32 bytes) a step
                        umma_e4m3<true>(d, da + 2, db + 2, idesc);
                        umma_e4m3<true>(d, da + 4, db + 4, idesc);
                        umma_e4m3<true>(d, da + 6, db + 6, idesc);
                    }
                    ptx::umma_commit(ptx::smem_u32(&ctrl->tfull[b]));
                    ptx::umma_commit(ptx::smem_u32(&ctrl->empty[s]));
                }
            }
        }
        __syncwarp();
    } else if (warp == WARP_SCALE) {
        // one product xs * ws per column and block; the loads of two steps run together, ahead of the waits
        constexpr int PER = (TN + 31) / 32;
        constexpr int AHEAD = 2 * PER_STEP;
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
                        next[u][j] = (kb + u < it.kb1 && m < a.M) ? a.xs[m * a.nkb + kb + u] * wrow[kb + u] : 0.f;
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
                for (int h = 0; h < 2; ++h) {
                    if (kb + h * PER_STEP >= it.kb1) break;
                    const uint32_t b = n % BUFS;
                    wait_bar(&ctrl->sempty[b], ((n / BUFS) & 1) ^ 1, ctrl, a.status);
#pragma unroll
                    for (int u = 0; u < PER_STEP; ++u)
#pragma unroll
                        for (int j = 0; j < PER; ++j)
                            if (j * 32 + lane < TN) scales[(b * PER_STEP + u) * TN + j * 32 + lane] = cur[h * PER_STEP + u][j];
                    ptx::mbar_arrive(ptx::smem_u32(&ctrl->sfull[b]));
                    ++n;
                }
            }
        }
    } else {
        const int half = warp >> 2, quad = warp & 3;      // a warp reads the 32 lanes of its place in its warpgroup
        const uint32_t t_lane = tmem + (static_cast<uint32_t>(quad * 32) << 16) + half * T::COLS;
        uint32_t n = 0;
        // (after an expired wait this loop and the scales' run on with waits that return at once)
        for (int i = blockIdx.x; i < items; i += gridDim.x) {
            const Item it = item_of(a, i, TN);
            float acc[T::COLS];
#pragma unroll
            for (int c = 0; c < T::COLS; ++c) acc[c] = 0.f;
            for (int kb = it.kb0; kb < it.kb1; kb += PER_STEP, ++n) {
                const uint32_t b = n % BUFS;
                wait_bar(&ctrl->sfull[b], (n / BUFS) & 1, ctrl, a.status);
                wait_bar(&ctrl->tfull[b], (n / BUFS) & 1, ctrl, a.status);
                ptx::tc_fence_after();
#pragma unroll
                for (int j = 0; j < PER_STEP; ++j) {
                    if (j > 0 && kb + j >= it.kb1) break;
                    const float* sc = scales + (b * PER_STEP + j) * TN + half * T::COLS;
                    uint32_t r[T::LD];
                    tmem_load<T::LD>(t_lane + (b * PER_STEP + j) * TN, r);
#pragma unroll
                    for (int c = 0; c < T::LD; c += 4) {
                        const float4 f = *reinterpret_cast<const float4*>(sc + c);
                        acc[c] = fmaf(__uint_as_float(r[c]), f.x, acc[c]);
                        acc[c + 1] = fmaf(__uint_as_float(r[c + 1]), f.y, acc[c + 1]);
                        acc[c + 2] = fmaf(__uint_as_float(r[c + 2]), f.z, acc[c + 2]);
                        acc[c + 3] = fmaf(__uint_as_float(r[c + 3]), f.w, acc[c + 3]);
                    }
                }
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(ptx::smem_u32(&ctrl->tempty[b]));
                    ptx::mbar_arrive(ptx::smem_u32(&ctrl->sempty[b]));
                }
            }
            if (a.splits == 1) {
#pragma unroll
                for (int c = 0; c < T::COLS; ++c) store_one(a, static_cast<i64>(it.m0) + half * T::COLS + c, it.n0 + quad * 32 + lane, acc[c]);
            } else {
                // (the ring is free: every copy has landed and every instruction that read it is complete)
#pragma unroll
                for (int c = 0; c < T::COLS; ++c) part[(half * T::COLS + c) * TM + quad * 32 + lane] = acc[c];
            }
        }
    }
    if (a.splits > 1) {
        // ---- The parts of a tile's contraction lie in the shared memories of the CTAs of a cluster (a tile each, in one round): every CTA
        // adds up its share of the columns, in the order of the parts, and stores it
        __syncwarp();
        ptx::cluster_sync_all();
        const Item it = item_of(a, blockIdx.x, TN);
        const int c0 = it.split * TN / a.splits, c1 = (it.split + 1) * TN / a.splits;
        const uint32_t mine = ptx::smem_u32(part);
        const int w4 = 4 * (threadIdx.x % (TM / 4));       // four rows of W
        for (int c = c0 + threadIdx.x / (TM / 4); c < c1; c += THREADS / (TM / 4)) {
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int s = 0; s < a.splits; ++s) {
                uint32_t from;
                float4 v;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(mine + (c * TM + w4) * 4), "r"(s));
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(from) : "memory");
                sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
            }
            const i64 row = static_cast<i64>(it.m0) + c;
            const int col = it.n0 + w4;
            if (a.out_wide && row < a.M && col + 4 <= a.N) {
                if (a.fp32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + row * a.out_stride + col) = sum;
                else *reinterpret_cast<uint2*>(static_cast<cake_bf16*>(a.out) + row * a.out_stride + col) = make_uint2(pack_bf16(sum.x, sum.y), pack_bf16(sum.z, sum.w));
            } else {
                store_one(a, row, col, sum.x), store_one(a, row, col + 1, sum.y), store_one(a, row, col + 2, sum.z), store_one(a, row, col + 3, sum.w);
            }
        }
        ptx::cluster_sync_all();                           // no CTA leaves while another reads its part
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == WARP_MMA) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, T::TMEM_COLS);
    }
}

// ------------------------------------------------------------------------------------------------------ more rows: CTA pairs
namespace wide {

constexpr int BM = 256;                        // rows of X of a pair's tile
constexpr int PAIR_EPI = 8;                    // epilogue warps
constexpr int PAIR_TMA = 8, PAIR_MMA = 9, PAIR_MMA1 = 10;
// registers: 12 warps start with 168 each; the two epilogue warpgroups take what the third gives up (2 * 232 + 40 = 3 * 168)
constexpr int EPI_REGS = 232, AUX_REGS = 40;
constexpr int GROUP = 4;                       // blocks whose scales are fetched together
constexpr int PAIR_THREADS = 12 * 32;
constexpr int OUT_PITCH = 80;                  // bytes of a staged row: 64 and a shift of the banks
constexpr uint32_t OUT_BYTES = PAIR_EPI * 32 * OUT_PITCH;
constexpr int BAND = 8;                        // tiles of X's rows that are worked on together, for the L2
constexpr int ACC = 128;                       // columns of an accumulator (and of an instruction); four of them fill tensor memory

// BN: rows of W of a pair's tile.  256: an issuing thread and two accumulators for each half of the columns, read by a warpgroup each.
// 128: the issuing threads take turns block by block, all epilogue warps read every accumulator.
template <int BN>
struct Shape {
    static constexpr bool HALVES = BN == 256;
    static constexpr uint32_t X_BYTES = 128 * KB, W_PART = 64 * KB;       // a CTA's 128 rows of X; its 64 rows of an instruction's W
    static constexpr uint32_t STAGE = X_BYTES + (HALVES ? 2 : 1) * W_PART;
    static constexpr int STAGES = HALVES ? 6 : 8;
    static constexpr int COLS = BN / 2;                                   // columns of an epilogue thread
};

struct __align__(16) PairCtrl {
    uint64_t full[8], empty[8], tfull[4], tempty[4];      // accumulators 0, 1: the first issuing thread's; 2, 3: the second's
    uint32_t tmem;
    int abort_flag;
};
template <int BN>
constexpr uint32_t pair_smem() { return 1024 + Shape<BN>::STAGES * Shape<BN>::STAGE + OUT_BYTES + sizeof(PairCtrl); }
static_assert(pair_smem<256>() <= 227 * 1024 && pair_smem<128>() <= 227 * 1024, "");

__device__ __forceinline__ void pair_wait(uint64_t* bar, uint32_t parity, PairCtrl* ctrl, int* status) {
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
__device__ __forceinline__ bool pair_aborted(PairCtrl* ctrl) { return *reinterpret_cast<volatile int*>(&ctrl->abort_flag) != 0; }
// the same place in rank 0's shared memory
__device__ __forceinline__ uint32_t at_rank0(const void* p) { return ptx::smem_u32(p) & ~ptx::CLUSTER_PEER_BIT; }

template <bool ACC>
__device__ __forceinline__ void umma_pair_e4m3(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "n"(ACC ? 1 : 0)
        : "memory");
}
// acc (two floats) += r * s
__device__ __forceinline__ void fma2(float2& acc, uint32_t r0, uint32_t r1, float s) {
    asm("{\n\t.reg .b64 a, b, c;\n\t"
        "mov.b64 a, {%2, %3};\n\t"
        "mov.b64 b, {%4, %4};\n\t"
        "mov.b64 c, {%0, %1};\n\t"
        "fma.rn.f32x2 c, a, b, c;\n\t"
        "mov.b64 {%0, %1}, c;\n\t}"
        : "+f"(acc.x), "+f"(acc.y) : "r"(r0), "r"(r1), "f"(s));
}

struct PairItem {
    int m0, n0, kb0, kb1, split, tile;
};
// Tiles in bands of BAND tiles of X's rows, all of W's tiles through a band; the parts of a tile next to each other.
template <int BN>
__device__ __forceinline__ PairItem pair_item(const GemmArgs& a, int i) {
    PairItem it;
    it.split = i % a.splits;
    it.tile = i / a.splits;
    const int band = it.tile / (BAND * a.tiles_n);
    const int in_band = it.tile - band * BAND * a.tiles_n;
    const int high = min(BAND, a.tiles_m - band * BAND);
    const int nt = in_band / high;
    it.m0 = (band * BAND + in_band - nt * high) * BM;
    it.n0 = nt * BN;
    it.kb0 = static_cast<int>(static_cast<i64>(it.split) * a.nkb / a.splits);
    it.kb1 = static_cast<int>(static_cast<i64>(it.split + 1) * a.nkb / a.splits);
    return it;
}

template <int BN>
__global__ void __launch_bounds__(PAIR_THREADS, 1)
gemm_fp8_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const GemmArgs a) {
    using S = Shape<BN>;
    constexpr int STAGES = S::STAGES, COLS = S::COLS;
    constexpr uint32_t STAGE = S::STAGE;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* const tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* const staging = tiles + STAGES * STAGE;
    PairCtrl* const ctrl = reinterpret_cast<PairCtrl*>(staging + OUT_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_ctarank();
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const int items = a.tiles_m * a.tiles_n * a.splits;

    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctrl->full[i]), 1);          // rank 0's: both CTAs' bytes
            ptx::mbar_init(ptx::smem_u32(&ctrl->empty[i]), S::HALVES ? 2 : 1);     // issuing threads that read a stage
        }
        for (int i = 0; i < 4; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctrl->tfull[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctrl->tempty[i]), S::HALVES ? PAIR_EPI : 2 * PAIR_EPI);   // rank 0's: warps of both CTAs
        }
        ctrl->abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&map_w);
        ptx::prefetch_tensormap(&map_x);
    }
    if (warp == PAIR_MMA) {
        ptx::tmem_alloc_pair(ptx::smem_u32(&ctrl->tmem), 4 * ACC);
        ptx::tmem_relinquish_pair();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::cluster_sync_all();         // both CTAs' barriers and tensor memory are set up
    ptx::tc_fence_after();
    const uint32_t tmem = ctrl->tmem;
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();

    if (warp >= PAIR_EPI) {
    ptx::setmaxnreg_dec<AUX_REGS>();
    if (warp == PAIR_TMA) {
        if (ptx::elect_one()) {
            uint32_t n = 0;
            for (int i = pair; i < items && !pair_aborted(ctrl); i += n_pairs) {
                const PairItem it = pair_item<BN>(a, i);
                const int x_row = it.m0 + static_cast<int>(rank) * 128, w_row = it.n0 + static_cast<int>(rank) * 64;
                for (int kb = it.kb0; kb < it.kb1; ++kb, ++n) {
                    const uint32_t s = n % STAGES;
                    pair_wait(&ctrl->empty[s], ((n / STAGES) & 1) ^ 1, ctrl, a.status);
                    if (pair_aborted(ctrl)) break;
                    if (rank == 0) ptx::mbar_arrive_expect_tx(ptx::smem_u32(&ctrl->full[s]), 2 * STAGE);
                    const uint32_t bar = at_rank0(&ctrl->full[s]), dst = ptx::smem_u32(tiles + s * STAGE);
                    ptx::tma_load_2d_pair(dst, &map_x, bar, kb * KB, x_row);
                    ptx::tma_load_2d_pair(dst + S::X_BYTES, &map_w, bar, kb * KB, w_row);
                    if (S::HALVES) ptx::tma_load_2d_pair(dst + S::X_BYTES + S::W_PART, &map_w, bar, kb * KB, w_row + 128);
                }
            }
            if (pair_aborted(ctrl)) {        // give copies in flight a bounded time to land
                const uint64_t t0 = ptx::globaltimer_ns();
                while (ptx::globaltimer_ns() - t0 < 1000000ull) {}
            }
        }
        __syncwarp();
    } else if (warp == PAIR_MMA || warp == PAIR_MMA1) {
        // Two issuing threads (rank 0): an instruction is accepted at the tensor core's pace, and one thread's waits and commits on top
        // of that left it idle.  Each has two accumulators of 128 columns, so the tensor core comes back to one as soon as the warps that
        // read it are done.  An instruction's 128 rows of W lie in both CTAs, 64 each
        if (rank == 0 && ptx::elect_one()) {
            const uint32_t who = warp == PAIR_MMA ? 0 : 1;
            uint32_t n = 0, u = 0;      // blocks; blocks that are this thread's
            constexpr uint32_t idesc = idesc_e4m3(BM, ACC);
            constexpr uint16_t BOTH = 3;
            for (int i = pair; i < items && !pair_aborted(ctrl); i += n_pairs) {
                const PairItem it = pair_item<BN>(a, i);
                for (int kb = it.kb0; kb < it.kb1; ++kb, ++n) {
                    if (!S::HALVES && (n & 1) != who) continue;
                    const uint32_t s = n % STAGES, acc = 2 * who + (u & 1);
                    pair_wait(&ctrl->full[s], (n / STAGES) & 1, ctrl, a.status);
                    pair_wait(&ctrl->tempty[acc], ((u >> 1) & 1) ^ 1, ctrl, a.status);
                    if (pair_aborted(ctrl)) break;
                    ptx::tc_fence_after();
                    const uint32_t d = tmem + acc * ACC;
                    const uint32_t base = ptx::smem_u32(tiles + s * STAGE);
                    const uint64_t da = ptx::umma_desc_sw128(base), db = ptx::umma_desc_sw128(base + S::X_BYTES + (S::HALVES ? who * S::W_PART : 0));
                    umma_pair_e4m3<false>(d, da, db, idesc);
                    umma_pair_e4m3<true>(d, da + 2, db + 2, idesc);
                    umma_pair_e4m3<true>(d, da + 4, db + 4, idesc);
                    umma_pair_e4m3<true>(d, da + 6, db + 6, idesc);
                    ptx::umma_pair_commit(ptx::smem_u32(&ctrl->tfull[acc]), BOTH);
                    ptx::umma_pair_commit(ptx::smem_u32(&ctrl->empty[s]), BOTH);
                    ++u;
                }
            }
        }
        __syncwarp();
    }
    } else {
        ptx::setmaxnreg_inc<EPI_REGS>();
        const int half = warp >> 2, quad = warp & 3;
        const uint32_t t_lane = tmem + (static_cast<uint32_t>(quad * 32) << 16) + (S::HALVES ? 0 : half * COLS);
        // block n is in accumulator acc_of(n), completed for the round_of(n)-th time
        auto acc_of = [&](uint32_t n) { return S::HALVES ? 2 * half + (n & 1) : 2 * (n & 1) + ((n >> 1) & 1); };
        auto round_of = [&](uint32_t n) { return S::HALVES ? n >> 1 : n >> 2; };
        const int local_row = quad * 32 + lane;                        // of the CTA's 128
        uint8_t* const stage_out = staging + warp * 32 * OUT_PITCH;
        const int n_blocks = (a.N + 127) / 128;
        uint32_t n = 0;
        for (int i = pair; i < items; i += n_pairs) {                  // (every warp takes every step, also after an expired wait)
            const PairItem it = pair_item<BN>(a, i);
            float2 acc[COLS / 2];
#pragma unroll
            for (int c = 0; c < COLS / 2; ++c) acc[c] = make_float2(0.f, 0.f);
            // The scales of four blocks at a time, one such group ahead and without a barrier: at this thread's pace (about 500 clocks a
            // block) a wait on a barrier, even a completed one, is dearer than the loads
            const i64 row = static_cast<i64>(it.m0) + rank * 128 + local_row;
            const int block = it.n0 / 128 + (S::HALVES ? half : 0);
            const bool live = row < a.M && block < n_blocks;
            const float* const xs = a.xs + (live ? row : 0) * a.nkb;
            const float* const ws = a.ws + static_cast<i64>(live ? block : 0) * a.nkb;
            float xn[GROUP], wn[GROUP], sc[GROUP], s_now = 0.f;
            auto fetch = [&](int kb) {
                if (a.xs_wide && kb % GROUP == 0 && kb + GROUP <= it.kb1) {
                    const float4 u = *reinterpret_cast<const float4*>(xs + kb), v = *reinterpret_cast<const float4*>(ws + kb);
                    xn[0] = u.x, xn[1] = u.y, xn[2] = u.z, xn[3] = u.w;
                    wn[0] = v.x, wn[1] = v.y, wn[2] = v.z, wn[3] = v.w;
                } else {
#pragma unroll
                    for (int u = 0; u < GROUP; ++u) {
                        xn[u] = kb + u < it.kb1 ? xs[kb + u] : 0.f;
                        wn[u] = kb + u < it.kb1 ? ws[kb + u] : 0.f;
                    }
                }
            };
            fetch(it.kb0);
            // The block's columns in loads of 32, each in flight while the one before is added up; the first of the next block as well,
            // if that block is done already
            constexpr int LOADS = COLS / 32;
            uint32_t r[2][32];
            auto add = [&](int c) {
#pragma unroll
                for (int q = 0; q < 16; ++q) fma2(acc[c * 16 + q], r[c & 1][2 * q], r[c & 1][2 * q + 1], s_now);
            };
            pair_wait(&ctrl->tfull[acc_of(n)], round_of(n) & 1, ctrl, a.status);
            ptx::tc_fence_after();
            ptx::tmem_ld_x32(t_lane + acc_of(n) * ACC, r[0]);
            for (int kb0 = it.kb0; kb0 < it.kb1; kb0 += GROUP) {
#pragma unroll
                for (int u = 0; u < GROUP; ++u) sc[u] = live ? xn[u] * wn[u] : 0.f;
                if (kb0 + GROUP < it.kb1) fetch(kb0 + GROUP);
#pragma unroll
                for (int u = 0; u < GROUP; ++u) {
                    const int kb = kb0 + u;
                    if (kb >= it.kb1) break;
                    s_now = sc[u];
                    const uint32_t b = acc_of(n);
                    const uint32_t t = t_lane + b * ACC;
                    ++n;
                    const uint32_t nb = acc_of(n);
                    uint64_t* const next = &ctrl->tfull[nb];
                    const uint32_t parity = round_of(n) & 1;
                    const bool more = kb + 1 < it.kb1;
                    bool ready = false;
#pragma unroll
                    for (int c = 0; c < LOADS; ++c) {
                        ptx::tmem_ld_wait(r[c & 1]);
                        if (c + 1 < LOADS) {
                            ptx::tmem_ld_x32(t + 32 * (c + 1), r[(c + 1) & 1]);
                            if (c + 2 == LOADS) ready = more && ptx::mbar_test_wait(ptx::smem_u32(next), parity);
                            add(c);
                        }
                    }
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive_cluster(at_rank0(&ctrl->tempty[b]));
                    if (__all_sync(0xffffffffu, ready)) {
                        ptx::tc_fence_after();
                        ptx::tmem_ld_x32(t_lane + nb * ACC, r[0]);
                        add(LOADS - 1);
                    } else {
                        add(LOADS - 1);
                        if (more) {
                            pair_wait(next, parity, ctrl, a.status);
                            ptx::tc_fence_after();
                            ptx::tmem_ld_x32(t_lane + nb * ACC, r[0]);
                        }
                    }
                }
            }
            // ---- out: 64 bytes of each of the warp's 32 rows at a time through shared memory, so that a store instruction covers whole
            // sectors of 8 rows instead of 16 bytes of 32.  (A part of a split contraction goes to the workspace, as a matrix of its own)
            const bool part = a.splits > 1, fp32 = part || a.fp32;
            const int elem = fp32 ? 4 : 2, per = 16 / elem;                 // bytes of an element, elements of 16 bytes
            const int col0 = (part ? 0 : it.n0) + half * COLS + (lane & 3) * per;
            const int n_cols = part ? BN : a.N;
            const i64 row0 = (part ? 0 : static_cast<i64>(it.m0)) + rank * 128 + quad * 32 + (lane >> 2);
            const i64 n_rows = part ? min(static_cast<i64>(BM), a.M - it.m0) : a.M;
            const i64 pitch = (part ? BN : a.out_stride) * elem;
            uint8_t* const to = (part ? reinterpret_cast<uint8_t*>(a.parts + static_cast<i64>(i) * (BM * BN)) : static_cast<uint8_t*>(a.out)) +
                                row0 * pitch + static_cast<i64>(col0) * elem;
            const bool whole = (part || a.out_wide) && (part ? 0 : it.n0) + BN <= n_cols;
            uint4* const put = reinterpret_cast<uint4*>(stage_out + lane * OUT_PITCH);
            const uint8_t* const get = stage_out + (lane >> 2) * OUT_PITCH + (lane & 3) * 16;
            auto flush = [&](int run) {                                     // the run-th 64 bytes of the warp's rows
                __syncwarp();
                if (whole) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint4 u = *reinterpret_cast<const uint4*>(get + k * 8 * OUT_PITCH);
                        if (row0 + 8 * k < n_rows) *reinterpret_cast<uint4*>(to + 8 * k * pitch + run * 64) = u;
                    }
                } else {        // edges, and rows that are no multiple of 16 bytes apart: element by element, a row's next to each other
                    const int wide = 64 / elem, c = lane % wide, col = it.n0 + half * COLS + run * wide + c;
                    const i64 first = static_cast<i64>(it.m0) + rank * 128 + quad * 32;
                    if (col < n_cols) {
#pragma unroll 4
                        for (int r = lane / wide; r < 32; r += 32 / wide) {
                            if (first + r >= n_rows) break;
                            const uint8_t* from = stage_out + r * OUT_PITCH + c * elem;
                            uint8_t* dst = static_cast<uint8_t*>(a.out) + (first + r) * pitch + static_cast<i64>(col) * elem;
                            if (fp32) *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(from);
                            else *reinterpret_cast<uint16_t*>(dst) = *reinterpret_cast<const uint16_t*>(from);
                        }
                    }
                }
                __syncwarp();
            };
#pragma unroll
            for (int c = 0; c < COLS / 32; ++c) {
                const float2* f = acc + 16 * c;
                if (fp32) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            put[q] = make_uint4(__float_as_uint(f[8 * h + 2 * q].x), __float_as_uint(f[8 * h + 2 * q].y),
                                                __float_as_uint(f[8 * h + 2 * q + 1].x), __float_as_uint(f[8 * h + 2 * q + 1].y));
                        flush(2 * c + h);
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        put[q] = make_uint4(pack_bf16(f[4 * q].x, f[4 * q].y), pack_bf16(f[4 * q + 1].x, f[4 * q + 1].y),
                                            pack_bf16(f[4 * q + 2].x, f[4 * q + 2].y), pack_bf16(f[4 * q + 3].x, f[4 * q + 3].y));
                    flush(c);
                }
            }
        }
    }
    // neither CTA leaves while the other's MMAs, loads or arrivals can still reach it
    ptx::tc_fence_before();
    __syncthreads();
    ptx::cluster_sync_all();
    if (warp == PAIR_MMA) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc_pair(tmem, 4 * ACC);
    }
}

// (the parts of a split contraction are no more than the pairs of SMs: one round)
static_assert(kHeaderBytes + static_cast<size_t>(SMS / 2) * BM * 256 * 4 == CAKE_GEMM_FP8_MOST_WORKSPACE_BYTES, "the most that a plan asks for, and the ABI's constant");

// Sums of the parts of a split contraction, in order; four columns to a thread.
template <int BN>
__global__ void __launch_bounds__(256)
gemm_join_kernel(const GemmArgs a) {
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    const int quads = (a.N + 3) / 4;
    const i64 total = a.M * quads;
    for (i64 e = static_cast<i64>(blockIdx.x) * blockDim.x + threadIdx.x; e < total; e += static_cast<i64>(gridDim.x) * blockDim.x) {
        const i64 m = e / quads;
        const int n = 4 * static_cast<int>(e - m * quads);
        const int tm = static_cast<int>(m / BM), tn = n / BN;
        const int band = tm / BAND, high = min(BAND, a.tiles_m - band * BAND);
        const i64 tile = static_cast<i64>(band) * BAND * a.tiles_n + tn * high + (tm - band * BAND);
        const float4* from = reinterpret_cast<const float4*>(a.parts + tile * a.splits * (BM * BN) + (m - static_cast<i64>(tm) * BM) * BN + (n - tn * BN));
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s) {
            const float4 v = __ldcg(from + static_cast<i64>(s) * (BM * BN / 4));
            sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
        }
        const float f[4] = {sum.x, sum.y, sum.z, sum.w};
        if (a.fp32) {
            float* dst = static_cast<float*>(a.out) + m * a.out_stride + n;
            if (a.out_wide && n + 4 <= a.N) *reinterpret_cast<float4*>(dst) = sum;
            else
                for (int q = 0; q < 4; ++q)
                    if (n + q < a.N) dst[q] = f[q];
        } else {
            cake_bf16* dst = static_cast<cake_bf16*>(a.out) + m * a.out_stride + n;
            if (a.out_wide && n + 4 <= a.N) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
            else
                for (int q = 0; q < 4; ++q)
                    if (n + q < a.N) dst[q] = to_bf16(f[q]);
        }
    }
}

}  // namespace wide

// ---------------------------------------------------------------------------------------------------------------- host
constexpr int MOST_PARTS = 8;      // CTAs of a cluster
// Clusters of so many CTAs of the narrow kernel (one to an SM) that a B200 runs at once, as the occupancy query counts them: fewer than
// the SMs divided by their size, since a cluster stays inside one group of SMs.  A chip grouped otherwise runs some of them later
constexpr int CLUSTERS[MOST_PARTS + 1] = {0, SMS, 74, 45, 33, 26, 22, 15, 15};
struct Plan {
    bool pair;
    int tn, bn, tiles_m, tiles_n, splits, nkb;
    size_t part_bytes;
};
Plan plan_of(i64 M, int N, int K) {
    Plan p;
    p.nkb = (K + KB - 1) / KB;
    p.pair = M > NARROW_M;
    p.tn = p.pair ? wide::BM : M <= 16 ? 16 : M <= 32 ? 32 : 64;
    p.tiles_m = static_cast<int>((M + p.tn - 1) / p.tn);
    const int units = p.pair ? SMS / 2 : SMS;        // that work on a tile each
    // The shape of a pair's tile, and parts of the contraction (all of them in one round): what needs the least time, counted in
    // nanoseconds of a block (measured over 128 blocks: 510 of 256 x 256, 290 of 256 x 128), of a tile's start and end, and of
    // writing and joining the parts.  517 x 2624 x 5120: 22.3 us in 256 x 256 tiles and two parts, 15.7 - 18.3 in 256 x 128
    double least = 1e300;
    for (int bn : {256, 128}) {
        if (!p.pair && bn == 256) continue;
        const int tiles_n = (N + bn - 1) / bn;
        const i64 tiles = static_cast<i64>(p.tiles_m) * tiles_n;
        const double block = !p.pair ? 150 : bn == 256 ? 510 : 290, tile = p.pair ? (bn == 256 ? 2000 : 1200) : 1000;
        for (int s = 1; s == 1 || (s <= p.nkb / 2 && s <= (p.pair ? 32 : MOST_PARTS) && tiles * s <= units); ++s) {
            if (!p.pair && tiles > CLUSTERS[s] && s > 1) continue;
            const double rounds = static_cast<double>((tiles * s + units - 1) / units);
            double cost = rounds * ((p.nkb + s - 1) / s * block + tile);
            if (s > 1) cost += p.pair ? 3000 + (bn == 256 ? 2000 : 1000) + 300 * s : 700 + 30 * s;
            if (cost < least) least = cost, p.bn = bn, p.tiles_n = tiles_n, p.splits = s;
        }
    }
    const i64 tiles = static_cast<i64>(p.tiles_m) * p.tiles_n;
    p.part_bytes = p.pair && p.splits > 1 ? static_cast<size_t>(tiles) * p.splits * wide::BM * p.bn * 4 : 0;
    return p;
}

template <int TN>
int launch(const GemmArgs& a, const CUtensorMap& mw, const CUtensorMap& mx, const DeviceInfo& di, cudaStream_t s) {
    using T = Tile<TN>;
    static PerDevice ready;
    if (!ready.get(di.device, [] { return allow_smem(gemm_fp8_kernel<TN>, T::SMEM); })) return CAKE_ERR_CUDA;
    const i64 items = static_cast<i64>(a.tiles_m) * a.tiles_n * a.splits;
    if (a.splits == 1) {
        const int ctas = static_cast<int>(items < di.sm_count ? items : di.sm_count);
        return launch_early(gemm_fp8_kernel<TN>, dim3(ctas), dim3(THREADS), T::SMEM, s, mw, mx, a) == cudaSuccess ? CAKE_OK : CAKE_ERR_CUDA;
    }
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;      // the parts of a tile
    at[0].val.clusterDim.x = a.splits;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // as launch_early
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(items));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = T::SMEM;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, gemm_fp8_kernel<TN>, mw, mx, a) != cudaSuccess) {
        cudaGetLastError();
        return CAKE_ERR_CUDA;
    }
    note_launches(1);
    return CAKE_OK;
}

template <int BN>
int launch_pair(const GemmArgs& a, const CUtensorMap& mw, const CUtensorMap& mx, const DeviceInfo& di, cudaStream_t s) {
    static PerDevice ready;
    if (!ready.get(di.device, [] { return allow_smem(wide::gemm_fp8_pair_kernel<BN>, wide::pair_smem<BN>()); })) return CAKE_ERR_CUDA;
    const i64 items = static_cast<i64>(a.tiles_m) * a.tiles_n * a.splits;
    const int pairs = static_cast<int>(items < di.sm_count / 2 ? items : di.sm_count / 2);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * pairs);
    cfg.blockDim = dim3(wide::PAIR_THREADS);
    cfg.dynamicSmemBytes = wide::pair_smem<BN>();
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // as launch_early
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, wide::gemm_fp8_pair_kernel<BN>, mw, mx, a) != cudaSuccess) {
        cudaGetLastError();
        return CAKE_ERR_CUDA;
    }
    note_launches(1);
    if (a.splits == 1) return CAKE_OK;
    const i64 threads = a.M * ((a.N + 3) / 4);
    const i64 blocks = threads / 256 + 1;
    return launch_early(wide::gemm_join_kernel<BN>, dim3(static_cast<unsigned>(blocks < 8 * di.sm_count ? blocks : 8 * di.sm_count)), dim3(256), 0, s, a) ==
                   cudaSuccess ? CAKE_OK : CAKE_ERR_CUDA;
}

int check_shape(i64 M, int N, int K) {
    if (M < 0 || N < 1 || K < 1 || M > INT_MAX - 1024 || N > INT_MAX - 1024 || K > INT_MAX - 1024) return CAKE_ERR_SHAPE;
    if (((M + 127) / 128) * ((static_cast<i64>(N) + TM - 1) / TM) > INT_MAX / 64) return CAKE_ERR_SHAPE;
    return CAKE_OK;
}

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
    *out_bytes = kHeaderBytes + plan_of(M, N, K).part_bytes;
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
    const Plan p = plan_of(M, N, K);
    if (ws_bytes < kHeaderBytes + p.part_bytes) return CAKE_ERR_WORKSPACE;
    DeviceInfo di;
    rc = current_device_info(&di);
    if (rc != CAKE_OK) return rc;
    if (di.cc_major != 10) return CAKE_ERR_DEVICE;
    CUtensorMap mw, mx;
    rc = make_tmap_bytes(&mw, W, K, N, w_stride, p.pair ? 64 : TM);
    if (rc != CAKE_OK) return rc;
    rc = make_tmap_bytes(&mx, X, K, M, x_stride, p.pair ? 128 : p.tn);
    if (rc != CAKE_OK) return rc;
    GemmArgs a;
    a.xs = x_scale, a.ws = w_scale, a.out = out, a.status = static_cast<int*>(ws);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + kHeaderBytes);
    a.M = M, a.out_stride = out_stride, a.N = N, a.nkb = p.nkb, a.tiles_m = p.tiles_m, a.tiles_n = p.tiles_n, a.splits = p.splits;
    a.fp32 = flags & CAKE_GEMM_OUT_FP32;
    a.xs_wide = aligned(x_scale, 16) && aligned(w_scale, 16) && p.nkb % 4 == 0;
    a.out_wide = aligned(out, 16) && out_stride % (a.fp32 ? 4 : 8) == 0;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (p.pair) return p.bn == 256 ? launch_pair<256>(a, mw, mx, di, s) : launch_pair<128>(a, mw, mx, di, s);
    switch (p.tn) {
        case 16: return launch<16>(a, mw, mx, di, s);
        case 32: return launch<32>(a, mw, mx, di, s);
        default: return launch<64>(a, mw, mx, di, s);
    }
}

}  // extern "C"
