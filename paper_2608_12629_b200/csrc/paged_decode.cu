// Attention of one new token per sequence over a paged cache, split over the cache's length and joined.
//
//   out = sum_t exp(x_t - m) v_t / sum_t exp(x_t - m),   x_t = scale * q . k_t,   m = max_t x_t
//
// One pass over the keys and values with the running maximum m, sum l and weighted sum O of a softmax; parts (m, l, O) of
// the same row join by  m = max m_i,  l = sum l_i e^(m_i - m),  O = sum O_i e^(m_i - m).  Bound by memory: every key and
// value is read once, so everything here serves to keep loads in flight.
//
// Work is the list of tiles (16 keys for each of a CTA's warps: 64; 32 for bf16 heads of 256) of all (sequence, key-value head) entries, one after the other; CTA c of n takes tiles
// [c T / n, (c+1) T / n): equal shares whatever the lengths are.  An entry that several CTAs share is joined from parts
// in the workspace, in the order of the CTAs: by the last of them to arrive, in two levels, or by a second kernel where either would be much for one SM.
//
// A warp works on 16 keys at a time, with a ring of its own in shared memory and no barrier between warps.  Long rows are
// fetched by one instruction of the warp a step: each lane copies one row (bulk copy; lanes 0-15 the keys, 16-31 the values); short
// ones 16 bytes per lane and instruction.  They land at a pitch at which the reads below meet no bank twice.
//   scores:  S^T[key][head] = K Q^T   (m16n8k16: 16 keys x 8 heads; the contraction's order of elements is permuted the same way
//            in both operands so that a lane's 16-byte run of a key feeds whole k-steps)
//   output:  O^T[d][head] += V^T P    (16 values of d x 8 heads x 16 keys; V^T by transposing matrix loads, P's operand from
//            S^T's accumulators by an 8x8 transpose between lanes)
// Query heads that share a key-value head sit side by side in the 8 (or 16) columns, so the group costs one read.
//
// Measured (32 query, 8 key-value heads of 128, bf16): 64 sequences of 512 to 8,192 tokens 187 us, 6.20 TB/s, 95 % of the copy rate, bound by
// memory.  Four of up to 131,072 tokens, 64 query heads, 8-bit: 141 us, 4.93 TB/s, 75 %: 16-byte copies, conversions and the softmax of
// twice the keys per byte keep the schedulers half busy and a warp's chain of steps is what is left.  One of 777 tokens: 7.8 us, all latency (lengths, table,
// keys, join).  First form (lane-wise 16-byte copies everywhere, maximum exact at every step): 301, 253 and 30 us.
#include "ptx.cuh"
#include "serving.cuh"

namespace cake {
namespace serving {

int check_cache(const cake_paged_cache* c);   // kv_append.cu

namespace {

constexpr int KEYS = 16;                 // keys of a warp's step
constexpr int MOST_WARPS = 4;
constexpr int kPartCtas = 1024;          // CTAs that the workspace has room for parts of (two each)
static_assert(3 * kPartCtas <= kMaxCtas, "arrival counters: of entries, of groups, of entries' first groups");
constexpr int PART_BATCH = 8;            // parts that a join has in flight
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NEG_INF = -INFINITY;
constexpr int WAIT_TRIES = 100000;       // of 20 us each

// an entry that several CTAs share
struct Split {
    int b, g, run, c0, c1;           // the CTAs
    int pad[3];
};

// where finished rows go
struct Rows {
    cake_bf16* out;
    float* lse;
    bool wide;                       // 8-byte stores
};

struct DecodeArgs {
    cake_paged_cache c;
    const cake_bf16* q;
    const int* table;
    const int* lens;
    Rows rows;
    int* status;
    int* counters;
    float* parts;
    struct Split* splits;
    int* n_splits;                   // entries in `splits`; [1]: join blocks that are done
    bool defer;                      // entries that several CTAs share are joined by a second kernel
    int few;                         // else: parts that the last CTA joins by itself
    i64 q_stride, q_head_stride, table_stride, table_head_stride, lens_stride, lens_head_stride;
    bool q_wide;                     // 16-byte loads
    int B, Hq, G, chunks, max_pages, window;   // chunks: runs of at most 8 * NT query heads of a key-value head
    float scale;
};

template <int D, bool E4M3>
struct Layout {
    static constexpr int ELEM = E4M3 ? 1 : 2;
    static constexpr int ROW = D * ELEM;                                            // bytes of a key
    // a key's row is read in runs of VK bytes by four lanes, eight rows at a time: 8 rows apart by 64 (32) bytes modulo 128
    static constexpr int VK = ROW % 64 == 0 ? 16 : 8;
    static constexpr int CK = ROW / (4 * VK);                                       // runs of a lane per key
    static constexpr int K_PITCH = VK == 16 ? (ROW % 128 == 64 ? ROW : ROW + 64) : (ROW / 128 * 128 + 160);
    // a value's row is read 16 bytes at a time, eight rows at once: an odd number of 16-byte units apart
    static constexpr int V_PITCH = (ROW / 16) % 2 == 1 ? ROW : ROW + 16;
    static constexpr int K_BYTES = KEYS * K_PITCH;
    // Rows of 256 bytes and more: one bulk copy per row.  An SM takes about 160 bulk copies a microsecond, whatever their size, so that
    // shorter rows (128 bytes: 2.8 TB/s) are fetched by 16-byte asynchronous copies of all lanes instead
    static constexpr bool BULK = ROW >= 256;
    static constexpr int UNITS = ROW / 16;                                          // 16-byte units of a row
    static constexpr int STAGE = KEYS * (K_PITCH + V_PITCH);                        // of a warp
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool ok) {      // zeros where !ok
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int N>
__device__ __forceinline__ void lds(uint32_t addr, uint32_t (&w)[N / 4]) {
    if constexpr (N == 16) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
    else if constexpr (N == 8) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(addr) : "memory");
    else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(addr) : "memory");
}

template <bool F16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], const uint32_t b0, const uint32_t b1) {
    if (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {      // 2 ulp; below 2^-126 flushed to zero
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// four 8x8 matrices of 16-bit elements, each transposed; lane i gives the address of row i % 8 of matrix i / 8
__device__ __forceinline__ void ldmatrix_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// four e4m3 values to two pairs of f16: exact
__device__ __forceinline__ void e4m3_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    const uint16_t a = static_cast<uint16_t>(w & 0xffffu), b = static_cast<uint16_t>(w >> 16);
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"(a));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"(b));
}

// tokens of sequence b and key-value head g that are attended to: [first, first + count)
__device__ __forceinline__ void span_of(const DecodeArgs& a, int b, int g, int& first, int& count, bool& cut) {
    const i64 room = static_cast<i64>(a.max_pages) * a.c.page_size;
    i64 n = a.lens[b * a.lens_stride + g * a.lens_head_stride];
    cut = n > room;
    if (cut) n = room;
    if (n < 0) n = 0;
    const i64 w = (a.window > 0 && a.window < n) ? a.window : n;
    first = static_cast<int>(n - w);
    count = static_cast<int>(w);
}
template <int TILE>
__device__ __forceinline__ int tiles_of(int count) { return count > 0 ? (count - 1) / TILE + 1 : 1; }   // an empty row still has to be written

// four values of a finished row: (their sum, the row's maximum and sum of exponentials)
template <int D>
__device__ __forceinline__ void write_out(const Rows& r, i64 row, int d, const float4& acc, float top, float sum, float vs) {
    const float f = sum == 0.f ? 0.f : vs / sum;                    // no token weighs anything: zeros
    const uint2 w = make_uint2(pack_bf16(acc.x * f, acc.y * f), pack_bf16(acc.z * f, acc.w * f));
    cake_bf16* dst = r.out + row * D + d;
    if (r.wide) {
        *reinterpret_cast<uint2*>(dst) = w;
    } else {
        dst[0] = w.x & 0xffff, dst[1] = w.x >> 16, dst[2] = w.y & 0xffff, dst[3] = w.y >> 16;
    }
    if (r.lse && d == 0) r.lse[row] = (top + log2f(sum)) * LN2;
}

// The work list: entries in the order (sequence, key-value head, run of query heads), each of tiles_of(its tokens) tiles.
struct Cursor {
    int b, g, run, first, count, tiles;
    i64 start;        // number of the entry's first tile in the list
};

// parts c, c + step, ... of four values of a row, joined
struct Joined {
    float top = NEG_INF, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);

    __device__ __forceinline__ void rescale(float up) {
        const float f = ex2(top - (up == NEG_INF ? 0.f : up));
        sum *= f, acc.x *= f, acc.y *= f, acc.z *= f, acc.w *= f;
        top = up;
    }
    // ml_at: where a part's m and l are
    template <int D, int HEADS>
    __device__ __forceinline__ void add(const float* parts, int c, int c1, int step, int c0, int h, int d, int ml_at = HEADS * D) {
        constexpr int BATCH = PART_BATCH;
        constexpr i64 PART = HEADS * (D + 4);
        for (; c <= c1; c += BATCH * step) {
            float4 u[BATCH];
            float2 ml[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                u[k] = make_float4(0.f, 0.f, 0.f, 0.f), ml[k] = make_float2(NEG_INF, 0.f);
                const int ck = c + k * step;
                if (ck <= c1) {
                    const float* p = parts + (2 * ck + (ck == c0 ? 1 : 0)) * PART;      // an entry's beginning is the second of its CTA's parts
                    u[k] = __ldcg(reinterpret_cast<const float4*>(p + h * D + d));
                    ml[k] = __ldcg(reinterpret_cast<const float2*>(p + ml_at + 2 * h));
                }
            }
            float up = top;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) up = fmaxf(up, ml[k].x);
            rescale(up);
            const float base = up == NEG_INF ? 0.f : up;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const float f = ex2(ml[k].x - base);
                sum = fmaf(ml[k].y, f, sum);
                acc.x = fmaf(u[k].x, f, acc.x), acc.y = fmaf(u[k].y, f, acc.y);
                acc.z = fmaf(u[k].z, f, acc.z), acc.w = fmaf(u[k].w, f, acc.w);
            }
        }
    }
};

// true for the last of `others` + 1 CTAs to arrive: releases what the CTA wrote (ordered before thread 0 by the barrier) and acquires what
// those ahead of it did.  The counter is zero again then, ready for the next call
__device__ __forceinline__ bool arrive(int* counter, int others, int* flag) {
    __syncthreads();
    if (threadIdx.x == 0) {
        int before_me;
        asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before_me) : "l"(counter) : "memory");
        *flag = before_me == others;
        if (*flag) *counter = 0;
    }
    __syncthreads();
    return *flag;
}

// An entry of many parts without a second kernel: groups of neighbouring parts are joined by the last CTA of each group, the groups' sums by the
// last group's.  One row of 131,072 tokens beside 255 of 100, 16 heads of 256: 99 us, and 375 by a single CTA; 8 heads of 128 beside 511: 28 and 61.
// (Out of line, all arguments by value: inside the kernel it made rows of 64 bytes 7 % slower)
template <int D, int HEADS>
__device__ __noinline__ void join_in_groups(Rows rows, float* parts, int* counters, int cta, int c0, int c1, int heads, i64 out0, float vs, int* flag) {
    constexpr int ML_AT = HEADS * D + 2 * HEADS;         // of a group's sum: beside the first part's m and l, which other threads still read
    // groups of about the square root of the parts, a power of two, at least a batch
    const int parts_n = c1 - c0 + 1, shift = parts_n <= 64 ? 3 : parts_n <= 256 ? 4 : 5, step = 1 << shift;
    const int first = c0 + ((cta - c0) >> shift << shift), last = min(first + step - 1, c1);
    // (a CTA may begin the last group of one entry and the first of the next)
    if (!arrive(counters + (first == c0 ? 2 : 1) * kPartCtas + first, last - first, flag)) return;
    float* const sum = parts + (2 * first + (first == c0 ? 1 : 0)) * static_cast<i64>(HEADS * (D + 4));
    for (int i = threadIdx.x; i < heads * (D / 4); i += blockDim.x) {
        const int h = i / (D / 4), d = 4 * (i - h * (D / 4));
        Joined j;
        j.add<D, HEADS>(parts, first, last, 1, c0, h, d);
        __stcg(reinterpret_cast<float4*>(sum + h * D + d), j.acc);
        if (d == 0) __stcg(reinterpret_cast<float2*>(sum + ML_AT + 2 * h), make_float2(j.top, j.sum));
    }
    if (!arrive(counters + c0, (c1 - c0) >> shift, flag)) return;
    for (int i = threadIdx.x; i < heads * (D / 4); i += blockDim.x) {
        const int h = i / (D / 4), d = 4 * (i - h * (D / 4));
        Joined j;
        j.add<D, HEADS>(parts, c0, c1, step, c0, h, d, ML_AT);
        write_out<D>(rows, out0 + h, d, j.acc, j.top, j.sum, vs);
    }
}

// One row (an entry's query head) to a block and step: D / 4 threads across the row, four such groups share its parts.
template <int D, int HEADS>
__global__ void __launch_bounds__(D, 2)
paged_join_kernel(const DecodeArgs a, bool e4m3) {
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    __shared__ float4 accs[4][D / 4];
    __shared__ float2 mls[4];
    const int group = threadIdx.x / (D / 4), d = 4 * (threadIdx.x % (D / 4));
    const int rows = *reinterpret_cast<volatile int*>(a.n_splits) * HEADS;
    if (rows == 0) return;           // (for all blocks alike: the list is emptied when all of them are done)
    for (int u = blockIdx.x; u < rows; u += gridDim.x) {
        const Split e = a.splits[u / HEADS];
        const int h = u % HEADS;
        if (h >= min(HEADS, a.G - e.run * HEADS)) continue;
        Joined j;
        j.add<D, HEADS>(a.parts, e.c0 + group, e.c1, 4, e.c0, h, d);
        accs[group][d / 4] = j.acc;
        if (d == 0) mls[group] = make_float2(j.top, j.sum);
        __syncthreads();
        if (group == 0) {
            float up = NEG_INF;
#pragma unroll
            for (int k = 0; k < 4; ++k) up = fmaxf(up, mls[k].x);
            const float base = up == NEG_INF ? 0.f : up;
            float sum = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = ex2(mls[k].x - base);
                const float4 v = accs[k][d / 4];
                sum = fmaf(mls[k].y, f, sum);
                acc.x = fmaf(v.x, f, acc.x), acc.y = fmaf(v.y, f, acc.y), acc.z = fmaf(v.z, f, acc.z), acc.w = fmaf(v.w, f, acc.w);
            }
            const float vs = e4m3 && a.c.v_scale ? a.c.v_scale[e.g] : 1.f;
            write_out<D>(a.rows, static_cast<i64>(e.b) * a.Hq + e.g * a.G + e.run * HEADS + h, d, acc, up, sum, vs);
        }
        __syncthreads();
    }
    // the last block empties the list for the next call
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(a.n_splits + 1, 1) == static_cast<int>(gridDim.x) - 1) a.n_splits[0] = 0, a.n_splits[1] = 0;
    }
}

template <int D, bool E4M3, int NT, int STAGES, int WARPS, int PER_SM>
__global__ void __launch_bounds__(WARPS * 32, PER_SM)
paged_decode_kernel(const DecodeArgs a) {
    using L = Layout<D, E4M3>;
    constexpr int HEADS = 8 * NT;
    constexpr int THREADS = WARPS * 32;
    constexpr int TILE = WARPS * KEYS;       // keys of a CTA's tile
    // What is subtracted from the scores: LIFT below their maximum, which it follows when it lies SLACK behind.  8-bit values take p in f16, whose
    // full range serves: p of the heaviest key is 2^11 to 2^15, 11 bits are held down to 2^-25 of it and a step of 2^-35 below that.  (With the
    // heaviest at 1, keys below 2^-25 of it were lost, thousands of them and all)
    constexpr float LIFT = E4M3 ? 11.f : 0.f, SLACK = E4M3 ? 4.f : 8.f;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ i64 scan[WARPS];
    __shared__ i64 found_start;
    __shared__ int found_b;
    __shared__ float wm[WARPS][HEADS], wl[WARPS][HEADS];
    __shared__ int last_flag;
    __shared__ uint64_t bars[WARPS][STAGES];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3;
    const int Hkv = a.c.Hkv;
    const bool shared_lens = a.lens_head_stride == 0;
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) ptx::mbar_init(ptx::smem_u32(&bars[warp][s]), 1);
        ptx::fence_mbar_init();
    }

    ptx::grid_dep_wait();
    // ---- the number of tiles of all entries, and the one that holds this CTA's first tile
    // A unit is a sequence (all heads alike) or, where heads have lengths of their own, one head of a sequence
    const int units = shared_lens ? a.B : a.B * Hkv;
    const int per = (units + THREADS - 1) / THREADS;
    const int repeats = (shared_lens ? Hkv : 1) * a.chunks;          // entries of a unit, all of as many tiles
    auto tiles_of_unit = [&](int u) -> int {
        int first, count;
        bool cut;
        span_of(a, shared_lens ? u : u / Hkv, shared_lens ? 0 : u % Hkv, first, count, cut);
        return tiles_of<TILE>(count);
    };
    i64 mine = 0;
    for (int u = tid * per; u < min(units, (tid + 1) * per); ++u) mine += static_cast<i64>(tiles_of_unit(u)) * repeats;
    i64 before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const i64 u = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += u;
    }
    if (lane == 31) scan[warp] = before;
    __syncthreads();
    i64 total = 0;
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) before += scan[w];
        total += scan[w];
    }
    before -= mine;
    const i64 n_ctas = min(static_cast<i64>(gridDim.x), total);     // no CTA without a tile between two of an entry's
    const i64 cta = blockIdx.x;
    if (cta >= n_ctas) return;
    const i64 lo = cta * total / n_ctas, hi = (cta + 1) * total / n_ctas;
    if (before <= lo && lo < before + mine) {
        i64 at = before;
        int u = tid * per;
        i64 n;
        for (;; ++u, at += n) {
            n = static_cast<i64>(tiles_of_unit(u)) * repeats;
            if (lo < at + n) break;
        }
        found_b = u;
        found_start = at;
    }
    __syncthreads();
    Cursor e{};
    bool cut;
    auto look = [&]() {
        span_of(a, e.b, e.g, e.first, e.count, cut);
        e.tiles = tiles_of<TILE>(e.count);
        if (cut && tid == 0) raise_bad_index(a.status);
    };
    auto next = [&]() {
        e.start += e.tiles;
        if (++e.run == a.chunks) {
            e.run = 0;
            if (++e.g == Hkv) e.g = 0, ++e.b;
        }
    };
    e.b = shared_lens ? found_b : found_b / Hkv, e.g = shared_lens ? 0 : found_b % Hkv;
    look();
    {
        const int skip = static_cast<int>((lo - found_start) / e.tiles);      // entries of the unit ahead of the CTA's first
        e.g += skip / a.chunks, e.run = skip % a.chunks;
        e.start = found_start + static_cast<i64>(skip) * e.tiles;
    }

    // ---- the warp's ring
    const uint32_t ring = ptx::smem_u32(smem) + warp * STAGES * L::STAGE;
    const uint32_t bar0 = ptx::smem_u32(&bars[warp][0]);
    uint32_t phases = 0;             // bit s: parity of the next completion of stage s
    bool dead = false;               // a wait has expired: no more copies, and a bounded wait for each that is under way
    const int row = lane & 15;
    const bool is_v = lane >= 16;
    const uint32_t row_dst = ring + (is_v ? L::K_BYTES + row * L::V_PITCH : row * L::K_PITCH);
    const i64 page_bytes = (is_v ? a.c.v_page_stride : a.c.k_page_stride) * L::ELEM;
    const i64 token_bytes = (is_v ? a.c.v_token_stride : a.c.k_token_stride) * L::ELEM;
    const unsigned page_size = a.c.page_size;
    // a token's page and place in it; powers of two (almost every cache) without the division's twenty instructions
    const bool pow2 = (page_size & (page_size - 1)) == 0;
    const int page_shift = 31 - __clz(page_size);
    auto page_of = [&](int key) -> unsigned { return pow2 ? static_cast<unsigned>(key) >> page_shift : static_cast<unsigned>(key) / page_size; };
    auto place_of = [&](int key) -> unsigned { return pow2 ? static_cast<unsigned>(key) & (page_size - 1) : static_cast<unsigned>(key) % page_size; };
    const uint32_t v_read = ring + L::K_BYTES + ((lane & 7) + ((lane >> 4) << 3)) * L::V_PITCH + ((lane >> 3) & 1) * 16;
    const uint32_t k_read = ring + g8 * L::K_PITCH + t4 * L::VK;

    for (i64 at = lo; at < hi;) {
        const int tile0 = static_cast<int>(at - e.start);
        const int n_tiles = static_cast<int>(min(hi - at, static_cast<i64>(e.tiles - tile0)));
        const int heads = min(HEADS, a.G - e.run * HEADS);        // query heads of this run
        const int h0 = e.g * a.G + e.run * HEADS;
        const int* table = a.table + e.b * a.table_stride + e.g * a.table_head_stride;
        const int end = e.first + e.count;
        const int key0 = e.first + tile0 * TILE + warp * KEYS + row;       // this lane's key of the segment's first step
        const uint8_t* const base = is_v ? static_cast<const uint8_t*>(a.c.v) + e.g * a.c.v_head_stride * L::ELEM
                                         : static_cast<const uint8_t*>(a.c.k) + e.g * a.c.k_head_stride * L::ELEM;

        // the table entry of this lane's key of a step; -1: no such key
        auto page_at = [&](int step) -> int {
            const int key = key0 + step * TILE;
            return (step < n_tiles && key < end) ? table[page_of(key)] : -1;
        };
        // fetches a step; returns the mask of its keys that are there
        auto copy = [&](int step, int entry, uint32_t s) -> uint32_t {
            const int key = key0 + step * TILE;
            const bool asked = step < n_tiles && key < end;
            const bool there = asked && entry >= 0 && entry < a.c.num_pages;
            const uint32_t mask = __ballot_sync(0xffffffffu, there) & 0xffffu;
            if (asked && !there) raise_bad_index(a.status);
            if (!L::BULK) {
                if (mask != 0) {
                    const unsigned off = place_of(key);
                    const uint64_t mine = reinterpret_cast<uint64_t>(base + (there ? entry * page_bytes + off * token_bytes : 0));
                    const uint32_t stage = ring + s * L::STAGE;
#pragma unroll
                    for (int i = 0; i < L::UNITS; ++i) {          // first the keys' 16 * UNITS units, then the values'
                        const int v = i >= L::UNITS / 2;
                        const int unit = (i - v * (L::UNITS / 2)) * 32 + lane;
                        const int r = unit / L::UNITS, c = unit - r * L::UNITS;
                        const uint8_t* src = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, mine, r + 16 * v)) + c * 16;
                        cp_async16(stage + (v ? L::K_BYTES + r * L::V_PITCH : r * L::K_PITCH) + c * 16, src, (mask >> r) & 1);
                    }
                }
                cp_commit();
                return mask;
            }
            if (mask == 0 || dead) return 0;
            const uint32_t bar = bar0 + 8 * s;
            if (lane == 0) ptx::mbar_arrive_expect_tx(bar, 2 * __popc(mask) * L::ROW);
            if (there) {
                const unsigned off = place_of(key);
                ptx::bulk_load(row_dst + s * L::STAGE, base + entry * page_bytes + off * token_bytes, L::ROW, bar);
            } else if (is_v) {
                // 0 * v has to be 0 for a value that is not there; ordered ahead of a later copy to the same place
#pragma unroll
                for (int i = 0; i < L::ROW; i += 16)
                    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(row_dst + s * L::STAGE + i), "r"(0) : "memory");
                ptx::fence_proxy_async_smem();
            }
            return mask;
        };

        uint32_t masks[STAGES];      // of the next STAGES - 1 steps
        int entry;
        {
            int entries[STAGES];
#pragma unroll
            for (int s = 0; s < STAGES; ++s) entries[s] = page_at(s);
#pragma unroll
            for (int s = 0; s < STAGES - 1; ++s) masks[s] = copy(s, entries[s], s);
            entry = entries[STAGES - 1];
        }

        // ---- queries: operand b of the score product, lane (head g8, element runs of t4), and their factor
        constexpr int EL = L::VK / L::ELEM;      // elements of a run
        uint32_t qf[NT][L::CK * EL / 4][2];
        float factor[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int h = n * 8 + g8;
            const cake_bf16* src = a.q + e.b * a.q_stride + (h0 + h) * a.q_head_stride + t4 * EL;
            uint32_t w[L::CK][EL / 2];
#pragma unroll
            for (int c = 0; c < L::CK; ++c)
#pragma unroll
                for (int j = 0; j < EL / 8; ++j) {
                    uint4 u = make_uint4(0, 0, 0, 0);
                    if (h < heads) {
                        const cake_bf16* from = src + 4 * c * EL + 8 * j;
                        if (a.q_wide) {
                            u = *reinterpret_cast<const uint4*>(from);
                        } else {
                            auto two = [&](int i) { return static_cast<uint32_t>(from[i]) | (static_cast<uint32_t>(from[i + 1]) << 16); };
                            u = make_uint4(two(0), two(2), two(4), two(6));
                        }
                    }
                    w[c][4 * j] = u.x, w[c][4 * j + 1] = u.y, w[c][4 * j + 2] = u.z, w[c][4 * j + 3] = u.w;
                }
            // 8-bit keys are widened to f16 (exact), so the query is too: divided by a power of two that leaves its largest
            // element in [1, 2), which keeps 11 bits where bf16 has 8; elements below 2^-14 of the largest are held to 2^-25 of it
            float unit = 1.f;
            if (E4M3) {
                float most = 0.f;
#pragma unroll
                for (int c = 0; c < L::CK; ++c)
#pragma unroll
                    for (int j = 0; j < EL / 2; ++j) most = fmaxf(most, fmaxf(fabsf(bf16_lo(w[c][j])), fabsf(bf16_hi(w[c][j]))));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
                const uint32_t ex = __float_as_uint(most) & 0x7f800000u;
                if (ex > (2u << 23) && ex < (252u << 23)) unit = __uint_as_float(ex);
                const float down = __uint_as_float((254u << 23) - __float_as_uint(unit));
#pragma unroll
                for (int c = 0; c < L::CK; ++c)
#pragma unroll
                    for (int j = 0; j < EL / 2; ++j) w[c][j] = pack_f16(bf16_lo(w[c][j]) * down, bf16_hi(w[c][j]) * down);
            }
#pragma unroll
            for (int c = 0; c < L::CK; ++c)
#pragma unroll
                for (int j = 0; j < EL / 2; ++j) qf[n][c * (EL / 4) + j / 2][j & 1] = w[c][j];
            const float ks = E4M3 && a.c.k_scale ? a.c.k_scale[e.g] : 1.f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                factor[n][i] = a.scale * LOG2E * ks * __shfl_sync(0xffffffffu, unit, (2 * t4 + i) * 4);
        }

        float o[D / 16][NT][4];      // O^T: per 16 values of d, (d, head 2t4), (d, head 2t4+1), (d', ...), (d', ...)
        float m[NT][2], l[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < 2; ++i) m[n][i] = NEG_INF, l[n][i] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[j][n][i] = 0.f;
        }
        uint32_t s = 0;              // stage of the step
        for (int step = 0; step < n_tiles; ++step) {
            const int following = page_at(step + STAGES);
            __syncwarp();            // every lane has read the stage that is filled next
            const uint32_t s_next = s == 0 ? STAGES - 1 : s - 1;
            const uint32_t coming = copy(step + STAGES - 1, entry, s_next);
            entry = following;
            const uint32_t mask = masks[0];
#pragma unroll
            for (int i = 0; i + 1 < STAGES - 1; ++i) masks[i] = masks[i + 1];
            masks[STAGES - 2] = coming;
            const uint32_t here = s;
            s = s + 1 == STAGES ? 0 : s + 1;
            if (mask == 0) continue;
            if (!L::BULK) {
                cp_wait<STAGES - 1>();
                __syncwarp();
            } else {                 // (also after a wait that expired: no copy in flight is left behind unwaited for)
                const uint32_t bar = bar0 + 8 * here, parity = (phases >> here) & 1;
                int tries = 0;
                while (!ptx::mbar_try_wait_hint(bar, parity, 20000) && tries < WAIT_TRIES) ++tries;
                if (__any_sync(0xffffffffu, tries == WAIT_TRIES)) {
                    dead = true;
                    if (lane == 0) atomicCAS(a.status, CAKE_OK, CAKE_ERR_TIMEOUT);
                }
                phases ^= 1u << here;
            }

            // ---- scores of 16 keys
            float x[NT][4];
            const uint32_t k_at = k_read + here * L::STAGE;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[n][i] = 0.f;
#pragma unroll
            for (int c = 0; c < L::CK; ++c) {
                uint32_t k0[L::VK / 4], k1[L::VK / 4];
                lds<L::VK>(k_at + c * 4 * L::VK, k0);
                lds<L::VK>(k_at + 8 * L::K_PITCH + c * 4 * L::VK, k1);
                if (E4M3) {
#pragma unroll
                    for (int j = 0; j < L::VK / 4; ++j) {
                        uint32_t f[4];
                        e4m3_to_f16(k0[j], f[0], f[2]);
                        e4m3_to_f16(k1[j], f[1], f[3]);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma<true>(x[n], f, qf[n][c * (L::VK / 4) + j][0], qf[n][c * (L::VK / 4) + j][1]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < L::VK / 8; ++j) {
                        const uint32_t f[4] = {k0[2 * j], k1[2 * j], k0[2 * j + 1], k1[2 * j + 1]};
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma<false>(x[n], f, qf[n][c * (L::VK / 8) + j][0], qf[n][c * (L::VK / 8) + j][1]);
                    }
                }
            }

            // ---- running maximum (m: LIFT below it) and sum.  It may lag behind the true one by up to SLACK (p stays below 2^(LIFT + SLACK),
            // inside every format it passes through), so it moves, and O is rescaled, only a few times per row
            uint32_t ph[NT][2], pl[NT][2];
            const bool ok0 = (mask >> g8) & 1, ok1 = (mask >> (g8 + 8)) & 1;
            bool higher = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x[n][i] = ok0 ? x[n][i] * factor[n][i] : NEG_INF;
                    x[n][2 + i] = ok1 ? x[n][2 + i] * factor[n][i] : NEG_INF;
                    higher |= fmaxf(x[n][i], x[n][2 + i]) > m[n][i] + (LIFT + SLACK);
                }
            if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float top = fmaxf(x[n][i], x[n][2 + i]);
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        top = fmaxf(m[n][i], top - LIFT);
                        const float keep = ex2(m[n][i] - (top == NEG_INF ? 0.f : top));
                        m[n][i] = top;
                        l[n][i] *= keep;
#pragma unroll
                        for (int j = 0; j < D / 16; ++j) o[j][n][i] *= keep, o[j][n][2 + i] *= keep;
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float p[4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float base_m = m[n][i] == NEG_INF ? 0.f : m[n][i];     // every score so far is -inf: they all weigh nothing
                    p[i] = ex2(x[n][i] - base_m);
                    p[2 + i] = ex2(x[n][2 + i] - base_m);
                    l[n][i] += p[i] + p[2 + i];
                }
                if (E4M3) {
                    // f16 holds 11 bits of p: its rounding is an eighth of the output's (the lightest keys': see LIFT)
                    ph[n][0] = transpose8x8(pack_f16(p[0], p[1]));
                    ph[n][1] = transpose8x8(pack_f16(p[2], p[3]));
                } else {
                    // p as the sum of two bf16, so that its rounding (2^-8 in one of them) does not add to the output's own
                    const uint32_t a0 = pack_bf16(p[0], p[1]), a1 = pack_bf16(p[2], p[3]);
                    pl[n][0] = transpose8x8(pack_bf16(p[0] - bf16_lo(a0), p[1] - bf16_hi(a0)));
                    pl[n][1] = transpose8x8(pack_bf16(p[2] - bf16_lo(a1), p[3] - bf16_hi(a1)));
                    ph[n][0] = transpose8x8(a0);
                    ph[n][1] = transpose8x8(a1);
                }
            }

            // ---- weighted sum of 16 values: 32 bytes of each at a time
#pragma unroll
            for (int j = 0; j < L::ROW / 32; ++j) {
                uint32_t v[4];
                ldmatrix_trans(v_read + here * L::STAGE + j * 32, v);
                if (E4M3) {
                    // v[0], v[2]: elements (d, d+1) of two keys each, d = 32j + 2 g8; v[1], v[3]: 16 further on
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t f[4];
                        e4m3_to_f16(__byte_perm(v[i], 0, 0x3120), f[0], f[1]);
                        e4m3_to_f16(__byte_perm(v[2 + i], 0, 0x3120), f[2], f[3]);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma<true>(o[2 * j + i][n], f, ph[n][0], ph[n][1]);
                    }
                } else {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma<false>(o[j][n], v, ph[n][0], ph[n][1]);
                        mma<false>(o[j][n], v, pl[n][0], pl[n][1]);
                    }
                }
            }
        }
        if (!L::BULK) cp_wait<0>();

        // ---- the warps' parts: maxima and sums first, then the weighted sums through the ring's memory
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], d);
                if (g8 == 0) wm[warp][n * 8 + 2 * t4 + i] = m[n][i], wl[warp][n * 8 + 2 * t4 + i] = l[n][i];
            }
        __syncthreads();             // (also: every warp has drained its ring)
        float* const osum = reinterpret_cast<float*>(smem);      // [WARPS][HEADS][O_PITCH]
        constexpr int O_PITCH = D + 4;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int h = n * 8 + 2 * t4 + i;
                float top = NEG_INF;
#pragma unroll
                for (int w = 0; w < WARPS; ++w) top = fmaxf(top, wm[w][h]);
                const float f = ex2(m[n][i] - (top == NEG_INF ? 0.f : top));
                float* dst = osum + (warp * HEADS + h) * O_PITCH;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    if (E4M3) {
                        *reinterpret_cast<float2*>(dst + 16 * j + 2 * g8) = make_float2(o[j][n][i] * f, o[j][n][2 + i] * f);
                    } else {
                        dst[16 * j + g8] = o[j][n][i] * f;
                        dst[16 * j + 8 + g8] = o[j][n][2 + i] * f;
                    }
                }
            }
        __syncthreads();
        const bool whole = tile0 == 0 && n_tiles == e.tiles;
        constexpr int PART = HEADS * (D + 4);            // floats of a part: O of the run's heads, then m and l (and padding)
        float* const part = a.parts + (2 * cta + (tile0 == 0 ? 1 : 0)) * static_cast<i64>(PART);
        const float vs = E4M3 && a.c.v_scale ? a.c.v_scale[e.g] : 1.f;
        const i64 out0 = static_cast<i64>(e.b) * a.Hq + h0;
        auto finish = [&](int h, int d, const float4& acc, float top, float sum) { write_out<D>(a.rows, out0 + h, d, acc, top, sum, vs); };
        for (int i = tid; i < heads * (D / 4); i += THREADS) {
            const int h = i / (D / 4), d = 4 * (i - h * (D / 4));
            float top = NEG_INF;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) top = fmaxf(top, wm[w][h]);
            const float base_m = top == NEG_INF ? 0.f : top;
            float sum = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                sum += wl[w][h] * ex2(wm[w][h] - base_m);
                const float4 u = *reinterpret_cast<const float4*>(osum + (w * HEADS + h) * O_PITCH + d);
                acc.x += u.x, acc.y += u.y, acc.z += u.z, acc.w += u.w;
            }
            if (whole) {
                finish(h, d, acc, top, sum);
            } else {
                __stcg(reinterpret_cast<float4*>(part + h * D + d), acc);
                if (d == 0) __stcg(reinterpret_cast<float2*>(part + HEADS * D + 2 * h), make_float2(top, sum));
            }
        }
        if (!whole) {
            // ---- The entry's CTAs are neighbours.  A few parts are joined, in order, by the last of them to arrive; more in two levels; or
            // all of them by a second kernel, for which the first of them notes the entry
            const i64 s0 = e.start, s1 = e.start + e.tiles - 1;
            const int c0 = static_cast<int>(((s0 + 1) * n_ctas - 1) / total), c1 = static_cast<int>(((s1 + 1) * n_ctas - 1) / total);
            if (a.defer) {
                if (tid == 0 && cta == c0) a.splits[atomicAdd(a.n_splits, 1)] = Split{e.b, e.g, e.run, c0, c1, {0, 0, 0}};
            } else if (c1 - c0 >= a.few) {
                if (at + n_tiles >= hi) ptx::grid_dep_launch();      // the CTA's last: the next kernel may start beside the join
                join_in_groups<D, HEADS>(a.rows, a.parts, a.counters, static_cast<int>(cta), c0, c1, heads, out0, vs, &last_flag);
            } else if (arrive(a.counters + c0, c1 - c0, &last_flag)) {
                for (int i = tid; i < heads * (D / 4); i += THREADS) {
                    const int h = i / (D / 4), d = 4 * (i - h * (D / 4));
                    Joined j;
                    j.add<D, HEADS>(a.parts, c0, c1, 1, c0, h, d);
                    finish(h, d, j.acc, j.top, j.sum);
                }
            }
        }
        __syncthreads();             // the ring's memory, wm and wl are free again
        ptx::fence_proxy_async_smem();       // plain accesses to the ring's memory come before the next copies into it
        at += n_tiles;
        if (at < hi) next(), look();
    }
}

struct Shape {
    int nt, chunks;
};
Shape shape_of(int Hq, int Hkv) {
    const int G = Hq / Hkv;
    Shape s;
    s.nt = G <= 8 ? 1 : 2;
    s.chunks = (G + 8 * s.nt - 1) / (8 * s.nt);
    return s;
}

template <int D, bool E4M3, int NT, int STAGES, int WARPS, int PER_SM>
int launch(DecodeArgs& a, const DeviceInfo& di, cudaStream_t s) {
    using L = Layout<D, E4M3>;
    constexpr int RING1 = WARPS * L::STAGE;
    constexpr int RING = RING1 * STAGES;
    constexpr int MERGE = WARPS * 8 * NT * (D + 4) * 4;
    constexpr int SMEM = RING > MERGE ? RING : MERGE;
    const auto kernel = paged_decode_kernel<D, E4M3, NT, STAGES, WARPS, PER_SM>;
    static PerDevice resident;
    const int per_sm = resident.get(di.device, [kernel]() -> int {
        int n = 0;
        if (!allow_smem(kernel, SMEM)) return 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, WARPS * 32, SMEM) == cudaSuccess) return n;
        cudaGetLastError();
        return 0;
    });
    if (per_sm < 1) return CAKE_ERR_CUDA;
    const int ctas = min(di.sm_count * per_sm, kPartCtas);
    // Whether a second kernel joins the parts has to be said here, where the lengths are not known: from the parts of an entry if all are about as
    // long, no more than the page table and the window leave room for.  Behind short rows it is 1.2 - 1.8 us for nothing (one row of 777 tokens, a
    // table for 16,384: 9.2 us with it, 7.7 without).  Two levels in this kernel lose less than that where a CTA has a thread for each four values of
    // a part (32 query, 8 key-value heads of 128, one row of 4,000 tokens 11.4 -> 11.3 us, of 30,000 30.4 -> 31.0; 4 heads to a single
    // key-value head 17.2 -> 13.6), but more in several passes (8 heads, 4,000 tokens: 9.2 and 10.1; 16 heads, 30,000: 19.1 and 24.9), from
    // 64 KiB of parts on (about 2 us of one SM's reads).  One CTA joins up to `few` parts of an entry by itself: batches of eight, 0.6 us each and pass;
    // two levels are an arrival (about two batches) more
    const i64 entries = static_cast<i64>(a.B) * a.c.Hkv * a.chunks;
    i64 most = static_cast<i64>(a.max_pages) * a.c.page_size;
    if (a.window > 0 && a.window < most) most = a.window;
    const i64 most_tiles = (most + WARPS * KEYS - 1) / (WARPS * KEYS);
    const i64 share = (ctas + entries - 1) / entries, parts = share < most_tiles ? share : most_tiles;
    const int part_bytes = min(8 * NT, a.G) * D * 4;
    const int passes = (part_bytes / 16 + WARPS * 32 - 1) / (WARPS * 32);
    a.defer = passes > 1 && parts * part_bytes > 64 * 1024;
    a.few = passes == 1 ? 32 : 16;
    if (launch_early(kernel, dim3(ctas), dim3(WARPS * 32), SMEM, s, a) != cudaSuccess) return CAKE_ERR_CUDA;
    if (!a.defer) return CAKE_OK;
    return launch_early(paged_join_kernel<D, 8 * NT>, dim3(2 * di.sm_count), dim3(D), 0, s, a, E4M3) == cudaSuccess ? CAKE_OK : CAKE_ERR_CUDA;
}

// Two stages a warp and as many warps as fit: a warp's step is a chain of dependent instructions, other warps fill its gaps.
template <int D>
int launch_d(DecodeArgs& a, bool e4m3, int nt, const DeviceInfo& di, cudaStream_t s) {
    constexpr int W16 = D == 256 ? 2 : 4;
    constexpr int P8 = D <= 128 ? 4 : 2, P16 = D <= 64 ? 4 : 3;
    if (e4m3) return nt == 1 ? launch<D, true, 1, 2, 4, P8>(a, di, s) : launch<D, true, 2, 2, 4, D == 256 ? 2 : 3>(a, di, s);
    return nt == 1 ? launch<D, false, 1, 2, W16, P16>(a, di, s) : launch<D, false, 2, 2, W16, 3>(a, di, s);
}

int check_heads(long long B, int Hq, int Hkv, int D) {
    if (B < 0 || Hkv < 1 || B > INT_MAX / 2 / Hkv || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return CAKE_ERR_SHAPE;
    if (D != 64 && D != 96 && D != 128 && D != 256) return CAKE_ERR_UNSUPPORTED;
    return CAKE_OK;
}
size_t workspace_bytes(int Hq, int Hkv, int D) {
    const Shape sh = shape_of(Hq, Hkv);
    return round_up(static_cast<i64>(kHeaderBytes + kPartCtas * sizeof(Split) + sizeof(float) * 2 * kPartCtas * 8 * sh.nt * (D + 4)), 256);
}

}  // namespace
}  // namespace serving
}  // namespace cake

using namespace cake;
using namespace cake::serving;

extern "C" {

int cake_paged_decode_workspace_bytes(long long B, int Hq, int Hkv, int D, size_t* out_bytes) {
    if (!out_bytes) return CAKE_ERR_NULL;
    const int rc = check_heads(B, Hq, Hkv, D);
    if (rc != CAKE_OK) return rc;
    *out_bytes = workspace_bytes(Hq, Hkv, D);
    return CAKE_OK;
}

int cake_paged_decode(const cake_bf16* q, long long q_stride, long long q_head_stride, const cake_paged_cache* cache,
                      const int* page_table, long long table_stride, long long table_head_stride, int max_pages,
                      const int* seq_lens, long long lens_stride, long long lens_head_stride, long long B, int Hq, float scale,
                      int window, cake_bf16* out, float* out_lse, void* ws, size_t ws_bytes, cake_stream_t stream) {
    int rc = check_cache(cache);
    if (rc != CAKE_OK) return rc;
    rc = check_heads(B, Hq, cache->Hkv, cache->D);
    if (rc != CAKE_OK) return rc;
    if (max_pages < 0 || static_cast<i64>(max_pages) * cache->page_size > INT_MAX - 16 * MOST_WARPS * KEYS || window < 0) return CAKE_ERR_SHAPE;
    if (table_stride < 0 || table_head_stride < 0 || lens_stride < 0 || lens_head_stride < 0 || q_stride < 0 || q_head_stride < 0)
        return CAKE_ERR_SHAPE;
    if (!ws) return CAKE_ERR_NULL;
    if (!aligned(ws, 256)) return CAKE_ERR_ALIGN;
    if (ws_bytes < workspace_bytes(Hq, cache->Hkv, cache->D)) return CAKE_ERR_WORKSPACE;
    if (B == 0) return CAKE_OK;
    if (!q || !seq_lens || !out || (max_pages > 0 && !page_table)) return CAKE_ERR_NULL;
    if (!aligned(q, 2) || !aligned(out, 2) || !aligned(out_lse, 4) || !aligned(page_table, 4) || !aligned(seq_lens, 4)) return CAKE_ERR_ALIGN;
    DeviceInfo di;
    rc = current_device_info(&di);
    if (rc != CAKE_OK) return rc;
    if (di.cc_major != 10) return CAKE_ERR_DEVICE;
    const Shape sh = shape_of(Hq, cache->Hkv);
    DecodeArgs a;
    a.c = *cache, a.q = q, a.table = page_table, a.lens = seq_lens, a.rows = Rows{out, out_lse, aligned(out, 8)};
    a.status = static_cast<int*>(ws);
    a.counters = static_cast<int*>(ws) + 64;
    a.n_splits = static_cast<int*>(ws) + 16;
    a.splits = reinterpret_cast<Split*>(static_cast<char*>(ws) + kHeaderBytes);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + kHeaderBytes + kPartCtas * sizeof(Split));
    a.q_stride = q_stride, a.q_head_stride = q_head_stride, a.table_stride = table_stride, a.table_head_stride = table_head_stride;
    a.lens_stride = lens_stride, a.lens_head_stride = lens_head_stride;
    a.B = static_cast<int>(B), a.Hq = Hq, a.G = Hq / cache->Hkv, a.chunks = sh.chunks, a.max_pages = max_pages, a.window = window;
    a.scale = scale;
    a.q_wide = aligned(q, 16) && q_stride % 8 == 0 && q_head_stride % 8 == 0;
    const bool e4m3 = cache->type == CAKE_KV_E4M3;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    switch (cache->D) {
        case 64: return launch_d<64>(a, e4m3, sh.nt, di, s);
        case 96: return launch_d<96>(a, e4m3, sh.nt, di, s);
        case 128: return launch_d<128>(a, e4m3, sh.nt, di, s);
        default: return launch_d<256>(a, e4m3, sh.nt, di, s);
    }
}

}  // extern "C"
