// Attention of many query tokens: softmax(scale Q K^T) V, keys and values packed by sequence or in a paged cache.
//
//   out_i = sum_t exp(x_it - m_i) v_t / sum_t exp(x_it - m_i),   x_it = scale * q_i . k_t  over the keys t that token i sees
//
// One pass over the keys with the running maximum m, sum l and weighted sum O of a softmax.  Both products run on the tensor cores:
//   S = Q K^T   [128 rows x 128 keys], Q and K from shared memory, S in tensor memory
//   O += P V    P (16-bit, over S's columns in tensor memory) times V from shared memory, O in tensor memory
// and the threads between them have a row of S each (tensor memory's lanes): no exchange between threads for maximum and sum.
//
// Rows are (token, query head of the key-value head's group) pairs, tokens outermost, so a key-value head is read once for its
// whole group, whatever the group's size; a tile of 128 rows holds 128 / group tokens.
//
// A CTA works on two tiles of rows at a time (heads of 256: one, its O fills tensor memory), so that the tensor cores multiply for
// one while the other's exponentials are taken: both need about as long (128 x 128 scores: 1,024 clocks of two products at
// D = 128, 1,024 clocks of 2^x).  Two tiles are either
//   different rows that share each tile of keys (DUAL), or, where an item has no more than 128 rows,
//   the same rows over every other tile of keys (ALT), joined at the end.
//
// Work is the list of all keys of all items (sequence, key-value head, block of rows), one after the other, with some for an item's
// start and end; CTA c of n takes the c-th of n equal shares, whatever the lengths are, in whole tiles and moved to the end of an item where that is near.  Items that several
// CTAs share are joined from parts in the workspace by a second kernel, in the order of the CTAs.
//
// Warps: a warpgroup of softmax rows for each row tile; four warps that load pages (paged caches only: two for the keys, two for the values); four
// of one job each: the scheduler, which loads queries and packed keys as it goes, the loads of packed values, the issue of Q K^T, the issue of P V.
// Keys and values have a ring each, and each product a warp that issues it, since one that waits for weights would hold up the other's scores (one
// issuing warp and one ring: 2.18 ms for 16,384 causal tokens where this takes 1.72).
//
// Tensor memory has one place for scores, between the weights of the two row tiles, and O: scores are loaded as soon as they are there (128
// registers a thread), which frees the place for the other tile's.
//
// What bounds it (one B200, D = 128, 32 query heads to 8): 16,384 causal tokens 1.72 ms in short runs = 1,280 TFLOP/s, 77 % of the rate measured for a library
// product (1.97 ms in long runs, under the power cap): 2^x and the tensor cores are both busy for two thirds of the time, two softmax warps to a
// scheduler do not hide all of a tile's chain (load, 2^x, sum, store, wait).  Short items: their end (O of the last products, 1/l, stores) and start are not hidden,
// and they are run so rarely that their instructions come from the L2: code is kept small for that reason (a loader of 92 KB of unrolled code for one of 16: 107 -> 70 us
// for 64 tokens over 16 x 4,097 cached).  8-bit caches: widening, 16 bytes read and 32 written in shared memory for every 16 elements.
#pragma once
#include "ptx.cuh"
#include "serving.cuh"

namespace cake {
namespace serving {

int check_cache(const cake_paged_cache* c);   // kv_append.cu

namespace attn {

constexpr int KT = 128;                        // keys of a tile
constexpr int MT = 128;                        // rows of a tile
constexpr int MOST_CTAS = 148;                 // that the workspace has room for parts of (two each)
constexpr int SEGS = 4;                        // segments of work that the scheduler is ahead
constexpr int FLAGS_AHEAD = 16;                // tiles of keys whose page flags are kept
constexpr int OVERHEAD = 576;                  // keys that an item's start and end cost (four tiles of them, and half of one that is not full)
constexpr int SNAP = 4;                        // a share's end within fewer tiles of an item's is moved there
constexpr int MIN_SHARE = OVERHEAD / 4;        // of a CTA, in keys
constexpr uint64_t WAIT_LIMIT_NS = 8000000000ull;      // (a warp that computes its rows again, mend_rows, keeps the others waiting)
constexpr float LEAST = 1.4012985e-45f;        // 2^-149
constexpr float LN2 = 0.6931471805599453f;
constexpr float NEG_INF = -INFINITY;

// Tensor memory: scores of one row tile between the weights (16 bits) of two, then the weighted sums (of the one row tile: both places)
constexpr uint32_t S_COL = KT / 2, O_COL = 2 * KT;
__device__ __forceinline__ uint32_t p_col(int pb) { return pb ? KT / 2 + KT : 0; }

enum Kind { PACKED = 0, PAGED_BF16 = 1, PAGED_E4M3 = 2 };

// An item that several CTAs share: `cta` has the beginning, the ones up to c1 the rest; count = 0: none.
struct Split {
    i64 tok;                                   // first token among all queries'
    int head0, heads, ntok, c1, valid, g;
};

struct Args {
    cake_paged_cache c;                        // paged
    const cake_bf16 *q, *k, *v;
    const int *starts, *k_starts;              // of the sequences' queries; of their keys (packed)
    const int *table, *lens;                   // paged
    cake_bf16* out;
    float* lse;
    int* status;
    float* parts;
    Split* splits;
    i64 T, Tk, q_stride, q_head_stride, k_stride, k_head_stride, v_stride, v_head_stride;
    i64 table_stride, table_head_stride, lens_stride, lens_head_stride;
    int entries;                               // sequences * key-value heads * runs
    uint32_t per_mul, per_shift;               // e / (heads * runs) = mulhi(e, per_mul) >> per_shift (per_mul 0: e)
    uint32_t page_mul, page_shift;             // the same for a page's tokens
    uint64_t share_mul;                        // 2^64 / CTAs
    int Hq, Hkv, G, runs, heads, tokens;    // heads: of a run of a group's query heads; tokens: of a tile of rows
    int max_pages, window;
    float scale_log2;                          // |scale| log2 e
    bool negative, causal;                     // sign of the scale
    bool wide;                                 // out is a multiple of 32 bytes
    bool cuts;                                 // an item may be shared by CTAs
    bool maps;                                 // paged: mk and mv are maps of the pages, boxes of `box` tokens
    int box;
};

// A share of an item: what every role of a CTA is told of it.
struct Seg {
    i64 tok;                                   // first token among all queries'
    i64 k0;                                    // first key among all keys (packed); the table's row (paged)
    int g, head0, heads, ntok, pos, klen, ja, jb;   // pos: position of the first token; tiles of keys [ja, jb)
    int part;                                  // slot among the parts, -1: the whole item
    int negative, done;
};

template <int D_, int KIND_>
struct Traits {
    static constexpr int D = D_;
    static constexpr int KIND = KIND_;
    static constexpr bool PAGED = KIND != PACKED, F16 = KIND == PAGED_E4M3;
    static constexpr int TILES = D == 256 ? 1 : 2;
    // Keys and values have a ring of places each (64 KiB), a tile of them comes in units of KC (VC) columns, in slabs of 64: 128-byte rows,
    // 128-byte swizzle.  Heads of 256: smaller units of keys, so that the next tile's come in behind this one's products (8-bit ones: a unit's start and
    // end is most of what it costs to widen it)
    static constexpr uint32_t SLAB = MT * 128;
    static constexpr int SLABS = (D + 63) / 64;
    static constexpr int KC = D == 256 ? (F16 ? 128 : 64) : D, VC = D == 256 ? 128 : D;
    static constexpr int NKU = D / KC, NVU = D / VC;
    static constexpr int K_SLABS = (KC + 63) / 64, V_SLABS = (VC + 63) / 64;
    static constexpr uint32_t K_UNIT = K_SLABS * SLAB, V_UNIT = V_SLABS * SLAB;
    // (8-bit caches: what has come from memory and is not widened yet takes half of the values' room)
    static constexpr uint32_t K_BYTES = 4 * SLAB, V_BYTES = (F16 ? 2 : 4) * SLAB;
    static constexpr int K_STAGES = K_BYTES / K_UNIT, V_STAGES = V_BYTES / V_UNIT;
    static constexpr uint32_t RAW = SLAB;                    // 128 bytes of 128 keys
    static constexpr int RAW_STAGES = F16 ? 3 : 0;
    static constexpr int WARPS_SM = 4 * TILES, WARPS_LD = PAGED ? 4 : 0;
    static constexpr int WARP_SCHED = WARPS_SM + WARPS_LD, WARP_VALUES = WARP_SCHED + 1, WARP_MMA = WARP_SCHED + 2;
    static constexpr int WARPS = WARP_SCHED + 4, THREADS = 32 * WARPS;
    static constexpr uint32_t Q_TILE = SLABS * SLAB, Q_BYTES = TILES * Q_TILE;
    // registers: what a block starts with (65,536 / threads), shared out again between the warpgroups
    static constexpr bool SPLIT_REGS = TILES == 2 || PAGED;
    static constexpr int REGS_SM = TILES == 2 ? (PAGED ? 184 : 224) : 232;
    static constexpr int REGS_LD = TILES == 2 ? 96 : 192, REGS_AUX = TILES == 2 ? (PAGED ? 48 : 56) : 80;
    static constexpr int REGS_START = 65536 / THREADS / 8 * 8 > 255 ? 255 : 65536 / THREADS / 8 * 8;
    static_assert(!SPLIT_REGS || TILES * REGS_SM + (PAGED ? REGS_LD : 0) + REGS_AUX <= REGS_START * (THREADS / 128), "registers of the block");
    // Who says that a tile's queries are done with.  A barrier's parity names every other load, so nobody who looks at a load may miss it:
    // the issuing warp and, of 16-bit copies, the second warpgroup look at every load of the first tile
    static __host__ __device__ constexpr int q_readers(int t) { return TILES == 2 && t == 0 && F16 ? 5 : 1; }
    static constexpr int PART_ROWS = TILES * MT;
    static constexpr i64 PART = static_cast<i64>(PART_ROWS) * (D + 2);       // floats
};

struct __align__(16) Ctrl {
    uint64_t seg_full[SEGS], seg_empty[SEGS];
    uint64_t q_full[2], q_empty[2], q_conv[2];
    uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4], v_end;
    uint64_t raw_full[4][3];                   // of a loading warp's places
    uint64_t s_full[2], p_ready[2], o_done[2], o_free[2], s_free, x_full, x_empty, drained[2];
    Seg seg[SEGS];
    i64 sums[16];
    uint4 flags[FLAGS_AHEAD];                  // a bit for each key of a tile: its page exists
    float2 ml[MT];                             // maximum and sum of the second tile (ALT)
    float q_scale[2][MT];                      // powers of two that 16-bit queries were divided by
    uint32_t tmem;
    int abort_flag;
};

template <class T>
constexpr uint32_t smem_bytes() {
    return 1024 + T::Q_BYTES + T::K_BYTES + T::V_BYTES + T::RAW_STAGES * T::RAW + sizeof(Ctrl);
}
// what a CTA's shared memory holds
struct Room {
    uint8_t *q, *k, *v, *raw;
};

__device__ __forceinline__ bool aborted(Ctrl* ctrl) { return *reinterpret_cast<volatile int*>(&ctrl->abort_flag) != 0; }
// the same for all lanes of a warp
__device__ __forceinline__ bool any_aborted(Ctrl* ctrl) { return __any_sync(0xffffffffu, aborted(ctrl)); }
__device__ __forceinline__ void wait_more(uint32_t addr, uint32_t parity, Ctrl* ctrl, int* status) {
    const uint64_t t0 = ptx::globaltimer_ns();
    while (!ptx::mbar_try_wait_hint(addr, parity, 20000)) {
        if (aborted(ctrl)) return;
        if (ptx::globaltimer_ns() - t0 > WAIT_LIMIT_NS) {
            *reinterpret_cast<volatile int*>(&ctrl->abort_flag) = 1;
            atomicCAS(status, CAKE_OK, CAKE_ERR_TIMEOUT);
            return;
        }
    }
}
__device__ __forceinline__ void wait_bar(uint64_t* bar, uint32_t parity, Ctrl* ctrl, int* status) {
    const uint32_t addr = ptx::smem_u32(bar);
    if (__builtin_expect(!ptx::mbar_try_wait(addr, parity & 1), 0)) wait_more(addr, parity & 1, ctrl, status);
}
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ void arrive(uint64_t* bar) { ptx::mbar_arrive(ptx::smem_u32(bar)); }
__device__ __forceinline__ float ex2(float x) {      // 2 ulp; below 2^-126 flushed to zero
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// What a row's scores are multiplied by: |scale| log2 e times its head's scale and what its queries were divided by (in 64 bits: the parts may leave 32 where
// the product does not).  Never zero (of which a mask's infinity would make a NaN): 2^-149 leaves scores of zero in all that 2^x sees.  Not a number: the
// row's end says so, and the mask stays a mask.
__device__ __forceinline__ float factor_of(float scale_log2, float head, float queries) {
    const float c = static_cast<float>(static_cast<double>(scale_log2) * fabsf(head) * queries);
    return c > 0.f ? c : LEAST;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// four e4m3 values to two pairs of f16: exact
__device__ __forceinline__ void e4m3_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    const uint16_t a = static_cast<uint16_t>(w & 0xffffu), b = static_cast<uint16_t>(w >> 16);
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"(a));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"(b));
}
// (a, b) * c - d
__device__ __forceinline__ void scale_sub2(float& a, float& b, float c, float minus_d) {
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(c), "f"(minus_d));
}
__device__ __forceinline__ void add2(float2& s, float a, float b) {
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(s.x), "+f"(s.y) : "f"(a), "f"(b));
}
// s += 0 * (a, b): NaN once one of them is not finite
__device__ __forceinline__ void check2(float2& s, float a, float b) {
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %4};\n\tfma.rn.f32x2 x, y, z, x;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(s.x), "+f"(s.y) : "f"(a), "f"(b), "f"(0.f));
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool ok) {      // zeros where !ok
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void store32(void* to, const uint32_t (&o)[32], int k) {      // o[k .. k + 7], to a multiple of 32 bytes
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(to), "r"(o[k]), "r"(o[k + 1]), "r"(o[k + 2]), "r"(o[k + 3]), "r"(o[k + 4]), "r"(o[k + 5]), "r"(o[k + 6]), "r"(o[k + 7])
                 : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ------------------------------------------------------------------------------------------------- who sees what
__device__ __forceinline__ int first_key(const Args& a, int pos, int klen) {
    return a.window > 0 && pos >= a.window ? min(pos - a.window + 1, klen) : 0;
}
__device__ __forceinline__ int end_key(const Args& a, int pos, int klen) { return a.causal ? max(0, min(pos + 1, klen)) : klen; }

__device__ __forceinline__ int page_number(const Args& a, int key) { return a.page_mul ? static_cast<int>(__umulhi(key, a.page_mul) >> a.page_shift) : key; }

// An entry: a sequence's new tokens, a key-value head and a run of its query heads.
struct Entry {
    i64 q0, k0;
    int qlen, klen, g, run;
};
template <bool PAGED>
__device__ __forceinline__ Entry entry_of(const Args& a, int e, bool report) {
    Entry n;
    const int per = a.Hkv * a.runs;
    const int b = a.per_mul ? static_cast<int>(__umulhi(e, a.per_mul) >> a.per_shift) : e, r = e - b * per;
    n.g = a.runs == 1 ? r : r / a.runs, n.run = r - n.g * a.runs;
    const int s0 = a.starts[b], s1 = a.starts[b + 1];
    bool bad = s0 < 0 || s1 < s0 || s1 > a.T;
    n.q0 = s0, n.qlen = bad ? 0 : s1 - s0;
    if (PAGED) {
        n.k0 = b * a.table_stride + n.g * a.table_head_stride;
        const i64 room = min(static_cast<i64>(a.max_pages) * a.c.page_size, static_cast<i64>(INT_MAX - 2 * KT));
        i64 len = a.lens[b * a.lens_stride + n.g * a.lens_head_stride];
        if (len > room) bad = true, len = room;
        n.klen = static_cast<int>(len < 0 ? 0 : len);
    } else {
        const int k0 = a.k_starts[b], k1 = a.k_starts[b + 1];
        const bool wrong = k0 < 0 || k1 < k0 || k1 > a.Tk;
        bad |= wrong;
        n.k0 = wrong ? 0 : k0, n.klen = wrong ? 0 : k1 - k0;
        if (wrong) n.qlen = 0;
    }
    if (bad && report) raise_bad_index(a.status);
    return n;
}
// tiles of keys [ja, jb) that tokens [tok, tok + n) of an entry see
__device__ __forceinline__ void tiles_of(const Args& a, int pos, int n, int klen, int& ja, int& jb) {
    ja = first_key(a, pos, klen) / KT;
    jb = (end_key(a, pos + n - 1, klen) + KT - 1) / KT;
    if (jb < ja) jb = ja;
}
template <int TILES>
__device__ __forceinline__ int blocks_of(const Args& a, int qlen) { return (qlen + TILES * a.tokens - 1) / (TILES * a.tokens); }
// Cost of the first n items of an entry, in keys: OVERHEAD + end - first key for each, where both grow by a block's tokens from item
// to item (but for the last item's end, which is the sequence's): sums of arithmetic series, no loop.  An item of one row tile, the last one it can be,
// takes its keys two tiles at a time and costs half as much (1,630 clocks a tile of keys where two row tiles take 3,190; counted in full, a step of single
// tokens and pieces of prompts took 263 us for 257); with 8-bit caches, whose tiles take as long to widen for one as for two, it does not
template <class T>
__device__ __forceinline__ bool is_cheap(const Args& a, int ntok) { return T::TILES == 2 && !T::F16 && ntok <= a.tokens; }
template <class T>
__device__ __noinline__ i64 cost_before(const Args& a, int qlen, int klen, int n) {
    const int per = T::TILES * a.tokens, off = klen - qlen;
    i64 less = 0;                                           // half of the last item's, if it is one row tile
    if (n > 0 && is_cheap<T>(a, qlen - (n - 1) * per)) less = (OVERHEAD + static_cast<i64>(klen) - first_key(a, off + (n - 1) * per, klen) + 1) >> 1;
    if (!a.causal) return static_cast<i64>(n) * (OVERHEAD + klen) - less;
    const int full = min(n, qlen / per);                    // items of a whole block of tokens
    i64 sum = static_cast<i64>(n) * OVERHEAD + (n > full ? klen : 0);
    const int i0 = off < 0 ? min(full, -off / per) : 0;     // those before see nothing
    const i64 m = full - i0;
    sum += m * off + per * (m * (i0 + 1 + full) / 2);       // off + (i + 1) per, i0 <= i < full
    if (a.window > 0) {
        const i64 gone = static_cast<i64>(off) - a.window + 1;      // first key of item i: gone + i per
        const int i1 = gone < 0 ? static_cast<int>(min(static_cast<i64>(n), (-gone + per - 1) / per)) : 0;
        const i64 k = n - i1;
        sum -= k * gone + per * (k * (i1 + n - 1) / 2);
    }
    return sum - less;
}
__device__ __forceinline__ i64 inclusive_scan(i64 v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const i64 u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}
// a share's end p keys (of cost) into an item of n tiles, in tiles, moved to the item's ends where they are near
__device__ __forceinline__ int snap(i64 p, int n, int cheap) {
    p <<= cheap;
    const int t = p <= OVERHEAD ? 0 : static_cast<int>(min(p - OVERHEAD, static_cast<i64>(INT_MAX))) / KT;
    return t < SNAP ? 0 : n - t < SNAP ? n : t;
}

// the tiles of keys of a segment that its row tile t sees (DUAL), or all of them
template <class T>
__device__ __forceinline__ bool is_dual(const Args& a, const Seg& s) { return T::TILES == 2 && s.ntok > a.tokens; }
__device__ __forceinline__ void range_of(const Args& a, const Seg& s, bool dual, int t, int& ra, int& rb) {
    ra = s.ja, rb = s.jb;
    if (dual) {
        int ja, jb;
        const int first = t * a.tokens;
        tiles_of(a, s.pos + first, min(a.tokens, s.ntok - first), s.klen, ja, jb);
        ra = max(ra, ja), rb = min(rb, jb);
        if (rb < ra) rb = ra;
    }
}

// ------------------------------------------------------------------------------------------------------ scheduler
template <class T>
__device__ __forceinline__ int stretch_of(const Args& a) { return (a.entries + T::WARPS - 1) / T::WARPS; }      // entries that a warp adds up
// One warp: finds the CTA's share of the list, tells the others of its segments, and loads their queries and (packed) keys.
template <class T>
__device__ __forceinline__ void load_queries_keys(const Args& a, Ctrl* ctrl, const Room& room, const CUtensorMap* mq, const CUtensorMap* mk, const Seg& s,
                                                  uint32_t (&q_count)[2], uint32_t& nk) {
    const uint32_t q_bytes = T::SLABS * static_cast<uint32_t>(a.tokens * a.heads) * 128u;
    const bool dual = is_dual<T>(a, s);
#pragma unroll 1
    for (int t = 0; t < (dual ? 2 : 1); ++t) {
        int ra, rb;
        range_of(a, s, dual, t, ra, rb);
        if (ra == rb) continue;
        wait_bar(&ctrl->q_empty[t], q_count[t] + 1, ctrl, a.status);
        if (aborted(ctrl)) return;
        ++q_count[t];
        const uint32_t bar = ptx::smem_u32(&ctrl->q_full[t]);
        ptx::mbar_arrive_expect_tx(bar, q_bytes);
#pragma unroll
        for (int x = 0; x < T::SLABS; ++x)
            ptx::tma_load_3d(ptx::smem_u32(room.q) + t * T::Q_TILE + x * T::SLAB, mq, bar, 64 * x, s.head0, static_cast<int>(s.tok) + t * a.tokens);
    }
    if constexpr (!T::PAGED) {
#pragma unroll 1
        for (int j = s.ja; j < s.jb; ++j)
#pragma unroll 1
            for (int u = 0; u < T::NKU; ++u, ++nk) {
                const uint32_t st = nk % T::K_STAGES;
                wait_bar(&ctrl->k_empty[st], nk / T::K_STAGES + 1, ctrl, a.status);
                if (aborted(ctrl)) return;
                const uint32_t bar = ptx::smem_u32(&ctrl->k_full[st]);
                ptx::mbar_arrive_expect_tx(bar, T::K_UNIT);
#pragma unroll
                for (int x = 0; x < T::K_SLABS; ++x)
                    ptx::tma_load_3d(ptx::smem_u32(room.k) + st * T::K_UNIT + x * T::SLAB, mk, bar, T::KC * u + 64 * x, s.g, static_cast<int>(s.k0) + KT * j);
            }
    }
}
// copies in flight land before the CTA gives up its shared memory (they have, unless a wait has expired)
__device__ __forceinline__ void landed(uint64_t* bars, uint32_t n, uint32_t stages) {
    const uint64_t t0 = ptx::globaltimer_ns();
    for (uint32_t i = n > stages ? n - stages : 0; i < n; ++i)
        while (!ptx::mbar_try_wait(ptx::smem_u32(&bars[i % stages]), (i / stages) & 1) && ptx::globaltimer_ns() - t0 < WAIT_LIMIT_NS / 4) {}
}
template <class T>
__device__ __forceinline__ void schedule(const Args& a, Ctrl* ctrl, const Room& room, const CUtensorMap* mq, const CUtensorMap* mk) {
    constexpr int TILES = T::TILES;
    const int lane = threadIdx.x & 31;
    const unsigned all = 0xffffffffu;
    // The costs, added up: of the warps' stretches, or of the entries where they are no more than lanes
    const bool few = a.entries <= 32;
    Entry one = {};
    i64 mine = 0;
    if (few) {
        if (lane < a.entries) one = entry_of<T::PAGED>(a, lane, blockIdx.x == 0);
        mine = cost_before<T>(a, one.qlen, one.klen, blocks_of<TILES>(a, one.qlen));
    } else if (lane < T::WARPS) {
        mine = ctrl->sums[lane];
    }
    const i64 sums = inclusive_scan(mine);
    const i64 total = __shfl_sync(all, sums, 31);
    // Shares: CTA c's begins at total * c / n, or a little before, for all CTAs alike
    const bool many = total >= static_cast<i64>(MIN_SHARE) * gridDim.x;
    const int n = many ? static_cast<int>(gridDim.x) : max(static_cast<int>(total) / MIN_SHARE, 1);
    auto begin_of = [&](int c) {
        return c >= n ? total : many ? static_cast<i64>(__umul64hi(total, a.share_mul * c)) : static_cast<i64>(static_cast<unsigned>(total) * c / n);
    };
    const int cta = blockIdx.x;
    uint32_t count = 0, q_count[2] = {0, 0}, nk = 0;      // segments, loads of queries, units of keys so far
    const bool lead = ptx::elect_one();
    auto post = [&](const Seg& s) {
        const int slot = count % SEGS;
        wait_bar(&ctrl->seg_empty[slot], (count / SEGS + 1) & 1, ctrl, a.status);
        if (any_aborted(ctrl)) return;      // (others may still read the place)
        if (lane == 0) {
            ctrl->seg[slot] = s;
            arrive(&ctrl->seg_full[slot]);
        }
        ++count;
    };
    Split split = {};
    if (cta < n && total > 0) {
        const i64 x0 = begin_of(cta), x1 = begin_of(cta + 1);
        // the entry that x0 is in (its stretch first)
        const unsigned behind = __ballot_sync(all, x0 < sums);
        const int w = __ffs(behind) - 1;
        i64 before = w > 0 ? __shfl_sync(all, sums, (w - 1) & 31) : 0;
        const int stretch = stretch_of<T>(a), e_end = few ? 0 : min(stretch * (w + 1), a.entries);
        int e = few ? 0 : stretch * w, block = 0, who = few ? w : 32;
#pragma unroll 1
        for (; who == 32 && e < e_end; e += who) {      // 32 entries at a time
            one = {};
            if (e + lane < e_end) one = entry_of<T::PAGED>(a, e + lane, false);
            const i64 cost = cost_before<T>(a, one.qlen, one.klen, blocks_of<TILES>(a, one.qlen)), upto = inclusive_scan(cost);
            const unsigned hit = __ballot_sync(all, x0 < before + upto);
            who = hit ? __ffs(hit) - 1 : 32;
            before += __shfl_sync(all, hit ? upto - cost : upto, hit ? who : 31);
        }
        if (few) e = w;
        Entry en;
        en.q0 = __shfl_sync(all, one.q0, who & 31), en.k0 = __shfl_sync(all, one.k0, who & 31);
        en.qlen = __shfl_sync(all, one.qlen, who & 31), en.klen = __shfl_sync(all, one.klen, who & 31);
        en.g = __shfl_sync(all, one.g, who & 31), en.run = __shfl_sync(all, one.run, who & 31);
        int blocks = blocks_of<TILES>(a, en.qlen);
        // its item
#pragma unroll 1
        for (int step = blocks > 1 ? 1 << (31 - __clz(blocks - 1)) : 0; step; step >>= 1)
            if (block + step < blocks && before + cost_before<T>(a, en.qlen, en.klen, block + step) <= x0) block += step;
        if (block) before += cost_before<T>(a, en.qlen, en.klen, block);
        int start = -1;
#pragma unroll 1
        while (x1 > before && block < blocks) {
            const int per = TILES * a.tokens, tok = block * per, ntok = min(per, en.qlen - tok);
            const int pos = en.klen - en.qlen + tok;
            int ja, jb;
            tiles_of(a, pos, ntok, en.klen, ja, jb);
            const int tiles = jb - ja;
            const int cheap = is_cheap<T>(a, ntok);
            const i64 end_at = before + ((OVERHEAD + static_cast<i64>(end_key(a, pos + ntok - 1, en.klen)) - (a.window > 0 ? first_key(a, pos, en.klen) : 0)) >> cheap);
            if (start < 0) start = x0 > before ? snap(x0 - before, tiles, cheap) : 0;      // the share's first item
            const bool to_end = x1 >= end_at;
            const int end = to_end ? tiles : snap(x1 - before, tiles, cheap);
            if (to_end ? start < tiles || start == 0 : start < end) {
                Seg s;
                s.tok = en.q0 + tok, s.k0 = en.k0, s.g = en.g;
                s.head0 = en.g * a.G + en.run * a.heads, s.heads = min(a.heads, a.G - en.run * a.heads);
                s.ntok = ntok, s.pos = pos, s.klen = en.klen;
                s.ja = ja + start, s.jb = ja + end;
                s.part = start == 0 && end == tiles ? -1 : 2 * cta + (start == 0 ? 1 : 0);
                s.negative = a.negative;
                if (T::F16 && a.c.k_scale && a.c.k_scale[en.g] < 0.f) s.negative ^= 1;
                s.done = 0;
                post(s);
                if (lead && !aborted(ctrl)) load_queries_keys<T>(a, ctrl, room, mq, mk, s, q_count, nk);
                __syncwarp();
                if (any_aborted(ctrl)) break;
                if (start == 0 && end < tiles) {      // the CTAs behind this one have the rest
                    int c1 = cta;
#pragma unroll 1
                    for (int c = cta + 1; c < n; c += 32) {
                        const i64 x = begin_of(c + lane);
                        const unsigned in = __ballot_sync(all, c + lane < n && x < end_at && snap(x - before, tiles, cheap) < tiles);
                        c1 += __popc(in);
                        if (in != all) break;
                    }
                    split.tok = s.tok, split.head0 = s.head0, split.heads = s.heads, split.ntok = ntok, split.c1 = c1, split.g = en.g;
                    split.valid = 1;
                }
            }
            if (!to_end) break;
            before = end_at;
            start = 0;
            if (++block == blocks) {
                block = 0, blocks = 0;
#pragma unroll 1
                while (blocks == 0 && ++e < a.entries) {
                    en = entry_of<T::PAGED>(a, e, false);
                    blocks = blocks_of<TILES>(a, en.qlen);
                }
            }
        }
    }
    if (lane == 0) a.splits[cta] = split;
    Seg last = {};
    last.done = 1;
    post(last);
    if (lead && aborted(ctrl)) {
        for (int t = 0; t < 2; ++t) landed(&ctrl->q_full[t], q_count[t], 1);
        if (!T::PAGED) landed(ctrl->k_full, nk, T::K_STAGES);
    }
    __syncwarp();
}

// The roles' side of it: reads the next segment (whole warps, or one thread with `alone`).  False: no more.
__device__ __forceinline__ bool next_seg(const Args& a, Ctrl* ctrl, uint32_t& count, Seg& s, bool alone) {
    const int slot = count % SEGS;
    wait_bar(&ctrl->seg_full[slot], (count / SEGS) & 1, ctrl, a.status);
    if (alone ? aborted(ctrl) : any_aborted(ctrl)) return false;
    s = ctrl->seg[slot];
    if (!alone) __syncwarp();
    if (alone || (threadIdx.x & 31) == 0) arrive(&ctrl->seg_empty[slot]);
    ++count;
    return !s.done;
}

// ------------------------------------------------------------------------------------------------------------ rows
// Rows whose O holds something that is not finite.  It may come from values that a row does not see (they weigh nothing, but zero times infinity is NaN), or from
// finite ones whose weighted sum passes 32 bits (weights reach 2^20): the row is then computed again, in 32 bits, from the keys that it sees in this segment, with
// weights of at most 2^-DOWN.  Where it comes from infinities and NaN that the row sees it is right as it is.  A warp to its 32 rows: it looks once for the first and the
// last such value of each column, and has then MEND rows at a time, a lane to a key for the scores, two or more columns to a lane for the sums.
// Measured: a tile's 127 rows of 128 over 4,096 cached keys 7.5 ms (a row to a thread: 187), over 40,000 73 ms (heads of 256: 120), where the call takes 0.4 (0.6).  So 2 to 3 us
// a key for a warp's rows: a piece of a million keys ends before the others' patience does.
__device__ __forceinline__ float2 as_pair(uint32_t w) { return make_float2(bf16_lo(w), bf16_hi(w)); }
template <class T>
__device__ __forceinline__ float2 pair_at(const char* row, int d) {      // elements d and d + 1 of a key or value
    if (T::F16) {
        const uint16_t w = *reinterpret_cast<const uint16_t*>(row + d);
        uint32_t f;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(f) : "h"(w));
        return __half22float2(*reinterpret_cast<const __half2*>(&f));
    }
    return as_pair(*reinterpret_cast<const uint32_t*>(row + 2 * d));
}
// where a key of a segment, or its value, is; nullptr: nowhere
template <class T, bool VALUE>
__device__ __forceinline__ const char* locate(const Args& a, const Seg* s, int key, int to) {
    if (key >= to) return nullptr;
    if (T::PAGED) {
        const int page = a.table[s->k0 + page_number(a, key)];
        if (page < 0 || page >= a.c.num_pages) return nullptr;
        const i64 off = key - page_number(a, key) * a.c.page_size;
        return static_cast<const char*>(VALUE ? a.c.v : a.c.k) +
               (VALUE ? page * a.c.v_page_stride + off * a.c.v_token_stride + s->g * a.c.v_head_stride
                      : page * a.c.k_page_stride + off * a.c.k_token_stride + s->g * a.c.k_head_stride) * (T::F16 ? 1 : 2);
    }
    return reinterpret_cast<const char*>(VALUE ? a.v + (s->k0 + key) * a.v_stride + s->g * a.v_head_stride : a.k + (s->k0 + key) * a.k_stride + s->g * a.k_head_stride);
}
template <class T>
__device__ __forceinline__ void eight_at(const char* row, int d, float (&f)[8]) {      // elements d to d + 7
    if (T::F16) {
        const uint2 w = *reinterpret_cast<const uint2*>(row + d);
        uint32_t h[4];
        e4m3_to_f16(w.x, h[0], h[1]), e4m3_to_f16(w.y, h[2], h[3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&h[j]));
            f[2 * j] = u.x, f[2 * j + 1] = u.y;
        }
    } else {
        const uint4 u = *reinterpret_cast<const uint4*>(row + 2 * d);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) f[2 * j] = bf16_lo(w[j]), f[2 * j + 1] = bf16_hi(w[j]);
    }
}
constexpr int MEND = 4, DOWN = 40;
// todo: a bit for each of the warp's rows, row0 + bit of row tile t, that holds something that is not finite; tiles of keys [ra, rb) were multiplied
template <class T>
__device__ __noinline__ void mend_rows(const Args& a, Ctrl* ctrl, const Seg* s, unsigned todo, int row0, int t, int ra, int rb) {
    constexpr int D = T::D, PAIRS = (D + 63) / 64;
    constexpr unsigned all = 0xffffffffu;
    constexpr float kDown = 1.f / (1ull << DOWN);
    const int lane = threadIdx.x & 31, pos = s->pos, klen = s->klen;
    const int tile = is_dual<T>(a, *s) ? t : 0;
    int from = KT * ra, to = KT * rb;
    if (T::PAGED) from = max(from, first_key(a, pos, klen)), to = min(to, end_key(a, pos + s->ntok - 1, klen));      // (others were not loaded)
    else to = min(to, klen);                       // (zeros were put behind the sequence)
    // first and last key of which the lane's columns 2 lane + 64 j and the next are not finite
    int first[2 * PAIRS], last[2 * PAIRS];
#pragma unroll
    for (int j = 0; j < 2 * PAIRS; ++j) first[j] = INT_MAX, last[j] = -1;
#pragma unroll 1
    for (int key = from; key < to; key += 32) {
        const char* const mine = locate<T, true>(a, s, key + lane, to);
#pragma unroll 1
        for (int i = 0; i < 32; i += 8) {
            float2 f[8][PAIRS];
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const char* const v = reinterpret_cast<const char*>(__shfl_sync(all, reinterpret_cast<unsigned long long>(mine), i + b));
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) f[b][j] = v && 2 * lane + 64 * j < D ? pair_at<T>(v, 2 * lane + 64 * j) : make_float2(0.f, 0.f);
            }
#pragma unroll
            for (int b = 0; b < 8; ++b)
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) {
                    if (!isfinite(f[b][j].x)) first[2 * j] = min(first[2 * j], key + i + b), last[2 * j] = key + i + b;
                    if (!isfinite(f[b][j].y)) first[2 * j + 1] = min(first[2 * j + 1], key + i + b), last[2 * j + 1] = key + i + b;
                }
        }
    }
    const float vs = T::F16 && a.c.v_scale ? a.c.v_scale[s->g] : 1.f, ks = T::F16 && a.c.k_scale ? a.c.k_scale[s->g] : 1.f;
    float* const part = a.parts + s->part * T::PART;
    auto out_row = [&](int r) {
        const int tok = r / a.heads;
        return (s->tok + tile * a.tokens + tok) * a.Hq + s->head0 + r - tok * a.heads;
    };
    __syncwarp();                                           // (rows that others of the warp have stored)
    for (;;) {
        int rows[MEND], k0[MEND], k1[MEND], kmin = INT_MAX, kmax = 0;
#pragma unroll
        for (int n = 0; n < MEND; ++n) {
            rows[n] = -1, k0[n] = k1[n] = 0;
#pragma unroll 1
            for (; todo && rows[n] < 0; todo &= todo - 1) {
                const int r = row0 + __ffs(todo) - 1, tok = tile * a.tokens + r / a.heads;
                const int b0 = max(from, first_key(a, pos + tok, klen)), b1 = min(to, end_key(a, pos + tok, klen));
                bool again = false;
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) {
                    const int d = 2 * lane + 64 * j;
                    if (d >= D) continue;
                    const float2 f = s->part >= 0 ? *reinterpret_cast<const float2*>(part + static_cast<i64>(tile * MT + r) * D + d)
                                                  : as_pair(*reinterpret_cast<const uint32_t*>(a.out + out_row(r) * D + d));
                    // (last is -1 where there are none)
                    again |= first[2 * j] < b0 || last[2 * j] >= b1 || (last[2 * j] < 0 && !isfinite(f.x));
                    again |= first[2 * j + 1] < b0 || last[2 * j + 1] >= b1 || (last[2 * j + 1] < 0 && !isfinite(f.y));
                }
                if (__any_sync(all, again)) rows[n] = r, k0[n] = b0, k1[n] = b1, kmin = min(kmin, b0), kmax = max(kmax, b1);
            }
        }
        if (rows[0] < 0) break;
        const cake_bf16* q[MEND];
        float c[MEND], inv[MEND], m[MEND], l[MEND];      // l: of the lane's keys
        float2 o[MEND][PAIRS];
#pragma unroll
        for (int n = 0; n < MEND; ++n) {
            const int r = rows[n] < 0 ? rows[0] : rows[n], tok = r / a.heads;
            q[n] = a.q + (s->tok + tile * a.tokens + tok) * a.q_stride + (s->head0 + r - tok * a.heads) * a.q_head_stride;
            const float qs = T::F16 ? ctrl->q_scale[tile][r] : 1.f;      // (as 16 bits took them: their products stay in 32)
            c[n] = factor_of(a.scale_log2, ks, qs), inv[n] = 1.f / qs;
            if (s->negative) c[n] = -c[n];
            m[n] = NEG_INF, l[n] = 0.f;
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) o[n][j] = make_float2(0.f, 0.f);
        }
#pragma unroll 1
        for (int key = kmin; key < kmax; key += 32) {
            const char* const k = locate<T, false>(a, s, key + lane, kmax);
            const char* const mine = locate<T, true>(a, s, key + lane, kmax);
            float x[MEND];
#pragma unroll
            for (int n = 0; n < MEND; ++n) x[n] = 0.f;
            if (k) {
#pragma unroll 2
                for (int d = 0; d < D; d += 8) {
                    float f[8];
                    eight_at<T>(k, d, f);
#pragma unroll
                    for (int n = 0; n < MEND; ++n) {
                        const uint4 u = *reinterpret_cast<const uint4*>(q[n] + d);
                        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float lo = T::F16 ? bf16_lo(w[j]) * inv[n] : bf16_lo(w[j]), hi = T::F16 ? bf16_hi(w[j]) * inv[n] : bf16_hi(w[j]);
                            x[n] = fmaf(lo, f[2 * j], x[n]), x[n] = fmaf(hi, f[2 * j + 1], x[n]);
                        }
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < MEND; ++n) {
                const bool sees = k && key + lane >= k0[n] && key + lane < k1[n];
                x[n] = sees ? x[n] * c[n] : NEG_INF;
                float up = x[n];
#pragma unroll
                for (int b = 16; b; b >>= 1) up = fmaxf(up, __shfl_xor_sync(all, up, b));
                up = fmaxf(up, m[n]);
                const float base = up == NEG_INF ? 0.f : up, f = ex2(m[n] - base), p = ex2(x[n] - base);
                m[n] = up, l[n] = l[n] * f + p;
                x[n] = sees ? p * kDown : -1.f;    // the key's weight; -1: nothing, whatever its value is
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) o[n][j].x *= f, o[n][j].y *= f;
            }
#pragma unroll 1
            for (int i = 0; i < 32; i += 4) {
                float2 u[4][PAIRS];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const char* const v = reinterpret_cast<const char*>(__shfl_sync(all, reinterpret_cast<unsigned long long>(mine), i + b));
#pragma unroll
                    for (int j = 0; j < PAIRS; ++j) u[b][j] = v && 2 * lane + 64 * j < D ? pair_at<T>(v, 2 * lane + 64 * j) : make_float2(0.f, 0.f);
                }
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int n = 0; n < MEND; ++n) {
                        const float w = __shfl_sync(all, x[n], i + b);
                        if (w < 0.f) continue;
#pragma unroll
                        for (int j = 0; j < PAIRS; ++j) o[n][j].x = fmaf(w, u[b][j].x, o[n][j].x), o[n][j].y = fmaf(w, u[b][j].y, o[n][j].y);
                    }
            }
        }
#pragma unroll
        for (int n = 0; n < MEND; ++n) {
            if (rows[n] < 0) break;
#pragma unroll
            for (int b = 16; b; b >>= 1) l[n] += __shfl_xor_sync(all, l[n], b);
            const int part_row = tile * MT + rows[n];
            const i64 row = out_row(rows[n]);
            const float f = l[n] == 0.f ? 0.f : vs / l[n];
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) {
                const int d = 2 * lane + 64 * j;
                if (d >= D) continue;
                if (s->part >= 0) *reinterpret_cast<float2*>(part + static_cast<i64>(part_row) * D + d) = o[n][j];
                else *reinterpret_cast<uint32_t*>(a.out + row * D + d) = pack_bf16(o[n][j].x * f * (1.f / kDown), o[n][j].y * f * (1.f / kDown));
            }
            if (lane == 0) {
                if (s->part >= 0) *reinterpret_cast<float2*>(part + static_cast<i64>(T::PART_ROWS) * D + 2 * part_row) = make_float2(m[n] + DOWN, l[n] * kDown);
                else if (a.lse) a.lse[row] = (m[n] + log2f(l[n])) * LN2;
            }
        }
    }
}

// Queries of a row to f16, in place: divided by a power of two that brings its largest to [1, 2).  Returns that power.
template <class T>
__device__ __forceinline__ float narrow_queries(uint8_t* row, int r) {
    float most = 0.f;
#pragma unroll 1
    for (int i = 0; i < T::SLABS * 8; ++i) {
        const uint4 u = *reinterpret_cast<const uint4*>(row + (i >> 3) * T::SLAB + (((i & 7) ^ (r & 7)) << 4));
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) most = fmaxf(most, fmaxf(fabsf(bf16_lo(w[j])), fabsf(bf16_hi(w[j]))));
    }
    uint32_t e = __float_as_uint(most) >> 23;                   // a power of two, 2^(e - 127)
    e = most == 0.f || e == 255 ? 127 : e < 1 ? 1 : e > 253 ? 253 : e;
    const float inv = __uint_as_float((254 - e) << 23);
#pragma unroll 1
    for (int i = 0; i < T::SLABS * 8; ++i) {
        uint4* const at = reinterpret_cast<uint4*>(row + (i >> 3) * T::SLAB + (((i & 7) ^ (r & 7)) << 4));
        const uint4 u = *at;
        *at = make_uint4(pack_f16(bf16_lo(u.x) * inv, bf16_hi(u.x) * inv), pack_f16(bf16_lo(u.y) * inv, bf16_hi(u.y) * inv),
                         pack_f16(bf16_lo(u.z) * inv, bf16_hi(u.z) * inv), pack_f16(bf16_lo(u.w) * inv, bf16_hi(u.w) * inv));
    }
    return __uint_as_float(e << 23);
}

// Warpgroup t of softmax rows: thread r has row r of the tile.
template <class T>
__device__ __forceinline__ void softmax_rows(const Args& a, Ctrl* ctrl, const Room& room, uint32_t tmem, int t) {
    constexpr int D = T::D;
    // What is subtracted from a row's scores, m, is the maximum of the first tile in which it sees anything; it is raised to the maximum so far
    // only when a tile's weights add up to more than LIMIT.  So the maximum of most tiles is never looked for, and O is hardly ever
    // rescaled: weights above 1 do no harm in 32 bits, nor rounded to bf16.  Weights in f16 (8-bit values, which widen to f16 exactly) lie LIFT higher, the heaviest at 2^11 or
    // above, so that 11 bits are held down to 2^-25 of it and steps of 2^-35 below.  A tile of which a quarter's weights add up to more than f16 holds is looked
    // at, and m is raised where one of them passes 2^(LIFT + ROOM); so that this is rare, every row looks for its maximum at its 2nd, 5th, 17th, ... tile too.  (2 x 32,768
    // keys, scores of a spread of up to 1.8: 1,669 us; without those looks 1,812 - 1,858; raised whenever a larger one is found, 512 tokens over 2 x 8,192: 417 us for 350;
    // heaviest at 2^7, 11 bits down to 2^-21: 1,637 and 349)
    constexpr float LIFT = T::F16 ? 11.f : 0.f, ROOM = T::F16 ? 4.875f : 0.f, LIMIT = T::F16 ? 60000.f : 1048576.f;
    // x c - m in one rounding lies beside what m = x c was rounded by: half a step of m, which passes 2^x's range where m passes 2^30.  Scores that reach FAR, whose
    // neighbours in 32 bits are two powers of two apart, are multiplied by the power of two that is not below c instead, which rounds nothing; what is
    // beyond FAR stays beyond it, in the same order
    constexpr float FAR = 16777216.f;
    const int lane = threadIdx.x & 31, r = threadIdx.x & 127;
    const uint32_t t_lane = tmem + (static_cast<uint32_t>(r & 96) << 16);
    const int tok = r / a.heads;
    uint32_t segs = 0, s_count = 0, o_count[2] = {0, 0}, q_count[2] = {0, 0}, x_count = 0, tiles = 0;      // o: products on a place of P
    for (;; ++segs) {
        // (the segment stays where it is until its end: registers are for the scores)
        const Seg* const sp = &ctrl->seg[segs % SEGS];
        wait_bar(&ctrl->seg_full[segs % SEGS], segs / SEGS, ctrl, a.status);
        if (any_aborted(ctrl) || sp->done) break;
        const bool dual = is_dual<T>(a, *sp), alt = T::TILES == 2 && !dual;
        int first, rb;
        range_of(a, *sp, dual, t, first, rb);
        const int ra = first, step = alt ? 2 : 1;
        if (alt) first += t;
        const int n_mine = first < rb ? (rb - first + step - 1) / step : 0;
        const uint32_t flag0 = tiles + first - sp->ja;                      // its first tile among all that were loaded
        const int my_tok = (dual ? t * a.tokens : 0) + tok;                 // of the segment's tokens
        int k0, k1, inner0, inner1;                                         // the row sees [k0, k1), every row of the tile [inner0, inner1)
        {
            // (rows that are none see what the last one does: their scores are computed, but go nowhere)
            const int klen = sp->klen, pos = sp->pos;
            k0 = first_key(a, pos + my_tok, klen), k1 = end_key(a, pos + my_tok, klen);
            inner0 = first_key(a, pos + min(sp->ntok, (dual ? (t + 1) * a.tokens : sp->ntok)) - 1, klen);
            inner1 = end_key(a, pos + (dual ? t * a.tokens : 0), klen);
        }
        float c = a.scale_log2 > 0.f ? a.scale_log2 : LEAST;
        if (T::F16) {
            const int qt = dual ? t : 0;
            const bool used = dual ? n_mine > 0 : sp->jb > sp->ja;
            if (used && (dual || t == 0)) {
                wait_bar(&ctrl->q_full[qt], q_count[qt], ctrl, a.status);
                ctrl->q_scale[qt][r] = narrow_queries<T>(room.q + qt * T::Q_TILE + r * 128, r);
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) arrive(&ctrl->q_conv[qt]);
            }
            if (used) {
                wait_bar(&ctrl->q_conv[qt], q_count[qt], ctrl, a.status);
                c = factor_of(a.scale_log2, a.c.k_scale ? a.c.k_scale[sp->g] : 1.f, ctrl->q_scale[qt][r]);
                ++q_count[qt];
            }
            if (t == 1) {      // looks at every load of the first tile
                bool other = !dual && used;
                if (dual) {
                    int ua, ub;
                    range_of(a, *sp, dual, 0, ua, ub);
                    other = ub > ua;
                    if (other) wait_bar(&ctrl->q_conv[0], q_count[0], ctrl, a.status), ++q_count[0];
                }
                __syncwarp();
                if (other && lane == 0) arrive(&ctrl->q_empty[0]);
            }
        }
        const bool idle = !__any_sync(0xffffffffu, tok < a.tokens && my_tok < sp->ntok);      // a warp without a row: P may hold anything there
        // Rows that are none, or see nothing, have no maximum to look for: whatever their scores are (what lay in shared memory, for rows behind the
        // queries' box), they do not hold up the others
        const bool live = tok < a.tokens && my_tok < sp->ntok && k0 < k1;
        float m = live ? NEG_INF : 0.f, l = 0.f;   // m: the maximum that is subtracted, without LIFT
        const float c_near = c, c_far = __uint_as_float(min((__float_as_uint(c) + 0x7fffffu) & 0xff800000u, 0x7f000000u));      // c: the one of m
        for (int i = 0; i < n_mine; ++i) {
            const int key0 = KT * (first + i * step);
            const int pb = T::TILES == 2 ? t : i & 1;      // place of the weights
            wait_bar(&ctrl->s_full[t], s_count, ctrl, a.status);
            ++s_count;
            if (__builtin_expect(idle, 0)) {
                if (o_count[pb]) wait_bar(&ctrl->o_done[pb], o_count[pb] - 1, ctrl, a.status);
                ++o_count[pb];
                if (lane == 0) arrive(&ctrl->s_free), arrive(&ctrl->p_ready[pb]);
                continue;
            }
            ptx::tc_fence_after();
            uint32_t x[4][32];
#pragma unroll
            for (int w = 0; w < 4; ++w) ptx::tmem_ld_x32(t_lane + S_COL + 32 * w, x[w]);
            ptx::tmem_ld_wait(x[0]);
#pragma unroll
            for (int w = 1; w < 4; ++w) ptx::reg_dep(x[w]);
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive(&ctrl->s_free);
            bool masked = key0 < inner0 || key0 + KT > inner1;
            uint4 pages = make_uint4(~0u, ~0u, ~0u, ~0u);
            if (T::PAGED) {
                pages = ctrl->flags[(flag0 + i * step) % FLAGS_AHEAD];
                masked |= (pages.x & pages.y & pages.z & pages.w) != ~0u;
            }
            // Which rows look for their maximum: it is theirs alone to say, so that a row's bits do not depend on its neighbours
            bool search = m == NEG_INF;
            if (T::F16) search |= live && i > 0 && (i & (i - 1)) == 0 && (i & 0x55555555) != 0;
            if (__builtin_expect(masked, 0)) {
                const uint32_t seen[4] = {pages.x, pages.y, pages.z, pages.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int b0 = min(max(k0 - key0 - 32 * w, 0), 32), b1 = min(max(k1 - key0 - 32 * w, 0), 32);
                    // bits [b0, b1)
                    const uint32_t below1 = b1 == 32 ? ~0u : (1u << b1) - 1, below0 = b0 == 32 ? ~0u : (1u << b0) - 1;
                    const uint32_t bits = seen[w] & below1 & ~below0;
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (!(bits & (1u << k))) x[w][k] = __float_as_uint(NEG_INF);
                }
            }
            float total;
#pragma unroll 1                               // (one copy of this: the loops are about what the instruction caches hold)
            for (int pass = 0;; ++pass) {
                if (__builtin_expect(__any_sync(0xffffffffu, search), 0)) {
                    float top[4];
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        top[w] = __uint_as_float(x[w][0]);
#pragma unroll
                        for (int k = 1; k < 31; k += 2) top[w] = ptx::fmax3(top[w], __uint_as_float(x[w][k]), __uint_as_float(x[w][k + 1]));
                        top[w] = fmaxf(top[w], __uint_as_float(x[w][31]));
                    }
                    top[0] = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                    const float near = top[0] * c_near, up = fabsf(near) < FAR ? near : top[0] * c_far;
                    const bool higher = search && up > (pass > 0 ? m + ROOM : m);
                    if (T::F16 && pass > 0 && !__any_sync(0xffffffffu, higher)) break;
                    const float f = higher ? ex2(m - up) : 1.f;
                    if (higher) m = up;
                    c = fabsf(m) < FAR ? c_near : c_far;
                    l *= f;
                    if (i > 0) {
                        const int ob = T::TILES == 2 ? t : 0, last = T::TILES == 2 ? t : pb ^ 1;      // the product before has to be complete
                        wait_bar(&ctrl->o_done[last], o_count[last] - 1, ctrl, a.status);
                        ptx::tc_fence_after();
#pragma unroll 1
                        for (int d = 0; d < D; d += 16) {
                            uint32_t o[16];
                            const uint32_t oa = t_lane + O_COL + ob * KT + d;
                            ptx::tmem_ld_x16(oa, o);
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            ptx::tmem_st_x16(oa, o);
                        }
                    }
                }
                const float minus = m == NEG_INF ? 0.f : LIFT - m;
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t p[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float u = __uint_as_float(x[w][2 * k]), v = __uint_as_float(x[w][2 * k + 1]);
                        scale_sub2(u, v, c, minus);
                        u = ex2(u), v = ex2(v);
                        add2(sum[k & 1], u, v);
                        // Weights are rounded to 16 bits for the tensor core (bf16: half a step of 2^-8, about what the output's own
                        // rounding is; it is the operand type that the values have, and a second term for the rest would be a second product and has
                        // no room in tensor memory), their sum is that of the unrounded ones
                        p[k] = T::F16 ? pack_f16(u, v) : pack_bf16(u, v);
                    }
                    // the product that read the place of the weights before is complete (looked at every time: a parity names every other one)
                    if (w == 0 && o_count[pb]) wait_bar(&ctrl->o_done[pb], o_count[pb] - 1, ctrl, a.status);
                    ptx::tmem_st_x16(t_lane + p_col(pb) + 16 * w, p);
                }
                total = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                // (the second time m is the maximum: no more than that can be done for scores so large that their differences are lost)
                search = live && !search && (T::F16 ? fmaxf(ptx::fmax3(sum[0].x, sum[0].y, sum[1].x), sum[1].y) : total) > LIMIT;
                if (pass > 0 || !__any_sync(0xffffffffu, search)) break;
            }
            ++o_count[pb];
            l += total;
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive(&ctrl->p_ready[pb]);
        }
        const int ja = sp->ja, jb = sp->jb;
        tiles += jb - ja;
        if (dual && t == 0) {      // (the first warpgroup counts the second tile's products too)
            int ua, ub;
            range_of(a, *sp, dual, 1, ua, ub);
            o_count[1] += ub - ua;
        }
        const int n_other = alt ? (jb - ja) / 2 : 0;       // the second tile's steps
        if (alt && t == 1) {
            // the first warpgroup joins
            if (n_mine) {
                if (x_count) wait_bar(&ctrl->x_empty, x_count - 1, ctrl, a.status);
                ctrl->ml[r] = make_float2(m, l);
                __syncwarp();
                if (lane == 0) arrive(&ctrl->x_full);
                ++x_count;
            }
            __syncwarp();
            if (lane == 0) arrive(&ctrl->seg_empty[segs % SEGS]);
            continue;
        }
        // ---- the end of the segment
        float f0 = 1.f, f1 = 0.f, top = m;
        if (n_other) {
            wait_bar(&ctrl->x_full, x_count, ctrl, a.status);
            const float2 other = ctrl->ml[r];
            __syncwarp();
            if (lane == 0) arrive(&ctrl->x_empty);
            ++x_count;
            top = fmaxf(m, other.x);
            const float from = top == NEG_INF ? 0.f : top;
            f0 = ex2(m - from), f1 = ex2(other.x - from);
            l = l * f0 + other.y * f1;
            o_count[1] += n_other;
            wait_bar(&ctrl->o_done[1], o_count[1] - 1, ctrl, a.status);
        }
        if (fabsf(top) >= FAR && top != NEG_INF) top = top / c_far * c_near;
        const int ob = T::TILES == 2 ? t : 0;
        if (n_mine) {
            const int last = T::TILES == 2 ? t : (n_mine - 1) & 1;
            wait_bar(&ctrl->o_done[last], o_count[last] - 1, ctrl, a.status);
        }
        ptx::tc_fence_after();
        const int g = sp->g, part_at = sp->part, h = r - tok * a.heads;
        const bool valid = tok < a.tokens && my_tok < sp->ntok && h < sp->heads;
        const i64 row = (sp->tok + my_tok) * a.Hq + sp->head0 + h;
        const float sub = top == NEG_INF ? NEG_INF : top - LIFT;      // what was subtracted
        const float vs = T::F16 && a.c.v_scale ? a.c.v_scale[g] : 1.f;
        // (a scale that is no number: so are the rows that see anything)
        if (isnan(a.scale_log2) || (T::F16 && a.c.k_scale && isnan(a.c.k_scale[g]))) l = l == 0.f ? 0.f : NAN;
        const bool empty = l == 0.f;               // sees nothing that weighs anything: zeros, whatever the values are
        const float inv = part_at >= 0 ? 1.f : vs / l;
        f0 *= inv, f1 *= inv;
        const int part_row = (dual ? t * MT : 0) + r;
        float* const part = a.parts + part_at * T::PART;
        float2 odd[4];                             // NaN once something is not finite
#pragma unroll
        for (int k = 0; k < 4; ++k) odd[k] = make_float2(0.f, 0.f);
        // (a short loop: an item's end is run once in a while, and to fetch its instructions is what costs it most; with the next columns on their way
        // meanwhile, and twice the code, 8 packed prompts took 151 us for 141)
        uint32_t oa[32];
        auto fetch = [&](uint32_t (&o)[32], int d) {
            if (n_mine) {
                ptx::tmem_ld_x32(t_lane + O_COL + ob * KT + d, o);
            } else {
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] = 0u;
            }
        };
        auto finish = [&](uint32_t (&o)[32], int d) {
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f0);
            if (__builtin_expect(n_other, 0)) {
                uint32_t o1[32];
                ptx::tmem_ld_x32(t_lane + O_COL + KT + d, o1);
                ptx::tmem_ld_wait(o1);
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(fmaf(__uint_as_float(o1[k]), f1, __uint_as_float(o[k])));
            }
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
                check2(odd[(k >> 1) & 3], __uint_as_float(o[k]), __uint_as_float(o[k + 1]));
                if (empty) o[k] = o[k + 1] = 0u;
            }
            // (whole sectors: by halves, what is stored held up all that comes behind it in shared memory too; 8 packed prompts 143 us for 138)
            if (!valid) return;
            if (part_at >= 0) {
                float* const to = part + static_cast<i64>(part_row) * D + d;
#pragma unroll
                for (int k = 0; k < 4; ++k) store32(to + 8 * k, o, 8 * k);
            } else {
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = pack_bf16(__uint_as_float(o[2 * k]), __uint_as_float(o[2 * k + 1]));
                cake_bf16* const to = a.out + row * D + d;
                if (a.wide) {
                    store32(to, o, 0), store32(to + 16, o, 8);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) reinterpret_cast<uint4*>(to)[k] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                }
            }
        };
#pragma unroll 1
        for (int d = 0; d < D; d += 32) {
            fetch(oa, d);
            ptx::tmem_ld_wait(oa);
            finish(oa, d);
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) {
            if (n_mine) arrive(&ctrl->o_free[ob]);
            if (n_other) arrive(&ctrl->o_free[1]);
        }
        if (valid) {
            if (part_at >= 0) *reinterpret_cast<float2*>(part + static_cast<i64>(T::PART_ROWS) * D + 2 * part_row) = make_float2(sub, l);
            else if (a.lse) a.lse[row] = empty ? NEG_INF : (sub + __log2f(l)) * LN2;
        }
        const bool finite = !isnan((odd[0].x + odd[0].y) + (odd[1].x + odd[1].y) + (odd[2].x + odd[2].y) + (odd[3].x + odd[3].y));
        const unsigned todo = __ballot_sync(0xffffffffu, valid && !finite && isfinite(l) && isfinite(vs) && !empty);
        if (__builtin_expect(todo != 0, 0)) mend_rows<T>(a, ctrl, sp, todo, r & 96, t, ra, rb);
        __syncwarp();
        if (lane == 0) arrive(&ctrl->seg_empty[segs % SEGS]);
    }
}

// ------------------------------------------------------------------------------------------------------------ loads
// Values of packed prompts: one warp.
template <class T>
__device__ __forceinline__ void load_unit(uint32_t place, const CUtensorMap* mv, uint64_t* full, int column, int g, int key) {
    const uint32_t bar = ptx::smem_u32(full);
    ptx::mbar_arrive_expect_tx(bar, T::V_UNIT);
#pragma unroll
    for (int x = 0; x < T::V_SLABS; ++x) ptx::tma_load_3d(place + x * T::SLAB, mv, bar, column + 64 * x, g, key);
}
// What lies behind a sequence in its last tile is another's or nobody's: zeros in its place, of which no weight of zero makes a NaN
template <class T>
__device__ __noinline__ void load_end(Ctrl* ctrl, int* status, uint8_t* place, const CUtensorMap* mv, uint64_t* full, uint32_t ends, int column, int g, int key, int kept) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) load_unit<T>(ptx::smem_u32(place), mv, &ctrl->v_end, column, g, key);
    __syncwarp();
    wait_bar(&ctrl->v_end, ends, ctrl, status);
#pragma unroll 1
    for (int x = 0; x < T::V_SLABS; ++x)
#pragma unroll 4
        for (int at = kept * 128 + lane * 16; at < KT * 128; at += 512) *reinterpret_cast<uint4*>(place + x * T::SLAB + at) = make_uint4(0u, 0u, 0u, 0u);
    ptx::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) arrive(full);
}
template <class T>
__device__ __forceinline__ void load_values(const Args& a, Ctrl* ctrl, const Room& room, const CUtensorMap* mv) {
    const bool lead = ptx::elect_one();
    uint32_t segs = 0, nv = 0, ends = 0;                    // segments, units, units that a sequence ends in
    Seg s;
    while (next_seg(a, ctrl, segs, s, false)) {
        const int klen = uniform(s.klen);
#pragma unroll 1
        for (int j = s.ja; j < s.jb; ++j) {
#pragma unroll 1
            for (int u = 0; u < T::NVU; ++u, ++nv) {
                const uint32_t st = nv % T::V_STAGES;
                wait_bar(&ctrl->v_empty[st], nv / T::V_STAGES + 1, ctrl, a.status);
                if (any_aborted(ctrl)) break;
                uint8_t* const place = room.v + st * T::V_UNIT;
                const int key = static_cast<int>(s.k0) + KT * j;
                if (__builtin_expect(klen < KT * (j + 1), 0)) load_end<T>(ctrl, a.status, place, mv, &ctrl->v_full[st], ends++, T::VC * u, s.g, key, klen - KT * j);
                else if (lead) load_unit<T>(ptx::smem_u32(place), mv, &ctrl->v_full[st], T::VC * u, s.g, key);
                __syncwarp();
            }
            if (any_aborted(ctrl)) break;
        }
        if (any_aborted(ctrl)) break;
    }
    if (lead && aborted(ctrl)) {
        landed(ctrl->v_full, nv, T::V_STAGES);
        landed(&ctrl->v_end, ends, 1);
    }
    __syncwarp();
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y, int z, int w) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}
// Pages by four warps, two for the keys and two for the values: lane i of a warp looks up keys i and 32 + i of its half of a tile.  Keys that are
// all there come in boxes of up to 32 tokens of a page; others (the sequence's end, a window's begin, pages that are no multiple of 8) by
// 16-byte copies, zeros where nothing is to be read.  e4m3: into a ring of their own, 32 keys at a time, from where the warp widens them.
template <class T>
__device__ __forceinline__ void load_pages(const Args& a, Ctrl* ctrl, const Room& room, const CUtensorMap* mk, const CUtensorMap* mv) {
    constexpr int ELEM = T::F16 ? 1 : 2;
    const int lane = threadIdx.x & 31, warp = uniform((threadIdx.x >> 5) & 3);
    const bool values = warp >= 2;
    const int half = 64 * (warp & 1);                       // the warp's first key of a tile
    const int pieces = (values ? T::VC : T::KC) * ELEM / 16, units = values ? T::NVU : T::NKU;      // 16-byte pieces of a key in a unit
    // (units of two sizes: powers of two)
    static_assert(T::KC == T::VC || (T::VC == 2 * T::KC && T::KC == 64), "");
    auto over_pieces = [&](int i) { return T::KC == T::VC ? i / (T::KC * ELEM / 16) : i >> ((ELEM == 1 ? 2 : 3) + (values ? 1 : 0)); };
    const uint32_t stages = values ? T::V_STAGES : T::K_STAGES, unit_bytes = values ? T::V_UNIT : T::K_UNIT;
    uint8_t* const ring = values ? room.v : room.k;
    uint64_t* const full = values ? ctrl->v_full : ctrl->k_full;
    uint64_t* const empty = values ? ctrl->v_empty : ctrl->k_empty;
    const CUtensorMap* const map = values ? mv : mk;
    const char* const base = static_cast<const char*>(values ? a.c.v : a.c.k);
    const i64 page_stride = values ? a.c.v_page_stride : a.c.k_page_stride, token_stride = values ? a.c.v_token_stride : a.c.k_token_stride,
              head_stride = values ? a.c.v_head_stride : a.c.k_head_stride;
    uint32_t segs = 0, n = 0, tiles = 0;                    // segments, units, tiles so far
    // e4m3: pieces of work of 32 keys that were fetched into the warp's ring, and those of them that are not widened yet; a bit for each of these,
    // oldest highest, says that it came by 16-byte copies
    constexpr uint32_t RING = T::F16 ? T::RAW_STAGES : 1;
    uint32_t raw = 0, waiting = 0, copied = 0;
    uint8_t* const mine = room.raw + warp * (T::RAW / 4);
    auto widen = [&]() {
        const uint32_t at = raw - waiting, st = at % RING, unit = at >> 1, keys = half + 32 * (at & 1);
        uint64_t* const bar = &ctrl->raw_full[warp][st];
        if ((copied >> (waiting - 1)) & 1) {
            cp_wait<0>();
            __syncwarp();
            if (lane == 0) arrive(bar);                     // (a parity names every other use of the place)
        } else {
            wait_bar(bar, at / RING, ctrl, a.status);
        }
        wait_bar(&empty[unit % stages], unit / stages + 1, ctrl, a.status);
        __syncwarp();
        const uint8_t* const src = mine + st * T::RAW;
        uint8_t* const place = ring + unit % stages * unit_bytes + keys * 128;
        // (all of a unit's loads in flight: 1,508 us for 32,768 cached tokens where four at a time took 1,640)
#pragma unroll 8
        for (int i = 0; i < pieces; ++i) {
            const int flat = i * 32 + lane, key = over_pieces(flat), piece = flat - key * pieces;      // 16 elements
            const uint4 x = *reinterpret_cast<const uint4*>(src + flat * 16);
            uint32_t f[8];
            e4m3_to_f16(x.x, f[0], f[1]), e4m3_to_f16(x.y, f[2], f[3]), e4m3_to_f16(x.z, f[4], f[5]), e4m3_to_f16(x.w, f[6], f[7]);
            // (the second slab's lanes store their halves in the other order: eight lanes then meet every bank once)
            const int c = (piece & 3) * 2, odd = piece >> 2 & 1;
            uint8_t* const dst = place + (piece >> 2) * T::SLAB + key * 128;
            const uint4 lo = make_uint4(f[0], f[1], f[2], f[3]), hi = make_uint4(f[4], f[5], f[6], f[7]);
            *reinterpret_cast<uint4*>(dst + (((c + odd) ^ (key & 7)) << 4)) = odd ? hi : lo;
            *reinterpret_cast<uint4*>(dst + (((c + 1 - odd) ^ (key & 7)) << 4)) = odd ? lo : hi;
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) arrive(&full[unit % stages]);
        --waiting;
    };
    Seg s = {};
    int from = 0, to = 0;                                   // keys that some row of the item sees
    // the page of a key; INT_MIN: not to be read
    auto page_of = [&](int key) {
        if (key < from || key >= to) return INT_MIN;
        return max(a.table[s.k0 + page_number(a, key)], -1);
    };
    for (;;) {
        // (what is still under way is widened before the warp waits for more work)
        while (T::F16 && waiting && !__all_sync(0xffffffffu, ptx::mbar_test_wait(ptx::smem_u32(&ctrl->seg_full[segs % SEGS]), (segs / SEGS) & 1))) widen();
        tiles += s.jb - s.ja;
        if (!next_seg(a, ctrl, segs, s, false)) break;
        from = first_key(a, s.pos, s.klen), to = end_key(a, s.pos + s.ntok - 1, s.klen);
        to = min(to, KT * s.jb);
        int key = KT * s.ja + half + lane;
        int next[2] = {page_of(key), page_of(key + 32)};    // (of the tile after: looked up while this one is fetched)
#pragma unroll 1
        for (int j = s.ja; j < s.jb; ++j, key += KT) {
            const int p[2] = {next[0], next[1]};
            if (j + 1 < s.jb) next[0] = page_of(key + KT), next[1] = page_of(key + KT + 32);
            bool ok[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ok[h] = p[h] >= 0 && p[h] < a.c.num_pages;
                if (!values) {
                    const unsigned bits = __ballot_sync(0xffffffffu, ok[h] || p[h] == INT_MIN);
                    if (lane == 0) reinterpret_cast<uint32_t*>(&ctrl->flags[(tiles + j - s.ja) % FLAGS_AHEAD])[(half >> 5) + h] = bits;
                    if (!ok[h] && p[h] != INT_MIN) raise_bad_index(a.status);
                }
            }
            const int off[2] = {key - page_number(a, key) * a.c.page_size, key + 32 - page_number(a, key + 32) * a.c.page_size};
            // n 64 keys, or 32 at a time (e4m3)
            constexpr int STEP = T::F16 ? 1 : 2;
#pragma unroll 1
            for (int u = 0; u < units; ++u) {
                if (!T::F16) wait_bar(&empty[n % stages], n / stages + 1, ctrl, a.status);
#pragma unroll 1
                for (int h = 0; h < 2; h += STEP) {
                    const bool boxes = a.maps && __all_sync(0xffffffffu, T::F16 ? (h ? ok[1] : ok[0]) : ok[0] && ok[1]);
                    const uint32_t st = T::F16 ? raw % RING : n % stages;
                    const uint32_t place = T::F16 ? ptx::smem_u32(mine) + st * T::RAW : ptx::smem_u32(ring) + st * unit_bytes + half * 128;
                    uint64_t* const bar = T::F16 ? &ctrl->raw_full[warp][st] : &full[st];
                    if (boxes) {
                        // (8-bit: rows of a unit as they are, one behind the other; else slabs of 64 columns)
                        const int slabs = T::F16 ? 1 : (pieces + 7) / 8, pitch = T::F16 ? pieces * 16 : 128;
                        if (lane == 0) ptx::mbar_arrive_expect_tx(ptx::smem_u32(bar), slabs * 32 * STEP * pitch);
                        __syncwarp();
                        const int x = slabs == 2 ? lane & 1 : 0, first = (slabs == 2 ? lane >> 1 : lane) * a.box;      // slab; of the keys
                        const int p0 = __shfl_sync(0xffffffffu, p[0], first & 31), p1 = __shfl_sync(0xffffffffu, p[1], first & 31);
                        const int o0 = __shfl_sync(0xffffffffu, off[0], first & 31), o1 = __shfl_sync(0xffffffffu, off[1], first & 31);
                        const bool second = h + (first >> 5) != 0;
                        if (first < 32 * STEP)
                            tma_load_4d(place + x * T::SLAB + first * pitch, map, ptx::smem_u32(bar), u * pieces * (16 / ELEM) + 64 * x, s.g, second ? o1 : o0, second ? p1 : p0);
                    } else {
#pragma unroll 1
                        for (int g = h; g < h + STEP; ++g) {
                            const char* row = nullptr;      // of the lane's key
                            if (g ? ok[1] : ok[0])
                                row = base + ((g ? p[1] : p[0]) * page_stride + (g ? off[1] : off[0]) * token_stride + s.g * head_stride) * ELEM + u * pieces * 16;
#pragma unroll 4
                            for (int i = 0; i < pieces; ++i) {      // 32 keys' pieces, 32 at a time
                                const int flat = i * 32 + lane, k = over_pieces(flat), piece = flat - k * pieces;
                                const char* const src = reinterpret_cast<const char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), k));
                                const uint32_t dst = T::F16 ? place + flat * 16 : place + (piece >> 3) * T::SLAB + (32 * g + k) * 128 + (((piece & 7) ^ (k & 7)) << 4);
                                cp_async16(dst, src ? src + piece * 16 : base, src != nullptr);
                            }
                        }
                        cp_commit();
                        if (!T::F16) {
                            cp_wait<0>();
                            ptx::fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) arrive(bar);
                        }
                    }
                    if (T::F16) {
                        copied = copied << 1 | (boxes ? 0u : 1u), ++waiting, ++raw;
                        if (waiting == RING) widen();
                    }
                }
                ++n;
            }
            if (any_aborted(ctrl)) break;
        }
        if (any_aborted(ctrl)) break;
    }
    while (T::F16 && waiting && !any_aborted(ctrl)) widen();
    cp_wait<0>();
    if (lane == 0 && aborted(ctrl)) {
        if (T::F16) landed(ctrl->raw_full[warp], raw, RING);
        else landed(full, n, stages);
    }
    __syncwarp();
}

// ---------------------------------------------------------------------------------------------------------- products
// One warp issues the scores' products, another the weighted sums': neither waits for what the other's operands wait for.  The whole warp
// walks through its loop, so that addresses and descriptors are the same in all lanes as the compiler sees it (a tensor instruction
// takes them from uniform registers); one lane issues.

__device__ __forceinline__ void drain(Ctrl* ctrl, int who) {      // products under way end before shared and tensor memory are given up
    ptx::umma_commit(ptx::smem_u32(&ctrl->drained[who]));
    const uint64_t t0 = ptx::globaltimer_ns();
    while (!ptx::mbar_try_wait(ptx::smem_u32(&ctrl->drained[who]), 0) && ptx::globaltimer_ns() - t0 < WAIT_LIMIT_NS / 4) {}
}

// S = Q K^T for the row tiles in turn, all into one place of tensor memory, which is free again as soon as a row tile's threads have
// their scores in registers: the next scores are there when they are done with these.
template <class T>
__device__ __forceinline__ void scores_warp(const Args& a, Ctrl* ctrl, uint32_t q_smem, uint32_t k_smem, uint32_t tmem) {
    const bool lead = ptx::elect_one();
    uint32_t segs = 0, n = 0, q0_count = 0, q1_count = 0, uses = 0;      // n: units of keys
    Seg s = {};
    while (next_seg(a, ctrl, segs, s, false)) {
        const int ja = uniform(s.ja), steps = uniform(s.jb) - ja;
        if (steps == 0) continue;
        const uint32_t idesc = (ptx::umma_idesc_bf16(MT, KT) & ~(T::F16 ? ptx::UMMA_IDESC_F16 : 0u)) | (uniform(s.negative) ? ptx::UMMA_IDESC_NEGATE_B : 0u);
        const bool dual = uniform(is_dual<T>(a, s));
        int ra0 = 0, rb0 = steps, ra1 = 0, rb1 = 0;
        if (dual) {
            range_of(a, s, true, 0, ra0, rb0), range_of(a, s, true, 1, ra1, rb1);
            ra0 = uniform(ra0) - ja, rb0 = uniform(rb0) - ja, ra1 = uniform(ra1) - ja, rb1 = uniform(rb1) - ja;
        }
        auto product = [&](int qt, int t, bool loaded) {      // loaded: the tile's keys have been waited for
            if (uses) wait_bar(&ctrl->s_free, uses - 1, ctrl, a.status);
            ++uses;
            ptx::tc_fence_after();
#pragma unroll
            for (int u = 0; u < T::NKU; ++u) {
                const uint32_t st = (n + u) % T::K_STAGES;
                if (!loaded) {
                    wait_bar(&ctrl->k_full[st], (n + u) / T::K_STAGES, ctrl, a.status);
                    ptx::tc_fence_after();
                }
                const uint32_t qa = ptx::umma_desc_lo_sw128(q_smem + qt * T::Q_TILE + u * T::K_UNIT);
                const uint32_t ka = ptx::umma_desc_lo_sw128(k_smem + st * T::K_UNIT);
                if (lead) {
#pragma unroll
                    for (int k = 0; k < T::KC / 16; ++k) {
                        const uint32_t add = (k >> 2) * (T::SLAB >> 4) + (k & 3) * 2;
                        if (u == 0 && k == 0) ptx::umma_bf16_lohi<false>(tmem + S_COL, qa + add, ptx::UMMA_DESC_HI_SW128, ka + add, ptx::UMMA_DESC_HI_SW128, idesc);
                        else ptx::umma_bf16_lohi<true>(tmem + S_COL, qa + add, ptx::UMMA_DESC_HI_SW128, ka + add, ptx::UMMA_DESC_HI_SW128, idesc);
                    }
                    if (T::NKU > 1) ptx::umma_commit(ptx::smem_u32(&ctrl->k_empty[st]));
                }
            }
            if (lead) ptx::umma_commit(ptx::smem_u32(&ctrl->s_full[t]));
        };
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
            if (any_aborted(ctrl)) break;
            bool loaded = false;
#pragma unroll 1
            for (int t = 0; t < (dual ? 2 : 1); ++t) {
                const int ra = t ? ra1 : ra0, rb = t ? rb1 : rb0;
                if (i < ra || i >= rb) continue;
                if (i == ra) {
                    wait_bar(T::F16 ? &ctrl->q_conv[t] : &ctrl->q_full[t], t ? q1_count : q0_count, ctrl, a.status);
                    if (t) ++q1_count;
                    else ++q0_count;
                }
                product(t, dual ? t : T::TILES == 2 ? i & 1 : 0, loaded);
                loaded = true;
                if (i == rb - 1 && lead) ptx::umma_commit(ptx::smem_u32(&ctrl->q_empty[t]));
            }
            if (!loaded) wait_bar(&ctrl->k_full[n % T::K_STAGES], n / T::K_STAGES, ctrl, a.status);      // (no row tile sees them)
            if (T::NKU == 1 && lead) ptx::umma_commit(ptx::smem_u32(&ctrl->k_empty[n % T::K_STAGES]));
            n += T::NKU;
        }
        if (any_aborted(ctrl)) break;
    }
    if (lead && aborted(ctrl)) drain(ctrl, 0);
    __syncwarp();
}

// O += P V
template <class T>
__device__ __forceinline__ void sums_warp(const Args& a, Ctrl* ctrl, uint32_t v_smem, uint32_t tmem) {
    constexpr uint32_t idesc = (ptx::umma_idesc_bf16(MT, T::VC) & ~(T::F16 ? ptx::UMMA_IDESC_F16 : 0u)) | ptx::UMMA_IDESC_B_MN_MAJOR;
    const bool lead = ptx::elect_one();
    uint32_t segs = 0, n = 0, p0_count = 0, p1_count = 0, o0_uses = 0, o1_uses = 0;      // n: units of values
    Seg s = {};
    while (next_seg(a, ctrl, segs, s, false)) {
        const int ja = uniform(s.ja), steps = uniform(s.jb) - ja;
        if (steps == 0) continue;
        const bool dual = uniform(is_dual<T>(a, s));
        int ra0 = 0, rb0 = steps, ra1 = 0, rb1 = 0;
        if (dual) {
            range_of(a, s, true, 0, ra0, rb0), range_of(a, s, true, 1, ra1, rb1);
            ra0 = uniform(ra0) - ja, rb0 = uniform(rb0) - ja, ra1 = uniform(ra1) - ja, rb1 = uniform(rb1) - ja;
        }
        auto product = [&](int pb, int ob, bool fresh, bool loaded) {
            if (fresh) {                       // the rows of the segment before have been read
                const uint32_t uses = ob ? o1_uses : o0_uses;
                if (uses) wait_bar(&ctrl->o_free[ob], uses - 1, ctrl, a.status);
                if (ob) ++o1_uses;
                else ++o0_uses;
            }
            wait_bar(&ctrl->p_ready[pb], pb ? p1_count : p0_count, ctrl, a.status);
            if (pb) ++p1_count;
            else ++p0_count;
            ptx::tc_fence_after();
#pragma unroll
            for (int u = 0; u < T::NVU; ++u) {
                const uint32_t st = (n + u) % T::V_STAGES;
                if (!loaded) {
                    wait_bar(&ctrl->v_full[st], (n + u) / T::V_STAGES, ctrl, a.status);
                    ptx::tc_fence_after();
                }
                // values as they lie there: 64-column slabs (leading offset), groups of eight keys 1024 bytes apart
                const uint32_t lo = (((v_smem + st * T::V_UNIT) & 0x3FFFFu) >> 4) | ((T::SLAB >> 4) << 16);
                if (lead) {
#pragma unroll
                    for (int k = 0; k < KT / 16; ++k)
                        ptx::umma_f16_ta(tmem + O_COL + ob * KT + u * T::VC, tmem + p_col(pb) + k * 8, lo + k * (2048u >> 4), ptx::UMMA_DESC_HI_SW128, idesc, !fresh || k > 0);
                    if (T::NVU > 1) ptx::umma_commit(ptx::smem_u32(&ctrl->v_empty[st]));
                }
            }
            if (lead) ptx::umma_commit(ptx::smem_u32(&ctrl->o_done[pb]));
        };
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
            if (any_aborted(ctrl)) break;
            bool loaded = false;
#pragma unroll 1
            for (int t = 0; t < (dual ? 2 : 1); ++t) {
                const int ra = t ? ra1 : ra0, rb = t ? rb1 : rb0;
                if (i < ra || i >= rb) continue;
                const int at = dual ? t : i & 1;
                product(at, T::TILES == 2 ? at : 0, dual ? i == ra : i < T::TILES, loaded);
                loaded = true;
            }
            if (!loaded) wait_bar(&ctrl->v_full[n % T::V_STAGES], n / T::V_STAGES, ctrl, a.status);
            if (T::NVU == 1 && lead) ptx::umma_commit(ptx::smem_u32(&ctrl->v_empty[n % T::V_STAGES]));
            n += T::NVU;
        }
        if (any_aborted(ctrl)) break;
    }
    if (lead && aborted(ctrl)) drain(ctrl, 1);
    __syncwarp();
}

template <class T>
__global__ void __launch_bounds__(T::THREADS, 1)
attention_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                 const __grid_constant__ Args a) {
    extern __shared__ uint8_t smem_raw[];
    Room room;
    room.q = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    room.k = room.q + T::Q_BYTES, room.v = room.k + T::K_BYTES, room.raw = room.v + T::V_BYTES;
    Ctrl* const ctrl = reinterpret_cast<Ctrl*>(room.raw + T::RAW_STAGES * T::RAW);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        auto init = [](uint64_t* bar, int n) { ptx::mbar_init(ptx::smem_u32(bar), n); };
        for (int i = 0; i < SEGS; ++i) {
            init(&ctrl->seg_full[i], 1);
            init(&ctrl->seg_empty[i], 2 + T::WARPS_SM + (T::PAGED ? T::WARPS_LD : 1));
        }
        for (int i = 0; i < 2; ++i) {
            init(&ctrl->q_full[i], 1), init(&ctrl->q_empty[i], T::q_readers(i)), init(&ctrl->q_conv[i], 4);
            init(&ctrl->s_full[i], 1), init(&ctrl->p_ready[i], 4), init(&ctrl->o_done[i], 1), init(&ctrl->o_free[i], 4);
        }
        for (int i = 0; i < T::K_STAGES; ++i) init(&ctrl->k_full[i], T::F16 ? 4 : T::PAGED ? 2 : 1), init(&ctrl->k_empty[i], 1);
        for (int i = 0; i < T::V_STAGES; ++i) init(&ctrl->v_full[i], T::F16 ? 4 : T::PAGED ? 2 : 1), init(&ctrl->v_empty[i], 1);
        if (T::F16)
            for (int i = 0; i < 12; ++i) init(&ctrl->raw_full[i / 3][i % 3], 1);
        init(&ctrl->v_end, 1), init(&ctrl->x_full, 4), init(&ctrl->x_empty, 4), init(&ctrl->s_free, 4), init(&ctrl->drained[0], 1), init(&ctrl->drained[1], 1);
        ctrl->abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&mq);
        if (!T::PAGED || a.maps) ptx::prefetch_tensormap(&mk), ptx::prefetch_tensormap(&mv);
    }
    if (warp == T::WARP_MMA) {
        ptx::tmem_alloc(ptx::smem_u32(&ctrl->tmem), 512);
        ptx::tmem_relinquish();
    }
    ptx::grid_dep_wait();
    if (a.entries > 32) {      // the list's length: every warp adds up a stretch of entries (of few, the scheduler does it all)
        const int stretch = stretch_of<T>(a), e0 = min(stretch * warp, a.entries), e1 = min(e0 + stretch, a.entries);
        i64 sum = 0;
#pragma unroll 1
        for (int e = e0; e < e1; e += 32) {
            Entry en = {};
            if (e + lane < e1) en = entry_of<T::PAGED>(a, e + lane, blockIdx.x == 0);
            sum += cost_before<T>(a, en.qlen, en.klen, blocks_of<T::TILES>(a, en.qlen));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) ctrl->sums[warp] = sum;
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ctrl->tmem;

    if (warp >= T::WARP_SCHED) {
        if (T::SPLIT_REGS) ptx::setmaxnreg_dec<T::REGS_AUX>();
        if (warp == T::WARP_SCHED) {
            schedule<T>(a, ctrl, room, &mq, &mk);
        } else if (warp == T::WARP_VALUES) {
            if (!T::PAGED) load_values<T>(a, ctrl, room, &mv);
        } else if (warp == T::WARP_MMA) {
            scores_warp<T>(a, ctrl, ptx::smem_u32(room.q), ptx::smem_u32(room.k), tmem);
        } else {
            sums_warp<T>(a, ctrl, ptx::smem_u32(room.v), tmem);
        }
    } else if (T::PAGED && warp >= T::WARPS_SM) {
        if constexpr (T::SPLIT_REGS) {
            if constexpr (T::REGS_LD < T::REGS_START) ptx::setmaxnreg_dec<T::REGS_LD>();
            else ptx::setmaxnreg_inc<T::REGS_LD>();
        }
        if constexpr (T::PAGED) load_pages<T>(a, ctrl, room, &mk, &mv);
    } else {
        if (T::SPLIT_REGS) ptx::setmaxnreg_inc<T::REGS_SM>();
        softmax_rows<T>(a, ctrl, room, tmem, warp >> 2);
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == T::WARP_MMA) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

// ------------------------------------------------------------------------------------------------------------- join
// out = sum O_i 2^(m_i - m) / sum l_i 2^(m_i - m), m = max m_i, over the parts of an item, in order.  A warp to a row, or, for few rows of many
// parts, a block to a row (its warps share the parts).  Sums lie 2^8 lower (MOST_CTAS parts at most), so that those of finite parts are finite.
static_assert(MOST_CTAS <= 256, "");
constexpr int JOIN_WARPS = 8, JOIN_BATCH = 4, JOIN_SLICES = 16;      // SLICES: blocks to an item
template <int D, int ROWS, int TILES>
__global__ void __launch_bounds__(32 * JOIN_WARPS)
attention_join_kernel(const Args a) {
    constexpr int V = (D + 127) / 128;           // float4 of a lane
    constexpr i64 PART = static_cast<i64>(ROWS) * (D + 2);
    __shared__ float4 accs[JOIN_WARPS][V][32];
    __shared__ float2 mls[JOIN_WARPS];
    ptx::grid_dep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.x / JOIN_SLICES, slice = blockIdx.x % JOIN_SLICES;
    const Split e = a.splits[c0];
    if (!e.valid) return;
    const int rows = e.ntok * e.heads, parts = e.c1 - c0 + 1;
    // rounds of loads, one behind the other: a row to a warp, or to a block
    const bool many = (rows + JOIN_SLICES - 1) / JOIN_SLICES * ((parts + JOIN_WARPS * JOIN_BATCH - 1) / (JOIN_WARPS * JOIN_BATCH) + 1) <
                      (rows + JOIN_SLICES * JOIN_WARPS - 1) / (JOIN_SLICES * JOIN_WARPS) * ((parts + JOIN_BATCH - 1) / JOIN_BATCH);
    const float vs = a.c.type == CAKE_KV_E4M3 && a.c.v_scale ? a.c.v_scale[e.g] : 1.f;
    const bool dual = TILES == 2 && e.ntok > a.tokens;
    for (int i = many ? slice : slice * JOIN_WARPS + warp; i < rows; i += many ? JOIN_SLICES : JOIN_SLICES * JOIN_WARPS) {
        const int tok = i / e.heads, h = i - tok * e.heads;
        const int t = dual && tok >= a.tokens ? 1 : 0;
        const int row = t * MT + (tok - t * a.tokens) * a.heads + h;
        float m = NEG_INF, l = 0.f;
        float4 acc[V];
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](float pm, float pl, const float4 (&u)[V], float down) {
            const float up = fmaxf(m, pm), from = up == NEG_INF ? 0.f : up;
            const float f = ex2(m - from), g = ex2(pm - from) * down;
            m = up, l = l * f + pl * g;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                acc[v].x = acc[v].x * f + u[v].x * g, acc[v].y = acc[v].y * f + u[v].y * g;
                acc[v].z = acc[v].z * f + u[v].z * g, acc[v].w = acc[v].w * f + u[v].w * g;
            }
        };
        const int step = many ? JOIN_WARPS : 1;
        constexpr int BATCH = JOIN_BATCH;
        for (int c = c0 + (many ? warp : 0); c <= e.c1; c += BATCH * step) {
            float4 u[BATCH][V];
            float2 ml[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int cb = c + b * step;
                ml[b] = make_float2(NEG_INF, 0.f);
#pragma unroll
                for (int v = 0; v < V; ++v) u[b][v] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (cb <= e.c1) {
                    const float* p = a.parts + (2 * cb + (cb == c0 ? 1 : 0)) * PART;
                    ml[b] = *reinterpret_cast<const float2*>(p + static_cast<i64>(ROWS) * D + 2 * row);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (128 * v + 4 * lane < D) u[b][v] = *reinterpret_cast<const float4*>(p + static_cast<i64>(row) * D + 128 * v + 4 * lane);
                }
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) add(ml[b].x, ml[b].y, u[b], 1.f / 256.f);
        }
        if (many) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v) accs[warp][v][lane] = acc[v];
            if (lane == 0) mls[warp] = make_float2(m, l);
            __syncthreads();
            if (warp != 0) continue;
            for (int w = 1; w < JOIN_WARPS; ++w) {
                float4 u[V];
#pragma unroll
                for (int v = 0; v < V; ++v) u[v] = accs[w][v][lane];
                add(mls[w].x, mls[w].y, u, 1.f);
            }
        }
        const float f = l == 0.f ? 0.f : vs / l;
        const i64 out_row = (e.tok + tok) * a.Hq + e.head0 + h;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int d = 128 * v + 4 * lane;
            if (d >= D) continue;
            const uint2 w = make_uint2(pack_bf16(acc[v].x * f, acc[v].y * f), pack_bf16(acc[v].z * f, acc[v].w * f));
            cake_bf16* const to = a.out + out_row * D + d;
            *reinterpret_cast<uint2*>(to) = w;
        }
        if (a.lse && lane == 0) a.lse[out_row] = l == 0.f ? NEG_INF : (m + log2f(l * 256.f)) * LN2;
    }
}

// ------------------------------------------------------------------------------------------------------------- host
struct Maps {
    CUtensorMap q, k, v;
};
inline int ctas_of(const DeviceInfo& di) { return di.sm_count < MOST_CTAS ? di.sm_count : MOST_CTAS; }
int launch_64(const Args& a, const Maps& m, int kind, const DeviceInfo& di, cudaStream_t s);
int launch_96(const Args& a, const Maps& m, int kind, const DeviceInfo& di, cudaStream_t s);
int launch_128(const Args& a, const Maps& m, int kind, const DeviceInfo& di, cudaStream_t s);
int launch_256(const Args& a, const Maps& m, int kind, const DeviceInfo& di, cudaStream_t s);

template <class T>
int launch(const Args& a, const Maps& m, const DeviceInfo& di, cudaStream_t s) {
    constexpr uint32_t SMEM = smem_bytes<T>();
    static_assert(SMEM <= 227 * 1024, "");
    static PerDevice ready;
    const bool ok = ready.get(di.device, [] {
        // the split of the registers counts on what the block starts with
        cudaFuncAttributes at;
        if (cudaFuncGetAttributes(&at, attention_kernel<T>) != cudaSuccess) {
            cudaGetLastError();
            return 0;
        }
        const int sum = 128 * (T::TILES * T::REGS_SM + (T::PAGED ? T::REGS_LD : 0) + T::REGS_AUX);
        if (T::SPLIT_REGS && at.numRegs * T::THREADS < sum) return 0;
        return allow_smem(attention_kernel<T>, SMEM);
    });
    if (!ok) return CAKE_ERR_CUDA;
    const int ctas = ctas_of(di);
    if (launch_early(attention_kernel<T>, dim3(ctas), dim3(T::THREADS), SMEM, s, m.q, m.k, m.v, a) != cudaSuccess) return CAKE_ERR_CUDA;
    if (!a.cuts) return CAKE_OK;
    return launch_early(attention_join_kernel<T::D, T::PART_ROWS, T::TILES>, dim3(ctas * JOIN_SLICES), dim3(32 * JOIN_WARPS), 0, s, a) == cudaSuccess
               ? CAKE_OK : CAKE_ERR_CUDA;
}
template <int D>
int launch_kind(const Args& a, const Maps& m, int kind, const DeviceInfo& di, cudaStream_t s) {
    switch (kind) {
        case PACKED: return launch<Traits<D, PACKED>>(a, m, di, s);
        case PAGED_BF16: return launch<Traits<D, PAGED_BF16>>(a, m, di, s);
        default: return launch<Traits<D, PAGED_E4M3>>(a, m, di, s);
    }
}

}  // namespace attn
}  // namespace serving
}  // namespace cake
