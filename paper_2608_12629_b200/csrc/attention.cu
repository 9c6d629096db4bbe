// Entry points of the attention of many query tokens (attention.cuh): packed prompts, and chunks over a paged cache.
#include <math.h>

#include "attention.cuh"

namespace cake {
namespace serving {
namespace attn {
namespace {

static_assert(kHeaderBytes % 256 == 0, "parts are written by 32 bytes");
constexpr size_t kSplitBytes = (MOST_CTAS * sizeof(Split) + 255) / 256 * 256;
size_t part_floats(int D) { return static_cast<size_t>(D == 256 ? MT : 2 * MT) * (D + 2); }
bool supported(int D) { return D == 64 || D == 96 || D == 128 || D == 256; }

// bf16 [tokens][heads][D]: box of 64 columns x `box_heads` heads x `box_tokens` tokens, 128-byte swizzle, zeros outside
int make_map(CUtensorMap* m, const void* base, int D, int heads, i64 head_stride, i64 tokens, i64 stride, int box_heads, int box_tokens) {
    // (the stride of a dimension of one element says nothing)
    if (heads == 1) head_stride = D;
    if (tokens == 1) stride = static_cast<i64>(D) * heads;
    return make_tmap_heads(m, base, D, heads, head_stride * 2, tokens, stride * 2, box_heads, box_tokens);
}

// boxes of the columns that a unit of loads has (bf16: 64, swizzled; e4m3: all of the unit's) x `box` tokens of a page
int make_map_pages(CUtensorMap* m, const void* base, const cake_paged_cache& c, i64 head, i64 token, i64 page, int columns, int box) {
    if (c.Hkv == 1) head = c.D;
    if (c.page_size == 1) token = c.D;
    if (c.num_pages == 1) page = c.D;
    if (head < c.D || token < c.D || page < c.D) return CAKE_ERR_UNSUPPORTED;      // (strides of zero: expanded tensors)
    const int size = c.type == CAKE_KV_BF16 ? 2 : 1;
    return make_tmap_pages(m, base, c.D, c.Hkv, head * size, c.page_size, token * size, c.num_pages, page * size, columns, box, size == 1);
}

bool strides_ok(int D, i64 heads, i64 head_stride, i64 tokens, i64 stride) {
    return (heads == 1 || head_stride >= D) && (tokens <= 1 || stride >= D);
}
bool strides_aligned(i64 heads, i64 head_stride, i64 tokens, i64 stride) {
    return (heads == 1 || head_stride % 8 == 0) && (tokens <= 1 || stride % 8 == 0);
}

int check_heads(int Hq, int Hkv, int D) {
    if (Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return CAKE_ERR_SHAPE;
    return supported(D) ? CAKE_OK : CAKE_ERR_UNSUPPORTED;
}

// e / d for e < 2^31: mulhi(e, ceil(2^(31 + k) / d)) >> (k - 1) with 2^k >= d; 0 for d = 1
void division(uint32_t d, uint32_t* mul, uint32_t* shift) {
    uint32_t k = 0;
    while ((1ull << k) < d) ++k;
    *mul = d == 1 ? 0 : static_cast<uint32_t>(((1ull << (31 + k)) + d - 1) / d);
    *shift = d == 1 ? 0 : k - 1;
}

// what both entry points share: everything of a but the keys
int prepare(Args& a, Maps& maps, i64 B, int D, float scale, void* ws, size_t ws_bytes, DeviceInfo* di) {
    if (!a.q || !a.starts || !a.out) return CAKE_ERR_NULL;
    if (!aligned(a.q, 16) || !strides_aligned(a.Hq, a.q_head_stride, a.T, a.q_stride)) return CAKE_ERR_ALIGN;
    if (!aligned(a.out, 16) || !aligned(a.lse, 4) || !aligned(a.starts, 4)) return CAKE_ERR_ALIGN;
    if (ws_bytes < kHeaderBytes + kSplitBytes + 2 * MOST_CTAS * part_floats(D) * 4) return CAKE_ERR_WORKSPACE;
    const int rc = current_device_info(di);
    if (rc != CAKE_OK) return rc;
    if (di->cc_major != 10) return CAKE_ERR_DEVICE;
    a.G = a.Hq / a.Hkv;
    a.runs = (a.G + MT - 1) / MT;
    a.heads = (a.G + a.runs - 1) / a.runs;
    a.tokens = MT / a.heads;
    if (B > INT_MAX / 64 / (static_cast<i64>(a.Hkv) * a.runs)) return CAKE_ERR_SHAPE;
    a.entries = static_cast<int>(B) * a.Hkv * a.runs;
    division(static_cast<uint32_t>(a.Hkv) * a.runs, &a.per_mul, &a.per_shift);
    a.share_mul = ~0ull / ctas_of(*di);
    a.negative = scale < 0.f;
    a.wide = aligned(a.out, 32);
    a.scale_log2 = static_cast<float>(fabs(static_cast<double>(scale)) * 1.4426950408889634);
    a.status = static_cast<int*>(ws);
    a.splits = reinterpret_cast<Split*>(static_cast<char*>(ws) + kHeaderBytes);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + kHeaderBytes + kSplitBytes);
    return make_map(&maps.q, a.q, D, a.Hq, a.q_head_stride, a.T, a.q_stride, a.heads, a.tokens);
}

// Whether an item can have so many tiles of keys that its share may be cut (`most`: keys of a sequence).  If not, nothing has to be joined: one launch
// (a prompt of 201 tokens 17.3 us with the join, 15.8 without)
bool may_cut(const Args& a, int D, i64 most) {
    const i64 tokens = static_cast<i64>(D == 256 ? 1 : 2) * a.tokens;
    const i64 tiles = a.window > 0 && a.window + tokens < most ? (a.window + tokens) / KT + 2 : (most + KT - 1) / KT;
    return tiles >= 2 * SNAP;
}

int launch_any(const Args& a, const Maps& m, int D, int kind, const DeviceInfo& di, cudaStream_t s) {
    switch (D) {
        case 64: return launch_64(a, m, kind, di, s);
        case 96: return launch_96(a, m, kind, di, s);
        case 128: return launch_128(a, m, kind, di, s);
        default: return launch_256(a, m, kind, di, s);
    }
}

}  // namespace
}  // namespace attn
}  // namespace serving
}  // namespace cake

using namespace cake;
using namespace cake::serving;
using namespace cake::serving::attn;

extern "C" {

int cake_attention_workspace_bytes(int Hq, int Hkv, int D, size_t* out_bytes) {
    if (!out_bytes) return CAKE_ERR_NULL;
    const int rc = check_heads(Hq, Hkv, D);
    if (rc != CAKE_OK) return rc;
    *out_bytes = kHeaderBytes + kSplitBytes + 2 * MOST_CTAS * part_floats(D) * 4;
    return CAKE_OK;
}

int cake_prompt_attention(const cake_bf16* q, long long q_stride, long long q_head_stride, const cake_bf16* k, long long k_stride,
                          long long k_head_stride, const cake_bf16* v, long long v_stride, long long v_head_stride, const int* starts,
                          const int* k_starts, long long B, long long T, long long Tk, int Hq, int Hkv, int D, float scale, int window,
                          cake_bf16* out, float* out_lse, void* ws, size_t ws_bytes, cake_stream_t stream, unsigned flags) {
    int rc = check_heads(Hq, Hkv, D);
    if (rc != CAKE_OK) return rc;
    if ((flags & ~CAKE_ATTENTION_CAUSAL) != 0 || (window > 0 && !(flags & CAKE_ATTENTION_CAUSAL))) return CAKE_ERR_UNSUPPORTED;
    if (B < 0 || T < 0 || Tk < 0 || B > INT_MAX - 1 || T > INT_MAX - 1024 || Tk > INT_MAX - 1024 || window < 0) return CAKE_ERR_SHAPE;
    if (!strides_ok(D, Hq, q_head_stride, T, q_stride) || !strides_ok(D, Hkv, k_head_stride, Tk, k_stride) ||
        !strides_ok(D, Hkv, v_head_stride, Tk, v_stride))
        return CAKE_ERR_SHAPE;
    if (!ws) return CAKE_ERR_NULL;
    if (!aligned(ws, 256)) return CAKE_ERR_ALIGN;
    if (B == 0 || T == 0) return CAKE_OK;
    if (Tk > 0 && (!k || !v)) return CAKE_ERR_NULL;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_starts, 4) || !strides_aligned(Hkv, k_head_stride, Tk, k_stride) ||
        !strides_aligned(Hkv, v_head_stride, Tk, v_stride))
        return CAKE_ERR_ALIGN;
    Args a = {};
    Maps maps;
    DeviceInfo di;
    a.q = q, a.k = k, a.v = v, a.starts = starts, a.k_starts = k_starts ? k_starts : starts, a.out = out, a.lse = out_lse;
    a.T = T, a.Tk = Tk, a.q_stride = q_stride, a.q_head_stride = q_head_stride, a.k_stride = k_stride, a.k_head_stride = k_head_stride;
    a.v_stride = v_stride, a.v_head_stride = v_head_stride;
    a.Hq = Hq, a.Hkv = Hkv, a.window = window, a.causal = flags & CAKE_ATTENTION_CAUSAL;
    rc = prepare(a, maps, B, D, scale, ws, ws_bytes, &di);
    if (rc != CAKE_OK) return rc;
    a.cuts = may_cut(a, D, Tk);
    if (Tk == 0) {      // (no keys at all: nothing is loaded, any map will do)
        maps.k = maps.v = maps.q;
    } else {
        rc = make_map(&maps.k, k, D, Hkv, k_head_stride, Tk, k_stride, 1, KT);
        if (rc != CAKE_OK) return rc;
        rc = make_map(&maps.v, v, D, Hkv, v_head_stride, Tk, v_stride, 1, KT);
        if (rc != CAKE_OK) return rc;
    }
    return launch_any(a, maps, D, PACKED, di, reinterpret_cast<cudaStream_t>(stream));
}

int cake_paged_chunk(const cake_bf16* q, long long q_stride, long long q_head_stride, const cake_paged_cache* cache,
                     const int* page_table, long long table_stride, long long table_head_stride, int max_pages, const int* seq_lens,
                     long long lens_stride, long long lens_head_stride, const int* starts, long long B, long long T, int Hq, float scale,
                     int window, cake_bf16* out, float* out_lse, void* ws, size_t ws_bytes, cake_stream_t stream) {
    int rc = check_cache(cache);
    if (rc != CAKE_OK) return rc;
    rc = check_heads(Hq, cache->Hkv, cache->D);
    if (rc != CAKE_OK) return rc;
    if (B < 0 || T < 0 || B > INT_MAX - 1 || T > INT_MAX - 1024 || window < 0 || max_pages < 0 ||
        max_pages > (INT_MAX - 2 * KT) / cache->page_size)
        return CAKE_ERR_SHAPE;
    if (table_stride < 0 || table_head_stride < 0 || lens_stride < 0 || lens_head_stride < 0) return CAKE_ERR_SHAPE;
    if (!strides_ok(cache->D, Hq, q_head_stride, T, q_stride)) return CAKE_ERR_SHAPE;
    if (!ws) return CAKE_ERR_NULL;
    if (!aligned(ws, 256)) return CAKE_ERR_ALIGN;
    if (B == 0 || T == 0) return CAKE_OK;
    if (!page_table || !seq_lens) return CAKE_ERR_NULL;
    if (!aligned(page_table, 4) || !aligned(seq_lens, 4)) return CAKE_ERR_ALIGN;
    Args a = {};
    Maps maps;
    DeviceInfo di;
    a.c = *cache;
    a.q = q, a.starts = starts, a.table = page_table, a.lens = seq_lens, a.out = out, a.lse = out_lse;
    a.T = T, a.q_stride = q_stride, a.q_head_stride = q_head_stride, a.table_stride = table_stride, a.table_head_stride = table_head_stride;
    a.lens_stride = lens_stride, a.lens_head_stride = lens_head_stride, a.max_pages = max_pages;
    a.Hq = Hq, a.Hkv = cache->Hkv, a.window = window, a.causal = true;
    rc = prepare(a, maps, B, cache->D, scale, ws, ws_bytes, &di);
    if (rc != CAKE_OK) return rc;
    a.cuts = may_cut(a, cache->D, static_cast<i64>(max_pages) * cache->page_size);
    division(static_cast<uint32_t>(cache->page_size), &a.page_mul, &a.page_shift);
    // Pages come in boxes where a warp's 32 keys are whole boxes of a page: 8, 16 or 32 tokens, or 32 of a page of several times that
    const cake_paged_cache& c = *cache;
    a.box = c.page_size < 32 ? c.page_size : 32;
    const bool bytes = c.type == CAKE_KV_E4M3;
    const int columns = bytes ? (c.D == 256 ? 128 : c.D) : 64;
    a.maps = (c.page_size % 32 == 0 || c.page_size == 16 || c.page_size == 8) &&
             make_map_pages(&maps.k, c.k, c, c.k_head_stride, c.k_token_stride, c.k_page_stride, columns, a.box) == CAKE_OK &&
             make_map_pages(&maps.v, c.v, c, c.v_head_stride, c.v_token_stride, c.v_page_stride, columns, a.box) == CAKE_OK;
    if (!a.maps) maps.k = maps.v = maps.q;      // (not used)
    return launch_any(a, maps, cache->D, cache->type == CAKE_KV_E4M3 ? PAGED_E4M3 : PAGED_BF16, di, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
