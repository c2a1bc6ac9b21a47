// Host side of the cache calls: argument checks, how attention is laid out, launches.  Included by srs.hip behind what it uses of it (the
// context, the device guard, the limits); the calls are documented in include/srs.h.
#pragma once
#include "attention_kernels.hpp"
#include "cache_kernels.hpp"

#include <cmath>

namespace {
uint32_t elem_bytes(int dtype) { return dtype == SRS_BF16 || dtype == SRS_FP16 ? 2u : dtype == SRS_FP32 ? 4u : 0u; }

bool stride_ok(int64_t s) { return s >= -(1ll << 40) && s <= (1ll << 40); }

// A launch has below 2^32 threads.
bool grid_ok(uint64_t workgroups, uint32_t threads) { return workgroups * threads <= 0xffffffffull; }

// Pointer and strides of rows of `tokens` tokens; `align` in bytes.
bool rows_ok(const srs_rows *r, uint32_t align) {
    return r && r->p && r->heads > 0 && r->heads <= 65536 && ((uintptr_t)r->p & (align - 1)) == 0 && stride_ok(r->token_stride) && stride_ok(r->head_stride);
}

bool cache_ok(const srs_cache *c, uint32_t align) {
    if (!c || (c->pages && (!c->k || !c->v)) || !elem_bytes(c->dtype) || c->page_tokens == 0 || c->heads == 0 || c->heads > 65536 || c->head_dim == 0 || c->head_dim > 65536)
        return false;
    if (c->pages > kMaxIndexable || c->page_tokens > kMaxIndexable || (((uintptr_t)c->k | (uintptr_t)c->v) & (align - 1))) return false;
    const auto within = [](uint64_t n, int64_t stride) { return n == 0 || (uint64_t)(stride < 0 ? -stride : stride) <= kMaxSlots / n; };
    if (!within(c->pages, c->k_page) || !within(c->pages, c->v_page) || !within(c->page_tokens, c->k_token) || !within(c->page_tokens, c->v_token)) return false;
    return stride_ok(c->k_page) && stride_ok(c->k_token) && stride_ok(c->k_head) && stride_ok(c->v_page) && stride_ok(c->v_token) && stride_ok(c->v_head);
}

RowsArg rows_arg(const srs_rows *r) { return RowsArg{(unsigned char *)r->p, r->token_stride, r->head_stride, r->heads}; }

bool rotation_ok(uint32_t rot_dim, uint32_t head_dim, uint32_t flags, const int32_t *positions, const double *inv_freq, float magnitude) {
    if (rot_dim > head_dim || (rot_dim & 1u) || (flags & ~(SRS_ROPE_INTERLEAVED | SRS_ROPE_TRANSPOSE))) return false;
    if (rot_dim == 0) return true;
    return positions && inv_freq && !((uintptr_t)positions & 3u) && !((uintptr_t)inv_freq & 7u) && std::isfinite(magnitude);
}

// Do all rows and strides let 16-byte pieces be read and written, and whole pieces be turned?
bool rope_in_pieces(const RopeArgs &a, uint32_t size, bool interleaved) {
    const uint32_t n = 16 / size;
    if (a.head_dim % n || a.rot % (interleaved ? n : 2 * n) || a.rot / 2 > kTurns) return false;
    auto rows = [n](const RowsArg &r) { return r.heads == 0 || (((uintptr_t)r.p & 15u) == 0 && r.token_stride % n == 0 && r.head_stride % n == 0); };
    if (!rows(a.x) || !rows(a.out) || !rows(a.k) || !rows(a.v)) return false;
    if (!a.slots) return true;
    return (((uintptr_t)a.k_cache | (uintptr_t)a.v_cache) & 15u) == 0 &&
           ((a.k_page | a.k_token | a.k_head | a.v_page | a.v_token | a.v_head) & (int64_t)(n - 1)) == 0;
}

int launch_rope(RopeArgs &a, int dtype, uint32_t flags, hipStream_t st) {
    const uint32_t size = elem_bytes(dtype);
    const bool transpose = (flags & SRS_ROPE_TRANSPOSE) != 0, interleaved = (flags & SRS_ROPE_INTERLEAVED) != 0;
    const bool pieces = rope_in_pieces(a, size, interleaved);
    const uint64_t heads = (uint64_t)a.x.heads + a.k.heads + a.v.heads;
    const uint64_t each = !pieces ? a.rot / 2 + (a.head_dim - a.rot) : (interleaved ? a.rot : a.rot / 2) / (16 / size) + (a.head_dim - a.rot) / (16 / size);
    if (heads * each > 0x7fffffffull - 65536) return SRS_ERR_INVALID;
    // a workgroup for a token; where that leaves CUs idle, for as much of one as its threads take at once (up to 1 / 1024 / 4096 workgroups,
    // us: rows of 48 heads of 128, 1 token 3.5 / 3.2 / 3.2, 64 tokens 3.8 / 3.3 / 3.3, 1024 tokens 6.2 / 6.2 / 7.1)
    const uint64_t most = (heads * each + 255) / 256, wanted = (1024 + a.tokens - 1) / a.tokens;
    a.shares = (uint32_t)(most < wanted ? most : wanted);
    const uint64_t blocks = (uint64_t)a.tokens * a.shares;
    if (!grid_ok(blocks, 256)) return SRS_ERR_INVALID;
#define SRS_ROPE_LAUNCH(T)                                                                                                      \
    do {                                                                                                                        \
        const dim3 grid((uint32_t)blocks);                                                                                      \
        if (pieces && interleaved) hipLaunchKernelGGL((rope_pieces_kernel<T, true>), grid, dim3(256), 0, st, a, transpose);     \
        else if (pieces) hipLaunchKernelGGL((rope_pieces_kernel<T, false>), grid, dim3(256), 0, st, a, transpose);              \
        else if (interleaved) hipLaunchKernelGGL((rope_kernel<T, true>), grid, dim3(256), 0, st, a, transpose);                 \
        else hipLaunchKernelGGL((rope_kernel<T, false>), grid, dim3(256), 0, st, a, transpose);                                 \
    } while (0)
    if (dtype == SRS_BF16) SRS_ROPE_LAUNCH(__bf16);
    else if (dtype == SRS_FP16) SRS_ROPE_LAUNCH(_Float16);
    else SRS_ROPE_LAUNCH(float);
#undef SRS_ROPE_LAUNCH
    SRS_HIP(hipGetLastError());
    return SRS_OK;
}
}  // namespace

namespace {
constexpr uint64_t kMaxKeys = 1ull << 30;              // of one request
constexpr float kLog2e = 1.44269504088896340736f;

// How the attention of one call is laid out.
struct AttnPlan {
    AttnShape narrow, wide;
    uint32_t narrow_most, split_tokens, wide_tiles;
    uint32_t places;                    // of the wide kernel's workgroups, where its last round is shared out; else 0
    bool ranked;                        // requests in order of length
    bool eight;                         // waves of the narrow kernel, instead of four
    uint64_t workspace;
};

// Workgroups that a launch should have where rows are few (two of either kernel fit a CU), and the fewest key tiles worth one.
// The narrow kernel's are short and even out requests of unlike length; more are not worth their beginning and end (6 / 12 / 24 a CU,
// us: 128 requests of up to 8192 keys 580 / 464 / 472, two of up to 131072 136 / 138 / 164).
// The wide kernel's (256 / 512 / 1024, us, 32 heads over eight key heads, one request each: 16 tokens over 60,000 keys 65 / 58 / 69, 32
// 118 / 77 / 74, 128 over 30,000 140 / 130 / 143, 512 over 8000 136 / 113 / 122; four of 64 over 16,000 187 / 134 / 189).  At least 2 / 4 / 8 key
// tiles: 16 tokens over 8000 keys 27 / 25 / 29.
// Where tiles nearly fill the card without parts (three quarters of those workgroups), parts cost the wide kernel a pass over all results:
// 528 full tiles of 35 key tiles 152 us, in two parts 178.  Those behind the last whole round are shared out instead (116), where there are at
// most kTailRounds of them, which bounds the gain, and kTailKeys key tiles, which pay for the join.  Tiles of few rows come in two all the same, which evens out the end: 64 requests
// of 5 tokens over 4000 keys 276 / 226.
constexpr uint64_t kNarrowWorkgroups = 12 * 256, kWideWorkgroups = 512;
constexpr uint64_t kTailKeys = 24, kTailRounds = 6;
constexpr uint64_t kLeastNarrowTiles = 2, kLeastWideTiles = 4, kFewRows = 32;

// The narrow kernel's parts are joined by a launch of their own.  The workgroup that ends last could do it, but what the others wrote has to
// pass from XCD to XCD for that, and the release and acquire of each workgroup empty its L2: separate / last, us: 8 requests of up to 1000
// keys 13.3 / 16.9, 128 of up to 8192 413 / 738.
// Where it would share keys out, its workgroups may have eight waves and go through all of them instead, which saves joining
// parts: for up to kEightTiles key tiles, and, where there are tiles enough for most CUs, up to kEightWork over all of them.
// Four waves and parts / eight, us (heads of 128, requests times key heads, longest context, the shortest an eighth of it): 32 of 500 keys 12.2 / 10.6, of 1000
// 12.3 / 15.2, 128 of 1000 17.3 / 18.3, 256 of 500 17.6 / 13.0, of 1000 29.4 / 21.1, of 4000 65.8 / 65.7, 512 of 2000 71.3 / 63.8, of
// 4000 116.1 / 114.7, 1024 of 500 54.8 / 50.2, of 1000 73.3 / 72.3, of 2000 116.3 / 120.5.
constexpr uint64_t kEightTiles = 4, kEightUnits = 192, kEightWork = 8192;

uint64_t parts_over(uint64_t n, uint64_t each) { return (n + each - 1) / each; }

// The tiles of a kernel with `rows` rows.
void attention_tiles(AttnShape &w, uint32_t rows, uint32_t group) {
    w.head_blocks = (group + rows - 1) / rows;
    w.block = (group + w.head_blocks - 1) / w.head_blocks;
    w.tile_tokens = rows / w.block;
    w.part_o = w.part_lse = nullptr; w.slots = 0;
}

// Key tiles of `step` keys that a tile reads at most.
uint64_t attention_key_tiles(const AttnShape &w, uint64_t step, uint64_t keys, uint32_t window, uint32_t sinks) {
    const uint64_t all = parts_over(keys, step), seen = parts_over(sinks, step) + parts_over((uint64_t)window + w.tile_tokens, step) + 1;
    return window && seen < all ? seen : all;
}

void attention_split(AttnShape &w, uint64_t key_tiles, uint64_t each, uint64_t least) {
    each = each < least ? least : each;
    const uint64_t splits = parts_over(key_tiles, each);
    w.split_tiles = (uint32_t)each; w.splits = splits < 1 ? 1 : (uint32_t)splits;
}

AttnPlan attention_plan(uint32_t nrequests, uint64_t tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, uint32_t table_width,
                        uint32_t page_tokens, uint32_t window, uint32_t sinks, uint64_t most_tokens, uint64_t most_keys) {
    AttnPlan p;
    const uint32_t group = q_heads / kv_heads;
    uint64_t keys = (uint64_t)table_width * page_tokens;
    if (most_keys && most_keys < keys) keys = most_keys;
    attention_tiles(p.narrow, 16, group);
    attention_tiles(p.wide, 128, group);
    const uint64_t busy = tokens < nrequests ? tokens : nrequests, units = busy * kv_heads * p.narrow.head_blocks;
    const uint64_t key_tiles = attention_key_tiles(p.narrow, kSplitKeys, keys, window, sinks);
    attention_split(p.narrow, key_tiles, parts_over(units * key_tiles, kNarrowWorkgroups), kLeastNarrowTiles);
    p.eight = p.narrow.splits > 1 && head_dim <= 128 && (key_tiles <= kEightTiles || (units >= kEightUnits && units * key_tiles <= kEightWork));
    if (p.eight) { p.narrow.splits = 1; p.narrow.split_tiles = 0x7fffffff; }
    // A request whose new tokens fit one narrow tile is read once by it; the wide kernel takes the others, unless there are none.
    const bool only_narrow = most_tokens && most_tokens <= p.narrow.tile_tokens;
    p.narrow_most = only_narrow ? 0x7fffffffu : p.narrow.tile_tokens;
    p.split_tokens = only_narrow ? (uint32_t)most_tokens : p.narrow.tile_tokens;
    p.narrow.slots = (uint64_t)nrequests * p.split_tokens;
    p.wide.slots = tokens; p.wide.splits = 1; p.wide.split_tiles = 0x7fffffff; p.wide_tiles = 0; p.places = 0; p.ranked = false;
    if (!only_narrow) {
        p.wide_tiles = (uint32_t)(tokens / p.wide.tile_tokens + nrequests);
        // of the tiles, those that hold something: a request's last is the only one that may be less than full
        const uint64_t chunks = tokens / (p.narrow.tile_tokens + 1), wide_busy = tokens / p.wide.tile_tokens + (chunks < nrequests ? chunks : nrequests);
        const uint64_t wide_units = wide_busy * kv_heads * p.wide.head_blocks, wide_keys = attention_key_tiles(p.wide, head_dim <= 128 ? 64 : 32, keys, window, sinks);
        const bool nearly_full = wide_units * 4 >= kWideWorkgroups * 3, few_rows = tokens * group <= kFewRows * wide_busy;
        attention_split(p.wide, wide_keys, !nearly_full ? parts_over(wide_units * wide_keys, kWideWorkgroups)
                                          : few_rows && wide_units < 2 * kWideWorkgroups ? parts_over(wide_keys, 2) : wide_keys, kLeastWideTiles);
        const uint32_t places = 256 * (head_dim <= 64 ? 3 : head_dim <= 128 ? 2 : 1);                  // registers allow so many
        p.ranked = nrequests <= kRanked && p.wide.splits == 1 && wide_units > places;
        if (p.ranked && wide_keys >= kTailKeys && wide_units <= kTailRounds * places) p.places = places;
    }
    p.workspace = 0;
    if (p.narrow.splits > 1) p.workspace += p.narrow.splits * p.narrow.slots * q_heads * 4 * (head_dim + 4);
    if (p.wide.splits > 1) p.workspace += p.wide.splits * p.wide.slots * q_heads * 4 * (head_dim + 4);
    p.workspace += (uint64_t)p.places * 128 * 4 * (head_dim + 4);
    return p;
}

// Where the parts lie in the workspace: results, then their lse (four words' room for each, which keeps what follows aligned).
void attention_parts(AttnShape &w, uint64_t cells, uint32_t head_dim, float *&at) {
    w.part_o = at; w.part_lse = at + cells * head_dim;
    at += cells * (head_dim + 4);
}

// Pages that hold whole blocks of 16 keys, alike for keys and values, whose rows a 32-bit offset spans: a block is looked up once, its address
// is scalar and serves both.
bool in_blocks(const srs_cache *c) {
    return c->page_tokens % 16 == 0 && c->k_page == c->v_page && c->k_token == c->v_token && c->k_token >= 0 && c->k_token <= 1ll << 26;
}

template <class T, bool WIDE>
int launch_join(const AttnArgs &a, const AttnShape &w, hipStream_t st) {
    if (w.splits <= 1) return SRS_OK;
    const uint64_t cells = w.slots * a.heads;
    if (w.splits <= kFewParts) hipLaunchKernelGGL((attention_join_kernel<T, WIDE, false>), dim3((uint32_t)((cells + 3) / 4)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((attention_join_kernel<T, WIDE, true>), dim3((uint32_t)cells), dim3(1024), 0, st, a);
    SRS_HIP(hipGetLastError());
    return SRS_OK;
}

template <class T, int DP>
int launch_attention(const AttnArgs &a, bool blocks, bool eight, hipStream_t st) {
    const dim3 narrow(a.nrequests * a.narrow.splits * a.kv_heads * a.narrow.head_blocks), wide(a.wide_tiles * a.wide.splits * a.kv_heads * a.wide.head_blocks + a.places);
#define SRS_ATTENTION(BLOCKS, EXACT)                                                                                    \
    do {                                                                                                                \
        if (a.wide_tiles) {                                                                                             \
            hipLaunchKernelGGL((attention_wide_kernel<T, DP, BLOCKS, EXACT>), wide, dim3(256), 0, st, a);               \
            SRS_HIP(hipGetLastError());                                                                                 \
        }                                                                                                               \
        if constexpr (DP <= 128) {                                                                                      \
            if (eight) hipLaunchKernelGGL((attention_narrow_kernel<T, DP, BLOCKS, EXACT, 8>), narrow, dim3(512), 0, st, a); \
        }                                                                                                               \
        if (!eight) hipLaunchKernelGGL((attention_narrow_kernel<T, DP, BLOCKS, EXACT, 4>), narrow, dim3(256), 0, st, a); \
        SRS_HIP(hipGetLastError());                                                                                     \
    } while (0)
    if (blocks && a.head_dim == DP) SRS_ATTENTION(true, true);
    else if (blocks) SRS_ATTENTION(true, false);
    else SRS_ATTENTION(false, false);
#undef SRS_ATTENTION
    int rc = launch_join<T, false>(a, a.narrow, st);
    if (rc == SRS_OK) rc = launch_join<T, true>(a, a.wide, st);
    if (rc == SRS_OK && a.places) {
        hipLaunchKernelGGL((attention_tail_join_kernel<T>), dim3(1024), dim3(256), 0, st, a);
        SRS_HIP(hipGetLastError());
    }
    return rc;
}

template <class T>
int launch_attention(const AttnArgs &a, bool blocks, bool eight, hipStream_t st) {
    if (a.head_dim <= 64) return launch_attention<T, 64>(a, blocks, eight, st);
    if (a.head_dim <= 128) return launch_attention<T, 128>(a, blocks, eight, st);
    return launch_attention<T, 256>(a, blocks, eight, st);
}
}  // namespace

extern "C" {

// New tokens, and pages of the free list, that a workgroup of the table calls is there for, of 256 and 64 at most.  512 / 2048 / 8192 tokens, us:
// 4,200 5.7 / 6.1 / 6.7, 34,000 6.0 / 6.7 / 10.2, 136,000 7.9 / 7.2 / 11.3; 1024 / 8192 / 65,536 pages of the list: 16,400 pages taken and
// released 14.4 / 16.9 / 32.6, 64,000 19.5 / 23.3 / 83.1.
// Where one is enough and requests are few it has 256 threads instead of 1024, whose sums and barriers are what such a call consists of: tables and release
// together, 1024 / 256, us: 1 request 8.2 / 5.6, 128 of one token 9.7 / 7.0, 256 10.0 / 7.4, 64 of up to 16 9.6 / 8.2, 200 of up to 5 10.0 / 9.0.
constexpr uint64_t kTokensEach = 1024;
constexpr uint32_t kPagesEach = 1024, kFewRequests = 256;

int srs_cache_tables(srs_ctx *ctx, const int32_t *start, const int32_t *count, uint32_t nrequests, uint32_t page_tokens,
                     int32_t *held, int32_t *table, uint32_t table_width, const int32_t *free_pages, int32_t *free_count,
                     uint32_t free_cap, int32_t *token_begin, int64_t *slots, int32_t *positions, uint64_t max_tokens, void *stream) {
    if (!ctx || page_tokens == 0 || !token_begin || !free_count || max_tokens > kMaxIndexable || free_cap > kMaxIndexable) return SRS_ERR_INVALID;
    if (nrequests > kMaxIndexable || (uint64_t)table_width * page_tokens > kMaxIndexable) return SRS_ERR_INVALID;
    if (nrequests && (!start || !count || !held || (table_width && !table))) return SRS_ERR_INVALID;
    if ((free_cap && !free_pages) || (max_tokens && (!slots || !positions))) return SRS_ERR_INVALID;
    if (((uintptr_t)start | (uintptr_t)count | (uintptr_t)held | (uintptr_t)table | (uintptr_t)free_pages | (uintptr_t)free_count |
         (uintptr_t)token_begin | (uintptr_t)positions) & 3u || (uintptr_t)slots & 7u)
        return SRS_ERR_INVALID;
    hipStream_t st = (hipStream_t)stream;
    SRS_ON_DEVICE(ctx->device);
    TablesArgs a{start, count, nrequests, page_tokens, held, table, table_width, free_pages, free_count, free_cap,
                 token_begin, slots, positions, (uint32_t)max_tokens, ctx->flags, ctx->flags + kTicketWord};
    const uint64_t grid = (max_tokens + kTokensEach - 1) / kTokensEach;
    if (nrequests <= kFewRequests && grid <= 1) hipLaunchKernelGGL((cache_tables_kernel<256>), dim3(1), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((cache_tables_kernel<1024>), dim3((uint32_t)(grid < 1 ? 1 : grid > 256 ? 256 : grid)), dim3(1024), 0, st, a);
    SRS_HIP(hipGetLastError());
    return SRS_OK;
}

int srs_cache_release(srs_ctx *ctx, const int32_t *keep, uint32_t nrequests, int32_t *held, const int32_t *table,
                      uint32_t table_width, int32_t *free_pages, int32_t *free_count, uint32_t free_cap, void *stream) {
    if (!ctx || !free_count || free_cap > kMaxIndexable || nrequests > kMaxIndexable || table_width > kMaxIndexable) return SRS_ERR_INVALID;
    if (nrequests == 0) return SRS_OK;
    if (!keep || !held || (table_width && !table) || (free_cap && !free_pages)) return SRS_ERR_INVALID;
    if (((uintptr_t)keep | (uintptr_t)held | (uintptr_t)table | (uintptr_t)free_pages | (uintptr_t)free_count) & 3u) return SRS_ERR_INVALID;
    hipStream_t st = (hipStream_t)stream;
    SRS_ON_DEVICE(ctx->device);
    ReleaseArgs a{keep, nrequests, held, table, table_width, free_pages, free_count, free_cap, ctx->flags, ctx->flags + kTicketWord};
    const uint32_t grid = free_cap / kPagesEach;         // as if all that the list has room for came back
    if (nrequests <= kFewRequests && grid <= 1) hipLaunchKernelGGL((cache_release_kernel<256>), dim3(1), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((cache_release_kernel<1024>), dim3(grid < 1 ? 1 : grid > 64 ? 64 : grid), dim3(1024), 0, st, a);
    SRS_HIP(hipGetLastError());
    return SRS_OK;
}


int srs_rope(srs_ctx *ctx, int dtype, const srs_rows *x, const srs_rows *out, uint64_t tokens, uint32_t head_dim,
             const int32_t *positions, const double *inv_freq, uint32_t rot_dim, uint32_t flags, float magnitude, void *stream) {
    const uint32_t size = elem_bytes(dtype);
    if (!ctx || !size || head_dim == 0 || head_dim > 65536 || tokens > kMaxIndexable) return SRS_ERR_INVALID;
    if (!rotation_ok(rot_dim, head_dim, flags, positions, inv_freq, magnitude)) {
        if (tokens || rot_dim > head_dim || (rot_dim & 1u)) return SRS_ERR_INVALID;
    }
    if (tokens == 0) return SRS_OK;
    if (!rows_ok(x, size) || !rows_ok(out, size) || x->heads != out->heads) return SRS_ERR_INVALID;
    hipStream_t st = (hipStream_t)stream;
    SRS_ON_DEVICE(ctx->device);
    RopeArgs a;
    std::memset(&a, 0, sizeof(a));
    a.x = rows_arg(x); a.out = rows_arg(out);
    a.tokens = (uint32_t)tokens; a.head_dim = head_dim; a.rot = rot_dim; a.page = 1;
    a.positions = positions; a.inv_freq = inv_freq; a.magnitude = magnitude; a.flags = ctx->flags;
    return launch_rope(a, dtype, flags, st);
}

int srs_cache_write(srs_ctx *ctx, const srs_cache *cache, const srs_rows *k, const srs_rows *v, uint64_t tokens,
                    const int64_t *slots, const srs_rows *q, const srs_rows *q_out, const int32_t *positions, const double *inv_freq,
                    uint32_t rot_dim, uint32_t flags, float magnitude, void *stream) {
    if (!ctx || !cache || tokens > kMaxIndexable) return SRS_ERR_INVALID;
    const uint32_t size = elem_bytes(cache->dtype);
    if (!size || !cache_ok(cache, size)) return SRS_ERR_INVALID;
    if (tokens == 0) return SRS_OK;
    if (!rotation_ok(rot_dim, cache->head_dim, flags, positions, inv_freq, magnitude)) return SRS_ERR_INVALID;
    if (!rows_ok(k, size) || !rows_ok(v, size) || k->heads != cache->heads || v->heads != cache->heads || !slots || ((uintptr_t)slots & 7u)) return SRS_ERR_INVALID;
    const bool queries = rot_dim > 0 && q;
    if (queries && (!rows_ok(q, size) || !rows_ok(q_out, size) || q->heads != q_out->heads)) return SRS_ERR_INVALID;
    hipStream_t st = (hipStream_t)stream;
    SRS_ON_DEVICE(ctx->device);
    RopeArgs a;
    std::memset(&a, 0, sizeof(a));
    if (queries) { a.x = rows_arg(q); a.out = rows_arg(q_out); }
    a.k = rows_arg(k); a.v = rows_arg(v);
    a.k_cache = (unsigned char *)cache->k; a.v_cache = (unsigned char *)cache->v;
    a.k_page = cache->k_page; a.k_token = cache->k_token; a.k_head = cache->k_head;
    a.v_page = cache->v_page; a.v_token = cache->v_token; a.v_head = cache->v_head;
    a.slots = slots; a.places = (uint64_t)cache->pages * cache->page_tokens; a.page = cache->page_tokens;
    a.tokens = (uint32_t)tokens; a.head_dim = cache->head_dim; a.rot = rot_dim;
    a.positions = positions; a.inv_freq = inv_freq; a.magnitude = magnitude; a.flags = ctx->flags;
    return launch_rope(a, cache->dtype, flags, st);
}


uint64_t srs_cache_attention_workspace(uint32_t nrequests, uint64_t tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim,
                                       uint32_t table_width, uint32_t page_tokens, uint32_t window, uint32_t sinks,
                                       uint64_t most_tokens, uint64_t most_keys) {
    if (nrequests == 0 || tokens == 0 || kv_heads == 0 || q_heads < kv_heads || tokens > kMaxIndexable || nrequests > kMaxIndexable) return 0;
    return attention_plan(nrequests, tokens, q_heads, kv_heads, head_dim, table_width, page_tokens, window, sinks, most_tokens, most_keys).workspace;
}

int srs_cache_attention(srs_ctx *ctx, const srs_cache *cache, const srs_rows *q, const srs_rows *out, float *lse, uint64_t tokens,
                        const int32_t *token_begin, const int32_t *start, const int32_t *table, uint32_t table_width,
                        uint32_t nrequests, float scale, uint32_t flags, uint32_t window, uint32_t sinks, uint64_t most_tokens,
                        uint64_t most_keys, void *workspace, uint64_t workspace_bytes, void *stream) {
    if (!ctx || !cache || tokens > kMaxIndexable || nrequests > kMaxIndexable || (flags & ~SRS_ATTN_FULL) || !std::isfinite(scale * kLog2e)) return SRS_ERR_INVALID;
    if ((cache->dtype != SRS_BF16 && cache->dtype != SRS_FP16) || !cache_ok(cache, 16)) return SRS_ERR_INVALID;
    if (cache->head_dim > 256 || (cache->head_dim & 7u) || window > kMaxIndexable || sinks > kMaxIndexable || (sinks && !window)) return SRS_ERR_INVALID;
    if ((flags & SRS_ATTN_FULL) && (window || sinks)) return SRS_ERR_INVALID;
    if (((cache->k_page | cache->k_token | cache->k_head | cache->v_page | cache->v_token | cache->v_head) & 7) != 0) return SRS_ERR_INVALID;
    if (tokens == 0 || nrequests == 0) return SRS_OK;
    if (!rows_ok(q, 16) || !rows_ok(out, 16) || q->heads != out->heads || q->heads % cache->heads) return SRS_ERR_INVALID;
    if (((q->token_stride | q->head_stride | out->token_stride | out->head_stride) & 7) != 0) return SRS_ERR_INVALID;
    if (!token_begin || !start || (table_width && !table) || (uint64_t)table_width * cache->page_tokens > kMaxKeys) return SRS_ERR_INVALID;
    if (((uintptr_t)token_begin | (uintptr_t)start | (uintptr_t)table | (uintptr_t)lse) & 3u) return SRS_ERR_INVALID;
    const AttnPlan p = attention_plan(nrequests, tokens, q->heads, cache->heads, cache->head_dim, table_width, cache->page_tokens, window, sinks,
                                      most_tokens, most_keys);
    if (p.workspace && (!workspace || ((uintptr_t)workspace & 15u) || workspace_bytes < p.workspace)) return SRS_ERR_INVALID;
    if (!grid_ok((uint64_t)nrequests * p.narrow.splits * cache->heads * p.narrow.head_blocks, p.eight ? 512 : 256) ||
        !grid_ok((uint64_t)p.wide_tiles * p.wide.splits * cache->heads * p.wide.head_blocks + p.places, 256) || tokens * q->heads > 0x7fffffffull ||
        (p.narrow.splits > 1 && !grid_ok(p.narrow.slots * q->heads, p.narrow.splits <= kFewParts ? 64 : 1024)) ||
        (p.wide.splits > 1 && !grid_ok(p.wide.slots * q->heads, p.wide.splits <= kFewParts ? 64 : 1024)))
        return SRS_ERR_INVALID;
    hipStream_t st = (hipStream_t)stream;
    SRS_ON_DEVICE(ctx->device);
    AttnArgs a;
    std::memset(&a, 0, sizeof(a));
    a.q = (const unsigned char *)q->p; a.out = (unsigned char *)out->p; a.lse = lse;
    a.k = (const unsigned char *)cache->k; a.v = (const unsigned char *)cache->v;
    a.q_token = q->token_stride; a.q_head = q->head_stride; a.o_token = out->token_stride; a.o_head = out->head_stride;
    a.k_page = cache->k_page; a.k_token = cache->k_token; a.k_head = cache->k_head;
    a.v_page = cache->v_page; a.v_token = cache->v_token; a.v_head = cache->v_head;
    a.token_begin = token_begin; a.start = start; a.table = table;
    a.tokens = (uint32_t)tokens; a.nrequests = nrequests; a.width = table_width; a.page = cache->page_tokens; a.pages = cache->pages;
    uint32_t log = 0;                                   // ceil(log2(page)): the quotient is exact for numerators below 2^31; a page of 1 takes none
    while ((1ull << log) < cache->page_tokens) ++log;
    a.page_magic = (uint32_t)(((1ull << (31 + log)) + cache->page_tokens - 1) / cache->page_tokens); a.page_shift = log ? log - 1 : 0;
    a.heads = q->heads; a.kv_heads = cache->heads; a.head_dim = cache->head_dim; a.group = q->heads / cache->heads;
    a.window = window; a.sinks = sinks; a.full = (flags & SRS_ATTN_FULL) != 0; a.flags = ctx->flags;
    a.scale = scale == 0.f ? 1.f : std::fabs(scale) * kLog2e;
    a.sign = scale > 0.f ? 1.f : scale < 0.f ? -1.f : 0.f;
    a.narrow = p.narrow; a.wide = p.wide; a.narrow_most = p.narrow_most; a.split_tokens = p.split_tokens; a.wide_tiles = p.wide_tiles; a.ranked = p.ranked; a.places = p.places;
    float *at = (float *)workspace;
    if (p.narrow.splits > 1) attention_parts(a.narrow, p.narrow.splits * p.narrow.slots * q->heads, cache->head_dim, at);
    if (p.wide.splits > 1) attention_parts(a.wide, p.wide.splits * p.wide.slots * q->heads, cache->head_dim, at);
    if (p.places) attention_parts(a.wide, (uint64_t)p.places * 128, cache->head_dim, at);
    const bool blocks = in_blocks(cache);
    if (cache->dtype == SRS_BF16) return launch_attention<__bf16>(a, blocks, p.eight, st);
    return launch_attention<_Float16>(a, blocks, p.eight, st);
}

}  // extern "C"
