// Device code of srs_cache_attention for gfx950.
#pragma once
#include "srs_kernels.hpp"

namespace srs {

// The work: a tile is up to `rows` rows that share a key head, `block` heads of each of `tile_tokens` successive tokens of one
// request.  Tiles are numbered so that a workgroup finds its own without a table: request r's begin at
// token_begin[r] / tile_tokens + r, which leaves room for at least as many as it has.
struct AttnArgs {
    const unsigned char *q, *k, *v;
    unsigned char *out;
    float *lse;
    int64_t q_token, q_head, o_token, o_head;
    int64_t k_page, k_token, k_head, v_page, v_token, v_head;
    const int32_t *token_begin, *start, *table;
    uint32_t tokens, nrequests, width, page, page_shift, pages;     // page_shift: log2 of page, or 32
    uint32_t heads, kv_heads, head_dim, group;
    uint32_t window, sinks;
    float scale;                                                    // times log2(e)
    bool full;
    uint32_t *flags;
    uint32_t block, head_blocks, tile_tokens, tiles;                // of this launch
    uint32_t splits, split_tiles;                                   // parts of a request's keys, key tiles in each (the last: what is left)
    float *part_o, *part_lse;                                       // [splits][tokens][heads][head_dim], [splits][tokens][heads]
    uint32_t *part_n;                                               // [tokens][heads] parts that hold something
};

template <class T> struct AttnTypes;
template <> struct AttnTypes<__bf16> {
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x4 __attribute__((ext_vector_type(4)));
    static constexpr float kShift = 0.f;
    static constexpr uint32_t kExponent = 0x7f80u;
};
template <> struct AttnTypes<_Float16> {
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x4 __attribute__((ext_vector_type(4)));
    // weights are carried times 2^12: halves lose bits below 2^-14, where the weights of a long row of keys lie
    static constexpr float kShift = 12.f;
    static constexpr uint32_t kExponent = 0x7c00u;
};
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma_16x16x32(AttnTypes<__bf16>::x8 a, AttnTypes<__bf16>::x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_16x16x32(AttnTypes<_Float16>::x8 a, AttnTypes<_Float16>::x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Four elements from LDS, transposed within each group of 16 lanes: lane i names the 8 bytes at row i / 4, columns 4 * (i % 4) .. + 3 of a
// 4 x 16 block and gets column i.
__device__ __forceinline__ s16x4 lds_transposed(const unsigned char *p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}

// the block table is read by scalar loads where a whole wave asks for the same entry
typedef const int32_t __attribute__((address_space(4))) const_i32;

template <class T> __device__ __forceinline__ T uniform_value(T x) { return (T)__builtin_amdgcn_readfirstlane((int)x); }

struct AttnTile {
    int32_t r, first_row;              // request, row of its first token in the batch
    int32_t i0, i1;                    // tokens of the tile, counted inside the request
    int64_t start;
    int32_t end;                       // keys that some row may see lie below
    int32_t low, sinks;                // and at or above low, or below sinks
    bool narrow;                       // the table ends before the keys do
};

// The request whose tiles hold number `tile`, by a search with 64 probes at a time; nothing where the tile is empty.
__device__ __forceinline__ bool find_tile(const AttnArgs &a, uint32_t tile, AttnTile &t) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t lo = 0, hi = a.nrequests;
    while (true) {
        const uint32_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        bool before = false;
        if (at < hi) {
            const int32_t b = a.token_begin[at];
            before = b >= 0 && (uint64_t)((uint32_t)b / a.tile_tokens) + at <= tile;
        }
        const uint32_t n = (uint32_t)__popcll(__ballot(before));
        if (n == 0) return false;
        lo += (n - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
        if (step == 1) break;
    }
    lo = uniform_value(lo);
    const int32_t b0 = a.token_begin[lo], b1 = a.token_begin[lo + 1], start = a.start[lo];
    if (b0 < 0 || b1 < b0 || (uint32_t)b1 > a.tokens || start < 0) return false;
    const int64_t i0 = (int64_t)(tile - ((uint32_t)b0 / a.tile_tokens + lo)) * a.tile_tokens;
    if (i0 >= b1 - b0) return false;
    t.r = (int32_t)lo; t.first_row = b0; t.start = start;
    t.i0 = (int32_t)i0; t.i1 = b1 - b0 - t.i0 < (int32_t)a.tile_tokens ? b1 - b0 : t.i0 + (int32_t)a.tile_tokens;
    const int64_t end = a.full ? (int64_t)start + (b1 - b0) : (int64_t)start + t.i1, room = (int64_t)a.width * a.page;
    t.narrow = end > room;
    t.end = (int32_t)(end < room ? end : room);
    int64_t low = a.window ? (int64_t)start + t.i0 - a.window + 1 : 0;
    low = low < 0 ? 0 : low;
    t.low = (int32_t)(low < 0x7fffffff ? low : 0x7fffffff);
    t.sinks = a.window ? (int32_t)a.sinks : 0;
    return true;
}

// The keys that a row at position pos sees: those before end, and at or after low or below the tile's sinks.
__device__ __forceinline__ void span(const AttnArgs &a, const AttnTile &t, int64_t pos, int32_t &low, int32_t &end) {
    end = a.full || pos + 1 >= t.end ? t.end : (int32_t)(pos + 1);
    const int64_t l = a.window ? pos - a.window + 1 : 0;
    low = l < 0 ? 0 : l < 0x7fffffff ? (int32_t)l : 0x7fffffff;
}

// Requests that cannot be computed are reported by the launch's first workgroup.
__device__ __forceinline__ void check_requests(const AttnArgs &a) {
    bool bad = false;
    for (uint32_t r = threadIdx.x; r < a.nrequests; r += blockDim.x) {
        const int32_t b0 = a.token_begin[r], b1 = a.token_begin[r + 1];
        bad |= b0 < 0 || b1 < b0 || b1 > (int32_t)a.tokens || a.start[r] < 0;
    }
    if (bad) atomicOr(a.flags, kFlagBadIndex);
}

// The key tiles of `step` keys that a tile reads: those of the first tokens that stay visible, then those from the window's beginning on.
struct KeyTiles {
    int32_t low, first, all;            // first: number of tiles below low
    __device__ __forceinline__ KeyTiles(const AttnTile &t, int32_t step) {
        low = t.low / step * step;
        int32_t s = t.sinks < low ? t.sinks : low;
        s = s < t.end ? s : t.end;
        first = (s + step - 1) / step;
        all = first + (t.end > low ? (t.end - low + step - 1) / step : 0);
    }
    __device__ __forceinline__ int32_t key(int32_t i, int32_t step) const { return i < first ? i * step : low + (i - first) * step; }
};

// This part's share of them; the number of parts that have one.
__device__ __forceinline__ uint32_t part_of(const AttnArgs &a, uint32_t split, int32_t all, int32_t &from, int32_t &to) {
    uint32_t n = ((uint32_t)all + a.split_tiles - 1) / a.split_tiles;
    n = n < 1 ? 1 : n > a.splits ? a.splits : n;
    from = (int32_t)(split * a.split_tiles);
    to = split + 1 == n ? all : from + (int32_t)a.split_tiles;
    return n;
}

// o (normalised) and lse in base 2 of a row to where they belong.
__device__ __forceinline__ void store_row_lse(const AttnArgs &a, uint64_t row, uint32_t head, uint32_t split, uint32_t n, float lse2) {
    const uint64_t at = row * a.heads + head;
    if (n > 1) {
        a.part_lse[(uint64_t)split * a.tokens * a.heads + at] = lse2;
        if (split == 0) a.part_n[at] = n;
    } else {
        if (a.splits > 1) a.part_n[at] = 1;
        if (a.lse) a.lse[at] = lse2 * 0.69314718055994530942f;
    }
}

// ---- few rows: decoding ------------------------------------------------------------------------------------------------------
// 16 rows to a workgroup, 32 keys of a tile of 128 to each of its four waves, which join their results at the end.  Scores come as
// K Q^T (keys down, rows across: v_mfma 16x16x32, keys straight from memory in the operand's own layout), so that a lane holds
// the weights of one row for eight keys, which is how the second product V^T P^T takes them if its keys are counted in the
// same order.  V passes through LDS, wave by wave, for its transposed read; its 16-byte pieces are rearranged in each row so that eight
// rows' reads fall on all banks.  The next tile's rows are in flight meanwhile.
// Bound: the cache's bytes.  Weights meet the values in two parts (value and remainder of its rounding): the second product costs
// nothing here.
constexpr int kNarrowKeys = 128;

template <class T, int DP, bool BLOCKS, bool EXACT>
__global__ __launch_bounds__(256, DP == 64 ? 3 : DP == 128 ? 2 : 1) void attention_narrow_kernel(const AttnArgs a) {
    typedef typename AttnTypes<T>::x8 x8;
    typedef typename AttnTypes<T>::x4 x4;
    constexpr int kQC = DP / 32, kVC = DP / 16, kRegion = 64 * DP + 256, kRowPieces = DP / 8;      // pieces of 16 bytes
    __shared__ __attribute__((aligned(16))) unsigned char s_mem[4 * kRegion];
    __shared__ float s_m[4][16], s_l[4][16];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform_value(tid >> 6), g = lane >> 4, n = lane & 15;
    uint32_t id = blockIdx.x;
    const uint32_t hb = id % (a.kv_heads * a.head_blocks), kh = hb / a.head_blocks, block = hb % a.head_blocks;
    id /= a.kv_heads * a.head_blocks;
    const uint32_t split = id % a.splits, tile = id / a.splits;
    if (blockIdx.x == 0) check_requests(a);
    AttnTile t;
    if (!find_tile(a, tile, t)) return;
    const KeyTiles tiles(t, kNarrowKeys);
    int32_t from, to;
    const uint32_t parts = part_of(a, split, tiles.all, from, to);
    if (split >= parts) return;
    if (a.pages == 0) to = from;
    bool bad = t.narrow || (a.pages == 0 && tiles.all > 0);

    // this lane's row: keys before row_end, and at or after row_low or before the sinks' end
    const uint32_t token = n / a.block, head = block * a.block + n % a.block;
    const bool row_ok = t.i0 + (int32_t)token < t.i1 && head < a.group && token < a.tile_tokens;
    const uint64_t row = (uint64_t)(t.first_row + t.i0) + token;
    int32_t row_low, row_end, all_low, all_end;                                      // all: what every row of the tile sees
    span(a, t, t.start + t.i0 + token, row_low, row_end);
    {
        int32_t unused;
        span(a, t, t.start + t.i1 - 1, all_low, unused);
        span(a, t, t.start + t.i0, unused, all_end);
    }

    x8 q[kQC];
    {
        const T *p = (const T *)a.q + (int64_t)row * a.q_token + (int64_t)(kh * a.group + head) * a.q_head;
#pragma unroll
        for (int c = 0; c < kQC; ++c) {
            x8 z = {};
            q[c] = row_ok && (EXACT || c * 32 + g * 8 < a.head_dim) ? *(const x8 *)(p + c * 32 + g * 8) : z;
        }
    }

    // Where this lane's pieces lie behind the base of a block of 16 keys: of K the row of key n, piece g of every 32 elements; of V
    // piece vpiece of row vrow of every kRowsPerLoad.  Pieces behind the head's end are read from its beginning and dropped.
    constexpr int kRowsPerLoad = 64 / kRowPieces;
    const uint32_t vpiece = lane % kRowPieces, vrow = lane / kRowPieces;
    const uint32_t k_lane = n * (uint32_t)a.k_token * 2 + g * 16, v_lane = vrow * (uint32_t)a.v_token * 2 + (EXACT || vpiece * 8 < a.head_dim ? vpiece * 16 : 0);
    const unsigned char *const k_base = a.k + (int64_t)kh * a.k_head * 2, *const v_base = a.v + (int64_t)kh * a.v_head * 2;
    const const_i32 *const table = (const const_i32 *)(a.table + (int64_t)t.r * a.width);

    // What the table says for the 32 keys from `key` on: for both blocks of 16 where pages hold whole blocks (scalar loads), else for key +
    // lane % 32.  Nothing is asked where no row sees a key; the answer is looked at a tile later, when it is there.
    struct Asked { int32_t page[BLOCKS ? 2 : 1]; int32_t place[BLOCKS ? 2 : 1]; };
    auto ask = [&](int32_t key, bool live) {
        Asked w;
#pragma unroll
        for (int b = 0; b < (BLOCKS ? 2 : 1); ++b) {
            const int32_t j = BLOCKS ? key + 16 * b : key + (int32_t)(lane & 31);
            const uint32_t at = a.page_shift < 32 ? (uint32_t)j >> a.page_shift : (uint32_t)j / a.page;
            const bool seen = live && j < t.end && (j + (BLOCKS ? 15 : 0) >= t.low || j < t.sinks);
            w.page[b] = -1; w.place[b] = -1;
            if (seen) {
                w.page[b] = BLOCKS ? table[at] : a.table[(int64_t)t.r * a.width + at];
                w.place[b] = j - (int32_t)(at * a.page);
            }
        }
        return w;
    };
    struct Pages { int32_t page[BLOCKS ? 2 : 1]; int32_t place[BLOCKS ? 2 : 1]; bool ok[BLOCKS ? 2 : 1]; };
    auto take = [&](const Asked &w) {
        Pages p;
#pragma unroll
        for (int b = 0; b < (BLOCKS ? 2 : 1); ++b) {
            p.ok[b] = (uint32_t)w.page[b] < a.pages;                                // -1 is not
            bad |= w.place[b] >= 0 && !p.ok[b];
            p.page[b] = p.ok[b] ? w.page[b] : 0;
            p.place[b] = w.place[b] >= 0 ? w.place[b] : 0;
        }
        return p;
    };
    x8 kreg[2][kQC];
    u32x4 vreg[kVC];
    auto load_k = [&](const Pages &w) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            gptr<const unsigned char> p;
            uint32_t off = k_lane;
            if constexpr (BLOCKS) {
                p = scalar_base(as_global(k_base + ((int64_t)w.page[b] * a.k_page + (int64_t)w.place[b] * a.k_token) * 2));
            } else {
                p = as_global(k_base + ((int64_t)__shfl(w.page[0], 16 * b + n) * a.k_page + (int64_t)__shfl(w.place[0], 16 * b + n) * a.k_token) * 2);
                off = g * 16;
            }
#pragma unroll
            for (int c = 0; c < kQC; ++c) {
                if constexpr (EXACT) {
                    kreg[b][c] = *(gptr<const x8>)(p + off + c * 64);
                } else {
                    const bool inside = c * 32 + g * 8 < a.head_dim;
                    const u32x4 x = *(gptr<const u32x4>)(p + (inside ? off + c * 64 : off - g * 16));
                    const u32x4 y = {inside ? x[0] : 0u, inside ? x[1] : 0u, inside ? x[2] : 0u, inside ? x[3] : 0u};
                    kreg[b][c] = __builtin_bit_cast(x8, y);
                }
            }
        }
    };
    auto load_v = [&](const Pages &w) {
#pragma unroll
        for (int c = 0; c < kVC; ++c) {
            constexpr int kLoads = 16 / kRowsPerLoad;                               // of a block
            if constexpr (BLOCKS) {
                const int b = c / kLoads;
                const auto p = scalar_base(as_global(v_base + ((int64_t)w.page[b] * a.v_page + ((int64_t)w.place[b] + (c % kLoads) * kRowsPerLoad) * a.v_token) * 2));
                vreg[c] = *(gptr<const u32x4>)(p + v_lane);
            } else {
                const uint32_t k = c * kRowsPerLoad + vrow;
                const auto p = as_global(v_base + ((int64_t)__shfl(w.page[0], k) * a.v_page + (int64_t)__shfl(w.place[0], k) * a.v_token) * 2);
                vreg[c] = *(gptr<const u32x4>)(p + (v_lane - vrow * (uint32_t)a.v_token * 2));
            }
        }
    };
    unsigned char *const mine = s_mem + wave * kRegion;
    auto place_of = [&](uint32_t key, uint32_t piece) { return key * (DP * 2) + ((piece ^ ((key & 7) << 1)) & (kRowPieces - 1)) * 16; };
    auto visible = [&](const Pages &w, int32_t key, uint32_t k) {                   // key + k to this lane's row
        const int32_t j = key + (int32_t)k;
        const bool ok = BLOCKS ? (k < 16 ? w.ok[0] : w.ok[BLOCKS ? 1 : 0]) : __shfl((int)w.ok[0], (int)k) != 0;
        return ok & (j < row_end) & ((j >= row_low) | (j < t.sinks));
    };

    f32x4 o[kVC];
#pragma unroll
    for (int c = 0; c < kVC; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const int32_t shift = 32 * (int32_t)wave;
    Pages now = take(ask(tiles.key(from, kNarrowKeys) + shift, from < to));
    Asked next = ask(tiles.key(from + 1, kNarrowKeys) + shift, from + 1 < to);
    if (from < to) { load_v(now); load_k(now); }
#pragma unroll 1
    for (int32_t i = from; i < to; ++i) {
        const int32_t key = tiles.key(i, kNarrowKeys) + shift;
        const bool more = i + 1 < to;
        // does every row see every one of these keys?
        const bool whole = key + 32 <= all_end && (key >= all_low || key + 32 <= t.sinks) && (BLOCKS ? now.ok[0] && now.ok[BLOCKS ? 1 : 0] : (bool)__all(now.ok[0]));
        if (!whole) {
            // values that no row sees are 0: a weight of 0 does not hide what is not a number
#pragma unroll
            for (int c = 0; c < kVC; ++c) {
                const uint32_t k = c * kRowsPerLoad + vrow;
                const int32_t j = key + (int32_t)k;
                const bool ok = BLOCKS ? now.ok[BLOCKS ? (c * kRowsPerLoad) >> 4 : 0] : __shfl((int)now.ok[0], (int)k) != 0;
                const bool any = ok & (j < t.end) & ((j >= t.low) | (j < t.sinks));
                vreg[c] = u32x4{any ? vreg[c][0] : 0u, any ? vreg[c][1] : 0u, any ? vreg[c][2] : 0u, any ? vreg[c][3] : 0u};
            }
        }
        // values that are not finite are left out of the product and added row by row, for the rows that see them: the product would
        // take them times the weights of the others, and times both parts of a weight
        u16x2 largest = {0, 0};
#pragma unroll
        for (int c = 0; c < kVC; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, vreg[c][e] & 0x7fff7fffu));
        const bool dirty = __any((largest[0] >= AttnTypes<T>::kExponent) | (largest[1] >= AttnTypes<T>::kExponent));
#pragma unroll
        for (int c = 0; c < kVC; ++c) *(u32x4 *)(mine + place_of(c * kRowsPerLoad + vrow, vpiece)) = vreg[c];
        const Pages cur = now;
        now = take(next);
        next = ask(tiles.key(i + 2, kNarrowKeys) + shift, i + 2 < to);
        if (more) load_v(now);
        float x[8], top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < kQC; ++c) s = mfma_16x16x32(kreg[b][c], q[c], s);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * b + e] = s[e] * a.scale;
        }
        if (more) load_k(now);
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = visible(cur, key, 16 * (e >> 2) + 4 * g + (e & 3)) ? x[e] : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > m)) {
            const float m2 = fmaxf(m, top), keep = m2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m2);
            l *= keep;
#pragma unroll
            for (int c = 0; c < kVC; ++c) o[c] *= keep;
            m = m2;
        }
        const float base = (m == -INFINITY ? 0.f : m) - AttnTypes<T>::kShift;
        x8 high, rest;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = __builtin_amdgcn_exp2f(x[e] - base);
            l += x[e];
            high[e] = (T)x[e];
            rest[e] = (T)(x[e] - (float)high[e]);
        }
        if (dirty) {
            // weights times values that are not finite, for the rows that see them; then the values are 0
#pragma unroll 1
            for (uint32_t k = 0; k < 32; ++k) {
                float w = x[0];
#pragma unroll
                for (int e = 1; e < 8; ++e) w = (k >> 4) * 4 + (k & 3) == (uint32_t)e ? x[e] : w;
                w = __shfl(w, (int)((k >> 2 & 3) * 16 + n));
                const bool sees = visible(cur, key, k);
#pragma unroll
                for (int c = 0; c < kVC; ++c) {
                    const T *const at = (const T *)(mine + place_of(k, 2 * c + (g >> 1)) + (g & 1) * 8);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = (float)at[e];
                        o[c][e] += (sees && !(fabsf(v) < INFINITY)) ? w * v : 0.f;
                    }
                }
            }
#pragma unroll 1
            for (uint32_t c = 0; c < (uint32_t)kVC; ++c) {
                uint32_t *const at = (uint32_t *)(mine + place_of(c * kRowsPerLoad + vrow, vpiece));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t E = AttnTypes<T>::kExponent, y = at[e];
                    at[e] = y & ((y & E) == E ? 0xffff0000u : ~0u) & ((y >> 16 & E) == E ? 0xffffu : ~0u);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < kVC; ++c) {
            s16x4 v[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) v[b] = lds_transposed(mine + place_of(16 * b + 4 * g + (n >> 2), 2 * c + ((n & 3) >> 1)) + (n & 1) * 8);
            const x8 vt = __builtin_bit_cast(x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
            o[c] = mfma_16x16x32(vt, high, o[c]);
            o[c] = mfma_16x16x32(vt, rest, o[c]);
        }
    }
    if (bad) atomicOr(a.flags, kFlagBadIndex);

    // the four waves' results, in each wave's own region
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    float *const os = (float *)mine;
#pragma unroll
    for (int c = 0; c < kVC; ++c) *(f32x4 *)(os + n * (DP + 4) + c * 16 + g * 4) = o[c];
    if (lane < 16) { s_m[wave][lane] = m; s_l[wave][lane] = l; }
    __syncthreads();
    const uint32_t orow = tid >> 4, otoken = orow / a.block, ohead = block * a.block + orow % a.block;
    if (t.i0 + (int32_t)otoken >= t.i1 || ohead >= a.group || otoken >= a.tile_tokens) return;
    float M = -INFINITY, L = 0.f, w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) M = fmaxf(M, s_m[k][orow]);
    const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int k = 0; k < 4; ++k) { w[k] = __builtin_amdgcn_exp2f(s_m[k][orow] - base); L += w[k] * s_l[k][orow]; }
    const bool some = !(M == -INFINITY && L == 0.f);
    const float inv = some ? 1.f / L : 0.f;
    const uint64_t out_row = (uint64_t)(t.first_row + t.i0) + otoken;
    const uint32_t out_head = kh * a.group + ohead;
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) {
        const uint32_t d = c * 64 + (tid & 15) * 4;
        if (d >= a.head_dim) continue;
        float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const f32x4 part = *(const f32x4 *)((const float *)(s_mem + k * kRegion) + orow * (DP + 4) + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] += w[k] * part[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = some ? y[e] * inv : 0.f;
        if (parts > 1) {
            *(f32x4 *)(a.part_o + (((uint64_t)split * a.tokens + out_row) * a.heads + out_head) * a.head_dim + d) = f32x4{y[0], y[1], y[2], y[3]};
        } else {
            *(x4 *)((T *)a.out + (int64_t)out_row * a.o_token + (int64_t)out_head * a.o_head + d) = x4{(T)y[0], (T)y[1], (T)y[2], (T)y[3]};
        }
    }
    if ((tid & 15) == 0) store_row_lse(a, out_row, out_head, split, parts, some ? base + __builtin_amdgcn_logf(L) - AttnTypes<T>::kShift : -INFINITY);
}

// ---- joining the parts -------------------------------------------------------------------------------------------------------
// A wave per row and head whose keys were shared out: parts' results weighted by exp2 of their lse.
template <class T>
__global__ __launch_bounds__(256) void attention_join_kernel(const AttnArgs a) {
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t at = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= (uint64_t)a.tokens * a.heads) return;
    const uint32_t row = (uint32_t)(at / a.heads), head = (uint32_t)(at % a.heads);
    // is the row one of a request that was computed?
    uint32_t lo = 0, hi = a.nrequests;
    while (true) {
        const uint32_t step = (hi - lo + 63) / 64, k = lo + lane * step;
        const bool before = k < hi && a.token_begin[k] >= 0 && a.token_begin[k] <= (int32_t)row;
        const uint32_t n = (uint32_t)__popcll(__ballot(before));
        if (n == 0) return;
        lo += (n - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
        if (step == 1) break;
    }
    const int32_t b0 = a.token_begin[lo], b1 = a.token_begin[lo + 1];
    if (b1 < b0 || b1 <= (int32_t)row || (uint32_t)b1 > a.tokens || a.start[lo] < 0) return;
    const uint32_t n = a.part_n[at];
    if (n <= 1 || n > a.splits) return;
    const uint64_t stride = (uint64_t)a.tokens * a.heads;
    float M = -INFINITY;
    for (uint32_t s = lane; s < n; s += 64) M = fmaxf(M, a.part_lse[s * stride + at]);
#pragma unroll
    for (int x = 1; x < 64; x *= 2) M = fmaxf(M, __shfl_xor(M, x));
    const float base = M == -INFINITY ? 0.f : M;
    float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t s = 0; s < n; ++s) {
        const float w = __builtin_amdgcn_exp2f(a.part_lse[s * stride + at] - base);
        L += w;
        const float *p = a.part_o + (s * stride + at) * a.head_dim;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (lane + 64 * e < a.head_dim) o[e] += w * p[lane + 64 * e];
    }
    const bool some = !(M == -INFINITY && L == 0.f);
    const float inv = some ? 1.f / L : 0.f;
    T *out = (T *)a.out + (int64_t)row * a.o_token + (int64_t)head * a.o_head;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (lane + 64 * e < a.head_dim) out[lane + 64 * e] = (T)(some ? o[e] * inv : 0.f);
    if (lane == 0 && a.lse) a.lse[at] = some ? (base + __builtin_amdgcn_logf(L)) * 0.69314718055994530942f : -INFINITY;
}

}  // namespace srs
