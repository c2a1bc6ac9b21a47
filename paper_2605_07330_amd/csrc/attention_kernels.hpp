// Device code of srs_cache_attention for gfx950.
#pragma once
#include "srs_kernels.hpp"

namespace srs {

// How one of the two kernels lays its work out.  A tile is up to 16 (narrow) or 128 (wide) rows that share a key head: `block` heads of
// each of `tile_tokens` successive tokens of one request.  Its keys may be shared out over `splits` workgroups, split_tiles key
// tiles to each (the last takes what is left), whose results go to part_o [splits][slots][heads][head_dim] and part_lse [splits][slots][heads].
struct AttnShape {
    uint32_t block, head_blocks, tile_tokens, splits, split_tiles;
    float *part_o, *part_lse;
    uint64_t slots;
};

struct AttnArgs {
    const unsigned char *q, *k, *v;
    unsigned char *out;
    float *lse;
    int64_t q_token, q_head, o_token, o_head;
    int64_t k_page, k_token, k_head, v_page, v_token, v_head;
    const int32_t *token_begin, *start, *table;
    uint32_t tokens, nrequests, width, page, pages;
    uint32_t page_magic, page_shift;                                // j / page = j * page_magic >> 32 + page_shift for j below 2^31, unless page is 1
    uint32_t heads, kv_heads, head_dim, group;
    uint32_t window, sinks;
    float scale;                                                    // its size times log2(e); 1 where it is 0
    float sign;                                                     // -1, 0 or 1: taken by the queries
    bool full;
    uint32_t *flags;
    AttnShape narrow, wide;
    uint32_t narrow_most;                                           // requests of more new tokens are the wide kernel's
    uint32_t split_tokens;                                          // of more: not split by the narrow kernel
    uint32_t wide_tiles;                                            // 0: there is no wide launch
    bool ranked;                                                    // up to kRanked requests, in order of length
    uint32_t places;                                                // wide workgroups that the card holds, where the last round's are shared out; else 0
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
    // weights are carried times 2^12, as halves lose bits below 2^-14; what they still lose goes in products of its own (kLift)
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

template <class T> __device__ __forceinline__ T uniform_value(T x) { return (T)__builtin_amdgcn_readfirstlane((int)x); }

// Values that are not finite may not meet the weights of rows that do not see them (0 hides nothing), nor weights that their rounding may make
// 0, nor weights in two parts.  They are taken out of every tile, and where there were any, what they add to the rows that do see them, themselves
// whatever their weights, is added by a second walk over the keys when all else is done: all of them where tokens are few, else those of the
// 64th of the tiles that had some.  Looking at every value costs the wide kernel 1 to 3 % (8192 re-encoded 633 / 651 us); one infinite value
// makes it 1250 us, the walk over all keys 19,300, and a decoding batch 412 / 1370.
template <class T> __device__ __forceinline__ u32x4 finite_values(u32x4 x) {
    constexpr uint32_t E = AttnTypes<T>::kExponent;
    u32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = x[e] & ((x[e] & E) == E ? 0xffff0000u : ~0u) & ((x[e] >> 16 & E) == E ? 0xffffu : ~0u);
    return y;
}

// Halves hold numbers to within 2^-25.  What they lose so of a weight below 2^-14 (or, in two halves, below 2^-3) is added times 2^40 by products of
// its own in those tiles that have such weights; what these lose again is 2^-65, which not even 2^30 keys of the largest value make a half of.
// Without it a key whose value is 0 and whose score lies 20 above 8000 others took 10 % of the result, 24 above all of it.  us, without this and without
// looking at every value / as it is: scores of unit spread, 8192 re-encoded, heads of 128, 670 / 700, 24 chunks of heads of 64 261 / 268, 3000 tokens
// over 1000, heads of 256, 490 / 529, a decoding batch 416 / 416; of spread 4, where nearly every tile has such weights, 673 / 1057, 258 / 412,
// 514 / 1124 and 416 / 424.
constexpr float kLift = 0x1p40f;
// Of one half, and of two.  The bounds are held whole, so that larger weights taken as these lose nothing.
__device__ __forceinline__ float lost_weight(float x) {
    x = fminf(x, 0x1p-14f);
    return (x - (float)(_Float16)x) * kLift;
}
__device__ __forceinline__ float lost_in_two(float x) {
    x = fminf(x, 0x1p-3f);
    const float rest = x - (float)(_Float16)x;
    return (rest - (float)(_Float16)rest) * kLift;
}

// A part of a result under its share of the weights.  A value that is not finite is itself, also where the part lies so far below the others that
// its share is 0.
__device__ __forceinline__ void add_part(f32x4 &sum, float share, f32x4 part) {
    if (share != 0.f) {
        sum += share * part;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += fabsf(part[e]) < INFINITY ? 0.f : part[e];
    }
}

// Queries take the scale's sign, so that the largest score is that of the largest product; 0 where there is none.
template <class T> __device__ __forceinline__ typename AttnTypes<T>::x8 signed_query(typename AttnTypes<T>::x8 q, bool there, float sign) {
    typename AttnTypes<T>::x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (T)(there ? (float)q[e] * sign : 0.f);
    return y;
}

// What the block table says about keys of a request: each lane asks for one, a tile early, and looks at the answer when it is there.
// Nothing is asked where no row sees the key, nor, with BLOCKS, any of the 16 keys that it is the first of: place is then -1.
struct Asked { int32_t page, place; };
template <bool BLOCKS>
__device__ __forceinline__ Asked ask_table(const AttnArgs &a, const int32_t *table, int32_t j, bool seen) {
    const uint32_t at = !BLOCKS && a.page == 1 ? (uint32_t)j : __umulhi((uint32_t)j, a.page_magic) >> a.page_shift;
    Asked x;
    x.page = table[seen ? at : 0u];
    x.place = seen ? j - (int32_t)(at * a.page) : -1;
    return x;
}

// Where a lane's key (or block) lies behind the bases of K and V, in bytes; with BLOCKS both are the same.  Page 0 where there is none.
struct Found { int64_t k, v; bool there, hole; };
template <bool BLOCKS>
__device__ __forceinline__ Found find_row(const AttnArgs &a, const Asked &x) {
    Found f;
    f.there = x.place >= 0 && (uint32_t)x.page < a.pages;
    f.hole = x.place >= 0 && !f.there;
    const int64_t page = f.there ? x.page : 0, place = x.place >= 0 ? x.place : 0;
    f.k = (page * a.k_page + place * a.k_token) * 2;
    f.v = BLOCKS ? f.k : (page * a.v_page + place * a.v_token) * 2;
    return f;
}
__device__ __forceinline__ int64_t lane_value(int64_t x, uint32_t lane) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, (int)lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)x >> 32), (int)lane);
    return (int64_t)(((uint64_t)hi << 32) | lo);
}
// Bit k: key k of a tile is there.  lanes: bit i, lane i's is.
template <bool BLOCKS, int KEYS> __device__ __forceinline__ uint64_t there_bits(uint64_t lanes) {
    if (!BLOCKS) return lanes;
    uint64_t x = 0;
#pragma unroll
    for (int b = 0; b < KEYS / 16; ++b) x |= (lanes >> b & 1ull) * (0xffffull << (16 * b));
    return x;
}

// Bits 0 .. 63 of the keys from `key` on that a row sees: those before end, and at or after low or below sinks.
__device__ __forceinline__ uint64_t bits_below(int32_t n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }
__device__ __forceinline__ uint64_t seen_bits(int32_t key, int32_t low, int32_t end, int32_t sinks) {
    return bits_below(end - key) & (~bits_below(low - key) | bits_below(sinks - key));
}

struct AttnTile {
    int32_t r, first_row;              // request, row of its first token in the batch
    int32_t i0, i1, n;                 // tokens of the tile, counted inside the request; of the request
    int64_t start;
    int32_t end;                       // keys that some row may see lie below
    int32_t low, sinks;                // and at or above low, or below sinks
    bool narrow;                       // the table ends before the keys do
};

// Request r, if it can be computed and has new tokens.
__device__ __forceinline__ bool open_request(const AttnArgs &a, uint32_t r, AttnTile &t) {
    const int32_t b0 = a.token_begin[r], b1 = a.token_begin[r + 1], start = a.start[r];
    if (b0 < 0 || b1 <= b0 || (uint32_t)b1 > a.tokens || start < 0) return false;
    t.r = (int32_t)r; t.first_row = b0; t.start = start; t.n = b1 - b0;
    return true;
}

// Its tile that begins with token i0.
__device__ __forceinline__ void open_tile(const AttnArgs &a, int32_t i0, uint32_t tile_tokens, AttnTile &t) {
    t.i0 = i0; t.i1 = t.n - i0 < (int32_t)tile_tokens ? t.n : i0 + (int32_t)tile_tokens;
    const int64_t end = t.start + (a.full ? t.n : t.i1), room = (int64_t)a.width * a.page;
    t.narrow = end > room;
    t.end = (int32_t)(end < room ? end : room);
    int64_t low = a.window ? t.start + t.i0 - a.window + 1 : 0;
    low = low < 0 ? 0 : low;
    t.low = (int32_t)(low < 0x7fffffff ? low : 0x7fffffff);
    t.sinks = a.window ? (int32_t)a.sinks : 0;
}

// The last request r with begin(r) <= at, begin(r) = token_begin[r] / tile_tokens + r * each, by a search with 64 probes at a time; -1
// where there is none.
__device__ __forceinline__ int32_t find_request(const AttnArgs &a, uint32_t at, uint32_t tile_tokens, uint32_t each) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t lo = 0, hi = a.nrequests;
    while (true) {
        const uint32_t step = (hi - lo + 63) / 64, r = lo + lane * step;
        bool before = false;
        if (r < hi) {
            const int32_t b = a.token_begin[r];
            before = b >= 0 && (uint64_t)((uint32_t)b / tile_tokens) + (uint64_t)r * each <= at;
        }
        const uint32_t n = (uint32_t)__popcll(__ballot(before));
        if (n == 0) return -1;
        lo += (n - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
        if (step == 1) return uniform_value((int32_t)lo);
    }
}

// The keys that a row at position pos sees: those before end, and at or after low or below the tile's sinks.
__device__ __forceinline__ void span(const AttnArgs &a, const AttnTile &t, int64_t pos, int32_t &low, int32_t &end) {
    end = a.full || pos + 1 >= t.end ? t.end : (int32_t)(pos + 1);
    const int64_t l = a.window ? pos - a.window + 1 : 0;
    low = l < 0 ? 0 : l < 0x7fffffff ? (int32_t)l : 0x7fffffff;
}

// add(row of V, whether this lane's row sees it) for the keys key .. key + n - 1 that some row sees
template <class T, class F>
__device__ __forceinline__ void walk_values(const AttnArgs &a, const AttnTile &t, uint32_t kh, int32_t key, int32_t n, int32_t row_low, int32_t row_end, F add) {
    for (int32_t k = 0; k < n; ++k) {
        const int32_t j = key + k;
        if (j >= t.end || !(j >= t.low || j < t.sinks)) continue;
        const uint32_t at = a.page == 1 ? (uint32_t)j : __umulhi((uint32_t)j, a.page_magic) >> a.page_shift;
        const int32_t page = a.table[(int64_t)t.r * a.width + at];
        if ((uint32_t)page >= a.pages) continue;
        add((const T *)a.v + (int64_t)page * a.v_page + (int64_t)(j - (int32_t)(at * a.page)) * a.v_token + (int64_t)kh * a.v_head,
            (j < row_end) & ((j >= row_low) | (j < t.sinks)));
    }
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

// How many parts the keys of a tile come in.
__device__ __forceinline__ uint32_t parts_of(const AttnShape &w, int32_t all) {
    const uint32_t n = ((uint32_t)all + w.split_tiles - 1) / w.split_tiles;
    return n < 1 ? 1 : n > w.splits ? w.splits : n;
}

// Up to 64 requests, one to a lane, whose tiles are taken from the one with the longest keys on, later tokens first, so that the last
// workgroups are short ones.  In the batch's order / in this and the last round shared out as below, us: 24 requests of up to 512 new tokens
// behind up to 4096, heads of 64, 276 / 266, 60 of up to 64 behind 4000 143 / 112; heads of 128, 16 of up to 300 behind 8000 308 / 286.
constexpr uint32_t kRanked = 64;
struct Ranked {
    int32_t first_row, n, start;
    uint32_t tiles, before, all;        // this lane's, those of the requests before it, and all
    __device__ __forceinline__ Ranked(const AttnArgs &a, uint32_t tile_tokens) {
        const uint32_t lane = threadIdx.x & 63;
        AttnTile t;
        const bool open = lane < a.nrequests && open_request(a, lane, t) && (uint32_t)t.n > a.narrow_most;
        first_row = open ? t.first_row : 0; n = open ? t.n : 0; start = open ? (int32_t)t.start : 0;
        tiles = ((uint32_t)n + tile_tokens - 1) / tile_tokens;
        const uint32_t place = (((uint32_t)start + (uint32_t)n) & ~63u) | (63u - lane);      // the longest in steps of 64 keys, then the first
        before = all = 0;
        for (uint32_t r = 0; r < a.nrequests; r += 4) {
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) {
                const uint32_t its = (uint32_t)__builtin_amdgcn_readlane((int)tiles, (int)(r + k)), its_place = (uint32_t)__builtin_amdgcn_readlane((int)place, (int)(r + k));
                before += its_place > place ? its : 0u;
                all += its;
            }
        }
    }
    // Request and first token of tile `at` of all; -1 where there are fewer.
    __device__ __forceinline__ int32_t find(uint32_t at, uint32_t tile_tokens, AttnTile &t) const {
        const uint64_t here = __ballot(at - before < tiles);
        if (!here) return -1;
        const int r = __builtin_ctzll(here);
        t.r = r;
        t.first_row = __builtin_amdgcn_readlane(first_row, r); t.n = __builtin_amdgcn_readlane(n, r); t.start = __builtin_amdgcn_readlane(start, r);
        const uint32_t its = (uint32_t)__builtin_amdgcn_readlane((int)tiles, r), its_before = (uint32_t)__builtin_amdgcn_readlane((int)before, r);
        return (int32_t)((its - 1 - (at - its_before)) * tile_tokens);
    }
};

// Workgroups beyond the last whole number of rounds on a card of `places` leave most of it idle while they run: from `full` on, each of
// `units` is shared out over `most` workgroups, whose results go to part_o [places][128][head_dim] and part_lse [places][128].
// One request, whole workgroups on 512 places / the last round shared out, us: 552 of them over 30,000 keys 1785 / 1220, over 8000
// 497 / 368, over 1500 129 / 117; 1056 over 8000 832 / 713, 1552 1210 / 1085, 2600 2090 / 1965.
constexpr uint32_t kTailParts = 16, kTailTiles = 4;     // at most, and key tiles of a part at least
struct Tail {
    uint32_t units, full, most;
    __device__ __forceinline__ Tail(uint32_t n, uint32_t places) {
        const uint32_t rest = places && n > places ? n % places : 0u;
        most = rest ? places / rest : 1u;
        most = most < kTailParts ? most : kTailParts;
        units = n; full = most > 1 ? n - rest : n;
    }
    __device__ __forceinline__ uint32_t each(int32_t all) const {
        const uint32_t e = ((uint32_t)all + most - 1) / most;
        return e < kTailTiles ? kTailTiles : e;
    }
    __device__ __forceinline__ uint32_t parts(int32_t all) const { return all > 0 ? ((uint32_t)all + each(all) - 1) / each(all) : 1u; }
};

// ---- few rows: decoding ------------------------------------------------------------------------------------------------------
// 16 rows to a workgroup, 32 keys of a tile to each of its four or eight waves, which join their results at the end.  Scores come as
// K Q^T (keys down, rows across: v_mfma 16x16x32), so that a lane holds the weights of one row for eight keys, which is how the second
// product V^T P^T takes them if its keys are counted in the same order.  K and V pass through LDS, wave by wave: V for its transposed
// read, K so that memory is read by whole rows, past the caches (128 requests of up to 8192 keys: 464 us with K straight from
// memory in the operand's layout, half a line to an instruction, where the hint did nothing; 417 this way).  Pieces of 16 bytes are rearranged
// in each row so that neither read meets itself on a bank.  The next tile's rows are in flight meanwhile.
// Weights meet the values in two parts, value and remainder of its rounding, as the second product costs nothing here: the output is
// then off by its own rounding alone.
// Bound: the cache's bytes.  2.42 GB of them in 408 us (5.9 TB/s; two plain read streams reach 6.98), 0.60 GB of two requests in 106.  Heads of 256
// leave one workgroup to a CU (132 KB of LDS): 8 requests of 8000 keys over 8 key heads 146 us, 3.6 TB/s.
template <class T, int DP, bool BLOCKS, bool EXACT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP == 64 ? 3 : DP == 128 ? 2 : 1) void attention_narrow_kernel(const AttnArgs a) {
    constexpr int kNarrowKeys = 32 * WAVES;
    constexpr bool kHalf = AttnTypes<T>::kShift != 0.f;
    typedef typename AttnTypes<T>::x8 x8;
    typedef typename AttnTypes<T>::x4 x4;
    constexpr int kQC = DP / 32, kVC = DP / 16, kRegion = 64 * DP + 256, kRowPieces = DP / 8;      // 32 rows of V, or 16 of float results; pieces of 16 bytes
    __shared__ __attribute__((aligned(16))) unsigned char s_mem[WAVES * kRegion];
    __shared__ __attribute__((aligned(16))) unsigned char s_keys[WAVES][64 * DP];
    __shared__ float s_m[WAVES][16], s_l[WAVES][16];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform_value(tid >> 6), g = lane >> 4, n = lane & 15;
    const AttnShape &w = a.narrow;
    uint32_t id = blockIdx.x;
    const uint32_t hb = id % (a.kv_heads * w.head_blocks), kh = hb / w.head_blocks, block = hb % w.head_blocks;
    id /= a.kv_heads * w.head_blocks;
    const uint32_t split = id % w.splits;
    if (blockIdx.x == 0) check_requests(a);
    AttnTile t;
    if (!open_request(a, id / w.splits, t) || (uint32_t)t.n > a.narrow_most) return;
    for (int32_t i0 = 0; i0 < t.n; i0 += (int32_t)w.tile_tokens) {                  // one tile, unless the caller's hint was wrong
    if (i0) __syncthreads();
    open_tile(a, i0, w.tile_tokens, t);
    const KeyTiles tiles(t, kNarrowKeys);
    const uint32_t parts = (uint32_t)t.n > a.split_tokens ? 1 : parts_of(w, tiles.all);
    if (split >= parts) return;
    const int32_t from = (int32_t)(split * w.split_tiles);
    int32_t to = split + 1 == parts ? tiles.all : from + (int32_t)w.split_tiles;
    if (a.pages == 0) to = from;
    bool bad = t.narrow || (a.pages == 0 && tiles.all > 0);

    // this lane's row: keys before row_end, and at or after row_low or before the sinks' end
    const uint32_t token = n / w.block, head = block * w.block + n % w.block;
    const bool row_ok = t.i0 + (int32_t)token < t.i1 && head < a.group && token < w.tile_tokens;
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
        const T *p = (const T *)a.q + (int64_t)(row_ok ? row : (uint64_t)(t.first_row + t.i0)) * a.q_token + (int64_t)(kh * a.group + (row_ok ? head : 0u)) * a.q_head;
#pragma unroll
        for (int c = 0; c < kQC; ++c) {
            const bool there = EXACT || c * 32 + g * 8 < a.head_dim;
            q[c] = signed_query<T>(*(const x8 *)(p + (there ? c * 32 + g * 8 : 0)), row_ok && there, a.sign);
        }
    }

    // This lane carries piece `piece` of row my_row of every kRowsPerLoad of K and of V: whole rows go out in one load instruction.  Pieces
    // behind the head's end are read from its beginning and dropped.
    constexpr int kRowsPerLoad = 64 / kRowPieces;
    const uint32_t piece = lane % kRowPieces, my_row = lane / kRowPieces;
    const bool inside = EXACT || piece * 8 < a.head_dim;
    const uint32_t piece_off = inside ? piece * 16 : 0;
    const uint32_t row_off = my_row * (uint32_t)a.k_token * 2 + piece_off;           // BLOCKS: of K and V
    const unsigned char *const k_base = a.k + (int64_t)kh * a.k_head * 2, *const v_base = a.v + (int64_t)kh * a.v_head * 2;
    const int32_t *const table = a.table + (int64_t)t.r * a.width;
    // of the 32 keys from `key` on: the two blocks of 16 where pages hold whole blocks, else every key
    auto ask = [&](int32_t key, bool live) {
        const int32_t j = key + (int32_t)(BLOCKS ? 16 * (lane & 1) : lane & 31);
        return ask_table<BLOCKS>(a, table, j, live & (j < t.end) & ((j + (BLOCKS ? 15 : 0) >= t.low) | (j < t.sinks)));
    };
    u32x4 kreg[kVC], vreg[kVC];
    auto load_rows = [&](int64_t found, const unsigned char *base, u32x4 (&to)[kVC]) {
        constexpr int kLoads = 16 / kRowsPerLoad;                                   // of a block
        if constexpr (BLOCKS) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const auto p = scalar_base(as_global(base + lane_value(found, b)));
#pragma unroll
                for (int c = 0; c < kLoads; ++c) to[b * kLoads + c] = __builtin_nontemporal_load((gptr<const u32x4>)(p + (row_off + c * (kRowsPerLoad * 2) * (uint32_t)a.k_token)));
            }
        } else {
#pragma unroll
            for (int c = 0; c < kVC; ++c)
                to[c] = __builtin_nontemporal_load((gptr<const u32x4>)as_global(base + __shfl(found, c * kRowsPerLoad + my_row) + piece_off));
        }
    };
    uint64_t ok = 0;                                                                // of the keys whose rows are in kreg and vreg
    auto load = [&](const Asked &x) {
        const Found f = find_row<BLOCKS>(a, x);
        bad |= f.hole;
        ok = there_bits<BLOCKS, 32>(__ballot(f.there));
        load_rows(f.v, v_base, vreg);
        load_rows(f.k, k_base, kreg);
    };
    unsigned char *const mine = s_mem + wave * kRegion, *const keys = s_keys[wave];
    auto place_of = [&](uint32_t key, uint32_t p) { return key * (DP * 2) + ((p ^ ((key & 7) << 1)) & (kRowPieces - 1)) * 16; };
    auto k_place = [&](uint32_t key, uint32_t p) { return key * (DP * 2) + (p ^ (DP == 64 ? (key >> 1) & 7 : key & 15)) * 16; };
    f32x4 o[kVC];
#pragma unroll
    for (int c = 0; c < kVC; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    bool dirty = false;
    const int32_t shift = 32 * (int32_t)wave;
    if (from < to) {
    Asked next = ask(tiles.key(from, kNarrowKeys) + shift, true);
    load(next);
    next = ask(tiles.key(from + 1, kNarrowKeys) + shift, from + 1 < to);
#pragma unroll 1
    for (int32_t i = from; i < to; ++i) {
        const int32_t key = tiles.key(i, kNarrowKeys) + shift;
        const bool more = i + 1 < to;
        // does every row see every one of these keys?
        const bool whole = key + 32 <= all_end && (key >= all_low || key + 32 <= t.sinks) && (uint32_t)ok == ~0u;
        if (!whole) {
            // values that no row sees are 0: a weight of 0 does not hide what is not a number
            const uint32_t any = (uint32_t)(seen_bits(key, t.low, t.end, t.sinks) & ok);
#pragma unroll
            for (int c = 0; c < kVC; ++c) {
                const bool here = any >> (c * kRowsPerLoad + my_row) & 1u;
                vreg[c] = u32x4{here ? vreg[c][0] : 0u, here ? vreg[c][1] : 0u, here ? vreg[c][2] : 0u, here ? vreg[c][3] : 0u};
            }
        }
        u16x2 largest = {0, 0};
#pragma unroll
        for (int c = 0; c < kVC; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, vreg[c][e] & 0x7fff7fffu));
        if (__any((largest[0] >= AttnTypes<T>::kExponent) | (largest[1] >= AttnTypes<T>::kExponent))) {
            dirty = true;
#pragma unroll
            for (int c = 0; c < kVC; ++c) vreg[c] = finite_values<T>(vreg[c]);
        }
#pragma unroll
        for (int c = 0; c < kVC; ++c) {
            *(u32x4 *)(mine + place_of(c * kRowsPerLoad + my_row, piece)) = vreg[c];
            if constexpr (EXACT) *(u32x4 *)(keys + k_place(c * kRowsPerLoad + my_row, piece)) = kreg[c];
            else *(u32x4 *)(keys + k_place(c * kRowsPerLoad + my_row, piece)) = u32x4{inside ? kreg[c][0] : 0u, inside ? kreg[c][1] : 0u, inside ? kreg[c][2] : 0u, inside ? kreg[c][3] : 0u};
        }
        const uint32_t here = (uint32_t)ok;
        if (more) load(next);
        next = ask(tiles.key(i + 2, kNarrowKeys) + shift, i + 2 < to);
        float x[8], top = -INFINITY, low = INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < kQC; ++c) s = mfma_16x16x32(*(const x8 *)(keys + k_place(16 * b + n, 4 * c + g)), q[c], s);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * b + e] = s[e] * a.scale;
        }
        if constexpr (kHalf) {
#pragma unroll
            for (int e = 0; e < 8; ++e) low = fminf(low, x[e]);
        }
        if (!whole) {
            const uint32_t sees = ((uint32_t)seen_bits(key, row_low, row_end, t.sinks) & here) >> (4 * g);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = sees >> (16 * (e >> 2) + (e & 3)) & 1u ? x[e] : -INFINITY;
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
        auto values = [&](int c, int b) { return lds_transposed(mine + place_of(16 * b + 4 * g + (n >> 2), 2 * c + ((n & 3) >> 1)) + (n & 1) * 8); };
#pragma unroll
        for (int c = 0; c < kVC; ++c) {
            const x8 vt = __builtin_bit_cast(x8, __builtin_shufflevector(values(c, 0), values(c, 1), 0, 1, 2, 3, 4, 5, 6, 7));
            o[c] = mfma_16x16x32(vt, high, o[c]);
            o[c] = mfma_16x16x32(vt, rest, o[c]);
        }
        if constexpr (kHalf) {
            if (__any(low - base < -3.f)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = lost_in_two(x[e]);
                    high[e] = (T)x[e];
                    rest[e] = (T)(x[e] - (float)high[e]);
                }
#pragma unroll
                for (int c = 0; c < kVC; ++c) {
                    const x8 vt = __builtin_bit_cast(x8, __builtin_shufflevector(values(c, 0), values(c, 1), 0, 1, 2, 3, 4, 5, 6, 7));
                    o[c] += mfma_16x16x32(vt, rest, mfma_16x16x32(vt, high, f32x4{0.f, 0.f, 0.f, 0.f})) * (1.f / kLift);
                }
            }
        }
    }
    if (dirty) {
        for (int32_t i = from; i < to; ++i)
            walk_values<T>(a, t, kh, tiles.key(i, kNarrowKeys) + shift, 32, row_low, row_end, [&](const T *v, bool sees) {
#pragma unroll
                for (int c = 0; c < kVC; ++c)
                    if (EXACT || c * 16 + g * 4 < a.head_dim) {
                        const x4 y = *(const x4 *)(v + c * 16 + g * 4);
                        o[c] += f32x4{sees && !(fabsf((float)y[0]) < INFINITY) ? (float)y[0] : 0.f, sees && !(fabsf((float)y[1]) < INFINITY) ? (float)y[1] : 0.f,
                                      sees && !(fabsf((float)y[2]) < INFINITY) ? (float)y[2] : 0.f, sees && !(fabsf((float)y[3]) < INFINITY) ? (float)y[3] : 0.f};
                    }
            });
    }
    }
    if (bad) atomicOr(a.flags, kFlagBadIndex);

    // the waves' results, in each wave's own region
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    float *const os = (float *)mine;
#pragma unroll
    for (int c = 0; c < kVC; ++c) *(f32x4 *)(os + n * (DP + 4) + c * 16 + g * 4) = o[c];
    if (lane < 16) { s_m[wave][lane] = m; s_l[wave][lane] = l; }
    __syncthreads();
    const uint32_t orow = tid >> 4, otoken = orow / w.block, ohead = block * w.block + orow % w.block;
    if (t.i0 + (int32_t)otoken >= t.i1 || ohead >= a.group || otoken >= w.tile_tokens || tid >= 256) continue;
    float M = -INFINITY, L = 0.f, share[WAVES];
#pragma unroll
    for (int k = 0; k < WAVES; ++k) M = fmaxf(M, s_m[k][orow]);
    const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) { share[k] = __builtin_amdgcn_exp2f(s_m[k][orow] - base); L += share[k] * s_l[k][orow]; }
    const bool some = !(M == -INFINITY && L == 0.f);
    const float inv = some ? 1.f / L : 0.f;
    const uint64_t out_row = (uint64_t)(t.first_row + t.i0) + otoken;
    const uint32_t out_head = kh * a.group + ohead;
    const uint64_t cell = (split * w.slots + (uint64_t)t.r * a.split_tokens + otoken) * a.heads + out_head;     // where parts > 1
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) {
        const uint32_t d = c * 64 + (tid & 15) * 4;
        if (d >= a.head_dim) continue;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            add_part(y, share[k], *(const f32x4 *)((const float *)(s_mem + k * kRegion) + orow * (DP + 4) + d));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = some ? y[e] * inv : 0.f;
        if (parts > 1) {
            *(f32x4 *)(w.part_o + cell * a.head_dim + d) = f32x4{y[0], y[1], y[2], y[3]};
        } else {
            *(x4 *)((T *)a.out + (int64_t)out_row * a.o_token + (int64_t)out_head * a.o_head + d) = x4{(T)y[0], (T)y[1], (T)y[2], (T)y[3]};
        }
    }
    if ((tid & 15) == 0) {
        const float lse2 = some ? base + __builtin_amdgcn_logf(L) - AttnTypes<T>::kShift : -INFINITY;
        if (parts > 1) w.part_lse[cell] = lse2;
        else if (a.lse) a.lse[out_row * a.heads + out_head] = lse2 * 0.69314718055994530942f;
    }
    }
}

// ---- many rows: chunks ---------------------------------------------------------------------------------------------------------
// 128 rows to a workgroup, 32 to each of its four waves, which all go through the tile's keys, 64 at a time (32 above heads of 128).  K and
// V of a key tile pass through LDS (two buffers; the next tile is on its way in registers meanwhile), where every wave takes them as
// the left operand of v_mfma 32x32x16: S^T = K Q^T, so that a lane holds the weights of one row, and O^T = V^T P^T with P^T straight from
// those registers, the keys of a product counted in the order in which the lanes have them.  Pieces of 16 bytes are rearranged in
// each row so that neither the rows of K nor the transposed reads of V meet on a bank (no conflicts counted).  Weights are rounded to
// the element type for the second product: of the order of the output's own rounding.  A row's accumulators follow its running maximum
// only when that has grown by 2^kSlack (less in halves, where it costs the small weights bits).  Workgroups of a key head follow each other in
// steps of the number of key heads, so that an XCD keeps few of them in its L2.
// Bound: a wave's products and its exponentials, one after the other.  8192 new tokens of 32 heads of 128 over 4 key heads, 550 GFLOP: 640 to 680
// us (810 to 860 TFLOP/s; a plain 8192^3 product 1120); matrix units busy 39 % of the time and vector units 50 %, which adds up to little less
// than all of it: with two waves a SIMD they seldom work side by side.  One row's scores held a key tile ahead, so that products stand beside
// exponentials, fewer vector instructions for the maximum and wave priorities changed nothing.
// Of few rows: a wave owns 32 of the 128, so tiles of up to 32 rows keep one wave of four at the products, of up to 64 two: 16 tokens of
// 32 heads over 8 key heads, 64 rows, take 27 us over 8000 keys and 72 over 60,000, whose bytes take 4.7 and 35.
// Heads of 256: 256 + 256 registers and 128 bytes of scratch a lane, one wave a SIMD; 3000 tokens over 4000 at 530 TFLOP/s.
typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mfma_32x32x16(AttnTypes<__bf16>::x8 a, AttnTypes<__bf16>::x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma_32x32x16(AttnTypes<_Float16>::x8 a, AttnTypes<_Float16>::x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

template <class T, int DP, bool BLOCKS, bool EXACT>
__global__ __launch_bounds__(256, DP == 64 ? 3 : DP == 128 ? 2 : 1) void attention_wide_kernel(const AttnArgs a) {
    typedef typename AttnTypes<T>::x8 x8;
    typedef typename AttnTypes<T>::x4 x4;
    constexpr int KT = DP <= 128 ? 64 : 32, kB = KT / 32, kQC = DP / 16, kDB = DP / 32, kRowPieces = DP / 8;
    constexpr int kRowsPerLoad = 256 / kRowPieces, kRowsPerWave = kRowsPerLoad / 4, kLoads = KT / kRowsPerLoad, kBytes = KT * DP * 2;
    constexpr bool kHalf = AttnTypes<T>::kShift != 0.f;
    constexpr float kSlack = kHalf ? 4.f : 8.f, kShift = kHalf ? 10.f : 0.f;         // at most 2^14 in a half
    __shared__ __attribute__((aligned(16))) unsigned char s_k[2][kBytes], s_v[2][kBytes];
    __shared__ uint32_t s_dirty[2];                                                // bit k: in which 64th of the tiles a value was not finite
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform_value(tid >> 6), h = lane >> 5, n = lane & 31;
    const AttnShape &w = a.wide;
    const uint32_t heads = a.kv_heads * w.head_blocks;
    uint32_t unit = blockIdx.x / (heads * w.splits) * heads + blockIdx.x % heads, split = blockIdx.x / heads % w.splits, tail_part = 0;
    AttnTile t;
    Tail tail(0, 0);
    if (a.ranked) {
        const Ranked order(a, w.tile_tokens);
        tail = Tail(order.all * heads, a.places);
        if (tail.most > 1 && blockIdx.x >= tail.full) {                             // w.splits is 1 then
            tail_part = blockIdx.x - tail.full;
            if (tail_part / tail.most >= tail.units - tail.full) return;
            unit = tail.full + tail_part / tail.most; split = tail_part % tail.most;
        }
        const int32_t i0 = order.find(unit / heads, w.tile_tokens, t);
        if (i0 < 0) return;
        open_tile(a, i0, w.tile_tokens, t);
    } else {
        const uint32_t tile = a.wide_tiles - 1 - unit / heads;                      // later tokens, which see more keys, first
        const int32_t r = find_request(a, tile, w.tile_tokens, 1);
        if (r < 0 || !open_request(a, (uint32_t)r, t) || (uint32_t)t.n <= a.narrow_most) return;
        const int64_t i0 = (int64_t)(tile - ((uint32_t)t.first_row / w.tile_tokens + (uint32_t)r)) * w.tile_tokens;
        if (i0 >= t.n) return;
        open_tile(a, (int32_t)i0, w.tile_tokens, t);
    }
    // the same in all lanes, which the compiler does not see behind the two ways
    t.r = uniform_value(t.r); t.first_row = uniform_value(t.first_row); t.n = uniform_value(t.n); t.i0 = uniform_value(t.i0); t.i1 = uniform_value(t.i1);
    t.end = uniform_value(t.end); t.low = uniform_value(t.low); t.sinks = uniform_value(t.sinks); t.start = uniform_value((int32_t)t.start);
    unit = uniform_value(unit); split = uniform_value(split);
    const uint32_t hb = unit % heads, kh = hb / w.head_blocks, block = hb % w.head_blocks;
    const KeyTiles tiles(t, KT);
    const bool in_tail = tail.most > 1 && unit >= tail.full;
    const uint32_t parts = in_tail ? tail.parts(tiles.all) : parts_of(w, tiles.all), each_part = in_tail ? tail.each(tiles.all) : w.split_tiles;
    if (split >= parts) return;
    // one part: ~0, one of the last round's: its number, top bit set, else the part's: as one number, it costs the loop one register
    const uint32_t part = uniform_value(parts == 1 ? ~0u : in_tail ? tail_part | 1u << 31 : split);
    const int32_t from = (int32_t)(split * each_part);
    int32_t to = split + 1 == parts ? tiles.all : from + (int32_t)each_part;
    if (a.pages == 0) to = from;
    bool bad = t.narrow || (a.pages == 0 && tiles.all > 0);

    // this lane's row, and what some and all rows of the wave see
    const uint32_t slot = wave * 32 + n, token = slot / w.block, head = block * w.block + slot % w.block;
    const bool row_ok = t.i0 + (int32_t)token < t.i1 && head < a.group && token < w.tile_tokens;
    const uint64_t row = (uint64_t)(t.first_row + t.i0) + token;
    const int32_t tokens = t.i1 - t.i0, first = (int32_t)(wave * 32 / w.block), last_full = (int32_t)((wave * 32 + 31) / w.block);
    const int32_t last = last_full < tokens ? last_full : tokens - 1;
    int32_t row_low, row_end, all_low, all_end, any_low, any_end;
    span(a, t, t.start + t.i0 + token, row_low, row_end);
    span(a, t, t.start + t.i0 + first, any_low, all_end);
    span(a, t, t.start + t.i0 + last, all_low, any_end);
    if (first >= tokens) any_end = 0;                                              // no row at all

    x8 q[kQC];
    {
        const T *p = (const T *)a.q + (int64_t)(row_ok ? row : (uint64_t)(t.first_row + t.i0)) * a.q_token + (int64_t)(kh * a.group + (row_ok ? head : 0u)) * a.q_head;
#pragma unroll
        for (int c = 0; c < kQC; ++c) {
            const bool there = EXACT || c * 16 + h * 8 < a.head_dim;
            q[c] = signed_query<T>(*(const x8 *)(p + (there ? c * 16 + h * 8 : 0)), row_ok && there, a.sign);
        }
    }

    // A thread carries piece `piece` of row c * kRowsPerLoad + my_row of every key tile, of K and of V.
    const uint32_t piece = lane % kRowPieces, lane_row = lane / kRowPieces, my_row = wave * kRowsPerWave + lane_row;
    const bool inside = EXACT || piece * 8 < a.head_dim;
    const uint32_t piece_off = inside ? piece * 16 : 0;
    const uint32_t row_off = my_row % 16 * (uint32_t)a.k_token * 2 + piece_off;      // BLOCKS: of K and V
    const unsigned char *const k_base = a.k + (int64_t)kh * a.k_head * 2, *const v_base = a.v + (int64_t)kh * a.v_head * 2;
    const int32_t *const table = a.table + (int64_t)t.r * a.width;
    // of the tile's keys from `key` on: the blocks of 16 where pages hold whole blocks, else every key
    auto ask = [&](int32_t key, bool live) {
        const int32_t j = key + (int32_t)(BLOCKS ? 16 * (lane % (KT / 16)) : lane % KT);
        return ask_table<BLOCKS>(a, table, j, live & (j < t.end) & ((j + (BLOCKS ? 15 : 0) >= t.low) | (j < t.sinks)));
    };
    u32x4 kst[kLoads], vst[kLoads];
    uint64_t ok = 0;                                                               // of the keys whose rows are in kst and vst; bit i: lane i's answer
    bool hole = false;
    auto load = [&](const Asked &x) {
        const Found f = find_row<BLOCKS>(a, x);
        bad |= f.hole;
        hole = __any(f.hole);
        ok = __ballot(f.there);
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
            if constexpr (BLOCKS) {
                const int64_t at = lane_value(f.k, (c * kRowsPerLoad + wave * kRowsPerWave) / 16);
                const uint32_t off = row_off + (kRowsPerLoad < 16 ? c * kRowsPerLoad % 16 * (uint32_t)a.k_token * 2 : 0);
                kst[c] = *(gptr<const u32x4>)(scalar_base(as_global(k_base + at)) + off);
                vst[c] = *(gptr<const u32x4>)(scalar_base(as_global(v_base + at)) + off);
            } else {
                kst[c] = *(gptr<const u32x4>)as_global(k_base + __shfl(f.k, c * kRowsPerLoad + my_row) + piece_off);
                vst[c] = *(gptr<const u32x4>)as_global(v_base + __shfl(f.v, c * kRowsPerLoad + my_row) + piece_off);
            }
            if constexpr (!EXACT) kst[c] = u32x4{inside ? kst[c][0] : 0u, inside ? kst[c][1] : 0u, inside ? kst[c][2] : 0u, inside ? kst[c][3] : 0u};
        }
    };
    auto k_place = [&](uint32_t key, uint32_t p) { return key * (DP * 2) + (p ^ (DP == 64 ? (key >> 1) & 7 : key & 15)) * 16; };
    auto v_place = [&](uint32_t key, uint32_t p) { return key * (DP * 2) + (p ^ (DP == 64 ? ((key >> 1) & 1) << 2 : (key & 3) << 2)) * 16; };
    const uint32_t walked = ((uint32_t)(to - from) + 63) / 64;                     // tiles to a bit of s_dirty
    // what the registers hold, tile i with keys from `key` on, into LDS
    auto put = [&](int32_t i, int32_t key) {
        const int buf = i & 1;
        const bool edge = !(key + KT <= t.end && (key >= t.low || key + KT <= t.sinks));
        u16x2 largest = {0, 0};
        if (edge || hole) {                                                       // values that no row sees are 0
            const uint64_t any = (seen_bits(key, t.low, t.end, t.sinks) & there_bits<BLOCKS, KT>(ok)) >> my_row;
#pragma unroll
            for (int c = 0; c < kLoads; ++c) {
                const bool here = any >> (c * kRowsPerLoad) & 1u;
                vst[c] = u32x4{here ? vst[c][0] : 0u, here ? vst[c][1] : 0u, here ? vst[c][2] : 0u, here ? vst[c][3] : 0u};
            }
        }
#pragma unroll
        for (int c = 0; c < kLoads; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, vst[c][e] & 0x7fff7fffu));
        if (__any((largest[0] >= AttnTypes<T>::kExponent) | (largest[1] >= AttnTypes<T>::kExponent))) {
            if (lane == 0) {
                const uint32_t k = (uint32_t)(i - from) / walked;
                atomicOr(&s_dirty[k / 32], 1u << k % 32);
            }
#pragma unroll
            for (int c = 0; c < kLoads; ++c) vst[c] = finite_values<T>(vst[c]);
        }
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
            const uint32_t row = c * kRowsPerLoad + my_row;
            *(u32x4 *)(s_k[buf] + k_place(row, piece)) = kst[c];
            *(u32x4 *)(s_v[buf] + v_place(row, piece)) = vst[c];
        }
    };

    f32x16 o[kDB];
#pragma unroll
    for (int d = 0; d < kDB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float m = -INFINITY, l = 0.f;
    if (tid < 2) s_dirty[tid] = 0;
    __syncthreads();
    if (from < to) {
    Asked next = ask(tiles.key(from, KT), true);
    {
        load(next);
        next = ask(tiles.key(from + 1, KT), from + 1 < to);
        put(from, tiles.key(from, KT));
    }
    __syncthreads();

#pragma unroll 1
    for (int32_t i = from; i < to; ++i) {
        const int buf = i & 1;
        const int32_t key = tiles.key(i, KT);
        const bool more = i + 1 < to;
        const uint64_t here = ok;
        const bool holes = hole;
        if (more) load(next);
        next = ask(tiles.key(i + 2, KT), i + 2 < to);
        if (key < any_end && (key + KT > any_low || key < t.sinks)) {              // some row of the wave sees something
            const bool whole = key + KT <= all_end && (key >= all_low || key + KT <= t.sinks) && !holes;
            float x[kB][16], top = -INFINITY, low = INFINITY;
#pragma unroll
            for (int b = 0; b < kB; ++b) {
                f32x16 s;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
                for (int c = 0; c < kQC; ++c) s = mfma_32x32x16(*(const x8 *)(s_k[buf] + k_place(32 * b + n, 2 * c + h)), q[c], s);
#pragma unroll
                for (int e = 0; e < 16; ++e) x[b][e] = s[e];
                if constexpr (kHalf) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) low = fminf(low, s[e]);
                }
            }
            // taken here, or the compiler keeps all scores beside what is left of them (277 / 271 us; above heads of 128 533 / 594)
            if constexpr (kHalf && DP <= 128) asm volatile("" : "+v"(low));
            if (!whole) {
                uint64_t sees = seen_bits(key, row_low, row_end, t.sinks);
                if (holes) sees &= there_bits<BLOCKS, KT>(here);
                const uint64_t mine = sees >> (4 * h);
#pragma unroll
                for (int b = 0; b < kB; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[b][e] = (uint32_t)(mine >> (32 * b)) >> (8 * (e / 4) + e % 4) & 1u ? x[b][e] : -INFINITY;
            }
#pragma unroll
            for (int b = 0; b < kB; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, x[b][e]);
            top = fmaxf(top, __shfl_xor(top, 32)) * a.scale;
            if (__any(top > m + kSlack)) {
                const float m2 = fmaxf(m, top), keep = m2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m2);
                l *= keep;
#pragma unroll
                for (int d = 0; d < kDB; ++d) o[d] *= keep;
                m = m2;
            }
            const float base = kShift - (m == -INFINITY ? 0.f : m);
            if constexpr (kHalf) {
                if (__any(__builtin_fmaf(low, a.scale, base) < -14.f)) {
                    // copies that the compiler cannot see through: it would keep what it has here, registers full of it, for the products below
                    float base_here = base;
                    uint32_t key_here = 0;
                    asm volatile("" : "+v"(base_here), "+v"(key_here));
                    auto values_here = [&](int d, int b, int c, int u) {
                        return lds_transposed(s_v[buf] + v_place(key_here + 32 * b + 16 * c + 8 * u + 4 * h + ((lane & 15) >> 2), 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + (lane & 1) * 8);
                    };
#pragma unroll
                    for (int d = 0; d < kDB; ++d) o[d] *= kLift;
#pragma unroll
                    for (int b = 0; b < kB; ++b)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            x8 r;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][8 * c + e], a.scale, base_here));
                                r[e] = (T)lost_weight(y);
                            }
#pragma unroll
                            for (int d = 0; d < kDB; ++d)
                                o[d] = mfma_32x32x16(__builtin_bit_cast(x8, __builtin_shufflevector(values_here(d, b, c, 0), values_here(d, b, c, 1), 0, 1, 2, 3, 4, 5, 6, 7)), r, o[d]);
                            __builtin_amdgcn_sched_barrier(0);
                        }
#pragma unroll
                    for (int d = 0; d < kDB; ++d) o[d] *= 1.f / kLift;
                }
            }
            x8 p[kB][2];
#pragma unroll
            for (int b = 0; b < kB; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    x[b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][e], a.scale, base));
                    l += x[b][e];
                    p[b][e / 8][e % 8] = (T)x[b][e];
                }
            auto values = [&](int d, int b, int c, int u) {
                return lds_transposed(s_v[buf] + v_place(32 * b + 16 * c + 8 * u + 4 * h + ((lane & 15) >> 2), 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + (lane & 1) * 8);
            };
#pragma unroll
            for (int b = 0; b < kB; ++b)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int d = 0; d < kDB; ++d)
                        o[d] = mfma_32x32x16(__builtin_bit_cast(x8, __builtin_shufflevector(values(d, b, c, 0), values(d, b, c, 1), 0, 1, 2, 3, 4, 5, 6, 7)), p[b][c], o[d]);
        }
        if (more) put(i + 1, tiles.key(i + 1, KT));
        __syncthreads();
    }
    uint64_t dirty = uniform_value(s_dirty[0]) | (uint64_t)uniform_value(s_dirty[1]) << 32;
    if (dirty) {
        uint32_t left = walked;
        for (int32_t i = from; i < to; ++i) {
            if (dirty & 1)
                walk_values<T>(a, t, kh, tiles.key(i, KT), KT, row_low, row_end, [&](const T *v, bool sees) {
#pragma unroll
                    for (int d = 0; d < kDB; ++d)
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (EXACT || 32 * d + 8 * u + 4 * h < a.head_dim) {
                                const x4 y = *(const x4 *)(v + 32 * d + 8 * u + 4 * h);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[d][4 * u + e] += sees && !(fabsf((float)y[e]) < INFINITY) ? (float)y[e] : 0.f;
                            }
                });
            if (--left == 0) { left = walked; dirty >>= 1; }
        }
    }
    }
    if (bad) atomicOr(a.flags, kFlagBadIndex);

    l += __shfl_xor(l, 32);
    if (!row_ok) return;
    const bool some = !(m == -INFINITY && l == 0.f);
    const float inv = some ? 1.f / l : 0.f;
    const uint32_t out_head = kh * a.group + head;
    const uint64_t cell = part >> 31 ? (uint64_t)(part & 0x7fffffffu) * 128 + slot : (part * w.slots + row) * a.heads + out_head;
    auto each = [&](auto store) {
#pragma unroll
        for (int d = 0; d < kDB; ++d)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t at = 32 * d + 8 * u + 4 * h;
                if (EXACT || at < a.head_dim)
                    store(at, some ? o[d][4 * u] * inv : 0.f, some ? o[d][4 * u + 1] * inv : 0.f, some ? o[d][4 * u + 2] * inv : 0.f, some ? o[d][4 * u + 3] * inv : 0.f);
            }
    };
    if (part != ~0u) {
        float *const to_p = w.part_o + cell * a.head_dim;
        each([&](uint32_t at, float y0, float y1, float y2, float y3) { *(f32x4 *)(to_p + at) = f32x4{y0, y1, y2, y3}; });
    } else {
        T *const to_p = (T *)a.out + (int64_t)row * a.o_token + (int64_t)out_head * a.o_head;
        each([&](uint32_t at, float y0, float y1, float y2, float y3) { *(x4 *)(to_p + at) = x4{(T)y0, (T)y1, (T)y2, (T)y3}; });
    }
    if (h == 0) {
        const float lse2 = some ? m + __builtin_amdgcn_logf(l) - kShift : -INFINITY;
        if (part != ~0u) w.part_lse[cell] = lse2;
        else if (a.lse) a.lse[row * a.heads + out_head] = lse2 * 0.69314718055994530942f;
    }
}

constexpr int kSplitKeys = 128;                             // keys of a tile of the narrow kernel where they are shared out: four waves

// ---- joining the parts -------------------------------------------------------------------------------------------------------
// The parts' results of a row and head weighted by exp2 of their lse; 32 threads take four elements each (eight above 128) of a part.  Few
// parts: a wave to a row and head, two parts at once.  Many: a workgroup of 32 such groups, so that hundreds of parts cost a few round trips
// (171 parts: 17 us with 8 groups, 11 with 32).
constexpr uint32_t kFewParts = 8;

struct Joined {
    float L;
    f32x4 x;                            // lane: elements 4 * lane on
};
// Parts `from`, from + step and so on, to each half of the wave its own.
__device__ __forceinline__ Joined join_parts(const AttnArgs &a, const float *lse, const float *part, uint64_t stride, uint32_t from, uint32_t step, uint32_t n, float base) {
    const uint32_t lane = threadIdx.x & 63, piece = lane & 31;
    float L = 0.f;
    f32x4 o[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll 4
    for (uint32_t s = from; s < n; s += step) {
        const float share = __builtin_amdgcn_exp2f(lse[s * stride] - base);
        L += share;
        const float *p = part + s * stride * a.head_dim;
        if (piece * 4 < a.head_dim) add_part(o[0], share, *(const f32x4 *)(p + piece * 4));
        if (piece * 4 + 128 < a.head_dim) add_part(o[1], share, *(const f32x4 *)(p + piece * 4 + 128));
    }
    L += __shfl_xor(L, 32);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[k][e] += __shfl_xor(o[k][e], 32);
    return Joined{L, lane < 32 ? o[0] : o[1]};
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int k = 1; k < 64; k *= 2) x = fmaxf(x, __shfl_xor(x, k));
    return x;
}
template <class T>
__device__ __forceinline__ void store_joined(const AttnArgs &a, const Joined &y, float M, float base, uint64_t row, uint32_t head) {
    typedef typename AttnTypes<T>::x4 x4;
    const uint32_t lane = threadIdx.x & 63;
    const bool some = !(M == -INFINITY && y.L == 0.f);
    if (lane * 4 < a.head_dim) {
        const float inv = some ? 1.f / y.L : 0.f;
        *(x4 *)((T *)a.out + (int64_t)row * a.o_token + (int64_t)head * a.o_head + lane * 4) =
            x4{(T)(some ? y.x[0] * inv : 0.f), (T)(some ? y.x[1] * inv : 0.f), (T)(some ? y.x[2] * inv : 0.f), (T)(some ? y.x[3] * inv : 0.f)};
    }
    if (lane == 0 && a.lse) a.lse[row * a.heads + head] = some ? (base + __builtin_amdgcn_logf(y.L)) * 0.69314718055994530942f : -INFINITY;
}
// A wave joins n parts that lie `stride` cells apart.
template <class T>
__device__ __forceinline__ void join_row(const AttnArgs &a, const float *lse, const float *part, uint64_t stride, uint32_t n, uint64_t row, uint32_t head) {
    const uint32_t lane = threadIdx.x & 63;
    float M = -INFINITY;
    for (uint32_t s = lane; s < n; s += 64) M = fmaxf(M, lse[s * stride]);
    M = wave_max(M);
    const float base = M == -INFINITY ? 0.f : M;
    store_joined<T>(a, join_parts(a, lse, part, stride, lane >> 5, 2, n, base), M, base, row, head);
}

template <class T, bool WIDE, bool MANY>
__global__ __launch_bounds__(MANY ? 1024 : 256) void attention_join_kernel(const AttnArgs a) {
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform_value(tid >> 6);
    const AttnShape &w = WIDE ? a.wide : a.narrow;
    const uint64_t cell = MANY ? blockIdx.x : (uint64_t)blockIdx.x * 4 + wave;
    if (cell >= w.slots * a.heads) return;
    const uint32_t slot = (uint32_t)(cell / a.heads), head = (uint32_t)(cell % a.heads);
    // the row's tile, and how many parts its keys came in
    AttnTile t;
    uint32_t i;
    if constexpr (WIDE) {
        const int32_t r = find_request(a, slot, 1, 0);
        if (r < 0 || !open_request(a, (uint32_t)r, t) || (uint32_t)t.n <= a.narrow_most) return;
        i = slot - (uint32_t)t.first_row;
    } else {
        if (!open_request(a, slot / a.split_tokens, t) || (uint32_t)t.n > a.narrow_most || (uint32_t)t.n > a.split_tokens) return;
        i = slot % a.split_tokens;
    }
    if (i >= (uint32_t)t.n) return;
    open_tile(a, (int32_t)(i / w.tile_tokens * w.tile_tokens), w.tile_tokens, t);
    const uint32_t n = parts_of(w, KeyTiles(t, WIDE ? (a.head_dim <= 128 ? 64 : 32) : kSplitKeys).all);
    if (n <= 1) return;
    const uint64_t row = (uint64_t)t.first_row + i, stride = w.slots * a.heads;
    const float *const lse = w.part_lse + cell, *const part = w.part_o + cell * a.head_dim;
    if constexpr (!MANY) {
        join_row<T>(a, lse, part, stride, n, row, head);
    } else {
        constexpr int kWaves = 16;
        __shared__ float s_top[kWaves], s_sum[kWaves];
        __shared__ f32x4 s_o[kWaves][64];
        float M = -INFINITY;
        for (uint32_t s = tid; s < n; s += 64 * kWaves) M = fmaxf(M, lse[s * stride]);
        M = wave_max(M);
        if (lane == 0) s_top[wave] = M;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kWaves; ++k) M = fmaxf(M, s_top[k]);
        const float base = M == -INFINITY ? 0.f : M;
        Joined y = join_parts(a, lse, part, stride, tid >> 5, 2 * kWaves, n, base);
        s_o[wave][lane] = y.x;
        if (lane == 0) s_sum[wave] = y.L;
        __syncthreads();
        if (wave) return;
        y.L = 0.f;
        y.x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) { y.L += s_sum[k]; y.x += s_o[k][lane]; }
        store_joined<T>(a, y, M, base, row, head);
    }
}

// The parts of the last round's workgroups, row by row (11,000 rows in 8 parts of heads of 64 14 us, none 4; on twice and four times the workgroups
// the same within the scatter).
template <class T>
__global__ __launch_bounds__(256) void attention_tail_join_kernel(const AttnArgs a) {
    const AttnShape &w = a.wide;
    const uint32_t wave = uniform_value(threadIdx.x >> 6), heads = a.kv_heads * w.head_blocks;
    const Ranked order(a, w.tile_tokens);
    const Tail tail(order.all * heads, a.places);
    if (tail.most <= 1) return;
    for (uint32_t at = blockIdx.x * 4 + wave; at < (tail.units - tail.full) * 128; at += gridDim.x * 4) {
        const uint32_t first_part = at / 128 * tail.most, slot = at % 128, unit = tail.full + at / 128, hb = unit % heads;
        AttnTile t;
        const int32_t i0 = order.find(unit / heads, w.tile_tokens, t);
        if (i0 < 0) return;
        open_tile(a, i0, w.tile_tokens, t);
        const uint32_t n = tail.parts(KeyTiles(t, a.head_dim <= 128 ? 64 : 32).all);
        const uint32_t token = slot / w.block, head = hb % w.head_blocks * w.block + slot % w.block;
        if (n <= 1 || t.i0 + (int32_t)token >= t.i1 || head >= a.group || token >= w.tile_tokens) continue;
        const uint64_t cell = (uint64_t)first_part * 128 + slot;
        join_row<T>(a, w.part_lse + cell, w.part_o + cell * a.head_dim, 128, n, (uint64_t)(t.first_row + i0) + token, hb / w.head_blocks * a.group + head);
    }
}

}  // namespace srs
