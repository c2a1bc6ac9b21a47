// Device code of the cache calls for gfx950: block tables and slots from request lengths, rotary positions, rows into the paged cache.
#pragma once
#include "srs_kernels.hpp"

namespace srs {

// ---- block tables -----------------------------------------------------------------------------------------------------

struct TablesArgs {
    const int32_t *start, *count;
    uint32_t nrequests, page;
    int32_t *held, *table;
    uint32_t width;
    const int32_t *free_pages;
    int32_t *free_count;
    uint32_t free_cap;
    int32_t *token_begin;
    int64_t *slots;
    int32_t *positions;
    uint32_t max_tokens;
    uint32_t *flags, *ticket;
};

// Whether this workgroup is the last of the launch to come here; the counter is 0 again afterwards.  What the others have read before
// is then theirs to overwrite.
__device__ __forceinline__ bool last_workgroup(uint32_t *ticket) {
    __shared__ uint32_t s_last;
    if (gridDim.x == 1) return true;
    __syncthreads();
    if (threadIdx.x == 0) s_last = atomicInc(ticket, gridDim.x - 1) == gridDim.x - 1;
    __syncthreads();
    return s_last != 0;
}

// Exclusive sums of two numbers per thread over the workgroup; totals in the last two.
template <int kTableThreads>
__device__ __forceinline__ void block_sums(int64_t a, int64_t b, int64_t &before_a, int64_t &before_b, int64_t &all_a, int64_t &all_b) {
    __shared__ int64_t wave_sums[2][kTableThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x = a, y = b;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const int64_t u = __shfl_up(x, k), v = __shfl_up(y, k);
        if (lane >= k) { x += u; y += v; }
    }
    if (lane == 63) { wave_sums[0][wave] = x; wave_sums[1][wave] = y; }
    __syncthreads();
    all_a = all_b = 0;
    before_a = x - a; before_b = y - b;
#pragma unroll
    for (int w = 0; w < kTableThreads / 64; ++w) {
        if (w == wave) { before_a += all_a; before_b += all_b; }
        all_a += wave_sums[0][w]; all_b += wave_sums[1][w];
    }
    __syncthreads();
}

// largest q < n with at[q] <= k (at ascending, at[0] <= k)
__device__ __forceinline__ uint32_t last_at_most(const uint32_t *at, uint32_t n, uint32_t k) {
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (at[mid] <= k) lo = mid; else hi = mid;
    }
    return lo;
}

// Requests come in chunks of one per thread; their tokens and the pages they ask for are numbered by two prefix sums, which every
// workgroup works out for itself, and both are then spread over all threads of the launch, which find their request by bisection.
// The pages that tokens lie in are known from the sums, whether they are in the table yet or not; the numbers that the call
// changes are written by the workgroup that finishes last, when nobody reads them any more.  Bound: latency (a load, two sums, a
// bisection, a load), 3.9 us for a decoding step; with many tokens what each of them costs besides, a bisection, a division and two stores: 557,000
// of 256 requests 10.7 us, of which their bytes take 1.5 (one workgroup for everything: 485).
template <int kTableThreads>
__global__ __launch_bounds__(kTableThreads) void cache_tables_kernel(const TablesArgs a) {
    __shared__ uint32_t s_tok[kTableThreads + 1], s_page[kTableThreads + 1], s_start[kTableThreads], s_held[kTableThreads];
    const uint32_t tid = threadIdx.x, worker = blockIdx.x * kTableThreads + tid, workers = gridDim.x * kTableThreads;
    const int32_t listed = *a.free_count;
    const uint32_t avail = listed < 0 ? 0u : (uint32_t)listed > a.free_cap ? a.free_cap : (uint32_t)listed;
    uint32_t flags = (listed < 0 || (uint32_t)listed > a.free_cap) ? kFlagBadIndex : 0u;
    int64_t tokens = 0, pages = 0;                          // of the requests before this chunk
    uint32_t start = 0, held = 0, now_held = 0;             // of this thread's request
    // numbers the chunk's tokens and pages; leaves room for the next call
    auto number = [&](uint32_t base, uint32_t n) {
        const uint32_t r = base + tid;
        int64_t cnt = 0, want = 0;
        start = held = 0;
        if (tid < n) {
            const int32_t s = a.start[r], c = a.count[r], h = a.held[r];
            if (s < 0 || c < 0 || h < 0 || (uint32_t)(h < 0 ? 0 : h) > a.width) flags |= kFlagBadIndex;
            start = s < 0 ? 0u : (uint32_t)s; cnt = c < 0 ? 0 : c; held = h < 0 ? 0u : (uint32_t)h > a.width ? a.width : (uint32_t)h;
            const uint32_t need = (uint32_t)(((uint64_t)start + (uint64_t)cnt + a.page - 1) / a.page);
            if (need > a.width && cnt > 0) flags |= kFlagOverflow;
            const uint32_t most = need < a.width ? need : a.width;
            want = most > held ? (int64_t)(most - held) : 0;
        }
        int64_t t0, p0, t_all, p_all;
        block_sums<kTableThreads>(cnt, want, t0, p0, t_all, p_all);
        t0 += tokens; p0 += pages;
        tokens += t_all; pages += p_all;
        s_tok[tid] = t0 < (int64_t)a.max_tokens ? (uint32_t)t0 : a.max_tokens;
        s_page[tid] = p0 < (int64_t)avail ? (uint32_t)p0 : avail;
        s_start[tid] = start; s_held[tid] = held;
        if (tid == n - 1) {
            s_tok[n] = tokens < (int64_t)a.max_tokens ? (uint32_t)tokens : a.max_tokens;
            s_page[n] = pages < (int64_t)avail ? (uint32_t)pages : avail;
        }
        __syncthreads();
        now_held = held + (tid < n ? s_page[tid + 1] - s_page[tid] : 0u);
    };
    auto chunk_of = [&](uint32_t base) { return a.nrequests - base < (uint32_t)kTableThreads ? a.nrequests - base : (uint32_t)kTableThreads; };
    for (uint32_t base = 0; base < a.nrequests; base += kTableThreads) {
        const uint32_t n = chunk_of(base);
        number(base, n);
        if (blockIdx.x == 0 && tid < n) a.token_begin[base + tid] = (int32_t)s_tok[tid];
        for (uint32_t k = s_page[0] + worker; k < s_page[n]; k += workers) {
            const uint32_t q = last_at_most(s_page, n, k);
            a.table[(uint64_t)(base + q) * a.width + s_held[q] + (k - s_page[q])] = a.free_pages[avail - 1 - k];
        }
        for (uint32_t t = s_tok[0] + worker; t < s_tok[n]; t += workers) {
            const uint32_t q = last_at_most(s_tok, n, t);
            const uint32_t pos = s_start[q] + (t - s_tok[q]), at = pos / a.page, h = s_held[q], got = s_page[q + 1] - s_page[q];
            int32_t page = -1;
            if (at < h) page = a.table[(uint64_t)(base + q) * a.width + at];
            else if (at - h < got) page = a.free_pages[avail - 1 - (s_page[q] + (at - h))];
            a.slots[t] = page < 0 ? -1ll : (int64_t)page * a.page + (pos - at * a.page);
            a.positions[t] = pos > 0x7fffffffu ? 0x7fffffff : (int32_t)pos;
        }
        __syncthreads();
    }
    const uint32_t t_end = tokens < (int64_t)a.max_tokens ? (uint32_t)tokens : a.max_tokens, taken = pages < (int64_t)avail ? (uint32_t)pages : avail;
    for (uint32_t t = t_end + worker; t < a.max_tokens; t += workers) { a.slots[t] = -1; a.positions[t] = 0; }
    if (blockIdx.x == 0) {
        if (tokens > (int64_t)a.max_tokens || pages > (int64_t)avail) flags |= kFlagOverflow;
        if (flags) atomicOr(a.flags, flags);
        if (tid == 0) a.token_begin[a.nrequests] = (int32_t)t_end;
    }
    if (!last_workgroup(a.ticket)) return;
    if (a.nrequests <= (uint32_t)kTableThreads) {
        if (tid < a.nrequests && now_held != held) a.held[tid] = (int32_t)now_held;
    } else {
        tokens = pages = 0;
        for (uint32_t base = 0; base < a.nrequests; base += kTableThreads) {
            const uint32_t n = chunk_of(base);
            number(base, n);
            if (tid < n && now_held != held) a.held[base + tid] = (int32_t)now_held;
            __syncthreads();
        }
    }
    if (tid == 0) *a.free_count = (int32_t)(avail - taken);
}

struct ReleaseArgs {
    const int32_t *keep;
    uint32_t nrequests;
    int32_t *held;
    const int32_t *table;
    uint32_t width;
    int32_t *free_pages, *free_count;
    uint32_t free_cap;
    uint32_t *flags, *ticket;
};

// The surplus pages, numbered in the order in which srs_cache_tables would have handed them out, go to the end of the free list from the
// last to the first.
template <int kTableThreads>
__global__ __launch_bounds__(kTableThreads) void cache_release_kernel(const ReleaseArgs a) {
    __shared__ uint32_t s_page[kTableThreads + 1], s_keep[kTableThreads];
    const uint32_t tid = threadIdx.x, worker = blockIdx.x * kTableThreads + tid, workers = gridDim.x * kTableThreads;
    const int32_t listed = *a.free_count;
    const uint32_t have = listed < 0 ? 0u : (uint32_t)listed > a.free_cap ? a.free_cap : (uint32_t)listed, room = a.free_cap - have;
    uint32_t flags = (listed < 0 || (uint32_t)listed > a.free_cap) ? kFlagBadIndex : 0u;
    uint32_t keep = 0, extra = 0;                           // of this thread's request
    auto look = [&](uint32_t base) {
        const uint32_t r = base + tid;
        keep = extra = 0;
        if (r < a.nrequests) {
            const int32_t k = a.keep[r], h = a.held[r];
            if (k < 0 || h < 0 || (uint32_t)(h < 0 ? 0 : h) > a.width) flags |= kFlagBadIndex;
            const uint32_t held = h < 0 ? 0u : (uint32_t)h > a.width ? a.width : (uint32_t)h;
            keep = k < 0 ? 0u : (uint32_t)k;
            extra = held > keep ? held - keep : 0;
        }
    };
    int64_t all = 0, before = 0, x, y, n, z;
    for (uint32_t base = 0; base < a.nrequests; base += kTableThreads) {       // how many there are
        look(base);
        block_sums<kTableThreads>(extra, 0, x, y, n, z);
        all += n;
    }
    for (uint32_t base = 0; base < a.nrequests; base += kTableThreads) {
        const uint32_t count = a.nrequests - base < (uint32_t)kTableThreads ? a.nrequests - base : (uint32_t)kTableThreads;
        if (a.nrequests > (uint32_t)kTableThreads) {                            // else they are still there
            look(base);
            block_sums<kTableThreads>(extra, 0, x, y, n, z);
        }
        s_page[tid] = (uint32_t)x; s_keep[tid] = keep;
        if (tid == count - 1) s_page[count] = (uint32_t)n;
        __syncthreads();
        for (uint32_t k = worker; k < (uint32_t)n; k += workers) {
            const uint32_t q = last_at_most(s_page, count, k);
            const int64_t to = all - 1 - (before + k);                          // places behind the list's end
            if (to < (int64_t)room) a.free_pages[have + (uint32_t)to] = a.table[(uint64_t)(base + q) * a.width + s_keep[q] + (k - s_page[q])];
        }
        before += n;
        __syncthreads();
    }
    if (blockIdx.x == 0) {
        if (all > (int64_t)room) flags |= kFlagOverflow;
        if (flags) atomicOr(a.flags, flags);
    }
    if (!last_workgroup(a.ticket)) return;
    for (uint32_t base = 0; base < a.nrequests; base += kTableThreads) {
        if (a.nrequests > (uint32_t)kTableThreads) look(base);
        if (extra) a.held[base + tid] = (int32_t)keep;
    }
    if (tid == 0) *a.free_count = (int32_t)(have + (all < (int64_t)room ? (uint32_t)all : room));
}

// ---- rotary positions and rows into the cache --------------------------------------------------------------------------

struct RowsArg {
    unsigned char *p;
    int64_t token_stride, head_stride;
    uint32_t heads;
};

struct RopeArgs {
    RowsArg x, out;                 // srs_rope: x -> out; srs_cache_write: q -> q_out (heads 0: none)
    RowsArg k, v;                   // srs_cache_write only
    unsigned char *k_cache, *v_cache;
    int64_t k_page, k_token, k_head, v_page, v_token, v_head;
    const int64_t *slots;           // NULL: no cache
    uint64_t places;                // pages * page
    uint32_t page;
    uint32_t tokens, head_dim, rot;
    uint32_t shares;                // workgroups to a token
    const int32_t *positions;
    const double *inv_freq;
    float magnitude;
    uint32_t *flags;
};

// Sine and cosine of position * frequency.  The turns are counted in double and reduced to one there: a binary32 product is off by
// 2^-24 of up to a million radians at far positions.  What is left, at most half a turn, is binary32.
__device__ __forceinline__ void turn_of(int32_t position, double inv_freq, float &c, float &s) {
    const double turns = (double)position * (inv_freq * 0.15915494309189533576888376337251436);
    const float half_turns = (float)(2.0 * (turns - rint(turns)));
    sincospif(half_turns, &s, &c);
}

// Where row t's head `head` (queries, then keys, then values) comes from and goes to; whether it is turned.  Nothing where its slot is none.
template <class T>
__device__ __forceinline__ bool rope_row(const RopeArgs &a, uint32_t t, uint32_t head, int64_t page, int64_t place, bool slot_ok, const T *&from, T *&to, bool &turned) {
    turned = true;
    if (head < a.x.heads) {
        from = (const T *)a.x.p + (int64_t)t * a.x.token_stride + (int64_t)head * a.x.head_stride;
        to = (T *)a.out.p + (int64_t)t * a.out.token_stride + (int64_t)head * a.out.head_stride;
        return true;
    }
    if (!slot_ok) return false;
    uint32_t h = head - a.x.heads;
    if (h < a.k.heads) {
        from = (const T *)a.k.p + (int64_t)t * a.k.token_stride + (int64_t)h * a.k.head_stride;
        to = (T *)a.k_cache + page * a.k_page + place * a.k_token + (int64_t)h * a.k_head;
    } else {
        h -= a.k.heads;
        from = (const T *)a.v.p + (int64_t)t * a.v.token_stride + (int64_t)h * a.v.head_stride;
        to = (T *)a.v_cache + page * a.v_page + place * a.v_token + (int64_t)h * a.v_head;
        turned = false;
    }
    return true;
}

__device__ __forceinline__ bool rope_slot(const RopeArgs &a, uint32_t t, int64_t &page, int64_t &place) {
    page = place = 0;
    if (!a.slots) return false;
    const int64_t slot = a.slots[t];
    if (slot < 0 || (uint64_t)slot >= a.places) {
        if (slot != -1 && threadIdx.x == 0) atomicOr(a.flags, kFlagBadIndex);
        return false;
    }
    page = slot / a.page; place = slot - page * a.page;
    return true;
}

// Any strides, alignment and sizes: one thread per pair, or per element that is copied.  Bound: the sines, one for each pair and head: 8192 tokens of
// 40 heads of 80, half of them turned in halves, 63 us in 16 bits (1.7 TB/s), of 128 off the 16-byte boundaries 62 (2.7; in pieces 28).
template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a, bool transpose) {
    const uint32_t units = a.rot / 2 + (a.head_dim - a.rot), heads = a.x.heads + a.k.heads + a.v.heads;
    const uint32_t t = blockIdx.x / a.shares;
    int64_t page, place;
    const bool slot_ok = rope_slot(a, t, page, place);
    for (uint32_t i = (blockIdx.x % a.shares) * 256 + threadIdx.x; i < heads * units; i += a.shares * 256) {
        const uint32_t head = i / units, u = i % units;
        const T *from;
        T *to;
        bool turned;
        if (!rope_row(a, t, head, page, place, slot_ok, from, to, turned)) continue;
        if (u >= a.rot / 2) {
            const uint32_t d = a.rot + (u - a.rot / 2);
            to[d] = from[d];
            continue;
        }
        const uint32_t d1 = INTERLEAVED ? 2 * u : u, d2 = INTERLEAVED ? 2 * u + 1 : u + a.rot / 2;
        const T x1 = from[d1], x2 = from[d2];
        float c = 1.f, s = 0.f;
        if (turned) {
            turn_of(a.positions[t], a.inv_freq[u], c, s);
            c *= a.magnitude; s *= transpose ? -a.magnitude : a.magnitude;
        }
        to[d1] = turned ? (T)((float)x1 * c - (float)x2 * s) : x1;
        to[d2] = turned ? (T)((float)x2 * c + (float)x1 * s) : x2;
    }
}

// Rows in 16-byte pieces: a workgroup takes a token, or a share of its heads where there are few tokens.  Its sines and cosines are
// worked out once, a thread each, while the first pieces are on their way, and serve all heads from LDS; a thread then turns
// the two pieces that hold a run of pairs (or the one, interleaved).  Bound: memory.  One thread per pair and head, each with
// its own sine, took three times as long (8192 tokens of 40 heads of 128 80 us, now 29: 5.9 TB/s read and written).
constexpr uint32_t kTurns = 512;                            // pairs that the table holds

template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_pieces_kernel(const RopeArgs a, bool transpose) {
    constexpr int N = 16 / sizeof(T), kAhead = 2;           // elements of a piece; units of a thread in flight
    typedef T piece __attribute__((ext_vector_type(N)));
    __shared__ __attribute__((aligned(16))) float s_cos[kTurns], s_sin[kTurns];
    const uint32_t turning = INTERLEAVED ? a.rot / N : a.rot / 2 / N, units = turning + (a.head_dim - a.rot) / N, heads = a.x.heads + a.k.heads + a.v.heads;
    const uint32_t t = blockIdx.x / a.shares, step = a.shares * 256;
    int64_t page, place;
    const bool slot_ok = rope_slot(a, t, page, place);
    struct Unit { T *to; piece x, y; uint32_t d; bool there, turns, turned; };
    auto open = [&](uint32_t i) {
        Unit z;
        const uint32_t head = i / units, u = i - head * units;
        const T *from = nullptr;
        z.there = i < heads * units && rope_row(a, t, head, page, place, slot_ok, from, z.to, z.turned);
        z.turns = u < turning;
        z.d = z.turns ? u * N : a.rot + (u - turning) * N;
        if (z.there) {
            z.x = *(const piece *)(from + z.d);
            if (!INTERLEAVED && z.turns) z.y = *(const piece *)(from + z.d + a.rot / 2);
        }
        return z;
    };
    auto close = [&](const Unit &z) {
        if (!z.there) return;
        piece x = z.x, y = z.y;
        if (z.turns && z.turned) {
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const float c = s_cos[z.d / 2 + e / 2], s = s_sin[z.d / 2 + e / 2], x1 = (float)z.x[e], x2 = (float)z.x[e + 1];
                    x[e] = (T)(x1 * c - x2 * s);
                    x[e + 1] = (T)(x2 * c + x1 * s);
                }
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float c = s_cos[z.d + e], s = s_sin[z.d + e], x1 = (float)z.x[e], x2 = (float)z.y[e];
                    x[e] = (T)(x1 * c - x2 * s);
                    y[e] = (T)(x2 * c + x1 * s);
                }
            }
        }
        *(piece *)(z.to + z.d) = x;
        if (!INTERLEAVED && z.turns) *(piece *)(z.to + z.d + a.rot / 2) = y;
    };
    uint32_t i = (blockIdx.x % a.shares) * 256 + threadIdx.x;
    Unit z[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) z[k] = open(i + k * step);
    for (uint32_t u = threadIdx.x; u < a.rot / 2; u += 256) {
        float c, s;
        turn_of(a.positions[t], a.inv_freq[u], c, s);
        s_cos[u] = c * a.magnitude; s_sin[u] = s * (transpose ? -a.magnitude : a.magnitude);
    }
    __syncthreads();
    while (true) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) close(z[k]);
        i += kAhead * step;
        if (i >= heads * units) break;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) z[k] = open(i + k * step);
    }
}

}  // namespace srs
