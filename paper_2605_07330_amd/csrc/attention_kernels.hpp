// Device code of srs_cache_attention for gfx950.
#pragma once
#include "srs_kernels.hpp"

namespace srs {

struct AttnArgs {
    const unsigned char *q, *k, *v;
    unsigned char *out;
    float *lse;
    int64_t q_token, q_head, o_token, o_head;
    int64_t k_page, k_token, k_head, v_page, v_token, v_head;
    const int32_t *token_begin, *start, *table;
    uint32_t tokens, nrequests, width, page, pages;
    uint32_t heads, kv_heads, head_dim;
    uint32_t window, sinks;
    float scale;
    bool full;
    uint32_t *flags;
};

// A wave per row and head: lanes take one key each of 64, then one or more elements each of the output.
template <class T>
__global__ __launch_bounds__(64) void attention_rows_kernel(const AttnArgs a) {
    __shared__ float s_q[256];
    const uint32_t lane = threadIdx.x, t = blockIdx.x / a.heads, h = blockIdx.x % a.heads, kh = h / (a.heads / a.kv_heads);
    uint32_t lo = 0, hi = a.nrequests;                      // the last request that begins at or before t
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (a.token_begin[mid] <= (int32_t)t) lo = mid; else hi = mid;
    }
    const int32_t r = (int32_t)lo;
    const int32_t b0 = a.token_begin[r], b1 = a.token_begin[r + 1], start = a.start[r];
    if (b0 < 0 || b1 > (int32_t)a.tokens || start < 0 || b1 < b0) {
        if (lane == 0) atomicOr(a.flags, kFlagBadIndex);
        return;
    }
    if ((int32_t)t < b0 || (int32_t)t >= b1) return;
    const int64_t pos = (int64_t)start + ((int32_t)t - b0), keys = (int64_t)start + (b1 - b0);
    const int64_t end = a.full ? keys : pos + 1;
    const T *q = (const T *)a.q + (int64_t)t * a.q_token + (int64_t)h * a.q_head;
    for (uint32_t d = lane; d < a.head_dim; d += 64) s_q[d] = (float)q[d] * a.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    bool bad = false;
    for (int64_t j0 = 0; j0 < end; j0 += 64) {
        if (a.window && j0 >= (int64_t)a.sinks && j0 + 64 <= pos - (int64_t)a.window + 1) continue;
        const int64_t j = j0 + lane;
        bool seen = j < end && (!a.window || pos - j < (int64_t)a.window || j < (int64_t)a.sinks);
        int64_t vrow = 0;
        float s = -INFINITY;
        if (seen) {
            const int64_t pi = j / a.page;
            const int32_t page = pi < (int64_t)a.width ? a.table[(int64_t)r * a.width + pi] : -1;
            if (page < 0 || (uint32_t)page >= a.pages) { bad = true; seen = false; }
            else {
                const int64_t place = j - pi * a.page;
                const T *k = (const T *)a.k + page * a.k_page + place * a.k_token + (int64_t)kh * a.k_head;
                vrow = page * a.v_page + place * a.v_token + (int64_t)kh * a.v_head;
                float sum = 0.f;
                for (uint32_t d = 0; d < a.head_dim; ++d) sum += s_q[d] * (float)k[d];
                s = sum;
            }
        }
        float top = s;
        for (int x = 32; x; x /= 2) top = fmaxf(top, __shfl_xor(top, x));
        const float m2 = fmaxf(m, top), base = m2 == -INFINITY ? 0.f : m2, keep = expf(m - base);
        const float p = seen ? expf(s - base) : 0.f;
        float sum = p;
        for (int x = 32; x; x /= 2) sum += __shfl_xor(sum, x);
        l = l * keep + sum; m = m2;
        for (int e = 0; e < 4; ++e) o[e] *= keep;
        for (unsigned long long left = __ballot(seen); left; left &= left - 1) {
            const int from = __ffsll((unsigned long long)left) - 1;
            const float w = __shfl(p, from);
            const T *v = (const T *)a.v + __shfl(vrow, from);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (lane + 64 * e < a.head_dim) o[e] += w * (float)v[lane + 64 * e];
        }
    }
    T *out = (T *)a.out + (int64_t)t * a.o_token + (int64_t)h * a.o_head;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (lane + 64 * e < a.head_dim) out[lane + 64 * e] = (T)(l > 0.f || l != l ? o[e] / l : 0.f);
    if (lane == 0 && a.lse) a.lse[(uint64_t)t * a.heads + h] = m == -INFINITY && l == 0.f ? -INFINITY : m + logf(l);
    if (bad) atomicOr(a.flags, kFlagBadIndex);
}

}  // namespace srs
