// Eviction from a paged cache by accumulated attention weight (include/poss.h: poss_kv_evict).
//
// Slots are ranked by a 32-bit key: those that always stay above all, NaN below all, the others by their weight, mapped so that unsigned order is
// the order of the numbers (-0 as 0).  Of the n = min(length, budget) that stay, the n-th largest key is found digit by digit
// (four counts of 8 bits each); of the slots with that very key the lowest stay.  Holes below n and kept slots from n on are equally many:
// the j-th hole is filled from the j-th of those.  No source is a destination, so the moves need no order.
#include "kv.h"

namespace poss {

__device__ __forceinline__ uint32_t weight_key(float w) {      // 1 .. 0xfffffffe; NaN: 0
    if (w != w) return 0;
    const uint32_t b = __builtin_bit_cast(uint32_t, w + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct EvictArgs {
    const float *weights; const int32_t *positions, *lengths;
    int budget, first, recent;
    int32_t *kept; float *weights_out; int32_t *positions_out, *lengths_out;
};

constexpr int EVICT_THREADS = 1024;

// Sum over the workgroup of the threads before this one, and of all (LDS: 17 ints).
__device__ __forceinline__ int block_scan(int x, int *red, int &all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = x;
    for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(s, o); if (lane >= o) s += y; }
    __syncthreads();
    if (lane == 63) red[wave] = s;
    __syncthreads();
    int before = 0; all = 0;
    for (int w = 0; w < EVICT_THREADS / 64; ++w) { if (w < wave) before += red[w]; all += red[w]; }
    return before + s - x;
}

// One workgroup per sequence and key head.
__global__ void __launch_bounds__(EVICT_THREADS) evict_select_kernel(KvView c, EvictArgs a) {
    __shared__ int hist[256], red[17], pick[2];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int64_t row = (int64_t)b * c.hkv + h, base = row * c.slots;
    const float *w = a.weights + base;
    const int32_t *pos = a.positions + base;
    int32_t *kept = a.kept + row * a.budget;
    float *wo = a.weights_out + base;
    int32_t *po = a.positions_out + base;
    int len = a.lengths[b];
    len = len < 0 ? 0 : len > c.slots ? c.slots : len;
    const int n = len < a.budget ? len : a.budget;
    if (h == 0 && tid == 0) a.lengths_out[b] = n;
    for (int i = n + tid; i < a.budget; i += EVICT_THREADS) kept[i] = -1;
    for (int i = n + tid; i < c.slots; i += EVICT_THREADS) { wo[i] = 0.f; po[i] = -1; }
    if (n == len) {
        for (int i = tid; i < n; i += EVICT_THREADS) { kept[i] = i; wo[i] = w[i]; po[i] = pos[i]; }
        return;
    }
    // the newest position
    int newest = INT32_MIN;
    for (int i = tid; i < len; i += EVICT_THREADS) newest = max(newest, pos[i]);
    for (int o = 32; o; o >>= 1) newest = max(newest, __shfl_xor(newest, o));
    if ((tid & 63) == 0) red[tid >> 6] = newest;
    __syncthreads();
    for (int i = 0; i < EVICT_THREADS / 64; ++i) newest = max(newest, red[i]);
    const int64_t border = (int64_t)newest - a.recent;
    auto key_of = [&](int i) { const int p = pos[i]; return p < a.first || p > border ? 0xffffffffu : weight_key(w[i]); };
    // the n-th largest key
    uint32_t prefix = 0;
    int want = n;                                    // which one of the keys that share the digits found so far
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = tid; i < 256; i += EVICT_THREADS) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < len; i += EVICT_THREADS) {
            const uint32_t k = key_of(i);
            if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int d = 255;
            while (want > hist[d]) want -= hist[d--];
            pick[0] = d; pick[1] = want;
        }
        __syncthreads();
        prefix = prefix << 8 | (uint32_t)pick[0];
        want = pick[1];
    }
    // kept: keys above the prefix, and the first `want` with it.  First the holes and movers are counted off in index order.
    int equal_before = 0, holes_before = 0, movers_before = 0;
    for (int i0 = 0; i0 < len; i0 += EVICT_THREADS) {
        const int i = i0 + tid;
        const uint32_t k = i < len ? key_of(i) : 0;
        const bool in = i < len, eq = in && k == prefix;
        int all;
        const int rank = equal_before + block_scan(eq, red, all);
        equal_before += all;
        const bool stays = in && (k > prefix || (eq && rank < want));
        const bool mover = stays && i >= n, hole = in && i < n && !stays;
        int holes, movers;
        const int hr = holes_before + block_scan(hole, red, holes), mr = movers_before + block_scan(mover, red, movers);
        holes_before += holes; movers_before += movers;
        // the lists meet in `kept`: a hole notes its rank as -2 - rank, and po[n ..] lends its room to the movers
        if (hole) kept[i] = -2 - hr;
        else if (in && i < n) { kept[i] = i; wo[i] = w[i]; po[i] = pos[i]; }
        if (mover) po[n + mr] = i;
    }
    __syncthreads();
    __threadfence_block();
    for (int i = tid; i < n; i += EVICT_THREADS) {
        const int k = kept[i];
        if (k >= 0) continue;
        const int s = po[n + (-2 - k)];
        kept[i] = s; wo[i] = w[s]; po[i] = pos[s];
    }
    __syncthreads();
    for (int i = n + tid; i < n + movers_before; i += EVICT_THREADS) po[i] = -1;
}

// 64 slots below the budget of one sequence and head per workgroup: those whose source is another take its key and value.
template <typename T>
__global__ void __launch_bounds__(256) evict_move_kernel(KvView c, const int32_t *__restrict__ kept, int budget) {
    const int h = blockIdx.y, b = blockIdx.z, d0 = threadIdx.x & 31;
    const int32_t *list = kept + ((int64_t)b * c.hkv + h) * budget;
    T *k = static_cast<T *>(c.k), *v = static_cast<T *>(c.v);
    for (int j = threadIdx.x >> 5; j < 64; j += 8) {
        const int to = blockIdx.x * 64 + j;
        if (to >= budget) break;
        const int from = list[to];
        if (from < 0 || from == to) continue;
        const int pf = kv_page(c, b, from), pt = kv_page(c, b, to);
        if (pf < 0 || pt < 0) continue;
        for (int d = d0; d < c.dh; d += 32) {
            k[kv_key_at(c, pt, h, to) + d] = k[kv_key_at(c, pf, h, from) + d];
            v[kv_value_at(c, pt, h, d, to)] = v[kv_value_at(c, pf, h, d, from)];
        }
    }
}

}  // namespace poss

// ------------------------------------------------------------------------------------------ C entry point (include/poss.h)
using namespace poss;

extern "C" int poss_kv_evict(const poss_kv_cache *cache, const float *weights, const int32_t *positions, const int32_t *lengths, int32_t budget, int32_t first, int32_t recent,
                             int32_t *kept, float *weights_out, int32_t *positions_out, int32_t *lengths_out, void *hip_stream) {
    const char *who = "poss_kv_evict";
    if (const char *why = kv_cache_bad(cache)) return set_error(POSS_E_INVALID_ARG, "%s: %s", who, why);
    if (budget < 1 || budget > 1 << 30 || first < 0 || recent < 0 || (int64_t)first + recent > budget) return set_error(POSS_E_INVALID_ARG, "%s: 0 <= first + recent <= budget, and a budget, are wanted", who);
    if (cache->n_seq == 0) return POSS_OK;
    if (!weights || !positions || !lengths || !kept || !weights_out || !positions_out || !lengths_out) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    for (const void *p : {(const void *)weights, (const void *)positions, (const void *)lengths, (const void *)kept, (const void *)weights_out, (const void *)positions_out, (const void *)lengths_out})
        if (!kv_aligned(p, 4)) return set_error(POSS_E_INVALID_ARG, "%s: an array is not aligned to its type", who);
    if (weights == weights_out || positions == positions_out || lengths == lengths_out) return set_error(POSS_E_INVALID_ARG, "%s: outputs must be arrays of their own", who);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const KvView c = kv_view(*cache);
    const EvictArgs a{weights, positions, lengths, budget, first, recent, kept, weights_out, positions_out, lengths_out};
    evict_select_kernel<<<dim3(c.hkv, c.n_seq), EVICT_THREADS, 0, st>>>(c, a);
    const int most = budget < c.slots ? budget : c.slots;
    const dim3 grid((most + 63) / 64, c.hkv, c.n_seq);
    if (cache->dtype == DT_F32) evict_move_kernel<float><<<grid, 256, 0, st>>>(c, kept, budget);
    else if (cache->dtype == DT_BF16) evict_move_kernel<bf16_t><<<grid, 256, 0, st>>>(c, kept, budget);
    else evict_move_kernel<f16_t><<<grid, 256, 0, st>>>(c, kept, budget);
    return kv_launched(who);
}
