// Log-probabilities of given tokens, entropy and the best alternatives of rows of logits (include/poss.h: poss_logprobs).
//
// With m = max x, d = (x - m) / T:  S = sum e^d, log p = d - log S, entropy = log S - sum(e^d d) / S.  Everything is formed from differences to the
// maximum: large logits cancel nothing, and x / T cannot overflow where p has a value.
#include "kv.h"

namespace poss {

constexpr float LOG2_E = 1.4426950408889634f;

// A row is read once, by one workgroup or by several that share it; each thread keeps S and sum(e^d d) relative to the maximum that its wave has seen.
//
// The best n of a row as 64-bit numbers, larger is better: the value, mapped so that unsigned order is the order of the numbers (NaN 0, -0 as 0), above the
// complement of its id.  A tile's values that can still be among them go to a list in LDS: those above the n-th best so far (tiles ascend, so an equal value loses by its
// id); at first, those from the n-th largest of the threads' maxima on, which is no more than the n-th best.  A list too long for another tile is
// cut to its n best.  Random rows put a few dozen values there, a rising row every one of them.
typedef unsigned long long Best;

__device__ __forceinline__ Best best_of(float v, int id) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f), key = v != v ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
    return (Best)key << 32 | (uint32_t)~id;
}
__device__ __forceinline__ int best_id(Best b) { return (int)~(uint32_t)b; }
__device__ __forceinline__ float best_value(Best b) {
    const uint32_t key = (uint32_t)(b >> 32);
    return key == 0 ? NAN : __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// m: the largest logit seen (-infinity: none), s: sum 2^((x - m) c), t: sum of the same times (x - m) c;  c = log2(e) / temperature.
struct Sums { float m, s, t; };

__device__ __forceinline__ Sums add_sums(Sums a, Sums b, float c) {
    const float m = fmaxf(a.m, b.m);
    Sums r = {m, 0.f, 0.f};
    if (a.m != -INFINITY || a.s != a.s) { const float d = fmaxf((a.m - m) * c, -1e4f), f = __builtin_amdgcn_exp2f((a.m - m) * c); r.s += a.s * f; r.t += (a.t + a.s * d) * f; }
    if (b.m != -INFINITY || b.s != b.s) { const float d = fmaxf((b.m - m) * c, -1e4f), f = __builtin_amdgcn_exp2f((b.m - m) * c); r.s += b.s * f; r.t += (b.t + b.s * d) * f; }
    return r;
}
// The sums of all threads (first WAVES waves of a workgroup), to every thread: all brought to the largest maximum, then added.
template <int WAVES>
__device__ __forceinline__ Sums block_sums(Sums q, float c, float *red /* 3 * WAVES */) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto all = [&](float v, float *at, bool largest) {
        v = largest ? wave_max(v) : wave_sum(v);
        if constexpr (WAVES > 1) {
            if (lane == 0) at[wave] = v;
            __syncthreads();
            v = at[0];
            for (int w = 1; w < WAVES; ++w) v = largest ? fmaxf(v, at[w]) : v + at[w];
        }
        return v;
    };
    const float m = all(q.m, red, true);
    const Sums r = add_sums(q, Sums{m, 0.f, 0.f}, c);
    return Sums{m, all(r.s, red + WAVES, false), all(r.t, red + 2 * WAVES, false)};
}

constexpr int LP_THREADS = 256, LP_PER = 16, LP_TILE = LP_THREADS * LP_PER, LP_LIST = 768, LP_MOST_PARTS = 64;

// The n best of list[0 .. count) to the front, in order; the rest of the first n are 0.  All threads; barriers on both sides.
__device__ __forceinline__ void keep_best(Best *list, int count, int n, Best *room /* POSS_LOGPROBS_TOP + 8 */) {
    const int tid = threadIdx.x;
    __syncthreads();
    if (count <= LP_THREADS) {                             // a thread per number: how many are better
        const Best mine = tid < count ? list[tid] : 0;
        int rank = 0;
        for (int i = 0; i < count; ++i) rank += list[i] > mine;
        if (tid < n) room[tid] = 0;
        __syncthreads();
        if (tid < count && rank < n) room[rank] = mine;
    } else {
        Best last = ~0ull;
        for (int j = 0; j < n; ++j) {
            Best top = 0;
            for (int i = tid; i < count; i += LP_THREADS) { const Best b = list[i]; if (b < last && b > top) top = b; }
            for (int o = 32; o; o >>= 1) { const Best b = __shfl_xor(top, o); if (b > top) top = b; }
            if ((tid & 63) == 0) room[POSS_LOGPROBS_TOP + (j & 1) * 4 + (tid >> 6)] = top;
            __syncthreads();
            for (int v = 0; v < 4; ++v) { const Best b = room[POSS_LOGPROBS_TOP + (j & 1) * 4 + v]; if (b > top) top = b; }
            last = top;
            if (tid == 0) room[j] = top;
        }
    }
    __syncthreads();
    if (tid < n) list[tid] = room[tid];
    __syncthreads();
}
// The n-th largest of 64 numbers, the largest of four neighbouring threads' each (n <= 64), in every thread: no more than the n-th largest of what they stand for.
__device__ __forceinline__ float nth_of_threads(float v, int n, float *all /* 65 */) {
    v = fmaxf(v, xor1(v));
    v = fmaxf(v, xor2(v));
    if ((threadIdx.x & 3) == 0) all[threadIdx.x >> 2] = v;
    __syncthreads();
    if (threadIdx.x < 64) {
        v = all[threadIdx.x];
        int above = 0, least = 0;
        for (int i = 0; i < 64; ++i) { const float o = lane_value(v, i); above += o > v; least += o >= v; }
        if (above < n && least >= n) all[64] = v;          // (equal ones write the same)
    }
    __syncthreads();
    return all[64];
}

struct LogprobsArgs {
    const void *x; int64_t ldx; int vocab, parts, per; float temperature;      // per: ids of a part
    const int32_t *tokens; int n_tokens; float *logp, *entropy;
    int n_top; int32_t *top_ids; float *top_logp;
    Sums *part_sums; Best *part_best;           // [rows][parts], [rows][parts][n_top]
};

// What a row's sums and best ids give.
template <typename T>
__device__ __forceinline__ void write_row(const LogprobsArgs &a, int64_t r, Sums q, const Best *best) {
    const T *row = static_cast<const T *>(a.x) + r * a.ldx;
    const float log_s = logf(q.s);                         // NaN where a logit is NaN or +infinity; -infinity, and x - m NaN, where none is above -infinity
    if (threadIdx.x == 0 && a.entropy) a.entropy[r] = log_s - q.t * 0.6931471805599453f / q.s;
    for (int j = threadIdx.x; j < a.n_tokens; j += LP_THREADS) {
        const int id = a.tokens[r * a.n_tokens + j];
        a.logp[r * a.n_tokens + j] = (unsigned)id < (unsigned)a.vocab ? (to_f(row[id]) - q.m) / a.temperature - log_s : NAN;
    }
    if ((int)threadIdx.x < a.n_top) {
        const Best b = best[threadIdx.x];
        a.top_ids[r * a.n_top + threadIdx.x] = best_id(b);
        a.top_logp[r * a.n_top + threadIdx.x] = (best_value(b) - q.m) / a.temperature - log_s;
    }
}

// A workgroup per row and part of it.  TOP: 0 no alternatives, 1 one (each wave keeps its best), 2 up to POSS_LOGPROBS_TOP.
template <typename T, int TOP>
__global__ void __launch_bounds__(LP_THREADS) logprobs_kernel(LogprobsArgs a) {
    constexpr int E = 16 / sizeof(T), VECS = LP_PER / E;
    typedef T vec __attribute__((ext_vector_type(E)));
    __shared__ Best list[TOP == 2 ? LP_LIST : 1], room[POSS_LOGPROBS_TOP + 8];
    __shared__ float all[65], red[12];
    __shared__ int count;
    const int tid = threadIdx.x;
    const int64_t r = blockIdx.x;
    const float c = LOG2_E / a.temperature;
    // this part's ids [lo, hi); tiles are counted from the 16-byte boundary at or before lo, so that whole pieces are aligned loads
    const T *row = static_cast<const T *>(a.x) + r * a.ldx;
    const int lo = (int)blockIdx.y * a.per, hi = min(a.vocab, lo + a.per);
    const int start = lo - (int)(reinterpret_cast<uintptr_t>(row + lo) % 16 / sizeof(T));
    auto whole = [&](int i0) { return i0 >= lo && i0 + LP_TILE <= hi; };
    auto fetch = [&](int i0, vec *raw) {                   // the pieces of this thread in the whole tile at id i0
#pragma unroll
        for (int v = 0; v < VECS; ++v) raw[v] = *reinterpret_cast<const vec *>(row + i0 + (v * LP_THREADS + tid) * E);
    };
    auto fetch_guarded = [&](int i0, vec *raw) {           // a tile that begins before lo or ends behind hi
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            const int i = i0 + (v * LP_THREADS + tid) * E;
            if (i >= lo && i + E <= hi) raw[v] = *reinterpret_cast<const vec *>(row + i);
            else {                                         // its values one by one, all asked for before the first is waited for
                T at[E];
#pragma unroll
                for (int e = 0; e < E; ++e) at[e] = row[min(max(i + e, lo), hi - 1)];
#pragma unroll
                for (int e = 0; e < E; ++e) raw[v][e] = i + e >= lo && i + e < hi ? at[e] : (T)-INFINITY;
            }
        }
    };
    auto id_of = [&](int i0, int e) { return i0 + (e / E * LP_THREADS + tid) * E + e % E; };
    if (tid == 0) count = 0;
    Sums q = {-INFINITY, 0.f, 0.f};
    float border = -INFINITY;                              // TOP 2: what a value has to exceed; NaN: any value may pass
    int best_at = 0;                                       // TOP 1: the lowest id with the wave's maximum
    auto take = [&](int i0, const vec *raw) {
        float x[LP_PER];
#pragma unroll
        for (int e = 0; e < LP_PER; ++e) x[e] = to_f(raw[e / E][e % E]);
        float top = -INFINITY;                             // (of what is a number)
#pragma unroll
        for (int e = 0; e < LP_PER; ++e) top = fmaxf(top, x[e]);
        // the reference is the wave's maximum: few tiles of a row have a new one, where nearly every tile has a new one for some thread of 64
        if (__any(top > q.m)) {
            const float m = wave_max(top);
            q = add_sums(q, Sums{m, 0.f, 0.f}, c);
            if constexpr (TOP == 1) {
                best_at = INT32_MAX;
#pragma unroll
                for (int e = LP_PER - 1; e >= 0; --e) best_at = x[e] == m ? id_of(i0, e) : best_at;
                for (int o = 32; o; o >>= 1) best_at = min(best_at, __shfl_xor(best_at, o));
            }
        }
        const float ref = q.m == -INFINITY ? 0.f : q.m;
#pragma unroll
        for (int e = 0; e < LP_PER; ++e) {
            const float d = (x[e] - ref) * c, p = __builtin_amdgcn_exp2f(d);
            q.s += p;
            q.t += p * fmaxf(d, -1e4f);
        }
        if constexpr (TOP == 2) {
            const bool first = i0 == start;
            float from = border;
            if (first) from = nth_of_threads(top, a.n_top, all);
            const bool any = first ? from == -INFINITY : border != border;
            uint32_t passes = 0;
            if (any || (first ? top >= from : top > from)) {
#pragma unroll
                for (int e = 0; e < LP_PER; ++e) {
                    const int i = id_of(i0, e);
                    if (i >= lo && i < hi && (any || (first ? x[e] >= from : x[e] > from))) passes |= 1u << e;
                }
            }
            const int have = count;                        // (nobody adds before the barrier below)
            __syncthreads();
            int at = passes ? atomicAdd(&count, __builtin_popcount(passes)) : 0;
            __syncthreads();
            int n = count;
            if (n <= LP_LIST) {
                if (passes)
#pragma unroll
                    for (int e = 0; e < LP_PER; ++e) if (passes >> e & 1) list[at++] = best_of(x[e], id_of(i0, e));
            } else {                                       // too many at once: one of each thread at a time
                __syncthreads();
                if (tid == 0) count = have;
                __syncthreads();
#pragma unroll 1
                for (int e = 0; e < LP_PER; ++e) {
                    if (count > LP_LIST - LP_THREADS) {
                        keep_best(list, count, a.n_top, room);
                        if (tid == 0) count = a.n_top;
                    }
                    __syncthreads();
                    float xe = x[0];
#pragma unroll
                    for (int k = 1; k < LP_PER; ++k) xe = e == k ? x[k] : xe;
                    if (passes >> e & 1) list[atomicAdd(&count, 1)] = best_of(xe, id_of(i0, e));
                    __syncthreads();
                }
                n = count;
            }
            if (first || n > LP_LIST / 2 || i0 + LP_TILE >= hi) {
                keep_best(list, n, a.n_top, room);
                border = best_value(list[a.n_top - 1]);
                if (tid == 0) count = a.n_top;
            }
            __syncthreads();
        }
    };
    for (int i0 = start; i0 < hi;) {
        vec raw[VECS];
        if (!whole(i0)) {
            fetch_guarded(i0, raw);
            take(i0, raw);
            i0 += LP_TILE;
            continue;
        }
        fetch(i0, raw);
        for (bool more = true; more; i0 += LP_TILE) {      // the next whole tile is under way while one is summed
            vec next[VECS];
            more = whole(i0 + LP_TILE);
            fetch(more ? i0 + LP_TILE : i0, next);
            take(i0, raw);
#pragma unroll
            for (int v = 0; v < VECS; ++v) raw[v] = next[v];
        }
    }
    const float own_m = q.m;
    q = block_sums<LP_THREADS / 64>(q, c, red);
    const Best *best = list;
    if constexpr (TOP == 1) {
        Best mine = own_m > -INFINITY ? best_of(own_m, best_at) : 0;
        if (q.m == -INFINITY)                              // nothing but -infinity and NaN
            for (int i = lo + tid; i < hi; i += LP_THREADS) { const Best b = best_of(to_f(row[i]), i); if (b > mine) mine = b; }
        for (int o = 32; o; o >>= 1) { const Best b = __shfl_xor(mine, o); if (b > mine) mine = b; }
        if ((tid & 63) == 0) room[4 + (tid >> 6)] = mine;
        __syncthreads();
        if (tid == 0) { for (int v = 0; v < 4; ++v) if (room[4 + v] > mine) mine = room[4 + v]; room[0] = mine; }      // (thread 0 alone reads it)
        best = room;
    }
    if (a.parts == 1) return write_row<T>(a, r, q, best);
    const int64_t at = r * a.parts + blockIdx.y;
    if (tid == 0) a.part_sums[at] = q;
    if (tid < a.n_top) a.part_best[at * a.n_top + tid] = best[tid];
}

// Joins a row's parts: a workgroup per row.  Of their best, those from the n-th largest of the parts' first on can be among the n best.
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_join_kernel(LogprobsArgs a) {
    __shared__ Best list[LP_MOST_PARTS * POSS_LOGPROBS_TOP], room[POSS_LOGPROBS_TOP + 8];
    __shared__ Sums joined;
    __shared__ int count;
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, n = a.n_top;
    const float c = LOG2_E / a.temperature;
    if (tid == 0) count = 0;
    if (tid < 64) {
        const Sums q = block_sums<1>(tid < a.parts ? a.part_sums[r * a.parts + tid] : Sums{-INFINITY, 0.f, 0.f}, c, nullptr);
        if (tid == 0) joined = q;
    }
    __syncthreads();
    if (n) {
        const Best *best = a.part_best + r * a.parts * n;
        Best from = 0;
        if (n <= a.parts) {
            Best first = 0;
            if (tid < a.parts) first = best[tid * n];
            if (tid < a.parts) list[tid] = first;
            __syncthreads();
            int rank = 0;
            for (int i = 0; i < a.parts; ++i) rank += list[i] > first || (list[i] == first && i < tid);
            if (tid < a.parts && rank == n - 1) room[0] = first;
            __syncthreads();
            from = room[0];
            __syncthreads();
        }
        for (int i = tid; i < a.parts * n; i += LP_THREADS) {
            const Best b = best[i];
            if (b >= from) list[atomicAdd(&count, 1)] = b;
        }
        __syncthreads();
        keep_best(list, count, n, room);
    }
    write_row<T>(a, r, joined, list);
}

// Parts of a row: as many as give the chip two thousand workgroups, none of less than a tile.  per: ids of each, whole pieces of 16 bytes.
static int logprobs_parts(int rows, int vocab, int *per = nullptr) {
    int p = rows ? 2048 / rows : 1;
    const int most = (vocab + LP_TILE - 1) / LP_TILE;
    p = p < most ? p : most;
    p = p < 1 ? 1 : p > LP_MOST_PARTS ? LP_MOST_PARTS : p;
    const int ids = ((vocab + p - 1) / p + 7) / 8 * 8;
    if (per) *per = ids;
    return (vocab + ids - 1) / ids;
}

template <typename T>
static void launch_logprobs(const LogprobsArgs &a, int rows, hipStream_t st) {
    const dim3 grid(rows, a.parts);
    if (a.n_top == 0) logprobs_kernel<T, 0><<<grid, LP_THREADS, 0, st>>>(a);
    else if (a.n_top == 1) logprobs_kernel<T, 1><<<grid, LP_THREADS, 0, st>>>(a);
    else logprobs_kernel<T, 2><<<grid, LP_THREADS, 0, st>>>(a);
    if (a.parts > 1) logprobs_join_kernel<T><<<rows, LP_THREADS, 0, st>>>(a);
}

}  // namespace poss

// ------------------------------------------------------------------------------------------ C entry points (include/poss.h)
using namespace poss;

namespace {
bool logprobs_ok(int32_t rows, int32_t vocab, int32_t n_top) { return rows >= 0 && rows <= 1 << 23 && vocab >= 1 && vocab <= 1 << 30 && n_top >= 0 && n_top <= POSS_LOGPROBS_TOP && n_top <= vocab; }
size_t sums_bytes(int32_t rows, int parts) { return ((size_t)rows * parts * sizeof(Sums) + 255) / 256 * 256; }
}  // namespace

extern "C" {

size_t poss_logprobs_scratch_bytes(int32_t rows, int32_t vocab, int32_t n_top) {
    if (!logprobs_ok(rows, vocab, n_top)) return 0;
    const int parts = logprobs_parts(rows, vocab);
    return parts == 1 ? 256 : 256 + sums_bytes(rows, parts) + (size_t)rows * parts * n_top * sizeof(Best);
}

int poss_logprobs(int32_t dtype, const void *x, int64_t ldx, int32_t rows, int32_t vocab, float temperature, const int32_t *tokens, int32_t n_tokens, float *logp, float *entropy,
                  int32_t n_top, int32_t *top_ids, float *top_logp, void *scratch, size_t scratch_bytes, void *hip_stream) {
    const char *who = "poss_logprobs";
    if (kv_bad_dtype(dtype) || !logprobs_ok(rows, vocab, n_top) || n_tokens < 0 || (rows > 1 && ldx < vocab)) return set_error(POSS_E_INVALID_ARG, "%s: bad shape or type", who);
    if (!(temperature > 0) || !(temperature < INFINITY)) return set_error(POSS_E_INVALID_ARG, "%s: temperature must be positive", who);
    if (rows == 0) return POSS_OK;
    if (!x || !scratch || (n_tokens && (!tokens || !logp)) || (n_top && (!top_ids || !top_logp))) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    if (!kv_aligned(x, dtype_size(dtype)) || !kv_aligned(tokens, 4) || !kv_aligned(logp, 4) || !kv_aligned(entropy, 4) || !kv_aligned(top_ids, 4) || !kv_aligned(top_logp, 4))
        return set_error(POSS_E_INVALID_ARG, "%s: an array is not aligned to its type", who);
    if (!kv_aligned(scratch, 256)) return set_error(POSS_E_INVALID_ARG, "%s: scratch must be aligned to 256 bytes", who);
    const size_t need = poss_logprobs_scratch_bytes(rows, vocab, n_top);
    if (scratch_bytes < need) return set_error(POSS_E_CAPACITY, "%s: rows=%d vocab=%d n_top=%d needs %zu bytes of scratch, got %zu", who, rows, vocab, n_top, need, scratch_bytes);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    int per;
    const int parts = logprobs_parts(rows, vocab, &per);
    char *base = static_cast<char *>(scratch);
    const LogprobsArgs a{x, ldx, vocab, parts, per, temperature, tokens, n_tokens, logp, entropy, n_top, top_ids, top_logp, reinterpret_cast<Sums *>(base),
                         reinterpret_cast<Best *>(base + sums_bytes(rows, parts))};
    if (dtype == DT_F32) launch_logprobs<float>(a, rows, st);
    else if (dtype == DT_BF16) launch_logprobs<bf16_t>(a, rows, st);
    else launch_logprobs<f16_t>(a, rows, st);
    return kv_launched(who);
}

}  // extern "C"
