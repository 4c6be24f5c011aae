// Log-probabilities of given tokens, entropy and the best alternatives of rows of logits (include/poss.h: poss_logprobs).
//
// With m = max x, d = (x - m) / T:  S = sum e^d, log p = d - log S, entropy = log S - sum(e^d d) / S.  Everything is formed from differences to the
// maximum: large logits cancel nothing, and x / T cannot overflow where p has a value (logits 2^128 or more below the largest have none here, at any temperature).
#include "kv.h"

#include <float.h>

namespace poss {

constexpr float LOG2_E = 1.4426950408889634f;

// Bound by memory for many rows (4095 x 32001 bf16, 262 MB: 53 us, 4.9 TB/s), by instructions beside it where alternatives are wanted (61 x 128256 float32, ten of them: 14.6 us for
// 31 MB, some thousand instructions a wave, and 3.9 for the join), by latency for a row (6.5 + 3.3 us).
//
// A row is read once, by one workgroup or by several that share it; each thread keeps S and sum(e^d d) relative to the maximum that its wave has seen.
//
// The best n of a row as 64-bit numbers, larger is better: the value, mapped so that unsigned order is the order of the numbers (NaN 0, -0 as 0), above the
// complement of its id.  Each wave keeps a list of its own in LDS: of its first tile the values from about the n-th largest of its lanes' maxima on (never
// above it), then what exceeds that (tiles ascend, so an equal value loses by its id).  A list too long for another 64 is cut to its n best, whose last is the
// border from then on.  Nothing waits for other waves until the end.  Random rows put a few dozen values there, a rising row every one of them.
// -infinity and NaN are looked for at the end, where fewer than n others are there.
typedef unsigned long long Best;

__device__ __forceinline__ Best best_of(float v, int id) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f), key = v != v ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
    return (Best)key << 32 | (uint32_t)~id;
}
// A number on a wave's list: the value as it is above its id, made comparable when the list is looked at.
__device__ __forceinline__ Best listed(float v, int id) { return (Best)__builtin_bit_cast(uint32_t, v) << 32 | (uint32_t)id; }
__device__ __forceinline__ Best best_of_listed(Best b) { return best_of(__builtin_bit_cast(float, (uint32_t)(b >> 32)), (int)(uint32_t)b); }
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

constexpr int LP_THREADS = 256, LP_PER = 16, LP_TILE = LP_THREADS * LP_PER, LP_LIST = 192, LP_MOST_PARTS = 64;

// A lower bound of the n-th largest of the wave's 64 values, near it (its upper 16 bits as a key); -infinity where fewer than n are above that.
__device__ __forceinline__ float near_nth(float v, int n) {
    const uint32_t key = (uint32_t)(best_of(v, 0) >> 48);
    uint32_t found = 0;
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
        const uint32_t more = found | 1u << bit;
        if (__popcll(__ballot(key >= more)) >= n) found = more;
    }
    return found < 0x80u ? -INFINITY : best_value((Best)found << 48);
}
// A wave's list of `count` numbers (at most LP_LIST), its n best to the front.  All lanes.
__device__ __forceinline__ void cut_list(Best *list, int count, int n) {      // (its numbers as `listed` leaves them)
    const int lane = threadIdx.x & 63;
    Best mine[LP_LIST / 64];
    int rank[LP_LIST / 64];
    wave_lds_sync();
#pragma unroll
    for (int k = 0; k < LP_LIST / 64; ++k) { mine[k] = k * 64 + lane < count ? best_of_listed(list[k * 64 + lane]) : 0; rank[k] = 0; }
    for (int i = 0; i < count; ++i) {
        const Best o = best_of_listed(list[i]);
#pragma unroll
        for (int k = 0; k < LP_LIST / 64; ++k) rank[k] += o > mine[k];
    }
    wave_lds_sync();
#pragma unroll
    for (int k = 0; k < LP_LIST / 64; ++k) if (k * 64 + lane < count && rank[k] < n) list[rank[k]] = listed(best_value(mine[k]), best_id(mine[k]));
    wave_lds_sync();
}
// The n best of list[0 .. count), in order, to room[0 .. n); returns how many there are.  The workgroup, behind a barrier; a barrier at the end.
__device__ __forceinline__ int rank_list(const Best *list, int count, int n, Best *room) {
    for (int at = threadIdx.x; at < count; at += LP_THREADS) {
        const Best mine = list[at];
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += list[j] > mine;
        if (rank < n) room[rank] = mine;
    }
    __syncthreads();
    return count < n ? count : n;
}
// room[have .. n) from the ids [lo, hi): -infinity by id, then NaN by id, then 0.  The workgroup.
template <typename T>
__device__ __forceinline__ void fill_rest(const T *row, int lo, int hi, int have, int n, Best *room, int *red /* 4 */) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int what = 0; what < 2; ++what)
        for (int i0 = lo; i0 < hi && have < n; i0 += LP_THREADS) {
            const int i = i0 + (int)threadIdx.x;
            const float v = i < hi ? to_f(row[i]) : 0.f;
            const bool it = what ? v != v : v == -INFINITY;
            const unsigned long long them = __ballot(it);
            __syncthreads();
            if (lane == 0) red[wave] = __popcll(them);
            __syncthreads();
            int at = have + __popcll(them & ((1ull << lane) - 1));
            for (int w = 0; w < LP_THREADS / 64; ++w) { if (w < wave) at += red[w]; have += red[w]; }
            if (it && at < n) room[at] = best_of(v, i);
        }
    if ((int)threadIdx.x < n && (int)threadIdx.x >= have) room[threadIdx.x] = 0;
    __syncthreads();
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
    constexpr int WAVES = LP_THREADS / 64;
    __shared__ Best lists[TOP == 2 ? WAVES : 1][LP_LIST], joint[TOP == 2 ? WAVES * LP_LIST : WAVES], room[POSS_LOGPROBS_TOP];
    __shared__ float red[3 * WAVES], borders[WAVES];
    __shared__ int joined, found[WAVES];
    const int tid = threadIdx.x;
    const int64_t r = blockIdx.x;
    const float c = LOG2_E / a.temperature;
    // this part's ids [lo, hi); tiles are counted from the 16-byte boundary at or before the row, so that whole pieces are aligned loads, and parts are whole
    // tiles: only a row's first and last one may be less
    const T *row = static_cast<const T *>(a.x) + r * a.ldx;
    const int shift = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T)), start = (int)blockIdx.y * a.per - shift;
    const int lo = max(start, 0), hi = min(a.vocab, start + a.per);
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
            else if (i + E <= lo || i >= hi) raw[v] = (vec)((T)-INFINITY);
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
    Sums q = {-INFINITY, 0.f, 0.f};
    Best *const list = lists[TOP == 2 ? tid >> 6 : 0];     // TOP 2: the wave's list, how long it is, what a value has to exceed
    int count = 0;
    float border = -INFINITY, tops = -INFINITY;            // tops: this lane's maximum
    int tile = 0;
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
            bool equal = false;                            // whether a value may equal the border
            if (i0 == start) { border = near_nth(top, a.n_top); equal = border > -INFINITY; }
            else if (tile > 1 && (tile & (tile - 1)) == 0) border = fmaxf(border, near_nth(tops, a.n_top));      // of 2, 4, 8 .. tiles before: a tile puts fewer on the list
            tops = fmaxf(tops, top);
            ++tile;
            if (__any(equal ? top >= border : top > border)) {
#pragma unroll
                for (int e = 0; e < LP_PER; ++e) {
                    const unsigned long long them = __ballot(equal ? x[e] >= border : x[e] > border);      // (ids outside the part stand as -infinity)
                    if (!them) continue;
                    if (count > LP_LIST - 64) {
                        // its n best, a border that may rise: an equal value of this tile with a lower id can still be to come, so the border of this tile stays
                        cut_list(list, count, a.n_top);
                        count = a.n_top;
                    }
                    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(them >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)them, 0));
                    if (equal ? x[e] >= border : x[e] > border) list[count + before] = listed(x[e], id_of(i0, e));
                    count += __popcll(them);
                }
                if (count > LP_LIST / 2) {
                    cut_list(list, count, a.n_top);
                    count = a.n_top;
                    border = __builtin_bit_cast(float, (uint32_t)(list[a.n_top - 1] >> 32));
                }
            }
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
    q = block_sums<WAVES>(q, c, red);
    if constexpr (TOP > 0) {
        if (TOP == 1) {
            if ((tid & 63) == 0) joint[tid >> 6] = best_of(own_m, best_at);
            __syncthreads();
        } else {
            // each wave has n / WAVES numbers from its border here on, so the lowest of the borders is no more than the part's n-th best
            const float b = near_nth(tops, (a.n_top + WAVES - 1) / WAVES);
            if ((tid & 63) == 0) borders[tid >> 6] = b;
            if (tid == 0) joined = 0;
            __syncthreads();
            float from = borders[0];
            for (int w = 1; w < WAVES; ++w) from = fminf(from, borders[w]);
            for (int i = tid & 63; i < count; i += 64) {
                const Best o = list[i];
                if (__builtin_bit_cast(float, (uint32_t)(o >> 32)) >= from) joint[atomicAdd(&joined, 1)] = best_of_listed(o);
            }
            __syncthreads();
        }
        int have = rank_list(joint, TOP == 1 ? WAVES : joined, a.n_top, room);
        if (TOP == 1 && q.m == -INFINITY) have = 0;
        if (have < a.n_top) fill_rest(row, lo, hi, have, a.n_top, room, found);
    }
    const Best *best = room;
    if (a.parts == 1) return write_row<T>(a, r, q, best);
    const int64_t at = r * a.parts + blockIdx.y;
    if (tid == 0) a.part_sums[at] = q;
    if (tid < a.n_top) a.part_best[at * a.n_top + tid] = best[tid];
}

// Joins a row's parts: a workgroup per row.  Of their best, those from about the n-th largest of the parts' first on can be among the n best.
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_join_kernel(LogprobsArgs a) {
    constexpr int EACH = LP_MOST_PARTS * POSS_LOGPROBS_TOP / LP_THREADS;
    __shared__ Best list[LP_MOST_PARTS * POSS_LOGPROBS_TOP], room[POSS_LOGPROBS_TOP];
    __shared__ Sums joined;
    __shared__ uint32_t from;
    __shared__ int count;
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, n = a.n_top;
    const float c = LOG2_E / a.temperature;
    const Best *best = a.part_best + r * a.parts * n;
    Best mine[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) mine[k] = tid + k * LP_THREADS < a.parts * n ? best[tid + k * LP_THREADS] : 0;
    if (tid < 64) {
        const Sums part = tid < a.parts ? a.part_sums[r * a.parts + tid] : Sums{-INFINITY, 0.f, 0.f};
        uint32_t key = 0, found = 0;
        if (n) {
            key = tid < a.parts ? (uint32_t)(best[tid * n] >> 48) : 0;
            for (int bit = 15; bit >= 0; --bit)
                if (__popcll(__ballot(key >= (found | 1u << bit))) >= n) found |= 1u << bit;
        }
        const Sums q = block_sums<1>(part, c, nullptr);
        if (tid == 0) { joined = q; from = found; count = 0; }
    }
    __syncthreads();
    if (n) {
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            if (tid + k * LP_THREADS < a.parts * n && (uint32_t)(mine[k] >> 48) >= from && mine[k]) list[atomicAdd(&count, 1)] = mine[k];
        __syncthreads();
        rank_list(list, count, n, room);
    }
    write_row<T>(a, r, joined, room);
}

// Parts of a row: as many as give the chip four workgroups a CU, whole tiles each.  (A row that begins off alignment by less than 16 bytes has up to 7 ids more to cover.)
static int logprobs_parts(int rows, int vocab, int *per = nullptr) {
    const int tiles = (vocab + 7 + LP_TILE - 1) / LP_TILE;
    int p = rows ? 1024 / rows : 1;
    p = p < tiles ? p : tiles;
    p = p < 1 ? 1 : p > LP_MOST_PARTS ? LP_MOST_PARTS : p;
    const int each = (tiles + p - 1) / p;
    if (per) *per = each * LP_TILE;
    return (tiles + each - 1) / each;
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
    if (!(temperature >= FLT_MIN) || !(temperature < INFINITY)) return set_error(POSS_E_INVALID_ARG, "%s: temperature must be a positive number, not a subnormal one", who);
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
