// Attention of one new token per sequence over a paged cache (include/poss.h: poss_kv_attend).
//
// Online softmax in the log2 domain: a wave keeps, per query head, the maximum m of its scores z = scale * log2(e) * q.k, l = sum 2^(z-m) and
// O = sum 2^(z-m) v; two such triples join as m = max, l and O scaled by 2^(m_i - m) and added.  out = O / l, lse = (m + log2 l) * ln 2.
// What bounds it: keys and values are read once; the matrix instructions, of whose 16 columns the heads that share a key head use theirs, have ten times the rate that
// is wanted.  Operands go straight from the pages into registers.  One row of 131072 slots, 8 key heads of 128, bf16 (537 MB): 95 us, 5.7 TB/s, and 5.7 us for the join; 64 ragged
// rows of up to 8192 with weights 225 + 14.6 us.  A second block on its way while one is worked on takes half of the waves a CU holds and is slower (102 -> 105 us, 40 key heads
// 74 -> 82); so are three waves a SIMD with fewer registers (102 -> 108).
//
// Work is cut along the batch's slots laid end to end, in blocks of 32: workgroup w of a key head takes blocks [w T / W, (w + 1) T / W) of all T, so
// that ragged batches are even without the host knowing a length.  A row that lies in one workgroup is written there; pieces of others
// go to scratch (at most two a workgroup: the end of a row that began before, the beginning of one that goes on) and are joined in order by a second launch.
#include "kv.h"

namespace poss {

typedef float  f32x4 __attribute__((ext_vector_type(4)));

constexpr int ATT_BLOCK = 32;                 // slots of a block: never across pages
constexpr int ATT_WAVES = 4;
constexpr int ATT_LEAST = 2, ATT_MOST = 512;   // blocks of a workgroup at least, workgroups of a launch at most
constexpr int ATT_ROW = 2 * ATT_WAVES;        // blocks of a row that one workgroup takes
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct AttendArgs {
    int hq, tiles;        // tiles: groups of 16 query heads of a key head
    const void *q; int64_t q_row; void *out; int64_t out_row;
    const int32_t *lengths; int max_len; float scale;
    float *lse; const float *weights; float *weights_out;
    int W;                // workgroups along the batch's slots; 0: one for each row
    float *part;          // [2 W][hkv * tiles][16][dh]
    float2 *part_ml;      // [2 W][hkv * tiles][16]
    float *scores; int64_t score_row;   // [n_seq][hq][score_row], log2 domain
    float *row_lse;       // [n_seq][hq], log2 domain: of rows that lie in one workgroup
};

// Blocks of a row; one whose length is beyond the bound has none and is NaN.
__device__ __forceinline__ int row_blocks(int len, int max_len) { return len <= 0 || len > max_len ? 0 : (len + ATT_BLOCK - 1) / ATT_BLOCK; }

// Workgroups that the slots are cut among: no more than W, and none with less than ATT_LEAST blocks' worth.
__device__ __forceinline__ int64_t attend_parts(int64_t all, int W) {
    const int64_t p = (all + ATT_LEAST - 1) / ATT_LEAST;
    return p < W ? p : W;
}

// a * b / c, rounded down: in 32 bits where they hold it (a 64-bit division takes some hundred instructions).
__device__ __forceinline__ int64_t times_over(int64_t a, int64_t b, int64_t c) {
    if (a < 1 << 20 && b <= 1 << 10) return (uint32_t)a * (uint32_t)b / (uint32_t)c;
    return a * b / c;
}
// Sum over the wave's lanes up to this one (64 rows' blocks fit: a row has 2^25 at most).
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    for (int o = 1; o < 64; o <<= 1) { const uint32_t y = __shfl_up(x, o); if ((int)(threadIdx.x & 63) >= o) x += y; }
    return x;
}
// The batch's rows as blocks laid end to end, by every wave for itself.  Up to 64 rows are looked at once: x and end are lane i's blocks and those up to it; of more, a
// pass for the sum comes first.
struct Batch { int64_t all; uint32_t x, end; };
__device__ __forceinline__ Batch count_blocks(const int32_t *lengths, int n, int max_len) {
    const int lane = threadIdx.x & 63;
    Batch r{0, 0, 0};
    if (n == 1) { r.x = r.end = row_blocks(lengths[0], max_len); r.all = r.x; return r; }
    if (n <= 64) {
        r.x = lane < n ? row_blocks(lengths[lane], max_len) : 0;
        r.end = wave_scan(r.x);
        r.all = (uint32_t)__builtin_amdgcn_readlane(r.end, 63);
        return r;
    }
    int64_t a = 0;
    for (int i = lane; i < n; i += 64) a += row_blocks(lengths[i], max_len);
    for (int o = 32; o; o >>= 1) a += __shfl_xor(a, o);
    r.all = a;
    return r;
}
// Blocks before row b.
__device__ __forceinline__ int64_t blocks_before(const Batch &r, const int32_t *lengths, int n, int max_len, int b) {
    if (n == 1) return 0;
    if (n <= 64) return (uint32_t)__builtin_amdgcn_readlane(r.end - r.x, b);
    int64_t a = 0;
    for (int i = threadIdx.x & 63; i < b; i += 64) a += row_blocks(lengths[i], max_len);
    for (int o = 32; o; o >>= 1) a += __shfl_xor(a, o);
    return a;
}
// The row that holds block `at` (0 <= at < all) and its first block.
__device__ __forceinline__ void find_row(const Batch &r, const int32_t *lengths, int n, int max_len, int64_t at, int &row, int64_t &first) {
    row = 0; first = 0;
    if (n == 1) return;
    int64_t base = 0;
    for (int i0 = 0; i0 < n; i0 += 64) {
        const int i = i0 + (int)(threadIdx.x & 63);
        const uint32_t x = n <= 64 ? r.x : i < n ? row_blocks(lengths[i], max_len) : 0, end = n <= 64 ? r.end : wave_scan(x);
        const unsigned long long past = __ballot(base + end > at);
        if (past) {
            const int lane = __ffsll(past) - 1;
            row = i0 + lane;
            first = base + (uint32_t)__builtin_amdgcn_readlane(end - x, lane);
            return;
        }
        base += (uint32_t)__builtin_amdgcn_readlane(end, 63);
    }
}

// What a wave does with a block of 32 slots, 16-bit types.  Scores: K as the A operand, its rows ordered so that the lane of group g = lane / 16 gets the scores of slots
// 8g .. 8g + 7 for head lane % 16 - the B operand of O^T = V^T P^T as it stands.
template <typename T, int DH> struct Tile {
    typedef T x8 __attribute__((ext_vector_type(8)));
    x8 q[DH / 32], k[2][DH / 32], v[DH / 16];
    static __device__ __forceinline__ int slot_of(int j) { return 8 * ((threadIdx.x & 63) >> 4) + j; }
    __device__ __forceinline__ void load_q(const T *row, bool there) {
        const int g = (threadIdx.x & 63) >> 4;
        for (int s = 0; s < DH / 32; ++s) q[s] = there ? *reinterpret_cast<const x8 *>(row + 32 * s + 8 * g) : x8{};
    }
    __device__ __forceinline__ void load(const T *kb, const T *vb, int P) {
        const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const T *row = kb + (8 * (i >> 2) + 4 * t + (i & 3)) * DH + 8 * g;
#pragma unroll
            for (int s = 0; s < DH / 32; ++s) k[t][s] = *reinterpret_cast<const x8 *>(row + 32 * s);
        }
#pragma unroll
        for (int d = 0; d < DH / 16; ++d) v[d] = *reinterpret_cast<const x8 *>(vb + (16 * d + i) * P + 8 * g);
    }
    static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) {
        if constexpr (sizeof(T) == 2 && __is_same(T, bf16_t)) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    __device__ __forceinline__ void scores(float *z) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < DH / 32; ++s) c = mfma(k[t][s], q[s], c);
            for (int r = 0; r < 4; ++r) z[4 * t + r] = c[r];
        }
    }
    __device__ __forceinline__ void clear_beyond(int n) {        // what lies behind the length may be anything
#pragma unroll
        for (int d = 0; d < DH / 16; ++d)
            for (int j = 0; j < 8; ++j) if (slot_of(j) >= n) v[d][j] = (T)0.f;
    }
    // A probability enters as the sum of two 16-bit numbers: rounded once to 8 bits (bf16) it alone would be off by more than the result's half step.  fp16
    // holds numbers below 2^-14 with fewer bits: there probabilities, and their sum with them, are 2^12 times larger (lift()), so that those of 2^-26 of the largest have all.
    __device__ __forceinline__ void add_values(const float *p, f32x4 *o) const {
        x8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) { hi[j] = (T)p[j]; lo[j] = (T)(p[j] - (float)hi[j]); }
#pragma unroll
        for (int d = 0; d < DH / 16; ++d) { o[d] = mfma(v[d], hi, o[d]); o[d] = mfma(v[d], lo, o[d]); }
    }
};
// float32: the instruction of four products deep; slot 4g + r (r < 4) and 16 + 4g + r.
template <int DH> struct Tile<float, DH> {
    f32x4 q[DH / 16], k[2][DH / 16], v[2][DH / 16];
    static __device__ __forceinline__ int slot_of(int j) { return 16 * (j >> 2) + 4 * ((threadIdx.x & 63) >> 4) + (j & 3); }
    __device__ __forceinline__ void load_q(const float *row, bool there) {
        const int g = (threadIdx.x & 63) >> 4;
        for (int s = 0; s < DH / 16; ++s) q[s] = there ? *reinterpret_cast<const f32x4 *>(row + 16 * s + 4 * g) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void load(const float *kb, const float *vb, int P) {
        const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int s = 0; s < DH / 16; ++s) k[t][s] = *reinterpret_cast<const f32x4 *>(kb + (16 * t + i) * DH + 16 * s + 4 * g);
#pragma unroll
            for (int d = 0; d < DH / 16; ++d) v[t][d] = *reinterpret_cast<const f32x4 *>(vb + (16 * d + i) * P + 16 * t + 4 * g);
        }
    }
    __device__ __forceinline__ void scores(float *z) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < DH / 16; ++s)
                for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][s][j], q[s][j], c, 0, 0, 0);
            for (int r = 0; r < 4; ++r) z[4 * t + r] = c[r];
        }
    }
    __device__ __forceinline__ void clear_beyond(int n) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
            for (int d = 0; d < DH / 16; ++d)
                for (int r = 0; r < 4; ++r) if (slot_of(4 * t + r) >= n) v[t][d][r] = 0.f;
    }
    __device__ __forceinline__ void add_values(const float *p, f32x4 *o) const {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int d = 0; d < DH / 16; ++d) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[t][d][r], p[4 * t + r], o[d], 0, 0, 0);
    }
};

template <typename T> constexpr float lift() { return __is_same(T, f16_t) ? 12.f : 0.f; }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
// 2^(m - to) for a running maximum that may be -infinity (nothing yet: 0).
__device__ __forceinline__ float back_by(float m, float to) { return m == -INFINITY ? 0.f : exp2_of(m - to); }

__device__ __forceinline__ bool any_nan(f32x4 o) { return __builtin_isunordered(o[0], o[1]) || __builtin_isunordered(o[2], o[3]); }
// An infinite value counts as such wherever its score is above -infinity.  Where its probability, the second number that stands for it or a factor on the way is 0, or that
// number is below 0, NaN has come of it.  So this is what a sum over the slots s0 .. s1 - 1 has to be that is NaN while the probabilities are not: the infinities and NaN among
// the values (row d) times 1, or times 0 where the score is -infinity.  (If there are none it is left: numbers whose sums float32 does not hold.)  A thread looks through the
// slots by itself, which costs the tiles nothing (131072 slots of 8 key heads: 0.18 ms with one infinity, 0.49 with a slot of them, for 0.1); to take their blocks once
// more, with such values apart, cost every call 0.2 to 0.5 us.
template <typename T, int DH>
__device__ __forceinline__ float sum_of_infinities(const T *q, const KvView &c, const int32_t *table, int hk, int d, int s0, int s1, float scale) {
    constexpr int E = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(E)));
    float sum = 0.f;
#pragma unroll 1
    for (int s = s0; s < s1 && sum == sum; s += E) {           // (s0 is a block's first slot)
        const int page = table[s >> c.shift];                  // (there: the row's probabilities are numbers)
        const T *v = static_cast<const T *>(c.v) + kv_value_at(c, page, hk, d, s), *k = static_cast<const T *>(c.k) + kv_key_at(c, page, hk, s);
        const vec x = *reinterpret_cast<const vec *>(v);
        bool numbers = true;
#pragma unroll
        for (int e = 0; e < E; ++e) numbers &= fabsf(to_f(x[e])) < INFINITY;
        if (numbers) continue;
#pragma unroll 1
        for (int e = 0; e < min(E, s1 - s); ++e) {
            if (fabsf(to_f(v[e])) < INFINITY) continue;
            float z = 0.f;
#pragma unroll 1
            for (int i = 0; i < DH; ++i) z += to_f(q[i]) * to_f(k[e * DH + i]);
            sum += to_f(v[e]) * (z * scale == -INFINITY ? 0.f : 1.f);
        }
    }
    return sum == 0.f ? NAN : sum;
}
// A piece's sums brought to another maximum; an infinity stays one, however small the factor.
__device__ __forceinline__ f32x4 brought(f32x4 o, float f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fabsf(o[e]) == INFINITY ? o[e] : o[e] * f;
    return o;
}

template <typename T, int DH, bool WEIGHED>
__global__ void __launch_bounds__(64 * ATT_WAVES) attend_kernel(KvView c, AttendArgs a) {
    constexpr int ROW = DH + 4;
    __shared__ float lds_o[ATT_WAVES * 16 * ROW];
    __shared__ float2 lds_ml[ATT_WAVES][16];
    __shared__ float lds_lse[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g4 = lane >> 4;
    const int w = blockIdx.x, hk = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles;
    const int group = a.hq / c.hkv, head0 = hk * group + tile * 16, heads = min(16, group - tile * 16);
    const T *ks = static_cast<const T *>(c.k), *vs = static_cast<const T *>(c.v), *qs = static_cast<const T *>(a.q);
    T *out = static_cast<T *>(a.out);
    const int P = 1 << c.shift;
    const bool by_rows = a.W == 0;                             // a workgroup is a row
    // rows without a block are nobody's: workgroup b % W writes row b
    for (int b = w; b < c.n_seq; b += by_rows ? c.n_seq : a.W) {
        const int len = a.lengths[b];
        if (row_blocks(len, a.max_len)) continue;
        for (int i = threadIdx.x; i < heads * DH; i += 64 * ATT_WAVES) out[b * a.out_row + (int64_t)head0 * DH + i] = from_f<T>(len > 0 ? NAN : 0.f);
        if ((int)threadIdx.x < heads && a.lse) a.lse[(int64_t)b * a.hq + head0 + threadIdx.x] = len > 0 ? NAN : -INFINITY;
    }
    int64_t at = 0, end, first = 0;
    int b = w;
    if (by_rows) end = row_blocks(a.lengths[w], a.max_len);
    else {
        const Batch batch = count_blocks(a.lengths, c.n_seq, a.max_len);
        const int64_t parts = attend_parts(batch.all, a.W);
        if (w >= parts) return;
        at = times_over(batch.all, w, parts);
        end = times_over(batch.all, w + 1, parts);
        find_row(batch, a.lengths, c.n_seq, a.max_len, at, b, first);
    }
    const float scale = a.scale * LOG2E;
    Tile<T, DH> t;
    while (at < end) {
        const int len = a.lengths[b], blocks = row_blocks(len, a.max_len);
        if (at >= first + blocks) { first += blocks; ++b; continue; }          // (an empty row)
        const int i0 = (int)(at - first), i1 = (int)(first + blocks < end ? blocks : end - first);
        t.load_q(qs + b * a.q_row + (int64_t)(head0 + col) * DH, col < heads);
        float m = -INFINITY, l = 0.f;
        f32x4 o[DH / 16];
        for (int d = 0; d < DH / 16; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int32_t *table = c.table + (int64_t)b * c.table_stride;
        float *score = WEIGHED ? a.scores + ((int64_t)b * a.hq + head0 + col) * a.score_row : nullptr;
        // this wave's blocks: every fourth; the pages of 64 of them are looked up at once
        for (int i64 = i0 + wave; i64 < i1; i64 += 64 * ATT_WAVES) {
            const int mine = i64 + lane * ATT_WAVES;
            const int looked = mine < i1 ? table[(mine * ATT_BLOCK) >> c.shift] : 0;
            for (int j = 0; j < 64 && i64 + j * ATT_WAVES < i1; ++j) {
                const int i = i64 + j * ATT_WAVES, s0 = i * ATT_BLOCK;
                int page = __builtin_amdgcn_readlane(looked, j);
                const bool there = (unsigned)page < (unsigned)c.n_pages;
                page = there ? page : 0;
                const int off = s0 & (P - 1);
                t.load(ks + page * c.k_page + ((int64_t)(hk << c.shift) + off) * DH, vs + page * c.v_page + ((int64_t)(hk * DH) << c.shift) + off, P);
                float z[8];
                t.scores(z);
                const int live = len - s0;
                float top = -INFINITY;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    z[x] = !there ? NAN : t.slot_of(x) < live ? z[x] * scale : -INFINITY;
                    top = fmaxf(top, z[x]);
                }
                if (live < ATT_BLOCK) t.clear_beyond(live);
                if constexpr (WEIGHED) {
                    if (col < heads)
#pragma unroll
                        for (int x = 0; x < 8; x += 4) *reinterpret_cast<f32x4 *>(score + s0 + t.slot_of(x)) = f32x4{z[x], z[x + 1], z[x + 2], z[x + 3]};
                }
                top = rows_max(top);
                if (__any(top > m)) {
                    const float now = fmaxf(m, top), back = back_by(m, now);
                    m = now;
                    l *= back;
#pragma unroll
                    for (int d = 0; d < DH / 16; ++d) o[d] *= back;
                }
                const float ref = (m == -INFINITY ? 0.f : m) - lift<T>();
#pragma unroll
                for (int x = 0; x < 8; ++x) { z[x] = exp2_of(z[x] - ref); l += z[x]; }
                t.add_values(z, o);
            }
        }
        // the four waves' triples become one
        {
            float x, y;
            swap16(l, x, y); l = x + y;
            swap32(l, x, y); l = x + y;
        }
        __syncthreads();
        if (g4 == 0) lds_ml[wave][col] = make_float2(m, l);
        if (col < heads)
#pragma unroll
            for (int d = 0; d < DH / 16; ++d) *reinterpret_cast<f32x4 *>(&lds_o[(wave * 16 + col) * ROW + 16 * d + 4 * g4]) = o[d];
        __syncthreads();
        const bool starts = i0 == 0, ends = i1 == blocks;
        const int64_t slot = (int64_t)(2 * w + (starts ? 1 : 0)) * c.hkv * a.tiles + blockIdx.y;
        for (int x = threadIdx.x; x < heads * (DH / 4); x += 64 * ATT_WAVES) {
            const int h = x / (DH / 4), d = x % (DH / 4) * 4;
            float top = -INFINITY;
            for (int v = 0; v < ATT_WAVES; ++v) top = fmaxf(top, lds_ml[v][h].x);
            float sum = 0.f;
            f32x4 r = {0.f, 0.f, 0.f, 0.f};
            for (int v = 0; v < ATT_WAVES; ++v) {
                const float f = back_by(lds_ml[v][h].x, top);
                const f32x4 ov = *reinterpret_cast<const f32x4 *>(&lds_o[(v * 16 + h) * ROW + d]);
                sum += lds_ml[v][h].y * f;                 // (a wave that saw nothing adds 0, one that saw only NaN shows it: 0 * NaN)
                r += ov * f;
            }
            if (any_nan(r) && sum == sum)
#pragma unroll 1
                for (int e = 0; e < 4; ++e)
                    if (r[e] != r[e]) r[e] = sum_of_infinities<T, DH>(qs + b * a.q_row + (int64_t)(head0 + h) * DH, c, table, hk, d + e, i0 * ATT_BLOCK, min(i1 * ATT_BLOCK, len), scale);
            if (starts && ends) {
                const float inv = 1.f / sum;
                T *to = out + b * a.out_row + (int64_t)(head0 + h) * DH + d;
                for (int e = 0; e < 4; ++e) to[e] = from_f<T>(r[e] * inv);
                if (d == 0) {
                    const float lse2 = top + __builtin_amdgcn_logf(sum) - lift<T>();
                    if (a.lse) a.lse[(int64_t)b * a.hq + head0 + h] = lse2 * LN2;
                    if (WEIGHED) { if (by_rows && a.tiles == 1) lds_lse[h] = lse2; else a.row_lse[(int64_t)b * a.hq + head0 + h] = lse2; }
                }
            } else {
                *reinterpret_cast<f32x4 *>(a.part + (slot * 16 + h) * DH + d) = r;
                if (d == 0) a.part_ml[slot * 16 + h] = make_float2(top, sum);
            }
        }
        at = first + i1;
        if constexpr (WEIGHED) {
            if (by_rows && a.tiles == 1) {                     // all the key head's heads are here: their weights need no second launch
                __syncthreads();
                const int64_t row = ((int64_t)b * c.hkv + hk) * c.slots;
                for (int s = threadIdx.x; s < len; s += 64 * ATT_WAVES) {
                    const float *z = a.scores + ((int64_t)b * a.hq + head0) * a.score_row + s;
                    float x = 0.f;
                    for (int h = 0; h < heads; ++h) x += exp2_of(z[h * a.score_row] - lds_lse[h]);
                    a.weights_out[row + s] = (a.weights ? a.weights[row + s] : 0.f) + x;
                }
            }
        }
    }
}

// What is left once every piece of every row is there.  A row's pieces lie in workgroups w0 .. w1; a workgroup per row and query head joins them, and one per 1024 slots
// of a row and key head gives the slots their weights: 2^(score - lse), summed over the heads that share the key head.  The latter form a head's lse
// from its pieces' maxima and sums by themselves, so that one launch does both (131072 slots in 64 pieces a head: 62 us with a thread
// per value that walks the pieces one after the other, 5 with all of them asked for at once).
constexpr int FINISH_SLOTS = 1024, FINISH_HEADS = 64;

// WAVES waves join a head: all four where heads are few, one of them each where there are thousands, most of which have one piece and nothing to join (100 rows of 64
// heads, the whole call: 72 us with a workgroup per head, 61 with a wave).
template <typename T, int WAVES>
__global__ void __launch_bounds__(256) attend_finish_kernel(KvView c, AttendArgs a, int joins) {
    constexpr int THREADS = 64 * WAVES, TEAMS = 4 / WAVES;
    __shared__ float factors[TEAMS][ATT_MOST];
    __shared__ f32x4 sums[256];
    __shared__ float red[8];
    const int b = blockIdx.z, hk = blockIdx.y, tid = threadIdx.x, group = a.hq / c.hkv, dh = c.dh;
    const int len = a.lengths[b], blocks = row_blocks(len, a.max_len);
    if (!blocks) return;
    const int chunk = (int)blockIdx.x - joins;
    if (chunk >= 0 && chunk * FINISH_SLOTS >= len) return;
    int w0 = 0, n = 1;
    if (a.W) {
        const Batch batch = count_blocks(a.lengths, c.n_seq, a.max_len);
        const int64_t parts = attend_parts(batch.all, a.W), first = blocks_before(batch, a.lengths, c.n_seq, a.max_len, b);
        // the last workgroup w with w * all / parts <= block
        auto holder = [&](int64_t block) {
            const int64_t x = (block + 1) * parts - 1;
            return x < 1ll << 32 && batch.all < 1ll << 32 ? (int)((uint32_t)x / (uint32_t)batch.all) : (int)(x / batch.all);
        };
        w0 = holder(first); n = holder(first + blocks - 1) - w0 + 1;
    }
    // piece p of the head of this group's index j
    auto slot = [&](int p, int j) { return ((int64_t)(2 * (w0 + p) + (p == 0 ? 1 : 0)) * c.hkv * a.tiles + hk * a.tiles + j / 16) * 16 + j % 16; };
    if (chunk < 0) {
        if (n == 1) return;
        const int team = tid / THREADS, t = tid % THREADS, j = blockIdx.x * TEAMS + team;
        const bool there = j < group;
        float *factor = factors[team];
        auto all_of = [&](float v, float *at, bool largest) {  // over the team
            v = largest ? wave_max(v) : wave_sum(v);
            if constexpr (WAVES == 1) return v;
            if ((tid & 63) == 0) at[tid >> 6] = v;
            __syncthreads();
            return largest ? fmaxf(fmaxf(at[0], at[1]), fmaxf(at[2], at[3])) : at[0] + at[1] + at[2] + at[3];
        };
        float2 ml[ATT_MOST / THREADS];
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k < ATT_MOST / THREADS; ++k) {
            const int p = k * THREADS + t;
            ml[k] = there && p < n ? a.part_ml[slot(p, j)] : make_float2(-INFINITY, 0.f);
            top = fmaxf(top, ml[k].x);
        }
        top = all_of(top, red, true);
#pragma unroll
        for (int k = 0; k < ATT_MOST / THREADS; ++k) {
            const float f = back_by(ml[k].x, top);
            factor[k * THREADS + t] = f;
            sum += ml[k].y * f;
        }
        sum = all_of(sum, red + 4, false);
        __syncthreads();
        // a thread adds four values of every (THREADS / quads)-th piece
        const int quads = dh / 4, ways = THREADS / quads, way = t / quads, d = t % quads * 4;
        f32x4 r = {0.f, 0.f, 0.f, 0.f};
        if (there && way < ways) {
#pragma unroll 8
            for (int p = way; p < n; p += ways) r += *reinterpret_cast<const f32x4 *>(a.part + slot(p, j) * dh + d) * factor[p];
            if (any_nan(r)) {
                r = f32x4{0.f, 0.f, 0.f, 0.f};
                for (int p = way; p < n; p += ways) r += brought(*reinterpret_cast<const f32x4 *>(a.part + slot(p, j) * dh + d), factor[p]);
            }
        }
        sums[tid] = r;
        __syncthreads();
        if (there && way == 0) {
            for (int v = 1; v < ways; ++v) r += sums[team * THREADS + v * quads + t];
            const float inv = 1.f / sum;
            T *to = static_cast<T *>(a.out) + b * a.out_row + (int64_t)(hk * group + j) * dh + d;
            for (int e = 0; e < 4; ++e) to[e] = from_f<T>(r[e] * inv);
        }
        if (there && t == 0 && a.lse) a.lse[(int64_t)b * a.hq + hk * group + j] = (top + __builtin_amdgcn_logf(sum) - lift<T>()) * LN2;
        return;
    }
    float *factor = factors[0];
    const int s = chunk * FINISH_SLOTS + tid * 4, live = len - s;
    f32x4 w = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < group; j0 += FINISH_HEADS) {
        const int heads = min(FINISH_HEADS, group - j0);
        __syncthreads();
        for (int j = tid >> 6; j < heads; j += 4) {        // a wave per head: its lse in `factor`
            float lse;
            if (n == 1) lse = a.row_lse[(int64_t)b * a.hq + hk * group + j0 + j];
            else {
                float top = -INFINITY, sum = 0.f;
                for (int p = tid & 63; p < n; p += 64) top = fmaxf(top, a.part_ml[slot(p, j0 + j)].x);
                top = wave_max(top);
                for (int p = tid & 63; p < n; p += 64) { const float2 ml = a.part_ml[slot(p, j0 + j)]; sum += ml.y * back_by(ml.x, top); }
                lse = top + __builtin_amdgcn_logf(wave_sum(sum)) - lift<T>();
            }
            if ((tid & 63) == 0) factor[j] = lse;
        }
        __syncthreads();
        if (live > 0) {
            const float *row = a.scores + ((int64_t)b * a.hq + hk * group + j0) * a.score_row + s;
#pragma unroll 4
            for (int j = 0; j < heads; ++j) {
                const f32x4 z = *reinterpret_cast<const f32x4 *>(row + j * a.score_row);
                for (int e = 0; e < 4; ++e) w[e] += exp2_of(z[e] - factor[j]);
            }
        }
    }
    if (live <= 0) return;
    const int64_t at = ((int64_t)b * c.hkv + hk) * c.slots + s;
    if (live >= 4 && (reinterpret_cast<uintptr_t>(a.weights) | reinterpret_cast<uintptr_t>(a.weights_out)) % 16 == 0) {
        if (a.weights) w += *reinterpret_cast<const f32x4 *>(a.weights + at);
        *reinterpret_cast<f32x4 *>(a.weights_out + at) = w;
        return;
    }
    for (int e = 0; e < min(4, live); ++e) a.weights_out[at + e] = (a.weights ? a.weights[at + e] : 0.f) + w[e];
}

// How a call runs: workgroups along the slots, and its scratch.
struct AttendPlan { int tiles, W; int64_t score_row; size_t part, part_ml, row_lse, scores, bytes; };
static AttendPlan attend_plan(const KvView &c, int esize, int hq, int max_len, bool weighed) {
    AttendPlan p{};
    p.tiles = (hq / c.hkv + 15) / 16;
    const int64_t per = (int64_t)c.hkv * p.tiles, longest = (max_len + ATT_BLOCK - 1) / ATT_BLOCK, blocks = c.n_seq * longest;
    // As many workgroups as the registers let a CU hold, and never more: a third round of a few costs as much as a whole one (40 key heads, 16 rows: 94 us with 13 x 40
    // workgroups, 74 with 12 x 40).
    const bool two = esize == 2 ? c.dh <= 160 : c.dh <= (weighed ? 96 : 128);
    int64_t W = (two ? ATT_MOST : ATT_MOST / 2) / per;
    if (W > (blocks + ATT_LEAST - 1) / ATT_LEAST) W = (blocks + ATT_LEAST - 1) / ATT_LEAST;
    p.W = W < 1 ? 1 : (int)W;
    // Rows of a few blocks are a workgroup each, without a join: up to two blocks a wave, or four where rows and heads are many (8 rows of up to 250 slots 12.8 -> 8.2 us,
    // 64 of up to 500 weighed 28.7 -> 24.7; 4 of up to 1000 15.2 -> 18.8, so not those; 2 of up to 318 with one key head 12.2 -> 13.9).
    if (longest <= ATT_ROW || (longest <= 2 * ATT_ROW && c.n_seq * per >= 64)) p.W = 0;
    p.score_row = (max_len + ATT_BLOCK - 1) / ATT_BLOCK * ATT_BLOCK;
    auto take = [&](size_t n) { const size_t at = p.bytes; p.bytes += (n + 255) / 256 * 256; return at; };
    if (p.W > 1) {
        p.part = take((size_t)2 * p.W * per * 16 * c.dh * 4);
        p.part_ml = take((size_t)2 * p.W * per * 16 * 8);
    }
    if (weighed) {
        p.row_lse = take((size_t)c.n_seq * hq * 4);
        p.scores = take((size_t)c.n_seq * hq * p.score_row * 4);
    }
    if (p.bytes == 0) p.bytes = 256;
    return p;
}

template <typename T, int DH>
static void launch_attend(const KvView &c, const AttendArgs &a, bool weighed, hipStream_t st) {
    const dim3 grid(a.W ? a.W : c.n_seq, c.hkv * a.tiles);
    if (weighed) attend_kernel<T, DH, true><<<grid, 64 * ATT_WAVES, 0, st>>>(c, a);
    else attend_kernel<T, DH, false><<<grid, 64 * ATT_WAVES, 0, st>>>(c, a);
}
template <typename T>
static void launch_attend_t(const KvView &c, const AttendArgs &a, bool weighed, hipStream_t st) {
    switch (c.dh) {
        case 32: launch_attend<T, 32>(c, a, weighed, st); break;
        case 64: launch_attend<T, 64>(c, a, weighed, st); break;
        case 96: launch_attend<T, 96>(c, a, weighed, st); break;
        case 128: launch_attend<T, 128>(c, a, weighed, st); break;
        case 160: launch_attend<T, 160>(c, a, weighed, st); break;
        case 192: launch_attend<T, 192>(c, a, weighed, st); break;
        case 224: launch_attend<T, 224>(c, a, weighed, st); break;
        default: launch_attend<T, 256>(c, a, weighed, st); break;
    }
    const int chunks = weighed && (a.W || a.tiles > 1) ? (a.max_len + FINISH_SLOTS - 1) / FINISH_SLOTS : 0;
    const bool many = (int64_t)c.n_seq * a.hq > 1024;
    const int joins = a.W <= 1 ? 0 : many ? (a.hq / c.hkv + 3) / 4 : a.hq / c.hkv;
    const dim3 grid(joins + chunks, c.hkv, c.n_seq);
    if (joins + chunks == 0) return;
    if (many) attend_finish_kernel<T, 1><<<grid, 256, 0, st>>>(c, a, joins);
    else attend_finish_kernel<T, 4><<<grid, 256, 0, st>>>(c, a, joins);
}

}  // namespace poss

// ------------------------------------------------------------------------------------------ C entry points (include/poss.h)
using namespace poss;

namespace {
// max_len as it counts, or -1
int attend_max_len(const poss_kv_cache &c, int32_t max_len) {
    const int slots = c.table_pages * c.page_tokens;
    return max_len < 0 || max_len > slots ? -1 : max_len == 0 ? slots : max_len;
}
const char *attend_bad(const poss_kv_cache *c, int32_t hq, int32_t max_len) {
    if (const char *why = kv_cache_bad(c)) return why;
    if (hq < 1 || hq > 65535 || hq % c->n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads";
    if (attend_max_len(*c, max_len) < 0) return "max_len is more than the slots";
    return nullptr;
}
}  // namespace

extern "C" {

size_t poss_kv_attend_scratch_bytes(const poss_kv_cache *cache, int32_t n_q_heads, int32_t max_len, int32_t weighed) {
    return attend_bad(cache, n_q_heads, max_len) ? 0 : attend_plan(kv_view(*cache), (int)dtype_size(cache->dtype), n_q_heads, attend_max_len(*cache, max_len), weighed != 0).bytes;
}

int poss_kv_attend(const poss_kv_cache *cache, int32_t n_q_heads, const void *q, int64_t q_row, void *out, int64_t out_row, const int32_t *lengths, int32_t max_len, float scale,
                   float *lse, const float *weights, float *weights_out, void *scratch, size_t scratch_bytes, void *hip_stream) {
    const char *who = "poss_kv_attend";
    if (const char *why = attend_bad(cache, n_q_heads, max_len)) return set_error(POSS_E_INVALID_ARG, "%s: %s", who, why);
    if (!(fabsf(scale) * LOG2E < INFINITY)) return set_error(POSS_E_INVALID_ARG, "%s: scale, and scale times log2(e), must be finite", who);
    if (weights && !weights_out) return set_error(POSS_E_INVALID_ARG, "%s: weights without weights_out", who);
    if (cache->n_seq == 0) return POSS_OK;
    if (!q || !out || !lengths || !scratch) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    const int64_t whole = 16 / (int64_t)dtype_size(cache->dtype), row = (int64_t)n_q_heads * cache->head_dim;
    if (!kv_aligned(q, 16) || !kv_aligned(out, 16) || q_row % whole || out_row % whole) return set_error(POSS_E_INVALID_ARG, "%s: q and out must be aligned to 16 bytes, with rows whole 16 bytes apart", who);
    if (cache->n_seq > 1 && (q_row < row || out_row < row)) return set_error(POSS_E_INVALID_ARG, "%s: rows overlap", who);
    if (!kv_aligned(lengths, 4) || !kv_aligned(lse, 4) || !kv_aligned(weights, 4) || !kv_aligned(weights_out, 4)) return set_error(POSS_E_INVALID_ARG, "%s: an array is not aligned to its type", who);
    if (!kv_aligned(scratch, 256)) return set_error(POSS_E_INVALID_ARG, "%s: scratch must be aligned to 256 bytes", who);
    const KvView c = kv_view(*cache);
    const int most = attend_max_len(*cache, max_len);
    const bool weighed = weights_out != nullptr;
    const AttendPlan p = attend_plan(c, (int)dtype_size(cache->dtype), n_q_heads, most, weighed);
    if (scratch_bytes < p.bytes) return set_error(POSS_E_CAPACITY, "%s: needs %zu bytes of scratch, got %zu", who, p.bytes, scratch_bytes);
    char *base = static_cast<char *>(scratch);
    AttendArgs a{n_q_heads, p.tiles, q, q_row, out, out_row, lengths, most, scale, lse, weights, weights_out, p.W, reinterpret_cast<float *>(base + p.part),
                 reinterpret_cast<float2 *>(base + p.part_ml), weighed ? reinterpret_cast<float *>(base + p.scores) : nullptr, p.score_row,
                 weighed ? reinterpret_cast<float *>(base + p.row_lse) : nullptr};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (cache->dtype == DT_F32) launch_attend_t<float>(c, a, weighed, st);
    else if (cache->dtype == DT_BF16) launch_attend_t<bf16_t>(c, a, weighed, st);
    else launch_attend_t<f16_t>(c, a, weighed, st);
    return kv_launched(who);
}

}  // extern "C"
