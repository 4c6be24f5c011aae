// Rotary positions, alone and on the way into a paged cache (include/poss.h: poss_rope_fill, poss_rotary, poss_kv_append).
//
// Pairs (a, b) -> magnitude (a cos - b sin, b cos + a sin), in float32, rounded once.  Bound by memory: everything is read once and written once.  8192 rows of 32 + 8 + 8
// heads of 128 (bf16, 201 MB): 45 us, 4.5 TB/s, with no more traffic than that (102 MB read, 101 MB written); 8192 x 40 heads alone 38 us.  A row alone 4.7 us: launch, position
// and slot, the page, the row.
#include "kv.h"
#include "pieces.h"

#include <math.h>

namespace poss {

// The table of one row, times magnitude, into LDS: by the threads first, first + step ..  Angle, cosine and sine are formed in 64 bits, as a context's are: with its
// frequencies, keys get the bits that they get there.  (A series in 32 bits behind a 64-bit reduction took 4.7 us for a token where this takes 4.9, and the same for a prompt.)
__device__ __forceinline__ void rope_angles(const poss_rope &rope, int pos, float sign, float2 *cs, int first, int step) {
    for (int i = first; i < rope.rot_dim / 2; i += step) {
        double s, c;
        sincos((double)pos * rope.freq[i], &s, &c);
        cs[i] = make_float2((float)(c * rope.magnitude), (float)(s * rope.magnitude) * sign);
    }
}

// ------------------------------------------------------------------------------------------ any size and alignment, few rows
// One head: a lane takes pairs, and the values that stay.
template <typename T>
__device__ __forceinline__ void rotate_head(const T *x, T *y, int dh, int rot, int interleaved, const float2 *cs) {
    const int half = rot >> 1;
    for (int i = threadIdx.x & 63; i < half + dh - rot; i += 64) {
        if (i >= half) { y[i + half] = x[i + half]; continue; }
        const int a = interleaved ? 2 * i : i, b = interleaved ? 2 * i + 1 : i + half;
        float o1, o2;
        rope_pair(to_f(x[a]), to_f(x[b]), cs[i], o1, o2);
        y[a] = round_f<T>(o1); y[b] = round_f<T>(o2);
    }
}

// A workgroup per row, a wave per head.
template <typename T>
__global__ void __launch_bounds__(1024) rotary_kernel(const T *x, int64_t x_row, int64_t x_head, T *y, int64_t y_row, int64_t y_head, int heads, int dh,
                                                     const int32_t *__restrict__ positions, poss_rope rope, float sign) {
    __shared__ float2 cs[POSS_ROPE_PAIRS];
    const int64_t r = blockIdx.x;
    rope_angles(rope, positions[r], sign, cs, threadIdx.x, blockDim.x);
    __syncthreads();
    for (int64_t h = threadIdx.x >> 6; h < heads; h += blockDim.x >> 6)
        rotate_head(x + r * x_row + h * x_head, y + r * y_row + h * y_head, dh, rope.rot_dim, rope.interleaved, cs);
}

struct AppendArgs {
    int rows, hq;
    const void *q; int64_t q_row; void *q_out; int64_t q_out_row;
    const void *k; int64_t k_row; const void *v; int64_t v_row;
    const int32_t *seq, *slots, *positions;
    int32_t *slot_positions;
};

// The page that a row goes to (-1: nowhere), its sequence and slot.
__device__ __forceinline__ int append_page(const KvView &c, const AppendArgs &a, int r, int &b, int &slot) {
    b = a.seq ? a.seq[r] : r;
    slot = a.slots[r];
    return (unsigned)b < (unsigned)c.n_seq ? kv_page(c, b, slot) : -1;
}
__device__ __forceinline__ void note_positions(const KvView &c, const AppendArgs &a, int r, int b, int slot, int first, int step) {
    if (a.slot_positions)
        for (int h = first; h < c.hkv; h += step) a.slot_positions[((int64_t)b * c.hkv + h) * c.slots + slot] = a.positions[r];
}

template <typename T>
__global__ void __launch_bounds__(1024) append_kernel(KvView c, AppendArgs a, poss_rope rope) {
    __shared__ float2 cs[POSS_ROPE_PAIRS];
    const int r = blockIdx.x, dh = c.dh;
    int b, slot;
    const int page = append_page(c, a, r, b, slot);
    if (rope.rot_dim) rope_angles(rope, a.positions[r], 1.f, cs, threadIdx.x, blockDim.x);
    __syncthreads();
    const T *q = static_cast<const T *>(a.q) + r * a.q_row, *k = static_cast<const T *>(a.k) + r * a.k_row, *v = static_cast<const T *>(a.v) + r * a.v_row;
    T *qo = static_cast<T *>(a.q_out) + r * a.q_out_row, *ck = static_cast<T *>(c.k), *cv = static_cast<T *>(c.v);
    const int heads = page < 0 ? a.hq : a.hq + 2 * c.hkv;
    for (int h = threadIdx.x >> 6; h < heads; h += blockDim.x >> 6) {          // heads of queries, keys, values
        const int hk = h - a.hq, hv = hk - c.hkv;
        if (hv >= 0)
            for (int d = threadIdx.x & 63; d < dh; d += 64) cv[kv_value_at(c, page, hv, d, slot)] = v[hv * dh + d];
        else rotate_head(hk < 0 ? q + h * dh : k + hk * dh, hk < 0 ? qo + h * dh : ck + kv_key_at(c, page, hk, slot), dh, rope.rot_dim, rope.interleaved, cs);
    }
    if (page < 0) return;
    note_positions(c, a, r, b, slot, threadIdx.x, blockDim.x);
}

// ------------------------------------------------------------------------------------------ whole pieces of 16 bytes, many rows
// A wave's part of a row, in units of pieces.h; four waves share a row where rows alone would leave the chip idle (274 rows of 64 + 8 + 8 heads of 256: 26 -> 11 us).
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void rotate_pieces(const T *x, int64_t x_head, T *y, int64_t y_head, int heads, int rot, Units n, int part, const float2 *cs) {
    constexpr int E = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(E)));
    const int half = rot >> 1, turned = INTERLEAVED ? rot / E : half / E, all = heads * n.units;
#pragma unroll 2
    for (int j = part * 64 + (threadIdx.x & 63); j < all; j += 64 * n.parts) {
        const int h = unit_head(j, n.of_units), u = j - h * n.units;
        const T *xi = x + h * x_head;
        T *yi = y + h * y_head;
        if (u >= turned) {                                 // values that stay
            const int d = rot + (u - turned) * E;
            *reinterpret_cast<vec *>(yi + d) = *reinterpret_cast<const vec *>(xi + d);
        } else if (INTERLEAVED) {
            const vec p = *reinterpret_cast<const vec *>(xi + u * E);
            vec o;
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                float o1, o2;
                rope_pair(to_f(p[e]), to_f(p[e + 1]), cs[u * (E / 2) + e / 2], o1, o2);
                o[e] = round_f<T>(o1); o[e + 1] = round_f<T>(o2);
            }
            *reinterpret_cast<vec *>(yi + u * E) = o;
        } else {
            const vec p = *reinterpret_cast<const vec *>(xi + u * E), q = *reinterpret_cast<const vec *>(xi + half + u * E);
            vec o, s;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float o1, o2;
                rope_pair(to_f(p[e]), to_f(q[e]), cs[u * E + e], o1, o2);
                o[e] = round_f<T>(o1); s[e] = round_f<T>(o2);
            }
            *reinterpret_cast<vec *>(yi + u * E) = o;
            *reinterpret_cast<vec *>(yi + half + u * E) = s;
        }
    }
}

// A wave per row, or n.parts of them.
template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(256) rotary_rows_kernel(const T *x, int64_t x_row, int64_t x_head, T *y, int64_t y_row, int64_t y_head, int rows, int heads, Units n,
                                                          const int32_t *__restrict__ positions, poss_rope rope, float sign) {
    __shared__ __align__(16) float2 cs[4][POSS_ROPE_PAIRS];
    const int wave = threadIdx.x >> 6;
    const int64_t r = n.parts == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    if (r >= rows) return;
    rope_angles(rope, positions[r], sign, cs[wave], threadIdx.x & 63, 64);
    wave_lds_sync();
    rotate_pieces<T, INTERLEAVED>(x + r * x_row, x_head, y + r * y_row, y_head, heads, rope.rot_dim, n, n.parts == 1 ? 0 : wave, cs[wave]);
}

// Queries and keys: a wave per row (or n.parts), in the first workgroups.  Values: behind them, a wave per square of eight by eight pieces - 16-bit types 64 rows by 64 dims -
// of which a lane turns a square of E by E values over in its registers, so that the rows of consecutive slots leave as whole lines of a value row.
// That needs E rows with consecutive slots, the first at a multiple of E; squares are laid so for the rows that follow the call's first slot.
// In other squares a lane takes a row and writes value by value: of consecutive slots 64 stand side by side (all squares so: 49 us for the 45 above).
template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(256) append_rows_kernel(KvView c, AppendArgs a, poss_rope rope, Units n, int row_groups) {
    constexpr int E = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(E)));
    __shared__ __align__(16) float2 cs[4][POSS_ROPE_PAIRS];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, dh = c.dh;
    if ((int)blockIdx.x < row_groups) {
        const int r = n.parts == 1 ? blockIdx.x * 4 + wave : blockIdx.x, part = n.parts == 1 ? 0 : wave;
        if (r >= a.rows) return;
        int b, slot;
        const int page = append_page(c, a, r, b, slot);
        if (rope.rot_dim) rope_angles(rope, a.positions[r], 1.f, cs[wave], lane, 64);
        wave_lds_sync();
        rotate_pieces<T, INTERLEAVED>(static_cast<const T *>(a.q) + r * a.q_row, dh, static_cast<T *>(a.q_out) + r * a.q_out_row, dh, a.hq, rope.rot_dim, n, part, cs[wave]);
        if (page < 0) return;
        rotate_pieces<T, INTERLEAVED>(static_cast<const T *>(a.k) + r * a.k_row, dh, static_cast<T *>(c.k) + kv_key_at(c, page, 0, slot), (int64_t)dh << c.shift, c.hkv, rope.rot_dim, n, part,
                                      cs[wave]);
        if (part == 0) note_positions(c, a, r, b, slot, lane, 64);
        return;
    }
    const int across = (c.hkv * dh + 8 * E - 1) / (8 * E);                     // squares of a row of values
    const int64_t square = (int64_t)(blockIdx.x - row_groups) * 4 + wave;
    const int sr = (int)(square / across), dims = c.hkv * dh, d_first = (int)(square - (int64_t)sr * across) * 8 * E;
    const int shift = a.slots[0] > 0 ? a.slots[0] & (E - 1) : 0, r_first = sr * 8 * E - shift;
    const T *v = static_cast<const T *>(a.v);
    T *cv = static_cast<T *>(c.v);
    // lane i looks up row i of the square's 8 E
    const int mine = r_first + lane;
    int b = -1, slot = -1;
    const int page = lane < 8 * E && mine >= 0 && mine < a.rows ? append_page(c, a, mine, b, slot) : -1;
    const int place = lane & (E - 1), head_slot = __shfl(slot, lane - place), head_b = __shfl(b, lane - place);
    const bool run = page >= 0 && head_slot % E == 0 && slot == head_slot + place && b == head_b;
    if (__all(run || (lane >= 8 * E))) {
        const int g = lane & 7, d0 = d_first + (lane >> 3) * E, r0 = r_first + g * E;
        const int page0 = __shfl(page, g * E), slot0 = __shfl(slot, g * E);
        if (d0 >= dims) return;
        vec in[E];
#pragma unroll
        for (int e = 0; e < E; ++e) in[e] = *reinterpret_cast<const vec *>(v + (int64_t)(r0 + e) * a.v_row + d0);
        T *to = cv + kv_value_at(c, page0, 0, d0, slot0);                      // (heads and dims are one sequence of value rows)
#pragma unroll
        for (int d = 0; d < E; ++d) {
            vec o;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = in[e][d];
            *reinterpret_cast<vec *>(to + ((int64_t)d << c.shift)) = o;
        }
        return;
    }
    // any rows: a lane per row, so that what lies side by side in a value row leaves side by side
    if (page < 0) return;
    T *to = cv + kv_value_at(c, page, 0, d_first, slot);
    const int across_d = min(8 * E, dims - d_first);
#pragma unroll 2
    for (int d = 0; d < across_d; d += E) {
        const vec in = *reinterpret_cast<const vec *>(v + mine * a.v_row + d_first + d);
#pragma unroll
        for (int e = 0; e < E; ++e) to[(int64_t)(d + e) << c.shift] = in[e];
    }
}

}  // namespace poss

// ------------------------------------------------------------------------------------------ C entry points (include/poss.h)
using namespace poss;

namespace {
// From ROWS_MANY rows on a wave takes a row.  Below, a workgroup does: 64 sequences' tokens 5.6 us for 13.9 (their values go to 64 pages); 100 rows of a prompt 5.5 for 4.7.
constexpr int ROWS_MANY = 200, ROWS_MOST = 1 << 21;     // (threads of a launch are counted in 32 bits)
int row_threads(int heads) { return heads >= 16 ? 1024 : heads > 4 ? 512 : 256; }
bool rope_ok(const poss_rope &r, int head_dim) { return r.rot_dim >= 2 && r.rot_dim <= 2 * POSS_ROPE_PAIRS && r.rot_dim % 2 == 0 && r.rot_dim <= head_dim; }
}  // namespace

extern "C" {

int poss_rope_fill(int32_t rot_dim, int32_t interleaved, double theta, int32_t scaling, double factor, double low, double high, double original, double magnitude, poss_rope *out) {
    const char *who = "poss_rope_fill";
    if (!out) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    if (rot_dim < 2 || rot_dim > 2 * POSS_ROPE_PAIRS || rot_dim % 2) return set_error(POSS_E_INVALID_ARG, "%s: rot_dim must be even, 2 to %d", who, 2 * POSS_ROPE_PAIRS);
    if (!(theta > 0) || !isfinite(theta) || !isfinite((float)magnitude)) return set_error(POSS_E_INVALID_ARG, "%s: theta must be positive, magnitude finite", who);
    if (scaling < POSS_ROPE_NONE || scaling > POSS_ROPE_RAMP) return set_error(POSS_E_INVALID_ARG, "%s: no such scaling", who);
    if (scaling != POSS_ROPE_NONE && (!(factor > 0) || !isfinite(factor))) return set_error(POSS_E_INVALID_ARG, "%s: factor must be positive", who);
    const bool parts = scaling == POSS_ROPE_BANDS || scaling == POSS_ROPE_RAMP;
    if (parts && (!(low > 0) || !(high > low) || !isfinite(high) || !(original > 0) || !isfinite(original)))
        return set_error(POSS_E_INVALID_ARG, "%s: 0 < low < high and original > 0 are wanted", who);
    if (scaling == POSS_ROPE_RAMP && !(theta > 1)) return set_error(POSS_E_INVALID_ARG, "%s: a ramp needs theta > 1", who);
    if (scaling == POSS_ROPE_BASE) {
        if (rot_dim < 4) return set_error(POSS_E_INVALID_ARG, "%s: another base needs rot_dim of at least 4", who);
        theta *= pow(factor, (double)rot_dim / (rot_dim - 2));
    }
    const double two_pi = 6.283185307179586476925;
    poss_rope r{};
    r.rot_dim = rot_dim; r.interleaved = interleaved != 0; r.magnitude = (float)magnitude;
    double lo = 0, hi = 0;
    if (scaling == POSS_ROPE_RAMP) {
        lo = floor(rot_dim * log(original / (high * two_pi)) / (2 * log(theta)));
        hi = ceil(rot_dim * log(original / (low * two_pi)) / (2 * log(theta)));
        lo = lo < 0 ? 0 : lo; hi = hi > rot_dim - 1 ? rot_dim - 1 : hi;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double w = pow(theta, -2.0 * i / rot_dim);
        double g = 1;
        if (scaling == POSS_ROPE_LINEAR) g = 0;
        if (scaling == POSS_ROPE_BANDS) g = (original * w / two_pi - low) / (high - low);
        if (scaling == POSS_ROPE_RAMP) g = 1 - (i - lo) / (hi - lo > 1e-3 ? hi - lo : 1e-3);
        g = g < 0 ? 0 : g > 1 ? 1 : g;
        r.freq[i] = g * w + (1 - g) * w / (scaling == POSS_ROPE_NONE || scaling == POSS_ROPE_BASE ? 1 : factor);
        if (!isfinite(r.freq[i])) return set_error(POSS_E_INVALID_ARG, "%s: theta and factor give a frequency that is not finite", who);
    }
    *out = r;
    return POSS_OK;
}

int poss_rotary(int32_t dtype, const void *x, int64_t x_row, int64_t x_head, void *y, int64_t y_row, int64_t y_head, int32_t rows, int32_t heads, int32_t head_dim,
                const int32_t *positions, const poss_rope *rope, int32_t inverse, void *hip_stream) {
    const char *who = "poss_rotary";
    if (kv_bad_dtype(dtype) || rows < 0 || rows > ROWS_MOST || heads < 1 || head_dim < 2) return set_error(POSS_E_INVALID_ARG, "%s: bad shape or type", who);
    if (!rope || !rope_ok(*rope, head_dim)) return set_error(POSS_E_INVALID_ARG, "%s: rope: an even rot_dim up to the head's values is wanted", who);
    if (rows == 0) return POSS_OK;
    if (!x || !y || !positions) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    const size_t e = dtype_size(dtype);
    if (!kv_aligned(x, e) || !kv_aligned(y, e) || !kv_aligned(positions, 4)) return set_error(POSS_E_INVALID_ARG, "%s: x, y or positions is not aligned to its type", who);
    if ((heads > 1 && (x_head < head_dim || y_head < head_dim)) || (rows > 1 && (x_row < head_dim || y_row < head_dim)))
        return set_error(POSS_E_INVALID_ARG, "%s: rows or heads overlap", who);
    if (x == y && ((rows > 1 && x_row != y_row) || (heads > 1 && x_head != y_head))) return set_error(POSS_E_INVALID_ARG, "%s: y is x with other distances", who);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const float sign = inverse ? -1.f : 1.f;
    const int64_t whole = 16 / (int64_t)e;
    const int threads = row_threads(heads);
    Units n{};
    const bool pieces = rows >= ROWS_MANY && units_of((int)whole, rows, heads, head_dim, rope->rot_dim, rope->interleaved, n) && kv_aligned(x, 16) && kv_aligned(y, 16) &&
                        x_row % whole == 0 && y_row % whole == 0 && x_head % whole == 0 && y_head % whole == 0;
    const int row_groups = n.parts == 4 ? rows : (rows + 3) / 4;
#define POSS_ROTARY(T)                                                                                                                                    \
    do {                                                                                                                                                  \
        const T *xt = static_cast<const T *>(x); T *yt = static_cast<T *>(y);                                                                             \
        if (!pieces) rotary_kernel<T><<<rows, threads, 0, st>>>(xt, x_row, x_head, yt, y_row, y_head, heads, head_dim, positions, *rope, sign);               \
        else if (rope->interleaved) rotary_rows_kernel<T, true><<<row_groups, 256, 0, st>>>(xt, x_row, x_head, yt, y_row, y_head, rows, heads, n, positions, *rope, sign); \
        else rotary_rows_kernel<T, false><<<row_groups, 256, 0, st>>>(xt, x_row, x_head, yt, y_row, y_head, rows, heads, n, positions, *rope, sign);  \
    } while (0)
    if (dtype == DT_F32) POSS_ROTARY(float); else if (dtype == DT_BF16) POSS_ROTARY(bf16_t); else POSS_ROTARY(f16_t);
#undef POSS_ROTARY
    return kv_launched(who);
}

int poss_kv_append(const poss_kv_cache *cache, const poss_rope *rope, int32_t rows, int32_t n_q_heads, const void *q, int64_t q_row, void *q_out, int64_t q_out_row,
                   const void *k, int64_t k_row, const void *v, int64_t v_row, const int32_t *seq, const int32_t *slots, const int32_t *positions,
                   int32_t *slot_positions, void *hip_stream) {
    const char *who = "poss_kv_append";
    if (const char *why = kv_cache_bad(cache)) return set_error(POSS_E_INVALID_ARG, "%s: %s", who, why);
    if (rows < 0 || rows > ROWS_MOST || n_q_heads < 0 || n_q_heads > 65535) return set_error(POSS_E_INVALID_ARG, "%s: bad shape", who);
    if (rope && !rope_ok(*rope, cache->head_dim)) return set_error(POSS_E_INVALID_ARG, "%s: rope: an even rot_dim up to the head's values is wanted", who);
    if (rows == 0 || cache->n_seq == 0) return POSS_OK;
    if (!k || !v || !slots || (n_q_heads && (!q || !q_out)) || ((rope || slot_positions) && !positions)) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    const size_t e = dtype_size(cache->dtype);
    if (!kv_aligned(k, e) || !kv_aligned(v, e) || (n_q_heads && (!kv_aligned(q, e) || !kv_aligned(q_out, e))) || !kv_aligned(seq, 4) || !kv_aligned(slots, 4) || !kv_aligned(positions, 4) ||
        !kv_aligned(slot_positions, 4))
        return set_error(POSS_E_INVALID_ARG, "%s: an array is not aligned to its type", who);
    const int64_t kv_len = (int64_t)cache->n_kv_heads * cache->head_dim, q_len = (int64_t)n_q_heads * cache->head_dim;
    if (rows > 1 && (k_row < kv_len || v_row < kv_len || (n_q_heads && (q_row < q_len || q_out_row < q_len)))) return set_error(POSS_E_INVALID_ARG, "%s: rows overlap", who);
    if (n_q_heads && rows > 1 && q == q_out && q_row != q_out_row) return set_error(POSS_E_INVALID_ARG, "%s: q_out is q with another distance", who);
    poss_rope none{};
    const AppendArgs a{rows, n_q_heads, q, q_row, q_out, q_out_row, k, k_row, v, v_row, seq, slots, positions, slot_positions};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const KvView c = kv_view(*cache);
    const poss_rope &r = rope ? *rope : none;
    const int64_t whole = 16 / (int64_t)e;
    const int threads = row_threads(n_q_heads + 2 * cache->n_kv_heads);
    Units n{};
    const bool pieces = rows >= ROWS_MANY && units_of((int)whole, rows, n_q_heads > cache->n_kv_heads ? n_q_heads : cache->n_kv_heads, cache->head_dim, r.rot_dim, r.interleaved, n) && kv_aligned(k, 16) && kv_aligned(v, 16) && k_row % whole == 0 &&
                        v_row % whole == 0 && (!n_q_heads || (kv_aligned(q, 16) && kv_aligned(q_out, 16) && q_row % whole == 0 && q_out_row % whole == 0));
    const int row_groups = n.parts == 4 ? rows : (rows + 3) / 4;
    const int64_t squares = ((int64_t)rows + whole - 1 + 8 * whole - 1) / (8 * whole) * ((kv_len + 8 * whole - 1) / (8 * whole));      // (the first rows may begin inside a piece)
    const int64_t groups = row_groups + (squares + 3) / 4;
#define POSS_APPEND(T)                                                                                                     \
    do {                                                                                                                   \
        if (!pieces || groups > 1 << 23) append_kernel<T><<<rows, threads, 0, st>>>(c, a, r);                                  \
        else if (r.interleaved) append_rows_kernel<T, true><<<(unsigned)groups, 256, 0, st>>>(c, a, r, n, row_groups);     \
        else append_rows_kernel<T, false><<<(unsigned)groups, 256, 0, st>>>(c, a, r, n, row_groups);                       \
    } while (0)
    if (cache->dtype == DT_F32) POSS_APPEND(float); else if (cache->dtype == DT_BF16) POSS_APPEND(bf16_t); else POSS_APPEND(f16_t);
#undef POSS_APPEND
    return kv_launched(who);
}

}  // extern "C"
