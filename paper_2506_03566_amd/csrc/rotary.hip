// Rotary positions, alone and on the way into a paged cache (include/poss.h: poss_rope_fill, poss_rotary, poss_kv_append).
#include "kv.h"

#include <math.h>

namespace poss {

// Cosine and sine of position * freq[i], times magnitude, for the pairs of one row: into LDS, by the row's workgroup.
__device__ __forceinline__ void rope_angles(const poss_rope &rope, int pos, float sign, float2 *cs) {
    for (int i = threadIdx.x; i < rope.rot_dim / 2; i += blockDim.x) {
        double s, c;
        sincos((double)pos * rope.freq[i], &s, &c);
        cs[i] = make_float2((float)(c * rope.magnitude), (float)(s * rope.magnitude) * sign);
    }
}

// What value d of a head at x becomes.
template <typename T>
__device__ __forceinline__ T rope_value(const T *x, int d, int rot, int interleaved, const float2 *cs) {
    if (d >= rot) return x[d];
    const int half = rot >> 1;
    const int i = interleaved ? d >> 1 : d < half ? d : d - half;
    const bool second = interleaved ? d & 1 : d >= half;
    float a, b;
    rope_pair(to_f(x[interleaved ? 2 * i : i]), to_f(x[interleaved ? 2 * i + 1 : i + half]), cs[i], a, b);
    return from_f<T>(second ? b : a);
}

// A workgroup per row.
template <typename T>
__global__ void __launch_bounds__(256) rotary_kernel(const T *x, int64_t x_row, int64_t x_head, T *y, int64_t y_row, int64_t y_head, int heads, int dh,
                                                     const int32_t *__restrict__ positions, poss_rope rope, float sign) {
    __shared__ float2 cs[POSS_ROPE_PAIRS];
    const int64_t r = blockIdx.x;
    rope_angles(rope, positions[r], sign, cs);
    __syncthreads();
    const int half = rope.rot_dim >> 1, rest = dh - rope.rot_dim, per = half + rest;      // a thread takes a pair, or a value that stays
    for (int64_t j = threadIdx.x; j < (int64_t)heads * per; j += blockDim.x) {
        const int64_t h = j / per;
        const int i = (int)(j - h * per);
        const T *xi = x + r * x_row + h * x_head;
        T *yi = y + r * y_row + h * y_head;
        if (i >= half) { yi[i + half] = xi[i + half]; continue; }
        const int a = rope.interleaved ? 2 * i : i, b = rope.interleaved ? 2 * i + 1 : i + half;
        float o1, o2;
        rope_pair(to_f(xi[a]), to_f(xi[b]), cs[i], o1, o2);
        yi[a] = from_f<T>(o1); yi[b] = from_f<T>(o2);
    }
}

struct AppendArgs {
    int hq;
    const void *q; int64_t q_row; void *q_out; int64_t q_out_row;
    const void *k; int64_t k_row; const void *v; int64_t v_row;
    const int32_t *seq, *slots, *positions;
    int32_t *slot_positions;
};

template <typename T>
__global__ void __launch_bounds__(256) append_kernel(KvView c, AppendArgs a, poss_rope rope) {
    __shared__ float2 cs[POSS_ROPE_PAIRS];
    const int r = blockIdx.x, dh = c.dh, half = rope.rot_dim >> 1;
    if (half) rope_angles(rope, a.positions[r], 1.f, cs);
    __syncthreads();
    const int rest = dh - rope.rot_dim, per = half + rest;
    const T *q = static_cast<const T *>(a.q) + r * a.q_row;
    T *qo = static_cast<T *>(a.q_out) + r * a.q_out_row;
    for (int j = threadIdx.x; j < a.hq * per; j += blockDim.x) {
        const int h = j / per, i = j - h * per;
        if (i >= half) { qo[h * dh + i + half] = q[h * dh + i + half]; continue; }
        const int x = h * dh + (rope.interleaved ? 2 * i : i), y = h * dh + (rope.interleaved ? 2 * i + 1 : i + half);
        float o1, o2;
        rope_pair(to_f(q[x]), to_f(q[y]), cs[i], o1, o2);
        qo[x] = from_f<T>(o1); qo[y] = from_f<T>(o2);
    }
    const int b = a.seq ? a.seq[r] : r, slot = a.slots[r];
    if ((unsigned)b >= (unsigned)c.n_seq) return;
    const int page = kv_page(c, b, slot);
    if (page < 0) return;
    const T *k = static_cast<const T *>(a.k) + r * a.k_row, *v = static_cast<const T *>(a.v) + r * a.v_row;
    T *ck = static_cast<T *>(c.k), *cv = static_cast<T *>(c.v);
    for (int j = threadIdx.x; j < c.hkv * dh; j += blockDim.x) {
        const int h = j / dh, d = j - h * dh;
        ck[kv_key_at(c, page, h, slot) + d] = rope_value(k + h * dh, d, rope.rot_dim, rope.interleaved, cs);
        cv[kv_value_at(c, page, h, d, slot)] = v[j];
    }
    if (a.slot_positions)
        for (int h = threadIdx.x; h < c.hkv; h += blockDim.x) a.slot_positions[((int64_t)b * c.hkv + h) * c.slots + slot] = a.positions[r];
}

}  // namespace poss

// ------------------------------------------------------------------------------------------ C entry points (include/poss.h)
using namespace poss;

namespace {
bool rope_ok(const poss_rope &r, int head_dim) { return r.rot_dim >= 2 && r.rot_dim <= 2 * POSS_ROPE_PAIRS && r.rot_dim % 2 == 0 && r.rot_dim <= head_dim; }
}  // namespace

extern "C" {

int poss_rope_fill(int32_t rot_dim, int32_t interleaved, double theta, int32_t scaling, double factor, double low, double high, double original, double magnitude, poss_rope *out) {
    const char *who = "poss_rope_fill";
    if (!out) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    if (rot_dim < 2 || rot_dim > 2 * POSS_ROPE_PAIRS || rot_dim % 2) return set_error(POSS_E_INVALID_ARG, "%s: rot_dim must be even, 2 to %d", who, 2 * POSS_ROPE_PAIRS);
    if (!(theta > 0) || !isfinite(theta) || !isfinite(magnitude)) return set_error(POSS_E_INVALID_ARG, "%s: theta must be positive, magnitude finite", who);
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
    }
    *out = r;
    return POSS_OK;
}

int poss_rotary(int32_t dtype, const void *x, int64_t x_row, int64_t x_head, void *y, int64_t y_row, int64_t y_head, int32_t rows, int32_t heads, int32_t head_dim,
                const int32_t *positions, const poss_rope *rope, int32_t inverse, void *hip_stream) {
    const char *who = "poss_rotary";
    if (kv_bad_dtype(dtype) || rows < 0 || heads < 1 || head_dim < 2) return set_error(POSS_E_INVALID_ARG, "%s: bad shape or type", who);
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
#define POSS_ROTARY(T) rotary_kernel<T><<<rows, 256, 0, st>>>(static_cast<const T *>(x), x_row, x_head, static_cast<T *>(y), y_row, y_head, heads, head_dim, positions, *rope, sign)
    if (dtype == DT_F32) POSS_ROTARY(float); else if (dtype == DT_BF16) POSS_ROTARY(bf16_t); else POSS_ROTARY(f16_t);
#undef POSS_ROTARY
    return kv_launched(who);
}

int poss_kv_append(const poss_kv_cache *cache, const poss_rope *rope, int32_t rows, int32_t n_q_heads, const void *q, int64_t q_row, void *q_out, int64_t q_out_row,
                   const void *k, int64_t k_row, const void *v, int64_t v_row, const int32_t *seq, const int32_t *slots, const int32_t *positions,
                   int32_t *slot_positions, void *hip_stream) {
    const char *who = "poss_kv_append";
    if (const char *why = kv_cache_bad(cache)) return set_error(POSS_E_INVALID_ARG, "%s: %s", who, why);
    if (rows < 0 || n_q_heads < 0 || n_q_heads > 65535) return set_error(POSS_E_INVALID_ARG, "%s: bad shape", who);
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
    const AppendArgs a{n_q_heads, q, q_row, q_out, q_out_row, k, k_row, v, v_row, seq, slots, positions, slot_positions};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const KvView c = kv_view(*cache);
    const poss_rope &r = rope ? *rope : none;
    if (cache->dtype == DT_F32) append_kernel<float><<<rows, 256, 0, st>>>(c, a, r);
    else if (cache->dtype == DT_BF16) append_kernel<bf16_t><<<rows, 256, 0, st>>>(c, a, r);
    else append_kernel<f16_t><<<rows, 256, 0, st>>>(c, a, r);
    return kv_launched(who);
}

}  // extern "C"
