// Attention of one new token per sequence over a paged cache (include/poss.h: poss_kv_attend).
#include "kv.h"

namespace poss {

struct AttendArgs {
    int hq;
    const void *q; int64_t q_row; void *out; int64_t out_row;
    const int32_t *lengths; int max_len; float scale;
    float *lse; const float *weights; float *weights_out;
    float *scores;        // [n_seq][hq][max_len]
    float *row_lse;       // [n_seq][hq]
};

// A workgroup per sequence and query head: scores of 256 slots at a time, the running maximum and sum, then the values.
template <typename T>
__global__ void __launch_bounds__(256) attend_kernel(KvView c, AttendArgs a) {
    __shared__ float qs[256], ps[256], red_v[17];
    __shared__ int red_i[17];
    __shared__ int pages[256];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, g = a.hq / c.hkv, hk = h / g, dh = c.dh;
    if (tid < dh) qs[tid] = to_f(static_cast<const T *>(a.q)[b * a.q_row + (int64_t)h * dh + tid]);
    __syncthreads();
    int len = a.lengths[b];
    const bool bad = len > a.max_len;
    len = len < 0 ? 0 : bad ? 0 : len;
    const T *k = static_cast<const T *>(c.k), *v = static_cast<const T *>(c.v);
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int s0 = 0; s0 < len; s0 += 256) {
        const int s = s0 + tid;
        float z = -INFINITY;
        int page = -1;
        if (s < len) {
            page = kv_page(c, b, s);
            z = NAN;
            if (page >= 0) {
                z = 0.f;
                const T *key = k + kv_key_at(c, page, hk, s);
                for (int d = 0; d < dh; ++d) z += qs[d] * to_f(key[d]);
                z *= a.scale;
            }
            if (a.scores) a.scores[((int64_t)b * a.hq + h) * a.max_len + s] = z;
        }
        float top = z; int id = tid;
        block_argmax(top, id, red_v, red_i);
        const float now = fmaxf(m, top), ref = now == -INFINITY ? 0.f : now, back = m == -INFINITY ? 0.f : expf(m - ref);
        const float p = expf(z - ref);
        l = l * back + block_sum(p, red_v);
        ps[tid] = p; pages[tid] = page;
        __syncthreads();
        if (tid < dh) {
            o *= back;
            const int n = min(256, len - s0);
            for (int j = 0; j < n; ++j) o += pages[j] >= 0 ? ps[j] * to_f(v[kv_value_at(c, pages[j], hk, tid, s0 + j)]) : NAN;
        }
        m = now;
        __syncthreads();
    }
    const float sum = m + logf(l);
    if (tid < dh) static_cast<T *>(a.out)[b * a.out_row + (int64_t)h * dh + tid] = from_f<T>(bad ? NAN : len ? o / l : 0.f);
    if (tid == 0) {
        const float lse = bad ? NAN : len ? sum : -INFINITY;
        if (a.lse) a.lse[(int64_t)b * a.hq + h] = lse;
        if (a.row_lse) a.row_lse[(int64_t)b * a.hq + h] = lse;
    }
}

__global__ void __launch_bounds__(256) attend_weights_kernel(KvView c, AttendArgs a) {
    const int hk = blockIdx.y, b = blockIdx.z, s = blockIdx.x * 256 + threadIdx.x, g = a.hq / c.hkv;
    const int len = min(a.lengths[b], a.max_len);
    if (s >= len) return;
    const int64_t at = ((int64_t)b * c.hkv + hk) * c.slots + s;
    float w = 0.f;
    for (int j = 0; j < g; ++j) {
        const int64_t row = (int64_t)b * a.hq + hk * g + j;
        w += expf(a.scores[row * a.max_len + s] - a.row_lse[row]);
    }
    a.weights_out[at] = (a.weights ? a.weights[at] : 0.f) + w;
}

static size_t attend_scores_bytes(const KvView &c, int hq, int max_len) { return (size_t)c.n_seq * hq * max_len * 4; }

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
size_t attend_scratch(const poss_kv_cache &c, int32_t hq, int max_len, bool weighed) {
    return 256 + (weighed ? attend_scores_bytes(kv_view(c), hq, max_len) + (size_t)c.n_seq * hq * 4 : 0);
}
}  // namespace

extern "C" {

size_t poss_kv_attend_scratch_bytes(const poss_kv_cache *cache, int32_t n_q_heads, int32_t max_len, int32_t weighed) {
    return attend_bad(cache, n_q_heads, max_len) ? 0 : attend_scratch(*cache, n_q_heads, attend_max_len(*cache, max_len), weighed != 0);
}

int poss_kv_attend(const poss_kv_cache *cache, int32_t n_q_heads, const void *q, int64_t q_row, void *out, int64_t out_row, const int32_t *lengths, int32_t max_len, float scale,
                   float *lse, const float *weights, float *weights_out, void *scratch, size_t scratch_bytes, void *hip_stream) {
    const char *who = "poss_kv_attend";
    if (const char *why = attend_bad(cache, n_q_heads, max_len)) return set_error(POSS_E_INVALID_ARG, "%s: %s", who, why);
    if (!(scale > -INFINITY && scale < INFINITY)) return set_error(POSS_E_INVALID_ARG, "%s: scale must be finite", who);
    if (weights && !weights_out) return set_error(POSS_E_INVALID_ARG, "%s: weights without weights_out", who);
    if (cache->n_seq == 0) return POSS_OK;
    if (!q || !out || !lengths || !scratch) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    const int64_t whole = 16 / (int64_t)dtype_size(cache->dtype), row = (int64_t)n_q_heads * cache->head_dim;
    if (!kv_aligned(q, 16) || !kv_aligned(out, 16) || q_row % whole || out_row % whole) return set_error(POSS_E_INVALID_ARG, "%s: q and out must be aligned to 16 bytes, with rows whole 16 bytes apart", who);
    if (cache->n_seq > 1 && (q_row < row || out_row < row)) return set_error(POSS_E_INVALID_ARG, "%s: rows overlap", who);
    if (!kv_aligned(lengths, 4) || !kv_aligned(lse, 4) || !kv_aligned(weights, 4) || !kv_aligned(weights_out, 4)) return set_error(POSS_E_INVALID_ARG, "%s: an array is not aligned to its type", who);
    if (!kv_aligned(scratch, 256)) return set_error(POSS_E_INVALID_ARG, "%s: scratch must be aligned to 256 bytes", who);
    const int most = attend_max_len(*cache, max_len);
    const size_t need = attend_scratch(*cache, n_q_heads, most, weights_out != nullptr);
    if (scratch_bytes < need) return set_error(POSS_E_CAPACITY, "%s: needs %zu bytes of scratch, got %zu", who, need, scratch_bytes);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const KvView c = kv_view(*cache);
    AttendArgs a{n_q_heads, q, q_row, out, out_row, lengths, most, scale, lse, weights, weights_out, nullptr, nullptr};
    if (weights_out) {
        a.row_lse = static_cast<float *>(scratch);
        a.scores = a.row_lse + (size_t)c.n_seq * n_q_heads;
    }
    const dim3 grid(n_q_heads, c.n_seq);
    if (cache->dtype == DT_F32) attend_kernel<float><<<grid, 256, 0, st>>>(c, a);
    else if (cache->dtype == DT_BF16) attend_kernel<bf16_t><<<grid, 256, 0, st>>>(c, a);
    else attend_kernel<f16_t><<<grid, 256, 0, st>>>(c, a);
    if (weights_out) attend_weights_kernel<<<dim3((most + 255) / 256, c.hkv, c.n_seq), 256, 0, st>>>(c, a);
    return kv_launched(who);
}

}  // extern "C"
