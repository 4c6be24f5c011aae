// Log-probabilities of given tokens, entropy and the best alternatives of rows of logits (include/poss.h: poss_logprobs).
//
// With m = max x, d = (x - m) / T:  S = sum e^d, log p = d - log S, entropy = log S - sum(e^d d) / S.  Everything is formed from differences to the
// maximum: large logits cancel nothing, and x / T cannot overflow where p has a value.
#include "kv.h"

namespace poss {

// One workgroup per row: a pass for the maximum, one for the sums, one for each alternative.
template <typename T>
__global__ void __launch_bounds__(1024) logprobs_kernel(const T *x, int64_t ldx, int vocab, float temperature, const int32_t *__restrict__ tokens, int n_tokens,
                                                        float *__restrict__ logp, float *__restrict__ entropy, int n_top, int32_t *__restrict__ top_ids, float *__restrict__ top_logp) {
    __shared__ float red[17], red_v[17];
    __shared__ int red_i[17];
    const int64_t r = blockIdx.x;
    const T *row = x + r * ldx;
    float m = -INFINITY;
    for (int i = threadIdx.x; i < vocab; i += 1024) m = fmaxf(m, to_f(row[i]));
    int dummy = threadIdx.x;
    block_argmax(m, dummy, red_v, red_i);
    float s = 0.f, t = 0.f;
    for (int i = threadIdx.x; i < vocab; i += 1024) {
        const float d = (to_f(row[i]) - m) / temperature, e = expf(d);
        s += e;
        t += e * fmaxf(d, -1e4f);
    }
    s = block_sum(s, red);
    t = block_sum(t, red);
    const float log_s = logf(s);                           // NaN where a logit is NaN or +infinity, or none is above -infinity
    if (entropy && threadIdx.x == 0) entropy[r] = log_s - t / s;
    for (int j = threadIdx.x; j < n_tokens; j += 1024) {
        const int id = tokens[r * n_tokens + j];
        logp[r * n_tokens + j] = (unsigned)id < (unsigned)vocab ? (to_f(row[id]) - m) / temperature - log_s : NAN;
    }
    // numbers by (value, id), then NaN by id: NaN stands as the value below -infinity, told apart by `nan`
    float last = INFINITY; int last_id = -1; bool nans = false;
    for (int j = 0; j < n_top; ++j) {
        float v = -INFINITY; int id = 0x7fffffff;
        if (!nans)
            for (int i = threadIdx.x; i < vocab; i += 1024) {
                const float z = to_f(row[i]);
                if (z == z && (z < last || (z == last && i > last_id)) && better(z, i, v, id)) { v = z; id = i; }
            }
        block_argmax(v, id, red_v, red_i);
        if (id == 0x7fffffff) {
            if (!nans) { nans = true; last_id = -1; }
            v = 0.f;
            for (int i = threadIdx.x; i < vocab; i += 1024)
                if (row[i] != row[i] && i > last_id) { id = i; break; }
            block_argmax(v, id, red_v, red_i);
        }
        last = v; last_id = id;
        if (threadIdx.x == 0) {
            top_ids[r * n_top + j] = id;
            top_logp[r * n_top + j] = (to_f(row[id]) - m) / temperature - log_s;
        }
    }
}

}  // namespace poss

// ------------------------------------------------------------------------------------------ C entry points (include/poss.h)
using namespace poss;

namespace {
bool logprobs_ok(int32_t rows, int32_t vocab, int32_t n_top) { return rows >= 0 && vocab >= 1 && vocab <= 1 << 30 && n_top >= 0 && n_top <= POSS_LOGPROBS_TOP && n_top <= vocab; }
}  // namespace

extern "C" {

size_t poss_logprobs_scratch_bytes(int32_t rows, int32_t vocab, int32_t n_top) { return logprobs_ok(rows, vocab, n_top) ? 256 : 0; }

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
#define POSS_LOGPROBS(T) logprobs_kernel<T><<<rows, 1024, 0, st>>>(static_cast<const T *>(x), ldx, vocab, temperature, tokens, n_tokens, logp, entropy, n_top, top_ids, top_logp)
    if (dtype == DT_F32) POSS_LOGPROBS(float); else if (dtype == DT_BF16) POSS_LOGPROBS(bf16_t); else POSS_LOGPROBS(f16_t);
#undef POSS_LOGPROBS
    return kv_launched(who);
}

}  // extern "C"
