// Y[m][n] = sum_k X[m][k] W[n][k] with W microscaled in 4 bits and packed in operand order (mx.hip), X in 32 or 16 bits or
// microscaled as well.
//
// 16-bit X: a weight becomes c * 2^(s - ref) in the type of X (one conversion instruction for two, exact) and enters
// v_mfma_f32_16x16x32; the 32 codes that a lane holds per k-step are the k values of four such instructions, lane / 16 choosing the block of
// 32 and the instruction eight values of it, so that X is read in the same order: 64 contiguous bytes of a row per lane.
// float32 X: the sum of three bf16 numbers, three instructions.  Microscaled X: v_mfma_scale with both scales, one block per lane.
// The sums are multiplied by 2^ref at the end.  Products are formed transposed (weights as MFMA rows): a lane holds four consecutive
// columns of a row of Y.
#include "mx.h"

namespace poss {

constexpr int F16_SHIFT = 13;     // fp16 operands carry 2^13: 6 * 2^13 is finite, and c * 2^(s - ref) exact down to s = ref - 36

template <typename T> struct MxOp;
template <> struct MxOp<bf16_t> {
    static constexpr int SHIFT = 0;
    static __device__ __forceinline__ u32x4 weights(unsigned q, float s) {     // eight codes as operand values
        union { u32x4 v; bf16x2 p[4]; } u;
        u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 0); u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 1);
        u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 2); u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 3);
        return u.v;
    }
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct MxOp<f16_t> {
    static constexpr int SHIFT = F16_SHIFT;
    static __device__ __forceinline__ u32x4 weights(unsigned q, float s) {
        union { u32x4 v; f16x2 p[4]; } u;
        u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, s, 0); u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, s, 1);
        u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, s, 2); u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, s, 3);
        return u.v;
    }
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};
// The scale of k-step s (of a group of four) as the conversion's scale operand: its exponent field is the byte.
template <typename T, int S> __device__ __forceinline__ float mx_scale(unsigned four) {
    const unsigned f = (S < 3 ? four << (23 - 8 * S) : four >> 1) & 0x7f800000u;
    return __builtin_bit_cast(float, f + ((unsigned)MxOp<T>::SHIFT << 23));
}

__device__ const u32x4 mx_zero_piece = {0u, 0u, 0u, 0u};  // what a lane reads where its k lies beyond K

// The sums of four consecutive columns n.. of row m, times 2^ref, to Y.
template <typename Y> struct __attribute__((aligned(4 * sizeof(Y)))) MxQuad { Y v[4]; };
template <typename Y> __device__ __forceinline__ void mx_store(Y *__restrict__ y, int64_t ldy, bool quads, int m, int n, int N, f32x4 acc, const int32_t *__restrict__ ref, int shift) {
    MxQuad<Y> o;
    const int4 e = *reinterpret_cast<const int4 *>(ref + n);
    const int es[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
    for (int r = 0; r < 4; ++r) o.v[r] = from_f<Y>(es[r] == 255 ? __builtin_nanf("") : __builtin_ldexpf(acc[r], es[r] - 127 - shift));
    Y *dst = y + (int64_t)m * ldy + n;
    if (quads) *reinterpret_cast<MxQuad<Y> *>(dst) = o;   // (n, N and ldy are multiples of four then, and y is aligned)
    else
#pragma unroll
        for (int r = 0; r < 4; ++r) if (n + r < N) dst[r] = o.v[r];
}

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// X as the 16-bit kernels read it: rows of 16-byte pieces.  PARTS > 1: the parts lie `part` values apart.
struct MxRows { const void *x; int64_t ldx, part; int K; };

// ------------------------------------------------------------------------------------------ staging
// float32 activations enter as the sum of three bf16 numbers, each the leading eight bits of what is left: exact.  Infinities and NaN
// are the first number alone.
__device__ __forceinline__ void split3(float x, bf16_t &a, bf16_t &b, bf16_t &c) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const bool special = (u & 0x7f800000u) == 0x7f800000u;
    const unsigned top = special && (u & 0x7fffffu) ? (u >> 16) | 0x40u : u >> 16;
    const float r1 = special ? 0.f : x - __builtin_bit_cast(float, u & 0xffff0000u);
    const unsigned u1 = __builtin_bit_cast(unsigned, r1);
    const float r2 = r1 - __builtin_bit_cast(float, u1 & 0xffff0000u);
    a = __builtin_bit_cast(bf16_t, (uint16_t)top);
    b = __builtin_bit_cast(bf16_t, (uint16_t)(u1 >> 16));
    c = (bf16_t)r2;                                       // at most eight bits: no rounding but below 2^-133
}

// X whose rows cannot be read in 16-byte pieces (odd lengths, distances or addresses), and float32 X: a copy in rows of Kp values,
// zeros beyond K; of float32 the three parts, a matrix each.
template <typename X> __global__ __launch_bounds__(256) void mx_stage_kernel(const X *__restrict__ x, int64_t ldx, int M, int K, int Kp, u32x4 *__restrict__ out) {
    const int k0 = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (k0 >= Kp) return;
    for (int m = blockIdx.y; m < M; m += gridDim.y) {
        const X *row = x + (int64_t)m * ldx;
        X v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = k0 + j < K ? row[k0 + j] : from_f<X>(0.f);
        u32x4 *dst = out + ((int64_t)m * Kp + k0) / 8;
        if constexpr (sizeof(X) == 2) {
            union { X e[8]; u32x4 u; } o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o.e[j] = v[j];
            *dst = o.u;
        } else {
            union { bf16_t e[8]; u32x4 u; } a, b, c;
#pragma unroll
            for (int j = 0; j < 8; ++j) split3(v[j], a.e[j], b.e[j], c.e[j]);
            const int64_t part = (int64_t)M * Kp / 8;
            dst[0] = a.u; dst[part] = b.u; dst[2 * part] = c.u;
        }
    }
}

// ------------------------------------------------------------------------------------------ few rows
// Up to 64 rows: the weights are what is read.  A workgroup owns NT column tiles and all of K, cut among its waves in whole groups of four
// k-steps; each wave reads its weights (1 KB per tile and k-step, contiguous) and its part of X (from the L2) straight into
// operand registers, the next group's on the way while this one is multiplied, and the waves' sums are added in LDS, in wave order.
// No planes, no second launch.
constexpr int mx_waves_max(int mt, int nt) { return 64 / (mt * nt) < 16 ? 64 / (mt * nt) : 16; }   // the waves' sums stay within 64 KB of LDS

template <typename T, typename Y, int MT, int NT, int PARTS>
__global__ __launch_bounds__(mx_waves_max(MT, NT) * 64) void mx_stream_kernel(MxPacked w, MxRows x, Y *__restrict__ y, int64_t ldy, bool quads, int M, int N) {
    extern __shared__ f32x4 red[];
    typedef MxOp<T> Op;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int ct0 = blockIdx.x * NT, g0 = wave * w.kgroups / waves, g1 = (wave + 1) * w.kgroups / waves;
    f32x4 acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (g0 < g1) {
        const u32x4 *wp[NT];
        const uint32_t *sp[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int ct = min(ct0 + nt, w.tiles - 1);    // tiles beyond the matrix repeat the last one (never stored)
            wp[nt] = w.codes + ((size_t)ct * w.ksteps + g0 * 4) * 64 + lane;
            sp[nt] = w.scales + ((size_t)ct * w.kgroups + g0) * 64 + lane;
        }
        const T *xp[MT];
        const int kl = (lane >> 4) * MX_BLOCK;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) xp[mt] = static_cast<const T *>(x.x) + (int64_t)min(mt * 16 + (lane & 15), M - 1) * x.ldx + g0 * 4 * MX_KSTEP + kl;
        u32x4 c[4][NT], xv[4][PARTS][MT];
        uint32_t sc[NT], sn[NT];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) c[s][nt] = wp[nt][s * 64];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sn[nt] = *sp[nt];
        // piece i of k-step s (of the group at g) for every row tile
        auto load_x = [&](auto tail, int g, int s, int i) {
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const T *a = xp[mt] + p * x.part + s * MX_KSTEP + i * 8;
                    if constexpr (decltype(tail)::value) a = (g * 4 + s) * MX_KSTEP + kl + i * 8 < x.K ? a : reinterpret_cast<const T *>(&mx_zero_piece);
                    xv[i][p][mt] = *reinterpret_cast<const u32x4 *>(a);
                }
        };
        // one group; `more`: another follows, whose weights are asked for as this one's are used up
        auto group = [&](auto more, auto tail, int g) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) { sc[nt] = sn[nt]; if constexpr (decltype(more)::value) { sp[nt] += 64; sn[nt] = *sp[nt]; } }
#pragma unroll
            for (int i = 0; i < 4; ++i) load_x(tail, g, 0, i);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                float f[NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) f[nt] = s == 0 ? mx_scale<T, 0>(sc[nt]) : s == 1 ? mx_scale<T, 1>(sc[nt]) : s == 2 ? mx_scale<T, 2>(sc[nt]) : mx_scale<T, 3>(sc[nt]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const u32x4 v = Op::weights(c[s][nt][i], f[nt]);
#pragma unroll
                        for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) acc[mt][nt] = Op::mfma(v, xv[i][p][mt], acc[mt][nt]);
                    }
                    if (s < 3) load_x(tail, g, s + 1, i);
                }
                if constexpr (decltype(more)::value)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) c[s][nt] = wp[nt][(s + 4) * 64];
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) wp[nt] += 256;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) xp[mt] += 4 * MX_KSTEP;
        };
        int g = g0;
        for (; g + 1 < g1; ++g) group(Yes{}, No{}, g);
        if ((g + 1) * 4 * MX_KSTEP <= x.K) group(No{}, No{}, g); else group(No{}, Yes{}, g);
    }
    // the waves' sums
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) red[((wave * MT + mt) * NT + nt) * 64 + lane] = acc[mt][nt];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * NT * 64; i += blockDim.x) {
        f32x4 a = red[i];
        for (int v = 1; v < waves; ++v) a += red[v * MT * NT * 64 + i];
        const int l = i & 63, nt = (i >> 6) % NT, m = ((i >> 6) / NT) * 16 + (l & 15), n = (ct0 + nt) * 16 + (l >> 4) * 4;
        if (m < M && n < N) mx_store<Y>(y, ldy, quads, m, n, N, a, w.ref, Op::SHIFT);
    }
}

// The same with microscaled X: a block of 16 bytes and its scale per lane, row tile and k-step.
template <typename Y, int MT, int NT>
__global__ __launch_bounds__(mx_waves_max(MT, NT) * 64) void mx_stream_both_kernel(MxPacked w, const u32x4 *__restrict__ x, const uint8_t *__restrict__ xs, int blocks, Y *__restrict__ y, int64_t ldy,
                                                              bool quads, int M, int N) {
    extern __shared__ f32x4 red[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int ct0 = blockIdx.x * NT, g0 = wave * w.kgroups / waves, g1 = (wave + 1) * w.kgroups / waves;
    f32x4 acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (g0 < g1) {
        const u32x4 *wp[NT];
        const uint32_t *sp[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int ct = min(ct0 + nt, w.tiles - 1);
            wp[nt] = w.codes + ((size_t)ct * w.ksteps + g0 * 4) * 64 + lane;
            sp[nt] = w.scales + ((size_t)ct * w.kgroups + g0) * 64 + lane;
        }
        int64_t xr[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) xr[mt] = (int64_t)min(mt * 16 + (lane & 15), M - 1) * blocks;
        u32x4 c[4][NT], xv[4][MT];
        uint32_t sc[NT], sn[NT];
        int xc[4][MT];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) c[s][nt] = wp[nt][s * 64];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sn[nt] = *sp[nt];
        auto load_x = [&](int g, int s) {
            const int b = (g * 4 + s) * 4 + (lane >> 4);
            const bool in = b < blocks;                    // (a block of another row must not lend its scale: it may be NaN)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                xv[s][mt] = *(in ? x + xr[mt] + b : &mx_zero_piece);
                const int t = xs[xr[mt] + (in ? b : blocks - 1)];
                xc[s][mt] = in ? t : 127;
            }
        };
#pragma unroll
        for (int s = 0; s < 4; ++s) load_x(g0, s);
        auto group = [&](auto more, int g) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) { sc[nt] = sn[nt]; if constexpr (decltype(more)::value) { sp[nt] += 64; sn[nt] = *sp[nt]; } }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const i32x8 a = {(int)c[s][nt].x, (int)c[s][nt].y, (int)c[s][nt].z, (int)c[s][nt].w, 0, 0, 0, 0};
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        const i32x8 b = {(int)xv[s][mt].x, (int)xv[s][mt].y, (int)xv[s][mt].z, (int)xv[s][mt].w, 0, 0, 0, 0};
                        if (s == 0) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[mt][nt], 4, 4, 0, (int)sc[nt], 0, xc[s][mt]);
                        else if (s == 1) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[mt][nt], 4, 4, 1, (int)sc[nt], 0, xc[s][mt]);
                        else if (s == 2) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[mt][nt], 4, 4, 2, (int)sc[nt], 0, xc[s][mt]);
                        else acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[mt][nt], 4, 4, 3, (int)sc[nt], 0, xc[s][mt]);
                    }
                }
                if constexpr (decltype(more)::value) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) c[s][nt] = wp[nt][(s + 4) * 64];
                    load_x(g + 1, s);
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) wp[nt] += 256;
        };
        int g = g0;
        for (; g + 1 < g1; ++g) group(Yes{}, g);
        group(No{}, g);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) red[((wave * MT + mt) * NT + nt) * 64 + lane] = acc[mt][nt];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * NT * 64; i += blockDim.x) {
        f32x4 a = red[i];
        for (int v = 1; v < waves; ++v) a += red[v * MT * NT * 64 + i];
        const int l = i & 63, nt = (i >> 6) % NT, m = ((i >> 6) / NT) * 16 + (l & 15), n = (ct0 + nt) * 16 + (l >> 4) * 4;
        if (m < M && n < N) mx_store<Y>(y, ldy, quads, m, n, N, a, w.ref, 0);
    }
}

// ------------------------------------------------------------------------------------------ launches
constexpr int MX_STREAM_ROWS = 64;

template <typename T, typename Y, int MT, int NT, int PARTS>
static void launch_stream_c(const MxPacked &w, const MxRows &x, void *y, int64_t ldy, bool quads, int M, int N, int waves, hipStream_t st) {
    if (waves > mx_waves_max(MT, NT)) waves = mx_waves_max(MT, NT);
    mx_stream_kernel<T, Y, MT, NT, PARTS><<<(w.tiles + NT - 1) / NT, waves * 64, waves * MT * NT * 1024, st>>>(w, x, static_cast<Y *>(y), ldy, quads, M, N);
}
template <typename T, typename Y, int PARTS>
static void launch_stream(const MxPacked &w, const MxRows &x, void *y, int64_t ldy, bool quads, int M, int N, int nt, int waves, hipStream_t st) {
    const int mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
#define POSS_MX(MT, NT) return launch_stream_c<T, Y, MT, NT, PARTS>(w, x, y, ldy, quads, M, N, waves, st)
    if (mt == 1) { if (nt == 1) POSS_MX(1, 1); if (nt == 2) POSS_MX(1, 2); POSS_MX(1, 4); }
    if constexpr (PARTS == 3) { if (nt == 1) POSS_MX(2, 1); POSS_MX(2, 2); }
    else {
        if (mt == 2) { if (nt == 1) POSS_MX(2, 1); if (nt == 2) POSS_MX(2, 2); POSS_MX(2, 4); }
        if (nt == 1) POSS_MX(4, 1); if (nt == 2) POSS_MX(4, 2); POSS_MX(4, 4);
    }
#undef POSS_MX
}
template <typename Y>
static void launch_stream_both(const MxPacked &w, const void *x, const void *xs, int blocks, void *y, int64_t ldy, bool quads, int M, int N, int nt, int waves, hipStream_t st) {
    const int mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    if (waves > mx_waves_max(mt, nt)) waves = mx_waves_max(mt, nt);
#define POSS_MX(MT, NT) return mx_stream_both_kernel<Y, MT, NT><<<(w.tiles + NT - 1) / NT, waves * 64, waves * MT * NT * 1024, st>>>( \
        w, static_cast<const u32x4 *>(x), static_cast<const uint8_t *>(xs), blocks, static_cast<Y *>(y), ldy, quads, M, N)
    if (mt == 1) { if (nt == 1) POSS_MX(1, 1); if (nt == 2) POSS_MX(1, 2); POSS_MX(1, 4); }
    if (mt == 2) { if (nt == 1) POSS_MX(2, 1); if (nt == 2) POSS_MX(2, 2); POSS_MX(2, 4); }
    if (nt == 1) POSS_MX(4, 1); if (nt == 2) POSS_MX(4, 2); POSS_MX(4, 4);
#undef POSS_MX
}

struct StreamShape { int nt, waves; };
static StreamShape stream_shape(int, int, int) { return StreamShape{1, 8}; }

// Whether X can be read as it is: rows of whole 16-byte pieces.
static bool rows_ok(int x_dt, const void *x, int64_t ldx, int K) {
    return x_dt != DT_F32 && reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx % 8 == 0 && K % 8 == 0;
}
static bool quads_ok(const void *y, int64_t ldy, int N, int y_dt) {
    return N % 4 == 0 && ldy % 4 == 0 && reinterpret_cast<uintptr_t>(y) % (4 * dtype_size(y_dt)) == 0;
}

size_t mx_gemm_scratch_size(int x_dt, int M, int N, int K) {
    if (x_dt == DT_MX) return 256;
    const size_t kp = (size_t)(K + 4 * MX_KSTEP - 1) / (4 * MX_KSTEP) * (4 * MX_KSTEP);
    return ((size_t)M * kp * 2 * (x_dt == DT_F32 ? 3 : 1) + 255) / 256 * 256 + 256;
}

static MxRows stage(int x_dt, const void *x, int64_t ldx, int M, int K, int kp, void *scratch, hipStream_t st) {
    const dim3 grid((kp / 8 + 255) / 256, M < 65535 ? M : 65535);
    u32x4 *o = static_cast<u32x4 *>(scratch);
    if (x_dt == DT_F32) mx_stage_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float *>(x), ldx, M, K, kp, o);
    else mx_stage_kernel<uint16_t><<<grid, 256, 0, st>>>(static_cast<const uint16_t *>(x), ldx, M, K, kp, o);
    return MxRows{scratch, kp, (int64_t)M * kp, kp};
}

template <typename T, int PARTS>
static void launch_gemm_t(const MxPacked &w, MxRows x, int y_dt, char *y, int64_t ldy, bool quads, int M, int N, hipStream_t st) {
    const int rows = PARTS == 3 ? 32 : MX_STREAM_ROWS;
    const StreamShape sh = stream_shape(M, N, w.kgroups);
    for (int m = 0; m < M; m += rows) {
        MxRows xr = x;
        xr.x = static_cast<const T *>(x.x) + m * x.ldx;
        char *yr = y + m * ldy * (int64_t)dtype_size(y_dt);
        const int n = M - m < rows ? M - m : rows;
        if (y_dt == DT_F32) launch_stream<T, float, PARTS>(w, xr, yr, ldy, quads, n, N, sh.nt, sh.waves, st);
        else if (y_dt == DT_BF16) launch_stream<T, bf16_t, PARTS>(w, xr, yr, ldy, quads, n, N, sh.nt, sh.waves, st);
        else launch_stream<T, f16_t, PARTS>(w, xr, yr, ldy, quads, n, N, sh.nt, sh.waves, st);
    }
}

void launch_mx_gemm(int x_dt, const void *x, int64_t ldx, const void *packed, int y_dt, void *y, int64_t ldy, int M, int N, int K, void *scratch, hipStream_t st) {
    const MxPacked w = mx_packed_at(packed, N, K);
    const MxRows r = rows_ok(x_dt, x, ldx, K) ? MxRows{x, ldx, 0, K} : stage(x_dt, x, ldx, M, K, w.ksteps * MX_KSTEP, scratch, st);
    const bool quads = quads_ok(y, ldy, N, y_dt);
    if (x_dt == DT_F32) launch_gemm_t<bf16_t, 3>(w, r, y_dt, static_cast<char *>(y), ldy, quads, M, N, st);
    else if (x_dt == DT_BF16) launch_gemm_t<bf16_t, 1>(w, r, y_dt, static_cast<char *>(y), ldy, quads, M, N, st);
    else launch_gemm_t<f16_t, 1>(w, r, y_dt, static_cast<char *>(y), ldy, quads, M, N, st);
}

void launch_mx_gemm_mx(const void *x_codes, const void *x_scales, const void *packed, int y_dt, void *y, int64_t ldy, int M, int N, int K, void *, hipStream_t st) {
    const MxPacked w = mx_packed_at(packed, N, K);
    const bool quads = quads_ok(y, ldy, N, y_dt);
    const int nb = mx_blocks(K);
    const StreamShape sh = stream_shape(M, N, w.kgroups);
    for (int m = 0; m < M; m += MX_STREAM_ROWS) {
        const char *c = static_cast<const char *>(x_codes) + (int64_t)m * nb * 16, *s = static_cast<const char *>(x_scales) + (int64_t)m * nb;
        char *yr = static_cast<char *>(y) + m * ldy * (int64_t)dtype_size(y_dt);
        const int n = M - m < MX_STREAM_ROWS ? M - m : MX_STREAM_ROWS;
        if (y_dt == DT_F32) launch_stream_both<float>(w, c, s, nb, yr, ldy, quads, n, N, sh.nt, sh.waves, st);
        else if (y_dt == DT_BF16) launch_stream_both<bf16_t>(w, c, s, nb, yr, ldy, quads, n, N, sh.nt, sh.waves, st);
        else launch_stream_both<f16_t>(w, c, s, nb, yr, ldy, quads, n, N, sh.nt, sh.waves, st);
    }
}

}  // namespace poss
