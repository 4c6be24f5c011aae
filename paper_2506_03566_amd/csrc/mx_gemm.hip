// Y[m][n] = sum_k X[m][k] W[n][k] with W microscaled in 4 bits and packed in operand order (mx.hip), X in 32 or 16 bits or
// microscaled as well.
//
// 16-bit X: a weight becomes a number in the type of X (one conversion instruction for two, exact; fp16: relative to its row's largest) and enters
// v_mfma_f32_16x16x32; the 32 codes that a lane holds per k-step are the k values of four such instructions, lane / 16 choosing the block of
// 32 and the instruction eight values of it, so that a lane takes 64 contiguous bytes of a row of X.
// float32 X: the sum of three bf16 numbers, three instructions.  Microscaled X: v_mfma_scale with both scales, one block per lane.
// What the operands leave out of 2^ref is applied to the sums at the end.  Products are formed transposed (weights as MFMA rows): a lane holds four consecutive
// columns of a row of Y.
#include "mx.h"

namespace poss {

constexpr int F16_SHIFT = 13;     // fp16 operands are c * 2^(s - ref) times 2^13: 6 * 2^13 is finite, and they are exact down to s = ref - 36

// SHIFT: 0 where operands are as the packed scales have them.  scale: a block's scale as the conversion's operand, whose exponent field is the byte,
// moved by what move gives for the block's row; weights below what fp16 can hold round to zero there, at 2^-127 too.
template <typename T> struct MxOp;
template <> struct MxOp<bf16_t> {
    static constexpr int SHIFT = 0;
    static __device__ __forceinline__ int move(const int32_t *, int) { return 0; }
    static __device__ __forceinline__ float scale(unsigned byte_at_23, int) { return __builtin_bit_cast(float, byte_at_23); }
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
    static __device__ __forceinline__ int move(const int32_t *__restrict__ ref, int n) { return (127 + SHIFT - mx_held(mx_row_top(ref[n]))) * (1 << 23); }
    static __device__ __forceinline__ float scale(unsigned byte_at_23, int move) { return __builtin_bit_cast(float, max(0, (int)byte_at_23 + move)); }
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
template <typename T, int S> __device__ __forceinline__ float mx_scale(unsigned four, int move) {
    return MxOp<T>::scale((S < 3 ? four << (23 - 8 * S) : four >> 1) & 0x7f800000u, move);
}

__device__ const u32x4 mx_zero_piece = {0u, 0u, 0u, 0u};  // what a lane reads where its k lies beyond K

// The sums of four consecutive columns n.. of row m to Y, times what their operands leave out: shift 0: of the packed form, otherwise all of 2^ref.
__device__ __forceinline__ float mx_result(float a, int ref, int shift) {
    return ref == MX_NAN_ROW ? __builtin_nanf("") : __builtin_ldexpf(a, shift ? mx_row_top(ref) - 127 - shift : mx_row_power(ref));
}
template <typename Y> struct __attribute__((aligned(4 * sizeof(Y)))) MxQuad { Y v[4]; };
template <typename Y> __device__ __forceinline__ MxQuad<Y> mx_scaled(f32x4 a, int4 e, int shift) {
    MxQuad<Y> o;
    const int es[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
    for (int r = 0; r < 4; ++r) o.v[r] = from_f<Y>(mx_result(a[r], es[r], shift));
    return o;
}
template <typename Y> __device__ __forceinline__ MxQuad<Y> mx_scaled(f32x4 a, const int32_t *__restrict__ ref, int n, int shift) {
    return mx_scaled<Y>(a, *reinterpret_cast<const int4 *>(ref + n), shift);
}
template <typename Y> __device__ __forceinline__ MxQuad<Y> mx_raw(f32x4 a) { MxQuad<Y> o; for (int r = 0; r < 4; ++r) o.v[r] = (Y)a[r]; return o; }
template <typename Y> __device__ __forceinline__ void mx_store_quad(Y *__restrict__ dst, bool quads, int left, const MxQuad<Y> &o) {
    if (quads) *reinterpret_cast<MxQuad<Y> *>(dst) = o;   // (columns, N and ldy are multiples of four then, and y is aligned)
    else
#pragma unroll
        for (int r = 0; r < 4; ++r) if (r < left) dst[r] = o.v[r];
}
template <typename Y> __device__ __forceinline__ void mx_store(Y *__restrict__ y, int64_t ldy, bool quads, int m, int n, int N, f32x4 acc, const int32_t *__restrict__ ref, int shift) {
    mx_store_quad<Y>(y + (int64_t)m * ldy + n, quads, N - n, mx_scaled<Y>(acc, ref, n, shift));
}

// Results of the largest tiles go past the caches: 8192 x 28672 x 4096 in 480 us instead of 503 (16-bit X 1314, 1361); a pass over the results right
// behind it makes the pair take as long either way (659 us).  Planes are read at once and stay.
template <typename Y> __device__ __forceinline__ void mx_store_piece(Y *p, u32x4 v, bool past) {
    if (past) __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
    else *reinterpret_cast<u32x4 *>(p) = v;
}

// ROWS rows x COLS columns of float32 sums that a wave holds, to Y (times what the operands leave out) or to a plane, in pieces of 16 bytes: from the lanes' quads
// through LDS of the wave's own (rows padded by 16 bytes).  A lane's quads of a row, as they are, would be written 8 bytes here and
// there: 256 x 256 tiles of 8192 x 28672 results took 24 us a round for them, of 59.
// put(f): calls f(row, column, sums) for each quad.
template <typename Y, int ROWS, int COLS, bool PAST, typename Put>
__device__ __forceinline__ void mx_store_rows(char *lds, Put put, int m0, int n0, int M, int N, Y *__restrict__ y, int64_t ldy) {
    constexpr int ROW = COLS * (int)sizeof(Y) + 16, LPR = COLS * (int)sizeof(Y) / 16, RPI = 64 / LPR;      // lanes a row, rows an instruction
    const int lane = threadIdx.x & 63;
    put([&](int r, int c, const MxQuad<Y> &v) { *reinterpret_cast<MxQuad<Y> *>(lds + r * ROW + c * (int)sizeof(Y)) = v; });
    wave_lds_sync();
    const int c = (lane % LPR) * (16 / (int)sizeof(Y));
#pragma unroll
    for (int r = lane / LPR; r < ROWS; r += RPI) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(lds + r * ROW + c * (int)sizeof(Y));
        if (m0 + r < M && n0 + c < N) mx_store_piece(y + (int64_t)(m0 + r) * ldy + n0 + c, v, PAST);
    }
    wave_lds_sync();                                      // (the next rows go to the same place)
}
template <typename T> __device__ __forceinline__ MxQuad<T> mx_silu_quad(const MxQuad<float> &gate, const MxQuad<float> &up) {
    MxQuad<T> o;
#pragma unroll
    for (int r = 0; r < 4; ++r) o.v[r] = mul_round<T>(gate.v[r] / (1.0f + expf(-gate.v[r])), up.v[r]);
    return o;
}

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };
template <int I> struct Num { static constexpr int value = I; };

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
// zeros beyond K; of float32 the three parts, one after the other.  wide: rows of x can be read in pieces of 16 bytes.
template <typename X> __global__ __launch_bounds__(256) void mx_stage_kernel(const X *__restrict__ x, int64_t ldx, bool wide, int M, int K, int Kp, u32x4 *__restrict__ out) {
    const int k0 = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (k0 >= Kp) return;
    for (int m = blockIdx.y; m < M; m += gridDim.y) {
        const X *row = x + (int64_t)m * ldx;
        union { u32x4 u[sizeof(X) / 2]; X v[8]; } in;
        if (wide && k0 + 8 <= K)
#pragma unroll
            for (int j = 0; j < (int)sizeof(X) / 2; ++j) in.u[j] = reinterpret_cast<const u32x4 *>(row + k0)[j];
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) in.v[j] = k0 + j < K ? row[k0 + j] : from_f<X>(0.f);
        u32x4 *dst = out + ((int64_t)m * Kp * (sizeof(X) == 2 ? 1 : 3) + k0) / 8;
        if constexpr (sizeof(X) == 2) *dst = in.u[0];
        else {
            union { bf16_t e[8]; u32x4 u; } a, b, c;
#pragma unroll
            for (int j = 0; j < 8; ++j) split3(in.v[j], a.e[j], b.e[j], c.e[j]);
            dst[0] = a.u; dst[Kp / 8] = b.u; dst[Kp / 4] = c.u;
        }
    }
}

// ------------------------------------------------------------------------------------------ few rows
// Up to sixteen rows: a workgroup owns a column tile and all of K, cut among its waves in whole groups of four k-steps.  Each wave reads its
// weights (1 KB per k-step, contiguous) and its part of X (from the L2) straight into operand registers, the next group's on the way while
// this one is multiplied; the waves' sums are added in LDS, in wave order.  Nothing is waited for but memory: one row of 28672 x 4096 11.9 us
// (62.5 MB at 5.3 TB/s), 4096 x 4096 3.7.  Slower: X through LDS (a barrier behind a trip to memory: 6.0 for 3.7), two groups ahead (6144 x 4096
// 6.5 for 5.5).  With rows X counts (16 bytes at a time, once per column tile): 16 rows 30 us, where mx_fed_kernel takes 12.8.
// The waves' sums in the first wave (true there).
__device__ __forceinline__ bool mx_stream_sum(f32x4 *red, f32x4 &acc) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    red[wave * 64 + lane] = acc;
    __syncthreads();
    if (wave) return false;
    for (int v = 1; v < waves; ++v) acc += red[v * 64 + lane];
    return true;
}

template <typename T, typename Y, int PARTS>
__global__ __launch_bounds__(1024) void mx_stream_kernel(MxPacked w, MxRows x, Y *__restrict__ y, int64_t ldy, bool quads, int M, int N) {
    extern __shared__ f32x4 red[];
    typedef MxOp<T> Op;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int ct = blockIdx.x, g0 = wave * w.kgroups / waves, g1 = (wave + 1) * w.kgroups / waves, kl = (lane >> 4) * MX_BLOCK;     // (every wave has a group)
    const u32x4 *wp = w.codes + ((size_t)ct * w.ksteps + g0 * 4) * 64 + lane;
    const uint32_t *sp = w.scales + ((size_t)ct * w.kgroups + g0) * 64 + lane;
    const T *xp = static_cast<const T *>(x.x) + (int64_t)min(lane & 15, M - 1) * x.ldx + g0 * 4 * MX_KSTEP + kl;
    const int move = Op::move(w.ref, ct * 16 + (lane & 15));
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    u32x4 c[4], xv[4][PARTS];
    uint32_t next = *sp;
#pragma unroll
    for (int s = 0; s < 4; ++s) c[s] = wp[s * 64];
    // piece i of k-step s of the group at g
    auto load_x = [&](auto tail, int g, int s, int i) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const T *a = xp + p * x.part + s * MX_KSTEP + i * 8;
            if constexpr (decltype(tail)::value) a = (g * 4 + s) * MX_KSTEP + kl + i * 8 < x.K ? a : reinterpret_cast<const T *>(&mx_zero_piece);
            xv[i][p] = *reinterpret_cast<const u32x4 *>(a);
        }
    };
    // one group; `more`: another follows, whose weights are asked for as this one's are used up; `tail`: X ends in it
    auto group = [&](auto more, auto tail, int g) {
        const uint32_t sc = next;
        if constexpr (decltype(more)::value) { sp += 64; next = *sp; }
#pragma unroll
        for (int i = 0; i < 4; ++i) load_x(tail, g, 0, i);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const float f = s == 0 ? mx_scale<T, 0>(sc, move) : s == 1 ? mx_scale<T, 1>(sc, move) : s == 2 ? mx_scale<T, 2>(sc, move) : mx_scale<T, 3>(sc, move);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32x4 v = Op::weights(c[s][i], f);
#pragma unroll
                for (int p = PARTS - 1; p >= 0; --p) acc = Op::mfma(v, xv[i][p], acc);
                if (s < 3) load_x(tail, g, s + 1, i);
            }
            if constexpr (decltype(more)::value) c[s] = wp[(s + 4) * 64];
        }
        wp += 256;
        xp += 4 * MX_KSTEP;
    };
    int g = g0;
    for (; g + 1 < g1; ++g) group(Yes{}, No{}, g);
    if ((g + 1) * 4 * MX_KSTEP <= x.K) group(No{}, No{}, g); else group(No{}, Yes{}, g);
    if (!mx_stream_sum(red, acc)) return;
    const int m = lane & 15, n = ct * 16 + (lane >> 4) * 4;
    if (m < M && n < N) mx_store<Y>(y, ldy, quads, m, n, N, acc, w.ref, Op::SHIFT);
}

// The same with microscaled X: a block of 16 bytes and its scale per lane and k-step.
template <typename Y>
__global__ __launch_bounds__(1024) void mx_stream_both_kernel(MxPacked w, const u32x4 *__restrict__ x, const uint8_t *__restrict__ xs, int blocks, Y *__restrict__ y, int64_t ldy,
                                                              bool quads, int M, int N) {
    extern __shared__ f32x4 red[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int ct = blockIdx.x, g0 = wave * w.kgroups / waves, g1 = (wave + 1) * w.kgroups / waves;
    const u32x4 *wp = w.codes + ((size_t)ct * w.ksteps + g0 * 4) * 64 + lane;
    const uint32_t *sp = w.scales + ((size_t)ct * w.kgroups + g0) * 64 + lane;
    const int64_t xr = (int64_t)min(lane & 15, M - 1) * blocks;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    u32x4 c[4], xv[4];
    uint32_t next = *sp;
    int xc[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) c[s] = wp[s * 64];
    auto load_x = [&](int g, int s) {
        const int b = (g * 4 + s) * 4 + (lane >> 4);
        const bool in = b < blocks;                        // (a block of another row must not lend its scale: it may be NaN)
        xv[s] = *(in ? x + xr + b : &mx_zero_piece);
        const int t = xs[xr + (in ? b : blocks - 1)];
        xc[s] = in ? t : 127;
    };
#pragma unroll
    for (int s = 0; s < 4; ++s) load_x(g0, s);
    auto group = [&](auto more, int g) {
        const uint32_t sc = next;
        if constexpr (decltype(more)::value) { sp += 64; next = *sp; }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const i32x8 a = {(int)c[s].x, (int)c[s].y, (int)c[s].z, (int)c[s].w, 0, 0, 0, 0}, b = {(int)xv[s].x, (int)xv[s].y, (int)xv[s].z, (int)xv[s].w, 0, 0, 0, 0};
            if (s == 0) acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, (int)sc, 0, xc[s]);
            else if (s == 1) acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 1, (int)sc, 0, xc[s]);
            else if (s == 2) acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 2, (int)sc, 0, xc[s]);
            else acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 3, (int)sc, 0, xc[s]);
            if constexpr (decltype(more)::value) {
                c[s] = wp[(s + 4) * 64];
                load_x(g + 1, s);
            }
        }
        wp += 256;
    };
    int g = g0;
    for (; g + 1 < g1; ++g) group(Yes{}, g);
    group(No{}, g);
    if (!mx_stream_sum(red, acc)) return;
    const int m = lane & 15, n = ct * 16 + (lane >> 4) * 4;
    if (m < M && n < N) mx_store<Y>(y, ldy, quads, m, n, N, acc, w.ref, 0);
}

// ------------------------------------------------------------------------------------------ many rows
// A workgroup owns TM rows x TN columns and all of K or a part of it (whose sums go to a plane).  X goes from memory straight into LDS,
// one k-step of 128 per stage, two stages; the codes of a wave's own columns go into its registers (the weights of a k-step are a
// quarter of X's bytes, and LDS reads are what a tile has least of) and are converted there, one k-step ahead.  A k-step is four
// substeps of one matrix instruction per 16 x 16 tile; while a wave multiplies a substep it converts the next one's weights and reads
// X's operands a few tiles ahead from LDS.  One barrier per k-step, where those reads pass into the next stage: that has landed by then,
// and every operand of this one has been read, so that its place can be asked for again.
struct MxGeom {
    int M, N, steps;              // k-steps of the product: float32 X is three times as long (its parts one after the other)
    int full;                     // k-steps that lie inside X's rows as a whole
    int tiles_m, tiles_n, splits;
    int plane_ld;                 // planes: [M][plane_ld] each,
    bool plane_scaled;            // times what the operands leave out already
};

// Workgroup -> tile: consecutive ids go to the 8 XCDs in turn; an XCD is given a contiguous run of tiles, ordered so that those it works
// on at a time share rows and columns in its L2.
__device__ __forceinline__ void mx_tile_of(const MxGeom &g, int bid, int gm_rows, int &tm, int &tn) {
    const int n = g.tiles_m * g.tiles_n, q = n >> 3, r = n & 7, x = bid & 7;
    const int id = x * q + (x < r ? x : r) + (bid >> 3);
    const int grp = id / (gm_rows * g.tiles_n), in_grp = id - grp * (gm_rows * g.tiles_n), gm = min(gm_rows, g.tiles_m - grp * gm_rows);
    tm = grp * gm_rows + in_grp % gm;
    tn = in_grp / gm;
}

// This split's k-steps: whole groups of four, the last split's as far as the product goes.
__device__ __forceinline__ void mx_split_of(const MxGeom &g, int &s0, int &n) {
    const int groups = (g.steps + 3) >> 2;
    s0 = (int)((int64_t)blockIdx.y * groups / g.splits) * 4;
    n = min((int)((int64_t)(blockIdx.y + 1) * groups / g.splits) * 4, g.steps) - s0;
}

// Four consecutive columns to a plane.
template <int SHIFT> __device__ __forceinline__ void mx_store_plane(float *p, f32x4 a, const MxGeom &g, const MxPacked &w, int col) {
    *reinterpret_cast<MxQuad<float> *>(p) = g.plane_scaled ? mx_scaled<float>(a, w.ref, col, SHIFT) : __builtin_bit_cast(MxQuad<float>, a);
}

// A wave's tiles to Y, or to this split's plane.  D tile: lane -> row lane % 16, register r -> column 4 (lane / 16) + r.
template <typename T, typename Y, int MTW, int NTW, bool SPLIT>
__device__ __forceinline__ void mx_tile_store(const f32x4 (&acc)[MTW][NTW], int row0, int ct0, const MxGeom &g, const MxPacked &w, Y *__restrict__ y, int64_t ldy, bool quads) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int mt = 0; mt < MTW; ++mt) {
        const int m = row0 + mt * 16 + (lane & 15);
        if (m >= g.M) continue;
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) {
            const int col = (ct0 + nt) * 16 + (lane >> 4) * 4;
            if (col >= g.N) continue;
            if constexpr (SPLIT) mx_store_plane<MxOp<T>::SHIFT>(y + ((size_t)blockIdx.y * g.M + m) * g.plane_ld + col, acc[mt][nt], g, w, col);
            else mx_store<Y>(y, ldy, quads, m, col, g.N, acc[mt][nt], w.ref, MxOp<T>::SHIFT);
        }
    }
}

// The same through LDS of the wave's own (16 rows of NTW * 16 columns and padding), where pieces of 16 bytes can be written.
template <typename T, typename Y, int MTW, int NTW, bool SPLIT>
__device__ __forceinline__ void mx_tile_store_wide(char *own, const f32x4 (&acc)[MTW][NTW], int row0, int ct0, const MxGeom &g, const MxPacked &w, Y *__restrict__ y, int64_t ldy) {
    const int lane = threadIdx.x & 63, cols = SPLIT ? w.tiles * 16 : g.N;
    Y *dst = SPLIT ? y + (size_t)blockIdx.y * g.M * g.plane_ld : y;
#pragma unroll
    for (int mt = 0; mt < MTW; ++mt)
        mx_store_rows<Y, 16, NTW * 16, !SPLIT && MTW >= 8>(own, [&](auto f) {
#pragma unroll
            for (int nt = 0; nt < NTW; ++nt) {
                const int c = nt * 16 + (lane >> 4) * 4;
                if (SPLIT && !g.plane_scaled) f(lane & 15, c, mx_raw<Y>(acc[mt][nt]));
                else f(lane & 15, c, mx_scaled<Y>(acc[mt][nt], w.ref, min(ct0 + nt, w.tiles - 1) * 16 + (lane >> 4) * 4, MxOp<T>::SHIFT));
            }
        }, row0 + mt * 16, ct0 * 16, g.M, cols, dst, SPLIT ? g.plane_ld : ldy);
}

template <typename T, typename Y, int TM, int TN, int WM, int WN, bool SPLIT>
__global__ __launch_bounds__(WM * WN * 64, 2) void mx_tile_kernel(MxPacked w, MxRows x, MxGeom g, Y *__restrict__ y, int64_t ldy, bool quads, bool wide) {
    typedef __attribute__((address_space(3))) void *LdsPtr;
    typedef MxOp<T> Op;
    constexpr int WAVES = WM * WN, MTW = TM / (16 * WM), NTW = TN / (16 * WN), UNITS = TM / 16 * 4, UPW = UNITS / WAVES;   // 1 KB units: 16 rows x 64 bytes
    static_assert(UPW * WAVES == UNITS && MTW >= 1 && NTW >= 1, "tile shape");
    __shared__ __attribute__((aligned(1024))) u32x4 xs[2 * UNITS * 64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, wm = wave % WM, wn = wave / WM;
    int tm, tn;
    mx_tile_of(g, blockIdx.x, 8, tm, tn);
    const int m0 = tm * TM, ct0 = tn * (TN / 16) + wn * NTW;
    int s0, n;
    mx_split_of(g, s0, n);

    // Unit u of a stage: rows 16 (u / 4).., columns 32 (u % 4).. of the k-step, four lanes per row; piece p (eight columns) of row r lies at
    // position p ^ (r / 4 % 4), so that sixteen lanes that read the same piece of sixteen rows meet every bank once.
    const int x_piece = (lane & 3) ^ ((lane >> 4) & 3);
    const T *x_base = static_cast<const T *>(x.x) + (int64_t)m0 * x.ldx;
    const unsigned lds0 = (unsigned)(uintptr_t)(LdsPtr)&xs[0];
    auto issue_one = [&](int j, int s, int st) {          // unit j (static) of this wave's share of k-step s, into stage st
        const int u = wave + WAVES * j, m = min((u >> 2) * 16 + (lane >> 2), g.M - 1 - m0);
        const unsigned dst = lds0 + (unsigned)((st * UNITS + u) * 1024);
        const int k = (u & 3) * MX_BLOCK + x_piece * 8;
        const unsigned off = ((unsigned)m * (unsigned)x.ldx + (unsigned)k) * 2u;     // (TM rows are below 4 GiB: checked on the host)
        const T *src = x_base + (int64_t)s * MX_KSTEP;
        if (s < g.full) lds_dma16_s(dst, src, off);
        else {
            const char *p = reinterpret_cast<const char *>(src) + off;
            lds_dma16(dst, s * MX_KSTEP + k < x.K ? static_cast<const void *>(p) : static_cast<const void *>(&mx_zero_piece));
        }
    };
    int ws = s0 % w.ksteps;                               // k-step of the weights: the next one to load
    const u32x4 *wp[NTW];
    const uint32_t *sp[NTW];
    int move[NTW];
#pragma unroll
    for (int nt = 0; nt < NTW; ++nt) {
        const int ct = min(ct0 + nt, w.tiles - 1);        // tiles beyond the matrix repeat the last one (never stored)
        wp[nt] = w.codes + (size_t)ct * w.ksteps * 64;
        sp[nt] = w.scales + (size_t)ct * w.kgroups * 64;
        move[nt] = Op::move(w.ref, ct * 16 + (lane & 15));
    }
    auto load_w = [&](u32x4 (&c)[NTW], float (&f)[NTW]) {
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) {
            c[nt] = wp[nt][ws * 64 + lane];
            f[nt] = Op::scale((sp[nt][(ws >> 2) * 64 + lane] >> (8 * (ws & 3)) & 255u) << 23, move[nt]);
        }
        ws = ws + 1 == w.ksteps ? 0 : ws + 1;
    };
    f32x4 acc[MTW][NTW];
#pragma unroll
    for (int mt = 0; mt < MTW; ++mt)
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};

    // A k-step is 4 MTW slots, one row tile of one substep each.  Operands of X are read AHEAD slots ahead, into a ring of four.
    constexpr int SLOTS = 4 * MTW, AHEAD = 3;
    u32x4 c[NTW], cn[NTW], xf[4], wf[2][NTW];
    float f[NTW], fn[NTW];
#pragma unroll
    for (int j = 0; j < UPW; ++j) issue_one(j, s0, 0);
    load_w(c, f);
    dma_wait<0>();
    __syncthreads();
    const int rd = (wm * MTW * 4 + (lane >> 4)) * 64 + (lane & 15) * 4, rs = (lane >> 2) & 3;      // + 256 per row tile, piece i at i ^ rs
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) xf[q] = xs[rd + (q % MTW) * 256 + ((q / MTW) ^ rs)];
#pragma unroll
    for (int nt = 0; nt < NTW; ++nt) wf[0][nt] = Op::weights(c[nt][0], f[nt]);

    for (int s = 0; s < n; ++s) {
        const u32x4 *cur = xs + (s & 1) * UNITS * 64, *nxt = xs + (~s & 1) * UNITS * 64;
        const bool more = s + 1 < n;
#pragma unroll
        for (int q = 0; q < SLOTS; ++q) {
            const int i = q / MTW, mt = q % MTW;
            if (q == SLOTS - AHEAD) {                     // (nobody reads this stage any more, and the next one has landed)
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                __syncthreads();
            }
            if (more && q == 0) load_w(cn, fn);
            if (more && q < MTW)
#pragma unroll
                for (int j = mt; j < UPW; j += MTW) issue_one(j, s0 + s + 1, ~s & 1);
            const int qa = (q + AHEAD) % SLOTS;
            xf[(q + AHEAD) & 3] = (q + AHEAD >= SLOTS ? nxt : cur)[rd + (qa % MTW) * 256 + ((qa / MTW) ^ rs)];
#pragma unroll
            for (int nt = mt; nt < NTW; nt += MTW)
                wf[(i + 1) & 1][nt] = i == 3 ? Op::weights(cn[nt][0], fn[nt]) : Op::weights(c[nt][(i + 1) & 3], f[nt]);
#pragma unroll
            for (int nt = 0; nt < NTW; ++nt) acc[mt][nt] = Op::mfma(wf[i & 1][nt], xf[q & 3], acc[mt][nt]);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) { c[nt] = cn[nt]; f[nt] = fn[nt]; }
    }
    if (!wide) {
        mx_tile_store<T, Y, MTW, NTW, SPLIT>(acc, m0 + wm * MTW * 16, ct0, g, w, y, ldy, quads);
        return;
    }
    __syncthreads();                                      // nobody reads X any more
    mx_tile_store_wide<T, Y, MTW, NTW, SPLIT>(reinterpret_cast<char *>(xs) + wave * (16 * (NTW * 16 * (int)sizeof(Y) + 16)), acc, m0 + wm * MTW * 16, ct0, g, w, y, ldy);
}

// ------------------------------------------------------------------------------------------ tens of rows
// Up to some hundred rows: what bounds a product is how fast a CU draws weights and X through its L1 together (some 45 GB/s measured, whatever
// the shape of a load), and what comes between: a wave that waits for X cannot ask for weights.  So FW waves of a workgroup do nothing but
// fetch X into LDS, a group of four k-steps a stage, two stages; the others keep the codes of their own columns four k-steps
// ahead in registers, and multiply.  One barrier per stage, where reads pass into the next one, as in mx_tile_kernel.
// SILU: the columns alternate in groups of 16 gates and 16 ups (PackSrc::interleave16), and what is written is SiLU(gate) * up, [M][ldy].
template <typename T, typename Y, int TM, int TN, int WM, int WN, int FW, bool SPLIT, bool SILU = false>
__global__ __launch_bounds__((WM * WN + FW) * 64) void mx_fed_kernel(MxPacked w, MxRows x, MxGeom g, Y *__restrict__ y, int64_t ldy, bool quads, bool wide) {
    typedef __attribute__((address_space(3))) void *LdsPtr;
    typedef MxOp<T> Op;
    constexpr int WAVES = WM * WN, MTW = TM / (16 * WM), NTW = TN / (16 * WN), UNITS = TM, UPW = UNITS / FW;         // 1 KB units of a stage
    constexpr int SLOTS = 16 * MTW, AHEAD = 3;
    static_assert(UPW * FW == UNITS, "tile shape");
    __shared__ __attribute__((aligned(1024))) u32x4 xs[2 * UNITS * 64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    int tm, tn;
    mx_tile_of(g, blockIdx.x, 16, tm, tn);
    const int m0 = tm * TM;
    int g0, n;                                            // groups of four k-steps
    mx_split_of(g, g0, n);
    g0 >>= 2; n = (n + 3) >> 2;

    if (wave >= WAVES) {                                  // a wave that fetches
        const int fw = wave - WAVES, x_piece = (lane & 3) ^ ((lane >> 4) & 3);
        const unsigned lds0 = (unsigned)(uintptr_t)(LdsPtr)&xs[0];
        const T *src = static_cast<const T *>(x.x) + (int64_t)m0 * x.ldx + (int64_t)g0 * 4 * MX_KSTEP;
        auto issue = [&](int t) {                         // stage t
            const int k0 = (g0 + t) * 4 * MX_KSTEP;
            const bool whole = (g0 + t + 1) * 4 <= g.full;
#pragma unroll
            for (int j = 0; j < UPW; ++j) {
                const int u = fw + FW * j, m = min((u >> 4) * 16 + (lane >> 2), g.M - 1 - m0), k = (u & 15) * MX_BLOCK + x_piece * 8;
                const unsigned off = ((unsigned)m * (unsigned)x.ldx + (unsigned)k) * 2u, dst = lds0 + (unsigned)(((t & 1) * UNITS + u) * 1024);
                if (whole) lds_dma16_s(dst, src + (int64_t)t * 4 * MX_KSTEP, off);
                else {
                    const char *p = reinterpret_cast<const char *>(src + (int64_t)t * 4 * MX_KSTEP) + off;
                    lds_dma16(dst, k0 + k < x.K ? static_cast<const void *>(p) : static_cast<const void *>(&mx_zero_piece));
                }
            }
        };
        issue(0);
        for (int t = 0; t < n; ++t) {
            dma_wait<0>();
            __syncthreads();                              // stage t has landed; nobody reads stage t - 1 any more
            if (t + 1 < n) issue(t + 1);
        }
        if (TM >= 64 && !SILU && wide) __syncthreads();   // (the others write their results through LDS)
        return;
    }
    const int wm = wave % WM, wn = wave / WM, ct0 = tn * (TN / 16) + wn * NTW;
    const u32x4 *wp[NTW];
    const uint32_t *sp[NTW];
    int move[NTW];
#pragma unroll
    for (int nt = 0; nt < NTW; ++nt) {
        const int ct = min(ct0 + nt, w.tiles - 1);        // tiles beyond the matrix repeat the last one (never stored)
        wp[nt] = w.codes + (size_t)ct * w.ksteps * 64 + lane;
        sp[nt] = w.scales + (size_t)ct * w.kgroups * 64 + lane;
        move[nt] = Op::move(w.ref, ct * 16 + (lane & 15));
    }
    int wg = g0 % w.kgroups;                              // group of the weights (float32 X passes over them three times)
    f32x4 acc[MTW][NTW];
#pragma unroll
    for (int mt = 0; mt < MTW; ++mt)
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 c[4][NTW], xf[4], wf[2][NTW];
    unsigned sc[NTW], sn[NTW];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) c[s][nt] = wp[nt][(wg * 4 + s) * 64];
#pragma unroll
    for (int nt = 0; nt < NTW; ++nt) sc[nt] = sp[nt][wg * 64];
    // X: sixteen units per row tile, a block of columns each; slot q of a stage: k-step q / (4 MTW), substep q / MTW % 4, row tile q % MTW
    const int rd = (wm * MTW * 16 + (lane >> 4)) * 64 + (lane & 15) * 4, rs = (lane >> 2) & 3;
    auto x_at = [&](int q) { return rd + ((q % MTW) * 16 + q / (4 * MTW) * 4) * 64 + ((q / MTW & 3) ^ rs); };
    auto scale = [&](int s, unsigned four, int nt) {
        return s == 0 ? mx_scale<T, 0>(four, move[nt]) : s == 1 ? mx_scale<T, 1>(four, move[nt]) : s == 2 ? mx_scale<T, 2>(four, move[nt]) : mx_scale<T, 3>(four, move[nt]);
    };
    __syncthreads();
    int st = 0;
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) xf[q] = xs[x_at(q)];
#pragma unroll
    for (int nt = 0; nt < NTW; ++nt) wf[0][nt] = Op::weights(c[0][nt][0], scale(0, sc[nt], nt));
    auto group = [&](auto more_) {
        constexpr bool more = decltype(more_)::value;
        const u32x4 *cur = xs + st * UNITS * 64, *nxt = xs + (st ^ 1) * UNITS * 64;
        const int wn_ = wg + 1 == w.kgroups ? 0 : wg + 1;
        if constexpr (more)
#pragma unroll
            for (int nt = 0; nt < NTW; ++nt) sn[nt] = sp[nt][wn_ * 64];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int mt = 0; mt < MTW; ++mt) {
                    const int q = (s * 4 + i) * MTW + mt;
                    if (more && q == SLOTS - AHEAD) {
                        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                        __syncthreads();
                    }
                    xf[(q + AHEAD) & 3] = q + AHEAD >= SLOTS ? nxt[x_at(q + AHEAD - SLOTS)] : cur[x_at(q + AHEAD)];
#pragma unroll
                    for (int nt = mt; nt < NTW; nt += MTW) {
                        // the next substep's weights
                        if (i < 3) wf[(i + 1) & 1][nt] = Op::weights(c[s][nt][(i + 1) & 3], scale(s, sc[nt], nt));
                        else if (s < 3) wf[0][nt] = Op::weights(c[(s + 1) & 3][nt][0], scale(s + 1, sc[nt], nt));
                        else if constexpr (more) wf[0][nt] = Op::weights(c[0][nt][0], scale(0, sn[nt], nt));
                    }
#pragma unroll
                    for (int nt = 0; nt < NTW; ++nt) acc[mt][nt] = Op::mfma(wf[i & 1][nt], xf[q & 3], acc[mt][nt]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (i == 2)                                // all of these codes are converted: the next group's on their way
                    if constexpr (more)
#pragma unroll
                        for (int nt = 0; nt < NTW; ++nt) c[s][nt] = wp[nt][(wn_ * 4 + s) * 64];
            }
        }
        st ^= 1;
        wg = wn_;
        if constexpr (more)
#pragma unroll
            for (int nt = 0; nt < NTW; ++nt) sc[nt] = sn[nt];
    };
    for (int t = 0; t + 1 < n; ++t) group(Yes{});
    group(No{});
    if constexpr (SILU) {
        static_assert(NTW % 2 == 0, "a wave holds gates with their ups");
#pragma unroll
        for (int mt = 0; mt < MTW; ++mt) {
            const int m = m0 + (wm * MTW + mt) * 16 + (lane & 15);
            if (m >= g.M) continue;
#pragma unroll
            for (int nt = 0; nt < NTW; nt += 2) {
                const int f = (ct0 + nt) * 8 + (lane >> 4) * 4, n = min(ct0 + nt, w.tiles - 2) * 16 + (lane >> 4) * 4;
                if (f >= ldy) continue;                   // (a multiple of eight)
                const MxQuad<float> gate = mx_scaled<float>(acc[mt][nt], w.ref, n, Op::SHIFT), up = mx_scaled<float>(acc[mt][nt + 1], w.ref, n + 16, Op::SHIFT);
                *reinterpret_cast<MxQuad<T> *>(y + (int64_t)m * ldy + f) = mx_silu_quad<T>(gate, up);
            }
        }
    } else if (TM >= 64 && wide) {
        __syncthreads();                                  // nobody reads X any more
        mx_tile_store_wide<T, Y, MTW, NTW, SPLIT>(reinterpret_cast<char *>(xs) + wave * (16 * (NTW * 16 * (int)sizeof(Y) + 16)), acc, m0 + wm * MTW * 16, ct0, g, w, y, ldy);
    } else mx_tile_store<T, Y, MTW, NTW, SPLIT>(acc, m0 + wm * MTW * 16, ct0, g, w, y, ldy, quads);
}

__device__ __forceinline__ void lds_dma4_s(unsigned lds_base, const void *g, unsigned off) {     // 4 bytes a lane (device_utils.h has 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds_base), "v"(off), "s"(g) : "memory");
}

// ------------------------------------------------------------------------------------------ both operands in 4 bits, tens of rows
// mx_fed_kernel for microscaled X: a lane's block of 16 bytes is an operand as it is, so a stage is codes (a 1 KB unit per row tile and
// k-step: four lanes fetch a row's 64 bytes, block b of row r to position b ^ (r / 4 % 4)) and, for each row tile and group, the scales of
// a lane's four blocks in one word, which the fetching waves put together from the rows' bytes.  KG groups of four k-steps a stage.
// (Sixteen lanes fetching one block each of sixteen rows took four times as long to issue: 8192 x 28672 x 4096 843 us, now 558 with the
// results' way out.)
template <typename Y, int TM, int TN, int WM, int WN, int FW, int KG, bool SPLIT>
__global__ __launch_bounds__((WM * WN + FW) * 64) void mx_fed_both_kernel(MxPacked w, const u32x4 *__restrict__ x, const uint8_t *__restrict__ xs_, int blocks, MxGeom g, Y *__restrict__ y,
                                                                          int64_t ldy, bool quads, bool wide) {
    typedef __attribute__((address_space(3))) void *LdsPtr;
    constexpr int WAVES = WM * WN, MTW = TM / (16 * WM), NTW = TN / (16 * WN), RT = TM / 16, UNITS = RT * 4 * KG;
    constexpr int STAGE = UNITS * 64 + RT * KG * 16, SLOTS = 4 * KG * MTW, AHEAD = 3;      // (16 bytes each: codes, then scales)
    constexpr int UPW = (UNITS + FW - 1) / FW, SPW = (RT * KG + FW - 1) / FW;
    static_assert(SLOTS > AHEAD, "tile shape");
    __shared__ __attribute__((aligned(1024))) u32x4 xs[2 * STAGE];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    int tm, tn;
    mx_tile_of(g, blockIdx.x, 16, tm, tn);
    const int m0 = tm * TM;
    const int n_groups = w.kgroups, g0 = (int)((int64_t)blockIdx.y * n_groups / g.splits), n = (int)((int64_t)(blockIdx.y + 1) * n_groups / g.splits) - g0;
    const int stages = (n + KG - 1) / KG;

    if (wave >= WAVES) {
        const int fw = wave - WAVES;
        const unsigned lds0 = (unsigned)(uintptr_t)(LdsPtr)&xs[0];
        unsigned sc[SPW];
        auto issue = [&](int t) {
            const int b0 = (g0 + t * KG) * 16;            // first block of the stage
#pragma unroll
            for (int j = 0; j < UPW; ++j) {
                const int u = fw + FW * j;
                if (UPW * FW != UNITS && u >= UNITS) break;
                const int m = min(m0 + u / (4 * KG) * 16 + (lane >> 2), g.M - 1), b = b0 + u % (4 * KG) * 4 + ((lane & 3) ^ (lane >> 4));
                lds_dma16(lds0 + (unsigned)(((t & 1) * STAGE + u * 64) * 16), b < blocks ? x + ((int64_t)m * blocks + b) : &mx_zero_piece);
            }
#pragma unroll
            for (int j = 0; j < SPW; ++j) {
                const int u = fw + FW * j, m = min(m0 + u / KG * 16 + (lane & 15), g.M - 1), b = b0 + u % KG * 16 + (lane >> 4);
                sc[j] = 0;
                if (SPW * FW != RT * KG && u >= RT * KG) break;
#pragma unroll
                for (int s = 0; s < 4; ++s) sc[j] |= (unsigned)(b + s * 4 < blocks ? xs_[(int64_t)m * blocks + b + s * 4] : 127) << (8 * s);
            }
        };
        auto put = [&](int t) {
#pragma unroll
            for (int j = 0; j < SPW; ++j) {
                const int u = fw + FW * j;
                if (SPW * FW != RT * KG && u >= RT * KG) break;
                reinterpret_cast<unsigned *>(xs + (t & 1) * STAGE + UNITS * 64)[u * 64 + lane] = sc[j];
            }
        };
        issue(0);
        for (int t = 0; t < stages; ++t) {
            put(t);
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __syncthreads();
            if (t + 1 < stages) issue(t + 1);
        }
        if (TM >= 64 && wide) __syncthreads();            // (the others write their results through LDS)
        return;
    }
    const int wm = wave % WM, wn = wave / WM, ct0 = tn * (TN / 16) + wn * NTW;
    const u32x4 *wp[NTW];
    const uint32_t *sp[NTW];
#pragma unroll
    for (int nt = 0; nt < NTW; ++nt) {
        const int ct = min(ct0 + nt, w.tiles - 1);
        wp[nt] = w.codes + ((size_t)ct * w.ksteps + g0 * 4) * 64 + lane;
        sp[nt] = w.scales + ((size_t)ct * w.kgroups + g0) * 64 + lane;
    }
    f32x4 acc[MTW][NTW];
#pragma unroll
    for (int mt = 0; mt < MTW; ++mt)
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 c[4][NTW], xf[4];
    unsigned sc[NTW], sn[NTW], xsc[MTW];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) c[s][nt] = wp[nt][s * 64];
#pragma unroll
    for (int nt = 0; nt < NTW; ++nt) sn[nt] = *sp[nt];
    const int rd = wm * MTW * 4 * KG * 64 + (lane & 15) * 4 + ((lane >> 4) ^ ((lane >> 2) & 3));
    auto x_at = [&](int q) { return rd + ((q % MTW) * 4 * KG + q / MTW) * 64; };            // slot q of a stage: k-step q / MTW
    __syncthreads();
    int st = 0;                                           // stage buffer
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) xf[q] = xs[x_at(q)];
    auto group = [&](auto more_, auto gi_, bool next_stage) {
        constexpr bool more = decltype(more_)::value;
        constexpr int GI = decltype(gi_)::value;          // group within the stage (static)
        const u32x4 *cur = xs + st * STAGE, *nxt = xs + (st ^ 1) * STAGE;
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) { sc[nt] = sn[nt]; if constexpr (more) { sp[nt] += 64; sn[nt] = *sp[nt]; } }
#pragma unroll
        for (int mt = 0; mt < MTW; ++mt) xsc[mt] = reinterpret_cast<const unsigned *>(cur + UNITS * 64)[((wm * MTW + mt) * KG + GI) * 64 + lane];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int mt = 0; mt < MTW; ++mt) {
                const int q = (GI * 4 + s) * MTW + mt;
                if (q == SLOTS - AHEAD && next_stage) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    __syncthreads();
                }
                xf[(q + AHEAD) & 3] = q + AHEAD >= SLOTS ? nxt[x_at(q + AHEAD - SLOTS)] : cur[x_at(q + AHEAD)];
                const u32x4 &xv = xf[q & 3];
                const i32x8 b = {(int)xv.x, (int)xv.y, (int)xv.z, (int)xv.w, 0, 0, 0, 0};
#pragma unroll
                for (int nt = 0; nt < NTW; ++nt) {
                    const i32x8 a = {(int)c[s][nt].x, (int)c[s][nt].y, (int)c[s][nt].z, (int)c[s][nt].w, 0, 0, 0, 0};
                    if (s == 0) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[mt][nt], 4, 4, 0, (int)sc[nt], 0, (int)xsc[mt]);
                    else if (s == 1) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[mt][nt], 4, 4, 1, (int)sc[nt], 1, (int)xsc[mt]);
                    else if (s == 2) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[mt][nt], 4, 4, 2, (int)sc[nt], 2, (int)xsc[mt]);
                    else acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[mt][nt], 4, 4, 3, (int)sc[nt], 3, (int)xsc[mt]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (more)
#pragma unroll
                for (int nt = 0; nt < NTW; ++nt) c[s][nt] = wp[nt][(s + 4) * 64];
        }
#pragma unroll
        for (int nt = 0; nt < NTW; ++nt) wp[nt] += 256;
    };
    // whole stages but the last, then what is left of it
    for (int t = 0; t + 1 < stages; ++t) {
        group(Yes{}, Num<0>{}, true);
        if constexpr (KG == 2) group(Yes{}, Num<1>{}, true);
        st ^= 1;
    }
    if (KG == 1 || n % KG != 0) group(No{}, Num<0>{}, false);
    else {
        group(Yes{}, Num<0>{}, false);
        if constexpr (KG == 2) group(No{}, Num<1>{}, false);
    }
    if (TM >= 64 && wide) {
        __syncthreads();                                  // nobody reads X any more
        mx_tile_store_wide<bf16_t, Y, MTW, NTW, SPLIT>(reinterpret_cast<char *>(xs) + wave * (16 * (NTW * 16 * (int)sizeof(Y) + 16)), acc, m0 + wm * MTW * 16, ct0, g, w, y, ldy);
    } else mx_tile_store<bf16_t, Y, MTW, NTW, SPLIT>(acc, m0 + wm * MTW * 16, ct0, g, w, y, ldy, quads);
}

// ------------------------------------------------------------------------------------------ both operands in 4 bits, many rows
// X's scales as the packed weights have theirs: [row tile][group][lane], the four k-steps of a lane's block row in a word.
__global__ __launch_bounds__(256) void mx_scales_kernel(const uint8_t *__restrict__ xs, int M, int blocks, int groups, uint32_t *__restrict__ out) {
    const int i = blockIdx.x * 256 + threadIdx.x, grp = i >> 6, lane = i & 63;
    if (grp >= groups) return;
    for (int rt = blockIdx.y; rt * 16 < M; rt += gridDim.y) {
        const int m = min(rt * 16 + (lane & 15), M - 1);
        unsigned v = 0;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int b = grp * 16 + s * 4 + (lane >> 4);
            v |= (unsigned)(b < blocks ? xs[(int64_t)m * blocks + b] : 127) << (8 * s);
        }
        out[((size_t)rt * groups + grp) * 64 + lane] = v;
    }
}

// 256 x 256 tiles, eight waves of 128 x 64 with the 32 x 32 x 64 instruction (registers alone, random codes: 6.3 PFLOP/s where the
// 16 x 16 x 128 one gives 5.2).  Codes of both operands go into LDS by LDS-direct loads, a k-step of 128 a stage, four stages in a ring,
// one barrier per k-step; the scales of a group of four k-steps likewise, an eighth of them by each wave, half of that in each of the first two k-steps of the group before; two buffers.
// A workgroup per CU takes one tile after the other, and the loads run on into the next one: when a tile's sums are written, the next
// tile's first three stages and scales are there or on their way.  8192 x 28672 x 4096: 480 us, 4.0 PFLOP/s; the matrix pipes are busy half the
// cycles of a clock that their load has brought to 1.7 GHz (registers alone: all cycles at 1.5).
template <typename Y>
__global__ __launch_bounds__(512, 2) void mx_block_both_kernel(MxPacked w, const u32x4 *__restrict__ x, const uint32_t *__restrict__ xscales, int blocks, MxGeom g, Y *__restrict__ y,
                                                               int64_t ldy, bool quads, bool wide) {
    typedef __attribute__((address_space(3))) void *LdsPtr;
    constexpr int NST = 4, STAGE = 32 * 64;               // units 0..15: X's row tiles, 16..31: column tiles
    __shared__ __attribute__((aligned(1024))) u32x4 xs[NST * STAGE];
    __shared__ __attribute__((aligned(1024))) unsigned scs[2][32 * 64];
    __shared__ __attribute__((aligned(1024))) int refs[8 * 64];       // of each wave's 64 columns
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, wm = wave & 1, wn = wave >> 1;
    const unsigned lds0 = (unsigned)(uintptr_t)(LdsPtr)&xs[0], lds1 = (unsigned)(uintptr_t)(LdsPtr)&scs[0][0], lds2 = (unsigned)(uintptr_t)(LdsPtr)&refs[0];
    const int x_b = (lane & 3) ^ (lane >> 4);             // block b of row r of a unit of X lies at position b ^ (r / 4 % 4)
    const bool planes = g.splits > 1;                     // (Y is float then)
    const int tiles = g.tiles_m * g.tiles_n, items = tiles * g.splits, rts = (g.M + 15) / 16;
    // A tile (of a split) as the loads see it.  Scales of a group: unit wave + 8 j (j = 0, 1: row tiles; 2, 3: column tiles).
    struct Item { int m0, ct0, split, g0, n; };
    auto item_of = [&](int i) {
        Item t;
        int tm, tn;
        t.split = i / tiles;
        mx_tile_of(g, i - t.split * tiles, 8, tm, tn);
        t.m0 = tm * 256; t.ct0 = tn * 16;
        t.g0 = (int)((int64_t)t.split * w.kgroups / g.splits);
        t.n = ((int)((int64_t)(t.split + 1) * w.kgroups / g.splits) - t.g0) * 4;       // k-steps: whole groups
        return t;
    };
    const u32x4 *xp, *wp[2];
    const uint32_t *sp[4];
    unsigned xo[2];                                       // (256 rows of 2^16 blocks: 32 bits)
    int x_left;                                           // blocks of a row of X from the item's first on
    auto codes_at = [&](const Item &t) {
        xp = x + (int64_t)t.m0 * blocks + t.g0 * 16;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            xo[j] = (unsigned)(min((wave + 8 * j) * 16 + (lane >> 2), g.M - 1 - t.m0) * blocks + x_b) * 16u;
            wp[j] = w.codes + ((size_t)min(t.ct0 + wave + 8 * j, w.tiles - 1) * w.ksteps + t.g0 * 4) * 64;
        }
        x_left = blocks - t.g0 * 16;
    };
    auto scales_at = [&](const Item &t) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            sp[j] = xscales + ((size_t)min(t.m0 / 16 + wave + 8 * j, rts - 1) * w.kgroups + t.g0) * 64;
            sp[2 + j] = w.scales + ((size_t)min(t.ct0 + wave + 8 * j, w.tiles - 1) * w.kgroups + t.g0) * 64;
        }
    };
    auto issue = [&](int j, int s, int st) {              // load j (static, 0..3) of k-step s of the item, into stage st
        const unsigned base = lds0 + (unsigned)(st * STAGE * 16);
        if (j < 2) {
            const void *p = reinterpret_cast<const char *>(xp + s * 4) + xo[j];
            lds_dma16(base + (wave + 8 * j) * 1024, s * 4 + x_b < x_left ? p : &mx_zero_piece);
        } else lds_dma16_s(base + (16 + wave + 8 * (j - 2)) * 1024, wp[j - 2] + s * 64, lane * 16);
    };
    auto issue_scales = [&](int j, int grp, int buf) {    // unit j (static) of group grp of the item
        lds_dma4_s(lds1 + (unsigned)((buf * 32 + wave + 8 * j) * 256), sp[j] + grp * 64, lane * 4);
    };
    auto issue_refs = [&](const Item &t) { lds_dma4_s(lds2 + (unsigned)(wave * 256), w.ref, (unsigned)min((t.ct0 + wn * 4) * 16 + lane, w.tiles * 16 - 1) * 4u); };
    f32x16 acc[4][2];
    // an operand of 32 rows x 64 columns (half h of a k-step): lane -> row lane % 32 (of two units), block 2 h + lane / 32
    const int fr = ((lane >> 4) & 1) * 64 + (lane >> 5) * 16 + (lane & 15);
    const int xr = wm * 8 * 64 + fr, wr = (16 + wn * 4) * 64 + fr;                       // + 128 per 32 rows, + 32 for the second half
    int xc[2];                                            // X's codes
#pragma unroll
    for (int h = 0; h < 2; ++h) xc[h] = wm * 8 * 64 + ((lane >> 4) & 1) * 64 + (lane & 15) * 4 + ((h * 2 + (lane >> 5)) ^ ((lane >> 2) & 3));
    u32x4 xf[2][4], wf[2][2];
    unsigned xsc[2][4], wsc[2][2];
    auto read_scales = [&](int buf) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) wsc[h][nt] = scs[buf][wr + nt * 128 + h * 32];
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) xsc[h][mt] = scs[buf][xr + mt * 128 + h * 32];
        }
    };

    // Loads of a wave: four pieces a k-step, in the first two of a group two units each of the next group's scales, in the second the refs
    // too: they have landed with the pieces by the group's end.  Behind the stage that k-step s waits for: those of s - 1 and of s.
    // (Stores of the tile before are behind it too, or done: the wait is longer for them, never shorter.)
    Item cur = item_of(blockIdx.x);
    codes_at(cur);
    scales_at(cur);
#pragma unroll
    for (int j = 0; j < 4; ++j) issue_scales(j, 0, 0);
#pragma unroll
    for (int s = 0; s < NST - 1; ++s) {                   // (n is at least four)
#pragma unroll
        for (int j = 0; j < 4; ++j) issue(j, s, s);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NST - 2) * 4) : "memory");
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) wf[0][nt] = xs[wr + nt * 128];
#pragma unroll
    for (int mt = 0; mt < 4; ++mt) xf[0][mt] = xs[xc[0] + mt * 128];
    read_scales(0);
    int buf = 0;
    Item next;
    // a group of four k-steps, the item's last one or not: there the scales that follow are the next item's, from its second k-step on the codes
    auto group = [&](auto last_, int s4) {
        constexpr bool last = decltype(last_)::value;
        const int gi = last ? 0 : (s4 >> 2) + 1;
        if (last) scales_at(next);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (last && s == 1) codes_at(next);
            const int ai = (s + 3) & 3, si = last && s > 0 ? s - 1 : s4 + s + 3;      // (k-step s of a group lies in stage s)
            const u32x4 *st = xs + s * STAGE, *nxt = xs + ((s + 1) & 3) * STAGE;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h == 1) {                         // the next stage has landed; behind the barrier the last one's place is free
                    if (s == 0) asm volatile("s_waitcnt vmcnt(10) lgkmcnt(0)" ::: "memory");
                    else if (s == 1) asm volatile("s_waitcnt vmcnt(13) lgkmcnt(0)" ::: "memory");
                    else if (s == 2) asm volatile("s_waitcnt vmcnt(11) lgkmcnt(0)" ::: "memory");
                    else asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
                    __syncthreads();
                }
#pragma unroll
                for (int mt = 0; mt < 4; ++mt) {
                    if (h == 0) issue(mt, si, ai);
                    if (h == 0 && mt >= 2 && s < 2) issue_scales(2 * s + mt - 2, gi, buf ^ 1);
                    if (h == 0 && mt == 3 && s == 1) issue_refs(cur);
                    const u32x4 *from = h == 1 ? nxt : st;
                    if (mt == 0) {                        // the next half's operands in the first two of four turns: six matrix instructions to arrive in
                        wf[h ^ 1][0] = from[wr + (h ^ 1) * 32];
                        wf[h ^ 1][1] = from[wr + 128 + (h ^ 1) * 32];
                        xf[h ^ 1][0] = from[xc[h ^ 1]];
                    } else if (mt == 1) {
                        xf[h ^ 1][1] = from[xc[h ^ 1] + 128];
                        xf[h ^ 1][2] = from[xc[h ^ 1] + 256];
                        xf[h ^ 1][3] = from[xc[h ^ 1] + 384];
                    }
                    const i32x8 b = {(int)xf[h][mt].x, (int)xf[h][mt].y, (int)xf[h][mt].z, (int)xf[h][mt].w, 0, 0, 0, 0};
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) {
                        const i32x8 a = {(int)wf[h][nt].x, (int)wf[h][nt].y, (int)wf[h][nt].z, (int)wf[h][nt].w, 0, 0, 0, 0};
                        if (s == 0) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc[mt][nt], 4, 4, 0, (int)wsc[h][nt], 0, (int)xsc[h][mt]);
                        else if (s == 1) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc[mt][nt], 4, 4, 1, (int)wsc[h][nt], 1, (int)xsc[h][mt]);
                        else if (s == 2) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc[mt][nt], 4, 4, 2, (int)wsc[h][nt], 2, (int)xsc[h][mt]);
                        else acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc[mt][nt], 4, 4, 3, (int)wsc[h][nt], 3, (int)xsc[h][mt]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        buf ^= 1;
        read_scales(buf);
    };
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        next = item_of(item + (int)gridDim.x < items ? item + (int)gridDim.x : item);      // (none: this one's again, valid memory that is never used)
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[mt][nt][r] = 0.f;
        for (int s4 = 0; s4 + 4 < cur.n; s4 += 4) group(No{}, s4);
        group(Yes{}, cur.n - 4);
        // D tile: lane -> row lane % 32, register r -> column 8 (r / 4) + 4 (lane / 32) + r % 4.  Thirty-two rows of 128 bytes at a time
        // through the stage that nobody reads and nothing is on its way to: the four units of it that this wave itself fills
        // next (eight rows each; piece p of a row at p ^ (row % 8)).  So waves need not wait for each other here.
        auto quad = [&](int mt, int nt, int q) { return f32x4{acc[mt][nt][q * 4], acc[mt][nt][q * 4 + 1], acc[mt][nt][q * 4 + 2], acc[mt][nt][q * 4 + 3]}; };
        auto scaled = [&](int mt, int nt, int q) {
            const int4 e = *reinterpret_cast<const int4 *>(&refs[wave * 64 + nt * 32 + q * 8 + (lane >> 5) * 4]);
            return mx_scaled<Y>(quad(mt, nt, q), planes ? int4{0, 0, 0, 0} : e, 0);
        };
        const int row0 = cur.m0 + wm * 128, n0 = (cur.ct0 + wn * 4) * 16;
        if (wide) {
            constexpr int NTS = sizeof(Y) == 2 ? 2 : 1;   // 32-column tiles of a piece of 128 bytes
            const int64_t ldd = planes ? (int64_t)g.plane_ld : ldy;
            const int half = lane >> 5, r_out = lane >> 3, cols = (planes ? w.tiles * 16 : g.N) - n0 - (lane & 7) * (16 / (int)sizeof(Y));
            char *const lds = reinterpret_cast<char *>(xs);
            const int own = (NST - 1) * (STAGE * 16) + wave * 1024, get = own + r_out * 128 + (((lane & 7) ^ r_out) << 4);
            const int put = own + ((lane >> 3) & 3) * 8192 + (lane & 7) * 128 + (NTS == 2 ? ((lane & 7) << 4) + half * 8 : ((lane & 7) ^ half) << 4);
            Y *to = y + (planes ? (size_t)cur.split * g.M * g.plane_ld : 0) + (int64_t)(row0 + r_out) * ldd + n0 + (lane & 7) * (16 / (int)sizeof(Y));
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
                for (int nt0 = 0; nt0 < 2; nt0 += NTS) {
#pragma unroll
                    for (int nt = nt0; nt < nt0 + NTS; ++nt)
#pragma unroll
                        for (int q = 0; q < 4; ++q)       // (quad q: piece nt * 4 + q or, of four bytes a value, 2 q + half)
                            *reinterpret_cast<MxQuad<Y> *>(lds + (put ^ (NTS == 2 ? nt * 4 + q : 2 * q) << 4)) = scaled(mt, nt, q);
                    wave_lds_sync();
                    Y *p = to;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const u32x4 v = *reinterpret_cast<const u32x4 *>(lds + get + i * 8192);
                        if (row0 + mt * 32 + i * 8 + r_out < g.M && nt0 * 32 < cols) mx_store_piece(p + nt0 * 32, v, !planes);
                        p += 8 * ldd;
                    }
                    wave_lds_sync();
                    if (nt0 + NTS == 2) to = p;
                    asm volatile("" : "+v"(to));          // (one address at a time: registers)
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
                const int m = row0 + mt * 32 + (lane & 31);
                if (m >= g.M) continue;
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int col = n0 + nt * 32 + q * 8 + (lane >> 5) * 4;
                        if (col < g.N) mx_store_quad<Y>(y + (int64_t)m * ldy + col, quads, g.N - col, scaled(mt, nt, q));
                    }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (loads go to that stage again)
        cur = next;
    }
    dma_wait<0>();                                        // (what nobody reads: LDS is given back)
}

// The planes of a product, added in order.
template <typename Y>
__global__ __launch_bounds__(256) void mx_planes_kernel(const f32x4 *__restrict__ part, int splits, int M, int N, int quads_row, const int32_t *__restrict__ ref, int shift,
                                                        Y *__restrict__ y, int64_t ldy, bool quads) {
    const int q = blockIdx.x * 256 + threadIdx.x;          // four columns
    if (q * 4 >= N) return;
    const size_t plane = (size_t)M * quads_row;
    for (int m = blockIdx.y; m < M; m += gridDim.y) {
        const f32x4 *p = part + (size_t)m * quads_row + q;
        f32x4 a = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; s += 8) {              // eight planes on the way at a time
            f32x4 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p[min(s + j, splits - 1) * plane];
#pragma unroll
            for (int j = 0; j < 8; ++j) if (s + j < splits) a += v[j];
        }
        mx_store<Y>(y, ldy, quads, m, q * 4, N, a, ref, shift);
    }
}

// ------------------------------------------------------------------------------------------ launches
// Whether X can be read as it is: rows of whole 16-byte pieces.
static bool rows_ok(int x_dt, const void *x, int64_t ldx, int K) {
    return x_dt != DT_F32 && reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx % 8 == 0 && K % 8 == 0 && ldx < (1 << 22);   // (offsets within a tile's rows are 32 bits)
}
static bool quads_ok(const void *y, int64_t ldy, int N, int y_dt) {
    return N % 4 == 0 && ldy % 4 == 0 && reinterpret_cast<uintptr_t>(y) % (4 * dtype_size(y_dt)) == 0;
}

// Whether rows of Y can be written in pieces of 16 bytes.
template <typename Y> static bool wide_ok(const Y *y, int64_t ldy, int N) {
    return reinterpret_cast<uintptr_t>(y) % 16 == 0 && ldy * sizeof(Y) % 16 == 0 && N * sizeof(Y) % 16 == 0;
}

static MxRows stage(int x_dt, const void *x, int64_t ldx, int M, int K, int kp, void *scratch, hipStream_t st) {
    const dim3 grid((kp / 8 + 255) / 256, M < 65535 ? M : 65535);
    u32x4 *o = static_cast<u32x4 *>(scratch);
    const bool wide = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx * dtype_size(x_dt) % 16 == 0;
    if (x_dt == DT_F32) { mx_stage_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float *>(x), ldx, wide, M, K, kp, o); return MxRows{scratch, 3 * (int64_t)kp, kp, kp}; }
    mx_stage_kernel<uint16_t><<<grid, 256, 0, st>>>(static_cast<const uint16_t *>(x), ldx, wide, M, K, kp, o);
    return MxRows{scratch, kp, 0, kp};
}

// Scratch: what stands in X's place (a staged copy; X's scales in operand order), then the planes.  Its size is asked for by type and shape: the copy's
// room is there for 16-bit rows of any distance and address, also where rows can be read as they are.
static size_t stage_bytes(int x_dt, int M, int K, const MxPlan &p) {
    const size_t groups = mx_groups(K);
    if (x_dt == DT_MX) return MX_BOTH_TILES[p.shape].tm == 256 ? (size_t)((M + 15) / 16) * groups * 256 : 0;
    return ((size_t)M * groups * 4 * MX_KSTEP * 2 * (x_dt == DT_F32 ? 3 : 1) + 255) / 256 * 256;
}
static MxPlan plan_of(int x_dt, int M, int N, int K) { return mx_plan_of(x_dt == DT_MX, x_dt == DT_F32 ? 3 : 1, M, N, K); }
size_t mx_gemm_scratch_size(int x_dt, int M, int N, int K) {
    if (M == 0) return 256;
    const MxPlan p = plan_of(x_dt, M, N, K);
    return stage_bytes(x_dt, M, K, p) + (p.splits > 1 ? (size_t)p.splits * M * ((N + 15) / 16 * 16) * sizeof(float) : 0) + 256;
}

template <typename Y>
static void add_planes(const MxPacked &w, const float *part, int splits, int M, int N, int shift, Y *y, int64_t ldy, bool quads, hipStream_t st) {
    mx_planes_kernel<Y><<<dim3(((N + 3) / 4 + 255) / 256, M < 65535 ? M : 65535), 256, 0, st>>>(reinterpret_cast<const f32x4 *>(part), splits, M, N, w.tiles * 4, w.ref, shift, y, ldy, quads);
}

template <typename T, typename Y>
static void run_tiles(const MxPacked &w, const MxRows &x, MxGeom g, const MxPlan &p, Y *y, int64_t ldy, bool quads, float *part, hipStream_t st) {
    const MxTile t = MX_TILES[p.shape];
    g.splits = p.splits; g.tiles_m = (g.M + t.tm - 1) / t.tm; g.tiles_n = (g.N + t.tn - 1) / t.tn;
    const dim3 grid(g.tiles_m * g.tiles_n, g.splits);
    const bool wide = wide_ok(y, ldy, g.N);
#define POSS_MX_FED(TM, TN, WM, WN, FW)                                                                                                      \
    do {                                                                                                                                     \
        if (g.splits > 1) mx_fed_kernel<T, float, TM, TN, WM, WN, FW, true><<<grid, (WM * WN + FW) * 64, 0, st>>>(w, x, g, part, 0, true, true); \
        else mx_fed_kernel<T, Y, TM, TN, WM, WN, FW, false><<<grid, (WM * WN + FW) * 64, 0, st>>>(w, x, g, y, ldy, quads, wide);         \
    } while (0)
    switch (p.shape) {
        case 1: POSS_MX_FED(16, 64, 1, 4, 2); break;
        case 2: POSS_MX_FED(32, 128, 1, 8, 4); break;
        case 3: POSS_MX_FED(32, 256, 1, 8, 4); break;
        case 4: POSS_MX_FED(64, 128, 2, 4, 4); break;
        case 5: POSS_MX_FED(64, 256, 1, 8, 4); break;
        default:
            if (g.splits > 1) mx_tile_kernel<T, float, 256, 256, 2, 4, true><<<grid, 512, 0, st>>>(w, x, g, part, 0, true, true);
            else mx_tile_kernel<T, Y, 256, 256, 2, 4, false><<<grid, 512, 0, st>>>(w, x, g, y, ldy, quads, wide);
    }
#undef POSS_MX_FED
}
template <typename T, typename Y, int PARTS>
static void run_gemm(const MxPacked &w, const MxRows &x, MxGeom g, const MxPlan &p, Y *y, int64_t ldy, bool quads, float *part, hipStream_t st) {
    if (p.shape == MX_STREAM) {
        const int waves = stream_waves(w.tiles, w.kgroups);
        mx_stream_kernel<T, Y, PARTS><<<w.tiles, waves * 64, waves * 1024, st>>>(w, x, y, ldy, quads, g.M, g.N);
        return;
    }
    g.plane_ld = w.tiles * 16; g.plane_scaled = false;
    run_tiles<T, Y>(w, x, g, p, y, ldy, quads, part, st);
    if (p.splits > 1) add_planes<Y>(w, part, p.splits, g.M, g.N, MxOp<T>::SHIFT, y, ldy, quads, st);
}

// X microscaled.  xscales: scratch for its scales in operand order.
template <typename Y>
static void run_both(const MxPacked &w, const u32x4 *x, const uint8_t *xs, int blocks, MxGeom g, const MxPlan &p, Y *y, int64_t ldy, bool quads, uint32_t *xscales, float *part, hipStream_t st) {
    if (p.shape == MX_STREAM) {
        const int waves = stream_waves(w.tiles, w.kgroups);
        mx_stream_both_kernel<Y><<<w.tiles, waves * 64, waves * 1024, st>>>(w, x, xs, blocks, y, ldy, quads, g.M, g.N);
        return;
    }
    const MxTile t = MX_BOTH_TILES[p.shape];
    g.plane_ld = w.tiles * 16; g.plane_scaled = false;
    g.splits = p.splits; g.tiles_m = (g.M + t.tm - 1) / t.tm; g.tiles_n = (g.N + t.tn - 1) / t.tn;
    const dim3 grid(g.tiles_m * g.tiles_n, g.splits);
    const bool wide = wide_ok(y, ldy, g.N);
#define POSS_MX_FED(TM, TN, WM, WN, FW, KG)                                                                                                        \
    do {                                                                                                                                           \
        if (g.splits > 1) mx_fed_both_kernel<float, TM, TN, WM, WN, FW, KG, true><<<grid, (WM * WN + FW) * 64, 0, st>>>(w, x, xs, blocks, g, part, 0, true, true); \
        else mx_fed_both_kernel<Y, TM, TN, WM, WN, FW, KG, false><<<grid, (WM * WN + FW) * 64, 0, st>>>(w, x, xs, blocks, g, y, ldy, quads, wide); \
    } while (0)
    switch (p.shape) {
        case 1: POSS_MX_FED(16, 64, 1, 4, 2, 1); break;
        case 2: POSS_MX_FED(32, 128, 1, 8, 4, 1); break;
        case 3: POSS_MX_FED(64, 128, 1, 8, 4, 2); break;
        case 4: POSS_MX_FED(64, 256, 1, 8, 4, 2); break;
        default: {
            const int rts = (g.M + 15) / 16;
            mx_scales_kernel<<<dim3((w.kgroups * 64 + 255) / 256, rts < 65535 ? rts : 65535), 256, 0, st>>>(xs, g.M, blocks, w.kgroups, xscales);
            const int items = g.tiles_m * g.tiles_n * g.splits, wgs = items < CHIP_CUS ? items : CHIP_CUS;
            if (g.splits > 1) mx_block_both_kernel<float><<<wgs, 512, 0, st>>>(w, x, xscales, blocks, g, part, 0, true, true);
            else mx_block_both_kernel<Y><<<wgs, 512, 0, st>>>(w, x, xscales, blocks, g, y, ldy, quads, wide);
        }
    }
#undef POSS_MX_FED
    if (g.splits > 1) add_planes<Y>(w, part, g.splits, g.M, g.N, 0, y, ldy, quads, st);
}

template <typename T, int PARTS>
static void run_gemm_t(const MxPacked &w, const MxRows &x, const MxGeom &g, const MxPlan &p, int y_dt, void *y, int64_t ldy, float *part, hipStream_t st) {
    const bool quads = quads_ok(y, ldy, g.N, y_dt);
    if (y_dt == DT_F32) run_gemm<T, float, PARTS>(w, x, g, p, static_cast<float *>(y), ldy, quads, part, st);
    else if (y_dt == DT_BF16) run_gemm<T, bf16_t, PARTS>(w, x, g, p, static_cast<bf16_t *>(y), ldy, quads, part, st);
    else run_gemm<T, f16_t, PARTS>(w, x, g, p, static_cast<f16_t *>(y), ldy, quads, part, st);
}

// ------------------------------------------------------------------------------------------ a context's layers
bool launch_mx_planes(int dt, const void *packed, int N, int K, const void *X, int ldx, int M, float *part, int ld, int splits, hipStream_t st) {
    if (!packed || !X || !part || M < 1 || N < 4 || N % 4 || K < 8 || K % 8 || ld % 4 || ld < (N + 15) / 16 * 16 || splits < 1 || splits > 16 || splits > mx_groups(K) ||
        !rows_ok(dt, X, ldx, K) || ldx < K) return false;
    const MxPacked w = mx_packed_at(packed, N, K);
    const MxPlan p = best_plan(MX_TILES, M, N, w.kgroups, splits);
    const MxGeom g{M, N, (K + MX_KSTEP - 1) / MX_KSTEP, K / MX_KSTEP, 0, 0, 1, ld, true};
    const MxRows x{X, ldx, 0, K};
    if (dt == DT_BF16) run_tiles<bf16_t, float>(w, x, g, p, part, ld, true, part, st);
    else run_tiles<f16_t, float>(w, x, g, p, part, ld, true, part, st);
    return true;
}
// A thread per four units; the planes come from the L2s for the most part.
template <typename T>
__global__ __launch_bounds__(256) void mx_silu_kernel(const float *__restrict__ part, int splits, int M, int ld, int F, T *__restrict__ act) {
    const int f = (blockIdx.x * 256 + threadIdx.x) * 4, m = blockIdx.y;
    if (f >= F) return;                                   // (F is a multiple of eight)
    const float *p = part + (size_t)m * ld + (f >> 4) * 32 + (f & 15);
    const size_t plane = (size_t)M * ld;
    f32x4 gate = *reinterpret_cast<const f32x4 *>(p), up = *reinterpret_cast<const f32x4 *>(p + 16);
    for (int s = 1; s < splits; ++s) {
        gate += *reinterpret_cast<const f32x4 *>(p + s * plane);
        up += *reinterpret_cast<const f32x4 *>(p + s * plane + 16);
    }
    *reinterpret_cast<MxQuad<T> *>(act + (size_t)m * F + f) = mx_silu_quad<T>(__builtin_bit_cast(MxQuad<float>, gate), __builtin_bit_cast(MxQuad<float>, up));
}
static void launch_mx_silu(int dt, const float *part, int splits, int M, int ld, int F, void *act, hipStream_t st) {
    const dim3 grid((F / 4 + 255) / 256, M);
    if (dt == DT_BF16) mx_silu_kernel<bf16_t><<<grid, 256, 0, st>>>(part, splits, M, ld, F, static_cast<bf16_t *>(act));
    else mx_silu_kernel<f16_t><<<grid, 256, 0, st>>>(part, splits, M, ld, F, static_cast<f16_t *>(act));
}

// act[M][F] = SiLU(gate) * up.  Unsplit (enough column tiles for the chip) the product does it itself: tiles whose waves hold a gate column with its up.
template <typename T>
static void run_silu(const MxPacked &w, const MxRows &x, MxGeom g, T *act, int F, hipStream_t st) {
#define POSS_MX_SILU(TM, TN, WM, WN, FW)                                                                                                     \
    do {                                                                                                                                     \
        g.tiles_m = (g.M + TM - 1) / TM; g.tiles_n = (g.N + TN - 1) / TN;                                                                    \
        mx_fed_kernel<T, T, TM, TN, WM, WN, FW, false, true><<<dim3(g.tiles_m * g.tiles_n), (WM * WN + FW) * 64, 0, st>>>(w, x, g, act, F, true, false); \
    } while (0)
    if (g.M <= 16) POSS_MX_SILU(16, 128, 1, 4, 2);
    else if (g.M <= 32) POSS_MX_SILU(32, 256, 1, 8, 4);
    else if (g.M <= 64) POSS_MX_SILU(64, 128, 2, 4, 4);
    else POSS_MX_SILU(64, 256, 1, 8, 4);
#undef POSS_MX_SILU
}
bool launch_mx_gate_up(int dt, const void *packed, int F, int K, const void *X, int ldx, int M, float *part, int ld, void *act, hipStream_t st) {
    const int N = gate_up_rows(F), splits = mx_plane_splits(N, K);
    if (!act || F % 8) return false;
    if (splits > 1) {
        if (!launch_mx_planes(dt, packed, N, K, X, ldx, M, part, ld, splits, st)) return false;
        launch_mx_silu(dt, part, splits, M, ld, F, act, st);
        return true;
    }
    if (!packed || !X || M < 1 || K < 8 || ldx < K || !rows_ok(dt, X, ldx, K)) return false;
    const MxPacked w = mx_packed_at(packed, N, K);
    const MxGeom g{M, N, (K + MX_KSTEP - 1) / MX_KSTEP, K / MX_KSTEP, 0, 0, 1, 0, false};
    if (dt == DT_BF16) run_silu<bf16_t>(w, MxRows{X, ldx, 0, K}, g, static_cast<bf16_t *>(act), F, st);
    else run_silu<f16_t>(w, MxRows{X, ldx, 0, K}, g, static_cast<f16_t *>(act), F, st);
    return true;
}

void launch_mx_gemm(int x_dt, const void *x, int64_t ldx, const void *packed, int y_dt, void *y, int64_t ldy, int M, int N, int K, void *scratch, hipStream_t st) {
    const MxPacked w = mx_packed_at(packed, N, K);
    const MxPlan p = plan_of(x_dt, M, N, K);
    const bool as_is = rows_ok(x_dt, x, ldx, K);
    const MxRows r = as_is ? MxRows{x, ldx, 0, K} : stage(x_dt, x, ldx, M, K, w.ksteps * MX_KSTEP, scratch, st);
    MxGeom g{M, N, x_dt == DT_F32 ? 3 * w.ksteps : (K + MX_KSTEP - 1) / MX_KSTEP, 0, 0, 0, 1, 0, false};
    g.full = as_is ? K / MX_KSTEP : x_dt == DT_F32 ? g.steps : w.ksteps;
    float *part = reinterpret_cast<float *>(static_cast<char *>(scratch) + stage_bytes(x_dt, M, K, p));
    if (x_dt == DT_F32) run_gemm_t<bf16_t, 3>(w, r, g, p, y_dt, y, ldy, part, st);
    else if (x_dt == DT_BF16) run_gemm_t<bf16_t, 1>(w, r, g, p, y_dt, y, ldy, part, st);
    else run_gemm_t<f16_t, 1>(w, r, g, p, y_dt, y, ldy, part, st);
}

void launch_mx_gemm_mx(const void *x_codes, const void *x_scales, const void *packed, int y_dt, void *y, int64_t ldy, int M, int N, int K, void *scratch, hipStream_t st) {
    const MxPacked w = mx_packed_at(packed, N, K);
    const MxPlan p = plan_of(DT_MX, M, N, K);
    const bool quads = quads_ok(y, ldy, N, y_dt);
    const MxGeom g{M, N, w.ksteps, 0, 0, 0, 1, 0, false};
    const u32x4 *c = static_cast<const u32x4 *>(x_codes);
    const uint8_t *s = static_cast<const uint8_t *>(x_scales);
    uint32_t *xs = static_cast<uint32_t *>(scratch);
    float *part = reinterpret_cast<float *>(static_cast<char *>(scratch) + stage_bytes(DT_MX, M, K, p));
    if (y_dt == DT_F32) run_both<float>(w, c, s, mx_blocks(K), g, p, static_cast<float *>(y), ldy, quads, xs, part, st);
    else if (y_dt == DT_BF16) run_both<bf16_t>(w, c, s, mx_blocks(K), g, p, static_cast<bf16_t *>(y), ldy, quads, xs, part, st);
    else run_both<f16_t>(w, c, s, mx_blocks(K), g, p, static_cast<f16_t *>(y), ldy, quads, xs, part, st);
}

}  // namespace poss
