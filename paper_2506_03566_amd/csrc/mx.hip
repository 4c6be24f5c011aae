// Products with microscaled 4-bit weights, and the quantisation to that form.
//
// The format: 32 values of a row share a power of two (e8m0: a byte b stands for 2^(b - 127), 255 for NaN); a value is a sign, two
// bits of exponent and one of mantissa (e2m1, magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6).  In memory a row is ceil(cols / 32) blocks of
// 16 bytes, the even column in the low half of a byte, and as many scale bytes; columns beyond the row's end are codes of zero.
//
// Packed weights (what the products read) are those blocks in operand order of the 16 x 16 x 128 matrix instruction:
//   codes  [column tile][k-step][lane]  16 bytes: the block of weight row tile * 16 + lane % 16, columns k-step * 128 + lane / 16 * 32 ...
//          (k-steps of 128, in whole groups of four; zeros beyond the matrix)
//   scales [column tile][k-step / 4][lane]  4 bytes: the scales of that lane's blocks of four k-steps, moved with the row's largest to where mx_held has it
//   ref    [row]  the largest scale byte of the row's blocks that are not all zero, and what the row's sums are multiplied by (mx_row_ref)
// A wave reads 1 KB of codes per k-step, contiguous along k.  bf16 and scaled operands are those numbers, mostly the weights themselves; an fp16
// number reaches from 2^-24 to 2^16 only: there operands are c * 2^(s - ref), times a constant.  The float32 sums are multiplied by what is left
// of 2^ref, exactly.
#include "../../include/poss.h"
#include "mx.h"

namespace poss {

// ------------------------------------------------------------------------------------------ quantisation
// Bound by memory.  Four lanes per block, a piece of eight values each: 16 or 32 bytes read, a word of codes written.  Scale byte = exponent field of
// the block's largest magnitude - 2, at least 0: that magnitude lies in [4, 8) then, and 6 to 8 saturates.  Magnitudes compare as integers,
// NaN above infinity above the rest.  The conversion instruction divides by the power of two and rounds to nearest, ties to even.
// A matrix without gaps whose rows are whole blocks is one long row (`flat`: no division per piece).
template <typename T> struct MxIn;
template <> struct MxIn<float> {
    union { u32x4 u[2]; float e[8]; unsigned w[8]; } v;
    __device__ __forceinline__ void load(const float *p) { v.u[0] = reinterpret_cast<const u32x4 *>(p)[0]; v.u[1] = reinterpret_cast<const u32x4 *>(p)[1]; }

    __device__ __forceinline__ void set(int j, float x) { v.e[j] = x; }
    __device__ __forceinline__ unsigned top() const {
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, v.w[j] & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ unsigned codes(float s) const {
        unsigned q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v.e[0], v.e[1], s, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v.e[2], v.e[3], s, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v.e[4], v.e[5], s, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v.e[6], v.e[7], s, 3);
    }
};
template <typename T> struct MxIn16 {
    union { u32x4 u; T e[8]; } v;
    __device__ __forceinline__ void load(const T *p) { v.u = *reinterpret_cast<const u32x4 *>(p); }

    __device__ __forceinline__ void set(int j, T x) { v.e[j] = x; }
    __device__ __forceinline__ unsigned top() const {      // the largest magnitude's 16 bits
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = max(m, max(v.u[j] & 0x7fffu, v.u[j] >> 16 & 0x7fffu));
        return m;
    }
};
template <> struct MxIn<bf16_t> : MxIn16<bf16_t> {
    __device__ __forceinline__ unsigned top() const { return MxIn16<bf16_t>::top() << 16; }
    __device__ __forceinline__ unsigned codes(float s) const {
        const bf16x2 *p = reinterpret_cast<const bf16x2 *>(&v);
        unsigned q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, p[0], s, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, p[1], s, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, p[2], s, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, p[3], s, 3);
    }
};
template <> struct MxIn<f16_t> : MxIn16<f16_t> {
    __device__ __forceinline__ unsigned top() const {
        const uint16_t b = (uint16_t)MxIn16<f16_t>::top();
        return __builtin_bit_cast(unsigned, (float)__builtin_bit_cast(f16_t, b));      // (infinity and NaN stay above the rest)
    }
    __device__ __forceinline__ unsigned codes(float s) const {
        const f16x2 *p = reinterpret_cast<const f16x2 *>(&v);
        unsigned q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(0u, p[0], s, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, p[1], s, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, p[2], s, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, p[3], s, 3);
    }
};
__device__ __forceinline__ unsigned quad_max(unsigned v) {
    v = max(v, __builtin_bit_cast(unsigned, xor1(__builtin_bit_cast(float, v))));
    return max(v, __builtin_bit_cast(unsigned, xor2(__builtin_bit_cast(float, v))));
}

// Piece i of a matrix of `pieces` pieces a row (a multiple of four): its row and place.  Index: 32 bits wherever they hold all pieces.
template <typename I> __device__ __forceinline__ void piece_at(I i, int pieces, bool flat, int64_t &row, int64_t &piece) {
    if (flat) { row = 0; piece = (int64_t)i; }
    else { const I r = i / (I)pieces; row = (int64_t)r; piece = (int64_t)(i - r * (I)pieces); }
}

// wide: rows of x can be read in pieces of 16 bytes.
template <typename T, typename I> __global__ __launch_bounds__(256) void mx_quantize_kernel(const T *__restrict__ x, int64_t ldx, int64_t total, int64_t cols, int pieces, bool flat,
                                                                                            bool wide, uint32_t *__restrict__ codes, uint8_t *__restrict__ scales) {
    for (I i = (I)blockIdx.x * 256 + threadIdx.x; i < (I)total; i += (I)gridDim.x * 256) {       // (total is a multiple of four: the lanes of a block go together)
        int64_t row, piece;
        piece_at<I>(i, pieces, flat, row, piece);
        const T *p = x + row * ldx + piece * 8;
        MxIn<T> in;
        if (wide && piece * 8 + 8 <= cols) in.load(p);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) in.set(j, piece * 8 + j < cols ? p[j] : from_f<T>(0.f));
        const unsigned field = quad_max(in.top()) >> 23, s = field == 255 ? 255u : field < 2 ? 0u : field - 2;
        codes[i] = field == 255 ? 0u : in.codes(mx_power(s));
        if ((i & 3) == 0) scales[i >> 2] = (uint8_t)s;
    }
}

// A piece: 16 bytes of y, so that a wave's stores are a kilobyte without gaps, past the caches: 28672 x 4096 to bf16 80 -> 42 us (with a pass
// over y behind it 159 -> 136), to float32 152 -> 73; float32 in pieces of 32 bytes 190.
template <typename T, typename I> __global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t total,
                                                                                              int64_t cols, int pieces, bool flat, bool wide, T *__restrict__ y, int64_t ldy) {
    constexpr int V = 16 / (int)sizeof(T), PER = 32 / V;  // values of a piece, pieces of a block
    for (I i = (I)blockIdx.x * 256 + threadIdx.x; i < (I)total; i += (I)gridDim.x * 256) {
        int64_t row, piece;
        piece_at<I>(i, pieces, flat, row, piece);
        const unsigned q = V == 8 ? codes[i] : reinterpret_cast<const uint16_t *>(codes)[i];
        const float s = mx_power(scales[i / PER]);
        union { T v[V]; u32x4 u; } o;
        // (values times the power of two in float32, exactly; then rounded to T once)
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1);
        o.v[0] = from_f<T>(a.x * s); o.v[1] = from_f<T>(a.y * s); o.v[2] = from_f<T>(b.x * s); o.v[3] = from_f<T>(b.y * s);
        if constexpr (V == 8) {
            const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3);
            o.v[4] = from_f<T>(c.x * s); o.v[5] = from_f<T>(c.y * s); o.v[6] = from_f<T>(d.x * s); o.v[7] = from_f<T>(d.y * s);
        }
        T *p = y + row * ldy + piece * V;
        if (wide && piece * V + V <= cols) __builtin_nontemporal_store(o.u, reinterpret_cast<u32x4 *>(p));
        else
#pragma unroll
            for (int j = 0; j < V; ++j) if (piece * V + j < cols) p[j] = o.v[j];
    }
}

// ------------------------------------------------------------------------------------------ packing
static inline int mx_ksteps(int K) { return mx_groups(K) * 4; }
static inline int mx_tiles(int N) { return (N + 15) / 16; }

MxPacked mx_packed_at(const void *packed, int N, int K) {
    const size_t tiles = mx_tiles(N), ks = mx_ksteps(K);
    const char *p = static_cast<const char *>(packed);
    MxPacked w;
    w.codes = reinterpret_cast<const u32x4 *>(p);
    p += tiles * ks * 1024;
    w.scales = reinterpret_cast<const uint32_t *>(p);
    p += tiles * (ks / 4) * 256;
    w.ref = reinterpret_cast<const int32_t *>(p);
    w.ksteps = (int)ks; w.kgroups = (int)(ks / 4); w.tiles = (int)tiles;
    return w;
}

size_t mx_packed_size(int N, int K) {
    const size_t tiles = mx_tiles(N), ks = mx_ksteps(K);
    return (tiles * ks * 1024 + tiles * (ks / 4) * 256 + tiles * 64 + 255) / 256 * 256;
}

__device__ __forceinline__ bool mx_all_zero(u32x4 c) { return ((c.x | c.y | c.z | c.w) & 0x77777777u) == 0; }

// The byte of a block's scale s in the packed form (blocks of zeros may lie above their row's largest).  Negative where the block lies further below the
// largest of a row above 2^0 than a byte reaches: it is taken for zero then.
__device__ __forceinline__ int mx_packed_scale(int s, int top) { return min(top, s) - top + mx_held(top); }

// A workgroup per column tile: first the rows' largest scales, then the blocks in their order.
__global__ __launch_bounds__(256) void mx_pack_kernel(const u32x4 *__restrict__ codes, const uint8_t *__restrict__ scales, int N, int blocks, int ksteps,
                                                      u32x4 *__restrict__ out, uint32_t *__restrict__ out_scales, int32_t *__restrict__ ref) {
    __shared__ int top[16];
    const int tile = blockIdx.x, tid = threadIdx.x;
    if (tid < 16) top[tid] = 0;
    __syncthreads();
    {
        const int r = tid >> 4, n = tile * 16 + r;
        int t = 0;
        if (n < N)
            for (int b = tid & 15; b < blocks; b += 16) {
                const int s = scales[(size_t)n * blocks + b];
                if (s == 255 || !mx_all_zero(codes[(size_t)n * blocks + b])) t = max(t, s);
            }
        atomicMax(&top[r], t);                            // (the largest: the same in any order)
    }
    __syncthreads();
    if (tid < 16) ref[tile * 16 + tid] = mx_row_ref(top[tid]);
    const int lane = tid & 63, r = lane & 15, n = tile * 16 + r, groups = ksteps / 4;
    for (int g = tid >> 6; g < groups; g += 4) {
        uint32_t packed = 0;
        for (int i = 0; i < 4; ++i) {
            const int ks = g * 4 + i, b = ks * 4 + (lane >> 4);
            u32x4 c = {0u, 0u, 0u, 0u};
            int s = 127;
            if (n < N && b < blocks) {
                s = mx_packed_scale(scales[(size_t)n * blocks + b], top[r]);
                if (s >= 0) c = codes[(size_t)n * blocks + b];
                else s = 0;
            }
            out[((size_t)tile * ksteps + ks) * 64 + lane] = c;
            packed |= (uint32_t)s << (8 * i);
        }
        out_scales[((size_t)tile * groups + g) * 64 + lane] = packed;
    }
}

// Quantisation and packing of a context's matrices in one kernel, when it is loaded: a workgroup per column tile reads its rows (the packed order's:
// gate and up alternate, heads have their rotary pairs side by side) once for the rows' largest scales and once for the codes.  What poss_mx_quantize and
// poss_mx_pack give for the same rows.
template <typename T> __global__ __launch_bounds__(256) void mx_pack_rows_kernel(PackSrc src, int K, int ksteps, u32x4 *__restrict__ out, uint32_t *__restrict__ out_scales,
                                                                                 int32_t *__restrict__ ref) {
    __shared__ int top[16];
    const int tile = blockIdx.x, tid = threadIdx.x, blocks = (K + MX_BLOCK - 1) / MX_BLOCK, groups = ksteps / 4;
    if (tid < 16) top[tid] = 0;
    __syncthreads();
    auto row_of = [&](int r) {
        int which, row;
        return pack_source_row(src, tile * 16 + r, which, row) ? static_cast<const T *>(src.ptr[which]) + (size_t)row * K : nullptr;
    };
    auto load = [&](const T *row, int b, MxIn<T> (&in)[4]) {      // (K is a multiple of eight)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (row && b * MX_BLOCK + i * 8 < K) in[i].load(row + b * MX_BLOCK + i * 8);
            else in[i].v.u = u32x4{0u, 0u, 0u, 0u};
        }
    };
    auto scale_of = [&](const MxIn<T> (&in)[4]) {
        const unsigned field = max(max(in[0].top(), in[1].top()), max(in[2].top(), in[3].top())) >> 23;
        return field == 255 ? 255 : field < 2 ? 0 : (int)field - 2;
    };
    {
        const T *row = row_of(tid >> 4);
        int t = 0;
        for (int b = tid & 15; b < blocks; b += 16) {
            MxIn<T> in[4];
            load(row, b, in);
            t = max(t, scale_of(in));
        }
        atomicMax(&top[tid >> 4], t);                     // (the largest: the same in any order)
    }
    __syncthreads();
    if (tid < 16) ref[tile * 16 + tid] = mx_row_ref(top[tid]);
    const int lane = tid & 63, r = lane & 15;
    const T *row = row_of(r);
    for (int g = tid >> 6; g < groups; g += 4) {
        uint32_t packed = 0;
        for (int i = 0; i < 4; ++i) {
            const int ks = g * 4 + i, b = ks * 4 + (lane >> 4);
            u32x4 c = {0u, 0u, 0u, 0u};
            int s = 127;
            if (row && b < blocks) {
                MxIn<T> in[4];
                load(row, b, in);
                const int sb = scale_of(in);
                s = mx_packed_scale(sb, top[r]);
                if (s < 0) s = 0;
                else if (sb != 255) c = u32x4{in[0].codes(mx_power(sb)), in[1].codes(mx_power(sb)), in[2].codes(mx_power(sb)), in[3].codes(mx_power(sb))};
            }
            out[((size_t)tile * ksteps + ks) * 64 + lane] = c;
            packed |= (uint32_t)s << (8 * i);
        }
        out_scales[((size_t)tile * groups + g) * 64 + lane] = packed;
    }
}

// ------------------------------------------------------------------------------------------ launches
// A matrix as the kernels walk it.
struct MxWalk { int64_t total, cols; int pieces; bool flat, wide, small; unsigned grid; };
static MxWalk walk_of(int dt, const void *rows_at, int64_t ld, int rows, int cols, int per_block) {
    MxWalk k;
    k.pieces = mx_blocks(cols) * per_block;
    k.total = (int64_t)rows * k.pieces;
    k.flat = cols % MX_BLOCK == 0 && (ld == cols || rows == 1);
    k.cols = k.flat ? (int64_t)rows * cols : cols;
    k.wide = reinterpret_cast<uintptr_t>(rows_at) % 16 == 0 && (rows == 1 || ld * dtype_size(dt) % 16 == 0);
    k.small = k.total < (1ll << 31);
    const int64_t g = (k.total + 255) / 256;
    k.grid = (unsigned)(g < (1 << 20) ? g : 1 << 20);
    return k;
}

#define POSS_MX_TYPES(KERNEL, ...)                                                                                   \
    do {                                                                                                             \
        if (dt == DT_F32) { typedef float T; if (k.small) KERNEL<T, uint32_t> __VA_ARGS__; else KERNEL<T, uint64_t> __VA_ARGS__; }          \
        else if (dt == DT_BF16) { typedef bf16_t T; if (k.small) KERNEL<T, uint32_t> __VA_ARGS__; else KERNEL<T, uint64_t> __VA_ARGS__; }   \
        else { typedef f16_t T; if (k.small) KERNEL<T, uint32_t> __VA_ARGS__; else KERNEL<T, uint64_t> __VA_ARGS__; }                       \
    } while (0)

void launch_mx_quantize(int dt, const void *x, int64_t ldx, int rows, int cols, void *codes, void *scales, hipStream_t st) {
    const MxWalk k = walk_of(dt, x, ldx, rows, cols, 4);
    POSS_MX_TYPES(mx_quantize_kernel, <<<k.grid, 256, 0, st>>>(static_cast<const T *>(x), ldx, k.total, k.cols, k.pieces, k.flat, k.wide, static_cast<uint32_t *>(codes),
                                                               static_cast<uint8_t *>(scales)));
}

void launch_mx_dequantize(int dt, const void *codes, const void *scales, int rows, int cols, void *y, int64_t ldy, hipStream_t st) {
    const MxWalk k = walk_of(dt, y, ldy, rows, cols, dt == DT_F32 ? 8 : 4);
    POSS_MX_TYPES(mx_dequantize_kernel, <<<k.grid, 256, 0, st>>>(static_cast<const uint32_t *>(codes), static_cast<const uint8_t *>(scales), k.total, k.cols, k.pieces, k.flat,
                                                                 k.wide, static_cast<T *>(y), ldy));
}
#undef POSS_MX_TYPES

void launch_mx_pack(const void *codes, const void *scales, int N, int K, void *packed, hipStream_t st) {
    const MxPacked w = mx_packed_at(packed, N, K);
    mx_pack_kernel<<<w.tiles, 256, 0, st>>>(static_cast<const u32x4 *>(codes), static_cast<const uint8_t *>(scales), N, mx_blocks(K), w.ksteps,
                                            const_cast<u32x4 *>(w.codes), const_cast<uint32_t *>(w.scales), const_cast<int32_t *>(w.ref));
}

void launch_mx_pack_rows(int dt, const PackSrc &src, int N, int K, void *packed, hipStream_t st) {
    const MxPacked w = mx_packed_at(packed, N, K);
    u32x4 *c = const_cast<u32x4 *>(w.codes); uint32_t *s = const_cast<uint32_t *>(w.scales); int32_t *r = const_cast<int32_t *>(w.ref);
    if (dt == DT_BF16) mx_pack_rows_kernel<bf16_t><<<w.tiles, 256, 0, st>>>(src, K, w.ksteps, c, s, r);
    else mx_pack_rows_kernel<f16_t><<<w.tiles, 256, 0, st>>>(src, K, w.ksteps, c, s, r);
}

}  // namespace poss

// ------------------------------------------------------------------------------------------ C entry points (include/poss.h)
using namespace poss;

namespace {
bool bad_dtype(int32_t t) { return t < 0 || t > 2; }
int launched(const char *who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? POSS_OK : set_error(POSS_E_HIP, "%s: %s", who, hipGetErrorString(e));
}
bool weight_ok(int32_t N, int32_t K) { return N > 0 && N <= MX_MOST_N && K > 0 && K <= MX_MOST_K; }
bool product_ok(int32_t M, int32_t N, int32_t K) { return weight_ok(N, K) && M >= 0 && M <= MX_MOST_M && (int64_t)M * N <= MX_MOST_MN; }
bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
// what both products check
int check_product(const char *who, const void *packed, const void *y, int32_t y_dtype, int64_t ldy, int32_t M, int32_t N, int32_t K, const void *scratch, size_t scratch_bytes, size_t need) {
    if (!product_ok(M, N, K) || ldy < N || bad_dtype(y_dtype)) return set_error(POSS_E_INVALID_ARG, "%s: bad shape or type", who);
    if (M == 0) return POSS_OK;
    if (!packed || !y || !scratch) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    if (reinterpret_cast<uintptr_t>(packed) % 256 || reinterpret_cast<uintptr_t>(scratch) % 256)
        return set_error(POSS_E_INVALID_ARG, "%s: packed weights and scratch must be aligned to 256 bytes", who);
    if (reinterpret_cast<uintptr_t>(y) % dtype_size(y_dtype)) return set_error(POSS_E_INVALID_ARG, "%s: y is not aligned to its type", who);
    if (scratch_bytes < need) return set_error(POSS_E_CAPACITY, "%s: M=%d N=%d K=%d needs %zu bytes of scratch, got %zu", who, M, N, K, need, scratch_bytes);
    return POSS_OK;
}
}  // namespace

extern "C" {

int poss_mx_quantize(int32_t dtype, const void *x, int64_t ldx, int32_t rows, int32_t cols, void *codes, void *scales, void *hip_stream) {
    if (bad_dtype(dtype) || rows < 0 || cols < 1 || ldx < cols) return set_error(POSS_E_INVALID_ARG, "poss_mx_quantize: bad shape or type");
    if (rows == 0) return POSS_OK;
    if (!x || !codes || !scales) return set_error(POSS_E_INVALID_ARG, "poss_mx_quantize: null argument");
    if (!aligned16(codes) || reinterpret_cast<uintptr_t>(x) % dtype_size(dtype)) return set_error(POSS_E_INVALID_ARG, "poss_mx_quantize: codes must be aligned to 16 bytes, x to its type");
    launch_mx_quantize(dtype, x, ldx, rows, cols, codes, scales, static_cast<hipStream_t>(hip_stream));
    return launched("poss_mx_quantize");
}

int poss_mx_dequantize(int32_t dtype, const void *codes, const void *scales, int32_t rows, int32_t cols, void *y, int64_t ldy, void *hip_stream) {
    if (bad_dtype(dtype) || rows < 0 || cols < 1 || ldy < cols) return set_error(POSS_E_INVALID_ARG, "poss_mx_dequantize: bad shape or type");
    if (rows == 0) return POSS_OK;
    if (!y || !codes || !scales) return set_error(POSS_E_INVALID_ARG, "poss_mx_dequantize: null argument");
    if (!aligned16(codes) || reinterpret_cast<uintptr_t>(y) % dtype_size(dtype)) return set_error(POSS_E_INVALID_ARG, "poss_mx_dequantize: codes must be aligned to 16 bytes, y to its type");
    launch_mx_dequantize(dtype, codes, scales, rows, cols, y, ldy, static_cast<hipStream_t>(hip_stream));
    return launched("poss_mx_dequantize");
}

size_t poss_mx_packed_bytes(int32_t N, int32_t K) { return weight_ok(N, K) ? mx_packed_size(N, K) : 0; }

int poss_mx_pack(const void *codes, const void *scales, int32_t N, int32_t K, void *packed, void *hip_stream) {
    if (!weight_ok(N, K)) return set_error(POSS_E_INVALID_ARG, "poss_mx_pack: bad shape");
    if (!codes || !scales || !packed) return set_error(POSS_E_INVALID_ARG, "poss_mx_pack: null argument");
    if (!aligned16(codes) || reinterpret_cast<uintptr_t>(packed) % 256) return set_error(POSS_E_INVALID_ARG, "poss_mx_pack: codes must be aligned to 16 bytes, packed to 256");
    launch_mx_pack(codes, scales, N, K, packed, static_cast<hipStream_t>(hip_stream));
    return launched("poss_mx_pack");
}

size_t poss_mx_gemm_scratch_bytes(int32_t x_dtype, int32_t M, int32_t N, int32_t K) {
    if ((bad_dtype(x_dtype) && x_dtype != POSS_MX) || !product_ok(M, N, K)) return 0;
    return mx_gemm_scratch_size(x_dtype, M, N, K);
}

int poss_mx_gemm(int32_t x_dtype, const void *x, int64_t ldx, const void *packed, int32_t y_dtype, void *y, int64_t ldy, int32_t M, int32_t N, int32_t K,
                 void *scratch, size_t scratch_bytes, void *hip_stream) {
    if (bad_dtype(x_dtype) || ldx < K) return set_error(POSS_E_INVALID_ARG, "poss_mx_gemm: bad shape or type");
    const int rc = check_product("poss_mx_gemm", packed, y, y_dtype, ldy, M, N, K, scratch, scratch_bytes, poss_mx_gemm_scratch_bytes(x_dtype, M, N, K));
    if (rc != POSS_OK || M == 0) return rc;
    if (!x) return set_error(POSS_E_INVALID_ARG, "poss_mx_gemm: null argument");
    if (reinterpret_cast<uintptr_t>(x) % dtype_size(x_dtype)) return set_error(POSS_E_INVALID_ARG, "poss_mx_gemm: x is not aligned to its type");
    launch_mx_gemm(x_dtype, x, ldx, packed, y_dtype, y, ldy, M, N, K, scratch, static_cast<hipStream_t>(hip_stream));
    return launched("poss_mx_gemm");
}

int poss_mx_gemm_mx(const void *x_codes, const void *x_scales, const void *packed, int32_t y_dtype, void *y, int64_t ldy, int32_t M, int32_t N, int32_t K,
                    void *scratch, size_t scratch_bytes, void *hip_stream) {
    const int rc = check_product("poss_mx_gemm_mx", packed, y, y_dtype, ldy, M, N, K, scratch, scratch_bytes, poss_mx_gemm_scratch_bytes(POSS_MX, M, N, K));
    if (rc != POSS_OK || M == 0) return rc;
    if (!x_codes || !x_scales) return set_error(POSS_E_INVALID_ARG, "poss_mx_gemm_mx: null argument");
    if (!aligned16(x_codes)) return set_error(POSS_E_INVALID_ARG, "poss_mx_gemm_mx: x_codes must be aligned to 16 bytes");
    launch_mx_gemm_mx(x_codes, x_scales, packed, y_dtype, y, ldy, M, N, K, scratch, static_cast<hipStream_t>(hip_stream));
    return launched("poss_mx_gemm_mx");
}

}  // extern "C"
