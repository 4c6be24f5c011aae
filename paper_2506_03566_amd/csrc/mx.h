// Microscaled 4-bit weights: the packed form, its device pieces and its launches (mx.hip, mx_gemm.hip).
#pragma once
#include "device_utils.h"
#include "mx_plan.h"

namespace poss {

typedef float  f32x2 __attribute__((ext_vector_type(2)));
typedef float  f32x4 __attribute__((ext_vector_type(4)));
typedef float  f32x16 __attribute__((ext_vector_type(16)));
typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t  f16x2 __attribute__((ext_vector_type(2)));
typedef f16_t  f16x8 __attribute__((ext_vector_type(8)));
typedef int    i32x8 __attribute__((ext_vector_type(8)));

constexpr int MX_BLOCK = 32;      // values that share a scale
constexpr int MX_KSTEP = 128;     // columns of a k-step: a block for each sixteen lanes
static_assert(MX_GROUP == 4 * MX_KSTEP, "a scale word holds a group");

// Packed weights as the kernels see them (the layout stands in mx.hip).
struct MxPacked { const u32x4 *codes; const uint32_t *scales; const int32_t *ref; int ksteps, kgroups, tiles; };
MxPacked mx_packed_at(const void *packed, int N, int K);

enum { DT_MX = 4 };               // activations that are microscaled too
size_t mx_gemm_scratch_size(int x_dt, int M, int N, int K);
void launch_mx_gemm(int x_dt, const void *x, int64_t ldx, const void *packed, int y_dt, void *y, int64_t ldy, int M, int N, int K, void *scratch, hipStream_t st);
void launch_mx_gemm_mx(const void *x_codes, const void *x_scales, const void *packed, int y_dt, void *y, int64_t ldy, int M, int N, int K, void *scratch, hipStream_t st);


// For a context's layers (16-bit types).  A matrix of packed rows, as launch_pack takes them, quantised and packed; N: its rows, padding ones among them.
size_t mx_packed_size(int N, int K);
void launch_mx_pack_rows(int dt, const PackSrc &src, int N, int K, void *packed, hipStream_t st);
// The planes of X W^T: plane s < splits of part (mx_plane_splits of them), [M][ld], ld a multiple of four and at least N.  A row's planes are the same for
// every M.
bool launch_mx_planes(int dt, const void *packed, int N, int K, const void *X, int ldx, int M, float *part, int ld, int splits, hipStream_t st);
// act[M][F] = SiLU(gate) * up of X with a matrix whose rows alternate in groups of 16 (PackSrc::interleave16).  part as above, for the planes of a split product.
bool launch_mx_gate_up(int dt, const void *packed, int F, int K, const void *X, int ldx, int M, float *part, int ld, void *act, hipStream_t st);

// Leaves the message that poss_last_error(NULL) returns; the code is handed through.
int set_error(int code, const char *fmt, ...);

static inline int mx_blocks(int cols) { return (cols - 1) / MX_BLOCK + 1; }     // cols > 0
// What a product takes: offsets within a tile's rows are 32 bits (256 rows of three times K 16-bit values), and so are a launch's threads.
constexpr int MX_MOST_M = 1 << 24, MX_MOST_N = 1 << 27, MX_MOST_K = 1 << 21;
constexpr int64_t MX_MOST_MN = 1ll << 38;

// Where a row's largest scale stands in the packed form: as it is between 2^-24 and 2^0, moved there otherwise, the row's sums brought back at the end.  So
// no sum of ordinary activations with large weights leaves float32's range on the way, and none of activations as large as float32 has them with small
// weights: 2^21 terms of 3.4e38 * 6 * 2^-24 do not; between the two a sum overflows where its terms take it.
__device__ __forceinline__ int mx_held(int top) { return min(127, max(103, top)); }
// A row's largest scale byte as the packed form keeps it: that byte and, ready for the sums, the power of two that they are to be multiplied by.
constexpr int MX_NAN_ROW = 0x7fffffff;
__device__ __forceinline__ int mx_row_ref(int top) { return top == 255 ? MX_NAN_ROW : (top - mx_held(top)) * 256 + top; }
__device__ __forceinline__ int mx_row_top(int ref) { return ref & 255; }
__device__ __forceinline__ int mx_row_power(int ref) { return ref >> 8; }

// 2^(b - 127) of a scale byte, exactly (2^-127 is subnormal).
__device__ __forceinline__ float mx_power(unsigned b) {
    return __builtin_bit_cast(float, b == 255 ? 0x7fc00000u : b == 0 ? 0x00400000u : b << 23);
}

}  // namespace poss
