// The pieces of 16 bytes of a row's heads, plain C++ (the same on the host, where it is compared with the division).
#pragma once
#include <stdint.h>
#ifdef __HIPCC__
#define POSS_HD __host__ __device__ __forceinline__
#else
#define POSS_HD static inline
#endif

namespace poss {

// A unit is a piece of a head or, where pairs lie half the rotated values apart, a piece of the first half and its partner of the second.  units: of one head; of_units: 2^31 / units,
// rounded up (31 bits, as 2^32 / 1 would not fit); parts: waves that share a row.
struct Units { int units; uint32_t of_units; int parts; };

// The head of a row's unit j: j / units.  of_units * units exceeds 2^31 by less than units, so this is the quotient while j * units < 2^31.
POSS_HD int unit_head(int j, uint32_t of_units) {
#ifdef __HIP_DEVICE_COMPILE__
    return (int)__umulhi((uint32_t)j << 1, of_units);
#else
    return (int)((uint64_t)((uint32_t)j << 1) * of_units >> 32);
#endif
}

constexpr int ROWS_FULL = 2048;                              // two waves a SIMD
// Whether heads of dh values, rot of them rotated, are whole pieces of E values whose head unit_head() finds, and their units.
static inline bool units_of(int E, int rows, int heads, int dh, int rot, bool interleaved, Units &n) {
    const int half = rot / 2;
    if (dh % E || rot % E || (!interleaved && half % E)) return false;
    n.units = dh / E - (interleaved ? 0 : half / E);
    n.parts = rows < ROWS_FULL ? 4 : 1;
    n.of_units = (uint32_t)(((1ull << 31) + n.units - 1) / n.units);
    const int64_t all = (int64_t)heads * n.units;
    return all < 1 << 24 && all * n.units <= 1ll << 31;
}

}  // namespace poss
