// Eviction from a paged cache by accumulated attention weight (include/poss.h: poss_kv_evict).
//
// Slots are ranked by a 32-bit key: those that always stay above all, NaN below all, the others by their weight, mapped so that unsigned order is
// the order of the numbers (-0 as 0).  Of the n = min(length, budget) that stay the n-th largest key is found; of the slots with that very key the lowest
// stay.  Holes below n and kept slots from n on are equally many:
// the j-th hole is filled from the j-th of those.  No source is a destination, so the moves need no order.
//
// A workgroup per head chooses, bound by latency (1025 slots of 8 heads 12 us, 4096 of 256 heads 16, 18580 of one 31, 131072 of 8 238); a second launch moves.  Keys move as rows; a
// value row gives and takes single values, so that whole lines are read and parts of lines written: 32 sequences of up to 4096 slots to 2000, 8 heads of 128, bf16: 57 us for 105 MB
// read and 91 written, 17 us of them the keys'.  Reading and writing the destinations' lines whole took as long.
#include "kv.h"

namespace poss {

__device__ __forceinline__ uint32_t weight_key(float w) {      // 1 .. 0xfffffffe; NaN: 0
    if (w != w) return 0;
    const uint32_t b = __builtin_bit_cast(uint32_t, w + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct EvictArgs {
    const float *weights; const int32_t *positions, *lengths;
    int budget, first, recent;
    int32_t *kept; float *weights_out; int32_t *positions_out, *lengths_out;
};

constexpr int EVICT_THREADS = 1024, EVICT_WAVES = EVICT_THREADS / 64;

__device__ __forceinline__ int lanes_below(unsigned long long them) {      // of them, those before this lane
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(them >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)them, 0));
}
// Sum of a number per wave over the waves; one barrier.
template <int WAVES>
__device__ __forceinline__ int waves_sum(int x, int *red) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    int s = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += red[w];
    return s;
}
template <int WAVES>
__device__ __forceinline__ int block_newest(int newest, int *red) {
    for (int o = 32; o; o >>= 1) newest = max(newest, __shfl_xor(newest, o));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = newest;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) newest = max(newest, red[w]);
    return newest;
}
__device__ __forceinline__ uint32_t slot_key(float w, int pos, int first, int64_t border) { return pos < first || pos > border ? 0xffffffffu : weight_key(w); }

// One head's rows of the arrays, and what every kernel does with them first: what lies beyond the new length, and a head that loses nothing.
struct EvictHead { const float *w; const int32_t *pos; int32_t *kept; float *wo; int32_t *po; int len, n; };
template <int THREADS>
__device__ __forceinline__ EvictHead evict_head(const KvView &c, const EvictArgs &a) {
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int64_t row = (int64_t)b * c.hkv + h, base = row * c.slots;
    EvictHead e{a.weights + base, a.positions + base, a.kept + row * a.budget, a.weights_out + base, a.positions_out + base, a.lengths[b], 0};
    e.len = e.len < 0 ? 0 : e.len > c.slots ? c.slots : e.len;
    e.n = e.len < a.budget ? e.len : a.budget;
    if (h == 0 && tid == 0) a.lengths_out[b] = e.n;
    for (int i = e.n + tid; i < a.budget; i += THREADS) e.kept[i] = -1;
    for (int i = e.n + tid; i < c.slots; i += THREADS) { e.wo[i] = 0.f; e.po[i] = -1; }
    if (e.n == e.len)
        for (int i = tid; i < e.n; i += THREADS) { e.kept[i] = i; e.wo[i] = e.w[i]; e.po[i] = e.pos[i]; }
    return e;
}

// One workgroup per sequence and key head, up to K * THREADS slots: slot k * THREADS + t is thread t's k-th, its key stays in a register.  The n-th largest key is found from the
// highest bit down, two bits at a time, by counting the keys from each candidate on: counting is ballots, with no contention for
// a histogram's few busy bins.  It ends as soon as exactly n keys are counted, for distinct weights long before the last bit.
template <int THREADS, int K>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(KvView c, EvictArgs a) {
    constexpr int WAVES = THREADS / 64;
    __shared__ int red[2][3][WAVES], before[K][WAVES];
    __shared__ uint16_t movers[K * THREADS / 2];       // as many as there are holes, at most half of the slots
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const EvictHead e = evict_head<THREADS>(c, a);
    const int len = e.len, n = e.n;
    if (n == len) return;
    float w[K];
    int pos[K];
    int newest = INT32_MIN;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = k * THREADS + tid;
        w[k] = i < len ? e.w[i] : 0.f;
        pos[k] = i < len ? e.pos[i] : INT32_MIN;
        newest = max(newest, pos[k]);
    }
    const int64_t border = (int64_t)block_newest<WAVES>(newest, red[0][0]) - a.recent;
    uint32_t key[K];
#pragma unroll
    for (int k = 0; k < K; ++k) key[k] = k * THREADS + tid < len ? slot_key(w[k], pos[k], a.first, border) : 0;
    uint32_t found = 0;                                      // the keys from here on are at least n
    int above = 0;                                           // the keys beyond it, once it is the n-th
    bool exact = false;                                      // just n keys from `found` on
    int turn = 1;
    for (int shift = 30; shift >= 0 && !exact; shift -= 2, turn ^= 1) {
        int many[3] = {0, 0, 0};
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 3; ++j) many[j] += __popcll(__ballot(key[k] >= (found | (uint32_t)(j + 1) << shift)));
        if (lane == 0)
            for (int j = 0; j < 3; ++j) red[turn][j][wave] = many[j];
        __syncthreads();
        for (int j = 0; j < 3; ++j) {
            many[j] = 0;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) many[j] += red[turn][j][v];
        }
        const int step = many[2] >= n ? 3 : many[1] >= n ? 2 : many[0] >= n ? 1 : 0;
        found |= (uint32_t)step << shift;
        exact = step && many[step - 1] == n;
    }
    // of the keys equal to the n-th the first `want`, in slot order
    int want = 0;
    if (!exact) {
        int more = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) more += __popcll(__ballot(key[k] > found));
        above = waves_sum<WAVES>(more, red[turn][0]);
        want = n - above;
    }
    uint32_t stays = 0;
    if (exact) {
#pragma unroll
        for (int k = 0; k < K; ++k) if (k * THREADS + tid < len && key[k] >= found) stays |= 1u << k;
    } else {
        unsigned long long equal[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            equal[k] = __ballot(k * THREADS + tid < len && key[k] == found);
            if (lane == 0) before[k][wave] = __popcll(equal[k]);
        }
        __syncthreads();
        int base = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            int mine = base;
            for (int v = 0; v < WAVES; ++v) { const int x = before[k][v]; base += x; if (v < wave) mine += x; }
            const bool eq = equal[k] >> lane & 1;
            if (k * THREADS + tid < len && (key[k] > found || (eq && mine + lanes_below(equal[k]) < want))) stays |= 1u << k;
        }
        __syncthreads();
    }
    // holes below n and movers from n on, counted off in slot order in the two halves of a number
    unsigned long long holes[K], moves[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = k * THREADS + tid;
        holes[k] = __ballot(i < n && !(stays >> k & 1));
        moves[k] = __ballot(i >= n && (stays >> k & 1));
        if (lane == 0) before[k][wave] = __popcll(holes[k]) | __popcll(moves[k]) << 16;
    }
    __syncthreads();
    int hole_at[K], base = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        int mine = base;
        for (int v = 0; v < WAVES; ++v) { const int x = before[k][v]; base += x; if (v < wave) mine += x; }
        hole_at[k] = holes[k] >> lane & 1 ? (mine & 0xffff) + lanes_below(holes[k]) : -1;
        if (moves[k] >> lane & 1) movers[(mine >> 16) + lanes_below(moves[k])] = (uint16_t)(k * THREADS + tid);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = k * THREADS + tid;
        if (i >= n) continue;
        int from = i;
        if (hole_at[k] >= 0) { from = movers[hole_at[k]]; w[k] = e.w[from]; pos[k] = e.pos[from]; }
        e.kept[i] = from; e.wo[i] = w[k]; e.po[i] = pos[k];
    }
}

// More slots: the 12 highest bits of the n-th key (sign, exponent, three bits of mantissa) come from a histogram, the others by counting among the keys that share
// them, in LDS; where those are too many (equal weights), from two more histograms.  each(f): f of every key of this thread; 1024 threads.
// The n-th key, how many of the keys equal to it stay (the first in slot order), and how many there are.
constexpr int BINS = 4096;
struct NthKey { uint32_t key; int want, share; };
struct NthRoom { int hist[BINS], red[2][3][EVICT_WAVES], pick[3], taken; };
template <class Each>
__device__ __forceinline__ NthKey nth_key(Each each, int n, int len, NthRoom &room) {
    constexpr int EACH = BINS / EVICT_THREADS, FEW = 8;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // the digit of `bits` bits at `shift` of the key that is the want-th largest of those with this prefix: prefix, want, and how many share the new prefix
    uint32_t prefix = 0;
    int want = n, share = len;
    auto digit = [&](int shift, int bits) {
        __syncthreads();
        for (int i = tid; i < BINS; i += EVICT_THREADS) room.hist[i] = 0;
        __syncthreads();
        each([&](uint32_t k) { if (shift + bits == 32 || k >> (shift + bits & 31) == prefix) atomicAdd(&room.hist[k >> shift & ((1 << bits) - 1)], 1); });
        __syncthreads();
        // thread t looks at bins EACH t .. EACH t + EACH - 1, counted from the last
        int mine[EACH], sum = 0;
#pragma unroll
        for (int j = 0; j < EACH; ++j) sum += mine[j] = room.hist[BINS - 1 - (tid * EACH + j)];
        int at = sum;
        for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(at, o); if (lane >= o) at += y; }
        if (lane == 63) room.red[1][0][wave] = at;
        __syncthreads();
        at -= sum;
        for (int v = 0; v < wave; ++v) at += room.red[1][0][v];
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            if (at < want && want <= at + mine[j]) { room.pick[0] = BINS - 1 - (tid * EACH + j); room.pick[1] = want - at; room.pick[2] = mine[j]; }
            at += mine[j];
        }
        __syncthreads();
        prefix = prefix << bits | (uint32_t)room.pick[0];
        want = room.pick[1]; share = room.pick[2];
    };
    if (tid == 0) room.taken = 0;                              // (seen by all behind digit()'s barriers)
    digit(20, 12);
    if (share > BINS) {
        digit(8, 12);
        digit(0, 8);
        return NthKey{prefix, want, share};
    }
    each([&](uint32_t k) { if (k >> 20 == prefix) room.hist[atomicAdd(&room.taken, 1)] = (int)k; });      // (in any order: they are counted)
    __syncthreads();
    if (share <= 64 * FEW) {                                   // few: one wave counts them bit by bit, without a barrier
        if (wave == 0) {
            uint32_t key[FEW], found = prefix << 20;
#pragma unroll
            for (int j = 0; j < FEW; ++j) key[j] = j * 64 + lane < share ? (uint32_t)room.hist[j * 64 + lane] : 0;
            int from = share, beyond = 0;                      // keys from `found` on, and those beyond its stretch
            for (int bit = 19; bit >= 0 && from != want; --bit) {
                int many = 0;
#pragma unroll
                for (int j = 0; j < FEW; ++j) many += __popcll(__ballot(j * 64 + lane < share && key[j] >= (found | 1u << bit)));
                if (many >= want) { found |= 1u << bit; from = many; } else beyond = many;
            }
            // with `from` of them exactly as many as stay, the lowest of these is the n-th and none of its equals goes
            if (from == want) {
                uint32_t low = ~0u;
#pragma unroll
                for (int j = 0; j < FEW; ++j) if (j * 64 + lane < share && key[j] >= found) low = min(low, key[j]);
                for (int o = 32; o; o >>= 1) low = min(low, (uint32_t)__shfl_xor((int)low, o));
                found = low; beyond = want - 1; from = want;
            }
            if (lane == 0) { room.pick[0] = (int)found; room.pick[1] = want - beyond; room.pick[2] = from - beyond; }
        }
        __syncthreads();
        return NthKey{(uint32_t)room.pick[0], room.pick[1], room.pick[2]};
    }
    uint32_t key[EACH], found = prefix << 20;
    bool in[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) { in[j] = j * EVICT_THREADS + tid < share; key[j] = in[j] ? (uint32_t)room.hist[j * EVICT_THREADS + tid] : 0; }
    // often all are the same number (weights of zero)
    uint32_t differ = 0;
#pragma unroll
    for (int j = 0; j < EACH; ++j) if (in[j]) differ |= key[j] ^ (uint32_t)room.hist[0];
    if (__any(differ) && lane == 0) room.pick[0] = -1;         // (`prefix` has been read from there: barriers behind that)
    __syncthreads();
    if (room.pick[0] != -1) return NthKey{(uint32_t)room.hist[0], want, share};
    int turn = 0, beyond = 0, least = share;                   // keys above `found`'s stretch, and from it on
    for (int shift = 18; shift >= 0; shift -= 2, turn ^= 1) {
        int many[3] = {0, 0, 0};
#pragma unroll
        for (int k = 0; k < EACH; ++k)
#pragma unroll
            for (int j = 0; j < 3; ++j) many[j] += __popcll(__ballot(in[k] && key[k] >= (found | (uint32_t)(j + 1) << shift)));
        if (lane == 0)
            for (int j = 0; j < 3; ++j) room.red[turn][j][wave] = many[j];
        __syncthreads();
        for (int j = 0; j < 3; ++j) {
            many[j] = 0;
#pragma unroll
            for (int v = 0; v < EVICT_WAVES; ++v) many[j] += room.red[turn][j][v];
        }
        const int step = many[2] >= want ? 3 : many[1] >= want ? 2 : many[0] >= want ? 1 : 0;
        found |= (uint32_t)step << shift;
        if (step < 3) beyond = many[step];                     // (with step 3 what lies above is as before)
        if (step) least = many[step - 1];
    }
    return NthKey{found, want - beyond, least - beyond};
}

// Up to K * 1024 slots, keys in registers: slot k * 1024 + t is thread t's k-th.
template <int K>
__global__ void __launch_bounds__(EVICT_THREADS) evict_select_wide_kernel(KvView c, EvictArgs a) {
    constexpr int COUNTS = K * EVICT_WAVES, AHEAD = 8;
    __shared__ NthRoom room;
    __shared__ int before[COUNTS];
    __shared__ uint16_t movers[K * EVICT_THREADS / 2];         // as many as there are holes, at most half of the slots
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const EvictHead e = evict_head<EVICT_THREADS>(c, a);
    const int len = e.len, n = e.n;
    if (n == len) return;
    uint32_t key[K];
    int newest = INT32_MIN;
    {
        int pos[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = k * EVICT_THREADS + tid;
            pos[k] = i < len ? e.pos[i] : INT32_MIN;
            newest = max(newest, pos[k]);
        }
        const int64_t border = (int64_t)block_newest<EVICT_WAVES>(newest, room.red[0][0]) - a.recent;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = k * EVICT_THREADS + tid;
            key[k] = slot_key(i < len ? e.w[i] : 0.f, pos[k], a.first, border);
        }
    }
    const NthKey nth = nth_key([&](auto f) {
#pragma unroll
        for (int k = 0; k < K; ++k) if (k * EVICT_THREADS + tid < len) f(key[k]);
    }, n, len, room);
    // counts[k][wave], in slot order, become sums of those before
    auto count_off = [&]() {
        __syncthreads();
        if (wave == 0) {
            int x[COUNTS / 64], sum = 0;
#pragma unroll
            for (int j = 0; j < COUNTS / 64; ++j) sum += x[j] = before[lane * (COUNTS / 64) + j];
            int at = sum;
            for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(at, o); if (lane >= o) at += y; }
            at -= sum;
#pragma unroll
            for (int j = 0; j < COUNTS / 64; ++j) { before[lane * (COUNTS / 64) + j] = at; at += x[j]; }
        }
        __syncthreads();
    };
    const bool ties = nth.want < nth.share;
    uint32_t stays = 0;
    if (ties) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const unsigned long long eq = __ballot(k * EVICT_THREADS + tid < len && key[k] == nth.key);
            if (lane == 0) before[k * EVICT_WAVES + wave] = __popcll(eq);
        }
        count_off();
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool in = k * EVICT_THREADS + tid < len;
        const unsigned long long eq = __ballot(in && key[k] == nth.key);
        if (in && (key[k] > nth.key || (key[k] == nth.key && (!ties || before[k * EVICT_WAVES + wave] + lanes_below(eq) < nth.want)))) stays |= 1u << k;
    }
    // holes below n and movers from n on, counted off in the two halves of a number
    __syncthreads();
    auto holes_at = [&](int k) { return __ballot(k * EVICT_THREADS + tid < n && !(stays >> k & 1)); };
    auto moves_at = [&](int k) { return __ballot(k * EVICT_THREADS + tid >= n && (stays >> k & 1)); };
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const unsigned long long holes = holes_at(k), moves = moves_at(k);
        if (lane == 0) before[k * EVICT_WAVES + wave] = __popcll(holes) | __popcll(moves) << 16;
    }
    count_off();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const unsigned long long moves = moves_at(k);
        if (moves >> lane & 1) movers[(before[k * EVICT_WAVES + wave] >> 16) + lanes_below(moves)] = (uint16_t)(k * EVICT_THREADS + tid);
    }
    __syncthreads();
#pragma unroll
    for (int k0 = 0; k0 < K; k0 += AHEAD) {
        int from[AHEAD], pos[AHEAD];
        float w[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int k = k0 + u, i = k * EVICT_THREADS + tid;
            const unsigned long long holes = holes_at(k);
            from[u] = i >= n ? -1 : holes >> lane & 1 ? movers[(before[k * EVICT_WAVES + wave] & 0xffff) + lanes_below(holes)] : i;
            if (from[u] >= 0) { w[u] = e.w[from[u]]; pos[u] = e.pos[from[u]]; }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = (k0 + u) * EVICT_THREADS + tid;
            if (from[u] >= 0) { e.kept[i] = from[u]; e.wo[i] = w[u]; e.po[i] = pos[u]; }
        }
    }
}

// The same for any number of slots: what is read is read again for every pass, by each wave its own stretch of slots, 64 side by side, with a barrier only between passes.
__global__ void __launch_bounds__(EVICT_THREADS) evict_select_long_kernel(KvView c, EvictArgs a) {
    constexpr int AHEAD = 16;                                  // loads of an array on their way at a time
    __shared__ NthRoom room;
    int (*const red)[3][EVICT_WAVES] = room.red;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const EvictHead e = evict_head<EVICT_THREADS>(c, a);
    const int len = e.len, n = e.n;
    if (n == len) return;
    const int per = (len + 64 * EVICT_WAVES - 1) / (64 * EVICT_WAVES) * 64, i0 = wave * per + lane, i1 = min(len, (wave + 1) * per);
    int newest = INT32_MIN;
    for (int i = i0; i < i1; i += 64 * AHEAD) {
        int pos[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) pos[u] = i + 64 * u < i1 ? e.pos[i + 64 * u] : INT32_MIN;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) newest = max(newest, pos[u]);
    }
    const int64_t border = (int64_t)block_newest<EVICT_WAVES>(newest, red[0][0]) - a.recent;
    float w[AHEAD];
    int pos[AHEAD];
    auto load = [&](int i) {                                   // slots i, i + 64 ..
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) { const bool in = i + 64 * u < i1; w[u] = in ? e.w[i + 64 * u] : 0.f; pos[u] = in ? e.pos[i + 64 * u] : 0; }
    };
    auto key_of = [&](int u) { return slot_key(w[u], pos[u], a.first, border); };
    const NthKey nth = nth_key([&](auto f) {
        for (int i = i0; i < i1; i += 64 * AHEAD) {
            load(i);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) if (i + 64 * u < i1) f(key_of(u));
        }
    }, n, len, room);
    const uint32_t prefix = nth.key;
    const int want = nth.want, share = nth.share;
    // kept: keys above the prefix, and the first `want` of the `share` with it.  Each wave counts its equal ones, then its holes and movers, then writes.
    __syncthreads();
    const bool ties = want < share;
    if (ties) {
        int many = 0;
        for (int i = i0; i - lane < i1; i += 64 * AHEAD) {
            load(i);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) many += __popcll(__ballot(i + 64 * u < i1 && key_of(u) == prefix));
        }
        if (lane == 0) red[0][0][wave] = many;
    }
    __syncthreads();
    int equal_first = 0;
    if (ties) for (int v = 0; v < wave; ++v) equal_first += red[0][0][v];
    auto stays_at = [&](int i, int u, int &equal) {            // of the 64 slots side by side, the u-th loaded; equal: equal ones before them, brought forward
        const uint32_t k = key_of(u);
        const unsigned long long eq = __ballot(i < i1 && k == prefix);
        const bool stays = i < i1 && (k > prefix || (k == prefix && (!ties || equal + lanes_below(eq) < want)));
        equal += __popcll(eq);
        return stays;
    };
    int holes = 0, movers = 0, equal = equal_first;
    for (int j = i0; j - lane < i1; j += 64 * AHEAD) {
        load(j);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = j + 64 * u;
            const unsigned long long stay = __ballot(stays_at(i, u, equal)), low = __ballot(i < n), in = __ballot(i < i1);
            holes += __popcll(in & low & ~stay); movers += __popcll(stay & ~low);
        }
    }
    if (lane == 0) { red[0][1][wave] = holes; red[0][2][wave] = movers; }
    __syncthreads();
    int hole = 0, mover = 0, all = 0;
    for (int v = 0; v < EVICT_WAVES; ++v) { if (v < wave) { hole += red[0][1][v]; mover += red[0][2][v]; } all += red[0][2][v]; }
    equal = equal_first;
    for (int j = i0; j - lane < i1; j += 64 * AHEAD) {
        load(j);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = j + 64 * u;
            const bool stays = stays_at(i, u, equal), is_hole = i < i1 && i < n && !stays, is_mover = stays && i >= n;
            const unsigned long long them = __ballot(is_hole), those = __ballot(is_mover);
            // the lists meet in the outputs: a hole notes its rank as -2 - rank, and po[n ..] lends its room to the movers
            if (is_hole) e.kept[i] = -2 - (hole + lanes_below(them));
            else if (stays && i < n) { e.kept[i] = i; e.wo[i] = w[u]; e.po[i] = pos[u]; }
            if (is_mover) e.po[n + mover + lanes_below(those)] = i;
            hole += __popcll(them); mover += __popcll(those);
        }
    }
    __syncthreads();
    for (int i = tid; i < n; i += EVICT_THREADS * AHEAD) {
        int from[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) from[u] = i + u * EVICT_THREADS < n ? e.kept[i + u * EVICT_THREADS] : 0;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) from[u] = from[u] < 0 ? e.po[n + (-2 - from[u])] : -1;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) if (from[u] >= 0) { w[u] = e.w[from[u]]; pos[u] = e.pos[from[u]]; }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) if (from[u] >= 0) { const int to = i + u * EVICT_THREADS; e.kept[to] = from[u]; e.wo[to] = w[u]; e.po[to] = pos[u]; }
    }
    __syncthreads();
    for (int i = n + tid; i < n + all; i += EVICT_THREADS) e.po[i] = -1;
}

// The slots 256 x .. below the budget of one sequence and head whose source is another, 64 (or 32) of the dims: listed, then moved, keys in pieces of 16 bytes, values with a lane per
// slot: sources ascend with destinations, so that the values of 64 of them lie in a few lines of each value row.  A launch has MOVE_GROUPS times as many slots side by side at most (threads
// are counted in 32 bits: 2^30 slots of heads of 256 dims, cut in four, are 2^32 of them); a workgroup goes on to others.
constexpr int MOVE_SLOTS = 256, MOVE_GROUPS = 1024;
template <typename T>
__global__ void __launch_bounds__(256) evict_move_kernel(KvView c, const int32_t *__restrict__ kept, int budget, int splits, int most) {
    constexpr int E = 16 / sizeof(T), AHEAD = 8;
    typedef T vec __attribute__((ext_vector_type(E)));
    __shared__ int64_t key_from[MOVE_SLOTS], key_to[MOVE_SLOTS], value_from[MOVE_SLOTS], value_to[MOVE_SLOTS];
    __shared__ int count;
    const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, dims = c.dh / splits, first = blockIdx.x % splits * dims;
    T *k = static_cast<T *>(c.k), *v = static_cast<T *>(c.v);
    for (int chunk = blockIdx.x / splits; chunk * MOVE_SLOTS < most; chunk += MOVE_GROUPS) {
        const int to = chunk * MOVE_SLOTS + tid, from = to < most ? kept[((int64_t)b * c.hkv + h) * budget + to] : -1;
        int pf = -1, pt = -1;
        if (from >= 0 && from != to) { pf = kv_page(c, b, from); pt = kv_page(c, b, to); }
        const bool moves = pf >= 0 && pt >= 0;
        if (chunk >= MOVE_GROUPS) __syncthreads();             // the lists of the slots before are done with
        if (tid == 0) count = 0;
        __syncthreads();
        // (the order between waves does not matter, a wave's own slots stay together)
        const unsigned long long them = __ballot(moves);
        int at = 0;
        if ((tid & 63) == 0 && them) at = atomicAdd(&count, __popcll(them));
        at = __shfl(at, 0) + lanes_below(them);
        if (moves) {
            key_from[at] = kv_key_at(c, pf, h, from); key_to[at] = kv_key_at(c, pt, h, to);
            value_from[at] = kv_value_at(c, pf, h, 0, from); value_to[at] = kv_value_at(c, pt, h, 0, to);
        }
        __syncthreads();
        const int n = count, pieces = dims / E;
#pragma unroll 2
        for (int x = tid; x < n * pieces; x += 256) {
            const int i = x / pieces, d = first + (x - i * pieces) * E;
            *reinterpret_cast<vec *>(k + key_to[i] + d) = *reinterpret_cast<const vec *>(k + key_from[i] + d);
        }
        const int each = dims / 4, d0 = first + (tid >> 6) * each;      // a wave takes a quarter of the value rows (a multiple of AHEAD)
        for (int i = tid & 63; i < n; i += 64) {
            const T *vf = v + value_from[i];
            T *vt = v + value_to[i];
            for (int d = d0; d < d0 + each; d += AHEAD) {
                T got[AHEAD];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) got[j] = vf[(int64_t)(d + j) << c.shift];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) vt[(int64_t)(d + j) << c.shift] = got[j];
            }
        }
    }
}

}  // namespace poss

// ------------------------------------------------------------------------------------------ C entry point (include/poss.h)
using namespace poss;

extern "C" int poss_kv_evict(const poss_kv_cache *cache, const float *weights, const int32_t *positions, const int32_t *lengths, int32_t budget, int32_t first, int32_t recent,
                             int32_t *kept, float *weights_out, int32_t *positions_out, int32_t *lengths_out, void *hip_stream) {
    const char *who = "poss_kv_evict";
    if (const char *why = kv_cache_bad(cache)) return set_error(POSS_E_INVALID_ARG, "%s: %s", who, why);
    if (budget < 1 || budget > 1 << 30 || first < 0 || recent < 0 || (int64_t)first + recent > budget) return set_error(POSS_E_INVALID_ARG, "%s: 0 <= first + recent <= budget, and a budget, are wanted", who);
    if (cache->n_seq == 0) return POSS_OK;
    if (!weights || !positions || !lengths || !kept || !weights_out || !positions_out || !lengths_out) return set_error(POSS_E_INVALID_ARG, "%s: null argument", who);
    for (const void *p : {(const void *)weights, (const void *)positions, (const void *)lengths, (const void *)kept, (const void *)weights_out, (const void *)positions_out, (const void *)lengths_out})
        if (!kv_aligned(p, 4)) return set_error(POSS_E_INVALID_ARG, "%s: an array is not aligned to its type", who);
    if (weights == weights_out || positions == positions_out || lengths == lengths_out) return set_error(POSS_E_INVALID_ARG, "%s: outputs must be arrays of their own", who);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const KvView c = kv_view(*cache);
    const EvictArgs a{weights, positions, lengths, budget, first, recent, kept, weights_out, positions_out, lengths_out};
    const dim3 heads(c.hkv, c.n_seq);
#define POSS_SELECT(THREADS, K) if (c.slots <= THREADS * K) evict_select_kernel<THREADS, K><<<heads, THREADS, 0, st>>>(c, a)
    POSS_SELECT(256, 3);
    else POSS_SELECT(256, 6);
    else POSS_SELECT(512, 4);
    else POSS_SELECT(512, 8);
    else POSS_SELECT(512, 16);
#undef POSS_SELECT
    else if (c.slots <= 16 * EVICT_THREADS) evict_select_wide_kernel<16><<<heads, EVICT_THREADS, 0, st>>>(c, a);
    else if (c.slots <= 32 * EVICT_THREADS) evict_select_wide_kernel<32><<<heads, EVICT_THREADS, 0, st>>>(c, a);
    else evict_select_long_kernel<<<heads, EVICT_THREADS, 0, st>>>(c, a);
    const int most = budget < c.slots ? budget : c.slots;
    const int splits = c.dh % 64 ? c.dh / 32 : c.dh / 64;
    const int chunks = (most + MOVE_SLOTS - 1) / MOVE_SLOTS;
    const dim3 grid((chunks < MOVE_GROUPS ? chunks : MOVE_GROUPS) * splits, c.hkv, c.n_seq);
    if (cache->dtype == DT_F32) evict_move_kernel<float><<<grid, 256, 0, st>>>(c, kept, budget, splits, most);
    else if (cache->dtype == DT_BF16) evict_move_kernel<bf16_t><<<grid, 256, 0, st>>>(c, kept, budget, splits, most);
    else evict_move_kernel<f16_t><<<grid, 256, 0, st>>>(c, kept, budget, splits, most);
    return kv_launched(who);
}
