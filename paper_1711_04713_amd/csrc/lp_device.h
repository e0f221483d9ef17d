// Device-side helpers shared by the gfx950 kernels of this library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lp.h"

namespace lp {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef short v2s __attribute__((ext_vector_type(2)));
typedef unsigned short v2us __attribute__((ext_vector_type(2)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

// Requantization parameters of the LPAct step (Sec. 2.1): divide by 2^s,
// round to nearest, clip to [lo, hi].
struct ActParams {
    int s;        // f_acc - f_out; > 0 shifts right, <= 0 shifts left
    int relu;     // clamp negatives to zero first
    int even;     // tie rule: 0 away from zero, 1 to even
    int lo, hi;   // code range of the output format
};

__host__ inline ActParams make_act_params(int f_acc, lp_qfmt qy, int relu, lp_round r)
{
    ActParams a;
    a.s = f_acc - qy.f;
    a.relu = relu ? 1 : 0;
    a.even = (r == LP_ROUND_NEAREST_EVEN) ? 1 : 0;
    a.lo = -(1 << (qy.n - 1));
    a.hi = (1 << (qy.n - 1)) - 1;
    return a;
}

// One accumulator -> one output code.  |v| < 2^62.  sat: the rounded value lay outside
// [lo, hi] and was clipped.
__device__ __forceinline__ int act_one(int64_t v, const ActParams &p, bool &sat)
{
    if (p.relu && v < 0) v = 0;
    int64_t r;
    if (p.s > 0) {
        const int64_t half = (int64_t)1 << (p.s - 1);
        if (!p.even) {
            const int64_t mag = v < 0 ? -v : v;
            const int64_t q = (mag + half) >> p.s;
            r = v < 0 ? -q : q;
        } else {
            int64_t q = v >> p.s;                       // floor
            const int64_t rem = v & (((int64_t)1 << p.s) - 1);
            if (rem > half || (rem == half && (q & 1))) q += 1;
            r = q;
        }
    } else {
        // beyond the code range the product stays beyond it: one step outside keeps it in 64 bits
        int64_t c = v;
        if (c > p.hi) c = (int64_t)p.hi + 1;
        if (c < p.lo) c = (int64_t)p.lo - 1;
        r = c * ((int64_t)1 << (-p.s));
    }
    sat = r > p.hi || r < p.lo;
    if (r > p.hi) r = p.hi;
    if (r < p.lo) r = p.lo;
    return (int)r;
}

__device__ __forceinline__ int act_one(int64_t v, const ActParams &p)
{
    bool sat;
    return act_one(v, p, sat);
}

// Number of lanes of the wavefront for which pred holds (ballot + popcount).
__device__ __forceinline__ unsigned wave_count(bool pred)
{
    return (unsigned)__popcll(__ballot(pred));
}

// Adds a block's counts to the caller's counters (either may be null): the waves' totals meet in LDS
// and the block issues one atomic per counter.  The atomics of a launch all hit one address and are
// served one after the other, 12 to 14 ns each: with one per wave and counter (16 k of them) a counting
// lp_quantize of 25.7 M elements took 207 us instead of 29, a counting lp_act to 8 bits (32 k) 398 instead of 44.
template <int THREADS>
__device__ __forceinline__ void add_block_counts(unsigned zeros, unsigned sats, unsigned long long *zero_count,
                                                 unsigned long long *sat_count)
{
    __shared__ unsigned part[2][THREADS / 64];
    if ((threadIdx.x & 63) == 0) {
        part[0][threadIdx.x >> 6] = zeros;
        part[1][threadIdx.x >> 6] = sats;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        unsigned total = 0;
        for (int w = 0; w < THREADS / 64; ++w) total += part[threadIdx.x][w];
        unsigned long long *out = threadIdx.x ? sat_count : zero_count;
        if (out && total) atomicAdd(out, (unsigned long long)total);
    }
}

// ------------------------------------------------------------------ Philox4x32-10
// Counter-based generator of Salmon, Moraes, Dror, Shaw (SC'11): ten rounds of two
// 32x32->64 multiplies and xors, key bumped by the Weyl constants each round.  One block gives four
// words; element i of a tensor draws word i % 4 of the block with counter (i / 4, 0).
struct PhiloxBlock {
    uint32_t w[4];
};
__device__ __forceinline__ PhiloxBlock philox4x32_10(uint64_t ctr, uint64_t key)
{
    uint32_t c0 = (uint32_t)ctr, c1 = (uint32_t)(ctr >> 32), c2 = 0, c3 = 0;
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0;
        const uint64_t p1 = (uint64_t)0xCD9E8D57u * c2;
        const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
        const uint32_t n1 = (uint32_t)p1;
        const uint32_t n2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        const uint32_t n3 = (uint32_t)p0;
        c0 = n0; c1 = n1; c2 = n2; c3 = n3;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return PhiloxBlock{{c0, c1, c2, c3}};
}
// the draw of element i by itself (ragged tails)
__device__ __forceinline__ uint32_t philox_draw(uint64_t i, uint64_t key)
{
    const PhiloxBlock b = philox4x32_10(i >> 2, key);
    const unsigned k = (unsigned)i & 3u;
    return k == 0 ? b.w[0] : k == 1 ? b.w[1] : k == 2 ? b.w[2] : b.w[3];
}

inline hipStream_t as_stream(void *s) { return reinterpret_cast<hipStream_t>(s); }

inline bool fmt_ok(lp_qfmt q)
{
    return q.n >= 2 && q.n <= 16 && q.m >= 1 && q.m <= q.n && q.f >= 0 && q.n == q.m + q.f;
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Status of the launches this call has made.  clear_stale_error() at the call's entry drops an
// error that an earlier, unrelated HIP call left pending, so that it is not reported as this
// call's.
inline void clear_stale_error() { (void)hipGetLastError(); }
inline lp_status launch_status()
{
    return hipGetLastError() == hipSuccess ? LP_OK : LP_EDEVICE;
}

} // namespace lp
