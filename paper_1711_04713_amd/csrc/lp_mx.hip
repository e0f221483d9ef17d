// HBM-bound kernels of the microscaled formats: floats to mx4 and back, activations to ckpt8 with the activation function in
// the same pass, the kept values and the activation function's gradient from them.
//
// A thread takes pieces of eight neighbouring elements; a block of 32 is four neighbouring lanes, whose largest
// magnitude meets in two lane permutations.
#include <algorithm>

#include "lp_mx.h"

namespace lp {

constexpr int kThreads = 256;
// Counting launches: few blocks, so that the atomics of a counter (12 to 14 ns each, one after the other) hide behind the streaming.
constexpr unsigned kCountThreads = 1024, kCountBlocks = 512;

struct PieceGrid {
    unsigned rows, cols, per_row, magic, total; // pieces of eight per row (a multiple of 4) and in all
};

static bool piece_grid(size_t rows, size_t cols, size_t blocks, PieceGrid *g)
{
    if (cols >= ((size_t)1 << 31) || rows >= ((size_t)1 << 31) || rows * (blocks * 4) >= ((size_t)1 << 31)) return false;
    g->rows = (unsigned)rows;
    g->cols = (unsigned)cols;
    g->per_row = (unsigned)(blocks * 4);
    g->magic = piece_magic(g->per_row);
    g->total = (unsigned)(rows * (blocks * 4));
    return true;
}

static dim3 blocks_for(const PieceGrid &g) { return dim3((g.total + kThreads - 1) / kThreads); }

// the draws of elements i .. i + 7; whole: i is a multiple of 4 in every row
__device__ __forceinline__ void draws8(uint64_t i, bool whole, uint64_t seed, uint32_t (&w)[8])
{
    if (whole) {
        const PhiloxBlock a = philox4x32_10(i >> 2, seed), b = philox4x32_10((i >> 2) + 1, seed);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = j < 4 ? a.w[j & 3] : b.w[j & 3];
    } else { // (three blocks: one a piece for each element took twice as long, 258 us for 117 M bfloat16 in rows of an odd length)
        const PhiloxBlock a = philox4x32_10(i >> 2, seed), b = philox4x32_10((i >> 2) + 1, seed), c = philox4x32_10((i >> 2) + 2, seed);
        const uint32_t all[12] = {a.w[0], a.w[1], a.w[2], a.w[3], b.w[0], b.w[1], b.w[2], b.w[3], c.w[0], c.w[1], c.w[2], c.w[3]};
        const uint32_t one = 0u - ((uint32_t)i & 1), two = 0u - ((uint32_t)i >> 1 & 1);
        uint32_t t[10];
#pragma unroll
        for (int j = 0; j < 10; ++j) t[j] = (all[j + 1] & one) | (all[j] & ~one);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = (t[j + 2] & two) | (t[j] & ~two);
    }
}

// One magnitude t >= 0 (in units of the block's scale, exact) to its code 0..8; 8 does not exist and saturates.  The
// magnitudes go in steps of 1/2 below 2, of 1 below 4 and of 2 above: with t in units of the step, the codes of a segment are
// consecutive.  (Nearest even is the hardware's own conversion, mx4_word.)
template <int MODE>
__device__ __forceinline__ int mx4_code(float t, uint32_t draw)
{
    t = fminf(t, 8.0f);
    const float u = t < 2.0f ? 2.0f * t : t < 4.0f ? t : 0.5f * t;
    const int first = t < 2.0f ? 0 : t < 4.0f ? 2 : 4;
    float r;
    if (MODE == LP_ROUND_NEAREST_AWAY) {
        r = roundf(u);
    } else {
        r = floorf(u);
        r += (double)draw < (double)(u - r) * 4294967296.0 ? 1.0f : 0.0f;
    }
    return first + (int)r;
}

template <typename T, int MODE, bool COUNT>
__global__ __launch_bounds__(COUNT ? kCountThreads : kThreads) void mx4_quantize_kernel(const T *__restrict__ x, size_t ldx, PieceGrid g, unsigned *__restrict__ codes,
                                                                unsigned char *__restrict__ scales, uint64_t seed,
                                                                unsigned long long *zero_count, unsigned long long *sat_count)
{
    constexpr unsigned THREADS = COUNT ? kCountThreads : kThreads;
    unsigned zeros = 0, sats = 0;
#pragma unroll MODE == LP_ROUND_STOCHASTIC ? 1 : 2
    for (unsigned p = blockIdx.x * THREADS + threadIdx.x; p < g.total; p += gridDim.x * THREADS) {
        unsigned row, piece;
        piece_place(p, g.per_row, g.magic, row, piece);
        const unsigned col = 8 * piece;
        const int n = (int)min(g.cols - min(col, g.cols), 8u);
        v8f v = load8(x + row * ldx + col, n);
        const int e = mx4_scale_byte(block_exponent(v));
        unsigned w = 0;
        if constexpr (MODE == LP_ROUND_NEAREST_EVEN) {
            w = mx4_word(v, e);
            if (COUNT) {
                // (elements that do not exist are zeros)
                zeros += n - __builtin_popcount(((w & 0x77777777u) + 0x77777777u) & 0x88888888u);
                const float over = 7.0f * power_of_byte(e); // rounds to 8
#pragma unroll
                for (int j = 0; j < 8; ++j) sats += fabsf(v[j]) >= over;
            }
        } else {
            const float inv = power_of_byte(254 - e);
            uint32_t draw[8] = {};
            if constexpr (MODE == LP_ROUND_STOCHASTIC) draws8((uint64_t)row * g.cols + col, (g.cols & 3) == 0, seed, draw);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float a = v[j] == v[j] ? v[j] : 0.0f;
                const int c = mx4_code<MODE>(fabsf(a) * inv, draw[j]);
                w |= ((unsigned)min(c, 7) | (__float_as_uint(a) >> 28 & 8)) << (4 * j); // (-0 too)
                if (COUNT) {
                    zeros += j < n && c == 0;
                    sats += j < n && c > 7;
                }
            }
        }
        codes[p] = w;
        if ((p & 3) == 0) scales[p >> 2] = (unsigned char)e;
    }
    if constexpr (COUNT) {
        for (int d = 32; d; d >>= 1) {
            zeros += __shfl_xor(zeros, d);
            sats += __shfl_xor(sats, d);
        }
        add_block_counts<THREADS>(zeros, sats, zero_count, sat_count);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void mx4_dequantize_kernel(const unsigned *__restrict__ codes, const unsigned char *__restrict__ scales,
                                                                  PieceGrid g, T *__restrict__ y, size_t ldy)
{
    const unsigned p = blockIdx.x * kThreads + threadIdx.x;
    if (p >= g.total) return;
    unsigned row, piece;
    piece_place(p, g.per_row, g.magic, row, piece);
    const unsigned col = 8 * piece;
    if (col >= g.cols) return;
    store8(y + row * ldy + col, (int)min(g.cols - col, 8u), mx4_values(codes[p], scales[p >> 2]));
}

template <typename T, int MODE>
__global__ __launch_bounds__(kThreads) void ckpt8_save_kernel(const T *x, size_t ldx, PieceGrid g, v2u *__restrict__ codes,
                                                              unsigned char *__restrict__ scales, uint64_t seed, lp_actfn act, T *y, size_t ldy)
{
    const unsigned p = blockIdx.x * kThreads + threadIdx.x;
    if (p >= g.total) return;
    unsigned row, piece;
    piece_place(p, g.per_row, g.magic, row, piece);
    const unsigned col = 8 * piece;
    const int n = (int)min(g.cols - min(col, g.cols), 8u);
    v8f v = load8(x + row * ldx + col, n);
    const int e = min(max(block_exponent(v), 7), 254);
    const float inv = power_of_byte(260 - e);
    uint32_t draw[8] = {};
    if constexpr (MODE == LP_ROUND_STOCHASTIC) draws8((uint64_t)row * g.cols + col, (g.cols & 3) == 0, seed, draw);
    v2u w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float t = v[j] * inv; // exact (a power of two), or so small that it is 0 in every mode
        float r;
        if (MODE == LP_ROUND_NEAREST_AWAY) {
            r = roundf(t);
        } else if (MODE == LP_ROUND_NEAREST_EVEN) {
            r = rintf(t);
        } else {
            // in double: for a negative t just below zero t - floor(t) needs more bits than float has
            const float fl = floorf(t);
            r = (double)draw[j] < ((double)t - (double)fl) * 4294967296.0 ? fl + 1.0f : fl;
        }
        if (!(t == t)) r = 0.0f;
        const int q = (int)fminf(fmaxf(r, -127.0f), 127.0f);
        w[j >> 2] |= (unsigned)(q & 255) << (8 * (j & 3));
    }
    codes[p] = w;
    if ((p & 3) == 0) scales[p >> 2] = (unsigned char)e;
    if (y) {
        store8(y + row * ldy + col, n, act_values<T>(v, act));
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void ckpt8_load_kernel(const v2u *__restrict__ codes, const unsigned char *__restrict__ scales, PieceGrid g,
                                                              T *__restrict__ y, size_t ldy)
{
    const unsigned p = blockIdx.x * kThreads + threadIdx.x;
    if (p >= g.total) return;
    unsigned row, piece;
    piece_place(p, g.per_row, g.magic, row, piece);
    const unsigned col = 8 * piece;
    if (col >= g.cols) return;
    store8(y + row * ldy + col, (int)min(g.cols - col, 8u), ckpt8_values(codes[p], scales[p >> 2]));
}

template <typename T>
__global__ __launch_bounds__(kThreads) void ckpt8_act_bwd_kernel(const v2u *__restrict__ codes, const unsigned char *__restrict__ scales, PieceGrid g,
                                                                 const T *dy, size_t lddy, lp_actfn act, T *dx, size_t lddx)
{
    const unsigned p = blockIdx.x * kThreads + threadIdx.x;
    if (p >= g.total) return;
    unsigned row, piece;
    piece_place(p, g.per_row, g.magic, row, piece);
    const unsigned col = 8 * piece;
    if (col >= g.cols) return;
    const int n = (int)min(g.cols - col, 8u);
    const v8f h = ckpt8_values(codes[p], scales[p >> 2]);
    store8(dx + row * lddx + col, n, act_gradients<T>(load8(dy + row * lddy + col, n), h, act));
}

// ---------------------------------------------------------------------------------- launches

template <typename F>
static void with_mode(lp_round r, F f)
{
    if (r == LP_ROUND_NEAREST_AWAY) f(std::integral_constant<int, LP_ROUND_NEAREST_AWAY>());
    else if (r == LP_ROUND_NEAREST_EVEN) f(std::integral_constant<int, LP_ROUND_NEAREST_EVEN>());
    else f(std::integral_constant<int, LP_ROUND_STOCHASTIC>());
}

void mx4_quantize_launch(const void *x, lp_dtype xt, size_t rows, size_t cols, size_t ldx, void *codes, void *scales, hipStream_t st)
{
    const size_t blocks = mx4_blocks(cols), most = (((size_t)1 << 31) - 1) / (blocks * 4); // rows of a launch
    for (size_t r = 0; r < rows; r += most) {
        PieceGrid g;
        if (!piece_grid(std::min(rows - r, most), cols, blocks, &g)) return; // (a row has at most 2^24 columns)
        with_type(xt, [&](auto *tag) {
            typedef std::remove_pointer_t<decltype(tag)> T;
            hipLaunchKernelGGL((mx4_quantize_kernel<T, LP_ROUND_NEAREST_EVEN, false>), blocks_for(g), dim3(kThreads), 0, st, (const T *)x + r * ldx, ldx, g,
                               (unsigned *)codes + r * blocks * 4, (unsigned char *)scales + r * blocks, (uint64_t)0, (unsigned long long *)nullptr,
                               (unsigned long long *)nullptr);
        });
    }
}

} // namespace lp

// ------------------------------------------------------------------------------------ C ABI

using namespace lp;

extern "C" lp_status lp_mx4_bytes(size_t rows, size_t cols, size_t *codes_bytes_host, size_t *scales_bytes_host)
{
    if (!codes_bytes_host || !scales_bytes_host) return LP_EINVAL;
    PieceGrid g;
    if (!piece_grid(rows, cols, mx4_blocks(cols), &g)) return LP_EUNSUPPORTED;
    *scales_bytes_host = rows * mx4_blocks(cols);
    *codes_bytes_host = *scales_bytes_host * 16;
    return LP_OK;
}

extern "C" lp_status lp_ckpt8_bytes(size_t rows, size_t cols, size_t *codes_bytes_host, size_t *scales_bytes_host)
{
    if (!codes_bytes_host || !scales_bytes_host) return LP_EINVAL;
    PieceGrid g;
    if (!piece_grid(rows, cols, ckpt8_blocks(cols), &g)) return LP_EUNSUPPORTED;
    *scales_bytes_host = rows * ckpt8_blocks(cols);
    *codes_bytes_host = *scales_bytes_host * 32;
    return LP_OK;
}

extern "C" lp_status lp_mx4_quantize(const void *x_dev, lp_dtype xt, size_t rows, size_t cols, size_t ldx, void *codes_dev,
                                     void *scales_dev, lp_round r, uint64_t seed, uint64_t *zero_count_dev,
                                     uint64_t *sat_count_dev, void *stream)
{
    if (!dtype_ok(xt) || (int)r < 0 || (int)r > 2) return LP_EINVAL;
    if (rows == 0 || cols == 0) return LP_OK;
    if (!floats_ok(x_dev, xt, cols, ldx) || !codes_dev || !aligned16(codes_dev) || !scales_dev || !aligned_to(scales_dev, 8)) return LP_EINVAL;
    if (!aligned_to(zero_count_dev, 8) || !aligned_to(sat_count_dev, 8)) return LP_EINVAL;
    PieceGrid g;
    if (!piece_grid(rows, cols, mx4_blocks(cols), &g)) return LP_EUNSUPPORTED;
    hipStream_t st = as_stream(stream);
    clear_stale_error();
    const bool count = zero_count_dev || sat_count_dev;
    with_type(xt, [&](auto *tag) {
        typedef std::remove_pointer_t<decltype(tag)> T;
        with_mode(r, [&](auto mode) {
            constexpr int MODE = decltype(mode)::value;
            const dim3 grid = count ? dim3(std::min((g.total + kCountThreads - 1) / kCountThreads, kCountBlocks)) : blocks_for(g);
            hipLaunchKernelGGL((count ? mx4_quantize_kernel<T, MODE, true> : mx4_quantize_kernel<T, MODE, false>), grid, dim3(count ? kCountThreads : kThreads), 0, st,
                               (const T *)x_dev, ldx, g, (unsigned *)codes_dev, (unsigned char *)scales_dev, seed,
                               (unsigned long long *)zero_count_dev, (unsigned long long *)sat_count_dev);
        });
    });
    return launch_status();
}

extern "C" lp_status lp_mx4_dequantize(const void *codes_dev, const void *scales_dev, size_t rows, size_t cols, void *y_dev,
                                       lp_dtype yt, size_t ldy, void *stream)
{
    if (!dtype_ok(yt)) return LP_EINVAL;
    if (rows == 0 || cols == 0) return LP_OK;
    if (!floats_ok(y_dev, yt, cols, ldy) || !codes_dev || !aligned16(codes_dev) || !scales_dev || !aligned_to(scales_dev, 8)) return LP_EINVAL;
    PieceGrid g;
    if (!piece_grid(rows, cols, mx4_blocks(cols), &g)) return LP_EUNSUPPORTED;
    clear_stale_error();
    with_type(yt, [&](auto *tag) {
        typedef std::remove_pointer_t<decltype(tag)> T;
        hipLaunchKernelGGL(mx4_dequantize_kernel<T>, blocks_for(g), dim3(kThreads), 0, as_stream(stream), (const unsigned *)codes_dev,
                           (const unsigned char *)scales_dev, g, (T *)y_dev, ldy);
    });
    return launch_status();
}

extern "C" lp_status lp_ckpt8_save(const void *x_dev, lp_dtype xt, size_t rows, size_t cols, size_t ldx, void *codes_dev,
                                   void *scales_dev, lp_round r, uint64_t seed, lp_actfn act, void *y_dev, size_t ldy,
                                   void *stream)
{
    if (!dtype_ok(xt) || (int)r < 0 || (int)r > 2 || !actfn_ok(act)) return LP_EINVAL;
    if (rows == 0 || cols == 0) return LP_OK;
    if (!floats_ok(x_dev, xt, cols, ldx) || !codes_dev || !aligned16(codes_dev) || !scales_dev) return LP_EINVAL;
    if (y_dev && (!floats_ok(y_dev, xt, cols, ldy) || (y_dev == x_dev && ldy != ldx))) return LP_EINVAL;
    PieceGrid g;
    if (!piece_grid(rows, cols, ckpt8_blocks(cols), &g)) return LP_EUNSUPPORTED;
    clear_stale_error();
    with_type(xt, [&](auto *tag) {
        typedef std::remove_pointer_t<decltype(tag)> T;
        with_mode(r, [&](auto mode) {
            hipLaunchKernelGGL((ckpt8_save_kernel<T, decltype(mode)::value>), blocks_for(g), dim3(kThreads), 0, as_stream(stream), (const T *)x_dev, ldx,
                               g, (v2u *)codes_dev, (unsigned char *)scales_dev, seed, act, (T *)y_dev, ldy);
        });
    });
    return launch_status();
}

extern "C" lp_status lp_ckpt8_load(const void *codes_dev, const void *scales_dev, size_t rows, size_t cols, void *y_dev,
                                   lp_dtype yt, size_t ldy, void *stream)
{
    if (!dtype_ok(yt)) return LP_EINVAL;
    if (rows == 0 || cols == 0) return LP_OK;
    if (!floats_ok(y_dev, yt, cols, ldy) || !codes_dev || !aligned16(codes_dev) || !scales_dev) return LP_EINVAL;
    PieceGrid g;
    if (!piece_grid(rows, cols, ckpt8_blocks(cols), &g)) return LP_EUNSUPPORTED;
    clear_stale_error();
    with_type(yt, [&](auto *tag) {
        typedef std::remove_pointer_t<decltype(tag)> T;
        hipLaunchKernelGGL(ckpt8_load_kernel<T>, blocks_for(g), dim3(kThreads), 0, as_stream(stream), (const v2u *)codes_dev,
                           (const unsigned char *)scales_dev, g, (T *)y_dev, ldy);
    });
    return launch_status();
}

extern "C" lp_status lp_ckpt8_act_bwd(const void *codes_dev, const void *scales_dev, size_t rows, size_t cols, const void *dy_dev,
                                      lp_dtype t, size_t lddy, lp_actfn act, void *dx_dev, size_t lddx, void *stream)
{
    if (!dtype_ok(t) || !actfn_ok(act)) return LP_EINVAL;
    if (rows == 0 || cols == 0) return LP_OK;
    if (!floats_ok(dy_dev, t, cols, lddy) || !floats_ok(dx_dev, t, cols, lddx) || (dx_dev == dy_dev && lddx != lddy)) return LP_EINVAL;
    if (!codes_dev || !aligned16(codes_dev) || !scales_dev) return LP_EINVAL;
    PieceGrid g;
    if (!piece_grid(rows, cols, ckpt8_blocks(cols), &g)) return LP_EUNSUPPORTED;
    clear_stale_error();
    with_type(t, [&](auto *tag) {
        typedef std::remove_pointer_t<decltype(tag)> T;
        hipLaunchKernelGGL(ckpt8_act_bwd_kernel<T>, blocks_for(g), dim3(kThreads), 0, as_stream(stream), (const v2u *)codes_dev,
                           (const unsigned char *)scales_dev, g, (const T *)dy_dev, lddy, act, (T *)dx_dev, lddx);
    });
    return launch_status();
}
