// The inner products of the microscaled formats: mx4 times mx4 (forward), bfloat16 times mx4 (gradient of the
// input) and bfloat16 times ckpt8 (gradient of the weights).
//
//     C[i][j] = sum_c A(i, c) * B(c, j)
#include <algorithm>

#include "lp_mx.h"

namespace lp {

constexpr int PT = 64;  // rows and columns of a tile
constexpr int PC = 16;  // positions of the reduction per step

struct Mx4Rows { // element (row, pos) of an mx4 tensor
    const unsigned char *codes, *scales;
    size_t blocks;
    __device__ float at(int row, int pos) const
    {
        const int code = codes[(size_t)row * blocks * 16 + (pos >> 1)] >> (4 * (pos & 1)) & 15;
        const int e = code >> 1 & 3, m = code & 1;
        const float v = e ? (float)((2 + m) << (e - 1)) * 0.5f : 0.5f * m;
        return (code & 8 ? -v : v) * power_of_byte(scales[(size_t)row * blocks + (pos >> 5)]);
    }
};
struct Ckpt8Rows {
    const signed char *codes;
    const unsigned char *scales;
    size_t blocks;
    __device__ float at(int row, int pos) const
    {
        return (float)codes[(size_t)row * blocks * 32 + pos] * power_of_byte(scales[(size_t)row * blocks + (pos >> 5)] - 6);
    }
};
struct Bf16Rows {
    const __bf16 *p;
    size_t ld;
    __device__ float at(int row, int pos) const { return (float)p[(size_t)row * ld + pos]; }
};

struct Output {
    void *y;
    lp_dtype t;
    size_t ld;
    const float *bias;
    lp_actfn act;
    int accumulate;
    __device__ void put(int i, int j, float v) const
    {
        const size_t at = (size_t)i * ld + j;
        if (bias) v += bias[j];
        if (accumulate) v += t == LP_F32 ? ((float *)y)[at] : (float)((__bf16 *)y)[at];
        v = act_value(v, act);
        if (t == LP_F32) ((float *)y)[at] = v;
        else if (t == LP_BF16) ((__bf16 *)y)[at] = (__bf16)v;
        else ((_Float16 *)y)[at] = (_Float16)v;
    }
};

// A(i, c): a.at(i, c), or a.at(c, i) where the reduction runs over a's rows; B(c, j) likewise: b.at(j, c) or b.at(c, j).
template <bool A_BY_POS, bool B_BY_POS, typename A, typename B>
__global__ __launch_bounds__(256) void product_kernel(A a, B b, Output out, int I, int J, int C)
{
    __shared__ float ta[PC][PT + 1], tb[PC][PT + 1];
    const int tiles_i = (I + PT - 1) / PT, i0 = blockIdx.x % tiles_i * PT, j0 = blockIdx.x / tiles_i * PT, ti = threadIdx.x & 15, tj = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int c0 = 0; c0 < C; c0 += PC) {
        for (int k = threadIdx.x; k < PC * PT; k += 256) {
            const int ac = A_BY_POS ? k / PT : k % PC, ai = A_BY_POS ? k % PT : k / PC;
            ta[ac][ai] = i0 + ai < I && c0 + ac < C ? (A_BY_POS ? a.at(c0 + ac, i0 + ai) : a.at(i0 + ai, c0 + ac)) : 0.0f;
            const int bc = B_BY_POS ? k / PT : k % PC, bj = B_BY_POS ? k % PT : k / PC;
            tb[bc][bj] = j0 + bj < J && c0 + bc < C ? (B_BY_POS ? b.at(c0 + bc, j0 + bj) : b.at(j0 + bj, c0 + bc)) : 0.0f;
        }
        __syncthreads();
        for (int c = 0; c < PC; ++c)
            for (int u = 0; u < 4; ++u)
                for (int v = 0; v < 4; ++v) acc[u][v] += ta[c][ti + 16 * u] * tb[c][tj * 4 + v];
        __syncthreads();
    }
    for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v) {
            const int i = i0 + ti + 16 * u, j = j0 + tj * 4 + v;
            if (i < I && j < J) out.put(i, j, acc[u][v]);
        }
}

// dbias[j] (+)= sum over the rows of dY
__global__ __launch_bounds__(256) void column_sums_kernel(Bf16Rows dy, int M, int N, float *out, int accumulate)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= N) return;
    float s = 0.0f;
    for (int m = 0; m < M; ++m) s += dy.at(m, j);
    out[j] = accumulate ? out[j] + s : s;
}

static dim3 product_grid(int I, int J) { return dim3((unsigned)((I + PT - 1) / PT) * (unsigned)((J + PT - 1) / PT)); }

static bool sizes_ok(int M, int K, int Nout) { return M >= 0 && K > 0 && Nout > 0; }
static bool sizes_taken(int M, int K, int Nout) { return M <= (1 << 24) && K <= (1 << 24) && Nout <= (1 << 24); }

static bool mx4_ok(const void *codes, const void *scales) { return codes && aligned16(codes) && scales && aligned_to(scales, 8); }
static bool floats_ok(const void *p, lp_dtype t, size_t cols, size_t ld) { return p && aligned_to(p, dtype_size(t)) && ld >= cols; }

static size_t fwd_workspace(int M, int K, int Nout)
{
    const size_t blocks = (size_t)M * mx4_blocks((size_t)K);
    return (blocks * 17 + 255) / 256 * 256;
}

} // namespace lp

// ------------------------------------------------------------------------------------ C ABI

using namespace lp;

extern "C" lp_status lp_mx4_fc_workspace_bytes(int M, int K, int Nout, size_t *bytes_host)
{
    if (!bytes_host || !sizes_ok(M, K, Nout)) return LP_EINVAL;
    if (!sizes_taken(M, K, Nout)) return LP_EUNSUPPORTED;
    *bytes_host = fwd_workspace(M, K, Nout);
    return LP_OK;
}

extern "C" lp_status lp_mx4_fc_fwd(int M, int K, int Nout, const void *x_dev, lp_dtype xt, size_t ldx, const void *x_scales_dev,
                                   const void *w_codes_dev, const void *w_scales_dev, const float *bias_dev, void *y_dev,
                                   lp_dtype yt, size_t ldy, lp_actfn act, void *workspace_dev, size_t workspace_bytes,
                                   void *stream)
{
    if (!sizes_ok(M, K, Nout) || !dtype_ok(yt) || !actfn_ok(act) || (!x_scales_dev && !dtype_ok(xt))) return LP_EINVAL;
    if (!sizes_taken(M, K, Nout)) return LP_EUNSUPPORTED;
    if (M == 0) return LP_OK;
    if (x_scales_dev ? !mx4_ok(x_dev, x_scales_dev) : !floats_ok(x_dev, xt, (size_t)K, ldx)) return LP_EINVAL;
    if (!mx4_ok(w_codes_dev, w_scales_dev) || !floats_ok(y_dev, yt, (size_t)Nout, ldy) || !aligned_to(bias_dev, 4)) return LP_EINVAL;
    const size_t need = fwd_workspace(M, K, Nout);
    if (need && (!workspace_dev || workspace_bytes < need)) return LP_EWORKSPACE;
    if (need && !aligned16(workspace_dev)) return LP_EINVAL;
    hipStream_t st = as_stream(stream);
    clear_stale_error();
    const size_t blocks = mx4_blocks((size_t)K);
    const unsigned char *xc = (const unsigned char *)x_dev, *xs = (const unsigned char *)x_scales_dev;
    if (!xs) {
        unsigned char *w = (unsigned char *)workspace_dev;
        mx4_quantize_launch(x_dev, xt, (size_t)M, (size_t)K, ldx, w, w + (size_t)M * blocks * 16, st);
        xc = w;
        xs = w + (size_t)M * blocks * 16;
    }
    const Mx4Rows a{xc, xs, blocks}, b{(const unsigned char *)w_codes_dev, (const unsigned char *)w_scales_dev, blocks};
    hipLaunchKernelGGL((product_kernel<false, false, Mx4Rows, Mx4Rows>), product_grid(M, Nout), dim3(256), 0, st, a, b,
                       Output{y_dev, yt, ldy, bias_dev, act, 0}, M, Nout, K);
    return launch_status();
}

extern "C" lp_status lp_mx4_fc_dgrad_workspace_bytes(int M, int K, int Nout, size_t *bytes_host)
{
    if (!bytes_host || !sizes_ok(M, K, Nout)) return LP_EINVAL;
    if (!sizes_taken(M, K, Nout)) return LP_EUNSUPPORTED;
    *bytes_host = 0;
    return LP_OK;
}

extern "C" lp_status lp_mx4_fc_dgrad(int M, int K, int Nout, const void *dy_dev, size_t lddy, const void *w_codes_dev,
                                     const void *w_scales_dev, void *dx_dev, lp_dtype dxt, size_t lddx, void *workspace_dev,
                                     size_t workspace_bytes, void *stream)
{
    if (!sizes_ok(M, K, Nout) || !dtype_ok(dxt)) return LP_EINVAL;
    if (!sizes_taken(M, K, Nout) || dxt == LP_F16) return LP_EUNSUPPORTED;
    if (M == 0) return LP_OK;
    if (!floats_ok(dy_dev, LP_BF16, (size_t)Nout, lddy) || !mx4_ok(w_codes_dev, w_scales_dev) || !floats_ok(dx_dev, dxt, (size_t)K, lddx)) return LP_EINVAL;
    clear_stale_error();
    const Bf16Rows a{(const __bf16 *)dy_dev, lddy};
    const Mx4Rows b{(const unsigned char *)w_codes_dev, (const unsigned char *)w_scales_dev, mx4_blocks((size_t)K)};
    hipLaunchKernelGGL((product_kernel<false, true, Bf16Rows, Mx4Rows>), product_grid(M, K), dim3(256), 0, as_stream(stream), a, b,
                       Output{dx_dev, dxt, lddx, nullptr, LP_ACT_NONE, 0}, M, K, Nout);
    return launch_status();
}

extern "C" lp_status lp_ckpt8_fc_wgrad_workspace_bytes(int M, int K, int Nout, size_t *bytes_host)
{
    if (!bytes_host || !sizes_ok(M, K, Nout)) return LP_EINVAL;
    if (!sizes_taken(M, K, Nout)) return LP_EUNSUPPORTED;
    *bytes_host = 0;
    return LP_OK;
}

extern "C" lp_status lp_ckpt8_fc_wgrad(int M, int K, int Nout, const void *dy_dev, size_t lddy, const void *x_codes_dev,
                                       const void *x_scales_dev, void *dw_dev, lp_dtype dwt, size_t lddw, float *dbias_dev,
                                       int accumulate, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    if (!sizes_ok(M, K, Nout) || !dtype_ok(dwt)) return LP_EINVAL;
    if (!sizes_taken(M, K, Nout) || dwt == LP_F16) return LP_EUNSUPPORTED;
    if (M && (!floats_ok(dy_dev, LP_BF16, (size_t)Nout, lddy) || !x_codes_dev || !aligned16(x_codes_dev) || !x_scales_dev)) return LP_EINVAL;
    if (!floats_ok(dw_dev, dwt, (size_t)K, lddw) || !aligned_to(dbias_dev, 4)) return LP_EINVAL;
    hipStream_t st = as_stream(stream);
    clear_stale_error();
    const Bf16Rows a{(const __bf16 *)dy_dev, lddy};
    const Ckpt8Rows b{(const signed char *)x_codes_dev, (const unsigned char *)x_scales_dev, ckpt8_blocks((size_t)K)};
    hipLaunchKernelGGL((product_kernel<true, true, Bf16Rows, Ckpt8Rows>), product_grid(Nout, K), dim3(256), 0, st, a, b,
                       Output{dw_dev, dwt, lddw, nullptr, LP_ACT_NONE, accumulate != 0}, Nout, K, M);
    if (dbias_dev) hipLaunchKernelGGL(column_sums_kernel, dim3((Nout + 255) / 256), dim3(256), 0, st, a, M, Nout, dbias_dev, accumulate != 0);
    return launch_status();
}
