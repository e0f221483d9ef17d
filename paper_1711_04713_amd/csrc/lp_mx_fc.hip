// The inner products of the microscaled formats: mx4 times mx4 (forward), bfloat16 times mx4 (gradient of the
// input) and bfloat16 times ckpt8 (gradient of the weights).
//
//     C[i][j] = sum_c A(i, c) * B(c, j)
#include <algorithm>
#include <type_traits>

#include "lp_mx.h"

namespace lp {

constexpr int kCUs = 256;
constexpr int kXCDs = 8;

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void *LdsPtr;

// 16 bytes per lane from memory to LDS without a register: lane l's land at to + 16 l.  (A function of its own: the host
// pass does not know the builtin's width.)
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t from, unsigned char *to, unsigned lane_offset, int offset)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (LdsPtr)to, 16, lane_offset, offset, 0, 0);
}
__device__ __forceinline__ void load_lds4(__amdgpu_buffer_rsrc_t from, unsigned char *to, unsigned lane_offset, int offset)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (LdsPtr)to, 4, lane_offset, offset, 0, 0);
}

// -------------------------------------------------------------------------------- results

// Where a product's sums go: out[i][j] = act(sum + bias[j]), rounded once.  A product that is cut along its reduction
// writes 32-bit sums of its parts to the workspace in the same way (no bias, no function), part p `part` elements further.
struct Sink {
    void *y;
    size_t ld, part;
    const float *bias;
    lp_actfn act;
};

// y = act(sum of the parts + bias): a thread takes eight neighbours of a row
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(const float *__restrict__ parts, int count, size_t part, size_t ldp, T *__restrict__ y, size_t ldy,
                                                         int I, int J, unsigned per_row, unsigned magic, unsigned total, const float *__restrict__ bias,
                                                         lp_actfn act)
{
    const unsigned p = blockIdx.x * 256 + threadIdx.x;
    if (p >= total) return;
    unsigned row, piece;
    piece_place(p, per_row, magic, row, piece);
    const int j = 8 * (int)piece, n = min(J - j, 8);
    const float *q = parts + row * ldp + j; // (rows of the parts are whole pieces)
    v8f v = load8(q, 8);
    for (int k = 1; k < count; ++k) v += load8(q + k * part, 8);
    if (bias) v += load8(bias + j, n);
    store8(y + row * ldy + j, n, act_values(v, act));
}

// ------------------------------------------------------------------------------- mx4 times mx4

// y[m][n] = sum_k x[m][k] w[n][k] on v_mfma_scale_f32_32x32x64_f8f6f4, whose lane takes one block of 32 neighbours of a row
// (16 bytes of codes) and that block's scale byte.
//
// A workgroup owns TM rows of x times TN rows of w, one wave MB x NB blocks of 32 x 32; two waves per SIMD, so that the
// one's reads and address arithmetic hide behind the other's products.  A stage is 256 positions: 128 bytes of each row (a
// whole cache line: 64 bytes of twice as many rows come at 54 GB/s a CU instead of 90), brought to LDS by loads that do not
// pass through registers, into one of two buffers; one stage is on its way while the other is multiplied.  16-byte piece p
// of row r lies at place p ^ (r % 8) of the row, so that the eight rows that a read takes together lie in different banks.
// Within a stage the order of the reduction is free as long as both sides share it: in step s (of four) the lower half of
// the lanes takes block s, the upper half block 4 + s, so that a lane's scale bytes of a stage are one word.  Scale bytes
// come the same way, those of four stages at a time.
//
// Weights are the row operand: a lane ends up with four neighbouring columns of one row of y.
struct Mx4Args {
    const unsigned char *xc, *xs, *wc, *ws;
    int M, N, blocks, stages, stages_per_part, tiles_m, tiles_n, parts, work, per_xcd; // stages_per_part: a multiple of 4
    Sink out;
};

constexpr int kTileGroup = 4; // row tiles that are walked together: 32 workgroups of a die share 4 x 8 tiles

template <int MB, int NB, int WM, int WN, typename OutT>
__global__ __launch_bounds__(WM *WN * 64, 2) void mx4_product_kernel(const Mx4Args a)
{
    constexpr int TM = MB * 32 * WM, TN = NB * 32 * WN, WAVES = WM * WN, ROWS = TM + TN, STAGE = ROWS * 128, PER = ROWS / 8 / WAVES;
    constexpr int SROWS = ROWS / WAVES, SPER = SROWS / 32; // rows whose scale bytes a wave brings, loads that takes
    static_assert(TM % SROWS == 0, "of one tensor");
    constexpr int OUTROW = NB * 32 + 4; // a wave's row of results in LDS, floats, padded
    constexpr int OUTWAVE = 32 * OUTROW * 4;
    // (the scale bytes of a row's stages that do not exist are read too, from whatever follows: 32 bytes more)
    __shared__ __align__(1024) unsigned char lds[2 * STAGE + ROWS * 32 + 32];
    static_assert(WAVES * OUTWAVE <= (int)sizeof(lds), "results pass through the same memory");
    // work item: consecutive workgroups go round the dies, each die has a run of consecutive items
    const int item = (blockIdx.x % kXCDs) * a.per_xcd + blockIdx.x / kXCDs;
    if (item >= a.work) return;
    // (divisions run on the vector unit: what comes back is said to be the same in all lanes)
    const int tiles = a.tiles_m * a.tiles_n, part = __builtin_amdgcn_readfirstlane(item / tiles), tile = item - part * tiles;
    const int group = __builtin_amdgcn_readfirstlane(tile / (kTileGroup * a.tiles_n)), in_group = tile - group * kTileGroup * a.tiles_n;
    const int rows = min(kTileGroup, a.tiles_m - group * kTileGroup), tile_n = __builtin_amdgcn_readfirstlane(in_group / rows);
    const int m0 = (group * kTileGroup + in_group - tile_n * rows) * TM, n0 = tile_n * TN;
    const int first = part * a.stages_per_part, last = min(a.stages, first + a.stages_per_part);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h = lane >> 5, wm = wave % WM, wn = wave / WM;
    const size_t pitch = (size_t)a.blocks * 16;
    // place of tile row r (x's rows, then w's) among its tensor's rows; rows beyond the last are read as the last one and not stored
    auto row_of = [&](int r) __attribute__((always_inline)) { return (unsigned)(r < TM ? min(r, a.M - 1 - m0) : min(r - TM, a.N - 1 - n0)); };
    unsigned at[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = (wave * PER + i) * 8 + lane / 8;
        at[i] = row_of(r) * (unsigned)pitch + ((lane & 7) ^ (r & 7)) * 16;
    }
    // loads FROM .. TO - 1 of a wave's share of stage t
    auto stage = [&](int t, int buf, auto from, auto to) __attribute__((always_inline)) {
        // (behind the last stage the descriptors are empty: the loads touch no memory)
        const int size = __builtin_amdgcn_readfirstlane(t < last ? -1 : 0);
        const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.xc) + m0 * pitch, 0, size, 0x00020000);
        const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.wc) + n0 * pitch, 0, size, 0x00020000);
#pragma unroll
        for (int i = decltype(from)::value; i < decltype(to)::value; ++i) {
            unsigned char *place = lds + buf * STAGE + (wave * PER + i) * 1024;
            if ((wave * PER + i) * 8 < TM) load_lds16(xr, place, at[i], t * 128);
            else load_lds16(wr, place, at[i], t * 128);
        }
    };
    constexpr std::integral_constant<int, 0> L0;
    constexpr std::integral_constant<int, 3 * PER / 8> L1;
    constexpr std::integral_constant<int, 6 * PER / 8> L2;
    constexpr std::integral_constant<int, PER> L3;
    // Scale bytes of stages t .. t + 3 (t a multiple of 4), 32 for each row, two lanes a row; where a row ends before that its last
    // 32.  Rows of fewer than 32 come a word a lane: the rows' eight bytes of the first stage, then those of the next.
    unsigned char *const scales = lds + 2 * STAGE;
    const bool narrow = a.blocks < 32;
    const int row_step = narrow ? 8 : 32, stage_step = narrow ? ROWS * 8 : 8;
    auto scales_of = [&](int size) __attribute__((always_inline)) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(wave * SROWS < TM ? a.xs + (size_t)m0 * a.blocks : a.ws + (size_t)n0 * a.blocks), 0,
                                                 size, 0x00020000);
    };
    unsigned scale_at[SPER];
#pragma unroll
    for (int i = 0; i < SPER; ++i) scale_at[i] = row_of(wave * SROWS + i * 32 + lane / 2) * (unsigned)a.blocks + (lane & 1) * 16;
    auto load_scales = [&](int t) __attribute__((always_inline)) {
        const __amdgpu_buffer_rsrc_t from = scales_of(__builtin_amdgcn_readfirstlane(t < last ? -1 : 0));
#pragma unroll
        for (int i = 0; i < SPER; ++i) load_lds16(from, scales + wave * SROWS * 32 + i * 1024, scale_at[i], min(8 * t, a.blocks - 32));
    };
    auto load_narrow_scales = [&]() __attribute__((always_inline)) {
        const __amdgpu_buffer_rsrc_t from = scales_of(-1);
        for (int q = 0; q < a.stages; ++q)
#pragma unroll
            for (int i = 0; i < SPER; ++i)
                load_lds4(from, scales + q * ROWS * 8 + wave * SROWS * 8 + i * 256, row_of(wave * SROWS + i * 32 + lane / 2) * (unsigned)a.blocks + 4 * (lane & 1), 8 * q);
    };
    int xscale[4][MB], wscale[4][NB];
    auto take_scales = [&](int t) __attribute__((always_inline)) {
        const int moved = narrow ? 0 : max(8 * t - (a.blocks - 32), 0);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const unsigned char *from = scales + moved + 4 * h + q * stage_step;
#pragma unroll
            for (int i = 0; i < MB; ++i) xscale[q][i] = *(const int *)(from + ((wm * MB + i) * 32 + l32) * row_step);
#pragma unroll
            for (int i = 0; i < NB; ++i) wscale[q][i] = *(const int *)(from + (TM + (wn * NB + i) * 32 + l32) * row_step);
        }
    };
    v16f acc[NB][MB] = {};
    v4i fx[2][MB], fw[2][NB];
    const unsigned char *xl = lds + (wm * MB * 32 + l32) * 128, *wl = lds + (TM + wn * NB * 32 + l32) * 128;
    auto fragments = [&](int buf, int s) __attribute__((always_inline)) {
        const int o = buf * STAGE + ((4 * h + s) ^ (l32 & 7)) * 16;
#pragma unroll
        for (int i = 0; i < MB; ++i) fx[s & 1][i] = *(const v4i *)(xl + i * 4096 + o);
#pragma unroll
        for (int i = 0; i < NB; ++i) fw[s & 1][i] = *(const v4i *)(wl + i * 4096 + o);
    };
    // step S of the four-stage's stage Q (constants: the scale byte is chosen by the instruction), with the reads for the next
    // step and a few of the loads between its products
#define LP_STEP(Q, S, LOADS)                                                                                                                \
    _Pragma("unroll") for (int j = 0; j < NB; ++j) _Pragma("unroll") for (int i = 0; i < MB; ++i)                                            \
    {                                                                                                                                       \
        const v4i &wf = fw[S & 1][j], &xf = fx[S & 1][i];                                                                                   \
        const v8i w = {wf[0], wf[1], wf[2], wf[3], 0, 0, 0, 0}, x = {xf[0], xf[1], xf[2], xf[3], 0, 0, 0, 0};                               \
        acc[j][i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, acc[j][i], 4, 4, S, wscale[Q][j], S, xscale[Q][i]);               \
    }                                                                                                                                       \
    _Pragma("unroll") for (int q = 0; q < MB * NB; ++q)                                                                                      \
    {                                                                                                                                       \
        if (q < MB + NB) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                                                                 \
        if (LOADS && q % 2 == 1) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);                                                         \
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                                                                  \
    }                                                                                                                                       \
    __builtin_amdgcn_sched_barrier(0);
    // Stage t, number Q of its four.  At its last step the next stage has arrived in every wave, its own buffer is free and the
    // stage after that is asked for, over three steps: 64 loads at once take the address unit so long that every wave waits
    // for its turn.  At the first one's the scale bytes are in registers and the next four's are asked for.
    auto whole_stage = [&](int t, auto number) __attribute__((always_inline)) {
        constexpr int Q = decltype(number)::value, B = Q & 1;
        __builtin_amdgcn_sched_barrier(0);
        fragments(B, 1);
        stage(t + 1, B ^ 1, L1, L2);
        LP_STEP(Q, 0, true)
        fragments(B, 2);
        stage(t + 1, B ^ 1, L2, L3);
        LP_STEP(Q, 1, true)
        fragments(B, 3);
        LP_STEP(Q, 2, false)
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_s_barrier();
        fragments(B ^ 1, 0);
        stage(t + 2, B, L0, L1);
        if (Q == 0) load_scales(t + 4);
        LP_STEP(Q, 3, true)
    };
#undef LP_STEP
    if (narrow) load_narrow_scales();
    else load_scales(first);
    stage(first, 0, L0, L3);
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    stage(first + 1, 1, L0, L1);
    fragments(0, 0);
    for (int t = first;; t += 4) {
        take_scales(t);
        whole_stage(t, std::integral_constant<int, 0>());
        if (t + 1 >= last) break;
        whole_stage(t + 1, std::integral_constant<int, 1>());
        if (t + 2 >= last) break;
        whole_stage(t + 2, std::integral_constant<int, 2>());
        if (t + 3 >= last) break;
        whole_stage(t + 3, std::integral_constant<int, 3>());
        if (t + 4 >= last) break;
    }
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    // Results: 32 rows at a time through the wave's own piece of LDS, so that they leave as whole rows, eight neighbours a lane.
    float *mine = (float *)(lds + wave * OUTWAVE);
    OutT *y = (OutT *)a.out.y + part * a.out.part;
    const int nw = n0 + wn * NB * 32;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int mw = m0 + (wm * MB + i) * 32;
        if (mw >= a.M) break;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const v16f &c = acc[j][i];
                *(v4f *)(mine + l32 * OUTROW + j * 32 + 8 * g + 4 * h) = v4f{c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll 2
        for (int q = 0; q < 2 * NB; ++q) {
            const int k = q * 64 + lane, row = k / (NB * 4), col = k % (NB * 4) * 8;
            const v4f lo = *(const v4f *)(mine + row * OUTROW + col), hi = *(const v4f *)(mine + row * OUTROW + col + 4);
            v8f v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            const int m = mw + row, n = nw + col;
            if (m < a.M && n < a.N) {
                if (a.out.bias) v += load8(a.out.bias + n, a.N - n);
                store8(y + m * a.out.ld + n, a.N - n, act_values(v, a.out.act));
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// -------------------------------------------------------------------------------- gradients

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

static size_t round256(size_t v) { return (v + 255) / 256 * 256; }

struct Mx4Plan {
    bool large;                 // tiles of 256 x 256, else 128 x 128
    int tiles_m, tiles_n, stages, parts, stages_per_part;
    size_t blocks, ldp;         // blocks of 32 per row; row length of the parts' sums
    size_t codes, scales, sums; // workspace: quantized x (if the call brings floats), sums of the parts
    size_t total() const { return codes + scales + sums; }
};

static Mx4Plan mx4_plan(int M, int K, int Nout)
{
    Mx4Plan p = {};
    p.blocks = mx4_blocks((size_t)K);
    p.stages = (int)(p.blocks / 8);
    const auto tiles = [&](int side) { return ((size_t)M + side - 1) / side * (((size_t)Nout + side - 1) / side); };
    p.large = tiles(256) >= 192;
    const int side = p.large ? 256 : 128;
    p.tiles_m = (M + side - 1) / side;
    p.tiles_n = (Nout + side - 1) / side;
    p.parts = 1;
    if (!p.large) p.parts = (int)std::min<size_t>(std::max<size_t>(2 * kCUs / std::max<size_t>(tiles(side), 1), 1), (size_t)std::max(p.stages / 4, 1));
    p.stages_per_part = ((p.stages + p.parts - 1) / p.parts + 3) / 4 * 4;
    p.parts = (p.stages + p.stages_per_part - 1) / p.stages_per_part;
    p.ldp = ((size_t)Nout + 7) / 8 * 8;
    p.codes = round256((size_t)M * p.blocks * 16);
    p.scales = round256((size_t)M * p.blocks);
    p.sums = p.parts > 1 ? round256((size_t)p.parts * M * p.ldp * 4) : 0;
    return p;
}

template <typename T>
static void mx4_launch_tiles(const Mx4Plan &p, Mx4Args a, hipStream_t st)
{
    a.tiles_m = p.tiles_m;
    a.tiles_n = p.tiles_n;
    a.stages = p.stages;
    a.stages_per_part = p.stages_per_part;
    a.parts = p.parts;
    a.work = p.tiles_m * p.tiles_n * p.parts;
    a.per_xcd = (a.work + kXCDs - 1) / kXCDs;
    const dim3 grid((unsigned)a.per_xcd * kXCDs);
    if (p.large) hipLaunchKernelGGL((mx4_product_kernel<4, 2, 2, 4, T>), grid, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((mx4_product_kernel<2, 2, 2, 2, T>), grid, dim3(256), 0, st, a);
}

// f(type tag) for the element type of t
template <typename F>
static void with_type(lp_dtype t, F f)
{
    if (t == LP_F32) f((float *)nullptr);
    else if (t == LP_BF16) f((__bf16 *)nullptr);
    else f((_Float16 *)nullptr);
}

// y = act(sum of the parts + bias)
static void join_parts(const float *sums, int parts, size_t part, size_t ldp, void *y, lp_dtype yt, size_t ldy, int I, int J, const float *bias, lp_actfn act,
                       hipStream_t st)
{
    const unsigned per_row = (unsigned)(ldp / 8), total = per_row * (unsigned)I;
    with_type(yt, [&](auto *tag) {
        typedef std::remove_pointer_t<decltype(tag)> T;
        hipLaunchKernelGGL(join_parts_kernel<T>, dim3((total + 255) / 256), dim3(256), 0, st, sums, parts, part, ldp, (T *)y, ldy, I, J, per_row,
                           piece_magic(per_row), total, bias, act);
    });
}

} // namespace lp

// ------------------------------------------------------------------------------------ C ABI

using namespace lp;

extern "C" lp_status lp_mx4_fc_workspace_bytes(int M, int K, int Nout, size_t *bytes_host)
{
    if (!bytes_host || !sizes_ok(M, K, Nout)) return LP_EINVAL;
    if (!sizes_taken(M, K, Nout)) return LP_EUNSUPPORTED;
    *bytes_host = mx4_plan(M, K, Nout).total();
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
    const Mx4Plan p = mx4_plan(M, K, Nout);
    if (p.total() && (!workspace_dev || workspace_bytes < p.total())) return LP_EWORKSPACE;
    if (p.total() && !aligned16(workspace_dev)) return LP_EINVAL;
    hipStream_t st = as_stream(stream);
    clear_stale_error();
    unsigned char *work = (unsigned char *)workspace_dev;
    Mx4Args a = {};
    a.xc = (const unsigned char *)x_dev;
    a.xs = (const unsigned char *)x_scales_dev;
    a.wc = (const unsigned char *)w_codes_dev;
    a.ws = (const unsigned char *)w_scales_dev;
    a.M = M;
    a.N = Nout;
    a.blocks = (int)p.blocks;
    if (!a.xs) {
        mx4_quantize_launch(x_dev, xt, (size_t)M, (size_t)K, ldx, work, work + p.codes, st);
        a.xc = work;
        a.xs = work + p.codes;
    }
    if (p.parts > 1) {
        float *sums = (float *)(work + p.codes + p.scales);
        const size_t part = (size_t)M * p.ldp;
        a.out = Sink{sums, p.ldp, part, nullptr, LP_ACT_NONE};
        mx4_launch_tiles<float>(p, a, st);
        join_parts(sums, p.parts, part, p.ldp, y_dev, yt, ldy, M, Nout, bias_dev, act, st);
    } else {
        a.out = Sink{y_dev, ldy, 0, bias_dev, act};
        with_type(yt, [&](auto *tag) { mx4_launch_tiles<std::remove_pointer_t<decltype(tag)>>(p, a, st); });
    }
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
