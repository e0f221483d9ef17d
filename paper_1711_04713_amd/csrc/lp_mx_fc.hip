// The inner products of the microscaled formats: mx4 times mx4 (forward), bfloat16 times mx4 (gradient of the
// input) and bfloat16 times ckpt8 (gradient of the weights).
//
//     C[i][j] = sum_c A(i, c) * B(c, j)
#include <algorithm>
#include <type_traits>

#include "lp_mx.h"
#include "lp_mx_tile.h"

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

// Everything that this wave has asked for has arrived but the last LATER loads from memory, and so it is in every other wave of
// the workgroup.
template <int LATER>
__device__ __forceinline__ void arrived_but()
{
    static_assert(LATER < 64, "what the counter holds");
    __builtin_amdgcn_s_waitcnt((LATER & 15) | (LATER >> 4) << 14 | 7 << 4);
    asm volatile("s_barrier" ::: "memory");
}
__device__ __forceinline__ void all_arrived() { arrived_but<0>(); }

// -------------------------------------------------------------------------------- results

// Where a product's sums go: out[i][j] = act(sum + bias[j]), rounded once.  accumulate: what is there is added before the
// rounding.  (db, weights only, may be null: the sums of dY, one for each row of out.)
struct Sink {
    void *y;
    size_t ld;
    const float *bias;
    float *db;
    lp_actfn act;
    int accumulate;
};

// W neighbouring results of a row, n of which exist.
template <int W, typename T>
__device__ __forceinline__ void put(const Sink &s, T *to, const float *bias, int n, typename Floats<W>::V v)
{
    if (s.bias) v += load_floats<W>(bias, n);
    if (s.accumulate) v += load_floats<W>(to, n);
    store_floats<W>(to, n, act_values<T>(v, s.act));
}

// A wave's results, MB x NB blocks of 32 rows x 32 columns from (i0, j0) of a tile on, of which I x J exist: 32 rows at a time
// through a piece of LDS of its own, so that they leave as whole rows, W neighbours a lane: 16 bytes, so that what the lanes of a
// store write lies together.  In the accumulators a lane holds, of row lane % 32 of a block, columns 8 g + 4 (lane / 32) + 0..3 in registers 4 g ..
constexpr int result_row(int NB) { return NB * 32 + 4; } // floats, padded
constexpr int result_bytes(int NB) { return 32 * result_row(NB) * 4; }
template <int MB, int NB, int W, typename PUT>
__device__ __forceinline__ void put_blocks(float *mine, const v16f (&acc)[NB][MB], int i0, int j0, int I, int J, PUT put)
{
    constexpr int ROW = result_row(NB);
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int ib = i0 + b * 32;
        if (ib >= I) break;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const v16f &c = acc[j][b];
                *(v4f *)(mine + l32 * ROW + j * 32 + 8 * g + 4 * h) = v4f{c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // (one wave: its own writes are all there)
#pragma unroll 4
        for (int q = 0; q < 16 * NB / W; ++q) {
            const int k = q * 64 + lane, row = k / (NB * 32 / W), col = k % (NB * 32 / W) * W;
            const float *from = mine + row * ROW + col;
            const int i = ib + row, j = j0 + col;
            typename Floats<W>::V v;
#pragma unroll
            for (int p = 0; p < W; p += 4) {
                const v4f part = *(const v4f *)(from + p);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[p + e] = part[e];
            }
            if (i < I && j < J) put(i, j, v);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// Which tile a workgroup computes, and which stages of the reduction.  The first `whole` tiles, a multiple of the compute
// units, are one workgroup each and go straight to the results; every one of the rest is cut along the reduction into `parts`,
// whose 32-bit sums meet in the workspace (one part: straight to the results too).  A last round that fills a few of the
// units, and a product that has few tiles, are spread over all of them this way.
//
// Consecutive workgroups go round the dies, each die has a run of consecutive tiles, row tiles walked kTileGroup at a time: 32
// workgroups of a die share 4 x 8 tiles.
constexpr int kTileGroup = 4;
struct Grid {
    int tiles_i, tiles_j, stages, whole, rest, parts, stages_per_part, work, per_xcd; // work = rest * parts
    float *sums;                                                                      // TI * TJ of each part and tile, then TI of dY
};
struct Place {
    int tile_i, tile_j, first, last; // stages first .. last - 1
    int sums;                        // number of the part and tile, or -1
};
__device__ __forceinline__ void place_tile(const Grid &g, int tile, Place *p)
{
    // (divisions run on the vector unit: what comes back is said to be the same in all lanes)
    const int group = __builtin_amdgcn_readfirstlane(tile / (kTileGroup * g.tiles_j));
    const int in_group = tile - group * kTileGroup * g.tiles_j, rows = min(kTileGroup, g.tiles_i - group * kTileGroup);
    p->tile_j = __builtin_amdgcn_readfirstlane(in_group / rows);
    p->tile_i = group * kTileGroup + in_group - p->tile_j * rows;
}
__device__ __forceinline__ bool find_place(const Grid &g, Place *p)
{
    const bool whole = (int)blockIdx.x < g.whole;
    const int b = blockIdx.x - (whole ? 0 : g.whole), item = (b % kXCDs) * (whole ? g.whole / kXCDs : g.per_xcd) + b / kXCDs;
    if (whole) {
        place_tile(g, item, p);
        p->first = 0;
        p->last = g.stages;
        p->sums = -1;
        return true;
    }
    if (item >= g.work) return false;
    const int part = __builtin_amdgcn_readfirstlane(item / g.rest);
    place_tile(g, g.whole + item - part * g.rest, p);
    p->first = part * g.stages_per_part;
    p->last = min(g.stages, p->first + g.stages_per_part);
    p->sums = g.parts > 1 ? item : -1;
    return true;
}
constexpr size_t tile_sums(int TI, int TJ) { return (size_t)TI * TJ + TI; } // floats

template <int TI, int TJ, int MB, int NB, typename OutT>
__device__ __forceinline__ void put_results(const Grid &g, const Sink &out, const Place &p, float *mine, const v16f (&acc)[NB][MB], int i0, int j0, int I, int J)
{
    const int ti = p.tile_i * TI, tj = p.tile_j * TJ;
    if (p.sums >= 0) {
        float *to = g.sums + p.sums * tile_sums(TI, TJ);
        put_blocks<MB, NB, 4>(mine, acc, i0, j0, I - ti, J - tj, [&](int i, int j, v4f v) __attribute__((always_inline)) {
            *(v4f *)(to + i * TJ + j) = v; // (whole pieces, where the row ends inside too)
        });
    } else {
        OutT *to = (OutT *)out.y + ti * out.ld + tj;
        const float *bias = out.bias + tj;
        constexpr int W = 16 / sizeof(OutT);
        put_blocks<MB, NB, W>(mine, acc, i0, j0, I - ti, J - tj, [&](int i, int j, typename Floats<W>::V v) __attribute__((always_inline)) {
            put<W>(out, to + i * out.ld + j, bias + j, J - tj - j, v);
        });
    }
}

// y = act(sum of the parts + bias), db the same of the rows' sums: a thread takes kJoinW neighbours of a row of a tile
constexpr int kJoinW = 4; // (16 bytes of each part, so that a load's lanes lie together)
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(const Grid g, Sink out, int TI, int TJ, int I, int J, int per_tile)
{
    const int rest = blockIdx.x / per_tile, within = blockIdx.x - rest * per_tile;
    Place p;
    place_tile(g, g.whole + rest, &p);
    const size_t tile = (size_t)TI * TJ + TI, part = tile * g.rest;
    const float *sums = g.sums + rest * tile;
    auto joined = [&](const float *q, auto load) __attribute__((always_inline)) {
        auto v = load(q);
        int k = 1;
        for (; k + 8 <= g.parts; k += 8) { // eight on their way at a time
            decltype(v) w[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) w[u] = load(q + (k + u) * part);
#pragma unroll
            for (int u = 0; u < 8; ++u) v += w[u];
        }
#pragma unroll 4
        for (; k < g.parts; ++k) v += load(q + k * part);
        return v;
    };
    const int piece = within * 256 + threadIdx.x, row = piece / (TJ / kJoinW), col = piece % (TJ / kJoinW) * kJoinW;
    const int i = p.tile_i * TI + row, j = p.tile_j * TJ + col;
    if (row < TI && i < I && j < J)
        put<kJoinW>(out, (T *)out.y + i * out.ld + j, out.bias + j, J - j, joined(sums + row * TJ + col, [](const float *q) { return *(const v4f *)q; }));
    const int r = p.tile_i * TI + threadIdx.x;
    if (out.db && p.tile_j == 0 && within == 0 && threadIdx.x < TI && r < I) {
        const float v = joined(sums + TI * TJ + threadIdx.x, [](const float *q) { return *q; });
        out.db[r] = out.accumulate ? out.db[r] + v : v;
    }
}

// ------------------------------------------------------------------------------- mx4 times mx4

// y[m][n] = sum_k x[m][k] w[n][k] on v_mfma_scale_f32_32x32x64_f8f6f4, whose lane takes one block of 32 neighbours of a row
// (16 bytes of codes) and that block's scale byte.
//
// A workgroup owns TM rows of x times TN rows of w, one wave MB x NB blocks of 32 x 32; two waves per SIMD, so that the
// one's reads and address arithmetic hide behind the other's products.  A stage is 256 positions: 128 bytes of each row (a
// whole cache line: 64 bytes of twice as many rows come at 54 GB/s a CU instead of 90), brought to LDS by loads that do not
// pass through registers, into one of BUFFERS buffers; the others are on their way while one is multiplied.  16-byte piece p
// of row r lies at place p ^ (r % 8) of the row, so that the eight rows that a read takes together lie in different banks.
// Within a stage the order of the reduction is free as long as both sides share it: in step s (of four) the lower half of
// the lanes takes block s, the upper half block 4 + s, so that a lane's scale bytes of a stage are one word.  Scale bytes
// come the same way, those of four stages at a time.
//
// Weights are the row operand: a lane ends up with four neighbouring columns of one row of y.
//
// Measured with codes in hand: 8192 x 14336 from 4096 250 to 260 us, 3.7 to 3.85 PFLOP/s (with SiLU 265 to 300).
// Its clock is 1.57 GHz and a stage 3030 cycles, 2048 of them the products'; with loads that
// touch no memory 1.89 GHz and 2870 cycles: what bounds the large tiles is first the clock under this load.  256 x 4096 from 25088 26 to
// 28 us (39 where the weights come from memory), 64 x 4096 from 4096 6.0: tiles of 64 rows are bound by their loads (0.2 us for 16 KB a stage and unit) and,
// alone on a unit, by the chain of a stage's barrier, reads and products: 540 cycles a stage, 480 with loads that touch no memory.
struct Mx4Args {
    const unsigned char *xc, *xs, *wc, *ws;
    int M, N, K, blocks;
    Grid grid; // stages_per_part: a multiple of 4
    Sink out;
};

template <int MB, int NB, int WM, int WN, int BUFFERS, typename OutT>
__global__ __launch_bounds__(WM *WN * 64, WM *WN == 4 && MB * NB * BUFFERS == 16 ? 1 : 2) void mx4_product_kernel(const Mx4Args a)
{
    static_assert(BUFFERS == 2 || BUFFERS == 4, "a stage's buffer is known where it is written out");
    constexpr int TM = MB * 32 * WM, TN = NB * 32 * WN, WAVES = WM * WN, ROWS = TM + TN, STAGE = ROWS * 128, PER = ROWS / 8 / WAVES;
    constexpr int SROWS = ROWS / WAVES, SPER = SROWS / 32; // rows whose scale bytes a wave brings, loads that takes
    static_assert(TM % SROWS == 0, "of one tensor");
    __shared__ __align__(1024) unsigned char lds[BUFFERS * STAGE + ROWS * 32];
    static_assert(WAVES * result_bytes(NB) <= (int)sizeof(lds), "results pass through the same memory");
    Place p;
    if (!find_place(a.grid, &p)) return;
    const int m0 = p.tile_i * TM, n0 = p.tile_j * TN, first = p.first, last = p.last;

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
    // Scale bytes of stages t .. t + 3 (t a multiple of 4), 32 for each row: of 32 rows the first 16 each, then the others, so
    // that a read's lanes lie side by side.  (A row's 32 bytes together, read a word at a time, cost half of all LDS cycles.)
    // Bytes of stages that do not exist are the next row's, or zeros behind the last: the descriptor ends with the tensor.
    unsigned char *const scales = lds + BUFFERS * STAGE;
    const bool of_x = wave * SROWS < TM;
    unsigned scale_at[SPER];
#pragma unroll
    for (int i = 0; i < SPER; ++i) scale_at[i] = row_of(wave * SROWS + i * 32 + l32) * (unsigned)a.blocks + h * 16;
    auto load_scales = [&](int t) __attribute__((always_inline)) {
        const unsigned char *base = (of_x ? a.xs + (size_t)m0 * a.blocks : a.ws + (size_t)n0 * a.blocks) + 8 * t;
        const long long rest = (long long)(of_x ? a.M - m0 : a.N - n0) * a.blocks - 8 * t;
        const int size = __builtin_amdgcn_readfirstlane(t < last ? (int)(unsigned)std::min(rest, 0xffffffffLL) : 0);
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(base), 0, size, 0x00020000);
#pragma unroll
        for (int i = 0; i < SPER; ++i) load_lds16(from, scales + wave * SROWS * 32 + i * 1024, scale_at[i], 0);
    };
    int xscale[4][MB], wscale[4][NB];
    auto take_scales = [&]() __attribute__((always_inline)) {
        auto take = [&](int block, int q) __attribute__((always_inline)) { return *(const v4i *)(scales + block * 1024 + q / 2 * 512 + l32 * 16); };
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const v4i v = take(wm * MB + i, q);
                xscale[q][i] = h ? v[1] : v[0];
                xscale[q + 1][i] = h ? v[3] : v[2];
            }
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const v4i v = take(TM / 32 + wn * NB + i, q);
                wscale[q][i] = h ? v[1] : v[0];
                wscale[q + 1][i] = h ? v[3] : v[2];
            }
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
    // stage that will have it is asked for, over three steps: 64 loads at once take the address unit so long that every wave
    // waits for its turn.  At the first one's the scale bytes are in registers and the next four's are asked for.
    auto whole_stage = [&](int t, auto number) __attribute__((always_inline)) {
        constexpr int Q = decltype(number)::value, B = Q % BUFFERS, BEFORE = (Q + BUFFERS - 1) % BUFFERS;
        // loads that may still be on their way when the next stage has arrived: the stages behind it, the scale bytes
        constexpr int LATER = (BUFFERS - 2) * PER + (Q >= 1 && Q <= BUFFERS - 2 ? SPER : 0);
        __builtin_amdgcn_sched_barrier(0);
        fragments(B, 1);
        stage(t + BUFFERS - 1, BEFORE, L1, L2);
        LP_STEP(Q, 0, true)
        fragments(B, 2);
        stage(t + BUFFERS - 1, BEFORE, L2, L3);
        LP_STEP(Q, 1, true)
        fragments(B, 3);
        LP_STEP(Q, 2, false)
        arrived_but<LATER>();
        fragments((Q + 1) % BUFFERS, 0);
        stage(t + BUFFERS, B, L0, L1);
        if (Q == 0) load_scales(t + 4);
        LP_STEP(Q, 3, true)
    };
#undef LP_STEP
    load_scales(first);
#pragma unroll
    for (int b = 0; b < BUFFERS - 1; ++b) stage(first + b, b, L0, L3);
    arrived_but<(BUFFERS - 2) * PER>();
    stage(first + BUFFERS - 1, BUFFERS - 1, L0, L1);
    fragments(0, 0);
    for (int t = first;; t += 4) {
        take_scales();
        whole_stage(t, std::integral_constant<int, 0>());
        if (t + 1 >= last) break;
        whole_stage(t + 1, std::integral_constant<int, 1>());
        if (t + 2 >= last) break;
        whole_stage(t + 2, std::integral_constant<int, 2>());
        if (t + 3 >= last) break;
        whole_stage(t + 3, std::integral_constant<int, 3>());
        if (t + 4 >= last) break;
    }
    all_arrived();
    put_results<TM, TN, MB, NB, OutT>(a.grid, a.out, p, (float *)(lds + wave * result_bytes(NB)), acc, wm * MB * 32, wn * NB * 32, a.M, a.N);
}

// Few rows (16 at most): the weights are all that matters, and every byte of them is read once, straight into the registers that the matrix
// instruction (16 x 16 x 128) takes: 16 rows of w a workgroup, the reduction cut among its eight waves in chunks of 512 positions.
// A lane holds 64 neighbouring bytes of a row in four operands, whose scale bytes are one word.  Rows of x come as codes from
// memory, or, X a float type, are brought to codes by every wave for its own chunks: the rows are short, and a launch that
// does it beforehand takes longer.  The waves' sums meet in LDS, added in order.
constexpr int kFewWaves = 8;

template <typename X, typename OutT>
__global__ __launch_bounds__(kFewWaves * 64, 2) void mx4_few_kernel(const Mx4Args a, const X *x, size_t ldx)
{
    constexpr bool CODES = std::is_same<X, unsigned char>::value;
    constexpr int QROW = 256 + 16; // a quantized row of a chunk in LDS: codes, scale bytes
    __shared__ __align__(16) unsigned char lds[CODES ? 16 : kFewWaves * 16 * QROW];
    __shared__ __align__(32) float sums[kFewWaves][16][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16, chunks = (a.blocks + 15) / 16;
    const unsigned pitch = (unsigned)a.blocks * 16;
    // rows beyond the last lie outside the descriptors, and so is what lies behind a row: zeros
    const int wrows = min(a.N - n0, 16);
    const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.wc) + (size_t)n0 * pitch, 0, wrows * pitch, 0x00020000);
    const __amdgpu_buffer_rsrc_t wsr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.ws) + (size_t)n0 * a.blocks, 0, wrows * a.blocks, 0x00020000);
    const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.xc), 0, CODES ? a.M * pitch : 0, 0x00020000);
    const __amdgpu_buffer_rsrc_t xsr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.xs), 0, CODES ? a.M * a.blocks : 0, 0x00020000);
    struct Operand {
        v4i f[4];
        int s;
    };
    auto load = [&](Operand &o, __amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t scales, int row, int chunk) __attribute__((always_inline)) {
        const unsigned block = row * (unsigned)a.blocks + 16 * chunk + 4 * q;
        const bool there = 16 * chunk + 4 * q < a.blocks;
        const unsigned at = there ? block * 16 : 0xfffffff0u - 64;
#pragma unroll
        for (int k = 0; k < 4; ++k) o.f[k] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(codes, at + 16 * k, 0, 0));
        o.s = __builtin_amdgcn_raw_buffer_load_b32(scales, there ? block : 0xfffffff0u, 0, 0);
    };
    v4f acc = 0.0f;
    Operand w, v;
#define LP_PART(S)                                                                                                                          \
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v8i{w.f[S][0], w.f[S][1], w.f[S][2], w.f[S][3], 0, 0, 0, 0},                     \
                                                           v8i{v.f[S][0], v.f[S][1], v.f[S][2], v.f[S][3], 0, 0, 0, 0}, acc, 4, 4, S, w.s, S, v.s);
    for (int c = wave; c < chunks; c += kFewWaves) {
        load(w, wr, wsr, r16, c);
        if constexpr (CODES) {
            load(v, xr, xsr, r16, c);
        } else {
            unsigned char *mine = lds + wave * 16 * QROW;
            const int at = c * 512 + lane * 8, n = (int)a.K - at;
#pragma unroll 4
            for (int r = 0; r < a.M; ++r) {
                const v8f f = load8(x + r * ldx + at, n);
                const int e = mx4_scale_byte(block_exponent(f));
                *(unsigned *)(mine + r * QROW + lane * 4) = mx4_word(f, e);
                if ((lane & 3) == 0) mine[r * QROW + 256 + lane / 4] = (unsigned char)e;
            }
            const int row = min(r16, a.M - 1);
#pragma unroll
            for (int k = 0; k < 4; ++k) v.f[k] = *(const v4i *)(mine + row * QROW + (4 * q + k) * 16);
            v.s = *(const int *)(mine + row * QROW + 256 + 4 * q);
        }
        LP_PART(0)
        LP_PART(1)
        LP_PART(2)
        LP_PART(3)
    }
#undef LP_PART
    *(v4f *)&sums[wave][r16][4 * q] = acc;
    __syncthreads();
    const int m = threadIdx.x / 2, n = n0 + threadIdx.x % 2 * 8;
    if (m < 16 && m < a.M && n < a.N) {
        v8f sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) sum += *(const v8f *)&sums[k][m][n - n0];
        put<8>(a.out, (OutT *)a.out.y + m * a.out.ld + n, a.out.bias + n, a.N - n, sum);
    }
}

// -------------------------------------------------------------------------------- gradients

// D[i][j] = sum_c A(i, c) B(c, j) on v_mfma_f32_32x32x16_bf16, A the bfloat16 gradient dY, B an mx4 or ckpt8 tensor whose rows are
// the reduction.  Values of either format have at most seven significant bits: they are exact in bfloat16.
//   gradient of the input:    i = m, c = n, j = k; A(i, c) = dY[i][c], B = Wq
//   gradient of the weights:  i = n, c = m, j = k; A(i, c) = dY[c][i], B = X8
//
// A workgroup owns TI x TJ results, a wave MB x NB blocks of 32 x 32; a stage is 64 positions of the reduction in one of two
// LDS buffers.  B's codes pass through registers, a block of 32 a thread, and are decoded one stage ahead; dY
// comes by loads to LDS (or, where its rows do not start on words, through registers like the codes: 200 x 4096 from 1001
// columns 11.5 us, from 1002 10.9; 8192 x 4096 from 14337 880 to 925, from 14338 740 to 785).  The matrix
// instruction wants eight neighbouring positions of a row or column in a lane: those of dY's rows lie together in memory
// (16-byte piece p of row r at place p ^ (r % 8), as above); tiles with the reduction along their rows are read by
// ds_read_b64_tr_b16, which hands each of 16 lanes four rows' elements of its column.  Their rows are 512 (or 256) bytes, so
// the four rows of such a read lie in the same banks unless the 64-byte pieces of row r change places with r % 4 (r % 2 where a row has two).  Decoded
// codes also swap neighbouring 16 bytes where (column / 128 + row) is odd, for the sake of the writes.
//
// B is the row operand of the instruction, so that a lane ends up with four neighbouring columns of one row of D.
//
// Measured: 8192 x 4096 from 14336 715 to 760 us, 1.27 to 1.34 PFLOP/s; weights 14336 x 4096 over 8192 850 to 900, 1.07 to
// 1.13 (a library product of two bfloat16 tensors of these sizes reaches 1.2 to 1.5).  A stage of the large tile takes 2890 cycles (2048 are
// the products') at 1.85 GHz; with codes that are not decoded 2880 at 2.02, 680 us: the decoding costs clock, not cycles.  Weights 3270
// at 1.87, 3000 at 2.01 and 750 us.  256 x 4096 weights over 256 rows 21 us: 16.8 MB leave at 3 TB/s.
struct GradArgs {
    const __bf16 *dy;
    size_t ld;
    const unsigned char *codes, *scales;
    int I, J, C, blocks; // blocks of 32 in a row of B
    Grid grid;
    Sink out;
};

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s *LdsV4;

// Eight neighbouring positions of a lane's column: four rows from one place, four from the other.  (No load to LDS that is on
// its way writes there: the arguments say so, or the compiler would wait for all of them first.)
__device__ __forceinline__ v8s read_columns(const unsigned char *__restrict__ first, const unsigned char *__restrict__ next)
{
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsV4)first), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsV4)next);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

constexpr size_t kNearRows = (size_t)1 << 22; // dY's row strides up to which a tile's offsets fit 32 bits

// n (at most 8) bfloat16 of a row as one 16-byte piece, zeros behind them
__device__ __forceinline__ v4u load_piece(const __bf16 *p, int n)
{
    typedef unsigned short V __attribute__((ext_vector_type(8), aligned(2)));
    typedef unsigned short W __attribute__((ext_vector_type(8)));
    const unsigned short *q = reinterpret_cast<const unsigned short *>(p);
    W v = 0;
    if (n >= 8) {
        v = *reinterpret_cast<const V *>(q);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) v[e] = q[e];
    }
    return __builtin_bit_cast(v4u, v);
}

// A block of 32 codes with its scale byte: 16 bytes of mx4, 32 of ckpt8.
template <bool WEIGHTS>
struct RawBlock {
    v4u w[WEIGHTS ? 2 : 1];
    int e;
    // what lies outside the descriptors comes as zeros
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t scales, unsigned block)
    {
#pragma unroll
        for (int k = 0; k < (WEIGHTS ? 2 : 1); ++k)
            w[k] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(codes, block * (WEIGHTS ? 32 : 16) + 16 * k, 0, 0));
        e = __builtin_amdgcn_raw_buffer_load_b8(scales, block, 0, 0);
    }
    // sixteen-byte piece k of the block's values: elements 8 k .. 8 k + 7
    __device__ __forceinline__ v4u piece(int k) const
    {
        if constexpr (WEIGHTS) {
            const float s = power_of_byte(e - 6);
            v4u r;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const unsigned word = w[k >> 1][(k & 1) * 2 + (d >> 1)] >> (16 * (d & 1));
                const float lo = (float)(signed char)word * s, hi = (float)(signed char)(word >> 8) * s;
                r[d] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u); // (their low halves are zero)
            }
            return r;
        } else {
            const float s = power_of_byte(e);
            v4u r;
            r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0][k], s, 0));
            r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0][k], s, 1));
            r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0][k], s, 2));
            r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0][k], s, 3));
            return r;
        }
    }
};

// The eight from column `col` on of a row of `cols`, 8 at least; zeros where it has ended.  One load, that lies within the row,
// and a shift.
__device__ __forceinline__ v4u load_tail(const __bf16 *row, int col, int cols)
{
    typedef unsigned short V __attribute__((ext_vector_type(8), aligned(2)));
    const int from = min(col, cols - 8), gone = col - from;
    v4u v = __builtin_bit_cast(v4u, *reinterpret_cast<const V *>(row + from));
    if (gone & 1) v = v4u{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
    if (gone & 2) v = v4u{v[1], v[2], v[3], 0};
    if (gone & 4) v = v4u{v[2], v[3], 0, 0};
    return gone >= 8 ? v4u{0, 0, 0, 0} : v;
}

template <int MB, int NB, int WM, int WN, bool WEIGHTS, bool WORDS, typename OutT>
__global__ __launch_bounds__(WM *WN * 64, 2) void gradient_kernel(const GradArgs a)
{
    constexpr int TI = MB * 32 * WM, TJ = NB * 32 * WN, WAVES = WM * WN, THREADS = WAVES * 64;
    constexpr int ABYTES = TI * 128, BBYTES = TJ * 128, STAGE = ABYTES + BBYTES;
    typedef DyTile<TI, WAVES, WEIGHTS> Dy;
    constexpr int PER = Dy::PER, AROW = Dy::ROW, ATURN = Dy::TURN, BROW = TJ * 2;
    constexpr int BTURN = (BROW < 256 ? BROW / 64 : 4) - 1; // 64-byte pieces that change places
    static_assert((BROW & (BROW - 1)) == 0, "places are exchanged within a row");
    static_assert(TJ * 2 == THREADS, "a thread decodes one block of 32 per stage");
    __shared__ __align__(1024) unsigned char lds[2 * STAGE];
    static_assert(WAVES * result_bytes(NB) <= (int)sizeof(lds), "results pass through the same memory");
    Place p;
    if (!find_place(a.grid, &p)) return;
    const int i0 = p.tile_i * TI, j0 = p.tile_j * TJ, first = p.first, last = p.last;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h = lane >> 5, wm = wave % WM, wn = wave / WM;

    // dY.  The last stage of the whole reduction comes through registers where it, or a row, ends inside a piece: what lies
    // behind must not be multiplied, not even by zero.
    const bool ragged = last == a.grid.stages && (last * 64 != a.C || (WEIGHTS && i0 + TI > a.I));
    // Stages first .. whole - 1 come in whole pieces.  (Through registers only where offsets are 32 bits, and a piece reaches no
    // further than into the next row.)
    const bool direct = WORDS || (a.ld < kNearRows && (!WEIGHTS || a.ld >= 8));
    const int whole = direct ? last - ragged : first;
    // row and piece of the row that this lane brings, and where in a stage's buffer
    auto dy_row = [&](int q) __attribute__((always_inline)) { return Dy::row(Dy::number(wave, q, lane)); };
    auto dy_piece = [&](int q) __attribute__((always_inline)) { return Dy::piece(Dy::number(wave, q, lane)); };
    auto dy_place = [&](int buf, int q) __attribute__((always_inline)) { return lds + buf * STAGE + Dy::number(wave, q, lane) * 16; };
    unsigned at[PER];
#pragma unroll
    for (int q = 0; q < PER; ++q) at[q] = (unsigned)(WEIGHTS ? dy_row(q) : min(dy_row(q), a.I - 1 - i0)) * (unsigned)(a.ld * 2) + dy_piece(q) * 16;
    // loads FROM .. TO - 1 of a wave's share of stage t; where nothing is to come the descriptor is empty and zeros arrive
    auto load_dy = [&](int t, int buf, auto from, auto to) __attribute__((always_inline)) {
        if constexpr (WORDS) {
            const __bf16 *base = WEIGHTS ? a.dy + (size_t)t * 64 * a.ld + i0 : a.dy + (size_t)i0 * a.ld + t * 64;
            // Weights: a tile's row may reach past the end of dY's, over several of them where these are short; not past the last
            // one's.  (Whole words: the last row is not brought this way.)
            const long long rest = ((long long)(a.C - 1 - t * 64) * (long long)a.ld + (a.I - i0)) * 2;
            const int all = WEIGHTS ? (int)(unsigned)std::min(rest & ~3LL, 0xfffffffcLL) : -1;
            const int size = __builtin_amdgcn_readfirstlane(t < whole ? all : 0);
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<__bf16 *>(base), 0, size, 0x00020000);
#pragma unroll
            for (int q = decltype(from)::value; q < decltype(to)::value; ++q) load_lds16(rsrc, lds + buf * STAGE + Dy::number(wave, q, 0) * 16, at[q], 0);
        }
    };
    // A thread's pieces of a stage at once, or in two halves where registers are short beside a large tile's sums.  (8192 x 4096
    // from 14337: 1.10 ms at once, 0.92 in halves; weights 14337 x 4096 over 8192 the same in both.)
    constexpr int HALF = MB * NB >= 8 && !WEIGHTS ? PER / 2 : PER;
    v4u raw_dy[HALF] = {};
    auto fetch_dy = [&](int t, int half) __attribute__((always_inline)) {
        if (t >= whole) return;
        typedef unsigned short V __attribute__((ext_vector_type(8), aligned(2)));
        const size_t from = WEIGHTS ? (size_t)t * 64 * a.ld + i0 : (size_t)i0 * a.ld + t * 64;
        // (weights: a row's last piece reaches into the next row, the tile's into the one behind, but not past the end)
        const unsigned most = WEIGHTS ? (unsigned)std::min(((size_t)(a.C - 1) * a.ld + a.I - 8 - from) * 2, (size_t)0x7ffffffe) : 0;
#pragma unroll
        for (int q = 0; q < HALF; ++q) {
            const unsigned o = at[half * HALF + q];
            raw_dy[q] = __builtin_bit_cast(v4u, *reinterpret_cast<const V *>(reinterpret_cast<const char *>(a.dy + from) + (WEIGHTS ? std::min(o, most) : o)));
        }
    };
    // A stage at once, the ragged one for instance: as many pieces on their way together as there are registers for beside the sums.
    // (Where dY comes by loads to LDS, empty ones of this stage left zeros in the pieces that are written here.  They are this
    // wave's own, and it has waited for them; other waves' may still be on their way.)
    auto bring_dy = [&](int t, int buf) __attribute__((always_inline)) {
        constexpr int TOGETHER = MB * NB >= 8 ? 1 : PER;
        const int rows = WEIGHTS ? a.C : a.I, cols = WEIGHTS ? a.I : a.C;
#pragma unroll 1
        for (int q0 = 0; q0 < PER; q0 += TOGETHER) {
            v4u piece[TOGETHER];
#pragma unroll
            for (int q = 0; q < TOGETHER; ++q) {
                const int r = dy_row(q0 + q), s = dy_piece(q0 + q);
                const int row = WEIGHTS ? t * 64 + r : i0 + r, col = WEIGHTS ? i0 + s * 8 : t * 64 + s * 8;
                if (rows < 1 || cols < 8) piece[q] = load_piece(a.dy + row * a.ld + col, row < rows ? cols - col : 0);
                else piece[q] = load_tail(a.dy + min(row, rows - 1) * a.ld, row < rows ? col : cols, cols);
            }
            __builtin_amdgcn_s_waitcnt(0); // (and the zeros of this wave's empty loads have arrived)
#pragma unroll
            for (int q = 0; q < TOGETHER; ++q) *(v4u *)dy_place(buf, q0 + q) = piece[q];
        }
    };
    auto place_dy = [&](int buf, int half) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < HALF; ++q) *(v4u *)dy_place(buf, half * HALF + q) = raw_dy[q];
    };

    // B: thread's row of the stage and block of the row.  The descriptors start at a stage's first row and end with the tensor.
    RawBlock<WEIGHTS> raw;
    const int brow = threadIdx.x / (TJ / 32), bblock = threadIdx.x % (TJ / 32);
    const unsigned bat = j0 / 32 + bblock < a.blocks ? (unsigned)brow * (unsigned)a.blocks + (unsigned)(j0 / 32 + bblock) : 0x07ffffffu;
    // (eight lanes that write together hold one piece of each 64 bytes of a row, or of two rows: half of them swap neighbours)
    unsigned char *const bplace = lds + ABYTES + brow * BROW + (bblock ^ (brow & BTURN)) * 64;
    const int bswap = ((bblock >> 2 ^ brow) & 1) * 16;
    const int end = min(last * 64, a.C);
    auto load_b = [&](int t) __attribute__((always_inline)) {
        constexpr int BLOCK = WEIGHTS ? 32 : 16;
        const long long left = std::min(std::max((long long)(end - t * 64) * a.blocks, 0LL), 0x07ffffffLL); // blocks
        const int scales = __builtin_amdgcn_readfirstlane((int)left), codes = (int)((unsigned)scales * BLOCK);
        const size_t from = (size_t)t * 64 * a.blocks;
        raw.load(__builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.codes) + from * BLOCK, 0, codes, 0x00020000),
                 __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(a.scales) + from, 0, scales, 0x00020000), bat);
    };
    auto place_b = [&](int buf, int from, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int k = from; k < to; ++k) *(v4u *)(bplace + buf * STAGE + (k * 16 ^ bswap)) = raw.piece(k);
    };

    v16f acc[NB][MB] = {};
    v8s fa[2][MB], fb[2][NB];
    // this lane's place in a read of four rows x 16 columns (x0: the tile column of its block of 32)
    const int tr_row = 8 * h + (lane & 15) / 4, tr_col = (lane >> 4 & 1) * 32 + (lane & 3) * 8;
    auto tr_place = [&](int x0, int row_bytes, int turn) __attribute__((always_inline)) { return tr_row * row_bytes + ((x0 / 32) ^ (tr_row & turn)) * 64 + tr_col; };
    int apos[MB], bpos[NB];
#pragma unroll
    for (int b = 0; b < MB; ++b) apos[b] = WEIGHTS ? tr_place((wm * MB + b) * 32, AROW, ATURN) : ((wm * MB + b) * 32 + l32) * 128;
#pragma unroll
    for (int b = 0; b < NB; ++b) bpos[b] = ABYTES + (tr_place((wn * NB + b) * 32, BROW, BTURN) ^ (((wn * NB + b) >> 2 ^ tr_row) & 1) * 16);
    auto tr_read = [&](int pos, int row_bytes) __attribute__((always_inline)) { return read_columns(lds + pos, lds + pos + 4 * row_bytes); };
    auto fragments = [&](int buf, int s) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            if constexpr (WEIGHTS) fa[s & 1][b] = tr_read(buf * STAGE + apos[b] + s * 16 * AROW, AROW);
            else fa[s & 1][b] = *(const v8s *)(lds + buf * STAGE + apos[b] + ((2 * s + h) ^ (l32 & 7)) * 16);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) fb[s & 1][b] = tr_read(buf * STAGE + bpos[b] + s * 16 * BROW, BROW);
    };
    // sums of dY: a lane's eight positions of its column of each block
    const bool sum_dy = WEIGHTS && a.out.db && p.tile_j == 0 && wn == 0;
    float db[MB] = {};
    auto add_dy = [&](int s) __attribute__((always_inline)) {
        if constexpr (WEIGHTS) {
            if (sum_dy) {
                const v2bf one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
                for (int b = 0; b < MB; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        typedef short v2sh __attribute__((ext_vector_type(2)));
                        const v2sh two = {fa[s & 1][b][2 * e], fa[s & 1][b][2 * e + 1]};
                        db[b] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, two), one, db[b], false);
                    }
            }
        }
    };
#define LP_STEP(S)                                                                                                                          \
    _Pragma("unroll") for (int j = 0; j < NB; ++j) _Pragma("unroll") for (int i = 0; i < MB; ++i) acc[j][i] =                                \
        __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, fb[S & 1][j]), __builtin_bit_cast(v8bf, fa[S & 1][i]), acc[j][i], 0, 0, 0); \
    _Pragma("unroll") for (int q = 0; q < MB * NB; ++q)                                                                                      \
    {                                                                                                                                       \
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);                                                                                  \
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                                                                  \
    }                                                                                                                                       \
    __builtin_amdgcn_sched_barrier(0);                                                                                                      \
    add_dy(S);
    constexpr std::integral_constant<int, 0> L0;
    constexpr std::integral_constant<int, PER / 2> L1;
    constexpr std::integral_constant<int, PER> L2;
    // Stage t in buffer B: while it is multiplied the next one is completed in the other buffer.
    auto whole_stage = [&](int t, auto buffer) __attribute__((always_inline)) {
        constexpr int B = decltype(buffer)::value;
        // loads that may still be on their way when the next stage's dY has arrived: the codes of the one behind it (all of them
        // where dY is written to LDS from registers)
        constexpr int LATER = WORDS ? (WEIGHTS ? 3 : 2) : 63;
        __builtin_amdgcn_sched_barrier(0);
        fragments(B, 1);
        load_dy(t + 1, B ^ 1, L1, L2);
        place_b(B ^ 1, 0, 2);
        LP_STEP(0)
        if constexpr (!WORDS && HALF < PER) {
            place_dy(B ^ 1, 0);
            fetch_dy(t + 1, 1);
        }
        fragments(B, 2);
        place_b(B ^ 1, 2, 4);
        load_b(t + 2);
        LP_STEP(1)
        if constexpr (!WORDS && HALF == PER) {
            place_dy(B ^ 1, 0);
            fetch_dy(t + 2, 0);
        }
        fragments(B, 3);
        LP_STEP(2)
        if constexpr (!WORDS && HALF < PER) {
            place_dy(B ^ 1, 1);
            fetch_dy(t + 2, 0);
        }
        if (t + 1 >= whole && t + 1 < last) bring_dy(t + 1, B ^ 1);
        arrived_but<LATER>();
        fragments(B ^ 1, 0);
        load_dy(t + 2, B, L0, L1);
        LP_STEP(3)
    };
    load_b(first);
    load_dy(first, 0, L0, L2);
    place_b(0, 0, 4);
    load_b(first + 1);
    if (whole == first) {
        bring_dy(first, 0);
    } else if constexpr (!WORDS) {
        for (int half = 0; half < PER / HALF; ++half) {
            fetch_dy(first, half);
            place_dy(0, half);
        }
    }
    if constexpr (!WORDS) fetch_dy(first + 1, 0);
    all_arrived();
    load_dy(first + 1, 1, L0, L1);
    fragments(0, 0);
    for (int t = first;; t += 2) {
        whole_stage(t, std::integral_constant<int, 0>());
        if (t + 1 >= last) break;
        whole_stage(t + 1, std::integral_constant<int, 1>());
        if (t + 2 >= last) break;
    }
#undef LP_STEP
    all_arrived();
    if (sum_dy) {
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            const float v = db[b] + __shfl_xor(db[b], 32);
            const int i = (wm * MB + b) * 32 + l32;
            if (h != 0 || i0 + i >= a.I) continue;
            if (p.sums >= 0) a.grid.sums[p.sums * tile_sums(TI, TJ) + TI * TJ + i] = v;
            else a.out.db[i0 + i] = a.out.accumulate ? a.out.db[i0 + i] + v : v;
        }
    }
    put_results<TI, TJ, MB, NB, OutT>(a.grid, a.out, p, (float *)(lds + wave * result_bytes(NB)), acc, wm * MB * 32, wn * NB * 32, a.I, a.J);
}

// ------------------------------------------------------------------------------------- plans

static bool sizes_ok(int M, int K, int Nout) { return M >= 0 && K > 0 && Nout > 0; }
static bool sizes_taken(int M, int K, int Nout)
{
    const long long most = 1LL << 40;
    return M <= (1 << 24) && K <= (1 << 24) && Nout <= (1 << 24) && (long long)M * K < most && (long long)M * Nout < most && (long long)K * Nout < most;
}

static bool mx4_ok(const void *codes, const void *scales) { return codes && aligned16(codes) && scales && aligned_to(scales, 8); }

static size_t round256(size_t v) { return (v + 255) / 256 * 256; }

// Tiles that a product's kernel is built for, and what they cost in us: a stage of one workgroup on an idle chip and, per
// compute unit, with all of them at work (clocks fall under full load); a first workgroup's beginning and end, what they add for
// each further one (others of the same unit go on meanwhile).
struct TileCost {
    int i, j;
    double alone, full, ends, more;
};
// A stage of each of `work` workgroups.
static double stage_cost(const TileCost &c, long long work)
{
    const double last = work % kCUs ? std::min(c.alone, c.full) + std::max(0.0, c.full - c.alone) * (work % kCUs) / kCUs : 0.0;
    return std::max(c.alone, (double)(work / kCUs) * c.full + last);
}
// 64 x 64, 128 x 128 (four buffers each), 256 x 256 (two), 128 x 128 with two, which lets two workgroups of a unit work and end
// side by side; a stage is 256 positions
constexpr TileCost kMx4Tiles[4] = {{64, 64, 0.175, 0.2, 1.9, 0.8}, {128, 128, 0.345, 0.51, 3.35, 2.85}, {256, 256, 1.03, 1.58, 4.9, 3.2}, {128, 128, 0.54, 0.49, 2.6, 1.35}};
// 64 x 128, 128 x 128, 256 x 256; a stage is 64 positions
constexpr TileCost kInputTiles[3] = {{64, 128, 0.39, 0.315, 2.65, 0.45}, {128, 128, 0.505, 0.455, 3.15, 0.0}, {256, 256, 1.19, 1.34, 4.1, 0.0}};
// The weights' gradient, whichever way dY comes to LDS: the timings of both ways are fitted together, so that the choice depends on
// the sizes alone.  (With a table for each, chosen by the parity of Nout, a dY whose stride had the other parity got the other's
// tile, and 600 x 768 over 256 rows took 9.4 us instead of 7.2.)
constexpr TileCost kWeightTiles[3] = {{64, 128, 0.59, 0.42, 3.85, 0.565}, {128, 128, 0.825, 0.56, 4.68, 1.455}, {256, 256, 1.3, 1.605, 8.265, 3.825}};

// How a product I x J with `stages` stages of its reduction is cut into workgroups.
struct Cut {
    int size, i, j; // which of the tiles
    Grid grid;
    size_t sums;    // bytes (0: one part)
    double us;
};

// The cheapest of the tiles and numbers of parts, by an estimate that the tables above were fitted to (2915 timings of 380
// problems with operands in the caches: against the best of each the choice costs 0.2 % of a forward product on the average, 1 to 1.6 %
// of a gradient; it is a part too many or too few, 10 to 25 %, where it is worst).  What operands take that come from
// memory is not in it.  Results leave at 44 GB/s a compute unit; joining the parts is a launch, and their sums go through memory at
// 7.5 TB/s.  A part has `step` stages or a multiple of them, and `least` at least.
template <int SIZES>
static Cut cut_product(int I, int J, int stages, int step, int least, const TileCost (&tiles)[SIZES], int out_bytes)
{
    Cut best = {};
    for (int size = 0; size < SIZES; ++size) {
        const TileCost &c = tiles[size];
        const long long ti = (I + c.i - 1) / c.i, tj = (J + c.j - 1) / c.j, all = ti * tj;
        // all tiles in parts, or those of the last round only
        for (int keep = 0; keep < (all > kCUs && all % kCUs ? 2 : 1); ++keep) {
            const long long full = keep ? all / kCUs : 0, rest = all - full * kCUs;
            for (int parts = 1 + keep; parts <= 32; parts += parts < 4 ? 1 : parts / 2) { // 1 2 3 4 6 9 13 19 28
                if (parts > 1 && (stages < parts * least || rest * parts > 4 * kCUs)) break;
                const int each = ((stages + parts - 1) / parts + step - 1) / step * step, real = (stages + each - 1) / each;
                if (keep && real == 1) continue;
                const long long work = rest * real, rounds = (work + kCUs - 1) / kCUs;
                const double ends = 2.5 + c.ends + (full + rounds - 1) * c.more, out = (double)c.i * c.j / 45056.0;
                const double leave = full * out * out_bytes + rounds * out * std::min(1.0, (double)work / kCUs) * (real > 1 ? 4 : out_bytes);
                double us = ends + leave + full * stages * c.full + std::min(each, stages) * (stage_cost(c, full * kCUs + work) - full * c.full);
                if (real > 1) us += 2.3 + (double)real * (keep ? (double)rest * c.i * c.j : (double)I * J) * 8 / 7.5e6;
                if (best.us == 0 || us < best.us) {
                    best.us = us;
                    best.size = size;
                    best.i = c.i;
                    best.j = c.j;
                    best.grid = Grid{(int)ti, (int)tj, stages, (int)full * kCUs, (int)rest, real, each, (int)work, (int)((work + kXCDs - 1) / kXCDs), nullptr};
                }
            }
        }
    }
    const Grid &g = best.grid;
    best.sums = g.parts > 1 ? round256(g.work * tile_sums(best.i, best.j) * 4) : 0;
    return best;
}

static unsigned workgroups(const Grid &g) { return (unsigned)g.whole + (unsigned)g.per_xcd * kXCDs; }

// out = act(sum of the parts + bias)
static void join_parts(const Cut &c, const Grid &g, lp_dtype t, const Sink &out, int I, int J, hipStream_t st)
{
    const int per_tile = (std::min(c.i, I) * (c.j / kJoinW) + 255) / 256;
    with_type(t, [&](auto *tag) {
        typedef std::remove_pointer_t<decltype(tag)> T;
        hipLaunchKernelGGL(join_parts_kernel<T>, dim3((unsigned)g.rest * per_tile), dim3(256), 0, st, g, out, c.i, c.j, I, J, per_tile);
    });
}

struct Mx4Plan {
    bool few;             // the kernel for few rows, else tiles
    bool floats;          // it takes x as floats
    Cut cut;
    size_t blocks;        // of 32 per row
    size_t codes, scales; // workspace: quantized x (if the call brings floats), then the sums of the parts
    size_t total() const { return codes + scales + cut.sums; }
};

static Mx4Plan mx4_plan(int M, int K, int Nout)
{
    Mx4Plan p = {};
    p.blocks = mx4_blocks((size_t)K);
    double few_us = 0.0, few_floats = 0.0;
    if (M <= 16) {
        // Few rows: every workgroup reads 16 rows of w and all of x, 8 TB/s in all, a wave's chunk takes half a microsecond.
        // Quantizing x is a launch of 2.3 us, or 0.35 us a row and chunk where every wave does it.
        // us, few rows : tiles, bf16: 1 x 4096 -> 14336 9.0 : 9.9, 16 rows 15.7 : 10.7, 1 x 14336 -> 4096 8.3 : 13.3, 8 rows 12.8 : 13.8.
        // (The rate is the caches'.  Weights that come from memory take longer in either, which leaves the choice as it is: with ten
        // layers' in turn 9.7 : 10.7, 17.8 : 11.5, 9.2 : 14.2, 13.3 : 14.8; 1 x 4096 -> 131072, 285 MB, 50.7 : 49.8.)
        const double chunks = (double)((p.blocks + 16 * kFewWaves - 1) / (16 * kFewWaves));
        const double read = (double)Nout * p.blocks * 17 * (1 + M / 16.0) / 8e6;
        few_floats = 0.35 * M * chunks;
        few_us = 3.0 + std::max(0.5 * chunks, read) + std::min(few_floats, 2.3);
        p.few = few_us < 2.5 + kMx4Tiles[0].ends + 2.3; // (what no tiles go below; an estimate of them takes half a microsecond)
    }
    if (!p.few) {
        p.cut = cut_product(M, Nout, (int)(p.blocks / 8), 4, 4, kMx4Tiles, 2);
        p.few = M <= 16 && few_us < p.cut.us + 2.3;
    }
    p.floats = p.few && few_floats < 2.8;
    if (p.few) p.cut = Cut{};
    if (p.floats) return p;
    p.codes = round256((size_t)M * p.blocks * 16);
    p.scales = round256((size_t)M * p.blocks);
    return p;
}

template <typename T>
static void mx4_launch(const Cut &c, const Mx4Args &a, hipStream_t st)
{
    const dim3 grid(workgroups(a.grid));
    if (c.size == 0) hipLaunchKernelGGL((mx4_product_kernel<1, 1, 2, 2, 4, T>), grid, dim3(256), 0, st, a);
    else if (c.size == 1) hipLaunchKernelGGL((mx4_product_kernel<2, 2, 2, 2, 4, T>), grid, dim3(256), 0, st, a);
    else if (c.size == 2) hipLaunchKernelGGL((mx4_product_kernel<4, 2, 2, 4, 2, T>), grid, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((mx4_product_kernel<2, 2, 2, 2, 2, T>), grid, dim3(256), 0, st, a);
}

template <typename T>
static void few_launch(const Mx4Args &a, const void *x, lp_dtype xt, size_t ldx, hipStream_t st)
{
    const dim3 grid((unsigned)((a.N + 15) / 16)), block(kFewWaves * 64);
    if (a.xs) {
        hipLaunchKernelGGL((mx4_few_kernel<unsigned char, T>), grid, block, 0, st, a, (const unsigned char *)nullptr, ldx);
    } else {
        with_type(xt, [&](auto *tag) {
            typedef std::remove_pointer_t<decltype(tag)> X;
            hipLaunchKernelGGL((mx4_few_kernel<X, T>), grid, block, 0, st, a, (const X *)x, ldx);
        });
    }
}

static Cut grad_cut(int I, int J, int C, bool weights)
{
    return cut_product(I, J, std::max((C + 63) / 64, 1), 1, 4, weights ? kWeightTiles : kInputTiles, 4);
}

template <bool WEIGHTS, typename T>
static void grad_launch(const Cut &c, const GradArgs &a, hipStream_t st)
{
    const dim3 grid(workgroups(a.grid));
    // Loads to LDS ask for words, and reach 2^31 bytes from a tile's first row.
    const bool words = aligned_to(a.dy, 4) && a.ld % 2 == 0 && a.ld < kNearRows;
#define LP_TILES(MB, NB, WM, WN)                                                                                                             \
    hipLaunchKernelGGL((words ? gradient_kernel<MB, NB, WM, WN, WEIGHTS, true, T> : gradient_kernel<MB, NB, WM, WN, WEIGHTS, false, T>), grid, \
                       dim3(WM * WN * 64), 0, st, a)
    if (c.size == 0) LP_TILES(1, 2, 2, 2);
    else if (c.size == 1) LP_TILES(2, 2, 2, 2);
    else LP_TILES(4, 2, 2, 4);
#undef LP_TILES
}

template <bool WEIGHTS>
static void gradient(const Cut &c, GradArgs a, lp_dtype t, const Sink &out, void *work, hipStream_t st)
{
    a.grid = c.grid;
    a.grid.sums = (float *)work;
    a.out = out;
    if (t == LP_F32) grad_launch<WEIGHTS, float>(c, a, st);
    else grad_launch<WEIGHTS, __bf16>(c, a, st);
    if (a.grid.parts > 1) join_parts(c, a.grid, t, out, a.I, a.J, st);
}

} // namespace lp

// ------------------------------------------------------------------------------------ C ABI

using namespace lp;

static lp_status workspace_status(size_t need, const void *workspace, size_t bytes)
{
    if (need && (!workspace || bytes < need)) return LP_EWORKSPACE;
    return need && !aligned16(workspace) ? LP_EINVAL : LP_OK;
}

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
    if (const lp_status s = workspace_status(p.total(), workspace_dev, workspace_bytes)) return s;
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
    a.K = K;
    a.blocks = (int)p.blocks;
    a.grid = p.cut.grid;
    if (!a.xs && !p.floats) {
        mx4_quantize_launch(x_dev, xt, (size_t)M, (size_t)K, ldx, work, work + p.codes, st);
        a.xc = work;
        a.xs = work + p.codes;
    }
    a.grid.sums = (float *)(work + p.codes + p.scales);
    a.out = Sink{y_dev, ldy, bias_dev, nullptr, act, 0};
    with_type(yt, [&](auto *tag) {
        typedef std::remove_pointer_t<decltype(tag)> T;
        if (p.few) few_launch<T>(a, x_dev, xt, ldx, st);
        else mx4_launch<T>(p.cut, a, st);
    });
    if (a.grid.parts > 1) join_parts(p.cut, a.grid, yt, a.out, M, Nout, st);
    return launch_status();
}

extern "C" lp_status lp_mx4_fc_dgrad_workspace_bytes(int M, int K, int Nout, size_t *bytes_host)
{
    if (!bytes_host || !sizes_ok(M, K, Nout)) return LP_EINVAL;
    if (!sizes_taken(M, K, Nout)) return LP_EUNSUPPORTED;
    *bytes_host = M ? grad_cut(M, K, Nout, false).sums : 0;
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
    const Cut c = grad_cut(M, K, Nout, false);
    if (const lp_status s = workspace_status(c.sums, workspace_dev, workspace_bytes)) return s;
    clear_stale_error();
    GradArgs a = {};
    a.dy = (const __bf16 *)dy_dev;
    a.ld = lddy;
    a.codes = (const unsigned char *)w_codes_dev;
    a.scales = (const unsigned char *)w_scales_dev;
    a.I = M;
    a.J = K;
    a.C = Nout;
    a.blocks = (int)mx4_blocks((size_t)K);
    gradient<false>(c, a, dxt, Sink{dx_dev, lddx, nullptr, nullptr, LP_ACT_NONE, 0}, workspace_dev, as_stream(stream));
    return launch_status();
}

extern "C" lp_status lp_ckpt8_fc_wgrad_workspace_bytes(int M, int K, int Nout, size_t *bytes_host)
{
    if (!bytes_host || !sizes_ok(M, K, Nout)) return LP_EINVAL;
    if (!sizes_taken(M, K, Nout)) return LP_EUNSUPPORTED;
    *bytes_host = grad_cut(Nout, K, M, true).sums;
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
    const Cut c = grad_cut(Nout, K, M, true);
    if (const lp_status s = workspace_status(c.sums, workspace_dev, workspace_bytes)) return s;
    clear_stale_error();
    GradArgs a = {};
    a.dy = (const __bf16 *)dy_dev;
    a.ld = lddy;
    a.codes = (const unsigned char *)x_codes_dev;
    a.scales = (const unsigned char *)x_scales_dev;
    a.I = Nout;
    a.J = K;
    a.C = M;
    a.blocks = (int)ckpt8_blocks((size_t)K);
    gradient<true>(c, a, dwt, Sink{dw_dev, lddw, nullptr, dbias_dev, LP_ACT_NONE, accumulate != 0}, workspace_dev, as_stream(stream));
    return launch_status();
}
