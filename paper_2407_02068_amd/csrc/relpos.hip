// relpos.hip -- attention with a learned relative position bias (gfx950): forward and
// gradients.
//
// Per sequence and head h, over T tokens:
//   s_ij = q_i . k_j / sqrt(hd) + table[index_ij][h],  P = softmax over j,  O = P V
// and, for dO = dL/dO with D_i = sum_j P_ij dP_ij = dO_i . O_i, dP = dO V^T,
//   dS = P (dP - D),  dV = P^T dO,  dQ = dS K / sqrt(hd),  dK = dS^T Q / sqrt(hd),
//   dtable[b][h] = sum over sequences and over the pairs with index_ij = b of dS_ij.
// A pair takes no part where its index is -1, its bias -inf or the type's lowest value,
// or its tokens' region labels differ or are negative; a row without pairs gives zeros.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "lpv_attention.h"
#include "lpv_grid.h"
#include "lpv_internal.h"

namespace lpv {
namespace {

constexpr float LAZY = 8.0f;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// What the kernels read: qkv rows of the framework's layout, region labels.
struct Rp {
    const uint16_t* qkv;
    int64_t ldq;
    const int32_t* region;  // n_region x T, or NULL
    int64_t n_region, n_seq;
    int32_t T, H, nt;  // nt: tiles of 32 tokens
    const float* bias;  // tiles of the bias (k_relpos_bias)
};

// The labels of a sequence (n_seq and n_region are below 2^31).
__device__ inline const int32_t* labels(const Rp& p, int64_t seq)
{
    return p.region + (int64_t)((uint32_t)seq % (uint32_t)p.n_region) * p.T;
}

template <int HD> struct Row {
    static constexpr int KS = HD / 16;     // 16-dimension steps of a product over the head
    static constexpr int DT = HD / 32;     // 32-dimension tiles of an output
    static constexpr int RS = HD * 2 + 16; // bytes per staged row: 16 consecutive rows of one
                                           // 16-byte column sit in distinct banks
};

// The wave's number in the workgroup, as the uniform value that it is.
__device__ inline int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

__device__ inline uint32_t lds32(const void* p)
{
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// A tile's bias in matrix-core accumulator order, times sqrt(hd) (so that it is the
// accumulator's start value), -inf where the pair takes no part.  idx: Tp x Tp, -1 past T.
// Tile (a, b): rows 32 a of idx, columns 32 b; lane l holds row l % 32 and, in element r,
// column 8 (r / 4) + 4 (l / 32) + r % 4; in memory [r / 4][lane][r % 4], so that a wave's
// loads and stores are whole lines.

// A bias as the accumulator's start.  Finite ones saturate at 2^15: in a row whose every pair
// has one of -1e9, say, the weights would be differences of numbers whose float32 steps are
// far over 1, and infinite where the gradients take them from lse; at 2^15 they are right to 2^-9.
constexpr float MOST_BIAS = 32768.0f;
template <int DT> __device__ inline float ready_bias(uint16_t t, float root)
{
    constexpr uint16_t LOWEST = DT == LPV_BF16 ? 0xff7f : 0xfbff, NEG_INF = DT == LPV_BF16 ? 0xff80 : 0xfc00;
    return t == LOWEST || t == NEG_INF ? -INFINITY
                                       : fminf(fmaxf(Elem<DT>::to_f32(t), -MOST_BIAS), MOST_BIAS) * root;
}

// Elements 4 g .. 4 g + 3 of this lane.
template <int DT>
__device__ inline float4 gather_bias(const uint16_t* idx, int nt, int a, int b, int g, int lane,
                                     const uint16_t* table, int H, int h, float root)
{
    constexpr uint16_t NEG_INF = DT == LPV_BF16 ? 0xff80 : 0xfc00;
    const uint2 v = *(const uint2*)(idx + ((int64_t)a * 32 + (lane & 31)) * (nt * 32) + b * 32 + 4 * (lane >> 5) + 8 * g);
    const uint16_t* e = (const uint16_t*)&v;
    float4 o;
    float* of = (float*)&o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint16_t t = e[j] == 0xffff ? NEG_INF : table[(int64_t)e[j] * H + h];
        of[j] = ready_bias<DT>(t, root);
    }
    return o;
}

// D = dO . O of every row and head, hd / 8 lanes to a row, by `wgs` workgroups.  (4 x 777
// tokens, 8 heads of 64: beside the bias's tiles 1 us, in a launch of its own 4.)
struct RowsCall {
    const uint16_t *out, *dout;
    int64_t ldo, ldg, M;
    int32_t T;
    float* Dv;
};
template <int DT, int HD> __device__ inline void row_products(const RowsCall& c, int H, uint32_t wg, uint32_t wgs)
{
    using F = typename Elem<DT>::frag;
    constexpr int CH = HD / 8;
    // (the lanes of a row leave together)
    for (int64_t i = (int64_t)wg * 256 + threadIdx.x; i / CH < c.M * H; i += (int64_t)wgs * 256) {
        const int64_t r = i / CH, row = r / H, seq = row / c.T;
        const int h = (int)(r - row * H), k = (int)(i % CH) * 8;
        const F g = *(const F*)(c.dout + row * c.ldg + h * HD + k), o = *(const F*)(c.out + row * c.ldo + h * HD + k);
        float v = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v = fmaf((float)g[j], (float)o[j], v);
#pragma unroll
        for (int d = 1; d < CH; d <<= 1)
            v += __shfl_xor(v, d, 64);
        if (k == 0)
            c.Dv[(seq * H + h) * c.T + (row - seq * c.T)] = v;
    }
}

// The bias tiles of every head: blockIdx.z 0 those of idx, 1 those of its transpose; 2 (with
// HD): the rows' products, which the gradients that take both wait for as well.  A
// workgroup takes a head and `per` tiles; a head's column of the table is made ready in
// LDS once, where its gathers cost no more than reads of consecutive values do (the lanes of
// a tile's row differ by a constant in most indexes); larger tables are gathered in memory.
// (Forward of 8 x 1024 tokens, 12 heads, 2000 buckets: 61 us, 71 gathered; 11000: 84 and 88.)
// Bound: writes.  1025 tokens, 12 heads (52 MB): 18 us, 2.9 TB/s; more tiles or threads to a
// workgroup, or the next tile's buckets asked for ahead, gained there what they lost on
// smaller ones.
constexpr int BIAS_LDS = 12288;  // buckets

template <int DT, int HD>
__global__ __launch_bounds__(256) void k_relpos_bias(const uint16_t* __restrict__ idx,
                                                     const uint16_t* __restrict__ idx_t, int32_t nt,
                                                     const uint16_t* __restrict__ table, int32_t n_buckets,
                                                     int32_t H, float root, int32_t per,
                                                     float* __restrict__ bias, float* __restrict__ bias_t,
                                                     RowsCall rows)
{
    extern __shared__ float column[];  // n_buckets, or none
    if constexpr (HD > 0) {
        if (blockIdx.z == 2) {
            row_products<DT, HD>(rows, H, blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y);
            return;
        }
    }
    const int n_tiles = nt * nt, h = blockIdx.y, lane = threadIdx.x & 63;
    if ((int)blockIdx.x * per >= n_tiles)
        return;
    const bool in_lds = n_buckets <= BIAS_LDS;
    if (in_lds) {
        for (int i = threadIdx.x; i < n_buckets; i += 256)
            column[i] = ready_bias<DT>(table[(int64_t)i * H + h], root);
        __syncthreads();
    }
    const uint16_t* from = blockIdx.z ? idx_t : idx;
    float* to = (blockIdx.z ? bias_t : bias) + (int64_t)h * n_tiles * 1024 + lane * 4;
    const int end = min(((int)blockIdx.x + 1) * per, n_tiles);
    for (int tile = blockIdx.x * per + wave_id(); tile < end; tile += 4) {
        const int a = tile / nt, b = tile - a * nt;
        const uint16_t* src = from + ((int64_t)a * 32 + (lane & 31)) * (nt * 32) + b * 32 + 4 * (lane >> 5);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float4 o;
            if (in_lds) {
                const uint2 v = *(const uint2*)(src + 8 * g);
                const uint32_t e[4] = {v.x & 0xffffu, v.x >> 16, v.y & 0xffffu, v.y >> 16};
                float* of = (float*)&o;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    of[j] = e[j] == 0xffffu ? -INFINITY : column[e[j]];
            } else {
                o = gather_bias<DT>(from, nt, a, b, g, lane, table, H, h, root);
            }
            *(float4*)(to + (int64_t)tile * 1024 + 256 * g) = o;
        }
    }
}

__device__ inline f32x16 load_bias(const float* p)
{
    f32x16 s;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const float4 v = *(const float4*)(p + 256 * g);
        s[4 * g] = v.x;
        s[4 * g + 1] = v.y;
        s[4 * g + 2] = v.z;
        s[4 * g + 3] = v.w;
    }
    return s;
}

// A chunk of a row, or zero for a padding token's.
template <bool REG> __device__ inline uint4 unless_padding(uint4 v, int lab)
{
    if (REG && lab < 0)
        v = uint4{0u, 0u, 0u, 0u};
    return v;
}

// ROWS rows of a head's slices of two matrices, from global memory through registers into
// LDS, zero past T and for padding tokens (whose values, NaN too, then reach nothing).
template <int HD, int NT, int ROWS, bool REG> struct Stage {
    static constexpr int CH = HD / 8;                    // 16-byte chunks per row
    static constexpr int N = (ROWS * CH + NT - 1) / NT;   // chunks per thread and matrix
    uint4 a[N], b[N];
    int lab[N];  // the rows' labels: asked for beside them, so that neither waits for the other
    __device__ inline void load(const uint16_t* pa, int64_t lda, const uint16_t* pb, int64_t ldb,
                                int row0, int T, const int32_t* reg)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * NT, r = row0 + c / CH, k = c % CH;
            a[i] = uint4{0u, 0u, 0u, 0u};
            b[i] = uint4{0u, 0u, 0u, 0u};
            lab[i] = 0;
            if (r < T && c < ROWS * CH) {
                a[i] = *(const uint4*)(pa + (int64_t)r * lda + 8 * k);
                b[i] = *(const uint4*)(pb + (int64_t)r * ldb + 8 * k);
                if (REG)
                    lab[i] = reg[r];
            }
        }
    }
    __device__ inline void store(char* la, char* lb) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * NT;
            const uint4 va = unless_padding<REG>(a[i], lab[i]), vb = unless_padding<REG>(b[i], lab[i]);
            if (ROWS * CH % NT == 0 || c < ROWS * CH) {
                *(uint4*)(la + c / CH * Row<HD>::RS + 16 * (c % CH)) = va;
                *(uint4*)(lb + c / CH * Row<HD>::RS + 16 * (c % CH)) = vb;
            }
        }
    }
};

// A fragment of 8 head dimensions (8 half + 16 ks ..) of one row per lane, zero unless ok
// (the row, which exists, is read either way: it does not wait for its label).
template <typename F, int HD>
__device__ inline void load_frags(F* f, const uint16_t* row, int half, bool ok)
{
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks)
        f[ks] = as_frag<F>(unless_padding<true>(*(const uint4*)(row + 8 * half + 16 * ks), ok ? 0 : -1));
}

// This lane's address for transposing reads of row-major staged rows: 16-lane group g
// takes dimensions 16 (g % 2) + 0..15 and rows 4 (g / 2) + 0..3.
template <int HD> __device__ inline uint32_t tr_base(const char* p, int lane)
{
    const int g = lane >> 4, j = lane & 15;
    return lds32(p) + ((j >> 2) + 4 * (g >> 1)) * Row<HD>::RS + (16 * (g & 1) + 4 * (j & 3)) * 2;
}

// The matrix-core operand of 16 rows (their slots in accumulator order) of 32 dimensions.
template <typename F, int HD> __device__ inline F tr_frag(uint32_t base, int row, int dt)
{
    const uint32_t at = base + row * Row<HD>::RS + 64 * dt;
    const uint2 lo = att_tr_read(at), hi = att_tr_read(at + 8 * Row<HD>::RS);
    return as_frag<F>(uint4{lo.x, lo.y, hi.x, hi.y});
}

// The maximum, or sum, of a value in lanes l and l ^ 32.
__device__ inline float half_max(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float half_add(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// s = -inf where the labels of this lane's token and of the element's differ.
__device__ inline void mask_region(f32x16& s, int mine, const int32_t* lab, int half)
{
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int4 o = *(const int4*)(lab + 8 * g + 4 * half);
        s[4 * g] = o.x == mine ? s[4 * g] : -INFINITY;
        s[4 * g + 1] = o.y == mine ? s[4 * g + 1] : -INFINITY;
        s[4 * g + 2] = o.z == mine ? s[4 * g + 2] : -INFINITY;
        s[4 * g + 3] = o.w == mine ? s[4 * g + 3] : -INFINITY;
    }
}

// What the labels of 32 rows have in common: their value, DEAD (all padding) or MIXED.  lab:
// this lane's row's (negative: -1); lanes 0-31 and 32-63 are a tile each.
constexpr int32_t DEAD = -1, MIXED = -2;
__device__ inline int32_t tile_state(int32_t lab, int half)
{
    const int32_t first = __shfl(lab, 32 * half, 64);
    return (uint32_t)(__ballot(lab == first) >> (32 * half)) == 0xffffffffu ? first : MIXED;
}

// The label of a padding token as the one that attends; as the one attended it is -1, so
// that the two never match.
constexpr int32_t NO_LABEL = INT32_MIN;

// 32 rows of an output whose accumulators hold one row per lane (l % 32), dimensions
// 8 (r / 4) + 4 half + r % 4 of each 32-dimension tile: lanes l and l ^ 32 swap halves, so
// that each stores 16 bytes at a time.
template <int DT, int HD>
__device__ inline void store_rows(uint16_t* row, const f32x16* o, float f, int half)
{
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            uint32_t w[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    w[i][j] = pack2<DT>(o[dt][4 * (g + i) + 2 * j] * f, o[dt][4 * (g + i) + 2 * j + 1] * f);
            const auto x = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
            *(uint4*)(row + 32 * dt + 8 * g + 8 * half) = uint4{x[0], y[0], x[1], y[1]};
        }
}

// How a workgroup of the general kernels is laid out: QW 32-row tiles of one sequence and
// head, KS waves to each; the other side's rows pass in blocks of 64, of which a wave takes
// NI 32-row tiles.
template <int QW_, int KS_> struct Shape {
    static constexpr int QW = QW_, KS = KS_, NW = QW_ * KS_, NT = 64 * NW, B = 64, NI = 2 / KS_;
};

// Workgroups of a launch in an order in which each XCD (workgroup L runs on XCD L % 8) takes
// one run of neighbours, which find each other's rows and bias in its L2.  (8 x 1000 tokens,
// 12 heads of 64: forward 59 us, 80 in the launch's order; gradients 230 and 247.)
__device__ inline uint32_t xcd_order(uint32_t n, uint32_t id)
{
    const uint32_t per = n / 8, rest = n % 8, x = id % 8;
    return id < n ? x * per + min(x, rest) + id / 8 : n;
}

// Workgroup -> (sequence, head, block of row tiles).  A head's blocks of a sequence follow
// each other while its bias is small (they share K and V); else the sequences of a block do
// (they share its bias: 4 KB a pair of tiles).  Gradients of 64 x 300 tokens, 12 heads:
// 196 us the first way, 205 the second; of 4 x 2000 tokens 650 and 633; 8 x 1000: the same.
constexpr int BIAS_SMALL = 256;  // tiles of a head's bias: 1 MB
struct Place {
    int64_t seq;
    int h, blk;
};
__device__ inline Place place(const Rp& p, int n_blk, uint32_t id)
{
    const uint32_t seqs = (uint32_t)p.n_seq;
    const uint32_t inner = p.nt * p.nt <= BIAS_SMALL ? (uint32_t)n_blk : seqs;
    const uint32_t u = id / inner, in = id - u * inner;
    const uint32_t outer = p.nt * p.nt <= BIAS_SMALL ? seqs : (uint32_t)n_blk;
    const uint32_t h = u / outer, out = u - h * outer;
    return p.nt * p.nt <= BIAS_SMALL ? Place{(int64_t)out, (int)h, (int)in}
                                     : Place{(int64_t)in, (int)h, (int)out};
}

// The label of a token that attends (mine) or is attended (theirs); 0 without labels.
template <bool REG> __device__ inline int label_mine(const int32_t* reg, int i)
{
    return !REG ? 0 : reg[i] < 0 ? NO_LABEL : reg[i];
}

// The pipeline of a general kernel: the next block's rows are in flight while a block is
// worked on, and the bias of the next tile.  step(first row of the tile in the block, the
// block's rows in LDS, block % 2, the tile's bias) takes a tile; load_more(block) and
// store_more(buffer) go along with the rows.  (In a block the bias is asked for before the
// rows, so that its wait is not for those.  Two blocks ahead, and the bias two tiles, cost a
// third of the waves: 64 x 197 tokens x 12 heads of 64 35.4 us against 29.0.)
template <int HD, typename Sh, bool REG, typename LoadMore, typename StoreMore, typename Step>
__device__ inline void pass_blocks(const Rp& p, const uint16_t* a, int64_t lda, const uint16_t* b,
                                   int64_t ldb, const int32_t* reg, const float* bias, bool busy, int part,
                                   char* buf, LoadMore&& load_more, StoreMore&& store_more, Step&& step)
{
    constexpr int HALF = Sh::B * Row<HD>::RS;  // buf: [2][2][HALF]
    constexpr int NI = Sh::NI;
    const int n_b = (p.T + Sh::B - 1) / Sh::B;
    Stage<HD, Sh::NT, Sh::B, REG> st;
    auto load_tile = [&](int blk, int i) {
        return load_bias(bias + (int64_t)min(blk * NI * Sh::KS + part + i, p.nt - 1) * 1024);
    };
    f32x16 next = load_tile(0, 0);
    st.load(a, lda, b, ldb, 0, p.T, reg);
    load_more(0);
    st.store(buf, buf + HALF);
    store_more(0);
    __syncthreads();
    for (int blk = 0; blk < n_b; ++blk) {
        char* at = buf + (blk & 1) * 2 * HALF;
        char* to = buf + (~blk & 1) * 2 * HALF;
        const bool more = blk + 1 < n_b;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const f32x16 cur = next;
            next = i + 1 < NI ? load_tile(blk, i + 1) : load_tile(blk + 1, 0);
            if (i == 0 && more) {
                st.load(a, lda, b, ldb, (blk + 1) * Sh::B, p.T, reg);
                load_more(blk + 1);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (busy && blk * NI * Sh::KS + part + i < p.nt)
                step(32 * (part + i), at, at + HALF, blk & 1, cur);
        }
        if (more) {
            st.store(to, to + HALF);
            store_more(~blk & 1);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- forward

// A wave holds a 32-query tile; the keys pass in blocks through a double buffer in LDS.
// S^T = K Q^T starts from the bias in the accumulator, so a row of the softmax lives in
// lanes l and l ^ 32; the weights, rounded once to the element type, are then the B operand
// of O^T = V^T P^T (V^T by transposing LDS reads).  The row's sum adds the weights before
// that rounding, so that lse is exact to float32; each lane adds its own, the two of a row
// meet at the end.  With KS = 2 two waves share a tile's keys and join their rows in LDS.
// Bound: waits between a tile's dependent steps at three waves to a SIMD (the softmax's vector
// instructions take 37% of a SIMD's time, the matrix cores 14%).  64 x 197 tokens, 12 heads
// of 64: 28 us, 272 TFLOP/s; 8 x 1025, fp16, padded: 62 us, 417 TFLOP/s.  Four waves to a
// SIMD, at 128 registers, gained nothing (28.9 and 68), nor did five to a workgroup (64 x 144
// tokens, 12 heads of 64: 26.0, four 24.0, three 22.9).
template <int DT, int HD, typename Sh, bool REG>
__global__ __launch_bounds__(Sh::NT, HD == 32 ? 4 : 3) void k_relpos_fwd(Rp p, uint16_t* __restrict__ out, int64_t ldo,
                                                       float* __restrict__ lse, float scale)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS, ND = Row<HD>::DT;
    __shared__ __attribute__((aligned(16))) char kv[4 * Sh::B * RS];
    __shared__ __attribute__((aligned(16))) int32_t lab[2][Sh::B];
    __shared__ int32_t states[2][2];
    static_assert(Sh::B == 64, "a wave stages a block's labels");
    const int T = p.T;
    const int n_blk = (p.nt + Sh::QW - 1) / Sh::QW;
    const uint32_t n = (uint32_t)p.n_seq * (uint32_t)(p.H * n_blk);
    const uint32_t id = xcd_order(n, blockIdx.y * gridDim.x + blockIdx.x);  // (below 2^31 + 2^20)
    if (id >= n)
        return;
    const Place at = place(p, n_blk, id);
    const int lane = threadIdx.x & 63, wave = wave_id(), l32 = lane & 31, half = lane >> 5;
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    const uint16_t* base = p.qkv + at.seq * T * ldq + at.h * HD;
    const int32_t* reg = REG ? labels(p, at.seq) : nullptr;
    const int part = wave % Sh::KS, qt = at.blk * Sh::QW + wave / Sh::KS, q = qt * 32 + l32;
    const bool busy = qt < p.nt;
    const int mine = label_mine<REG>(reg, min(q, T - 1));
    const bool steps = busy && (!REG || !__all(mine == NO_LABEL));
    F qf[KS];
    load_frags<F, HD>(qf, base + (int64_t)min(q, T - 1) * ldq, half, busy && mine != NO_LABEL);
    f32x16 o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
        o[d] = f32x16{};
    float m = -INFINITY, l = 0.0f;
    int32_t lv = -1;
    pass_blocks<HD, Sh, REG>(
        p, base + hw, ldq, base + 2 * hw, ldq, reg,
        p.bias + ((int64_t)at.h * p.nt + min(qt, p.nt - 1)) * p.nt * 1024 + lane * 4, steps, part, kv,
        [&](int blk) {
            const int r = blk * Sh::B + threadIdx.x;
            if (REG && threadIdx.x < Sh::B)
                lv = r < T ? max(reg[r], -1) : -1;
        },
        [&](int b) {
            if (REG && wave == 0) {
                lab[b][lane] = lv;
                states[b][half] = tile_state(lv, half);
            }
        },
        [&](int row0, const char* kb, const char* vb, int b, const f32x16& bias) {
            const uint32_t ka = lds32(kb) + (row0 + l32) * RS + half * 16;
            const uint32_t va = tr_base<HD>(vb, lane) + row0 * RS;
            const int state = REG ? states[b][row0 / 32] : 0;
            if (REG && state == DEAD)
                return;
            f32x16 s = bias;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                s = E::mma(att_frag<F>(ka + 32 * ks), qf[ks], s);
            if (REG && !__all(mine == state))
                mask_region(s, mine, lab[b] + row0, half);
            float t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                t[j] = fmaxf(fmaxf(s[j], s[j + 4]), fmaxf(s[j + 8], s[j + 12]));
            float mt = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
            mt = half_max(mt);
            // the weights' reference m follows a row's maximum when that is over 2^8 weights
            // above it: most tiles then need no rescaling (each row by its own scores)
            const bool far = mt > m + LAZY / scale;
            if (__any(far)) {
                const float alpha = far ? __builtin_amdgcn_exp2f((m - mt) * scale) : 1.0f;
                m = far ? mt : m;
                l *= alpha;
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[d] *= alpha;
            }
            const float nms = m == -INFINITY ? 0.0f : -m * scale;  // (nothing yet: all weights 0)
            float ps[2] = {0.0f, 0.0f};
            uint32_t pb[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e0 = __builtin_amdgcn_exp2f(fmaf(s[2 * j], scale, nms));
                const float e1 = __builtin_amdgcn_exp2f(fmaf(s[2 * j + 1], scale, nms));
                ps[0] += e0;
                ps[1] += e1;
                pb[j] = pack2<DT>(e0, e1);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const F pf = as_frag<F>(uint4{pb[4 * u], pb[4 * u + 1], pb[4 * u + 2], pb[4 * u + 3]});
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[d] = E::mma(tr_frag<F, HD>(va, 16 * u, d), pf, o[d]);
            }
            l += ps[0] + ps[1];
        });
    l = half_add(l);
    if constexpr (Sh::KS == 2) {  // (every wave has left the blocks)
        float* j = (float*)kv + (wave / 2) * (ND * 16 + 2) * 64 + lane;
        static_assert(Sh::QW * (ND * 16 + 2) * 256 <= (int)sizeof(kv), "the joined rows fit");
        if (part == 1) {
            j[0] = m;
            j[64] = l;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    j[64 * (2 + 16 * d + r)] = o[d][r];
        }
        __syncthreads();
        if (part == 1)
            return;
        const float m1 = j[0], mn = fmaxf(m, m1), ref = mn == -INFINITY ? 0.0f : mn;
        const float a0 = __builtin_amdgcn_exp2f((m - ref) * scale), a1 = __builtin_amdgcn_exp2f((m1 - ref) * scale);
        m = mn;
        l = l * a0 + j[64] * a1;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                o[d][r] = o[d][r] * a0 + j[64 * (2 + 16 * d + r)] * a1;
    }
    if (busy && q < T) {
        store_rows<DT, HD>(out + (at.seq * T + q) * ldo + at.h * HD, o, l > 0.0f ? 1.0f / l : 0.0f, half);
        if (lse && half == 0)
            lse[(at.seq * p.H + at.h) * T + q] = l > 0.0f ? LN2 * (m * scale + __log2f(l)) : -INFINITY;
    }
}

// ---------------------------------------------------------------- gradients

// Adds the accumulators of the second of two waves to the first's; false for the second.
template <int N> __device__ inline bool join_sums(char* buf, f32x16* o, int wave)
{
    float* j = (float*)buf + (wave / 2) * N * 1024 + (threadIdx.x & 63);
    if (wave % 2) {
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                j[64 * (16 * d + r)] = o[d][r];
    }
    __syncthreads();
    if (wave % 2)
        return false;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            o[d][r] += j[64 * (16 * d + r)];
    return true;
}

// What the gradient kernels take beside Rp.
struct Gp {
    const float* lse;
    const float* Dv;  // dO . O of each row, in lse's layout (anything for a row without pairs)
    float* Dc;        // the same without the rounding of O: grad_q's, for the bias's sums
    const uint16_t* dout;
    int64_t ldg;
    uint16_t* dqkv;
    int64_t lddq;
    const float* bias_t;  // the bias of the transposed index
    float* part;
    int32_t chunks;
    float scale, rroot;
};

// LDS of a workgroup of the general gradients, whichever part it does.
template <int HD> struct GradLds {
    __attribute__((aligned(16))) char rows[4 * 64 * Row<HD>::RS];
    __attribute__((aligned(16))) float stats[2][2][64];
    __attribute__((aligned(16))) int32_t lab[2][64];
    int32_t states[2][2];
};

// dQ, tiled as the forward: the weights come back from lse, dP^T = V dO^T, and dS^T,
// rounded once, is the B operand of dQ^T = K^T dS^T.  A row of dS sums to zero; what it sums
// to here is what D is off by, O having been rounded: with it D is right for the bias's sums.
template <int DT, int HD, typename Sh, bool REG>
__device__ inline void grad_q(const Rp& p, const Gp& c, uint32_t id, GradLds<HD>& sh)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS, ND = Row<HD>::DT;
    static_assert(Sh::B == 64, "a wave stages a block's labels");
    char* kv = sh.rows;
    auto& lab = sh.lab;
    auto& states = sh.states;
    const int64_t ldg = c.ldg, lddq = c.lddq;
    const float scale = c.scale, rroot = c.rroot;
    const int T = p.T;
    const Place at = place(p, (p.nt + Sh::QW - 1) / Sh::QW, id);
    const int lane = threadIdx.x & 63, wave = wave_id(), l32 = lane & 31, half = lane >> 5;
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    const uint16_t* base = p.qkv + at.seq * T * ldq + at.h * HD;
    const int32_t* reg = REG ? labels(p, at.seq) : nullptr;
    const int part = wave % Sh::KS, qt = at.blk * Sh::QW + wave / Sh::KS, q = qt * 32 + l32;
    const int qc = min(q, T - 1);
    const bool busy = qt < p.nt;
    const int mine = label_mine<REG>(reg, qc);
    const bool live = busy && mine != NO_LABEL, steps = busy && (!REG || !__all(mine == NO_LABEL));
    F qf[KS], gf[KS];
    load_frags<F, HD>(qf, base + (int64_t)qc * ldq, half, live);
    load_frags<F, HD>(gf, c.dout + (at.seq * T + qc) * ldg + at.h * HD, half, live);
    const int64_t stat = (at.seq * p.H + at.h) * T;
    // (a row without pairs, padding for one, whose D may be anything: every weight 2^-inf)
    const float v = c.lse[stat + qc], D = v == -INFINITY ? 0.0f : c.Dv[stat + qc];
    const float nl = v == -INFINITY ? -INFINITY : -v * LOG2E;
    f32x16 dq[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
        dq[d] = f32x16{};
    float off[2] = {0.0f, 0.0f};
    int32_t lv = -1;
    pass_blocks<HD, Sh, REG>(
        p, base + hw, ldq, base + 2 * hw, ldq, reg,
        p.bias + ((int64_t)at.h * p.nt + min(qt, p.nt - 1)) * p.nt * 1024 + lane * 4, steps, part, kv,
        [&](int blk) {
            const int r = blk * Sh::B + threadIdx.x;
            if (REG && threadIdx.x < Sh::B)
                lv = r < T ? max(reg[r], -1) : -1;
        },
        [&](int b) {
            if (REG && wave == 0) {
                lab[b][lane] = lv;
                states[b][half] = tile_state(lv, half);
            }
        },
        [&](int row0, const char* kb, const char* vb, int b, const f32x16& bias) {
            const uint32_t ka = lds32(kb) + (row0 + l32) * RS + half * 16;
            const uint32_t va = lds32(vb) + (row0 + l32) * RS + half * 16;
            const uint32_t kt = tr_base<HD>(kb, lane) + row0 * RS;
            const int state = REG ? states[b][row0 / 32] : 0;
            if (REG && state == DEAD)
                return;
            f32x16 s = bias, dp = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = E::mma(att_frag<F>(ka + 32 * ks), qf[ks], s);
                dp = E::mma(att_frag<F>(va + 32 * ks), gf[ks], dp);
            }
            if (REG && !__all(mine == state))
                mask_region(s, mine, lab[b] + row0, half);
            uint32_t db[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f0 = __builtin_amdgcn_exp2f(fmaf(s[2 * j], scale, nl)) * (dp[2 * j] - D);
                const float f1 = __builtin_amdgcn_exp2f(fmaf(s[2 * j + 1], scale, nl)) * (dp[2 * j + 1] - D);
                off[0] += f0;
                off[1] += f1;
                db[j] = pack2<DT>(f0, f1);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const F df = as_frag<F>(uint4{db[4 * u], db[4 * u + 1], db[4 * u + 2], db[4 * u + 3]});
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    dq[d] = E::mma(tr_frag<F, HD>(kt, 16 * u, d), df, dq[d]);
            }
        });
    float miss = half_add(off[0] + off[1]);
    if constexpr (Sh::KS == 2) {
        static_assert(Sh::QW * ND * 4096 <= (int)sizeof(sh.rows), "the joined rows fit");
        float* other = (float*)sh.stats + wave / 2 * 32 + l32;
        if (part == 1 && half == 0)
            *other = miss;
        if (!join_sums<ND>(kv, dq, wave))
            return;
        miss += *other;
    }
    if (busy && q < T) {
        store_rows<DT, HD>(c.dqkv + (at.seq * T + q) * lddq + at.h * HD, dq, rroot, half);
        if (half == 0)
            c.Dc[stat + q] = D + miss;
    }
}

// dK and dV: a wave holds a 32-key tile, the queries pass in blocks with their lse and D.
// S = Q K^T and dP = dO V^T (lane = key) make P and dS the B operands of dV^T = dO^T P and
// dK^T = Q^T dS as they stand.  The bias tiles are those of the transposed index.
template <int DT, int HD, typename Sh, bool REG>
__device__ inline void grad_kv(const Rp& p, const Gp& c, uint32_t id, GradLds<HD>& sh)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS, ND = Row<HD>::DT;
    char* qg = sh.rows;
    auto& stats = sh.stats;
    auto& lab = sh.lab;
    auto& states = sh.states;
    const int64_t ldg = c.ldg, lddq = c.lddq;
    const float scale = c.scale, rroot = c.rroot;
    const int T = p.T;
    const Place at = place(p, (p.nt + Sh::QW - 1) / Sh::QW, id);
    const int lane = threadIdx.x & 63, wave = wave_id(), l32 = lane & 31, half = lane >> 5;
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    const uint16_t* base = p.qkv + at.seq * T * ldq + at.h * HD;
    const int32_t* reg = REG ? labels(p, at.seq) : nullptr;
    const int part = wave % Sh::KS, kt = at.blk * Sh::QW + wave / Sh::KS, k = kt * 32 + l32;
    const int kc = min(k, T - 1);
    const bool busy = kt < p.nt;
    const int mine = label_mine<REG>(reg, kc);
    const bool live = busy && k < T && mine != NO_LABEL;
    const bool steps = busy && (!REG || !__all(mine == NO_LABEL));
    F kf[KS], vf[KS];
    load_frags<F, HD>(kf, base + hw + (int64_t)kc * ldq, half, live);
    load_frags<F, HD>(vf, base + 2 * hw + (int64_t)kc * ldq, half, live);
    const int64_t stat = (at.seq * p.H + at.h) * T;
    f32x16 acc[2 * ND];  // dK, dV
#pragma unroll
    for (int d = 0; d < 2 * ND; ++d)
        acc[d] = f32x16{};
    float sl, sd;
    int32_t lv;
    pass_blocks<HD, Sh, REG>(
        p, base, ldq, c.dout + at.seq * T * ldg + at.h * HD, ldg, reg,
        c.bias_t + ((int64_t)at.h * p.nt + min(kt, p.nt - 1)) * p.nt * 1024 + lane * 4, steps, part, qg,
        [&](int blk) {
            // -lse in base 2 (-inf past T and for rows without pairs: every weight 0), D, label
            sl = -INFINITY;
            sd = 0.0f;
            lv = -1;
            const int r = blk * Sh::B + threadIdx.x;
            if (threadIdx.x < Sh::B && r < T) {
                const float v = c.lse[stat + r];
                sl = v == -INFINITY ? -INFINITY : -v * LOG2E;
                sd = v == -INFINITY ? 0.0f : c.Dv[stat + r];
                if (REG)
                    lv = max(reg[r], -1);
            }
        },
        [&](int b) {
            if (wave == 0) {
                stats[b][0][lane] = sl;
                stats[b][1][lane] = sd;
                if (REG) {
                    lab[b][lane] = lv;
                    states[b][half] = tile_state(lv, half);
                }
            }
        },
        [&](int row0, const char* qb, const char* gb, int b, const f32x16& bias) {
            const uint32_t qa = lds32(qb) + (row0 + l32) * RS + half * 16;
            const uint32_t ga = lds32(gb) + (row0 + l32) * RS + half * 16;
            const uint32_t qtr = tr_base<HD>(qb, lane) + row0 * RS;
            const uint32_t gtr = tr_base<HD>(gb, lane) + row0 * RS;
            const int state = REG ? states[b][row0 / 32] : 0;
            if (REG && state == DEAD)
                return;
            f32x16 s = bias, dp = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = E::mma(att_frag<F>(qa + 32 * ks), kf[ks], s);
                dp = E::mma(att_frag<F>(ga + 32 * ks), vf[ks], dp);
            }
            if (REG && !__all(mine == state))
                mask_region(s, mine, lab[b] + row0, half);
            uint32_t pb[8], db[8];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 nl = *(const float4*)(stats[b][0] + row0 + 8 * g + 4 * half);
                const float4 D = *(const float4*)(stats[b][1] + row0 + 8 * g + 4 * half);
                const float e0 = __builtin_amdgcn_exp2f(fmaf(s[4 * g], scale, nl.x));
                const float e1 = __builtin_amdgcn_exp2f(fmaf(s[4 * g + 1], scale, nl.y));
                const float e2 = __builtin_amdgcn_exp2f(fmaf(s[4 * g + 2], scale, nl.z));
                const float e3 = __builtin_amdgcn_exp2f(fmaf(s[4 * g + 3], scale, nl.w));
                pb[2 * g] = pack2<DT>(e0, e1);
                pb[2 * g + 1] = pack2<DT>(e2, e3);
                db[2 * g] = pack2<DT>(e0 * (dp[4 * g] - D.x), e1 * (dp[4 * g + 1] - D.y));
                db[2 * g + 1] = pack2<DT>(e2 * (dp[4 * g + 2] - D.z), e3 * (dp[4 * g + 3] - D.w));
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const F pf = as_frag<F>(uint4{pb[4 * u], pb[4 * u + 1], pb[4 * u + 2], pb[4 * u + 3]});
                const F df = as_frag<F>(uint4{db[4 * u], db[4 * u + 1], db[4 * u + 2], db[4 * u + 3]});
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    acc[d] = E::mma(tr_frag<F, HD>(qtr, 16 * u, d), df, acc[d]);
                    acc[ND + d] = E::mma(tr_frag<F, HD>(gtr, 16 * u, d), pf, acc[ND + d]);
                }
            }
        });
    if constexpr (Sh::KS == 2) {
        static_assert(Sh::QW * 2 * ND * 4096 <= (int)sizeof(sh.rows), "the joined rows fit");
        if (!join_sums<2 * ND>(qg, acc, wave))
            return;
    }
    if (busy && k < T) {
        uint16_t* row = c.dqkv + (at.seq * T + k) * lddq + at.h * HD;
        store_rows<DT, HD>(row + hw, acc, rroot, half);
        store_rows<DT, HD>(row + 2 * hw, acc + ND, 1.0f, half);
    }
}

// Sum over a chunk of sequences of dS of one head's pairs, 64 x 64 pairs to a workgroup of
// four waves (a 32 x 32 tile each, summed in its accumulators' places in float32), the four
// matrices' rows staged in LDS a sequence ahead.  part: [head][chunk][tile][r / 4][lane][r % 4].
template <int DT, int HD, bool REG>
__device__ inline void grad_bias(const Rp& p, const Gp& c, const float* Dv, uint32_t id, char* lds)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS;
    char(&rows)[4][64 * RS] = *(char(*)[4][64 * RS])lds;  // Q, dO, K, V
    const int64_t ldg = c.ldg;
    const int32_t chunks = c.chunks;
    const float scale = c.scale;
    const int T = p.T, n_blk = (p.nt + 1) / 2;
    // (the blocks of pairs of one head and chunk follow each other: they share the rows)
    const uint32_t n2 = (uint32_t)(n_blk * n_blk);
    const uint32_t u = id / n2;
    const int ab = (int)(id - u * n2), h = (int)(u / (uint32_t)chunks), chunk = (int)(u - (uint32_t)(h * chunks));
    const int lane = threadIdx.x & 63, wave = wave_id(), l32 = lane & 31, half = lane >> 5;
    const int qb = ab / n_blk, kb = ab - qb * n_blk;
    const int qt = 2 * qb + (wave >> 1), kt = 2 * kb + (wave & 1);
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    const bool busy = qt < p.nt && kt < p.nt;
    const int q = qt * 32 + l32, qc = min(q, T - 1);
    const f32x16 bias = load_bias(
        p.bias + (((int64_t)h * p.nt + min(qt, p.nt - 1)) * p.nt + min(kt, p.nt - 1)) * 1024 + lane * 4);
    const int64_t s0 = p.n_seq * chunk / chunks, s1 = p.n_seq * (chunk + 1) / chunks;
    Stage<HD, 256, 64, REG> sq, sk;
    auto load = [&](int64_t seq) {
        const uint16_t* base = p.qkv + seq * T * ldq + h * HD;
        const int32_t* reg = REG ? labels(p, seq) : nullptr;
        sq.load(base, ldq, c.dout + seq * T * ldg + h * HD, ldg, qb * 64, T, reg);
        sk.load(base + hw, ldq, base + 2 * hw, ldq, kb * 64, T, reg);
    };
    f32x16 sum = {};
    if (s0 < s1)
        load(s0);
    const uint32_t qa = lds32(rows[0]) + ((wave >> 1) * 32 + l32) * RS + half * 16;
    const uint32_t ga = lds32(rows[1]) + ((wave >> 1) * 32 + l32) * RS + half * 16;
    const uint32_t ka = lds32(rows[2]) + ((wave & 1) * 32 + l32) * RS + half * 16;
    const uint32_t va = lds32(rows[3]) + ((wave & 1) * 32 + l32) * RS + half * 16;
    for (int64_t seq = s0; seq < s1; ++seq) {
        sq.store(rows[0], rows[1]);
        sk.store(rows[2], rows[3]);
        const int64_t stat = (seq * p.H + h) * T;
        const float v = c.lse[stat + qc], D = v == -INFINITY ? 0.0f : Dv[stat + qc];
        // (a query past T: every weight 2^-inf)
        const float nl = v == -INFINITY || q >= T ? -INFINITY : -v * LOG2E;
        __syncthreads();
        if (seq + 1 < s1)
            load(seq + 1);
        if (busy) {
            f32x16 s = bias, dp = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = E::mma(att_frag<F>(ka + 32 * ks), att_frag<F>(qa + 32 * ks), s);
                dp = E::mma(att_frag<F>(va + 32 * ks), att_frag<F>(ga + 32 * ks), dp);
            }
            if (REG) {
                const int32_t* reg = labels(p, seq);
                int mine = reg[qc];
                mine = mine < 0 ? NO_LABEL : mine;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int k = kt * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                    s[r] = max(reg[min(k, T - 1)], -1) == mine ? s[r] : -INFINITY;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r)
                sum[r] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[r], scale, nl)), dp[r] - D, sum[r]);
        }
        __syncthreads();
    }
    if (busy) {
        float* dst = c.part + (((int64_t)h * chunks + chunk) * p.nt * p.nt + (int64_t)qt * p.nt + kt) * 1024 +
                     lane * 4;
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(float4*)(dst + 256 * g) = float4{sum[4 * g], sum[4 * g + 1], sum[4 * g + 2], sum[4 * g + 3]};
    }
}

// All gradients of longer sequences in one launch, so that its parts fill the chip together:
// workgroups of dQ, then of dK and dV, then (unless n_pairs is 0) of the bias's.  Nine products
// of T^2 hd in all, of which five would do where dS could stay in registers.  Bound: chains of
// dependent steps at two waves to a SIMD (registers).  4 x 777 tokens, 8 heads of 64, distinct
// buckets along a row: 51 us, 435 TFLOP/s of the nine; in a launch each the parts made forward and
// gradients 115 us long, together 107.  With 32 buckets, whose sums follow: 36 and 18 us.
template <int DT, int HD, typename Sh, bool REG>
__global__ __launch_bounds__(256, 2) void k_relpos_grad(Rp p, Gp c, uint32_t n_tiles, uint32_t n_pairs)
{
    static_assert(Sh::NT == 256, "every part has 256 threads");
    __shared__ GradLds<HD> sh;
    // (each part's workgroups in runs per XCD: the counts but the last are multiples of 8)
    const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x, span = (n_tiles + 7) / 8 * 8;
    if (id < 2 * span) {
        const uint32_t i = xcd_order(n_tiles, id % span);
        if (i >= n_tiles)
            return;
        if (id < span)
            grad_q<DT, HD, Sh, REG>(p, c, i, sh);
        else
            grad_kv<DT, HD, Sh, REG>(p, c, i, sh);
    } else {
        const uint32_t i = xcd_order(n_pairs, id - 2 * span);
        if (i < n_pairs)
            grad_bias<DT, HD, REG>(p, c, c.Dv, i, sh.rows);
    }
}

// The bias's part alone, behind the others, with the D that grad_q has put right: for indexes
// with a row that gives some bucket several pairs, whose gradient D's error would show in (as
// in k_relpos_mid_grad).  8 x 1025 tokens, 12 heads of 64, a class token: 135 and 62 us, in one
// launch 195; 32 x 290: 64 and 25, in one 87.
template <int DT, int HD, bool REG>
__global__ __launch_bounds__(256) void k_relpos_pairs(Rp p, Gp c, uint32_t n_pairs)
{
    __shared__ __attribute__((aligned(16))) char rows[4 * 64 * Row<HD>::RS];
    const uint32_t i = xcd_order(n_pairs, blockIdx.y * gridDim.x + blockIdx.x);
    if (i < n_pairs)
        grad_bias<DT, HD, REG>(p, c, c.Dc, i, rows);
}

// The chunks' sums of each pair: CL threads of a workgroup share a pair's chunks (each in
// order, then the threads'), 4 pairs to a thread.  per > 0: of a head's slots, those that
// k_relpos_mid_grad's workgroups have filled, which take `per` of all heads' sequences each.
// CL = 16 from 16 chunks on: gradients of 64 x 100 tokens, 2 heads (65 chunks) 26 us, with
// CL = 1 39; of 64 x 300 tokens, 12 heads (4 chunks) 202 and 197.
template <int CL>
__global__ __launch_bounds__(256) void k_relpos_fold(const float* __restrict__ part, int32_t slots,
                                                     uint32_t n_seq, uint32_t per, int64_t n_pos,
                                                     float* __restrict__ sum)
{
    __shared__ float4 red[256];
    const int x = threadIdx.x % (256 / CL), c0 = threadIdx.x / (256 / CL), h = blockIdx.y;
    const int64_t i = ((int64_t)blockIdx.x * (256 / CL) + x) * 4;  // (n_pos is a multiple of 1024)
    const float* at = part + (int64_t)h * slots * n_pos + i;
    const int chunks = per ? (int)(((h + 1) * n_seq - 1) / per - h * n_seq / per) + 1 : slots;
    float4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int c = c0; c < chunks; c += CL) {
        const float4 w = *(const float4*)(at + c * n_pos);
        v.x += w.x;
        v.y += w.y;
        v.z += w.z;
        v.w += w.w;
    }
    if (CL > 1) {
        red[threadIdx.x] = v;
        __syncthreads();
        if (c0 > 0)
            return;
        for (int c = 1; c < CL; ++c) {
            const float4 w = red[c * (256 / CL) + x];
            v.x += w.x;
            v.y += w.y;
            v.z += w.z;
            v.w += w.w;
        }
    }
    *(float4*)(sum + h * n_pos + i) = v;
}

// The pairs of a bucket, in segments: order[seg_ptr[g] .. seg_ptr[g + 1]) are places in a
// head's tiles.  A wave adds one segment, each lane its pairs in order, then a fixed tree; out:
// [segment][head], or the table's gradient where every bucket is one segment.  sum NULL: no
// sequences, all zero.  Bound: reads of 4 bytes where a bucket's pairs lie on diagonals (777
// tokens, 8 heads, 32 buckets: 8 us; 197 tokens, 12 heads, 732 buckets: 5).
template <int DT>
__global__ __launch_bounds__(256) void k_relpos_segments(const int32_t* __restrict__ order,
                                                         const int32_t* __restrict__ seg_ptr, int32_t n_segs,
                                                         const float* __restrict__ sum, int64_t n_pos,
                                                         int32_t H, float* __restrict__ sums,
                                                         uint16_t* __restrict__ dtable)
{
    const int g = blockIdx.x * 4 + wave_id(), h = blockIdx.y, lane = threadIdx.x & 63;
    if (g >= n_segs)
        return;
    float v = 0.0f;
    if (sum) {
        const float* at = sum + h * n_pos;
        const int begin = seg_ptr[g], end = seg_ptr[g + 1], i = begin + lane;
        static_assert(RELPOS_SEG == 512, "a segment is one turn");
        if (begin < end) {  // (all loads at once: those past the segment ask for its last pair)
            int o[8];
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                o[j] = order[min(i + 64 * j, end - 1)];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                w[j] = at[o[j]];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v += i + 64 * j < end ? w[j] : 0.0f;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v += __shfl_xor(v, o, 64);
    if (lane)
        return;
    if (dtable)
        dtable[(int64_t)g * H + h] = Elem<DT>::from_f32(v);
    else
        sums[(int64_t)g * H + h] = v;
}

// The segments of a bucket: a wave adds them, each lane its own in order, then a fixed tree.
template <int DT>
__global__ __launch_bounds__(256) void k_relpos_buckets(const int32_t* __restrict__ bucket_seg,
                                                        const float* __restrict__ sums, int32_t n_buckets,
                                                        int32_t H, uint16_t* __restrict__ dtable)
{
    const int b = blockIdx.x * 4 + wave_id(), h = blockIdx.y, lane = threadIdx.x & 63;
    if (b >= n_buckets)
        return;
    float v = 0.0f;
    for (int g = bucket_seg[b] + lane; g < bucket_seg[b + 1]; g += 64)
        v += sums[(int64_t)g * H + h];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v += __shfl_xor(v, o, 64);
    if (lane == 0)
        dtable[(int64_t)b * H + h] = Elem<DT>::from_f32(v);
}

// ---------------------------------------------------------------- up to 64 tokens

// Windows of at most 64 tokens: everything of a window and head fits a wave's (forward) or a
// small workgroup's (gradients) registers and LDS, so a workgroup stays with one head, whose
// bias its registers hold as the accumulators' start, and takes one window after the other,
// the next one's rows in flight.  Against the general kernels (us of a call): 2048 x 49
// tokens, 3 heads of 32, forward 20 / 28, gradients 42 / 111; 4096 x 16 tokens, 6 heads, 19 /
// 61 and 47 / 281; 512 x 64 tokens, 6 heads of 64, 24 / 26 and 54 / 110.

// Workgroup -> head and run of windows.  Workgroups L and L + 8 share an XCD: the heads of a
// run of windows are 8 apart, so that the lines that rows of two heads share are fetched and
// written back once.
struct WindowPlace {
    int h, chunk, of;
};
__device__ inline WindowPlace window_place(int H)
{
    const uint32_t j = blockIdx.x / 8, of = gridDim.x / (uint32_t)H, c = j / (uint32_t)H;
    if (of < 8)
        return {(int)(blockIdx.x % (uint32_t)H), (int)(blockIdx.x / (uint32_t)H), (int)of};
    return {(int)(j - c * (uint32_t)H), (int)(8 * c + blockIdx.x % 8), (int)of};
}

// Runs of windows (a multiple of 8, or fewer) for a launch of at most `most` workgroups of `each`
// windows at a time: no more passes than needed, and in them as few as do.
int window_runs(int64_t n_seq, int32_t H, int64_t most, int each)
{
    const int64_t need = (n_seq + each - 1) / each;
    if (need < 8)
        return (int)need;
    int64_t runs = most / H / 8 * 8;
    if (runs < 8)
        runs = 8;
    const int64_t its = (n_seq + runs * each - 1) / (runs * each);
    return (int)((n_seq + its * each * 8 - 1) / (its * each * 8) * 8);
}

// Forward: a wave to a window, four windows to a workgroup.  Q is read as the operand that it
// is, K and V pass through the wave's LDS rows.  Bound: HBM.  4096 x 49 tokens, 3 heads of 32,
// labels: 37 us, 4.1 TB/s.
template <int DT, int HD, int NT, bool REG>
__global__ __launch_bounds__(256, HD == 32 ? 2 : 1) void k_relpos_window_fwd(
    Rp p, const uint16_t* __restrict__ idx, const uint16_t* __restrict__ table, uint16_t* __restrict__ out,
    int64_t ldo, float* __restrict__ lse, float scale, float root)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS, ND = Row<HD>::DT, CH = HD / 8;
    constexpr int RPC = 64 / CH, NC = 32 * NT / RPC;  // rows to a chunk of 64 lanes, chunks
    __shared__ __attribute__((aligned(16))) char rows[4][2][32 * NT * RS];
    __shared__ __attribute__((aligned(16))) int32_t labs[4][64];
    __shared__ float4 tiles[NT * NT * 4 * 64];
    const int T = p.T, lane = threadIdx.x & 63, wave = wave_id(), l32 = lane & 31, half = lane >> 5;
    const WindowPlace at = window_place(p.H);
    const int h = at.h;
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD, step = (int64_t)at.of * 4;
    int64_t n = (int64_t)at.chunk * 4 + wave;
    // the next window: Q fragments, K and V chunks (row lane / CH of each RPC), its label
    F qn[NT][KS];
    uint4 kn[NC], vn[NC];
    int labn = 0;
    auto load = [&](int64_t seq) {
        const uint16_t* base = p.qkv + seq * T * ldq + h * HD;
        if (REG)
            labn = lane < T ? max(labels(p, seq)[lane], -1) : -1;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int r = i * RPC + lane / CH;
            kn[i] = vn[i] = uint4{0u, 0u, 0u, 0u};
            if (r < T) {
                const uint16_t* at = base + (int64_t)r * ldq + 8 * (lane % CH);
                kn[i] = *(const uint4*)(at + hw);
                vn[i] = *(const uint4*)(at + 2 * hw);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
            load_frags<F, HD>(qn[t], base + (int64_t)min(32 * t + l32, T - 1) * ldq, half, true);
    };
    if (n < p.n_seq)
        load(n);
    for (int i = wave; i < NT * NT * 4; i += 4)
        tiles[i * 64 + lane] = gather_bias<DT>(idx, NT, i / 4 / NT, i / 4 % NT, i % 4, lane, table, p.H, h, root);
    __syncthreads();
    f32x16 bias[NT][NT];
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b)
            bias[a][b] = load_bias((const float*)(tiles + (a * NT + b) * 256 + lane));
    char* kb = rows[wave][0];
    char* vb = rows[wave][1];
    const uint32_t ka = lds32(kb) + l32 * RS + half * 16, va = tr_base<HD>(vb, lane);
    for (; n < p.n_seq; n += step) {
        F qf[NT][KS];
        const int lab = labn;
        bool cut = false;  // the window has more than one label, or padding
        if (REG) {
            labs[wave][lane] = lab;
            cut = !__all(lane >= T || (lab == __builtin_amdgcn_readfirstlane(lab) && lab >= 0));
        }
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int r = i * RPC + lane / CH;
            if (REG && cut && __shfl(lab, r, 64) < 0)  // (padding may hold anything)
                vn[i] = uint4{0u, 0u, 0u, 0u};
            *(uint4*)(kb + r * RS + 16 * (lane % CH)) = kn[i];
            *(uint4*)(vb + r * RS + 16 * (lane % CH)) = vn[i];
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                qf[t][ks] = qn[t][ks];
        if (n + step < p.n_seq)
            load(n + step);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (a wave's LDS accesses run in order)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f32x16 s[NT], o[ND];
#pragma unroll
            for (int i = 0; i < NT; ++i)
                s[i] = bias[t][i];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int i = 0; i < NT; ++i)
                    s[i] = E::mma(att_frag<F>(ka + i * 32 * RS + 32 * ks), qf[t][ks], s[i]);
            if (REG && cut) {
                const int mine = __shfl(lab, 32 * t + l32, 64);
#pragma unroll
                for (int i = 0; i < NT; ++i)
                    mask_region(s[i], mine < 0 ? NO_LABEL : mine, labs[wave] + 32 * i, half);
            }
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    m = fmaxf(m, fmaxf(fmaxf(s[i][j], s[i][j + 4]), fmaxf(s[i][j + 8], s[i][j + 12])));
            m = half_max(m);
            const float nms = m == -INFINITY ? 0.0f : -m * scale;
            float ps[2] = {0.0f, 0.0f};
#pragma unroll
            for (int d = 0; d < ND; ++d)
                o[d] = f32x16{};
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                uint32_t pb[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float e0 = __builtin_amdgcn_exp2f(fmaf(s[i][2 * j], scale, nms));
                    const float e1 = __builtin_amdgcn_exp2f(fmaf(s[i][2 * j + 1], scale, nms));
                    ps[0] += e0;
                    ps[1] += e1;
                    pb[j] = pack2<DT>(e0, e1);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const F pf = as_frag<F>(uint4{pb[4 * u], pb[4 * u + 1], pb[4 * u + 2], pb[4 * u + 3]});
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        o[d] = E::mma(tr_frag<F, HD>(va, 32 * i + 16 * u, d), pf, o[d]);
                }
            }
            const float l = half_add(ps[0] + ps[1]);
            const int q = 32 * t + l32;
            if (q < T) {
                store_rows<DT, HD>(out + (n * T + q) * ldo + h * HD, o, l > 0.0f ? 1.0f / l : 0.0f, half);
                if (lse && half == 0)
                    lse[(n * p.H + h) * T + q] = l > 0.0f ? LN2 * (m * scale + __log2f(l)) : -INFINITY;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Gradients: a workgroup of NT waves to a window, all four matrices' rows in LDS.  First a
// wave holds a 32-query tile (lane = query): S^T, dP^T, D from the weights themselves, dS^T,
// which its registers add up over the windows for the bias's gradient, and dQ^T = K^T dS^T.
// P and dS, rounded once, cross to the other operand order through LDS; then a wave holds a
// 32-key tile: dV^T = dO^T P, dK^T = Q^T dS.  Bound: HBM as far as four workgroups to a
// compute unit (LDS and registers) keep it busy.  4096 x 49 tokens, 3 heads of 32, labels: 81
// us, 3.3 TB/s.
template <int DT, int HD, int NT, bool REG>
__global__ __launch_bounds__(64 * NT, HD == 32 ? 2 : 1) void k_relpos_window_grad(
    Rp p, const uint16_t* __restrict__ idx, const uint16_t* __restrict__ table,
    const float* __restrict__ lse, const uint16_t* __restrict__ dout, int64_t ldg,
    uint16_t* __restrict__ dqkv, int64_t lddq, float* __restrict__ part, float scale, float root, float rroot)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS, ND = Row<HD>::DT, CH = HD / 8;
    constexpr int N = 32 * CH / 64;  // chunks of each matrix to a thread
    constexpr int PS = 64 * NT + 16;  // bytes of a row of P and dS
    __shared__ __attribute__((aligned(16))) char rows[4][32 * NT * RS];  // Q, K, V, dO
    __shared__ __attribute__((aligned(16))) char cross[2][32 * NT * PS];
    __shared__ __attribute__((aligned(16))) int32_t labs[32 * NT];
    __shared__ int32_t states[NT];
    const int T = p.T, tid = threadIdx.x, lane = tid & 63, wave = wave_id(), l32 = lane & 31, half = lane >> 5;
    const WindowPlace at = window_place(p.H);
    const int h = at.h, chunk = at.chunk, chunks = at.of;
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    uint4 next[4][N];
    float lsen = 0.0f;
    int labn = 0, rlab[N] = {};
    const int q = 32 * wave + l32;
    auto load = [&](int64_t seq) {
        const uint16_t* base = p.qkv + seq * T * ldq + h * HD;
        const uint16_t* g = dout + seq * T * ldg + h * HD;
        const int32_t* reg = REG ? labels(p, seq) : nullptr;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = tid + i * 64 * NT, r = c / CH, k = 8 * (c % CH);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                next[j][i] = uint4{0u, 0u, 0u, 0u};
            if (r < T) {
                if (REG)
                    rlab[i] = reg[r];
                const uint16_t* at = base + (int64_t)r * ldq + k;
                next[0][i] = *(const uint4*)at;
                next[1][i] = *(const uint4*)(at + hw);
                next[2][i] = *(const uint4*)(at + 2 * hw);
                next[3][i] = *(const uint4*)(g + (int64_t)r * ldg + k);
            }
        }
        lsen = q < T ? lse[(seq * p.H + h) * T + q] : -INFINITY;
        if (REG)
            labn = q < T ? max(reg[q], -1) : -1;
    };
    int64_t n = chunk;
    if (n < p.n_seq)
        load(n);
    f32x16 bias[NT], sum[NT];
#pragma unroll
    for (int b = 0; b < NT; ++b) {
        sum[b] = f32x16{};
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 v = gather_bias<DT>(idx, NT, wave, b, g, lane, table, p.H, h, root);
            bias[b][4 * g] = v.x;
            bias[b][4 * g + 1] = v.y;
            bias[b][4 * g + 2] = v.z;
            bias[b][4 * g + 3] = v.w;
        }
    }
    const uint32_t qa = lds32(rows[0]) + q * RS + half * 16, ga = lds32(rows[3]) + q * RS + half * 16;
    const uint32_t ka = lds32(rows[1]) + l32 * RS + half * 16, va = lds32(rows[2]) + l32 * RS + half * 16;
    const uint32_t qtr = tr_base<HD>(rows[0], lane), ktr = tr_base<HD>(rows[1], lane),
                   gtr = tr_base<HD>(rows[3], lane);
    // this lane's transposing read of P and dS: rows are queries, columns this wave's keys
    const int g16 = lane >> 4, j16 = lane & 15;
    const uint32_t ptr = lds32(cross[0]) + ((j16 >> 2) + 4 * (g16 >> 1)) * PS +
                         (32 * wave + 16 * (g16 & 1) + 4 * (j16 & 3)) * 2;
    auto cross_frag = [&](uint32_t base, int row) {
        const uint32_t at = base + row * PS;
        const uint2 lo = att_tr_read(at), hi = att_tr_read(at + 8 * PS);
        return as_frag<F>(uint4{lo.x, lo.y, hi.x, hi.y});
    };
    for (; n < p.n_seq; n += chunks) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = tid + i * 64 * NT;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(uint4*)(rows[j] + c / CH * RS + 16 * (c % CH)) = unless_padding<REG>(next[j][i], rlab[i]);
        }
        const float nl = lsen == -INFINITY ? -INFINITY : -lsen * LOG2E;
        const int mine = labn < 0 ? NO_LABEL : labn;
        if (REG) {
            const int32_t state = tile_state(labn, half);  // (both halves hold the same rows)
            if (half == 0)
                labs[q] = labn;
            if (lane == 0)
                states[wave] = state;
        }
        __syncthreads();
        if (n + chunks < p.n_seq)
            load(n + chunks);
        F qf[KS], gf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks] = att_frag<F>(qa + 32 * ks);
            gf[ks] = att_frag<F>(ga + 32 * ks);
        }
        f32x16 s[NT], dp[NT];
        float D = 0.0f;
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            s[b] = bias[b];
            dp[b] = f32x16{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s[b] = E::mma(att_frag<F>(ka + b * 32 * RS + 32 * ks), qf[ks], s[b]);
                dp[b] = E::mma(att_frag<F>(va + b * 32 * RS + 32 * ks), gf[ks], dp[b]);
            }
            if (REG && !__all(q >= T || mine == states[b]))
                mask_region(s[b], mine, labs + 32 * b, half);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], scale, nl));
                D = fmaf(s[b][r], dp[b][r], D);
            }
        }
        D = half_add(D);
        f32x16 dq[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d)
            dq[d] = f32x16{};
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            uint32_t db[8];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float e[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    e[j] = s[b][4 * g + j] * (dp[b][4 * g + j] - D);
                    sum[b][4 * g + j] += e[j];
                }
                db[2 * g] = pack2<DT>(e[0], e[1]);
                db[2 * g + 1] = pack2<DT>(e[2], e[3]);
                const int at = q * PS + (32 * b + 8 * g + 4 * half) * 2;
                *(uint2*)(cross[0] + at) = uint2{pack2<DT>(s[b][4 * g], s[b][4 * g + 1]),
                                                 pack2<DT>(s[b][4 * g + 2], s[b][4 * g + 3])};
                *(uint2*)(cross[1] + at) = uint2{db[2 * g], db[2 * g + 1]};
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const F df = as_frag<F>(uint4{db[4 * u], db[4 * u + 1], db[4 * u + 2], db[4 * u + 3]});
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    dq[d] = E::mma(tr_frag<F, HD>(ktr, 32 * b + 16 * u, d), df, dq[d]);
            }
        }
        uint16_t* row = dqkv + (n * T + q) * lddq + h * HD;
        if (q < T)
            store_rows<DT, HD>(row, dq, rroot, half);
        __syncthreads();
        f32x16 dk[ND], dv[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            dk[d] = f32x16{};
            dv[d] = f32x16{};
        }
#pragma unroll
        for (int u = 0; u < 2 * NT; ++u) {
            const F pf = cross_frag(ptr, 16 * u), df = cross_frag(ptr + 32 * NT * PS, 16 * u);
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                dv[d] = E::mma(tr_frag<F, HD>(gtr, 16 * u, d), pf, dv[d]);
                dk[d] = E::mma(tr_frag<F, HD>(qtr, 16 * u, d), df, dk[d]);
            }
        }
        if (q < T) {
            store_rows<DT, HD>(row + hw, dk, rroot, half);
            store_rows<DT, HD>(row + 2 * hw, dv, 1.0f, half);
        }
        __syncthreads();
    }
    float* dst = part + (((int64_t)h * chunks + chunk) * NT + wave) * NT * 1024 + lane * 4;
#pragma unroll
    for (int b = 0; b < NT; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(float4*)(dst + b * 1024 + 256 * g) =
                float4{sum[b][4 * g], sum[b][4 * g + 1], sum[b][4 * g + 2], sum[b][4 * g + 3]};
}

int64_t tile_floats(const lpv_relpos* h) { return (int64_t)h->nt * h->nt * 1024; }

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// ---------------------------------------------------------------- gradients, 65 to 224 tokens

// Gradients of sequences whose tiles of dS a workgroup's registers can add up: a wave to a
// 32-query tile, all of a sequence's in one workgroup, and one wave more.  A workgroup takes
// the `per` next sequences, head after head.  The key tiles pass one at a time: every query
// wave forms S^T, P, dS of its queries (lane = query), adds dS to its sums and dS K to its dQ,
// and leaves P and dS, rounded once, in one of two LDS buffers; meanwhile the last wave turns
// the tile before into dV^T = dO^T P and dK^T = Q^T dS over all queries.  So every score is
// formed once, with five products, where the general kernels form it three times with nine.
// LDS holds all rows of Q and dO, two key tiles and the two buffers.  D is dO . O with O as it
// was rounded, so that it is off by E = dO . (O's rounding) and dS_ij by P_ij E: a rounding like
// others where a row's pairs go to distinct buckets, but a bucket that takes several pairs of a
// row adds P_ij E over them while the sum of their dS cancels (a class token's row is one bucket: at
// 197 tokens its gradient was off by 3% in bf16).  A row of dS sums to -E, which is known behind
// its last tile: the waves of crowded tiles leave P, rounded once, in `kept` as they go and
// then take P_ij times that sum off their sums (64 x 197 tokens, 12 heads of 64: 74 us without,
// 77 for the class token's tile, 83 for all seven).  Bound: LDS reads and the chain of a tile at two
// waves to a SIMD (the sums leave registers for no more).  64 x 197 tokens, 12 heads of 64: 247
// TFLOP/s; 256 x 144, 6 heads of 32, labels: 66 us.
constexpr int MID_TILES = 7;  // with the wave more two waves to a SIMD, which the sums' registers allow
constexpr int MID_XS = 72;  // bytes of a row of P or dS, 32 keys: the writes of 32 rows' 8 bytes meet all banks
template <int DT, int HD, bool REG>
__global__ __launch_bounds__(64 * (MID_TILES + 1)) void k_relpos_mid_grad(
    Rp p, const uint16_t* __restrict__ out, int64_t ldo, const float* __restrict__ lse,
    const uint16_t* __restrict__ dout, int64_t ldg, uint16_t* __restrict__ dqkv, int64_t lddq,
    float* __restrict__ part, int32_t per, int32_t slots, uint32_t crowded, char* __restrict__ kept,
    float scale, float rroot)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS, ND = Row<HD>::DT, CH = HD / 8;
    constexpr int XS = MID_XS;
    constexpr int KV = 32 * RS;             // a key tile of K or V
    constexpr int NR = 32 * CH / 64;        // a tile's chunks to a lane
    constexpr int NK = (64 * CH + 191) / 192;  // a key tile's chunks of K and V to a thread (3 query waves or more)
    constexpr bool KEEP = HD == 32;  // the operands of Q and dO stay in registers; else LDS has them
    extern __shared__ uint4 mid_lds[];
    const int T = p.T, nt = p.nt, tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    const int l32 = lane & 31, half = lane >> 5, threads = 64 * nt;
    char* Qr = (char*)mid_lds;
    char* Gr = Qr + 32 * nt * RS;
    char* kv = Gr + 32 * nt * RS;  // [2][K, V][KV]
    char* X = kv + 4 * KV;         // [2][P, dS][32 nt][XS]
    int32_t* labs = (int32_t*)(X + 4 * 32 * nt * XS);
    int32_t* states = labs + 32 * nt;
    const uint32_t units = (uint32_t)p.n_seq * (uint32_t)p.H, wgs = (units + per - 1) / per, wg = xcd_order(wgs, blockIdx.x);
    if (wg >= wgs)
        return;
    const uint32_t u0 = wg * per, u1 = min(u0 + per, units), seqs = (uint32_t)p.n_seq;
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    const uint32_t qtr = tr_base<HD>(Qr, lane), gtr = tr_base<HD>(Gr, lane);
    if (wave == nt) {  // dK and dV
        // this lane's transposing read of P and dS (rows are queries, columns the tile's keys)
        const int g16 = lane >> 4, j16 = lane & 15;
        const uint32_t xtr = lds32(X) + ((j16 >> 2) + 4 * (g16 >> 1)) * XS + (16 * (g16 & 1) + 4 * (j16 & 3)) * 2;
        for (uint32_t u = u0; u < u1; ++u) {
            const uint32_t h = u / seqs;
            const int64_t seq = u - h * seqs;
            auto outputs = [&](int kt) {
                f32x16 dk[ND], dv[ND];
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    dk[d] = f32x16{};
                    dv[d] = f32x16{};
                }
                const uint32_t x = xtr + (kt & 1) * 2 * 32 * nt * XS;
                auto x_frag = [&](uint32_t at) {
                    const uint2 lo = att_tr_read(at), hi = att_tr_read(at + 8 * XS);
                    return as_frag<F>(uint4{lo.x, lo.y, hi.x, hi.y});
                };
                // a step's operands are read while the step before is multiplied
                struct Step {
                    F p, ds, g[ND], q[ND];
                } step[2];
                auto read = [&](Step& t, int row) {
                    t.p = x_frag(x + row * XS);
                    t.ds = x_frag(x + (32 * nt + row) * XS);
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        t.g[d] = tr_frag<F, HD>(gtr, row, d);
                        t.q[d] = tr_frag<F, HD>(qtr, row, d);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                auto multiply = [&](const Step& t) {
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        dv[d] = E::mma(t.g[d], t.p, dv[d]);
                        dk[d] = E::mma(t.q[d], t.ds, dk[d]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                read(step[0], 0);
                for (int row = 0; row < 32 * nt; row += 32) {
                    read(step[1], row + 16);
                    multiply(step[0]);
                    read(step[0], row + 32 < 32 * nt ? row + 32 : 0);  // (the last one's is not used)
                    multiply(step[1]);
                }
                const int k = 32 * kt + l32;
                if (k < T) {
                    uint16_t* row = dqkv + (seq * T + k) * lddq + h * HD;
                    store_rows<DT, HD>(row + hw, dk, rroot, half);
                    store_rows<DT, HD>(row + 2 * hw, dv, 1.0f, half);
                }
            };
            __syncthreads();
            __syncthreads();
            for (int kt = 0; kt < nt; ++kt) {
                if (kt > 0)
                    outputs(kt - 1);
                __syncthreads();
            }
            outputs(nt - 1);
        }
        return;
    }
    const int q = 32 * wave + l32;
    // P of this wave's rows of a sequence: [key tile][r / 4][lane][r % 4], read by the lane that wrote it
    const bool crowd = (crowded >> wave) & 1;
    uint2* mine_p = (uint2*)kept +
                    ((int64_t)wg * __popc(crowded) + __popc(crowded & ((1u << wave) - 1))) * nt * 256 + lane;
    const uint32_t qa = lds32(Qr) + q * RS + half * 16, ga = lds32(Gr) + q * RS + half * 16;
    for (uint32_t unit = u0; unit < u1;) {  // a head
        const uint32_t h = unit / seqs, end = min(u1, (h + 1) * seqs);
        float* slot = part + (((int64_t)h * slots + (wg - h * seqs / per)) * nt + wave) * nt * 1024 + lane * 4;
        f32x16 sum[MID_TILES];
#pragma unroll
        for (int b = 0; b < MID_TILES; ++b)
            sum[b] = f32x16{};
        auto store_sum = [&](const f32x16& v, int kt) {  // to this workgroup's slot of the head
            int at = 1024 * kt;
            asm volatile("" : "+v"(at));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(float4*)(slot + at + 256 * i) = float4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
        };
        for (; unit < end; ++unit) {
            const int64_t seq = unit - h * seqs;
            const uint16_t* base = p.qkv + seq * T * ldq + h * HD;
            const uint16_t* g = dout + seq * T * ldg + h * HD;
            const int32_t* reg = REG ? labels(p, seq) : nullptr;
            const float* bias = p.bias + ((int64_t)h * nt + wave) * nt * 1024 + lane * 4;
            uint4 kvr[NK];
            int kvl[NK];  // (the rows' labels, asked for beside them)
            // (the thread's number as no constant: its chunks' places would be kept in registers)
            auto load_kv = [&](int kt) {
                int t = tid;
                asm volatile("" : "+v"(t));
#pragma unroll
                for (int i = 0; i < NK; ++i) {
                    const int c = t + i * threads, m = c / (32 * CH), r = 32 * kt + c / CH % 32;
                    kvr[i] = uint4{0u, 0u, 0u, 0u};
                    kvl[i] = 0;
                    if (c < 64 * CH && r < T) {
                        kvr[i] = *(const uint4*)(base + (1 + m) * hw + (int64_t)r * ldq + 8 * (c % CH));
                        if (REG)
                            kvl[i] = reg[r];
                    }
                }
            };
            auto store_kv = [&](int buf) {
                int t = tid;
                asm volatile("" : "+v"(t));
#pragma unroll
                for (int i = 0; i < NK; ++i) {
                    const int c = t + i * threads;
                    if (c < 64 * CH)
                        *(uint4*)(kv + (2 * buf + c / (32 * CH)) * KV + c / CH % 32 * RS + 16 * (c % CH)) =
                            unless_padding<REG>(kvr[i], kvl[i]);
                }
            };
            f32x16 s = load_bias(bias);
            load_kv(0);
            uint4 qr[NR], gr[NR];
            int ql[NR];
            int lo = lane;
            asm volatile("" : "+v"(lo));
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const int c = lo + 64 * i, r = 32 * wave + c / CH, k = 8 * (c % CH);
                qr[i] = gr[i] = uint4{0u, 0u, 0u, 0u};
                ql[i] = 0;
                if (r < T) {
                    qr[i] = *(const uint4*)(base + (int64_t)r * ldq + k);
                    gr[i] = *(const uint4*)(g + (int64_t)r * ldg + k);
                    if (REG)
                        ql[i] = reg[r];
                }
            }
            const int lab = REG && q < T ? max(reg[q], -1) : -1;
            const int mine = !REG ? 0 : lab < 0 ? NO_LABEL : lab;
            float D = 0.0f, nl = -INFINITY;
            float miss = 0.0f;  // the sum of this lane's row of dS: -E
            F qf[KS], gf[KS];
            {
                F of[KS];
                load_frags<F, HD>(of, out + (seq * T + min(q, T - 1)) * ldo + h * HD, half,
                                  q < T && (!REG || lab >= 0));
                if (q < T) {
                    const float v = lse[(seq * p.H + h) * T + q];
                    nl = v == -INFINITY ? -INFINITY : -v * LOG2E;
                }
                __syncthreads();  // (the last sequence's rows have been read)
#pragma unroll
                for (int i = 0; i < NR; ++i) {
                    const int c = lo + 64 * i, at = (32 * wave + c / CH) * RS + 16 * (c % CH);
                    *(uint4*)(Qr + at) = unless_padding<REG>(qr[i], ql[i]);
                    *(uint4*)(Gr + at) = unless_padding<REG>(gr[i], ql[i]);
                }
                if (REG) {
                    const int32_t state = tile_state(lab, half);  // (both halves hold the same rows)
                    if (half == 0)
                        labs[q] = lab;
                    if (lane == 0)
                        states[wave] = state;
                }
                store_kv(0);
                if (nt > 1)
                    load_kv(1);
                __syncthreads();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    qf[ks] = att_frag<F>(qa + 32 * ks);
                    gf[ks] = att_frag<F>(ga + 32 * ks);
                }
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        D = fmaf((float)gf[ks][j], (float)of[ks][j], D);
                D = half_add(D);
            }
            f32x16 dq[ND];
#pragma unroll
            for (int d = 0; d < ND; ++d)
                dq[d] = f32x16{};
#pragma unroll
            for (int sk = 0; sk < MID_TILES; ++sk) {
                if (sk >= nt)
                    break;
                int kt = sk;  // (as no constant, for the same reason)
                asm volatile("" : "+s"(kt));
                const uint32_t kb = lds32(kv) + (kt & 1) * 2 * KV;
                const uint32_t ka = kb + l32 * RS + half * 16, va = ka + KV;
                const uint32_t ktr = tr_base<HD>(kv, lane) + (kt & 1) * 2 * KV;
                char* x = X + (kt & 1) * 2 * 32 * nt * XS;
                f32x16 dp = {};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    s = E::mma(att_frag<F>(ka + 32 * ks), KEEP ? qf[ks] : att_frag<F>(qa + 32 * ks), s);
                    dp = E::mma(att_frag<F>(va + 32 * ks), KEEP ? gf[ks] : att_frag<F>(ga + 32 * ks), dp);
                }
                if (REG && !__all(mine == states[kt]))
                    mask_region(s, mine, labs + 32 * kt, half);
                uint32_t db[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float e[4], f[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        e[j] = __builtin_amdgcn_exp2f(fmaf(s[4 * i + j], scale, nl));
                        f[j] = e[j] * (dp[4 * i + j] - D);
                        sum[sk][4 * i + j] += f[j];
                    }
                    db[2 * i] = pack2<DT>(f[0], f[1]);
                    db[2 * i + 1] = pack2<DT>(f[2], f[3]);
                    const int at = q * XS + (8 * i + 4 * half) * 2;
                    const uint2 pb = {pack2<DT>(e[0], e[1]), pack2<DT>(e[2], e[3])};
                    *(uint2*)(x + at) = pb;
                    *(uint2*)(x + 32 * nt * XS + at) = uint2{db[2 * i], db[2 * i + 1]};
                    if (crowd) {
                        miss += (f[0] + f[1]) + (f[2] + f[3]);
                        mine_p[(4 * kt + i) * 64] = pb;
                    }
                }
                if (kt + 1 < nt) {
                    s = load_bias(bias + (kt + 1) * 1024);
                    store_kv(1 - (kt & 1));
                    if (kt + 2 < nt)
                        load_kv(kt + 2);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const F df = as_frag<F>(uint4{db[4 * u], db[4 * u + 1], db[4 * u + 2], db[4 * u + 3]});
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        dq[d] = E::mma(tr_frag<F, HD>(ktr, 16 * u, d), df, dq[d]);
                }
                if (unit + 1 == end && !crowd)  // the tile's sum is whole
                    store_sum(sum[sk], kt);
                __syncthreads();
            }
            if (q < T)
                store_rows<DT, HD>(dqkv + (seq * T + q) * lddq + h * HD, dq, rroot, half);
            if (crowd) {
                miss = half_add(miss);
                uint2 pb[2][4];
                auto load_p = [&](uint2* to, int kt) {
                    int at = 256 * kt;
                    asm volatile("" : "+v"(at));
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        to[i] = mine_p[at + 64 * i];
                };
                load_p(pb[0], 0);
#pragma unroll
                for (int sk = 0; sk < MID_TILES; ++sk) {
                    if (sk >= nt)
                        break;
                    load_p(pb[~sk & 1], sk + 1 < nt ? sk + 1 : sk);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const uint2 v = pb[sk & 1][r >> 2];
                        sum[sk][r] -= Elem<DT>::to_f32((uint16_t)((r & 2 ? v.y : v.x) >> (16 * (r & 1)))) * miss;
                    }
                    if (unit + 1 == end)
                        store_sum(sum[sk], sk);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }
}

constexpr int WINDOW_TILES = 2;  // tiles of 32 tokens that the window kernels take
bool is_window(const lpv_relpos* h) { return h->nt <= WINDOW_TILES; }

// Against the general kernels (us of both passes' calls): 64 sequences of 197 tokens, 12 heads
// of 64, 89 / 123; 224 tokens, heads of 32, 71 / 89; 66 tokens 32 / 39; 8 sequences 41 / 44.
bool is_mid(const lpv_relpos* h) { return !is_window(h) && h->nt <= MID_TILES; }
size_t mid_lds_bytes(int nt, int hd)
{
    const size_t rs = (size_t)hd * 2 + 16;
    return 2 * 32 * nt * rs + 4 * 32 * rs + 4 * 32 * (size_t)nt * MID_XS + 33 * nt * 4;
}
// Sequences of a head to a workgroup, one to a compute unit.
int32_t mid_per(int64_t n_seq, int32_t H) { return (int32_t)((n_seq * H + 255) / 256); }
int64_t mid_workgroups(int64_t n_seq, int32_t H)
{
    const int32_t per = mid_per(n_seq, H);
    return (n_seq * H + per - 1) / per;
}

// Chunks of sequences of the bias gradient: 1024 workgroups, four to a compute unit.
int bias_chunks(const lpv_relpos* h, int64_t n_seq, int32_t H)
{
    if (is_window(h)) {
        // 4 workgroups to a compute unit, or more where there are more heads
        return window_runs(n_seq, H, 1024, 1);
    }
    if (is_mid(h)) {  // (a head's sequences may begin and end inside a workgroup's)
        const int32_t per = mid_per(n_seq, H);
        return per ? (int)((n_seq + per - 1) / per + 1) : 0;
    }
    const int64_t n_blk = (h->nt + 1) / 2, wgs = (int64_t)H * n_blk * n_blk;
    const int64_t c = (1024 + wgs - 1) / wgs;
    return (int)(c < n_seq ? c : n_seq);
}

struct Ws {  // places in a gradient's workspace
    float *bias, *bias_t, *D, *Dc, *kept, *part, *sum, *sums;
    size_t bytes;
};
Ws grad_ws(const lpv_relpos* h, int64_t n_seq, int32_t H, void* ws)
{
    size_t at = 0;
    auto take = [&](size_t floats) {
        float* p = (float*)((char*)ws + at);
        at += up256(floats * sizeof(float));
        return p;
    };
    Ws w;
    const bool window = is_window(h), mid = is_mid(h);
    const int chunks = bias_chunks(h, n_seq, H);
    w.bias = take(window ? 0 : (size_t)(H * tile_floats(h)));
    w.bias_t = take(window || mid ? 0 : (size_t)(H * tile_floats(h)));
    w.D = take(window || mid ? 0 : (size_t)(n_seq * H * h->T));
    w.Dc = take(window || mid ? 0 : (size_t)(n_seq * H * h->T));
    w.kept = take(mid && chunks ? (size_t)mid_workgroups(n_seq, H) * __builtin_popcountll(h->crowded) * h->nt * 512 : 0);
    w.part = take((size_t)(H * chunks * tile_floats(h)));
    w.sum = chunks > 1 ? take((size_t)(H * tile_floats(h))) : w.part;
    w.sums = take((size_t)((int64_t)h->n_segs * H));
    w.bytes = at;
    return w;
}

// bias_t, rows: for the gradients that take the transposed tiles and the rows' products (HD,
// else 0).
template <int DT, int HD>
hipError_t expand_bias(const lpv_relpos* h, const void* table, int32_t H, int32_t hd, float* bias,
                       float* bias_t, const RowsCall& rows, hipStream_t s)
{
    // (a tile to a wave, or more of them where that makes over 1024 workgroups, each of which
    // makes the column ready for itself)
    const int tiles = h->nt * h->nt, per = std::max(4, (tiles * H + 1023) / 1024);
    // (rows: hd / 8 lanes each, up to 4096 workgroups' of them at once)
    const int64_t lanes = rows.M * H * (HD / 8), wgs = std::min<int64_t>(4096, (lanes + 255) / 256);
    const dim3 grid(std::max((tiles + per - 1) / per, (int)((wgs + H - 1) / H)), H, HD ? 3 : 1);
    hipLaunchKernelGGL((k_relpos_bias<DT, HD>), grid, dim3(256), h->n_buckets <= BIAS_LDS ? h->n_buckets * 4 : 0, s,
                       h->idx, h->idx_t, h->nt, (const uint16_t*)table, h->n_buckets, H, sqrtf((float)hd), per,
                       bias, bias_t, rows);
    return hipGetLastError();
}

// The general kernels' layout: a wave to a 32-row tile, four tiles to a workgroup; where
// that leaves the chip with few waves, two waves to a tile: `few` below six tiles to a
// compute unit in the forward pass, below two in the gradients, of which there are two kinds of
// workgroups.  (us of the call, two waves / one, 600 tokens, 8 heads of 64: forward 20.6 / 23.8 with
// 304 tiles, 27.5 / 28.5 with 1216, 37.4 / 36.7 with 1976; gradients with the bias's sums behind
// 55.7 / 57.0 with 304, 58.3 / 59.6 with 456, 69.2 / 67.0 with 608, 132 / 121 with 1976; beside
// them 51.2 / 52.9, 58.2 / 53.9, 64.1 / 59.2 and 127 / 111.  Four waves to a tile: 777 tokens, 4 sequences,
// 8 heads, the forward kernel 26.8 against 19.8.)
bool few_tiles(const lpv_relpos* h, const RelposCall& c, int64_t few) { return c.n_seq * c.H * h->nt < few; }

// Three tiles to a workgroup of the forward pass where that takes a quarter of the waves
// fewer, the others being idle (3, 5, 6 and 9 tiles): smaller groups stage K and V more often.
// (us of the call, three / four, 12 heads of 64: 256 x 144 tokens 59.9 / 69.2, 64 x 190 25.7 /
// 27.5, 64 x 280 41.5 / 46.4; with 17 tiles, a tenth fewer, 67.0 / 63.4.)
bool groups_of_three(int nt) { return (nt + 2) / 3 * 3 * 4 <= (nt + 3) / 4 * 4 * 3; }

template <int DT, int HD, bool REG, typename Sh>
hipError_t forward_tiles(const lpv_relpos* h, const RelposCall& c, hipStream_t s)
{
    const Rp p = {(const uint16_t*)c.qkv, c.ldq, c.region, c.n_region, c.n_seq, h->T, c.H, h->nt,
                  (const float*)c.ws};
    const Grid2 g = grid_of(c.n_seq * c.H * ((h->nt + Sh::QW - 1) / Sh::QW));
    hipLaunchKernelGGL((k_relpos_fwd<DT, HD, Sh, REG>), dim3(g.x, g.y), dim3(Sh::NT), 0, s, p,
                       (uint16_t*)c.out, c.ldo, c.lse, LOG2E / sqrtf((float)HD));
    return hipGetLastError();
}

// Workgroups of four windows: at most two (32 dimensions) or one to a compute unit at once.
template <int DT, int HD, bool REG, int NT>
hipError_t forward_windows(const lpv_relpos* h, const RelposCall& c, hipStream_t s)
{
    const Rp p = {(const uint16_t*)c.qkv, c.ldq, c.region, c.n_region, c.n_seq, h->T, c.H, h->nt, nullptr};
    const int runs = window_runs(c.n_seq, c.H, HD == 32 ? 512 : 256, 4);
    hipLaunchKernelGGL((k_relpos_window_fwd<DT, HD, NT, REG>), dim3((uint32_t)runs * c.H),
                       dim3(256), 0, s, p, h->idx, (const uint16_t*)c.table, (uint16_t*)c.out, c.ldo, c.lse,
                       LOG2E / sqrtf((float)HD), sqrtf((float)HD));
    return hipGetLastError();
}

template <int DT, int HD, bool REG, int NT>
hipError_t grad_windows(const lpv_relpos* h, const RelposCall& c, const Ws& w, int chunks, hipStream_t s)
{
    const Rp p = {(const uint16_t*)c.qkv, c.ldq, c.region, c.n_region, c.n_seq, h->T, c.H, h->nt, nullptr};
    hipLaunchKernelGGL((k_relpos_window_grad<DT, HD, NT, REG>), dim3((uint32_t)chunks * c.H), dim3(64 * NT), 0, s,
                       p, h->idx, (const uint16_t*)c.table, c.lse, (const uint16_t*)c.dout, c.ldg,
                       (uint16_t*)c.dqkv, c.lddq, w.part, LOG2E / sqrtf((float)HD), sqrtf((float)HD),
                       1.0f / sqrtf((float)HD));
    return hipGetLastError();
}

template <int DT, int HD, bool REG> hipError_t forward_as(const lpv_relpos* h, const RelposCall& c, hipStream_t s)
{
    if (is_window(h))
        return h->nt == 1 ? forward_windows<DT, HD, REG, 1>(h, c, s) : forward_windows<DT, HD, REG, 2>(h, c, s);
    const hipError_t e = expand_bias<DT, 0>(h, c.table, c.H, HD, (float*)c.ws, nullptr, {}, s);
    if (e != hipSuccess)
        return e;
    if (few_tiles(h, c, 1536))
        return forward_tiles<DT, HD, REG, Shape<2, 2>>(h, c, s);
    return groups_of_three(h->nt) ? forward_tiles<DT, HD, REG, Shape<3, 1>>(h, c, s)
                                  : forward_tiles<DT, HD, REG, Shape<4, 1>>(h, c, s);
}

template <int DT, int HD, bool REG, typename Sh>
hipError_t grad_tiles(const lpv_relpos* h, const RelposCall& c, const Ws& w, int chunks, hipStream_t s)
{
    const Rp p = {(const uint16_t*)c.qkv, c.ldq, c.region, c.n_region, c.n_seq, h->T, c.H, h->nt, w.bias};
    const Gp g = {c.lse, w.D, w.Dc, (const uint16_t*)c.dout, c.ldg, (uint16_t*)c.dqkv, c.lddq, w.bias_t, w.part, chunks,
                  LOG2E / sqrtf((float)HD), 1.0f / sqrtf((float)HD)};
    const int64_t n_tiles = c.n_seq * c.H * ((h->nt + Sh::QW - 1) / Sh::QW), n_blk = (h->nt + 1) / 2;
    const int64_t n_pairs = (int64_t)c.H * n_blk * n_blk * chunks;
    const bool behind = h->crowded != 0;
    const Grid2 t = grid_of(2 * ((n_tiles + 7) / 8 * 8) + (behind ? 0 : n_pairs)), q = grid_of(n_pairs);
    hipLaunchKernelGGL((k_relpos_grad<DT, HD, Sh, REG>), dim3(t.x, t.y), dim3(256), 0, s, p, g, (uint32_t)n_tiles,
                       behind ? 0u : (uint32_t)n_pairs);
    if (behind)
        hipLaunchKernelGGL((k_relpos_pairs<DT, HD, REG>), dim3(q.x, q.y), dim3(256), 0, s, p, g,
                           (uint32_t)n_pairs);
    return hipGetLastError();
}

template <int DT, int HD, bool REG>
hipError_t grad_mid(const lpv_relpos* h, const RelposCall& c, const Ws& w, int chunks, hipStream_t s)
{
    // LDS beyond 64 KB is allowed per kernel and device (idempotent: a race is harmless)
    static bool allowed[64] = {};
    if (h->device >= 64 || !allowed[h->device]) {
        const hipError_t e = hipFuncSetAttribute((const void*)k_relpos_mid_grad<DT, HD, REG>,
                                                 hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)mid_lds_bytes(MID_TILES, HD));
        if (e != hipSuccess)
            return e;
        if (h->device < 64)
            allowed[h->device] = true;
    }
    const Rp p = {(const uint16_t*)c.qkv, c.ldq, c.region, c.n_region, c.n_seq, h->T, c.H, h->nt, w.bias};
    const int32_t per = mid_per(c.n_seq, c.H);
    hipLaunchKernelGGL((k_relpos_mid_grad<DT, HD, REG>), dim3((uint32_t)mid_workgroups(c.n_seq, c.H)),
                       dim3(64 * (h->nt + 1)), mid_lds_bytes(h->nt, HD), s, p, (const uint16_t*)c.out, c.ldo, c.lse,
                       (const uint16_t*)c.dout, c.ldg, (uint16_t*)c.dqkv, c.lddq, w.part, per, chunks,
                       (uint32_t)h->crowded, (char*)w.kept, LOG2E / sqrtf((float)HD), 1.0f / sqrtf((float)HD));
    return hipGetLastError();
}

template <int DT, int HD, bool REG>
hipError_t grad_as(const lpv_relpos* h, const RelposCall& c, hipStream_t s)
{
    const Ws w = grad_ws(h, c.n_seq, c.H, c.ws);
    const int chunks = bias_chunks(h, c.n_seq, c.H);
    const int64_t n_pos = tile_floats(h);
    hipError_t e = hipSuccess;
    if (chunks > 0 && is_window(h)) {
        e = h->nt == 1 ? grad_windows<DT, HD, REG, 1>(h, c, w, chunks, s)
                       : grad_windows<DT, HD, REG, 2>(h, c, w, chunks, s);
    } else if (chunks > 0 && is_mid(h)) {
        e = expand_bias<DT, 0>(h, c.table, c.H, HD, w.bias, nullptr, {}, s);
        if (e == hipSuccess)
            e = grad_mid<DT, HD, REG>(h, c, w, chunks, s);
    } else if (chunks > 0) {  // (n_seq > 0)
        const RowsCall rows = {(const uint16_t*)c.out, (const uint16_t*)c.dout, c.ldo, c.ldg, c.n_seq * h->T, h->T,
                               w.D};
        e = expand_bias<DT, HD>(h, c.table, c.H, HD, w.bias, w.bias_t, rows, s);
        if (e == hipSuccess)
            e = few_tiles(h, c, 512) ? grad_tiles<DT, HD, REG, Shape<2, 2>>(h, c, w, chunks, s)
                                     : grad_tiles<DT, HD, REG, Shape<4, 1>>(h, c, w, chunks, s);
    }
    if (e != hipSuccess)
        return e;
    const uint32_t per = is_mid(h) ? (uint32_t)mid_per(c.n_seq, c.H) : 0;
    if (chunks >= 16)
        hipLaunchKernelGGL((k_relpos_fold<16>), dim3((uint32_t)(n_pos / 64), c.H), dim3(256), 0, s, w.part,
                           chunks, (uint32_t)c.n_seq, per, n_pos, w.sum);
    else if (chunks > 1)
        hipLaunchKernelGGL((k_relpos_fold<1>), dim3((uint32_t)(n_pos / 1024), c.H), dim3(256), 0, s,
                           w.part, chunks, (uint32_t)c.n_seq, per, n_pos, w.sum);
    const bool whole = h->n_segs == h->n_buckets;
    hipLaunchKernelGGL((k_relpos_segments<DT>), dim3((h->n_segs + 3) / 4, c.H), dim3(256), 0, s, h->order,
                       h->seg_ptr, h->n_segs, chunks > 0 ? w.sum : nullptr, n_pos, c.H, w.sums, whole ? (uint16_t*)c.dtable : nullptr);
    if (!whole)
        hipLaunchKernelGGL((k_relpos_buckets<DT>),
                           dim3((h->n_buckets + 3) / 4, c.H), dim3(256), 0, s, h->bucket_seg,
                           w.sums, h->n_buckets, c.H, (uint16_t*)c.dtable);
    return hipGetLastError();
}

}  // namespace

size_t relpos_workspace_bytes(const lpv_relpos* h, int64_t n_seq, int32_t H, bool grad)
{
    if (grad)
        return grad_ws(h, n_seq, H, nullptr).bytes;
    return is_window(h) ? 0 : up256((size_t)(H * tile_floats(h)) * sizeof(float));
}

RelposSizes relpos_sizes(const int32_t* index, int32_t T, int32_t n_buckets, int32_t* count, int32_t* last)
{
    RelposSizes z = {};
    z.bad = -1;
    for (int32_t b = 0; b < n_buckets; ++b) {
        count[b] = 0;
        last[b] = -1;  // the last row with a pair of the bucket
    }
    for (int32_t i = 0; i < T; ++i) {
        bool twice = false;
        for (int32_t j = 0; j < T; ++j) {
            const int32_t b = index[(int64_t)i * T + j];
            if (b < -1 || b >= n_buckets) {
                z.bad = (int64_t)i * T + j;
                return z;
            }
            if (b >= 0) {
                ++count[b];
                twice |= last[b] == i;
                last[b] = i;
            }
        }
        if (twice)
            z.crowded |= (uint64_t)1 << (i / 32);
    }
    for (int32_t b = 0; b < n_buckets; ++b) {
        z.n_pairs += count[b];
        z.n_segs += count[b] ? (count[b] + RELPOS_SEG - 1) / RELPOS_SEG : 1;
    }
    return z;
}

void relpos_tables(const int32_t* index, int32_t T, int32_t n_buckets, int32_t nt, int32_t* count,
                   uint16_t* idx, uint16_t* idx_t, int32_t* order, int32_t* seg_ptr, int32_t* bucket_seg)
{
    const int64_t Tp = (int64_t)nt * 32;
    memset(idx, 0xff, (size_t)(Tp * Tp) * 2);
    memset(idx_t, 0xff, (size_t)(Tp * Tp) * 2);
    int32_t seg = 0, at = 0;
    for (int32_t b = 0; b < n_buckets; ++b) {  // count[b] becomes the bucket's next place
        bucket_seg[b] = seg;
        const int32_t n = count[b];
        count[b] = at;
        for (int32_t i = 0; i == 0 || i < n; i += RELPOS_SEG)
            seg_ptr[seg++] = at + i;
        at += n;
    }
    bucket_seg[n_buckets] = seg;
    seg_ptr[seg] = at;
    // a bucket's pairs in the order of their places (so that neighbours are read together):
    // tile after tile, in one [c / 8][lane][c % 4] with row i % 32 in the lanes
    for (int32_t a = 0; a < nt; ++a)
        for (int32_t c = 0; c < nt; ++c)
            for (int32_t at = 0; at < 1024; ++at) {
                const int32_t lane = at / 4 % 64, i = 32 * a + lane % 32;
                const int32_t j = 32 * c + at / 256 * 8 + lane / 32 * 4 + at % 4;
                const int32_t b = i < T && j < T ? index[(int64_t)i * T + j] : -1;
                if (b >= 0) {
                    idx[i * Tp + j] = (uint16_t)b;
                    idx_t[j * Tp + i] = (uint16_t)b;
                    order[count[b]++] = (a * nt + c) * 1024 + at;
                }
            }
}

#define LPV_RP(FN_)                                                                          \
    (c.dtype == LPV_BF16                                                                     \
         ? (c.hd == 32 ? (c.region ? FN_<LPV_BF16, 32, true>(h, c, s) : FN_<LPV_BF16, 32, false>(h, c, s))  \
                       : (c.region ? FN_<LPV_BF16, 64, true>(h, c, s) : FN_<LPV_BF16, 64, false>(h, c, s))) \
         : (c.hd == 32 ? (c.region ? FN_<LPV_F16, 32, true>(h, c, s) : FN_<LPV_F16, 32, false>(h, c, s))    \
                       : (c.region ? FN_<LPV_F16, 64, true>(h, c, s) : FN_<LPV_F16, 64, false>(h, c, s))))

hipError_t launch_relpos_attention(const lpv_relpos* h, const RelposCall& c, hipStream_t s)
{
    return LPV_RP(forward_as);
}

hipError_t launch_relpos_grad(const lpv_relpos* h, const RelposCall& c, hipStream_t s)
{
    return LPV_RP(grad_as);
}
#undef LPV_RP

}  // namespace lpv
