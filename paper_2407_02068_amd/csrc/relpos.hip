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

#include "lpv_attention.h"
#include "lpv_grid.h"
#include "lpv_internal.h"

namespace lpv {
namespace {

constexpr int BLK = 64;  // rows of a staged block
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

template <int HD> struct Row {
    static constexpr int KS = HD / 16;     // 16-dimension steps of a product over the head
    static constexpr int DT = HD / 32;     // 32-dimension tiles of an output
    static constexpr int RS = HD * 2 + 16; // bytes per staged row: 16 consecutive rows of one
                                           // 16-byte column sit in distinct banks
};

__device__ inline uint32_t lds32(const void* p)
{
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// The tile's bias in matrix-core accumulator order, times sqrt(hd) (so that it is the
// accumulator's start value), -inf where the pair takes no part.  idx: Tp x Tp, -1 past T.
// Tile (a, b): rows 32 a of idx, columns 32 b; lane l holds row l % 32 and, in element r,
// column 8 (r / 4) + 4 (l / 32) + r % 4.
template <int DT>
__global__ __launch_bounds__(256) void k_relpos_bias(const uint16_t* __restrict__ idx, int32_t nt,
                                                     const uint16_t* __restrict__ table, int32_t H,
                                                     float root, float* __restrict__ bias)
{
    const int64_t n_tiles = (int64_t)nt * nt;
    const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int h = blockIdx.y, lane = threadIdx.x & 63;
    if (tile >= n_tiles)
        return;
    const int a = (int)(tile / nt), b = (int)(tile - (int64_t)a * nt);
    const uint16_t* src = idx + ((int64_t)a * 32 + (lane & 31)) * (nt * 32) + b * 32 + 4 * (lane >> 5);
    float* dst = bias + ((int64_t)h * n_tiles + tile) * 1024 + lane * 16;
    constexpr uint16_t LOWEST = DT == LPV_BF16 ? 0xff7f : 0xfbff, NEG_INF = DT == LPV_BF16 ? 0xff80 : 0xfc00;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const uint2 v = *(const uint2*)(src + 8 * g);
        const uint16_t* e = (const uint16_t*)&v;
        float4 o;
        float* of = (float*)&o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint16_t t = e[j] == 0xffff ? NEG_INF : table[(int64_t)e[j] * H + h];
            // (a finite bias stays finite: the product's overflow would mask the pair)
            const float f = fminf(fmaxf(Elem<DT>::to_f32(t) * root, -3e38f), 3e38f);
            of[j] = t == LOWEST || t == NEG_INF ? -INFINITY : f;
        }
        *(float4*)(dst + 4 * g) = o;
    }
}

__device__ inline f32x16 load_bias(const float* p)
{
    f32x16 s;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const float4 v = *(const float4*)(p + 4 * g);
        s[4 * g] = v.x;
        s[4 * g + 1] = v.y;
        s[4 * g + 2] = v.z;
        s[4 * g + 3] = v.w;
    }
    return s;
}

// BLK rows of a head's slices of two matrices, from global memory through registers into
// LDS, zero past T and for padding tokens (whose values, NaN too, then reach nothing).
template <int HD, int NT, bool REG> struct Stage {
    static constexpr int CH = HD / 8;                    // 16-byte chunks per row
    static constexpr int N = (BLK * CH + NT - 1) / NT;   // chunks per thread and matrix
    uint4 a[N], b[N];
    __device__ inline void load(const uint16_t* pa, int64_t lda, const uint16_t* pb, int64_t ldb,
                                int row0, int T, const int32_t* reg)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * NT, r = row0 + c / CH, k = c % CH;
            a[i] = uint4{0u, 0u, 0u, 0u};
            b[i] = uint4{0u, 0u, 0u, 0u};
            bool ok = r < T && c < BLK * CH;
            if (REG && ok)
                ok = reg[r] >= 0;
            if (ok) {
                a[i] = *(const uint4*)(pa + (int64_t)r * lda + 8 * k);
                b[i] = *(const uint4*)(pb + (int64_t)r * ldb + 8 * k);
            }
        }
    }
    __device__ inline void store(char* la, char* lb) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * NT;
            if (BLK * CH % NT == 0 || c < BLK * CH) {
                *(uint4*)(la + c / CH * Row<HD>::RS + 16 * (c % CH)) = a[i];
                *(uint4*)(lb + c / CH * Row<HD>::RS + 16 * (c % CH)) = b[i];
            }
        }
    }
};

// A fragment of 8 head dimensions (8 half + 16 ks ..) of one row per lane, zero unless ok.
template <typename F, int HD>
__device__ inline void load_frags(F* f, const uint16_t* row, int half, bool ok)
{
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks)
        f[ks] = as_frag<F>(ok ? *(const uint4*)(row + 8 * half + 16 * ks) : uint4{0u, 0u, 0u, 0u});
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

// The label of a padding token as the one that attends; as the one attended it is -1, so
// that the two never match.
constexpr int32_t NO_LABEL = INT32_MIN;

// 32 rows of an output whose accumulators hold one row per lane (l % 32), dimensions
// 8 (r / 4) + 4 half + r % 4 of each 32-dimension tile.
template <int DT, int HD>
__device__ inline void store_rows(uint16_t* row, const f32x16* o, float f, int half)
{
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(uint2*)(row + 32 * dt + 8 * g + 4 * half) =
                uint2{pack2<DT>(o[dt][4 * g] * f, o[dt][4 * g + 1] * f),
                      pack2<DT>(o[dt][4 * g + 2] * f, o[dt][4 * g + 3] * f)};
}

// Workgroup -> (sequence, head, block of row tiles).
struct Place {
    int64_t seq;
    int h, blk;
    bool ok;
};
__device__ inline Place place(const Rp& p, int n_blk)
{
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t u = id / p.n_seq;  // the sequences of one head's block follow each other
    return {id - u * p.n_seq, (int)(u / n_blk), (int)(u % n_blk), u < (int64_t)p.H * n_blk};
}

// ---------------------------------------------------------------- forward

// A workgroup of NW waves takes NW 32-query tiles of one sequence and head, a wave one of
// them; the keys pass in blocks of 64 through a double buffer in LDS, the next block's
// loads in flight meanwhile.  S^T = K Q^T starts from the bias in the accumulator, so a row
// of the softmax lives in lanes l and l ^ 32; the weights, rounded once to the element
// type, are then the B operand of O^T = V^T P^T (V^T by transposing LDS reads).  The
// row's sum adds the weights before that rounding, so that lse is exact to float32.
template <int DT, int HD, int NW, bool REG>
__global__ __launch_bounds__(64 * NW) void k_relpos_fwd(Rp p, uint16_t* __restrict__ out, int64_t ldo,
                                                        float* __restrict__ lse, float scale)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS, ND = Row<HD>::DT;
    __shared__ __attribute__((aligned(16))) char kv[2][2][BLK * RS];
    __shared__ __attribute__((aligned(16))) int32_t lab[2][BLK];
    const int T = p.T, n_blk = (p.nt + NW - 1) / NW;
    const Place at = place(p, n_blk);
    if (!at.ok)
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    const uint16_t* base = p.qkv + at.seq * T * ldq + at.h * HD;
    const int32_t* reg = REG ? p.region + at.seq % p.n_region * T : nullptr;
    const int qt = at.blk * NW + wave, q = qt * 32 + l32;
    const bool busy = qt < p.nt;
    F qf[KS];
    load_frags<F, HD>(qf, base + (int64_t)min(q, T - 1) * ldq, half, busy);
    int mine = 0;
    if (REG) {
        mine = reg[min(q, T - 1)];
        mine = mine < 0 ? NO_LABEL : mine;
    }
    Stage<HD, 64 * NW, REG> st;
    auto load_labels = [&](int b) {
        int32_t v = -1;
        const int r = b * BLK + threadIdx.x;
        if (REG && threadIdx.x < BLK && r < T)
            v = max(reg[r], -1);
        return v;
    };
    st.load(base + hw, ldq, base + 2 * hw, ldq, 0, T, reg);
    int32_t lv = load_labels(0);
    const int n_kb = (T + BLK - 1) / BLK;
    const float* bt = p.bias + (((int64_t)at.h * p.nt + min(qt, p.nt - 1)) * p.nt) * 1024 + lane * 16;
    f32x16 bn = load_bias(bt);
    st.store(kv[0][0], kv[0][1]);
    if (REG && threadIdx.x < BLK)
        lab[0][threadIdx.x] = lv;
    __syncthreads();
    f32x16 o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
        o[d] = f32x16{};
    float m = -INFINITY, l = 0.0f;
    for (int b = 0; b < n_kb; ++b) {
        const int cur = b & 1;
        if (b + 1 < n_kb) {
            st.load(base + hw, ldq, base + 2 * hw, ldq, (b + 1) * BLK, T, reg);
            lv = load_labels(b + 1);
        }
        if (busy) {
            const uint32_t ka = lds32(kv[cur][0]) + l32 * RS + half * 16;
            const uint32_t va = tr_base<HD>(kv[cur][1], lane);
            for (int i = 0; i < 2; ++i) {
                const int kt = 2 * b + i;
                if (kt >= p.nt)
                    break;
                f32x16 s = bn;
                bn = load_bias(bt + (int64_t)min(kt + 1, p.nt - 1) * 1024);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    s = E::mma(as_frag<F>(att_read16(ka + i * 32 * RS + 32 * ks)), qf[ks], s);
                if (REG)
                    mask_region(s, mine, lab[cur] + 32 * i, half);
                float mt = s[0];
#pragma unroll
                for (int r = 1; r < 16; ++r)
                    mt = fmaxf(mt, s[r]);
                mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
                const float mn = fmaxf(m, mt);
                const float ref = mn == -INFINITY ? 0.0f : mn;  // (nothing yet: all weights 0)
                const float nms = -ref * scale;
                const float alpha = __builtin_amdgcn_exp2f((m - ref) * scale);
                float ps = 0.0f;
                uint32_t pb[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float e0 = __builtin_amdgcn_exp2f(fmaf(s[2 * j], scale, nms));
                    const float e1 = __builtin_amdgcn_exp2f(fmaf(s[2 * j + 1], scale, nms));
                    ps += e0 + e1;
                    pb[j] = pack2<DT>(e0, e1);
                }
                ps += __shfl_xor(ps, 32, 64);
                l = l * alpha + ps;
                m = mn;
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[d] *= alpha;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const F pf = as_frag<F>(uint4{pb[4 * t], pb[4 * t + 1], pb[4 * t + 2], pb[4 * t + 3]});
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        o[d] = E::mma(tr_frag<F, HD>(va, 32 * i + 16 * t, d), pf, o[d]);
                }
            }
        }
        if (b + 1 < n_kb) {
            st.store(kv[1 - cur][0], kv[1 - cur][1]);
            if (REG && threadIdx.x < BLK)
                lab[1 - cur][threadIdx.x] = lv;
        }
        __syncthreads();
    }
    if (busy && q < T) {
        store_rows<DT, HD>(out + (at.seq * T + q) * ldo + at.h * HD, o, l > 0.0f ? 1.0f / l : 0.0f, half);
        if (lse && half == 0)
            lse[(at.seq * p.H + at.h) * T + q] =
                l > 0.0f ? LN2 * (m * scale + __log2f(l)) : -INFINITY;
    }
}

// ---------------------------------------------------------------- gradients

// dQ, tiled as the forward: the weights come back from lse, dP^T = V dO^T, and dS^T,
// rounded once, is the B operand of dQ^T = K^T dS^T.  D = dO . O is formed first and kept
// for the next kernel.
template <int DT, int HD, int NW, bool REG>
__global__ __launch_bounds__(64 * NW) void k_relpos_dq(Rp p, const uint16_t* __restrict__ out,
                                                       int64_t ldo, const float* __restrict__ lse,
                                                       const uint16_t* __restrict__ dout, int64_t ldg,
                                                       float* __restrict__ Dv,
                                                       uint16_t* __restrict__ dqkv, int64_t lddq,
                                                       float scale, float rroot)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS, ND = Row<HD>::DT;
    __shared__ __attribute__((aligned(16))) char kv[2][2][BLK * RS];
    __shared__ __attribute__((aligned(16))) int32_t lab[2][BLK];
    const int T = p.T, n_blk = (p.nt + NW - 1) / NW;
    const Place at = place(p, n_blk);
    if (!at.ok)
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    const uint16_t* base = p.qkv + at.seq * T * ldq + at.h * HD;
    const int32_t* reg = REG ? p.region + at.seq % p.n_region * T : nullptr;
    const int qt = at.blk * NW + wave, q = qt * 32 + l32, qc = min(q, T - 1);
    const bool busy = qt < p.nt;
    int mine = 0;
    if (REG) {
        mine = reg[qc];
        mine = mine < 0 ? NO_LABEL : mine;
    }
    const bool live = busy && mine != NO_LABEL;
    F qf[KS], gf[KS], of[KS];
    load_frags<F, HD>(qf, base + (int64_t)qc * ldq, half, live);
    load_frags<F, HD>(gf, dout + (at.seq * T + qc) * ldg + at.h * HD, half, live);
    load_frags<F, HD>(of, out + (at.seq * T + qc) * ldo + at.h * HD, half, live);
    float D = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            D = fmaf((float)gf[ks][j], (float)of[ks][j], D);
    D += __shfl_xor(D, 32, 64);
    const int64_t stat = (at.seq * p.H + at.h) * T;
    float nl = -INFINITY;  // -lse in base 2; a row without pairs: every weight 2^-inf
    if (busy) {
        const float v = lse[stat + qc];
        nl = v == -INFINITY ? -INFINITY : -v * LOG2E;
        if (half == 0 && q < T)
            Dv[stat + q] = D;
    }
    Stage<HD, 64 * NW, REG> st;
    auto load_labels = [&](int b) {
        int32_t v = -1;
        const int r = b * BLK + threadIdx.x;
        if (REG && threadIdx.x < BLK && r < T)
            v = max(reg[r], -1);
        return v;
    };
    st.load(base + hw, ldq, base + 2 * hw, ldq, 0, T, reg);
    int32_t lv = load_labels(0);
    const int n_kb = (T + BLK - 1) / BLK;
    const float* bt = p.bias + (((int64_t)at.h * p.nt + min(qt, p.nt - 1)) * p.nt) * 1024 + lane * 16;
    f32x16 bn = load_bias(bt);
    st.store(kv[0][0], kv[0][1]);
    if (REG && threadIdx.x < BLK)
        lab[0][threadIdx.x] = lv;
    __syncthreads();
    f32x16 dq[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
        dq[d] = f32x16{};
    for (int b = 0; b < n_kb; ++b) {
        const int cur = b & 1;
        if (b + 1 < n_kb) {
            st.load(base + hw, ldq, base + 2 * hw, ldq, (b + 1) * BLK, T, reg);
            lv = load_labels(b + 1);
        }
        if (busy) {
            const uint32_t ka = lds32(kv[cur][0]) + l32 * RS + half * 16;
            const uint32_t va = lds32(kv[cur][1]) + l32 * RS + half * 16;
            const uint32_t kt_a = tr_base<HD>(kv[cur][0], lane);
            for (int i = 0; i < 2; ++i) {
                const int kt = 2 * b + i;
                if (kt >= p.nt)
                    break;
                f32x16 s = bn, dp = {};
                bn = load_bias(bt + (int64_t)min(kt + 1, p.nt - 1) * 1024);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    s = E::mma(as_frag<F>(att_read16(ka + i * 32 * RS + 32 * ks)), qf[ks], s);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    dp = E::mma(as_frag<F>(att_read16(va + i * 32 * RS + 32 * ks)), gf[ks], dp);
                if (REG)
                    mask_region(s, mine, lab[cur] + 32 * i, half);
                uint32_t db[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float e0 = __builtin_amdgcn_exp2f(fmaf(s[2 * j], scale, nl));
                    const float e1 = __builtin_amdgcn_exp2f(fmaf(s[2 * j + 1], scale, nl));
                    db[j] = pack2<DT>(e0 * (dp[2 * j] - D), e1 * (dp[2 * j + 1] - D));
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const F df = as_frag<F>(uint4{db[4 * t], db[4 * t + 1], db[4 * t + 2], db[4 * t + 3]});
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        dq[d] = E::mma(tr_frag<F, HD>(kt_a, 32 * i + 16 * t, d), df, dq[d]);
                }
            }
        }
        if (b + 1 < n_kb) {
            st.store(kv[1 - cur][0], kv[1 - cur][1]);
            if (REG && threadIdx.x < BLK)
                lab[1 - cur][threadIdx.x] = lv;
        }
        __syncthreads();
    }
    if (busy && q < T)
        store_rows<DT, HD>(dqkv + (at.seq * T + q) * lddq + at.h * HD, dq, rroot, half);
}

// dK and dV: a wave holds a 32-key tile, the queries pass in blocks with their lse and D.
// S = Q K^T and dP = dO V^T (lane = key) make P and dS the B operands of dV^T = dO^T P and
// dK^T = Q^T dS as they stand.  The bias tiles are those of the transposed index.
template <int DT, int HD, int NW, bool REG>
__global__ __launch_bounds__(64 * NW) void k_relpos_dkv(Rp p, const float* __restrict__ lse,
                                                        const float* __restrict__ Dv,
                                                        const uint16_t* __restrict__ dout, int64_t ldg,
                                                        uint16_t* __restrict__ dqkv, int64_t lddq,
                                                        float scale, float rroot)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS, ND = Row<HD>::DT;
    __shared__ __attribute__((aligned(16))) char qg[2][2][BLK * RS];
    __shared__ __attribute__((aligned(16))) float stats[2][2][BLK];
    __shared__ __attribute__((aligned(16))) int32_t lab[2][BLK];
    const int T = p.T, n_blk = (p.nt + NW - 1) / NW;
    const Place at = place(p, n_blk);
    if (!at.ok)
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    const uint16_t* base = p.qkv + at.seq * T * ldq + at.h * HD;
    const uint16_t* gbase = dout + at.seq * T * ldg + at.h * HD;
    const int32_t* reg = REG ? p.region + at.seq % p.n_region * T : nullptr;
    const int kt = at.blk * NW + wave, k = kt * 32 + l32, kc = min(k, T - 1);
    const bool busy = kt < p.nt;
    int mine = 0;
    if (REG) {
        mine = reg[kc];
        mine = mine < 0 ? NO_LABEL : mine;
    }
    const bool live = busy && k < T && mine != NO_LABEL;
    F kf[KS], vf[KS];
    load_frags<F, HD>(kf, base + hw + (int64_t)kc * ldq, half, live);
    load_frags<F, HD>(vf, base + 2 * hw + (int64_t)kc * ldq, half, live);
    const int64_t stat = (at.seq * p.H + at.h) * T;
    Stage<HD, 64 * NW, REG> st;
    float sl, sd;
    int32_t lv;
    // -lse in base 2 (-inf past T and for rows without pairs: every weight 0), D and label
    auto load_stats = [&](int b) {
        sl = -INFINITY;
        sd = 0.0f;
        lv = -1;
        const int r = b * BLK + threadIdx.x;
        if (threadIdx.x < BLK && r < T) {
            const float v = lse[stat + r];
            sl = v == -INFINITY ? -INFINITY : -v * LOG2E;
            sd = Dv[stat + r];
            if (REG)
                lv = max(reg[r], -1);
        }
    };
    auto store_stats = [&](int buf) {
        if (threadIdx.x < BLK) {
            stats[buf][0][threadIdx.x] = sl;
            stats[buf][1][threadIdx.x] = sd;
            if (REG)
                lab[buf][threadIdx.x] = lv;
        }
    };
    st.load(base, ldq, gbase, ldg, 0, T, reg);
    load_stats(0);
    const int n_qb = (T + BLK - 1) / BLK;
    const float* bt = p.bias + (((int64_t)at.h * p.nt + min(kt, p.nt - 1)) * p.nt) * 1024 + lane * 16;
    f32x16 bn = load_bias(bt);
    st.store(qg[0][0], qg[0][1]);
    store_stats(0);
    __syncthreads();
    f32x16 dk[ND], dv[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) {
        dk[d] = f32x16{};
        dv[d] = f32x16{};
    }
    for (int b = 0; b < n_qb; ++b) {
        const int cur = b & 1;
        if (b + 1 < n_qb) {
            st.load(base, ldq, gbase, ldg, (b + 1) * BLK, T, reg);
            load_stats(b + 1);
        }
        if (busy) {
            const uint32_t qa = lds32(qg[cur][0]) + l32 * RS + half * 16;
            const uint32_t ga = lds32(qg[cur][1]) + l32 * RS + half * 16;
            const uint32_t qtr = tr_base<HD>(qg[cur][0], lane), gtr = tr_base<HD>(qg[cur][1], lane);
            for (int i = 0; i < 2; ++i) {
                const int qt = 2 * b + i;
                if (qt >= p.nt)
                    break;
                f32x16 s = bn, dp = {};
                bn = load_bias(bt + (int64_t)min(qt + 1, p.nt - 1) * 1024);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    s = E::mma(as_frag<F>(att_read16(qa + i * 32 * RS + 32 * ks)), kf[ks], s);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    dp = E::mma(as_frag<F>(att_read16(ga + i * 32 * RS + 32 * ks)), vf[ks], dp);
                if (REG)
                    mask_region(s, mine, lab[cur] + 32 * i, half);
                uint32_t pb[8], db[8];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 nl = *(const float4*)(stats[cur][0] + 32 * i + 8 * g + 4 * half);
                    const float4 D = *(const float4*)(stats[cur][1] + 32 * i + 8 * g + 4 * half);
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
                for (int t = 0; t < 2; ++t) {
                    const F pf = as_frag<F>(uint4{pb[4 * t], pb[4 * t + 1], pb[4 * t + 2], pb[4 * t + 3]});
                    const F df = as_frag<F>(uint4{db[4 * t], db[4 * t + 1], db[4 * t + 2], db[4 * t + 3]});
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        dv[d] = E::mma(tr_frag<F, HD>(gtr, 32 * i + 16 * t, d), pf, dv[d]);
                        dk[d] = E::mma(tr_frag<F, HD>(qtr, 32 * i + 16 * t, d), df, dk[d]);
                    }
                }
            }
        }
        if (b + 1 < n_qb) {
            st.store(qg[1 - cur][0], qg[1 - cur][1]);
            store_stats(1 - cur);
        }
        __syncthreads();
    }
    if (busy && k < T) {
        uint16_t* row = dqkv + (at.seq * T + k) * lddq + at.h * HD;
        store_rows<DT, HD>(row + hw, dk, rroot, half);
        store_rows<DT, HD>(row + 2 * hw, dv, 1.0f, half);
    }
}

// Sum over a chunk of sequences of dS of one head's pairs, 64 x 64 pairs to a workgroup of
// four waves (a 32 x 32 tile each, summed in its accumulators' places in float32), the four
// matrices' rows staged in LDS a sequence ahead.  part: [head][chunk][tile][lane][16].
template <int DT, int HD, bool REG>
__global__ __launch_bounds__(256) void k_relpos_dbias(Rp p, const float* __restrict__ lse,
                                                      const float* __restrict__ Dv,
                                                      const uint16_t* __restrict__ dout, int64_t ldg,
                                                      float* __restrict__ part, int32_t chunks,
                                                      float scale)
{
    using E = Elem<DT>;
    using F = typename E::frag;
    constexpr int RS = Row<HD>::RS, KS = Row<HD>::KS;
    __shared__ __attribute__((aligned(16))) char rows[4][BLK * RS];  // Q, dO, K, V
    const int T = p.T, n_blk = (p.nt + 1) / 2;
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t u = id / chunks;
    const int chunk = (int)(id - u * chunks);
    const int h = (int)(u / ((int64_t)n_blk * n_blk)), ab = (int)(u % ((int64_t)n_blk * n_blk));
    if (h >= p.H)
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
    const int qb = ab / n_blk, kb = ab - qb * n_blk;
    const int qt = 2 * qb + (wave >> 1), kt = 2 * kb + (wave & 1);
    const int64_t ldq = p.ldq, hw = (int64_t)p.H * HD;
    const bool busy = qt < p.nt && kt < p.nt;
    const int q = qt * 32 + l32, qc = min(q, T - 1);
    const f32x16 bias = load_bias(
        p.bias + (((int64_t)h * p.nt + min(qt, p.nt - 1)) * p.nt + min(kt, p.nt - 1)) * 1024 + lane * 16);
    const int64_t s0 = p.n_seq * chunk / chunks, s1 = p.n_seq * (chunk + 1) / chunks;
    Stage<HD, 256, REG> sq, sk;
    auto load = [&](int64_t seq) {
        const uint16_t* base = p.qkv + seq * T * ldq + h * HD;
        const int32_t* reg = REG ? p.region + seq % p.n_region * T : nullptr;
        sq.load(base, ldq, dout + seq * T * ldg + h * HD, ldg, qb * BLK, T, reg);
        sk.load(base + hw, ldq, base + 2 * hw, ldq, kb * BLK, T, reg);
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
        const float v = lse[stat + qc], D = Dv[stat + qc];
        // (a query past T: every weight 2^-inf)
        const float nl = v == -INFINITY || q >= T ? -INFINITY : -v * LOG2E;
        __syncthreads();
        if (seq + 1 < s1)
            load(seq + 1);
        if (busy) {
            f32x16 s = bias, dp = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = E::mma(as_frag<F>(att_read16(ka + 32 * ks)), as_frag<F>(att_read16(qa + 32 * ks)), s);
                dp = E::mma(as_frag<F>(att_read16(va + 32 * ks)), as_frag<F>(att_read16(ga + 32 * ks)), dp);
            }
            if (REG) {
                const int32_t* reg = p.region + seq % p.n_region * T;
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
        float* dst = part + (((int64_t)h * chunks + chunk) * p.nt * p.nt + (int64_t)qt * p.nt + kt) * 1024 +
                     lane * 16;
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(float4*)(dst + 4 * g) = float4{sum[4 * g], sum[4 * g + 1], sum[4 * g + 2], sum[4 * g + 3]};
    }
}

// The pairs of a bucket, in segments: order[seg_ptr[g] .. seg_ptr[g + 1]) are places in a
// head's tiles.  A workgroup adds one segment over all chunks, each thread its pairs in
// order, then a fixed tree; out: [segment][head] (16-bit: the table's gradient itself,
// where every bucket is one segment).
template <int DT>
__global__ __launch_bounds__(256) void k_relpos_segments(const int32_t* __restrict__ order,
                                                         const int32_t* __restrict__ seg_ptr,
                                                         const float* __restrict__ part, int32_t chunks,
                                                         int64_t n_pos, int32_t H, float* __restrict__ sums,
                                                         uint16_t* __restrict__ dtable)
{
    __shared__ float red[4];
    const int g = blockIdx.x, h = blockIdx.y;
    const float* base = part + (int64_t)h * chunks * n_pos;
    float v = 0.0f;
    for (int i = seg_ptr[g] + threadIdx.x; i < seg_ptr[g + 1]; i += 256) {
        const float* at = base + order[i];
        for (int c = 0; c < chunks; ++c)
            v += at[c * n_pos];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0)
        red[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        v = (red[0] + red[1]) + (red[2] + red[3]);
        if (dtable)
            dtable[(int64_t)g * H + h] = Elem<DT>::from_f32(v);
        else
            sums[(int64_t)g * H + h] = v;
    }
}

// The segments of each bucket, in order.
template <int DT>
__global__ __launch_bounds__(256) void k_relpos_buckets(const int32_t* __restrict__ bucket_seg,
                                                        const float* __restrict__ sums, int32_t n_buckets,
                                                        int32_t H, uint16_t* __restrict__ dtable)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)n_buckets * H)
        return;
    const int b = (int)(i / H), h = (int)(i - (int64_t)b * H);
    float v = 0.0f;
    for (int g = bucket_seg[b]; g < bucket_seg[b + 1]; ++g)
        v += sums[(int64_t)g * H + h];
    dtable[i] = Elem<DT>::from_f32(v);
}

int64_t tile_floats(const lpv_relpos* h) { return (int64_t)h->nt * h->nt * 1024; }

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Chunks of sequences of the bias gradient: 1024 workgroups, four to a compute unit.
int bias_chunks(const lpv_relpos* h, int64_t n_seq, int32_t H)
{
    const int64_t n_blk = (h->nt + 1) / 2, wgs = (int64_t)H * n_blk * n_blk;
    const int64_t c = (1024 + wgs - 1) / wgs;
    return (int)(c < n_seq ? c : n_seq);
}

struct Ws {  // places in a gradient's workspace
    float *bias, *bias_t, *D, *part, *sums;
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
    w.bias = take((size_t)(H * tile_floats(h)));
    w.bias_t = take((size_t)(H * tile_floats(h)));
    w.D = take((size_t)(n_seq * H * h->T));
    w.part = take((size_t)(H * bias_chunks(h, n_seq, H) * tile_floats(h)));
    w.sums = take((size_t)((int64_t)h->n_segs * H));
    w.bytes = at;
    return w;
}

template <int DT>
hipError_t expand_bias(const lpv_relpos* h, bool transposed, const void* table, int32_t H, int32_t hd,
                       float* bias, hipStream_t s)
{
    const int64_t tiles = (int64_t)h->nt * h->nt;
    hipLaunchKernelGGL((k_relpos_bias<DT>), dim3((uint32_t)((tiles + 3) / 4), H), dim3(256), 0, s,
                       transposed ? h->idx_t : h->idx, h->nt, (const uint16_t*)table, H,
                       sqrtf((float)hd), bias);
    return hipGetLastError();
}

constexpr int NW = 4;

template <int DT, int HD, bool REG> hipError_t forward_as(const lpv_relpos* h, const RelposCall& c, hipStream_t s)
{
    hipError_t e = expand_bias<DT>(h, false, c.table, c.H, HD, (float*)c.ws, s);
    if (e != hipSuccess)
        return e;
    const Rp p = {(const uint16_t*)c.qkv, c.ldq, c.region, c.n_region, c.n_seq, h->T, c.H, h->nt,
                  (const float*)c.ws};
    const int64_t wgs = c.n_seq * c.H * ((h->nt + NW - 1) / NW);
    const Grid2 g = grid_of(wgs);
    hipLaunchKernelGGL((k_relpos_fwd<DT, HD, NW, REG>), dim3(g.x, g.y), dim3(64 * NW), 0, s, p,
                       (uint16_t*)c.out, c.ldo, c.lse, LOG2E / sqrtf((float)HD));
    return hipGetLastError();
}

template <int DT, int HD, bool REG>
hipError_t grad_as(const lpv_relpos* h, const RelposCall& c, hipStream_t s)
{
    const Ws w = grad_ws(h, c.n_seq, c.H, c.ws);
    const int chunks = bias_chunks(h, c.n_seq, c.H);
    if (chunks > 0) {  // (n_seq > 0)
        const float scale = LOG2E / sqrtf((float)HD), rroot = 1.0f / sqrtf((float)HD);
        hipError_t e = expand_bias<DT>(h, false, c.table, c.H, HD, w.bias, s);
        if (e == hipSuccess)
            e = expand_bias<DT>(h, true, c.table, c.H, HD, w.bias_t, s);
        if (e != hipSuccess)
            return e;
        Rp p = {(const uint16_t*)c.qkv, c.ldq, c.region, c.n_region, c.n_seq, h->T, c.H, h->nt, w.bias};
        const Grid2 g = grid_of(c.n_seq * c.H * ((h->nt + NW - 1) / NW));
        hipLaunchKernelGGL((k_relpos_dq<DT, HD, NW, REG>), dim3(g.x, g.y), dim3(64 * NW), 0, s, p,
                           (const uint16_t*)c.out, c.ldo, c.lse, (const uint16_t*)c.dout, c.ldg, w.D,
                           (uint16_t*)c.dqkv, c.lddq, scale, rroot);
        p.bias = w.bias_t;
        hipLaunchKernelGGL((k_relpos_dkv<DT, HD, NW, REG>), dim3(g.x, g.y), dim3(64 * NW), 0, s, p, c.lse, w.D,
                           (const uint16_t*)c.dout, c.ldg, (uint16_t*)c.dqkv, c.lddq, scale, rroot);
        p.bias = w.bias;
        const int64_t n_blk = (h->nt + 1) / 2;
        const Grid2 gb = grid_of((int64_t)c.H * n_blk * n_blk * chunks);
        hipLaunchKernelGGL((k_relpos_dbias<DT, HD, REG>), dim3(gb.x, gb.y), dim3(256), 0, s, p, c.lse, w.D,
                           (const uint16_t*)c.dout, c.ldg, w.part, chunks, scale);
    }
    const bool whole = h->n_segs == h->n_buckets;
    hipLaunchKernelGGL((k_relpos_segments<DT>), dim3(h->n_segs, c.H), dim3(256), 0, s, h->order, h->seg_ptr,
                       w.part, chunks, tile_floats(h), c.H, w.sums, whole ? (uint16_t*)c.dtable : nullptr);
    if (!whole)
        hipLaunchKernelGGL((k_relpos_buckets<DT>),
                           dim3((uint32_t)(((int64_t)h->n_buckets * c.H + 255) / 256)), dim3(256), 0, s,
                           h->bucket_seg, w.sums, h->n_buckets, c.H, (uint16_t*)c.dtable);
    return hipGetLastError();
}

}  // namespace

size_t relpos_workspace_bytes(const lpv_relpos* h, int64_t n_seq, int32_t H, bool grad)
{
    if (grad)
        return grad_ws(h, n_seq, H, nullptr).bytes;
    return up256((size_t)(H * tile_floats(h)) * sizeof(float));
}

RelposSizes relpos_sizes(const int32_t* index, int32_t T, int32_t n_buckets, int32_t* count)
{
    RelposSizes z = {};
    z.bad = -1;
    for (int32_t b = 0; b < n_buckets; ++b)
        count[b] = 0;
    for (int64_t i = 0; i < (int64_t)T * T; ++i) {
        if (index[i] < -1 || index[i] >= n_buckets) {
            z.bad = i;
            return z;
        }
        if (index[i] >= 0)
            ++count[index[i]];
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
    for (int32_t i = 0; i < T; ++i)
        for (int32_t j = 0; j < T; ++j) {
            const int32_t b = index[(int64_t)i * T + j];
            if (b < 0)
                continue;
            idx[i * Tp + j] = (uint16_t)b;
            idx_t[j * Tp + i] = (uint16_t)b;
            // the pair's place in a head's tiles: row i % 32 in the lanes
            const int32_t c = j % 32, lane = i % 32 + 32 * (c / 4 % 2), r = 4 * (c / 8) + c % 4;
            order[count[b]++] = ((i / 32) * nt + j / 32) * 1024 + lane * 16 + r;
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
