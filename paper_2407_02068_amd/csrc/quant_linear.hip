// quant_linear.hip -- the linear layer over 8-bit codes: a weight packed with a scale for each
// output, its kept blocks only or all of them, times activations with a scale for each
// token (gfx950).
//
//   Y[m][n] = g(xs[m] ws[n] sum_k Xq[m][k] Wq[n][k] + b[n])
//
// The sums are integers (v_mfma_i32_32x32x32_i8, K <= 65536: below 2^31), so they are the
// same in any order; then one float32 conversion, the two scales, bias, g, one rounding.
//
// The weight lies in 32 x 32 tiles of 1 KB in operand order: lane l holds the 16 codes of row
// l % 32 from column 16 (l / 32) on.  As A operand a tile meets X^T as B: lane l brings the
// 16 codes of token l % 32 from the same columns, and holds in accumulator register r
// output 8 (r / 4) + 4 (l / 32) + r % 4 of that token.  A 0 for a dropped 16 x 16 part of a
// tile is exact in integers, whatever X holds.
#include "lpv_device.h"
#include "lpv_grid.h"
#include "lpv_internal.h"
#include "lpv_lds.h"

namespace lpv {
namespace {

typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ inline i32x16 mma8(v4i w, v4i x, i32x16 acc)
{
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x, acc, 0, 0, 0);
}

// ---------------------------------------------------------------- packing

// The tile (row tr, column tc) has a kept block.
__device__ inline bool tile_kept(const lpv_quant& h, const uint8_t* mask, int tr, int tc)
{
    if (tr >= h.n_tile_rows || tc >= h.n_tile_cols)
        return false;
    if (!mask)
        return true;
    const int r0 = tr * TILE / h.b_r, r1 = min((tr * TILE + TILE - 1) / h.b_r, h.R - 1);
    const int c0 = tc * TILE / h.b_c, c1 = min((tc * TILE + TILE - 1) / h.b_c, h.C - 1);
    bool kept = false;
    for (int r = r0; r <= r1; ++r)
        for (int c = c0; c <= c1; ++c)
            kept |= mask[(int64_t)r * h.C + c] != 0;
    return kept;
}

__device__ inline int groups_of(uint32_t bits)
{
    return max((__popc((bits | bits >> 16) & 0xffff) + 3) / 4, 1);
}

// One wave to a pair of tile rows: the kept columns of its chunks.
__global__ __launch_bounds__(64) void k_quant_bits(const lpv_quant h, const uint8_t* __restrict__ mask)
{
    const int pair = blockIdx.x, lane = threadIdx.x;
    for (int c = 0; c < h.n_chunks; ++c) {
        const bool kept = lane < 32 && tile_kept(h, mask, 2 * pair + (lane >> 4), c * QUANT_CHUNK + (lane & 15));
        const uint32_t bits = (uint32_t)__ballot(kept);
        if (lane == 0)
            h.bits[(int64_t)pair * h.n_chunks + c] = bits;
    }
}

// One workgroup: a thread to a pair (at most 1024), the sums over the pairs before it.
__global__ __launch_bounds__(1024) void k_quant_scan(const lpv_quant h, const uint8_t* __restrict__ mask,
                                                     QuantTotals* __restrict__ totals)
{
    __shared__ int s_tiles[1024], s_groups[1024], s_blocks;
    const int p = threadIdx.x;
    if (p == 0)
        s_blocks = 0;
    int even = 0, odd = 0, groups = 0;
    if (p < h.n_pairs)
        for (int c = 0; c < h.n_chunks; ++c) {
            const uint32_t b = h.bits[(int64_t)p * h.n_chunks + c];
            even += __popc(b & 0xffff);
            odd += __popc(b >> 16);
            groups += groups_of(b);
        }
    s_tiles[p] = even + odd;
    s_groups[p] = groups;
    __syncthreads();
    for (int d = 1; d < 1024; d <<= 1) {  // inclusive sums
        const int t = p >= d ? s_tiles[p - d] : 0, g = p >= d ? s_groups[p - d] : 0;
        __syncthreads();
        s_tiles[p] += t;
        s_groups[p] += g;
        __syncthreads();
    }
    if (p < h.n_pairs) {
        const int t0 = s_tiles[p] - even - odd;
        h.tile0[p] = t0;
        h.group0[p] = s_groups[p] - groups;
        if (2 * p < h.n_tile_rows)
            h.row_tile0[2 * p] = t0;
        if (2 * p + 1 < h.n_tile_rows)
            h.row_tile0[2 * p + 1] = t0 + even;
        if (p == h.n_pairs - 1) {
            h.tile0[h.n_pairs] = h.row_tile0[h.n_tile_rows] = s_tiles[p];
            h.group0[h.n_pairs] = s_groups[p];
        }
    }
    if (mask) {
        int n = 0;
        for (int64_t i = p; i < (int64_t)h.R * h.C; i += 1024)
            n += mask[i] != 0;
        n = wave_sum(n);
        if ((p & 63) == 0)
            atomicAdd(&s_blocks, n);  // (a count: any order)
        __syncthreads();
    }
    if (p == 0)
        *totals = QuantTotals{s_tiles[1023], s_groups[1023], mask ? s_blocks : h.R * h.C};
}

// One workgroup of 4 waves to a pair: wave w its chunks w, w + 4, ...
__global__ __launch_bounds__(256) void k_quant_fill(const lpv_quant h, const int8_t* __restrict__ W,
                                                    int64_t ldw, const float* __restrict__ scale,
                                                    const uint8_t* __restrict__ mask)
{
    const int pair = blockIdx.x, lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (wave == 0) {
        const int64_t n = (int64_t)pair * 64 + lane;
        h.scale[n] = n < h.N ? scale[n] : 0.0f;
    }
    const uint32_t* bits = h.bits + (int64_t)pair * h.n_chunks;
    int tile = h.tile0[pair], group = h.group0[pair];
    int at[2] = {0, 0};  // this pair's entries of either row in list
    if (2 * pair < h.n_tile_rows)
        at[0] = h.row_tile0[2 * pair];
    if (2 * pair + 1 < h.n_tile_rows)
        at[1] = h.row_tile0[2 * pair + 1];
    for (int c = 0; c < h.n_chunks; ++c) {
        const uint32_t b = __builtin_amdgcn_readfirstlane(bits[c]);
        const uint32_t e = b & 0xffff, o = b >> 16, any = e | o;
        if ((c & 3) == wave) {
            uint32_t left = any, desc = 0;
            const uint32_t last = 1u << 24 | (c == h.n_chunks - 1 ? 1u << 25 : 0u);
            int t = tile, n = 0, g = group, first = tile;
            if (any == 0 && lane == 0)
                h.groups[g] = uint2{last, (uint32_t)first};
            while (left) {
                const int col = __builtin_ctz(left);
                left &= left - 1;
                const uint32_t kept = (e >> col & 1) | (o >> col & 1) << 1;
                desc |= (uint32_t)(col | kept << 4) << (6 * n++);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (kept >> j & 1) {
                        const int tc = c * QUANT_CHUNK + col;
                        const int64_t row = (int64_t)(2 * pair + j) * TILE + (lane & 31);
                        const int64_t k = (int64_t)tc * TILE + 16 * (lane >> 5);
                        uint4 v = {0, 0, 0, 0};
                        if (row < h.N && k < h.K && (!mask || mask[row / h.b_r * h.C + k / h.b_c]))
                            v = *(const uint4*)(W + row * ldw + k);
                        *(uint4*)(h.tiles + (int64_t)t * 1024 + lane * 16) = v;
                        if (lane == 0)
                            h.list[at[j] + __popc((j ? o : e) & ((1u << col) - 1))] = int2{tc, t};
                        ++t;
                    }
                if (n == 4 || left == 0) {
                    if (lane == 0)
                        h.groups[g] = uint2{left ? desc : desc | last, (uint32_t)first};
                    ++g;
                    n = 0;
                    desc = 0;
                    first = t;
                }
            }
        }
        tile += __popc(e) + __popc(o);
        at[0] += __popc(e);
        at[1] += __popc(o);
        group += groups_of(b);
    }
}

// ---------------------------------------------------------------- the epilogue's arithmetic

// GELU for float32 outputs, to their own rounding (gelu_erf's 5e-6 would show there).
__device__ inline float gelu_f32(float v) { return 0.5f * v * erfcf(v * -0.70710678118654752f); }

// Four outputs of a token: sums, the token's scale, the outputs' scales and bias.
template <int OUT, bool GELU> __device__ inline void finish4(const int s[4], float xs, float4 ws, float4 b, float out[4])
{
    const float w[4] = {ws.x, ws.y, ws.z, ws.w}, c[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        out[i] = fmaf((float)s[i] * xs, w[i], c[i]);
        if (GELU)
            out[i] = OUT == LPV_F32 ? gelu_f32(out[i]) : gelu_erf(out[i]);
    }
}

// Four neighbours of the bias from output n on (a multiple of 4, below N).
template <int OUT> __device__ inline float4 bias4(const char* bias, int64_t n)
{
    if (!bias)
        return float4{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (OUT == LPV_F32) {
        return *(const float4*)(bias + n * 4);
    } else {
        const uint2 v = *(const uint2*)(bias + n * 2);
        using E = Elem<OUT>;
        return float4{E::to_f32((uint16_t)v.x), E::to_f32((uint16_t)(v.x >> 16)),
                      E::to_f32((uint16_t)v.y), E::to_f32((uint16_t)(v.y >> 16))};
    }
}

// ---------------------------------------------------------------- few tokens

struct QuantDims {
    int64_t ldx, M, K, N, ldy;
    int32_t n_tile_rows;
    int64_t n_units;
};

// 32 TU tokens times one tile row to a workgroup, whose 8 waves share the row's kept tiles, 8
// neighbours of the list at a time; the partial sums meet in LDS.  Both operands come
// straight from memory in operand order, so any size will do.
constexpr int FEW_WAVES = 8;

template <int OUT, bool GELU, int TU>
__global__ __launch_bounds__(64 * FEW_WAVES) void k_quant_few(
    const QuantDims a, const int8_t* __restrict__ X, const float* __restrict__ xscale,
    const char* __restrict__ tiles, const int2* __restrict__ list, const int32_t* __restrict__ row_tile0,
    const float* __restrict__ wscale, const char* __restrict__ bias, char* __restrict__ Y)
{
    constexpr int ES = OUT == LPV_F32 ? 4 : 2, U = 4;  // tiles asked for at a time
    __shared__ v4i s_part[FEW_WAVES][TU * 4][64];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int64_t unit = blockIdx.x; unit < a.n_units; unit += gridDim.x) {
        const int64_t mt = unit / a.n_tile_rows;
        const int row = (int)(unit - mt * a.n_tile_rows);
        const int64_t m0 = mt * (32 * TU);
        const int8_t* xr[TU];
#pragma unroll
        for (int u = 0; u < TU; ++u)
            xr[u] = X + min(m0 + 32 * u + (lane & 31), a.M - 1) * a.ldx;
        i32x16 acc[TU];
#pragma unroll
        for (int u = 0; u < TU; ++u)
            acc[u] = i32x16{};
        const int t0 = row_tile0[row], n = row_tile0[row + 1] - t0;
        // this wave's tiles: places wave, wave + 8, ... of the row's
        const int mine = n > wave ? (n - wave + FEW_WAVES - 1) / FEW_WAVES : 0;
        for (int base = 0; base < mine; base += 64) {
            const int2 e = list[t0 + wave + FEW_WAVES * min(base + lane, mine - 1)];
            const int here = min(mine - base, 64);
            for (int i0 = 0; i0 < here; i0 += U) {
                v4i w[U], x[U][TU];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int p = min(i0 + i, here - 1);
                    const int col = __builtin_amdgcn_readlane(e.x, p), t = __builtin_amdgcn_readlane(e.y, p);
                    w[i] = *(const v4i*)(tiles + (int64_t)t * 1024 + lane * 16);
                    // (a half past K is zero in the tile: any codes do, the row's first)
                    int k = col * TILE + 16 * h;
                    k = k < a.K ? k : 0;
#pragma unroll
                    for (int u = 0; u < TU; ++u)
                        x[i][u] = *(const v4i*)(xr[u] + k);
                }
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (i0 + i < here)
#pragma unroll
                        for (int u = 0; u < TU; ++u)
                            acc[u] = mma8(w[i], x[i][u], acc[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < TU; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                s_part[wave][u * 4 + q][lane] = v4i{acc[u][4 * q], acc[u][4 * q + 1], acc[u][4 * q + 2],
                                                    acc[u][4 * q + 3]};
        __syncthreads();
        for (int i = tid; i < TU * 256; i += 64 * FEW_WAVES) {
            const int uq = i >> 6, l = i & 63;
            int s[4] = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < FEW_WAVES; ++w) {
                const v4i v = s_part[w][uq][l];
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    s[b] += v[b];
            }
            const int64_t m = m0 + 32 * (uq >> 2) + (l & 31);
            const int64_t at = (int64_t)row * TILE + 8 * (uq & 3) + 4 * (l >> 5);
            if (m < a.M && at < a.N) {
                float o[4];
                finish4<OUT, GELU>(s, xscale[m], *(const float4*)(wscale + at), bias4<OUT>(bias, at), o);
                char* y = Y + (m * a.ldy + at) * ES;
                if constexpr (OUT == LPV_F32)
                    *(float4*)y = float4{o[0], o[1], o[2], o[3]};
                else
                    *(uint2*)y = uint2{pack2<OUT>(o[0], o[1]), pack2<OUT>(o[2], o[3])};
            }
        }
        __syncthreads();  // (the sums are read: the next unit's may be written)
    }
}

template <int OUT, bool GELU, int TU>
hipError_t launch_few(const lpv_quant* h, const QuantLinearCall& c, hipStream_t s)
{
    QuantDims d = {c.ldx, c.M, h->K, h->N, c.ldy, h->n_tile_rows, 0};
    d.n_units = (c.M + 32 * TU - 1) / (32 * TU) * h->n_tile_rows;
    const dim3 grid((unsigned)(d.n_units < GRID_ROW ? d.n_units : GRID_ROW)), block(64 * FEW_WAVES);
    hipLaunchKernelGGL((k_quant_few<OUT, GELU, TU>), grid, block, 0, s, d, c.X, c.xscale, h->tiles, h->list,
                       h->row_tile0, h->scale, (const char*)c.bias, (char*)c.Y);
    return hipGetLastError();
}

template <int OUT, bool GELU> hipError_t launch_as(const lpv_quant* h, const QuantLinearCall& c, hipStream_t s)
{
    if (c.M <= 32)
        return launch_few<OUT, GELU, 1>(h, c, s);
    return launch_few<OUT, GELU, 2>(h, c, s);
}

template <int OUT> hipError_t launch_out(const lpv_quant* h, const QuantLinearCall& c, hipStream_t s)
{
    return c.gelu ? launch_as<OUT, true>(h, c, s) : launch_as<OUT, false>(h, c, s);
}

}  // namespace

hipError_t launch_quant_plan(const lpv_quant* h, const uint8_t* mask, QuantTotals* totals, hipStream_t s)
{
    hipLaunchKernelGGL(k_quant_bits, dim3((unsigned)h->n_pairs), dim3(64), 0, s, *h, mask);
    hipLaunchKernelGGL(k_quant_scan, dim3(1), dim3(1024), 0, s, *h, mask, totals);
    return hipGetLastError();
}

hipError_t launch_quant_fill(const lpv_quant* h, const int8_t* W, int64_t ldw, const float* scale,
                             const uint8_t* mask, hipStream_t s)
{
    hipLaunchKernelGGL(k_quant_fill, dim3((unsigned)h->n_pairs), dim3(256), 0, s, *h, W, ldw, scale, mask);
    return hipGetLastError();
}

hipError_t launch_quant_linear(const lpv_quant* h, const QuantLinearCall& c, hipStream_t s)
{
    if (c.M == 0)
        return hipSuccess;
    switch (c.dtype) {
    case LPV_F32: return launch_out<LPV_F32>(h, c, s);
    case LPV_F16: return launch_out<LPV_F16>(h, c, s);
    default: return launch_out<LPV_BF16>(h, c, s);
    }
}

}  // namespace lpv
