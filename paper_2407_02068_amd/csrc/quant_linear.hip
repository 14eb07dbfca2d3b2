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
#include "lpv_internal.h"
#include "lpv_lds.h"

namespace lpv {
namespace {

typedef int i32x16 __attribute__((ext_vector_type(16)));
// (one LDS area holds values of several types in turn: accesses that may alias)
typedef __attribute__((may_alias)) uint32_t u32a;
typedef __attribute__((may_alias)) uint64_t u64a;
typedef __attribute__((address_space(3))) u32a* lds_u32;
typedef __attribute__((address_space(3))) u64a* lds_u64;

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

// Halves (two columns) of a chunk's groups: one at least.
__device__ inline int halves_of(uint32_t bits)
{
    return max((__popc((bits | bits >> 16) & 0xffff) + 1) / 2, 1);
}

// One wave to a pair of tile rows: the kept columns of its chunks.
__global__ __launch_bounds__(64) void k_quant_bits(const lpv_quant h, const uint8_t* __restrict__ mask)
{
    const int pair = blockIdx.x, lane = threadIdx.x;
    for (int c = 0; c < h.n_chunks; ++c) {
        const int col = lane & 15;
        const bool kept = lane < 32 && col < QUANT_CHUNK &&
                          tile_kept(h, mask, 2 * pair + (lane >> 4), c * QUANT_CHUNK + col);
        const uint32_t bits = (uint32_t)__ballot(kept);
        if (lane == 0)
            h.bits[(int64_t)pair * h.n_chunks + c] = bits;
    }
}

// One workgroup: a thread to a pair (at most 1024), the sums over the pairs before it.
__global__ __launch_bounds__(1024) void k_quant_scan(const lpv_quant h, const uint8_t* __restrict__ mask,
                                                     QuantTotals* __restrict__ totals)
{
    __shared__ int s_tiles[1024], s_blocks;
    const int p = threadIdx.x;
    if (p == 0)
        s_blocks = 0;
    int even = 0, odd = 0;
    if (p < h.n_pairs)
        for (int c = 0; c < h.n_chunks; ++c) {
            const uint32_t b = h.bits[(int64_t)p * h.n_chunks + c];
            even += __popc(b & 0xffff);
            odd += __popc(b >> 16);
        }
    s_tiles[p] = even + odd;
    __syncthreads();
    for (int d = 1; d < 1024; d <<= 1) {  // inclusive sums
        const int t = p >= d ? s_tiles[p - d] : 0;
        __syncthreads();
        s_tiles[p] += t;
        __syncthreads();
    }
    if (p < h.n_pairs) {
        const int t0 = s_tiles[p] - even - odd;
        h.tile0[p] = t0;
        if (2 * p < h.n_tile_rows)
            h.row_tile0[2 * p] = t0;
        if (2 * p + 1 < h.n_tile_rows)
            h.row_tile0[2 * p + 1] = t0 + even;
        if (p == h.n_pairs - 1)
            h.row_tile0[h.n_tile_rows] = s_tiles[p];
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
        *totals = QuantTotals{s_tiles[1023], mask ? s_blocks : h.R * h.C};
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
    int tile = h.tile0[pair], half = 0;
    uint2* groups = h.groups + (int64_t)pair * QUANT_GROUPS * h.n_chunks;
    int at[2] = {0, 0};  // this pair's entries of either row in list
    if (2 * pair < h.n_tile_rows)
        at[0] = h.row_tile0[2 * pair];
    if (2 * pair + 1 < h.n_tile_rows)
        at[1] = h.row_tile0[2 * pair + 1];
    for (int c = 0; c < h.n_chunks; ++c) {
        const uint32_t b = __builtin_amdgcn_readfirstlane(bits[c]);
        const uint32_t e = b & 0xffff, o = b >> 16, any = e | o;
        if ((c & 3) == wave) {
            uint32_t left = any;
            int t = tile;
            for (int n = 0; n < halves_of(b); ++n) {
                uint32_t desc = 0;
                const int first = t;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (!left)
                        break;
                    const int col = __builtin_ctz(left);
                    left &= left - 1;
                    const uint32_t kept = (e >> col & 1) | (o >> col & 1) << 1;
                    desc |= (uint32_t)(col | kept << 4) << (6 * i);
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
                }
                // (16 bits of the group's word, so that no other wave's half is written)
                const int at_half = half + n;
                const bool end = n == halves_of(b) - 1;
                const bool pad = end && c == h.n_chunks - 1 && (at_half & 1) == 0;  // the pair's last half is empty
                if (lane == 0) {
                    uint16_t* w = (uint16_t*)(groups + at_half / 2);
                    w[at_half & 1] = (uint16_t)(desc | (end && !pad ? 1u << 12 : 0u) |
                                                (end && !pad && c == h.n_chunks - 1 ? 1u << 13 : 0u));
                    if ((at_half & 1) == 0)
                        groups[at_half / 2].y = (uint32_t)first;
                    if (pad)
                        w[1] = (uint16_t)(1u << 12 | 1u << 13);
                }
            }
        }
        tile += __popc(e) + __popc(o);
        at[0] += __popc(e);
        at[1] += __popc(o);
        half += halves_of(b);
    }
}

// ---------------------------------------------------------------- the epilogue's arithmetic

// GELU for float32 outputs, as gelu_erf with f of degree 11 (gelu_fit.fit(11)): positive
// outputs to 3e-7 relative, negative ones to 1e-7 (4e-6 relative at -5.5, where the
// rounding of the exponent itself shows), where gelu_erf's 3e-6 to 5e-6 would show in the
// outputs' own type.
__device__ inline float gelu_f32(float v)
{
    const float a = fabsf(v) * 0.70710678118654752f;
    float f = 1.137913372e-07f;
    f = fmaf(f, a, -2.993123871e-06f);
    f = fmaf(f, a, 3.500672756e-05f);
    f = fmaf(f, a, -2.377048368e-04f);
    f = fmaf(f, a, 1.005247817e-03f);
    f = fmaf(f, a, -2.407329390e-03f);
    f = fmaf(f, a, 8.043324488e-05f);
    f = fmaf(f, a, 2.782279439e-02f);
    f = fmaf(f, a, -1.483810395e-01f);
    f = fmaf(f, a, -9.184218049e-01f);
    f = fmaf(f, a, -1.627909422e+00f);
    f = fmaf(f, a, 3.518289304e-08f - 0.5f);
    const float e = __builtin_amdgcn_exp2f(f);  // erfc(a) / sqrt 2
    const float r = fmaxf(v, 0.0f);
    return a >= 4.0f ? r : fmaf(-a, e, r);
}

// A token's scale above 2^96: its product with a sum (below 2^31) may pass the largest float32 where
// the output does not (a row that holds a type's lowest value, say).  2^-32 of the scale and 2^32 times
// the outputs' scales give the same bits without that.  (An output's scale above 2^95 stays: there a
// sum that is not 0 is infinite either way, and a sum of 0 stays 0.)
__device__ inline bool is_far(float xs) { return fabsf(xs) > 0x1p96f && fabsf(xs) < __builtin_inff(); }
__device__ inline float lift(float ws) { return fabsf(ws) <= 0x1p95f ? ws * 0x1p32f : ws; }

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

// Four neighbouring outputs, to memory.
template <int OUT> __device__ inline void store4(char* y, const float o[4])
{
    if constexpr (OUT == LPV_F32)
        *(float4*)y = float4{o[0], o[1], o[2], o[3]};
    else
        *(uint2*)y = uint2{pack2<OUT>(o[0], o[1]), pack2<OUT>(o[2], o[3])};
}

// ---------------------------------------------------------------- few tokens

struct QuantDims {
    int64_t ldx, M, K, N, ldy;
    int32_t n_tile_rows;
};

// 32 tokens times one tile row to a workgroup, whose WV waves share the row's kept tiles, every
// WV-th of the list, U at a time and the next U already asked for; the partial sums meet in
// LDS.  Both operands come straight from memory in operand order, so any size will do.
// Bound by the round trips: list, tiles, sums.  One token through 4096 x 4096 5.7 us, 2.9 TB/s of
// the weight (a copy's rate would be 3.2 us); 197 tokens, 768 -> 2304 at 50%: 4.6 us.  Eight tiles
// at a time or 16 waves were no faster.
template <int OUT, bool GELU, int WV, int U>
__global__ __launch_bounds__(64 * WV) void k_quant_few(
    const QuantDims a, const int8_t* __restrict__ X, const float* __restrict__ xscale,
    const char* __restrict__ tiles, const int2* __restrict__ list, const int32_t* __restrict__ row_tile0,
    const float* __restrict__ wscale, const char* __restrict__ bias, char* __restrict__ Y)
{
    constexpr int ES = OUT == LPV_F32 ? 4 : 2;
    __shared__ v4i s_part[WV][4][64];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = (int)(blockIdx.x % (unsigned)a.n_tile_rows);
    const int64_t m0 = (int64_t)(blockIdx.x / (unsigned)a.n_tile_rows) * 32;
    const int8_t* xr = X + min(m0 + (lane & 31), a.M - 1) * a.ldx;
    i32x16 acc = {};
    const int t0 = row_tile0[row], n = row_tile0[row + 1] - t0;
    // this wave's tiles: places wave, wave + WV, ... of the row's
    const int mine = n > wave ? (n - wave + WV - 1) / WV : 0;
    for (int base = 0; base < mine; base += 64) {
        const int2 e = list[t0 + wave + WV * min(base + lane, mine - 1)];
        const int here = min(mine - base, 64);
        v4i w[2][U], x[2][U];
        auto load = [&](int i0, v4i(&wv)[U], v4i(&xv)[U]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int p = min(i0 + i, here - 1);  // (past the last: it again, and no product)
                const int col = __builtin_amdgcn_readlane(e.x, p), t = __builtin_amdgcn_readlane(e.y, p);
                wv[i] = *(const v4i*)(tiles + (int64_t)t * 1024 + lane * 16);
                // (a half past K is zero in the tile: any codes do, the row's first)
                int k = col * TILE + 16 * h;
                k = k < a.K ? k : 0;
                xv[i] = *(const v4i*)(xr + k);
            }
        };
        auto mul = [&](int i0, v4i(&wv)[U], v4i(&xv)[U]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (i0 + i < here)
                    acc = mma8(wv[i], xv[i], acc);
        };
        load(0, w[0], x[0]);
        for (int i0 = 0; i0 < here; i0 += 2 * U) {
            if (i0 + U < here)
                load(i0 + U, w[1], x[1]);
            mul(i0, w[0], x[0]);
            if (i0 + U < here) {
                if (i0 + 2 * U < here)
                    load(i0 + 2 * U, w[0], x[0]);
                mul(i0 + U, w[1], x[1]);
            }
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
        s_part[wave][q][lane] = v4i{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    if (tid < 256) {
        const int q = tid >> 6;
        int s[4] = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WV; ++w) {
            const v4i v = s_part[w][q][lane];
#pragma unroll
            for (int b = 0; b < 4; ++b)
                s[b] += v[b];
        }
        const int64_t m = m0 + (lane & 31), at = (int64_t)row * TILE + 8 * q + 4 * h;
        if (m < a.M && at < a.N) {
            float o[4], xs = xscale[m];
            float4 ws = *(const float4*)(wscale + at);
            if (__builtin_expect(is_far(xs), 0)) {
                xs *= 0x1p-32f;
                ws = float4{lift(ws.x), lift(ws.y), lift(ws.z), lift(ws.w)};
            }
            finish4<OUT, GELU>(s, xs, ws, bias4<OUT>(bias, at), o);
            store4<OUT>(Y + (m * a.ldy + at) * ES, o);
        }
    }
}

template <int OUT, bool GELU, int WV, int U>
hipError_t launch_few(const lpv_quant* h, const QuantLinearCall& c, hipStream_t s)
{
    const QuantDims d = {c.ldx, c.M, h->K, h->N, c.ldy, h->n_tile_rows};
    const dim3 grid((unsigned)((c.M + 31) / 32 * h->n_tile_rows)), block(64 * WV);
    hipLaunchKernelGGL((k_quant_few<OUT, GELU, WV, U>), grid, block, 0, s, d, c.X, c.xscale, h->tiles, h->list,
                       h->row_tile0, h->scale, (const char*)c.bias, (char*)c.Y);
    return hipGetLastError();
}

// ---------------------------------------------------------------- many tokens

// A workgroup of WV waves takes items of 32 TU tokens times WV pairs of tile rows (64 WV outputs), a
// pair to a wave.  X goes by DMA into LDS a chunk (256 columns) at a time, NS chunks in
// turn; the pair's tiles come straight from memory into registers, since no other wave needs
// them, four columns ahead.  A wave's work is a list of kept columns, made at pack time: for
// each it reads the tokens' codes from LDS, for one tile or both, and has TU products for
// each.  So dropped tiles cost nothing, a column of X is read from LDS once for two tiles, and
// waves meet at one barrier a chunk.
//
// LDS: panels of 128 columns, a row (token) of 128 bytes, its 16-byte piece c at
// c ^ xswz(row): the 16 rows that are read at once lie in distinct banks.
//
// What bounds it.  Dense and large, the matrix cores: 16384 x 4096 -> 8192 453 to 465 us, 2.36 to 2.43
// POP/s, a library's 8192^3 int8 product 2.49 (525 to 566 us in the tens of launches after a rest, while
// the clock settles, as the library's is slower there).  Pruned, no one thing:
// 50432 x 768 -> 2304 at 50% takes 78 us (a copy of its bytes 52), 74 if the waves did not wait for each
// other at a chunk's end, 71 without the chunks' DMA (the tiles' loads come back behind it), 66
// without the outputs' stores; 8192 x 4096 -> 4096 in blocks of 64 at 80% 48 us (22), 41 without the
// waves' waiting (a chunk has 0.8 kept blocks a pair, on average, and the wave with the most is waited
// for), 44 without the DMA, 35 without both.  Behind GELU its 16 instructions for every
// 64 outputs: 12608 x 384 -> 1536 at 75% 19 us (8.4), of its cycles 30% that, and 14% before the first
// product; a workgroup has two or three items, 2.3 on average.  With one wave a SIMD (777 x 1296 ->
// 5136 float32 with GELU, 16 us) a group of four columns takes 1580 cycles, 512 of them products;
// without loads, waits, LDS reads and products together its control still takes 1100, and DMA,
// waits or products alone can be left out at no more than 4% gain.  Chunks of 512 columns, tiles
// eight columns ahead, X two columns ahead and over a chunk's end, places for all of a column's
// tiles (fewer instructions for their addresses), three workgroups a compute unit and wave
// priorities were measured and are within 5%, one way here and the other there; X of all K resident
// in LDS takes 5 us from the first of these and adds to the others.
//
// The waits count: vector memory comes back in order, so that a DMA is there once no more are
// out than are known to be younger (the compiler's own waits know nothing of the DMA and wait for
// more than they need).
struct PanelDims {
    int64_t ldx, M, K, N, ldy;
    int32_t n_chunks, n_pairs;
    int32_t n_mt, n_pb;  // token tiles, blocks of WV pairs
    int32_t n_items;
    uint32_t per_inv, last_inv;  // 2^32 / d rounded up for the divisors of item(): PN_MG n_pb and n_mt % PN_MG
};
constexpr int PN_MG = 8;             // token tiles that share an XCD's L2 with several blocks of pairs
constexpr int PN_STAGE = 4096;       // bytes of a wave's staging area

// Global -> LDS DMA of 4 bytes per lane to 256 bytes at a wave-uniform LDS address.
__device__ inline void dma4(const char* base, uint32_t off, uint32_t lds)
{
    asm volatile(
        "s_nop 0\n"
        "global_load_lds_dword %0, %1"
        :
        : "v"(off), "s"(base), "{m0}"(lds)
        : "memory");
}

// The lane number made opaque: what only a rare part needs is not kept in registers through the
// loop.
__device__ inline int fresh(int l)
{
    asm volatile("" : "+v"(l));
    return l;
}

// What the outputs of a pair need, into the wave's staging area: the outputs' scales (256 bytes),
// their bias (256) and the tokens' scales.
template <int OUT, int TU>
__device__ inline void params_dma(const PanelDims& a, uint32_t stage, int lane, int64_t m0, int64_t n0,
                                  const char* xscale, const char* wscale, const char* bias)
{
    constexpr int ES = OUT == LPV_F32 ? 4 : 2;
    const int ln = fresh(lane);
    dma4(wscale + n0 * 4, (uint32_t)ln * 4, stage);
    if (bias) {
        const int n = (int)n0 + (OUT == LPV_F32 ? ln : 2 * (ln & 31));
        dma4(bias, (uint32_t)((n < a.N ? n : 0) * ES), stage + 256);
    } else {
        *(lds_u32)(uintptr_t)(stage + 256 + ln * 4) = 0;
    }
    const int last = (int)min((int64_t)32 * TU - 1, a.M - 1 - m0);
#pragma unroll
    for (int i = 0; i < (TU + 1) / 2; ++i)
        dma4(xscale + m0 * 4, (uint32_t)min(64 * i + ln, last) * 4, stage + 512 + i * 256);
}

// Four neighbours of the bias in the staging area, from the pair's output n on.
template <int OUT> __device__ inline float4 stage_bias4(uint32_t stage, int n)
{
    if constexpr (OUT == LPV_F32) {
        return __builtin_bit_cast(float4, lds_read16<256>(stage + n * 4));
    } else {
        using E = Elem<OUT>;
        const uint64_t v = *(lds_u64)(uintptr_t)(stage + 256 + n * 2);
        return float4{E::to_f32((uint16_t)v), E::to_f32((uint16_t)(v >> 16)),
                      E::to_f32((uint16_t)(v >> 32)), E::to_f32((uint16_t)(v >> 48))};
    }
}

// The outputs as panel_outputs gives them, for a wave with a far token: each lane stores its own.
template <int OUT, bool GELU, int TU>
__device__ inline void far_outputs(const PanelDims& a, i32x16 (&acc)[2][TU], const float (&xs)[TU], uint32_t stage,
                                   int lane, int64_t m0, int64_t n0, char* Y)
{
    constexpr int ES = OUT == LPV_F32 ? 4 : 2;
    const int fr = lane & 31, h = lane >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = 32 * j + 8 * q + 4 * h;
            const float4 ws = __builtin_bit_cast(float4, lds_read16<0>(stage + n * 4));
            const float4 b = stage_bias4<OUT>(stage, n);
#pragma unroll
            for (int u = 0; u < TU; ++u) {
                const int s[4] = {acc[j][u][4 * q], acc[j][u][4 * q + 1], acc[j][u][4 * q + 2], acc[j][u][4 * q + 3]};
                const bool far = is_far(xs[u]);
                const float4 wl = {far ? lift(ws.x) : ws.x, far ? lift(ws.y) : ws.y, far ? lift(ws.z) : ws.z,
                                   far ? lift(ws.w) : ws.w};
                float o[4];
                finish4<OUT, GELU>(s, far ? xs[u] * 0x1p-32f : xs[u], wl, b, o);
                const int64_t m = m0 + 32 * u + fr;
                if (m < a.M && n0 + n < a.N)
                    store4<OUT>(Y + (m * a.ldy + n0 + n) * ES, o);
            }
        }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int u = 0; u < TU; ++u)
            acc[j][u] = i32x16{};
}

// The outputs of 32 TU tokens (from m0) and a pair's 64 outputs (from n0); the sums are left at 0.
template <int OUT, bool GELU, int TU>
__device__ inline void panel_outputs(const PanelDims& a, i32x16 (&acc)[2][TU], uint32_t stage, int lane,
                                     int64_t m0, int64_t n0, char* Y)
{
    constexpr int ES = OUT == LPV_F32 ? 4 : 2;
    const int ln = fresh(lane), fr = ln & 31, h = ln >> 5;
    float xs[TU];
#pragma unroll
    for (int u = 0; u < TU; ++u)
        xs[u] = __uint_as_float(*(lds_u32)(uintptr_t)(stage + 512 + (32 * u + fr) * 4));
    bool any_far = false;
#pragma unroll
    for (int u = 0; u < TU; ++u)
        any_far |= is_far(xs[u]);
    if (__builtin_expect(__any(any_far), 0)) {
        far_outputs<OUT, GELU, TU>(a, acc, xs, stage, ln, m0, n0, Y);
        return;
    }
    uint2 pk[TU][2][4];    // 16-bit outputs: four to a place
    float4 pf[OUT == LPV_F32 ? TU : 1][2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = 32 * j + 8 * q + 4 * h;
            const float4 ws = __builtin_bit_cast(float4, lds_read16<0>(stage + n * 4));
            const float4 b = stage_bias4<OUT>(stage, n);
#pragma unroll
            for (int u = 0; u < TU; ++u) {
                const int s[4] = {acc[j][u][4 * q], acc[j][u][4 * q + 1], acc[j][u][4 * q + 2], acc[j][u][4 * q + 3]};
                float o[4];
                finish4<OUT, GELU>(s, xs[u], ws, b, o);
                if constexpr (OUT == LPV_F32)
                    pf[u][j][q] = float4{o[0], o[1], o[2], o[3]};
                else
                    pk[u][j][q] = uint2{pack2<OUT>(o[0], o[1]), pack2<OUT>(o[2], o[3])};
            }
        }
    // 32 tokens of 128 bytes at a time through the staging area (16-byte piece c of token t at
    // c ^ xswz(t)), so that whole lines leave; streamed past the caches, which X and the
    // tiles want
    const int lt = ln >> 3, lp = ln & 7;
    const bool inside = m0 + 32 * TU <= a.M && n0 + 64 <= a.N;
    typedef __attribute__((address_space(1))) char* global_w;
    // (32 bits: eight rows of a stride of at most 2^22)
    const uint32_t y_off = ((uint32_t)lt * (uint32_t)a.ldy + (uint32_t)lp * (16 / ES)) * ES;
#pragma unroll
    for (int u = 0; u < TU; ++u) {
#pragma unroll
        for (int half = 0; half < ES / 2; ++half) {
            const uint32_t at = stage + fr * 128;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (ES == 4 && j != half)
                    continue;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (OUT == LPV_F32)
                        lds_write16(at + (((2 * q + h) ^ xswz(fr)) << 4), __builtin_bit_cast(v4i, pf[u][j][q]));
                    else
                        *(lds_u64)(uintptr_t)(at + (((4 * j + q) ^ xswz(fr)) << 4) + 8 * h) =
                            __builtin_bit_cast(uint64_t, pk[u][j][q]);
                }
            }
            v4i v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 8 * i + lt;
                v[i] = lds_read16<0>(stage + t * 128 + ((lp ^ xswz(t)) << 4));
            }
            global_w y = (global_w)Y + ((m0 + 32 * u) * a.ldy + n0 + 32 * half) * ES;
            typedef __attribute__((address_space(1))) v4i* out4;
            if (inside) {
#pragma unroll
                for (int i = 0; i < 4; ++i, y += 8 * a.ldy * ES) {
                    asm volatile("" : "+s"(y));  // (the wave's address: the lane's offset stays 32 bits)
                    __builtin_nontemporal_store(v[i], (out4)(y + y_off));
                }
            } else {
                const int rows = (int)min((int64_t)32, a.M - (m0 + 32 * u));
                if (n0 + 32 * half + lp * (16 / ES) < a.N)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (8 * i + lt < rows)
                            __builtin_nontemporal_store(v[i], (out4)(y + 8 * i * a.ldy * ES + y_off));
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int u = 0; u < TU; ++u)
            acc[j][u] = i32x16{};
}

// The four columns of a group: place in the chunk, and which of the pair's tiles are kept.
__device__ inline uint32_t col_of(uint32_t desc, int i) { return desc >> (16 * (i / 2) + 6 * (i & 1)) & 15; }
__device__ inline uint32_t kept_of(uint32_t desc, int i) { return desc >> (16 * (i / 2) + 6 * (i & 1) + 4) & 3; }
// A half's end of the chunk (i = 1 or 3), and the group's of the pair.
__device__ inline bool chunk_end(uint32_t desc, int i) { return desc >> (i == 1 ? 12 : 28) & 1; }
__device__ inline bool pair_end(uint32_t desc) { return desc >> 29 & 1; }

template <int OUT, bool GELU, int TU, int WV, int NS>
__global__ __launch_bounds__(64 * WV, TU == 1 ? 3 : 2) void k_quant_panel(
    const PanelDims a, const char* X, const char* xscale, const char* tiles, const uint2* groups,
    const char* wscale, const char* bias, char* Y)
{
    constexpr int PANEL = TU * 4096, SLOT = 2 * PANEL;  // bytes
    constexpr int IPW = TU * 8 / WV;                    // DMA instructions of a wave and chunk
    __shared__ uint4 smem[(NS * SLOT + WV * PN_STAGE) / 16];
    static_assert(IPW * WV == TU * 8 && QUANT_CHUNK == 8, "a chunk is two panels, shared out evenly");
    // (an address that the compiler knows nothing about: loads from it stay on their side of the
    // DMA and of the waits, which count them)
    typedef const __attribute__((address_space(1))) char* global;
    global wt = (global)tiles;
    asm volatile("" : "+s"(wt));

    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t lds = lds_addr(smem), stage = lds + NS * SLOT + (uint32_t)wave * PN_STAGE;
    const uint32_t loff = (uint32_t)lane * 16;

    // Items in order: groups of PN_MG token tiles, in each the blocks of pairs, in each its token
    // tiles; XCD x (workgroups x, x + 8, ...) has a contiguous eighth of them, which its
    // workgroups take in turn.
    const int xcd = (int)(blockIdx.x & 7), C = (int)(gridDim.x >> 3);
    const int seg = (int)((int64_t)a.n_items * xcd / 8) + (int)(blockIdx.x >> 3);
    const int seg_end = (int)((int64_t)a.n_items * (xcd + 1) / 8);
    const int my_items = seg < seg_end ? (seg_end - seg + C - 1) / C : 0;
    if (my_items == 0)
        return;
    auto item = [&](int k, int& mt, int& pb) {
        // (below 2^30: the estimate of a quotient is right or one too many)
        const int i = seg + min(k, my_items - 1) * C, per = PN_MG * a.n_pb;
        int g = (int)__umulhi((uint32_t)i, a.per_inv), rest = i - g * per;
        if (rest < 0) {
            --g;
            rest += per;
        }
        const int mg = min(PN_MG, a.n_mt - g * PN_MG);
        pb = mg == PN_MG ? rest / PN_MG : mg == 1 ? rest : (int)__umulhi((uint32_t)rest, a.last_inv);
        mt = g * PN_MG + rest - pb * mg;
    };
    const int per_pair = QUANT_GROUPS * a.n_chunks;  // groups of a pair, at most
    auto lanes_of = [&](int pb, int from) {  // groups from .. from + 63 of this wave's pair
        const uint2* g = groups + (int64_t)(pb * WV + wave) * per_pair;
        return g[(uint32_t)min(from + fresh(lane), per_pair - 1)];
    };

    // ---- the DMA of a chunk: half of the waves to a panel, 8 IPW rows to a wave
    int d_k = 0, d_c = 0, d_slot = 0;  // its item, chunk and slot
    const char* d_base = nullptr;
    uint32_t d_row[IPW];
    const int d_panel = wave / (WV / 2), d_first = wave % (WV / 2) * (8 * IPW);
    auto set_x = [&]() {
        int mt, pb;
        item(d_k, mt, pb);
        const int64_t m0 = (int64_t)mt * (32 * TU);
        d_base = X + m0 * a.ldx;
        const int last = (int)min((int64_t)32 * TU - 1, a.M - 1 - m0);  // rows past M repeat the last
        const int ln = fresh(lane);
#pragma unroll
        for (int i = 0; i < IPW; ++i)
            d_row[i] = (uint32_t)min(d_first + 8 * i + (ln >> 3), last) * (uint32_t)a.ldx;
    };
    auto dma = [&]() {
        if (d_k >= my_items)
            return;
        const int ln = fresh(lane);
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const int row = d_first + 8 * i + (ln >> 3);
            const int k = (2 * d_c + d_panel) * 128 + ((ln & 7) ^ xswz(row)) * 16;
            // (past K the tiles are zero: any codes do, the row's first)
            dma16(d_base, d_row[i] + (uint32_t)(k < a.K ? k : 0),
                  smem + (d_slot * SLOT + d_panel * PANEL + d_first * 128 + i * 1024) / 16);
        }
        d_slot = d_slot + 1 == NS ? 0 : d_slot + 1;
        if (++d_c == a.n_chunks) {
            d_c = 0;
            if (++d_k < my_items)
                set_x();
        }
    };
    auto params = [&](int mt, int pb) {
        params_dma<OUT, TU>(a, stage, lane, (int64_t)mt * (32 * TU), (int64_t)(pb * WV + wave) * 64, xscale, wscale, bias);
    };

    set_x();
    dma();
    int mt, pb, mt1, pb1, mt2, pb2;  // this item, the next and the one after it
    item(0, mt, pb);
    item(1, mt1, pb1);
    params(mt, pb);
    uint2 dl = lanes_of(pb, 0);       // this item's groups, 64 at a time
    uint2 nd = lanes_of(pb1, 0), n2;  // the next item's, and the one's after it
    asm volatile("" : "+v"(dl.x), "+v"(dl.y), "+v"(nd.x), "+v"(nd.y));
    int gi = 0, from = 0;  // the group being worked on: lane gi of dl, whose first is `from`
    uint32_t cur = __builtin_amdgcn_readlane(dl.x, 0);

    // The tiles of four columns: of a column with one tile, that one twice.  (At most 2^22 tiles:
    // byte offsets fit 32 bits.)
    v4i w[4][2];
    typedef const __attribute__((address_space(1))) v4i* global4;
    auto load_w = [&](int i, uint32_t desc, uint32_t& at) __attribute__((always_inline)) {
        const uint32_t ab = kept_of(desc, i);
        w[i][0] = *(global4)(wt + (at + loff));
        at += ab == 3 ? 1024 : 0;
        w[i][1] = *(global4)(wt + (at + loff));
        at += ab ? 1024 : 0;
    };
    {
        uint32_t at = (uint32_t)__builtin_amdgcn_readlane(dl.y, 0) * 1024;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            load_w(i, cur, at);
    }
    // The codes of the tokens at a column of the chunk: lane l has row l % 32 (+ 32 u), pieces 2 c and
    // 2 c + 1 of the panel by l / 32.
    const int fr = lane & 31;
    const uint32_t xbase = lds + fr * 128, xpiece = (uint32_t)(h ^ xswz(fr)) << 4;
    v4i x[2][TU];
    auto read_x = [&](v4i(&o)[TU], uint32_t desc, int i, uint32_t slot) __attribute__((always_inline)) {
        const uint32_t c = col_of(desc, i);
        const uint32_t at = xbase + (xpiece ^ (c & 3) << 5) + (slot + (c >> 2) * PANEL);
#pragma unroll
        for (int u = 0; u < TU; ++u)
            o[u] = lds_read16<0>(at + u * 4096);
    };
    i32x16 acc[2][TU];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int u = 0; u < TU; ++u)
            acc[j][u] = i32x16{};

    uint32_t slot = 0;
    // The end of a chunk: the next one has landed (for every wave, behind the barrier), and every
    // wave has read this one, whose place the DMA takes.  What is younger than the next one's
    // DMA: 4 loads of tiles at least in each of the NS - 1 chunks since (fewer before there were
    // that many); what is younger than an item's scales and bias at its end: 8.
    // (At least: a count that is too low waits for more than it needs.  So any other load or store
    // in between, a spilled register's among them, leaves the waits right.)
    int chunks = 0;
    auto sync = [&](bool at_end) __attribute__((always_inline)) {
        constexpr int AHEAD = 4 * (NS - 1);
        if (NS > 2 && chunks >= NS - 1) {
            if (at_end)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n s_barrier" ::"i"(AHEAD < 8 ? AHEAD : 8) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n s_barrier" ::"i"(AHEAD) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)\n s_barrier" ::: "memory");
        }
        ++chunks;
    };
    asm volatile("s_waitcnt vmcnt(8)\n s_barrier" ::: "memory");  // (the tiles' loads are younger)
#pragma unroll
    for (int i = 1; i < NS; ++i)
        dma();
    for (int k = 0; k < my_items; ++k) {
        item(k + 2, mt2, pb2);
        n2 = lanes_of(pb2, 0);
        read_x(x[0], cur, 0, slot);
        bool done;
        do {  // the pair's groups
            uint32_t next, first;
            done = pair_end(cur);
            if (done) {
                next = __builtin_amdgcn_readlane(nd.x, 0);
                first = __builtin_amdgcn_readlane(nd.y, 0);
            } else {
                if (__builtin_expect(++gi == 64, 0)) {
                    gi = 0;
                    from += 64;
                    dl = lanes_of(pb, from);
                    asm volatile("" : "+v"(dl.x), "+v"(dl.y));
                }
                next = __builtin_amdgcn_readlane(dl.x, gi);
                first = __builtin_amdgcn_readlane(dl.y, gi);
            }
            uint32_t at = first * 1024;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool end = (i & 1) && chunk_end(cur, i);
                if (!end)
                    read_x(x[(i + 1) & 1], i < 3 ? cur : next, (i + 1) & 3, slot);
                if (kept_of(cur, i) & 1)
#pragma unroll
                    for (int u = 0; u < TU; ++u)
                        acc[0][u] = mma8(w[i][0], x[i & 1][u], acc[0][u]);
                if (kept_of(cur, i) & 2)
#pragma unroll
                    for (int u = 0; u < TU; ++u)
                        acc[1][u] = mma8(w[i][1], x[i & 1][u], acc[1][u]);
                load_w(i, next, at);
                if (end) {
                    sync(i == 3);
                    dma();
                    slot = slot + SLOT == NS * SLOT ? 0 : slot + SLOT;
                    if (i == 1)
                        read_x(x[0], cur, 2, slot);
                    else if (!done)
                        read_x(x[0], next, 0, slot);
                }
            }
            cur = next;
        } while (!done);
        asm volatile("" : "+v"(n2.x), "+v"(n2.y));
        panel_outputs<OUT, GELU, TU>(a, acc, stage, lane, (int64_t)mt * (32 * TU), (int64_t)(pb * WV + wave) * 64, Y);
        if (k + 1 < my_items)
            params(mt1, pb1);
        mt = mt1;
        pb = pb1;
        mt1 = mt2;
        pb1 = pb2;
        dl = nd;
        nd = n2;
        gi = from = 0;
    }
    // (nothing of this workgroup is in flight when it ends)
    __builtin_amdgcn_s_waitcnt(0);
}

template <int OUT, bool GELU, int TU, int WV, int NS>
hipError_t launch_panel(const lpv_quant* h, const QuantLinearCall& c, int n_cus, int per_cu, hipStream_t s)
{
    PanelDims d = {c.ldx, c.M, h->K, h->N, c.ldy, h->n_chunks, h->n_pairs};
    // token tiles of one launch: items in 31 bits
    d.n_pb = ((h->n_tile_rows + 1) / 2 + WV - 1) / WV;
    const int64_t most = ((int64_t)1 << 30) / d.n_pb;
    const int wgs = max(n_cus & ~7, 8) * per_cu;
    for (int64_t m = 0, n_mt = (c.M + 32 * TU - 1) / (32 * TU); n_mt > 0; m += most, n_mt -= most) {
        d.n_mt = (int32_t)(n_mt < most ? n_mt : most);
        d.n_items = d.n_mt * d.n_pb;
        auto inverse = [](int32_t n) { return (uint32_t)((((uint64_t)1 << 32) + n - 1) / n); };
        d.per_inv = inverse(PN_MG * d.n_pb);
        d.last_inv = d.n_mt % PN_MG > 1 ? inverse(d.n_mt % PN_MG) : 0;
        const int64_t m0 = m * (32 * TU);
        d.M = c.M - m0;
        const int need = (int)(((int64_t)d.n_items + 7) / 8 * 8);
        const dim3 grid((unsigned)(need < wgs ? need : wgs)), block(64 * WV);
        hipLaunchKernelGGL((k_quant_panel<OUT, GELU, TU, WV, NS>), grid, block, 0, s, d, (const char*)c.X + m0 * c.ldx,
                           (const char*)(c.xscale + m0), (const char*)h->tiles, (const uint2*)h->groups,
                           (const char*)h->scale, (const char*)c.bias,
                           (char*)c.Y + m0 * c.ldy * (OUT == LPV_F32 ? 4 : 2));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

// The kernel by the work there is, GPU us on 256 compute units (at up to 8192 outputs; wider ones follow
// the same rule untimed).
// - k_quant_few up to 1400 units of 32 tokens and a tile row (1380 units of 640 x 832 6.8, items of 32
//   tokens 7.0; 1600 of 656 x 688 9.5 / 7.5; 6400 of 5504 x 128 14.6 / 9.0), with 4 waves to a unit, or
//   8 where a tile row keeps more than 48 tiles (12: 4.7 / 5.5, 57: 4.7 / 4.6, 128: 7.0 / 6.1).
// - Items of 128 tokens x 8 pairs with four chunks on their way for a long reduction, if every
//   compute unit gets one (16384 x 4096 x 8192: 467, four pairs 480, 64 tokens 560), from 4096
//   columns on if half of them do (5832 x 7376 x 1424: 79 / 90 / 95).
// - Two workgroups of 128 tokens x 4 pairs to a compute unit, one's outputs beside the other's
//   products, if there are three items for each compute unit (50432 x 768 -> 2304 at 50%: 80, 8 pairs
//   84, 64 tokens 96; 594 items 20.8, 64 tokens 19.8).  Float32 outputs, which take twice the
//   registers there, go 64 tokens at a time (5506 x 640 -> 6848: 41 / 37).
// - 64 tokens if every compute unit gets an item (9933 x 528 x 528: 9.9, 32 tokens 11.7), else 32
//   (2353 x 2112 -> 896: 10.1 / 10.5).
template <int OUT, bool GELU> hipError_t launch_as(const lpv_quant* h, const QuantLinearCall& c, hipStream_t s)
{
    const int cus = h->n_cus;
    const int64_t pairs = (h->n_tile_rows + 1) / 2;
    auto items = [&](int tokens, int wv) { return (c.M + tokens - 1) / tokens * ((pairs + wv - 1) / wv); };
    if ((c.M + 31) / 32 * h->n_tile_rows <= 1400) {
        if (h->n_tiles <= 48 * (int64_t)h->n_tile_rows)
            return launch_few<OUT, GELU, 4, 4>(h, c, s);
        return launch_few<OUT, GELU, 8, 4>(h, c, s);
    }
    if (h->K >= 2048 && items(128, 8) >= (h->K >= 4096 ? cus / 2 : cus))
        return launch_panel<OUT, GELU, 4, 8, 4>(h, c, cus, 1, s);
    if constexpr (OUT != LPV_F32) {
        if (items(128, 4) >= 3 * cus)
            return launch_panel<OUT, GELU, 4, 4, 2>(h, c, cus, 2, s);
    }
    if (items(64, 4) >= cus)
        return launch_panel<OUT, GELU, 2, 4, 4>(h, c, cus, 2, s);
    return launch_panel<OUT, GELU, 1, 4, 4>(h, c, cus, 3, s);
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
