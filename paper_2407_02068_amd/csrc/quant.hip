// quant.hip -- rows in 8-bit codes with a scale for each row: as they are, or behind the
// residual's addition and a root-mean-square or layer norm (gfx950).
//
// A row's codes are q_j = rint(127 u_j / max|u|), ties to even, for u the row, or the
// row that the norm gives; its scale is max|u| / 127.  A root-mean-square norm's factor
// r = 1 / sqrt(mean s^2 + eps) divides out of the codes: u = s gamma, and r enters the
// scale alone.
//
// Arithmetic is float64: a code is a rounding of its own, and a value next to the border
// of two codes would else take one or the other by the order of a sum.  It costs nothing that
// shows: this card's float64 add, multiply and fma run at the rate of the (unpacked) float32
// ones, and the kernel waits for memory.  127 u / max|u| comes by a reciprocal, an error
// under 2^-44; in the sum with 6144.5 it is rounded to a multiple of 2^-40.  Where
// that is halfway between two codes, 127 u and that multiple of max|u| are compared as they
// are (settle): a float64 quotient that is past a border by 2^-50 takes its own code, and one that
// is on it the even one.  Elements themselves are never that near a border without being
// on it (24 bits each: 2^-33 at least); sums x + y and products with gamma are.  A layer
// norm's values have roundings of their own, and its quotients next to halfway go to the even code.
#include <math.h>

#include "lpv_device.h"
#include "lpv_internal.h"

namespace lpv {
namespace {

struct QuantDims {
    int64_t ldx, ldy, lds, ldq, M;
    int32_t D;
    double eps, per;  // 1 / D
};

// CH neighbours of a row as they lie in memory, and their values.
template <int DT, int CH> struct Raw {
    static constexpr int WORDS = DT == 0 ? CH : CH / 2;
    uint32_t w[WORDS];
    __device__ inline void load(const char* p)
    {
        if constexpr (WORDS == 2) {
            const uint2 v = *(const uint2*)p;
            w[0] = v.x;
            w[1] = v.y;
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; i += 4) {
                const uint4 v = *(const uint4*)(p + 4 * i);
                w[i] = v.x;
                w[i + 1] = v.y;
                w[i + 2] = v.z;
                w[i + 3] = v.w;
            }
        }
    }
    // element j alone, from its own address (element by element)
    __device__ inline void load1(int j, const char* p)
    {
        if constexpr (DT == 0)
            w[j] = *(const uint32_t*)p;
        else if (j & 1)
            w[j / 2] |= (uint32_t) * (const uint16_t*)p << 16;
        else
            w[j / 2] = *(const uint16_t*)p;
    }
    __device__ inline float at(int j) const
    {
        if constexpr (DT == 0)
            return __uint_as_float(w[j]);
        else
            return Elem<DT>::to_f32((uint16_t)(w[j / 2] >> (16 * (j & 1))));
    }
};

// CH values rounded to the element type, to CH neighbours.
template <int DT, int CH> __device__ inline void store_sum(char* p, const float v[CH])
{
    uint32_t w[Raw<DT, CH>::WORDS];
#pragma unroll
    for (int i = 0; i < Raw<DT, CH>::WORDS; ++i) {
        if constexpr (DT == 0)
            w[i] = __float_as_uint(v[i]);
        else
            w[i] = pack2<DT>(v[2 * i], v[2 * i + 1]);
    }
    if constexpr (Raw<DT, CH>::WORDS == 2) {
        *(uint2*)p = uint2{w[0], w[1]};
    } else {
#pragma unroll
        for (int i = 0; i < Raw<DT, CH>::WORDS; i += 4)
            *(uint4*)(p + 4 * i) = uint4{w[i], w[i + 1], w[i + 2], w[i + 3]};
    }
}

template <int DT> __device__ inline void store_sum1(char* p, float v)
{
    if constexpr (DT == 0)
        *(float*)p = v;
    else
        *(uint16_t*)p = Elem<DT>::from_f32(v);
}

// The same value of another lane of the row of 16: row_ror.
template <int N> __device__ inline double ror16(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)b, 0x120 + N, 0xf, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(b >> 32), 0x120 + N, 0xf, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// All-reduce over a wave in registers: rotations in rows of 16 lanes, then the rows change places
// (every lane adds the same pairs, in one order or the other: the same bits).
template <typename F> __device__ inline double wave_all(double v, F op)
{
    v = op(v, ror16<8>(v));
    v = op(v, ror16<4>(v));
    v = op(v, ror16<2>(v));
    v = op(v, ror16<1>(v));
#pragma unroll
    for (int half = 16; half <= 32; half *= 2) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t l = (uint32_t)b, h = (uint32_t)(b >> 32);
        const auto lo = half == 16 ? __builtin_amdgcn_permlane16_swap(l, l, false, false)
                                   : __builtin_amdgcn_permlane32_swap(l, l, false, false);
        const auto hi = half == 16 ? __builtin_amdgcn_permlane16_swap(h, h, false, false)
                                   : __builtin_amdgcn_permlane32_swap(h, h, false, false);
        v = op(__builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]),
               __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]));
    }
    return v;
}

struct Add {
    __device__ inline double operator()(double a, double b) const { return a + b; }
};
struct Max {
    __device__ inline double operator()(double a, double b) const { return fmax(a, b); }
};

// Over the NT threads of a row, the same in every thread: lanes, then waves in order.  `s` holds
// two reductions in turn, so that one barrier each is enough.
template <int NT, typename F> __device__ inline double row_all(double v, F op, double* s, int& turn)
{
    v = wave_all(v, op);
    if constexpr (NT > 64) {
        s += turn * (2 * (NT / 64));
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
            s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w)
            v = op(v, s[w]);
    }
    return v;
}

// Two sums at once.
template <int NT> __device__ inline void row_sums(double& a, double& b, double* s, int& turn)
{
    a = wave_all(a, Add());
    b = wave_all(b, Add());
    if constexpr (NT > 64) {
        constexpr int N = NT / 64;
        s += turn * (2 * N);
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
            s[threadIdx.x >> 6] = a;
            s[N + (threadIdx.x >> 6)] = b;
        }
        __syncthreads();
        a = s[0];
        b = s[N];
#pragma unroll
        for (int w = 1; w < N; ++w) {
            a += s[w];
            b += s[N + w];
        }
    }
}

// The value of a row's first thread, in every thread.
template <int NT> __device__ inline double first_of(double v, double* s, int& turn)
{
    if constexpr (NT > 64) {
        s += turn * (2 * (NT / 64));
        turn ^= 1;
        if (threadIdx.x == 0)
            s[0] = v;
        __syncthreads();
        return s[0];
    } else {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b);
        const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    }
}

// 1 / sqrt(x) and 1 / x to 2^-48 of them: the instructions' estimates (2^-22 at worst) and Newton's
// steps; an infinity or a NaN for x = 0, as long as nothing takes it.
__device__ inline double fast_rsqrt(double x)
{
    double r = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const double e = fma(-x * r, r, 1.0);
        r = fma(r * 0.5, e, r);
    }
    return r;
}
__device__ inline double fast_rcp(double x)
{
    double r = __builtin_amdgcn_rcp(x);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        r = fma(fma(-x, r, 1.0), r, r);
    return r;
}

// The code of u whose quotient 127 u / top is nearest to t, halfway between two codes: the sign of
// 127 u - t top decides.  The product's rounding error is exact in float64 (p and e), and so is
// 127 u - p, of two numbers that agree in 40 bits; the last difference has the right sign.
__device__ inline int settle(double u, double top, double t)
{
    const double p = t * top, e = fma(t, top, -p);
    const double d = fma(127.0, u, -p) - e;
    return (int)(d > 0.0 ? ceil(t) : d < 0.0 ? floor(t) : rint(t));
}

// NT threads to a row (64: four rows to a workgroup), NC chunks of CH elements to a thread, held
// in registers up to 8192 elements: the row is read once, the next one's loads going out before this
// one is worked on.  Bound by memory: 8192 x 4096 bf16 with its sum and a root-mean-square norm (two
// rows in, the sum and the codes out) 44 us, 5.3 TB/s, or 37, 6.4 TB/s, where the last-level cache
// still has the rows (60 before reductions in registers and the row ahead); 12608 x 768 fp16 with a
// layer norm 17.6 us, 3.9 TB/s (25.8), where a wave has a row of 12 elements a lane and the
// reductions' chain shows, bf16 as they are 8.5 us; 1777 x 5120 float32 10.4 us (14.8); one row of
// 4096 3.3 us, a launch.
// Past 8192 elements a row has 1024 threads, with 128 registers each.  They hold rows as they are (float32
// to 16384) and root-mean-square rows to 16384; the rest spills (bytes a lane, vectors / element by element):
// layer norms 184 to 252 up to 16384 and 384 to 956 / 892 to 1412 beyond, root-mean-square norms 36 to
// 352 / 336 to 576, float32 rows 120 / 128.  1024 x 32768 bf16 takes 39 us as a sum (6.0 TB/s with the
// cache's help), 90 behind a root-mean-square norm, 224 behind a layer norm.
// VEC: a chunk is CH neighbours; else (odd sizes, strides or addresses) the row's elements go
// to the threads one by one.
template <int DT, int KIND, int NT, int NC, int CH, bool VEC>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void k_quant_rows(
    const QuantDims d, const char* x, const char* y, const char* __restrict__ gamma,
    const char* __restrict__ beta, char* S, int8_t* __restrict__ q, float* __restrict__ scale)
{
    constexpr int ES = DT == 0 ? 4 : 2, E = NC * CH;
    constexpr int RPW = NT == 64 ? 4 : 1;  // rows per workgroup
    constexpr bool KEEP = E <= 16;         // gamma and beta stay in registers
    __shared__ double s_red[4 * (NT / 64)];
    int turn = 0;
    const int tid = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t step = (int64_t)gridDim.x * RPW;
    int64_t row = (int64_t)blockIdx.x * RPW + (NT == 64 ? (int)(threadIdx.x >> 6) : 0);
    // element of this thread's i-th chunk, j-th place
    auto at = [&](int i, int j) { return VEC ? (tid + NT * i) * CH + j : tid + NT * (CH * i + j); };
    typedef Raw<DT, CH> R;
    auto load = [&](R(&r)[NC], const char* p) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
#pragma unroll
            for (int k = 0; k < R::WORDS; ++k)
                r[i].w[k] = 0;
            if constexpr (VEC) {
                if (at(i, 0) < d.D)
                    r[i].load(p + at(i, 0) * ES);
            } else {
#pragma unroll
                for (int j = 0; j < CH; ++j)
                    if (at(i, j) < d.D)
                        r[i].load1(j, p + at(i, j) * ES);
            }
        }
    };
    R g[NC], b[NC], nx[NC], ny[NC];
    if (KEEP && KIND != QUANT_PLAIN)
        load(g, gamma);
    if (KEEP && KIND == QUANT_LAYER)
        load(b, beta);
    if (row < d.M) {
        load(nx, x + row * d.ldx * ES);
        if (y)
            load(ny, y + row * d.ldy * ES);
    }
    for (; row < d.M; row += step) {  // (the same rows for every thread of a workgroup, or of a wave)
        double v[E];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            float s[CH];
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const float a = nx[i].at(j);
                s[j] = a;
                v[CH * i + j] = a;
                if (y) {  // (float32 for S, as lpv_add_layernorm forms it; the codes take the sum itself)
                    s[j] += ny[i].at(j);
                    v[CH * i + j] += (double)ny[i].at(j);
                }
            }
            if (S) {
                char* sr = S + row * d.lds * ES;
                if constexpr (VEC) {
                    if (at(i, 0) < d.D)
                        store_sum<DT, CH>(sr + at(i, 0) * ES, s);
                } else {
#pragma unroll
                    for (int j = 0; j < CH; ++j)
                        if (at(i, j) < d.D)
                            store_sum1<DT>(sr + at(i, j) * ES, s[j]);
                }
            }
        }
        if (row + step < d.M) {
            load(nx, x + (row + step) * d.ldx * ES);
            if (y)
                load(ny, y + (row + step) * d.ldy * ES);
        }
        double sq = 0.0, factor = 1.0;
        if constexpr (KIND == QUANT_LAYER) {
            // Both sums in one go, of differences from the row's first element, which is no
            // further from the mean than sqrt(D) standard deviations: what the difference of
            // the two loses is at most 2^-52 D of the variance.
            const double v0 = first_of<NT>(v[0], s_red, turn);
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (at(i / CH, i % CH) < d.D) {
                    v[i] -= v0;
                    sum += v[i];
                    sq = fma(v[i], v[i], sq);
                }
            row_sums<NT>(sum, sq, s_red, turn);
            const double mean = sum * d.per;
            const double var = fmax(fma(-mean, mean, sq * d.per), 0.0) + d.eps;
            factor = var > 0.0 ? fast_rsqrt(var) : __builtin_inf();
#pragma unroll
            for (int i = 0; i < E; ++i)
                v[i] -= mean;
            if (!(sum == sum) || !(sq == sq))  // (a maximum passes over a NaN)
                factor = __builtin_nan("");
        }
        if constexpr (KIND == QUANT_RMS) {
#pragma unroll
            for (int i = 0; i < E; ++i)
                sq = fma(v[i], v[i], sq);
        }
        if (!KEEP && KIND != QUANT_PLAIN)
            load(g, gamma);
        if (!KEEP && KIND == QUANT_LAYER)
            load(b, beta);
        double top = 0.0, poison = 0.0;  // (poison: not zero where a value is not finite)
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (KIND == QUANT_RMS)
                v[i] *= (double)g[i / CH].at(i % CH);
            if constexpr (KIND == QUANT_LAYER)  // (past the row's end gamma and beta are zero)
                v[i] = fma(v[i] * factor, (double)g[i / CH].at(i % CH), (double)b[i / CH].at(i % CH));
            top = fmax(top, fabs(v[i]));
            poison = fma(v[i], 0.0, poison);
        }
        if constexpr (KIND == QUANT_RMS) {
            sq = row_all<NT>(sq, Add(), s_red, turn);
            factor = fast_rsqrt(fma(sq, d.per, d.eps));
            poison = fma(sq, 0.0, poison);
        }
        // a row that is not finite has no largest value: a NaN does not pass a maximum, an
        // infinity does
        if (!(poison == 0.0))
            top = __builtin_inf();
        top = row_all<NT>(top, Max(), s_red, turn);
        const bool bad = !(top < __builtin_inf());
        const double sc = (KIND == QUANT_RMS ? top * factor : top) * (1.0 / 127.0);
        if (tid == 0)
            scale[row] = bad ? __builtin_nanf("") : top == 0.0 ? 0.0f : (float)sc;
        const double inv = bad || top == 0.0 ? 0.0 : 127.0 * fast_rcp(top);
        int8_t* qr = q + row * d.ldq;
        // 24 * 2^8 + 1/2 + t, for the quotient t: its whole part's low byte is the code of t rounded half
        // up, and of its 40 bits of fraction none is set where t is halfway.
        constexpr double BIAS = 6144.5;
        auto quotient = [&](double u, double by, uint32_t& hi) {
            const uint64_t b = __builtin_bit_cast(uint64_t, fma(u, by, BIAS));
            hi = (uint32_t)(b >> 32);
            return (uint32_t)b | (hi & 0xff);  // zero: halfway
        };
        // The same to the even code at once: for a layer norm, which has nothing to settle (with the other
        // form 4% more time at 768 elements).
        auto even = [&](double u) {
            constexpr double WHOLE = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits are the integer
            return (uint32_t)__builtin_bit_cast(uint64_t, (fma(u, inv, 6144.0) - 6144.0) + WHOLE) & 0xff;
        };
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            uint32_t w[CH / 4] = {}, off = ~0u;
#pragma unroll
            for (int j = 0; j < CH; j += 4) {
                if constexpr (KIND == QUANT_LAYER) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        w[j / 4] |= even(v[CH * i + j + k]) << (8 * k);
                    continue;
                }
                uint32_t hi[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    off = min(off, quotient(v[CH * i + j + k], inv, hi[k]));
                // byte 1 of each
                w[j / 4] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(hi[3], hi[2], 0x0c0c0501),
                                                 __builtin_amdgcn_perm(hi[1], hi[0], 0x0c0c0501), 0x05040100);
            }
            if (KIND != QUANT_LAYER && __builtin_expect(off == 0, 0)) {
                double again = inv;  // (opaque, so that the quotients above need not be kept)
                asm volatile("" : "+v"(again));
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    uint32_t hi;
                    if (quotient(v[CH * i + j], again, hi) != 0)
                        continue;
                    if (KIND == QUANT_RMS || y) {
                        const int c = settle(v[CH * i + j], top, fma(v[CH * i + j], again, BIAS) - BIAS);
                        w[j / 4] = (w[j / 4] & ~(0xffu << (8 * (j & 3)))) | (uint32_t)(c & 0xff) << (8 * (j & 3));
                    } else {
                        w[j / 4] &= ~(1u << (8 * (j & 3)));  // (of the two codes the even one)
                    }
                }
            }
            if (bad)  // (the quotients of a NaN)
#pragma unroll
                for (int k = 0; k < CH / 4; ++k)
                    w[k] = 0;
            if constexpr (VEC) {
                if (at(i, 0) < d.D) {
                    if constexpr (CH == 4)
                        *(uint32_t*)(qr + at(i, 0)) = w[0];
                    else
                        *(uint2*)(qr + at(i, 0)) = uint2{w[0], w[1]};
                }
            } else {
#pragma unroll
                for (int j = 0; j < CH; ++j)
                    if (at(i, j) < d.D)
                        qr[at(i, j)] = (int8_t)(w[j / 4] >> (8 * (j & 3)));
            }
        }
    }
}

// Workgroups of 256 threads that fill the chip's 256 compute units eight times over: the
// rows past them follow, each behind its workgroup's last.
constexpr int QUANT_WGS = 2048;

template <int DT, int KIND> hipError_t launch_kind(const QuantRowsCall& c, hipStream_t s)
{
    const QuantDims d = {c.ldx, c.ldy, c.lds, c.ldq, c.M, c.D, c.eps, 1.0 / c.D};
    // a thread's neighbours by one load throughout: the row's length and every stride and address
    const int ch = c.D <= 1024 ? 4 : 8, unit = ch * (DT == 0 ? 4 : 2) < 16 ? 8 : 16;
    auto even = [&](const void* p, int64_t ld, int u) { return !p || ((uintptr_t)p % u == 0 && ld % ch == 0); };
    const bool vec = c.D % ch == 0 && even(c.x, c.ldx, unit) && even(c.y, c.ldy, unit) &&
                     even(c.S, c.lds, unit) && even(c.q, c.ldq, ch) && even(c.gamma, 0, unit) &&
                     even(c.beta, 0, unit);
#define LPV_ROWS(NT_, NC_, CH_)                                                                     \
    do {                                                                                            \
        const int64_t wgs = NT_ == 64 ? (c.M + 3) / 4 : c.M, most = NT_ == 1024 ? QUANT_WGS / 4 : QUANT_WGS; \
        const int64_t rounds = (wgs + most - 1) / most;  /* the same number of rows to each */      \
        const dim3 grid((unsigned)((wgs + rounds - 1) / rounds)), block(NT_ == 64 ? 256 : NT_);      \
        if (vec)                                                                                    \
            hipLaunchKernelGGL((k_quant_rows<DT, KIND, NT_, NC_, CH_, true>), grid, block, 0, s, d, \
                               (const char*)c.x, (const char*)c.y, (const char*)c.gamma,            \
                               (const char*)c.beta, (char*)c.S, c.q, c.scale);                      \
        else                                                                                        \
            hipLaunchKernelGGL((k_quant_rows<DT, KIND, NT_, NC_, CH_, false>), grid, block, 0, s, d, \
                               (const char*)c.x, (const char*)c.y, (const char*)c.gamma,            \
                               (const char*)c.beta, (char*)c.S, c.q, c.scale);                      \
        return hipGetLastError();                                                                   \
    } while (0)
    if (c.D <= 256)
        LPV_ROWS(64, 1, 4);
    if (c.D <= 512)
        LPV_ROWS(64, 2, 4);
    if (c.D <= 768)
        LPV_ROWS(64, 3, 4);
    if (c.D <= 1024)
        LPV_ROWS(64, 4, 4);
    if (c.D <= 2048)
        LPV_ROWS(256, 1, 8);
    if (c.D <= 4096)
        LPV_ROWS(256, 2, 8);
    if (c.D <= 8192)
        LPV_ROWS(256, 4, 8);
    if (c.D <= 16384)
        LPV_ROWS(1024, 2, 8);
    LPV_ROWS(1024, 4, 8);
#undef LPV_ROWS
}

template <int DT> hipError_t launch_type(const QuantRowsCall& c, hipStream_t s)
{
    switch (c.kind) {
    case QUANT_RMS: return launch_kind<DT, QUANT_RMS>(c, s);
    case QUANT_LAYER: return launch_kind<DT, QUANT_LAYER>(c, s);
    default: return launch_kind<DT, QUANT_PLAIN>(c, s);
    }
}

}  // namespace

hipError_t launch_quant_rows(const QuantRowsCall& c, hipStream_t s)
{
    if (c.M == 0)
        return hipSuccess;
    switch (c.dtype) {
    case LPV_F32: return launch_type<0>(c, s);
    case LPV_F16: return launch_type<1>(c, s);
    default: return launch_type<2>(c, s);
    }
}

}  // namespace lpv
