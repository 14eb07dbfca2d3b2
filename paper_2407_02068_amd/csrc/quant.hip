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
// under 2^-45; adding and subtracting 1.5 * 2^12 rounds it to a multiple of 2^-40 first, so
// that a quotient exactly between two codes stays there and goes to the even one.
#include <math.h>

#include "lpv_device.h"
#include "lpv_grid.h"
#include "lpv_internal.h"

namespace lpv {
namespace {

struct QuantDims {
    int64_t ldx, ldy, lds, ldq, M;
    int32_t D;
    double eps;
};

// Eight values of an element type, as doubles: 16-byte loads.
template <int DT> __device__ inline void load8(const char* p, double v[8])
{
    if constexpr (DT == 0) {
        const float4 a = *(const float4*)p, b = *(const float4*)(p + 16);
        const float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = f[j];
    } else {
        const uint4 a = *(const uint4*)p;
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = Elem<DT>::to_f32((uint16_t)(w[j / 2] >> (16 * (j & 1))));
    }
}

template <int DT> __device__ inline double load1(const char* p)
{
    if constexpr (DT == 0)
        return *(const float*)p;
    else
        return Elem<DT>::to_f32(*(const uint16_t*)p);
}

template <int DT> __device__ inline void store8(char* p, const double v[8])
{
    if constexpr (DT == 0) {
        *(float4*)p = float4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
        *(float4*)(p + 16) = float4{(float)v[4], (float)v[5], (float)v[6], (float)v[7]};
    } else {
        *(uint4*)p = uint4{pack2<DT>((float)v[0], (float)v[1]), pack2<DT>((float)v[2], (float)v[3]),
                           pack2<DT>((float)v[4], (float)v[5]), pack2<DT>((float)v[6], (float)v[7])};
    }
}

template <int DT> __device__ inline void store1(char* p, double v)
{
    if constexpr (DT == 0)
        *(float*)p = (float)v;
    else
        *(uint16_t*)p = Elem<DT>::from_f32((float)v);
}

// The row's sums (and its largest value) over its NT threads, the same in every thread:
// lanes by butterfly, then waves in order.
template <int NT> __device__ inline void row_reduce(double& a, double& b, double& top, double (*s)[3])
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        a += __shfl_xor(a, o, 64);
        b += __shfl_xor(b, o, 64);
        top = fmax(top, __shfl_xor(top, o, 64));
    }
    if constexpr (NT > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();  // (a reduction before this one has been read)
        if ((threadIdx.x & 63) == 0) {
            s[wave][0] = a;
            s[wave][1] = b;
            s[wave][2] = top;
        }
        __syncthreads();
        a = b = top = 0.0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) {
            a += s[w][0];
            b += s[w][1];
            top = fmax(top, s[w][2]);
        }
    }
}

// NT threads to a row (64: four rows to a workgroup), NC chunks of 8 elements to a thread,
// held in registers: the row is read once.  VEC: a chunk is 8 neighbours, by 16-byte
// loads; else (odd sizes, strides or addresses) the row's elements go to the threads
// one by one.
template <int DT, int KIND, int NT, int NC, bool VEC>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void k_quant_rows(
    const QuantDims d, const char* x, const char* y, const char* __restrict__ gamma,
    const char* __restrict__ beta, char* S, int8_t* __restrict__ q, float* __restrict__ scale)
{
    constexpr int ES = DT == 0 ? 4 : 2, E = 8 * NC;
    constexpr int RPW = NT == 64 ? 4 : 1;  // rows per workgroup
    __shared__ double s_red[NT / 64][3];
    const int tid = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * RPW +
                        (NT == 64 ? (int)(threadIdx.x >> 6) : 0);
    if (row >= d.M)
        return;  // (whole waves of a row each, or the whole workgroup)
    // element of this thread's i-th chunk, j-th place
    auto at = [&](int i, int j) { return VEC ? (tid + NT * i) * 8 + j : tid + NT * (8 * i + j); };
    const char* xr = x + row * d.ldx * ES;
    const char* yr = y ? y + row * d.ldy * ES : nullptr;
    char* sr = S ? S + row * d.lds * ES : nullptr;
    double v[E];
    double sum = 0.0, sq = 0.0, top = 0.0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        double* vi = v + 8 * i;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            vi[j] = 0.0;
        if constexpr (VEC) {
            const int c = at(i, 0);
            if (c < d.D) {
                load8<DT>(xr + (int64_t)c * ES, vi);
                if (y) {
                    double t[8];
                    load8<DT>(yr + (int64_t)c * ES, t);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        vi[j] += t[j];
                }
                if (S)
                    store8<DT>(sr + (int64_t)c * ES, vi);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = at(i, j);
                if (c < d.D) {
                    vi[j] = load1<DT>(xr + (int64_t)c * ES);
                    if (y)
                        vi[j] += load1<DT>(yr + (int64_t)c * ES);
                    if (S)
                        store1<DT>(sr + (int64_t)c * ES, vi[j]);
                }
            }
        }
    }
    double factor = 1.0;
    if constexpr (KIND == QUANT_LAYER) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            sum += v[i];
        row_reduce<NT>(sum, sq, top, s_red);
        const double mean = sum / d.D;
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (at(i / 8, i % 8) < d.D) {
                v[i] -= mean;
                sq += v[i] * v[i];
            }
        sum = 0.0;
        row_reduce<NT>(sum, sq, top, s_red);
        factor = 1.0 / sqrt(sq / d.D + d.eps);
    }
    if constexpr (KIND == QUANT_RMS) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            sq += v[i] * v[i];
    }
    double poison = 0.0;  // not zero where a value is not finite
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        double g[8], b[8];
        if constexpr (KIND != QUANT_PLAIN && VEC) {
            const int c = at(i, 0);
            if (c < d.D) {
                load8<DT>(gamma + (int64_t)c * ES, g);
                if constexpr (KIND == QUANT_LAYER)
                    load8<DT>(beta + (int64_t)c * ES, b);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = at(i, j);
            if (c < d.D) {
                if constexpr (KIND != QUANT_PLAIN && !VEC) {
                    g[j] = load1<DT>(gamma + (int64_t)c * ES);
                    if constexpr (KIND == QUANT_LAYER)
                        b[j] = load1<DT>(beta + (int64_t)c * ES);
                }
                double& u = v[8 * i + j];
                if constexpr (KIND == QUANT_RMS)
                    u *= g[j];
                if constexpr (KIND == QUANT_LAYER)
                    u = u * factor * g[j] + b[j];
                top = fmax(top, fabs(u));
                poison += u * 0.0;
            }
        }
    }
    row_reduce<NT>(sq, poison, top, s_red);
    if constexpr (KIND == QUANT_RMS) {
        factor = 1.0 / sqrt(sq / d.D + d.eps);
        poison += sq * 0.0;
    }
    // (the layer norm's factor is in u)
    const bool bad = !(poison == 0.0);
    double sc = KIND == QUANT_RMS ? top * factor / 127.0 : top / 127.0;
    if (top == 0.0)
        sc = 0.0;
    if (tid == 0)
        scale[row] = bad ? __builtin_nanf("") : (float)sc;
    const double inv = bad || top == 0.0 ? 0.0 : 127.0 / top;
    int8_t* qr = q + row * d.ldq;
    auto code = [&](double u) -> uint32_t {
        if (bad)
            u = 0.0;
        constexpr double FINE = 6144.0;              // 1.5 * 2^12
        constexpr double WHOLE = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits are the integer
        const double t = (fma(u, inv, FINE) - FINE) + WHOLE;
        return (uint32_t)__builtin_bit_cast(uint64_t, t) & 0xff;
    };
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        if constexpr (VEC) {
            const int c = at(i, 0);
            if (c < d.D) {
                uint32_t w[2] = {0, 0};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    w[j / 4] |= code(v[8 * i + j]) << (8 * (j & 3));
                *(uint2*)(qr + c) = uint2{w[0], w[1]};
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = at(i, j);
                if (c < d.D)
                    qr[c] = (int8_t)code(v[8 * i + j]);
            }
        }
    }
}

template <int DT, int KIND> hipError_t launch_kind(const QuantRowsCall& c, hipStream_t s)
{
    const QuantDims d = {c.ldx, c.ldy, c.lds, c.ldq, c.M, c.D, c.eps};
    // 16-byte pieces throughout: the row's length and every stride and address
    auto even = [](const void* p, int64_t ld, int unit) {
        return !p || ((uintptr_t)p % unit == 0 && ld % 8 == 0);
    };
    const bool vec = c.D % 8 == 0 && even(c.x, c.ldx, 16) && even(c.y, c.ldy, 16) &&
                     even(c.S, c.lds, 16) && even(c.q, c.ldq, 8) && even(c.gamma, 0, 16) &&
                     even(c.beta, 0, 16);
#define LPV_ROWS(NT_, NC_)                                                                          \
    do {                                                                                            \
        const Grid2 g = grid_of(NT_ == 64 ? (c.M + 3) / 4 : c.M);                                   \
        const dim3 grid(g.x, g.y), block(NT_ == 64 ? 256 : NT_);                                    \
        if (vec)                                                                                    \
            hipLaunchKernelGGL((k_quant_rows<DT, KIND, NT_, NC_, true>), grid, block, 0, s, d,      \
                               (const char*)c.x, (const char*)c.y, (const char*)c.gamma,            \
                               (const char*)c.beta, (char*)c.S, c.q, c.scale);                      \
        else                                                                                        \
            hipLaunchKernelGGL((k_quant_rows<DT, KIND, NT_, NC_, false>), grid, block, 0, s, d,     \
                               (const char*)c.x, (const char*)c.y, (const char*)c.gamma,            \
                               (const char*)c.beta, (char*)c.S, c.q, c.scale);                      \
        return hipGetLastError();                                                                   \
    } while (0)
    if (c.D <= 512)
        LPV_ROWS(64, 1);
    if (c.D <= 1024)
        LPV_ROWS(64, 2);
    if (c.D <= 2048)
        LPV_ROWS(256, 1);
    if (c.D <= 4096)
        LPV_ROWS(256, 2);
    if (c.D <= 8192)
        LPV_ROWS(256, 4);
    if (c.D <= 16384)
        LPV_ROWS(1024, 2);
    LPV_ROWS(1024, 4);
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
