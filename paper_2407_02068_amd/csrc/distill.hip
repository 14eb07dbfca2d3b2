// distill.hip -- the distillation loss from a teacher's top logits, with its gradient
// (gfx950).
//
// Per row, with the student's logits z, the teacher's logits t at the ids of its entries and
// the temperature tau:
//   p = softmax(z / tau) over all classes, q = softmax(t / tau) over the row's entries,
//   loss = tau^2 sum_j q_j (log q_j - log p[id_j]),   dz = dloss tau (p - q of each class).
// Entries without an id in [0, V) or with a logit of -inf are no entries; a row without any
// has loss 0 and gradient 0.  A class named twice has both shares.
//
// One pass over the data: a row is held in registers between its statistics and its
// gradient, so z is read once and dz written once (bound: HBM).  The teacher's part of a row
// is worked out while the row's own loads are in flight.  Rows too long for registers, or
// too few to fill the chip, are cut into chunks: one launch for each chunk's maximum and
// sum, a second that joins a row's and forms the gradient.
#include <float.h>
#include <math.h>

#include "lpv_device.h"
#include "lpv_grid.h"
#include "lpv_internal.h"

namespace lpv {
namespace {

constexpr float LN2 = 0.69314718055994530942f;

// Elements by type: a 16-byte chunk and its values.
template <int DT> struct Chunk {
    static constexpr int N = DT == LPV_F32 ? 4 : 8;
    static constexpr int ES = DT == LPV_F32 ? 4 : 2;
    __device__ static inline float get(const uint4& v, int i)
    {
        if constexpr (DT == LPV_F32)
            return __uint_as_float(((const uint32_t*)&v)[i]);
        else
            return Elem<DT>::to_f32((uint16_t)(((const uint32_t*)&v)[i >> 1] >> (16 * (i & 1))));
    }
    __device__ static inline uint4 pack(const float* f)
    {
        uint4 v;
        uint32_t* w = (uint32_t*)&v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == LPV_F32)
                w[i] = __float_as_uint(f[i]);
            else
                w[i] = pack2<DT>(f[2 * i], f[2 * i + 1]);
        }
        return v;
    }
    // element i of the row, and one element written
    __device__ static inline float load1(const char* row, int64_t i)
    {
        if constexpr (DT == LPV_F32)
            return ((const float*)row)[i];
        else
            return Elem<DT>::to_f32(((const uint16_t*)row)[i]);
    }
    __device__ static inline void store1(char* row, int64_t i, float f)
    {
        if constexpr (DT == LPV_F32)
            ((float*)row)[i] = f;
        else
            ((uint16_t*)row)[i] = Elem<DT>::from_f32(f);
    }
    // chunk c of a row of V elements; past the end -inf (no weight, no maximum)
    __device__ static inline uint4 load(const char* row, int c, int V)
    {
        const int i = c * N;
        if (i + N <= V)
            return *(const uint4*)(row + (int64_t)c * 16);
        float f[N];
#pragma unroll
        for (int j = 0; j < N; ++j)
            f[j] = i + j < V ? load1(row, i + j) : -INFINITY;
        return pack(f);
    }
    __device__ static inline void store(char* row, int c, int V, const float* f)
    {
        const int i = c * N;
        if (i + N <= V) {
            *(uint4*)(row + (int64_t)c * 16) = pack(f);
            return;
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (i + j < V)
                store1(row, i + j, f[j]);
    }
};

struct Ds {
    const char* z;
    int64_t ldz, M;  // row strides in elements
    int32_t V, k;
    const int32_t* ids;
    const float* t;
    int64_t ldt;
    float c, tau;        // log2(e) / tau
    const float* dloss;  // NULL: 1
    float* loss;
    char* dz;  // NULL: the loss alone
    int64_t ldd;
    int32_t Vd;  // dz's columns: those from V on are zero
};

__device__ inline float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
__device__ inline float wave_add(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v += __shfl_xor(v, o, 64);
    return v;
}

// Maximum or sum over the NT threads of a row (a wave's, or the workgroup's through red).
template <int NT, bool MAX> __device__ inline float row_reduce(float v, float* red)
{
    v = MAX ? wave_max(v) : wave_add(v);
    if constexpr (NT > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
            red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w)
            v = MAX ? fmaxf(v, red[w]) : v + red[w];
    }
    return v;
}

constexpr int MAX_K = DISTILL_MAX_K;

// The teacher's entries of a row, KPT to a thread.
template <int NT> struct Teacher {
    static constexpr int KPT = NT == 64 ? 1 : MAX_K / NT;
    static constexpr int NB = NT == 64 ? 4096 : 1 << 17;  // places of the table of ids seen
    int id[KPT];       // -1: none
    float q[KPT], lq[KPT], share[KPT];  // q, log2 q, the sum of q over the entries of that class
    float zi[KPT];     // z[id]
    bool some;
};

// LDS of a row: the table of ids, and the entries (read where an id came twice).
template <int NT> struct Shared {
    uint32_t seen[Teacher<NT>::NB / 32];
    int32_t id[NT == 64 ? 64 : MAX_K];
    float q[NT == 64 ? 64 : MAX_K];
};

template <int NT> __device__ inline void row_sync()
{
    if constexpr (NT > 64)
        __syncthreads();
    else
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (a wave's run in order)
}

// The entries' weights, and z at those with an id in [first, end).  tid: the thread's place
// in the row.
template <int DT, int NT>
__device__ inline void load_teacher(const Ds& a, int64_t row, int tid, Teacher<NT>& e, float* red,
                                    int first, int end)
{
    using C = Chunk<DT>;
    constexpr int KPT = Teacher<NT>::KPT;
    const char* z = a.z + row * a.ldz * C::ES;
    float tv[KPT], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int j = tid + i * NT;
        e.id[i] = -1;
        tv[i] = -INFINITY;
        e.zi[i] = 0.0f;
        if (j < a.k) {
            const int id = a.ids[row * a.ldt + j];
            const float t = a.t[row * a.ldt + j];
            if ((uint32_t)id < (uint32_t)a.V && t != -INFINITY) {
                e.id[i] = id;
                tv[i] = t;
                if (id >= first && id < end)
                    e.zi[i] = C::load1(z, id);
            }
        }
        // (an entry's NaN leaves it an entry, and is the loss's)
        top = fmaxf(top, e.id[i] < 0 ? -INFINITY : fmaxf(tv[i], -FLT_MAX));
    }
    top = row_reduce<NT, true>(top, red);
    e.some = top > -INFINITY;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        e.lq[i] = (tv[i] - top) * a.c;
        e.q[i] = e.id[i] < 0 ? 0.0f : __builtin_amdgcn_exp2f(e.lq[i]);
        sum += e.q[i];
    }
    sum = row_reduce<NT, false>(sum, red);
    const float inv = e.some ? 1.0f / sum : 0.0f, lsum = __log2f(sum);
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        e.q[i] *= inv;
        e.lq[i] -= lsum;
    }
}

// The share of each entry's class: its q, and where ids came twice (found by a table of the
// ids seen; above its size two classes may share a place, which only takes the longer way)
// the sum over the entries in order.
template <int NT>
__device__ inline void load_shares(const Ds& a, int tid, Teacher<NT>& e, Shared<NT>& sh)
{
    constexpr int KPT = Teacher<NT>::KPT;
    const int words = (min(a.V, Teacher<NT>::NB) + 31) / 32;
    for (int w = tid; w < words; w += NT)
        sh.seen[w] = 0;
    row_sync<NT>();
    bool again = false;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int j = tid + i * NT;
        e.share[i] = e.q[i];
        if (j < a.k) {
            sh.id[j] = e.id[i];
            sh.q[j] = e.q[i];
        }
        if (e.id[i] >= 0) {
            const uint32_t b = (uint32_t)e.id[i] % Teacher<NT>::NB;
            const uint32_t was = atomicOr(&sh.seen[b >> 5], 1u << (b & 31));
            again |= (was >> (b & 31)) & 1u;
        }
    }
    bool twice;
    if constexpr (NT > 64)
        twice = __syncthreads_or(again);
    else
        twice = __any(again);
    if (twice) {
        row_sync<NT>();
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            if (e.id[i] < 0)
                continue;
            float v = 0.0f;
            for (int j = 0; j < a.k; ++j)
                v += sh.id[j] == e.id[i] ? sh.q[j] : 0.0f;
            e.share[i] = v;
        }
    }
}

// sum_j q_j (log2 q_j - (z_j - m) / tau), so that the loss is tau^2 ln 2 times this plus
// log2 of the row's sum of exp((z - m) / tau).
template <int NT> __device__ inline float row_cross(const Ds& a, const Teacher<NT>& e, float m, float* red)
{
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < Teacher<NT>::KPT; ++i)
        if (e.q[i] != 0.0f)
            v += e.q[i] * (e.lq[i] - (e.zi[i] - m) * a.c);
    return row_reduce<NT, false>(v, red);
}

// The gradient at the classes of the row's entries with ids in [first, end), over what is
// there; and zero in the columns behind the classes.  w = dloss tau.
template <int DT, int NT>
__device__ inline void fix_entries(const Ds& a, const Teacher<NT>& e, char* dz, float m, float l, float w,
                                   int tid, int first, int end)
{
    if (end == a.V)
        for (int i = a.V + tid; i < a.Vd; i += NT)
            Chunk<DT>::store1(dz, i, 0.0f);
#pragma unroll
    for (int i = 0; i < Teacher<NT>::KPT; ++i)
        if (e.id[i] >= first && e.id[i] < end)
            Chunk<DT>::store1(dz, e.id[i],
                              w * (__builtin_amdgcn_exp2f((e.zi[i] - m) * a.c) / l - e.share[i]));
}

// Rows in registers: NT threads to a row (a wave's rows four to a workgroup), NC chunks of
// 16 bytes to a thread.  Bound: HBM where a row has many loads in flight (with the gradient, 2048
// rows of 21841 bf16 classes: 41 us, 4.4 TB/s), else a row's one round trip (the loss of 16384
// rows of 1000 fp16 classes: 11 us, 3.0 TB/s).
template <int DT, int NT, int NC>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void k_distill_row(Ds a)
{
    using C = Chunk<DT>;
    constexpr int RPW = NT == 64 ? 4 : 1;
    __shared__ Shared<NT> shared[RPW];
    __shared__ float red[NT / 64];
    const int sub = NT == 64 ? threadIdx.x >> 6 : 0, tid = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
    Shared<NT>& sh = shared[sub];
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * RPW + sub;
    if (row >= a.M)
        return;  // (a wave, or the whole workgroup)
    const char* z = a.z + row * a.ldz * C::ES;
    uint4 v[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = tid + i * NT;
        if (c * C::N < a.V)
            v[i] = C::load(z, c, a.V);
    }
    Teacher<NT> e;
    load_teacher<DT, NT>(a, row, tid, e, red, 0, a.V);
    if (a.dz)
        load_shares<NT>(a, tid, e, sh);
    const float g = a.dz && a.dloss ? a.dloss[row] : 1.0f;
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if ((tid + i * NT) * C::N < a.V)
#pragma unroll
            for (int j = 0; j < C::N; ++j)
                m = fmaxf(m, C::get(v[i], j));
    m = row_reduce<NT, true>(m, red);
    float l = 0.0f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if ((tid + i * NT) * C::N < a.V)
#pragma unroll
            for (int j = 0; j < C::N; ++j)
                l += __builtin_amdgcn_exp2f((C::get(v[i], j) - m) * a.c);
    l = row_reduce<NT, false>(l, red);
    const float cross = row_cross<NT>(a, e, m, red);
    if (tid == 0)
        a.loss[row] = e.some ? (cross + __log2f(l)) * LN2 * a.tau * a.tau : 0.0f;
    if (!a.dz)
        return;
    char* dz = a.dz + row * a.ldd * C::ES;
    const float w = g * a.tau, f = e.some ? w / l : 0.0f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = tid + i * NT;
        if (c * C::N < a.V) {
            float d[C::N];
#pragma unroll
            for (int j = 0; j < C::N; ++j)
                d[j] = e.some ? __builtin_amdgcn_exp2f((C::get(v[i], j) - m) * a.c) * f : 0.0f;
            C::store(dz, c, a.V, d);
        }
    }
    // the entries' classes again: their stores follow the row's
    __threadfence_block();
    if constexpr (NT > 64)
        __syncthreads();
    fix_entries<DT, NT>(a, e, dz, m, l, w, tid, 0, a.V);
}

// A chunk's maximum and sum: part[row][chunk] = (m, sum exp((z - m) / tau)).  The first
// chunk's workgroup also leaves what the teacher's entries add to the loss: the logits may be
// overwritten in the next launch.  The row's maximum is not known yet: row_cross is taken from
// the largest z of the entries, left beside it (NaN for a row without any, which a maximum never
// is: a NaN among the logits is the loss's), so that only differences of logits are formed and a
// common offset costs no accuracy.
// Bound: the two launches.  4 rows of 131072 fp32 classes: 4 us and 6 for the second.
template <int DT>
__global__ __launch_bounds__(256) void k_distill_part(Ds a, int32_t chunks, int32_t per,
                                                      float2* __restrict__ part, float2* __restrict__ cross)
{
    using C = Chunk<DT>;
    __shared__ float red[4];
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, row = id / chunks;
    const int chunk = (int)(id - row * chunks);
    if (row >= a.M)
        return;
    const char* z = a.z + row * a.ldz * C::ES;
    const int c0 = chunk * per, c1 = min((chunk + 1) * per, (a.V + C::N - 1) / C::N);
    float m = -INFINITY, l = 0.0f;
    for (int c = c0 + threadIdx.x; c < c1; c += 256) {
        const uint4 v = C::load(z, c, a.V);
        float n = m;
#pragma unroll
        for (int j = 0; j < C::N; ++j)
            n = fmaxf(n, C::get(v, j));
        const float ref = n == -INFINITY ? 0.0f : n;
        l *= __builtin_amdgcn_exp2f((m - ref) * a.c);
#pragma unroll
        for (int j = 0; j < C::N; ++j)
            l += __builtin_amdgcn_exp2f((C::get(v, j) - ref) * a.c);
        m = n;
    }
    const float mm = row_reduce<256, true>(m, red);
    l = m == -INFINITY ? 0.0f : l * __builtin_amdgcn_exp2f((m - mm) * a.c);
    l = row_reduce<256, false>(l, red);
    if (threadIdx.x == 0)
        part[id] = float2{mm, l};
    if (chunk == 0) {
        Teacher<256> e;
        load_teacher<DT, 256>(a, row, threadIdx.x, e, red, 0, a.V);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < Teacher<256>::KPT; ++i)
            top = e.q[i] > 0.0f ? fmaxf(top, e.zi[i]) : top;
        top = row_reduce<256, true>(top, red);
        const float ref = top == -INFINITY ? 0.0f : top;  // (no entries, or left out by the student)
        const float v = row_cross<256>(a, e, ref, red);
        if (threadIdx.x == 0)
            cross[row] = float2{v, e.some ? ref : NAN};
    }
}

// The loss of a row from its (m, sum) and cross.
__device__ inline float joined_loss(const Ds& a, float2 ml, float2 cross)
{
    return (cross.x + (ml.x - cross.y) * a.c + __log2f(ml.y)) * LN2 * a.tau * a.tau;
}

// (m, sum) of a row from its chunks'.
__device__ inline float2 join_parts(const Ds& a, const float2* part, int chunks, float* red)
{
    float m = -INFINITY, l = 0.0f;
    for (int i = threadIdx.x; i < chunks; i += 256)
        m = fmaxf(m, part[i].x);
    m = row_reduce<256, true>(m, red);
    for (int i = threadIdx.x; i < chunks; i += 256) {
        const float2 p = part[i];
        l += p.x == -INFINITY ? 0.0f : p.y * __builtin_amdgcn_exp2f((p.x - m) * a.c);
    }
    return float2{m, row_reduce<256, false>(l, red)};
}

// Joins a row's chunks: the first one's workgroup writes the loss, each its gradient.
template <int DT>
__global__ __launch_bounds__(256) void k_distill_join(Ds a, int32_t chunks, int32_t per,
                                                      const float2* __restrict__ part,
                                                      const float2* __restrict__ cross)
{
    using C = Chunk<DT>;
    __shared__ Shared<256> sh;
    __shared__ float red[4];
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, row = id / chunks;
    const int chunk = (int)(id - row * chunks);
    if (row >= a.M)
        return;
    const int c0 = chunk * per, c1 = min((chunk + 1) * per, (a.V + C::N - 1) / C::N);
    const int first = c0 * C::N, end = min(c1 * C::N, a.V);
    Teacher<256> e;
    load_teacher<DT, 256>(a, row, threadIdx.x, e, red, first, end);
    load_shares<256>(a, threadIdx.x, e, sh);
    const float2 ml = join_parts(a, part + row * chunks, chunks, red);
    const float m = ml.x, l = ml.y;
    if (chunk == 0 && threadIdx.x == 0)
        a.loss[row] = e.some ? joined_loss(a, ml, cross[row]) : 0.0f;
    const char* z = a.z + row * a.ldz * C::ES;
    char* dz = a.dz + row * a.ldd * C::ES;
    const float w = (a.dloss ? a.dloss[row] : 1.0f) * a.tau, f = e.some ? w / l : 0.0f;
    for (int c = c0 + threadIdx.x; c < c1; c += 256) {
        const uint4 v = C::load(z, c, a.V);
        float d[C::N];
#pragma unroll
        for (int j = 0; j < C::N; ++j)
            d[j] = e.some ? __builtin_amdgcn_exp2f((C::get(v, j) - m) * a.c) * f : 0.0f;
        C::store(dz, c, a.V, d);
    }
    __threadfence_block();
    __syncthreads();
    fix_entries<DT, 256>(a, e, dz, m, l, w, threadIdx.x, first, end);
}

// The same for the loss alone.
__global__ __launch_bounds__(256) void k_distill_loss(Ds a, int32_t chunks, const float2* __restrict__ part,
                                                      const float2* __restrict__ cross)
{
    __shared__ float red[4];
    const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (row >= a.M)
        return;
    const float2 ml = join_parts(a, part + row * chunks, chunks, red);
    const float2 x = cross[row];
    if (threadIdx.x == 0)
        a.loss[row] = x.y == x.y ? joined_loss(a, ml, x) : 0.0f;
}

// How a call is cut: threads to a row in registers (0: chunks), chunks a row, 16-byte
// chunks of data in each.
// A wave to a row where its registers hold it: 16384 rows of 1000 bf16 classes 10.7 us the
// loss, 19.2 with the gradient, a workgroup of 256 to a row 36 and 51; 2048 rows of 4000
// 9.0 and 11.1, 9.2 and 13.2.  Chunks past what registers hold (16 x 1024 threads), and for
// few rows of over half of that, where a row's own time is more than the second launch: 16
// rows of 131072 14.8 us with the gradient, as a workgroup each 22.9; 120 rows of 65000
// 19.3 and 17.7, 8 rows of 21841 14.9 and 12.7.
struct Cut {
    int nt, nc;  // rows in registers: threads and 16-byte chunks a thread
    int32_t chunks, per;
};

Cut cut_of(int64_t M, int64_t V, int32_t k, int dtype)
{
    const int64_t n = (V + (dtype == LPV_F32 ? 3 : 7)) / (dtype == LPV_F32 ? 4 : 8);
    if (n <= 64 * 8 && k <= 64)
        return {64, (int)((n + 63) / 64), 1, 0};
    if (n > 1024 * 16 || (M < 128 && n > 512 * 16)) {
        int64_t chunks = (1024 + M - 1) / M, most = (n + 511) / 512;
        chunks = chunks < 1 ? 1 : chunks > most ? most : chunks;
        const int64_t per = (n + chunks - 1) / chunks;
        return {0, 0, (int32_t)((n + per - 1) / per), (int32_t)per};
    }
    const int nt = n <= 256 * 16 ? 256 : n <= 512 * 16 ? 512 : 1024;
    return {nt, (int)((n + nt - 1) / nt), 1, 0};
}

template <int DT, int NT> hipError_t rows_as(const Ds& a, int nc, hipStream_t s)
{
    const Grid2 g = grid_of(NT == 64 ? (a.M + 3) / 4 : a.M);
    const dim3 grid(g.x, g.y), block(NT < 256 ? 256 : NT);
#define LPV_DS(NC_) hipLaunchKernelGGL((k_distill_row<DT, NT, NC_>), grid, block, 0, s, a)
    if constexpr (NT <= 256) {
        if (nc <= 1)
            LPV_DS(1);
        else if (nc <= 2)
            LPV_DS(2);
        else if (nc <= 4)
            LPV_DS(4);
        else if (nc <= 8)
            LPV_DS(8);
    }
    if constexpr (NT >= 256) {  // (512 and 1024 threads: rows of over 8 chunks to a thread)
        if (nc > 8 && nc <= 12)
            LPV_DS(12);
        else if (nc > 12)
            LPV_DS(16);
    }
#undef LPV_DS
    return hipGetLastError();
}

template <int DT> hipError_t distill_as(const Ds& a, void* ws, hipStream_t s)
{
    const Cut cut = cut_of(a.M, a.V, a.k, DT);
    switch (cut.nt) {
    case 64: return rows_as<DT, 64>(a, cut.nc, s);
    case 256: return rows_as<DT, 256>(a, cut.nc, s);
    case 512: return rows_as<DT, 512>(a, cut.nc, s);
    case 1024: return rows_as<DT, 1024>(a, cut.nc, s);
    default: break;
    }
    const Grid2 g = grid_of(a.M * cut.chunks);
    float2* part = (float2*)ws;
    float2* cross = part + a.M * cut.chunks;
    hipLaunchKernelGGL((k_distill_part<DT>), dim3(g.x, g.y), dim3(256), 0, s, a, cut.chunks, cut.per, part,
                       cross);
    if (a.dz) {
        hipLaunchKernelGGL((k_distill_join<DT>), dim3(g.x, g.y), dim3(256), 0, s, a, cut.chunks, cut.per,
                           part, cross);
    } else {
        const Grid2 j = grid_of(a.M);
        hipLaunchKernelGGL(k_distill_loss, dim3(j.x, j.y), dim3(256), 0, s, a, cut.chunks, part, cross);
    }
    return hipGetLastError();
}

}  // namespace

size_t distill_workspace_bytes(int64_t M, int64_t V, int32_t k, int dtype)
{
    if (M == 0)
        return 0;
    const Cut cut = cut_of(M, V, k, dtype);
    return cut.nt ? 0 : (size_t)M * (cut.chunks + 1) * sizeof(float2);
}

hipError_t launch_distill(const DistillCall& c, hipStream_t s)
{
    const Ds a = {(const char*)c.logits, c.ldz, c.M, (int32_t)c.V, c.k, c.ids, c.teacher, c.ldt,
                  (float)(1.4426950408889634074 / c.temperature), (float)c.temperature, c.dloss, c.loss,
                  (char*)c.dlogits, c.ldd, (int32_t)c.Vd};
    switch (c.dtype) {
    case LPV_BF16: return distill_as<LPV_BF16>(a, c.ws, s);
    case LPV_F16: return distill_as<LPV_F16>(a, c.ws, s);
    default: return distill_as<LPV_F32>(a, c.ws, s);
    }
}

}  // namespace lpv
