// lpv_internal.h -- host-side internals of liblpv: the handle, the schedule
// constants and the kernel launchers (implemented in pack.hip / linear.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/lpv.h"

namespace lpv {

// Schedule tile: 32 output rows x 32 reduction columns, the operand shape of
// one pair of 32x32x16 matrix-core instructions.
constexpr int TILE = 32;
// Tile rows per group: a workgroup owns one token tile times one group.
constexpr int GROUP_TILES = 8;
// Tokens per workgroup.
constexpr int BM = 256;

// Widest and tallest weight, in tiles, of the X-stationary kernel.
constexpr int XS_COLS = 24;
constexpr int XS_ROWS = 128;

struct Plan {  // sizes learnt on the device during pack
    int32_t nnzb, n_steps, n_tiles, n_walk;
};

}  // namespace lpv

struct lpv_bsr {
    int64_t N, K;
    int32_t b_r, b_c, R, C;
    int64_t nnzb;
    int32_t dtype;  // lpv_dtype
    int32_t device;
    void* meta;  // one allocation: the index arrays and the schedule (sizes known before the
                 // kept count is)
    void* data[4];  // values, stream_vals, row_vals and col_idx, in as few allocations as pay
    // canonical BSR
    int32_t* row_ptr;  // R + 1
    int32_t* col_idx;  // nnzb
    void* values;      // nnzb * b_r * b_c elements
    // tile schedule (16-bit element types only)
    int32_t n_tile_rows, n_tile_cols, n_groups;
    int64_t n_steps, n_tiles;
    int4* gdesc;           // n_groups: {group, first walk entry, walk length, rotation} per launch slot
    int4* gdesc_host;      // host copy of gdesc (sizes the linear kernel's launches)
    int32_t* group_order;  // n_groups
    int32_t* step_ptr;     // n_groups + 1
    int32_t* group_tile0;  // n_groups + 1, first stream tile of each group
    // half group (4 tile rows) x tile column (an even count, n_tile_cols rounded
    // up): kept rows << 28 | first kept tile in the stream (fewer than 2^21)
    uint32_t* half_tiles;
    int32_t* step_col;     // n_steps
    int32_t* step_bits;    // n_steps
    int32_t* step_tile;    // n_steps
    int64_t n_walk;
    int2* walk;            // n_walk: the launch slots' walks, {col | bits << 16 | last << 24, tile}
    void* stream_vals;     // n_tiles * TILE * TILE elements, operand order
    // the same tiles by tile row, ascending columns (weights that fit XS_COLS x
    // XS_ROWS tiles, K a multiple of 64; NULL otherwise): row r's are row_tile0[r] .. row_tile0[r + 1],
    // bit c of row_mask[r] set for tile column c
    void* row_vals;
    int32_t* row_tile0;    // n_tile_rows + 1
    uint32_t* row_mask;    // n_tile_rows
    // workspace of lpv_bsr_grad_w (per-chunk float32 partial sums of every
    // tile), allocated on the first call and kept until destroy
    mutable void* gradw_ws;
    mutable size_t gradw_ws_bytes;
};

// The bucket index of a position bias (lpv_relpos_create).
struct lpv_relpos {
    int32_t T, nt;  // tokens, and tiles of 32 of them
    int32_t n_buckets, n_segs;
    int32_t device;
    void* mem;              // one allocation, the arrays below in it
    uint16_t *idx, *idx_t;  // the index and its transpose, 32 nt x 32 nt, 0xffff: no pair
    // the pairs by bucket (their places in a head's tiles), cut into segments of at most
    // RELPOS_SEG; a bucket without pairs has one empty segment
    int32_t* order;
    int32_t* seg_ptr;     // n_segs + 1
    int32_t* bucket_seg;  // n_buckets + 1
    // the tiles of rows (a bit each) with a row that gives some bucket two pairs or more
    uint64_t crowded;
};

// A weight in 8-bit codes (lpv_quant_pack).  Its 32 x 32 tiles of codes go in pairs of tile
// rows (64 outputs) and chunks of QUANT_CHUNK tile columns: pair by pair, chunk by chunk,
// column by column, the even row's tile first.
struct lpv_quant {
    int64_t N, K;
    int32_t b_r, b_c, R, C;  // (dense: blocks of 16 x 16, all kept)
    int64_t nnzb, n_tiles;
    int32_t device, n_cus;
    int32_t n_tile_rows, n_tile_cols;
    int32_t n_pairs;   // of tile rows, filled up to a multiple of 8 with empty ones
    int32_t n_chunks;
    void* mem;         // one allocation: the arrays whose sizes are known before the kept count is
    void* data;        // another: tiles, list and groups
    uint32_t* bits;      // n_pairs x n_chunks: kept columns of the even row | of the odd row << 16
    int32_t* tile0;      // n_pairs: the first tile of each pair
    int32_t* row_tile0;  // n_tile_rows + 1: the first entry of each tile row in list
    float* scale;        // 64 n_pairs: the outputs' scales, zero past N
    char* tiles;         // n_tiles x 1 KB: lane l's 16 codes of row l % 32, from column 16 (l / 32)
    int2* list;          // n_tiles: by tile row, {tile column, place among the tiles}
    // Groups of two halves, a half up to two columns of a pair's chunk, in order.  A half is 16
    // bits: 6 for each column (its place in the chunk, even row kept << 4, odd row << 5), the
    // chunk's last half << 12, the pair's << 13; a chunk has one at least, a pair an even number.
    // Then the group's first tile.  Pair p's groups follow each other from QUANT_GROUPS
    // n_chunks p on.
    uint2* groups;       // QUANT_GROUPS n_chunks n_pairs
};

namespace lpv {

struct PackArgs {
    const void* W;  // NULL: the transpose of a packed weight, given by the next two
    int64_t ldw, N, K;
    const char* t_values;    // that weight's BSR values (blocks b_c x b_r) ...
    const int32_t* t_block;  // ... and, C x R, each kept block's number among them
    int32_t es;  // element size in bytes
    int32_t b_r, b_c, R, C;
    int32_t lr, lc;  // log2 of b_r, b_c
    const uint8_t* mask;
    int32_t n_tile_rows, n_tile_cols, n_groups;
    int32_t* row_tile0;  // NULL: no row-major tiles
    uint32_t* row_mask;
};

// pack.hip
// The counts, and (16-bit types) the schedule: everything that fits the handle's first
// allocation.  The Plan follows gdesc[n_groups] in memory.
hipError_t launch_pack_plan(const PackArgs& a, const lpv_bsr* h, Plan* plan, hipStream_t s);
// The block values, column indices and tile copies, into the second one.
hipError_t launch_pack_fill(const PackArgs& a, const lpv_bsr* h, hipStream_t s);
hipError_t launch_unpack(const lpv_bsr* h, void* W_out, int64_t ldw, hipStream_t s);

// linear.hip
struct LinearCall {
    const void* X;
    int64_t ldx, M;
    const void* bias;
    void* Y;
    int64_t ldy;
    int gelu;
};
hipError_t launch_bsr_linear(const lpv_bsr* h, const LinearCall& c, hipStream_t s);
hipError_t launch_dense_linear(const void* W, int64_t ldw, int64_t N, int64_t K, int dtype,
                               const LinearCall& c, hipStream_t s);
// stationary.hip: the product of a handle with row_vals, and whether it is the
// faster one for M tokens
bool use_xs(const lpv_bsr* h, int64_t M, bool gelu, int n_cus);
hipError_t launch_xs_linear(const lpv_bsr* h, const LinearCall& c, int n_cus, hipStream_t s);

// mask.hip
struct MaskCall {
    const void* W;
    int64_t ldw;
    const void* G;  // NULL: sum-of-squares scores
    int64_t ldg, N, K;
    int dtype;
    int32_t b_r, b_c;
    int64_t n_keep;
    uint8_t* mask;
    double* scores;
};
hipError_t launch_mask_topk(const MaskCall& m, hipStream_t s);
// Ranks by (-score, index): perm[rank] = block and / or mask[block] = rank < n_keep.
hipError_t launch_rank(const double* scores, int64_t nb, int64_t n_keep, int32_t* perm,
                       uint8_t* mask, hipStream_t s);

// delta.hip
constexpr int DELTA_MAX_POINTS = 128;
constexpr int64_t DELTA_MAX_BLOCKS = (int64_t)1 << 17;
struct DeltaCall {
    const void* W;  // N x K, row stride ldw
    int64_t ldw, N, K;
    int dtype;
    int32_t b_r, b_c;
    const void* grad;  // N x K, row stride ldg
    int64_t ldg;
    const void* samples;  // n_samples x (N x K, row stride lds), sample stride `stride`
    int64_t lds, stride, n_samples;
    double kappa;
    int32_t n_points;
    int32_t keep[DELTA_MAX_POINTS];  // kept blocks at each point, non-increasing
    double* delta;                   // n_points, device
    void* ws;                        // caller workspace, or NULL: allocated per call
    size_t ws_bytes;
};
size_t delta_workspace_bytes(int64_t N, int64_t K, int32_t b_r, int32_t b_c, int64_t n_samples,
                             int32_t n_points);
hipError_t launch_delta_curve(const DeltaCall& c, hipStream_t s);

// backward.hip
struct GradWCall {
    const void* G;  // M x N, row stride ldg
    int64_t ldg;
    const void* X;  // M x K, row stride ldx
    int64_t ldx, M;
    void* dW;  // nnzb x b_r x b_c, BSR order
    float* ws; // at least grad_w_workspace_bytes(h) bytes
};
// Bytes of the weight-gradient workspace of a handle (any M).
size_t grad_w_workspace_bytes(const lpv_bsr* h);
// The transposed mask (C x R) of a handle and its kept blocks' numbers (R x C).
hipError_t launch_transpose_maps(const lpv_bsr* h, uint8_t* maskT, int32_t* block, hipStream_t s);
hipError_t launch_grad_w(const lpv_bsr* h, const GradWCall& c, hipStream_t s);
// Encoder block around the pruned layers (encoder.hip).
constexpr int LN_MAX_D = 2048;     // widest row of the layer norm
constexpr int ATT_HD = 64;         // head dimension of the attention kernel
constexpr int ATT_MAX_T = 512;     // longest sequence (K and V staged in LDS)
hipError_t launch_add_layernorm(const void* x, const void* y, int64_t M, int32_t D, int dtype,
                                const void* gamma, const void* beta, float eps, void* S, void* out,
                                hipStream_t s);
hipError_t launch_attention(const void* qkv, int64_t n_seq, int32_t T, int32_t H, int dtype,
                            void* out, hipStream_t s);
// relpos.hip
constexpr int32_t RELPOS_MAX_T = 2048, RELPOS_MAX_BUCKETS = 65535, RELPOS_SEG = 512;
struct RelposCall {
    const void* table;  // n_buckets x H
    const void* qkv;
    int64_t ldq, n_seq;
    int32_t H, hd;
    int dtype;
    const int32_t* region;  // n_region x T, or NULL
    int64_t n_region;
    void* out;  // the gradient reads it
    int64_t ldo;
    float* lse;
    const void* dout;  // gradient only, as are the next
    int64_t ldg;
    void* dqkv;
    int64_t lddq;
    void* dtable;
    void* ws;
};
// The pairs and segments of an index, its crowded tiles, the pairs of each bucket (count), and
// the place of the first entry outside [-1, n_buckets) (bad, -1 if there is none); host memory
// (last: n_buckets of scratch).
struct RelposSizes {
    int64_t bad, n_pairs;
    uint64_t crowded;
    int32_t n_segs;
};
RelposSizes relpos_sizes(const int32_t* index, int32_t T, int32_t n_buckets, int32_t* count, int32_t* last);
// The handle's arrays (host memory; count as relpos_sizes left it, overwritten).
void relpos_tables(const int32_t* index, int32_t T, int32_t n_buckets, int32_t nt, int32_t* count,
                   uint16_t* idx, uint16_t* idx_t, int32_t* order, int32_t* seg_ptr,
                   int32_t* bucket_seg);
size_t relpos_workspace_bytes(const lpv_relpos* h, int64_t n_seq, int32_t H, bool grad);
hipError_t launch_relpos_attention(const lpv_relpos* h, const RelposCall& c, hipStream_t s);
hipError_t launch_relpos_grad(const lpv_relpos* h, const RelposCall& c, hipStream_t s);
// distill.hip
constexpr int32_t DISTILL_MAX_K = 1024;
struct DistillCall {
    const void* logits;  // M x V, row stride ldz
    int64_t ldz, M, V;
    int dtype;
    const int32_t* ids;  // M x k, row stride ldt, as is teacher
    const float* teacher;
    int64_t ldt;
    int32_t k;
    double temperature;
    const float* dloss;  // M, or NULL: 1
    float* loss;         // M
    void* dlogits;       // M x Vd, row stride ldd, or NULL
    int64_t ldd, Vd;
    void* ws;
};
size_t distill_workspace_bytes(int64_t M, int64_t V, int32_t k, int dtype);
hipError_t launch_distill(const DistillCall& c, hipStream_t s);
// quant.hip
constexpr int32_t QUANT_MAX_D = 32768;  // the longest row (32 elements to each of 1024 threads)
constexpr int QUANT_PLAIN = 0, QUANT_RMS = 1, QUANT_LAYER = 2;
struct QuantRowsCall {
    int kind;
    const void* x;
    int64_t ldx;
    const void* y;  // or NULL
    int64_t ldy, M;
    int32_t D;
    int dtype;
    const void *gamma, *beta;
    double eps;
    void* S;  // or NULL
    int64_t lds;
    int8_t* q;
    int64_t ldq;
    float* scale;
};
hipError_t launch_quant_rows(const QuantRowsCall& c, hipStream_t s);
// quant_linear.hip
constexpr int QUANT_CHUNK = 8;   // tile columns of a chunk (256 columns)
constexpr int QUANT_GROUPS = 2;  // groups of a chunk, at most
struct QuantTotals {
    int32_t n_tiles, n_blocks;
};
// Kept columns, counts and their sums (everything in h->mem but the scales); then tiles, list,
// groups and scales.
hipError_t launch_quant_plan(const lpv_quant* h, const uint8_t* mask, QuantTotals* totals, hipStream_t s);
hipError_t launch_quant_fill(const lpv_quant* h, const int8_t* W, int64_t ldw, const float* scale,
                             const uint8_t* mask, hipStream_t s);
struct QuantLinearCall {
    const int8_t* X;
    int64_t ldx;
    const float* xscale;
    int64_t M;
    const void* bias;
    void* Y;
    int64_t ldy;
    int dtype;
    int gelu;
};
hipError_t launch_quant_linear(const lpv_quant* h, const QuantLinearCall& c, hipStream_t s);
hipError_t launch_bias_grad(const void* G, int64_t ldg, int64_t M, int64_t N, int dtype, void* db,
                            hipStream_t s);
// The same with the partial sums in a fixed device array of this many floats
// (4 MiB per device, held until the process ends): no allocation.
constexpr int64_t BIAS_NOALLOC_SCRATCH_FLOATS = (int64_t)1 << 20;
hipError_t launch_bias_grad_noalloc(const void* G, int64_t ldg, int64_t M, int64_t N, int dtype,
                                    void* db, hipStream_t s);

}  // namespace lpv
