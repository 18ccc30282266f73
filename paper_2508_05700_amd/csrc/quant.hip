// Row-quantised tables (paper Section 4.1.2: the hosted tables are stored as
// INT4 after post-training quantisation): the pooled lookup that dequantises
// while it gathers.  (The quantisers are in quant_rows.hip.)
//
// Storage of one row of D elements, b = 8 or 4 bits per code:
//   bytes 0..3 scale (fp32), bytes 4..7 bias (fp32), then the codes (INT8: one
//   byte per element; INT4: element 2k in the low nibble of byte k, 2k+1 in the
//   high nibble), zero-padded to a multiple of 16 bytes (EMB_INT4_ROW64: of 64
//   bytes, otherwise the row of EMB_INT4).  Element value = scale * code + bias.
// MXFP4: D/2 bytes of codes (nibbles in the same order, each a 4-bit float), then
// one scale byte per 32 elements, zero-padded to a multiple of 16 bytes.  Codes
// come first so that the 16 bytes of a block are aligned: the matrix units take
// them as they are (product.hip).
//
// The kernel gives a lane 16 consecutive elements of a row, i.e. 8 (INT4, MXFP4)
// or 16 (INT8) code bytes, so a row of D elements takes LPR = D/16 lanes rounded up
// to a power of two; D must be a multiple of 16 (MXFP4: 32) and at most 1024.
#include "emb_internal.h"
#include "gather_quant.h"
#include "u64mod.h"

namespace {

// ---------------------------------------------------------------------------
// pooled lookup with dequantisation (the loop is in gather_quant.h)
// ---------------------------------------------------------------------------
// Rows come straight from the table in device memory.
struct QuantTableSource {
    const char *weights;
    uint64_t num_rows;
    int64_t row_bytes;
    uint32_t *status;
    __device__ __forceinline__ uint64_t resolve(int64_t r, int64_t) const
    {
        if ((uint64_t)r >= num_rows) {
            emb_flag(status, EMB_STATUS_BAD_INDEX);
            return 0ull;
        }
        return reinterpret_cast<uint64_t>(weights + r * row_bytes);
    }
};

// The entries are raw IDs: hashed by the lane that fetched them (Section 2.2), as in the lookup over
// fp32 / bf16 rows; the row numbers can be written out.
struct HashedQuantTableSource {
    const char *weights;
    uint64_t num_rows, salt, magic;
    int64_t row_bytes;
    int64_t *rows_out;   // nullable
    __device__ __forceinline__ uint64_t resolve(int64_t raw, int64_t j) const
    {
        const uint64_t r = emb_fast_mod(emb_splitmix64((uint64_t)raw ^ salt), num_rows, magic);
        if (rows_out) rows_out[j] = (int64_t)r;
        return reinterpret_cast<uint64_t>(weights + (int64_t)r * row_bytes);
    }
};

// MAKE_OFFSETS: as in bag_forward_kernel (forward.hip).
template <int LPR, int FMT, int UNROLL, bool HASHED, bool MAKE_OFFSETS>
__global__ __launch_bounds__(Q_BLOCK) void bag_forward_quant_kernel(const emb_table *__restrict__ tables, int32_t T,
                                                                    int64_t B, uint32_t blocks_per_table, int64_t nnz,
                                                                    const int64_t *__restrict__ rows,
                                                                    const int64_t *__restrict__ offsets, int32_t D,
                                                                    int64_t row_bytes, int32_t mode,
                                                                    float *__restrict__ out, uint32_t *status,
                                                                    int64_t *__restrict__ rows_out,
                                                                    int64_t *__restrict__ offsets_out,
                                                                    const int32_t *__restrict__ lengths)
{
    constexpr int GROUPS = Q_BLOCK / LPR;
    __shared__ int64_t tile_prefix[MAKE_OFFSETS ? Q_BLOCK + 1 : 1];
    __shared__ int64_t wave_sums[2 * Q_BLOCK / EMB_WAVE];
    const uint32_t lb = emb_xcd_block(blockIdx.x, gridDim.x);
    const uint32_t t_raw = lb / blocks_per_table;
    const bool tail = t_raw >= (uint32_t)T;          // the grid is rounded up to whole dies
    const int t = tail ? T - 1 : (int)t_raw;
    const int l = threadIdx.x % LPR;
    const int64_t b0 = tail ? B : (int64_t)(lb % blocks_per_table) * GROUPS;
    const int64_t b = b0 + threadIdx.x / LPR;
    const emb_table tb = tables[t];
    const int64_t bag = (int64_t)t * B + b;
    const bool live = b < B;
    int64_t s = 0, e = 0;
    if (MAKE_OFFSETS) {
        if (lengths) {   // uniform
            const int64_t left = B - b0;
            emb_bounds_from_lengths<Q_BLOCK, GROUPS>(lengths, (int64_t)t * B + b0, left < GROUPS ? (int)left : GROUPS,
                                                     threadIdx.x / LPR, tile_prefix, wave_sums, status, s, e);
        } else {
            emb_two_level_bounds<Q_BLOCK>(offsets, (int64_t)T * B, live, bag, tile_prefix, wave_sums, s, e);
        }
        if (live && l == 0) {
            offsets_out[bag + 1] = e;
            if (bag == 0) offsets_out[0] = 0;
        }
    } else if (live) {
        s = offsets[bag];
        e = offsets[bag + 1];
    }
    if (HASHED) {
        HashedQuantTableSource src{reinterpret_cast<const char *>(tb.weights), (uint64_t)tb.num_rows, tb.salt,
                                   tb.mod_magic, row_bytes, rows_out};
        gather_dequant_pool_range<LPR, FMT, UNROLL>(src, live, bag, s, e, l, nnz, rows, D, mode, out, status);
    } else {
        QuantTableSource src{reinterpret_cast<const char *>(tb.weights), (uint64_t)tb.num_rows, row_bytes, status};
        gather_dequant_pool_range<LPR, FMT, UNROLL>(src, live, bag, s, e, l, nnz, rows, D, mode, out, status);
    }
}

template <int LPR, int FMT>
int launch_quant_forward(hipStream_t s, const emb_table *tables, int32_t T, int64_t B, int64_t nnz, const int64_t *rows,
                         const int64_t *offsets, int32_t D, int64_t row_bytes, int32_t mode, float *out,
                         uint32_t *status, bool hashed, int64_t *rows_out, int64_t *offsets_out, const int32_t *lengths)
{
    constexpr int GROUPS = Q_BLOCK / LPR;
    constexpr int UNROLL = 8;
    const int64_t per_table = (B + GROUPS - 1) / GROUPS;
    const int64_t blocks = emb_round_up_xcds(per_table * T);
    if (blocks > (int64_t)0x7FFFFFFF) return EMB_ERR_UNSUPPORTED;
#define EMB_QK(HASHED, MAKE)                                                                                         \
    hipLaunchKernelGGL((bag_forward_quant_kernel<LPR, FMT, UNROLL, HASHED, MAKE>), dim3((unsigned)blocks), dim3(Q_BLOCK), \
                       0, s, tables, T, B, (uint32_t)per_table, nnz, rows, offsets, D, row_bytes, mode, out, status, \
                       rows_out, offsets_out, lengths)
    if (hashed) {
        if (offsets_out) EMB_QK(true, true); else EMB_QK(true, false);
    } else {
        if (offsets_out) EMB_QK(false, true); else EMB_QK(false, false);
    }
#undef EMB_QK
    EMB_RETURN_IF_LAUNCH_FAILED();
    return EMB_OK;
}

template <int FMT>
int dispatch_quant_forward(int lpr, hipStream_t s, const emb_table *tables, int32_t T, int64_t B, int64_t nnz,
                           const int64_t *rows, const int64_t *offsets, int32_t D, int64_t row_bytes, int32_t mode,
                           float *out, uint32_t *status, bool hashed, int64_t *rows_out, int64_t *offsets_out, const int32_t *lengths)
{
#define EMB_QF(L)                                                                                              \
    return launch_quant_forward<L, FMT>(s, tables, T, B, nnz, rows, offsets, D, row_bytes, mode, out, status, \
                                         hashed, rows_out, offsets_out, lengths)
    switch (lpr) {
        case 1: EMB_QF(1);
        case 2: EMB_QF(2);
        case 4: EMB_QF(4);
        case 8: EMB_QF(8);
        case 16: EMB_QF(16);
        case 32: EMB_QF(32);
        default: EMB_QF(64);
    }
#undef EMB_QF
}

}  // namespace

// Rows as such: INT8 / INT4 rows are made by a wavefront each, MXFP4 rows block by block.
int emb_check_quant_rows(int32_t D, int32_t dtype)
{
    if (!emb_is_quant(dtype)) return EMB_ERR_INVALID_ARG;
    if (D <= 0) return EMB_ERR_INVALID_ARG;
    if (dtype == EMB_MXFP4) return D % 32 != 0 || D > 65536 ? EMB_ERR_UNSUPPORTED : EMB_OK;
    if (D % Q_ELEMS != 0 || D > Q_ELEMS * EMB_WAVE) return EMB_ERR_UNSUPPORTED;
    return EMB_OK;
}

// Rows that a lookup reads: at most a wavefront of lanes.
int emb_check_quant_shape(int32_t D, int32_t dtype)
{
    const int rc = emb_check_quant_rows(D, dtype);
    if (rc != EMB_OK) return rc;
    return D > Q_ELEMS * EMB_WAVE ? EMB_ERR_UNSUPPORTED : EMB_OK;
}

extern "C" int64_t emb_row_bytes(int32_t D, int32_t dtype)
{
    if (D <= 0) return 0;
    switch (dtype) {
        case EMB_F32: return (int64_t)D * 4;
        case EMB_BF16: return (int64_t)D * 2;
        case EMB_INT8: return (8 + (int64_t)D + 15) / 16 * 16;
        case EMB_INT4: return D % 2 ? 0 : (8 + (int64_t)D / 2 + 15) / 16 * 16;
        case EMB_INT4_ROW64: return D % 2 ? 0 : (8 + (int64_t)D / 2 + 63) / 64 * 64;
        case EMB_MXFP4: return D % 32 ? 0 : ((int64_t)D / 2 + D / 32 + 15) / 16 * 16;
        default: return 0;
    }
}

// Called by emb_bag_forward (forward.hip) once the common arguments are checked.
// hashed: rows_dev holds raw IDs; rows_out_dev (nullable) then receives the row numbers.
// offsets_out_dev != NULL: the offsets are written there, made from lengths_dev or, where that is NULL, from the
// sums within tiles in offsets_dev.
int emb_forward_quant(const emb_table *tables_dev, int32_t T, int32_t D, int32_t dtype, const int64_t *rows_dev,
                      const int64_t *offsets_dev, int64_t B, int64_t nnz, int32_t mode, float *out_dev,
                      uint32_t *status_dev, hipStream_t s, bool hashed, int64_t *rows_out_dev,
                      int64_t *offsets_out_dev, const int32_t *lengths_dev)
{
    const int64_t rb = emb_row_bytes(D, dtype);
    const int lpr = emb_quant_lanes(D);
#define EMB_QFF(FMT)                                                                                               \
    return dispatch_quant_forward<FMT>(lpr, s, tables_dev, T, B, nnz, rows_dev, offsets_dev, D, rb, mode, out_dev,  \
                                       status_dev, hashed, rows_out_dev, offsets_out_dev, lengths_dev)
    switch (emb_quant_format(dtype)) {
        case EMB_FMT_INT8: EMB_QFF(EMB_FMT_INT8);
        case EMB_FMT_INT4: EMB_QFF(EMB_FMT_INT4);
        default: EMB_QFF(EMB_FMT_MXFP4);
    }
#undef EMB_QFF
}
