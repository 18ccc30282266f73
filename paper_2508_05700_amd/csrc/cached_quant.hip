// Hot-row cache of fewer bits than its table: rows are quantised as they are written to
// the cache, and the lookup reads hits from there and misses from the full-precision
// table (paper Section 3.3: tables hosted in CPU memory; Section 4.1.2: tables stored
// as INT4).  A cache of the same bytes holds five times the rows (fp32, D = 64, MXFP4:
// 48 for 256 bytes), and the rows it does not hold lose nothing.
//
// The cache's index and the order of its rows are those of the plain cache
// (cache_index.h); quant_rows.hip writes the rows.
//
// The lookup has the loop of gather_quant.h: a group of LPR = D/16 lanes owns a bag,
// 16 elements a lane.  The lane that resolves an entry marks the address of a table
// row (bit 0; rows are 16-byte aligned), and where a row is added, the lanes of
// a group go one way or the other: 8 or 16 bytes of codes and the scale, or 64
// (fp32) or 32 (bf16) bytes of the row.  Rows are added in the order of
// the bag's lookups, whichever side they come from.
#include "cache_index.h"
#include "emb_internal.h"
#include "gather_quant.h"
#include "u64mod.h"

namespace {

constexpr uint64_t TABLE_ROW = 1;

struct QuantCachedSource {
    const char *table;
    const char *cache_rows;
    const CacheEntry *index;
    uint64_t num_rows, num_hot;
    int64_t table_row_bytes, cache_row_bytes;
    uint32_t *status;
    uint32_t hits, misses;
    bool hashed;
    uint64_t salt, magic;
    __device__ __forceinline__ uint64_t resolve(int64_t r, int64_t)
    {
        if (hashed) r = (int64_t)emb_fast_mod(emb_splitmix64((uint64_t)r ^ salt), num_rows, magic);
        if ((uint64_t)r >= num_rows) {
            emb_flag(status, EMB_STATUS_BAD_INDEX);
            return 0ull;
        }
        const int64_t slot = cache_probe(index, (uint64_t)r, num_hot);
        if (slot >= 0) {
            ++hits;
            return reinterpret_cast<uint64_t>(cache_rows + slot * cache_row_bytes);
        }
        ++misses;
        return reinterpret_cast<uint64_t>(table + r * table_row_bytes) | TABLE_ROW;
    }
};

// N entries of a group's batch, from entry k0 on, each a cache row or a table row.
template <int LPR, int FMT, bool BF16, int N, int IPL>
__device__ __forceinline__ void gather_either_rows(float (&acc)[Q_ELEMS], const uint64_t (&mine)[IPL], int k0, QuantPlace at,
                                                   uint32_t table_off)
{
    constexpr int CW = FMT == EMB_FMT_INT8 ? 4 : 2;
    constexpr int CHUNKS = BF16 ? 2 : 4;      // 16-byte pieces of 16 elements
    uint4 v[N][CHUNKS];                       // a cache row: codes in the first, scale (and bias) in the second
    bool from_table[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint64_t p = reinterpret_cast<uint64_t>(group_bcast_ptr<LPR>(mine[IPL == 1 ? 0 : (k0 + i) / LPR], (k0 + i) % LPR));
        from_table[i] = (p & TABLE_ROW) != 0;
        const char *row = reinterpret_cast<const char *>(p & ~TABLE_ROW);
        if (from_table[i]) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) v[i][c] = load_chunk(row + table_off + 16 * c);
        } else if (FMT == EMB_FMT_MXFP4) {
            const uint2 w = load_u2(row + at.code);
            v[i][0] = make_uint4(w.x, w.y, 0u, 0u);
            v[i][1].x = *(const EMB_GLOBAL uint8_t *)(row + at.scale);
        } else {
            const uint2 h = load_u2(row), w = load_u2(row + at.code);
            v[i][1].x = h.x;
            v[i][1].y = h.y;
            v[i][0] = make_uint4(w.x, w.y, 0u, 0u);
            if (FMT == EMB_FMT_INT8) {
                const uint2 w2 = load_u2(row + at.code + 8);
                v[i][0].z = w2.x;
                v[i][0].w = w2.y;
            }
        }
    }
    __builtin_amdgcn_sched_barrier(0);   // every load of the batch before its first add
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (from_table[i]) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const uint32_t w[4] = {v[i][c].x, v[i][c].y, v[i][c].z, v[i][c].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (BF16) {
                        acc[(8 * c + 2 * j) % Q_ELEMS] += __uint_as_float(w[j] << 16);
                        acc[(8 * c + 2 * j + 1) % Q_ELEMS] += __uint_as_float(w[j] & 0xFFFF0000u);
                    } else {
                        acc[4 * c + j] += __uint_as_float(w[j]);
                    }
                }
            }
        } else {
            const uint32_t all[4] = {v[i][0].x, v[i][0].y, v[i][0].z, v[i][0].w};
            uint32_t w[CW];
#pragma unroll
            for (int j = 0; j < CW; ++j) w[j] = all[j];
            float f[Q_ELEMS];
            if constexpr (FMT == EMB_FMT_MXFP4) {
                mx_codes_to_float(w, v[i][1].x, f);
#pragma unroll
                for (int x = 0; x < Q_ELEMS; ++x) acc[x] += f[x];
            } else {
                const float scale = __uint_as_float(v[i][1].x), bias = __uint_as_float(v[i][1].y);
                codes_to_float<FMT>(w, f);
#pragma unroll
                for (int x = 0; x < Q_ELEMS; ++x) acc[x] += __builtin_fmaf(scale, f[x], bias);
            }
        }
    }
}

struct QuantCachedArgs {
    QuantCachedSource src;
    int64_t B, nnz;
    const int64_t *ids, *offsets;
    int32_t D, mode;
    float *out;
    unsigned long long *hit_miss;
    uint32_t *status;
    hipStream_t s;
};

constexpr int QC_UNROLL = 4;   // 16 registers an fp32 row and lane

template <int LPR, int FMT, bool BF16>
__global__ __launch_bounds__(Q_BLOCK) void bag_forward_cached_either_kernel(QuantCachedSource src, int64_t B, int64_t nnz,
                                                                            const int64_t *__restrict__ ids,
                                                                            const int64_t *__restrict__ offsets, int32_t D,
                                                                            int32_t mode, float *__restrict__ out,
                                                                            unsigned long long *hit_miss, uint32_t *status)
{
    constexpr int GROUPS = Q_BLOCK / LPR;
    constexpr int IPL = QC_UNROLL > LPR ? QC_UNROLL / LPR : 1;
    constexpr int IB = IPL * LPR;
    const int l = threadIdx.x % LPR;
    const int64_t bag = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LPR;
    const bool live = bag < B;
    const bool mine_elems = l * Q_ELEMS < D;
    const QuantPlace at = quant_place<FMT>(l, D);
    const uint32_t table_off = mine_elems ? (uint32_t)l * Q_ELEMS * (BF16 ? 2u : 4u) : 0u;
    int64_t s = 0, e = 0;
    if (live) {
        s = offsets[bag];
        e = offsets[bag + 1];
        if (s < 0 || e < s || e > nnz) {
            if (l == 0) emb_flag(status, EMB_STATUS_BAD_OFFSETS);
            s = e = 0;
        }
    }
    float acc[Q_ELEMS];
#pragma unroll
    for (int i = 0; i < Q_ELEMS; ++i) acc[i] = 0.f;
    const uint64_t zero_row = reinterpret_cast<uint64_t>(emb_zero_row);
    int64_t next[IPL];
#pragma unroll
    for (int m = 0; m < IPL; ++m) {
        const int64_t j = s + m * LPR + l;
        next[m] = j < e ? ids[j] : 0;
    }
    for (int64_t base = s; base < e; base += IB) {
        uint64_t mine[IPL];
#pragma unroll
        for (int m = 0; m < IPL; ++m) {
            const int64_t j = base + m * LPR + l;
            mine[m] = 0ull;
            if (j < e) mine[m] = src.resolve(next[m], j);
            if (mine[m] == 0ull) mine[m] = zero_row;
            if (j + IB < e) next[m] = ids[j + IB];
        }
#pragma unroll(LPR <= 16 ? IB / QC_UNROLL : 1)
        for (int u = 0; u < IB / QC_UNROLL; ++u) {
            const int64_t left = e - base - u * QC_UNROLL;
            if (left > 0)
                gather_batch<QC_UNROLL>(left, [&](auto n) {
                    gather_either_rows<LPR, FMT, BF16, decltype(n)::value>(acc, mine, u * QC_UNROLL, at, table_off);
                });
        }
    }
    if (live && mine_elems) {
        const int64_t len = e - s;
        const bool mean = (mode == EMB_POOL_MEAN) && len > 0;
        const float flen = (float)len;
        float4 *o = reinterpret_cast<float4 *>(out + bag * (int64_t)D + l * Q_ELEMS);
#pragma unroll
        for (int i = 0; i < Q_ELEMS / 4; ++i) {
            float4 v = make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
            if (mean) v = make_float4(v.x / flen, v.y / flen, v.z / flen, v.w / flen);
            o[i] = v;
        }
    }
    cache_add_hit_miss(src.hits, src.misses, hit_miss);
}

template <int FMT, bool BF16>
void launch_cached_either(const QuantCachedArgs &a)
{
#define EMB_CE(L)                                                                                                        \
    hipLaunchKernelGGL((bag_forward_cached_either_kernel<L, FMT, BF16>),                                                 \
                       dim3((unsigned)((a.B + Q_BLOCK / L - 1) / (Q_BLOCK / L))), dim3(Q_BLOCK), 0, a.s, a.src, a.B,      \
                       a.nnz, a.ids, a.offsets, a.D, a.mode, a.out, a.hit_miss, a.status)
    switch (emb_quant_lanes(a.D)) {
        case 1: EMB_CE(1); break;
        case 2: EMB_CE(2); break;
        case 4: EMB_CE(4); break;
        case 8: EMB_CE(8); break;
        case 16: EMB_CE(16); break;
        case 32: EMB_CE(32); break;
        default: EMB_CE(64);
    }
#undef EMB_CE
}

int check_types(int32_t D, int32_t dtype, int32_t cache_dtype)
{
    if (emb_elem_size(dtype) == 0) return EMB_ERR_INVALID_ARG;   // the table: fp32 or bf16
    const int rc = emb_check_quant_shape(D, cache_dtype);        // (D is then a multiple of 16: whole 16-byte pieces of a row)
    return rc != EMB_OK ? rc : emb_check_row_shape(D, dtype);
}

int build_entry(const void *table_dev, int64_t num_rows, int32_t D, int32_t dtype, int32_t cache_dtype,
                const void *old_rows_dev, const void *old_index_dev, int64_t old_num_hot, const int64_t *hot_rows_dev,
                int64_t num_hot, void *cache_rows_dev, void *cache_index_dev, uint64_t *moved_dev, uint32_t *status_dev,
                void *stream)
{
    int rc = check_types(D, dtype, cache_dtype);
    if (rc != EMB_OK) return rc;
    rc = emb_check_cache_build(table_dev, num_rows, D, dtype, old_rows_dev, old_index_dev, old_num_hot, hot_rows_dev, num_hot,
                               cache_rows_dev, cache_index_dev);
    if (rc != EMB_OK) return rc;
    hipStream_t s = emb_stream(stream);
    rc = emb_cache_index_launch(num_rows, hot_rows_dev, num_hot, cache_index_dev, status_dev, s);
    if (rc != EMB_OK || num_hot == 0) return rc;
    const emb_row_pick pick{hot_rows_dev, num_rows, old_index_dev, old_rows_dev, old_num_hot, moved_dev};
    return emb_quantize_launch(table_dev, dtype, (int64_t)D * emb_elem_size(dtype), num_hot, D, cache_dtype, cache_rows_dev, &pick, s);
}

int lookup_entry(const void *table_dev, int64_t num_rows, int32_t D, int32_t dtype, int32_t cache_dtype,
                 const void *cache_rows_dev, const void *cache_index_dev, int64_t num_hot, const int64_t *ids_dev,
                 const int64_t *offsets_dev, int64_t B, int64_t nnz, int32_t mode, float *out_dev, uint64_t *hit_miss_dev,
                 uint32_t *status_dev, void *stream, bool hashed, uint64_t salt)
{
    if (B < 0 || nnz < 0 || num_rows <= 0 || num_hot < 0) return EMB_ERR_INVALID_ARG;
    if (mode != EMB_POOL_SUM && mode != EMB_POOL_MEAN) return EMB_ERR_INVALID_ARG;
    const int rc = check_types(D, dtype, cache_dtype);
    if (rc != EMB_OK) return rc;
    if (B == 0) return EMB_OK;
    if (!table_dev || !cache_index_dev || (num_hot > 0 && !cache_rows_dev)) return EMB_ERR_INVALID_ARG;
    if (!offsets_dev || !out_dev || (nnz > 0 && !ids_dev)) return EMB_ERR_INVALID_ARG;
    if (!emb_aligned(table_dev, 16) || !emb_aligned(cache_index_dev, 16) || !emb_aligned(cache_rows_dev, 16) ||
        !emb_aligned(out_dev, 16))
        return EMB_ERR_INVALID_ARG;
    if (B > (int64_t)0x7FFFFFFF) return EMB_ERR_UNSUPPORTED;
    QuantCachedArgs a;
    a.src = QuantCachedSource{static_cast<const char *>(table_dev),
                              static_cast<const char *>(cache_rows_dev),
                              static_cast<const CacheEntry *>(cache_index_dev),
                              (uint64_t)num_rows,
                              (uint64_t)num_hot,
                              (int64_t)D * emb_elem_size(dtype),
                              emb_row_bytes(D, cache_dtype),
                              status_dev,
                              0u,
                              0u,
                              hashed,
                              salt,
                              emb_mod_magic((uint64_t)num_rows)};
    a.B = B; a.nnz = nnz;
    a.ids = ids_dev; a.offsets = offsets_dev;
    a.D = D; a.mode = mode;
    a.out = out_dev;
    a.hit_miss = reinterpret_cast<unsigned long long *>(hit_miss_dev);
    a.status = status_dev;
    a.s = emb_stream(stream);
    const bool bf16 = dtype == EMB_BF16;
    switch (emb_quant_format(cache_dtype)) {
        case EMB_FMT_INT8: bf16 ? launch_cached_either<EMB_FMT_INT8, true>(a) : launch_cached_either<EMB_FMT_INT8, false>(a); break;
        case EMB_FMT_INT4: bf16 ? launch_cached_either<EMB_FMT_INT4, true>(a) : launch_cached_either<EMB_FMT_INT4, false>(a); break;
        default: bf16 ? launch_cached_either<EMB_FMT_MXFP4, true>(a) : launch_cached_either<EMB_FMT_MXFP4, false>(a);
    }
    EMB_RETURN_IF_LAUNCH_FAILED();
    return EMB_OK;
}

}  // namespace

extern "C" int emb_cache_build_quantized(const void *table_dev, int64_t num_rows, int32_t D, int32_t dtype, int32_t cache_dtype,
                                         const int64_t *hot_rows_dev, int64_t num_hot, void *cache_rows_dev,
                                         void *cache_index_dev, uint32_t *status_dev, void *stream)
{
    return build_entry(table_dev, num_rows, D, dtype, cache_dtype, nullptr, nullptr, 0, hot_rows_dev, num_hot, cache_rows_dev,
                       cache_index_dev, nullptr, status_dev, stream);
}

extern "C" int emb_cache_rebuild_quantized(const void *table_dev, int64_t num_rows, int32_t D, int32_t dtype, int32_t cache_dtype,
                                           const void *old_cache_rows_dev, const void *old_cache_index_dev, int64_t old_num_hot,
                                           const int64_t *hot_rows_dev, int64_t num_hot, void *cache_rows_dev,
                                           void *cache_index_dev, uint64_t *moved_dev, uint32_t *status_dev, void *stream)
{
    if (!old_cache_index_dev) return EMB_ERR_INVALID_ARG;
    return build_entry(table_dev, num_rows, D, dtype, cache_dtype, old_cache_rows_dev, old_cache_index_dev, old_num_hot,
                       hot_rows_dev, num_hot, cache_rows_dev, cache_index_dev, moved_dev, status_dev, stream);
}

extern "C" int emb_bag_forward_cached_quantized(const void *table_dev, int64_t num_rows, int32_t D, int32_t dtype,
                                                int32_t cache_dtype, const void *cache_rows_dev, const void *cache_index_dev,
                                                int64_t num_hot, const int64_t *rows_dev, const int64_t *offsets_dev, int64_t B,
                                                int64_t nnz, int32_t mode, float *out_dev, uint64_t *hit_miss_dev,
                                                uint32_t *status_dev, void *stream)
{
    return lookup_entry(table_dev, num_rows, D, dtype, cache_dtype, cache_rows_dev, cache_index_dev, num_hot, rows_dev,
                        offsets_dev, B, nnz, mode, out_dev, hit_miss_dev, status_dev, stream, false, 0);
}

extern "C" int emb_bag_forward_cached_quantized_hashed(const void *table_dev, int64_t num_rows, int32_t D, int32_t dtype,
                                                       int32_t cache_dtype, const void *cache_rows_dev,
                                                       const void *cache_index_dev, int64_t num_hot, uint64_t salt,
                                                       const uint64_t *raw_dev, const int64_t *offsets_dev, int64_t B,
                                                       int64_t nnz, int32_t mode, float *out_dev, uint64_t *hit_miss_dev,
                                                       uint32_t *status_dev, void *stream)
{
    return lookup_entry(table_dev, num_rows, D, dtype, cache_dtype, cache_rows_dev, cache_index_dev, num_hot,
                        reinterpret_cast<const int64_t *>(raw_dev), offsets_dev, B, nnz, mode, out_dev, hit_miss_dev, status_dev,
                        stream, true, salt);
}
