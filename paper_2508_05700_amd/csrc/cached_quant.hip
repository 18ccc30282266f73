// Hot-row cache of fewer bits than its table: rows are quantised as they are written to
// the cache, and the lookup reads hits from there and misses from the full-precision
// table (paper Section 3.3: tables hosted in CPU memory; Section 4.1.2: tables stored
// as INT4).  A cache of the same bytes holds five times the rows (fp32, D = 64, MXFP4:
// 48 for 256 bytes), and the rows it does not hold lose nothing.
//
// The cache's index and the order of its rows are those of the plain cache
// (cache_index.h); quant_rows.hip writes the rows.
//
// The lookup has the loop of gather_quant.h: a group of LPR lanes owns a bag, 8 or 16
// elements a lane.  The lane that resolves an entry marks the address of a table
// row (bit 0; rows are 16-byte aligned).  Rows are added in the order of the bag's
// lookups, whichever side they come from.
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
    // An entry is resolved in two steps, so that the index can be asked for a batch ahead: its table row (num_rows for
    // one that is skipped) and entry of the index, then the address.
    __device__ __forceinline__ uint64_t row_of(int64_t r) const
    {
        if (hashed) r = (int64_t)emb_fast_mod(emb_splitmix64((uint64_t)r ^ salt), num_rows, magic);
        if ((uint64_t)r < num_rows) return (uint64_t)r;
        emb_flag(status, EMB_STATUS_BAD_INDEX);
        return num_rows;
    }
    __device__ __forceinline__ uint4 entry_of(uint64_t r) const   // (for a skipped one any entry)
    {
        return load_chunk(reinterpret_cast<const char *>(index + ((r < num_rows ? r : 0) >> 6)));
    }
    __device__ __forceinline__ uint64_t address(uint64_t r, const uint4 &entry)
    {
        if (r >= num_rows) return reinterpret_cast<uint64_t>(emb_zero_row);
        const int64_t slot = cache_slot(entry, (int)(r & 63), num_hot);
        if (slot >= 0) {
            ++hits;
            return reinterpret_cast<uint64_t>(cache_rows + slot * cache_row_bytes);
        }
        ++misses;
        return reinterpret_cast<uint64_t>(table + (int64_t)r * table_row_bytes) | TABLE_ROW;
    }
};

// The elements of a lane: 8 (rows of up to 512; 16 384 bags of 30 lookups of 64 elements 25 us, with 4 a lane 35 to 38), so that many
// rows can be in flight, or 16.  Its codes are W words; where they
// are in a row, and the scale of their block (MXFP4), lanes past the row reading its first ones.
template <int FMT, int E>
struct LaneCodes {
    static constexpr int W = E * (FMT == EMB_FMT_INT8 ? 8 : 4) / 32;
    static __device__ __forceinline__ QuantPlace place(int l, int32_t D)
    {
        const uint32_t at = l * E < D ? (uint32_t)l : 0u;
        if (FMT == EMB_FMT_MXFP4) return QuantPlace{at * (W * 4), (uint32_t)D / 2u + at * E / 32u};
        return QuantPlace{8u + at * (W * 4), 0u};
    }
    static __device__ __forceinline__ void load(const char *p, uint32_t (&w)[W])
    {
        if constexpr (W == 1) {
            w[0] = *(const EMB_GLOBAL uint32_t *)p;
        } else {
#pragma unroll
            for (int i = 0; i < W; i += 2) {   // (8-byte aligned, as lanes and headers are)
                const uint2 v = load_u2(p + 4 * i);
                w[i] = v.x;
                w[i + 1] = v.y;
            }
        }
    }
    // hdr: scale byte, or scale and bias
    static __device__ __forceinline__ void add(const uint32_t (&w)[W], const uint2 &hdr, float (&acc)[E])
    {
        const float scale = __uint_as_float(FMT == EMB_FMT_MXFP4 ? hdr.x << 23 : hdr.x), bias = __uint_as_float(hdr.y);
#pragma unroll
        for (int h = 0; h < W; ++h) {
            if constexpr (FMT == EMB_FMT_MXFP4) {
                const emb_f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[h], scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[h], scale, 1);
                const emb_f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[h], scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[h], scale, 3);
                const float f[8] = {a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[8 * h + i] += f[i];
            } else if constexpr (FMT == EMB_FMT_INT4) {
                const uint32_t even = w[h] & 0x0F0F0F0Fu, odd = (w[h] >> 4) & 0x0F0F0F0Fu;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    acc[8 * h + 2 * i] += __builtin_fmaf(scale, (float)((even >> (8 * i)) & 0xFFu), bias);
                    acc[8 * h + 2 * i + 1] += __builtin_fmaf(scale, (float)((odd >> (8 * i)) & 0xFFu), bias);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[4 * h + i] += __builtin_fmaf(scale, (float)((w[h] >> (8 * i)) & 0xFFu), bias);
            }
        }
    }
};

// N entries of a group's batch, from entry k0 on, each a cache row or a table row.  Both are read and added, the one that the
// entry does not select being the row of zeros (which stays in the L1): reads under a branch would share
// registers and wait for each other, row by row (16 384 bags of 30, one fifth of them misses, 16 elements a lane: 33 us, so 25).
template <int LPR, int FMT, int E, bool BF16, int N, int IPL>
__device__ __forceinline__ void gather_either_rows(float (&acc)[E], const uint64_t (&mine)[IPL], int k0, QuantPlace at,
                                                   uint32_t table_off)
{
    typedef LaneCodes<FMT, E> Codes;
    constexpr int CHUNKS = E * (BF16 ? 2 : 4) / 16;   // 16-byte pieces of a table row
    uint4 full[N][CHUNKS];
    uint32_t w[N][Codes::W];
    uint2 hdr[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint64_t p = reinterpret_cast<uint64_t>(group_bcast_ptr<LPR>(mine[IPL == 1 ? 0 : (k0 + i) / LPR], (k0 + i) % LPR));
        const bool from_table = (p & TABLE_ROW) != 0;
        const char *zeros = reinterpret_cast<const char *>(emb_zero_row), *row = reinterpret_cast<const char *>(p & ~TABLE_ROW);
        const char *const t = from_table ? row : zeros, *const q = from_table ? zeros : row;
        Codes::load(q + at.code, w[i]);
        hdr[i] = FMT == EMB_FMT_MXFP4 ? make_uint2(*(const EMB_GLOBAL uint8_t *)(q + at.scale), 0u) : load_u2(q);
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) full[i][k] = load_chunk(t + table_off + 16 * k);
    }
    __builtin_amdgcn_sched_barrier(0);   // every load of the batch before its first add
#pragma unroll
    for (int i = 0; i < N; ++i) {
        Codes::add(w[i], hdr[i], acc);
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            const uint32_t v[4] = {full[i][k].x, full[i][k].y, full[i][k].z, full[i][k].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (BF16) {
                    acc[(8 * k + 2 * j) % E] += __uint_as_float(v[j] << 16);
                    acc[(8 * k + 2 * j + 1) % E] += __uint_as_float(v[j] & 0xFFFF0000u);
                } else {
                    acc[(4 * k + j) % E] += __uint_as_float(v[j]);
                }
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

// What bounds the lookup is the time that a batch takes to come (its index entries, then its rows), so batches are long, 128
// registers of fp32 rows, and the next one's entries are under way with this one's rows.
template <int LPR, int FMT, int E, bool BF16>
__global__ __launch_bounds__(Q_BLOCK) void bag_forward_cached_either_kernel(QuantCachedSource src, int64_t B, int64_t nnz,
                                                                            const int64_t *__restrict__ ids,
                                                                            const int64_t *__restrict__ offsets, int32_t D,
                                                                            int32_t mode, float *__restrict__ out,
                                                                            unsigned long long *hit_miss, uint32_t *status)
{
    constexpr int GROUPS = Q_BLOCK / LPR;
    constexpr int UNROLL = 128 / E;
    constexpr int IPL = UNROLL > LPR ? UNROLL / LPR : 1;
    constexpr int IB = IPL * LPR;
    const int l = threadIdx.x % LPR;
    const int64_t bag = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LPR;
    const bool live = bag < B;
    const bool mine_elems = l * E < D;
    const QuantPlace at = LaneCodes<FMT, E>::place(l, D);
    const uint32_t table_off = mine_elems ? (uint32_t)l * E * (BF16 ? 2u : 4u) : 0u;
    int64_t s = 0, e = 0;
    if (live) {
        s = offsets[bag];
        e = offsets[bag + 1];
        if (s < 0 || e < s || e > nnz) {
            if (l == 0) emb_flag(status, EMB_STATUS_BAD_OFFSETS);
            s = e = 0;
        }
    }
    float acc[E];
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] = 0.f;
    int64_t id[IPL];          // of the batch after the next
    uint64_t row[IPL];        // of the next batch, with its index entries
    uint4 entry[IPL];
    auto fetch_ids = [&](int64_t base) {
#pragma unroll
        for (int m = 0; m < IPL; ++m) {
            const int64_t j = base + m * LPR + l;
            if (j < e) id[m] = ids[j];
        }
    };
    auto probe = [&](int64_t base) {
#pragma unroll
        for (int m = 0; m < IPL; ++m) {
            const int64_t j = base + m * LPR + l;
            row[m] = src.num_rows;
            if (j < e) {
                row[m] = src.row_of(id[m]);
                entry[m] = src.entry_of(row[m]);
            }
        }
    };
    fetch_ids(s);
    probe(s);
    fetch_ids(s + IB);
    for (int64_t base = s; base < e; base += IB) {
        uint64_t mine[IPL];
#pragma unroll
        for (int m = 0; m < IPL; ++m) mine[m] = src.address(row[m], entry[m]);
        probe(base + IB);
        fetch_ids(base + 2 * IB);
#pragma unroll(LPR <= 16 ? IB / UNROLL : 1)
        for (int u = 0; u < IB / UNROLL; ++u) {
            const int64_t left = e - base - u * UNROLL;
            if (left > 0)
                gather_batch<UNROLL>(left, [&](auto n) {
                    gather_either_rows<LPR, FMT, E, BF16, decltype(n)::value>(acc, mine, u * UNROLL, at, table_off);
                });
        }
    }
    if (live && mine_elems) {
        const int64_t len = e - s;
        const bool mean = (mode == EMB_POOL_MEAN) && len > 0;
        const float flen = (float)len;
        float4 *o = reinterpret_cast<float4 *>(out + bag * (int64_t)D + l * E);
#pragma unroll
        for (int i = 0; i < E / 4; ++i) {
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
#define EMB_CE(L, E)                                                                                                     \
    for (int64_t b = 0; b < a.B; b += emb_launch_items(L)) {                                                             \
        const int64_t n = a.B - b < emb_launch_items(L) ? a.B - b : emb_launch_items(L);                                 \
        hipLaunchKernelGGL((bag_forward_cached_either_kernel<L, FMT, E, BF16>),                                          \
                           dim3((unsigned)((n + Q_BLOCK / L - 1) / (Q_BLOCK / L))), dim3(Q_BLOCK), 0, a.s, a.src, n,      \
                           a.nnz, a.ids, a.offsets + b, a.D, a.mode, a.out + b * a.D, a.hit_miss, a.status);             \
    }
    if (a.D <= 16) EMB_CE(2, 8)
    else if (a.D <= 32) EMB_CE(4, 8)
    else if (a.D <= 64) EMB_CE(8, 8)
    else if (a.D <= 128) EMB_CE(16, 8)
    else if (a.D <= 256) EMB_CE(32, 8)
    else if (a.D <= 512) EMB_CE(64, 8)
    else EMB_CE(64, 16)
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
