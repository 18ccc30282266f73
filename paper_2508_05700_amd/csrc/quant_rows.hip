// Quantisers of table rows (paper Section 4.1.2: tables are stored as INT4 after
// post-training quantisation) and the way back.  The storage is described in
// quant.hip.
//
//   INT8, INT4   scale and bias of a row come from its smallest and largest
//                element, so a row is made by a group of LPR = D/16 lanes (rounded
//                up to a power of two), 16 elements each;
//   MXFP4        a block of 32 elements stands for itself: a thread takes 16 bytes
//                of the source (4 fp32 or 8 bf16 elements), the 8 (4) threads of a block
//                find its largest magnitude by data-parallel moves, and the hardware
//                rounds to 4-bit floats by a power of two, exactly as the definition
//                says (ties, saturation, subnormal scales).
//
// All are bound by the bytes of the source and of the rows (4e6 x 64 fp32 to MXFP4 240 us, 5.0 TB/s, and back 235; a copy
// gets 5.2; with the same rows again and again 207 and 247, INT8 232 and 238, INT4 215 and 209).  The same kernels fill a
// cache of quantised rows from a full-precision table (RowPick): the source row is then
// chosen by a list, and a row that an older cache of the same type holds is copied.
#include "cache_index.h"
#include "emb_internal.h"
#include "gather_quant.h"

namespace {

constexpr int PICK_BLOCK = 1024;   // a launch that counts kept and fetched rows has few workgroups: adds to one word
constexpr int PICK_GRID = 512;     // are served one at a time (as in the plain cache's copy)

// Where row k of a cache comes from: -1 nowhere (a bad entry of the list), else the table row; `kept` if the
// older cache has it, then at `old`.
struct PickedRow {
    int64_t row;
    const char *old;
};
__device__ __forceinline__ PickedRow pick_row(const emb_row_pick &p, int64_t k, int64_t row_bytes)
{
    PickedRow r{p.hot[k], nullptr};
    if (r.row < 0 || r.row >= p.num_rows) return PickedRow{-1, nullptr};
    if (p.old_index) {
        const int64_t slot = cache_probe(reinterpret_cast<const CacheEntry *>(p.old_index), (uint64_t)r.row, (uint64_t)p.old_num_hot);
        if (slot >= 0) r.old = static_cast<const char *>(p.old_rows) + slot * row_bytes;
    }
    return r;
}

// 16 elements of a source row, as fp32
template <bool BF16>
__device__ __forceinline__ void load_elems(const char *p, float (&x)[Q_ELEMS])
{
#pragma unroll
    for (int i = 0; i < (BF16 ? 2 : 4); ++i) {
        const uint4 v = load_chunk(p + 16 * i);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (BF16) {
                x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
                x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
            } else {
                x[4 * i + j] = __uint_as_float(w[j]);
            }
        }
    }
}

// One row by the LPR lanes of a group; src: the lane's 16 elements, row: where the row goes.  Every lane of the group
// calls this; live: the lane has elements.
template <int LPR, int BITS, bool BF16>
__device__ __forceinline__ void quantize_row(const char *src, bool live, int l, int32_t D, int64_t row_bytes, char *row)
{
    constexpr float QMAX = BITS == 8 ? 255.0f : 15.0f;
    float x[Q_ELEMS];
    if (live) {
        load_elems<BF16>(src, x);
    } else {
#pragma unroll
        for (int i = 0; i < Q_ELEMS; ++i) x[i] = 0.f;
    }
    // row minimum and maximum: exact, so the order of the comparisons does not matter
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < Q_ELEMS; ++i) {
        lo = x[i] < lo ? x[i] : lo;
        hi = x[i] > hi ? x[i] : hi;
    }
    if (!live) {     // lanes past the row must not take part in min / max
        lo = __builtin_inff();
        hi = -__builtin_inff();
    }
#pragma unroll
    for (int d = 1; d < LPR; d <<= 1) {
        const float ol = __shfl_xor(lo, d, LPR), oh = __shfl_xor(hi, d, LPR);
        lo = ol < lo ? ol : lo;
        hi = oh > hi ? oh : hi;
    }
    if (!live) return;
    // IEEE fp32 division and round-half-even, as the definition states
    const float scale = hi == lo ? 1.0f : (hi - lo) / QMAX;
    const float bias = lo;
    uint32_t code[Q_ELEMS];
#pragma unroll
    for (int i = 0; i < Q_ELEMS; ++i) {
        float q = rintf((x[i] - bias) / scale);
        q = q < 0.0f ? 0.0f : q;
        q = q > QMAX ? QMAX : q;
        code[i] = (uint32_t)q;
    }
    if (BITS == 4) {
        uint2 w = make_uint2(0u, 0u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w.x |= code[i] << (4 * i);
            w.y |= code[8 + i] << (4 * i);
        }
        *reinterpret_cast<uint2 *>(row + 8 + l * 8) = w;
    } else {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < Q_ELEMS; ++i) w[i / 4] |= code[i] << (8 * (i % 4));
        *reinterpret_cast<uint2 *>(row + 8 + l * 16) = make_uint2(w[0], w[1]);
        *reinterpret_cast<uint2 *>(row + 16 + l * 16) = make_uint2(w[2], w[3]);
    }
    if (l == 0) {
        *reinterpret_cast<uint2 *>(row) = make_uint2(__float_as_uint(scale), __float_as_uint(bias));
        // header and codes end on a multiple of 8 and so does the row: the padding is whole 8-byte words
        for (int64_t at = 8 + (int64_t)D * BITS / 8; at < row_bytes; at += 8)
            *reinterpret_cast<uint2 *>(row + at) = make_uint2(0u, 0u);
    }
}

template <int LPR, int BITS, bool BF16>
__global__ __launch_bounds__(Q_BLOCK) void quantize_rows_kernel(const char *__restrict__ src, int64_t src_pitch, int64_t R, int32_t D,
                                                                int64_t row_bytes, char *__restrict__ dst)
{
    constexpr int GROUPS = Q_BLOCK / LPR;
    const int l = threadIdx.x % LPR;
    const int64_t r = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LPR;
    quantize_row<LPR, BITS, BF16>(src + r * src_pitch + l * Q_ELEMS * (BF16 ? 2 : 4), r < R && l * Q_ELEMS < D, l, D,
                                  row_bytes, dst + r * row_bytes);
}

template <int LPR, int BITS, bool BF16>
__global__ __launch_bounds__(PICK_BLOCK) void quantize_picked_kernel(const char *__restrict__ src, int64_t src_pitch, int64_t R,
                                                                     int32_t D, int64_t row_bytes, char *__restrict__ dst,
                                                                     emb_row_pick pick)
{
    constexpr int GROUPS = PICK_BLOCK / LPR;
    const int l = threadIdx.x % LPR;
    uint32_t kept = 0, fetched = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * GROUPS; r0 < R; r0 += (int64_t)gridDim.x * GROUPS) {
        const int64_t r = r0 + threadIdx.x / LPR;
        PickedRow from{-1, nullptr};
        if (r < R) from = pick_row(pick, r, row_bytes);
        const bool fetch = from.row >= 0 && !from.old;
        quantize_row<LPR, BITS, BF16>(src + from.row * src_pitch + l * Q_ELEMS * (BF16 ? 2 : 4), fetch && l * Q_ELEMS < D, l, D,
                                      row_bytes, dst + r * row_bytes);
        if (from.old)
            for (int64_t at = l * 16; at < row_bytes; at += LPR * 16)
                *reinterpret_cast<uint4 *>(dst + r * row_bytes + at) = load_chunk(from.old + at);
        if (l == 0) {
            kept += from.old ? 1u : 0u;
            fetched += fetch ? 1u : 0u;
        }
    }
    cache_add_hit_miss(kept, fetched, reinterpret_cast<unsigned long long *>(pick.moved));
}

// ---------------------------------------------------------------------------
// MXFP4
// ---------------------------------------------------------------------------
// Scale byte of a block whose largest magnitude has the fp32 bits `top`: floor(log2) is the exponent field less 127,
// two less than that biased by 127 again, not below 0 (fp32 subnormals among it); infinities and NaN give 255.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : (e > 2u ? e : 2u) - 2u;
}
__device__ __forceinline__ uint32_t max_u32(uint32_t a, uint32_t b) { return a > b ? a : b; }
// Maximum over the aligned groups of 8 (4) lanes, in all of them.
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    v = max_u32(v, dpp_move<0xB1>(v));                        // lanes 1 apart
    v = max_u32(v, dpp_move<0x4E>(v));                        // lanes 2 apart
    if (LANES == 8) v = max_u32(v, dpp_move<0x141>(v));       // the other half of 8
    return v;
}

// Elements that a thread takes are 16 bytes of the source; `rest` is what a thread does for its row besides: the scale byte of
// its block, and its share of the padding.
template <bool BF16>
__device__ __forceinline__ void mx_quantize_chunk(const uint4 &v, uint32_t c, uint32_t cpr, uint32_t D, uint32_t row_bytes, char *row)
{
    constexpr int LANES = BF16 ? 4 : 8;   // of a block
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) top = max_u32(top, max_u32((w[i] << 16) & 0x7FFFFFFFu, w[i] & 0x7FFF0000u));
        else top = max_u32(top, w[i] & 0x7FFFFFFFu);
    }
    top = lanes_max<LANES>(top);
    const uint32_t byte = mx_scale_byte(top);
    const float scale = __uint_as_float(byte << 23);
    uint32_t code = 0;
    if (BF16) {
#define EMB_MXB(I) code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(emb_b2, w[I]), scale, I)
        EMB_MXB(0); EMB_MXB(1); EMB_MXB(2); EMB_MXB(3);
#undef EMB_MXB
    } else {
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, 1);
    }
    if (byte == 255u) code = 0;
    if (BF16) *reinterpret_cast<uint32_t *>(row + 4 * c) = code;
    else *reinterpret_cast<uint16_t *>(row + 2 * c) = (uint16_t)code;
    if (c % LANES == 0) row[D / 2 + c / LANES] = (char)byte;
    for (uint32_t at = D / 2 + D / 32 + c; at < row_bytes; at += cpr) row[at] = 0;
}

// A tile is BLOCK * U chunks of 16 source bytes, neighbouring threads on neighbouring chunks.  cpr: chunks of a row (a
// multiple of a block's, so that the lanes of a block go the same way everywhere); magic = floor(2^32 / cpr) + 1: the high
// half of its product with x is x / cpr for x < 2^32 / cpr (x is below cpr + 4096 and cpr at most 16384).
struct ChunkPlace {
    int64_t row;
    uint32_t c;
};
__device__ __forceinline__ ChunkPlace chunk_place(int64_t row0, uint32_t local, uint32_t cpr, uint32_t magic)
{
    const uint32_t q = __umulhi(local, magic);
    return ChunkPlace{row0 + q, local - q * cpr};
}

constexpr int MX_BLOCK = 256, MX_UNROLL = 4;

template <bool BF16>
__global__ __launch_bounds__(MX_BLOCK) void mx_quantize_kernel(const char *__restrict__ src, int64_t src_pitch, int64_t R, uint32_t D,
                                                               uint32_t cpr, uint32_t magic, uint32_t row_bytes,
                                                               char *__restrict__ dst)
{
    const int64_t first = (int64_t)blockIdx.x * (MX_BLOCK * MX_UNROLL);
    const int64_t row0 = first / cpr;
    const uint32_t rem = (uint32_t)(first - row0 * cpr) + threadIdx.x;
    uint4 v[MX_UNROLL];
    ChunkPlace at[MX_UNROLL];
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
        at[u] = chunk_place(row0, rem + u * MX_BLOCK, cpr, magic);
        if (at[u].row < R) v[u] = load_chunk(src + at[u].row * src_pitch + at[u].c * 16);
    }
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u)
        if (at[u].row < R) mx_quantize_chunk<BF16>(v[u], at[u].c, cpr, D, row_bytes, dst + at[u].row * row_bytes);
}

template <bool BF16>
__global__ __launch_bounds__(PICK_BLOCK) void mx_quantize_picked_kernel(const char *__restrict__ src, int64_t src_pitch, int64_t R,
                                                                        uint32_t D, uint32_t cpr, uint32_t magic,
                                                                        uint32_t row_bytes, char *__restrict__ dst, emb_row_pick pick)
{
    uint32_t kept = 0, fetched = 0;
    const int64_t total = R * cpr;
    for (int64_t first = (int64_t)blockIdx.x * PICK_BLOCK; first < total; first += (int64_t)gridDim.x * PICK_BLOCK) {
        const int64_t row0 = first / cpr;
        const ChunkPlace at = chunk_place(row0, (uint32_t)(first - row0 * cpr) + threadIdx.x, cpr, magic);
        if (at.row >= R) continue;
        const PickedRow from = pick_row(pick, at.row, row_bytes);
        if (from.row < 0) continue;
        char *row = dst + at.row * row_bytes;
        if (from.old) {
            if (at.c * 16 < row_bytes) *reinterpret_cast<uint4 *>(row + at.c * 16) = load_chunk(from.old + at.c * 16);
        } else {
            mx_quantize_chunk<BF16>(load_chunk(src + from.row * src_pitch + at.c * 16), at.c, cpr, D, row_bytes, row);
        }
        if (at.c == 0) {
            kept += from.old ? 1u : 0u;
            fetched += from.old ? 0u : 1u;
        }
    }
    cache_add_hit_miss(kept, fetched, reinterpret_cast<unsigned long long *>(pick.moved));
}

// ---------------------------------------------------------------------------
// rows read back
// ---------------------------------------------------------------------------
// A thread writes 16 bytes (4 fp32 or 8 bf16 elements), in tiles as above; cpr counts chunks of the destination row.
template <int FMT, bool BF16>
__global__ __launch_bounds__(MX_BLOCK) void dequantize_rows_kernel(const char *__restrict__ src, int64_t R, uint32_t D, uint32_t cpr,
                                                                   uint32_t magic, uint32_t row_bytes, char *__restrict__ dst,
                                                                   int64_t dst_pitch)
{
    constexpr int E = BF16 ? 8 : 4;
    const int64_t first = (int64_t)blockIdx.x * (MX_BLOCK * MX_UNROLL);
    const int64_t row0 = first / cpr;
    const uint32_t rem = (uint32_t)(first - row0 * cpr) + threadIdx.x;
    ChunkPlace at[MX_UNROLL];
    uint2 code[MX_UNROLL], hdr[MX_UNROLL];
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
        at[u] = chunk_place(row0, rem + u * MX_BLOCK, cpr, magic);
        if (at[u].row >= R) continue;
        const char *row = src + at[u].row * row_bytes;
        if (FMT == EMB_FMT_MXFP4) {
            hdr[u].x = *(const EMB_GLOBAL uint8_t *)(row + D / 2 + at[u].c * E / 32);
            code[u].x = BF16 ? *(const EMB_GLOBAL uint32_t *)(row + at[u].c * 4) : *(const EMB_GLOBAL uint16_t *)(row + at[u].c * 2);
        } else {
            hdr[u] = load_u2(row);
            if (FMT == EMB_FMT_INT4)
                code[u].x = BF16 ? *(const EMB_GLOBAL uint32_t *)(row + 8 + at[u].c * 4) : *(const EMB_GLOBAL uint16_t *)(row + 8 + at[u].c * 2);
            else if (BF16)
                code[u] = load_u2(row + 8 + at[u].c * 8);
            else
                code[u].x = *(const EMB_GLOBAL uint32_t *)(row + 8 + at[u].c * 4);
        }
    }
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
        if (at[u].row >= R) continue;
        uint4 o;
        if constexpr (FMT == EMB_FMT_MXFP4) {
            const float scale = __uint_as_float(hdr[u].x << 23);
            if (BF16) {
                o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u].x, scale, 0));
                o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u].x, scale, 1));
                o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u].x, scale, 2));
                o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u].x, scale, 3));
            } else {
                const emb_f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u].x, scale, 0);
                const emb_f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u].x, scale, 1);
                o = make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
            }
        } else {
            const float scale = __uint_as_float(hdr[u].x), bias = __uint_as_float(hdr[u].y);
            float f[E];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint32_t q = FMT == EMB_FMT_INT4 ? (code[u].x >> (4 * i)) & 15u : ((i < 4 ? code[u].x : code[u].y) >> (8 * (i % 4))) & 255u;
                f[i] = __builtin_fmaf(scale, (float)q, bias);
            }
            if (BF16) {
                uint32_t h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    emb_b2 p;
                    p.x = (__bf16)f[(2 * i) % E];       // to nearest-even
                    p.y = (__bf16)f[(2 * i + 1) % E];
                    h[i] = __builtin_bit_cast(uint32_t, p);
                }
                o = make_uint4(h[0], h[1], h[2], h[3]);
            } else {
                o = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            }
        }
        *reinterpret_cast<uint4 *>(dst + at[u].row * dst_pitch + at[u].c * 16) = o;
    }
}

struct RowsArgs {
    const char *src;
    int64_t src_pitch, R;
    int32_t D;
    int64_t row_bytes;
    char *dst;
    const emb_row_pick *pick;   // nullable
    hipStream_t s;
};

inline unsigned pick_grid(int64_t work)   // workgroups of PICK_BLOCK threads for `work` of them
{
    const int64_t want = (work + PICK_BLOCK - 1) / PICK_BLOCK;
    return (unsigned)(want > PICK_GRID ? PICK_GRID : want);
}

template <int LPR, int BITS, bool BF16>
void launch_quantize(const RowsArgs &a)
{
    if (a.pick)
        hipLaunchKernelGGL((quantize_picked_kernel<LPR, BITS, BF16>), dim3(pick_grid(a.R * LPR)), dim3(PICK_BLOCK), 0, a.s, a.src,
                           a.src_pitch, a.R, a.D, a.row_bytes, a.dst, *a.pick);
    else
        hipLaunchKernelGGL((quantize_rows_kernel<LPR, BITS, BF16>), dim3((unsigned)((a.R * LPR + Q_BLOCK - 1) / Q_BLOCK)),
                           dim3(Q_BLOCK), 0, a.s, a.src, a.src_pitch, a.R, a.D, a.row_bytes, a.dst);
}

template <int BITS, bool BF16>
void dispatch_quantize(const RowsArgs &a)
{
    switch (emb_quant_lanes(a.D)) {
        case 1: return launch_quantize<1, BITS, BF16>(a);
        case 2: return launch_quantize<2, BITS, BF16>(a);
        case 4: return launch_quantize<4, BITS, BF16>(a);
        case 8: return launch_quantize<8, BITS, BF16>(a);
        case 16: return launch_quantize<16, BITS, BF16>(a);
        case 32: return launch_quantize<32, BITS, BF16>(a);
        default: return launch_quantize<64, BITS, BF16>(a);
    }
}

template <bool BF16>
void launch_mx_quantize(const RowsArgs &a)
{
    const uint32_t cpr = (uint32_t)a.D * (BF16 ? 2 : 4) / 16, magic = (uint32_t)(((uint64_t)1 << 32) / cpr) + 1u;
    const int64_t chunks = a.R * (int64_t)cpr, blocks = (chunks + MX_BLOCK * MX_UNROLL - 1) / (MX_BLOCK * MX_UNROLL);
    if (a.pick)
        hipLaunchKernelGGL((mx_quantize_picked_kernel<BF16>), dim3(pick_grid(chunks)), dim3(PICK_BLOCK), 0, a.s, a.src, a.src_pitch,
                           a.R, (uint32_t)a.D, cpr, magic, (uint32_t)a.row_bytes, a.dst, *a.pick);
    else
        hipLaunchKernelGGL((mx_quantize_kernel<BF16>), dim3((unsigned)blocks), dim3(MX_BLOCK), 0, a.s, a.src, a.src_pitch, a.R,
                           (uint32_t)a.D, cpr, magic, (uint32_t)a.row_bytes, a.dst);
}

template <int FMT, bool BF16>
void launch_dequantize(const char *src, int64_t R, int32_t D, int64_t row_bytes, char *dst, int64_t dst_pitch, hipStream_t s)
{
    const uint32_t cpr = (uint32_t)D * (BF16 ? 2 : 4) / 16, magic = (uint32_t)(((uint64_t)1 << 32) / cpr) + 1u;
    const int64_t blocks = (R * (int64_t)cpr + MX_BLOCK * MX_UNROLL - 1) / (MX_BLOCK * MX_UNROLL);
    hipLaunchKernelGGL((dequantize_rows_kernel<FMT, BF16>), dim3((unsigned)blocks), dim3(MX_BLOCK), 0, s, src, R, (uint32_t)D, cpr,
                       magic, (uint32_t)row_bytes, dst, dst_pitch);
}

// Pitch in bytes of full-precision rows, or 0 if it is none the kernels take.
inline int64_t plain_pitch(int32_t D, int32_t dtype, int64_t stride)
{
    const int64_t esz = emb_elem_size(dtype);
    if (esz == 0 || stride < D || stride > INT64_MAX / 16) return 0;
    return stride * esz % 16 == 0 ? stride * esz : 0;
}

}  // namespace

int emb_quantize_launch(const void *src, int32_t src_dtype, int64_t src_pitch, int64_t R, int32_t D, int32_t dtype, void *dst,
                        const emb_row_pick *pick, hipStream_t s)
{
    const int64_t rb = emb_row_bytes(D, dtype);
    const bool bf16 = src_dtype == EMB_BF16;
    // threads of a row: 16 elements each, or (MXFP4) MX_UNROLL times 16 bytes; a launch that picks has a bounded grid
    const int threads = dtype == EMB_MXFP4 ? (D * emb_elem_size(src_dtype) + 63) / 64 : emb_quant_lanes(D);
    const int64_t most = pick ? R : emb_launch_items(threads);
    for (int64_t r = 0; r < R; r += most) {
        const RowsArgs a{static_cast<const char *>(src) + r * src_pitch, src_pitch, R - r < most ? R - r : most, D, rb,
                         static_cast<char *>(dst) + r * rb, pick, s};
        switch (emb_quant_format(dtype)) {
            case EMB_FMT_INT8: bf16 ? dispatch_quantize<8, true>(a) : dispatch_quantize<8, false>(a); break;
            case EMB_FMT_INT4: bf16 ? dispatch_quantize<4, true>(a) : dispatch_quantize<4, false>(a); break;
            default: bf16 ? launch_mx_quantize<true>(a) : launch_mx_quantize<false>(a);
        }
    }
    EMB_RETURN_IF_LAUNCH_FAILED();
    return EMB_OK;
}

extern "C" int emb_quantize_rows_from(const void *src_dev, int32_t src_dtype, int64_t src_stride, int64_t num_rows, int32_t D,
                                      int32_t dtype, void *dst_dev, void *stream)
{
    if (num_rows < 0) return EMB_ERR_INVALID_ARG;
    const int rc = emb_check_quant_rows(D, dtype);
    if (rc != EMB_OK) return rc;
    const int64_t pitch = plain_pitch(D, src_dtype, src_stride);
    if (pitch == 0) return EMB_ERR_INVALID_ARG;
    if (num_rows == 0) return EMB_OK;
    if (!src_dev || !dst_dev || !emb_aligned(src_dev, 16) || !emb_aligned(dst_dev, 16)) return EMB_ERR_INVALID_ARG;
    if (num_rows > (int64_t)0x7FFFFFFF) return EMB_ERR_UNSUPPORTED;
    return emb_quantize_launch(src_dev, src_dtype, pitch, num_rows, D, dtype, dst_dev, nullptr, emb_stream(stream));
}

extern "C" int emb_quantize_rows(const float *src_dev, int64_t num_rows, int32_t D, int32_t dtype, void *dst_dev, void *stream)
{
    if (num_rows < 0) return EMB_ERR_INVALID_ARG;
    const int rc = emb_check_quant_rows(D, dtype);
    if (rc != EMB_OK) return rc;
    return emb_quantize_rows_from(src_dev, EMB_F32, D, num_rows, D, dtype, dst_dev, stream);
}

extern "C" int emb_dequantize_rows(const void *src_dev, int32_t dtype, int64_t num_rows, int32_t D, void *dst_dev, int32_t dst_dtype,
                                   int64_t dst_stride, void *stream)
{
    if (num_rows < 0) return EMB_ERR_INVALID_ARG;
    const int rc = emb_check_quant_rows(D, dtype);
    if (rc != EMB_OK) return rc;
    const int64_t pitch = plain_pitch(D, dst_dtype, dst_stride);
    if (pitch == 0) return EMB_ERR_INVALID_ARG;
    if (num_rows == 0) return EMB_OK;
    if (!src_dev || !dst_dev || !emb_aligned(src_dev, 16) || !emb_aligned(dst_dev, 16)) return EMB_ERR_INVALID_ARG;
    if (num_rows > (int64_t)0x7FFFFFFF) return EMB_ERR_UNSUPPORTED;
    const char *src = static_cast<const char *>(src_dev);
    char *dst = static_cast<char *>(dst_dev);
    const int64_t rb = emb_row_bytes(D, dtype);
    hipStream_t s = emb_stream(stream);
    const int64_t most = emb_launch_items((D * emb_elem_size(dst_dtype) + 63) / 64);
#define EMB_DQ(FMT)                                                                                                  \
    dst_dtype == EMB_BF16 ? launch_dequantize<FMT, true>(src + r * rb, n, D, rb, dst + r * pitch, pitch, s)          \
                          : launch_dequantize<FMT, false>(src + r * rb, n, D, rb, dst + r * pitch, pitch, s)
    for (int64_t r = 0; r < num_rows; r += most) {
        const int64_t n = num_rows - r < most ? num_rows - r : most;
        switch (emb_quant_format(dtype)) {
            case EMB_FMT_INT8: EMB_DQ(EMB_FMT_INT8); break;
            case EMB_FMT_INT4: EMB_DQ(EMB_FMT_INT4); break;
            default: EMB_DQ(EMB_FMT_MXFP4);
        }
    }
#undef EMB_DQ
    EMB_RETURN_IF_LAUNCH_FAILED();
    return EMB_OK;
}
