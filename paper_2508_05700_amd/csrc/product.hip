// Product with the rows of an MXFP4 table: out[m, n] = sum over d of x[m, d] * W[n, d]:
// scores of vectors against a table's rows, or a dense layer over pooled rows (paper
// Section 3.1: the tables feed the ranking model; Section 4.1.2: 4-bit storage).
//
// Mathematics.  A block of 32 elements of W is 2^(s - 127) times 32 4-bit floats.  With x
// in MXFP4 too, the matrix unit takes both sides as stored, 16 bytes and one scale byte a
// lane (v_mfma_scale_f32_16x16x128_f8f6f4): products of 4-bit floats and powers of two are
// exact, sums are fp32.  With x in bf16, W's elements become bf16, exactly, and the product is
// bf16's.  With x in fp32, x = h + m + l with three bf16 parts of 8 bits each, exact unless a
// part falls below bf16's range: three bf16 products with the same W, summed in fp32 from the smallest part on.
//
// A wavefront holds a tile of 16*NT rows of W and 16*MT rows of x.  W is the unit's
// row operand, so that a lane ends with four neighbouring n of one m: one 16-byte store.
// The 32 elements of block b = 4 * step + g of a row go to lane group g = lane / 16.
#include "emb_internal.h"
#include "gather_quant.h"

namespace {

typedef int mx_i8 __attribute__((ext_vector_type(8)));
typedef float mx_f4 __attribute__((ext_vector_type(4)));
typedef __bf16 mx_b8 __attribute__((ext_vector_type(8)));
typedef float mx_f4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 mx_b4_any __attribute__((ext_vector_type(4), aligned(2)));

enum { X_MXFP4 = 0, X_BF16 = 1, X_F32 = 2 };

struct ProductArgs {
    const char *x, *w;
    int64_t x_pitch, w_pitch;      // bytes
    int64_t M, N;
    int32_t D;
    char *out;
    int64_t out_stride;            // elements
    int64_t tiles_m, tiles_n;      // workgroup tiles
};

__device__ __forceinline__ mx_i8 mx_operand(const uint4 &v)
{
    return mx_i8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
}

__device__ __forceinline__ uint32_t word_of(const uint4 &v, int j) { return j == 0 ? v.x : (j == 1 ? v.y : (j == 2 ? v.z : v.w)); }

// 8 codes of one word, by their block's power of two, as bf16 (exact)
__device__ __forceinline__ mx_b8 codes_to_bf16(uint32_t w, float scale)
{
    const emb_b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const emb_b2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return mx_b8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// Eight fp32 values as three bf16 parts: the upper 8 bits of the significand, the 8 after them and the last 8, all cut off, not
// rounded.  An infinity or a NaN is the first part alone.
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }
__device__ __forceinline__ void split_bf16(const uint4 &a, const uint4 &b, mx_b8 (&p)[3])
{
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, mid[8], low[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t top = w[i] & 0x7FFFFFFFu;
        const bool finite = top < 0x7F800000u;
        const float r = __uint_as_float(w[i]) - __uint_as_float(w[i] & 0xFFFF0000u);
        mid[i] = finite ? __float_as_uint(r) : 0u;
        low[i] = __float_as_uint(__uint_as_float(mid[i]) - __uint_as_float(mid[i] & 0xFFFF0000u));
        if (top > 0x7F800000u) w[i] |= 0x00400000u;   // a NaN whose mark is in the lower half stays one
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const uint32_t(&from)[8] = k == 0 ? w : (k == 1 ? mid : low);
        p[k] = __builtin_bit_cast(mx_b8, make_uint4(upper_halves(from[0], from[1]), upper_halves(from[2], from[3]),
                                                    upper_halves(from[4], from[5]), upper_halves(from[6], from[7])));
    }
}

template <int XT, int MT, int NT, int KS, bool OUT_BF16>
__global__ __launch_bounds__(KS > 1 ? 64 * KS : 256) void product_direct_kernel(ProductArgs a)
{
    constexpr int WAVES_N = KS > 1 ? 1 : 4;           // KS > 1: the wavefronts of a workgroup share a tile and split its K
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const uint32_t lb = emb_xcd_block(blockIdx.x, gridDim.x);
    const int64_t tile = lb;
    if (tile >= a.tiles_m * a.tiles_n) return;        // (the grid is rounded up to whole dies) uniform
    const int64_t tn = tile / a.tiles_m, tm = tile - tn * a.tiles_m;
    const int64_t m0 = tm * (16 * MT), n0 = (tn * WAVES_N + (KS > 1 ? 0 : wave)) * (16 * NT);
    const int nb = a.D / 32, supers = (nb + 15) / 16;

    const char *wp[NT], *xp[MT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {                    // rows past the end: the last row, not stored
        const int64_t n = n0 + 16 * t + r;
        wp[t] = a.w + (n < a.N ? n : a.N - 1) * a.w_pitch;
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t m = m0 + 16 * t + r;
        xp[t] = a.x + (m < a.M ? m : a.M - 1) * a.x_pitch;
    }
    mx_f4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = mx_f4{0.f, 0.f, 0.f, 0.f};

    for (int sup = KS > 1 ? wave : 0; sup < supers; sup += KS) {
        uint4 wc[NT][4], ws[NT];
        uint4 xc[XT == X_MXFP4 ? MT : 1][4], xs[XT == X_MXFP4 ? MT : 1];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            ws[t] = load_chunk(wp[t] + a.D / 2 + sup * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int b = sup * 16 + 4 * j + g;
                wc[t][j] = make_uint4(0, 0, 0, 0);
                if (b < nb) wc[t][j] = load_chunk(wp[t] + b * 16);
            }
        }
        if constexpr (XT == X_MXFP4) {
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                xs[t] = load_chunk(xp[t] + a.D / 2 + sup * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int b = sup * 16 + 4 * j + g;
                    xc[t][j] = make_uint4(0, 0, 0, 0);
                    if (b < nb) xc[t][j] = load_chunk(xp[t] + b * 16);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int b = sup * 16 + 4 * j + g;
            if (sup * 16 + 4 * j >= nb) break;        // uniform
            const bool in = b < nb;                   // blocks past the row: codes 0, a scale that is a number
            if constexpr (XT == X_MXFP4) {
                int wscale[NT], xscale[MT];
#pragma unroll
                for (int t = 0; t < NT; ++t) wscale[t] = in ? (int)((word_of(ws[t], j) >> (8 * g)) & 255u) : 127;
#pragma unroll
                for (int t = 0; t < MT; ++t) xscale[t] = in ? (int)((word_of(xs[t], j) >> (8 * g)) & 255u) : 127;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(wc[t][j]), mx_operand(xc[i][j]),
                                                                                    acc[i][t], 4, 4, 0, wscale[t], 0, xscale[i]);
            } else {
                float wscale[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) wscale[t] = __uint_as_float(in ? ((word_of(ws[t], j) >> (8 * g)) & 255u) << 23 : 127u << 23);
#pragma unroll
                for (int q = 0; q < 4; ++q) {         // 8 of the block's elements
                    constexpr int PARTS = XT == X_F32 ? 3 : 1;
                    mx_b8 xb[MT][PARTS];
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        if constexpr (XT == X_F32) {
                            uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
                            if (in) {
                                lo = load_chunk(xp[i] + (int64_t)b * 128 + q * 32);
                                hi = load_chunk(xp[i] + (int64_t)b * 128 + q * 32 + 16);
                            }
                            mx_b8 p[3];
                            split_bf16(lo, hi, p);
#pragma unroll
                            for (int k = 0; k < PARTS; ++k) xb[i][k] = p[k];
                        } else {
                            uint4 v = make_uint4(0, 0, 0, 0);
                            if (in) v = load_chunk(xp[i] + (int64_t)b * 64 + q * 16);
                            xb[i][0] = __builtin_bit_cast(mx_b8, v);
                        }
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const mx_b8 wb = codes_to_bf16(word_of(wc[t][j], q), wscale[t]);
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int k = PARTS - 1; k >= 0; --k)
                                acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, xb[i][k], acc[i][t], 0, 0, 0);
                    }
                }
            }
        }
    }

    if constexpr (KS > 1) {   // the wavefronts' sums, added in their order
        __shared__ mx_f4 part[KS - 1][MT * NT][64];
        if (wave > 0) {
#pragma unroll
            for (int i = 0; i < MT * NT; ++i) part[wave - 1][i][lane] = acc[i / NT][i % NT];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int k = 0; k < KS - 1; ++k)
#pragma unroll
            for (int i = 0; i < MT * NT; ++i) acc[i / NT][i % NT] += part[k][i][lane];
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = m0 + 16 * i + r;
        if (m >= a.M) continue;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int64_t n = n0 + 16 * t + 4 * g;
            if constexpr (OUT_BF16) {
                __bf16 *o = reinterpret_cast<__bf16 *>(a.out) + m * a.out_stride + n;
                const mx_b4_any v = {(__bf16)acc[i][t][0], (__bf16)acc[i][t][1], (__bf16)acc[i][t][2], (__bf16)acc[i][t][3]};
                if (n + 4 <= a.N) {
                    *reinterpret_cast<mx_b4_any *>(o) = v;
                } else {
                    for (int k = 0; k < 4; ++k)
                        if (n + k < a.N) o[k] = (__bf16)acc[i][t][k];
                }
            } else {
                float *o = reinterpret_cast<float *>(a.out) + m * a.out_stride + n;
                if (n + 4 <= a.N) {
                    *reinterpret_cast<mx_f4_any *>(o) = acc[i][t];
                } else {
                    for (int k = 0; k < 4; ++k)
                        if (n + k < a.N) o[k] = acc[i][t][k];
                }
            }
        }
    }
}

template <int XT, int MT, int NT, int KS, bool OUT_BF16>
int launch_direct(ProductArgs a, hipStream_t s)
{
    a.tiles_m = (a.M + 16 * MT - 1) / (16 * MT);
    const int64_t cols = 16 * NT * (KS > 1 ? 1 : 4);
    a.tiles_n = (a.N + cols - 1) / cols;
    if (a.tiles_n > (int64_t)0x7FFFFF00 / a.tiles_m) return EMB_ERR_UNSUPPORTED;
    const int64_t blocks = emb_round_up_xcds(a.tiles_m * a.tiles_n);
    hipLaunchKernelGGL((product_direct_kernel<XT, MT, NT, KS, OUT_BF16>), dim3((unsigned)blocks), dim3(KS > 1 ? 64 * KS : 256), 0, s, a);
    return EMB_OK;
}

template <int XT, bool OUT_BF16>
int dispatch_product(const ProductArgs &a, hipStream_t s)
{
    // With few tiles the chip is not filled: the wavefronts of a workgroup then split a tile's K.
    const bool few = (a.M + 15) / 16 * ((a.N + 31) / 32) < 2048 && a.D > 512;
    if (a.M <= 16 || few) {
        if (few) return launch_direct<XT, 1, 2, 8, OUT_BF16>(a, s);
        return launch_direct<XT, 1, 2, 1, OUT_BF16>(a, s);
    }
    if (a.M <= 32) return launch_direct<XT, 2, 2, 1, OUT_BF16>(a, s);
    return launch_direct<XT, 4, 4, 1, OUT_BF16>(a, s);
}

}  // namespace

extern "C" int emb_rows_product(const void *x_dev, int32_t x_dtype, int64_t x_stride, int64_t M, const void *w_rows_dev, int64_t N,
                                int32_t D, void *out_dev, int32_t out_dtype, int64_t out_stride, void *stream)
{
    if (M < 0 || N < 0) return EMB_ERR_INVALID_ARG;
    const int rc = emb_check_quant_rows(D, EMB_MXFP4);
    if (rc != EMB_OK) return rc;
    if (x_dtype != EMB_F32 && x_dtype != EMB_BF16 && x_dtype != EMB_MXFP4) return EMB_ERR_INVALID_ARG;
    if (out_dtype != EMB_F32 && out_dtype != EMB_BF16) return EMB_ERR_INVALID_ARG;
    const int64_t row = emb_row_bytes(D, EMB_MXFP4), esz = emb_elem_size(x_dtype);
    int64_t x_pitch = row;
    if (x_dtype != EMB_MXFP4) {
        if (x_stride < D || x_stride > INT64_MAX / 16 || x_stride * esz % 16 != 0) return EMB_ERR_INVALID_ARG;
        x_pitch = x_stride * esz;
    }
    if (out_stride < N) return EMB_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return EMB_OK;
    if (!x_dev || !w_rows_dev || !out_dev) return EMB_ERR_INVALID_ARG;
    if (!emb_aligned(x_dev, 16) || !emb_aligned(w_rows_dev, 16) || !emb_aligned(out_dev, emb_elem_size(out_dtype))) return EMB_ERR_INVALID_ARG;
    if (M > (int64_t)0x7FFFFFFF || N > (int64_t)0x7FFFFFFF) return EMB_ERR_UNSUPPORTED;
    const ProductArgs a{static_cast<const char *>(x_dev), static_cast<const char *>(w_rows_dev), x_pitch, row, M, N, D,
                        static_cast<char *>(out_dev), out_stride, 0, 0};
    hipStream_t s = emb_stream(stream);
    const bool b = out_dtype == EMB_BF16;
    int e;
    switch (x_dtype) {
        case EMB_MXFP4: e = b ? dispatch_product<X_MXFP4, true>(a, s) : dispatch_product<X_MXFP4, false>(a, s); break;
        case EMB_BF16: e = b ? dispatch_product<X_BF16, true>(a, s) : dispatch_product<X_BF16, false>(a, s); break;
        default: e = b ? dispatch_product<X_F32, true>(a, s) : dispatch_product<X_F32, false>(a, s);
    }
    if (e != EMB_OK) return e;
    EMB_RETURN_IF_LAUNCH_FAILED();
    return EMB_OK;
}
