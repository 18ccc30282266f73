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
// (Infinite elements of W are for mend_infinite_rows.)
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
typedef __bf16 mx_b8_any __attribute__((ext_vector_type(8), aligned(2)));

enum { X_MXFP4 = 0, X_BF16 = 1, X_F32 = 2 };

struct ProductArgs {
    const char *x, *w;
    int64_t x_pitch, w_pitch;      // bytes
    int64_t M, N;
    int32_t D;
    char *out;
    int64_t out_stride;            // elements
    int64_t tiles_m, tiles_n;      // workgroup tiles
    uint32_t die_rows;             // rows of dies that share them: 1, 2, 4 or 8
    uint32_t early;                // W's rows are asked for before the scores are written (early_rows)
};

__device__ __forceinline__ mx_i8 mx_operand(const uint4 &v)
{
    return mx_i8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
}

__device__ __forceinline__ uint32_t word_of(const uint4 &v, int j) { return j == 0 ? v.x : (j == 1 ? v.y : (j == 2 ? v.z : v.w)); }

// The unit's tiles take W's rows in an order that makes a lane's results 16 neighbouring bytes of the output and those of
// its four lane groups 64: for fp32 the rows' own, for bf16 place 16 * (2 * j + t) + 4 * a + b is row 32 * j + 4 * (2 * a + t) + b, so
// that two tiles end as 8 neighbouring n.  (Pieces of 16 bytes that only the L2 joins cost more the larger the output:
// 512 x 400000 x 128 to fp32 270 us, so 189.)
template <bool OUT_BF16>
constexpr int TILES = OUT_BF16 ? 2 : 1;   // that a store takes together
template <bool OUT_BF16>
__device__ __forceinline__ int w_row_at(int place)
{
    return OUT_BF16 ? (place & ~31) | ((place & 12) << 1) | ((place & 16) >> 2) | (place & 3) : place;
}

// 4 * V neighbouring elements of a row of the output, v[0] the first four.
template <int V, bool OUT_BF16>
__device__ __forceinline__ void store_run(char *out, int64_t row, int64_t n, int64_t N, const mx_f4 (&v)[V])
{
    if constexpr (OUT_BF16) {
        __bf16 *o = reinterpret_cast<__bf16 *>(out) + row + n;
#pragma unroll
        for (int h = 0; h < V / 2; ++h) {
            mx_b8_any b;
#pragma unroll
            for (int k = 0; k < 8; ++k) b[k] = (__bf16)v[2 * h + k / 4][k % 4];
            if (n + 8 * h + 8 <= N) {
                *reinterpret_cast<mx_b8_any *>(o + 8 * h) = b;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (n + 8 * h + k < N) o[8 * h + k] = b[k];
            }
        }
    } else {
        float *o = reinterpret_cast<float *>(out) + row + n;
#pragma unroll
        for (int t = 0; t < V; ++t) {
            if (n + 4 * t + 4 <= N) {
                *reinterpret_cast<mx_f4_any *>(o + 4 * t) = v[t];
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (n + 4 * t + k < N) o[4 * t + k] = v[t][k];
            }
        }
    }
}

// A lane's results for row m of x: NT tiles whose first place is n0.
template <int NT, bool OUT_BF16>
__device__ __forceinline__ void store_tiles(const ProductArgs &a, int64_t m, int64_t n0, int g, const mx_f4 (&v)[NT])
{
    constexpr int V = TILES<OUT_BF16>;
    static_assert(NT % V == 0, "whole stores");
    if (m >= a.M) return;
#pragma unroll
    for (int j = 0; j < NT / V; ++j)
        store_run<V, OUT_BF16>(a.out, m * a.out_stride, n0 + 16 * V * j + 4 * V * g, a.N, reinterpret_cast<const mx_f4(&)[V]>(v[V * j]));
}

// 8 codes of one word, by their block's power of two, as bf16 (exact)
__device__ __forceinline__ mx_b8 codes_to_bf16(uint32_t w, float scale)
{
    const emb_b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const emb_b2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return mx_b8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// Eight fp32 values as three bf16 parts: the upper 8 bits of the significand, the 8 after them and the last 8, all cut off, not
// rounded.  An infinity is the first part alone; of a NaN the other parts are NaN, wherever its mark is.
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }
__device__ __forceinline__ void split_bf16(const uint4 &a, const uint4 &b, mx_b8 (&p)[3])
{
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t mid[8], low[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float f = __uint_as_float(w[i]), r = f - __uint_as_float(w[i] & 0xFFFF0000u);
        mid[i] = __builtin_fabsf(f) == __builtin_inff() ? 0u : __float_as_uint(r);
        low[i] = __float_as_uint(__uint_as_float(mid[i]) - __uint_as_float(mid[i] & 0xFFFF0000u));
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const uint32_t(&from)[8] = k == 0 ? w : (k == 1 ? mid : low);
        p[k] = __builtin_bit_cast(mx_b8, make_uint4(upper_halves(from[0], from[1]), upper_halves(from[2], from[3]),
                                                    upper_halves(from[4], from[5]), upper_halves(from[6], from[7])));
    }
}

// Rows of W with infinite elements (under a scale byte of 253 or 254: 4 and 6 by 2^126, 2 to 6 by 2^127; the quantisers here
// write none) and an fp32 x.  A part of x that is zero makes NaN of an infinity, where fp32 has the infinity that the other parts
// make of it (theirs have the same sign, so nothing but NaN is ever wrong).  So a lane with a NaN among its sums makes
// that of a row with such bytes once more, an element of x at a time.  (Looking at the sums at the end of a tile takes up to 1 %; a
// maximum of the scale bytes kept along the way took 2 to 3 % of 4096 x 4096 x 1024.  16 x 100003 x 2048: 46 us, with a NaN in x 67, with a
// row of infinities in W 89; one of NaN 45.)
template <bool OUT_BF16>
__device__ __forceinline__ void redo_infinite_row(const ProductArgs &a, int64_t m, int64_t n)
{
    const char *const w = a.w + n * a.w_pitch, *const scales = w + a.D / 2, *const x = a.x + m * a.x_pitch;
    bool infinite = false;                             // (or not even so: a byte of the padding)
    for (int b = 0; b < a.D / 32; b += 16) {
        const uint4 v = load_chunk(scales + b);
#pragma unroll
        for (int k = 0; k < 16; ++k) infinite |= ((word_of(v, k / 4) >> (8 * (k % 4))) & 255u) - 253u < 2u;
    }
    if (!infinite) return;
    float sum = 0.f;
    for (int c = 0; c < a.D / 4; ++c) {                // 4 elements
        const uint32_t codes = *(const EMB_GLOBAL uint16_t *)(w + 2 * c), byte = *(const EMB_GLOBAL uint8_t *)(scales + c / 8);
        const float scale = __uint_as_float(byte << 23);
        const emb_f2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
        const uint4 v = load_chunk(x + 16 * c);
        sum = __builtin_fmaf(__uint_as_float(v.x), lo.x, sum);
        sum = __builtin_fmaf(__uint_as_float(v.y), lo.y, sum);
        sum = __builtin_fmaf(__uint_as_float(v.z), hi.x, sum);
        sum = __builtin_fmaf(__uint_as_float(v.w), hi.y, sum);
    }
    if (OUT_BF16) reinterpret_cast<__bf16 *>(a.out)[m * a.out_stride + n] = (__bf16)sum;
    else reinterpret_cast<float *>(a.out)[m * a.out_stride + n] = sum;
}
// acc: the lane's sums of rows m0 + 16 * i + r of x, tiles from place n0 on, which it has stored.
template <int XT, bool OUT_BF16, int MT, int NT>
__device__ __forceinline__ void mend_infinite_rows(const ProductArgs &a, int64_t m0, int64_t n0, int r, int g, const mx_f4 (&acc)[MT][NT])
{
    if constexpr (XT == X_F32) {
        static_assert(MT * NT <= 16, "a bit a sum");
        constexpr int V = NT % TILES<OUT_BF16> == 0 ? TILES<OUT_BF16> : 1;   // as in store_tiles
        bool any = false;
#pragma unroll
        for (int i = 0; i < MT * NT; ++i) {            // (two sums a comparison)
            const mx_f4 v = acc[i / NT][i % NT];
            any |= __builtin_isunordered(v[0], v[1]) | __builtin_isunordered(v[2], v[3]);
        }
        if (!any) return;
        uint64_t nan = 0;
#pragma unroll
        for (int i = 0; i < 4 * MT * NT; ++i) {
            const float v = acc[i / 4 / NT][i / 4 % NT][i % 4];
            if (v != v) nan |= UINT64_C(1) << i;
        }
        for (; nan; nan &= nan - 1) {
            const int i = __ffsll((unsigned long long)nan) - 1, t = i / 4 % NT;
            const int64_t m = m0 + 16 * (i / 4 / NT) + r, n = n0 + 16 * V * (t / V) + 4 * V * g + 4 * (t % V) + i % 4;
            if (m < a.M && n < a.N) redo_infinite_row<OUT_BF16>(a, m, n);
        }
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
        const int64_t n = n0 + (NT % TILES<OUT_BF16> == 0 ? w_row_at<OUT_BF16>(16 * t + r) : 16 * t + r);
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
        if constexpr (NT % TILES<OUT_BF16> == 0) {
            store_tiles<NT, OUT_BF16>(a, m0 + 16 * i + r, n0, g, acc[i]);
        } else if (m0 + 16 * i + r < a.M) {               // a single tile to bf16
            __bf16 *o = reinterpret_cast<__bf16 *>(a.out) + (m0 + 16 * i + r) * a.out_stride + n0 + 4 * g;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (n0 + 4 * g + k < a.N) o[k] = (__bf16)acc[i][0][k];
        }
    }
    mend_infinite_rows<XT, OUT_BF16>(a, m0, n0, r, g, acc);
}

// A grid holds fewer than 2^32 threads.
inline bool fits_a_grid(int64_t blocks, int64_t threads) { return blocks <= (int64_t)0xFFFFFFFF / threads; }

template <int XT, int MT, int NT, int KS, bool OUT_BF16>
int launch_direct(ProductArgs a, hipStream_t s)
{
    a.tiles_m = (a.M + 16 * MT - 1) / (16 * MT);
    const int64_t cols = 16 * NT * (KS > 1 ? 1 : 4);
    a.tiles_n = (a.N + cols - 1) / cols;
    if (a.tiles_n > (int64_t)0x7FFFFF00 / a.tiles_m) return EMB_ERR_UNSUPPORTED;
    const int64_t blocks = emb_round_up_xcds(a.tiles_m * a.tiles_n);
    if (!fits_a_grid(blocks, KS > 1 ? 64 * KS : 256)) return EMB_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((product_direct_kernel<XT, MT, NT, KS, OUT_BF16>), dim3((unsigned)blocks), dim3(KS > 1 ? 64 * KS : 256), 0, s, a);
    return EMB_OK;
}

// ---------------------------------------------------------------------------
// tiles in LDS
// ---------------------------------------------------------------------------
// Both operands MXFP4: a workgroup makes a tile of 256 x 256 (8 wavefronts of 128 x 64) or, where those would not fill the
// chip, 128 x 128 (4 of 64 x 64), from stages of 256 elements that go straight to LDS, two buffers in turn, the next stage's chunks
// requested one at a time between groups of this one's products (all ahead of them: 209 us for 8192 x 8192 x 4096, so 150 to 162, 3.4 to
// 3.7 PFLOP/s).  What bounds it: 4096 x 4096 x 16384 takes 138 us, without the requests 110, without LDS reads either 104, and as many
// products from registers alone 77 (the card's power: 57 on zeros); the stores of a round of tiles take 7.  A ring of four stages of half
// the length, requested three stages ahead, was slower (4096 x 4096 x 4096 54 us and 39): shorter pieces of rows cost more than the waits.
#define EMB_LDS __attribute__((address_space(3)))
typedef uint32_t mx_u4 __attribute__((ext_vector_type(4)));

// 256 elements of a row are 8 chunks of 16 bytes; a tile keeps them in 128 bytes a row, chunk c at place c ^ key(row).  LDS
// serves a 16-byte read 16 lanes at a time, of which 8 are of one lane group (rows 0-3 and 12-15 of a tile, or 4-11) and 8 of
// its neighbour (the other rows): groups that read neighbouring chunks then find 16 different places of 256 bytes.
// W's rows stand there in the order of the unit's tiles (w_row_at).
__device__ __forceinline__ int key_of(int place) { return (place >> 1) & 7; }

constexpr int STAGE_CHUNKS = 8;

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// The tile of a workgroup, if it has one.  The dies share the tiles as a grid of die_rows x 8 / die_rows, so that a die's L2 holds
// few panels of either operand; within its part a die goes row by row through strips of 8 columns.  (The quotients come from
// the vector unit: told to be uniform, so that addresses are scalar bases and 32-bit offsets.)
__device__ __forceinline__ bool tile_of(const ProductArgs &a, uint32_t &tm, uint32_t &tn)
{
    const uint32_t die = blockIdx.x % EMB_XCDS, i = blockIdx.x / EMB_XCDS, tiles_m = (uint32_t)a.tiles_m, tiles_n = (uint32_t)a.tiles_n;
    const uint32_t die_cols = EMB_XCDS / a.die_rows, high = uniform((tiles_m + a.die_rows - 1) / a.die_rows),
                   wide = uniform((tiles_n + die_cols - 1) / die_cols);
    const uint32_t row0 = die % a.die_rows * high, col0 = die / a.die_rows * wide;
    const uint32_t strip = uniform(i / (8 * high)), in_strip = i - strip * 8 * high;
    const uint32_t columns = wide - strip * 8 < 8 ? wide - strip * 8 : 8;
    const uint32_t row = uniform(in_strip / columns);
    tm = row0 + row;
    tn = col0 + strip * 8 + in_strip - row * columns;
    return tm < tiles_m && tn < tiles_n;
}

// Short rows make much more output than input, and reads of W that trickle in between the writes slow both.  So a die's first
// workgroups, one for each of its CUs, read its part of W at once (a word of every line, to no use), which brings it to the memory-side cache: with W
// in HBM 512 x 200000 x 128 from MXFP4 67 us, so 47; with W in the cache already 42.5 and 44.  A larger W is out of that cache again
// before it is used, and is read twice: 128 x 600000 x 128 (48 MB) 55 us, so 47; 128 x 1200000 x 64 (58 MB) 100 and 95; 512 x 800000 x 128
// (64 MB) 251 and 260; 128 x 1000000 x 128 (80 MB) 87 and 94; 128 x 4000000 x 128 (320 MB) 347 and 409.  So up to MOST_EARLY bytes of it.
constexpr int64_t MOST_EARLY = 48 << 20;
template <int BN, int THREADS>
__device__ __forceinline__ uint32_t early_rows(const ProductArgs &a)
{
    constexpr uint32_t FIRST = 32;
    const uint32_t die = blockIdx.x % EMB_XCDS, i = blockIdx.x / EMB_XCDS, die_cols = EMB_XCDS / a.die_rows;
    uint32_t seen = 0;
    if (a.early && i < FIRST) {   // uniform
        const int64_t part = (a.tiles_n + die_cols - 1) / die_cols * BN * a.w_pitch, from = die / a.die_rows * part;
        const int64_t to = from + part < a.N * a.w_pitch ? from + part : a.N * a.w_pitch;
        for (int64_t at = from + ((int64_t)i * THREADS + threadIdx.x) * 128; at < to; at += (int64_t)FIRST * THREADS * 128)
            seen ^= *(const EMB_GLOBAL uint32_t *)(a.w + at);
    }
    return seen;
}
__device__ __forceinline__ void use(uint32_t seen) { asm volatile("" ::"v"(seen)); }

// One operand's rows of a tile, seen as a buffer that begins with the tile's first row: 32-bit offsets, the stage's in a scalar,
// and what lies beyond its end reads as zero, which is where the chunks are sent that the last stage does not have.
constexpr uint32_t BUFFER_END = 1u << 30, BEYOND = 1u << 31;
constexpr int64_t MOST_PITCH = 1 << 22;    // of rows of x that are tiled: 128 of them end below BUFFER_END, as 256 MXFP4 rows do (34816 bytes)

template <int ROWS, int THREADS, bool IS_W, bool OUT_BF16>
struct StageOperand {
    static constexpr int LOADS = ROWS * STAGE_CHUNKS / THREADS;
    __amdgpu_buffer_rsrc_t rows;
    uint32_t off[LOADS];       // of this thread's chunk of the row at place u * THREADS / 8 + threadIdx / 8
    __device__ __forceinline__ static int chunk(int u)
    {
        return (threadIdx.x % STAGE_CHUNKS) ^ key_of(u * (THREADS / STAGE_CHUNKS) + threadIdx.x / STAGE_CHUNKS);
    }
    // have: how many rows there are (the others repeat the last)
    __device__ __forceinline__ void init(const char *base, int64_t have, int64_t pitch)
    {
        rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, BUFFER_END, 0x00020000);
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int place = u * (THREADS / STAGE_CHUNKS) + threadIdx.x / STAGE_CHUNKS, row = IS_W ? w_row_at<OUT_BF16>(place) : place;
            off[u] = __umul24((uint32_t)(row < have ? row : (int)have - 1), (uint32_t)pitch) + 16u * (uint32_t)chunk(u);
        }
    }
    // Chunks of a stage straight to LDS; the row still has `valid` of them.
    __device__ __forceinline__ void load(int u, int stage, char *lds, int valid) const
    {
        const uint32_t at = chunk(u) < valid ? off[u] : BEYOND;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (EMB_LDS void *)(lds + (u * THREADS + (threadIdx.x & ~63u)) * 16), 16, (int)at,
                                                 stage * (STAGE_CHUNKS * 16), 0, 0);
    }
};

// ONE: D is at most 128.
template <int WM, int WN, int MT, bool ONE, bool OUT_BF16>
__global__ __launch_bounds__(64 * WM * WN) void product_tiled_kernel(ProductArgs a)
{
    constexpr int NT = 4, THREADS = 64 * WM * WN, BM = WM * MT * 16, BN = WN * 64;
    static_assert(BM + BN == THREADS, "a thread fetches one row's scales");
    __shared__ __attribute__((aligned(16))) char x0[BM * 128], x1[BM * 128], w0[BN * 128], w1[BN * 128];
    __shared__ __attribute__((aligned(16))) uint16_t s0[THREADS * 4], s1[THREADS * 4];   // scales of a stage: x's rows, then W's
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
    const int wm = wave % WM, wn = wave / WM;
    uint32_t tm, tn, seen = 0;
    if constexpr (ONE) seen = early_rows<BN, THREADS>(a);
    if (!tile_of(a, tm, tn)) return;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const char *xbase = a.x + m0 * a.x_pitch, *wbase = a.w + n0 * a.w_pitch;
    const int64_t xrows = a.M - m0, wrows = a.N - n0;
    const int nb = a.D / 32, stages = (nb + STAGE_CHUNKS - 1) / STAGE_CHUNKS, last = nb - (stages - 1) * STAGE_CHUNKS;

    StageOperand<BM, THREADS, false, OUT_BF16> xo;
    StageOperand<BN, THREADS, true, OUT_BF16> wo;
    xo.init(xbase, xrows < BM ? xrows : BM, a.x_pitch);
    wo.init(wbase, wrows < BN ? wrows : BN, a.w_pitch);
    const char *srow;                                 // the scales that this thread fetches
    {
        const int64_t have = tid < BM ? xrows : wrows;
        int64_t row = tid < BM ? tid : w_row_at<OUT_BF16>(tid - BM);
        if (row >= have) row = have - 1;
        srow = (tid < BM ? xbase + row * a.x_pitch : wbase + row * a.w_pitch) + a.D / 2;
    }
    // the lane's first place in either tile; its others lie 16 places on, with the same key
    const int xrow0 = wm * MT * 16 + r, wrow0 = wn * 64 + r, key = key_of(r);
    uint2 sc;
    mx_f4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = mx_f4{0.f, 0.f, 0.f, 0.f};

    // (A stage past the last one reads nothing: the loop below stays one block of instructions, out of which the compiler
    // moves no MFMA.)
    auto fetch_scales = [&](int st) { sc = load_u2(srow + (st < stages ? st : stages - 1) * STAGE_CHUNKS); };
    auto fetch_part = [&](int part, int st, char *xl, char *wl) {
        if (part < xo.LOADS) xo.load(part, st, xl, nb - st * STAGE_CHUNKS);
        else wo.load(part - xo.LOADS, st, wl, nb - st * STAGE_CHUNKS);
    };
    constexpr int PARTS = (BM + BN) * STAGE_CHUNKS / THREADS;
    auto fetch = [&](int st, char *xl, char *wl) {
        fetch_scales(st);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) fetch_part(k, st, xl, wl);
    };
    // Scales in LDS: 16 bytes for a pair of the unit's tiles and a row of them, 4 for each lane group: its two blocks in the
    // first tile, then in the second.  One read gives a lane the scales of two tiles and both steps.
    int splace;
    {
        const int place = tid < BM ? tid : tid - BM;
        splace = (tid < BM ? 0 : BM * 4) + ((place >> 5) * 16 + (place & 15)) * 8 + ((place >> 4) & 1);
    }
    auto ready = [&](int st, uint16_t *sl) {
        __builtin_amdgcn_s_waitcnt(0x0F70);           // vmcnt(0): this thread's chunks of the stage are in LDS
        uint64_t v = (uint64_t)sc.y << 32 | sc.x;
        if (st + 1 == stages && last < STAGE_CHUNKS) {   // blocks past the row: a scale that is a number
            const uint64_t keep = (1ull << (8 * last)) - 1;
            v = (v & keep) | (0x7F7F7F7F7F7F7F7Full & ~keep);
        }
        const uint32_t lo = __builtin_amdgcn_perm((uint32_t)(v >> 32), (uint32_t)v, 0x05010400u),   // bytes 0 4 1 5
                       hi = __builtin_amdgcn_perm((uint32_t)(v >> 32), (uint32_t)v, 0x07030602u);   // 2 6 3 7
        sl[splace] = (uint16_t)lo;
        sl[splace + 2] = (uint16_t)(lo >> 16);
        sl[splace + 4] = (uint16_t)hi;
        sl[splace + 6] = (uint16_t)(hi >> 16);
        __syncthreads();                              // everyone's are, and nobody reads the other buffer any more
    };
    // One stage is two steps of the matrix unit: lane group g takes chunk g, then 4 + g, whose scale bytes lie side by side in
    // LDS.  Rows of at most 4 chunks are one step.
    auto compute = [&](const char *xl, const char *wl, const uint16_t *sl, int next, char *xnext, char *wnext) {
        constexpr bool HALF = ONE;
        const char *sx = reinterpret_cast<const char *>(sl) + (wm * (MT / 2) * 16 + r) * 16 + g * 4;
        const char *sw = reinterpret_cast<const char *>(sl) + BM * 8 + (wn * (NT / 2) * 16 + r) * 16 + g * 4;
        int xs[MT / 2], ws[NT / 2];                   // bytes: first tile, step 0 and 1; second tile
#pragma unroll
        for (int i = 0; i < MT / 2; ++i) xs[i] = *reinterpret_cast<const int *>(sx + i * 256);
#pragma unroll
        for (int t = 0; t < NT / 2; ++t) ws[t] = *reinterpret_cast<const int *>(sw + t * 256);
        // Reads run one group of MFMA ahead: 2 of x's tiles by 4 of W's, 128 cycles of the matrix unit.
        constexpr int XG = 2, PER_STEP = MT / XG, GROUPS = PER_STEP * (HALF ? 1 : 2);
        mx_u4 xv[2][XG], wv[2][NT];
        auto read_w = [&](int step) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
                wv[step][t] = *reinterpret_cast<const mx_u4 *>(wl + wrow0 * 128 + (((4 * step + g) ^ key) * 16) + t * 2048);
        };
        auto read_x = [&](int q) {
#pragma unroll
            for (int i = 0; i < XG; ++i)
                xv[q & 1][i] = *reinterpret_cast<const mx_u4 *>(xl + xrow0 * 128 + (((4 * (q / PER_STEP) + g) ^ key) * 16) +
                                                                ((q % PER_STEP) * XG + i) * 2048);
        };
        read_w(0);
        read_x(0);
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) {
            const int step = q / PER_STEP, i0 = (q % PER_STEP) * XG;
            if (!HALF && q == 0) read_w(1);
            if (q + 1 < GROUPS) read_x(q + 1);
            if (!HALF) {                              // the next stage's chunks, spread over this one's products
                if (q == 0) fetch_scales(next);
#pragma unroll
                for (int k = q * PARTS / GROUPS; k < (q + 1) * PARTS / GROUPS; ++k) fetch_part(k, next, xnext, wnext);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < XG; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const mx_u4 w = wv[step][t], x = xv[q & 1][i];
                    const mx_i8 wa = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
                    const mx_i8 xa = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
#define EMB_MFMA(WB, XB)                                                                                                    \
    acc[i0 + i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, xa, acc[i0 + i][t], 4, 4, WB, ws[t / 2], XB, xs[(i0 + i) / 2])
                    if (step == 0) {
                        if (t % 2 == 0) { if (i % 2 == 0) EMB_MFMA(0, 0); else EMB_MFMA(0, 2); }
                        else { if (i % 2 == 0) EMB_MFMA(2, 0); else EMB_MFMA(2, 2); }
                    } else {
                        if (t % 2 == 0) { if (i % 2 == 0) EMB_MFMA(1, 1); else EMB_MFMA(1, 3); }
                        else { if (i % 2 == 0) EMB_MFMA(3, 1); else EMB_MFMA(3, 3); }
                    }
#undef EMB_MFMA
                }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if constexpr (ONE) {
        fetch(0, x0, w0);
        use(seen);
        ready(0, s0);
        compute(x0, w0, s0, 0, x0, w0);
    } else {
        // Two buffers, of different names so that the compiler sees that what is fetched into one is not read from the other.
        int st = 0;
        if (stages & 1) {
            fetch(0, x1, w1);
            ready(0, s1);
            compute(x1, w1, s1, 1, x0, w0);
            st = 1;
        } else {
            fetch(0, x0, w0);
        }
        for (; st < stages; st += 2) {
            ready(st, s0);
            compute(x0, w0, s0, st + 1, x1, w1);
            ready(st + 1, s1);
            compute(x1, w1, s1, st + 2, x0, w0);
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);           // nothing is on its way to LDS when the workgroup ends
    }

#pragma unroll
    for (int i = 0; i < MT; ++i) {
        store_tiles<NT, OUT_BF16>(a, m0 + wm * MT * 16 + 16 * i + r, n0 + wn * 64, g, acc[i]);
    }
}

// The dies' part of the tiles: of the four ways to share them the one whose largest part is smallest, of equals the one with
// the fewest rows and columns in a part.  Returns the workgroups of the launch.
inline int64_t share_tiles(ProductArgs &a, int64_t bm, int64_t bn)
{
    a.tiles_m = (a.M + bm - 1) / bm;
    a.tiles_n = (a.N + bn - 1) / bn;
    int64_t best = INT64_MAX, around = 0;
    for (uint32_t rows = 1; rows <= EMB_XCDS; rows *= 2) {
        const int64_t high = (a.tiles_m + rows - 1) / rows, wide = (a.tiles_n + EMB_XCDS / rows - 1) / (EMB_XCDS / rows);
        if (high * wide < best || (high * wide == best && high + wide < around)) {
            best = high * wide;
            around = high + wide;
            a.die_rows = rows;
        }
    }
    // (a die holds up to 128 workgroups at once: fewer read W at once anyway)
    a.early = a.D <= 128 && best > 128 && a.N * a.w_pitch <= MOST_EARLY;
    return best * EMB_XCDS;
}

template <int WM, int WN, int MT, bool ONE, bool OUT_BF16>
int launch_tiled(ProductArgs a, hipStream_t s)
{
    const int64_t blocks = share_tiles(a, WM * MT * 16, WN * 64);
    if (!fits_a_grid(blocks, 64 * WM * WN)) return EMB_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((product_tiled_kernel<WM, WN, MT, ONE, OUT_BF16>), dim3((unsigned)blocks), dim3(64 * WM * WN), 0, s, a);
    return EMB_OK;
}

// x in bf16 or fp32: W's codes become bf16 in registers.  A stage is 256 bytes of a row of x (128 bf16 or 64 fp32 elements) and
// the 64 (32) bytes of codes that belong to them; scale bytes come from the row into a register, a stage ahead.  Lane group g
// takes the stage's elements from g * STAGE / 4 on, in steps of 8: chunk c of a row of x stands at place c ^ wide_key_x(row).
// Tiles are 128 x 128.  bf16: by wavefronts of 128 x 32, so that W's codes are widened once; two workgroups fill a CU's LDS
// exactly.  fp32: by wavefronts of 32 x 128, so that every element of x is split into its three parts once.
// 8192 x 8192 x 4096 bf16 1.0 PFLOP/s; 4096 x 4096 x 1024 bf16 38 us, fp32 122 to 144 by card: what keeps them from the matrix unit's rate is the vector
// work between its instructions (widening W; for fp32 six operations for an element's parts).
// Keys for rows of 256 bytes, chunks 4 apart in neighbouring lane groups, and of 64 bytes, chunks 1 apart.
__device__ __forceinline__ int wide_key_x(int row) { return (row & 3) | ((row >> 1) & 4) | (((row << 1) ^ row) & 8); }
__device__ __forceinline__ int wide_key_w(int row) { return ((row >> 1) & 2) ^ ((row >> 3) & 1) * 3; }
// HALF: tiles of 64 x 128, for few rows of x.
template <int XT, bool HALF, bool OUT_BF16>
__global__ __launch_bounds__(256, 2) void product_widened_kernel(ProductArgs a)
{
    constexpr bool F32 = XT == X_F32;
    constexpr int STAGE = F32 ? 64 : 128, WM = F32 ? 4 : 1, WN = F32 ? 1 : 4, MT = (F32 ? 2 : 8) / (HALF ? 2 : 1), NT = F32 ? 8 : 2;
    constexpr int BM = WM * MT * 16, BN = WN * NT * 16, THREADS = 256;
    constexpr int XC = 16, WC = STAGE / 32;                       // 16-byte chunks of a row in a stage
    constexpr int XL = BM * XC / THREADS, WL = BN * WC / THREADS; // that a thread fetches
    constexpr int STEPS = STAGE / 32, KPARTS = F32 ? 3 : 1;
    __shared__ __attribute__((aligned(16))) char x0[BM * 256], x1[BM * 256], w0[BN * WC * 16], w1[BN * WC * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
    const int wm = wave % WM, wn = wave / WM;
    uint32_t tm, tn;
    const uint32_t seen = early_rows<BN, THREADS>(a);
    if (!tile_of(a, tm, tn)) return;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int xhave = a.M - m0 < BM ? (int)(a.M - m0) : BM, whave = a.N - n0 < BN ? (int)(a.N - n0) : BN;
    const int nb = a.D / 32, stages = (a.D + STAGE - 1) / STAGE;
    const __amdgpu_buffer_rsrc_t xrows = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(a.x + m0 * a.x_pitch), 0, BUFFER_END, 0x00020000);
    const __amdgpu_buffer_rsrc_t wrows = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(a.w + n0 * a.w_pitch), 0, BUFFER_END, 0x00020000);

    uint32_t xoff[XL], woff[WL], soff[NT];
    const int xchunk = (tid % XC) ^ wide_key_x(tid / XC);            // (every row of this thread has the same place)
    auto wchunk = [&](int u) {
        const int place = (u * THREADS + tid) / WC;
        return (tid % WC) ^ (F32 ? (place >> 3) & 1 : wide_key_w(place));
    };
#pragma unroll
    for (int u = 0; u < XL; ++u) {
        const int row = u * (THREADS / XC) + tid / XC;
        xoff[u] = (uint32_t)(row < xhave ? row : xhave - 1) * (uint32_t)a.x_pitch + 16u * (uint32_t)xchunk;
    }
#pragma unroll
    for (int u = 0; u < WL; ++u) {
        const int row = w_row_at<OUT_BF16>((u * THREADS + tid) / WC);
        woff[u] = __umul24((uint32_t)(row < whave ? row : whave - 1), (uint32_t)a.w_pitch) + 16u * (uint32_t)wchunk(u);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = w_row_at<OUT_BF16>(wn * NT * 16 + 16 * t + r);
        soff[t] = __umul24((uint32_t)(row < whave ? row : whave - 1), (uint32_t)a.w_pitch) + (uint32_t)a.D / 2 + (uint32_t)(F32 ? g >> 1 : g);
    }
    uint32_t scale[NT], next_scale[NT];
    mx_f4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = mx_f4{0.f, 0.f, 0.f, 0.f};

    constexpr int PARTS = XL + WL;
    auto fetch_scales = [&](int st) {
        const int at = (st < stages ? st : stages - 1) * WC;
        const bool in = at + (F32 ? g >> 1 : g) < nb;             // a block past the row: a scale that is a number
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t b = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(wrows, (int)soff[t], at, 0);
            next_scale[t] = in ? b : 127u;
        }
    };
    auto fetch_part = [&](int part, int st, char *xl, char *wl) {
        if (part < XL) {
            const uint32_t at = xchunk < (a.D - st * STAGE) / (F32 ? 4 : 8) ? xoff[part] : BEYOND;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xrows, (EMB_LDS void *)(xl + (part * THREADS + (tid & ~63)) * 16), 16, (int)at, st * 256, 0, 0);
        } else {
            const int u = part - XL;
            const uint32_t at = wchunk(u) < nb - st * WC ? woff[u] : BEYOND;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wrows, (EMB_LDS void *)(wl + (u * THREADS + (tid & ~63)) * 16), 16, (int)at, st * WC * 16, 0, 0);
        }
    };
    const int xplace = (wm * MT * 16 + r) * 256, wplace = wn * NT * 16 + r;
    const int wkey = F32 ? (wplace >> 3) & 1 : wide_key_w(wplace), xkey = wide_key_x(r);
    auto compute = [&](const char *xl, const char *wl, int next, char *xnext, char *wnext) {
        // W's codes of the whole stage: 16 (8) bytes a row
        uint32_t code[NT][STEPS];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (F32) {
                const uint2 v = *reinterpret_cast<const uint2 *>(wl + (wplace + 16 * t) * 32 + (((g >> 1) ^ wkey) * 16) + (g & 1) * 8);
                code[t][0] = v.x;
                code[t][1] = v.y;
            } else {
                const mx_u4 v = *reinterpret_cast<const mx_u4 *>(wl + (wplace + 16 * t) * 64 + ((g ^ wkey) * 16));
#pragma unroll
                for (int k = 0; k < STEPS; ++k) code[t][k] = v[k];
            }
            scale[t] = next_scale[t];
        }
        // x's registers run one step ahead of the products
        mx_b8 xb[2][MT][KPARTS];
        uint4 raw[F32 ? MT : 1][2];
        auto read_x = [&](int k) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if constexpr (F32) {
                    raw[i][0] = *reinterpret_cast<const uint4 *>(xl + xplace + i * 4096 + (((4 * g + 2 * k) ^ xkey) * 16));
                    raw[i][1] = *reinterpret_cast<const uint4 *>(xl + xplace + i * 4096 + (((4 * g + 2 * k + 1) ^ xkey) * 16));
                } else {
                    xb[k & 1][i][0] = *reinterpret_cast<const mx_b8 *>(xl + xplace + i * 4096 + (((4 * g + k) ^ xkey) * 16));
                }
            }
        };
        auto split_x = [&](int k) {
            if constexpr (F32) {
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    mx_b8 p[3];
                    split_bf16(raw[i][0], raw[i][1], p);
#pragma unroll
                    for (int j = 0; j < KPARTS; ++j) xb[k & 1][i][j] = p[j];
                }
            }
        };
        read_x(0);
        split_x(0);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            if (k + 1 < STEPS) read_x(k + 1);
            if (k == 0) fetch_scales(next);
#pragma unroll
            for (int q = k * PARTS / STEPS; q < (k + 1) * PARTS / STEPS; ++q) fetch_part(q, next, xnext, wnext);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const mx_b8 wb = codes_to_bf16(code[t][k], __uint_as_float(scale[t] << 23));
#pragma unroll
                for (int j = KPARTS - 1; j >= 0; --j)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
                        acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, xb[k & 1][i][j], acc[i][t], 0, 0, 0);
            }
            if (k + 1 < STEPS) split_x(k + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto ready = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0F70);
        __syncthreads();
    };
    auto fetch = [&](int st, char *xl, char *wl) {
        fetch_scales(st);
#pragma unroll
        for (int q = 0; q < PARTS; ++q) fetch_part(q, st, xl, wl);
    };
    int st = 0;
    if (stages & 1) {
        fetch(0, x1, w1);
        use(seen);
        ready();
        compute(x1, w1, 1, x0, w0);
        st = 1;
    } else {
        fetch(0, x0, w0);
        use(seen);
    }
    for (; st < stages; st += 2) {
        ready();
        compute(x0, w0, st + 1, x1, w1);
        ready();
        compute(x1, w1, st + 2, x0, w0);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);               // nothing is on its way to LDS when the workgroup ends
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        store_tiles<NT, OUT_BF16>(a, m0 + wm * MT * 16 + 16 * i + r, n0 + wn * NT * 16, g, acc[i]);
    }
    mend_infinite_rows<XT, OUT_BF16>(a, m0 + wm * MT * 16, n0 + wn * NT * 16, r, g, acc);
}

template <int XT, bool HALF, bool OUT_BF16>
int launch_widened(ProductArgs a, hipStream_t s)
{
    const int64_t blocks = share_tiles(a, HALF ? 64 : 128, 128);
    if (!fits_a_grid(blocks, 256)) return EMB_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((product_widened_kernel<XT, HALF, OUT_BF16>), dim3((unsigned)blocks), dim3(256), 0, s, a);
    return EMB_OK;
}

// ---------------------------------------------------------------------------
// few rows of x in bf16 or fp32
// ---------------------------------------------------------------------------
// W passes through registers once, 32 rows a wavefront, and bounds it all; x stands in LDS, in bf16 parts, widened once by
// the workgroup, as much of K at a time as LDS_X holds (all of it for a single row of up to 8192 fp32 elements).  Rows of x
// lie a multiple of 256 bytes apart, 16-byte chunk c of row m at c ^ wide_key_x(m) within its 16.
constexpr int LDS_X = 49152;

template <int XT, int MT, bool OUT_BF16>
__global__ __launch_bounds__(256) void product_skinny_kernel(ProductArgs a, int rows, int kc)
{
    constexpr int NT = 2, KPARTS = XT == X_F32 ? 3 : 1, THREADS = 256;
    constexpr bool AHEAD = MT == 1;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
    const uint32_t tile = emb_xcd_block(blockIdx.x, gridDim.x);
    if (tile >= (uint32_t)a.tiles_n * (uint32_t)a.tiles_m) return;   // uniform
    const uint32_t tn = uniform(tile / (uint32_t)a.tiles_m), tm = tile - tn * (uint32_t)a.tiles_m;
    const int64_t n0 = ((int64_t)tn * 4 + wave) * (16 * NT), m0 = (int64_t)tm * MT * 16;
    const int nb = a.D / 32, have = a.M - m0 < rows ? (int)(a.M - m0) : rows;
    const int part = rows * kc * 2;                       // bytes of one part of x in LDS

    const char *wp[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t n = n0 + w_row_at<OUT_BF16>(16 * t + r);
        wp[t] = a.w + (n < a.N ? n : a.N - 1) * a.w_pitch;
    }
    int xrow[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) xrow[i] = 16 * i + r < have ? 16 * i + r : have - 1;
    mx_f4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = mx_f4{0.f, 0.f, 0.f, 0.f};

    // 512 elements of W's rows; with AHEAD requested while the 512 before them are multiplied (1 x 128000 x 2048 bf16 25.6 us,
    // without 29.8; 32 rows of x 52, without 43.8: too few wavefronts fit)
    uint4 next_wc[NT][4], next_ws[NT];
    auto load_w = [&](int b0) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            next_ws[t] = load_chunk(wp[t] + a.D / 2 + b0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int b = b0 + 4 * j + g;
                next_wc[t][j] = make_uint4(0, 0, 0, 0);
                if (b < nb) next_wc[t][j] = load_chunk(wp[t] + b * 16);
            }
        }
    };
    if (AHEAD) load_w(0);
    for (int k0 = 0; k0 < a.D; k0 += kc) {                // uniform
        if (k0) __syncthreads();                          // everyone is done with the part of K before
        const int chunks = kc / 8;
        for (int idx = tid; idx < have * chunks; idx += THREADS) {
            const int m = idx / chunks, c = idx - m * chunks, k = k0 + c * 8;
            char *to = lds + m * kc * 2 + ((c & ~15) | ((c ^ wide_key_x(m)) & 15)) * 16;
            const char *from = a.x + (m0 + m) * a.x_pitch + (int64_t)k * (XT == X_F32 ? 4 : 2);
            uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;   // past the row's end: zeros
            if (k < a.D) {
                lo = load_chunk(from);
                if (XT == X_F32) hi = load_chunk(from + 16);
            }
            if constexpr (XT == X_F32) {
                mx_b8 p[3];
                split_bf16(lo, hi, p);
#pragma unroll
                for (int j = 0; j < 3; ++j) *reinterpret_cast<mx_b8 *>(to + j * part) = p[j];
            } else {
                *reinterpret_cast<uint4 *>(to) = lo;
            }
        }
        __syncthreads();
        const int end = a.D - k0 < kc ? a.D - k0 : kc;
        for (int s = 0; s * 512 < end; ++s) {
            const int b0 = k0 / 32 + s * 16;              // first of 16 blocks
            if (!AHEAD) load_w(b0);
            uint4 wc[NT][4], ws[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                ws[t] = next_ws[t];
#pragma unroll
                for (int j = 0; j < 4; ++j) wc[t][j] = next_wc[t][j];
            }
            if (AHEAD && b0 + 16 < nb) load_w(b0 + 16);   // uniform
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (b0 + 4 * j >= nb) break;              // uniform
                const bool in = b0 + 4 * j + g < nb;      // blocks past the row: codes 0, a scale that is a number
                float scale[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) scale[t] = __uint_as_float(in ? ((word_of(ws[t], j) >> (8 * g)) & 255u) << 23 : 127u << 23);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    mx_b8 xb[MT][KPARTS];
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int k = 0; k < KPARTS; ++k)
                            xb[i][k] = *reinterpret_cast<const mx_b8 *>(lds + k * part + xrow[i] * kc * 2 + s * 1024 + j * 256 +
                                                                       (((4 * g + q) ^ wide_key_x(xrow[i])) & 15) * 16);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const mx_b8 wb = codes_to_bf16(word_of(wc[t][j], q), scale[t]);
#pragma unroll
                        for (int k = KPARTS - 1; k >= 0; --k)
#pragma unroll
                            for (int i = 0; i < MT; ++i) acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, xb[i][k], acc[i][t], 0, 0, 0);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        store_tiles<NT, OUT_BF16>(a, m0 + 16 * i + r, n0, g, acc[i]);
    }
    mend_infinite_rows<XT, OUT_BF16>(a, m0, n0, r, g, acc);
}

template <int XT, int MT, bool OUT_BF16>
int launch_skinny(ProductArgs a, hipStream_t s)
{
    constexpr int PARTS = XT == X_F32 ? 3 : 1;
    const int rows = a.M < MT * 16 ? (int)a.M : MT * 16;
    int kc = LDS_X / (rows * 2 * PARTS) / 512 * 512;      // (at least 512)
    const int all = (a.D + 511) / 512 * 512;
    if (kc > all) kc = all;
    a.tiles_m = (a.M + MT * 16 - 1) / (MT * 16);
    a.tiles_n = (a.N + 127) / 128;
    if (a.tiles_n > (int64_t)0x7FFFFF00 / a.tiles_m) return EMB_ERR_UNSUPPORTED;
    const int64_t blocks = emb_round_up_xcds(a.tiles_m * a.tiles_n);
    if (!fits_a_grid(blocks, 256)) return EMB_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((product_skinny_kernel<XT, MT, OUT_BF16>), dim3((unsigned)blocks), dim3(256), (size_t)rows * kc * 2 * PARTS, s, a,
                       rows, kc);
    return EMB_OK;
}

// Which kernel.  Times in us on an MI355X, outputs bf16 unless said.
//   A long K and tiles of 16 x 32 too few to fill the chip with wavefronts: the wavefronts of a workgroup split K, 16 ways where there
//   are very few (1 x 4096 x 4096 bf16 5.1, without 9.3; 8 x 512 x 16384 fp32 25, with 8 ways 39).  Beyond about 1024 tiles the other
//   kernels fill it (16 x 50000 x 512 bf16 5.3, split 12.9); the split parts of fp32, for which every wavefront makes three parts of its
//   x, lose from 512 on (1024 x 512 x 1024 8.9, split 18.8); few rows of MXFP4 that are very long, which have no other kernel that shares
//   a tile, gain up to 1536 (8 x 33792 x 4096 20.2, without 29.5; 16 x 49152 x 4096 28.2 and 34.9; 8 x 33792 x 2048 12.9 and 15.3, but 32 x 24576
//   x 2048 14.1 and 12.4), and lose at 2048 (32 x 32768 x 4096 31.6 and 25.2, 1 x 65536 x 2048 20.1 and 16.7).
//   Few rows of x: W streams through registers; MXFP4 and short rows straight from global memory (16 x 100003 x 64 fp32 6.4,
//   through LDS 8.5; from 256 elements on LDS is ahead: 16 x 100003 x 512 bf16 8.9, straight 11.6, fp32 11.9 and 19.4), others with x in
//   LDS (16 x 128000 x 2048 bf16 37, straight 50).  33 to 64 rows of MXFP4 are tiles where they are long and W has not rows enough for
//   straight wavefronts (64 x 16384 x 4096 16.5, straight 31; 64 x 128000 x 2048 44, tiles 50).
//   A row of x costs an fp32 product three MFMA, and the tiles for it are the less efficient: three passes over W are still quicker
//   than one over half-empty tiles (48 x 128000 x 2048: 114 and 188), and any number of them where tiles do not fill the
//   chip once (256 x 4096 x 1024 12.2, tiles 38.6; 512 x 2048 x 4096 46 and 142; the shorter the rows, the sooner tiles are ahead.  512
//   elements: 256 x 24576 28.9 and 33.4, 256 x 32768, 512 tiles, 36.9 and 34.6; 128 elements: 256 x 8192 8.8 and 9.5, 256 x 10240, 160 tiles, 10.2 and
//   9.9; between them a line at 160 is early for some, at 256 late for others: 256 x 10240 x 384 13.0 and 18.2, 256 x 15000 x 256 16.0 and 14.3).  bf16 takes half tiles there (512 x 4096 x 4096 29, whole 37.6).
//   Rows of x so far apart that 128 of them pass 32-bit offsets: LDS as well, any number of rows.
//   Up to 32 rows of x past whole tiles: a call of their own, where their tiles would begin another round of workgroups on the
//   chip (at_once of them) and rows are long enough for that to take longer than the call (4099 rows of x, 4096 of W: 1024 elements
//   bf16 45.2, so 42.7, fp32 180, so 163; 4096: MXFP4 63.8, so 44.1, bf16 167, so 142; with 512 elements bf16 nothing is won).  MXFP4 up to 65536
//   rows of W: 4099 x 32768 x 1024 148, so 145; 4099 x 61440 x 1024 254 and 253; 4099 x 131072 x 1024 547 and 561, 2050 x 131072 x 2048 432 and 456.
inline int64_t rows_of_full_rounds(const ProductArgs &a, int64_t tile, int64_t at_once)
{
    const int64_t whole = a.M / tile * tile, rest = a.M - whole;
    if (whole == 0 || rest == 0 || rest > 32) return a.M;
    ProductArgs all = a, without = a;
    without.M = whole;
    return (share_tiles(without, tile, tile) + at_once - 1) / at_once < (share_tiles(all, tile, tile) + at_once - 1) / at_once ? whole : a.M;
}

template <int XT, bool OUT_BF16>
int dispatch_product(const ProductArgs &a, hipStream_t s);

template <int XT, bool OUT_BF16>
int dispatch_in_two(ProductArgs a, int64_t whole, hipStream_t s)
{
    const int64_t rest = a.M - whole;
    a.M = whole;
    const int rc = dispatch_product<XT, OUT_BF16>(a, s);
    if (rc != EMB_OK) return rc;
    a.M = rest;
    a.x += whole * a.x_pitch;
    a.out += whole * a.out_stride * (OUT_BF16 ? 2 : 4);
    return dispatch_product<XT, OUT_BF16>(a, s);
}

template <int XT, bool OUT_BF16>
int dispatch_product(const ProductArgs &a, hipStream_t s)
{
    const int64_t tiles = (a.M + 15) / 16 * ((a.N + 31) / 32);
    const int64_t most_split = XT == X_F32 ? 512 : (XT == X_MXFP4 && a.M <= 32 && a.D >= 2048 ? 1536 : 1024);
    if (a.D > 512 && tiles <= most_split) return tiles < 256 ? launch_direct<XT, 1, 1, 16, OUT_BF16>(a, s) : launch_direct<XT, 1, 2, 8, OUT_BF16>(a, s);
    if constexpr (XT == X_MXFP4) {
        if (a.M <= 16) return launch_direct<XT, 1, 2, 1, OUT_BF16>(a, s);
        if (a.M <= 32) return launch_direct<XT, 2, 2, 1, OUT_BF16>(a, s);
        if (a.M <= 64 && (a.D < 1024 || a.N >= 65536)) return launch_direct<XT, 4, 2, 1, OUT_BF16>(a, s);
        if (a.D <= 128) return launch_tiled<2, 2, 4, true, OUT_BF16>(a, s);
        const bool big = (a.M + 255) / 256 * ((a.N + 255) / 256) >= 256;
        if (a.D >= 512 && a.N <= 65536) {             // (a strip of more tiles is rounds by itself, and the few rows read all of W)
            const int64_t whole = rows_of_full_rounds(a, big ? 256 : 128, big ? 256 : 512);
            if (whole < a.M) return dispatch_in_two<XT, OUT_BF16>(a, whole, s);
        }
        if (big) return launch_tiled<2, 4, 8, false, OUT_BF16>(a, s);
        return launch_tiled<2, 2, 4, false, OUT_BF16>(a, s);
    } else {
        constexpr bool BF16 = XT == X_BF16;
        const bool far = a.x_pitch > MOST_PITCH;
        const int64_t strips = (a.N + 127) / 128;
        if (a.D < 256 && a.M <= 16) return launch_direct<XT, 1, 2, 1, OUT_BF16>(a, s);
        if (a.D < 256 && a.M <= 32) return launch_direct<XT, 2, 2, 1, OUT_BF16>(a, s);
        if (a.M <= 16 || (!BF16 && (a.M <= 48 || far || (a.M + 127) / 128 * strips < (a.D >= 512 ? 512 : 160)))) return launch_skinny<XT, 1, OUT_BF16>(a, s);
        if constexpr (BF16) {
            if (a.M <= 32 || far) return launch_skinny<XT, 2, OUT_BF16>(a, s);
        }
        if (a.M <= 64 || (BF16 && (a.M + 63) / 64 * strips <= 512)) return launch_widened<XT, true, OUT_BF16>(a, s);
        if (a.D >= (BF16 ? 1024 : 512)) {
            const int64_t whole = rows_of_full_rounds(a, 128, 512);
            if (whole < a.M) return dispatch_in_two<XT, OUT_BF16>(a, whole, s);
        }
        return launch_widened<XT, false, OUT_BF16>(a, s);
    }
}

// W in halves where a launch would have more threads than a grid holds (33 rows of fp32 x by 7e8 rows of W).
template <int XT, bool OUT_BF16>
int product_in_launches(ProductArgs a, hipStream_t s)
{
    const int rc = dispatch_product<XT, OUT_BF16>(a, s);
    if (rc != EMB_ERR_UNSUPPORTED || a.N < 4096) return rc;
    ProductArgs rest = a;
    a.N = a.N / 2 / 2048 * 2048;                          // (whole tiles)
    rest.N -= a.N;
    rest.w += a.N * a.w_pitch;
    rest.out += a.N * (OUT_BF16 ? 2 : 4);
    const int half = product_in_launches<XT, OUT_BF16>(a, s);
    return half != EMB_OK ? half : product_in_launches<XT, OUT_BF16>(rest, s);
}

constexpr int64_t MOST_ROWS = ((int64_t)1 << 31) - 2048;   // of x and of W: row numbers, tiles of them included, are 32-bit

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
    if (M > MOST_ROWS || N > MOST_ROWS) return EMB_ERR_UNSUPPORTED;
    const ProductArgs a{static_cast<const char *>(x_dev), static_cast<const char *>(w_rows_dev), x_pitch, row, M, N, D,
                        static_cast<char *>(out_dev), out_stride, 0, 0, 1, 0};
    hipStream_t s = emb_stream(stream);
    const bool b = out_dtype == EMB_BF16;
    int e;
    switch (x_dtype) {
        case EMB_MXFP4: e = b ? product_in_launches<X_MXFP4, true>(a, s) : product_in_launches<X_MXFP4, false>(a, s); break;
        case EMB_BF16: e = b ? product_in_launches<X_BF16, true>(a, s) : product_in_launches<X_BF16, false>(a, s); break;
        default: e = b ? product_in_launches<X_F32, true>(a, s) : product_in_launches<X_F32, false>(a, s);
    }
    if (e != EMB_OK) return e;
    EMB_RETURN_IF_LAUNCH_FAILED();
    return EMB_OK;
}
