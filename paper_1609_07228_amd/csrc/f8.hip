// Matrices in 8-bit floating point with a power-of-two scale for each block of 128 (the format is described in efanna_f8.h),
// for gfx950: quantisation by rows and by tiles, rows by id, products of two tables, the gradient of a layer's weights.
//
// A power of two as a scale costs no precision (the codes are floating-point numbers themselves), and v_mfma_scale_f32_*_f8f6f4
// applies it.  A row's blocks are whole, 128 bytes of codes each, so that every product is made of whole steps.
#include "tables.h"

#include "../../include/efanna_f8.h"

namespace {

__host__ __device__ inline int f8_blocks(int d) { return (d + 127) >> 7; }
__host__ __device__ inline int f8_scale_pitch(int d) { return (f8_blocks(d) + 3) & ~3; }

struct F8 {
    const uint8_t *codes, *scales;
    int n, nb, sp;
    __device__ inline const uint8_t *row(long long r) const { return codes + (size_t)r * nb * 128; }
};

// ---- codes -----------------------------------------------------------------------------------------------
// Scale byte of a block whose largest finite magnitude has the bits `top`: the smallest power that leaves it within 1.75 * 2^8
// (E4M3) or 2^15 (E5M2): its own exponent, one more if its mantissa is beyond 1.75, less 8 or 15.
template <int FORMAT> __device__ inline u32 scale_byte(u32 top)
{
    const int e = (int)((top + 0x001FFFFFu) >> 23) - (FORMAT == EFANNA_E4M3 ? 8 : 15);
    return (u32)max(e, 0);
}
// 2^(127 - b) for such a byte, b <= 247
__device__ inline float inverse_scale(u32 b) { return __uint_as_float((254 - b) << 23); }

__device__ inline u32 finite_bits(float x)
{
    const u32 u = __float_as_uint(x) & 0x7FFFFFFFu;
    return u < 0x7F800000u ? u : 0;
}

// Codes of four values that are within the format's range (infinities and NaN become what the format has for them).
template <int FORMAT> __device__ inline u32 four_codes(float a, float b, float c, float d)
{
    int w = 0;
    if (FORMAT == EFANNA_E4M3) {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    }
    return (u32)w;
}
template <int FORMAT> __device__ inline void four_values(u32 w, float *v)
{
    const f32x2 lo = FORMAT == EFANNA_E4M3 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false) : __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false);
    const f32x2 hi = FORMAT == EFANNA_E4M3 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true) : __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
    v[0] = lo.x, v[1] = lo.y, v[2] = hi.x, v[3] = hi.y;
}

typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Sixteen codes as bfloat16 numbers, times their scale (exact from 2^-126 on).
template <int FORMAT> __device__ inline void sixteen_wide(i32x4 codes, float scale, bf16x8 (&v)[2])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf16x2 lo = FORMAT == EFANNA_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((u32)codes[i], scale, false)
                                                : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((u32)codes[i], scale, false);
        const bf16x2 hi = FORMAT == EFANNA_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((u32)codes[i], scale, true)
                                                : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((u32)codes[i], scale, true);
        v[i >> 1][(i & 1) * 4] = lo.x, v[i >> 1][(i & 1) * 4 + 1] = lo.y;
        v[i >> 1][(i & 1) * 4 + 2] = hi.x, v[i >> 1][(i & 1) * 4 + 3] = hi.y;
    }
}

// ---- quantisation of rows --------------------------------------------------------------------------------
// Sixteen lanes per block, eight coordinates each; a wave takes four blocks (their scales are one word), which are one row's
// four, or of rows of one or two blocks four or two rows (`group` lanes a row).
template <class T, int FORMAT>
__global__ __launch_bounds__(256) void f8_quantise_kernel(const T *X, u32 units, int d, long long ldx, int group, int nb, int sp,
                                                          uint8_t *codes, uint8_t *scales)
{
    const int lane = threadIdx.x & (group - 1), words = sp >> 2;
    const u32 unit = blockIdx.x * (256u / group) + threadIdx.x / group;
    if (unit >= units) return;
    const u32 row = words == 1 ? unit : unit / words, word = words == 1 ? 0 : unit - row * words;
    const int block = word * 4 + (lane >> 4), at = block * 128 + (lane & 15) * 8;
    float v[8];
    load_eight(X + row * ldx + at, d - at, v);
    u32 top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, finite_bits(v[j]));
    top = max(top, lane_from<kSwap1>(top));
    top = max(top, lane_from<kSwap2>(top));
    top = max(top, lane_from<kDown4>(top));
    top = max(top, lane_from<kDown8>(top));
    const u32 b = scale_byte<FORMAT>(top);
    const float inverse = inverse_scale(b);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= inverse;
    if (block < nb)
        *(u32x2 *)(codes + ((size_t)row * nb + block) * 128 + (lane & 15) * 8) =
            u32x2{four_codes<FORMAT>(v[0], v[1], v[2], v[3]), four_codes<FORMAT>(v[4], v[5], v[6], v[7])};
    u32 four = block < nb ? b : 0;
    if (group > 16) four |= __shfl_down(four, 16) << 8;
    if (group > 32) four |= __shfl_down(four, 32) << 16;
    if (lane == 0) *(u32 *)(scales + (size_t)row * sp + word * 4) = four;
}

// ---- quantisation of a matrix by tiles of 128 x 128 ------------------------------------------------------------
// A workgroup takes a tile: a thread holds 8 x 8 of it (rows 8 (tid / 16) on, columns 8 (tid % 16) on) in registers, all share the
// largest magnitude, and the codes of the transpose leave through LDS as whole lines.
template <class T, int FORMAT>
__global__ __launch_bounds__(256) void f8_weights_kernel(const T *W, int n, int d, long long ldw, uint8_t *codes, uint8_t *scales,
                                                         uint8_t *t_codes, uint8_t *t_scales)
{
    __shared__ u32 tops[4];
    __shared__ __align__(16) uint8_t turned[128][144];
    const int tid = threadIdx.x, nb = f8_blocks(d), sp = f8_scale_pitch(d), t_nb = f8_blocks(n), t_sp = f8_scale_pitch(n);
    const int bx = blockIdx.x, by = blockIdx.y, r0 = by * 128 + (tid >> 4) * 8, c0 = bx * 128 + (tid & 15) * 8;
    float v[8][8];
    u32 top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        load_eight(W + min(r0 + i, n - 1) * ldw + c0, r0 + i < n ? d - c0 : 0, v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, finite_bits(v[i][j]));
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = max(top, (u32)__shfl_xor((int)top, o));
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
    const u32 b = scale_byte<FORMAT>(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
    const float inverse = inverse_scale(b);
    u32 w[8][2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= inverse;
        w[i][0] = four_codes<FORMAT>(v[i][0], v[i][1], v[i][2], v[i][3]);
        w[i][1] = four_codes<FORMAT>(v[i][4], v[i][5], v[i][6], v[i][7]);
        if (r0 + i < n) *(u32x2 *)(codes + ((size_t)(r0 + i) * nb + bx) * 128 + (tid & 15) * 8) = u32x2{w[i][0], w[i][1]};
    }
    // scales of the tile's rows, with the padding after the last block
    const int pad = bx == nb - 1 ? sp - nb : 0, t_pad = by == t_nb - 1 ? t_sp - t_nb : 0;
    if (tid < 128 && by * 128 + tid < n) {
        uint8_t *s = scales + (size_t)(by * 128 + tid) * sp + bx;
        s[0] = (uint8_t)b;
        for (int i = 1; i <= pad; ++i) s[i] = 0;
    }
    if (!t_codes) return;
    if (tid >= 128 && bx * 128 + tid - 128 < d) {
        uint8_t *s = t_scales + (size_t)(bx * 128 + tid - 128) * t_sp + by;
        s[0] = (uint8_t)b;
        for (int i = 1; i <= t_pad; ++i) s[i] = 0;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        u32 col[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) col[i >> 2] |= ((w[i][j >> 2] >> (8 * (j & 3))) & 255u) << (8 * (i & 3));
        *(u32x2 *)&turned[(tid & 15) * 8 + j][(tid >> 4) * 8] = u32x2{col[0], col[1]};
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * 32 + (tid >> 3), part = (tid & 7) * 16;
        if (bx * 128 + c < d) *(u32x4 *)(t_codes + ((size_t)(bx * 128 + c) * t_nb + by) * 128 + part) = *(const u32x4 *)&turned[c][part];
    }
}

// ---- rows by id ------------------------------------------------------------------------------------------
// A lane per 16 bytes of an output row (4 or 8 coordinates: neighbouring lanes' stores touch), `group` lanes (a power of two)
// per row and kRows rows per lane, so that as many chains of id, codes, store run side by side.  Codes have at most four significant
// bits, so value * scale is exact; the factor's product is rounded to float32 and then once to the output's type.
constexpr int kRows = 4;
template <class T, int FORMAT, bool PAST_CACHE>
__global__ __launch_bounds__(256) void f8_rows_kernel(F8 t, int d, const int *ids, long long m, int group, float factor, T *out)
{
    constexpr int kPer = 16 / sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
    const int lane = threadIdx.x & (group - 1), per = 256 / group;
    const long long first = (long long)blockIdx.x * (per * kRows) + threadIdx.x / group;
    int id[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const long long row = min(first + (long long)i * per, m - 1);
        id[i] = ids ? ids[row] : (int)row;
    }
    for (int p = lane; p * kPer < d; p += group) {
        u32 word[kRows][2], b[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            word[i][0] = word[i][1] = 0, b[i] = 256;                   // (an empty slot)
            if (id[i] >= 0 && id[i] < t.n) {
                const uint8_t *from = t.row(id[i]) + p * kPer;
                if (kPer == 4) word[i][0] = *(const u32 *)from;
                else {
                    const u32x2 x = *(const u32x2 *)from;
                    word[i][0] = x.x, word[i][1] = x.y;
                }
                b[i] = t.scales[(size_t)id[i] * t.sp + p * kPer / 128];
            }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const long long row = first + (long long)i * per;
            float v[8];
            four_values<FORMAT>(word[i][0], v);
            if (kPer > 4) four_values<FORMAT>(word[i][1], v + 4);
            const float scale = scale_value(b[i] & 255);
            Piece x;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                float y = v[j] * scale * factor;
                if (sizeof(T) == 2) asm("" : "+v"(y));            // (a float32 number: not multiplied and rounded in one instruction)
                x[j] = from_float<T>(b[i] > 255 ? 0.0f : y);
            }
            if (row >= m) continue;
            T *o = out + (size_t)row * d + p * kPer;
            if (d - p * kPer >= kPer) {
                if (PAST_CACHE) __builtin_nontemporal_store(x, (Piece *)o);
                else *(Piece *)o = x;
            } else
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (p * kPer + j < d) o[j] = x[j];
        }
    }
}

// ---- matrix instructions ---------------------------------------------------------------------------------
// Lane l of an instruction of 32 x 32 brings its part of row l % 32 of an operand: 32 bytes of a step of 64 coordinates for
// 8-bit operands, 8 numbers of a step of 16 for bfloat16.  Which coordinates the two halves of the lanes bring does not matter as
// long as both operands agree.  The result's lane l holds column l % 32 (of the second operand), rows 8 c + 4 (l / 32) + 0..3.
template <int FA, int FB> __device__ inline f32x16 f8_mma(i32x4 a0, i32x4 a1, int a_scale, i32x4 b0, i32x4 b1, int b_scale, f32x16 c)
{
    const i32x8 a = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w}, b = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, FA, FB, 0, a_scale, 0, b_scale);
}

// Products: a wave per 32 x 32 results, operands from memory.
template <class T, int FA, int FB>
__global__ __launch_bounds__(256) void f8_product_kernel(F8 a, F8 b, T *out, long long ldo, int tiles_b, u32 tiles)
{
    const int lane = threadIdx.x & 63, r = lane & 31, half = lane >> 5;
    const u32 tile = min(blockIdx.x * 4 + (threadIdx.x >> 6), tiles - 1);
    const int i0 = (int)(tile / tiles_b) * 32, j0 = (int)(tile % tiles_b) * 32;
    const int ra = min(i0 + r, a.n - 1), rb = min(j0 + r, b.n - 1);
    f32x16 acc = {};
    for (int s = 0; s < a.nb; ++s) {
        const int sa = a.scales[(size_t)ra * a.sp + s], sb = b.scales[(size_t)rb * b.sp + s];
        const i32x4 *pa = (const i32x4 *)(a.row(ra) + s * 128) + half, *pb = (const i32x4 *)(b.row(rb) + s * 128) + half;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    bf16x8 x[2], y[2];
                    sixteen_wide<FB>(pb[4 * h + 2 * c], scale_value(sb), x);
                    sixteen_wide<FA>(pa[4 * h + 2 * c], scale_value(sa), y);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[0], y[0], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[1], y[1], acc, 0, 0, 0);
                }
            } else
                acc = f8_mma<FB, FA>(pb[4 * h], pb[4 * h + 2], sb, pa[4 * h], pa[4 * h + 2], sa, acc);
        }
    }
    if (i0 + r >= a.n) return;
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        const int j = j0 + 8 * (c >> 2) + 4 * half + (c & 3);
        if (j < b.n) out[(size_t)(i0 + r) * ldo + j] = from_float<T>(acc[c]);
    }
}

// ---- gradient of the weights -----------------------------------------------------------------------------
// A number as a sum of bfloat16 numbers, exactly (from 2^-110 on for float32): one of its own kind, two of half precision (11
// bits), three of float32 (24 bits).  Infinities and NaN are all in the first part.
template <class Y> struct Parts;
template <> struct Parts<__bf16> {
    static constexpr int count = 1;
    static __device__ inline void split(__bf16 x, __bf16 (&p)[1]) { p[0] = x; }
};
template <> struct Parts<_Float16> {
    static constexpr int count = 2;
    static __device__ inline void split(_Float16 h, __bf16 (&p)[2])
    {
        const float x = (float)h;
        p[0] = (__bf16)x;
        p[1] = (__bf16)(finite_bits(x) ? x - (float)p[0] : 0.0f);
    }
};
template <> struct Parts<float> {
    static constexpr int count = 3;
    static __device__ inline float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }
    static __device__ inline void split(float x, __bf16 (&p)[3])
    {
        const bool finite = finite_bits(x) != 0;
        const float first = finite ? cut(x) : x, rest = finite ? x - first : 0.0f, second = cut(rest);
        p[0] = (__bf16)first, p[1] = (__bf16)second, p[2] = (__bf16)(rest - second);
    }
};

// What the parts after the first are multiplied by: numbers without the infinities, which the first part meets (a later
// part that is zero would make a NaN of one).
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
__device__ inline bf16x8 without_infinities(bf16x8 x)
{
    u16x8 u = __builtin_bit_cast(u16x8, x);
    u *= __builtin_elementwise_min((u16x8)((u & (unsigned short)0x7FFF) ^ (unsigned short)0x7F80), (u16x8)(unsigned short)1);
    return __builtin_bit_cast(bf16x8, u);
}

// A wave per 32 x 32 results, elements from memory one by one.
template <class Y, class T, int FORMAT>
__global__ __launch_bounds__(256) void f8_gradient_kernel(const Y *dy, long long ldy, long long m, int n, F8 x, int d, T *out,
                                                          long long ldo, int tiles_d, u32 tiles)
{
    const int lane = threadIdx.x & 63, r = lane & 31, half = lane >> 5;
    const u32 tile = min(blockIdx.x * 4 + (threadIdx.x >> 6), tiles - 1);
    const int j = (int)(tile / tiles_d) * 32 + r, c0 = (int)(tile % tiles_d) * 32, c = min(c0 + r, d - 1);
    f32x16 acc = {};
    for (long long t0 = 0; t0 < m; t0 += 16) {
        bf16x8 held, part[Parts<Y>::count];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const long long t = t0 + 8 * half + k, row = min(t, m - 1);
            float v[4];
            four_values<FORMAT>(x.row(row)[c], v);
            held[k] = (__bf16)(t < m ? v[0] * scale_value(x.scales[(size_t)row * x.sp + (c >> 7)]) : 0.0f);
            __bf16 p[Parts<Y>::count];
            Parts<Y>::split(t < m ? dy[row * ldy + min(j, n - 1)] : (Y)0.0f, p);
#pragma unroll
            for (int i = 0; i < Parts<Y>::count; ++i) part[i][k] = p[i];
        }
#pragma unroll
        for (int i = 0; i < Parts<Y>::count; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(i ? without_infinities(held) : held, part[i], acc, 0, 0, 0);
    }
    if (j >= n) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int col = c0 + 8 * (i >> 2) + 4 * half + (i & 3);
        if (col < d) out[(size_t)j * ldo + col] = from_float<T>(acc[i]);
    }
}

inline bool table_ok(const uint8_t *codes, const uint8_t *scales, int32_t format, int64_t n, int32_t d)
{
    if (n < 0 || n > kMaxRows || d < 1 || d > EFANNA_F8_MAX_D || (format != EFANNA_E4M3 && format != EFANNA_E5M2)) return false;
    return n == 0 || (codes && scales && ((uintptr_t)codes & 15) == 0 && ((uintptr_t)scales & 3) == 0);
}
inline bool workspace_ok(const void *ws, size_t have, size_t need)
{
    return need == 0 || (ws && ((uintptr_t)ws & 255) == 0 && have >= need);
}

}  // namespace

#define EF_FORMAT(format, F, ...)                                                    \
    do {                                                                             \
        if ((format) == EFANNA_E4M3) { constexpr int F = EFANNA_E4M3; __VA_ARGS__; } \
        else { constexpr int F = EFANNA_E5M2; __VA_ARGS__; }                         \
    } while (0)

extern "C" int efanna_f8_quantise(const void *X, int32_t dtype, int64_t n, int32_t d, int64_t ldx, int32_t format,
                                  uint8_t *codes, uint8_t *scales, void *stream)
{
    if (!dtype_ok(dtype) || !table_ok(codes, scales, format, n, d) || ldx < d) return EFANNA_EINVAL;
    if (n == 0) return EFANNA_OK;
    if (!X || !aligned_for(X, dtype)) return EFANNA_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const int nb = f8_blocks(d), sp = f8_scale_pitch(d), words = sp / 4, group = nb == 1 ? 16 : nb == 2 ? 32 : 64;
    const int64_t units = 256 / group, slice = kSliceBlocks * units / words;      // of a workgroup; rows of a launch
    for (int64_t first = 0; first < n; first += slice) {
        const int64_t here = (n - first < slice ? n - first : slice) * words;
        EF_DTYPE(dtype, T, EF_FORMAT(format, F, (f8_quantise_kernel<T, F><<<(unsigned)((here + units - 1) / units), 256, 0, st>>>(
                                                    (const T *)X + first * ldx, (u32)here, d, ldx, group, nb, sp,
                                                    codes + (size_t)first * nb * 128, scales + (size_t)first * sp))));
        EF_HIP_CHECK(hipGetLastError());
    }
    return EFANNA_OK;
}

extern "C" int efanna_f8_weights(const void *W, int32_t dtype, int32_t n, int32_t d, int64_t ldw, int32_t format,
                                 uint8_t *codes, uint8_t *scales, uint8_t *t_codes, uint8_t *t_scales, void *stream)
{
    if (!dtype_ok(dtype) || !table_ok(codes, scales, format, n, d) || n > EFANNA_F8_MAX_D || ldw < d) return EFANNA_EINVAL;
    if ((t_codes || t_scales) && (n > 0 && !table_ok(t_codes, t_scales, format, d, n))) return EFANNA_EINVAL;
    if (n == 0) return EFANNA_OK;
    if (!W || !aligned_for(W, dtype)) return EFANNA_EINVAL;
    const dim3 grid((unsigned)f8_blocks(d), (unsigned)f8_blocks(n));
    EF_DTYPE(dtype, T, EF_FORMAT(format, F, (f8_weights_kernel<T, F><<<grid, 256, 0, (hipStream_t)stream>>>(
                                                (const T *)W, n, d, ldw, codes, scales, t_codes, t_scales))));
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
}

extern "C" int efanna_f8_rows(const uint8_t *codes, const uint8_t *scales, int32_t format, int64_t n, int32_t d,
                              const int32_t *ids, int64_t m, float factor, int32_t dtype, void *out, void *stream)
{
    if (!dtype_ok(dtype) || !table_ok(codes, scales, format, n, d) || m < 0 || m > kMaxRows || (!ids && m > n)) return EFANNA_EINVAL;
    if (m == 0) return EFANNA_OK;
    if (!out || !aligned_for(out, dtype) || ((uintptr_t)ids & 3)) return EFANNA_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const F8 t = {codes, scales, (int)n, f8_blocks(d), f8_scale_pitch(d)};
    const int per = dtype == EFANNA_F32 ? 4 : 8;
    const bool past_cache = m * d * (16 / per) > kStreamBytes;
    int group = 1;
    while (group < 64 && group * per < d) group <<= 1;
    const int64_t rows = kRows * (256 / group), slice = kSliceBlocks * rows;      // rows of a workgroup, of a launch
    for (int64_t first = 0; first < m; first += slice) {
        const int64_t here = m - first < slice ? m - first : slice;
        const unsigned blocks = (unsigned)((here + rows - 1) / rows);
        // (without ids the slice's rows are a table of their own)
        const F8 from = ids ? t : F8{codes + (size_t)first * t.nb * 128, scales + (size_t)first * t.sp, (int)(n - first), t.nb, t.sp};
        const int *slice_ids = ids ? ids + first : nullptr;
        EF_DTYPE(dtype, T, EF_FORMAT(format, F, {
            T *to = (T *)out + (size_t)first * d;
            if (past_cache) f8_rows_kernel<T, F, true><<<blocks, 256, 0, st>>>(from, d, slice_ids, here, group, factor, to);
            else f8_rows_kernel<T, F, false><<<blocks, 256, 0, st>>>(from, d, slice_ids, here, group, factor, to);
        }));
        EF_HIP_CHECK(hipGetLastError());
    }
    return EFANNA_OK;
}

extern "C" size_t efanna_f8_product_workspace_bytes(int64_t m, int64_t n, int32_t d) { return 0; }

extern "C" int efanna_f8_product(const uint8_t *a_codes, const uint8_t *a_scales, int32_t a_format, int64_t m,
                                 const uint8_t *b_codes, const uint8_t *b_scales, int32_t b_format, int64_t n, int32_t d,
                                 int32_t dtype, void *out, int64_t ldo, void *ws, size_t ws_bytes, void *stream)
{
    if (!dtype_ok(dtype) || !table_ok(a_codes, a_scales, a_format, m, d) || !table_ok(b_codes, b_scales, b_format, n, d) || ldo < n)
        return EFANNA_EINVAL;
    if (m == 0 || n == 0) return EFANNA_OK;
    if (!out || !aligned_for(out, dtype)) return EFANNA_EINVAL;
    if (!workspace_ok(ws, ws_bytes, efanna_f8_product_workspace_bytes(m, n, d))) return EFANNA_EWORKSPACE;
    const int nb = f8_blocks(d), sp = f8_scale_pitch(d);
    const F8 a = {a_codes, a_scales, (int)m, nb, sp}, b = {b_codes, b_scales, (int)n, nb, sp};
    const int64_t tiles_b = (n + 31) / 32, tiles = (m + 31) / 32 * tiles_b;
    if (tiles > 2147483647LL || !launch_fits((tiles + 3) / 4, 256)) return EFANNA_EUNSUPPORTED;
    EF_DTYPE(dtype, T, EF_FORMAT(a_format, FA, EF_FORMAT(b_format, FB, (f8_product_kernel<T, FA, FB><<<(unsigned)((tiles + 3) / 4), 256, 0, (hipStream_t)stream>>>(
                           a, b, (T *)out, ldo, (int)tiles_b, (u32)tiles)))));
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
}

extern "C" size_t efanna_f8_gradient_workspace_bytes(int64_t m, int32_t n, int32_t d) { return 0; }

extern "C" int efanna_f8_gradient(const void *dY, int32_t dtype, int64_t m, int32_t n, int64_t ldy, const uint8_t *codes,
                                  const uint8_t *scales, int32_t format, int32_t d, int32_t out_dtype, void *out,
                                  int64_t ldo, void *ws, size_t ws_bytes, void *stream)
{
    if (!dtype_ok(dtype) || !dtype_ok(out_dtype) || !table_ok(codes, scales, format, m, d) || n < 0 || n > EFANNA_F8_MAX_D || ldy < n || ldo < d)
        return EFANNA_EINVAL;
    if (n == 0) return EFANNA_OK;
    if ((m > 0 && !dY) || !out || !aligned_for(dY, dtype) || !aligned_for(out, out_dtype)) return EFANNA_EINVAL;
    if (!workspace_ok(ws, ws_bytes, efanna_f8_gradient_workspace_bytes(m, n, d))) return EFANNA_EWORKSPACE;
    const F8 x = {codes, scales, (int)m, f8_blocks(d), f8_scale_pitch(d)};
    const int tiles_d = (d + 31) / 32;
    const u32 tiles = (u32)((n + 31) / 32) * (u32)tiles_d;
    EF_DTYPE(dtype, Y, EF_DTYPE(out_dtype, T, EF_FORMAT(format, F, (f8_gradient_kernel<Y, T, F><<<(tiles + 3) / 4, 256, 0, (hipStream_t)stream>>>(
                           (const Y *)dY, ldy, m, n, x, d, (T *)out, ldo, tiles_d, tiles)))));
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
}
