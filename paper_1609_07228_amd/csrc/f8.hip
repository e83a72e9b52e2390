// Matrices in 8-bit floating point with a power-of-two scale for each block of 128 (the format is described in efanna_f8.h),
// for gfx950: quantisation by rows and by tiles, rows by id, products of two tables, the gradient of a layer's weights.
//
// A power of two as a scale costs no precision (the codes are floating-point numbers themselves), and v_mfma_scale_f32_*_f8f6f4
// applies it.  A row's blocks are whole, 128 bytes of codes each, so that every product is made of whole steps.
#include "pieces.h"
#include "tables.h"

#include "../../include/efanna_f8.h"

#include <type_traits>

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
// four, or of rows of one or two blocks four or two rows (`group` lanes a row).  Rows of up to 64 coordinates take eight lanes,
// which write the zeros after them too.  Bound: HBM (65 536 x 4096 bfloat16, 809 MB: 147 us, 5.5 TB/s), instructions for short rows
// (200 003 x 50 half precision: 13.0 us; with sixteen lanes a row 17.7).
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
    top = max(top, lane_from<kMirror8>(top));
    if (group > 8) top = max(top, lane_from<kDown8>(top));
    const u32 b = scale_byte<FORMAT>(top);
    const float inverse = inverse_scale(b);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= inverse;
    uint8_t *to = codes + ((size_t)row * nb + block) * 128 + (lane & 15) * 8;
    if (block < nb) *(u32x2 *)to = u32x2{four_codes<FORMAT>(v[0], v[1], v[2], v[3]), four_codes<FORMAT>(v[4], v[5], v[6], v[7])};
    if (group == 8) *(u32x2 *)(to + 64) = u32x2{0, 0};
    u32 four = block < nb ? b : 0;
    if (group > 16) four |= __shfl_down(four, 16) << 8;
    if (group > 32) four |= __shfl_down(four, 32) << 16;
    if (lane == 0) *(u32 *)(scales + (size_t)row * sp + word * 4) = four;
}

// ---- quantisation of a matrix by tiles of 128 x 128 ------------------------------------------------------------
// A workgroup takes a tile: a thread holds 4 x 8 of it (rows 4 (tid / 16) on, columns 8 (tid % 16) on) in registers, all share the
// largest magnitude, and the codes of the transpose leave through LDS as whole lines.  Bound: HBM (8192^2 float32 to both tables,
// 407 MB: 69 us, 5.9 TB/s); a few tiles (128 x 960: 5.1 us) the chain of loads, maximum and stores, which is why 512 threads share a
// tile (256 take 8.1).  Writes of the transpose to LDS meet in its banks (0.81 conflicts per active cycle), behind the loads from HBM.
template <class T, int FORMAT>
__global__ __launch_bounds__(512) void f8_weights_kernel(const T *W, int n, int d, long long ldw, uint8_t *codes, uint8_t *scales,
                                                         uint8_t *t_codes, uint8_t *t_scales)
{
    __shared__ u32 tops[8];
    __shared__ __align__(16) uint8_t turned[128][144];
    const int tid = threadIdx.x, nb = f8_blocks(d), sp = f8_scale_pitch(d), t_nb = f8_blocks(n), t_sp = f8_scale_pitch(n);
    const int bx = blockIdx.x, by = blockIdx.y, r0 = by * 128 + (tid >> 4) * 4, c0 = bx * 128 + (tid & 15) * 8;
    float v[4][8];
    u32 top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) load_eight(W + min(r0 + i, n - 1) * ldw + c0, r0 + i < n ? d - c0 : 0, v[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, finite_bits(v[i][j]));
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = max(top, (u32)__shfl_xor((int)top, o));
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
    top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, tops[i]);
    const u32 b = scale_byte<FORMAT>(top);
    const float inverse = inverse_scale(b);
    u32 w[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
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
    if (tid >= 128 && tid < 256 && bx * 128 + tid - 128 < d) {
        uint8_t *s = t_scales + (size_t)(bx * 128 + tid - 128) * t_sp + by;
        s[0] = (uint8_t)b;
        for (int i = 1; i <= t_pad; ++i) s[i] = 0;
    }
    // four rows' codes of a column are a word
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const u32 x = __builtin_amdgcn_perm(w[1][h], w[0][h], 0x05010400), y = __builtin_amdgcn_perm(w[1][h], w[0][h], 0x07030602);
        const u32 z = __builtin_amdgcn_perm(w[3][h], w[2][h], 0x05010400), u = __builtin_amdgcn_perm(w[3][h], w[2][h], 0x07030602);
        const u32 col[4] = {__builtin_amdgcn_perm(z, x, 0x05040100), __builtin_amdgcn_perm(z, x, 0x07060302), __builtin_amdgcn_perm(u, y, 0x05040100),
                            __builtin_amdgcn_perm(u, y, 0x07060302)};
#pragma unroll
        for (int j = 0; j < 4; ++j) *(u32 *)&turned[(tid & 15) * 8 + 4 * h + j][(tid >> 4) * 4] = col[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = i * 64 + (tid >> 3), part = (tid & 7) * 16;
        if (bx * 128 + c < d) *(u32x4 *)(t_codes + ((size_t)(bx * 128 + c) * t_nb + by) * 128 + part) = *(const u32x4 *)&turned[c][part];
    }
}

// ---- rows by id ------------------------------------------------------------------------------------------
// A lane per 16 bytes of an output row (4 or 8 coordinates: neighbouring lanes' stores touch), `group` lanes (a power of two)
// per row, or per piece of a row that a workgroup takes, and ROWS rows per lane, so that as many chains of id, codes, store run side
// by side.  Codes have at most four significant bits, so value * scale is exact; the factor's product is rounded to float32 and
// then once to the output's type.  Bound: HBM writes (65 536 x 4096 to bfloat16, 806 MB: 136 us, 5.9 TB/s; a wave per row that goes
// through its pieces took 160).
template <class T, int FORMAT, int ROWS, bool PAST_CACHE>
__global__ __launch_bounds__(256) void f8_rows_kernel(F8 t, int d, const int *ids, long long m, int group, int pieces, float factor, T *out)
{
    constexpr int kPer = 16 / sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
    const int per = 256 / group;
    const u32 rows = pieces == 1 ? blockIdx.x : blockIdx.x / pieces;
    const int p = (int)(blockIdx.x - rows * pieces) * group + (threadIdx.x & (group - 1));
    const long long first = (long long)rows * (per * ROWS) + threadIdx.x / group;
    if (p * kPer >= d) return;
    u32 word[ROWS][2], b[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const long long row = min(first + (long long)i * per, m - 1);
        const int id = ids ? ids[row] : (int)row;
        word[i][0] = word[i][1] = 0, b[i] = 256;                   // (an empty slot)
        if (id >= 0 && id < t.n) {
            const uint8_t *from = t.row(id) + p * kPer;
            if (kPer == 4) word[i][0] = *(const u32 *)from;
            else {
                const u32x2 x = *(const u32x2 *)from;
                word[i][0] = x.x, word[i][1] = x.y;
            }
            b[i] = t.scales[(size_t)id * t.sp + p * kPer / 128];
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
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

// ---- matrix instructions ---------------------------------------------------------------------------------
// Lane l of an instruction of 32 x 32 brings its part of row l % 32 of an operand: 32 bytes of a step of 64 coordinates for
// 8-bit operands, 8 numbers of a step of 16 for bfloat16.  Which coordinates the two halves of the lanes bring does not matter as
// long as both operands agree.  The result's lane l holds column l % 32 (of the second operand), rows 8 c + 4 (l / 32) + 0..3.
__device__ inline i32x8 both(i32x4 a, i32x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
template <int FA, int FB> __device__ inline f32x16 f8_mma(i32x4 a0, i32x4 a1, int a_scale, i32x4 b0, i32x4 b1, int b_scale, f32x16 c)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(both(a0, a1), both(b0, b1), c, FA, FB, 0, a_scale, 0, b_scale);
}

// Out through LDS, 32 rows of a wave's piece of 32 FA rows and 32 FB columns at a time, so that stores are whole rows of it.
template <class T, int FA, int FB>
__device__ inline void store_piece(const f32x16 (&acc)[FA][FB], char *lds, int lane, T *out, long long ldo, int rows, int columns)
{
    constexpr int kAcross = 32 * FB, kPitch = kAcross + 8, kPer = 16 / sizeof(T), kLanes = kAcross / kPer;      // lanes per row
    typedef T Out __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
    typedef T Turn __attribute__((ext_vector_type(4), aligned(8)));
    T *turn = (T *)lds;
    const int r = lane & 31, half = lane >> 5;
#pragma unroll
    for (int y = 0; y < FA; ++y) {
#pragma unroll
        for (int x = 0; x < FB; ++x)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *(Turn *)&turn[r * kPitch + 32 * x + 8 * c + 4 * half] =
                    Turn{from_float<T>(acc[y][x][4 * c]), from_float<T>(acc[y][x][4 * c + 1]), from_float<T>(acc[y][x][4 * c + 2]),
                         from_float<T>(acc[y][x][4 * c + 3])};
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        const int j = lane % kLanes * kPer, left = columns - j;
#pragma unroll
        for (int i = lane / kLanes; i < 32; i += 64 / kLanes) {
            if (32 * y + i >= rows) continue;
            T *o = out + (size_t)(32 * y + i) * ldo + j;
            const T *from = &turn[i * kPitch + j];
            if (left >= kPer) *(Out *)o = *(const Out *)from;
            else
                for (int c = 0; c < left; ++c) o[c] = from[c];
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
}

// Which tile (row, column of tiles) and part of the sum a workgroup takes: a chiplet (every eighth workgroup) gets a connected
// piece of them, part by part, in strips of eight rows of tiles, so that what runs there together shares operands in its L2.
struct Place {
    int y, x, part;
};
__device__ inline Place place_of(u32 id, int tiles_y, int tiles_x, int parts)
{
    const int tiles = tiles_y * tiles_x, all = tiles * parts, each = all / 8, more = all % 8, xcd = id & 7;
    int at = xcd * each + min(xcd, more) + (int)(id >> 3);
    const int part = parts > 1 ? at / tiles : 0;
    at -= part * tiles;
    const int strip = at / (8 * tiles_x), high = min(8, tiles_y - strip * 8), in = at - strip * 8 * tiles_x;
    return {strip * 8 + in % high, in / high, part};
}

// Sums of the parts, in their order: a lane per result, eight loads on their way (125 parts of 128 x 960: 10.6 us, 5.8 TB/s).
template <class T>
__global__ __launch_bounds__(256) void f8_join_kernel(const float *partial, int parts, u32 rows, u32 columns, T *out, long long ldo)
{
    const u32 row = blockIdx.y, c = blockIdx.x * 256 + threadIdx.x;
    if (c >= columns) return;
    const size_t step = (size_t)rows * columns;
    const float *from = partial + (size_t)row * columns + c;
    float sum = 0.0f;
    int p = 0;
    for (; p + 8 <= parts; p += 8, from += 8 * step) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = from[i * step];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i];
    }
    for (; p < parts; ++p, from += step) sum += *from;
    out[(size_t)row * ldo + c] = from_float<T>(sum);
}

template <class T>
int launch_join(const float *partial, int parts, int64_t rows, int64_t columns, T *out, int64_t ldo, hipStream_t st)
{
    const dim3 grid((unsigned)((columns + 255) / 256), (unsigned)rows);
    f8_join_kernel<T><<<grid, 256, 0, st>>>(partial, parts, (u32)rows, (u32)columns, out, ldo);
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
}

// ---- products --------------------------------------------------------------------------------------------
// out[i][j] = a_i . b_j.  The rows of b are the instruction's rows and those of a its columns, so that a lane ends up with
// consecutive values of an output row.

// WA x WB waves share a tile of a's rows by b's rows, FA x FB instructions of 32 x 32 each.  A stage is a block of both, whole
// lines of 128 bytes, and every fourth one brings the scales of four; while one is computed the next is on its way into LDS.  A
// load of codes brings 8 rows; the 16-byte pieces of row r lie in the order p ^ (r / 2) % 8, so that pieces p of 16 rows,
// which are read together, are in different ones of the 64 banks.
// The 8-bit matrix instructions multiply exactly, but cut each of eight products that they add first at 2^-14 of the largest of
// them (a product of 2^3 next to one of 2^17 is kept, one of 2^2 is not), which is below half a step of a 16-bit result wherever it is
// not much smaller than its terms, and too much for one of float32.  (8192^3 to bfloat16: 2.1 % of the results are a step beside the
// rounded exact sums, 0.01 % with sums of float32; the error against exact ones, 0.00166 of their norm, is the same.  1003 x 5001 x 960 to half
// precision: 2.7 % and 0.003 %, 0.0002078 and 0.0002074.)  WIDE, for those: codes are turned into bfloat16 numbers on their way
// from LDS, scales applied, and the bfloat16 instructions' sums are float32's (8192^3: 0.86 ms instead of 0.45).
// Bound: power.  8192^3 takes 0.45 ms, 2.4 PFLOP/s, at 1.87 GHz with the matrix units busy for 0.59 of the time (a library product of
// this size: 0.405); the same instructions on zeros run at 2.33 GHz, 0.37 ms.  Reading operands a piece of work ahead, as the gradient's
// kernel does, spills registers here (0.6 ms), and loads asked for before, between or after the reads make no difference.
template <int FA, int FB, int WA, int WB>
struct ProductTile {
    static constexpr int waves = WA * WB, side_a = 32 * FA * WA, side_b = 32 * FB * WB, sides = side_a + side_b;
    static constexpr int each = sides / 8 / waves, each_scales = sides / 64 / waves;      // loads of a wave
    static_assert(each_scales * 64 * waves == sides, "every wave loads as much");
    struct Lds {
        u32 codes[2][sides / 8][256];       // a's rows, then b's
        u32 scales[2][sides];               // of four blocks
    };
    static constexpr int turn_bytes = 32 * (32 * FB + 8) * 4;        // of a wave, at the end
    static constexpr int lds = (int)sizeof(Lds) > waves * turn_bytes ? (int)sizeof(Lds) : waves * turn_bytes;
};

template <bool WIDE, int FORMAT_A, int FORMAT_B, int FA, int FB, int WA, int WB>
__global__ __launch_bounds__(64 * WA * WB, FA * FB > 4 ? 1 : 2) void f8_product_tile_kernel(F8 a, F8 b, int dtype, void *out, long long ldo,
                                                                                           int tiles_a, int tiles_b, int parts, float *partial)
{
    typedef ProductTile<FA, FB, WA, WB> Tile;
    extern __shared__ __align__(16) char lds_raw[];
    typename Tile::Lds &lds = *(typename Tile::Lds *)lds_raw;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, half = lane >> 5;
    const Place at = place_of(blockIdx.x, tiles_a, tiles_b, parts);
    const int i0 = at.y * Tile::side_a, j0 = at.x * Tile::side_b;
    const int rows_a = a.n - i0, rows_b = b.n - j0;
    // a part is whole groups of four blocks
    const int fours = (a.nb + 3) / 4, s_lo = (int)((long long)fours * at.part / parts) * 4,
              s_hi = min((int)((long long)fours * (at.part + 1) / parts) * 4, a.nb);
    const uint8_t *codes_a = a.row(i0), *codes_b = b.row(j0), *scales_a = a.scales + (size_t)i0 * a.sp, *scales_b = b.scales + (size_t)j0 * b.sp;
    const auto row_of = [&](int row) { return (u32)(row < Tile::side_a ? min(row, rows_a - 1) : min(row - Tile::side_a, rows_b - 1)); };
    u32 at_codes[Tile::each], at_scales[Tile::each_scales];
#pragma unroll
    for (int i = 0; i < Tile::each; ++i) {
        const int row = (wave * Tile::each + i) * 8 + (lane >> 3);
        at_codes[i] = row_of(row) * a.nb * 128 + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    }
#pragma unroll
    for (int i = 0; i < Tile::each_scales; ++i) at_scales[i] = row_of((wave * Tile::each_scales + i) * 64 + lane) * a.sp;
    const auto load = [&](int stage, bool with_scales) {
        const uint8_t *from_a = codes_a + (size_t)stage * 128, *from_b = codes_b + (size_t)stage * 128;
        asm volatile("" : "+s"(from_a), "+s"(from_b));        // (or else every load's address stays in two registers)
#pragma unroll
        for (int i = 0; i < Tile::each; ++i) {
            const int op = wave * Tile::each + i;
            u32 at = at_codes[i];
            asm volatile("" : "+v"(at));        // (an offset of 32 bits: not kept as one of 64)
            stage_lds((op * 8 < Tile::side_a ? from_a : from_b) + at, &lds.codes[stage & 1][op][0], 1);
        }
        if (!with_scales) return;
#pragma unroll
        for (int i = 0; i < Tile::each_scales; ++i) {
            const int op = wave * Tile::each_scales + i;
            u32 at = at_scales[i];
            asm volatile("" : "+v"(at));
            stage_lds((op * 64 < Tile::side_a ? scales_a : scales_b) + stage + at, &lds.scales[(stage >> 2) & 1][op * 64], 0);
        }
    };
    f32x16 acc[FA][FB] = {};
    const int wa = wave % WA * 32 * FA, wb = wave / WA * 32 * FB;
    // where the lane's first piece is in a stage (other pieces: the offset ^ 16 p; 32 rows further down: 4096 bytes on)
    const int code_a = (wa + r) * 128 + (half ^ ((r >> 1) & 7)) * 16, code_b = code_a + (Tile::side_a + wb - wa) * 128;
    const auto piece = [&](int stage, int from, int p) { return *(const i32x4 *)((const char *)lds.codes[stage & 1] + (from ^ (16 * p))); };
    int sa[FA], sb[FB];
    const auto read_scales = [&](int stage) {
        const u32 *from = &lds.scales[(stage >> 2) & 1][r];
        const int shift = 8 * (stage & 3);
#pragma unroll
        for (int f = 0; f < FA; ++f) sa[f] = (int)(from[wa + 32 * f] >> shift);
#pragma unroll
        for (int f = 0; f < FB; ++f) sb[f] = (int)(from[Tile::side_a + wb + 32 * f] >> shift);
    };
    const auto multiply = [&](int stage) {
        read_scales(stage);
        if constexpr (WIDE) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                bf16x8 wide_b[FB][2];
#pragma unroll
                for (int f = 0; f < FB; ++f) sixteen_wide<FORMAT_B>(piece(stage, code_b + 4096 * f, 2 * p), scale_value(sb[f] & 255), wide_b[f]);
#pragma unroll
                for (int y = 0; y < FA; ++y) {
                    bf16x8 wide_a[2];
                    sixteen_wide<FORMAT_A>(piece(stage, code_a + 4096 * y, 2 * p), scale_value(sa[y] & 255), wide_a);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int x = 0; x < FB; ++x) acc[y][x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wide_b[x][h], wide_a[h], acc[y][x], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                i32x4 cb[FB][2], ca[FA][2];
#pragma unroll
                for (int f = 0; f < FB; ++f)
#pragma unroll
                    for (int q = 0; q < 2; ++q) cb[f][q] = piece(stage, code_b + 4096 * f, 4 * h + 2 * q);
#pragma unroll
                for (int f = 0; f < FA; ++f)
#pragma unroll
                    for (int q = 0; q < 2; ++q) ca[f][q] = piece(stage, code_a + 4096 * f, 4 * h + 2 * q);
#pragma unroll
                for (int y = 0; y < FA; ++y)
#pragma unroll
                    for (int x = 0; x < FB; ++x)
                        acc[y][x] = f8_mma<FORMAT_B, FORMAT_A>(cb[x][0], cb[x][1], sb[x], ca[y][0], ca[y][1], sa[y], acc[y][x]);
            }
        }
    };
    // a stage has arrived, and what was read of the one before it is in registers
    const auto arrived = [&]() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if (s_lo < s_hi) {
        load(s_lo, true);
        for (int stage = s_lo; stage < s_hi; ++stage) {
            arrived();
            if (stage + 1 < s_hi) load(stage + 1, ((stage + 1) & 3) == 0);
            multiply(stage);
        }
        arrived();
    }
    const size_t first_row = i0 + wa, first_col = j0 + wb;
    char *turn = lds_raw + wave * Tile::turn_bytes;
    if (parts > 1) store_piece<float>(acc, turn, lane, partial + ((size_t)at.part * a.n + first_row) * b.n + first_col, b.n, rows_a - wa, rows_b - wb);
    else if constexpr (WIDE) store_piece<float>(acc, turn, lane, (float *)out + first_row * ldo + first_col, ldo, rows_a - wa, rows_b - wb);
    else if (dtype == EFANNA_F16) store_piece<_Float16>(acc, turn, lane, (_Float16 *)out + first_row * ldo + first_col, ldo, rows_a - wa, rows_b - wb);
    else store_piece<__bf16>(acc, turn, lane, (__bf16 *)out + first_row * ldo + first_col, ldo, rows_a - wa, rows_b - wb);
}

// Few rows of one side, here a (16 M at most): bound by reading the other, b, once; step_a and step_b lead from a result to that of the
// next row of a and of b, one of them 1.  A workgroup takes 16 ROWS rows of b; its waves share the blocks, and
// their sums meet in LDS, in the waves' order.  Codes of both pass through LDS by direct loads, S blocks at a time (a load brings 8
// whole lines, ordered as in the tiles); operands are of 16 rows, lane l brings row l % 16 and the pieces l / 16 and l / 16 + 4.
// (16 rows against 8192 x 8192: 12 us, 5.7 TB/s; with a's operands straight from memory, rows apart in a load, 19; one row against
// 10^6 x 128: 19 us.)
template <int M, int ROWS, int S>
struct FewLds {
    u32 codes[S][2 * (ROWS + M)][256];       // b's rows, then a's
};
template <bool WIDE, int FORMAT_A, int FORMAT_B, int M, int ROWS, int S, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void f8_product_few_kernel(F8 a, F8 b, int dtype, void *out, long long step_a, long long step_b)
{
    static_assert(S <= 2, "a stage's scales are in one word");
    extern __shared__ __align__(16) char lds_raw[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    FewLds<M, ROWS, S> *lds = (FewLds<M, ROWS, S> *)lds_raw + wave;
    const int j0 = blockIdx.x * 16 * ROWS, left = b.n - j0;
    const int groups = (a.nb + S - 1) / S, s_lo = groups * wave / WAVES * S, s_hi = min(groups * (wave + 1) / WAVES * S, a.nb);
    const uint8_t *codes_b = b.row(j0);
    u32 at_b[2 * ROWS], at_a[2 * M];
    const int load_row = lane >> 3, load_piece = (lane & 7) ^ (load_row >> 1);      // of the rows 0 .. 7 of sixteen; 8 .. 15: the piece ^ 4
#pragma unroll
    for (int i = 0; i < 2 * ROWS; ++i) at_b[i] = (u32)min(8 * i + load_row, left - 1) * b.nb * 128 + (load_piece ^ (4 * (i & 1))) * 16;
#pragma unroll
    for (int i = 0; i < 2 * M; ++i) at_a[i] = (u32)min(8 * i + load_row, a.n - 1) * a.nb * 128 + (load_piece ^ (4 * (i & 1))) * 16;
    const uint8_t *scale_a[M], *scale_b[ROWS];
#pragma unroll
    for (int f = 0; f < M; ++f) scale_a[f] = a.scales + (size_t)min(16 * f + r, a.n - 1) * a.sp;
#pragma unroll
    for (int f = 0; f < ROWS; ++f) scale_b[f] = b.scales + (size_t)(j0 + min(16 * f + r, left - 1)) * b.sp;
    // where the lane's two pieces of its row are, within an operand of 16 rows
    const int first = r * 128 + (g ^ ((r >> 1) & 7)) * 16, second = first ^ 64;
    f32x4 acc[M][ROWS] = {};
    for (int s0 = s_lo; s0 < s_hi; s0 += S) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (S > 1 && s0 + s >= s_hi) break;
#pragma unroll
            for (int i = 0; i < 2 * ROWS; ++i) stage_lds(codes_b + (s0 + s) * 128 + at_b[i], &lds->codes[s][i][0], 1);
#pragma unroll
            for (int i = 0; i < 2 * M; ++i) stage_lds(a.codes + (s0 + s) * 128 + at_a[i], &lds->codes[s][2 * ROWS + i][0], 1);
        }
        u32 words_a[M], words_b[ROWS];
#pragma unroll
        for (int f = 0; f < M; ++f) words_a[f] = *(const u32 *)(scale_a[f] + (s0 & ~3)) >> (8 * (s0 & 3));
#pragma unroll
        for (int f = 0; f < ROWS; ++f) words_b[f] = *(const u32 *)(scale_b[f] + (s0 & ~3)) >> (8 * (s0 & 3));
        wait_loads<0>();
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (S > 1 && s0 + s >= s_hi) break;
            i32x4 y[M][2];
#pragma unroll
            for (int f = 0; f < M; ++f) {
                const char *from = (const char *)&lds->codes[s][2 * (ROWS + f)][0];
                y[f][0] = *(const i32x4 *)(from + first), y[f][1] = *(const i32x4 *)(from + second);
            }
#pragma unroll
            for (int t = 0; t < ROWS; ++t) {
                const char *from = (const char *)&lds->codes[s][2 * t][0];
                const i32x4 x[2] = {*(const i32x4 *)(from + first), *(const i32x4 *)(from + second)};
                const int x_scale = words_b[t] >> (8 * s) & 255;
                if constexpr (WIDE) {
                    bf16x8 wide_b[2][2];
#pragma unroll
                    for (int q = 0; q < 2; ++q) sixteen_wide<FORMAT_B>(x[q], scale_value(x_scale), wide_b[q]);
#pragma unroll
                    for (int f = 0; f < M; ++f)
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            bf16x8 wide_a[2];
                            sixteen_wide<FORMAT_A>(y[f][q], scale_value(words_a[f] >> (8 * s) & 255), wide_a);
#pragma unroll
                            for (int h = 0; h < 2; ++h) acc[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide_b[q][h], wide_a[h], acc[f][t], 0, 0, 0);
                        }
                } else
#pragma unroll
                    for (int f = 0; f < M; ++f)
                        acc[f][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(both(x[0], x[1]), both(y[f][0], y[f][1]), acc[f][t], FORMAT_B, FORMAT_A,
                                                                                     0, x_scale, 0, words_a[f] >> (8 * s) & 255);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (read before it is written again)
    }
    if (WAVES > 1) {
        f32x4 *share = (f32x4 *)lds_raw;          // [wave - 1][M * ROWS][lane]
        __syncthreads();
        if (wave > 0)
#pragma unroll
            for (int f = 0; f < M; ++f)
#pragma unroll
                for (int t = 0; t < ROWS; ++t) share[((wave - 1) * M * ROWS + f * ROWS + t) * 64 + lane] = acc[f][t];
        __syncthreads();
        if (wave > 0) return;
        for (int w = 0; w < WAVES - 1; ++w)
#pragma unroll
            for (int f = 0; f < M; ++f)
#pragma unroll
                for (int t = 0; t < ROWS; ++t) acc[f][t] += share[(w * M * ROWS + f * ROWS + t) * 64 + lane];
    }
    const auto store = [&](auto *to) {
        typedef typename std::remove_reference<decltype(*to)>::type T;
        typedef T Four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
#pragma unroll
        for (int f = 0; f < M; ++f)
#pragma unroll
            for (int t = 0; t < ROWS; ++t) {
                const int i = 16 * f + r, j = 16 * t + 4 * g;
                const f32x4 v = acc[f][t];
                if (i >= a.n || j >= left) continue;
                T *o = to + i * step_a + (j0 + j) * step_b;
                if (step_b == 1 && left - j >= 4) *(Four *)o = Four{from_float<T>(v[0]), from_float<T>(v[1]), from_float<T>(v[2]), from_float<T>(v[3])};
                else
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (c < left - j) o[c * step_b] = from_float<T>(v[c]);
            }
    };
    if constexpr (WIDE) store((float *)out);
    else if (dtype == EFANNA_F16) store((_Float16 *)out);
    else store((__bf16 *)out);
}

// Calls try_(parts, units of a part) for numbers of parts that a sum of `units` can be cut in: at most `fill`, or `most` where that is
// less, one at least.
template <class F> inline void least_of_parts(int64_t fill, int64_t units, int64_t most, F try_)
{
    if (fill < most) most = fill;
    if (most < 1) most = 1;
    for (int64_t p = 1;; p = p < 4 ? p + 1 : p * 5 / 4) {
        if (p > most) p = most;
        const int64_t each = units > p ? (units + p - 1) / p : 1;
        try_(units > 0 ? (units + each - 1) / each : 1, each);
        if (p == most) return;
    }
}

// How a product is cut: few rows of one side, or tiles of 128 or 256 a side, one of the larger or two of the smaller ones on a CU at a time,
// and in how many parts the sum: the least of estimated times, from what the kernels were measured at.  (1024 x 4096 x 4096 to bfloat16:
// 34 us in two parts of smaller tiles, 26 in one; 64 x 8192 x 8192 23 us in 8 parts, 20 in 4; 32 rows as few 15.7 us, in tiles 18.6.
// 10^6 x 1 x 128: 21 us as few rows, in tiles 68.)
struct ProductShape {
    bool few;
    int side, parts;
    size_t bytes;
};
constexpr int kFew = 32;
inline ProductShape product_shape(int64_t m, int64_t n, int32_t d, int32_t dtype)
{
    ProductShape best = {m <= kFew || n <= kFew, 128, 1, 0};
    if (best.few) return best;
    // microseconds of a block of 128 coordinates; of the smaller tiles where they are a CU's only ones, too
    const double large = dtype == EFANNA_F32 ? 3.4 : 1.8, small = dtype == EFANNA_F32 ? 2.1 : 1.2, alone = dtype == EFANNA_F32 ? 1.05 : 0.65;
    const int64_t fours = (f8_blocks(d) + 3) / 4;
    double least = 1e300;
    for (int side = 128; side <= 256; side += 128) {
        const int64_t tiles = ((m + side - 1) / side) * ((n + side - 1) / side), at_once = side == 128 ? 512 : 256;
        least_of_parts(at_once / tiles, fours, fours / 2, [&](int64_t parts, int64_t each) {
            const double rounds = (double)((tiles * parts + at_once - 1) / at_once);
            double time = rounds * (5.0 + (double)each * 4 * (side == 256 ? large : tiles * parts <= 256 ? alone : small));
            if (parts > 1) time += 3.0 + (double)parts * m * n * 8.0 / 4e6;      // written and read again
            if (time < least) {
                least = time;
                best.side = side, best.parts = (int)parts;
                best.bytes = parts > 1 ? align_up((size_t)parts * m * n * sizeof(float)) : 0;
            }
        });
    }
    return best;
}
template <bool WIDE, int FORMAT_A, int FORMAT_B, int FA, int FB, int WA, int WB>
int launch_tiles(const F8 &a, const F8 &b, int dtype, void *out, int64_t ldo, int parts, float *partial, hipStream_t st)
{
    typedef ProductTile<FA, FB, WA, WB> Tile;
    const int64_t ta = ((int64_t)a.n + Tile::side_a - 1) / Tile::side_a, tb = ((int64_t)b.n + Tile::side_b - 1) / Tile::side_b;
    if (ta * tb * parts > 2147483647LL || !launch_fits(ta * tb * parts, Tile::waves * 64)) return EFANNA_EUNSUPPORTED;
    EF_HIP_CHECK(allow_lds((const void *)f8_product_tile_kernel<WIDE, FORMAT_A, FORMAT_B, FA, FB, WA, WB>, Tile::lds));
    f8_product_tile_kernel<WIDE, FORMAT_A, FORMAT_B, FA, FB, WA, WB><<<(unsigned)(ta * tb * parts), Tile::waves * 64, Tile::lds, st>>>(
        a, b, dtype, out, ldo, (int)ta, (int)tb, parts, partial);
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
}
template <bool WIDE, int FORMAT_A, int FORMAT_B, int M, int ROWS, int S, int WAVES>
int launch_few(const F8 &a, const F8 &b, int dtype, void *out, int64_t step_a, int64_t step_b, hipStream_t st)
{
    const int stage = WAVES * (int)sizeof(FewLds<M, ROWS, S>), join = (WAVES - 1) * M * ROWS * 64 * 16, lds = stage > join ? stage : join;
    EF_HIP_CHECK(allow_lds((const void *)f8_product_few_kernel<WIDE, FORMAT_A, FORMAT_B, M, ROWS, S, WAVES>, lds));
    const int64_t slice = kSliceBlocks * 16 * ROWS * 4 / WAVES;      // rows of a launch
    for (int64_t first = 0; first < b.n; first += slice) {
        const int64_t here = b.n - first < slice ? b.n - first : slice;
        const F8 from = {b.codes + (size_t)first * b.nb * 128, b.scales + (size_t)first * b.sp, (int)here, b.nb, b.sp};
        f8_product_few_kernel<WIDE, FORMAT_A, FORMAT_B, M, ROWS, S, WAVES><<<(unsigned)((here + 16 * ROWS - 1) / (16 * ROWS)), 64 * WAVES, lds, st>>>(
            a, from, dtype, (char *)out + first * step_b * (dtype == EFANNA_F32 ? 4 : 2), step_a, step_b);
        EF_HIP_CHECK(hipGetLastError());
    }
    return EFANNA_OK;
}
template <bool WIDE, int FORMAT_A, int FORMAT_B, int M>
int launch_few_of(const F8 &a, const F8 &b, int dtype, void *out, int64_t step_a, int64_t step_b, hipStream_t st)
{
    if (a.nb < 4) return launch_few<WIDE, FORMAT_A, FORMAT_B, M, 4, 1, 1>(a, b, dtype, out, step_a, step_b, st);
    // (more waves for a sum where there are few rows of b; where they fill the GPU, 8192 x 8192, both take as long)
    if (a.nb < 16 || b.n > 4096) return launch_few<WIDE, FORMAT_A, FORMAT_B, M, 1, 2, 4>(a, b, dtype, out, step_a, step_b, st);
    return launch_few<WIDE, FORMAT_A, FORMAT_B, M, 1, 2, 8>(a, b, dtype, out, step_a, step_b, st);
}
template <bool WIDE, int FORMAT_A, int FORMAT_B>
int launch_product(const F8 &a, const F8 &b, int dtype, void *out, int64_t ldo, const ProductShape &sh, float *partial, hipStream_t st)
{
    if (sh.few && a.n <= kFew) return a.n <= 16 ? launch_few_of<WIDE, FORMAT_A, FORMAT_B, 1>(a, b, dtype, out, ldo, 1, st)
                                                : launch_few_of<WIDE, FORMAT_A, FORMAT_B, 2>(a, b, dtype, out, ldo, 1, st);
    if (sh.few) return b.n <= 16 ? launch_few_of<WIDE, FORMAT_B, FORMAT_A, 1>(b, a, dtype, out, 1, ldo, st)
                                 : launch_few_of<WIDE, FORMAT_B, FORMAT_A, 2>(b, a, dtype, out, 1, ldo, st);
    return sh.side == 256 ? launch_tiles<WIDE, FORMAT_A, FORMAT_B, 4, 2, 2, 4>(a, b, dtype, out, ldo, sh.parts, partial, st)
                          : launch_tiles<WIDE, FORMAT_A, FORMAT_B, 2, 2, 2, 2>(a, b, dtype, out, ldo, sh.parts, partial, st);
}

// ---- gradient of the weights -----------------------------------------------------------------------------
// A number as a sum of bfloat16 numbers, exactly (float32 from 2^-110 on): one of its own kind, two of half precision (11
// bits), three of float32 (24 bits).  A part is the upper half of what is left as a float32 number, eight bits of it.  An
// infinity is all in the first part.
template <class Y> struct Parts {
    static constexpr int count = sizeof(Y) == 4 ? 3 : 2;
    template <class Eight> static __device__ inline void split(Eight v, bf16x8 (&p)[count])
    {
        u32 left[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) left[k] = __float_as_uint((float)v[k]);
#pragma unroll
        for (int q = 0; q < count; ++q) {
            u32x4 halves;
#pragma unroll
            for (int k = 0; k < 4; ++k) halves[k] = __builtin_amdgcn_perm(left[2 * k + 1], left[2 * k], 0x07060302);
            p[q] = __builtin_bit_cast(bf16x8, halves);
            if (q + 1 < count)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float x = __uint_as_float(left[k]), rest = x - __uint_as_float(left[k] & 0xFFFF0000u);
                    left[k] = __float_as_uint(q == 0 && __builtin_amdgcn_classf(x, 0x204) ? 0.0f : rest);
                }
        }
    }
};
template <> struct Parts<__bf16> {
    static constexpr int count = 1;
    template <class Eight> static __device__ inline void split(Eight x, bf16x8 (&p)[1]) { p[0] = (bf16x8)x; }
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

// WY x WX waves share a tile of dY's columns by the table's, FY x FX instructions of 32 x 32 x 16 each, and STEP rows are a
// stage.  Both operands are wanted by columns and lie in rows: rows go to LDS as bfloat16 numbers (dY in its parts, codes with
// their scale applied, through registers, where AHEAD stages are on their way) and come back through transposing reads, of which a
// lane gets four rows' values of its column.
// Bound: power and the vector and LDS work between matrix instructions.  16 384 rows, 4096 x 4096, bfloat16: 0.47 ms, 1.17 PFLOP/s, at
// 1.84 GHz with the matrix units busy for 0.57 (zeros: 2.2 GHz, 0.41 ms; a library product of two bfloat16 matrices: 0.37); without
// putting stages down 0.39, without reading operands either 0.31.  Rows of dY straight into LDS or three stages of them were no faster;
// 64 rows a stage pay for the two smaller tiles only, the square one's spill, and so do waves of 128 x 128.
// A row's pieces of 16 columns (32 bytes) lie in the order u ^ turn_of(row), so that the eight rows that a read touches are in different
// banks (rows of 64 columns are four pieces: two of the eight rows in the same ones).
template <int ACROSS> __device__ inline int turn_of(int row) { return (2 * (row & 3) + ((row >> 2) & 1)) & (ACROSS / 16 - 1); }

// (a closure that is called twice and not inlined keeps what it captures, the accumulators too, in memory)
#define EF_INLINE __attribute__((always_inline))

template <class Y, int FY, int FX, int WY, int WX, int STEP>
struct GradientTile {
    static constexpr int waves = WY * WX, threads = 64 * waves, across_y = 32 * FY * WY, across_x = 32 * FX * WX, parts = Parts<Y>::count;
    static constexpr int pieces_y = across_y / 8 * STEP / threads, pieces_x = across_x / 16 * STEP / threads;      // of a thread
    static_assert(pieces_y * threads * 8 == across_y * STEP && pieces_x * threads * 16 == across_x * STEP, "every thread loads as much");
    struct Lds {
        __bf16 y[2][parts][STEP][across_y], x[2][STEP][across_x];
    };
    static constexpr int turn_bytes = 32 * (32 * FX + 8) * 4;        // of a wave, at the end
    static constexpr int lds = (int)sizeof(Lds) > waves * turn_bytes ? (int)sizeof(Lds) : waves * turn_bytes;
};

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

template <class Y, int FORMAT, int FY, int FX, int WY, int WX, int STEP, int AHEAD>
__global__ __launch_bounds__(64 * WY * WX, 2) void f8_gradient_kernel(const Y *dy, long long ldy, long long m, int n, F8 x, int d,
                                                                                       int dtype, void *out, long long ldo, int tiles_y,
                                                                                       int tiles_x, int parts, float *partial)
{
    typedef GradientTile<Y, FY, FX, WY, WX, STEP> Tile;
    typedef Y Eight __attribute__((ext_vector_type(8), aligned(sizeof(Y))));
    extern __shared__ __align__(16) char lds_raw[];
    typename Tile::Lds &lds = *(typename Tile::Lds *)lds_raw;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const Place at = place_of(blockIdx.x, tiles_y, tiles_x, parts);
    const int j0 = at.y * Tile::across_y, c0 = at.x * Tile::across_x;
    const long long all = (m + STEP - 1) / STEP, s_lo = all * at.part / parts, first = s_lo * STEP;
    const int stages = (int)(all * (at.part + 1) / parts - s_lo);
    const int rows_in = (int)min(m - first, (long long)stages * STEP);      // this part's rows: 0 .. rows_in - 1 from `first` on

    // A stage on its way.  Rows past the last one are loaded from it and put down as zeros; a stage past the last is loaded again
    // (nothing reads it).  Offsets within a stage are below 2^32.
    Eight raw_y[AHEAD][Tile::pieces_y];
    i32x4 raw_x[AHEAD][Tile::pieces_x];
    u32 raw_scale[AHEAD][Tile::pieces_x];
    const Y *dy0 = dy + first * ldy;
    const uint8_t *codes0 = x.row(first), *scales0 = x.scales + (size_t)first * x.sp;
    // (pieces past the last column, and the one that it is in, are loaded as the last eight columns and put in their place later; a
    // matrix of fewer columns is read one by one)
    const bool pieces_whole = n % 8 == 0;
    const int col_y = tid % (Tile::across_y / 8) * 8, row_y = tid / (Tile::across_y / 8), rows_y = Tile::threads / (Tile::across_y / 8);
    const int from_col = piece_from(j0 + col_y, n);      // 0 at least
    const int piece_x = min(c0 / 16 + tid % (Tile::across_x / 16), x.nb * 8 - 1), row_x = tid / (Tile::across_x / 16),
              rows_x = Tile::threads / (Tile::across_x / 16);
    const auto load_y = [&](int stage, int set, int i, auto inside) EF_INLINE {
        const int at = min(stage, stages - 1) * STEP, row = min(row_y + rows_y * i, rows_in - 1 - at);
        const Y *from = dy0 + at * ldy;
        const u32 offset = (u32)row * (u32)ldy;
        if (inside || n >= 8) raw_y[set][i] = *(const Eight *)(from + (offset + from_col));
        else
#pragma unroll
            for (int k = 0; k < 8; ++k) raw_y[set][i][k] = from[offset + piece_column(k, n)];
    };
    const auto load_x = [&](int stage, int set, int i) EF_INLINE {
        const int at = min(stage, stages - 1) * STEP, row = min(row_x + rows_x * i, rows_in - 1 - at);
        raw_x[set][i] = *(const i32x4 *)(codes0 + (size_t)at * x.nb * 128 + ((u32)row * x.nb * 128 + piece_x * 16));
        raw_scale[set][i] = *(const u32 *)(scales0 + (size_t)at * x.sp + ((u32)row * x.sp + (piece_x >> 5) * 4));
    };
    const int shift_x = 8 * ((piece_x >> 3) & 3);
    const auto put_y = [&](int stage, int set, int buffer, int i, auto inside) EF_INLINE {
        const int piece = col_y / 8, row = row_y + rows_y * i;
        const bool live = stage * STEP + row < rows_in;
        bf16x8 part[Tile::parts];
        Eight x = live ? raw_y[set][i] : (Eight)(Y)0.0f;
        if (!inside) x = moved_down<Y>(x, piece_moved(j0 + col_y, n));
        Parts<Y>::split(x, part);
#pragma unroll
        for (int q = 0; q < Tile::parts; ++q) *(bf16x8 *)&lds.y[buffer][q][row][((piece >> 1) ^ turn_of<Tile::across_y>(row)) * 16 + (piece & 1) * 8] = part[q];
    };
    const auto put_x = [&](int stage, int set, int buffer, int i) EF_INLINE {
        const int piece = tid % (Tile::across_x / 16), row = row_x + rows_x * i;
        const bool live = stage * STEP + row < rows_in;
        bf16x8 wide[2];
        u32 word = raw_scale[set][i];
        asm volatile("" : "+v"(word));
        const u32 scale = (word >> shift_x) & 255;
        // (the second four lanes of eight write their second half first: a write's 16 bytes per lane are in different banks)
        const bool swap = tid & 4;
        const i32x4 c = live ? raw_x[set][i] : i32x4{0, 0, 0, 0};
        sixteen_wide<FORMAT>(swap ? i32x4{c.z, c.w, c.x, c.y} : c, scale_value(live ? scale : 127), wide);
        __bf16 *to = &lds.x[buffer][row][(piece ^ turn_of<Tile::across_x>(row)) * 16 + (swap ? 8 : 0)];
        *(bf16x8 *)to = wide[0];
        *(bf16x8 *)(to + (swap ? -8 : 8)) = wide[1];
    };

    f32x16 acc[FY][FX] = {};
    const int wy = wave % WY, wx = wave / WY;
    // a lane's part of a transposing read: row 4 half + (lane / 4) % 4 of eight, a quarter of the piece of its 16 lanes
    const int row = 4 * half + ((lane >> 2) & 3), group = (lane >> 4) & 1, quarter = (lane & 3) * 4;
    int at_y[FY], at_x[FX];
#pragma unroll
    for (int f = 0; f < FY; ++f) at_y[f] = row * Tile::across_y + (((wy * FY + f) * 2 + group) ^ turn_of<Tile::across_y>(row)) * 16 + quarter;
#pragma unroll
    for (int f = 0; f < FX; ++f) at_x[f] = row * Tile::across_x + (((wx * FX + f) * 2 + group) ^ turn_of<Tile::across_x>(row)) * 16 + quarter;
    const auto columns = [](const __bf16 *from, int pitch) {      // sixteen rows' values of the lane's column, as an operand
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)from);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(from + 8 * pitch));
        return __builtin_bit_cast(bf16x8, (i16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // A stage is kUnits pieces of work, sixteen rows and a part of dY each; the next one's operands are read before one is done.
    constexpr int kUnits = STEP / 16 * Tile::parts;
    bf16x8 fx[2][FX], fy[2][FY];
    const auto read = [&](int buffer, int unit, int to) EF_INLINE {
        const int k = unit / Tile::parts * 16, q = unit % Tile::parts;
        if (q == 0)
#pragma unroll
            for (int f = 0; f < FX; ++f) fx[unit / Tile::parts & 1][f] = columns(&lds.x[buffer][k][0] + at_x[f], Tile::across_x);
#pragma unroll
        for (int f = 0; f < FY; ++f) fy[to][f] = columns(&lds.y[buffer][q][k][0] + at_y[f], Tile::across_y);
    };
    const auto multiply = [&](int unit, int from) EF_INLINE {
        const int q = unit % Tile::parts, k = unit / Tile::parts & 1;
        if (q == 1)
#pragma unroll
            for (int b = 0; b < FX; ++b) fx[k][b] = without_infinities(fx[k][b]);
#pragma unroll
        for (int a = 0; a < FY; ++a)
#pragma unroll
            for (int b = 0; b < FX; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[k][b], fy[from][a], acc[a][b], 0, 0, 0);
    };
    const auto meet = [&]() {          // what was written to LDS is there, what was read has arrived
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    static_assert(kUnits % 2 == 0 && AHEAD <= 2, "operands and sets alternate");
    constexpr int kPieces = Tile::pieces_x + Tile::pieces_y;
    const auto run = [&](auto inside) EF_INLINE {      // INSIDE: whole pieces of dY, without a look at where its rows end
        const auto load = [&](int stage, int set, int i) EF_INLINE {
            if (i < Tile::pieces_x) load_x(stage, set, i);
            else load_y(stage, set, i - Tile::pieces_x, inside);
        };
        const auto put = [&](int stage, int set, int buffer, int i) EF_INLINE {
            if (i < Tile::pieces_x) put_x(stage, set, buffer, i);
            else put_y(stage, set, buffer, i - Tile::pieces_x, inside);
        };
#pragma unroll
        for (int i = 0; i < kPieces; ++i) load(0, 0, i);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) put(0, 0, 0, i);
#pragma unroll
        for (int s = 1; s <= AHEAD; ++s)
#pragma unroll
            for (int i = 0; i < kPieces; ++i) load(s, s % AHEAD, i);
        meet();
        read(0, 0, 0);
        for (int stage = 0;; stage += 2) {
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
#pragma unroll
                for (int u = 0; u < kUnits - 1; ++u) {
                    read(odd, u + 1, (u + 1) & 1);
                    multiply(u, u & 1);
                    // the next stage is put down and another one asked for, a share of it with each piece of work but the last
#pragma unroll
                    for (int i = kPieces * u / (kUnits - 1); i < kPieces * (u + 1) / (kUnits - 1); ++i) {
                        put(stage + odd + 1, (odd + 1) % AHEAD, 1 - odd, i);
                        load(stage + odd + 1 + AHEAD, (odd + 1) % AHEAD, i);
                    }
                    // (between two matrix instructions there is room for so many others)
#pragma unroll
                    for (int i = 0; i < FY * FX; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);      // matrix
                        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);      // reads of LDS
                        __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);      // vector
                        __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);      // writes of LDS
                        __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
                        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);      // loads
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                meet();
                read(1 - odd, 0, 0);                  // (after the last stage: what was put down as one past it)
                multiply(kUnits - 1, 1);
                __builtin_amdgcn_sched_barrier(0);
                if (stage + odd + 1 >= stages) return;
            }
        }
    };
    if (stages > 0) {
        if (pieces_whole || j0 + Tile::across_y <= n) run(std::true_type());
        else run(std::false_type());
        meet();
    }
    const int rows = n - j0 - wy * FY * 32, cols = d - c0 - wx * FX * 32;
    const size_t first_row = j0 + wy * FY * 32, first_col = c0 + wx * FX * 32;
    char *turn = lds_raw + wave * Tile::turn_bytes;
    if (parts > 1) store_piece<float>(acc, turn, lane, partial + ((size_t)at.part * n + first_row) * d + first_col, d, rows, cols);
    else
        EF_DTYPE(dtype, T, store_piece<T>(acc, turn, lane, (T *)out + first_row * ldo + first_col, ldo, rows, cols));
}

// How a gradient is cut: which tile, and in how many parts the sum.  The larger tiles move half as much per operation, one at a time
// on a CU; the wide one is for few columns of dY; two of the small ones run on a CU and leave half as many sums to be joined, and the
// narrow one is for what would leave half of them empty.  The choice is the least of estimated times, from what the kernels were measured at.
// (100 000 x 128 x 960 in float32: small tiles in 64 parts 110 us and 6 for their sums, wide ones in 125 parts 79 and 11; 1000 x 50 x 300 in
// half precision: small tiles in 16 parts 7.8 and 2, in 4 parts 12, narrow ones in 16 parts 6.3 and 2; 8410 x 56 x 4585 in 14
// parts: small tiles 24.0, narrow ones 18.6.)
enum GradientKind { kSquare, kWide, kSmall, kNarrow };
struct GradientShape {
    int kind, parts;
    size_t bytes;
};
inline GradientShape gradient_shape(int64_t m, int32_t n, int32_t d, int32_t dtype)
{
    struct Kind {
        int y, x, at_once;             // sides, workgroups that run at once
        double stage[3];               // microseconds of 32 rows, by parts of an element of dY
    };
    static const Kind kinds[4] = {{256, 256, 256, {0.95, 1.75, 3.2}}, {128, 512, 256, {1.05, 1.9, 2.9}}, {128, 128, 512, {0.7, 1.3, 2.1}},
                                  {64, 128, 512, {0.5, 0.9, 1.45}}};
    const int p = dtype == EFANNA_F32 ? 2 : dtype == EFANNA_F16 ? 1 : 0;
    const int64_t stages = (m + 31) / 32;
    GradientShape best = {kSmall, 1, 0};
    double least = 1e300;
    for (int k = 0; k < 4; ++k) {
        const int64_t tiles = (int64_t)((n + kinds[k].y - 1) / kinds[k].y) * ((d + kinds[k].x - 1) / kinds[k].x);
        least_of_parts(kinds[k].at_once / tiles, stages, stages / 2, [&](int64_t parts, int64_t each) {
            const int64_t rounds = (tiles * parts + kinds[k].at_once - 1) / kinds[k].at_once;
            const double alone = 2 * tiles * parts <= kinds[k].at_once && k >= kSmall ? 0.65 : 1.0;      // a CU's only one
            double time = rounds * (6.0 + (double)each * kinds[k].stage[p] * alone);
            if (parts > 1) time += 3.0 + (double)parts * n * d * 8.0 / 4e6;      // written and read again
            if (time < least) {
                least = time;
                best = {k, (int)parts, parts > 1 ? align_up((size_t)parts * n * d * sizeof(float)) : 0};
            }
        });
    }
    return best;
}

template <class Y, int FORMAT, int FY, int FX, int WY, int WX, int STEP, int AHEAD>
int launch_gradient(const Y *dy, int64_t ldy, int64_t m, int n, const F8 &x, int d, int dtype, void *out, int64_t ldo, int parts,
                    float *partial, hipStream_t st)
{
    typedef GradientTile<Y, FY, FX, WY, WX, STEP> Tile;
    const int ty = (n + Tile::across_y - 1) / Tile::across_y, tx = (d + Tile::across_x - 1) / Tile::across_x;
    EF_HIP_CHECK(allow_lds((const void *)f8_gradient_kernel<Y, FORMAT, FY, FX, WY, WX, STEP, AHEAD>, Tile::lds));
    f8_gradient_kernel<Y, FORMAT, FY, FX, WY, WX, STEP, AHEAD><<<(unsigned)(ty * tx * parts), Tile::threads, Tile::lds, st>>>(
        dy, ldy, m, n, x, d, dtype, out, ldo, ty, tx, parts, partial);
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
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
    const int nb = f8_blocks(d), sp = f8_scale_pitch(d), words = sp / 4, group = d <= 64 ? 8 : nb == 1 ? 16 : nb == 2 ? 32 : 64;
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
    EF_DTYPE(dtype, T, EF_FORMAT(format, F, (f8_weights_kernel<T, F><<<grid, 512, 0, (hipStream_t)stream>>>(
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
    const int per = dtype == EFANNA_F32 ? 4 : 8, across = (d + per - 1) / per;      // coordinates of a lane, lanes of a row
    const bool past_cache = m * d * (16 / per) > kStreamBytes;
    int group = 1;
    while (group < 256 && group < across) group <<= 1;
    const int pieces = (across + group - 1) / group;
    const int each = m * pieces <= 2048 * (256 / group) ? 1 : 4;      // rows of a lane: one where four would leave CUs without work
    const int64_t rows = each * (256 / group), slice = kSliceBlocks / pieces * rows;      // rows of a workgroup, of a launch
    for (int64_t first = 0; first < m; first += slice) {
        const int64_t here = m - first < slice ? m - first : slice;
        const unsigned blocks = (unsigned)((here + rows - 1) / rows * pieces);
        // (without ids the slice's rows are a table of their own)
        const F8 from = ids ? t : F8{codes + (size_t)first * t.nb * 128, scales + (size_t)first * t.sp, (int)(n - first), t.nb, t.sp};
        const int *slice_ids = ids ? ids + first : nullptr;
        EF_DTYPE(dtype, T, EF_FORMAT(format, F, {
            const auto kernel = each == 1 ? f8_rows_kernel<T, F, 1, false> : past_cache ? f8_rows_kernel<T, F, 4, true> : f8_rows_kernel<T, F, 4, false>;
            kernel<<<blocks, 256, 0, st>>>(from, d, slice_ids, here, group, pieces, factor, (T *)out + (size_t)first * d);
        }));
        EF_HIP_CHECK(hipGetLastError());
    }
    return EFANNA_OK;
}

extern "C" size_t efanna_f8_product_workspace_bytes(int64_t m, int64_t n, int32_t d, int32_t dtype)
{
    if (m < 1 || m > kMaxRows || n < 1 || n > kMaxRows || d < 1 || d > EFANNA_F8_MAX_D || !dtype_ok(dtype)) return 0;
    return product_shape(m, n, d, dtype).bytes;
}

extern "C" int efanna_f8_product(const uint8_t *a_codes, const uint8_t *a_scales, int32_t a_format, int64_t m,
                                 const uint8_t *b_codes, const uint8_t *b_scales, int32_t b_format, int64_t n, int32_t d,
                                 int32_t dtype, void *out, int64_t ldo, void *ws, size_t ws_bytes, void *stream)
{
    if (!dtype_ok(dtype) || !table_ok(a_codes, a_scales, a_format, m, d) || !table_ok(b_codes, b_scales, b_format, n, d) || ldo < n)
        return EFANNA_EINVAL;
    if (m == 0 || n == 0) return EFANNA_OK;
    if (!out || !aligned_for(out, dtype)) return EFANNA_EINVAL;
    const ProductShape sh = product_shape(m, n, d, dtype);
    if (!workspace_ok(ws, ws_bytes, sh.bytes)) return EFANNA_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const int nb = f8_blocks(d), sp = f8_scale_pitch(d);
    const F8 a = {a_codes, a_scales, (int)m, nb, sp}, b = {b_codes, b_scales, (int)n, nb, sp};
    int rc = EFANNA_OK;
    EF_FORMAT(a_format, FA, EF_FORMAT(b_format, FB, {
        if (dtype == EFANNA_F32) rc = launch_product<true, FA, FB>(a, b, dtype, out, ldo, sh, (float *)ws, st);
        else rc = launch_product<false, FA, FB>(a, b, dtype, out, ldo, sh, (float *)ws, st);
    }));
    if (rc != EFANNA_OK || sh.parts == 1) return rc;
    EF_DTYPE(dtype, T, rc = launch_join<T>((const float *)ws, sh.parts, m, n, (T *)out, ldo, st));
    return rc;
}

extern "C" size_t efanna_f8_gradient_workspace_bytes(int64_t m, int32_t n, int32_t d, int32_t dtype)
{
    if (m < 0 || m > kMaxRows || n < 1 || n > EFANNA_F8_MAX_D || d < 1 || d > EFANNA_F8_MAX_D || !dtype_ok(dtype)) return 0;
    return gradient_shape(m, n, d, dtype).bytes;
}

extern "C" int efanna_f8_gradient(const void *dY, int32_t dtype, int64_t m, int32_t n, int64_t ldy, const uint8_t *codes,
                                  const uint8_t *scales, int32_t format, int32_t d, int32_t out_dtype, void *out,
                                  int64_t ldo, void *ws, size_t ws_bytes, void *stream)
{
    if (!dtype_ok(dtype) || !dtype_ok(out_dtype) || !table_ok(codes, scales, format, m, d) || n < 0 || n > EFANNA_F8_MAX_D || ldy < n || ldo < d)
        return EFANNA_EINVAL;
    if (n == 0) return EFANNA_OK;
    if (ldy >= EFANNA_F8_MAX_LDY) return EFANNA_EUNSUPPORTED;
    if ((m > 0 && !dY) || !out || !aligned_for(dY, dtype) || !aligned_for(out, out_dtype)) return EFANNA_EINVAL;
    const GradientShape sh = gradient_shape(m, n, d, dtype);
    if (!workspace_ok(ws, ws_bytes, sh.bytes)) return EFANNA_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const F8 x = {codes, scales, (int)m, f8_blocks(d), f8_scale_pitch(d)};
    int rc = EFANNA_OK;
    EF_DTYPE(dtype, Y, EF_FORMAT(format, F, {
        // (stages of 64 rows where dY is one part: 16 384 x 1024 x 1024 51 us instead of 56; the square tiles' would spill)
        constexpr int ahead = Parts<Y>::count == 3 ? 1 : 2, step = Parts<Y>::count == 1 ? 64 : 32, few_ahead = step == 64 ? 1 : 2;
        const auto run = sh.kind == kSquare ? launch_gradient<Y, F, 4, 2, 2, 4, 32, ahead>
                         : sh.kind == kWide ? launch_gradient<Y, F, 4, 2, 1, 8, 32, ahead>
                         : sh.kind == kSmall ? launch_gradient<Y, F, 2, 2, 2, 2, step, few_ahead>
                                             : launch_gradient<Y, F, 1, 2, 2, 2, step, few_ahead>;
        rc = run((const Y *)dY, ldy, m, n, x, d, out_dtype, out, ldo, sh.parts, (float *)ws, st);
    }));
    if (rc != EFANNA_OK || sh.parts == 1) return rc;
    EF_DTYPE(out_dtype, T, rc = launch_join<T>((const float *)ws, sh.parts, n, d, (T *)out, ldo, st));
    return rc;
}
