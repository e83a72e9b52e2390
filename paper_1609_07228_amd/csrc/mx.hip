// Tables of vectors in microscaled 4-bit floating point (MXFP4) for gfx950: quantisation, rows by id,
// products of two tables and the k nearest rows of one table to the rows of another.
//
// Format.  A row of d coordinates is nb = ceil(d / 32) blocks.  A block has a scale byte b, the power
// 2^(b - 127), and 32 codes of 4 bits (sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6),
// 16 bytes with the even coordinate in the low half.  codes: n x 16 nb bytes; scales: n x sp bytes, sp = nb
// rounded up to 4, so that four blocks' scales can be read as one word; norms: squared length of the row as held.
//
// A block is what one lane hands v_mfma_scale_f32_16x16x128_f8f6f4 as its part of an operand: lane l holds
// block 4 s + l / 16 of row l % 16 in step s, and its scale byte.  Row-major codes are therefore operands
// without any rearrangement, 16 bytes per lane and step.  The unit multiplies exactly and adds in float32.
#include "common.h"

#include <type_traits>

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kFp4 = 4;                    // the operand format's number in the matrix instruction
constexpr size_t kMaxWorkspace = (size_t)1 << 30;

__host__ __device__ inline int mx_blocks(int d) { return (d + 31) >> 5; }
__host__ __device__ inline int mx_scale_pitch(int d) { return (mx_blocks(d) + 3) & ~3; }
inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

struct Table {
    const uint8_t *codes, *scales;
    const float *norms;
    int n, nb, sp;
};

// 2^(b - 127); 255 stands for NaN
__device__ inline float mx_scale(u32 b)
{
    return __uint_as_float(b == 0 ? 0x00400000u : b == 255 ? 0x7FC00000u : b << 23);
}

// ---- element types -------------------------------------------------------------------------------------
template <class T> __device__ inline float to_float(T x) { return (float)x; }
template <class T> __device__ inline T from_float(float x) { return (T)x; }      // to nearest, ties to even

// ---- quantisation ----------------------------------------------------------------------------------------
// Four lanes per block, eight coordinates each; a row's lanes are `group` consecutive ones (a power of two), so
// a wave holds 64 / group rows and the row's squared length is a sum over those lanes.  Bound: HBM.
template <class T>
__global__ __launch_bounds__(256) void quantise_kernel(const T *X, long long n, int d, long long ldx, int group, int nb,
                                                       int sp, uint8_t *codes, uint8_t *scales, float *norms)
{
    const int lane = threadIdx.x & (group - 1);
    const long long row = ((long long)blockIdx.x * 256 + threadIdx.x) / group;
    if (row >= n) return;
    const T *x = X + row * ldx;
    float norm = 0.0f;
    const int pieces = 4 * sp;                 // lanes past the last block write the scales' padding
    for (int p = lane; p < pieces; p += group) {
        const int j0 = p * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j0 + j < d ? to_float(x[j0 + j]) : 0.0f;
        u32 top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
        top = max(top, (u32)__shfl_xor((int)top, 1));
        top = max(top, (u32)__shfl_xor((int)top, 2));
        const u32 e = top >> 23;
        const bool bad = e == 255;
        const u32 b = bad ? 255u : e > 2 ? e - 2 : 0u;
        const float scale = mx_scale(bad ? 127 : b);
        u32 word = 0;
        if (!bad) {
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[0], v[1], scale, 0);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2], v[3], scale, 1);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4], v[5], scale, 2);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6], v[7], scale, 3);
        }
        const int block = p >> 2;
        if (block < nb) *(u32 *)(codes + (size_t)row * nb * 16 + (size_t)p * 4) = word;
        if ((p & 3) == 0) scales[(size_t)row * sp + block] = (uint8_t)(block < nb ? b : 0);
        const f32x2 h0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 0);
        const f32x2 h1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 1);
        const f32x2 h2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 2);
        const f32x2 h3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 3);
        norm += (h0.x * h0.x + h0.y * h0.y) + (h1.x * h1.x + h1.y * h1.y) + (h2.x * h2.x + h2.y * h2.y) +
                (h3.x * h3.x + h3.y * h3.y);
        if (bad) norm = __uint_as_float(0x7FC00000u);
    }
    for (int o = 1; o < group; o <<= 1) norm += __shfl_xor(norm, o);
    if (lane == 0) norms[row] = norm;
}

// ---- rows by id ------------------------------------------------------------------------------------------
// A lane per eight coordinates of an output row: one word of codes in, eight values out.  Bound: HBM writes.
template <class T>
__global__ __launch_bounds__(256) void rows_kernel(Table t, int d, const int *ids, long long m, int lanes, float factor,
                                                   T *out)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long i = at / lanes;
    const int p = (int)(at - i * lanes);
    if (i >= m) return;
    const int id = ids ? ids[i] : (int)i;
    const int j0 = p * 8;
    float v[8] = {};
    if (id >= 0 && id < t.n) {
        const u32 word = *(const u32 *)(t.codes + (size_t)id * t.nb * 16 + (size_t)p * 4);
        const float scale = mx_scale(t.scales[(size_t)id * t.sp + (p >> 2)]);
        const f32x2 h0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 0);
        const f32x2 h1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 1);
        const f32x2 h2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 2);
        const f32x2 h3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 3);
        v[0] = h0.x * scale, v[1] = h0.y * scale, v[2] = h1.x * scale, v[3] = h1.y * scale;
        v[4] = h2.x * scale, v[5] = h2.y * scale, v[6] = h3.x * scale, v[7] = h3.y * scale;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= factor;
    }
    T *o = out + (size_t)i * d + j0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j0 + j < d) o[j] = from_float<T>(v[j]);
}

// ---- matrix instruction --------------------------------------------------------------------------------------
// Operand of 16 rows for step s: lane l brings block 4 s + l / 16 of its row (l % 16 of the 16), zero past the last block.
struct Operand {
    i32x4 codes;
    int scale;
};
__device__ inline Operand mx_load(const Table &t, int row, int block)
{
    Operand o = {{0, 0, 0, 0}, 0};
    if (block < t.nb) {
        o.codes = *(const i32x4 *)(t.codes + ((size_t)row * t.nb + block) * 16);
        o.scale = t.scales[(size_t)row * t.sp + block];
    }
    return o;
}
__device__ inline f32x4 mx_mma(const Operand &a, const Operand &b, f32x4 c)
{
    const i32x8 a8 = {a.codes.x, a.codes.y, a.codes.z, a.codes.w, 0, 0, 0, 0};
    const i32x8 b8 = {b.codes.x, b.codes.y, b.codes.z, b.codes.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, kFp4, kFp4, 0, a.scale, 0, b.scale);
}

// ---- product ---------------------------------------------------------------------------------------------
// out[i][j] = a_i . b_j.  The rows of b are the instruction's rows and those of a its columns, so that a lane
// ends up with four consecutive values of an output row.  A wave: 64 rows of a by 64 of b.
template <class T>
__global__ __launch_bounds__(256) void product_kernel(Table a, Table b, T *out, long long ldo)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int j0 = (blockIdx.x * 2 + (wave & 1)) * 64, i0 = (blockIdx.y * 2 + (wave >> 1)) * 64;
    if (i0 >= a.n || j0 >= b.n) return;
    f32x4 acc[4][4] = {};
    for (int s = 0; s < (a.nb + 3) / 4; ++s) {
        Operand oa[4], ob[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            oa[f] = mx_load(a, min(i0 + 16 * f + r, a.n - 1), 4 * s + g);
            ob[f] = mx_load(b, min(j0 + 16 * f + r, b.n - 1), 4 * s + g);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int x = 0; x < 4; ++x) acc[y][x] = mx_mma(ob[x], oa[y], acc[y][x]);
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        const int i = i0 + 16 * y + r;
        if (i >= a.n) continue;
        T *o = out + (size_t)i * ldo;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int j = j0 + 16 * x + 4 * g + c;
                if (j < b.n) o[j] = from_float<T>(acc[y][x][c]);
            }
    }
}

// ---- nearest rows ----------------------------------------------------------------------------------------
// u(q, x) = |x|^2 - 2 q . x orders the rows x of a query as their distances |q|^2 + u do.  |x|^2 is the start value
// of the accumulators, and -2 q is q with its signs turned and its scales' exponents one larger: no instruction is
// spent on either.  Rows are taken in groups of consecutive ones.  The k best rows, in the order (u, id), lie in the k
// groups that are best in the order (smallest u, number): each of those holds a row that precedes every row of
// any other group.  So
//   scan   computes all u and keeps the smallest of each group, and of each 16 groups (a super);
//   pick   per query: the k best supers, among their groups the k best, among their rows the k best.
// Nothing is appended, so nothing overflows and no order of updates matters; equal values cost no more than others.
// Rows (and queries) with |x|^2 >= 2^126 or NaN take part with scales of 2^-127 and u = inf: there is no NaN in the
// scan, and by Cauchy's inequality no sum of the others leaves the float32 range.
// Four groups are passed over together ("block"): tile t of `tiles` holds as instruction row r the block's row
// (r / 4) * 4 tiles + 4 t + r % 4, so that the four values of a lane belong to one group in every tile and its
// running minimum needs no other lane.  A group is 4 tiles rows, a super four blocks.
constexpr float kNormLimit = 8.507059173023462e37f;      // 2^126
__device__ inline bool mx_takes_part(float norm) { return norm < kNormLimit; }
__device__ inline float mx_min(float a, float b) { return __builtin_elementwise_minimum(a, b); }

// smaller value <-> smaller word; -0 and 0 the same
__device__ inline u32 mx_order(float x)
{
    const u32 u = __float_as_uint(x + 0.0f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ inline float mx_unorder(u32 o) { return __uint_as_float((o >> 31) ? o & 0x7FFFFFFFu : ~o); }
constexpr u32 kOrderInf = 0xFF800000u;

// -2 q as an operand
__device__ inline Operand mx_query(const Table &q, int row, int block, bool ok)
{
    Operand o = mx_load(q, row, block);
#pragma unroll
    for (int c = 0; c < 4; ++c) o.codes[c] ^= (int)0x88888888u;
    o.scale = ok && block < q.nb ? min(o.scale + 1, 254) : 0;
    return o;
}
__device__ inline int mx_tile_row(int row0, int tiles, int tile, int r) { return row0 + (r >> 2) * 4 * tiles + 4 * tile + (r & 3); }

struct Scan {
    Table t, q;
    int first, nq;               // queries first .. first + nq - 1
    int tiles, supers;           // tiles per block (a power of two), supers of the table
    int per_wg, q_parts;         // supers per workgroup, parts of the queries
    float *gmin, *smin;          // [q / 16][group][q % 16], [q / 16][super][q % 16]
};

// Rows of any length: operands of both sides from memory in every step.
__global__ __launch_bounds__(256) void scan_any_kernel(Scan a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int q0 = (blockIdx.y * 4 + wave) * 64;
    if (q0 >= a.nq) return;
    int qrow[4];
    bool qok[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
        qrow[f] = a.first + min(q0 + 16 * f + r, a.nq - 1);
        qok[f] = mx_takes_part(a.q.norms[qrow[f]]);
    }
    const int s1 = min(a.supers, ((int)blockIdx.x + 1) * a.per_wg);
    for (int super = blockIdx.x * a.per_wg; super < s1; ++super) {
        float best_s[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) best_s[f] = __builtin_inff();
        for (int four = 0; four < 4; ++four) {
            const int row0 = (super * 4 + four) * 16 * a.tiles;
            float best[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) best[f] = __builtin_inff();
            for (int tile = 0; tile < a.tiles; ++tile) {
                f32x4 start;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int x = mx_tile_row(row0, a.tiles, tile, 4 * g + c);
                    const float norm = x < a.t.n ? a.t.norms[x] : __builtin_inff();
                    start[c] = mx_takes_part(norm) ? norm : __builtin_inff();
                }
                const int row = min(mx_tile_row(row0, a.tiles, tile, r), a.t.n - 1);
                const bool ok = mx_takes_part(a.t.norms[row]);
                f32x4 acc[4] = {start, start, start, start};
                for (int s = 0; s < (a.t.nb + 3) / 4; ++s) {
                    Operand x = mx_load(a.t, row, 4 * s + g);
                    if (!ok) x.scale = 0;
#pragma unroll
                    for (int f = 0; f < 4; ++f) acc[f] = mx_mma(x, mx_query(a.q, qrow[f], 4 * s + g, qok[f]), acc[f]);
                }
#pragma unroll
                for (int f = 0; f < 4; ++f)
#pragma unroll
                    for (int c = 0; c < 4; ++c) best[f] = mx_min(best[f], acc[f][c]);
            }
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                if (q0 + 16 * f < a.nq)
                    a.gmin[((size_t)(q0 / 16 + f) * a.supers * 16 + super * 16 + four * 4) * 16 + lane] = best[f];
                best_s[f] = mx_min(best_s[f], best[f]);
            }
        }
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            float m = best_s[f];
            m = mx_min(m, __shfl_xor(m, 16));
            m = mx_min(m, __shfl_xor(m, 32));
            if (g == 0 && q0 + 16 * f < a.nq) a.smin[((size_t)(q0 / 16 + f) * a.supers + super) * 16 + r] = m;
        }
    }
}

// A wave's queries, QF times 16 of them, as operands that stay in registers: KS steps, scales of four steps in a word.
template <int KS, int QF>
struct Queries {
    i32x4 codes[KS][QF];
    int scale[(KS + 3) / 4][QF];
    __device__ inline void load(const Scan &a, int q0, int r, int g)
    {
#pragma unroll
        for (int f = 0; f < QF; ++f) {
            const int row = a.first + min(q0 + 16 * f + r, a.nq - 1);
            const bool ok = mx_takes_part(a.q.norms[row]);
#pragma unroll
            for (int w = 0; w < (KS + 3) / 4; ++w) scale[w][f] = 0;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const Operand o = mx_query(a.q, row, 4 * s + g, ok);
                codes[s][f] = o.codes;
                scale[s / 4][f] |= o.scale << (8 * (s % 4));
            }
        }
    }
    template <int S> __device__ inline f32x4 mma(int f, i32x4 x, int x_scale, f32x4 c) const
    {
        const i32x8 a8 = {x.x, x.y, x.z, x.w, 0, 0, 0, 0};
        const i32x4 y = codes[S][f];
        const i32x8 b8 = {y.x, y.y, y.z, y.w, 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, kFp4, kFp4, 0, x_scale, S % 4, scale[S / 4][f]);
    }
    // u of one tile's 16 rows: codes, scales of its KS steps from x, start values
    template <class X> __device__ inline void tile(const X &x, f32x4 start, f32x4 (&acc)[QF]) const
    {
#pragma unroll
        for (int f = 0; f < QF; ++f) acc[f] = start;
        step<0>(x, acc);
    }
    template <int S, class X> __device__ inline void step(const X &x, f32x4 (&acc)[QF]) const
    {
        if constexpr (S < KS) {
            const i32x4 c = x.codes(S);
            const int sc = x.scale(S);
#pragma unroll
            for (int f = 0; f < QF; ++f) acc[f] = mma<S>(f, c, sc, acc[f]);
            step<S + 1>(x, acc);
        }
    }
};

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

// Many queries: a workgroup of 8 waves holds 8 * QF * 16 queries in registers and passes the rows of its supers
// through LDS, a stage of kStage operands at a time, asynchronously loaded while the stage before is computed.
// An operand lies in LDS as the lanes read it (lane * 16 bytes), its rows gathered by the loading lanes' addresses.
constexpr int kStage = 32;
template <int KS>
struct StageLds {
    static constexpr int tiles = KS == 1 ? kStage : KS == 2 ? kStage / 2 : KS <= 4 ? kStage / 4 : kStage / 8;      // (a power of two)
    u32 codes[tiles * KS][256];
    u32 scales[(tiles * KS + 3) / 4 * 4][16];      // [tile * KS + s][row]: the scales of the row's blocks 4 s .. 4 s + 3
    float norms[tiles][16];
};

template <int KS, int QF>
__global__ __launch_bounds__(512, 2) void scan_wide_kernel(Scan a)
{
    typedef StageLds<KS> Lds;
    constexpr int TS = Lds::tiles, kOps = TS * KS;
    extern __shared__ __align__(16) char lds_raw[];
    Lds *stage = (Lds *)lds_raw;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    // workgroups that run together on one chiplet (every eighth) take the parts of the queries over the same rows
    const int xcd = blockIdx.x & 7, at = blockIdx.x >> 3;
    const int part = at % a.q_parts, slice = (at / a.q_parts) * 8 + xcd;
    const int s0 = slice * a.per_wg, s1 = min(a.supers, s0 + a.per_wg);
    if (s0 >= s1) return;
    const int q0 = (part * 8 + wave) * QF * 16;
    Queries<KS, QF> q;
    q.load(a, q0, r, g);
    const int tile_lo = s0 * 4 * a.tiles, tile_hi = s1 * 4 * a.tiles;      // tiles counted through the table
    const int log_tiles = 31 - __clz(a.tiles), run = min(TS, a.tiles);
    const auto row_of = [&](int tile, int row) {
        return mx_tile_row((tile >> log_tiles) * 16 * a.tiles, a.tiles, tile & (a.tiles - 1), row);
    };
    const auto load = [&](int buffer, int tile0) {
        Lds *to = stage + buffer;
#pragma unroll
        for (int i = 0; i < (kOps + 7) / 8; ++i) {
            const int op = wave + 8 * i;
            if (op < kOps) {
                const int s = op % KS, row = min(row_of(tile0 + op / KS, r), a.t.n - 1);
                const uint8_t *p = a.t.codes + ((size_t)row * a.t.nb + min(4 * s + g, a.t.nb - 1)) * 16;
                __builtin_amdgcn_global_load_lds((global_void *)p, (lds_void *)&to->codes[op][0], 16, 0, 0);
            }
        }
        constexpr int kScaleLoads = (kOps + 3) / 4;         // 64 words each
#pragma unroll
        for (int i = 0; i < (kScaleLoads + 7) / 8; ++i) {
            const int part4 = wave + 8 * i;
            if (part4 < kScaleLoads) {
                const int op = part4 * 4 + g;
                if (op < kOps) {
                    const int row = min(row_of(tile0 + op / KS, r), a.t.n - 1);
                    const uint8_t *p = a.t.scales + (size_t)row * a.t.sp + 4 * (op % KS);
                    __builtin_amdgcn_global_load_lds((global_void *)p, (lds_void *)&to->scales[part4 * 4][0], 4, 0, 0);
                }
            }
        }
        constexpr int kNormLoads = (TS * 16 + 63) / 64;
        if (wave < kNormLoads) {
            const int tile = wave * 4 + g;
            if (tile < TS) {
                const float *p = a.t.norms + min(row_of(tile0 + tile, r), a.t.n - 1);
                __builtin_amdgcn_global_load_lds((global_void *)p, (lds_void *)&to->norms[wave * 4][0], 4, 0, 0);
            }
        }
    };
    const auto arrived = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    float best[QF], best_s[QF];
#pragma unroll
    for (int f = 0; f < QF; ++f) best[f] = best_s[f] = __builtin_inff();
    load(0, tile_lo);
    arrived();
    for (int tile0 = tile_lo, buffer = 0; tile0 < tile_hi; tile0 += TS, buffer ^= 1) {
        if (tile0 + TS < tile_hi) load(buffer ^ 1, tile0 + TS);
        const Lds *from = stage + buffer;
        // rows that do not take part, or do not exist, anywhere in the stage?
        bool odd = row_of(min(tile0 + TS, tile_hi) - 1, 15) >= a.t.n;
#pragma unroll
        for (int i = 0; i < (TS * 16 + 63) / 64; ++i)
            if (i * 64 + lane < TS * 16) odd |= !mx_takes_part((&from->norms[0][0])[i * 64 + lane]);
        const bool careful = __any(odd);
        struct Rows {
            const Lds *l;
            int tile, lane, r, b, b_last;
            bool out;
            __device__ i32x4 codes(int s) const { return *(const i32x4 *)&l->codes[tile * KS + s][lane * 4]; }
            __device__ int scale(int s) const
            {
                const int v = ((const uint8_t *)&l->scales[tile * KS + s][r])[s < KS - 1 ? b : b_last];
                return out ? 0 : v;
            }
        };
        // (the last step's missing blocks: the scale of the block whose codes were loaded in their place)
        const int b_last = min(4 * (KS - 1) + g, a.t.nb - 1) & 3;
        const auto pass = [&](auto careful_, int first_tile) {
#pragma unroll 4
            for (int i = 0; i < run; ++i) {
                const int tile = first_tile + i;
                f32x4 start = *(const f32x4 *)&from->norms[tile][4 * g];
                Rows x = {from, tile, lane, r, g, b_last, false};
                if constexpr (decltype(careful_)::value) {
                    x.out = !mx_takes_part(from->norms[tile][r]);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (row_of(tile0 + tile, 4 * g + c) >= a.t.n || !mx_takes_part(start[c])) start[c] = __builtin_inff();
                }
                f32x4 acc[QF];
                q.tile(x, start, acc);
#pragma unroll
                for (int f = 0; f < QF; ++f) {
                    best[f] = mx_min(mx_min(best[f], acc[f][0]), acc[f][1]);
                    best[f] = mx_min(mx_min(best[f], acc[f][2]), acc[f][3]);
                }
            }
        };
        const int n_tiles = min(TS, tile_hi - tile0);
        for (int tile = 0; tile < n_tiles; tile += run) {
            if (careful) pass(std::true_type(), tile);
            else pass(std::false_type(), tile);
            const int done = tile0 + tile + run;
            if ((done & (a.tiles - 1)) != 0) continue;
            const int block = (done >> log_tiles) - 1;
#pragma unroll
            for (int f = 0; f < QF; ++f) {
                if (q0 + 16 * f < a.nq) a.gmin[((size_t)(q0 / 16 + f) * a.supers * 4 + block) * 64 + lane] = best[f];
                best_s[f] = mx_min(best_s[f], best[f]);
                best[f] = __builtin_inff();
            }
            if ((block & 3) != 3) continue;
#pragma unroll
            for (int f = 0; f < QF; ++f) {
                float m = best_s[f];
                m = mx_min(m, __shfl_xor(m, 16));
                m = mx_min(m, __shfl_xor(m, 32));
                if (g == 0 && q0 + 16 * f < a.nq) a.smin[((size_t)(q0 / 16 + f) * a.supers + (block >> 2)) * 16 + r] = m;
                best_s[f] = __builtin_inff();
            }
        }
        arrived();
    }
}

// Few queries: all four waves of a workgroup hold the same QF * 16 of them and take a block of a super each.  The rows
// are read once, straight into registers, many tiles ahead: bound by HBM.
template <int KS, int QF>
__global__ __launch_bounds__(256) void scan_narrow_kernel(Scan a)
{
    __shared__ float share[4][QF][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int super = blockIdx.x, q0 = blockIdx.y * QF * 16;
    Queries<KS, QF> q;
    q.load(a, q0, r, g);
    const int row0 = (super * 4 + wave) * 16 * a.tiles;
    float best[QF];
#pragma unroll
    for (int f = 0; f < QF; ++f) best[f] = __builtin_inff();
    constexpr int kAhead = KS >= 3 ? 1 : 4 / KS;              // tiles loaded together
    struct Rows {
        i32x4 c[KS];
        int sc[KS];
        __device__ i32x4 codes(int s) const { return c[s]; }
        __device__ int scale(int s) const { return sc[s]; }
    };
    for (int tile0 = 0; tile0 < a.tiles; tile0 += kAhead) {
        Rows x[kAhead];
        f32x4 start[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int tile = min(tile0 + i, a.tiles - 1);
            const int row = min(mx_tile_row(row0, a.tiles, tile, r), a.t.n - 1);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int block = min(4 * s + g, a.t.nb - 1);
                x[i].c[s] = *(const i32x4 *)(a.t.codes + ((size_t)row * a.t.nb + block) * 16);
                x[i].sc[s] = a.t.scales[(size_t)row * a.t.sp + block];
            }
            const bool ok = mx_takes_part(a.t.norms[row]);
#pragma unroll
            for (int s = 0; s < KS; ++s) x[i].sc[s] = ok ? x[i].sc[s] : 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int y = mx_tile_row(row0, a.tiles, tile, 4 * g + c);
                const float norm = y < a.t.n ? a.t.norms[y] : __builtin_inff();
                start[i][c] = mx_takes_part(norm) ? norm : __builtin_inff();
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            f32x4 acc[QF];
            q.tile(x[i], start[i], acc);
#pragma unroll
            for (int f = 0; f < QF; ++f)
#pragma unroll
                for (int c = 0; c < 4; ++c) best[f] = mx_min(best[f], acc[f][c]);
        }
    }
#pragma unroll
    for (int f = 0; f < QF; ++f) {
        if (q0 + 16 * f < a.nq) a.gmin[((size_t)(q0 / 16 + f) * a.supers * 4 + super * 4 + wave) * 64 + lane] = best[f];
        float m = best[f];
        m = mx_min(m, __shfl_xor(m, 16));
        m = mx_min(m, __shfl_xor(m, 32));
        if (g == 0) share[wave][f][r] = m;
    }
    __syncthreads();
    if (tid < QF * 16 && q0 + (tid & ~15) < a.nq) {
        const int f = tid >> 4;
        const float m = mx_min(mx_min(share[0][f][r], share[1][f][r]), mx_min(share[2][f][r], share[3][f][r]));
        a.smin[((size_t)(q0 / 16 + f) * a.supers + super) * 16 + r] = m;
    }
}

struct PickShared {
    u32 hist[256];
    u32 waves[8];
    u32 prefix, need, count;
};

// The `k` smallest of m words, ties by the lower index, as ascending indices in out; returns the last one's
// word (the largest there is if m <= k) and their number.  All threads of the block take part; value(i) is called
// for i < m only.
template <int THREADS, class Value>
__device__ u32 choose(Value value, int m, int k, int *out, PickShared &sh, int &count)
{
    const int tid = threadIdx.x;
    if (m <= k) {
        for (int i = tid; i < m; i += THREADS) out[i] = i;
        count = m;
        __syncthreads();
        return ~0u;
    }
    // the k-th smallest word, eight bits at a time from the top
    u32 prefix = 0, need = k;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += THREADS) sh.hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < m; i += THREADS) {
            const u32 v = value(i);
            if (shift == 24 || (v >> (shift + 8)) == prefix) atomicAdd(&sh.hist[(v >> shift) & 255], 1u);
        }
        __syncthreads();
        if (tid < 64) {        // lane l owns the digits 4 l .. 4 l + 3
            u32 c[4], sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += c[j] = sh.hist[4 * tid + j];
            u32 upto = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const u32 other = (u32)__shfl_up((int)upto, o);
                if (tid >= o) upto += other;
            }
            u32 before = upto - sum;
            if (before < need && upto >= need)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (before < need && before + c[j] >= need) {
                        sh.prefix = (prefix << 8) | (u32)(4 * tid + j);
                        sh.need = need - before;
                    }
                    before += c[j];
                }
        }
        __syncthreads();
        prefix = sh.prefix;
        need = sh.need;
        __syncthreads();
    }
    // all that are smaller, and the first `need` of the equal ones, in the order of their indices
    u32 equal_before = 0, before = 0;
    const int lane = tid & 63, wave = tid >> 6;
    const u64 below = (1ULL << lane) - 1;
    for (int i0 = 0; i0 < m; i0 += THREADS) {
        const int i = i0 + tid;
        const u32 v = i < m ? value(i) : ~0u;
        const u64 eq = __ballot(i < m && v == prefix);
        if (lane == 0) sh.waves[wave] = (u32)__popcll(eq);
        __syncthreads();
        u32 eq_rank = equal_before + (u32)__popcll(eq & below);
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) eq_rank += sh.waves[w];
            equal_before += sh.waves[w];
        }
        const bool take = i < m && (v < prefix || (v == prefix && eq_rank < need));
        const u64 taken = __ballot(take);
        __syncthreads();
        if (lane == 0) sh.waves[wave] = (u32)__popcll(taken);
        __syncthreads();
        u32 pos = before + (u32)__popcll(taken & below);
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) pos += sh.waves[w];
            before += sh.waves[w];
        }
        if (take) out[pos] = i;
        __syncthreads();
    }
    count = k;
    return prefix;
}

// One block per query.  LDS: keys (as many as the chosen groups have rows), then the values of the groups, then the lists.
__global__ __launch_bounds__(256) void pick_kernel(Scan a, int k, long long first_self, int *ids, float *dists)
{
    constexpr int kThreads = 256;
    extern __shared__ u64 lds[];
    __shared__ PickShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int qi = blockIdx.x, kk = k + (first_self >= 0 ? 1 : 0), group = 4 * a.tiles;
    const Table &t = a.t, &q = a.q;
    const int self = first_self >= 0 ? (int)min(first_self + a.first + qi, 0x7FFFFFFFLL) : -1;
    int key_slots = 1;
    while (key_slots < kk * group) key_slots <<= 1;
    u64 *keys = lds;
    u32 *values = (u32 *)(keys + key_slots);
    int *chosen_supers = (int *)(values + 16 * kk);
    int *chosen = chosen_supers + kk;
    int *out_ids = ids + (size_t)(a.first + qi) * k;
    float *out_dists = dists + (size_t)(a.first + qi) * k;
    const float qnorm = q.norms[a.first + qi];
    int found = 0;
    if (mx_takes_part(qnorm) && t.n > 0) {
        const float *sm = a.smin + ((size_t)(qi >> 4) * a.supers) * 16 + (qi & 15);
        const float *gm = a.gmin + ((size_t)(qi >> 4) * a.supers * 16) * 16 + (qi & 15);
        int n_supers, n_groups;
        choose<kThreads>([&](int i) { return mx_order(sm[(size_t)i * 16]); }, a.supers, kk, chosen_supers, sh, n_supers);
        for (int i = tid; i < n_supers * 16; i += kThreads)
            values[i] = mx_order(gm[((size_t)chosen_supers[i >> 4] * 16 + (i & 15)) * 16]);
        __syncthreads();
        const u32 limit = choose<kThreads>([&](int i) { return values[i]; }, n_supers * 16, kk, chosen, sh, n_groups);
        if (tid == 0) sh.count = 0;
        __syncthreads();
        // values of the chosen groups' rows; every column of the instruction holds the query
        const int r = lane & 15, g = lane >> 4, per_group = (group + 15) / 16;
        for (int tile = wave; tile < n_groups * per_group; tile += kThreads / 64) {
            const int c = chosen[tile / per_group];
            const int row0 = (chosen_supers[c >> 4] * 16 + (c & 15)) * group + (tile % per_group) * 16;
            f32x4 acc;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int x = row0 + 4 * g + j;
                const float norm = x < t.n ? t.norms[x] : __builtin_inff();
                acc[j] = mx_takes_part(norm) ? norm : __builtin_inff();
            }
            const int row = min(row0 + r, t.n - 1);
            const bool ok = mx_takes_part(t.norms[row]);
            for (int s = 0; s < (t.nb + 3) / 4; ++s) {
                Operand x = mx_load(t, row, 4 * s + g);
                if (!ok) x.scale = 0;
                acc = mx_mma(x, mx_query(q, a.first + qi, 4 * s + g, true), acc);
            }
            const float u = r == 0 ? acc[0] : r == 1 ? acc[1] : r == 2 ? acc[2] : acc[3];
            const int id = row0 + 4 * g + r;
            const u32 order = mx_order(u);
            if (r < 4 && id < t.n && id != self && order < kOrderInf && order <= limit)
                keys[atomicAdd(&sh.count, 1u)] = ((u64)order << 32) | (u32)id;
        }
        __syncthreads();
        found = (int)sh.count;
    }
    int pow2 = 1;
    while (pow2 < found) pow2 <<= 1;
    for (int i = found + tid; i < pow2; i += kThreads) keys[i] = ~0ULL;
    __syncthreads();
    for (int size = 2; size <= pow2; size <<= 1)
        for (int step = size >> 1; step > 0; step >>= 1) {
            for (int i = tid; i < pow2 / 2; i += kThreads) {
                const int lo = 2 * step * (i / step) + i % step, hi = lo + step;
                const u64 x = keys[lo], y = keys[hi];
                if ((x > y) == ((lo & size) == 0)) {
                    keys[lo] = y;
                    keys[hi] = x;
                }
            }
            __syncthreads();
        }
    for (int i = tid; i < k; i += kThreads) {
        const bool live = i < found;
        const float u = live ? mx_unorder((u32)(keys[i] >> 32)) : 0.0f;
        out_ids[i] = live ? (int)(u32)keys[i] : -1;
        out_dists[i] = live ? fmaxf(qnorm + u, 0.0f) : __builtin_inff();
    }
}

struct NearestShape {
    int tiles, supers, chunk;      // tiles per block, supers of the table, queries per pass
    size_t gmin_bytes, bytes, lds;
};
inline NearestShape nearest_shape(int64_t n, int64_t nq, int k)
{
    NearestShape s;
    // Group size: the scan writes a value per group, the pick reads the rows of k groups.
    s.tiles = 4;
    while (s.tiles < 16 && (int64_t)s.tiles * s.tiles * 4 * 300 * (k + 1) <= n && (k + 1) * 4 * s.tiles * 2 <= 8192) s.tiles *= 2;
    const int64_t super_rows = 64 * s.tiles;
    s.supers = (int)((n + super_rows - 1) / super_rows);
    const size_t per16 = (size_t)s.supers * 17 * 16 * sizeof(float);     // 16 queries: groups and supers
    size_t sixteens = per16 ? kMaxWorkspace / per16 : (size_t)nq;
    if (sixteens < 16) sixteens = 16;
    const size_t all = (size_t)(nq + 15) / 16;
    if (sixteens >= all) sixteens = all;
    else {                         // passes of equal size
        const size_t passes = (all + sixteens - 1) / sixteens;
        sixteens = (all + passes - 1) / passes;
    }
    s.chunk = (int)(sixteens * 16);
    s.gmin_bytes = align_up(sixteens * s.supers * 16 * 16 * sizeof(float));
    s.bytes = s.gmin_bytes + align_up(sixteens * s.supers * 16 * sizeof(float)) + 256;
    const int kk = k + 1;
    size_t slots = 1;
    while (slots < (size_t)kk * 4 * s.tiles) slots <<= 1;
    s.lds = slots * 8 + (size_t)kk * 16 * 4 + (size_t)kk * 8;
    return s;
}

template <int KS, int QF>
int launch_wide(Scan a, hipStream_t st)
{
    const int lds = 2 * (int)sizeof(StageLds<KS>);
    EF_HIP_CHECK(hipFuncSetAttribute((const void *)scan_wide_kernel<KS, QF>, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    a.q_parts = (a.nq + 128 * QF - 1) / (128 * QF);
    const int tiles = 256;                                // per workgroup, about
    a.per_wg = tiles / (4 * a.tiles) > 1 ? tiles / (4 * a.tiles) : 1;
    const int64_t slices = (a.supers + a.per_wg - 1) / a.per_wg;
    const int64_t grid = (slices + 7) / 8 * 8 * a.q_parts;
    if (grid > 2147483647LL) return EFANNA_EUNSUPPORTED;
    scan_wide_kernel<KS, QF><<<(unsigned)grid, 512, lds, st>>>(a);
    return EFANNA_OK;
}
template <int KS, int QF>
int launch_narrow(const Scan &a, hipStream_t st)
{
    scan_narrow_kernel<KS, QF><<<dim3((unsigned)a.supers, (unsigned)((a.nq + 16 * QF - 1) / (16 * QF))), 256, 0, st>>>(a);
    return EFANNA_OK;
}
template <int KS>
int launch_scan(const Scan &a, hipStream_t st)
{
    if (a.nq <= 16) return launch_narrow<KS, 1>(a, st);
    if (a.nq <= 64) return launch_narrow<KS, 4>(a, st);
    if (KS <= 4 && a.nq > 512) return launch_wide<KS, KS <= 4 ? 8 : 4>(a, st);
    return launch_wide<KS, 4>(a, st);
}
int launch_scan_any(Scan a, hipStream_t st)
{
    const int ks = (a.t.nb + 3) / 4;
    switch (ks) {
    case 1: return launch_scan<1>(a, st);
    case 2: return launch_scan<2>(a, st);
    case 3: return launch_scan<3>(a, st);
    case 4: return launch_scan<4>(a, st);
    case 5: return launch_scan<5>(a, st);
    case 6: return launch_scan<6>(a, st);
    case 7: return launch_scan<7>(a, st);
    case 8: return launch_scan<8>(a, st);
    default: break;
    }
    a.per_wg = 4;
    const dim3 grid((unsigned)((a.supers + a.per_wg - 1) / a.per_wg), (unsigned)((a.nq + 255) / 256));
    if (grid.y > 65535) return EFANNA_EUNSUPPORTED;
    scan_any_kernel<<<grid, 256, 0, st>>>(a);
    return EFANNA_OK;
}

constexpr int64_t kMaxRows = 2147483647LL - 65536;

inline bool table_ok(const uint8_t *codes, const uint8_t *scales, int64_t n, int32_t d)
{
    if (n < 0 || n > kMaxRows || d < 1 || d > EFANNA_MX_MAX_D) return false;
    return n == 0 || (codes && scales && ((uintptr_t)codes & 15) == 0 && ((uintptr_t)scales & 3) == 0);
}
inline bool dtype_ok(int32_t dtype) { return dtype == EFANNA_F32 || dtype == EFANNA_F16 || dtype == EFANNA_BF16; }
inline bool aligned_for(const void *p, int32_t dtype) { return ((uintptr_t)p & (dtype == EFANNA_F32 ? 3 : 1)) == 0; }

}  // namespace

#define EF_MX_DTYPE(dtype, T, ...)                                   \
    do {                                                             \
        if ((dtype) == EFANNA_F32) { typedef float T; __VA_ARGS__; } \
        else if ((dtype) == EFANNA_F16) { typedef _Float16 T; __VA_ARGS__; } \
        else { typedef __bf16 T; __VA_ARGS__; }                      \
    } while (0)

extern "C" int efanna_mx_quantise(const void *X, int32_t dtype, int64_t n, int32_t d, int64_t ldx, uint8_t *codes,
                                  uint8_t *scales, float *norms, void *stream)
{
    if (!dtype_ok(dtype) || !table_ok(codes, scales, n, d) || ldx < d) return EFANNA_EINVAL;
    if (n == 0) return EFANNA_OK;
    if (!X || !norms || !aligned_for(X, dtype) || ((uintptr_t)norms & 3)) return EFANNA_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const int nb = mx_blocks(d), sp = mx_scale_pitch(d);
    int group = 4;
    while (group < 64 && group < 4 * sp) group <<= 1;
    const int64_t blocks = (n * group + 255) / 256;
    EF_MX_DTYPE(dtype, T, (quantise_kernel<T><<<(unsigned)blocks, 256, 0, st>>>((const T *)X, n, d, ldx, group, nb, sp, codes, scales, norms)));
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
}

extern "C" int efanna_mx_rows(const uint8_t *codes, const uint8_t *scales, int64_t n, int32_t d, const int32_t *ids,
                              int64_t m, float factor, int32_t dtype, void *out, void *stream)
{
    if (!dtype_ok(dtype) || !table_ok(codes, scales, n, d) || m < 0 || m > kMaxRows || (!ids && m > n)) return EFANNA_EINVAL;
    if (m == 0) return EFANNA_OK;
    if (!out || !aligned_for(out, dtype) || ((uintptr_t)ids & 3)) return EFANNA_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const Table t = {codes, scales, nullptr, (int)n, mx_blocks(d), mx_scale_pitch(d)};
    const int lanes = (d + 7) / 8;
    const int64_t blocks = (m * lanes + 255) / 256;
    if (blocks > 2147483647LL) return EFANNA_EUNSUPPORTED;
    EF_MX_DTYPE(dtype, T, (rows_kernel<T><<<(unsigned)blocks, 256, 0, st>>>(t, d, ids, m, lanes, factor, (T *)out)));
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
}

extern "C" int efanna_mx_product(const uint8_t *a_codes, const uint8_t *a_scales, int64_t m, const uint8_t *b_codes,
                                 const uint8_t *b_scales, int64_t n, int32_t d, int32_t dtype, void *out, int64_t ldo,
                                 void *stream)
{
    if (!dtype_ok(dtype) || !table_ok(a_codes, a_scales, m, d) || !table_ok(b_codes, b_scales, n, d) || ldo < n)
        return EFANNA_EINVAL;
    if (m == 0 || n == 0) return EFANNA_OK;
    if (!out || !aligned_for(out, dtype)) return EFANNA_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const int nb = mx_blocks(d), sp = mx_scale_pitch(d);
    const Table a = {a_codes, a_scales, nullptr, (int)m, nb, sp}, b = {b_codes, b_scales, nullptr, (int)n, nb, sp};
    const dim3 grid((unsigned)((n + 127) / 128), (unsigned)((m + 127) / 128));
    if (grid.y > 65535) return EFANNA_EUNSUPPORTED;
    EF_MX_DTYPE(dtype, T, (product_kernel<T><<<grid, 256, 0, st>>>(a, b, (T *)out, ldo)));
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
}

extern "C" size_t efanna_mx_nearest_workspace_bytes(int64_t n, int64_t nq, int32_t k)
{
    if (n < 0 || nq < 0 || n > kMaxRows || nq > kMaxRows || k < 1 || k > EFANNA_MAX_K) return 0;
    return nearest_shape(n, nq, k).bytes;
}

extern "C" int efanna_mx_nearest(const uint8_t *codes, const uint8_t *scales, const float *norms, int64_t n, int32_t d,
                                 const uint8_t *q_codes, const uint8_t *q_scales, const float *q_norms, int64_t nq,
                                 int32_t k, int64_t first_self, int32_t *ids, float *dists, void *ws, size_t ws_bytes,
                                 void *stream)
{
    if (!table_ok(codes, scales, n, d) || !table_ok(q_codes, q_scales, nq, d) || k < 1 || k > EFANNA_MAX_K)
        return EFANNA_EINVAL;
    if (nq == 0) return EFANNA_OK;
    if ((n > 0 && !norms) || !q_norms || !ids || !dists || ((uintptr_t)norms & 15) || ((uintptr_t)q_norms & 3) ||
        ((uintptr_t)ids & 3) || ((uintptr_t)dists & 3))
        return EFANNA_EINVAL;
    const NearestShape sh = nearest_shape(n, nq, k);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < sh.bytes) return EFANNA_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const int nb = mx_blocks(d), sp = mx_scale_pitch(d);
    const Table t = {codes, scales, norms, (int)n, nb, sp}, q = {q_codes, q_scales, q_norms, (int)nq, nb, sp};
    Scan a = {t, q, 0, 0, sh.tiles, sh.supers, 0, 0, (float *)ws, (float *)((char *)ws + sh.gmin_bytes)};
    EF_HIP_CHECK(hipFuncSetAttribute((const void *)pick_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sh.lds));
    for (int64_t first = 0; first < nq; first += sh.chunk) {
        a.first = (int)first;
        a.nq = (int)(nq - first < sh.chunk ? nq - first : sh.chunk);
        if (a.supers > 0) {
            const int rc = launch_scan_any(a, st);
            if (rc != EFANNA_OK) return rc;
            EF_HIP_CHECK(hipGetLastError());
        }
        pick_kernel<<<(unsigned)a.nq, 256, sh.lds, st>>>(a, k, first_self, ids, dists);
        EF_HIP_CHECK(hipGetLastError());
    }
    return EFANNA_OK;
}
