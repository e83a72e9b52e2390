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

#include <stdint.h>
#include <type_traits>

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kFp4 = 4;                    // the operand format's number in the matrix instruction
// Outputs larger than the L2 caches are stored past them (10^6 x 128 float32 read back: 102 -> 81 us); smaller ones are left there
// for whoever reads them next.
constexpr int64_t kStreamBytes = (int64_t)32 << 20;
constexpr size_t kMaxWorkspace = (size_t)1 << 30;
// A launch takes fewer than 2^32 threads.  Rows that a kernel takes one by one go in slices of so many workgroups of 256.
constexpr int64_t kSliceBlocks = (int64_t)1 << 23;
inline bool launch_fits(int64_t blocks, int64_t threads) { return blocks <= 4294967295LL / threads; }

// (64 KiB and less need no leave, and asking for it takes a microsecond)
inline hipError_t allow_lds(const void *kernel, int bytes)
{
    return bytes > 65536 ? hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}
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

// Eight values from or to any address that suits the element (the last ones of a row: fewer).
template <class T>
__device__ inline void load_eight(const T *p, int left, float (&v)[8])
{
    typedef T Piece __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    constexpr int kPer = 16 / sizeof(T);
    if (left >= 8) {
#pragma unroll
        for (int i = 0; i < 8; i += kPer) {
            const Piece x = *(const Piece *)(p + i);
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[i + j] = to_float(x[j]);
        }
    } else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < left ? to_float(p[j]) : 0.0f;
}
// the eight values of a word of codes
__device__ inline void mx_values(u32 word, float scale, float (&v)[8])
{
    const f32x2 h0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 0), h1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 1);
    const f32x2 h2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 2), h3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 3);
    v[0] = h0.x, v[1] = h0.y, v[2] = h1.x, v[3] = h1.y, v[4] = h2.x, v[5] = h2.y, v[6] = h3.x, v[7] = h3.y;
}

// A neighbour's value by row operations (no trip through LDS): the other lane of a pair, of a pair of pairs; the lane 4 or
// 8 further within a row of 16, around its end.
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kDown4 = 0x120 + 12, kDown8 = 0x120 + 8;
template <int CTRL> __device__ inline u32 mx_from(u32 x) { return (u32)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true); }
template <int CTRL> __device__ inline float mx_from(float x) { return __uint_as_float(mx_from<CTRL>(__float_as_uint(x))); }

// ---- quantisation ----------------------------------------------------------------------------------------
// Four lanes per block, eight coordinates each; a row's lanes are `group` consecutive ones (4 for a row of one block, 8 for two,
// else a power of two from 16 on), so a wave holds 64 / group rows and the row's squared length is a sum over those lanes.
// Bound: HBM for rows that fill their lanes (10^6 x 128 float32, 590 MB: 103 us, 5.7 TB/s), instructions for short ones (200 003 x
// 50 half precision: 11.8 us, vector instructions for 0.73 of it).
template <class T>
__global__ __launch_bounds__(256) void quantise_kernel(const T *X, long long n, int d, long long ldx, int group, int nb,
                                                       int sp, uint8_t *codes, uint8_t *scales, float *norms)
{
    const int lane = threadIdx.x & (group - 1);
    const long long row = (long long)blockIdx.x * (256 / group) + threadIdx.x / group;
    if (row >= n) return;
    const T *x = X + row * ldx;
    uint8_t *row_codes = codes + (size_t)row * nb * 16, *row_scales = scales + (size_t)row * sp;
    float norm = 0.0f;
    const int pieces = group < 16 ? group : 4 * sp;      // lanes past the last block write the scales' padding
    for (int p = lane; p < pieces; p += group) {
        float v[8];
        load_eight(x + p * 8, d - p * 8, v);
        u32 top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
        top = max(top, mx_from<kSwap1>(top));
        top = max(top, mx_from<kSwap2>(top));
        const u32 e = top >> 23;
        const bool bad = e == 255;
        const u32 b = bad ? 255u : e > 2 ? e - 2 : 0u;
        const float scale = mx_scale(bad ? 127 : b);
        u32 word = 0;
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[0], v[1], scale, 0);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2], v[3], scale, 1);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4], v[5], scale, 2);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6], v[7], scale, 3);
        if (bad) word = 0;
        const int block = p >> 2;
        if (block < nb) *(u32 *)(row_codes + (size_t)p * 4) = word;
        // four blocks' scales as a word
        u32 four = block < nb ? b : 0;
        if (group > 4) four |= mx_from<kDown4>(four) << 8;
        if (group > 8) four |= mx_from<kDown8>(four) << 16;
        if ((p & 15) == 0) *(u32 *)(row_scales + block) = four;
        mx_values(word, scale, v);
        norm += (v[0] * v[0] + v[1] * v[1]) + (v[2] * v[2] + v[3] * v[3]) + (v[4] * v[4] + v[5] * v[5]) + (v[6] * v[6] + v[7] * v[7]);
        if (bad) norm = __uint_as_float(0x7FC00000u);
    }
    norm += mx_from<kSwap1>(norm);
    norm += mx_from<kSwap2>(norm);
    if (group > 4) norm += mx_from<kDown4>(norm);
    if (group > 8) norm += mx_from<kDown8>(norm);
    for (int o = 16; o < group; o <<= 1) norm += __shfl_xor(norm, o);
    if (lane == 0) norms[row] = norm;
}

// ---- rows by id ------------------------------------------------------------------------------------------
// A lane per 16 bytes of an output row (4 or 8 coordinates: neighbouring lanes' stores touch), `group` lanes (a power of two)
// per row and kRows rows per lane, so that as many chains of id, codes, store run side by side.  Bound: HBM writes (10^6 rows of 128
// to float32: 91 us, 6.4 TB/s with the table), and instructions for 16-bit outputs (2 * 10^6 rows by id to bf16, 512 MB: 92 us,
// 5.6 TB/s, vector instructions for 0.94 of the time).  Codes have two significant
// bits, so value * scale is exact; the factor's product is rounded to float32 and then once to the output's type.
constexpr int kRows = 4;
template <class T, bool PAST_CACHE>
__global__ __launch_bounds__(256) void rows_kernel(Table t, int d, const int *ids, long long m, int group, float factor, T *out)
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
        u32 word[kRows], b[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            word[i] = 0, b[i] = 256;                   // (an empty slot)
            if (id[i] >= 0 && id[i] < t.n) {
                word[i] = *(const u32 *)(t.codes + (size_t)id[i] * t.nb * 16 + (size_t)(p * kPer / 8) * 4);
                b[i] = t.scales[(size_t)id[i] * t.sp + p * kPer / 32];
            }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const long long row = first + (long long)i * per;
            float v[8];
            mx_values(kPer == 4 ? word[i] >> (16 * (p & 1)) : word[i], 1.0f, v);
            const float scale = mx_scale(b[i] & 255);
            Piece x;
#pragma unroll
            for (int j = 0; j < kPer; ++j) x[j] = from_float<T>(b[i] > 255 ? 0.0f : v[j] * scale * factor);
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

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

// Rows pass through LDS by loads that write there directly.  An operand (16 rows, a step's 4 blocks) is 1 KiB; lane l of
// its load brings a 16-byte block of row l / 4, so that four lanes share 64 consecutive bytes of memory (with the lanes in the
// order the matrix instruction wants them the loads return a quarter as fast).  The blocks of row r lie in the order
// b ^ (r / 2) % 4, so that blocks b of eight neighbouring rows, which are read together, are in different banks.
__device__ inline int mx_stage_block(int lane, int step, int nb) { return min(4 * step + ((lane & 3) ^ ((lane >> 3) & 3)), nb - 1); }
__device__ inline int mx_staged_at(int r, int g) { return (r * 4 + (g ^ ((r >> 1) & 3))) * 4; }      // word within the operand
__device__ inline void mx_stage(const void *from, void *to, int lane_bytes_16)
{
    if (lane_bytes_16) __builtin_amdgcn_global_load_lds((global_void *)from, (lds_void *)to, 16, 0, 0);
    else __builtin_amdgcn_global_load_lds((global_void *)from, (lds_void *)to, 4, 0, 0);
}

// ---- product ---------------------------------------------------------------------------------------------
// out[i][j] = a_i . b_j.  The rows of b are the instruction's rows and those of a its columns, so that a lane
// ends up with four consecutive values of an output row.
template <class T>
__device__ inline void store_four(T *o, f32x4 x, int left)
{
    if (left >= 4) {
        typedef T Unaligned __attribute__((ext_vector_type(4), aligned(sizeof(T))));
        *(Unaligned *)o = Unaligned{from_float<T>(x[0]), from_float<T>(x[1]), from_float<T>(x[2]), from_float<T>(x[3])};
    } else
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c < left) o[c] = from_float<T>(x[c]);
}

typedef float f32x16 __attribute__((ext_vector_type(16)));
template <int N> __device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// WA x WB waves share a tile of a's rows by b's rows, FA x FB instructions of 32 x 32 x 64 each.  A stage is 256
// coordinates of both, whole lines of 128 bytes (half lines cost the loads as much each), and the scales of 512 coordinates
// with every other one; while one is computed the next is on its way into LDS.  A load of codes brings 8 rows; the blocks of row
// r lie in the order b ^ (r / 2) % 8, so that blocks b of 16 rows, which are read together, are in different ones of the 64 banks.
// Bound: what a stage waits for, all eight waves at its one barrier, and clocks under load.  8192^3 takes 0.28 ms, 3.9 PFLOP/s, at
// 1.74 GHz with the matrix units busy for 0.55 and LDS for 0.34 of the time (a fifth of that are conflicts); all loads from the same
// eight rows (less to move and fewer bits that change) 0.24.
// Tiles of 128 x 128, two workgroups a CU, 0.36: they load twice as much.  Long outputs of short sums wait for their stores too:
// 4096 x 65536 x 960 to bf16 0.27 ms, without its stores 0.16; workgroups that stay and ask for the next tile before they store
// this one were no faster, and 0.27 with stores past the caches.
template <int FA, int FB, int WA, int WB>
struct Tiling {
    static constexpr int waves = WA * WB, side_a = 32 * FA * WA, side_b = 32 * FB * WB, sides = side_a + side_b;
    static constexpr int each = sides / 8 / waves, each_scales = sides / 16 / waves;      // loads of a wave
    static_assert(sides % (16 * waves) == 0, "every wave loads as much, an even number of groups of 8 rows");
    struct Lds {
        u32 codes[2][sides / 8][256];       // a's rows, then b's
        u32 scales[2][sides][4];
    };
    static constexpr int out_pitch = 32 * FB + 8;       // values of a row of the piece that a wave turns round at the end
};

template <class T, int FA, int FB, int WA, int WB>
__global__ __launch_bounds__(64 * WA * WB, FA * FB > 8 ? 1 : 2) void product_tile_kernel(Table a, Table b, T *out, long long ldo, int tiles_a,
                                                                                          int tiles_b)
{
    typedef Tiling<FA, FB, WA, WB> Tile;
    extern __shared__ __align__(16) char lds_raw[];
    typename Tile::Lds &lds = *(typename Tile::Lds *)lds_raw;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, half = lane >> 5;
    // A chiplet (every eighth workgroup) gets a connected piece of the tiles, walked in strips of eight rows of tiles: what runs
    // there together shares rows of a and of b in its L2.
    int ta, tb;
    {
        const int all = tiles_a * tiles_b, each = all / 8, more = all % 8, xcd = blockIdx.x & 7;
        const int at = xcd * each + min(xcd, more) + (blockIdx.x >> 3);
        const int strip = at / (8 * tiles_b), high = min(8, tiles_a - strip * 8), in = at - strip * 8 * tiles_b;
        ta = strip * 8 + in % high;
        tb = in / high;
    }
    const int i0 = ta * Tile::side_a, j0 = tb * Tile::side_b;
    const int rows_a = a.n - i0, rows_b = b.n - j0, n_stages = (a.nb + 7) / 8;
    const uint8_t *codes_a = a.codes + (size_t)i0 * a.nb * 16, *codes_b = b.codes + (size_t)j0 * b.nb * 16;
    const uint8_t *scales_a = a.scales + (size_t)i0 * a.sp, *scales_b = b.scales + (size_t)j0 * b.sp;
    const auto row_of = [&](int row) { return (u32)(row < Tile::side_a ? min(row, rows_a - 1) : min(row - Tile::side_a, rows_b - 1)); };
    u32 at_codes[Tile::each], at_scales[Tile::each_scales];
#pragma unroll
    for (int i = 0; i < Tile::each; ++i) at_codes[i] = row_of((wave * Tile::each + i) * 8 + (lane >> 3)) * a.nb * 16;
#pragma unroll
    for (int i = 0; i < Tile::each_scales; ++i) at_scales[i] = row_of((wave * Tile::each_scales + i) * 16 + (lane >> 2)) * a.sp;
    const auto load = [&](int stage, bool with_scales) {
        u32 block[2];          // of even and of odd groups of 8 rows
#pragma unroll
        for (int i = 0; i < 2; ++i) block[i] = min(8 * stage + ((lane & 7) ^ (4 * i + (lane >> 4))), a.nb - 1) * 16;
#pragma unroll
        for (int i = 0; i < Tile::each; ++i) {
            const int op = wave * Tile::each + i;
            mx_stage((op * 8 < Tile::side_a ? codes_a : codes_b) + at_codes[i] + block[i & 1], &lds.codes[stage & 1][op][0], 1);
        }
        if (!with_scales) return;
        const u32 word = min(8 * stage + 4 * (lane & 3), a.sp - 4);
#pragma unroll
        for (int i = 0; i < Tile::each_scales; ++i) {
            const int op = wave * Tile::each_scales + i;
            mx_stage((op * 16 < Tile::side_a ? scales_a : scales_b) + at_scales[i] + word, &lds.scales[(stage >> 1) & 1][op * 16][0], 0);
        }
    };
    f32x16 acc[FA][FB] = {};
    const int wa = wave % WA * 32 * FA, wb = wave / WA * 32 * FB;
    // where the lane's block of the first 64 coordinates is in a stage (64 coordinates on: the offset ^ 32; 32 rows further down:
    // 4096 bytes on), and its row's scales
    const int code_a = (wa + r) * 128 + (half ^ ((r >> 1) & 7)) * 16, code_b = code_a + (Tile::side_a + wb - wa) * 128;
    typedef u32 u32x2 __attribute__((ext_vector_type(2)));
    i32x4 ca[2][FA], cb[2][FB];
    u32x2 sa[2][FA], sb[2][FB];
    const auto read_codes = [&](int stage, int h, int to) {
        const char *pa = (const char *)lds.codes[stage & 1] + (code_a ^ (32 * h)), *pb = (const char *)lds.codes[stage & 1] + (code_b ^ (32 * h));
#pragma unroll
        for (int f = 0; f < FA; ++f) ca[to][f] = *(const i32x4 *)(pa + 32 * 128 * f);
#pragma unroll
        for (int f = 0; f < FB; ++f) cb[to][f] = *(const i32x4 *)(pb + 32 * 128 * f);
    };
    // a lane's blocks are the odd or the even ones: shifted, they are bytes 0 and 2 of two words
    const auto read_scales = [&](int stage, int to) {
        const u32 *from = &lds.scales[(stage >> 1) & 1][r][2 * (stage & 1)];
#pragma unroll
        for (int f = 0; f < FA; ++f) sa[to][f] = *(const u32x2 *)(from + 4 * (wa + 32 * f)) >> (u32)(8 * half);
#pragma unroll
        for (int f = 0; f < FB; ++f) sb[to][f] = *(const u32x2 *)(from + 4 * (Tile::side_a + wb + 32 * f)) >> (u32)(8 * half);
    };
    const auto multiply = [&](int h, int from, int scales) {
#pragma unroll
        for (int y = 0; y < FA; ++y)
#pragma unroll
            for (int x = 0; x < FB; ++x) {
                const i32x4 p = cb[from][x], q = ca[from][y];
                const i32x8 p8 = {p.x, p.y, p.z, p.w, 0, 0, 0, 0}, q8 = {q.x, q.y, q.z, q.w, 0, 0, 0, 0};
                const int s = (int)sb[scales][x][h >> 1], t = (int)sa[scales][y][h >> 1];
                acc[y][x] = h & 1 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p8, q8, acc[y][x], kFp4, kFp4, 2, s, 2, t)
                                  : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p8, q8, acc[y][x], kFp4, kFp4, 0, s, 0, t);
            }
    };
    // a stage has arrived, and what was read of the one before it is in registers
    const auto arrived = [&]() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    load(0, true);
    if (n_stages > 1) load(1, false);
    if (n_stages > 1) wait_loads<Tile::each>();      // (the second stage may still be out)
    else wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    // Stages in pairs, without a branch (behind one, the compiler would put the matrix instructions too).  The next operands are
    // read while the matrix unit works on these; before a stage's last piece of work the next stage has to be there, and the
    // one after it may take this one's place.
    const int whole = a.nb / 8;
    int stage = 0;
    if (stage + 2 < whole) {
        read_codes(0, 0, 0);
        read_scales(0, 0);
        for (; stage + 3 < n_stages && stage + 2 < whole; stage += 2)
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
#pragma unroll
                for (int h = 0; h < 3; ++h) {
                    read_codes(stage + odd, h + 1, (h + 1) & 1);
                    multiply(h, h & 1, odd);
                    __builtin_amdgcn_sched_barrier(0);        // (reads further ahead do not fit the registers)
                }
                arrived();
                load(stage + odd + 2, odd == 0);
                read_codes(stage + odd + 1, 0, 0);
                read_scales(stage + odd + 1, 1 - odd);
                multiply(3, 1, odd);
                __builtin_amdgcn_sched_barrier(0);
            }
    }
    // what is left: at most three stages and one that is not whole
    for (; stage < n_stages; ++stage) {
        const int have = min(a.nb - 8 * stage, 8);
        if (have & 1) {
            // the second half of the last instruction: nothing in a, and no scale of either
            for (int row = tid; row < Tile::sides; row += 64 * Tile::waves) {
                if (row < Tile::side_a)
                    *(i32x4 *)&lds.codes[stage & 1][row >> 3][((row & 7) * 8 + (have ^ ((row >> 1) & 7))) * 4] = i32x4{0, 0, 0, 0};
                ((uint8_t *)&lds.scales[(stage >> 1) & 1][row][2 * (stage & 1)])[have] = 0;
            }
            __syncthreads();
        }
        read_scales(stage, 0);
#pragma unroll 1
        for (int h = 0; 2 * h < have; ++h) {
            read_codes(stage, h, 0);
            multiply(0, 0, 0);
            // the next two blocks' scales into byte 0
#pragma unroll
            for (int f = 0; f < FA; ++f) sa[0][f].x = h & 1 ? sa[0][f].y : sa[0][f].x >> 16;
#pragma unroll
            for (int f = 0; f < FB; ++f) sb[0][f].x = h & 1 ? sb[0][f].y : sb[0][f].x >> 16;
        }
        if (stage + 1 < n_stages) {
            arrived();
            if (stage + 2 < n_stages) load(stage + 2, (stage & 1) == 0);
        }
    }
    // Out through LDS, 32 rows of a wave's piece at a time, so that stores are whole rows of it.  (Straight from the registers
    // a store instruction is 64 pieces of 8 or 16 bytes: 65 536 x 4096 of 16 bits took 1.9 ms.)
    __syncthreads();
    constexpr int kAcross = 32 * FB, kPitch = Tile::out_pitch, kPer = 16 / sizeof(T), kLanes = kAcross / kPer;      // lanes per row
    T *turn = (T *)lds_raw + wave * 32 * kPitch;
    typedef T Out __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
    typedef T Turn __attribute__((ext_vector_type(4), aligned(8)));
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
        const int j = lane % kLanes * kPer, left = rows_b - wb - j;
#pragma unroll
        for (int i = lane / kLanes; i < 32; i += 64 / kLanes) {
            const int row = wa + 32 * y + i;
            if (row >= rows_a) continue;
            T *o = out + (size_t)(i0 + row) * ldo + j0 + wb + j;
            const T *from = &turn[i * kPitch + j];
            if (left >= kPer) *(Out *)o = *(const Out *)from;
            else
                for (int c = 0; c < left; ++c) o[c] = from[c];
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
}

// Few rows of a (16 * M at most): bound by reading b once (one row against 10^6 x 128: 12 us, 5.9 TB/s with the output).  A wave takes 64 rows of b and its share of the steps, S of them in
// flight; the WAVES waves of a workgroup take the same rows, and their sums meet in LDS, in the waves' order.
template <int S>
struct FewLds {
    u32 codes[4 * S][256];
    u32 scales[S][4][16];
};
template <class T, int M, int S, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void product_few_kernel(Table a, Table b, T *out, long long ldo)
{
    extern __shared__ __align__(16) char lds_raw[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    FewLds<S> *lds = (FewLds<S> *)lds_raw + wave;
    const int j0 = blockIdx.x * 64, left = b.n - j0, at_lane = mx_staged_at(r, g);
    const int steps = (a.nb + 3) / 4, s_lo = steps * wave / WAVES, s_hi = steps * (wave + 1) / WAVES;
    const uint8_t *from_codes = b.codes + (size_t)j0 * b.nb * 16, *lane_scales = b.scales + (size_t)(j0 + min(lane, left - 1)) * b.sp;
    u32 at_codes[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) at_codes[i] = (u32)min(16 * i + (lane >> 2), left - 1) * b.nb * 16;
    f32x4 acc[M][4] = {};
    for (int s0 = s_lo; s0 < s_hi; s0 += S) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (S > 1 && s0 + s >= s_hi) break;
            const u32 block = mx_stage_block(lane, s0 + s, b.nb) * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) mx_stage(from_codes + at_codes[i] + block, &lds->codes[s * 4 + i][0], 1);
            mx_stage(lane_scales + 4 * (s0 + s), &lds->scales[s][0][0], 0);
        }
        Operand y[S][M];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int f = 0; f < M; ++f) y[s][f] = mx_load(a, min(16 * f + r, a.n - 1), 4 * (s0 + s) + g);
        wait_loads<0>();
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (S > 1 && s0 + s >= s_hi) break;
            // (missing blocks: zeros of a meet the row's last block)
            const int block = min(4 * (s0 + s) + g, b.nb - 1) & 3;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                Operand x;
                x.codes = *(const i32x4 *)&lds->codes[s * 4 + i][at_lane];
                const int scale = ((const uint8_t *)&lds->scales[s][i][r])[block];
                x.scale = 4 * (s0 + s) + g < b.nb ? scale : 0;
#pragma unroll
                for (int f = 0; f < M; ++f) acc[f][i] = mx_mma(x, y[s][f], acc[f][i]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (read before it is written again)
    }
    if (WAVES > 1) {
        f32x4 *share = (f32x4 *)lds_raw;          // [wave - 1][M * 4][lane]
        __syncthreads();
        if (wave > 0)
#pragma unroll
            for (int f = 0; f < M; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) share[((wave - 1) * M * 4 + f * 4 + i) * 64 + lane] = acc[f][i];
        __syncthreads();
        if (wave > 0) return;
        for (int w = 0; w < WAVES - 1; ++w)
#pragma unroll
            for (int f = 0; f < M; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 other = share[(w * M * 4 + f * 4 + i) * 64 + lane];
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[f][i][c] += other[c];
                }
    }
#pragma unroll
    for (int f = 0; f < M; ++f) {
        const int i = 16 * f + r;
        if (i >= a.n) continue;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int j = 16 * t + 4 * g;
            if (j < left) store_four(out + (size_t)i * ldo + j0 + j, acc[f][t], left - j);
        }
    }
}

template <class T, int FA, int FB, int WA, int WB>
int launch_tiles(const Table &a, const Table &b, T *out, int64_t ldo, hipStream_t st)
{
    typedef Tiling<FA, FB, WA, WB> Tile;
    const int stages = (int)sizeof(typename Tile::Lds), turn = Tile::waves * 32 * Tile::out_pitch * (int)sizeof(T);
    const int lds = stages > turn ? stages : turn;
    EF_HIP_CHECK(allow_lds((const void *)product_tile_kernel<T, FA, FB, WA, WB>, lds));
    const int64_t ta = (a.n + Tile::side_a - 1) / Tile::side_a, tb = (b.n + Tile::side_b - 1) / Tile::side_b;
    if (ta * tb > 2147483647LL || !launch_fits(ta * tb, 64 * Tile::waves)) return EFANNA_EUNSUPPORTED;
    product_tile_kernel<T, FA, FB, WA, WB><<<(unsigned)(ta * tb), 64 * Tile::waves, lds, st>>>(a, b, out, ldo, (int)ta, (int)tb);
    return EFANNA_OK;
}
template <class T, int M, int S, int WAVES>
int launch_few(const Table &a, const Table &b, T *out, int64_t ldo, hipStream_t st)
{
    const int stage = WAVES * (int)sizeof(FewLds<S>), join = (WAVES - 1) * M * 4 * 64 * 16, lds = stage > join ? stage : join;
    const int64_t blocks = ((int64_t)b.n + 63) / 64;
    if (!launch_fits(blocks, 64 * WAVES)) return EFANNA_EUNSUPPORTED;
    EF_HIP_CHECK(allow_lds((const void *)product_few_kernel<T, M, S, WAVES>, lds));
    product_few_kernel<T, M, S, WAVES><<<(unsigned)blocks, 64 * WAVES, lds, st>>>(a, b, out, ldo);
    return EFANNA_OK;
}
template <class T, int M>
int launch_few_of(const Table &a, const Table &b, T *out, int64_t ldo, hipStream_t st)
{
    const int steps = (a.nb + 3) / 4;
    if (steps == 1) return launch_few<T, M, 1, 1>(a, b, out, ldo, st);
    if (steps < 8) return launch_few<T, M, 2, 1>(a, b, out, ldo, st);
    return launch_few<T, M, 2, 4>(a, b, out, ldo, st);
}
template <class T>
int launch_product(const Table &a, const Table &b, T *out, int64_t ldo, hipStream_t st)
{
    // (32 rows against 10^6 x 128: 29 us, in tiles 69; against 8192 x 8192: 17 and 22)
    if (a.n <= 16) return launch_few_of<T, 1>(a, b, out, ldo, st);
    if (a.n <= 32) return launch_few_of<T, 2>(a, b, out, ldo, st);
    // The larger tile moves half as much per operation, one of them per CU at a time; two of the smaller ones run there, which is less
    // time where they all do at once (2816^2 x 4096: 26 us, larger tiles 34; 3584^2 x 4096: 46 and 37; x 1024: 18 and 16).
    const int64_t small = (int64_t)((a.n + 127) / 128) * ((b.n + 127) / 128);
    return small > 512 ? launch_tiles<T, 4, 2, 2, 4>(a, b, out, ldo, st) : launch_tiles<T, 2, 2, 2, 2>(a, b, out, ldo, st);
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
__device__ inline bool mx_takes_part(float norm) { return norm < EFANNA_MX_MAX_NORM; }
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


template <int TILES, int KS>
struct StageLds {
    static constexpr int tiles = TILES, ops = TILES * KS;
    u32 codes[ops][256];
    u32 scales[(ops + 3) / 4 * 4][16];       // [tile * KS + s][row]: the scales of the row's blocks 4 s .. 4 s + 3
    float norms[(TILES + 3) / 4 * 4][16];
    // The waves' share of loading: row_of(tile, r) is row r of a tile of the stage, and exists.
    template <int WAVES, class RowOf> __device__ inline void load(const Table &t, int wave, int lane, RowOf row_of)
    {
        const int r = lane & 15, g = lane >> 4;
#pragma unroll
        for (int i = 0; i < (ops + WAVES - 1) / WAVES; ++i) {
            const int op = wave + WAVES * i;
            if (WAVES * (i + 1) <= ops || op < ops)
                mx_stage(t.codes + ((size_t)row_of(op / KS, lane >> 2) * t.nb + mx_stage_block(lane, op % KS, t.nb)) * 16,
                         &codes[op][0], 1);
        }
#pragma unroll
        for (int i = 0; i < ((ops + 3) / 4 + WAVES - 1) / WAVES; ++i) {
            const int op = (wave + WAVES * i) * 4 + g;
            if (op < ops) mx_stage(t.scales + (size_t)row_of(op / KS, r) * t.sp + 4 * (op % KS), &scales[(wave + WAVES * i) * 4][0], 0);
        }
#pragma unroll
        for (int i = 0; i < ((TILES + 3) / 4 + WAVES - 1) / WAVES; ++i) {
            const int tile = (wave + WAVES * i) * 4 + g;
            if (tile < TILES) mx_stage(t.norms + row_of(tile, r), &norms[(wave + WAVES * i) * 4][0], 0);
        }
    }
    // whether a row of the stage does not take part
    __device__ inline bool odd(int lane) const
    {
        bool any = false;
#pragma unroll
        for (int i = 0; i < (TILES * 16 + 63) / 64; ++i)
            if (i * 64 + lane < TILES * 16) any |= !mx_takes_part((&norms[0][0])[i * 64 + lane]);
        return __any(any);
    }
};
// A tile of a stage as an operand for Queries::tile.  b, b_last: the lane's block in a step and in the last one, where the
// place of missing blocks is taken by the row's last (the queries' zeros there count).
template <class Lds, int KS>
struct StagedRows {
    const Lds *l;
    int tile, r, at, b, b_last;
    bool out;
    __device__ i32x4 codes(int s) const { return *(const i32x4 *)&l->codes[tile * KS + s][at]; }
    __device__ int scale(int s) const
    {
        const int v = ((const uint8_t *)&l->scales[tile * KS + s][r])[s < KS - 1 ? b : b_last];
        return out ? 0 : v;
    }
};
// Start values of the tile's rows 4 g .. 4 g + 3; CAREFUL: rows from `left` on do not exist, rows out of range do not take part.
template <bool CAREFUL, class Lds>
__device__ inline f32x4 mx_start(const Lds *l, int tile, int g, int left)
{
    f32x4 start = *(const f32x4 *)&l->norms[tile][4 * g];
    if (CAREFUL)
#pragma unroll
        for (int c = 0; c < 4; ++c) start[c] = c < left && mx_takes_part(start[c]) ? start[c] : __builtin_inff();
    return start;
}

// Many queries: a workgroup of 8 waves holds 8 * QF * 16 queries in registers and passes the rows of its supers
// through LDS, a stage of about kStage operands at a time; the next one is asked for before this one is computed.  10 000 queries of
// 10^6 x 128 take 0.57 ms, 4.5 PFLOP/s, at 1.9 GHz: matrix units busy for 0.57 of the time, other vector instructions, two minima per
// matrix instruction most of all, for 0.44.  <1, 8>, which is what they take, has seven values more than its 128 registers hold; four
// are read back in every stage behind the next stage's loads, and the wait for them is one for those loads too, so that in this variant
// loads and computation take turns within a wave (the other workgroup of the CU goes on).  1000 of 10^6 x 960: 0.45 ms, 4.3 PFLOP/s, at
// 2.0 GHz, matrix units busy for 0.56: a step's operand is read from LDS right before its matrix instructions, which wait for it.
constexpr int kStage = 32;

template <int KS, int QF>
__global__ __launch_bounds__(512, KS == 1 ? 4 : 2) void scan_wide_kernel(Scan a)
{
    constexpr int TS = KS == 1 ? kStage : KS == 2 ? kStage / 2 : KS <= 4 ? kStage / 4 : kStage / 8;      // (a power of two)
    typedef StageLds<TS, KS> Lds;
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
    const int at_lane = mx_staged_at(r, g), b_last = min(4 * (KS - 1) + g, a.t.nb - 1) & 3;
    const auto row_of = [&](int tile, int row) {
        return mx_tile_row((tile >> log_tiles) * 16 * a.tiles, a.tiles, tile & (a.tiles - 1), row);
    };
    const auto load = [&](int buffer, int tile0) {
        stage[buffer].template load<8>(a.t, wave, lane, [&](int tile, int row) { return min(row_of(tile0 + tile, row), a.t.n - 1); });
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
        const bool careful = from->odd(lane) || row_of(min(tile0 + TS, tile_hi) - 1, 15) >= a.t.n;
        const auto pass = [&](auto careful_, int first_tile) {
            constexpr bool kCareful = decltype(careful_)::value;
            constexpr int kTogether = kCareful || KS > 2 ? 1 : 2;
            for (int i0 = 0; i0 < run; i0 += kTogether)
#pragma unroll
                for (int i = 0; i < kTogether; ++i) {
                    const int tile = first_tile + i0 + i;
                    const f32x4 start = mx_start<kCareful>(from, tile, g, a.t.n - row_of(tile0 + tile, 4 * g));
                    StagedRows<Lds, KS> x = {from, tile, r, at_lane, g, b_last, false};
                    if (kCareful) x.out = !mx_takes_part(from->norms[tile][r]);
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
                if (q0 + 16 * f < a.nq) {
                    float *to = &a.gmin[((size_t)(q0 / 16 + f) * a.supers * 4 + block) * 64 + lane];
                    // (past the caches where there are many: 10^4 queries of 10^6 rows 755 -> 731 us)
                    if (QF == 8) __builtin_nontemporal_store(best[f], to);
                    else *to = best[f];
                }
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

// Few queries: all four waves of a workgroup hold the same QF * 16 of them and take a block of a super each, up to 16
// operands of it in flight.  Bound by HBM: the rows are read once (one query of 10^6 x 128, 72 MB: 14.7 us, 4.9 TB/s).  (<7, 4> has
// ten values more than its registers hold; the choice below counts that in.)
template <int KS, int QF>
__global__ __launch_bounds__(256, 2) void scan_narrow_kernel(Scan a)
{
    constexpr int TS = KS == 1 ? 16 : KS == 2 ? 8 : KS <= 4 ? 4 : 2;
    typedef StageLds<TS, KS> Lds;
    extern __shared__ __align__(16) char lds_raw[];
    __shared__ float share[4][QF][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int super = blockIdx.x, q0 = blockIdx.y * QF * 16;
    const int row0 = (super * 4 + wave) * 16 * a.tiles;
    Lds *stage = (Lds *)lds_raw + wave;
    const int at_lane = mx_staged_at(r, g), b_last = min(4 * (KS - 1) + g, a.t.nb - 1) & 3;
    Queries<KS, QF> q;
    float best[QF];
#pragma unroll
    for (int f = 0; f < QF; ++f) best[f] = __builtin_inff();
    for (int tile0 = 0; tile0 < a.tiles; tile0 += TS) {
        // (tiles past the block's end are its last one again)
        const auto row_of = [&](int tile, int row) {
            return min(mx_tile_row(row0, a.tiles, min(tile0 + tile, a.tiles - 1), row), a.t.n - 1);
        };
        stage->template load<1>(a.t, 0, lane, row_of);
        if (tile0 == 0) q.load(a, q0, r, g);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const auto pass = [&](auto careful_, int tile) {
            constexpr bool kCareful = decltype(careful_)::value;
            const int left = a.t.n - mx_tile_row(row0, a.tiles, min(tile0 + tile, a.tiles - 1), 4 * g);
            const f32x4 start = mx_start<kCareful>(stage, tile, g, left);
            StagedRows<Lds, KS> x = {stage, tile, r, at_lane, g, b_last, false};
            if (kCareful) x.out = !mx_takes_part(stage->norms[tile][r]);
            f32x4 acc[QF];
            q.tile(x, start, acc);
#pragma unroll
            for (int f = 0; f < QF; ++f) {
                best[f] = mx_min(mx_min(best[f], acc[f][0]), acc[f][1]);
                best[f] = mx_min(mx_min(best[f], acc[f][2]), acc[f][3]);
            }
        };
        if (stage->odd(lane) || row0 + 16 * a.tiles > a.t.n) {
#pragma unroll 1
            for (int tile = 0; tile < TS; ++tile) pass(std::true_type(), tile);
        } else if constexpr (KS <= 2) {
#pragma unroll 4
            for (int tile = 0; tile < TS; ++tile) pass(std::false_type(), tile);
        } else {
#pragma unroll 1
            for (int tile = 0; tile < TS; ++tile) pass(std::false_type(), tile);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (read before it is written again)
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

// One word from all of a wave's, by an operation that does not mind order or repetition
template <class Of> __device__ inline u32 wave_all(u32 x, Of of)
{
    x = of(x, mx_from<kSwap1>(x));
    x = of(x, mx_from<kSwap2>(x));
    x = of(x, mx_from<kDown4>(x));
    x = of(x, mx_from<kDown8>(x));
    const u32 a = __builtin_amdgcn_readlane(x, 0), b = __builtin_amdgcn_readlane(x, 16);
    const u32 c = __builtin_amdgcn_readlane(x, 32), d = __builtin_amdgcn_readlane(x, 48);
    return of(of(a, b), of(c, d));
}

// A word that separates the `want` smallest of a wave's 64 * R words from the others, bit by bit: exactly `want` of them do not
// exceed it (sharp), or it is the want-th smallest, which others equal; `less` are smaller then.  A word of all ones stands for
// nothing, and `want` at least are something.  The search counts from the smallest word on and leaves out the leading and the last
// bits that no word has there: values next to one another share the leading ones, products of codes end in zeros.
template <int R>
__device__ inline u32 wave_nth(const u32 (&v)[R], int want, int &less, bool &sharp)
{
    u32 low = v[0];
#pragma unroll
    for (int i = 1; i < R; ++i) low = min(low, v[i]);
    low = wave_all(low, [](u32 a, u32 b) { return min(a, b); });
    u32 above[R], bits = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        above[i] = v[i] - low;
        bits |= v[i] == ~0u ? 0 : above[i];
    }
    bits = wave_all(bits, [](u32 a, u32 b) { return a | b; });
    u32 t = 0;
    less = 0;
    sharp = false;
    const u32 last = bits & (0 - bits);
    for (u32 bit = bits ? 0x80000000u >> __clz(bits) : 0; bit >= last && bit != 0; bit >>= 1) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) n += __popcll(__ballot(above[i] < t + bit));
        if (n == want) {
            sharp = true;
            return low + min(t + bit - 1, ~0u - 1 - low);
        }
        if (n < want) {
            t += bit;
            less = n;
        }
    }
    return low + t;
}

// The smallest keys (word, index) that a wave has met, in LDS.  limit: a key that `want` keys of the list do not
// exceed, once there are so many (all ones until then); nothing above it is taken in.
constexpr int kListRoom = 512;             // entries beyond `want`
struct KeyList {
    u64 *keys;
    int want, count;
    u64 limit;
    __device__ inline void start(u64 *at, int want_) { keys = at, want = want_, count = 0, limit = ~0ULL; }
    // all lanes; room for 64 more is the caller's care
    __device__ inline void push(u64 key, bool take, int lane)
    {
        take = take && key < limit;
        const u64 mask = __ballot(take);
        if (take) keys[count + __popcll(mask & ((1ULL << lane) - 1))] = key;
        count += __popcll(mask);
    }
    // all of at most 64 * ROUNDS keys into ascending order, by their ranks, and down to `want`.  (Keys go from lane to
    // lane through scalar registers: reading them from LDS in the loop, a wave waits for each.)
    template <int ROUNDS> __device__ inline void sort_of(int lane)
    {
        u64 mine[ROUNDS];
        int rank[ROUNDS];
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            mine[i] = i * 64 + lane < count ? keys[i * 64 + lane] : ~0ULL;
            rank[i] = 0;
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int b = 0; b < ROUNDS; ++b) {
            const int n = min(count - b * 64, 64);
            for (int l = 0; l < n; ++l) {
                const u32 lo = (u32)__builtin_amdgcn_readlane((int)(u32)mine[b], l);
                const u32 hi = (u32)__builtin_amdgcn_readlane((int)(u32)(mine[b] >> 32), l);
                const u64 other = ((u64)hi << 32) | lo;
#pragma unroll
                for (int i = 0; i < ROUNDS; ++i) rank[i] += other < mine[i];
            }
        }
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i)
            if (i * 64 + lane < count && rank[i] < want) keys[rank[i]] = mine[i];
        __builtin_amdgcn_wave_barrier();
        count = min(count, want);
    }
    // down to the `want` smallest, in no order: the want-th word bit by bit, among equal words the want-th index likewise
    template <int ROUNDS> __device__ inline void cut_of(int lane)
    {
        u64 mine[ROUNDS];
        u32 word[ROUNDS];
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            mine[i] = i * 64 + lane < count ? keys[i * 64 + lane] : ~0ULL;
            word[i] = (u32)(mine[i] >> 32);
        }
        __builtin_amdgcn_wave_barrier();
        int less;
        bool sharp;
        const u32 w = wave_nth(word, want, less, sharp);
        u32 last = ~0u;
        if (!sharp) {
            u32 index[ROUNDS];
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i) index[i] = word[i] == w ? (u32)mine[i] : ~0u;
            int unused;
            last = wave_nth(index, want - less, unused, sharp);
        }
        limit = ((u64)w << 32) | last;
        count = 0;
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const bool keep = mine[i] <= limit;
            const u64 mask = __ballot(keep);
            if (keep) keys[count + __popcll(mask & ((1ULL << lane) - 1))] = mine[i];
            count += __popcll(mask);
        }
        __builtin_amdgcn_wave_barrier();
    }
    __device__ inline void cut(int lane)
    {
        __builtin_amdgcn_wave_barrier();
        if (count < want) return;
        if (count <= 64) cut_of<1>(lane);
        else if (count <= 256) cut_of<4>(lane);
        else cut_of<(kListRoom + 192) / 64>(lane);
    }
    __device__ inline void sort(int lane)
    {
        if (count > 192) cut(lane);
        __builtin_amdgcn_wave_barrier();
        if (count <= 64) sort_of<1>(lane);
        else sort_of<3>(lane);
    }
};

// Takes the keys (word(i), name(i)) of i0 <= i < min(m, i0 + 64 * C), one at least, into the list; a word of kOrderInf and more is nothing.
template <int C, class Word, class Name>
__device__ inline void choose_part(KeyList &list, int i0, int m, int lane, Word word, Name name)
{
    u32 v[C];
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = word(min(i0 + c * 64 + lane, m - 1));      // (no load waits behind a condition)
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = i0 + c * 64 + lane < m ? v[c] : ~0u;
    u32 bound = ~0u;
    if (list.limit == ~0ULL && m - i0 > list.want) {
        // the want-th of the words, or of the lanes' smallest words: at least want of the words do not exceed either, and
        // where want is far below 64 few more do
        int unused;
        bool sharp;
        if (list.want <= 32) {
            u32 low[1] = {v[0]};
#pragma unroll
            for (int c = 1; c < C; ++c) low[0] = min(low[0], v[c]);
            bound = wave_nth(low, list.want, unused, sharp);
        } else if (list.want < 64 * C) bound = wave_nth(v, list.want, unused, sharp);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const bool take = v[c] < kOrderInf && v[c] <= bound;
        if (__any(take)) list.push(((u64)v[c] << 32) | (u32)(take ? name(i0 + c * 64 + lane) : 0), take, lane);
    }
    list.cut(lane);
}
// The list's `want` smallest of m keys.  (Eight loads per lane at a time where there is so much; fewer cost fewer instructions.)
template <class Word, class Name>
__device__ inline void choose(KeyList &list, int m, int lane, Word word, Name name)
{
    if (m == 0) return;              // (a part reads one key at least)
    if (m <= 128) return choose_part<2>(list, 0, m, lane, word, name);
    if (m <= 256) return choose_part<4>(list, 0, m, lane, word, name);
    for (int i0 = 0; i0 < m; i0 += 512) choose_part<8>(list, i0, m, lane, word, name);
}

// u of 64 rows, a lane each: lane (g, r) asks for row 4 g + r % 4 of tile r / 4, which begins at row0[r / 4] (the same for all lanes)
// and is a row of the table.  Every column of the instruction is the query, so that of the four values that a lane gets of each tile
// it needs one, and start values elsewhere do not matter: all of a lane's are its row's norm.  S steps at a time pass through the
// wave's own piece of LDS.
template <int S>
struct ScoreLds {
    u32 codes[4 * S][256];
    u32 scales[S][4][16];
};
template <int S>
__device__ inline float score_rows(const Table &t, const Table &q, ScoreLds<S> *lds, const Operand &first, int qrow, int lane,
                                   const int (&row0)[4], float norm)
{
    const int steps = (t.nb + 3) / 4, r = lane & 15, g = lane >> 4, at_lane = mx_staged_at(r, g);
    const bool whole = max(max(row0[0], row0[1]), max(row0[2], row0[3])) + 16 <= t.n;
    const int scale_row = (g == 0 ? row0[0] : g == 1 ? row0[1] : g == 2 ? row0[2] : row0[3]) + r;
    const uint8_t *lane_scales = t.scales + (size_t)min(scale_row, t.n - 1) * t.sp;
    const u32 lane_codes = __umul24(lane >> 2, t.nb) * 16;
    f32x4 acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = f32x4{norm, norm, norm, norm};
    for (int s0 = 0; s0 < steps; s0 += S) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (S > 1 && s0 + s >= steps) break;
            const u32 block = mx_stage_block(lane, s0 + s, t.nb) * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32 row = whole ? lane_codes : __umul24(min(lane >> 2, t.n - 1 - row0[i]), t.nb) * 16;
                mx_stage(t.codes + (size_t)row0[i] * t.nb * 16 + (row + block), &lds->codes[s * 4 + i][0], 1);
            }
            mx_stage(lane_scales + 4 * (s0 + s), &lds->scales[s][0][0], 0);
        }
        Operand y[S];
#pragma unroll
        for (int s = 0; s < S; ++s) y[s] = S == 1 && s0 == 0 ? first : mx_query(q, qrow, 4 * (s0 + s) + g, true);
        wait_loads<0>();
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (S > 1 && s0 + s >= steps) break;
            const int block = min(4 * (s0 + s) + g, t.nb - 1) & 3;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                Operand x;
                x.codes = *(const i32x4 *)&lds->codes[s * 4 + i][at_lane];
                x.scale = ((const uint8_t *)&lds->scales[s][i][r])[block];
                acc[i] = mx_mma(x, y[s], acc[i]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (read before it is written again)
    }
    float u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = r & 1 ? acc[i][1] : acc[i][0], hi = r & 1 ? acc[i][3] : acc[i][2];
        u[i] = r & 2 ? hi : lo;
    }
    const float lo = r & 4 ? u[1] : u[0], hi = r & 4 ? u[3] : u[2];
    return r & 8 ? hi : lo;
}

// Bound: instructions and their latency (20 003 queries of as many rows of 50: 86 us, 1100 vector and 1600 scalar instructions per
// query; 10 000 of 10^6 x 128: 100 us; one: 13.5 us, a chain of some thirty dependent steps).
// WAVES waves per query (one: many queries; several: few).  All of them choose the same supers and groups; the rows of
// the groups are shared out, and the waves' lists meet in the first one's.
template <int WAVES, int S>
__global__ __launch_bounds__(64 * WAVES) void pick_kernel(Scan a, int k, long long first_self, int *ids, float *dists)
{
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    // sixteen neighbouring queries, whose minima lie side by side, on one chiplet (every eighth workgroup)
    const int qi = WAVES > 1 ? blockIdx.x : (blockIdx.x & ~127) + (blockIdx.x & 7) * 16 + ((blockIdx.x >> 3) & 15);
    if (qi >= a.nq) return;
    const int kk = k + (first_self >= 0 ? 1 : 0), group = 4 * a.tiles;
    const Table &t = a.t, &q = a.q;
    const int self = first_self >= 0 ? (int)min(first_self + a.first + qi, 0x7FFFFFFFLL) : -1;
    ScoreLds<S> *scores = (ScoreLds<S> *)lds + wave;
    u64 *lists = (u64 *)((ScoreLds<S> *)lds + WAVES), *mine = lists + wave * (2 * kk + kListRoom);
    u64 *chosen = mine + kk + kListRoom;
    int *out_ids = ids + (size_t)(a.first + qi) * k;
    float *out_dists = dists + (size_t)(a.first + qi) * k;
    const float qnorm = q.norms[a.first + qi];
    KeyList list;
    list.start(mine, kk);
    if (mx_takes_part(qnorm) && t.n > 0) {
        const float *sm = a.smin + ((size_t)(qi >> 4) * a.supers) * 16 + (qi & 15);
        const float *gm = a.gmin + ((size_t)(qi >> 4) * a.supers * 16) * 16 + (qi & 15);
        choose(list, a.supers, lane, [&](int i) { return mx_order(sm[(size_t)i * 16]); }, [&](int i) { return i; });
        const int n_supers = list.count;
        for (int i = lane; i < n_supers; i += 64) chosen[i] = mine[i];
        __builtin_amdgcn_wave_barrier();
        list.start(mine, kk);
        const auto group_of = [&](int i) { return (int)(u32)chosen[i >> 4] * 16 + (i & 15); };
        choose(list, n_supers * 16, lane, [&](int i) { return mx_order(gm[(size_t)group_of(i) * 16]); }, group_of);
        const int n_groups = list.count;
        const u32 bound = (u32)(list.limit >> 32);
        __builtin_amdgcn_wave_barrier();
        for (int i = lane; i < n_groups; i += 64) chosen[i] = mine[i];
        __builtin_amdgcn_wave_barrier();
        list.start(mine, kk);
        // values of the groups' rows, four tiles of 16 at a time
        const Operand first = mx_query(q, a.first + qi, g, true);
        const float farthest = bound < kOrderInf ? mx_unorder(bound) : 3.402823466e+38f;
        const int per_group = group / 16, log_per_group = 31 - __clz(per_group), n_tiles = n_groups << log_per_group;
        for (int tile0 = wave * 4; tile0 < n_tiles; tile0 += WAVES * 4) {
            int row0[4], row_lane = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int tile = min(tile0 + i, n_tiles - 1);
                const int at = __builtin_amdgcn_readfirstlane((int)(u32)chosen[tile >> log_per_group]) * group + (tile & (per_group - 1)) * 16;
                if (r >> 2 == i) row_lane = at;
                row0[i] = min(at, t.n - 1);            // (the table can end inside a group)
            }
            const int id = row_lane + 4 * g + (r & 3);
            const float norm = t.norms[min(id, t.n - 1)];
            const float u = score_rows<S>(t, q, scores, first, a.first + qi, lane, row0, norm);
            const bool take = u <= farthest && id != self && id < t.n && tile0 + (r >> 2) < n_tiles && mx_takes_part(norm);
            if (__any(take)) list.push(((u64)mx_order(u) << 32) | (u32)id, take, lane);
            if (list.count > kListRoom - 64) list.cut(lane);
        }
    }
    if (WAVES > 1) {
        if (list.count > kk) list.cut(lane);
        __shared__ int counts[WAVES];
        if (lane == 0) counts[wave] = list.count;
        __syncthreads();
        if (wave != 0) return;
        for (int w = 1; w < WAVES; ++w) {
            const u64 *theirs = lists + w * (2 * kk + kListRoom);
            const int c = counts[w];
            for (int i0 = 0; i0 < c; i0 += 64) list.push(i0 + lane < c ? theirs[i0 + lane] : 0, i0 + lane < c, lane);
            if (list.count > kListRoom - 256) list.cut(lane);
        }
    }
    list.sort(lane);
    for (int i = lane; i < k; i += 64) {
        const bool live = i < list.count;
        const u64 key = live ? mine[i] : 0;
        out_ids[i] = live ? (int)(u32)key : -1;
        out_dists[i] = live ? fmaxf(qnorm + mx_unorder((u32)(key >> 32)), 0.0f) : __builtin_inff();
    }
}

struct NearestShape {
    int tiles, supers, chunk;      // tiles per block, supers of the table, queries per pass
    size_t gmin_bytes, bytes;
};
inline NearestShape nearest_shape(int64_t n, int d, int64_t nq, int k)
{
    NearestShape s;
    // Group size: the scan writes a value per group, the pick reads the rows of k groups.
    s.tiles = 4;
    const int row = mx_blocks(d) > 4 ? mx_blocks(d) : 4;
    while (s.tiles < 32 && (int64_t)s.tiles * s.tiles * 120 * row * (k + 1) <= n) s.tiles *= 2;
    const int64_t super_rows = 64 * s.tiles;
    s.supers = (int)((n + super_rows - 1) / super_rows);
    const size_t per16 = (size_t)s.supers * 17 * 16 * sizeof(float);     // 16 queries: groups and supers
    size_t sixteens = per16 ? kMaxWorkspace / per16 : (size_t)nq;
    if (sixteens < 16) sixteens = 16;
    if (sixteens > (size_t)1 << 20) sixteens = (size_t)1 << 20;      // (no rows: what one launch of the choice takes)
    const size_t all = (size_t)(nq + 15) / 16;
    if (sixteens >= all) sixteens = all;
    else {                         // passes of equal size
        const size_t passes = (all + sixteens - 1) / sixteens;
        sixteens = (all + passes - 1) / passes;
    }
    s.chunk = (int)(sixteens * 16);
    s.gmin_bytes = align_up(sixteens * s.supers * 16 * 16 * sizeof(float));
    s.bytes = s.gmin_bytes + align_up(sixteens * s.supers * 16 * sizeof(float)) + 256;
    return s;
}

template <int WAVES, int S>
int launch_pick_of(const Scan &a, int k, int64_t first_self, int32_t *ids, float *dists, hipStream_t st)
{
    const int kk = k + (first_self >= 0 ? 1 : 0), lds = WAVES * ((2 * kk + kListRoom) * 8 + (int)sizeof(ScoreLds<S>));
    EF_HIP_CHECK(allow_lds((const void *)pick_kernel<WAVES, S>, lds));
    const int blocks = WAVES > 1 ? a.nq : (a.nq + 127) & ~127;
    pick_kernel<WAVES, S><<<(unsigned)blocks, 64 * WAVES, lds, st>>>(a, k, first_self, ids, dists);
    return EFANNA_OK;
}
template <int S>
int launch_pick(const Scan &a, int k, int64_t first_self, int32_t *ids, float *dists, hipStream_t st)
{
    // Waves per query, by how many queries there are to fill the CUs (10^6 x 128; one, four, eight waves: 16 queries 39, 33, 32 us;
    // 1000 queries 109, 102, 119; 4096 queries 290, 326, 376)
    if (a.nq > 2048) return launch_pick_of<1, S>(a, k, first_self, ids, dists, st);
    if (a.nq > 256) return launch_pick_of<4, S>(a, k, first_self, ids, dists, st);
    return launch_pick_of<8, S>(a, k, first_self, ids, dists, st);
}

template <int KS, int QF>
int launch_wide(Scan a, hipStream_t st)
{
    const int lds = 2 * (int)sizeof(StageLds<KS == 1 ? kStage : KS == 2 ? kStage / 2 : KS <= 4 ? kStage / 4 : kStage / 8, KS>);
    EF_HIP_CHECK(allow_lds((const void *)scan_wide_kernel<KS, QF>, lds));
    a.q_parts = (a.nq + 128 * QF - 1) / (128 * QF);
    // supers per workgroup: those that a chiplet is through with first, in rounds of the workgroups that run there at once, a
    // workgroup's start counted as 4 tiles (10^6 x 960, 1000 queries: 0.45 ms in two rounds of 4, 0.50 in three of 3)
    const int64_t at_once = KS == 1 ? 64 : 32, start = 4;
    int64_t best = INT64_MAX;
    for (int p = 1; p <= 64; ++p) {
        const int64_t groups = (int64_t)(((a.supers + p - 1) / p + 7) / 8) * a.q_parts;
        const int64_t cost = (groups + at_once - 1) / at_once * ((int64_t)p * 4 * a.tiles + start);
        if (cost < best) {
            best = cost;
            a.per_wg = p;
        }
    }
    const int64_t slices = (a.supers + a.per_wg - 1) / a.per_wg;
    const int64_t grid = (slices + 7) / 8 * 8 * a.q_parts;
    if (grid > 2147483647LL || !launch_fits(grid, 512)) return EFANNA_EUNSUPPORTED;
    scan_wide_kernel<KS, QF><<<(unsigned)grid, 512, lds, st>>>(a);
    return EFANNA_OK;
}
template <int KS, int QF>
int launch_narrow(const Scan &a, hipStream_t st)
{
    const int lds = 4 * (int)sizeof(StageLds<KS == 1 ? 16 : KS == 2 ? 8 : KS <= 4 ? 4 : 2, KS>);
    EF_HIP_CHECK(allow_lds((const void *)scan_narrow_kernel<KS, QF>, lds));
    scan_narrow_kernel<KS, QF><<<dim3((unsigned)a.supers, (unsigned)((a.nq + 16 * QF - 1) / (16 * QF))), 256, lds, st>>>(a);
    return EFANNA_OK;
}
template <int KS>
int launch_scan(const Scan &a, hipStream_t st)
{
    if (a.nq <= 16) return launch_narrow<KS, 1>(a, st);
    // (64 queries' operands of longer rows leave too few registers: 32 of 10^6 x 832 137 us, otherwise 144; of 10^6 x 960 166 and 152)
    if constexpr (KS <= 7)
        if (a.nq <= 64) return launch_narrow<KS, 4>(a, st);
    if (a.nq <= 128) return launch_wide<KS, 1>(a, st);
    if (a.nq <= 256) return launch_wide<KS, 2>(a, st);
    if (a.nq <= 512 || KS > 4) return launch_wide<KS, 4>(a, st);
    return launch_wide<KS, KS <= 4 ? 8 : 4>(a, st);
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
    int group = nb == 1 ? 4 : nb == 2 ? 8 : 16;      // (200 003 rows of 50 half-precision values: 8 lanes 11.7 us, 16 lanes 17.5)
    while (nb > 2 && group < 64 && group < 4 * sp) group <<= 1;
    const int64_t rows = 256 / group, slice = kSliceBlocks * rows;      // rows of a workgroup, of a launch
    for (int64_t first = 0; first < n; first += slice) {
        const int64_t here = n - first < slice ? n - first : slice;
        EF_MX_DTYPE(dtype, T, (quantise_kernel<T><<<(unsigned)((here + rows - 1) / rows), 256, 0, st>>>(
                                  (const T *)X + first * ldx, here, d, ldx, group, nb, sp, codes + (size_t)first * nb * 16,
                                  scales + (size_t)first * sp, norms + first)));
        EF_HIP_CHECK(hipGetLastError());
    }
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
    const int per = dtype == EFANNA_F32 ? 4 : 8;
    const bool past_cache = m * d * (16 / per) > kStreamBytes;
    int group = 1;
    while (group < 64 && group * per < d) group <<= 1;
    const int64_t rows = kRows * (256 / group), slice = kSliceBlocks * rows;      // rows of a workgroup, of a launch
    for (int64_t first = 0; first < m; first += slice) {
        const int64_t here = m - first < slice ? m - first : slice;
        const unsigned blocks = (unsigned)((here + rows - 1) / rows);
        // (without ids the slice's rows are a table of their own)
        const Table from = ids ? t : Table{codes + (size_t)first * t.nb * 16, scales + (size_t)first * t.sp, nullptr, (int)(n - first), t.nb, t.sp};
        const int *slice_ids = ids ? ids + first : nullptr;
        EF_MX_DTYPE(dtype, T, {
            T *to = (T *)out + (size_t)first * d;
            if (past_cache) rows_kernel<T, true><<<blocks, 256, 0, st>>>(from, d, slice_ids, here, group, factor, to);
            else rows_kernel<T, false><<<blocks, 256, 0, st>>>(from, d, slice_ids, here, group, factor, to);
        });
        EF_HIP_CHECK(hipGetLastError());
    }
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
    int rc = EFANNA_OK;
    EF_MX_DTYPE(dtype, T, rc = launch_product<T>(a, b, (T *)out, ldo, st));
    if (rc != EFANNA_OK) return rc;
    EF_HIP_CHECK(hipGetLastError());
    return EFANNA_OK;
}

extern "C" size_t efanna_mx_nearest_workspace_bytes(int64_t n, int32_t d, int64_t nq, int32_t k)
{
    if (d < 1 || d > EFANNA_MX_MAX_D || n < 0 || nq < 0 || n > kMaxRows || nq > kMaxRows || k < 1 || k > EFANNA_MAX_K) return 0;
    return nearest_shape(n, d, nq, k).bytes;
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
    const NearestShape sh = nearest_shape(n, d, nq, k);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < sh.bytes) return EFANNA_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const int nb = mx_blocks(d), sp = mx_scale_pitch(d);
    const Table t = {codes, scales, norms, (int)n, nb, sp}, q = {q_codes, q_scales, q_norms, (int)nq, nb, sp};
    Scan a = {t, q, 0, 0, sh.tiles, sh.supers, 0, 0, (float *)ws, (float *)((char *)ws + sh.gmin_bytes)};
    for (int64_t first = 0; first < nq; first += sh.chunk) {
        a.first = (int)first;
        a.nq = (int)(nq - first < sh.chunk ? nq - first : sh.chunk);
        if (a.supers > 0) {
            const int rc = launch_scan_any(a, st);
            if (rc != EFANNA_OK) return rc;
            EF_HIP_CHECK(hipGetLastError());
        }
        const int rc = a.t.nb <= 4 ? launch_pick<1>(a, k, first_self, ids, dists, st) : launch_pick<2>(a, k, first_self, ids, dists, st);
        if (rc != EFANNA_OK) return rc;
        EF_HIP_CHECK(hipGetLastError());
    }
    return EFANNA_OK;
}
