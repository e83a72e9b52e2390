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
// s(q, x) = q . x - |x|^2 / 2 orders the rows x of a query as their distances |q|^2 - 2 s do, and |x|^2 / 2 is
// the start value of the accumulators.  Rows are taken in groups of consecutive ones.  The k best rows, in the
// order (s descending, id ascending), lie in the k groups that are best in the order (largest s descending,
// number ascending): each of those holds a row that precedes every row of any other group.  So
//   scan   computes all s and keeps the largest of each group, and of each 16 groups (a super);
//   pick   per query: the k best supers, among their groups the k best, among their rows the k best.
// Nothing is appended, so nothing overflows and no order of updates matters; equal scores cost no more than others.
// Rows (and queries) whose norm is not finite get the scale 2^-127 and s = -inf: there is no NaN in the scan, and by
// Cauchy's inequality no sum of the others leaves the float32 range.
constexpr int kTiles = 4;                  // 16-row tiles per 4 groups: a group is 4 * kTiles rows
constexpr int kGroup = 4 * kTiles;
constexpr int kSuper = 16 * kGroup;

__device__ inline bool mx_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }
// larger score <-> larger word; -0 and 0 the same
__device__ inline u32 mx_order(float s)
{
    const u32 u = __float_as_uint(s + 0.0f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ inline float mx_unorder(u32 o) { return __uint_as_float((o >> 31) ? o & 0x7FFFFFFFu : ~o); }
constexpr u32 kOrderMinusInf = 0x007FFFFFu;

// largest score of the groups and supers of a slice.  gmax[q / 16][group][q % 16], smax[q / 16][super][q % 16].
// In a pass over 4 groups the instruction's row r of tile t is row (r / 4) * kGroup + 4 t + r % 4 of them, so that
// the four values of a lane belong to one group in every tile and its running maximum needs no other lane.
__global__ __launch_bounds__(256) void scan_kernel(Table t, Table q, int first, int nq, int supers, int per_block,
                                                   float *gmax, float *smax)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int q0 = (blockIdx.y * 4 + wave) * 64;
    if (q0 >= nq) return;
    const int groups = supers * 16;
    int qrow[4];
    bool qok[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
        qrow[f] = first + min(q0 + 16 * f + r, nq - 1);
        qok[f] = mx_finite(q.norms[qrow[f]]);
    }
    const int s1 = min(supers, ((int)blockIdx.x + 1) * per_block);
    for (int super = blockIdx.x * per_block; super < s1; ++super) {
        float best_s[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) best_s[f] = -__builtin_inff();
        for (int four = 0; four < 4; ++four) {
            const int row0 = super * kSuper + four * 4 * kGroup;
            float best[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) best[f] = -__builtin_inff();
            for (int tile = 0; tile < kTiles; ++tile) {
                f32x4 start;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int x = row0 + g * kGroup + 4 * tile + c;
                    const float norm = x < t.n ? t.norms[x] : __builtin_inff();
                    start[c] = mx_finite(norm) ? -0.5f * norm : -__builtin_inff();
                }
                const int row = min(row0 + (r >> 2) * kGroup + 4 * tile + (r & 3), t.n - 1);
                const bool ok = mx_finite(t.norms[row]);
                f32x4 acc[4] = {start, start, start, start};
                for (int s = 0; s < (t.nb + 3) / 4; ++s) {
                    Operand x = mx_load(t, row, 4 * s + g);
                    if (!ok) x.scale = 0;
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        Operand y = mx_load(q, qrow[f], 4 * s + g);
                        if (!qok[f]) y.scale = 0;
                        acc[f] = mx_mma(x, y, acc[f]);
                    }
                }
#pragma unroll
                for (int f = 0; f < 4; ++f)
#pragma unroll
                    for (int c = 0; c < 4; ++c) best[f] = __builtin_elementwise_maximum(best[f], acc[f][c]);
            }
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                if (q0 + 16 * f < nq)
                    gmax[((size_t)(q0 / 16 + f) * groups + super * 16 + four * 4 + g) * 16 + r] = best[f];
                best_s[f] = __builtin_elementwise_maximum(best_s[f], best[f]);
            }
        }
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            float s = best_s[f];
            s = __builtin_elementwise_maximum(s, __shfl_xor(s, 16));
            s = __builtin_elementwise_maximum(s, __shfl_xor(s, 32));
            if (g == 0 && q0 + 16 * f < nq) smax[((size_t)(q0 / 16 + f) * supers + super) * 16 + r] = s;
        }
    }
}

struct PickShared {
    u32 hist[256];
    u32 waves[8];
    u32 prefix, need, count;
};

// The `k` best of m ordered scores, ties by the lower index, as ascending indices in out; returns the last one's
// score (that of nothing if m <= k) and their number.  All threads of the block take part; value(i) is called
// for i < m only.
template <int THREADS, class Value>
__device__ u32 choose(Value value, int m, int k, int *out, PickShared &sh, int &count)
{
    const int tid = threadIdx.x;
    if (m <= k) {
        for (int i = tid; i < m; i += THREADS) out[i] = i;
        count = m;
        __syncthreads();
        return 0;
    }
    // the k-th largest word, eight bits at a time from the top
    u32 prefix = 0, need = k;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += THREADS) sh.hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < m; i += THREADS) {
            const u32 v = value(i);
            if (shift == 24 || (v >> (shift + 8)) == prefix) atomicAdd(&sh.hist[(v >> shift) & 255], 1u);
        }
        __syncthreads();
        if (tid < 64) {        // lane l owns the digits 255 - 4 l .. 252 - 4 l, best first
            u32 c[4], sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += c[j] = sh.hist[255 - 4 * tid - j];
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
                        sh.prefix = (prefix << 8) | (u32)(255 - 4 * tid - j);
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
    // all that are better, and the first `need` of the equal ones, in the order of their indices
    u32 equal_before = 0, before = 0;
    const int lane = tid & 63, wave = tid >> 6;
    const u64 below = (1ULL << lane) - 1;
    for (int i0 = 0; i0 < m; i0 += THREADS) {
        const int i = i0 + tid;
        const u32 v = i < m ? value(i) : 0;
        const u64 eq = __ballot(i < m && v == prefix);
        if (lane == 0) sh.waves[wave] = (u32)__popcll(eq);
        __syncthreads();
        u32 eq_rank = equal_before + (u32)__popcll(eq & below);
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) eq_rank += sh.waves[w];
            equal_before += sh.waves[w];
        }
        const bool take = i < m && (v > prefix || (v == prefix && eq_rank < need));
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

// One block per query.  LDS: keys (k * kGroup of them at most), then the values of the groups, then the lists.
__global__ __launch_bounds__(256) void pick_kernel(Table t, Table q, int first, int k, long long first_self, int supers,
                                                   const float *gmax, const float *smax, int *ids, float *dists)
{
    constexpr int kThreads = 256;
    extern __shared__ u64 lds[];
    __shared__ PickShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int qi = blockIdx.x, kk = k + (first_self >= 0 ? 1 : 0);
    const int self = first_self >= 0 ? (int)min(first_self + first + qi, 0x7FFFFFFFLL) : -1;
    int key_slots = 1;
    while (key_slots < kk * kGroup) key_slots <<= 1;
    u64 *keys = lds;
    u32 *values = (u32 *)(keys + key_slots);
    int *chosen_supers = (int *)(values + 16 * kk);
    int *chosen = chosen_supers + kk;
    int *out_ids = ids + (size_t)(first + qi) * k;
    float *out_dists = dists + (size_t)(first + qi) * k;
    const float qnorm = q.norms[first + qi];
    int found = 0;
    if (mx_finite(qnorm) && t.n > 0) {
        const int groups = supers * 16;
        const float *sm = smax + ((size_t)(qi >> 4) * supers) * 16 + (qi & 15);
        const float *gm = gmax + ((size_t)(qi >> 4) * groups) * 16 + (qi & 15);
        int n_supers, n_groups;
        choose<kThreads>([&](int i) { return mx_order(sm[(size_t)i * 16]); }, supers, kk, chosen_supers, sh, n_supers);
        for (int i = tid; i < n_supers * 16; i += kThreads)
            values[i] = mx_order(gm[((size_t)chosen_supers[i >> 4] * 16 + (i & 15)) * 16]);
        __syncthreads();
        const u32 limit = choose<kThreads>([&](int i) { return values[i]; }, n_supers * 16, kk, chosen, sh, n_groups);
        if (tid == 0) sh.count = 0;
        __syncthreads();
        // scores of the chosen groups' rows; every column of the instruction holds the query
        const int r = lane & 15, g = lane >> 4;
        for (int tile = wave; tile < n_groups * (kGroup / 16); tile += kThreads / 64) {
            const int c = chosen[tile / (kGroup / 16)];
            const int row0 = (chosen_supers[c >> 4] * 16 + (c & 15)) * kGroup + (tile % (kGroup / 16)) * 16;
            f32x4 acc;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int x = row0 + 4 * g + j;
                const float norm = x < t.n ? t.norms[x] : __builtin_inff();
                acc[j] = mx_finite(norm) ? -0.5f * norm : -__builtin_inff();
            }
            const int row = min(row0 + r, t.n - 1);
            const bool ok = mx_finite(t.norms[row]);
            for (int s = 0; s < (t.nb + 3) / 4; ++s) {
                Operand x = mx_load(t, row, 4 * s + g);
                if (!ok) x.scale = 0;
                acc = mx_mma(x, mx_load(q, first + qi, 4 * s + g), acc);
            }
            const float s = r == 0 ? acc[0] : r == 1 ? acc[1] : r == 2 ? acc[2] : acc[3];
            const int id = row0 + 4 * g + r;
            const u32 order = mx_order(s);
            if (r < 4 && id < t.n && id != self && order > kOrderMinusInf && order >= limit)
                keys[atomicAdd(&sh.count, 1u)] = ((u64)~order << 32) | (u32)id;
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
        const float s = live ? mx_unorder(~(u32)(keys[i] >> 32)) : 0.0f;
        out_ids[i] = live ? (int)(u32)keys[i] : -1;
        out_dists[i] = live ? fmaxf(fmaf(-2.0f, s, qnorm), 0.0f) : __builtin_inff();
    }
}

struct NearestShape {
    int supers, chunk;             // supers of the table, queries per pass
    size_t gmax_bytes, smax_bytes, bytes, lds;
};
inline NearestShape nearest_shape(int64_t n, int64_t nq, int k)
{
    NearestShape s;
    s.supers = (int)((n + kSuper - 1) / kSuper);
    const size_t per16 = (size_t)s.supers * 17 * 16 * sizeof(float);     // 16 queries: groups and supers
    size_t sixteens = per16 ? kMaxWorkspace / per16 : (size_t)nq;
    if (sixteens < 16) sixteens = 16;
    const size_t all = (size_t)(nq + 15) / 16;
    if (sixteens >= all) sixteens = all;
    else if (sixteens > 16) sixteens &= ~(size_t)15;
    s.chunk = (int)(sixteens * 16);
    s.gmax_bytes = align_up(sixteens * s.supers * 16 * 16 * sizeof(float));
    s.smax_bytes = align_up(sixteens * s.supers * 16 * sizeof(float));
    s.bytes = s.gmax_bytes + s.smax_bytes + 256;
    const int kk = k + 1;
    size_t slots = 1;
    while (slots < (size_t)kk * kGroup) slots <<= 1;
    s.lds = slots * 8 + (size_t)kk * 16 * 4 + (size_t)kk * 8;
    return s;
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
    float *gmax = (float *)ws, *smax = (float *)((char *)ws + sh.gmax_bytes);
    EF_HIP_CHECK(hipFuncSetAttribute((const void *)pick_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sh.lds));
    for (int64_t first = 0; first < nq; first += sh.chunk) {
        const int cnt = (int)(nq - first < sh.chunk ? nq - first : sh.chunk);
        if (sh.supers > 0) {
            const int per_block = 4;
            const dim3 grid((unsigned)((sh.supers + per_block - 1) / per_block), (unsigned)((cnt + 255) / 256));
            if (grid.y > 65535) return EFANNA_EUNSUPPORTED;
            scan_kernel<<<grid, 256, 0, st>>>(t, q, (int)first, cnt, sh.supers, per_block, gmax, smax);
            EF_HIP_CHECK(hipGetLastError());
        }
        pick_kernel<<<(unsigned)cnt, 256, sh.lds, st>>>(t, q, (int)first, k, first_self, sh.supers, gmax, smax, ids, dists);
        EF_HIP_CHECK(hipGetLastError());
    }
    return EFANNA_OK;
}
