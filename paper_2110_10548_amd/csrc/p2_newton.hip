// Newton-Schulz products: X = G / (||G|| + eps), then A = X X^T, B = b A + c A A, X = a X + B X, some steps long.
//
// Numbers.  Small singular values of X grow by a = 3.4445 a step, 485 times over five steps, and what a step rounds off grows
// with them: with 16-bit operands the result of a gradient of low rank is off by 4 % (fp16) or 29 % (bf16).  So a
// matrix is kept as pairs of fp16 numbers, value = (high + low) / 2^scale, 22 bits together, in every step, and a product takes three MFMA:
// high*high + high*low + low*high, summed in fp32 (low*low is below what sums of more than 64 terms round off).  The scales come from the bound that the
// polynomial sets on the singular values, so that no entry passes fp16's largest number (no entry is larger than the
// largest singular value).
//
// Layout.  Every operand is stored with the summed index contiguous, so a product is always rows times rows:
// C[i][j] = sum_k P[i][k] Q[j][k].  32 values of k lie together as 64 bytes of highs and 64 bytes of lows: what a
// stage of the product's loop needs of a row is one line of 128 bytes.  A and B are symmetric and are their own transposes; only
// tiles on and below the diagonal are computed, and written to both sides.  X is kept in both orders (m x n for X X^T, n x m
// for B X).  Sizes are padded to multiples of 64 with zeros, which stay zeros through all steps.
//
// What it reaches, and what bounds it as far as counters show.  4096 x 4096 3.48 ms: the large products do 1.21 to 1.27 P operations a second (the last one, which writes one
// order alone, 1.38), all three terms of the tiles computed, where the installed library's plain 16-bit product of that size does 1.24 to 1.27; the matrix units are busy
// for half of the time at 2.4 GHz.  Around 1000 rows (2777 x 1000 fp32 313 us) neither they (13 to 27 %) nor one wait alone: wavefronts wait 26 to 41 % of their
// time, and for an instruction 16 to 48 %; L2 is read at 12.0 TB/s by X X^T (255 MB in 21.2 us) and 13.3 by B X (392 in 29.5).  Stacks of 256 x 256: launches and the first
// loads of each (17 in 155 us; deeper prefetch changes nothing).  Up to 128 rows: one launch, one block's chain of steps (64 x 64 18 us).
#include <algorithm>
#include <cmath>

#include "p2_train_dev.h"

namespace p2 {

namespace {

typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef half_t half4 __attribute__((ext_vector_type(4)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4), may_alias));

constexpr int kLine = 128;                     // bytes of 32 pairs
constexpr int64_t kUnits = 256;                // compute units
constexpr int64_t kMostNormParts = 1024;       // blocks that a matrix's norm is summed by

// Byte of the high half of pair k in a row; its low half is 64 further.
__device__ __forceinline__ int64_t pair_at(int64_t k) { return (k >> 5) * kLine + (k & 31) * 2; }
__device__ __forceinline__ float4_t multiply(half8 p, half8 q, float4_t sum) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q, sum, 0, 0, 0); }
// v as a sum of two.  The compiler may make `high` twice, once for its store and once for `low`, and where v is a product round it to 32 bits first in
// only one of the two: next to a tie they differ by a step of 11 bits (one entry in some thousand).  After the empty statement v is a number in
// 32 bits, whose halves come out the same however often they are made.
__device__ __forceinline__ void split(float v, half_t& high, half_t& low) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm("" : "+v"(v));
#endif
    high = (half_t)v;
    low = (half_t)fmaf((float)high, -1.0f, v);             // (one instruction with the conversion)
}

__device__ __forceinline__ uint32_t pack(float v) {
    half_t h, l;
    split(v, h, l);
    return (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
}
__device__ __forceinline__ void store_pairs(char* at, const uint32_t (&v)[4]) {
    uint2 high, low;
    high.x = __builtin_amdgcn_perm(v[1], v[0], 0x05040100);
    high.y = __builtin_amdgcn_perm(v[3], v[2], 0x05040100);
    low.x = __builtin_amdgcn_perm(v[1], v[0], 0x07060302);
    low.y = __builtin_amdgcn_perm(v[3], v[2], 0x07060302);
    *reinterpret_cast<uint2*>(at) = high;
    *reinterpret_cast<uint2*>(at + kLine / 2) = low;
}

// Sum over a block of 256 threads, the same for all of them.
__device__ __forceinline__ double block_sum_256(double s, double* buf) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = s;
    __syncthreads();
    return (buf[0] + buf[1]) + (buf[2] + buf[3]);
}
// What a matrix whose squares sum to s is multiplied by, as part * 2^power; zeros stay zeros without an eps, too.  The power of two
// comes first, so that values of any size lose nothing, and one rounding to 32 bits is left (64-bit products took twice the time).
struct Factor {
    float part;
    int power;
    __device__ __forceinline__ Factor(double s, double eps, double unit) {
        s = sqrt(s) + eps;
        const double f = s == 0.0 ? 0.0 : unit / s;
        part = (float)__builtin_amdgcn_frexp_mant(f);
        power = __builtin_amdgcn_frexp_exp(f);
    }
    __device__ __forceinline__ float operator()(float v) const { return __builtin_amdgcn_ldexpf(v, power) * part; }
};

// Sum of squares, in 64 bits: entries of any size, and no overflow before the root.  `across` threads (a power of two) take a
// row, 256 / across rows at a time.
template <typename T> __global__ __launch_bounds__(256) void k_newton_norm(const T* g, int64_t stride, int64_t matrix_stride, int64_t rows, int64_t cols,
                                                                           int32_t across, double* parts) {
    constexpr int V = 16 / sizeof(T);
    __shared__ double buf[4];
    const T* m = g + (int64_t)blockIdx.y * matrix_stride;
    const int tall = 256 / across;
    double s = 0.0;
    for (int64_t r = (int64_t)blockIdx.x * tall + threadIdx.x / across; r < rows; r += (int64_t)gridDim.x * tall)
        for (int64_t c = (int64_t)(threadIdx.x % across) * V; c < cols; c += (int64_t)across * V) {
            float v[V];
            load_part<T, V>(m + r * stride + c, cols - c, v, 0.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) s += (double)v[i] * (double)v[i];
        }
    s = block_sum_256(s, buf);
    if (threadIdx.x == 0) parts[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

// G / (||G|| + eps) as pairs in both orders: `straight` (rows x cols) and `turned` (cols x rows), zeros in the padding.
template <typename T> __global__ __launch_bounds__(256) void k_newton_scale(const T* g, int64_t stride, int64_t matrix_stride, int64_t rows, int64_t cols,
                                                                            const double* parts, int32_t n_parts, double eps, double unit, char* straight,
                                                                            char* turned, int64_t rows_padded, int64_t cols_padded, int64_t plane) {
    __shared__ uint32_t tile[64][65];
    __shared__ double buf[4];
    const T* m = g + (int64_t)blockIdx.z * matrix_stride;
    const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
    const int x = (threadIdx.x & 15) * 4, y = threadIdx.x >> 4;
    float v[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + y + i * 16, c = c0 + x;
        load_part<T, 4>(m + r * stride + c, r < rows ? cols - c : 0, v[i], 0.0f);
    }
    double s = 0.0;
    for (int i = threadIdx.x; i < n_parts; i += 256) s += parts[(int64_t)blockIdx.z * n_parts + i];
    s = block_sum_256(s, buf);
    const Factor factor(s, eps, unit);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = pack(factor(v[i][j]));
            tile[y + i * 16][x + j] = w[j];
        }
        store_pairs(straight + blockIdx.z * plane + (r0 + y + i * 16) * cols_padded * 4 + pair_at(c0 + x), w);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = tile[x + j][y + i * 16];
        store_pairs(turned + blockIdx.z * plane + (c0 + y + i * 16) * rows_padded * 4 + pair_at(r0 + x), w);
    }
}

enum : int { kGram = 0, kPoly = 1, kApply = 2, kPart = 3, kLast = 4, kLastBrain = 5, kLastHalf = 6 };     // the last ones: fp32, bf16, fp16

struct Product {
    const char* p; const char* q;              // pairs: rows of P and of Q
    const char* old;                           // kPoly: A; kApply, the last ones: X turned
    char* straight;                            // result (kGram, kPoly: the whole result)
    char* turned;
    void* out;                                 // the last ones; kPart: sums of the parts of k, [parts][matrices][rows][cols]
    int64_t p_plane, q_plane, old_plane, out_plane;      // from matrix to matrix: bytes (out: elements)
    int64_t k;                                 // summed length, padded
    int64_t rows, cols;                        // padded size of the result
    int64_t out_rows, out_cols, out_stride;    // the last ones: the result's own, and whether it is to be written turned
    float old_factor, sum_factor, gain;        // (old * old_factor + sum * sum_factor) * gain
    int32_t out_turned;
    int32_t tiles, parts;                      // blocks of a matrix; kPart: parts that k is cut into
    int64_t matrices;
};

// Four values in a row of the result, of which `n` are inside it.
__device__ __forceinline__ void store_four(void* p, int32_t type, int64_t at, int64_t n, const float (&v)[4]) {
    if (type == P2_F32) store_part<float, 4>(static_cast<float*>(p) + at, n, v);
    else if (type == P2_BF16) store_part<bf16_t, 4>(static_cast<bf16_t*>(p) + at, n, v);
    else store_part<half_t, 4>(static_cast<half_t*>(p) + at, n, v);
}

// Rows of an operand, `bytes` long altogether, and 16 bytes a lane of them to LDS (`to`: the wavefront's, lanes one after
// the other); what lies past the end comes as zeros.  Only the device's compiler knows the descriptor's type.
struct Rows {
#if defined(__HIP_DEVICE_COMPILE__)
    __amdgpu_buffer_rsrc_t at;
    __device__ __forceinline__ Rows(const char* p, int bytes) : at(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, bytes, 0x00027000)) {}
    __device__ __forceinline__ void bring(char* to, int lane_offset, int offset) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(at, (__attribute__((address_space(3))) void*)to, 16, lane_offset, offset, 0, 0);
    }
#else
    __device__ Rows(const char*, int) {}
    __device__ void bring(char*, int, int) const {}
#endif
};

// Waits until at most kLoads of this wavefront's loads are under way (and all its LDS reads are done), then for the others.
template <int kLoads> __device__ __forceinline__ void stage_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((kLoads & 15) | (kLoads >> 4) << 14 | 0x70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int kKind> struct Result { typedef float type; };
template <> struct Result<kLastBrain> { typedef bf16_t type; };
template <> struct Result<kLastHalf> { typedef half_t type; };

// One tile of C = P Q^T.  The tiles of P and Q come to LDS in stages of kSub times 32 values of k, kStages - 1 of them under way while one
// is multiplied.  A row of a stage takes 128 bytes; its
// 16-byte parts are exchanged by the row's number, so that the 16 rows that a wavefront reads at once lie in different banks.
// Rows past the end of P or Q are zeros: the loads' descriptors end with the matrix.
template <int kTile, int kWavesM, int kWavesN, int kStages, int kSub, int kKind>
__global__ __launch_bounds__(kWavesM * kWavesN * 64) void k_newton_product(Product a) {
    constexpr bool kEnd = kKind >= kLast;
    typedef typename Result<kKind>::type Out;
    constexpr int kWaves = kWavesM * kWavesN;
    constexpr int FM = kTile / kWavesM / 16, FN = kTile / kWavesN / 16;
    constexpr int kLoads = kTile / 8 / kWaves;             // of each operand a stage; one brings 8 rows
    constexpr int kAhead = kStages - 1;
    constexpr int kPerRow = (2 * kLoads + FM - 1) / FM;    // loads issued with a row of fragments: all of them in the first half
    static_assert(kLoads * 8 * kWaves == kTile && FM * kWavesM * 16 == kTile && FN * kWavesN * 16 == kTile, "rows are dealt out evenly");
    static_assert(2 * kLoads * kSub * (kAhead - 1) < 64, "the loads' counter");
    __shared__ __attribute__((aligned(1024))) char lds[kStages][kSub][2][kTile * kLine];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // Blocks go to the eight dies in turn: tiles are dealt out so that those of a die are neighbours, of as few matrices as can be.
    int t;
    {
        const int whole = gridDim.x / 8, rest = gridDim.x % 8, die = blockIdx.x & 7;
        t = die * whole + min(die, rest) + (blockIdx.x >> 3);
    }
    const int64_t matrix = t / a.tiles;
    t %= a.tiles;
    int part_of_k = 0;
    if constexpr (kKind == kPart) {
        part_of_k = t % a.parts;
        t /= a.parts;
    }
    int bi, bj;
    if constexpr (kKind == kGram || kKind == kPart || kKind == kPoly) {      // the t-th tile on or below the diagonal
        bi = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
        while ((bi + 1) * (bi + 2) / 2 <= t) ++bi;
        while (bi * (bi + 1) / 2 > t) --bi;
        bj = t - bi * (bi + 1) / 2;
    } else {                                               // column by column of four rows of tiles
        const int down = (int)((a.rows + kTile - 1) / kTile), across = (int)((a.cols + kTile - 1) / kTile);
        const int band = t / (4 * across), first = band * 4, high = min(4, down - first), in = t - first * across;
        bi = first + in % high;
        bj = in / high;
    }
    const int64_t pitch = a.k * 4;
    auto rows_of = [&](const char* m, int64_t first, int64_t rows) {
        return Rows(m + first * pitch, (int)(min(rows - first, (int64_t)kTile) * pitch));
    };
    const Rows p = rows_of(a.p + matrix * a.p_plane, (int64_t)bi * kTile, a.rows);
    const Rows q = rows_of(a.q + matrix * a.q_plane, (int64_t)bj * kTile, a.cols);
    const int part = (lane & 7) ^ (lane >> 3);
    const int from = (wave * kLoads * 8 + (lane >> 3)) * (int)pitch + part * 16;
    auto bring_one = [&](int stage, int sub, int l, int at) {          // the l-th load of each operand
        const int src = from + l * 8 * (int)pitch;
        const int dst = (wave * kLoads + l) * 1024;
        p.bring(&lds[stage][sub][0][dst], src, at + sub * kLine);
        q.bring(&lds[stage][sub][1][dst], src, at + sub * kLine);
    };
    const int wm = wave / kWavesN, wn = wave % kWavesN;
    const int row = lane & 15, quad = lane >> 4;
    const int64_t i0 = (int64_t)bi * kTile + wm * FM * 16, j0 = (int64_t)bj * kTile + wn * FN * 16;
    // The result's old values are asked for first: they are there when the products are.
    half4 high[FN], low[FN];
    auto fetch = [&](int fi) {
        if constexpr (kKind != kGram && kKind != kPart) {
            if (i0 + fi * 16 >= a.rows) return;
#pragma unroll
            for (int fj = 0; fj < FN; ++fj) {
                if (j0 + fj * 16 >= a.cols) continue;
                const char* o = a.old + matrix * a.old_plane + (j0 + fj * 16 + row) * a.rows * 4 + pair_at(i0 + fi * 16 + quad * 4);
                high[fj] = *reinterpret_cast<const half4*>(o);
                low[fj] = *reinterpret_cast<const half4*>(o + kLine / 2);
            }
        }
    };
    fetch(0);
    int stages = (int)(a.k / (32 * kSub)), begin = 0;
    if constexpr (kKind == kPart) {                        // (every part has a stage at least)
        begin = (int)((int64_t)stages * part_of_k / a.parts);
        stages = (int)((int64_t)stages * (part_of_k + 1) / a.parts) - begin;
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s)
        if (s < stages)
#pragma unroll
            for (int l = 0; l < kSub * kLoads; ++l) bring_one(s, l / kLoads, l % kLoads, (begin + s) * kSub * kLine);
    float4_t acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    // where this lane's 16 bytes of a row lie: highs and lows
    const int at0 = row * kLine + (quad ^ (row & 7)) * 16, at1 = row * kLine + ((quad + 4) ^ (row & 7)) * 16;
    int stage = 0, next = kAhead;
    for (int s = 0; s < stages; ++s) {
        if (s + kAhead <= stages) stage_barrier<2 * kLoads * kSub * (kAhead - 1)>();
        else stage_barrier<0>();
        const bool more = s + kAhead < stages;
        const int at = (begin + s + kAhead) * kSub * kLine;
#pragma unroll
        for (int sub = 0; sub < kSub; ++sub) {
            const char* tp = lds[stage][sub][0] + wm * FM * 16 * kLine;
            const char* tq = lds[stage][sub][1] + wn * FN * 16 * kLine;
            half8 q0[FN], q1[FN], p0, p1;
            p0 = *reinterpret_cast<const half8*>(tp + at0);
            p1 = *reinterpret_cast<const half8*>(tp + at1);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                q0[j] = *reinterpret_cast<const half8*>(tq + j * 16 * kLine + at0);
                q1[j] = *reinterpret_cast<const half8*>(tq + j * 16 * kLine + at1);
            }
            // The loads of a stage to come are spread over the first rows of fragments: issued together they would hold up this
            // stage's products for as long as the compute unit's address unit takes for all of them.
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                half8 n0, n1;
                if (i + 1 < FM) {
                    n0 = *reinterpret_cast<const half8*>(tp + (i + 1) * 16 * kLine + at0);
                    n1 = *reinterpret_cast<const half8*>(tp + (i + 1) * 16 * kLine + at1);
                }
                if (more)
#pragma unroll
                    for (int l = i * kPerRow; l < (i + 1) * kPerRow && l < kLoads; ++l) bring_one(next, sub, l, at);
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = multiply(p1, q0[j], acc[i][j]);
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = multiply(p0, q1[j], acc[i][j]);
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = multiply(p0, q0[j], acc[i][j]);
                p0 = n0;
                p1 = n1;
                if constexpr (kSub == 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
        next = stage;
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    if constexpr (kKind == kPart) {
        float* sums = static_cast<float*>(a.out) + (part_of_k * a.matrices + matrix) * a.rows * a.cols;
#pragma unroll
        for (int fi = 0; fi < FM; ++fi)
#pragma unroll
            for (int fj = 0; fj < FN; ++fj)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int64_t i = i0 + fi * 16 + quad * 4 + r, j = j0 + fj * 16 + row;
                    if (i < a.rows && j < a.cols) sums[i * a.cols + j] = acc[fi][fj][r];
                }
        return;
    }
    stage_barrier<0>();                                    // LDS changes its use: a strip of 16 rows for each wavefront
    // A lane has four rows i of one column j, which are four values in a row of the transpose.  For the result's own rows a
    // strip goes through LDS, where a lane picks up four columns of one row.
    constexpr int kPitch = FN * 16 + 4;
    static_assert(kWaves * 16 * kPitch * 4 <= (int)sizeof(lds), "the strips fit");
    uint32_t* strip = reinterpret_cast<uint32_t*>(&lds[0][0][0][0]) + wave * 16 * kPitch;
#pragma unroll
    for (int fi = 0; fi < FM; ++fi) {
        if (i0 + fi * 16 >= a.rows) break;                 // (padded sizes are whole fragments)
        uint32_t w[FN][4];
#pragma unroll
        for (int fj = 0; fj < FN; ++fj)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float v = acc[fi][fj][r] * a.sum_factor;
                if constexpr (kKind != kGram) v = fmaf((float)high[fj][r], a.old_factor, fmaf((float)low[fj][r], a.old_factor, v));
                w[fj][r] = kEnd ? __float_as_uint(v * a.gain) : pack(v);
            }
        if (fi + 1 < FM) fetch(fi + 1);
        const int64_t i = i0 + fi * 16 + quad * 4;
        if (!kEnd || a.out_turned) {
            char* t = kKind == kApply ? a.turned + matrix * a.q_plane : kEnd ? nullptr : a.straight + matrix * a.old_plane;
#pragma unroll
            for (int fj = 0; fj < FN; ++fj) {
                const int64_t j = j0 + fj * 16 + row;
                if constexpr (kEnd) {
                    const float f[4] = {__uint_as_float(w[fj][0]), __uint_as_float(w[fj][1]), __uint_as_float(w[fj][2]), __uint_as_float(w[fj][3])};
                    if (j < a.out_cols) store_part<Out, 4>(static_cast<Out*>(a.out) + matrix * a.out_plane + j * a.out_stride + i, a.out_rows - i, f);
                } else {
                    if (j < a.cols) store_pairs(t + j * a.rows * 4 + pair_at(i), w[fj]);
                }
            }
        }
        if (kKind == kApply || (kEnd ? !a.out_turned : bi != bj)) {
#pragma unroll
            for (int fj = 0; fj < FN; ++fj)
#pragma unroll
                for (int r = 0; r < 4; ++r) strip[(quad * 4 + r) * kPitch + fj * 16 + row] = w[fj][r];
            wavefront_exchange();
#pragma unroll
            for (int x = 0; x < FN; ++x) {
                const int item = x * 64 + lane, si = item / (FN * 4), sj = item % (FN * 4) * 4;
                const u32x4 u = *reinterpret_cast<const u32x4*>(strip + si * kPitch + sj);
                const int64_t ri = i0 + fi * 16 + si, rj = j0 + sj;
                if constexpr (kEnd) {
                    const float f[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
                    if (ri < a.out_rows) store_part<Out, 4>(static_cast<Out*>(a.out) + matrix * a.out_plane + ri * a.out_stride + rj, a.out_cols - rj, f);
                } else if (rj < a.cols) {
                    const uint32_t f[4] = {u.x, u.y, u.z, u.w};
                    store_pairs(a.straight + matrix * a.old_plane + ri * a.cols * 4 + pair_at(rj), f);
                }
            }
            wavefront_exchange();
        }
    }
}

// v * factor + (high + low) * old_factor
__device__ __forceinline__ float4_t add_halves(float4_t v, float factor, const half_t* high, const half_t* low, float old_factor) {
    const half4 h = *reinterpret_cast<const half4*>(high), l = *reinterpret_cast<const half4*>(low);
    float4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = fmaf((float)h[i], old_factor, fmaf((float)l[i], old_factor, v[i] * factor));
    return r;
}
__device__ __forceinline__ void store_halves(half_t* high, half_t* low, float4_t v) {
    half4 h, l;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        half_t hr, lr;
        split(v[r], hr, lr);
        h[r] = hr;
        l[r] = lr;
    }
    *reinterpret_cast<half4*>(high) = h;
    *reinterpret_cast<half4*>(low) = l;
}

// A float's two halves in the places of a pair: the results, all 32 bits of them.
typedef uint32_t words2 __attribute__((ext_vector_type(2), may_alias));
__device__ __forceinline__ void store_bits(half_t* high, half_t* low, float4_t v) {
    const uint32_t b0 = __float_as_uint(v[0]), b1 = __float_as_uint(v[1]), b2 = __float_as_uint(v[2]), b3 = __float_as_uint(v[3]);
    *reinterpret_cast<words2*>(high) = words2{b0 >> 16 | (b1 & 0xffff0000u), b2 >> 16 | (b3 & 0xffff0000u)};
    *reinterpret_cast<words2*>(low) = words2{(b0 & 0xffffu) | b1 << 16, (b2 & 0xffffu) | b3 << 16};
}
__device__ __forceinline__ float4_t load_bits(const half_t* high, const half_t* low) {
    const words2 h = *reinterpret_cast<const words2*>(high), l = *reinterpret_cast<const words2*>(low);
    return float4_t{__uint_as_float(h.x << 16 | (l.x & 0xffffu)), __uint_as_float((h.x & 0xffff0000u) | l.x >> 16),
                    __uint_as_float(h.y << 16 | (l.y & 0xffffu)), __uint_as_float((h.y & 0xffff0000u) | l.y >> 16)};
}

// A matrix whose smaller side is at most 32 kBlocks (128) and which fits in LDS goes through all its steps there: one block
// of eight wavefronts a matrix, one launch altogether.  X lies in rows, highs and lows apart, A and then B beside it.  A product's operands come from
// there; only X in B X is needed by columns, and a wavefront picks those of its 16 columns up value by value, once for all
// rows of the result.  What it writes are the same 16 columns, which nobody else reads meanwhile.
struct Small {
    const void* g; void* out;
    int64_t stride, matrix_stride, out_stride, out_plane;
    int32_t rows, cols, n;                     // n: the longer side, padded to 64
    int32_t out_type, steps;
    double eps, unit;
    float gain;
    float gram[64], poly_old[64], poly_sum[64], apply_old[64], apply_sum[64];
};
constexpr int kSmallBlock = 512;
constexpr int64_t kLdsBytes = 160 * 1024;
constexpr int64_t kSmallSpare = 128;                       // for the sums at its beginning
// Halves from row to row of A, and where value (r, c) lies.  16 lanes read 16 bytes each at a time, of rows 0 to 3 and 12 to 15
// at one place and of 4 to 11 at the next: with rows of 128 bytes (an odd number of them) or of 256, pieces of 16 bytes exchanged
// by the row's lowest three or four bits, they lie in different banks.  (Rows 16 bytes longer than that: 41 cycles in 100
// went into conflicts.)
__host__ __device__ constexpr int small_pitch(int m) { return m <= 64 ? 64 : 128; }
__host__ __device__ constexpr int small_mask(int pitch) { return pitch % 128 ? 7 : 15; }
__device__ __forceinline__ int small_at(int r, int c, int pitch, int mask) { return r * pitch + (((c >> 3) ^ (r & mask)) << 3 | (c & 7)); }
inline int64_t small_length(int64_t rows, int64_t cols) { return ceil_div(std::max(rows, cols), 64) * 64; }
inline int64_t small_bytes(int64_t m, int64_t n) {         // X, A, and where eight wavefronts share A's only blocks their sums
    return kSmallSpare + 4 * m * n + 4 * m * small_pitch((int)m) + (m == 32 ? kSmallBlock / 64 * 2 * 64 * 16 : 0);
}

template <typename T, int kBlocks> __global__ __launch_bounds__(kSmallBlock) void k_newton_small(Small a) {
    constexpr int M = 32 * kBlocks, kWaves = kSmallBlock / 64;
    // A wavefront has one block of A, of FM x FN fragments of 16 x 16; where there are only two blocks four wavefronts share
    // one's sum, every fourth 32 values of k each.
    constexpr int FM = kBlocks < 3 ? 1 : 2, FN = kBlocks < 3 ? 2 : kBlocks;
    constexpr int kAcross = M / (16 * FN), kAll = M / (16 * FM) * kAcross, kSplit = kBlocks == 1 ? kWaves / kAll : 1;
    constexpr int AP = small_pitch(M), kAMask = small_mask(AP);
    // Low times low is 2^-22 of a term at most, 2^-24 as a rule.  Of few rows the sums have so few roundings of their own that it counts: off by (mean of
    // forty normal matrices; without it / with it / products in 32 bits) 5 x 7 1.04 / 0.78 / 0.69e-6, 33 x 90 1.63 / 1.31 / 1.24e-6, 64 x 200 1.59 / 1.30 /
    // 1.43e-6, but 96 x 120 1.00 / 0.94 / 1.36e-6, where it would take 13 % of the time of 128 x 128 (of 64 x 64 5 %).
    constexpr bool kLowest = kBlocks <= 2;
    extern __shared__ __attribute__((aligned(16))) char small_lds[];
    const int XP = a.n, x_mask = small_mask(a.n);
    half_t* xh = reinterpret_cast<half_t*>(small_lds + kSmallSpare);
    half_t* xl = xh + M * XP;
    half_t* ah = xl + M * XP;
    half_t* al = ah + M * AP;
    double* buf = reinterpret_cast<double*>(small_lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, quad = lane >> 4;
    const int block = wave % (kWaves / kSplit), share = wave / (kWaves / kSplit);
    const bool has_block = block < kAll;
    const int i0 = block / kAcross * FM * 16, j0 = block % kAcross * FN * 16;
    const T* g = static_cast<const T*>(a.g) + (int64_t)blockIdx.x * a.matrix_stride;
    const bool tall = a.rows > a.cols;
    // Squares of 4 x 4 values a thread, whose four rows are under way together: once for the norm, once more (from the cache) for
    // LDS, where four values of a row of X, which are a row or a column of the square, are written at a time.
    const int across = (a.cols + 3) / 4, squares = (a.rows + 3) / 4 * across;
    auto each = [&](auto&& use) {
        for (int at = threadIdx.x; at < squares; at += kSmallBlock) {
            const int r = at / across * 4, c = at % across * 4;
            float v[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u) load_part<T, 4>(g + (int64_t)min(r + u, a.rows - 1) * a.stride + c, r + u < a.rows ? a.cols - c : 0, v[u], 0.0f);
            use(r, c, v);
        }
    };
    double s = 0.0;
    each([&](int, int, const float (&v)[4][4]) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s += (double)v[u][e] * (double)v[u][e];
    });
    for (int i = threadIdx.x; i < 2 * M * XP / 8; i += kSmallBlock) reinterpret_cast<half8*>(xh)[i] = half8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if (lane == 0) buf[wave] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += buf[w];
    const Factor factor(s, a.eps, a.unit);
    each([&](int r, int c, const float (&v)[4][4]) {       // (what lies beyond the matrix is zeros, and inside the padding)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float4_t x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = factor(tall ? v[e][u] : v[u][e]);
            const int at = tall ? small_at(c + u, r, XP, x_mask) : small_at(r + u, c, XP, x_mask);
            store_halves(xh + at, xl + at, x);
        }
    });
    __syncthreads();
    for (int step = 0; step < a.steps; ++step) {
        const bool last = step + 1 == a.steps;
        float4_t acc[FM][FN];
        auto square = [&](const half_t* ph, const half_t* pl, int pitch, int mask, int length) {     // P P^T
#pragma unroll
            for (int x = 0; x < FM; ++x)
#pragma unroll
                for (int y = 0; y < FN; ++y) acc[x][y] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
            const int pi = (i0 + row) * pitch, pj = (j0 + row) * pitch;
            if (has_block)
                for (int k = share * 32; k < length; k += 32 * kSplit) {
                    half8 p0[FM], p1[FM], q0[FN], q1[FN];
                    const int kk = (((k >> 3) + quad) ^ (row & mask)) * 8;           // (of 16 rows in a row: the same for all of them)
#pragma unroll
                    for (int x = 0; x < FM; ++x) {
                        p0[x] = *reinterpret_cast<const half8*>(ph + pi + x * 16 * pitch + kk);
                        p1[x] = *reinterpret_cast<const half8*>(pl + pi + x * 16 * pitch + kk);
                    }
#pragma unroll
                    for (int y = 0; y < FN; ++y) {
                        q0[y] = *reinterpret_cast<const half8*>(ph + pj + y * 16 * pitch + kk);
                        q1[y] = *reinterpret_cast<const half8*>(pl + pj + y * 16 * pitch + kk);
                    }
#pragma unroll
                    for (int x = 0; x < FM; ++x)
#pragma unroll
                        for (int y = 0; y < FN; ++y) {
                            if constexpr (kLowest) acc[x][y] = multiply(p1[x], q1[y], acc[x][y]);
                            acc[x][y] = multiply(p1[x], q0[y], acc[x][y]);
                        }
#pragma unroll
                    for (int x = 0; x < FM; ++x)
#pragma unroll
                        for (int y = 0; y < FN; ++y) acc[x][y] = multiply(p0[x], q1[y], acc[x][y]);
#pragma unroll
                    for (int x = 0; x < FM; ++x)
#pragma unroll
                        for (int y = 0; y < FN; ++y) acc[x][y] = multiply(p0[x], q0[y], acc[x][y]);
                }
            if constexpr (kSplit > 1) {                    // the shares' sums in their order
                float4_t* part = reinterpret_cast<float4_t*>(al + M * AP);
#pragma unroll
                for (int y = 0; y < FN; ++y) part[(wave * FN + y) * 64 + lane] = acc[0][y];
                __syncthreads();
#pragma unroll
                for (int y = 0; y < FN; ++y) {
                    acc[0][y] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int p = 0; p < kSplit; ++p) acc[0][y] += part[((p * kAll + block) * FN + y) * 64 + lane];
                }
            }
        };
        // A and B are symmetric: a lane's four rows of one column are four values of a row
        auto at_of = [&](int x, int y) { return small_at(j0 + y * 16 + row, i0 + x * 16 + quad * 4, AP, kAMask); };
        auto place = [&](float factor) {
            if (!has_block || share) return;
#pragma unroll
            for (int x = 0; x < FM; ++x)
#pragma unroll
                for (int y = 0; y < FN; ++y) store_halves(ah + at_of(x, y), al + at_of(x, y), acc[x][y] * factor);
        };
        square(xh, xl, XP, x_mask, a.n);
        place(a.gram[step]);
        __syncthreads();
        square(ah, al, AP, kAMask, M);
        if (has_block)
#pragma unroll
            for (int x = 0; x < FM; ++x)
#pragma unroll
                for (int y = 0; y < FN; ++y)
                    acc[x][y] = add_halves(acc[x][y], a.poly_sum[step], ah + at_of(x, y), al + at_of(x, y), a.poly_old[step]);
        __syncthreads();                                   // everybody has read A
        place(1.0f);
        __syncthreads();
#pragma unroll 1
        for (int jb = wave * 16; jb < a.n; jb += kWaves * 16) {
            half8 q0[kBlocks], q1[kBlocks];
#pragma unroll
            for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = small_at(k * 32 + quad * 8 + e, jb + row, XP, x_mask);
                    q0[k][e] = xh[at];
                    q1[k][e] = xl[at];
                }
            // columns of X times rows of B: a lane has four columns j of one row i
            float4_t c[2 * kBlocks];
#pragma unroll
            for (int i = 0; i < 2 * kBlocks; ++i) {
                c[i] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < kBlocks; ++k) {
                    const int at = small_at(i * 16 + row, k * 32 + quad * 8, AP, kAMask);
                    const half8 p0 = *reinterpret_cast<const half8*>(ah + at), p1 = *reinterpret_cast<const half8*>(al + at);
                    if constexpr (kLowest) c[i] = multiply(q1[k], p1, c[i]);
                    c[i] = multiply(q0[k], p1, c[i]);
                    c[i] = multiply(q1[k], p0, c[i]);
                    c[i] = multiply(q0[k], p0, c[i]);
                }
            }
            // all old values before the first new one: no read then waits for a write
#pragma unroll
            for (int i = 0; i < 2 * kBlocks; ++i) {
                const int at = small_at(i * 16 + row, jb + quad * 4, XP, x_mask);
                c[i] = add_halves(c[i], a.apply_sum[step], xh + at, xl + at, a.apply_old[step]);
            }
            wavefront_exchange();                          // (all lanes have their columns)
#pragma unroll
            for (int i = 0; i < 2 * kBlocks; ++i) {
                const int ri = i * 16 + row, rj = jb + quad * 4;
                const int at = small_at(ri, rj, XP, x_mask);
                if (last) store_bits(xh + at, xl + at, c[i] * a.gain);
                else store_halves(xh + at, xl + at, c[i]);
            }
        }
        __syncthreads();
    }
    for (int at = threadIdx.x; at < squares; at += kSmallBlock) {
        const int r = at / across * 4, c = at % across * 4;
        float4_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int from = tall ? small_at(c + u, r, XP, x_mask) : small_at(r + u, c, XP, x_mask);
            v[u] = load_bits(xh + from, xl + from);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float o[4] = {tall ? v[0][u] : v[u][0], tall ? v[1][u] : v[u][1], tall ? v[2][u] : v[u][2], tall ? v[3][u] : v[u][3]};
            if (r + u < a.rows) store_four(a.out, a.out_type, (int64_t)blockIdx.x * a.out_plane + (r + u) * a.out_stride + c, a.cols - c, o);
        }
    }
}

constexpr int64_t kPad = 64;                   // two fragments of k, four of rows; tiles may be larger
inline int64_t padded(int64_t v) { return ceil_div(v, kPad) * kPad; }
inline int64_t align256(int64_t v) { return (v + 255) / 256 * 256; }

// Largest value of |a x + b x^3 + c x^5| on [0, top].
double poly_bound(double a, double b, double c, double top) {
    auto f = [&](double x) { return std::fabs(x * (a + x * x * (b + x * x * c))); };
    double most = f(top);
    // a + 3 b s + 5 c s^2 = 0 with s = x^2
    const double qa = 5 * c, qb = 3 * b, qc = a;
    double roots[2] = {-1.0, -1.0};
    if (qa != 0.0) {
        const double d = qb * qb - 4 * qa * qc;
        if (d >= 0.0) { roots[0] = (-qb + std::sqrt(d)) / (2 * qa); roots[1] = (-qb - std::sqrt(d)) / (2 * qa); }
    } else if (qb != 0.0) {
        roots[0] = -qc / qb;
    }
    for (double s : roots) if (s > 0.0 && s < top * top) most = std::max(most, f(std::sqrt(s)));
    return most;
}
// Largest value of |b s + c s^2| on [0, top].
double square_bound(double b, double c, double top) {
    auto f = [&](double s) { return std::fabs(s * (b + c * s)); };
    double most = f(top);
    const double s = c != 0.0 ? -b / (2 * c) : -1.0;
    if (s > 0.0 && s < top) most = std::max(most, f(s));
    return most;
}
// The power of two that brings `bound`, and a little more, just below fp16's largest number.
double unit_for(double bound) {
    int e;
    std::frexp(std::max(bound, 1e-4) * 1.02 / 65504.0, &e);
    return std::ldexp(1.0, -e);
}

// A = sum of its parts, in their order, as pairs on both sides of the diagonal: a block takes a tile of 64 x 64 on or below it.
__global__ __launch_bounds__(256) void k_newton_join(const float* sums, int32_t parts, int64_t matrices, int64_t m, float factor, char* to, int64_t plane) {
    __shared__ float tile[64][65];
    int bi = (int)((sqrtf(8.0f * (float)blockIdx.x + 1.0f) - 1.0f) * 0.5f);
    while ((bi + 1) * (bi + 2) / 2 <= (int)blockIdx.x) ++bi;
    while (bi * (bi + 1) / 2 > (int)blockIdx.x) --bi;
    const int bj = (int)blockIdx.x - bi * (bi + 1) / 2;
    const int64_t matrix = blockIdx.y, i0 = (int64_t)bi * 64, j0 = (int64_t)bj * 64;
    const int x = (threadIdx.x & 15) * 4, y = threadIdx.x >> 4;
    char* out = to + matrix * plane;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int64_t i = i0 + y + n * 16;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int p = 0; p < parts; ++p) {
            float w[4];
            load_vec<float, 4>(sums + ((p * matrices + matrix) * m + i) * m + j0 + x, w);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] += w[q];
        }
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] *= factor;
            tile[y + n * 16][x + q] = v[q];
            w[q] = pack(v[q]);
        }
        if (bi != bj) store_pairs(out + i * m * 4 + pair_at(j0 + x), w);
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = pack(tile[x + q][y + n * 16]);
        store_pairs(out + (j0 + y + n * 16) * m * 4 + pair_at(i0 + x), w);
    }
}

int64_t tiles_of(const Product& p, int64_t tile, int kind) {
    const int64_t down = ceil_div(p.rows, tile), across = ceil_div(p.cols, tile);
    return kind == kGram || kind == kPart || kind == kPoly ? down * (down + 1) / 2 : down * across;
}

template <int kTile, int kWavesM, int kWavesN, int kStages, int kSub> void product(Product p, int kind, hipStream_t s) {
    p.tiles = (int32_t)tiles_of(p, kTile, kind) * (kind == kPart ? p.parts : 1);
    const dim3 grid((unsigned)(p.tiles * p.matrices));
    const dim3 block(kWavesM * kWavesN * 64);
#define P2_PRODUCT(KIND) k_newton_product<kTile, kWavesM, kWavesN, kStages, kSub, KIND><<<grid, block, 0, s>>>(p)
    if (kind == kGram) P2_PRODUCT(kGram);
    else if (kind == kPoly) P2_PRODUCT(kPoly);
    else if (kind == kApply) P2_PRODUCT(kApply);
    else if (kind == kLastBrain) P2_PRODUCT(kLastBrain);
    else if (kind == kLastHalf) P2_PRODUCT(kLastHalf);
    else P2_PRODUCT(kLast);
#undef P2_PRODUCT
}

// The tile of a product.  What a stage of 32 values of k takes, in us on a compute unit that has one tile of its size
// (measured, products of 1000 to 4096 rows): 256 x 256 2.45, 192 x 192 1.4, 128 x 128 0.7; of 64 x 64 several share a
// unit's time, 0.25 for each.  Larger tiles need less of each operand's traffic and smaller ones leave fewer units idle:
// X X^T of 4096 x 4096 takes 266 us in 136 tiles of 256, 200 in 253 of 192, 240 in 528 of 128, 340 in 2080 of 64, and B X
// 329, 404, 355, 460; X X^T of 1000 x 2777 takes 165, 103, 66 and 30.  Where no unit has two tiles of 64 x 64 a stage's latency
// counts: eight wavefronts and 64 values of k between barriers (updates of 512 x 512 126 us for 141, 1024 x 1024 186 for
// 225); where units do, the LDS that this takes would keep their other tiles out (32 updates of 256 x 256 172 us for 152).
// Where the units suffice for tiles of 48 x 48, more of them have one: three wavefronts, each 16 rows of all columns, and three
// stages under way (updates of 1000 x 2777 288 us for 306, 1024 x 4096 351 for 367, 512 x 2048
// 168 for 173, two of 700 x 2000 230 for 242; with two stages under way 295, 356, 167 and 233).
void product_by_size(const Product& p, int kind, hipStream_t s) {
    auto cost = [&](int64_t tile, double stage, bool shared) {
        const int64_t tiles = tiles_of(p, tile, kind) * p.matrices;
        return stage * (shared ? std::max(1.0, (double)tiles / kUnits) : (double)ceil_div(tiles, kUnits));
    };
    const double c64 = cost(64, 0.25, true), c128 = cost(128, 0.7, false), c192 = cost(192, 1.4, false), c256 = cost(256, 2.45, false);
    const double least = std::min({c64, c128, c192, c256});
    if (c256 == least) product<256, 2, 4, 2, 1>(p, kind, s);
    else if (c192 == least) product<192, 2, 4, 3, 1>(p, kind, s);
    else if (c128 == least) product<128, 2, 4, 2, 1>(p, kind, s);
    else if (tiles_of(p, 48, kind) * p.matrices <= kUnits) product<48, 3, 1, 4, 2>(p, kind, s);
    else if (tiles_of(p, 64, kind) * p.matrices <= kUnits) product<64, 2, 4, 3, 2>(p, kind, s);
    else product<64, 2, 2, 3, 1>(p, kind, s);
}

// X X^T of a short and long X has few tiles and a long sum: it is cut into as many parts as there are compute units for, of 16
// stages at least, whose sums k_newton_join adds up.  1: it is not cut.
int64_t gram_parts(int64_t count, int64_t m, int64_t n) {
    const int64_t down = ceil_div(m, 64), tiles = down * (down + 1) / 2 * count;
    return std::max<int64_t>(1, std::min(kUnits / tiles, n / 512));
}

int64_t norm_parts(int64_t rows, int64_t cols) {           // 8192 values a block, and not more than rows
    return std::max<int64_t>(1, std::min({kMostNormParts, ceil_div(rows * cols, 8192), rows}));
}

template <typename T> void to_pairs(const Orthogonalize& a, double unit, double* parts, char* straight, char* turned, int64_t rp, int64_t cp,
                                    int64_t plane, hipStream_t s) {
    const T* g = static_cast<const T*>(a.g);
    const int n = (int)norm_parts(a.rows, a.cols);
    int across = 1;
    while (across < 256 && across * (16 / (int)sizeof(T)) < a.cols) across *= 2;
    k_newton_norm<T><<<dim3((unsigned)n, (unsigned)a.count), dim3(256), 0, s>>>(g, a.stride, a.matrix_stride, a.rows, a.cols, across, parts);
    k_newton_scale<T><<<dim3((unsigned)(cp / 64), (unsigned)(rp / 64), (unsigned)a.count), dim3(256), 0, s>>>(
        g, a.stride, a.matrix_stride, a.rows, a.cols, parts, n, a.eps, unit, straight, turned, rp, cp, plane);
}

}  // namespace

bool orthogonalize_bounds(const Orthogonalize& a, double* bounds) {
    double top = 1.0;
    for (int i = 0; i <= a.steps; ++i) {
        bounds[i] = top;
        if (!(top <= 1024.0)) return false;
        top = poly_bound(a.a, a.b, a.c, top * 1.001);      // (what rounding adds to the singular values, many times over)
    }
    return true;
}

namespace {

// The powers of two that a step's matrices are kept in, as factors of its products.
struct StepFactors {
    double unit;                               // of the X that the step makes
    float gram, poly_old, poly_sum, apply_old, apply_sum;
};
StepFactors step_factors(const Orthogonalize& a, int step, double unit) {
    const double top = a.bounds[step] * 1.001;
    const double ua = unit_for(top * top), ub = unit_for(square_bound(a.b, a.c, top * top));
    StepFactors f;
    f.unit = unit_for(a.bounds[step + 1]);
    f.gram = (float)(ua / (unit * unit));
    f.poly_old = (float)(a.b * ub / ua);
    f.poly_sum = (float)(a.c * ub / (ua * ua));
    f.apply_old = (float)(a.a * f.unit / unit);
    f.apply_sum = (float)(f.unit / (ub * unit));
    return f;
}

bool is_small(int64_t rows, int64_t cols) {
    const int64_t m = ceil_div(std::min(rows, cols), 32) * 32, n = small_length(rows, cols);
    return m <= 128 && small_bytes(m, n) <= kLdsBytes;
}

template <typename T, int kBlocks> hipError_t small_as(const Small& p, int64_t count, hipStream_t s) {
    const size_t bytes = (size_t)small_bytes(32 * kBlocks, p.n);
    if (bytes > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_newton_small<T, kBlocks>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLdsBytes);
        if (e != hipSuccess) return e;
    }
    k_newton_small<T, kBlocks><<<dim3((unsigned)count), dim3(kSmallBlock), bytes, s>>>(p);
    return hipGetLastError();
}
template <typename T> hipError_t small_of(const Small& p, int64_t count, hipStream_t s) {
    switch (ceil_div(std::min(p.rows, p.cols), 32)) {
        case 1: return small_as<T, 1>(p, count, s);
        case 2: return small_as<T, 2>(p, count, s);
        case 3: return small_as<T, 3>(p, count, s);
        default: return small_as<T, 4>(p, count, s);
    }
}

hipError_t launch_small(const Orthogonalize& a, hipStream_t s) {
    Small p = {};
    p.g = a.g; p.out = a.out;
    p.stride = a.stride; p.matrix_stride = a.matrix_stride; p.out_stride = a.out_stride; p.out_plane = a.out_matrix_stride;
    p.rows = (int32_t)a.rows; p.cols = (int32_t)a.cols; p.n = (int32_t)small_length(a.rows, a.cols);
    p.out_type = a.out_type; p.steps = a.steps;
    p.eps = a.eps;
    double unit = p.unit = unit_for(a.bounds[0]);
    for (int i = 0; i < a.steps; ++i) {
        const StepFactors f = step_factors(a, i, unit);
        p.gram[i] = f.gram; p.poly_old[i] = f.poly_old; p.poly_sum[i] = f.poly_sum; p.apply_old[i] = f.apply_old; p.apply_sum[i] = f.apply_sum;
        unit = f.unit;
    }
    p.gain = (float)(a.scale / unit);
    if (a.type == P2_F32) return small_of<float>(p, a.count, s);
    if (a.type == P2_BF16) return small_of<bf16_t>(p, a.count, s);
    return small_of<half_t>(p, a.count, s);
}

}  // namespace

int64_t orthogonalize_workspace(int64_t count, int64_t rows, int64_t cols) {
    if (is_small(rows, cols)) return 0;
    const int64_t m = padded(std::min(rows, cols)), n = padded(std::max(rows, cols));
    const int64_t parts = gram_parts(count, m, n);
    return align256(count * norm_parts(rows, cols) * 8) + count * 4 * (3 * m * n + (2 + (parts > 1 ? parts : 0)) * m * m);
}

hipError_t launch_orthogonalize(const Orthogonalize& a, hipStream_t s) {
    if (is_small(a.rows, a.cols)) return launch_small(a, s);
    const bool tall = a.rows > a.cols;
    const int64_t m = padded(std::min(a.rows, a.cols)), n = padded(std::max(a.rows, a.cols));
    const int64_t xb = m * n * 4, ab = m * m * 4;
    char* w = static_cast<char*>(a.workspace);
    double* squares = reinterpret_cast<double*>(w);
    w += align256(a.count * norm_parts(a.rows, a.cols) * 8);
    char* x = w; w += a.count * xb;
    char* xt[2];
    xt[0] = w; w += a.count * xb;
    xt[1] = w; w += a.count * xb;
    char* ga = w; w += a.count * ab;
    char* gb = w; w += a.count * ab;
    float* sums = reinterpret_cast<float*>(w);
    const int64_t parts = gram_parts(a.count, m, n);
    double unit = unit_for(a.bounds[0]);
    char* straight = tall ? xt[0] : x;
    char* turned = tall ? x : xt[0];
    const int64_t rp = tall ? n : m, cp = tall ? m : n;
    if (a.type == P2_F32) to_pairs<float>(a, unit, squares, straight, turned, rp, cp, xb, s);
    else if (a.type == P2_BF16) to_pairs<bf16_t>(a, unit, squares, straight, turned, rp, cp, xb, s);
    else to_pairs<half_t>(a, unit, squares, straight, turned, rp, cp, xb, s);
    hipError_t e = hipGetLastError();
    for (int i = 0; i < a.steps && e == hipSuccess; ++i) {
        const bool last = i + 1 == a.steps;
        // (Pairs in the last step, too, whatever the result's type: a X and B X may cancel, and then they magnify what upper halves round off.)
        const StepFactors f = step_factors(a, i, unit);
        Product p = {};
        p.matrices = a.count;
        p.p = p.q = x; p.p_plane = p.q_plane = xb;
        p.straight = ga; p.old_plane = ab;
        p.k = n; p.rows = p.cols = m;
        p.sum_factor = f.gram;
        if (parts > 1) {
            p.out = sums; p.parts = (int32_t)parts;
            p.tiles = (int32_t)(tiles_of(p, 64, kPart) * parts);
            k_newton_product<64, 2, 2, 3, 2, kPart><<<dim3((unsigned)(p.tiles * a.count)), dim3(256), 0, s>>>(p);
            k_newton_join<<<dim3((unsigned)tiles_of(p, 64, kPart), (unsigned)a.count), dim3(256), 0, s>>>(sums, (int32_t)parts, a.count, m, f.gram, ga, ab);
        } else {
            product_by_size(p, kGram, s);
        }
        p = {};
        p.matrices = a.count;
        p.p = p.q = p.old = ga; p.p_plane = p.q_plane = p.old_plane = ab;
        p.straight = gb;
        p.k = p.rows = p.cols = m;
        p.old_factor = f.poly_old;
        p.sum_factor = f.poly_sum;
        product_by_size(p, kPoly, s);
        p = {};
        p.matrices = a.count;
        p.p = gb; p.p_plane = ab;
        p.q = p.old = xt[i & 1]; p.q_plane = p.old_plane = xb;
        p.straight = x; p.turned = xt[(i + 1) & 1];
        p.k = p.rows = m; p.cols = n;
        p.old_factor = f.apply_old;
        p.sum_factor = f.apply_sum;
        if (last) {
            p.out = a.out; p.out_plane = a.out_matrix_stride; p.out_stride = a.out_stride;
            p.out_rows = std::min(a.rows, a.cols); p.out_cols = std::max(a.rows, a.cols);
            p.out_turned = tall;
            p.gain = (float)(a.scale / f.unit);
        }
        product_by_size(p, !last ? kApply : a.out_type == P2_BF16 ? kLastBrain : a.out_type == P2_F16 ? kLastHalf : kLast, s);
        unit = f.unit;
        e = hipGetLastError();
    }
    return e;
}

}  // namespace p2
