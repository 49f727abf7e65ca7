// Newton-Schulz products: X = G / (||G|| + eps), then A = X X^T, B = b A + c A A, X = a X + B X, some steps long.
//
// Numbers.  Small singular values of X grow by a = 3.4445 a step, 485 times over five steps, and what a step rounds off grows
// with them: with 16-bit operands the result of a gradient of low rank is off by 4 % (fp16) or 29 % (bf16).  So a
// matrix is kept as pairs of fp16 numbers, value = (high + low) / 2^scale, 22 bits together, and a product takes three MFMA:
// high*high + high*low + low*high, summed in fp32 (low*low is below what fp32 holds).  The scales come from the bound that the
// polynomial sets on the singular values, so that no entry passes fp16's largest number (no entry is larger than the
// largest singular value).
//
// Layout.  Every operand is stored with the summed index contiguous, so a product is always rows times rows:
// C[i][j] = sum_k P[i][k] Q[j][k].  32 values of k lie together as 64 bytes of highs and 64 bytes of lows: what one
// step of the product's loop needs of a row is one line of 128 bytes.  A and B are symmetric and are their own transposes; only
// tiles on and below the diagonal are computed, and written to both sides.  X is kept in both orders (m x n for X X^T, n x m
// for B X).  Sizes are padded to whole tiles with zeros, which stay zeros through all steps.
#include <algorithm>
#include <cmath>

#include "p2_train_dev.h"

namespace p2 {

namespace {

typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef half_t half4 __attribute__((ext_vector_type(4)));
typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr int kLine = 128;                     // bytes of 32 pairs
constexpr int kNormParts = 64;                 // blocks that a matrix's norm is summed by

// Byte of the high half of pair k in a row; its low half is 64 further.
__device__ __forceinline__ int64_t pair_at(int64_t k) { return (k >> 5) * kLine + (k & 31) * 2; }
__device__ __forceinline__ void split(float v, half_t& high, half_t& low) {
    high = (half_t)v;
    low = (half_t)(v - (float)high);
}

// Sum of squares, in 64 bits: entries of any size, and no overflow before the root.
template <typename T> __global__ __launch_bounds__(256) void k_newton_norm(const T* g, int64_t stride, int64_t matrix_stride, int64_t rows, int64_t cols,
                                                                           double* parts) {
    __shared__ double buf[4];
    const T* m = g + (int64_t)blockIdx.y * matrix_stride;
    double s = 0.0;
    for (int64_t r = blockIdx.x; r < rows; r += kNormParts)
        for (int64_t c = threadIdx.x; c < cols; c += 256) { const double v = (double)(float)m[r * stride + c]; s += v * v; }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) parts[(int64_t)blockIdx.y * kNormParts + blockIdx.x] = buf[0] + buf[1] + buf[2] + buf[3];
}

// G / (||G|| + eps) as pairs in both orders: `straight` (rows x cols) and `turned` (cols x rows), zeros in the padding.
template <typename T> __global__ __launch_bounds__(256) void k_newton_scale(const T* g, int64_t stride, int64_t matrix_stride, int64_t rows, int64_t cols,
                                                                            const double* parts, double eps, double unit, char* straight, char* turned,
                                                                            int64_t rows_padded, int64_t cols_padded, int64_t plane) {
    __shared__ float tile[32][33];
    __shared__ double factor;
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int i = 0; i < kNormParts; ++i) s += parts[(int64_t)blockIdx.z * kNormParts + i];
        s = sqrt(s) + eps;
        factor = s == 0.0 ? 0.0 : unit / s;
    }
    __syncthreads();
    const T* m = g + (int64_t)blockIdx.z * matrix_stride;
    const int64_t r0 = (int64_t)blockIdx.y * 32, c0 = (int64_t)blockIdx.x * 32;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    for (int i = y; i < 32; i += 8) {
        const int64_t r = r0 + i, c = c0 + x;
        const float v = r < rows && c < cols ? (float)((double)(float)m[r * stride + c] * factor) : 0.0f;
        tile[i][x] = v;
        half_t high, low;
        split(v, high, low);
        char* at = straight + blockIdx.z * plane + r * cols_padded * 4 + pair_at(c);
        *reinterpret_cast<half_t*>(at) = high;
        *reinterpret_cast<half_t*>(at + 64) = low;
    }
    __syncthreads();
    for (int i = y; i < 32; i += 8) {
        half_t high, low;
        split(tile[x][i], high, low);
        char* at = turned + blockIdx.z * plane + (c0 + i) * rows_padded * 4 + pair_at(r0 + x);
        *reinterpret_cast<half_t*>(at) = high;
        *reinterpret_cast<half_t*>(at + 64) = low;
    }
}

enum : int { kGram = 0, kPoly = 1, kApply = 2, kLast = 3 };

struct Product {
    const char* p; const char* q;              // pairs: rows of P and of Q
    const char* old;                           // kPoly: A; kApply, kLast: X turned
    char* straight;                            // result (kGram, kPoly: the whole result)
    char* turned;
    void* out;                                 // kLast
    int64_t p_plane, q_plane, old_plane, out_plane;      // from matrix to matrix: bytes (out: elements)
    int64_t k;                                 // summed length, padded
    int64_t rows, cols;                        // padded size of the result
    int64_t out_rows, out_cols, out_stride;    // kLast: the result's own, and whether it is to be written turned
    float old_factor, sum_factor, gain;        // (old * old_factor + sum * sum_factor) * gain
    int32_t out_turned, out_type;
};

// One tile of C = P Q^T.  kTerms 3: pairs; 1: their upper halves.  The tiles of P and Q for 32 (64) values of k are
// brought to LDS while those before are multiplied; a row takes 128 bytes there, its 16-byte pieces exchanged by the row's
// number, so that the 16 rows that a wavefront reads at once lie in different banks.
template <int kTile, int kWavesM, int kWavesN, int kTerms, int kKind>
__global__ __launch_bounds__(kWavesM * kWavesN * 64) void k_newton_product(Product a) {
    constexpr int kWaves = kWavesM * kWavesN;
    constexpr int FM = kTile / kWavesM / 16, FN = kTile / kWavesN / 16;
    constexpr int kStep = kTerms == 3 ? 32 : 64;
    constexpr int kStepBytes = kTerms == 3 ? kLine : 2 * kLine;
    constexpr int kLoads = kTile / 8 / kWaves;             // a wavefront's loads of each operand a step, 8 rows each
    static_assert(kLoads * 8 * kWaves == kTile, "rows are dealt out evenly");
    __shared__ __attribute__((aligned(1024))) char lds[2][2][kTile * kLine];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int bi, bj;
    if constexpr (kKind == kGram || kKind == kPoly) {      // the t-th tile on or below the diagonal
        const int t = blockIdx.x;
        bi = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
        while ((bi + 1) * (bi + 2) / 2 <= t) ++bi;
        while (bi * (bi + 1) / 2 > t) --bi;
        bj = t - bi * (bi + 1) / 2;
    } else {
        const int across = (int)(a.cols / kTile);
        bi = (int)blockIdx.x / across;
        bj = (int)blockIdx.x % across;
    }
    const int64_t pitch = a.k * 4;
    const char* p = a.p + blockIdx.y * a.p_plane + (int64_t)bi * kTile * pitch;
    const char* q = a.q + blockIdx.y * a.q_plane + (int64_t)bj * kTile * pitch;
    const int piece = (lane & 7) ^ (lane >> 3);
    const int64_t from = (int64_t)(wave * kLoads * 8 + (lane >> 3)) * pitch +
                         (kTerms == 3 ? piece * 16 : (piece >> 2) * kLine + (piece & 3) * 16);
    auto bring = [&](int buf, int64_t at) {
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const int64_t src = from + (int64_t)l * 8 * pitch + at;
            const int dst = (wave * kLoads + l) * 8 * kLine;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p + src),
                                             (__attribute__((address_space(3))) void*)(&lds[buf][0][dst]), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(q + src),
                                             (__attribute__((address_space(3))) void*)(&lds[buf][1][dst]), 16, 0, 0);
        }
    };
    const int wm = wave / kWavesN, wn = wave % kWavesN;
    const int row = lane & 15, quad = lane >> 4;
    float4_t acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (int)(a.k / kStep);
    bring(0, 0);
    for (int s = 0; s < steps; ++s) {
        __builtin_amdgcn_s_waitcnt(0x0f70);                // vmcnt(0): this wavefront's loads of the step are in LDS
        __syncthreads();
        if (s + 1 < steps) bring((s + 1) & 1, (int64_t)(s + 1) * kStepBytes);
        const char* tp = lds[s & 1][0] + (wm * FM * 16 + row) * kLine;
        const char* tq = lds[s & 1][1] + (wn * FN * 16 + row) * kLine;
        const int at0 = (quad ^ (row & 7)) * 16, at1 = ((quad + 4) ^ (row & 7)) * 16;
        half8 q0[FN], q1[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            q0[j] = *reinterpret_cast<const half8*>(tq + j * 16 * kLine + at0);
            q1[j] = *reinterpret_cast<const half8*>(tq + j * 16 * kLine + at1);
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const half8 p0 = *reinterpret_cast<const half8*>(tp + i * 16 * kLine + at0);
            const half8 p1 = *reinterpret_cast<const half8*>(tp + i * 16 * kLine + at1);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                if constexpr (kTerms == 3) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p1, q0[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, q1[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, q0[j], acc[i][j], 0, 0, 0);
                } else {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, q0[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p1, q1[j], acc[i][j], 0, 0, 0);
                }
            }
        }
    }
    // a lane has four rows i of one column j
#pragma unroll
    for (int fi = 0; fi < FM; ++fi)
#pragma unroll
        for (int fj = 0; fj < FN; ++fj) {
            const int64_t i = (int64_t)bi * kTile + wm * FM * 16 + fi * 16 + quad * 4;
            const int64_t j = (int64_t)bj * kTile + wn * FN * 16 + fj * 16 + row;
            float v[4];
            if constexpr (kKind == kGram) {
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = acc[fi][fj][r] * a.sum_factor;
            } else {
                const char* o = a.old + blockIdx.y * a.old_plane + j * a.rows * 4 + pair_at(i);
                const half4 high = *reinterpret_cast<const half4*>(o), low = *reinterpret_cast<const half4*>(o + 64);
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = ((float)high[r] + (float)low[r]) * a.old_factor + acc[fi][fj][r] * a.sum_factor;
            }
            if constexpr (kKind == kLast) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (i + r >= a.out_rows || j >= a.out_cols) continue;
                    const int64_t at = blockIdx.y * a.out_plane + (a.out_turned ? j * a.out_stride + i + r : (i + r) * a.out_stride + j);
                    store_typed(a.out, a.out_type, at, v[r] * a.gain);
                }
            } else {
                half4 high, low;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    half_t h, l;
                    split(v[r], h, l);
                    high[r] = h;
                    low[r] = l;
                }
                char* t = a.turned + blockIdx.y * a.q_plane;
                if constexpr (kKind != kApply) t = a.straight + blockIdx.y * a.old_plane;
                t += j * a.rows * 4 + pair_at(i);
                *reinterpret_cast<half4*>(t) = high;
                *reinterpret_cast<half4*>(t + 64) = low;
                if (kKind == kApply || bi != bj) {
                    char* st = a.straight + blockIdx.y * a.old_plane;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        char* at = st + (i + r) * a.cols * 4 + pair_at(j);
                        *reinterpret_cast<half_t*>(at) = high[r];
                        *reinterpret_cast<half_t*>(at + 64) = low[r];
                    }
                }
            }
        }
}

constexpr int64_t kPad = 128;                  // tiles divide it
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

template <int kTile, int kWavesM, int kWavesN> void product(const Product& p, int terms, int kind, int64_t count, hipStream_t s) {
    const int64_t tm = p.rows / kTile, tn = p.cols / kTile;
    const dim3 grid((unsigned)(kind == kGram || kind == kPoly ? tm * (tm + 1) / 2 : tm * tn), (unsigned)count);
    const dim3 block(kWavesM * kWavesN * 64);
#define P2_PRODUCT(TERMS, KIND) k_newton_product<kTile, kWavesM, kWavesN, TERMS, KIND><<<grid, block, 0, s>>>(p)
    if (terms == 3) {
        if (kind == kGram) P2_PRODUCT(3, kGram);
        else if (kind == kPoly) P2_PRODUCT(3, kPoly);
        else if (kind == kApply) P2_PRODUCT(3, kApply);
        else P2_PRODUCT(3, kLast);
    } else {
        if (kind == kGram) P2_PRODUCT(1, kGram);
        else if (kind == kPoly) P2_PRODUCT(1, kPoly);
        else P2_PRODUCT(1, kLast);
    }
#undef P2_PRODUCT
}

template <typename T> void to_pairs(const Orthogonalize& a, double unit, double* parts, char* straight, char* turned, int64_t rp, int64_t cp,
                                    int64_t plane, hipStream_t s) {
    const T* g = static_cast<const T*>(a.g);
    k_newton_norm<T><<<dim3(kNormParts, (unsigned)a.count), dim3(256), 0, s>>>(g, a.stride, a.matrix_stride, a.rows, a.cols, parts);
    k_newton_scale<T><<<dim3((unsigned)(cp / 32), (unsigned)(rp / 32), (unsigned)a.count), dim3(256), 0, s>>>(
        g, a.stride, a.matrix_stride, a.rows, a.cols, parts, a.eps, unit, straight, turned, rp, cp, plane);
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

int64_t orthogonalize_workspace(int64_t count, int64_t rows, int64_t cols) {
    const int64_t m = padded(std::min(rows, cols)), n = padded(std::max(rows, cols));
    return align256(count * kNormParts * 8) + count * 4 * (3 * m * n + 2 * m * m);
}

hipError_t launch_orthogonalize(const Orthogonalize& a, hipStream_t s) {
    const bool tall = a.rows > a.cols;
    const int64_t m = padded(std::min(a.rows, a.cols)), n = padded(std::max(a.rows, a.cols));
    const int64_t xb = m * n * 4, ab = m * m * 4;
    char* w = static_cast<char*>(a.workspace);
    double* parts = reinterpret_cast<double*>(w);
    w += align256(a.count * kNormParts * 8);
    char* x = w; w += a.count * xb;
    char* xt[2];
    xt[0] = w; w += a.count * xb;
    xt[1] = w; w += a.count * xb;
    char* ga = w; w += a.count * ab;
    char* gb = w;
    double ux = unit_for(a.bounds[0]);
    char* straight = tall ? xt[0] : x;
    char* turned = tall ? x : xt[0];
    const int64_t rp = tall ? n : m, cp = tall ? m : n;
    if (a.type == P2_F32) to_pairs<float>(a, ux, parts, straight, turned, rp, cp, xb, s);
    else if (a.type == P2_BF16) to_pairs<bf16_t>(a, ux, parts, straight, turned, rp, cp, xb, s);
    else to_pairs<half_t>(a, ux, parts, straight, turned, rp, cp, xb, s);
    hipError_t e = hipGetLastError();
    for (int i = 0; i < a.steps && e == hipSuccess; ++i) {
        const bool last = i + 1 == a.steps;
        const int terms = last && a.out_type == P2_BF16 ? 1 : 3;
        const double top = a.bounds[i] * 1.001;
        const double ua = unit_for(top * top), ub = unit_for(square_bound(a.b, a.c, top * top)), un = unit_for(a.bounds[i + 1]);
        Product p = {};
        p.p = p.q = x; p.p_plane = p.q_plane = xb;
        p.straight = ga; p.old_plane = ab;
        p.k = n; p.rows = p.cols = m;
        p.sum_factor = (float)(ua / (ux * ux));
        product<128, 2, 2>(p, terms, kGram, a.count, s);
        p = {};
        p.p = p.q = p.old = ga; p.p_plane = p.q_plane = p.old_plane = ab;
        p.straight = gb;
        p.k = p.rows = p.cols = m;
        p.old_factor = (float)(a.b * ub / ua);
        p.sum_factor = (float)(a.c * ub / (ua * ua));
        product<128, 2, 2>(p, terms, kPoly, a.count, s);
        p = {};
        p.p = gb; p.p_plane = ab;
        p.q = p.old = xt[i & 1]; p.q_plane = p.old_plane = xb;
        p.straight = x; p.turned = xt[(i + 1) & 1];
        p.k = p.rows = m; p.cols = n;
        p.old_factor = (float)(a.a * un / ux);
        p.sum_factor = (float)(un / (ub * ux));
        if (last) {
            p.out = a.out; p.out_plane = a.out_matrix_stride; p.out_stride = a.out_stride;
            p.out_rows = std::min(a.rows, a.cols); p.out_cols = std::max(a.rows, a.cols);
            p.out_turned = tall; p.out_type = a.out_type;
            p.gain = (float)(a.scale / un);
        }
        product<128, 2, 2>(p, terms, last ? kLast : kApply, a.count, s);
        ux = un;
        e = hipGetLastError();
    }
    return e;
}

}  // namespace p2
