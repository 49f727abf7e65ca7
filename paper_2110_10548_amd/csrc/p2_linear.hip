// Matrix products of a layer: y = activation(x W^T + bias) + residual, and its gradients dx = dz W, dW = dz^T x, dbias = sum dz with
// dz = dy * activation'(z).
//
// Every product is rows times rows, C[j][i] = sum_k A[i][k] B[j][k], with the summed index contiguous in both: the forward pass takes weight
// and x as they are; for the gradients weight, x and dz are written turned first, or, in large 16-bit products, turned by the reads from LDS.  A tile of C comes from stages of 128 bytes of
// each row (64 values of 16 bits, 32 of 32) that are brought to LDS straight from memory while the stage before is multiplied.  The MFMA's rows
// are A's: a lane has four neighbouring columns of one row of C.
#include <algorithm>
#include <cmath>
#include <limits>
#include <type_traits>

#include "p2_train_dev.h"

namespace p2 {

namespace {

typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr int kLine = 128;                     // bytes of a row in a stage
constexpr int64_t kUnits = 256;                // compute units
constexpr float kLog2e = 1.44269504088896340736f;

int64_t round_up(int64_t v, int64_t to) { return ceil_div(v, to) * to; }

// ---------------------------------------------------------------------------------------------- activations

// (The instructions for 2^x and 1 / x, which are off by a step of 32 bits: a division would take ten times as long, and the epilogue of a large product
// has nothing to hide behind.)
__device__ __forceinline__ float sigmoid_of(float v) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v * kLog2e)); }

// z (1 + tanh u) / 2 = z sigmoid(2 u), and 2 u = 2 sqrt(2 / pi) (z + 0.044715 z^3), here times -log2 e: the sigmoid.
__device__ __forceinline__ float gelu_part(float z, float square) {
    constexpr float kOne = -1.5957691216057308f * kLog2e;
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * fmaf(kOne * 0.044715f, square, kOne)));
}
template <int kActivation> __device__ __forceinline__ float activated(float z) {
    if constexpr (kActivation == P2_RELU) return z < 0.0f ? 0.0f : z;
    else if constexpr (kActivation == P2_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);
    else if constexpr (kActivation == P2_GELU_TANH) return z * gelu_part(z, z * z);
    else if constexpr (kActivation == P2_SILU) return z * sigmoid_of(z);
    else return z;
}
template <int kActivation> __device__ __forceinline__ float slope(float z) {
    if constexpr (kActivation == P2_RELU) {
        return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
    } else if constexpr (kActivation == P2_GELU) {
        return 0.5f * erfcf(-0.70710678118654752f * z) + z * 0.39894228040143268f * __builtin_amdgcn_exp2f(-0.5f * kLog2e * z * z);
    } else if constexpr (kActivation == P2_GELU_TANH) {
        const float square = z * z, p = gelu_part(z, square);
        const float flat = p * (1.0f - p);                 // (0 far out, where what it is multiplied by may be infinite)
        return flat == 0.0f ? p : fmaf(flat, z * fmaf(1.5957691216057308f * 0.134145f, square, 1.5957691216057308f), p);
    } else if constexpr (kActivation == P2_SILU) {
        const float p = sigmoid_of(z);
        return p * (1.0f + z * (1.0f - p));
    } else {
        return 1.0f;
    }
}
// One jump for all of v.
template <int N, typename F> __device__ __forceinline__ void with_activation(int32_t activation, F&& f) {
    switch (activation) {
        case P2_RELU: f(std::integral_constant<int, P2_RELU>()); break;
        case P2_GELU: f(std::integral_constant<int, P2_GELU>()); break;
        case P2_GELU_TANH: f(std::integral_constant<int, P2_GELU_TANH>()); break;
        case P2_SILU: f(std::integral_constant<int, P2_SILU>()); break;
        default: break;
    }
}
template <int N> __device__ __forceinline__ void activate(float (&v)[N], int32_t activation) {
    with_activation<N>(activation, [&](auto kind) {
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = activated<decltype(kind)::value>(v[q]);
    });
}
// v * activation'(z)
template <int N> __device__ __forceinline__ void times_slope(float (&v)[N], const float (&z)[N], int32_t activation) {
    with_activation<N>(activation, [&](auto kind) {
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] *= slope<decltype(kind)::value>(z[q]);
    });
}

// ------------------------------------------------------------------------------------------------ results

// What becomes of a sum: C's row j, column i.
struct Result {
    const void* bias; const void* residual; void* y; void* z;
    int64_t residual_stride, y_stride, z_stride;
    int32_t y_type, activation;        // (bias, residual and z have the operands' type)
};
template <typename T, int N> __device__ __forceinline__ void finish(const Result& r, int64_t j, int64_t i, int64_t n, float (&v)[N]) {
    if (r.bias) {
        float b[N];
        load_part<T, N>(static_cast<const T*>(r.bias) + i, n, b, 0.0f);
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] += b[q];
    }
    if (r.z) store_part<T, N>(static_cast<T*>(r.z) + j * r.z_stride + i, n, v);
    activate(v, r.activation);
    if (r.residual) {
        float b[N];
        load_part<T, N>(static_cast<const T*>(r.residual) + j * r.residual_stride + i, n, b, 0.0f);
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] += b[q];
    }
    if (r.y_type == P2_F32) store_part<float, N>(static_cast<float*>(r.y) + j * r.y_stride + i, n, v);
    else if (r.y_type == P2_BF16) store_part<bf16_t, N>(static_cast<bf16_t*>(r.y) + j * r.y_stride + i, n, v);
    else store_part<half_t, N>(static_cast<half_t*>(r.y) + j * r.y_stride + i, n, v);
}

// ------------------------------------------------------------------------------------------------ products

struct Product {
    const char* a; const char* b;      // rows, 16-byte aligned; a turned operand's are those of its transpose, `length` of them
    int64_t a_pitch, b_pitch;          // bytes from row to row, multiples of 16
    bool turned_a, turned_b;
    int64_t a_rows, b_rows, length;    // length: bytes of a row, a multiple of 16
    float* sums;                       // of the tiles in parts: [tile][part][tile's rows of B][of A]
    int32_t across, down, whole, parts;                    // tiles of A's and of B's rows; the first `whole` have one block, the others a block for each part of the length
    int32_t tile_a, tile_b;
    Result r;
};
// Products of one launch: the first has the first `blocks` blocks.
struct Products { Product p[2]; int32_t blocks; };

// 16 bytes of a row a lane: products of what 16 lanes x 4 have.
__device__ __forceinline__ void multiply(const half8& p, const half8& q, float4_t& c) { c = __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q, c, 0, 0, 0); }
__device__ __forceinline__ void multiply(const bf16x8& p, const bf16x8& q, float4_t& c) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, q, c, 0, 0, 0); }
__device__ __forceinline__ void multiply(const float4_t& p, const float4_t& q, float4_t& c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(p[i], q[i], c, 0, 0, 0);
}
template <typename T> struct Fragment;
template <> struct Fragment<half_t> { typedef half8 type; };
template <> struct Fragment<bf16_t> { typedef bf16x8 type; };
template <> struct Fragment<float> { typedef float4_t type; };

// Rows of an operand and 16 bytes a lane of them to LDS (`to`: the wavefront's, lanes one after the other); what lies past `bytes` comes as
// zeros.  Only the device's compiler knows the descriptor's type.
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

// Eight values a lane of a turned operand, whose rows in LDS are of the summed index: 16 lanes have four rows of 16 values at `from` (a lane points to four of
// a row), and get a column's four each.
template <typename F> __device__ __forceinline__ F read_turned(const char* __restrict from, int step) {
    F f = {};
#if defined(__HIP_DEVICE_COMPILE__)
    typedef short short4_t __attribute__((ext_vector_type(4)));
    const auto four = [&](const char* p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)p); };
    f = __builtin_bit_cast(F, __builtin_shufflevector(four(from), four(from + step), 0, 1, 2, 3, 4, 5, 6, 7));
#endif
    return f;
}

// Waits until at most kLoads of this wavefront's loads are under way (and all its LDS reads are done), then for the others.
template <int kLoads> __device__ __forceinline__ void stage_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((kLoads & 15) | (kLoads >> 4) << 14 | 0x70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr int kPastEnd = 0x7ffffff0;           // an offset that no descriptor reaches

// A tile's rows of A and of B come in halves of kWavesA * FA * 16 and kWavesB * FB * 16, and a stage is multiplied in four
// phases, half by half, A0 B0, A0 B1, A1 B1, A1 B0, so that each phase's fragments are read from LDS while the one before is multiplied, six
// reads of a fragment with every 16 MFMA, and a half's place in LDS is free for the stage after the next two phases after it has been
// read: loads have five to six phases to arrive.  Two barriers a stage.
template <typename T, int kWavesA, int kWavesB, int FA, int FB> struct Tile {
    typedef typename Fragment<T>::type F;
    static constexpr int kWaves = kWavesA * kWavesB;
    static constexpr int kHalfA = kWavesA * FA * 16, kHalfB = kWavesB * FB * 16;       // rows of a half
    static constexpr int kLoadsA = kHalfA / 8 / kWaves, kLoadsB = kHalfB / 8 / kWaves; // of a half by a wavefront; one brings 8 rows
    static constexpr int kBuffer = 2 * (kHalfA + kHalfB) * kLine;
    static_assert(kLoadsA * 8 * kWaves == kHalfA && kLoadsB * 8 * kWaves == kHalfB, "rows are dealt out evenly");
    static_assert(kWaves * 2 * FB * 16 * FA * 64 <= 2 * kBuffer, "half of the results fit");
};
// Eight rows from `first` on, of which those past the matrix's end are zeros; where all are, the first row again and zeros, whose results nobody writes
// (a descriptor has to reach past the place in the row that a load adds to it).
__device__ __forceinline__ Rows rows_from(const char* p, int64_t pitch, int64_t first, int64_t rows, int length) {
    const int64_t n = min(rows - first, (int64_t)8);
    return Rows(p + (n > 0 ? first : 0) * pitch, (n > 0 ? (int)((n - 1) * pitch) : 0) + length);
}
// A turned operand's rows of each stage, from a half's first column on (or, where there is none, from column 0).  (What it needs is kept in scalar registers:
// fetched anew from the kernel's arguments it would make LDS reads wait.)
struct Turned {
    const char* first;
    int pitch, left, extent;           // left: rows from the first stage on; extent: bytes of a row
    __device__ __forceinline__ Turned(const char* p, int64_t row, int begin, int rows, int64_t col, int64_t cols) {
        const int64_t c = col < cols ? col : 0;
        const uint64_t at = reinterpret_cast<uint64_t>(p + (int64_t)begin * 64 * row + c * 2);
        first = reinterpret_cast<const char*>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at));
        pitch = __builtin_amdgcn_readfirstlane((int)row);
        left = __builtin_amdgcn_readfirstlane(rows - begin * 64);
        extent = __builtin_amdgcn_readfirstlane((int)(cols - c) * 2);
    }
    __device__ __forceinline__ Rows stage(int s, bool last) const {
        const int n = last ? min(left - s * 64, 64) : 64;
        return Rows(first + (uint64_t)(uint32_t)(s * 64) * (uint32_t)pitch, (n - 1) * pitch + extent);
    }
};
__device__ __forceinline__ void in_this_order() { __builtin_amdgcn_sched_barrier(0); }

// Which tile, and which part of the length, a block has.  Blocks go to the eight dies in turn: tiles are dealt out so that those of a die are neighbours, column by
// column of four rows of tiles.
struct Place { int ti, tj, split, part; };     // split: the tile's number among those in parts, or -1
__device__ __forceinline__ Place place_of_tile(const Product& a, int t) {
    const int band = t / (4 * a.across), first = band * 4, high = min(4, a.down - first), in = t - first * a.across;
    return {in / high, first + in % high, t - a.whole, 0};
}
__device__ __forceinline__ Place place_of(const Product& a, int block) {
    const int rest = a.across * a.down - a.whole;
    const bool split = block >= a.whole;
    const int x = split ? block - a.whole : block, blocks = split ? rest * a.parts : a.whole;
    const int each = blocks / 8, more = blocks % 8, die = x & 7;
    const int t = die * each + min(die, more) + (x >> 3), part = split ? t / rest : 0;
    Place p = place_of_tile(a, split ? a.whole + t % rest : t);
    p.split = split ? p.split : -1;
    p.part = part;
    return p;
}

// A tile's results: `acc` of this wavefront.  LDS is free for them.
template <typename S, typename T, int kWavesB, int FA, int FB>
__device__ __forceinline__ void write_results(const Product& a, const Place& place, char* lds, const float4_t (&acc)[2][2][FA][FB]) {
    // A lane has four neighbouring columns of a row of C.  A wavefront's results go through LDS, half of the columns at a time, where a lane picks up eight.  A row's
    // 16-byte parts are exchanged by the row's number.  (One loop, not unrolled: a copy of the activations for each strip would not stay in the instruction cache.)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wa = wave / kWavesB, wb = wave % kWavesB, row = lane & 15, quad = lane >> 4;
    constexpr int kParts = FA * 4, kAcross = FA * 2, kRow = FA * 64;                    // of a row in LDS: 16-byte parts, lanes, bytes
    const Result result = a.r;
    const int64_t a_rows = a.a_rows, b_rows = a.b_rows;
    constexpr int kTileA = 2 * S::kHalfA, kTileB = 2 * S::kHalfB;
    float* const sums = place.split >= 0 ? a.sums + ((int64_t)place.split * a.parts + place.part) * (kTileA * kTileB) : nullptr;
    char* mine = lds + wave * 2 * FB * 16 * kRow;
#pragma unroll
    for (int ha = 0; ha < 2; ++ha) {
#pragma unroll
        for (int hb = 0; hb < 2; ++hb)
#pragma unroll
            for (int fj = 0; fj < FB; ++fj)
#pragma unroll
                for (int fi = 0; fi < FA; ++fi)
                    *reinterpret_cast<float4_t*>(mine + ((hb * FB + fj) * 16 + row) * kRow + ((fi * 4 + quad) ^ (row & (kParts - 1))) * 16) = acc[ha][hb][fi][fj];
        wavefront_exchange();
        const int i0 = ha * S::kHalfA + wa * FA * 16;
#pragma unroll 1
        for (int x = 0; x < FA * FB; ++x) {
            const int r = (x * 64 + lane) / kAcross, c = (x * 64 + lane) % kAcross, h = r / (16 * FB);
            const int in_j = h * S::kHalfB + wb * FB * 16 + r % (16 * FB), in_i = i0 + c * 8;
            const int64_t j = (int64_t)place.tj * kTileB + in_j, i = (int64_t)place.ti * kTileA + in_i;
            float v[8];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float4_t f = *reinterpret_cast<const float4_t*>(mine + r * kRow + ((c * 2 + q) ^ (r & 15 & (kParts - 1))) * 16);
#pragma unroll
                for (int w = 0; w < 4; ++w) v[q * 4 + w] = f[w];
            }
            if (j < b_rows && i < a_rows) {
                if (sums) store_vec<float, 8>(sums + in_j * kTileA + in_i, v);
                else finish<T, 8>(result, j, i, a_rows - i, v);
            }
        }
        wavefront_exchange();
    }
}

// An operand may be turned: its memory has the summed index's rows, of which a stage takes 64, and a half's columns of them lie in LDS as 64 rows of 256 bytes.  Their
// 32-byte parts are exchanged by the row's number, so that what is read at once lies in different banks.  (16 bits and 256 x 256 tiles alone.)
// Bound by the matrix units, which are busy for 70 to 77 % of the compute units' busy cycles, at the 1.8 to 2.0 GHz that such a load leaves (50 % of cycles at 2.4 GHz): 8192 x 4096 x 16384 bf16 843 to 860 us with gelu, bias and z, 1.28 to 1.30 P/s; its main loop alone runs at 1.56, and a tile's end takes 9 of 97 us, the
// epilogue's vector instructions, which 256 x 256 sums in registers leave no second block to hide behind.  Turned, 8192 x 4096 x 4096: 226 us with one operand, 220 with both, 1.22 and 1.25 P/s.
template <typename T, int kWavesA, int kWavesB, int FA, int FB, bool kTurnA = false, bool kTurnB = false>
__global__ __launch_bounds__(kWavesA * kWavesB * 64) void k_linear_wide(Products all_of) {
    const bool second = (int)blockIdx.x >= all_of.blocks;
    const Product& a = all_of.p[__builtin_amdgcn_readfirstlane(second ? 1 : 0)];
    const int block = (int)blockIdx.x - (second ? all_of.blocks : 0);
    typedef Tile<T, kWavesA, kWavesB, FA, FB> S;
    typedef typename S::F F;
    constexpr int LA = S::kLoadsA, LB = S::kLoadsB, kBoth = 2 * (LA + LB);
    static_assert(!(kTurnA || kTurnB) || (sizeof(T) == 2 && S::kHalfA == 128 && S::kHalfB == 128), "what a turned operand is laid out for");
    __shared__ __attribute__((aligned(1024))) char lds[2 * S::kBuffer];                // two stages of A0, A1, B0, B1
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const Place place = place_of(a, block);
    const int ti = place.ti, tj = place.tj, part = place.part, parts = place.split >= 0 ? a.parts : 1;
    const int length = (int)a.length;
    const int all = (length + kLine - 1) / kLine;
    const int begin = (int)((int64_t)all * part / parts), stages = (int)((int64_t)all * (part + 1) / parts) - begin;
    // A row's 16-byte parts are exchanged by the row's number, so that the 16 rows that a wavefront reads at once lie in different banks.
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const int from_a = (lane >> 3) * (int)a.a_pitch + piece, from_b = (lane >> 3) * (int)a.b_pitch + piece;
    // Every load of a stage has a descriptor of its own, which begins with its first row: lanes' offsets are the same for all of them.
    const auto rows_of_a = [&](int half, int l) { return rows_from(a.a, a.a_pitch, (int64_t)ti * 2 * S::kHalfA + half * S::kHalfA + (wave * LA + l) * 8, a.a_rows, length); };
    const auto rows_of_b = [&](int half, int l) { return rows_from(a.b, a.b_pitch, (int64_t)tj * 2 * S::kHalfB + half * S::kHalfB + (wave * LB + l) * 8, a.b_rows, length); };
    const Rows ra[2][2] = {{rows_of_a(0, 0), rows_of_a(0, LA - 1)}, {rows_of_a(1, 0), rows_of_a(1, LA - 1)}},
               rb[2][2] = {{rows_of_b(0, 0), rows_of_b(0, LB - 1)}, {rows_of_b(1, 0), rows_of_b(1, LB - 1)}};
    static_assert(LA <= 2 && LB <= 2, "descriptors");
    // A turned operand's loads bring four rows each, with a descriptor of the stage's rows from the half's first column on (or, where there is none, from column 0).
    const auto turned_from = [&](int64_t pitch, int load) { return (load * 4 + (lane >> 4)) * (int)pitch + ((lane & 15) ^ ((lane >> 4) * 2 + (load >> 1 & 1) * 8)) * 16; };
    const int turned_a[2] = {turned_from(a.a_pitch, wave * LA), turned_from(a.a_pitch, wave * LA + LA - 1)}, turned_b[2] = {turned_from(a.b_pitch, wave * LB), turned_from(a.b_pitch, wave * LB + LB - 1)};
    const Turned ta[2] = {Turned(a.a, a.a_pitch, begin, length / 2, (int64_t)ti * 2 * S::kHalfA, a.a_rows), Turned(a.a, a.a_pitch, begin, length / 2, (int64_t)ti * 2 * S::kHalfA + S::kHalfA, a.a_rows)},
                 tb[2] = {Turned(a.b, a.b_pitch, begin, length / 2, (int64_t)tj * 2 * S::kHalfB, a.b_rows), Turned(a.b, a.b_pitch, begin, length / 2, (int64_t)tj * 2 * S::kHalfB + S::kHalfB, a.b_rows)};
    // the l-th load of a half of stage s; `last` may be the row's last stage, whose rest is zeros
    const auto bring_a = [&](auto last, int half, int s, int l) {
        const int at = (begin + s) * kLine;
        char* to = &lds[(s & 1) * S::kBuffer + half * S::kHalfA * kLine + (wave * LA + l) * 1024];
        if constexpr (kTurnA) ta[half].stage(s, decltype(last)::value).bring(to, turned_a[l], 0);
        else ra[half][l].bring(to, !decltype(last)::value || at + piece < length ? from_a : kPastEnd, at);
    };
    const auto bring_b = [&](auto last, int half, int s, int l) {
        const int at = (begin + s) * kLine;
        char* to = &lds[(s & 1) * S::kBuffer + (2 * S::kHalfA + half * S::kHalfB) * kLine + (wave * LB + l) * 1024];
        if constexpr (kTurnB) tb[half].stage(s, decltype(last)::value).bring(to, turned_b[l], 0);
        else rb[half][l].bring(to, !decltype(last)::value || at + piece < length ? from_b : kPastEnd, at);
    };
    const auto bring_stage = [&](int s) {
#pragma unroll
        for (int l = 0; l < LA; ++l) bring_a(std::true_type(), 0, s, l);
#pragma unroll
        for (int l = 0; l < LB; ++l) bring_b(std::true_type(), 0, s, l);
#pragma unroll
        for (int l = 0; l < LB; ++l) bring_b(std::true_type(), 1, s, l);
#pragma unroll
        for (int l = 0; l < LA; ++l) bring_a(std::true_type(), 1, s, l);
    };
    const int wa = wave / kWavesB, wb = wave % kWavesB, row = lane & 15, quad = lane >> 4;
    const int slot[2] = {row * kLine + (quad ^ (row & 7)) * 16, row * kLine + ((4 + quad) ^ (row & 7)) * 16};
    // (of a turned operand: four rows from quad * 8 + row / 4 on, and four rows further down; 32-byte parts by the row's lowest two bits and its fourth)
    const int turned_slot = (quad * 8 + (row >> 2)) * 256 + (row & 3) * 8, exchanged = (row >> 2) + (quad & 1) * 4;
    const int slot_a = turned_slot + ((wa * FA) ^ exchanged) * 32, slot_b = turned_slot + ((wb * FB) ^ exchanged) * 32;
    const auto read_a = [&](int s, int half, int i, F (&f)[2]) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
            if constexpr (kTurnA) f[c] = read_turned<F>(lds + (slot_a ^ i * 32) + (s & 1) * S::kBuffer + half * S::kHalfA * kLine + c * 32 * 256, 4 * 256);
            else f[c] = *reinterpret_cast<const F*>(lds + (s & 1) * S::kBuffer + slot[c] + wa * FA * 16 * kLine + (half * S::kHalfA + i * 16) * kLine);
    };
    const auto read_b = [&](int s, int half, int j, F (&f)[2]) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
            if constexpr (kTurnB) f[c] = read_turned<F>(lds + (slot_b ^ j * 32) + (s & 1) * S::kBuffer + (2 * S::kHalfA + half * S::kHalfB) * kLine + c * 32 * 256, 4 * 256);
            else f[c] = *reinterpret_cast<const F*>(lds + (s & 1) * S::kBuffer + slot[c] + wb * FB * 16 * kLine + (2 * S::kHalfA + half * S::kHalfB + j * 16) * kLine);
    };
    float4_t acc[2][2][FA][FB];
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j) acc[h >> 1][h & 1][i][j] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    F a0[FA][2], a1[FA][2], bx[FB][2], by[FB][2];
    // One phase: the products of two halves, and between them `reads` (the r-th of kReads) and `loads` (the l-th of kLoads).
    const auto phase = [&](float4_t (&c)[FA][FB], const F (&fa)[FA][2], const F (&fb)[FB][2], auto reads_n, auto&& reads, auto loads_n, auto&& loads) {
        constexpr int kReads = decltype(reads_n)::value, kLoads = decltype(loads_n)::value, kProducts = FA * FB * 2;
#pragma unroll
        for (int n = 0; n < kProducts; ++n) {
            const int k = n / (FA * FB), i = n / FB % FA, j = n % FB;
            multiply(fa[i][k], fb[j][k], c[i][j]);
            // reads first, loads after them
            constexpr int kEvery = kReads + kLoads > 0 ? kReads + kLoads : 1;
#pragma unroll
            for (int x = n * kEvery / kProducts; x < (n + 1) * kEvery / kProducts; ++x) {
                if (x < kReads) reads(x);
                else if (x - kReads < kLoads) loads(x - kReads);
            }
            in_this_order();
        }
    };
    // kEnd: one of the last stages, after which fewer are left to bring.
    const auto step = [&](auto end, int s, F (&b0)[FB][2], F (&b1)[FB][2]) {
        constexpr bool kEnd = decltype(end)::value;
        const bool next = !kEnd || s + 1 < stages, after = !kEnd || s + 2 < stages;
        constexpr int kFew = FA >= 4 ? 1 : 0;              // fragments of A1 read in the first phase, of A0 in the last
        if (next) stage_barrier<kBoth>();
        else stage_barrier<0>();
        phase(acc[0][0], a0, b0, std::integral_constant<int, FB + kFew>(), [&](int x) { if (x < FB) read_b(s, 1, x, b1[x < FB ? x : 0]); else read_a(s, 1, x - FB, a1[x >= FB ? x - FB : 0]); },
              std::integral_constant<int, LA>(), [&](int l) { if (after) bring_a(end, 0, s + 2, l); });
        phase(acc[0][1], a0, b1, std::integral_constant<int, FA - kFew>(), [&](int x) { read_a(s, 1, x + kFew, a1[x + kFew]); },
              std::integral_constant<int, LB>(), [&](int l) { if (after) bring_b(end, 0, s + 2, l); });
        if (after) stage_barrier<kBoth>();
        else if (next) stage_barrier<LA + LB>();
        else stage_barrier<0>();
        phase(acc[1][1], a1, b1, std::integral_constant<int, FA - kFew>(), [&](int x) { if (next) read_a(s + 1, 0, x, a0[x]); },
              std::integral_constant<int, LB>(), [&](int l) { if (after) bring_b(end, 1, s + 2, l); });
        phase(acc[1][0], a1, b0, std::integral_constant<int, FB + kFew>(),
              [&](int x) { if (next) { if (x < FB) read_b(s + 1, 0, x, b1[x < FB ? x : 0]); else read_a(s + 1, 0, FA - 1, a0[FA - 1]); } },
              std::integral_constant<int, LA>(), [&](int l) { if (after) bring_a(end, 1, s + 2, l); });
    };
    bring_stage(0);
    if (stages > 1) {
        bring_stage(1);
        stage_barrier<kBoth + LA + LB>();
    } else {
        stage_barrier<LA + LB>();
    }
#pragma unroll
    for (int i = 0; i < FA; ++i) read_a(0, 0, i, a0[i]);
#pragma unroll
    for (int j = 0; j < FB; ++j) read_b(0, 0, j, bx[j]);
    int s = 0;
    for (; s + 4 < stages; s += 2) {
        step(std::false_type(), s, bx, by);
        step(std::false_type(), s + 1, by, bx);
    }
    for (; s + 1 < stages; s += 2) {
        step(std::true_type(), s, bx, by);
        step(std::true_type(), s + 1, by, bx);
    }
    if (s < stages) step(std::true_type(), s, bx, by);
    stage_barrier<0>();
    write_results<S, T, kWavesB, FA, FB>(a, place, lds, acc);
}

// The same for rows that cannot be brought to LDS as they are: of any alignment and length.  A stage's values are asked for while the one before is multiplied, and put
// into LDS after that; what lies past a row's end is zeros.  Rows past the matrix's end are the last one again, whose results nobody writes.  (Bound by the wait for a stage: 700 x 701 x 703
// bf16 10.9 us, 63 T/s.)
template <typename T, int kWavesA, int kWavesB, int FA, int FB> __global__ __launch_bounds__(kWavesA * kWavesB * 64) void k_linear_any(Product a) {
    typedef Tile<T, kWavesA, kWavesB, FA, FB> S;
    typedef typename S::F F;
    constexpr int V = 16 / sizeof(T), kLine16 = kLine / 16;
    constexpr int kRowsA = 2 * S::kHalfA, kRowsB = 2 * S::kHalfB, kThreads = S::kWaves * 64;
    constexpr int LA = kRowsA * kLine16 / kThreads, LB = kRowsB * kLine16 / kThreads;      // 16-byte parts of a stage a thread
    __shared__ __attribute__((aligned(1024))) char lds[2 * S::kBuffer];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const Place place = place_of(a, blockIdx.x);
    const int parts = place.split >= 0 ? a.parts : 1;
    const int64_t k = a.length / (int64_t)sizeof(T);       // (here the row's own length)
    const int all = (int)((a.length + kLine - 1) / kLine);
    const int begin = (int)((int64_t)all * place.part / parts), stages = (int)((int64_t)all * (place.part + 1) / parts) - begin;
    const int piece = threadIdx.x % kLine16, first = threadIdx.x / kLine16;                // this thread's part of a row, its first row
    const auto row_of = [&](const char* p, int64_t pitch, int64_t r, int64_t rows) { return reinterpret_cast<const T*>(p + min(r, rows - 1) * pitch) + piece * V; };
    const T *pa[LA], *pb[LB];
#pragma unroll
    for (int l = 0; l < LA; ++l) pa[l] = row_of(a.a, a.a_pitch, (int64_t)place.ti * kRowsA + first + l * (kThreads / kLine16), a.a_rows);
#pragma unroll
    for (int l = 0; l < LB; ++l) pb[l] = row_of(a.b, a.b_pitch, (int64_t)place.tj * kRowsB + first + l * (kThreads / kLine16), a.b_rows);
    vec_t<T, V> va[LA], vb[LB];
    const auto ask = [&](int s) {
        const int64_t at = (int64_t)(begin + s) * (kLine / (int)sizeof(T)), left = k - at - piece * V;
        if ((begin + s + 1) * (int64_t)kLine <= a.length) {
#pragma unroll
            for (int l = 0; l < LA; ++l) va[l] = *reinterpret_cast<const vec_t<T, V>*>(pa[l] + at);
#pragma unroll
            for (int l = 0; l < LB; ++l) vb[l] = *reinterpret_cast<const vec_t<T, V>*>(pb[l] + at);
        } else {                                           // the rows' last stage
            const auto some = [&](const T* p) {
                vec_t<T, V> v;
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = j < left ? p[at + j] : (T)0.0f;
                return v;
            };
#pragma unroll
            for (int l = 0; l < LA; ++l) va[l] = some(pa[l]);
#pragma unroll
            for (int l = 0; l < LB; ++l) vb[l] = some(pb[l]);
        }
    };
    const auto put = [&](int s) {
        char* to = lds + (s & 1) * S::kBuffer;
#pragma unroll
        for (int l = 0; l < LA; ++l) {
            const int r = first + l * (kThreads / kLine16);
            *reinterpret_cast<F*>(to + r * kLine + (piece ^ (r & 7)) * 16) = __builtin_bit_cast(F, va[l]);
        }
#pragma unroll
        for (int l = 0; l < LB; ++l) {
            const int r = first + l * (kThreads / kLine16);
            *reinterpret_cast<F*>(to + (kRowsA + r) * kLine + (piece ^ (r & 7)) * 16) = __builtin_bit_cast(F, vb[l]);
        }
    };
    float4_t acc[2][2][FA][FB];
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j) acc[h >> 1][h & 1][i][j] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const int wa = wave / kWavesB, wb = wave % kWavesB, row = lane & 15, quad = lane >> 4;
    ask(0);
    put(0);
    __syncthreads();
    for (int s = 0; s < stages; ++s) {
        if (s + 1 < stages) ask(s + 1);
        const char* from = lds + (s & 1) * S::kBuffer;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int at = row * kLine + ((c * 4 + quad) ^ (row & 7)) * 16;
            F fa[2][FA], fb[2][FB];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < FA; ++i) fa[h][i] = *reinterpret_cast<const F*>(from + (h * S::kHalfA + (wa * FA + i) * 16) * kLine + at);
#pragma unroll
                for (int j = 0; j < FB; ++j) fb[h][j] = *reinterpret_cast<const F*>(from + (kRowsA + h * S::kHalfB + (wb * FB + j) * 16) * kLine + at);
            }
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int i = 0; i < FA; ++i)
#pragma unroll
                    for (int j = 0; j < FB; ++j) multiply(fa[h >> 1][i], fb[h & 1][j], acc[h >> 1][h & 1][i][j]);
        }
        if (s + 1 < stages) put(s + 1);                    // (the other half of LDS: everyone has left it before the last barrier)
        __syncthreads();
    }
    write_results<S, T, kWavesB, FA, FB>(a, place, lds, acc);
}

// What is left of a call's products: parts of sums added up, in their order, and the tiles' lines of dbias, 16 columns a block and 16 threads a column.  (4 to 5 us, a launch and a chain of loads.)
struct Join {
    Product p[2];
    const float* lines; void* out;             // [n][cols]
    int64_t n, cols;
    int32_t blocks[2];                         // of each product
    int32_t type;
};
template <typename T> __global__ __launch_bounds__(256) void k_linear_join(Join all) {
    __shared__ float part[16][17];
    int block = blockIdx.x;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const Product& a = all.p[which];
        const int blocks = all.blocks[which];
        if (block < blocks) {
            const int across = a.tile_a / 4, plane = a.tile_a * a.tile_b, in_tile = across * a.tile_b;
            const int64_t items = (int64_t)(a.across * a.down - a.whole) * in_tile;
            for (int64_t x = (int64_t)block * 256 + threadIdx.x; x < items; x += (int64_t)blocks * 256) {
                const int tile = (int)(x / in_tile), in = (int)(x % in_tile);
                const Place place = place_of_tile(a, a.whole + tile);
                const int64_t j = (int64_t)place.tj * a.tile_b + in / across, i = (int64_t)place.ti * a.tile_a + in % across * 4;
                if (j >= a.b_rows || i >= a.a_rows) continue;
                const float* from = a.sums + (int64_t)tile * a.parts * plane + in * 4;
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
                for (int p = 0; p < a.parts; ++p) {
                    float w[4];
                    load_vec<float, 4>(from + (int64_t)p * plane, w);
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] += w[q];
                }
                finish<T, 4>(a.r, j, i, a.a_rows - i, v);
            }
            return;
        }
        block -= blocks;
    }
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
    const int64_t c = (int64_t)block * 16 + x;
    float s = 0.0f;
    if (c < all.cols)
#pragma unroll 4
        for (int64_t l = y; l < all.n; l += 16) s += all.lines[l * all.cols + c];
    part[y][x] = s;
    __syncthreads();
    if (y > 0 || c >= all.cols) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += part[i][x];
    store_typed(all.out, all.type, c, s);
}

// A few rows of x against all of the weight's, which are read once: a wavefront takes kEach of them at a time.  Bound by memory.
template <typename T, int kRows, int kEach, int kAhead> __global__ __launch_bounds__(256) void k_linear_rows(const T* x, int64_t x_stride, const T* weight, int64_t weight_stride, int64_t inner,
                                                                                                 int64_t outer, Result r) {
    constexpr int V = 16 / sizeof(T);
    const int lane = threadIdx.x & 63;
    const int64_t i0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * kEach;
    if (i0 >= outer) return;
    float sum[kRows][kEach] = {};
    int64_t k = lane * V;
    // of long rows, kAhead vectors of each under way at once (1 x 4096 x 16384 bf16 28.0 -> 24.3 us, the weight from memory, 5.5 TB/s, and 21.2 from the last cache; 1 x 8000 x 500 fp16 15.2 -> 7.4)
    if constexpr (kAhead > 1) for (int64_t whole = kAhead * 64 * V; whole <= inner; whole += kAhead * 64 * V, k += kAhead * 64 * V) {
        vec_t<T, V> w[kAhead][kEach], v[kAhead][kRows];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) w[u][e] = *reinterpret_cast<const vec_t<T, V>*>(weight + min(i0 + e, outer - 1) * weight_stride + k + u * 64 * V);
#pragma unroll
            for (int m = 0; m < kRows; ++m) v[u][m] = *reinterpret_cast<const vec_t<T, V>*>(x + m * x_stride + k + u * 64 * V);
        }
        in_this_order();
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int m = 0; m < kRows; ++m)
#pragma unroll
                for (int e = 0; e < kEach; ++e)
#pragma unroll
                    for (int q = 0; q < V; ++q) sum[m][e] = fmaf((float)v[u][m][q], (float)w[u][e][q], sum[m][e]);
    }
    for (; k < inner; k += 64 * V) {
        float p[kRows][V], q[kEach][V];
#pragma unroll
        for (int e = 0; e < kEach; ++e) load_part<T, V>(weight + min(i0 + e, outer - 1) * weight_stride + k, inner - k, q[e], 0.0f);
#pragma unroll
        for (int m = 0; m < kRows; ++m) load_part<T, V>(x + m * x_stride + k, inner - k, p[m], 0.0f);
#pragma unroll
        for (int m = 0; m < kRows; ++m)
#pragma unroll
            for (int e = 0; e < kEach; ++e)
#pragma unroll
                for (int v = 0; v < V; ++v) sum[m][e] = fmaf(p[m][v], q[e][v], sum[m][e]);
    }
#pragma unroll
    for (int m = 0; m < kRows; ++m) {
        float v[4] = {};
#pragma unroll
        for (int e = 0; e < kEach; ++e) v[e] = group_sum<64>(sum[m][e]);
        if (lane == m) finish<T, 4>(r, m, i0, min((int64_t)kEach, outer - i0), v);
    }
}

// Up to 32 rows of x against all of the weight's, straight into registers, of any alignment, without LDS and its barriers.  A block has kFragments * 16 of the weight's rows, and
// its eight wavefronts share their length in pieces of 128 bytes, kAhead of them under way at once; their sums are added up in order.  x has up to kRows * 16 rows.  Bound by memory, or by a
// wavefront's chain of loads: 16 x 4096 x 16384 bf16 34 to 37 us, 3.7 to 4.0 TB/s; 16 x 1000 x 1000 5.3 us.
template <typename T, int kRows, int kFragments, int kAhead> __global__ __launch_bounds__(512) void k_linear_thin(const T* x, int64_t x_stride, const T* weight, int64_t weight_stride, int64_t rows,
                                                                                                               int64_t inner, int64_t outer, Result r) {
    typedef typename Fragment<T>::type F;
    constexpr int V = 16 / sizeof(T), kPiece = kLine / (int)sizeof(T);
    __shared__ float4_t part[8][kRows * kFragments][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), row = lane & 15, quad = lane >> 4;
    const int64_t i0 = (int64_t)blockIdx.x * kFragments * 16;
    const T *pw[kFragments], *px[kRows];
#pragma unroll
    for (int f = 0; f < kFragments; ++f) pw[f] = weight + min(i0 + f * 16 + row, outer - 1) * weight_stride + quad * V;          // (rows past the end: the last one again, whose results nobody writes)
#pragma unroll
    for (int f = 0; f < kRows; ++f) px[f] = x + min((int64_t)f * 16 + row, rows - 1) * x_stride + quad * V;
    float4_t acc[kRows][kFragments];
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int f = 0; f < kFragments; ++f) acc[i][f] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const int whole = (int)(inner / kPiece);
    const auto pieces = [&](int first, auto n) {               // n pieces, eight apart
        constexpr int kN = decltype(n)::value;
        vec_t<T, V> w[kN][kFragments][2], v[kN][kRows][2];
#pragma unroll
        for (int u = 0; u < kN; ++u) {
            const int64_t at = (int64_t)(first + u * 8) * kPiece;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int f = 0; f < kFragments; ++f) w[u][f][c] = *reinterpret_cast<const vec_t<T, V>*>(pw[f] + at + c * 4 * V);
#pragma unroll
                for (int f = 0; f < kRows; ++f) v[u][f][c] = *reinterpret_cast<const vec_t<T, V>*>(px[f] + at + c * 4 * V);
            }
        }
        in_this_order();                                       // (or the compiler asks for a piece when the one before it is there)
#pragma unroll
        for (int u = 0; u < kN; ++u)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < kRows; ++i)
#pragma unroll
                    for (int f = 0; f < kFragments; ++f) multiply(__builtin_bit_cast(F, w[u][f][c]), __builtin_bit_cast(F, v[u][i][c]), acc[i][f]);
    };
    int s = wave;
    for (; s + 8 * (kAhead - 1) < whole; s += 8 * kAhead) pieces(s, std::integral_constant<int, kAhead>());
    for (; s < whole; s += 8) pieces(s, std::integral_constant<int, 1>());
    if (s == whole && inner % kPiece) {                        // the rest, past which there are zeros
        const auto some = [&](const T* p, int c) {
            const int64_t at = (int64_t)whole * kPiece + c * 4 * V;
            vec_t<T, V> o;
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = at + quad * V + j < inner ? p[at + j] : (T)0.0f;
            return __builtin_bit_cast(F, o);
        };
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            F v[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) v[i] = some(px[i], c);
#pragma unroll
            for (int f = 0; f < kFragments; ++f) {
                const F w = some(pw[f], c);
#pragma unroll
                for (int i = 0; i < kRows; ++i) multiply(w, v[i], acc[i][f]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int f = 0; f < kFragments; ++f) part[wave][i * kFragments + f][lane] = acc[i][f];
    __syncthreads();
    for (int t = wave; t < kRows * kFragments; t += 8) {
        float4_t sum = part[0][t][lane];
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += part[w][t][lane];
        const int64_t j = t / kFragments * 16 + row, i = i0 + t % kFragments * 16 + quad * 4;
        float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        if (j < rows && i < outer) finish<T, 4>(r, j, i, outer - i, v);
    }
}

// ------------------------------------------------------------------------------------- operands in order

// A matrix as a product takes it: straight, turned, or both, with zeros from its end to whole stages.  With z the values are dy activation'(z), and
// each tile's sums over its rows go to sums[tile][cols], or, where one tile has all rows, to dbias.
struct Pack {
    const void* from; const void* z; char* straight; char* turned; float* sums; void* dbias;
    int64_t from_stride, z_stride, straight_pitch, turned_pitch;       // pitches in bytes
    int64_t rows, cols;
    int32_t activation, dbias_type;
};
// dz is rounded to the operands' type, which the matrix units take: by half a step of each, so that 16-bit results are off by (relative norm) 2.35e-3 where
// rounding them alone gives 1.66e-3 (8192 x 4096 x 4096 bf16, gelu_tanh).  As a pair, which would keep 16 bits of it, both products would be twice as long: 439 -> some 790 us.  dbias adds
// up what has not been rounded.
// Bound by memory: dz of 8192 x 4096 bf16 with gelu_tanh's slope and dbias 42 us for 192 MB, 4.6 TB/s; small ones by the chain of a launch, a load and a store, 5.6 us and more.
// Several matrices in one launch: the m-th has the blocks from begin[m] on, across[m] of them side by side.
struct Packs { Pack p[3]; int32_t begin[4], across[3]; };
template <typename T> __global__ __launch_bounds__(256) void k_linear_pack(Packs all) {
    __shared__ float tile[64][65];
    const int m = (int)blockIdx.x >= all.begin[2] ? 2 : (int)blockIdx.x >= all.begin[1] ? 1 : 0;
    const Pack& a = all.p[__builtin_amdgcn_readfirstlane(m)];
    const int block = (int)blockIdx.x - all.begin[m], line = block / all.across[m];
    const int64_t r0 = (int64_t)line * 64, c0 = (int64_t)(block % all.across[m]) * 64;
    const int x = (threadIdx.x & 15) * 4, y = threadIdx.x >> 4;
    // All is asked for before any of it is waited for, without conditions: a vector that the row's end cuts is the row's last one, moved into place after that
    // (three matrices of 2001 x 1023 x 515 11.5 -> 11.4 us, 4001 x 2047 x 1029 20.9 -> 16.8, 8192 x 4096 x 4096 96 -> 87).
    vec_t<T, 4> raw[4], raw_z[4];
    const int64_t c = c0 + x, last = a.cols - 4, place = min(c, last);
    if (last >= 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = *reinterpret_cast<const vec_t<T, 4>*>(static_cast<const T*>(a.from) + min(r0 + y + i * 16, a.rows - 1) * a.from_stride + place);
        if (a.z)
#pragma unroll
            for (int i = 0; i < 4; ++i) raw_z[i] = *reinterpret_cast<const vec_t<T, 4>*>(static_cast<const T*>(a.z) + min(r0 + y + i * 16, a.rows - 1) * a.z_stride + place);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t r = min(r0 + y + i * 16, a.rows - 1), e = min(max(place, (int64_t)0) + q, a.cols - 1);
                raw[i][q] = static_cast<const T*>(a.from)[r * a.from_stride + e];
                if (a.z) raw_z[i][q] = static_cast<const T*>(a.z)[r * a.z_stride + e];
            }
    }
    const int moved = last >= 0 ? (int)min(c - place, (int64_t)4) : c == 0 ? 0 : 4, there = (int)min(max(a.cols - c, (int64_t)0), (int64_t)4);
    const bool inside = r0 + 64 <= a.rows && c0 + 64 <= a.cols;
    const auto in_place = [&](const vec_t<T, 4>& from, float (&v)[4], bool row) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (float)from[q];
        if (inside) return;
#pragma unroll
        for (int m = 0; m < 3; ++m)
            if (m < moved) { v[0] = v[1]; v[1] = v[2]; v[2] = v[3]; }
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = row && q < there ? v[q] : 0.0f;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + y + i * 16;
        float v[4];
        in_place(raw[i], v, r < a.rows);
        if (a.z) {
            float z[4];
            in_place(raw_z[i], z, r < a.rows);
            times_slope(v, z, a.activation);               // (past the matrix's end 0 times the slope at 0)
        }
        if (a.straight && r < a.rows) store_part<T, 4>(reinterpret_cast<T*>(a.straight + r * a.straight_pitch) + c, a.straight_pitch / (int)sizeof(T) - c, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) tile[y + i * 16][x + q] = v[q];
    }
    if (!a.turned && !a.sums && !a.dbias) return;
    __syncthreads();
    if (a.turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t c = c0 + y + i * 16, r = r0 + x;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = tile[x + q][y + i * 16];
            if (c < a.cols) store_part<T, 4>(reinterpret_cast<T*>(a.turned + c * a.turned_pitch) + r, a.turned_pitch / (int)sizeof(T) - r, v);
        }
    }
    if ((a.sums || a.dbias) && threadIdx.x < 64 && c0 + threadIdx.x < a.cols) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 64; ++i) s += tile[i][threadIdx.x];
        if (a.sums) a.sums[(int64_t)line * a.cols + c0 + threadIdx.x] = s;
        else store_typed(a.dbias, a.dbias_type, c0 + threadIdx.x, s);
    }
}

// The gradients of up to kRows rows, in one pass over weight and dweight: a wavefront has V columns a lane and kEach of the weight's rows, of which it reads each once, adds dz times it to dx's
// sums and writes what dz and x make of it.  A block's four wavefronts have the same columns; their sums, and those of the blocks along `outer`, are added up in order.  Lanes that the row's end
// cuts take its last V columns, which two lanes then work out alike.  Bound by memory:
// 1 x 4096 x 16384 bf16 48 us from memory, 5.6 TB/s of the two matrices, 8 rows 59 (as products of matrices that are put in order 121 and 122); small ones by two launches, 16 bits'
// eight rows by their vector instructions (least_thin): 8 x 1000 x 1000 bf16 12.9 (14.9), 8 x 1001 x 2003 fp32 13.0 (23.9).
struct Thin {
    const void* dy; const void* z; const void* x; const void* weight; void* dweight; void* dbias; float* sums;     // sums: [parts][rows][across * 64 V], or NULL
    int64_t dy_stride, z_stride, x_stride, weight_stride, dweight_stride, inner, outer;
    int32_t rows, activation, weight_type, across;
};
template <typename T, int kRows, int kEach> __global__ __launch_bounds__(256) void k_linear_thin_backward(Thin a) {
    constexpr int V = 16 / sizeof(T), kOuter = 4 * kEach, kAhead = 8;
    __shared__ float dz[kOuter][kRows];
    __shared__ float part[4][64 * V];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int group = blockIdx.x % a.across, line = blockIdx.x / a.across;
    const int64_t o0 = (int64_t)line * kOuter, c = min(((int64_t)group * 64 + lane) * V, a.inner - V);
    // (rows past the last are that one again, and zeros once they are there: loads without conditions are under way together)
    vec_t<T, V> raw[kRows];
    if (a.dweight)
#pragma unroll
        for (int j = 0; j < kRows; ++j) raw[j] = *reinterpret_cast<const vec_t<T, V>*>(static_cast<const T*>(a.x) + min(j, a.rows - 1) * a.x_stride + c);
    // dz, whose sums over the rows are dbias
    for (int t = threadIdx.x; t < kOuter; t += 256) {
        const int64_t o = min(o0 + t, a.outer - 1);
        T y[kRows], z[kRows];
#pragma unroll
        for (int j = 0; j < kRows; ++j) y[j] = static_cast<const T*>(a.dy)[min(j, a.rows - 1) * a.dy_stride + o];
        if (a.z)
#pragma unroll
            for (int j = 0; j < kRows; ++j) z[j] = static_cast<const T*>(a.z)[min(j, a.rows - 1) * a.z_stride + o];
        float v[kRows], slopes[kRows], sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kRows; ++j) { v[j] = (float)y[j]; slopes[j] = a.z ? (float)z[j] : 0.0f; }
        if (a.z) times_slope(v, slopes, a.activation);
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            if (j >= a.rows) v[j] = 0.0f;
            sum += v[j];
            dz[t][j] = v[j];                               // (32 bits: no matrix unit takes it)
        }
        if (a.dbias && group == 0 && o0 + t < a.outer) store_typed(a.dbias, a.weight_type, o, sum);
    }
    float x[kRows][V] = {}, dx[kRows][V] = {};
    if (a.dweight)
#pragma unroll
        for (int j = 0; j < kRows; ++j)
#pragma unroll
            for (int q = 0; q < V; ++q) x[j][q] = j < a.rows ? (float)raw[j][q] : 0.0f;
    __syncthreads();
    const int64_t first = o0 + wave * kEach;
    const int n = (int)max((int64_t)0, min(a.outer - first, (int64_t)kEach));
    for (int e0 = 0; e0 < n; e0 += kAhead) {
        vec_t<T, V> w[kAhead] = {};
        if (a.sums) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) w[u] = *reinterpret_cast<const vec_t<T, V>*>(static_cast<const T*>(a.weight) + (first + min(e0 + u, n - 1)) * a.weight_stride + c);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (e0 + u >= n) break;
            float d[kRows], out[V] = {};
#pragma unroll
            for (int j = 0; j < kRows; ++j) d[j] = dz[wave * kEach + e0 + u][j];
            if (a.sums) {
#pragma unroll
                for (int j = 0; j < kRows; ++j)
#pragma unroll
                    for (int q = 0; q < V; ++q) dx[j][q] = fmaf(d[j], (float)w[u][q], dx[j][q]);
            }
            if (a.dweight) {
#pragma unroll
                for (int j = 0; j < kRows; ++j)
#pragma unroll
                    for (int q = 0; q < V; ++q) out[q] = fmaf(d[j], x[j][q], out[q]);
                const int64_t at = (first + e0 + u) * a.dweight_stride + c;
                if (a.weight_type == P2_F32) store_vec<float, V>(static_cast<float*>(a.dweight) + at, out);
                else if (a.weight_type == P2_BF16) store_vec<bf16_t, V>(static_cast<bf16_t*>(a.dweight) + at, out);
                else store_vec<half_t, V>(static_cast<half_t*>(a.dweight) + at, out);
            }
        }
    }
    if (!a.sums) return;
    const int64_t pitch = (int64_t)a.across * 64 * V;
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
        if (j >= a.rows) break;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < V; ++q) part[wave][q * 64 + lane] = dx[j][q];
        __syncthreads();
        for (int t = threadIdx.x; t < 64 * V; t += 256) {
            const int at = t % V * 64 + t / V;                 // column t of the block's
            a.sums[((int64_t)line * a.rows + j) * pitch + (int64_t)group * 64 * V + t] = part[0][at] + part[1][at] + part[2][at] + part[3][at];
        }
    }
}
// dx from its parts: a block has 16 columns of a row, and 16 threads a column.
template <typename T> __global__ __launch_bounds__(256) void k_linear_thin_join(const float* sums, int64_t parts, int32_t rows, int64_t inner, int64_t pitch, T* dx, int64_t dx_stride) {
    constexpr int V = 16 / sizeof(T);
    __shared__ float part[16][17];
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4, across = (int)((inner + 15) / 16), j = blockIdx.x / across;
    const int64_t i = (int64_t)(blockIdx.x % across) * 16 + x, cut = inner / V * V;
    const int64_t at = i < cut ? i : cut + V - (inner - min(i, inner - 1));            // the last lane has the row's last V columns
    const float* from = sums + j * pitch + at;
    float s = 0.0f;
#pragma unroll 8
    for (int64_t p = y; p < parts; p += 16) s += from[p * rows * pitch];
    part[y][x] = s;
    __syncthreads();
    if (y > 0 || i >= inner) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) s += part[k][x];
    dx[j * dx_stride + i] = (T)s;
}

__global__ __launch_bounds__(256) void k_linear_zero(void* out, int32_t type, int64_t stride, int64_t rows, int64_t cols) {
    for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < rows * cols; x += (int64_t)gridDim.x * 256) store_typed(out, type, x / cols * stride + x % cols, 0.0f);
}

// ------------------------------------------------------------------------------------------------- plans

enum Cut : int32_t { k256, k128, k128x64, k64x128, k64 };      // tiles: rows of A by rows of B
constexpr Cut kCuts[] = {k256, k128, k128x64, k64x128, k64};
struct Plan { Cut cut; int64_t whole; int32_t parts; };        // (as in Product)
// What a cut takes, in us: a stage of one block that has its compute unit to itself (`alone`), a stage of each of more blocks that share one, a block's end.
struct Price { int64_t a, b; double alone, shared, end; };
constexpr Price kPrices16[] = {{256, 256, 1.38, 1.38, 9.0}, {128, 128, 0.60, 0.55, 2.2}, {128, 64, 0.38, 0.33, 1.1}, {64, 128, 0.40, 0.34, 1.1}, {64, 64, 0.29, 0.22, 0.6}};
constexpr Price kPrices32[] = {{256, 256, 7.0, 7.0, 18.0}, {128, 128, 1.9, 1.9, 4.4}, {128, 64, 0.94, 0.94, 2.2}, {64, 128, 0.95, 0.95, 2.2}, {64, 64, 0.47, 0.47, 1.2}};
int64_t tile_a(Cut c) { return kPrices16[c].a; }
int64_t tile_b(Cut c) { return kPrices16[c].b; }
// How a product of these sizes is cut: the cheapest by prices that were measured (blocks go to the 256 compute units one by one; a sum in parts is written and
// read once more, by a launch of its own).  us by 256 x 256, 128 x 128, 128 x 64, 64 x 64 tiles, with the best number of parts each, bf16: 8192 x 4096 x 4096
// 194, 240, 280, 330; 3000^3 73, 85, 102, 121; 2048^3 38, 23.5, 24.1, 28; 1024^3 23, 14, 9.5, 8.0; 512 x 4096 x 4096 36, 28, 27, 27; 64 x 4096 x 4096
// 20, 14.6, 13.4, 12.5; 256 x 8192 x 256 23.5, 16.3, 13.5, 11.8; fp32 1531 x 1000 x 776 54, 36, 34, 33.
// Tiles that fill the units whole times may have a block each and the rest be cut into parts (us, against all tiles cut alike: fp32 1531 x 1000 x 777 38 -> 29, 5000 x 800 x 600
// 54 -> 48; bf16 3500 x 8192 x 2500 152 -> 135, 4096 x 4096 x 5120 160 -> 152; 1500^3 31.4 -> 32.4).
// k_linear_any takes some half more (us, as they are against put in order first, bf16: 700 x 701 x 703 10.4 against 12.8, 100 x 5001 x 9001 50 against 67, 2000 x 1001 x 4001 32 against 36,
// 4085 x 2093 x 367 34 against 29; fp32 440 x 111 x 78 7.1 against 11.1, 3001 x 2001 x 1003 114 against 108).
constexpr double kAny = 1.5;
// A way to cut a product: blocks that have a tile and those that have a part of one, a tile's stages and a part's, what joining takes, and what all takes in one launch.
struct Offer { Plan plan; int64_t whole, rest, stages, part; double join, us; };
// (Of the numbers of parts that keep the units equally long, the one that is worth joining: a call is planned in a few us.)
constexpr int kOffers = 9;
int offers_of(Cut cut, int32_t type, int64_t a_rows, int64_t b_rows, int64_t length, Offer (&offers)[kOffers]) {
    const int64_t stages = ceil_div(length, kLine);
    const Price& price = type == P2_F32 ? kPrices32[cut] : kPrices16[cut];
    const int64_t tiles = ceil_div(a_rows, price.a) * ceil_div(b_rows, price.b), full = tiles / kUnits * kUnits;
    int n = 0;
    const auto offer = [&](int64_t whole, int64_t parts) {
        const int64_t part = ceil_div(stages, parts);
        const double before = (double)(whole / kUnits), after = (double)ceil_div((tiles - whole) * parts, kUnits), longest = (double)(whole ? stages : part);
        const double bytes = (double)parts * std::min((double)(tiles - whole) * (double)(price.a * price.b), (double)a_rows * (double)b_rows) * 8.0;
        const double join = parts == 1 ? 0.0 : 2.5 + 0.15 * (double)parts + bytes / 5e6;
        const double us = std::max(price.alone * longest, price.shared * (before * (double)stages + after * (double)part)) + (before + after) * price.end + join;
        if (parts == 1) offers[n++] = {{cut, tiles, 1}, tiles, 0, stages, 0, join, us};
        else offers[n++] = {{cut, whole, (int32_t)parts}, whole, (tiles - whole) * parts, stages, part, join, us};
    };
    offer(0, 1);
    for (const int64_t whole : {(int64_t)0, full}) {
        const int64_t rest = tiles - whole;
        if (rest == 0 || (whole == 0 && n > 1)) break;                                 // (full may be 0, too)
        const double each = 0.15 + std::min((double)rest * (double)(price.a * price.b), (double)a_rows * (double)b_rows) * 8.0 / 5e6;      // a part more, joined
        int64_t before = 1;
        for (int64_t load = 1; load <= 4; ++load) {
            const int64_t most = std::min({(int64_t)32, stages / 4, load * kUnits / rest}), worth = (int64_t)(std::sqrt((double)(stages * load) * price.shared / each) + 0.5);
            const int64_t parts = std::min(most, std::max<int64_t>(worth, 2));
            if (parts > before) { offer(whole, parts); before = parts; }
        }
    }
    return n;
}
Plan plan_of(int32_t type, int64_t a_rows, int64_t b_rows, int64_t length, bool small, double* us) {
    Offer best = {}, offers[kOffers];
    best.us = std::numeric_limits<double>::infinity();
    for (const Cut cut : kCuts) {
        if (small && cut == k256) continue;
        const int n = offers_of(cut, type, a_rows, b_rows, length, offers);
        for (int i = 0; i < n; ++i)
            if (offers[i].us < best.us) best = offers[i];
    }
    if (us) *us = best.us;
    return best.plan;
}
// Units that are done at the same time.
struct Shift {
    double at[16]; int64_t units[16];
    int n;
    // `blocks` of `us` each go to the units that are done first
    void take(int64_t blocks, double us) {
        while (blocks > 0) {
            int first = 0, last = 0;
            for (int i = 1; i < n; ++i) {
                if (at[i] < at[first]) first = i;
                if (at[i] > at[last]) last = i;
            }
            if (blocks >= kUnits && at[last] - at[first] <= us) {                      // all units alike
                for (int i = 0; i < n; ++i) at[i] += (double)(blocks / kUnits) * us;
                blocks %= kUnits;
                continue;
            }
            const int64_t some = n < 16 ? std::min(blocks, units[first]) : units[first];       // (16 shifts are more than four kinds of blocks make)
            blocks -= some;
            units[first] -= some;
            const double end = at[first] + us;
            int same = 0;
            while (same < n && !(std::fabs(at[same] - end) < 1e-6 && same != first)) ++same;
            if (same < n) {
                units[same] += some;
                if (units[first] == 0) { at[first] = at[n - 1]; units[first] = units[n - 1]; --n; }
            } else if (units[first] == 0) {
                at[first] = end;
                units[first] = some;
            } else {
                at[n] = end;
                units[n++] = some;
            }
        }
    }
    double end() const { return *std::max_element(at, at + n); }
};
// Two products of one launch have one cut.  (joined: there is a launch that joins dbias anyway.)  What they take is found by dealing their blocks out to the units, of each product's a few ways to cut it.  (us, against the cuts that are best for
// each by itself: fp16 2001 x 1023 x 515 29.7 -> 26.0, 3001 x 1501 x 2003 74 -> 66, fp32 100 x 3000 x 2000 56.6 -> 54.7; a plan takes the host 1 us)
void plan_both(int32_t type, int64_t a0, int64_t b0, int64_t length0, int64_t a1, int64_t b1, int64_t length1, bool joined, Plan& p0, Plan& p1) {
    double least = std::numeric_limits<double>::infinity();
    Offer o[2][kOffers];
    for (const Cut cut : kCuts) {
        const Price& price = type == P2_F32 ? kPrices32[cut] : kPrices16[cut];
        int n[2] = {offers_of(cut, type, a0, b0, length0, o[0]), offers_of(cut, type, a1, b1, length1, o[1])};
        if (price.shared * (double)(o[0][0].whole * o[0][0].stages + o[1][0].whole * o[1][0].stages) / kUnits >= least) continue;
        for (int k = 0; k < 2; ++k) {                          // uncut, and the best two of the others
            std::partial_sort(o[k] + 1, o[k] + std::min(n[k], 3), o[k] + n[k], [](const Offer& x, const Offer& y) { return x.us < y.us; });
            n[k] = std::min(n[k], 3);
        }
        for (int i = 0; i < n[0]; ++i)
            for (int k = 0; k < n[1]; ++k) {
                const Offer &x = o[0][i], &y = o[1][k];
                Shift shift;
                shift.n = 1; shift.at[0] = 0.0; shift.units[0] = kUnits;
                for (const Offer* f : {&x, &y}) {
                    shift.take(f->whole, price.shared * (double)f->stages + price.end);
                    shift.take(f->rest, price.shared * (double)f->part + price.end);
                }
                const double alone = price.alone * (double)std::max(x.whole ? x.stages : x.part, y.whole ? y.stages : y.part) + price.end;
                double us = std::max(shift.end(), alone) + std::max(0.0, x.join - 2.5) + std::max(0.0, y.join - 2.5) + (!joined && (x.rest || y.rest) ? 2.5 : 0.0);
                if (cut == k256 && type != P2_F32) us = x.us + y.us;                   // (turned operands: a launch each)
                if (us < least) { least = us; p0 = x.plan; p1 = y.plan; }
            }
    }
}
int64_t sums_bytes(const Plan& p, int64_t a_rows, int64_t b_rows) {
    const int64_t rest = ceil_div(a_rows, tile_a(p.cut)) * ceil_div(b_rows, tile_b(p.cut)) - p.whole;
    return p.parts > 1 ? rest * p.parts * tile_a(p.cut) * tile_b(p.cut) * 4 : 0;
}

// One product, or two of one cut; and the columns' sums of `join` where it has lines.  `any`: rows of any alignment, one product.
template <typename T> hipError_t multiply_rows(Product* p, const Plan* plan, int n, Join join, bool any, hipStream_t s) {
    Products all = {};
    int64_t blocks = 0, joined = 0;
    for (int i = 0; i < n; ++i) {
        p[i].tile_a = (int32_t)tile_a(plan[i].cut);
        p[i].tile_b = (int32_t)tile_b(plan[i].cut);
        p[i].across = (int32_t)ceil_div(p[i].a_rows, p[i].tile_a);
        p[i].down = (int32_t)ceil_div(p[i].b_rows, p[i].tile_b);
        p[i].whole = (int32_t)plan[i].whole;
        p[i].parts = plan[i].parts;
        all.p[i] = p[i];
        const int64_t rest = (int64_t)p[i].across * p[i].down - p[i].whole;
        blocks += p[i].whole + rest * p[i].parts;
        if (i == 0) all.blocks = (int32_t)blocks;
        if (p[i].parts > 1) {
            join.p[i] = p[i];
            join.blocks[i] = (int32_t)std::min<int64_t>(ceil_div(rest * p[i].tile_a * p[i].tile_b / 4, 256), 4096);
            joined += join.blocks[i];
        }
    }
    if (n > 0 && p[0].turned_a) {
        // (a launch each: of one cut and of some size they do not need each other's blocks)
        if constexpr (sizeof(T) == 2)
            for (int i = 0; i < n; ++i) {
                Products one = {};
                one.p[0] = all.p[i];
                one.blocks = (int32_t)(p[i].whole + ((int64_t)p[i].across * p[i].down - p[i].whole) * p[i].parts);
                if (p[i].turned_b) k_linear_wide<T, 2, 4, 4, 2, true, true><<<dim3((unsigned)one.blocks), dim3(512), 0, s>>>(one);
                else k_linear_wide<T, 2, 4, 4, 2, true, false><<<dim3((unsigned)one.blocks), dim3(512), 0, s>>>(one);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
    } else if (n > 0) {
        const dim3 grid((unsigned)blocks);
        if (any) switch (plan[0].cut) {
            case k256: case k128: k_linear_any<T, 2, 2, 2, 2><<<grid, dim3(256), 0, s>>>(p[0]); break;      // (k256: never planned)
            case k128x64: k_linear_any<T, 2, 2, 2, 1><<<grid, dim3(256), 0, s>>>(p[0]); break;
            case k64x128: k_linear_any<T, 2, 2, 1, 2><<<grid, dim3(256), 0, s>>>(p[0]); break;
            case k64: k_linear_any<T, 2, 2, 1, 1><<<grid, dim3(256), 0, s>>>(p[0]); break;
        } else switch (plan[0].cut) {
            case k256: k_linear_wide<T, 2, 4, 4, 2><<<grid, dim3(512), 0, s>>>(all); break;
            case k128: k_linear_wide<T, 2, 2, 2, 2><<<grid, dim3(256), 0, s>>>(all); break;
            case k128x64: k_linear_wide<T, 2, 2, 2, 1><<<grid, dim3(256), 0, s>>>(all); break;
            case k64x128: k_linear_wide<T, 2, 2, 1, 2><<<grid, dim3(256), 0, s>>>(all); break;
            case k64: k_linear_wide<T, 2, 2, 1, 1><<<grid, dim3(256), 0, s>>>(all); break;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (join.lines) joined += ceil_div(join.cols, 16);
    if (joined == 0) return hipSuccess;
    k_linear_join<T><<<dim3((unsigned)joined), dim3(256), 0, s>>>(join);
    return hipGetLastError();
}

// Up to three matrices.
template <typename T> hipError_t pack(const Pack* a, int n, hipStream_t s) {
    Packs all = {};
    int64_t blocks = 0;
    for (int m = 0; m < 3; ++m) {
        all.begin[m] = (int32_t)blocks;
        if (m >= n) continue;
        const int64_t cols = a[m].straight ? std::max<int64_t>(a[m].cols, a[m].straight_pitch / sizeof(T)) : a[m].cols;
        const int64_t rows = a[m].turned ? std::max<int64_t>(a[m].rows, a[m].turned_pitch / sizeof(T)) : a[m].rows;
        all.p[m] = a[m];
        all.across[m] = (int32_t)ceil_div(cols, 64);
        blocks += all.across[m] * ceil_div(rows, 64);
    }
    if (blocks == 0) return hipSuccess;
    k_linear_pack<T><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(all);
    return hipGetLastError();
}

// Whether rows can be brought to LDS as they are.
bool in_order(const void* p, int64_t stride, int32_t type, int64_t cols) {
    const int64_t size = (int64_t)type_bytes(type);
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0 && cols * size % 16 == 0 && stride * size <= ((int64_t)1 << 22);
}
// So few that the products are worked out beside the loads (3 and 4 of 16 bits, which have to be converted: 4 x 4096 x 16384 bf16 50 us, by matrix instructions 34).
bool few_rows(int64_t rows, int32_t type) { return rows <= (type == P2_F32 ? 4 : 2); }
// What k_linear_thin takes, in us, as in offers_of: a wavefront's pieces one after the other, or the weight's bytes (of rows that are not in order the caches pass each line several times).
double thin_us(const LinearForward& a, bool ordered) {
    const double bytes = (double)a.inner * (double)type_bytes(a.type), blocks = (double)a.outer / (a.outer >= 32 * kUnits ? 32.0 : 16.0);
    const double pieces = std::ceil(bytes / (8 * kLine)) * (a.rows <= 16 ? 0.55 : 1.2) * std::ceil(blocks / (2.0 * kUnits));
    return 0.8 + std::max(pieces, bytes * (double)a.outer / 4.3e6 * (ordered ? 1.0 : 3.0));
}

struct ForwardRoom { bool thin, pack_x, pack_weight, any; Plan plan; int64_t length, x, weight, sums, bytes; };
ForwardRoom forward_room(const LinearForward& a) {
    ForwardRoom r = {};
    if (few_rows(a.rows, a.type)) return r;
    const int64_t size = (int64_t)type_bytes(a.type), padded = round_up(a.inner * size, kLine);
    r.pack_x = !in_order(a.x, a.x_stride, a.type, a.inner);
    r.pack_weight = !in_order(a.weight, a.weight_stride, a.type, a.inner);
    r.length = r.pack_x && r.pack_weight ? padded : round_up(a.inner * size, 16);
    double us = 0.0, any_us = 0.0;
    r.plan = plan_of(a.type, a.outer, a.rows, r.length, false, &us);
    if (r.pack_x || r.pack_weight) {
        // rows that are not in order are put in order first, or multiplied as they are, by whichever takes less
        const Plan any = plan_of(a.type, a.outer, a.rows, a.inner * size, true, &any_us);
        us += 4.0 + ((r.pack_x ? a.rows : 0) + (r.pack_weight ? a.outer : 0)) * (double)a.inner * size * 2.0 / 3.5e6;
        if (any_us * kAny < us) {
            us = any_us * kAny;
            r.plan = any;
            r.any = true;
            r.pack_x = r.pack_weight = false;
            r.length = a.inner * size;
        }
    }
    // Few rows come out of registers where that takes less (rows x inner x outer, us: bf16 5 x 4096 x 16384 38 -> 34, 16 x 1000 x 1000 8.5 -> 5.3, fp32 8 x 4096 x 8192 44 -> 34, 8 x 1001 x 2003 10.6 -> 5.6; but
    // fp16 30 x 8000 x 500 11 -> 22, bf16 16 x 4097 x 16383 54 -> 77).
    const double weight_us = (double)a.outer * (double)a.inner * (double)size / 3.8e6;
    if (a.rows <= 32 && thin_us(a, in_order(a.x, a.x_stride, a.type, 16 / size) && in_order(a.weight, a.weight_stride, a.type, 16 / size)) < std::max(us, weight_us)) {
        ForwardRoom thin = {};
        thin.thin = true;
        return thin;
    }
    r.x = 0;
    r.weight = r.x + (r.pack_x ? round_up(a.rows * padded, 256) : 0);
    r.sums = r.weight + (r.pack_weight ? round_up(a.outer * padded, 256) : 0);
    r.bytes = r.sums + sums_bytes(r.plan, a.outer, a.rows);
    return r;
}

// From how many of the weight's rows on up to eight rows take k_linear_thin_backward, whose chain of vector instructions grows with x's rows (us on the device, against products of matrices put in
// order, at 16 and 100 / 500 / 1000 of the weight's: bf16 8 x 1000 12.2 and 12.5 against 8.4 and 9.0 / 12.7, 11.4 / the same within 3 %; 5 x 1000 10.9 and 11.2 against 8.4 and 9.0 / the same;
// 4 x 1000 9.2 and 9.5 against 8.5 and 9.0; fp32 8 x 1000 9.4 against 8.9 / less from 100 on; one and two rows less throughout; long rows pay earlier: 5 x 16384 14.2 against 12.9 at 100,
// 21.1 against 27.8 at 500).
int64_t least_thin(int32_t type, int64_t rows, int64_t inner) {
    const int64_t least = type == P2_F32 ? (rows > 4 ? 64 : 1) : rows > 4 ? 768 : rows > 2 ? 128 : 1;
    return inner > 8192 ? ceil_div(least, 3) : least;
}

struct BackwardRoom { bool thin; int64_t each, across, parts; Plan dx, dweight; int64_t along, deep, bytes; };      // bytes: enough for any call of these sizes
BackwardRoom backward_room(int32_t type, int64_t rows, int64_t inner, int64_t outer) {
    // (A call asks twice, for its workspace and for itself: the last sizes' answer is kept.)
    struct Last { int32_t type; int64_t rows, inner, outer; BackwardRoom room; };
    static thread_local Last last = {};
    if (last.rows == rows && last.type == type && last.inner == inner && last.outer == outer) return last.room;
    const int64_t size = (int64_t)type_bytes(type);
    BackwardRoom r = {};
    const int64_t values = 16 / size;
    if (rows <= 8 && inner >= values && outer >= least_thin(type, rows, inner)) {
        r.thin = true;
        r.across = ceil_div(inner, 64 * values);
        r.each = r.across * ceil_div(outer, 256) >= 2 * kUnits ? 64 : 8;               // of the weight's rows a wavefront
        r.parts = ceil_div(outer, 4 * r.each);
        r.bytes = round_up(r.parts * rows * r.across * 64 * values * 4, 256);
        last = {type, rows, inner, outer, r};
        return r;
    }
    r.along = round_up(outer * size, kLine);               // a row of dz, and of the weight turned
    r.deep = round_up(rows * size, kLine);                 // a row of dz turned, and of x turned
    plan_both(type, inner, rows, r.along, inner, outer, r.deep, rows > 64, r.dx, r.dweight);
    r.bytes = round_up(rows * r.along, 256) + round_up(outer * r.deep, 256) + round_up(inner * r.deep, 256) + round_up(inner * r.along, 256) + round_up(ceil_div(rows, 64) * outer * 4, 256) +
              sums_bytes(r.dx, inner, rows) + sums_bytes(r.dweight, inner, outer);
    last = {type, rows, inner, outer, r};
    return r;
}

// What a call of these arguments uses of its workspace, and where.
struct BackwardLayout { bool own_dz, turned; int64_t dz, dz_turned, x_turned, weight_turned, lines, sums, more_sums, bytes; };
BackwardLayout layout_of(const LinearBackward& a, const BackwardRoom& r) {
    BackwardLayout l = {};
    if (r.thin) {
        l.bytes = a.dx ? r.bytes : 0;
        return l;
    }
    l.own_dz = a.activation != P2_NO_ACTIVATION || !in_order(a.dy, a.dy_stride, a.type, a.outer);
    // Large 16-bit products take weight, x and dz turned as they lie in memory, and only dz is put in order
    // (us, bf16, without / with an activation: 8192 x 4096 x 4096 428 -> 394 / 460 -> 431, 32768 x 1024 x 1024 213 -> 156 / 248 -> 191, 4096^3 225 -> 207 / 238 -> 220).
    l.turned = a.type != P2_F32 && r.dx.cut == k256 && r.dweight.cut == k256 && a.outer % 8 == 0 && (!a.dx || in_order(a.weight, a.weight_stride, a.type, a.inner)) &&
               (!a.dweight || in_order(a.x, a.x_stride, a.type, a.inner));
    const auto place = [&](bool used, int64_t bytes) {
        const int64_t at = l.bytes;
        if (used) l.bytes += round_up(bytes, 256);
        return at;
    };
    l.dz = place(l.own_dz && (a.dx || (a.dweight && l.turned)), a.rows * r.along);
    l.dz_turned = place(a.dweight && !l.turned, a.outer * r.deep);
    l.x_turned = place(a.dweight && !l.turned, a.inner * r.deep);
    l.weight_turned = place(a.dx && !l.turned, a.inner * r.along);
    l.lines = place(a.dbias && a.rows > 64, ceil_div(a.rows, 64) * a.outer * 4);
    l.sums = place(a.dx != nullptr, sums_bytes(r.dx, a.inner, a.rows));
    l.more_sums = place(a.dweight != nullptr, sums_bytes(r.dweight, a.inner, a.outer));
    return l;
}

template <typename T> hipError_t forward(const LinearForward& a, hipStream_t s) {
    Result r = {};
    r.bias = a.bias; r.residual = a.residual; r.y = a.y; r.z = a.z;
    r.residual_stride = a.residual_stride; r.y_stride = a.y_stride; r.z_stride = a.z_stride;
    r.y_type = a.type; r.activation = a.activation;
    const T* x = static_cast<const T*>(a.x);
    const T* w = static_cast<const T*>(a.weight);
    if (few_rows(a.rows, a.type)) {
        const dim3 grid((unsigned)ceil_div(a.outer, 8)), block(256);
        const auto launch = [&](auto rows, auto ahead) {
            k_linear_rows<T, decltype(rows)::value, 2, decltype(ahead)::value><<<grid, block, 0, s>>>(x, a.x_stride, w, a.weight_stride, a.inner, a.outer, r);
        };
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 4> four;
        const bool ahead = a.inner * (int64_t)sizeof(T) >= 4 * 64 * 16;
        if (a.rows == 1) { if (ahead) launch(one, four); else launch(one, one); }
        else if (a.rows == 2) { if (ahead) launch(two, four); else launch(two, one); }
        else if constexpr (sizeof(T) == 4) {
            if (a.rows == 3) launch(std::integral_constant<int, 3>(), one);
            else launch(four, one);
        }
        return hipGetLastError();
    }
    const ForwardRoom room = forward_room(a);
    if (room.thin) {
        const auto launch = [&](auto rows, auto fragments, auto ahead) {
            constexpr int kFragments = decltype(fragments)::value;
            k_linear_thin<T, decltype(rows)::value, kFragments, decltype(ahead)::value>
                <<<dim3((unsigned)ceil_div(a.outer, kFragments * 16)), dim3(512), 0, s>>>(x, a.x_stride, w, a.weight_stride, a.rows, a.inner, a.outer, r);
        };
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 4> four;
        const bool wide = a.outer >= 32 * kUnits;              // (enough blocks of twice as many of the weight's rows)
        if (a.rows <= 16) { if (wide) launch(one, two, four); else launch(one, one, four); }
        else if (wide) launch(two, two, two);
        else launch(two, one, four);
        return hipGetLastError();
    }
    const int64_t padded = round_up(a.inner * (int64_t)sizeof(T), kLine);
    Product p = {};
    p.a = static_cast<const char*>(a.weight);
    p.a_pitch = a.weight_stride * (int64_t)sizeof(T);
    p.b = static_cast<const char*>(a.x);
    p.b_pitch = a.x_stride * (int64_t)sizeof(T);
    Pack k[2] = {};
    int packs = 0;
    if (room.pack_x) {
        k[packs].from = a.x; k[packs].from_stride = a.x_stride; k[packs].rows = a.rows;
        p.b = k[packs++].straight = a.workspace + room.x;
        p.b_pitch = padded;
    }
    if (room.pack_weight) {
        k[packs].from = a.weight; k[packs].from_stride = a.weight_stride; k[packs].rows = a.outer;
        p.a = k[packs++].straight = a.workspace + room.weight;
        p.a_pitch = padded;
    }
    for (int i = 0; i < packs; ++i) { k[i].straight_pitch = padded; k[i].cols = a.inner; }
    const hipError_t e = pack<T>(k, packs, s);
    if (e != hipSuccess) return e;
    p.a_rows = a.outer; p.b_rows = a.rows; p.length = room.length;
    p.sums = reinterpret_cast<float*>(a.workspace + room.sums);
    p.r = r;
    return multiply_rows<T>(&p, &room.plan, 1, Join(), room.any, s);
}

template <typename T> hipError_t backward(const LinearBackward& a, hipStream_t s) {
    const BackwardRoom room = backward_room(a.type, a.rows, a.inner, a.outer);
    if (room.thin) {
        Thin t = {};
        t.dy = a.dy; t.x = a.x; t.weight = a.weight; t.dweight = a.dweight; t.dbias = a.dbias;
        if (a.activation != P2_NO_ACTIVATION) t.z = a.z;
        if (a.dx) t.sums = reinterpret_cast<float*>(a.workspace);
        t.dy_stride = a.dy_stride; t.z_stride = a.z_stride; t.x_stride = a.x_stride; t.weight_stride = a.weight_stride; t.dweight_stride = a.dweight_stride;
        t.inner = a.inner; t.outer = a.outer; t.rows = (int32_t)a.rows; t.activation = a.activation; t.weight_type = a.weight_type; t.across = (int32_t)room.across;
        const auto launch = [&](auto rows) {
            constexpr int kRows = decltype(rows)::value;
            const dim3 grid((unsigned)(room.across * room.parts)), block(256);
            if (room.each == 64) k_linear_thin_backward<T, kRows, 64><<<grid, block, 0, s>>>(t);
            else k_linear_thin_backward<T, kRows, 8><<<grid, block, 0, s>>>(t);
        };
        if (a.rows == 1) launch(std::integral_constant<int, 1>());
        else if (a.rows == 2) launch(std::integral_constant<int, 2>());
        else if (a.rows <= 4) launch(std::integral_constant<int, 4>());
        else launch(std::integral_constant<int, 8>());
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || !a.dx) return e;
        k_linear_thin_join<T><<<dim3((unsigned)(a.rows * ceil_div(a.inner, 16))), dim3(256), 0, s>>>(t.sums, room.parts, t.rows, a.inner, room.across * 64 * (16 / (int64_t)sizeof(T)), static_cast<T*>(a.dx),
                                                                                                   a.dx_stride);
        return hipGetLastError();
    }
    const BackwardLayout at = layout_of(a, room);
    const bool own_dz = at.own_dz, turned = at.turned;
    const char* const dz_rows = own_dz ? a.workspace + at.dz : static_cast<const char*>(a.dy);
    const int64_t dz_pitch = own_dz ? room.along : a.dy_stride * (int64_t)sizeof(T);
    Pack k[3] = {};
    int packs = 0;
    Pack& dz = k[packs];
    dz.from = a.dy; dz.from_stride = a.dy_stride;
    if (a.activation != P2_NO_ACTIVATION) { dz.z = a.z; dz.z_stride = a.z_stride; }
    dz.rows = a.rows; dz.cols = a.outer; dz.activation = a.activation;
    if ((a.dx || (a.dweight && turned)) && own_dz) { dz.straight = a.workspace + at.dz; dz.straight_pitch = room.along; }
    if (a.dweight && !turned) { dz.turned = a.workspace + at.dz_turned; dz.turned_pitch = room.deep; }
    if (a.dbias && a.rows <= 64) { dz.dbias = a.dbias; dz.dbias_type = a.weight_type; }
    else if (a.dbias) dz.sums = reinterpret_cast<float*>(a.workspace + at.lines);
    if (dz.straight || dz.turned || dz.sums || dz.dbias) ++packs;
    Product p[2] = {};
    Plan plan[2];
    int products = 0;
    if (a.dx) {
        Product& q = p[products];
        if (turned) {
            q.a = static_cast<const char*>(a.weight); q.a_pitch = a.weight_stride * (int64_t)sizeof(T); q.turned_a = true;
        } else {
            Pack& w = k[packs++];
            w = Pack();
            w.from = a.weight; w.from_stride = a.weight_stride; w.rows = a.outer; w.cols = a.inner;
            w.turned = a.workspace + at.weight_turned; w.turned_pitch = room.along;
            q.a = w.turned; q.a_pitch = room.along;
        }
        q.a_rows = a.inner;
        q.b = dz_rows; q.b_pitch = dz_pitch; q.b_rows = a.rows;
        q.length = own_dz && !turned ? room.along : a.outer * (int64_t)sizeof(T);
        q.sums = reinterpret_cast<float*>(a.workspace + at.sums);
        q.r.y = a.dx; q.r.y_stride = a.dx_stride; q.r.y_type = a.type;
        plan[products++] = room.dx;
    }
    if (a.dweight) {
        Product& q = p[products];
        if (turned) {
            q.a = static_cast<const char*>(a.x); q.a_pitch = a.x_stride * (int64_t)sizeof(T); q.turned_a = true;
            q.b = dz_rows; q.b_pitch = dz_pitch; q.turned_b = true;
            q.length = a.rows * (int64_t)sizeof(T);
        } else {
            Pack& x = k[packs++];
            x = Pack();
            x.from = a.x; x.from_stride = a.x_stride; x.rows = a.rows; x.cols = a.inner;
            x.turned = a.workspace + at.x_turned; x.turned_pitch = room.deep;
            q.a = x.turned; q.a_pitch = room.deep;
            q.b = a.workspace + at.dz_turned; q.b_pitch = room.deep;
            q.length = room.deep;
        }
        q.a_rows = a.inner; q.b_rows = a.outer;
        q.sums = reinterpret_cast<float*>(a.workspace + at.more_sums);
        q.r.y = a.dweight; q.r.y_stride = a.dweight_stride; q.r.y_type = a.weight_type;
        plan[products++] = room.dweight;
    }
    const hipError_t e = pack<T>(k, packs, s);
    if (e != hipSuccess) return e;
    Join join = {};
    if (dz.sums) {
        join.lines = dz.sums; join.n = ceil_div(a.rows, 64); join.cols = a.outer;
        join.out = a.dbias; join.type = a.weight_type;
    }
    return multiply_rows<T>(p, plan, products, join, false, s);
}

}  // namespace

int64_t linear_forward_workspace(const LinearForward& a) { return a.rows ? forward_room(a).bytes : 0; }
int64_t linear_backward_workspace(const LinearBackward& a) { return a.rows ? layout_of(a, backward_room(a.type, a.rows, a.inner, a.outer)).bytes : 0; }
int64_t linear_backward_workspace(int32_t type, int64_t rows, int64_t inner, int64_t outer) { return rows ? backward_room(type, rows, inner, outer).bytes : 0; }

hipError_t launch_linear_forward(const LinearForward& a, hipStream_t s) {
    return a.type == P2_F32 ? forward<float>(a, s) : a.type == P2_BF16 ? forward<bf16_t>(a, s) : forward<half_t>(a, s);
}

hipError_t launch_linear_backward(const LinearBackward& a, hipStream_t s) {
    if (a.rows == 0) {
        if (a.dweight) {
            k_linear_zero<<<dim3((unsigned)std::min<int64_t>(ceil_div(a.outer * a.inner, 256), 65536)), dim3(256), 0, s>>>(a.dweight, a.weight_type, a.dweight_stride, a.outer, a.inner);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (!a.dbias) return hipSuccess;
        k_linear_zero<<<dim3((unsigned)ceil_div(a.outer, 256)), dim3(256), 0, s>>>(a.dbias, a.weight_type, a.outer, 1, a.outer);
        return hipGetLastError();
    }
    return a.type == P2_F32 ? backward<float>(a, s) : a.type == P2_BF16 ? backward<bf16_t>(a, s) : backward<half_t>(a, s);
}

}  // namespace p2
