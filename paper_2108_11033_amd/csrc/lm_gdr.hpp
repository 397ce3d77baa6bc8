// What the kernels of the gated delta rule share: matrices in LDS as sums of bf16 parts, products of them, chunks of packed sequences.
//
// A number is held as the sum of P bf16 parts, each the rounding of what the parts before it leave: two parts are off by at most 2^-17 of the number, three
// by 2^-25 or so.  The product of two numbers takes the parts' products whose numbers add up to less than the larger P, summed in fp32 by the matrix cores.  Operands
// that come as bf16 are one part, fp16 two, fp32 three, all exact; what is computed between products (states, differences) is two parts where operands are 16 bits
// wide, whose own roundings are 2^-8 and 2^-11, and three in fp32.  (The fp32 matrix instruction does a sixteenth of the work of the bf16 one.)
#pragma once
#include "lm_common.hpp"

namespace grim {
namespace lm {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Gdr;
// chunk: tokens that the matrix form takes at a time.  (In fp32 a chunk of 64 tokens has no room in LDS.)
template <>
struct Gdr<bf16> { static constexpr int data = 1, comp = 2, chunk = 64; };
template <>
struct Gdr<f16> { static constexpr int data = 2, comp = 2, chunk = 64; };
template <>
struct Gdr<float> { static constexpr int data = 3, comp = 3, chunk = 32; };

constexpr int kGdrColumns = 64;                 // columns of the states that a workgroup takes
constexpr int kGdrThreads = 256;
constexpr double kLeastDecay = -10000.;

// ---------------------------------------------------------------------------------------------------- matrices in LDS
// P parts of ROWS x COLS, rows 16 bytes longer than their elements: the rows that one instruction reads then lie in different banks.
template <int P, int ROWS, int COLS>
struct Tile {
    static constexpr int parts = P, ld = COLS + 8, part = ROWS * ld, bytes = P * part * 2;
    uint16_t *at;
};

template <int P>
struct Frag { s16x8 part[P]; };

// 16 rows from r, as an operand whose sum runs along them, over elements k .. k + 31.
template <int P, int R, int C>
__device__ __forceinline__ Frag<P> along(const Tile<P, R, C> &m, int r, int k) {
    const int lane = threadIdx.x & 63;
    Frag<P> f;
#pragma unroll
    for (int p = 0; p < P; ++p)
        f.part[p] = *reinterpret_cast<const s16x8 *>(m.at + p * m.part + (r + (lane & 15)) * m.ld + k + (lane >> 4) * 8);
    return f;
}

// 16 columns from c, as an operand whose sum runs over rows k .. k + 31: the transposing read hands each lane of 16 four rows at one column.
template <int P, int R, int C>
__device__ __forceinline__ Frag<P> across(const Tile<P, R, C> &m, int c, int k) {
    const int lane = threadIdx.x & 63, j = lane & 15;
    Frag<P> f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        uint16_t *from = m.at + p * m.part + (k + (lane >> 4) * 8 + j / 4) * m.ld + c + (j % 4) * 4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)from);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(from + 4 * m.ld));
        f.part[p] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    return f;
}

// acc + the 16 x 16 product: a lane has rows (lane / 16) 4 .. + 3 of a's at column lane % 16 of b's.  Small terms first.
template <int PA, int PB>
__device__ __forceinline__ f32x4 multiply(const Frag<PA> &a, const Frag<PB> &b, f32x4 acc) {
    constexpr int P = PA > PB ? PA : PB;
#pragma unroll
    for (int s = P - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (s - i >= 0 && s - i < PB)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a.part[i]), __builtin_bit_cast(b16x8, b.part[s - i]), acc, 0, 0, 0);
    return acc;
}

// Elements c .. c + 3 of row r.
template <int P, int R, int C>
__device__ __forceinline__ void put4(const Tile<P, R, C> &m, int r, int c, f32x4 v) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        bf16 h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            h[j] = (bf16)v[j];
            if (p + 1 < P) v[j] -= (float)h[j];
        }
        s16x4 w;
        __builtin_memcpy(&w, h, 8);
        *reinterpret_cast<s16x4 *>(m.at + p * m.part + r * m.ld + c) = w;
    }
}

template <int P, int R, int C, typename T>
__device__ __forceinline__ void put8(const Tile<P, R, C> &m, int r, int c, const Pack<T, 8> &raw, const float (&x)[8]) {
    if constexpr (__is_same(T, bf16) && P == 1) {
        __builtin_memcpy(m.at + r * m.ld + c, raw.w, 16);
    } else {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x[j];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            bf16 h[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[j] = (bf16)v[j];
                if (p + 1 < P) v[j] -= (float)h[j];
            }
            __builtin_memcpy(m.at + p * m.part + r * m.ld + c, h, 16);
        }
    }
}

// Rows of keys or queries on their way to LDS: COLS elements in pieces of 8, dealt to the workgroup's threads; zeros behind the head's
// width and the last row.
template <typename T, int ROWS, int COLS>
struct Rows {
    static constexpr int per_row = COLS / 8, PER = ROWS * per_row / kGdrThreads;
    static_assert(PER * kGdrThreads == ROWS * per_row, "whole pieces");
    Pack<T, 8> raw[PER];
    __device__ __forceinline__ static int row(int k) { return (k * kGdrThreads + (int)threadIdx.x) / per_row; }
    __device__ __forceinline__ static int col(int k) { return (k * kGdrThreads + (int)threadIdx.x) % per_row * 8; }
    __device__ __forceinline__ void fetch(const T *x, int64_t ld, int rows, int width) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int r = row(k), c = col(k);
#pragma unroll
            for (int i = 0; i < raw[k].W; ++i) raw[k].w[i] = 0;
            if (r >= rows) continue;
            const T *from = x + r * ld + c;
            if (c + 8 <= width) raw[k] = load<8>(from);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < width) put(raw[k], j, from[j]);
        }
    }
    // Into the tile; lengths (if asked for): of every row 1 / sqrt(sum of squares + eps), times `factor`; without eps `factor` alone.
    template <int P>
    __device__ __forceinline__ void place(const Tile<P, ROWS, COLS> &m, float *lengths, float eps, float factor) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            float v[8];
            unpack(raw[k], v);
            put8(m, row(k), col(k), raw[k], v);
            if (!lengths) continue;
            float sq = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sq = __builtin_fmaf(v[j], v[j], sq);
            sq += from_lane<0xb1>(sq);
            sq += from_lane<0x4e>(sq);
            sq += from_lane<0x141>(sq);
            if (per_row == 16) sq += from_lane<0x140>(sq);
            if (col(k) == 0) lengths[row(k)] = eps > 0.f ? factor / sqrtf(sq + eps) : factor;
        }
    }
};

// ---------------------------------------------------------------------------------------------------- chunks of sequences
struct GdrParams {
    const void *q, *k, *v;
    const float *decay, *beta, *s0;
    const int32_t *seq_start;
    void *y;
    float *s_last;
    char *saved;                // per chunk and head: what chunk_matrices leaves, and in training the states in front of it
    float *states;
    int64_t ldq, ldk, ldv, ldg, ldy, N;
    int32_t nseq, heads, group, dk, dv, blocks;         // group: heads of a key head; blocks: of columns of the states
    float scale, norm_eps;
};

// Sequence s: rows first .. end - 1, in the order of the buffers whatever the starts hold.
struct Span {
    int64_t first, end;
    __device__ __forceinline__ Span(const int32_t *starts, int s, int64_t N) : first(0), end(N) {
        if (!starts) return;
        end = min(max((int64_t)starts[s + 1], (int64_t)0), N);
        first = min(max((int64_t)starts[s], (int64_t)0), end);
    }
};

// The chunks of all sequences have places in one row: sequence s has the places from first / SIZE + s, one more than it needs at most, and there are
// N / SIZE + nseq in all.
template <int SIZE>
__device__ __forceinline__ int64_t place_of(const int32_t *starts, int s, int64_t N) {
    return Span(starts, s, N).first / SIZE + s;
}

// Which sequence place c belongs to.
template <int SIZE>
__device__ __forceinline__ int sequence_of(const int32_t *starts, int nseq, int64_t N, int64_t c) {
    int lo = 0, hi = nseq - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (place_of<SIZE>(starts, mid, N) <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// What is kept of a chunk for a head: the matrix M in parts, and the sums of the decays' logarithms in fp64.
template <typename T>
struct Saved {
    static constexpr int C = Gdr<T>::chunk, P = Gdr<T>::comp, matrix = P * C * C * 2, bytes = matrix + C * 8;
    char *at;
    __device__ __forceinline__ Saved(const GdrParams &p, int64_t place, int head) : at(p.saved + (place * p.heads + head) * bytes) {}
    __device__ __forceinline__ uint16_t *M() const { return reinterpret_cast<uint16_t *>(at); }
    __device__ __forceinline__ double *G() const { return reinterpret_cast<double *>(at + matrix); }
};

}  // namespace lm
}  // namespace grim
