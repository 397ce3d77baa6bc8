// What the kernels of the gated delta rule share: matrices in LDS as sums of bf16 parts, products of them, chunks of packed sequences.
//
// A number is held as the sum of up to three bf16 parts, each the rounding of what the parts before it leave: three are off by 2^-25 of the number or less.  The product of two
// numbers takes the parts' products whose numbers add up to two or less, summed in fp32 by the matrix cores: 2^-24 or so, as fp32 itself.  Operands
// that come as bf16 are one part, fp16 two, fp32 three, all exact but the last; what is computed between products (states, differences) is three.
// (Two parts for it would be off by 2^-17, which outputs of 16 bits hide but the states and the gates' gradients do not: those were 1e-6 to 6e-6 off in the 2-norm, and are 6e-8 to 4e-7
// with three.  What that costs: 32768 tokens x 8 heads of 128 x 128 in bf16, both directions, 1077 -> 1262 us.  The fp32 matrix instruction does a sixteenth of the work of the bf16 one.)
#pragma once
#include <atomic>

#include "lm_common.hpp"

namespace grim {
namespace lm {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Gdr;
// data: parts of an operand; comp: of what is computed; chunk: tokens that the matrix form takes at a time (fewer in fp32, whose products take up to three times as long)
template <>
struct Gdr<bf16> { static constexpr int data = 1, comp = 3, chunk = 64; };
template <>
struct Gdr<f16> { static constexpr int data = 2, comp = 3, chunk = 64; };
template <>
struct Gdr<float> { static constexpr int data = 3, comp = 3, chunk = 32; };

constexpr int kMatrixThreads = 256;            // of the kernel that forms the chunks' matrices
constexpr double kLeastDecay = -10000.;

// ---------------------------------------------------------------------------------------------------- matrices in LDS
// Sums run over 32 elements at a time.  A lane of the first operand holds 8 elements of row lane % 16, of the second 8 of column lane % 16; a result's lane
// has rows (lane / 16) 4 .. + 3 at column lane % 16.  Which 8 of the 32 a lane holds is free as long as both operands agree: here elements 4 g .. 4 g + 3 and
// 16 + 4 g .. 16 + 4 g + 3, g = lane / 16.  That is what two results of 16 rows above one another leave in a lane, so that a result is the
// next product's operand (first or second) as it stands, without a way through LDS.
template <int P>
struct Frag { s16x8 part[P]; };

// P parts of ROWS x COLS.  Rows are longer than their elements, so that the rows that one access reads lie in different banks.  Measured, in clocks per access of a
// compute unit of which 8-byte accesses take 1.85 and 16-byte ones 3 at best: rows of 36 or 76 words 8 bytes along the rows 1.85 (40, 72 words 3), transposing reads 3 (40, 72 words 1.85);
// 16 bytes along the rows (PAIRED: columns stored in the order that a lane reads them in, 32 m + 16 h + 4 g + r at 32 m + 8 g + 4 h + r) 6 with rows of 36 words, 3 of 40 and 72.
// TURNED: the longer rows with the columns in their own order, for tiles that only transposing reads read.
enum Order { PLAIN, PAIRED, TURNED };
template <int P, int ROWS, int COLS, int ORDER = PLAIN>
struct Tile {
    static constexpr int parts = P, ld = COLS == 128 ? (ORDER ? 144 : 152) : COLS == 64 ? (ORDER ? 80 : 72) : 40, part = ROWS * ld, bytes = P * part * 2;
    uint16_t *at;
};

__device__ __forceinline__ s16x8 both(s16x4 lo, s16x4 hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }

__device__ __forceinline__ int paired(int c) { return (c & ~31) + 8 * (c >> 2 & 3) + 4 * (c >> 4 & 1) + (c & 3); }

// 16 rows from r, as an operand whose sum runs along them, over elements k .. k + 31.
template <int P, int R, int C, int ORDER>
__device__ __forceinline__ Frag<P> along(const Tile<P, R, C, ORDER> &m, int r, int k) {
    const int lane = threadIdx.x & 63;
    Frag<P> f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const uint16_t *from = m.at + p * m.part + (r + (lane & 15)) * m.ld + k + (lane >> 4) * (ORDER == PAIRED ? 8 : 4);
        if (ORDER == PAIRED) f.part[p] = *reinterpret_cast<const s16x8 *>(from);
        else f.part[p] = both(*reinterpret_cast<const s16x4 *>(from), *reinterpret_cast<const s16x4 *>(from + 16));
    }
    return f;
}

// Four rows from r + (lane / 16) 4 at column c + lane % 16: the transposing read of 16 bits.
__device__ __forceinline__ s16x4 turned(const uint16_t *at, int ld, int r, int c) {
    const int lane = threadIdx.x & 63, j = lane & 15;
    uint16_t *from = const_cast<uint16_t *>(at) + (r + (lane >> 4) * 4 + j / 4) * ld + c + (j % 4) * 4;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)from);
}

// 16 columns from c (as they are stored), as an operand whose sum runs over rows k .. k + 31.
template <int P, int R, int C, int ORDER>
__device__ __forceinline__ Frag<P> across(const Tile<P, R, C, ORDER> &m, int c, int k) {
    Frag<P> f;
#pragma unroll
    for (int p = 0; p < P; ++p) f.part[p] = both(turned(m.at + p * m.part, m.ld, k, c), turned(m.at + p * m.part, m.ld, k + 16, c));
    return f;
}

// (lo, hi) rounded to bf16, in one word; what is left of them.  (Not by inline asm: the compiler keeps the matrix instructions' results from being read too early
// only where it knows the reader.)
__device__ __forceinline__ uint32_t round2(float lo, float hi) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), b16x2));
}
template <int V>
__device__ __forceinline__ void round_off(float (&v)[V], uint32_t (&w)[V / 2], bool more) {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
        w[j] = round2(v[2 * j], v[2 * j + 1]);
        if (more) v[2 * j] -= __builtin_bit_cast(float, w[j] << 16), v[2 * j + 1] -= __builtin_bit_cast(float, w[j] & 0xffff0000u);
    }
}

// Two results above one another, as the operand of a sum over their rows.
template <int P>
__device__ __forceinline__ Frag<P> operand(f32x4 lo, f32x4 hi) {
    Frag<P> f;
    float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
    for (int p = 0; p < P; ++p) {
        uint32_t w[4];
        round_off(v, w, p + 1 < P);
        __builtin_memcpy(&f.part[p], w, 16);
    }
    return f;
}

// acc + the 16 x 16 product, small terms first.
template <int PA, int PB>
__device__ __forceinline__ f32x4 multiply(const Frag<PA> &a, const Frag<PB> &b, f32x4 acc) {
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (s - i >= 0 && s - i < PB)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a.part[i]), __builtin_bit_cast(b16x8, b.part[s - i]), acc, 0, 0, 0);
    return acc;
}

// Elements c .. c + 3 of row r.
template <int P, int R, int C, int ORDER>
__device__ __forceinline__ void put4(const Tile<P, R, C, ORDER> &m, int r, int c, f32x4 v) {
    if (ORDER == PAIRED) c = paired(c);
    float t[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
    for (int p = 0; p < P; ++p) {
        uint32_t w[2];
        round_off(t, w, p + 1 < P);
        s16x4 o;
        __builtin_memcpy(&o, w, 8);
        *reinterpret_cast<s16x4 *>(m.at + p * m.part + r * m.ld + c) = o;
    }
}

// Elements c .. c + 7, c a multiple of 8.
template <int P, int R, int C, int ORDER>
__device__ __forceinline__ void put8(const Tile<P, R, C, ORDER> &m, int r, int c, s16x8 v, int p = 0) {
    uint16_t *to = m.at + p * m.part + r * m.ld;
    if (ORDER == PAIRED) {
        *reinterpret_cast<s16x4 *>(to + paired(c)) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
        *reinterpret_cast<s16x4 *>(to + paired(c) + 8) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
    } else {
        *reinterpret_cast<s16x8 *>(to + c) = v;
    }
}
template <int P, int R, int C, int ORDER>
__device__ __forceinline__ void put8(const Tile<P, R, C, ORDER> &m, int r, int c, float (&v)[8]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        uint32_t h[4];
        round_off(v, h, p + 1 < P);
        s16x8 w;
        __builtin_memcpy(&w, h, 16);
        put8(m, r, c, w, p);
    }
}

// C x C of which the products of chunks need the blocks of 32 x 32 on the diagonal and (C = 64) one beside it: below (UPPER: above) the diagonal.
template <int P, int C, int ORDER, bool UPPER = false>
struct Triangle {
    static constexpr int elements = C * 32 + (C - 32) * 32, bytes = Tile<P, C, 32, ORDER>::bytes + (C > 32 ? Tile<P, 32, 32, ORDER>::bytes : 0);
    Tile<P, C, 32, ORDER> tall;                             // columns 0 .. 31 of all rows (UPPER: the last 32)
    Tile<P, 32, 32, ORDER> rest;                            // the other diagonal block
    __device__ __forceinline__ void put(char *at) {
        tall.at = reinterpret_cast<uint16_t *>(at), rest.at = reinterpret_cast<uint16_t *>(at + Tile<P, C, 32, ORDER>::bytes);
    }
    // Where the n-th 8 elements of what is kept go (not UPPER).
    __device__ __forceinline__ uint16_t *piece(int n) const {
        const int p = n / (elements / 8), q = n % (elements / 8), r = q / 4, c = q % 4 * 8;
        return r < C ? tall.at + p * tall.part + r * tall.ld + c : rest.at + p * rest.part + (r - C) * rest.ld + c;
    }
    __device__ __forceinline__ static constexpr bool is_tall(int c) { return UPPER ? c >= C - 32 : c < 32; }
    __device__ __forceinline__ static constexpr int row(int r) { return UPPER ? r : r - 32; }       // of the rest
};
template <int P, int C, int ORDER, bool UPPER>
__device__ __forceinline__ Frag<P> along(const Triangle<P, C, ORDER, UPPER> &m, int r, int k) {
    return m.is_tall(k) ? along(m.tall, r, 0) : along(m.rest, m.row(r), 0);
}
template <int P, int C, int ORDER, bool UPPER>
__device__ __forceinline__ Frag<P> across(const Triangle<P, C, ORDER, UPPER> &m, int c, int k) {
    return m.is_tall(c) ? across(m.tall, c % 32, k) : across(m.rest, c % 32, m.row(k));
}
template <int P, int C, int ORDER, bool UPPER>
__device__ __forceinline__ void put4(const Triangle<P, C, ORDER, UPPER> &m, int r, int c, f32x4 v) {
    if (m.is_tall(__builtin_amdgcn_readfirstlane(c))) put4(m.tall, r, c % 32, v);         // (the same for all lanes)
    else put4(m.rest, m.row(r), c % 32, v);
}

// V elements from column c of a row of `width` (which may end inside them, or before) without a branch, so that loads do not wait for each other: those that end with the row,
// which settle() moves to their places when they have come.  WHOLE: the width is a multiple of V.
template <bool WHOLE, int V, typename T>
__device__ __forceinline__ Pack<T, V> reach(const T *row, int c, int width) {
    if (WHOLE || width >= V) return load<V>(row + max(0, min(c, width - V)));
    Pack<T, V> r = {};
#pragma unroll
    for (int j = 0; j < V; ++j) put(r, j, row[min(c + j, width - 1)]);
    return r;
}
template <bool WHOLE, int V, typename T>
__device__ __forceinline__ void settle(const Pack<T, V> &raw, int c, int width, bool there, float (&v)[V]) {
    unpack(raw, v);
    if (WHOLE) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = there && c < width ? v[j] : 0.f;
        return;
    }
    const int n = width >= V ? c - max(0, min(c, width - V)) : 0;
#pragma unroll
    for (int by = 1; by < V; by *= 2)
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = n & by ? (j + by < V ? v[j + by] : 0.f) : v[j];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = there && c + j < width ? v[j] : 0.f;
}

// Elements c .. c + 3 of a row of `width`.
template <bool WHOLE, typename T>
__device__ __forceinline__ void leave(T *row, int c, int width, f32x4 v) {
    if (c + 4 <= width) {
        const float t[4] = {v[0], v[1], v[2], v[3]};
        store(row + c, t);
    } else if (!WHOLE) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < width) row[c + j] = (T)v[j];
    }
}

// Rows of keys or queries on their way to LDS: COLS elements in pieces of 8, dealt to the workgroup's threads; zeros behind the head's
// width and the last row.
template <bool WHOLE, typename T, int THREADS, int ROWS, int COLS>
struct Rows {
    static constexpr int per_row = COLS / 8, PER = (ROWS * per_row + THREADS - 1) / THREADS;
    static constexpr bool even = PER * THREADS == ROWS * per_row;       // else some threads have a piece less
    Pack<T, 8> raw[PER];
    __device__ __forceinline__ static int row(int k) { return (k * THREADS + (int)threadIdx.x) / per_row; }
    __device__ __forceinline__ static int col(int k) { return (k * THREADS + (int)threadIdx.x) % per_row * 8; }
    __device__ __forceinline__ void fetch(const T *x, int64_t ld, int rows, int width) {
#pragma unroll
        for (int k = 0; k < PER; ++k) raw[k] = reach<WHOLE, 8>(x + min(row(k), rows - 1) * ld, col(k), width);
    }
    // Into the tile.
    template <int P, int ORDER>
    __device__ __forceinline__ void place(const Tile<P, ROWS, COLS, ORDER> &m, int rows, int width) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int r = row(k), c = col(k);
            if (!even && r >= ROWS) continue;
            if constexpr (WHOLE && P == 1) {
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = r < rows && c < width ? raw[k].w[i] : 0u;
                put8(m, r, c, __builtin_bit_cast(s16x8, w));
            } else {
                float v[8];
                settle<WHOLE>(raw[k], c, width, r < rows, v);
                put8(m, r, c, v);
            }
        }
    }
    // As they are, to rows of ld elements.
    __device__ __forceinline__ void keep(T *to, int ld, int rows, int width) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int r = row(k), c = col(k);
            if (!even && r >= ROWS) continue;
            if constexpr (WHOLE) {
#pragma unroll
                for (int i = 0; i < raw[k].W; i += 4) {
                    u32x4 w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = r < rows && c < width ? raw[k].w[i + j] : 0u;
                    __builtin_memcpy(to + r * ld + c + i * 4 / (int)sizeof(T), &w, 16);
                }
            } else {
                float v[8];
                settle<WHOLE>(raw[k], c, width, r < rows, v);
                T t[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = (T)v[j];
                __builtin_memcpy(to + r * ld + c, t, sizeof(t));
            }
        }
    }
    // Of every row factor / sqrt(sum of squares + eps), without eps `factor` alone; to be called by all lanes.
    __device__ __forceinline__ void lengths(int rows, int width, float *to, float eps, float factor) {
        static_assert(even, "whole pieces");
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            float v[8], sq = 0.f;
            settle<WHOLE>(raw[k], col(k), width, row(k) < rows, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) sq = __builtin_fmaf(v[j], v[j], sq);
            sq += from_lane<0xb1>(sq);
            sq += from_lane<0x4e>(sq);
            sq += from_lane<0x141>(sq);
            if (per_row == 16) sq += from_lane<0x140>(sq);
            if (col(k) == 0) to[row(k)] = eps > 0.f ? factor / sqrtf(sq + eps) : factor;
        }
    }
};

// ---------------------------------------------------------------------------------------------------- chunks of sequences
// Matrices that are kept (states, their gradients, E and its) lie in tiles of 16 x 16, a column's 16 rows one after another: a lane's four in one access.
struct GdrParams {
    const void *q, *k, *v;
    const float *decay, *beta, *s0;
    const int32_t *seq_start;
    void *y;
    float *s_last;
    char *saved;                // per chunk and head: what chunk_matrices leaves
    float *states, *E;          // for the backward pass, per chunk and head: the states in front of it, and E; or NULL
    float *starts;              // per run and head: the states in front of it (of a sequence's first run: not used)
    float *maps;                // per run and head: dk x dk, what the run makes of the states in front of it, less what it adds
    int64_t ldq, ldk, ldv, ldg, ldy, N;
    uint32_t size;              // tokens of a run
    int32_t nseq, heads, group, dk, dv, tiles;          // group: heads of a key head; tiles: of 16 columns of the states
    float scale, norm_eps;
};

// Of the backward pass; p.starts are the gradients of the states behind the runs.
struct GdrBack {
    GdrParams p;
    const void *dy;
    const float *ds_last;
    void *dq, *dk, *dv;
    float *ddecay, *dbeta, *ds0;
    float *A, *F;               // per chunk and head: the gradient of the states behind it, and of U over what later tokens make of it (lm_gdr_back.hip)
    int64_t lddy, lddq, lddk, lddv, lddg;
    int32_t key_heads;
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

// The chunks (or runs of chunks, of `size` tokens) of all sequences have places in one row: sequence s has the places from first / size + s, one more than it needs at
// most, and there are N / size + nseq in all.  (N is at most 2^30: 32-bit divisions.)
__device__ __forceinline__ uint32_t place_of(const Span &span, int s, uint32_t size) { return (uint32_t)span.first / size + s; }

// Which sequence a place belongs to: 64 lanes look at once, so that up to 64 sequences cost one wait for memory, 4096 two.
__device__ __forceinline__ int sequence_of(const int32_t *starts, int nseq, int64_t N, uint32_t size, uint32_t place) {
    int lo = 0, left = nseq;
    while (left > 1) {
        const int step = (left + 63) / 64, at = lo + (int)(threadIdx.x & 63) * step, in = at < lo + left;
        const bool before = in && place_of(Span(starts, in ? at : lo, N), at, size) <= place;
        const int n = __builtin_popcountll(__ballot(before));          // (in ascending order: the first ones)
        const int next = lo + (n > 0 ? n - 1 : 0) * step;
        left = min(step, lo + left - next);
        lo = __builtin_amdgcn_readfirstlane(next);
        left = __builtin_amdgcn_readfirstlane(left);
    }
    return lo;
}

// What is kept of a chunk for a head: the matrix M in parts, columns paired, the blocks of Triangle one after another; the running sums of the decays' base-2 logarithms in fp64; and of every token, with r the
// factors that its key and its query count with, beta (0 behind the last one), the decay since the chunk's start times r_k, the decay until its end times r_k, the
// decay since its start times r_q, r_k, r_q.
template <typename T>
struct Saved {
    static constexpr int C = Gdr<T>::chunk, P = Gdr<T>::comp, part = C * 32 + (C - 32) * 32, matrix = P * part * 2, bytes = matrix + C * 32;
    char *at;
    __device__ __forceinline__ Saved(const GdrParams &p, int64_t place, int head) : at(p.saved + (place * p.heads + head) * bytes) {}
    __device__ __forceinline__ uint16_t *M() const { return reinterpret_cast<uint16_t *>(at); }
    __device__ __forceinline__ double *G() const { return reinterpret_cast<double *>(at + matrix); }
    __device__ __forceinline__ float *tokens() const { return reinterpret_cast<float *>(at + matrix + C * 8); }
};

// Values in LDS as they come; what a lane of a 16 x 16 result takes of them.
template <typename T, int ROWS, int COLS>
struct Values {
    static constexpr int ld = sizeof(T) == 4 ? COLS + 4 : COLS == 128 ? 144 : COLS + 8, bytes = ROWS * ld * (int)sizeof(T);
    T *at;
    __device__ __forceinline__ f32x4 get(int r, int c) const {
        f32x4 v;
        if constexpr (sizeof(T) == 4) {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = at[(r + (lane >> 4) * 4 + e) * ld + c + (lane & 15)];
        } else {
            const s16x4 w = turned(reinterpret_cast<const uint16_t *>(at), ld, r, c);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (float)__builtin_bit_cast(T, (uint16_t)w[e]);
        }
        return v;
    }
};

// The decay between two places of a chunk.  (The argument's rounding is 2^-24 of it: 8e-7 of a decay to a millionth, less nearer by.)
__device__ __forceinline__ float decay_of(double from_to) { return __builtin_amdgcn_exp2f((float)from_to); }

// The 16 x 16 of a chunk's lower triangle that sums over 32 tokens read (all of a 32 x 32 block on the diagonal).
template <int C>
struct Lower {
    static constexpr int count = C == 64 ? 12 : 4;
    __device__ __forceinline__ static void get(int n, int &row, int &col) { row = n < 4 ? n / 2 : 2 + (n - 4) / 4, col = n < 4 ? n % 2 : (n - 4) % 4; }
};

template <typename T>
int64_t places_of(int64_t N, int32_t nseq) { return N / Gdr<T>::chunk + nseq; }

inline int padded(int dk) { return dk <= 64 ? 64 : 128; }
inline int tiles_of(int dv) { return (dv + 15) / 16; }

inline bool gdr_shape(int64_t N, int32_t nseq, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv) {
    return N >= 0 && N <= (int64_t)1 << 30 && nseq >= 1 && heads >= 1 && heads <= kMostHeads && key_heads >= 1 && heads % key_heads == 0 && dk >= 1 && dv >= 1;
}

inline grim_status gdr_check(int64_t N, int32_t nseq, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv) {
    if (!gdr_shape(N, nseq, heads, key_heads, dk, dv)) return GRIM_ERR_SHAPE;
    // (a launch has fewer than 2^32 threads: of a run 4 workgroups of 256 or one of 512, of a sequence that is long enough for the join, one of 5 chunks, 8 of 512)
    return dk > kMostHeadSize || dv > kMostHeadSize || (N / 32 + nseq) * heads > (int64_t)1 << 21 ? GRIM_ERR_UNSUPPORTED : GRIM_OK;
}
// (the lengths' squares, factors of queries and their reciprocals stay far from the ends of fp32)
inline bool gdr_factors(float scale, float eps) {
    return (scale == 0.f || (fabsf(scale) >= 1e-30f && fabsf(scale) <= 1e30f)) && (eps == 0.f || (eps >= 1e-16f && eps <= 1e30f));
}
inline grim_status gdr_check(grim_dtype dt, int64_t N, int32_t nseq, bool starts, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv, float scale, float eps) {
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if ((nseq > 1 && !starts) || !gdr_factors(scale, eps)) return GRIM_ERR_SHAPE;
    return gdr_check(N, nseq, heads, key_heads, dk, dv);
}

// Tokens of a run.  Over runs of s chunks a head of n chunks costs 2 s chunks (what a run does to the states has to be formed first) and n / s steps of the join instead of n chunks,
// some 5 us each where a step is 1.5 to 2: s is the root of n / 8, or what runs that fill the compute units once (twice where two workgroups share one) come to.  One sequence
// and 4 heads of 64 x 64 in bf16, runs of 2, 4, 8 chunks: 1024 tokens 38, 48, 70 us, 4096 63, 61, 79, 32768 213, 213, 173 (without runs some 5 us a chunk).  The lengths lie on the
// GPU, so that the mean stands for all of them: a long sequence among many short ones is walked chunk after chunk (32749 tokens in 256 sequences, one of 30000, 8 heads of 128 x 128 in bf16,
// both directions, 8.6 ms; the 30000 alone 1.2).
template <typename T>
uint32_t run_of(int64_t N, int32_t nseq, int32_t heads, int32_t dv) {
    constexpr int64_t C = Gdr<T>::chunk;
    const int64_t mean = N / nseq / C, each = (int64_t)heads * ((tiles_of(dv) + 7) / 8), runs = (tiles_of(dv) > 4 ? 1 : 2) * kComputeUnits / each;
    if (runs < 2 || mean < 4) return (uint32_t)1 << 31;
    int64_t size = 2;
    while (size * size * 8 < mean) ++size;
    // (every sequence but one may end in a part of a run: counted, unless there are so many that they take several turns anyway.  16384 tokens in 4, 8 heads of 128 x 128 in fp16, both
    // directions: 1017 -> 871 us)
    const int64_t whole = runs - (nseq - 1) >= runs / 2 ? runs - (nseq - 1) : runs, fill = ((N + whole - 1) / whole + C - 1) / C;
    return (uint32_t)((size > fill ? size : fill) * C);
}
inline int64_t runs_of(int64_t N, int32_t nseq, uint32_t size) { return N / size + nseq; }

// Bytes of what a call keeps, section by section: of the chunks their matrices, the states in front of them and E (or their gradients, and E's); of the runs their maps, and
// the states in front of them (or the gradients behind them).
template <typename T>
struct GdrRoom {
    int64_t saved, maps, states, E, starts;
    GdrRoom(int64_t N, int32_t nseq, int32_t heads, int32_t dk, int32_t dv) {
        const int64_t places = places_of<T>(N, nseq) * heads, d = padded(dk), columns = 16 * tiles_of(dv);
        const uint32_t size = run_of<T>(N, nseq, heads, dv);
        const int64_t runs = size < N ? runs_of(N, nseq, size) * heads : 0;
        saved = places * Saved<T>::bytes, states = places * columns * d * 4, E = places * columns * Gdr<T>::chunk * 4;
        maps = runs * d * d * 4, starts = runs * columns * d * 4;
    }
    int64_t kept() const { return saved + maps + states + E; }
    int64_t scratch() const {                               // forward without keeping, or backward
        const int64_t forward = saved + maps + starts, backward = starts + states + E;
        return forward > backward ? forward : backward;
    }
};

// S_(r + 1) = A_r S_r + B_r from run to run of every sequence and head; BACK: the gradients, the other way through the transposed maps (lm_gdr_join.hip).
template <typename T, int DK, bool BACK>
grim_status join_runs(const GdrParams &p, hipStream_t stream);

// Raises a kernel's LDS limit, once per process.
inline bool lds_of(const void *kernel, int bytes, std::atomic<bool> &grown) {
    if (grown) return true;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    return grown = true;
}

// The gradients of queries, keys, decays and betas from what the chunks left (lm_gdr_grad.hip).
template <typename T, int DK, bool WHOLE>
grim_status gdr_gradients(const GdrBack &b, hipStream_t stream);

}  // namespace lm
}  // namespace grim
