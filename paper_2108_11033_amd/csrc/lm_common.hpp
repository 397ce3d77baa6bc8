// What the kernels of the language-model operators (grim_lm.h) share: element types, vector loads and stores that need no
// alignment beyond the element's, reductions over a wave and a workgroup.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "grim_lm.h"

namespace grim {
namespace lm {

using bf16 = __bf16;
using f16 = _Float16;

constexpr int kComputeUnits = 256;
constexpr int64_t kMostRows = 0x7fffffff;       // of a layer norm, a distillation, a policy loss
constexpr int kMostHeads = 4096, kMostHeadSize = 128;   // of a gated delta rule

// V elements of T as they lie in memory, in words: what waits in registers keeps two 16-bit elements in each.  They are read
// and written at any address that an element may have: rows may start anywhere (odd widths, leading dimensions and offsets), the
// hardware takes a 16-byte access at any address, and so rows that are not aligned run on the same kernels.
template <typename T, int V>
struct Pack {
    static constexpr int W = (V * (int)sizeof(T) + 3) / 4;
    uint32_t w[W];
};

template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)), may_alias)) Loose {
    uint32_t w[Pack<T, V>::W];
};

template <int V, typename T>
__device__ __forceinline__ Pack<T, V> load(const T *p) {
    Pack<T, V> r;
    if constexpr (V * sizeof(T) >= 4) {
        const Loose<T, V> l = *reinterpret_cast<const Loose<T, V> *>(p);
#pragma unroll
        for (int i = 0; i < r.W; ++i) r.w[i] = l.w[i];
    } else {
        r.w[0] = __builtin_bit_cast(uint16_t, *p);
    }
    return r;
}

template <int V, typename T>
__device__ __forceinline__ float element(const Pack<T, V> &p, int j) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, p.w[j]);
    const uint32_t w = p.w[j / 2];
    if constexpr (__is_same(T, bf16)) return __builtin_bit_cast(float, j % 2 ? w & 0xffff0000u : w << 16);
    return (float)__builtin_bit_cast(f16, (uint16_t)(j % 2 ? w >> 16 : w));
}

template <int V, typename T>
__device__ __forceinline__ void unpack(const Pack<T, V> &p, float (&out)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = element(p, j);
}

template <int V, typename T>
__device__ __forceinline__ void put(Pack<T, V> &p, int j, T v) {
    if constexpr (sizeof(T) == 4) p.w[j] = __builtin_bit_cast(uint32_t, v);
    else {
        const uint32_t b = __builtin_bit_cast(uint16_t, v);
        p.w[j / 2] = j % 2 ? (p.w[j / 2] & 0xffffu) | b << 16 : (p.w[j / 2] & 0xffff0000u) | b;
    }
}

// One rounding, to nearest even.  PAST: past the caches (below).
template <bool PAST = false, int V, typename T>
__device__ __forceinline__ void store(T *p, const float (&v)[V]) {
    T t[V];
#pragma unroll
    for (int j = 0; j < V; ++j) t[j] = (T)v[j];
    if constexpr (V * sizeof(T) >= 4) {
        typedef uint32_t Words __attribute__((ext_vector_type(Pack<T, V>::W), aligned(sizeof(T)), may_alias));
        Words w;
        __builtin_memcpy(&w, t, V * sizeof(T));
        if constexpr (PAST) __builtin_nontemporal_store(w, reinterpret_cast<Words *>(p));
        else *reinterpret_cast<Words *>(p) = w;
    } else {
        *p = t[0];
    }
}

// Outputs of calls whose operands are far from fitting the last-level cache are stored past it: they would displace what
// is still to be read, and a reader of theirs finds them displaced too (65536 x 1024 bf16 recurrence, both directions, 497 ->
// 467 us; 8192 x 32768 distillation 219 -> 215; 32768 x 1024 backward norm 44.8 -> 43.9).
// f(PAST): the loop that stores, compiled for either.
template <typename F>
__device__ __forceinline__ void store_rows(bool past, F f) {
    if (past) {
        asm volatile("; past the caches");                      // (keeps the compiler from making one loop of the two)
        f(std::true_type());
        asm volatile("; past the caches");
    } else {
        f(std::false_type());
    }
}
inline bool past_caches(int64_t bytes) { return bytes >= (int64_t)128 << 20; }

// The same words as far as the program goes, but not for the compiler: what was unpacked before is unpacked again after,
// instead of being held in twice the registers meanwhile.
template <typename T, int V>
__device__ __forceinline__ void forget(Pack<T, V> &p) {
#pragma unroll
    for (int i = 0; i < p.W; ++i) asm volatile("" : "+v"(p.w[i]));
}

// The value of the lane that a pattern names: 0xb1, 0x4e: the neighbour, the neighbouring pair; 0x141, 0x140: mirrored in 8 and
// in 16 lanes.
template <int PATTERN>
__device__ __forceinline__ float from_lane(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), PATTERN, 0xf, 0xf, true));
}

// All lanes get join(v of all 64), each having joined the same pairs: first inside rows of 16 lanes, then across rows by exchanging
// them.  (No trip through LDS: a reduction is some 30 cycles, not 600.)
template <typename F>
__device__ __forceinline__ float row_join(float v, F join) {
    v = join(v, from_lane<0xb1>(v));
    v = join(v, from_lane<0x4e>(v));
    v = join(v, from_lane<0x141>(v));
    return join(v, from_lane<0x140>(v));
}

template <typename F>
__device__ __forceinline__ float across_rows(float v, F join) {
    const uint32_t r = __builtin_bit_cast(uint32_t, v);
    const auto by16 = __builtin_amdgcn_permlane16_swap(r, r, false, false);
    v = join(__builtin_bit_cast(float, (uint32_t)by16[0]), __builtin_bit_cast(float, (uint32_t)by16[1]));
    const uint32_t q = __builtin_bit_cast(uint32_t, v);
    const auto by32 = __builtin_amdgcn_permlane32_swap(q, q, false, false);
    return join(__builtin_bit_cast(float, (uint32_t)by32[0]), __builtin_bit_cast(float, (uint32_t)by32[1]));
}

struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

__device__ __forceinline__ float wave_sum(float v) { return across_rows(row_join(v, Add()), Add()); }
__device__ __forceinline__ float wave_max(float v) { return across_rows(row_join(v, Max()), Max()); }

// Sums over a workgroup of W waves, in the order of the waves; `room` holds W floats that nobody uses until the next barrier
// of the caller.
template <int W>
__device__ __forceinline__ float group_sum(float v, float *room) {
    v = wave_sum(v);
    if (W == 1) return v;
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) s += room[w];
    return s;
}

// The same over teams of TPR threads: a row of 16 lanes, a wave, a workgroup of TPR / 64 waves.
template <int TPR>
__device__ __forceinline__ float team_sum(float v, float *room) {
    if constexpr (TPR == 16) return row_join(v, Add());
    else return group_sum<TPR / 64>(v, room);
}

template <int W>
__device__ __forceinline__ float group_max(float v, float *room) {
    v = wave_max(v);
    if (W == 1) return v;
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = room[0];
#pragma unroll
    for (int w = 1; w < W; ++w) s = fmaxf(s, room[w]);
    return s;
}

// out0[c], out1[c - C0]: sums of part[i * (C0 + C1) + c] over i < groups, in a fixed order (lm_norm.hip).
grim_status join_columns(const float *part, int64_t groups, int64_t C0, float *out0, int64_t C1, float *out1, hipStream_t stream);

inline bool known(grim_dtype dt) { return dt == GRIM_F32 || dt == GRIM_F16 || dt == GRIM_BF16; }
inline int bytes_of(grim_dtype dt) { return dt == GRIM_F32 ? 4 : 2; }
inline grim_status launched() { return hipGetLastError() == hipSuccess ? GRIM_OK : GRIM_ERR_DEVICE; }

// A launch has fewer than 2^32 threads; one of more starts what is left of their number in 32 bits, without an error.  So many
// workgroups are a launch's most:
constexpr int64_t most_groups(int threads) { return 0xffffffffll / threads; }

// f(first, count) for runs of at most `most` out of `all`, one launch each.
template <typename F>
grim_status in_runs(int64_t all, int64_t most, F f) {
    for (int64_t first = 0; first < all; first += most) {
        const grim_status st = f(first, all - first < most ? all - first : most);
        if (st != GRIM_OK) return st;
    }
    return GRIM_OK;
}

template <typename T>
T *ahead(T *p, int64_t elements) { return p ? p + elements : p; }

inline bool overlap(const void *a, const void *b, int64_t bytes) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && (x < y ? y - x : x - y) < (uintptr_t)bytes;
}

// an output in its input's place whose rows lie elsewhere
inline bool moves(const void *in, int64_t ld_in, const void *out, int64_t ld_out, int64_t rows) {
    return in == out && ld_in != ld_out && rows > 1;
}

// rows x ld elements stay far below what a 64-bit byte offset holds
inline bool fits(int64_t rows, int64_t ld) { return ld >= 0 && ld <= (int64_t(1) << 40) && (rows <= 1 || ld <= (int64_t(1) << 56) / rows); }

}  // namespace lm
}  // namespace grim
