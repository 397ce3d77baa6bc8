// What the losses over a vocabulary (lm_distill.hip, lm_policy.hip) share: 16-byte pieces of a row, and slices of rows that are cut.
#pragma once
#include "lm_common.hpp"

namespace grim {
namespace lm {

constexpr float kLn2 = 0.69314718055994530942f;

// elements of a piece
template <typename T>
constexpr int piece() { return 16 / (int)sizeof(T); }

// Elements lo .. hi - 1 of a gradient row: zeros, by all threads of the workgroup.
template <typename T>
__device__ __forceinline__ void zero_row(T *dz, int64_t lo, int64_t hi) {
    constexpr int V = piece<T>();
    const float none[V] = {};
    for (int64_t c = lo + (int64_t)threadIdx.x * V; c < hi; c += (int64_t)blockDim.x * V) {
        if (c + V <= hi) store(dz + c, none);
        else
            for (int j = 0; c + j < hi; ++j) dz[c + j] = (T)0.f;
    }
}

constexpr int kSliceWaves = 4, kSlicePer = 4;               // a slice: 4 pieces of 16 bytes a thread

template <typename T>
constexpr int64_t slice_elements() { return 64 * kSliceWaves * kSlicePer * piece<T>(); }

// The pieces of a slice [lo, hi), element by element at its end.
template <typename T>
struct Slice {
    static constexpr int V = piece<T>();
    Pack<T, V> raw[kSlicePer];
    int have[kSlicePer];
    __device__ __forceinline__ static int64_t at(int64_t lo, int k) { return lo + (int64_t)(k * 64 * kSliceWaves + threadIdx.x) * V; }
    __device__ __forceinline__ Slice(const T *z, int64_t lo, int64_t hi) {
#pragma unroll
        for (int k = 0; k < kSlicePer; ++k) {
            const int64_t c = at(lo, k), left = hi - c;
            have[k] = left >= V ? V : left > 0 ? (int)left : 0;
            if (have[k] == V) raw[k] = load<V>(z + c);
            else
#pragma unroll
                for (int j = 0; j < V; ++j) put(raw[k], j, j < have[k] ? z[c + j] : (T)-INFINITY);
        }
    }
};

template <typename T>
int64_t slices_of(int64_t V) { return (V + slice_elements<T>() - 1) / slice_elements<T>(); }

}  // namespace lm
}  // namespace grim
