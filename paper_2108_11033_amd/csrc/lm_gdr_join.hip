// From run to run of a gated delta rule's sequences: S_(r + 1) = A_r S_r + B_r, and dS_(r - 1) = A_r' dS_r + B_r.
//
// A_r and B_r were formed for all runs at once; what is left is a chain of products of dk x dk matrices with a head's states, as long as a sequence has runs.  A wave has 16 columns of
// the states in registers; A comes through LDS, the next one on its way meanwhile.
#include "lm_gdr.hpp"

namespace grim {
namespace lm {

template <typename T, int DK, bool BACK>
__global__ void __launch_bounds__(256) join_kernel(GdrParams p) {
    constexpr int PC = Gdr<T>::comp, DT = DK / 16, DS = DK / 32;
    using Map = Tile<PC, DK, DK, BACK ? TURNED : PAIRED>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const Map A{reinterpret_cast<uint16_t *>(lds)};
    const uint32_t blocks = (p.tiles + 3) / 4, heads = (uint32_t)p.heads;
    const int block = (int)(blockIdx.x % blocks), h = (int)(blockIdx.x / blocks % heads), s = (int)(blockIdx.x / blocks / heads);
    const Span span(p.seq_start, s, p.N);
    const uint32_t run0 = place_of(span, s, p.size);
    const int runs = (int)((span.end - span.first + p.size - 1) / p.size);
    if (runs < 3) return;                                   // (the first step was made where the maps were formed)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tile = block * 4 + wave, own = (lane & 15) * 16 + (lane >> 4) * 4;
    const bool idle = tile >= p.tiles;
    // the states in front of run r (BACK: their gradient behind it)
    const auto at = [&](int r) { return p.starts + (((int64_t)(run0 + r) * p.heads + h) * p.tiles + (idle ? 0 : tile)) * DT * 256 + own; };
    const auto map = [&](int r) { return p.maps + ((int64_t)(run0 + r) * p.heads + h) * DK * DK; };
    // forward: runs 1 .. runs - 2 take the states in front of them to those in front of the next; back: runs - 2 .. 1
    const int step = BACK ? -1 : 1;
    int r = BACK ? runs - 2 : 1;
    f32x4 state[DT];
#pragma unroll
    for (int n = 0; n < DT; ++n) state[n] = *reinterpret_cast<const f32x4 *>(at(r) + n * 256);
    Rows<true, float, 256, DK, DK> next;
    next.fetch(map(r), DK, DK, DK);
    for (int left = runs - 2; left > 0; --left, r += step) {
        next.place(A, DK, DK);
        if (left > 1) next.fetch(map(r + step), DK, DK, DK);
        f32x4 sum[DT];
#pragma unroll
        for (int n = 0; n < DT; ++n) sum[n] = *reinterpret_cast<const f32x4 *>(at(r + step) + n * 256);
        __syncthreads();
        if (!idle) {
            Frag<PC> S[DS];
#pragma unroll
            for (int d = 0; d < DS; ++d) S[d] = operand<PC>(state[2 * d], state[2 * d + 1]);
#pragma unroll
            for (int n = 0; n < DT; ++n) {
#pragma unroll
                for (int d = 0; d < DS; ++d) sum[n] = multiply(BACK ? across(A, 16 * n, 32 * d) : along(A, 16 * n, 32 * d), S[d], sum[n]);
                state[n] = sum[n];
                *reinterpret_cast<f32x4 *>(at(r + step) + n * 256) = sum[n];
            }
        }
        __syncthreads();
    }
}

template <typename T, int DK, bool BACK>
grim_status join_runs(const GdrParams &p, hipStream_t stream) {
    constexpr int bytes = Tile<Gdr<T>::comp, DK, DK, BACK ? TURNED : PAIRED>::bytes;
    const auto kernel = join_kernel<T, DK, BACK>;
    static const hipError_t grown = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (grown != hipSuccess) return GRIM_ERR_DEVICE;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)p.nseq * p.heads * ((p.tiles + 3) / 4))), dim3(256), bytes, stream, p);
    return launched();
}

#define JOIN(T)                                                              \
    template grim_status join_runs<T, 64, false>(const GdrParams &, hipStream_t);  \
    template grim_status join_runs<T, 64, true>(const GdrParams &, hipStream_t);   \
    template grim_status join_runs<T, 128, false>(const GdrParams &, hipStream_t); \
    template grim_status join_runs<T, 128, true>(const GdrParams &, hipStream_t);
JOIN(float)
JOIN(f16)
JOIN(bf16)

}  // namespace lm
}  // namespace grim
