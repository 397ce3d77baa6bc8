// From run to run of a gated delta rule's sequences: S_(r + 1) = A_r S_r + B_r, and dS_(r - 1) = A_r' dS_r + B_r.
//
// A_r and B_r were formed for all runs at once; what is left is a chain of products of dk x dk matrices with a head's states, as long as a sequence has runs: what counts is the
// time of a step.  A workgroup takes 16 columns of the states; each of its waves has 16 rows of A, in registers two steps ahead, and leaves its 16 rows of the result in
// LDS as parts of the next step's operand, which all waves read after one barrier (two places in turn).
// A step is 2.1 us for 128 x 128 maps (64 KB that each compute unit fetches at some 31 GB/s), 0.75 to 1.5 for 64 x 64; 30 steps of 8 heads 66 us.
#include "lm_gdr.hpp"

namespace grim {
namespace lm {

template <typename T, int DK, bool BACK>
__global__ void __launch_bounds__(DK * 4) join_kernel(GdrParams p) {
    constexpr int PC = Gdr<T>::comp, DT = DK / 16, DS = DK / 32;
    __shared__ s16x8 operands[2][DS][PC][64];
    // (the workgroups that read the same maps are a multiple of the heads apart: with 8 heads or a multiple they share an L2)
    const uint32_t heads = (uint32_t)p.heads, chains = heads * (uint32_t)p.nseq, chain = blockIdx.x % chains;
    const int tile = (int)(blockIdx.x / chains), h = (int)(chain % heads), s = (int)(chain / heads);
    const Span span(p.seq_start, s, p.N);
    const uint32_t run0 = place_of(span, s, p.size);
    const int runs = (int)((span.end - span.first + p.size - 1) / p.size);
    if (runs < 3) return;                                   // (the first step was made where the maps were formed)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15, g4 = (lane >> 4) * 4;
    const uint32_t own = l15 * 16 + g4;
    // the states in front of run r (BACK: their gradient behind it), this wave's rows
    const auto at = [&](int r) { return p.starts + ((((int64_t)(run0 + r) * p.heads + h) * p.tiles + tile) * DT + wave) * 256; };
    const auto map = [&](int r) { return p.maps + ((int64_t)(run0 + r) * p.heads + h) * DK * DK; };
    // forward: runs 1 .. runs - 2 take the states in front of them to those in front of the next; back: runs - 2 .. 1
    const int step = BACK ? -1 : 1;
    int r = BACK ? runs - 2 : 1;
    struct Next {
        f32x4 A[2 * DS], B;
    } next[2];
    const auto fetch = [&](Next &n, int r) {
        const float *a = map(r) + (BACK ? 16 * wave : 16 * wave * DK);
#pragma unroll
        for (int i = 0; i < 2 * DS; ++i) {
            if (BACK) {
#pragma unroll
                for (int e = 0; e < 4; ++e) n.A[i][e] = a[(uint32_t)((16 * i + g4 + e) * DK + l15)];
            } else {
                n.A[i] = *reinterpret_cast<const f32x4 *>(a + (uint32_t)(l15 * DK + 16 * i + g4));
            }
        }
        n.B = *reinterpret_cast<const f32x4 *>(at(r + step) + own);
    };
    const auto leave_part = [&](int turn, f32x4 v) {        // rows 16 wave + g4 .. + 3: half a lane's elements of the sum over 32 (wave / 2)
        float t[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int c = 0; c < PC; ++c) {
            uint32_t w[2];
            round_off(t, w, c + 1 < PC);
            __builtin_memcpy(reinterpret_cast<char *>(&operands[turn][wave / 2][c][lane]) + wave % 2 * 8, w, 8);
        }
    };
    leave_part(0, *reinterpret_cast<const f32x4 *>(at(r) + own));
    const int steps = runs - 2;
    fetch(next[0], r);
    if (steps > 1) fetch(next[1], r + step);
    for (int n = 0; n < steps; n += 2)
#pragma unroll
        for (int turn = 0; turn < 2; ++turn) {
            if (n + turn >= steps) break;
            Frag<PC> A[DS];
#pragma unroll
            for (int d = 0; d < DS; ++d) A[d] = operand<PC>(next[turn].A[2 * d], next[turn].A[2 * d + 1]);
            f32x4 sum[DS] = {};
            sum[0] = next[turn].B;
            if (n + turn + 2 < steps) fetch(next[turn], r + 2 * step);
            __syncthreads();
#pragma unroll
            for (int d = 0; d < DS; ++d) {
                Frag<PC> S;
#pragma unroll
                for (int c = 0; c < PC; ++c) S.part[c] = operands[turn][d][c][lane];
                sum[d] = multiply(A[d], S, sum[d]);
            }
#pragma unroll
            for (int d = 1; d < DS; ++d) sum[0] += sum[d];
            leave_part(turn ^ 1, sum[0]);
            *reinterpret_cast<f32x4 *>(at(r + step) + own) = sum[0];
            r += step;
        }
}

template <typename T, int DK, bool BACK>
grim_status join_runs(const GdrParams &p, hipStream_t stream) {
    const int64_t groups = (int64_t)p.nseq * p.heads * p.tiles;
    hipLaunchKernelGGL((join_kernel<T, DK, BACK>), dim3((unsigned)groups), dim3(DK * 4), 0, stream, p);
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
