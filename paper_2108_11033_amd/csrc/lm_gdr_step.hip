// One token of the gated delta rule for a batch of callers.
//
//     D = exp(g) S    u = beta (v - k' D)    S_new = D + k u'    y = scale q' S_new = scale (q' D + (q . k) u)
//
// Bound by memory: a head's dk x dv states are read once and written once, held in registers between.  The second form of y takes all that has to be summed
// over the rows of the state (k'D, q'D, q . k and the lengths of q and k) from one pass, so that a workgroup meets at one barrier.
// 32 callers with 16 heads of 128 x 128: 13.6 us, 4.95 TB/s; one caller with 16 heads of 64 x 64 4.7 us of kernel.
#include "lm_gdr.hpp"

namespace grim {
namespace lm {

struct GdrStepParams {
    const float *q, *k, *v, *decay, *beta, *s;
    float *s_new;
    void *y;
    int64_t ldq, ldk, ldv, ldg, ldy;
    int32_t heads, group, dk, dv, blocks;       // group: value heads of a key head; blocks: of columns
    float scale, norm_eps;
};

constexpr int kStepColumns = 64;                // 16 lanes, four columns each

// A workgroup takes 64 columns of a caller's head: a row of 16 lanes per row of the state, 16 rows at a time.
template <typename T, int ROWS>
__global__ void __launch_bounds__(256) gdr_step(GdrStepParams p) {
    __shared__ float room[4][16][8];
    __shared__ float lengths[4][3];
    int64_t b = blockIdx.x;
    const int block = (int)(b % p.blocks);
    b /= p.blocks;
    const int h = (int)(b % p.heads);
    const int64_t caller = b / p.heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, row = threadIdx.x >> 4;
    const int c = block * kStepColumns + col * 4, have = min(p.dv - c, 4);      // (columns of this thread; none or fewer: <= 0)
    const int64_t key = (int64_t)(h / p.group) * p.dk, head = (caller * p.heads + h) * p.dk;
    float q[ROWS], k[ROWS], d[ROWS][4];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = i * 16 + row;
        q[i] = k[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) d[i][j] = 0.f;
        if (r >= p.dk) continue;
        q[i] = p.q[(key + r) * p.ldq + caller];
        k[i] = p.k[(key + r) * p.ldk + caller];
        const float *s = p.s + (head + r) * p.dv + c;
        if (have == 4) unpack(load<4>(s), d[i]);
        else
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < have) d[i][j] = s[j];
    }
    const float a = expf(p.decay[h * p.ldg + caller]), beta = p.beta[h * p.ldg + caller];
    float v[4], kd[4] = {}, qd[4] = {}, qk = 0.f, qq = 0.f, kk = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = j < have ? p.v[((int64_t)h * p.dv + c + j) * p.ldv + caller] : 0.f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        qk = __builtin_fmaf(q[i], k[i], qk);
        qq = __builtin_fmaf(q[i], q[i], qq);
        kk = __builtin_fmaf(k[i], k[i], kk);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            d[i][j] *= a;
            kd[j] = __builtin_fmaf(k[i], d[i][j], kd[j]);
            qd[j] = __builtin_fmaf(q[i], d[i][j], qd[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) kd[j] = across_rows(kd[j], Add()), qd[j] = across_rows(qd[j], Add());
    qk = across_rows(qk, Add()), qq = across_rows(qq, Add()), kk = across_rows(kk, Add());
    if (lane < 16)
#pragma unroll
        for (int j = 0; j < 4; ++j) room[wave][col][j] = kd[j], room[wave][col][4 + j] = qd[j];
    if (lane == 0) lengths[wave][0] = qk, lengths[wave][1] = qq, lengths[wave][2] = kk;
    __syncthreads();
    qk = qq = kk = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) kd[j] = qd[j] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        qk += lengths[w][0], qq += lengths[w][1], kk += lengths[w][2];
#pragma unroll
        for (int j = 0; j < 4; ++j) kd[j] += room[w][col][j], qd[j] += room[w][col][4 + j];
    }
    const float rk = p.norm_eps > 0.f ? 1.f / sqrtf(kk + p.norm_eps) : 1.f, rq = (p.norm_eps > 0.f ? 1.f / sqrtf(qq + p.norm_eps) : 1.f) * p.scale;
    float u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = beta * (v[j] - rk * kd[j]);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = i * 16 + row;
        if (r >= p.dk || have <= 0) continue;
        float *s = p.s_new + (head + r) * p.dv + c;
        const float ki = rk * k[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) d[i][j] = __builtin_fmaf(ki, u[j], d[i][j]);
        if (have == 4) store(s, d[i]);
        else
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < have) s[j] = d[i][j];
    }
    if (row != 0 || !p.y) return;
    T *y = static_cast<T *>(p.y) + ((int64_t)h * p.dv + c) * p.ldy + caller;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < have) y[j * p.ldy] = (T)(rq * __builtin_fmaf(rk * qk, u[j], qd[j]));
}

template <typename T>
grim_status gdr_step_typed(const GdrStepParams &call, int64_t batch, hipStream_t stream) {
    const int64_t each = (int64_t)call.heads * call.blocks;
    return in_runs(batch, most_groups(256) / each, [&](int64_t first, int64_t count) {
        GdrStepParams p = call;
        p.q += first, p.k += first, p.v += first, p.decay += first, p.beta += first;
        p.s += first * p.heads * p.dk * p.dv, p.s_new += first * p.heads * p.dk * p.dv;
        p.y = ahead(static_cast<T *>(p.y), first);
        const dim3 g((unsigned)(count * each)), b(256);
        if (p.dk <= 64) hipLaunchKernelGGL((gdr_step<T, 4>), g, b, 0, stream, p);
        else hipLaunchKernelGGL((gdr_step<T, 8>), g, b, 0, stream, p);
        return launched();
    });
}

}  // namespace lm
}  // namespace grim

extern "C" grim_status grim_gdr_step(const float *q_dev, const float *k_dev, const float *v_dev, int64_t ldq, int64_t ldk, int64_t ldv,
                                     const float *decay_dev, const float *beta_dev, int64_t ldg, const float *s_dev, float *s_new_dev, void *y_dev,
                                     grim_dtype dt, int64_t ldy, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv, float scale, float norm_eps,
                                     int32_t batch, void *hip_stream) {
    using namespace grim::lm;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if (heads < 1 || heads > kMostHeads || key_heads < 1 || heads % key_heads || dk < 1 || dv < 1 || batch < 0 || ldq < batch || ldk < batch || ldv < batch ||
        ldg < batch || (y_dev && ldy < batch) || !gdr_factors(scale, norm_eps))
        return GRIM_ERR_SHAPE;
    if (dk > kMostHeadSize || dv > kMostHeadSize) return GRIM_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)heads * kMostHeadSize;
    if (!fits(rows, ldq) || !fits(rows, ldk) || !fits(rows, ldv) || !fits(rows, ldg) || (y_dev && !fits(rows, ldy))) return GRIM_ERR_SHAPE;
    if (batch == 0) return GRIM_OK;
    if (!q_dev || !k_dev || !v_dev || !decay_dev || !beta_dev || !s_dev || !s_new_dev) return GRIM_ERR_NULL;
    if (s_dev != s_new_dev && overlap(s_dev, s_new_dev, (int64_t)batch * heads * dk * dv * 4)) return GRIM_ERR_UNSUPPORTED;
    const GdrStepParams p{q_dev, k_dev, v_dev, decay_dev, beta_dev, s_dev, s_new_dev, y_dev, ldq, ldk, ldv, ldg, ldy, heads, heads / key_heads, dk, dv,
                          (dv + kStepColumns - 1) / kStepColumns, scale, norm_eps};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dt == GRIM_F32   ? gdr_step_typed<float>(p, batch, stream)
           : dt == GRIM_F16 ? gdr_step_typed<f16>(p, batch, stream)
                            : gdr_step_typed<bf16>(p, batch, stream);
}
