// Layer norm over the rows of a matrix, forward and backward.
//
//     m = sum(x) / C    s = 1 / sqrt(sum((x - m)^2) / C + eps)    y = (x - m) s gamma + beta
//     dx = s (d - sum(d) / C - xh sum(d xh) / C),  d = dy gamma, xh = (x - m) s;   dgamma = sum_n dy xh,  dbeta = sum_n dy
//
// Both directions are bound by memory: a row is read once, stays in registers between its statistics and its result, and
// the variance is the centred one (the row is at hand, so nothing is saved by E(x^2) - m^2, which cancels).  Measured: 5003 x 1999 fp32
// forward 14.0 us (5.7 TB/s, part of it from the last-level cache), 32768 x 1024 bf16 backward 43.9 (37 of it the rows' pass at 5.5 TB/s),
// 8 x 1024 fp16 2.3 us of kernel.
#include "lm_common.hpp"

namespace grim {
namespace lm {

// A row of C elements dealt to TPR threads: PER pieces of V elements each, piece q = k * TPR + t.  PER is exact, so that only the last
// k has pieces that reach past the row; those are moved back to end with it (the row keeps no piece of its own that is
// narrower, hence C >= V), and the elements that another piece holds too are left out of the sums.
template <typename T>
constexpr int vec_of() { return 16 / (int)sizeof(T); }

template <int V, int TPR, int PER>
struct RowCut {
    int64_t at[PER];
    int first;              // elements of the last piece that belong to others (V and more: all of them)
    __device__ __forceinline__ RowCut(int t, int64_t C) {
#pragma unroll
        for (int k = 0; k < PER; ++k) at[k] = (int64_t)(k * TPR + t) * V;
        const int64_t over = at[PER - 1] - (C - V);
        first = over <= 0 ? 0 : over >= V ? V : (int)over;
        if (over > 0) at[PER - 1] = C - V;
    }
    template <typename F>
    __device__ __forceinline__ void own(F f) const {        // f(k, j) for every element of the thread's own
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (k < PER - 1 || j >= first) f(k, j);
    }
};

struct NormParams {
    const void *x;
    const float *gamma, *beta;
    void *y;
    float *mean, *rstd;
    int64_t ldx, ldy, N, C;
    float eps;
    bool past;
};

// TPR threads (16 lanes, one wave, or a workgroup of 4 or 16) per row.
template <typename T, int TPR, int PER>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_rows(NormParams p) {
    constexpr int V = vec_of<T>(), RPG = TPR < 256 ? 256 / TPR : 1;
    __shared__ float room[2][TPR < 64 ? 1 : TPR / 64];
    const int t = threadIdx.x % TPR;
    const int64_t n = (int64_t)blockIdx.x * RPG + threadIdx.x / TPR;
    if (TPR < 256 && n >= p.N) return;                     // (a team inside a wave: no barrier follows)
    const RowCut<V, TPR, PER> cut(t, p.C);
    const T *x = static_cast<const T *>(p.x) + n * p.ldx;
    Pack<T, V> raw[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) raw[k] = load<V>(x + cut.at[k]);
    float v[PER][V];
#pragma unroll
    for (int k = 0; k < PER; ++k) unpack(raw[k], v[k]);
    float sum = 0.f;
    cut.own([&](int k, int j) { sum += v[k][j]; });
    const float m = team_sum<TPR>(sum, room[0]) / (float)p.C;
    float sq = 0.f;
    cut.own([&](int k, int j) { const float d = v[k][j] - m; sq = __builtin_fmaf(d, d, sq); });
    const float s = 1.0f / sqrtf(team_sum<TPR>(sq, room[1]) / (float)p.C + p.eps);
    if (t == 0) {
        if (p.mean) p.mean[n] = m;
        if (p.rstd) p.rstd[n] = s;
    }
    T *y = static_cast<T *>(p.y) + n * p.ldy;
    store_rows(p.past, [&](auto past) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            float g[V], b[V], out[V];
#pragma unroll
            for (int j = 0; j < V; ++j) g[j] = 1.f, b[j] = 0.f;
            if (p.gamma) unpack(load<V>(p.gamma + cut.at[k]), g);
            if (p.beta) unpack(load<V>(p.beta + cut.at[k]), b);
#pragma unroll
            for (int j = 0; j < V; ++j) out[j] = __builtin_fmaf((v[k][j] - m) * s, g[j], b[j]);
            if (k < PER - 1 || cut.first < V) store<past.value>(y + cut.at[k], out);
        }
    });
}

// Rows narrower than one piece, or too wide for registers: a workgroup walks the row three times, an element a thread (1000 x 40000 bf16
// 160 us, a fifth of a copy's rate; 200000 x 7 133, most of a workgroup's threads without an element).
template <typename T>
__global__ void __launch_bounds__(256) norm_rows_any(NormParams p) {
    __shared__ float room[2][4];
    const int64_t n = blockIdx.x;
    const T *x = static_cast<const T *>(p.x) + n * p.ldx;
    T *y = static_cast<T *>(p.y) + n * p.ldy;
    float sum = 0.f, sq = 0.f;
    for (int64_t c = threadIdx.x; c < p.C; c += 256) sum += (float)x[c];
    const float m = group_sum<4>(sum, room[0]) / (float)p.C;
    for (int64_t c = threadIdx.x; c < p.C; c += 256) {
        const float d = (float)x[c] - m;
        sq = __builtin_fmaf(d, d, sq);
    }
    const float s = 1.0f / sqrtf(group_sum<4>(sq, room[1]) / (float)p.C + p.eps);
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[n] = m;
        if (p.rstd) p.rstd[n] = s;
    }
    for (int64_t c = threadIdx.x; c < p.C; c += 256)
        y[c] = (T)__builtin_fmaf(((float)x[c] - m) * s, p.gamma ? p.gamma[c] : 1.f, p.beta ? p.beta[c] : 0.f);
}

struct NormBackParams {
    const void *dy, *x;
    const float *gamma, *mean, *rstd;
    void *dx;
    float *part;            // [workgroup][dgamma | dbeta][C], or NULL
    int64_t lddy, ldx, lddx, N, C;
    bool past;
};

constexpr int kBackWaves = 4;           // waves of a workgroup whose waves take rows of their own

// A workgroup walks over rows blockIdx.x * RPG, + gridDim.x * RPG, ... (RPG teams of TPR threads); each thread keeps the sums of dgamma and dbeta for its
// columns in registers over all of them, so x and dy are read once for all three gradients.  The next row is asked for
// before the present one is summed.
template <typename T, int TPR, int PER>
__global__ void __launch_bounds__(TPR < 256 ? 64 * kBackWaves : TPR) norm_back_rows(NormBackParams p) {
    constexpr int V = vec_of<T>(), W = TPR < 64 ? 1 : TPR / 64, RPG = TPR < 256 ? 64 * kBackWaves / TPR : 1;
    __shared__ float room[2][2][W];
    extern __shared__ float sums[];                         // one wave per row: [dgamma | dbeta][C]
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR;
    const RowCut<V, TPR, PER> cut(t, p.C);
    float ag[PER][V], ab[PER][V], g[PER][V];
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) ag[k][j] = 0.f, ab[k][j] = 0.f, g[k][j] = 1.f;
    if (p.gamma)
#pragma unroll
        for (int k = 0; k < PER; ++k) unpack(load<V>(p.gamma + cut.at[k]), g[k]);
    const float inv = 1.0f / (float)p.C;
    const int64_t step = (int64_t)gridDim.x * RPG;
    int64_t n = (int64_t)blockIdx.x * RPG + team;
    Pack<T, V> xr[PER], dr[PER], xn[PER], dn[PER];          // this row and the next
    float mn = 0.f, sn = 0.f;
    auto fetch = [&](int64_t row) {
        const T *x = static_cast<const T *>(p.x) + row * p.ldx;
        const T *dy = static_cast<const T *>(p.dy) + row * p.lddy;
#pragma unroll
        for (int k = 0; k < PER; ++k) xn[k] = load<V>(x + cut.at[k]), dn[k] = load<V>(dy + cut.at[k]);
        mn = p.mean[row];
        sn = p.rstd[row];
    };
    if (n < p.N) fetch(n);
    int turn = 0;
    for (; n < p.N; n += step, turn ^= 1) {
#pragma unroll
        for (int k = 0; k < PER; ++k) xr[k] = xn[k], dr[k] = dn[k];
        const float m = mn, s = sn;
        if (n + step < p.N) fetch(n + step);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            float xh[V], d[V];
            unpack(xr[k], xh);
            unpack(dr[k], d);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (k == PER - 1 && j < cut.first) continue;
                const float h = (xh[j] - m) * s, dg = d[j] * g[k][j];
                ag[k][j] = __builtin_fmaf(d[j], h, ag[k][j]);
                ab[k][j] += d[j];
                s1 += dg;
                s2 = __builtin_fmaf(dg, h, s2);
            }
        }
        if (!p.dx) continue;
        // (two sets of words in turn: a wave may be one row ahead of another)
        s1 = row_join(s1, Add());
        s2 = row_join(s2, Add());
        if (TPR >= 64) s1 = across_rows(s1, Add()), s2 = across_rows(s2, Add());
        if (W > 1) {
            if ((threadIdx.x & 63) == 0) room[turn][0][threadIdx.x >> 6] = s1, room[turn][1][threadIdx.x >> 6] = s2;
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) s1 += room[turn][0][w], s2 += room[turn][1][w];
        }
        const float c1 = s1 * inv, c2 = s2 * inv;
        T *dx = static_cast<T *>(p.dx) + n * p.lddx;
        store_rows(p.past, [&](auto past) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                float xh[V], d[V], out[V];
                forget(xr[k]);
                forget(dr[k]);
                unpack(xr[k], xh);
                unpack(dr[k], d);
#pragma unroll
                for (int j = 0; j < V; ++j) out[j] = s * (d[j] * g[k][j] - c1 - (xh[j] - m) * s * c2);
                if (k < PER - 1 || cut.first < V) store<past.value>(dx + cut.at[k], out);
            }
        });
    }
    if (!p.part) return;
    float *part = p.part + (int64_t)blockIdx.x * 2 * p.C;
    if (TPR >= 256) {
        // (whole pieces at a time: 300 x 8192 fp16 16 us, 25 element by element)
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (k < PER - 1 || cut.first == 0) {
                store(part + cut.at[k], ag[k]);
                store(part + p.C + cut.at[k], ab[k]);
            } else
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (j >= cut.first) part[cut.at[k] + j] = ag[k][j], part[p.C + cut.at[k] + j] = ab[k][j];
        }
        return;
    }
    if (TPR < 64)
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) ag[k][j] = across_rows(ag[k][j], Add()), ab[k][j] = across_rows(ab[k][j], Add());
    for (int w = 0; w < kBackWaves; ++w) {                  // the waves' sums, in the order of the waves
        if ((int)threadIdx.x / 64 == w && threadIdx.x % 64 < TPR)
            cut.own([&](int k, int j) {
                const int64_t c = cut.at[k] + j;
                sums[c] = w ? sums[c] + ag[k][j] : ag[k][j];
                sums[p.C + c] = w ? sums[p.C + c] + ab[k][j] : ab[k][j];
            });
        __syncthreads();
    }
    for (int64_t c = threadIdx.x; c < 2 * p.C; c += blockDim.x) part[c] = sums[c];
}

// dx of rows that the kernel above has no form for (2000 x 10000 bf16 37 us, and 26 for the columns' sums below).
template <typename T>
__global__ void __launch_bounds__(256) norm_back_any(NormBackParams p) {
    __shared__ float room[2][4];
    const int64_t n = blockIdx.x;
    const T *x = static_cast<const T *>(p.x) + n * p.ldx, *dy = static_cast<const T *>(p.dy) + n * p.lddy;
    T *dx = static_cast<T *>(p.dx) + n * p.lddx;
    const float m = p.mean[n], s = p.rstd[n];
    float s1 = 0.f, s2 = 0.f;
    for (int64_t c = threadIdx.x; c < p.C; c += 256) {
        const float d = (float)dy[c] * (p.gamma ? p.gamma[c] : 1.f);
        s1 += d;
        s2 = __builtin_fmaf(d, ((float)x[c] - m) * s, s2);
    }
    const float c1 = group_sum<4>(s1, room[0]) / (float)p.C, c2 = group_sum<4>(s2, room[1]) / (float)p.C;
    for (int64_t c = threadIdx.x; c < p.C; c += 256) {
        const float d = (float)dy[c] * (p.gamma ? p.gamma[c] : 1.f);
        dx[c] = (T)(s * (d - c1 - ((float)x[c] - m) * s * c2));
    }
}

// The columns' sums of such rows: a thread per column and slab of rows.
template <typename T>
__global__ void __launch_bounds__(256) norm_back_columns(NormBackParams p, int64_t slab) {
    const int64_t c = (int64_t)blockIdx.y * 256 + threadIdx.x;
    if (c >= p.C) return;
    const int64_t n0 = blockIdx.x * slab, n1 = n0 + slab < p.N ? n0 + slab : p.N;
    float ag = 0.f, ab = 0.f;
    for (int64_t n = n0; n < n1; ++n) {
        const float d = (float)static_cast<const T *>(p.dy)[n * p.lddy + c];
        ag = __builtin_fmaf(d, ((float)static_cast<const T *>(p.x)[n * p.ldx + c] - p.mean[n]) * p.rstd[n], ag);
        ab += d;
    }
    float *part = p.part + (int64_t)blockIdx.x * 2 * p.C;
    part[c] = ag;
    part[p.C + c] = ab;
}

// Sums of the workgroups' columns, in a fixed order: 16 columns by 64 threads, each every 64th workgroup's, then four sums of 16
// and theirs.  (Short runs of columns: what it takes is the loads that follow each other in a thread.)
__global__ void __launch_bounds__(1024) join_columns_kernel(const float *part, int64_t groups, int64_t C0, float *out0, int64_t C1,
                                                            float *out1) {
    __shared__ float sums[64][17];
    const int col = threadIdx.x & 15, w = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + col, width = C0 + C1;
    float s = 0.f;
    if (c < width) {
#pragma unroll 16
        for (int64_t i = w; i < groups; i += 64) s += part[i * width + c];
    }
    sums[w][col] = s;
    __syncthreads();
    if (w < 4) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += sums[16 * w + i][col];
    }
    __syncthreads();
    if (w < 4) sums[w][col] = s;
    __syncthreads();
    if (w || c >= width) return;
    s = (sums[0][col] + sums[1][col]) + (sums[2][col] + sums[3][col]);
    if (c < C0) {
        if (out0) out0[c] = s;
    } else if (out1) out1[c - C0] = s;
}

grim_status join_columns(const float *part, int64_t groups, int64_t C0, float *out0, int64_t C1, float *out1, hipStream_t stream) {
    const int64_t grid = (C0 + C1 + 15) / 16;                   // (C0 + C1 below 2^26 in all calls)
    hipLaunchKernelGGL(join_columns_kernel, dim3((unsigned)grid), dim3(1024), 0, stream, part, groups, C0, out0, C1, out1);
    return launched();
}

// Threads per row: as few (16, a wave, 4 waves, 16) as hold the row in four pieces each; 0: the walking kernels.
template <typename T>
int threads_per_row(int64_t C) {
    const int64_t V = vec_of<T>();
    for (int tpr : {16, 64, 256, 1024})
        if (C >= V && C <= 4 * tpr * V) return tpr;
    return 0;
}

// The fewest pieces of a team of TPR threads: what the next smaller team, with `held` pieces each, has no room for.
constexpr int fewest_pieces(int tpr, int held) { return tpr == 16 ? 1 : held * (tpr / 4) / tpr + 1; }

// The same for the backward pass, whose threads hold five values per element: as many as leave no register spilled.
template <typename T>
constexpr int back_pieces(int tpr) { return (tpr == 1024 ? 8 : tpr == 256 && sizeof(T) == 2 ? 32 : 16) / vec_of<T>(); }
// (16 waves hold no more 16-bit features than 4 do)
template <typename T>
int back_threads_per_row(int64_t C) {
    const int64_t V = vec_of<T>();
    for (int tpr : {16, 64, 256, sizeof(T) == 4 ? 1024 : 256})
        if (C >= V && C <= back_pieces<T>(tpr) * tpr * V) return tpr;
    return 0;
}

// Workgroups of the backward pass.  A workgroup's column sums cost 8 C bytes written and read again.  Several rows at a time (teams of
// a wave or less): 64 rows each, 2 % of 6 C bytes a row in 16 bits, but at least 256 workgroups and at most 1024.  One row at a time: as
// many as have some 32 KB of rows on their way to a compute unit, up to 1024 with 8 rows or more each (12142 x 1038 bf16: 256
// workgroups 47 us, 1024 24), but no fewer than 256.
template <typename T>
int64_t back_groups_of(int64_t N, int64_t C) {
    const int tpr = back_threads_per_row<T>(C);
    const int at_once = tpr == 16 || tpr == 64 ? 64 * kBackWaves / tpr : 1;
    const int64_t all = (N + at_once - 1) / at_once;
    int64_t groups = N / 64;
    if (at_once == 1) {
        const int64_t each = 32768 / (2 * C * (int64_t)sizeof(T)), room = (each < 1 ? 1 : each) * kComputeUnits;
        groups = N / 8 < room ? N / 8 : room;
    }
    groups = groups < kComputeUnits ? kComputeUnits : groups > 4 * kComputeUnits ? 4 * kComputeUnits : groups;
    return all < groups ? all : groups;
}

// Rows first .. first + count - 1 of a call.
template <typename T>
NormParams rows_of(NormParams p, int64_t first, int64_t count) {
    p.x = static_cast<const T *>(p.x) + first * p.ldx;
    p.y = static_cast<T *>(p.y) + first * p.ldy;
    p.mean = ahead(p.mean, first), p.rstd = ahead(p.rstd, first);
    p.N = count;
    return p;
}

template <typename T, int TPR>
grim_status norm_launch(const NormParams &call, hipStream_t stream) {
    constexpr int RPG = TPR < 256 ? 256 / TPR : 1, threads = TPR < 256 ? 256 : TPR, fewest = fewest_pieces(TPR, 4);
    return in_runs(call.N, most_groups(threads) * RPG, [&](int64_t first, int64_t count) {
        const NormParams p = rows_of<T>(call, first, count);
        const dim3 g((unsigned)((p.N + RPG - 1) / RPG)), b(threads);
        switch ((p.C + TPR * vec_of<T>() - 1) / (TPR * vec_of<T>())) {
            case 1: hipLaunchKernelGGL((norm_rows<T, TPR, fewest>), g, b, 0, stream, p); break;
            case 2: hipLaunchKernelGGL((norm_rows<T, TPR, 2>), g, b, 0, stream, p); break;
            case 3: hipLaunchKernelGGL((norm_rows<T, TPR, 3>), g, b, 0, stream, p); break;
            default: hipLaunchKernelGGL((norm_rows<T, TPR, 4>), g, b, 0, stream, p); break;
        }
        return launched();
    });
}

template <typename T>
grim_status norm_typed(const NormParams &p, hipStream_t stream) {
    switch (threads_per_row<T>(p.C)) {
        case 16: return norm_launch<T, 16>(p, stream);
        case 64: return norm_launch<T, 64>(p, stream);
        case 256: return norm_launch<T, 256>(p, stream);
        case 1024: return norm_launch<T, 1024>(p, stream);
    }
    return in_runs(p.N, most_groups(256), [&](int64_t first, int64_t count) {
        hipLaunchKernelGGL(norm_rows_any<T>, dim3((unsigned)count), dim3(256), 0, stream, rows_of<T>(p, first, count));
        return launched();
    });
}

template <typename T, int TPR>
grim_status norm_back_launch(const NormBackParams &p, int64_t groups, hipStream_t stream) {
    const dim3 g((unsigned)groups), b(TPR < 256 ? 64 * kBackWaves : TPR);
    const size_t lds = TPR < 256 && p.part ? 2 * p.C * sizeof(float) : 0;
    constexpr int most = back_pieces<T>(TPR), fewest = fewest_pieces(TPR, back_pieces<T>(TPR / 4));
    switch ((p.C + TPR * vec_of<T>() - 1) / (TPR * vec_of<T>())) {
        case 1: hipLaunchKernelGGL((norm_back_rows<T, TPR, fewest>), g, b, lds, stream, p); break;
        case 2: hipLaunchKernelGGL((norm_back_rows<T, TPR, most < 2 ? most : 2>), g, b, lds, stream, p); break;
        case 3: hipLaunchKernelGGL((norm_back_rows<T, TPR, most < 3 ? most : 3>), g, b, lds, stream, p); break;
        default: hipLaunchKernelGGL((norm_back_rows<T, TPR, most>), g, b, lds, stream, p); break;
    }
    return launched();
}

template <typename T>
NormBackParams rows_of(NormBackParams p, int64_t first, int64_t count) {
    p.dy = static_cast<const T *>(p.dy) + first * p.lddy;
    p.x = static_cast<const T *>(p.x) + first * p.ldx;
    p.dx = static_cast<T *>(p.dx) + first * p.lddx;
    p.mean += first, p.rstd += first;
    p.N = count;
    return p;
}

constexpr int64_t kMostFeatures = 65535 * 256;              // of the backward pass: norm_back_columns has so many blocks of columns

template <typename T>
grim_status norm_back_typed(const NormBackParams &p, float *dgamma, float *dbeta, hipStream_t stream) {
    const int64_t groups = back_groups_of<T>(p.N, p.C);
    grim_status st = GRIM_OK;
    if (p.N > 0) {
        switch (back_threads_per_row<T>(p.C)) {
            case 16: st = norm_back_launch<T, 16>(p, groups, stream); break;
            case 64: st = norm_back_launch<T, 64>(p, groups, stream); break;
            case 256: st = norm_back_launch<T, 256>(p, groups, stream); break;
            case 1024:
                if constexpr (sizeof(T) == 4) st = norm_back_launch<T, 1024>(p, groups, stream);
                break;
            default:
                if (p.part) {                                               // first: dx may take dy's place
                    const int64_t slab = (p.N + groups - 1) / groups;
                    hipLaunchKernelGGL(norm_back_columns<T>, dim3((unsigned)groups, (unsigned)((p.C + 255) / 256)), dim3(256), 0,
                                       stream, p, slab);
                    st = launched();
                }
                if (p.dx && st == GRIM_OK)
                    st = in_runs(p.N, most_groups(256), [&](int64_t first, int64_t count) {
                        hipLaunchKernelGGL(norm_back_any<T>, dim3((unsigned)count), dim3(256), 0, stream, rows_of<T>(p, first, count));
                        return launched();
                    });
        }
    }
    if (st != GRIM_OK || !p.part) return st;
    return join_columns(p.part, p.N > 0 ? groups : 0, p.C, dgamma, p.C, dbeta, stream);
}

}  // namespace lm
}  // namespace grim

extern "C" {

grim_status grim_layer_norm(const void *x_dev, grim_dtype dt, int64_t ldx, const float *gamma_dev, const float *beta_dev,
                            float eps, int64_t N, int64_t C, void *y_dev, int64_t ldy, float *mean_dev, float *rstd_dev,
                            void *hip_stream) {
    using namespace grim::lm;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if (N < 0 || N > kMostRows || C < 1 || ldx < C || ldy < C || !fits(N, ldx) || !fits(N, ldy) || !(eps >= 0.f) || eps > 3.4e38f) return GRIM_ERR_SHAPE;
    if (N == 0) return GRIM_OK;
    if (!x_dev || !y_dev) return GRIM_ERR_NULL;
    if (moves(x_dev, ldx, y_dev, ldy, N)) return GRIM_ERR_SHAPE;
    const NormParams p{x_dev, gamma_dev, beta_dev, y_dev, mean_dev, rstd_dev, ldx, ldy, N, C, eps,
                       past_caches(2 * N * C * bytes_of(dt))};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dt == GRIM_F32 ? norm_typed<float>(p, stream) : dt == GRIM_F16 ? norm_typed<f16>(p, stream) : norm_typed<bf16>(p, stream);
}

int64_t grim_layer_norm_workspace(int64_t N, int64_t C) {
    using namespace grim::lm;
    if (N < 0 || N > kMostRows || C < 1 || C > kMostFeatures) return 0;
    const int64_t a = back_groups_of<float>(N, C), b = back_groups_of<f16>(N, C);
    const int64_t groups = a > b ? a : b;
    return (groups > 0 ? groups : 1) * 2 * C * (int64_t)sizeof(float);
}

grim_status grim_layer_norm_backward(const void *dy_dev, int64_t lddy, const void *x_dev, int64_t ldx, grim_dtype dt,
                                     const float *gamma_dev, const float *mean_dev, const float *rstd_dev, int64_t N,
                                     int64_t C, void *dx_dev, int64_t lddx, float *dgamma_dev, float *dbeta_dev,
                                     void *workspace, int64_t workspace_bytes, void *hip_stream) {
    using namespace grim::lm;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if (N < 0 || N > kMostRows || C < 1 || C > kMostFeatures || lddy < C || ldx < C || (dx_dev && lddx < C) || !fits(N, lddy) || !fits(N, ldx) ||
        (dx_dev && !fits(N, lddx)))
        return GRIM_ERR_SHAPE;
    const bool sums = dgamma_dev || dbeta_dev;
    if (N > 0 && (!dy_dev || !x_dev || !mean_dev || !rstd_dev)) return GRIM_ERR_NULL;
    if (sums && !workspace) return GRIM_ERR_NULL;
    if (moves(dy_dev, lddy, dx_dev, lddx, N)) return GRIM_ERR_SHAPE;
    if (sums && workspace_bytes < grim_layer_norm_workspace(N, C)) return GRIM_ERR_SHAPE;
    if (!sums && (!dx_dev || N == 0)) return GRIM_OK;
    const NormBackParams p{dy_dev, x_dev, gamma_dev, mean_dev, rstd_dev, dx_dev, sums ? static_cast<float *>(workspace) : nullptr,
                           lddy, ldx, lddx, N, C, past_caches(3 * N * C * bytes_of(dt))};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dt == GRIM_F32   ? norm_back_typed<float>(p, dgamma_dev, dbeta_dev, stream)
           : dt == GRIM_F16 ? norm_back_typed<f16>(p, dgamma_dev, dbeta_dev, stream)
                            : norm_back_typed<bf16>(p, dgamma_dev, dbeta_dev, stream);
}

}  // extern "C"
