// The clipped policy loss of chosen words, with a KL term against a reference: loss and gradient in one pass over the logits.
//
//     lp = log softmax(z / tau)[id]    r = exp(lp - old)    d = ref - lp
//     loss = w (kl (exp(d) - d - 1) - min(r A, clamp(r, 1 - low, 1 + high) A))
//     dloss/dlp = w (kl (1 - exp(d)) - (r A <= clamp(r) A ? r A : 0))    dz_j = dloss/dlp ([j = id] - softmax(z / tau)_j) / tau
//
// Bound by memory: z read once, dz written once.  A workgroup keeps its row in registers between the maximum, the sum and the gradient; the row's one word
// is looked up while the row is on its way, and its place in the gradient is the owner's, so nothing is stored twice.  Few rows of a large vocabulary,
// or rows that no workgroup's registers hold, are cut into slices: a first launch leaves every slice's maximum, sum and (where it lies) the word's logit,
// the second joins them and writes the gradient from a second read of z, which a few rows leave in the caches.
// 8192 x 32768 bf16: 218 us, 4.9 TB/s; 1024 x 1000 fp32: 5.7 us, a launch and one trip to memory; 24 x 131075 fp16, in slices: 10.2 us, two of each.
#include "lm_rows.hpp"

namespace grim {
namespace lm {

struct PolicyParams {
    const void *z;
    const int32_t *ids;
    const float *old_logp, *ref_logp, *advantage, *weight;
    float *loss, *logp;
    void *dz;
    float *part;                // [row][slice][maximum, sum, the word's logit, -]
    int64_t ldz, lddz, V;
    int32_t slices;
    float tau, scale;           // scale = log2(e) / tau
    float low, high, kl;        // the ratio's bounds
    bool past;
};

struct RowTerms {
    int32_t id;                 // -1: no word, the row counts for nothing
    float weight;
    __device__ __forceinline__ RowTerms(const PolicyParams &p, int64_t n) : id(p.ids[n]), weight(p.weight ? p.weight[n] : 1.f) {
        if (id < 0 || id >= p.V) id = -1;
    }
    __device__ __forceinline__ bool counts(const PolicyParams &p) const { return id >= 0 && weight != 0.f && (p.loss || p.dz); }
    // The loss of a row, and dloss/dlp / tau.
    __device__ __forceinline__ float loss(const PolicyParams &p, int64_t n, float lp, float &slope) const {
        const float A = p.advantage[n], r = p.old_logp ? expf(lp - p.old_logp[n]) : 1.f;
        const float plain = r * A, cut = fminf(fmaxf(r, p.low), p.high) * A;
        // (a NaN on either side stays one)
        float value = -(plain <= cut || plain != plain ? plain : cut), dlp = plain <= cut || plain != plain ? -plain : 0.f;
        if (p.ref_logp && p.kl != 0.f) {
            const float d = p.ref_logp[n] - lp, e = expm1f(d);
            value += p.kl * (e - d);
            dlp -= p.kl * e;
        }
        slope = weight * dlp / p.tau;
        return weight * value;
    }
};

// -------------------------------------------------------------------------------------------------- one workgroup per row
// W waves hold the row, at most PER pieces of 16 bytes a thread: pieces k < full are whole for all threads, piece `full` for
// some, the others are empty.  A piece that reaches past the row is moved back to end with it; what it shares counts in the other.
template <typename T, int W, int PER>
__global__ void __launch_bounds__(64 * W) policy_rows(PolicyParams p) {
    constexpr int V = piece<T>(), TPR = 64 * W;
    __shared__ float room[2][W];
    const int64_t n = blockIdx.x;
    const T *z = static_cast<const T *>(p.z) + n * p.ldz;
    T *dz = p.dz ? static_cast<T *>(p.dz) + n * p.lddz : nullptr;
    const RowTerms row(p, n);
    const bool counts = row.counts(p);
    if (!counts) {
        if (threadIdx.x == 0 && p.loss) p.loss[n] = 0.f;
        if (threadIdx.x == 0 && p.logp && row.id < 0) p.logp[n] = 0.f;
        if (row.id < 0 || !p.logp) {
            if (dz) zero_row(dz, 0, p.V);
            return;
        }
    }
    const int full = (int)(p.V / (TPR * V));
    const int mine = full * TPR * V + (int)threadIdx.x * V;   // where piece `full` would start
    const bool some = mine < p.V;
    const int tail = (int)min((int64_t)mine, p.V - V), first = mine - tail;
    Pack<T, V> raw[PER];
    float chosen = (float)z[row.id];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        if (k < full) raw[k] = load<V>(z + k * TPR * V + (int)threadIdx.x * V);
        else if (k == full && some) raw[k] = load<V>(z + tail);
    }
    asm volatile("" : "+v"(chosen));                        // (here before any barrier: dz may be z)
    auto own = [&](auto f) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (k > full || (k == full && !some)) continue;
            float v[V];
            forget(raw[k]);
            unpack(raw[k], v);
            if (k < full) {
#pragma unroll
                for (int j = 0; j < V; ++j) f(v[j]);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (j >= first) f(v[j]);
            }
        }
    };
    float peak = -INFINITY, sum = 0.f;
    own([&](float v) { peak = fmaxf(peak, v); });
    peak = group_max<W>(peak, room[0]);
    own([&](float v) { sum += __builtin_amdgcn_exp2f((v - peak) * p.scale); });
    sum = group_sum<W>(sum, room[1]);
    const float lp = (chosen - peak) / p.tau - kLn2 * log2f(sum);
    if (threadIdx.x == 0 && p.logp) p.logp[n] = lp;
    if (!counts) {
        if (dz) zero_row(dz, 0, p.V);
        return;
    }
    float slope;
    const float loss = row.loss(p, n, lp, slope);
    if (threadIdx.x == 0 && p.loss) p.loss[n] = loss;
    if (!dz) return;
    const float share = -slope * (1.f / sum);
    store_rows(p.past, [&](auto past) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (k > full || (k == full && !some)) continue;
            const int at = k < full ? k * TPR * V + (int)threadIdx.x * V : tail;
            float v[V], out[V];
            forget(raw[k]);
            unpack(raw[k], v);
#pragma unroll
            for (int j = 0; j < V; ++j) out[j] = share * __builtin_amdgcn_exp2f((v[j] - peak) * p.scale);
            const uint32_t here = (uint32_t)(row.id - at);
            if (here < V)
#pragma unroll
                for (int j = 0; j < V; ++j) out[j] += j == (int)here ? slope : 0.f;
            store<past.value>(dz + at, out);
        }
    });
}

// -------------------------------------------------------------------------------------------------- slices of rows
template <typename T>
__global__ void __launch_bounds__(64 * kSliceWaves) policy_slices(PolicyParams p) {
    constexpr int V = piece<T>(), W = kSliceWaves;
    __shared__ float room[2][W];
    const int64_t n = blockIdx.x / p.slices, s = blockIdx.x % p.slices;
    const RowTerms row(p, n);
    if (row.id < 0 || (!row.counts(p) && !p.logp)) return;
    const T *z = static_cast<const T *>(p.z) + n * p.ldz;
    const int64_t lo = s * slice_elements<T>(), hi = lo + slice_elements<T>() < p.V ? lo + slice_elements<T>() : p.V;
    const float chosen = row.id >= lo && row.id < hi ? (float)z[row.id] : 0.f;
    Slice<T> sl(z, lo, hi);
    float peak = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < kSlicePer; ++k) {
        float v[V];
        unpack(sl.raw[k], v);
#pragma unroll
        for (int j = 0; j < V; ++j) peak = fmaxf(peak, v[j]);
    }
    peak = group_max<W>(peak, room[0]);
    // (a slice of nothing but -infinity has the sum 0; one NaN makes the sum NaN)
    const float base = peak == -INFINITY ? 0.f : peak;
#pragma unroll
    for (int k = 0; k < kSlicePer; ++k) {
        float v[V];
        forget(sl.raw[k]);
        unpack(sl.raw[k], v);
#pragma unroll
        for (int j = 0; j < V; ++j) sum += __builtin_amdgcn_exp2f((v[j] - base) * p.scale);
    }
    sum = group_sum<W>(sum, room[1]);
    if (threadIdx.x == 0) {
        float *part = p.part + (int64_t)blockIdx.x * 4;
        part[0] = peak, part[1] = sum, part[2] = chosen;
    }
}

template <typename T>
__global__ void __launch_bounds__(64 * kSliceWaves) policy_join(PolicyParams p) {
    constexpr int V = piece<T>();
    const int64_t n = blockIdx.x / p.slices, s = blockIdx.x % p.slices;
    const T *z = static_cast<const T *>(p.z) + n * p.ldz;
    T *dz = p.dz ? static_cast<T *>(p.dz) + n * p.lddz : nullptr;
    const int64_t lo = s * slice_elements<T>(), hi = lo + slice_elements<T>() < p.V ? lo + slice_elements<T>() : p.V;
    const int lane = threadIdx.x & 63;
    const RowTerms row(p, n);
    const bool counts = row.counts(p), writer = threadIdx.x == 0 && s == 0;
    if (!counts) {
        if (writer && p.loss) p.loss[n] = 0.f;
        if (writer && p.logp && row.id < 0) p.logp[n] = 0.f;
        if (dz) zero_row(dz, lo, hi);
        if (row.id < 0 || !p.logp || s != 0) return;
    }
    const Slice<T> sl(z, lo, dz && counts ? hi : lo);
    // the maximum and the sum of the whole row from its slices', by every wave for itself
    const float *part = p.part + n * p.slices * 4;
    float own = -INFINITY, sum = 0.f;
    for (int i = lane; i < p.slices; i += 64) {
        const float m = part[4 * i], x = part[4 * i + 1], high = fmaxf(own, m);
        // (a slice without a maximum has the sum 0, or NaN)
        sum = (own == -INFINITY ? sum : sum * __builtin_amdgcn_exp2f((own - high) * p.scale)) +
              (m == -INFINITY ? x : x * __builtin_amdgcn_exp2f((m - high) * p.scale));
        own = high;
    }
    const float peak = wave_max(own);
    sum = wave_sum(own == -INFINITY && peak != -INFINITY ? sum : sum * __builtin_amdgcn_exp2f((own - peak) * p.scale));
    const float chosen = part[4 * (row.id / slice_elements<T>()) + 2];
    const float lp = (chosen - peak) / p.tau - kLn2 * log2f(sum);
    if (writer && p.logp) p.logp[n] = lp;
    if (!counts) return;
    float slope;
    const float loss = row.loss(p, n, lp, slope);
    if (writer && p.loss) p.loss[n] = loss;
    if (!dz) return;
    const float share = -slope * (1.f / sum);
#pragma unroll
    for (int k = 0; k < kSlicePer; ++k) {
        const int64_t at = Slice<T>::at(lo, k);
        float v[V];
        unpack(sl.raw[k], v);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = share * __builtin_amdgcn_exp2f((v[j] - peak) * p.scale) + (at + j == row.id ? slope : 0.f);
        T *to = dz + at;
        if (sl.have[k] == V) store(to, v);
        else
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < sl.have[k]) to[j] = (T)v[j];
    }
}

// -------------------------------------------------------------------------------------------------- launches
// A workgroup per row where its registers hold the row (16 pieces a thread of 16 waves) and the row is short or the rows
// fill the card: a second launch costs 3 us, a lone row of 65536 elements 4 us more in one workgroup than in slices.
// Measured, by rows and in slices, in us: bf16 4 x 16384 7.0 and 9.6, 64 x 32768 8.5 and 9.7, 64 x 50000 11.6 and 11.1,
// 32 x 65536 13.3 and 9.5, 128 x 131072 25.5 and 20.0, 160 x 131072 26.8 and 26.2, 192 x 131072 28.2 and 30.9,
// 512 x 65536 26.3 and 37.7; fp32 32 x 32768 9.2 and 9.8, 64 x 65536 14.7 and 12.2, 128 x 65536 18.7 both,
// 160 x 65536 20.6 and 24.3.
template <typename T>
bool policy_by_rows(int64_t N, int64_t V) {
    return V >= piece<T>() && V <= (int64_t)16 * 1024 * piece<T>() && (V <= 32768 || N >= (sizeof(T) == 2 ? 160 : 128));
}

// Rows first .. first + count - 1 of a call.
template <typename T>
PolicyParams rows_of(PolicyParams p, int64_t first) {
    p.z = static_cast<const T *>(p.z) + first * p.ldz;
    p.ids += first;
    p.old_logp = ahead(p.old_logp, first), p.ref_logp = ahead(p.ref_logp, first);
    p.advantage = ahead(p.advantage, first), p.weight = ahead(p.weight, first);
    p.loss = ahead(p.loss, first), p.logp = ahead(p.logp, first);
    p.dz = ahead(static_cast<T *>(p.dz), first * p.lddz);
    p.part += first * p.slices * 4;
    return p;
}

template <typename T>
grim_status policy_typed(PolicyParams call, int64_t N, hipStream_t stream) {
    if (policy_by_rows<T>(N, call.V)) {
        const int64_t pieces = (call.V + piece<T>() - 1) / piece<T>();
        const auto launch = [&](auto kernel, int threads) {
            return in_runs(N, most_groups(threads), [&](int64_t first, int64_t count) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(threads), 0, stream, rows_of<T>(call, first));
                return launched();
            });
        };
        if (pieces <= 128) return launch(policy_rows<T, 1, 2>, 64);
        if (pieces <= 256) return launch(policy_rows<T, 1, 4>, 64);
        if (pieces <= 1024) return launch(policy_rows<T, 4, 4>, 256);
        if (pieces <= 2048) return launch(policy_rows<T, 8, 4>, 512);
        if (pieces <= 4096) return launch(policy_rows<T, 8, 8>, 512);
        if (pieces <= 8192) return launch(policy_rows<T, 8, 16>, 512);
        return launch(policy_rows<T, 16, 16>, 1024);
    }
    call.slices = (int32_t)slices_of<T>(call.V);
    constexpr int threads = 64 * kSliceWaves;
    return in_runs(N, most_groups(threads) / call.slices, [&](int64_t first, int64_t count) {
        const PolicyParams p = rows_of<T>(call, first);
        const dim3 g((unsigned)(count * p.slices)), b(threads);
        hipLaunchKernelGGL(policy_slices<T>, g, b, 0, stream, p);
        const grim_status st = launched();
        if (st != GRIM_OK) return st;
        hipLaunchKernelGGL(policy_join<T>, g, b, 0, stream, p);
        return launched();
    });
}

}  // namespace lm
}  // namespace grim

extern "C" {

int64_t grim_policy_loss_workspace(int64_t N, int64_t V) {
    using namespace grim::lm;
    if (N < 0 || N > kMostRows || V < 1 || V >= (int64_t)1 << 31) return 0;
    // (whichever type comes: of fp32 a slice holds the fewest elements)
    int64_t bytes = 16;
    if (!policy_by_rows<float>(N, V)) bytes += N * slices_of<float>(V) * 16;
    else if (!policy_by_rows<f16>(N, V)) bytes += N * slices_of<f16>(V) * 16;
    return bytes;
}

grim_status grim_policy_loss(const void *z_dev, grim_dtype dt, int64_t ldz, const grim_policy *policy, int64_t N, int64_t V,
                             float *loss_dev, float *logp_dev, void *dz_dev, int64_t lddz, void *workspace,
                             int64_t workspace_bytes, void *hip_stream) {
    using namespace grim::lm;
    if (!policy) return GRIM_ERR_NULL;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    const bool learns = loss_dev || dz_dev;
    if (N < 0 || N > kMostRows || V < 1 || V >= (int64_t)1 << 31 || ldz < V || (dz_dev && lddz < V) || !fits(N, ldz) || (dz_dev && !fits(N, lddz)) ||
        !(policy->temperature >= 1e-30f) || policy->temperature > 1e30f)
        return GRIM_ERR_SHAPE;
    if (learns && (!(policy->clip_low >= 0.f) || policy->clip_low > 1.f || !(policy->clip_high >= 0.f) || policy->clip_high > 3e38f ||
                   !(policy->kl >= 0.f) || policy->kl > 3e38f))
        return GRIM_ERR_SHAPE;
    if (N == 0) return GRIM_OK;
    if (!z_dev || !policy->ids || (learns && !policy->advantage) || (!learns && !logp_dev) || !workspace) return GRIM_ERR_NULL;
    if (moves(z_dev, ldz, dz_dev, lddz, N)) return GRIM_ERR_SHAPE;
    if (workspace_bytes < grim_policy_loss_workspace(N, V)) return GRIM_ERR_SHAPE;
    const PolicyParams p{z_dev, policy->ids, policy->old_logp, policy->ref_logp, policy->advantage, policy->weight, loss_dev, logp_dev, dz_dev,
                         static_cast<float *>(workspace), ldz, lddz, V, 0, policy->temperature, 1.44269504088896340736f / policy->temperature,
                         1.f - policy->clip_low, 1.f + policy->clip_high, policy->kl, past_caches((dz_dev ? 2 : 1) * N * V * bytes_of(dt))};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dt == GRIM_F32   ? policy_typed<float>(p, N, stream)
           : dt == GRIM_F16 ? policy_typed<f16>(p, N, stream)
                            : policy_typed<bf16>(p, N, stream);
}

}  // extern "C"
