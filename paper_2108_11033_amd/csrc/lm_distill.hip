// Distillation from a teacher's top logits: loss and gradient in one pass over the student's logits.
//
//     p = softmax(top / tau) over the listed entries    q = softmax(z / tau) over all V
//     loss = w tau^2 sum_i p_i (log p_i - log q[id_i])    dz_j = w tau (q_j - sum of p_i with id_i = j)
//
// Bound by memory: z read once, dz written once.  Where the rows fill the compute units a workgroup keeps its row in registers
// between the maximum, the sum and the gradient.  With few rows, or rows that do not fit, a row is cut into slices: a first launch
// leaves every slice's maximum, sum and share of the loss, and the second joins them and writes the gradient from a second
// read of z, which a few rows leave in the caches.  Exponents are taken of differences from the maximum, (z - max) / tau, so that
// masks of the type's lowest value do not overflow on the way.  The loss is summed as
//     w tau sum_i p_i ((top_i - best) - (z_i - max) + tau (log sum_z - log sum_top))
// whose terms stay numbers where tau^2, or a difference over tau, is none.  Measured: 8192 x 32768 bf16 with 64 listed words 216 us (5.0 TB/s, a copy's
// rate), 24 x 131075 fp16 in slices 12 (two launches), 1024 x 1000 fp32 5.6.
#include "lm_rows.hpp"

namespace grim {
namespace lm {

constexpr int kMostEntries = 1024;

struct DistillParams {
    const void *z;
    const float *top, *weight;
    const int32_t *ids;
    float *loss;
    void *dz;
    float *part;                // [row][slice][maximum, sum, share of the loss / (w tau), probability listed in it]
    int64_t ldz, lddz, ldt, N, V;
    int32_t k, slices;
    float tau, scale;           // scale = log2(e) / tau
    bool past;                  // (not with many listed words, which are written a second time: 4000 x 32768 bf16 with 256 of
                                // them 133 us past the caches and 129 through them, with 65 112 and 116)
};

// The teacher's side of a row in LDS, with room for E entries: words (-1: absent), probabilities, the sums of the probabilities of
// entries that list the same word, below = top - best (log2 p is that times scale, less log2(total)), and z at the words.
template <int E>
struct Entries {
    static constexpr int kBits = E <= 64 ? 11 : 13;
    int32_t id[E];
    float p[E], sum[E], below[E], z[E];
    uint16_t table[1 << kBits];
    float total;                // sum of exponentials (0: nothing is listed; NaN: a listed logit is)
    // (two multiplications with a shift between them: words in even steps spread, whatever the step)
    static __device__ __forceinline__ int slot(int32_t id, uint32_t turn) {
        uint32_t h = ((uint32_t)id + turn) * 2654435761u;
        h = (h ^ h >> 15) * 0xa3d95fa7u;
        return (int)((h ^ h >> 14) >> (32 - kBits));
    }
};

// Formed by one wave.  The words lo .. hi - 1 get their z, others the word -1.  SUMS: words listed twice are looked for.
template <bool SUMS, int E, typename T>
__device__ __forceinline__ void teacher(const DistillParams &p, int64_t n, const T *z, int64_t lo, int64_t hi, Entries<E> &e) {
    const int lane = threadIdx.x & 63;
    const float *t = p.top + n * p.ldt;
    const int32_t *ids = p.ids + n * p.ldt;
    float m = -INFINITY;
    bool nan = false;
    // (up to 256 entries asked for at once, then their words: two waits for memory.  24 x 131075 fp16 in slices, 1000 listed words 32.9 us
    // against 34.7 one by one, and 28.2 since a slice leaves out the others' words here)
    constexpr int B = E < 256 ? E / 64 : 4;
    for (int i0 = lane; i0 < p.k; i0 += 64 * B) {
        int32_t id[B];
        float listed[B], z_at[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int i = i0 + 64 * b < p.k ? i0 + 64 * b : 0;
            id[b] = ids[i], listed[b] = t[i];
        }
#pragma unroll
        for (int b = 0; b < B; ++b) z_at[b] = (float)z[id[b] >= lo && id[b] < hi ? id[b] : lo];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int i = i0 + 64 * b;
            if (i >= p.k) break;
            const bool here = id[b] >= lo && id[b] < hi;
            const float v = id[b] >= 0 && id[b] < p.V ? listed[b] : -INFINITY;
            e.z[i] = here ? z_at[b] : 0.f;
            e.id[i] = here ? id[b] : -1;
            e.below[i] = v;
            nan |= v != v;
            m = fmaxf(m, v);
        }
    }
    m = wave_max(m);
    if (__any(nan)) m = NAN;
    float s = 0.f;
    for (int i = lane; i < p.k; i += 64) {
        const float v = e.below[i];
        const float d = v - m;                              // (of no use where p is 0)
        const float x = v == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(d * p.scale);
        e.below[i] = d;
        e.p[i] = x;
        s += x;
    }
    s = wave_sum(s);
    if (lane == 0) e.total = s;
    const float r = 1.f / s;
    for (int i = lane; i < p.k; i += 64) {
        const float x = s > 0.f ? e.p[i] * r : s;                        // (s: 0, or NaN)
        e.p[i] = x;
        if (SUMS) e.sum[i] = x;
    }
    if (!SUMS) return;
    // Words listed twice.  Every entry leaves its number in a table at its word's hash; one that finds another's there either
    // lists the same word, or takes part in a second turn with another hash.  Who then finds another's number once more, or has
    // found its own word, is looked up by the whole wave.  (Entries that list one word meet in the turn that they reach together.)
    const auto leave = [&](uint32_t turn, uint32_t who) {
        for (int i = lane, c = 0; i < p.k; i += 64, ++c)
            if (who >> c & 1 && e.id[i] >= 0) e.table[e.slot(e.id[i], turn)] = (uint16_t)i;
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
    };
    uint32_t again = 0, look = 0;                           // bit c: the lane's entry lane + 64 c
    leave(0, ~0u);
    for (int i = lane, c = 0; i < p.k; i += 64, ++c) {
        const int32_t id = e.id[i];
        const int other = id >= 0 ? e.table[e.slot(id, 0)] : i;
        if (other != i) (e.id[other] == id ? look : again) |= 1u << c;
    }
    __builtin_amdgcn_wave_barrier();
    __threadfence_block();
    if (__any(again != 0)) {
        leave(1, again);
        for (int i = lane, c = 0; i < p.k; i += 64, ++c)
            if (again >> c & 1 && e.table[e.slot(e.id[i], 1)] != i) look |= 1u << c;
    }
    for (int i0 = 0, c = 0; i0 < p.k; i0 += 64, ++c) {
        const int32_t id = i0 + lane < p.k ? e.id[i0 + lane] : -1;
        unsigned long long left = __ballot(look >> c & 1);
        while (left) {
            const int l = __builtin_ctzll(left);
            left &= left - 1;
            const int32_t word = __shfl(id, l, 64);
            float sum = 0.f;
            for (int j = lane; j < p.k; j += 64) sum += e.id[j] == word ? e.p[j] : 0.f;
            sum = wave_sum(sum);
            for (int j = lane; j < p.k; j += 64)
                if (e.id[j] == word) e.sum[j] = sum;
        }
    }
}

// weight tau (q_j - p_j) at the listed words, over what was streamed there.
template <int E, typename T>
__device__ __forceinline__ void write_listed(const DistillParams &p, const Entries<E> &e, T *dz, float peak, float rsum, float factor,
                                             int64_t lo, int64_t hi) {
    for (int i = threadIdx.x; i < p.k; i += blockDim.x) {
        const int32_t id = e.id[i];
        if (id >= lo && id < hi) dz[id] = (T)(factor * (__builtin_amdgcn_exp2f((e.z[i] - peak) * p.scale) * rsum - e.sum[i]));
    }
}

// -------------------------------------------------------------------------------------------------- one workgroup per row
// W waves hold the row, at most PER pieces of 16 bytes a thread: pieces k < full are whole for all threads, piece `full` for
// some, the others are empty.  A piece that reaches past the row is moved back to end with it; what it shares counts in
// the other.  One wave more forms the teacher's side meanwhile: its chain of loads and small reductions is as long as the row's own.
template <typename T, int E, int W, int PER>
__global__ void __launch_bounds__(64 * (W + 1)) distill_rows(DistillParams p) {
    constexpr int V = piece<T>(), TPR = 64 * W;
    __shared__ Entries<E> e;
    __shared__ float room[2][W];
    const int64_t n = blockIdx.x;
    const T *z = static_cast<const T *>(p.z) + n * p.ldz;
    T *dz = p.dz ? static_cast<T *>(p.dz) + n * p.lddz : nullptr;
    const float weight = p.weight ? p.weight[n] : 1.f;
    if (weight == 0.f) {
        if (threadIdx.x == 0) p.loss[n] = 0.f;
        if (dz) zero_row(dz, 0, p.V);
        return;
    }
    const bool aside = threadIdx.x >= TPR;
    const int full = (int)(p.V / (TPR * V));
    const int mine = full * TPR * V + (int)threadIdx.x * V;   // where piece `full` would start
    const bool some = !aside && mine < p.V;
    const int tail = (int)min((int64_t)mine, p.V - V), first = mine - tail;
    Pack<T, V> raw[PER];
    float peak = -INFINITY, sum = 0.f;
    if (aside) {
        teacher<true>(p, n, z, 0, p.V, e);
        __syncthreads();
        if (W > 1) __syncthreads();
        for (int w = 0; w < W; ++w) peak = fmaxf(peak, room[0][w]), sum += room[1][w];
    } else {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (k < full) raw[k] = load<V>(z + k * TPR * V + (int)threadIdx.x * V);
            else if (k == full && some) raw[k] = load<V>(z + tail);
        }
        // f(value) over the thread's own elements
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
        own([&](float v) { peak = fmaxf(peak, v); });
        peak = group_max<W>(peak, room[0]);
        own([&](float v) { sum += __builtin_amdgcn_exp2f((v - peak) * p.scale); });
        sum = group_sum<W>(sum, room[1]);                   // (its barrier also shows the teacher's side to all)
        if (W == 1) {                                       // (one wave: no barrier in either)
            room[0][0] = peak, room[1][0] = sum;
            __syncthreads();
        }
    }
    const float total = e.total;
    if (total == 0.f) {
        if (threadIdx.x == 0) p.loss[n] = 0.f;
        if (dz) zero_row(dz, 0, p.V);
        return;
    }
    const float rsum = 1.f / sum;
    const float factor = weight * p.tau * (total / total);  // (a NaN of the teacher reaches the whole row)
    if (aside) {
        const float lse = p.tau * (kLn2 * log2f(sum)), ltotal = p.tau * (kLn2 * log2f(total));
        float loss = 0.f;
        for (int i = threadIdx.x & 63; i < p.k; i += 64)
            if (e.p[i] != 0.f) loss += e.p[i] * ((e.below[i] - ltotal) - ((e.z[i] - peak) - lse));
        loss = wave_sum(loss);
        if (threadIdx.x == TPR) p.loss[n] = weight * p.tau * loss;
    } else if (dz) {
        const float slope = factor * rsum;
        store_rows(p.past, [&](auto past) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                if (k > full || (k == full && !some)) continue;
                float v[V], out[V];
                forget(raw[k]);
                unpack(raw[k], v);
#pragma unroll
                for (int j = 0; j < V; ++j) out[j] = slope * __builtin_amdgcn_exp2f((v[j] - peak) * p.scale);
                store<past.value>(dz + (k < full ? k * TPR * V + (int)threadIdx.x * V : tail), out);
            }
        });
    }
    if (!dz) return;
    __syncthreads();                                        // the listed words' places were written by other threads
    write_listed(p, e, dz, peak, rsum, factor, 0, p.V);
}

// -------------------------------------------------------------------------------------------------- slices of rows
// (kSliceWaves waves take the slice, one more the teacher's side meanwhile)
template <typename T, int E>
__global__ void __launch_bounds__(64 * (kSliceWaves + 1)) distill_slices(DistillParams p) {
    constexpr int V = piece<T>(), W = kSliceWaves;
    __shared__ Entries<E> e;
    __shared__ float room[2][W];
    const int64_t n = blockIdx.x / p.slices, s = blockIdx.x % p.slices;
    if (p.weight && p.weight[n] == 0.f) return;
    const T *z = static_cast<const T *>(p.z) + n * p.ldz;
    const int64_t lo = s * slice_elements<T>(), hi = lo + slice_elements<T>() < p.V ? lo + slice_elements<T>() : p.V;
    if (threadIdx.x >= 64 * W) {
        const int lane = threadIdx.x & 63;
        teacher<false>(p, n, z, lo, hi, e);
        __syncthreads();
        __syncthreads();
        float peak = -INFINITY, sum = 0.f;
        for (int w = 0; w < W; ++w) peak = fmaxf(peak, room[0][w]), sum += room[1][w];
        // (a slice of nothing but -infinity has the sum 0; one NaN makes the sum NaN)
        const float base = peak == -INFINITY ? 0.f : peak;
        // sum of p ((top - best) - (z - peak)) over the words in this slice, and of p
        float share = 0.f, there = 0.f;
        for (int i = lane; i < p.k; i += 64) {
            const int32_t id = e.id[i];
            if (id >= lo && id < hi && e.p[i] != 0.f) {
                share += e.p[i] * (e.below[i] - (e.z[i] - base));
                there += e.p[i];
            }
        }
        share = wave_sum(share);
        there = wave_sum(there);
        if (lane == 0) {
            float *part = p.part + (int64_t)blockIdx.x * 4;
            part[0] = peak, part[1] = sum, part[2] = share, part[3] = there;
        }
        return;
    }
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
    const float base = peak == -INFINITY ? 0.f : peak;
#pragma unroll
    for (int k = 0; k < kSlicePer; ++k) {
        float v[V];
        forget(sl.raw[k]);
        unpack(sl.raw[k], v);
#pragma unroll
        for (int j = 0; j < V; ++j) sum += __builtin_amdgcn_exp2f((v[j] - base) * p.scale);
    }
    group_sum<W>(sum, room[1]);
}

template <typename T, int E>
__global__ void __launch_bounds__(64 * (kSliceWaves + 1)) distill_join(DistillParams p) {
    constexpr int V = piece<T>(), W = kSliceWaves;
    __shared__ Entries<E> e;
    const int64_t n = blockIdx.x / p.slices, s = blockIdx.x % p.slices;
    const T *z = static_cast<const T *>(p.z) + n * p.ldz;
    T *dz = p.dz ? static_cast<T *>(p.dz) + n * p.lddz : nullptr;
    const int64_t lo = s * slice_elements<T>(), hi = lo + slice_elements<T>() < p.V ? lo + slice_elements<T>() : p.V;
    const float weight = p.weight ? p.weight[n] : 1.f;
    const int lane = threadIdx.x & 63;
    const bool aside = threadIdx.x >= 64 * W;
    const Slice<T> sl(z, lo, aside ? lo : hi);
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
    if (weight == 0.f) {
        if (threadIdx.x == 0 && s == 0) p.loss[n] = 0.f;
        if (dz) zero_row(dz, lo, hi);
        return;
    }
    if (aside) {
        // (z of this slice only: other slices' places may hold their gradient already, where dz is z)
        teacher<true>(p, n, z, lo, hi, e);
        if (s == 0) {
            // z - max = (z - base_i) + (base_i - peak)
            const float extra = p.tau * (kLn2 * (log2f(sum) - log2f(e.total)));
            float share = 0.f;
            for (int i = lane; i < p.slices; i += 64) {
                const float base = part[4 * i] == -INFINITY ? 0.f : part[4 * i], there = part[4 * i + 3];
                if (there != 0.f) share += part[4 * i + 2] + there * ((peak - base) + extra);
            }
            share = wave_sum(share);
            if (lane == 0) p.loss[n] = e.total == 0.f ? 0.f : weight * p.tau * share;
        }
    }
    if (!dz) return;
    const float rsum = 1.f / sum;
    float v[kSlicePer][V];
#pragma unroll
    for (int k = 0; k < kSlicePer; ++k) {
        unpack(sl.raw[k], v[k]);
#pragma unroll
        for (int j = 0; j < V; ++j) v[k][j] = rsum * __builtin_amdgcn_exp2f((v[k][j] - peak) * p.scale);
    }
    __syncthreads();                                        // (also: the words of this slice were read before it is written)
    const float total = e.total;
    if (total == 0.f) {
        zero_row(dz, lo, hi);
        return;
    }
    const float factor = weight * p.tau * (total / total);
    if (!aside) {
#pragma unroll
        for (int k = 0; k < kSlicePer; ++k) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[k][j] *= factor;
            T *to = dz + Slice<T>::at(lo, k);
            if (sl.have[k] == V) store(to, v[k]);
            else
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (j < sl.have[k]) to[j] = (T)v[k][j];
        }
    }
    __syncthreads();
    write_listed(p, e, dz, peak, rsum, factor, lo, hi);
}

// -------------------------------------------------------------------------------------------------- launches
// A workgroup per row where its registers hold the row: 18 pieces a thread of 15 waves.
template <typename T>
bool row_fits(int64_t V) { return V >= piece<T>() && V <= (int64_t)18 * 960 * piece<T>(); }

// Rows of up to 128 KB do so however few they are (100 x 32768 fp32 16.9 us against 20.1 in slices, 64 x 9000 7.0 against 10.1), longer ones
// if half of the compute units have one (62 x 90880 bf16 18.6 us against 14.5 in slices, 100 x 131072 28 against 22.5).
template <typename T>
bool by_rows(int64_t N, int64_t V) { return row_fits<T>(V) && (N >= 128 || V * (int64_t)sizeof(T) <= 128 * 1024); }

// Rows first .. first + count - 1 of a call.
template <typename T>
DistillParams rows_of(DistillParams p, int64_t first, int64_t count) {
    p.z = static_cast<const T *>(p.z) + first * p.ldz;
    p.top += first * p.ldt, p.ids += first * p.ldt;
    p.weight = ahead(p.weight, first);
    p.loss += first;
    p.dz = ahead(static_cast<T *>(p.dz), first * p.lddz);
    p.part += first * p.slices * 4;
    p.N = count;
    return p;
}

template <typename T, int E>
grim_status distill_launch(DistillParams call, hipStream_t stream) {
    if (by_rows<T>(call.N, call.V)) {
        const int64_t pieces = (call.V + piece<T>() - 1) / piece<T>();
        // 2, 4, 8 or 16 waves with the teacher's.  Short rows are bound by their workgroups' waves: 7180 x 512 bf16 8.5 us with 2 waves, 14.0
        // with 4; 20000 x 1000 fp32 30.4 and 38.6, 256 x 2000 bf16 6.8 and 6.6.  Long rows take 16 where a compute unit has one row, very long
        // ones where it has two (300 x 32768 fp32 19.3 us against 26.7 with 8, 269 x 19445 bf16 12.8 against 11.5, 512 x 32768 bf16 24.4 against 22.5).
        const bool many = call.N > (pieces > 4480 ? 2 : 1) * kComputeUnits;
        const auto launch = [&](auto kernel, int threads) {
            return in_runs(call.N, most_groups(threads), [&](int64_t first, int64_t count) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(threads), 0, stream, rows_of<T>(call, first, count));
                return launched();
            });
        };
        if (pieces <= 128) return launch(distill_rows<T, E, 1, 2>, 128);
        if (pieces <= 256) return launch(distill_rows<T, E, 1, 4>, 128);
        if (pieces <= 384) return launch(distill_rows<T, E, 3, 2>, 256);
        if (pieces <= 768) return launch(distill_rows<T, E, 3, 4>, 256);
        if (pieces <= 1792) return launch(distill_rows<T, E, 7, 4>, 512);
        if (!many && pieces <= 3840) return launch(distill_rows<T, E, 15, 4>, 1024);
        if (!many && pieces <= 9600) return launch(distill_rows<T, E, 15, 10>, 1024);
        if (pieces <= 2688) return launch(distill_rows<T, E, 7, 6>, 512);
        if (pieces <= 4480) return launch(distill_rows<T, E, 7, 10>, 512);
        if (pieces <= 8064) return launch(distill_rows<T, E, 7, 18>, 512);
        return launch(distill_rows<T, E, 15, 18>, 1024);
    }
    call.slices = (int32_t)slices_of<T>(call.V);
    constexpr int threads = 64 * (kSliceWaves + 1);
    return in_runs(call.N, most_groups(threads) / call.slices, [&](int64_t first, int64_t count) {
        const DistillParams p = rows_of<T>(call, first, count);
        const dim3 g((unsigned)(p.N * p.slices)), b(threads);
        hipLaunchKernelGGL((distill_slices<T, E>), g, b, 0, stream, p);
        const grim_status st = launched();
        if (st != GRIM_OK) return st;
        hipLaunchKernelGGL((distill_join<T, E>), g, b, 0, stream, p);
        return launched();
    });
}

// (room for 64 entries where they suffice: workgroups share a compute unit by their LDS)
template <typename T>
grim_status distill_typed(const DistillParams &p, hipStream_t stream) {
    return p.k <= 64 ? distill_launch<T, 64>(p, stream) : distill_launch<T, kMostEntries>(p, stream);
}

}  // namespace lm
}  // namespace grim

extern "C" {

int64_t grim_distill_topk_workspace(int64_t N, int64_t V) {
    using namespace grim::lm;
    if (N < 0 || N > kMostRows || V < 1 || V >= (int64_t)1 << 31) return 0;
    // (whichever type comes: of fp32 a slice holds the fewest elements)
    int64_t bytes = 16;
    if (!by_rows<float>(N, V)) bytes += N * slices_of<float>(V) * 16;
    else if (!by_rows<f16>(N, V)) bytes += N * slices_of<f16>(V) * 16;
    return bytes;
}

grim_status grim_distill_topk(const void *z_dev, grim_dtype dt, int64_t ldz, const float *top_logits_dev,
                              const int32_t *top_ids_dev, int32_t k, int64_t ldt, float temperature,
                              const float *weight_dev, int64_t N, int64_t V, float *loss_dev, void *dz_dev, int64_t lddz,
                              void *workspace, int64_t workspace_bytes, void *hip_stream) {
    using namespace grim::lm;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if (N < 0 || N > kMostRows || V < 1 || V >= (int64_t)1 << 31 || k < 1 || ldz < V || ldt < k || (dz_dev && lddz < V) || !fits(N, ldz) ||
        !fits(N, ldt) || (dz_dev && !fits(N, lddz)) || !(temperature >= 1e-30f) || temperature > 1e30f)
        return GRIM_ERR_SHAPE;
    if (k > kMostEntries) return GRIM_ERR_UNSUPPORTED;
    if (N == 0) return GRIM_OK;
    if (!z_dev || !top_logits_dev || !top_ids_dev || !loss_dev || !workspace) return GRIM_ERR_NULL;
    if (moves(z_dev, ldz, dz_dev, lddz, N)) return GRIM_ERR_SHAPE;
    if (workspace_bytes < grim_distill_topk_workspace(N, V)) return GRIM_ERR_SHAPE;
    const DistillParams p{z_dev, top_logits_dev, weight_dev, top_ids_dev, loss_dev, dz_dev, static_cast<float *>(workspace),
                          ldz, lddz, ldt, N, V, k, 0, temperature, 1.44269504088896340736f / temperature,
                          k <= 128 && past_caches(2 * N * V * bytes_of(dt))};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dt == GRIM_F32   ? distill_typed<float>(p, stream)
           : dt == GRIM_F16 ? distill_typed<f16>(p, stream)
                            : distill_typed<bf16>(p, stream);
}

}  // extern "C"
