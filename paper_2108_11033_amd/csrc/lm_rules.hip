// Rules applied to the logits of a served step: penalties for words of the history, biases, a grammar's mask.
//
//     z -> (z > 0 ? z / repetition : z repetition) - frequency count - presence      where count > 0
//     z -> z + bias    z -> -infinity where the word is not allowed
//
// One pass over the logits, bound by memory or, for a caller or two, by the launch.  A workgroup takes a tile of words and
// callers, counts the histories' words that fall into it in LDS (whole-number atomics: the order cannot matter), and then
// transforms the tile.  Every tile reads its callers' whole histories again (from L2), which costs less than a table of counts in
// memory, cleared, filled and read by three launches.  A word's place in LDS holds its count and, above it, the entry of the bias list
// that adds to it: four bytes a word, so that a compute unit holds four tiles of 8192.  Measured: 64 callers x 131072 words bf16 12.6 us (9.7
// without any rule, a copy 5.9: the phases of one round of workgroups follow each other), one caller x 32768 words 4.5 us of kernel.
#include "lm_common.hpp"

namespace grim {
namespace lm {

constexpr int kMostBias = 1024, kCountBits = 21;              // counts up to 2^21, entries 1 .. 1024
constexpr int32_t kMostHistory = 1 << 20;

struct RuleParams {
    const void *z;
    void *out;
    int64_t ldz, ldo, V;
    int32_t batch;
    grim_logit_rules r;
};

struct CallerRules {
    float repetition, inverse, frequency, presence;
    __device__ __forceinline__ CallerRules(const grim_logit_rules &r, int64_t b)
        : repetition(r.repetition ? r.repetition[b] : 1.f), frequency(r.frequency ? r.frequency[b] : 0.f),
          presence(r.presence ? r.presence[b] : 0.f) {
        inverse = 1.f / repetition;             // (a product for a division: one rounding of 2^-24 more)
    }
    // place: the word's place in LDS; biases: the end of the entries' sums.  Most words are in no list: the arithmetic is skipped where that holds
    // for all of a wave's.
    __device__ __forceinline__ float apply(float z, uint32_t place, const float *biases, bool allowed) const {
        if (__any(place != 0)) {
            const uint32_t count = place & ((1u << kCountBits) - 1), entry = place >> kCountBits;
            const float said = z * (z > 0.f ? inverse : repetition) - frequency * (float)count - presence;
            z = count ? said : z;
            if (entry) z += biases[-(int)entry];
        }
        return allowed ? z : -INFINITY;
    }
};

// A caller's history, walked by a team of `width` threads (this one is number t): its length and the first eight words of each
// thread are asked for before anything else (up to the most that a history may hold, so that they need not wait for the length).
struct History {
    const int32_t *h;
    int most, len, t, width;
    int32_t early[2][4];
    __device__ __forceinline__ History(const grim_logit_rules &r, int64_t b, int t_, int width_) : t(t_), width(width_) {
        most = r.history ? r.max_history : 0;
        h = r.history + b * r.ld_history;
        len = most > 0 && r.history_len ? min(max(r.history_len[b], 0), most) : most;
        take(t * 4, early[0]);
        take((width + t) * 4, early[1]);
    }
    __device__ __forceinline__ void take(int i, int32_t (&ids)[4]) const {
        if (i + 4 <= most) {
            const Pack<int32_t, 4> p = load<4>(h + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) ids[j] = (int32_t)p.w[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) ids[j] = i + j < most ? h[i + j] : -1;
        }
    }
    // Counts words lo .. lo + span - 1 at places[(word - lo) << shift].
    __device__ __forceinline__ void tally(int lo, int span, uint32_t *places, int shift) {
        const auto count = [&](int i, const int32_t (&ids)[4]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // (a word below lo wraps around to a large number; words of 2^31 and more do not exist)
                const uint32_t at = (uint32_t)ids[j] - (uint32_t)lo;
                if (i + j < len && ids[j] >= 0 && at < (uint32_t)span) atomicAdd(&places[at << shift], 1u);
            }
        };
        count(t * 4, early[0]);
        count((width + t) * 4, early[1]);
        constexpr int kAhead = 4;                               // loads on their way together: a long history is a chain of them
        for (int i = (2 * width + t) * 4; i < len; i += kAhead * width * 4) {
            int32_t ids[kAhead][4];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) take(i + k * width * 4, ids[k]);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) count(i + k * width * 4, ids[k]);
        }
    }
};

// A caller's biases, by thread t of `width`; the first two entries of each thread are asked for early.  Two steps, each behind a
// barrier: a place gets nbias - i for the first entry i of its word, by a maximum, before anything is counted there, and sums[i] the
// entry's value; and where `twice` says that a word of the tile is listed again, first entries add up their words' in the list's order.
// (43 callers x 18112 words fp32 in columns with 126 entries 8.5 us; 15.9 with every entry held against the whole list.)
struct Biases {
    const int32_t *ids;
    const float *values;
    int n, t, width;
    int32_t id[2];
    float value[2];
    __device__ __forceinline__ Biases(const grim_logit_rules &r, int64_t b, int t_, int width_)
        : ids(r.bias_ids + b * r.ld_bias), values(r.bias_values + b * r.ld_bias), n(r.nbias), t(t_), width(width_) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = t + k * width;
            id[k] = i < n ? ids[i] : -1;
            value[k] = i < n ? values[i] : 0.f;
        }
    }
    // f(entry, which of the thread's it is, word, its distance from lo) for the entries of words lo .. lo + span - 1
    template <typename F>
    __device__ __forceinline__ void each(int lo, int span, F f) const {
        for (int i = t, k = 0; i < n; i += width, ++k) {
            const int32_t word = k == 0 ? id[0] : k == 1 ? id[1] : ids[i];
            const uint32_t at = (uint32_t)word - (uint32_t)lo;
            if (word >= 0 && at < (uint32_t)span) f(i, k, word, at);
        }
    }
    __device__ __forceinline__ void place(int lo, int span, uint32_t *places, int shift, float *sums, int *twice) const {
        each(lo, span, [&](int i, int k, int32_t, uint32_t at) {
            sums[i] = k == 0 ? value[0] : k == 1 ? value[1] : values[i];
            if (atomicMax(&places[at << shift], (uint32_t)(n - i) << kCountBits)) *twice = 1;
        });
    }
    __device__ __forceinline__ void join(int lo, int span, const uint32_t *places, int shift, float *sums) const {
        each(lo, span, [&](int i, int, int32_t word, uint32_t at) {
            if (places[at << shift] >> kCountBits != (uint32_t)(n - i)) return;
            float sum = values[i];
#pragma unroll 8
            for (int j = i + 1; j < n; ++j)
                if (ids[j] == word) sum += values[j];
            sums[i] = sum;
        });
    }
};

// A row per caller: TILE words of one caller.  Everything that a tile reads is asked for at its start.
template <typename T, int TILE, int THREADS>
__global__ void __launch_bounds__(THREADS) rules_rows(RuleParams p, int tiles) {
    constexpr int V = 16 / (int)sizeof(T), PER = TILE / (THREADS * V);
    __shared__ __attribute__((aligned(16))) uint32_t places[TILE];
    __shared__ float sums[kMostBias];
    __shared__ int twice;
    const int64_t b = blockIdx.x / tiles, lo = (int64_t)(blockIdx.x % tiles) * TILE;
    const int64_t hi = lo + TILE < p.V ? lo + TILE : p.V;
    const T *z = static_cast<const T *>(p.z) + b * p.ldz + lo;
    T *out = static_cast<T *>(p.out) + b * p.ldo + lo;
    const int span = (int)(hi - lo);
    History history(p.r, b, threadIdx.x, THREADS);
    const Biases biases(p.r, b, threadIdx.x, THREADS);
    const CallerRules rules(p.r, b);
    const uint32_t *allowed = p.r.allowed ? p.r.allowed + b * p.r.ld_allowed + lo / 32 : nullptr;
    Pack<T, V> raw[PER];
    uint32_t bits[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = (k * THREADS + threadIdx.x) * V;
        if (c + V <= span) raw[k] = load<V>(z + c);
        else
#pragma unroll
            for (int j = 0; j < V; ++j) put(raw[k], j, c + j < span ? z[c + j] : (T)0.f);
        bits[k] = allowed && c < span ? allowed[c / 32] >> (c % 32) : 0xffffffffu;
    }
    const bool lists = history.most > 0 || p.r.nbias > 0;       // (a mask alone needs no places)
    if (lists) {
        for (int i = threadIdx.x; i < TILE / 4; i += THREADS) reinterpret_cast<uint4 *>(places)[i] = uint4{0, 0, 0, 0};
        if (threadIdx.x == 0) twice = 0;
        __syncthreads();
        if (p.r.nbias > 0) {
            biases.place((int)lo, span, places, 0, sums, &twice);
            __syncthreads();
            if (twice) biases.join((int)lo, span, places, 0, sums);
        }
        history.tally((int)lo, span, places, 0);
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = (k * THREADS + threadIdx.x) * V;
        if (c >= span) continue;
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = rules.apply(element(raw[k], j), lists ? places[c + j] : 0, sums + p.r.nbias, bits[k] >> j & 1);
        if (c + V <= span) store(out + c, v);
        else
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c + j < span) out[c + j] = (T)v[j];
    }
}

// A column per caller: TILE >> shift words of up to 1 << shift (at most kMostCallers) callers.  32 callers x 32768 words bf16 6.0 us of kernel,
// 64 x 50000 13.8, 64 x 131072 with all rules 24 to 29: with more than eight callers a line of logits is read and written in parts.
constexpr int kMostCallers = 8;

template <typename T, int TILE, int THREADS, int BIAS>
__global__ void __launch_bounds__(THREADS) rules_columns(RuleParams p, int tiles, int shift) {
    constexpr int PER = TILE / THREADS;
    __shared__ __attribute__((aligned(16))) uint32_t places[TILE];
    __shared__ float sums[kMostCallers][BIAS];
    __shared__ int twice[kMostCallers];
    const int words = TILE >> shift;
    const int64_t b0 = (int64_t)(blockIdx.x / tiles) << shift, lo = (int64_t)(blockIdx.x % tiles) * words;
    const int64_t hi = lo + words < p.V ? lo + words : p.V;
    const int span = (int)(hi - lo), callers = (int)min((int64_t)1 << shift, p.batch - b0);
    // (THREADS is a multiple of 1 << shift: a thread keeps its caller)
    const int mine = min((int)threadIdx.x & ((1 << shift) - 1), callers - 1);
    const bool live = ((int)threadIdx.x & ((1 << shift) - 1)) < callers;
    const CallerRules rules(p.r, b0 + mine);
    const uint32_t *allowed = p.r.allowed ? p.r.allowed + (b0 + mine) * p.r.ld_allowed : nullptr;
    const T *z = static_cast<const T *>(p.z) + b0 + mine;
    T *out = static_cast<T *>(p.out) + b0 + mine;
    // a few words a thread are asked for at the start; more would keep other workgroups from the compute unit
    constexpr bool early = PER <= 4;
    constexpr int STEP = early ? PER : 4;
    float v[STEP];
    uint32_t bits[STEP];
    auto fetch = [&](int k0) {
#pragma unroll
        for (int k = 0; k < STEP; ++k) {
            const int at = ((k0 + k) * THREADS + (int)threadIdx.x) >> shift;
            const int64_t word = lo + min(at, span - 1);
            v[k] = (float)z[word * p.ldz];
            bits[k] = allowed ? allowed[word / 32] >> (word % 32) : 1u;
        }
    };
    // as many waves per caller as there are
    static_assert(THREADS / 64 >= kMostCallers, "a wave per caller");
    const int each = THREADS / 64 >> shift, wave = threadIdx.x >> 6, b = wave / each;
    const int t = (wave % each) * 64 + (threadIdx.x & 63), width = each * 64;
    const bool lists = b < callers;
    const int64_t own = b0 + (lists ? b : 0);
    History history(p.r, own, t, width);
    const Biases biases(p.r, own, t, width);
    if (early) fetch(0);
    for (int i = threadIdx.x; i < TILE / 4; i += THREADS) reinterpret_cast<uint4 *>(places)[i] = uint4{0, 0, 0, 0};
    if (threadIdx.x < kMostCallers) twice[threadIdx.x] = 0;
    __syncthreads();
    if (p.r.nbias > 0) {
        if (lists) biases.place((int)lo, span, places + b, shift, sums[b], &twice[b]);
        __syncthreads();
        if (lists && twice[b]) biases.join((int)lo, span, places + b, shift, sums[b]);
    }
    if (lists) history.tally((int)lo, span, places + b, shift);
    __syncthreads();
    for (int k0 = 0; k0 < PER; k0 += STEP) {
        if (!early) fetch(k0);
#pragma unroll
        for (int k = 0; k < STEP; ++k) {
            const int i = (k0 + k) * THREADS + (int)threadIdx.x, at = i >> shift;
            if (live && at < span) out[(lo + at) * p.ldo] = (T)rules.apply(v[k], places[i], sums[mine] + p.r.nbias, bits[k] & 1);
        }
    }
}

// Callers first .. first + count - 1 of a call.
template <typename T>
RuleParams callers_of(RuleParams p, bool columns, int64_t first, int64_t count) {
    p.z = static_cast<const T *>(p.z) + first * (columns ? 1 : p.ldz);
    p.out = static_cast<T *>(p.out) + first * (columns ? 1 : p.ldo);
    p.r.history = ahead(p.r.history, first * p.r.ld_history);
    p.r.history_len = ahead(p.r.history_len, first);
    p.r.repetition = ahead(p.r.repetition, first);
    p.r.frequency = ahead(p.r.frequency, first);
    p.r.presence = ahead(p.r.presence, first);
    p.r.bias_ids = ahead(p.r.bias_ids, first * p.r.ld_bias);
    p.r.bias_values = ahead(p.r.bias_values, first * p.r.ld_bias);
    p.r.allowed = ahead(p.r.allowed, first * p.r.ld_allowed);
    p.batch = (int32_t)count;
    return p;
}

template <typename T, int TILE, int THREADS, bool COLUMNS>
grim_status rules_launch(const RuleParams &call, hipStream_t stream) {
    int shift = 0;
    if (COLUMNS)
        while ((1 << shift) < kMostCallers && (1 << shift) < call.batch) ++shift;    // 16 or 32 bytes of a row
    const int64_t words = TILE >> shift, tiles = (call.V + words - 1) / words;       // (up to 2^21: a launch has room for one block's)
    return in_runs(call.batch, most_groups(THREADS) / tiles << shift, [&](int64_t first, int64_t count) {
        const RuleParams p = callers_of<T>(call, COLUMNS, first, count);
        const dim3 g((unsigned)(tiles * ((p.batch + (1 << shift) - 1) >> shift))), b(THREADS);
        if constexpr (!COLUMNS) hipLaunchKernelGGL((rules_rows<T, TILE, THREADS>), g, b, 0, stream, p, (int)tiles);
        else if (p.r.nbias <= 128) hipLaunchKernelGGL((rules_columns<T, TILE, THREADS, 128>), g, b, 0, stream, p, (int)tiles, shift);
        else hipLaunchKernelGGL((rules_columns<T, TILE, THREADS, kMostBias>), g, b, 0, stream, p, (int)tiles, shift);
        return launched();
    });
}

// Tiles of 8192 places, of 2048 where those would leave compute units without one, or in columns, where a tile's chain is longer, with
// less than two.  (64 callers x 131072 words bf16, masks too, 12.6 us with 8192 places and 512 threads, 14.5 with 256 threads; 4096
// places 11.9, but 128 callers 19.9 against 18.3; 2048 places 14.0.  Columns bf16: 32 x 32768 9.1 us with 8192 places, 5.6 with 2048; 64 x 50000
// 17.0 and 13.7; 32 x 131072 13.1 and 13.3, 64 x 131072 18.2 and 27.)
template <typename T>
grim_status rules_typed(const RuleParams &p, bool columns, hipStream_t stream) {
    if (p.batch == 1 && p.ldz == 1 && p.ldo == 1) columns = false;   // a single dense column is a row
    if (p.V * p.batch >= (int64_t)(columns ? 16384 : 4096) * kComputeUnits)
        return columns ? rules_launch<T, 8192, 512, true>(p, stream) : rules_launch<T, 8192, 512, false>(p, stream);
    return columns ? rules_launch<T, 2048, 512, true>(p, stream) : rules_launch<T, 2048, 256, false>(p, stream);
}

}  // namespace lm
}  // namespace grim

extern "C" grim_status grim_apply_logit_rules(const void *z_dev, grim_dtype dt, int32_t columns, int64_t ldz, int64_t V, int32_t batch,
                                              const grim_logit_rules *rules, void *out_dev, int64_t ldo, void *hip_stream) {
    using namespace grim::lm;
    if (!rules) return GRIM_ERR_NULL;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if (V < 1 || V >= (int64_t)1 << 31 || batch < 0 || rules->max_history < 0 || rules->nbias < 0) return GRIM_ERR_SHAPE;
    const int64_t width = columns ? batch : V, rows = columns ? V : batch;
    if (ldz < width || ldo < width || !fits(rows, ldz) || !fits(rows, ldo)) return GRIM_ERR_SHAPE;
    if (rules->history && (rules->ld_history < rules->max_history || !fits(batch, rules->ld_history))) return GRIM_ERR_SHAPE;
    if (rules->nbias > 0 && (rules->ld_bias < rules->nbias || !fits(batch, rules->ld_bias))) return GRIM_ERR_SHAPE;
    if (rules->allowed && (rules->ld_allowed < (V + 31) / 32 || !fits(batch, rules->ld_allowed))) return GRIM_ERR_SHAPE;
    if (rules->nbias > kMostBias || (rules->history && rules->max_history > kMostHistory)) return GRIM_ERR_UNSUPPORTED;
    if (rules->nbias > 0 && (!rules->bias_ids || !rules->bias_values)) return GRIM_ERR_NULL;
    if (batch == 0) return GRIM_OK;
    if (!z_dev || !out_dev) return GRIM_ERR_NULL;
    if (moves(z_dev, ldz, out_dev, ldo, rows)) return GRIM_ERR_SHAPE;
    const RuleParams p{z_dev, out_dev, ldz, ldo, V, batch, *rules};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dt == GRIM_F32   ? rules_typed<float>(p, columns != 0, stream)
           : dt == GRIM_F16 ? rules_typed<f16>(p, columns != 0, stream)
                            : rules_typed<bf16>(p, columns != 0, stream);
}
