// Gated linear recurrence over packed sequences, forward and backward, and its single-token step.
//
//     f = sigmoid(u)    h_t = f h_(t-1) + (1 - f) c    y = sigmoid(v) h
//     G_t = dy_t sigmoid(v_t) + R_t,  R_(t-1) = f_t G_t     (R after the last token: dh_last)
//     du = G f (1 - f) (h_(t-1) - c)    dc = G (1 - f)    dv = dy h sigmoid(v) (1 - sigmoid(v))    dh0 = f_0 G_0
//
// Both directions are linear in the state that is handed on: what a run of tokens does to it is a map S -> A S + B per unit, and
// maps compose.  The rows of all sequences are cut alike, whatever their lengths, into chunks (one wave, 64 to 256 units)
// and sets of kWaves chunks (one workgroup).  A first launch forms the maps of the chunks and sets; the second composes the maps of the
// sets in front of its own, which gives every wave its state, and walks its rows again.  That reads u and c (backward: u, v
// and dy) twice, the price of the parallelism along the sequence; the sets are walked in the opposite order so that what was
// read last is still in the last-level cache.  A sequence that starts inside a run makes the map forget what came before: A = -0, told
// apart from a product of gates that has underflowed, so that an infinity or NaN crosses underflow but no start.
//
// What it measured (both directions, bf16): 65536 x 1024 459 us, of which maps 55 + 79, forward 110, backward 202, at 4.4 to 5.2 TB/s each
// of what they read and write; 512 x 1024 23.7 us, where launches and the chain starts -> rows -> maps through LDS count.
//
// The backward pass needs h_(t-1).  The forward pass leaves the state in front of every kGroup-th row (fp32: 4 bytes for 8 rows of
// 2 to 4 bytes each), from which a group's states are formed again in registers.
#include "lm_common.hpp"

namespace grim {
namespace lm {

constexpr int kWaves = 8;       // waves, and chunks, of a workgroup
// Waves per SIMD that the kernels are held to: what the loads of a group of rows leave room for.  Waves that wait for each other's
// loads hide more than a second group in flight per wave does (at 65536 x 1024 bf16: forward 125 against 112 us, backward 247
// against 212).
constexpr int kWavesMaps = 8;
template <int VEC> constexpr int waves_forward() { return VEC == 1 ? 8 : VEC == 2 ? 6 : 4; }
// (two 16-bit units a lane backward want a few registers more than the 128 that four waves leave: 4 are spilled, 20 bytes of scratch a lane)
template <int VEC> constexpr int waves_backward() { return VEC <= 2 ? 4 : 2; }
// Units of a lane where there are rows enough: 4 bytes, 256 of a row per wave.  (bf16, both directions: 65536 x 1024 555 us with one
// unit, 479 with two, 490 with four; fp32: 896 with one, 903 with two.)
template <typename T> constexpr int wide() { return sizeof(T) == 2 ? 2 : 1; }
constexpr int kGroup = 8;       // rows whose loads are in flight together, and between two saved states
constexpr float kLog2e = 1.44269504088896340736f;

struct GlrParams {
    const void *gates;
    const float *bias, *h0;
    const int32_t *seq;             // nseq + 1 starts, or NULL: one sequence
    void *y;
    float *h_last, *states;
    const void *dy;
    const float *dh_last;
    void *dgates;
    float *dh0, *dbias_part;        // [set][3H]
    float *chunk_maps, *set_maps;   // [chunk or set][A | B][H]
    int64_t ldg, ldy, lddy, lddg, N, H;
    int32_t nseq, L, sets, tiles;   // rows of a chunk (a multiple of kGroup), sets of kWaves chunks, column blocks
    bool torn;                      // rows that are not whole cache lines
};

// f = sigmoid(z) and k = 1 - f = sigmoid(-z) of t = -z log2(e), without cancellation: k = 2^t f.  2^126 is as good as
// infinity for f, and keeps k = 1 there; a NaN stays one.
__device__ __forceinline__ void gate(float t, float &f, float &k) {
    t = t > 126.f ? 126.f : t;
    const float e = __builtin_amdgcn_exp2f(t);
    f = __builtin_amdgcn_rcpf(1.f + e);
    k = e * f;
}

// sigmoid(z) alone needs no bound: the reciprocal of infinity is 0
__device__ __forceinline__ float open(float t) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(t)); }

__device__ __forceinline__ bool forgets(float a) { return __builtin_bit_cast(unsigned, a) == 0x80000000u; }
__device__ __forceinline__ float apply(float a, float b, float s) { return forgets(a) ? b : __builtin_fmaf(a, s, b); }
// (a, b) after (a0, b0)
__device__ __forceinline__ void compose(float a0, float b0, float &a, float &b) {
    b = apply(a, b, b0);
    a = forgets(a) ? a : a0 * a;
}

// ---------------------------------------------------------------------------------------------- where sequences start
// The starts of fewer than 64 sequences are kept in a register, one a lane.
struct Starts {
    const int32_t *seq;
    int32_t nseq, N, held;
    bool in_lanes;
    __device__ __forceinline__ Starts(const GlrParams &p) : seq(p.seq), nseq(p.nseq), N((int32_t)p.N), held(0), in_lanes(p.nseq < 64) {
        const int lane = threadIdx.x & 63;
        if (in_lanes) held = seq ? seq[min(lane, nseq)] : lane ? N : 0;
    }
    __device__ __forceinline__ int at(int i) const { return in_lanes ? __builtin_amdgcn_readlane(held, i) : seq[i]; }
    // how many of the starts of sequences 0 .. nseq - 1 lie below `row`; the whole wave asks
    __device__ __forceinline__ int below(int row) const {
        const int lane = threadIdx.x & 63;
        if (in_lanes) return __popcll(__ballot(lane < nseq && held < row));
        int lo = 0, n = nseq;
        while (n > 64) {
            const int step = (n + 63) / 64;
            const bool under = lane * step < n && seq[lo + lane * step] < row;
            const int c = __popcll(__ballot(under));
            if (c == 0) return lo;
            lo += (c - 1) * step;
            n = min(step, n - (c - 1) * step);
        }
        return __builtin_amdgcn_readfirstlane(lo + __popcll(__ballot(lane < n && seq[lo + lane] < row)));
    }
};

// The unit(s) of a lane: VEC side by side.  Lanes past the last unit repeat it and write nothing; a last lane that would reach past it
// is moved back and shares units with its neighbour (same values, same bits).
template <int VEC>
struct Units {
    int64_t at;
    bool live;
    __device__ __forceinline__ Units(int tile, int64_t H) {
        at = ((int64_t)tile * 64 + (threadIdx.x & 63)) * VEC;
        live = at < H;
        if (at > H - VEC) at = H - VEC;
    }
};

template <int VEC>
__device__ __forceinline__ void take(const float *from, float (&v)[VEC]) {
    unpack(load<VEC>(from), v);
}

// The biases, asked for early; scaled when the rows are in hand: the gates' exponents are one multiply-add each.
template <int VEC>
struct Bias {
    float u[VEC], c[VEC], v[VEC];
    __device__ __forceinline__ Bias(const GlrParams &p, int64_t at) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) u[j] = c[j] = v[j] = 0.f;
        if (p.bias) {
            take<VEC>(p.bias + at, u);
            take<VEC>(p.bias + p.H + at, c);
            take<VEC>(p.bias + 2 * p.H + at, v);
        }
    }
    __device__ __forceinline__ void scale() {
#pragma unroll
        for (int j = 0; j < VEC; ++j) u[j] *= -kLog2e, v[j] *= -kLog2e;
    }
};

// Rows g .. of a group, at most `have` of them (the last is read again for those that are missing), of one column block.
template <typename T, int VEC>
struct Rows {
    Pack<T, VEC> r[kGroup];
    __device__ __forceinline__ void fetch(const void *base, int64_t ld, int64_t column, int g, int have) {
        const T *p = static_cast<const T *>(base) + (int64_t)g * ld;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) r[i] = load<VEC>(p + (int64_t)min(i, have - 1) * ld + column);
    }
};

// ---------------------------------------------------------------------------------------------- maps of the chunks
// What rows r0 .. r1 - 1 do to the state that enters in front of them.
template <typename T, int VEC>
__device__ __forceinline__ void forward_map(const GlrParams &p, const Starts &starts, const Units<VEC> &un, Bias<VEC> &bias, int r0, int r1,
                                            float (&A)[VEC], float (&B)[VEC]) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) A[j] = 1.f, B[j] = 0.f;
    Rows<T, VEC> u, c;
    auto fetch = [&](int at) {
        u.fetch(p.gates, p.ldg, un.at, at, r1 - at);
        c.fetch(p.gates, p.ldg, p.H + un.at, at, r1 - at);
    };
    if (r0 < r1) fetch(r0);
    bias.scale();
    if (r0 >= r1) return;
    int s = starts.below(r0) - 1, bound = starts.at(s + 1);
    for (int g = r0; g < r1; g += kGroup) {
        if (g > r0) fetch(g);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
            const int r = g + i;
            if (r < r1) {
                if (r == bound && s + 1 < p.nseq) {
                    do ++s;
                    while (s + 1 < p.nseq && starts.at(s + 1) <= r);
                    bound = starts.at(s + 1);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) A[j] = -0.f, B[j] = 0.f;
                    if (p.h0) take<VEC>(p.h0 + s * p.H + un.at, B);
                }
                float zu[VEC], zc[VEC];
                unpack(u.r[i], zu);
                unpack(c.r[i], zc);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    float f, k;
                    gate(__builtin_fmaf(zu[j], -kLog2e, bias.u[j]), f, k);
                    A[j] *= f;
                    B[j] = __builtin_fmaf(f, B[j], k * (zc[j] + bias.c[j]));
                }
            }
        }
    }
}

// What rows r1 - 1 .. r0 do to the gradient R that enters behind them.
template <typename T, int VEC>
__device__ __forceinline__ void backward_map(const GlrParams &p, const Starts &starts, const Units<VEC> &un, Bias<VEC> &bias, int r0, int r1,
                                             float (&A)[VEC], float (&B)[VEC]) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) A[j] = 1.f, B[j] = 0.f;
    const int last = r0 + (r1 - 1 - r0) / kGroup * kGroup;
    Rows<T, VEC> u, v, d;
    auto fetch = [&](int at) {
        u.fetch(p.gates, p.ldg, un.at, at, r1 - at);
        v.fetch(p.gates, p.ldg, 2 * p.H + un.at, at, r1 - at);
        d.fetch(p.dy, p.lddy, un.at, at, r1 - at);
    };
    if (r0 < r1) fetch(last);
    bias.scale();
    if (r0 >= r1) return;
    int s = starts.below(r1) - 1;                               // the sequence of row r1 - 1, and where it ends and starts
    int end = s >= 0 ? starts.at(s + 1) : -1, begin = s >= 0 ? starts.at(s) : 0;
    for (int g = last; g >= r0; g -= kGroup) {
        if (g < last) fetch(g);
#pragma unroll
        for (int i = kGroup - 1; i >= 0; --i) {
            const int r = g + i;
            if (r < r1) {
                if (r < begin && s > 0) {
                    do --s;
                    while (s > 0 && starts.at(s) > r);
                    end = starts.at(s + 1), begin = starts.at(s);
                }
                if (r + 1 == end) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) A[j] = -0.f, B[j] = 0.f;
                    if (p.dh_last) take<VEC>(p.dh_last + s * p.H + un.at, B);
                }
                float zu[VEC], zv[VEC], dy[VEC];
                unpack(u.r[i], zu);
                unpack(v.r[i], zv);
                unpack(d.r[i], dy);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float f = open(__builtin_fmaf(zu[j], -kLog2e, bias.u[j])), o = open(__builtin_fmaf(zv[j], -kLog2e, bias.v[j]));
                    A[j] *= f;
                    B[j] = f * __builtin_fmaf(dy[j], o, B[j]);
                }
            }
        }
    }
}

// The maps of a workgroup's chunks in the order that the state passes them (wave `place` is the place-th), from LDS: what those in front of
// this one do together (A, B), and what all do (SA, SB).
template <int VEC>
__device__ __forceinline__ void compose_chunks(float (*maps)[2][64 * VEC], int place, const float (&a)[VEC], const float (&b)[VEC],
                                               float (&A)[VEC], float (&B)[VEC], float (&SA)[VEC], float (&SB)[VEC]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < VEC; ++j) maps[place][0][lane * VEC + j] = a[j], maps[place][1][lane * VEC + j] = b[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < VEC; ++j) A[j] = SA[j] = 1.f, B[j] = SB[j] = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w == place) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) A[j] = SA[j], B[j] = SB[j];
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            float na = maps[w][0][lane * VEC + j], nb = maps[w][1][lane * VEC + j];
            compose(SA[j], SB[j], na, nb);
            SA[j] = na, SB[j] = nb;
        }
    }
}

// The set and column block of a workgroup.  Workgroups are dealt to the eight XCDs in turn.  Where rows are whole cache lines, the column blocks of a
// set are: one XCD reads the same units of all sets, and its L2 still holds their maps in the second launch.  Where lines are torn
// between column blocks, all blocks of a set go to one XCD, whose L2 reads a line once for both (24007 x 1000 fp16, both directions, 193 against
// 173 us; 65536 x 1024 bf16, whole lines, 458 against 460, fp32 2048 x 1024 33.6 against 35.2).  LAST: the sets in descending order.
template <bool LAST>
struct Place {
    int set, tile;
    __device__ __forceinline__ Place(const GlrParams &p) {
        const int b = blockIdx.x;
        if (p.torn) {
            set = b % 8 + 8 * (LAST ? (p.sets + 7) / 8 - 1 - b / 8 / p.tiles : b / 8 / p.tiles);      // (set may be one of up to 7 too many)
            tile = b / 8 % p.tiles;
        } else {
            set = LAST ? p.sets - 1 - b / p.tiles : b / p.tiles;
            tile = b % p.tiles;
        }
    }
};
inline unsigned workgroups(const GlrParams &p) { return (unsigned)(p.torn ? (p.sets + 7) / 8 * 8 : p.sets) * p.tiles; }

// Rows of this wave's chunk.
struct Chunk {
    int wave, index, r0, r1;
    __device__ __forceinline__ Chunk(const GlrParams &p, int set) {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        index = set * kWaves + wave;
        const int64_t a = (int64_t)index * p.L, b = a + p.L;
        r0 = (int)(a < p.N ? a : p.N), r1 = (int)(b < p.N ? b : p.N);
    }
};

template <typename T, int VEC, bool BACK>
__global__ void __launch_bounds__(64 * kWaves, kWavesMaps) glr_maps(GlrParams p) {
    __shared__ float maps[kWaves][2][64 * VEC];
    const Starts starts(p);
    const Place<false> here(p);
    const int set = here.set;
    if (set >= p.sets) return;
    const Units<VEC> un(here.tile, p.H);
    Bias<VEC> bias(p, un.at);
    const Chunk ch(p, set);
    float a[VEC], b[VEC], A[VEC], B[VEC], SA[VEC], SB[VEC];
    if (BACK) backward_map<T, VEC>(p, starts, un, bias, ch.r0, ch.r1, a, b);
    else forward_map<T, VEC>(p, starts, un, bias, ch.r0, ch.r1, a, b);
    const int place = BACK ? kWaves - 1 - ch.wave : ch.wave;
    compose_chunks<VEC>(maps, place, a, b, A, B, SA, SB);
    if (!un.live) return;
    float *mine = p.chunk_maps + (int64_t)ch.index * 2 * p.H + un.at;
    store(mine, A);
    store(mine + p.H, B);
    if (place == kWaves - 1) {
        float *all = p.set_maps + (int64_t)set * 2 * p.H + un.at;
        store(all, SA);
        store(all + p.H, SB);
    }
}

// The state that enters this wave's chunk: the sets in front of its own (first, in steps of `dir`, to the one before `set`) dealt to the
// waves as runs, composed through LDS, then the chunk's own prefix.  Nothing enters the first set: A counts for nothing there.
template <int VEC>
__device__ __forceinline__ void entering(const GlrParams &p, float (*maps)[2][64 * VEC], const Units<VEC> &un, const Chunk &ch, int set,
                                         int first, int dir, int ahead, float (&S)[VEC]) {
    float a[VEC], b[VEC], pa[VEC], pb[VEC];
    const float *prefix = p.chunk_maps + (int64_t)ch.index * 2 * p.H + un.at;
    take<VEC>(prefix, pa);
    take<VEC>(prefix + p.H, pb);
#pragma unroll
    for (int j = 0; j < VEC; ++j) a[j] = 1.f, b[j] = 0.f;
    const int per = (ahead + kWaves - 1) / kWaves;
    const int from = min(ch.wave * per, ahead), to = min(from + per, ahead);
    constexpr int kBatch = 8;                                   // maps on their way together
    for (int i = from; i < to; i += kBatch) {
        Pack<float, VEC> na[kBatch], nb[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const float *m = p.set_maps + (int64_t)(first + dir * min(i + k, to - 1)) * 2 * p.H + un.at;
            na[k] = load<VEC>(m);
            nb[k] = load<VEC>(m + p.H);
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (i + k < to) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    float ka = element(na[k], j), kb = element(nb[k], j);
                    compose(a[j], b[j], ka, kb);
                    a[j] = ka, b[j] = kb;
                }
            }
    }
    float A[VEC], B[VEC], SA[VEC], SB[VEC];
    compose_chunks<VEC>(maps, ch.wave, a, b, A, B, SA, SB);
#pragma unroll
    for (int j = 0; j < VEC; ++j) S[j] = apply(pa[j], pb[j], SB[j]);
}

// ---------------------------------------------------------------------------------------------- forward
// ALONE: one set holds all rows, and its workgroup forms the maps of its chunks itself.
template <typename T, int VEC, bool ALONE, bool PAST>
__global__ void __launch_bounds__(64 * kWaves, waves_forward<VEC>()) glr_forward(GlrParams p) {
    __shared__ float maps[kWaves][2][64 * VEC];
    const Starts starts(p);
    const Place<true> here(p);
    const int set = ALONE ? 0 : here.set;
    if (set >= p.sets) return;
    const Units<VEC> un(ALONE ? (int)blockIdx.x : here.tile, p.H);
    Bias<VEC> bias(p, un.at);
    const Chunk ch(p, set);
    const int r0 = ch.r0, r1 = ch.r1;
    Rows<T, VEC> u, c, v;
    auto fetch = [&](int at) {
        u.fetch(p.gates, p.ldg, un.at, at, r1 - at);
        c.fetch(p.gates, p.ldg, p.H + un.at, at, r1 - at);
        v.fetch(p.gates, p.ldg, 2 * p.H + un.at, at, r1 - at);
    };
    // With few rows the first group is on its way while the state is put together; with many, other waves are.
    constexpr bool early = !ALONE && VEC == 1;
    if (early && r0 < r1) fetch(r0);
    float h[VEC];
    if (ALONE) {
        float a[VEC], b[VEC], A[VEC], SA[VEC], SB[VEC];
        forward_map<T, VEC>(p, starts, un, bias, ch.r0, ch.r1, a, b);
        compose_chunks<VEC>(maps, ch.wave, a, b, A, h, SA, SB);
    } else {
        entering<VEC>(p, maps, un, ch, set, 0, 1, set, h);
        bias.scale();
    }
    if (p.h_last)                                               // sequences without a token keep their state
        for (int s = ch.index; s < p.nseq; s += p.sets * kWaves)
            if (starts.at(s) == starts.at(s + 1) && un.live) {
                float v[VEC] = {};
                if (p.h0) take<VEC>(p.h0 + s * p.H + un.at, v);
                store(p.h_last + s * p.H + un.at, v);
            }
    if (r0 >= r1) return;
    int s = starts.below(r0) - 1, bound = starts.at(s + 1);
    T *y = static_cast<T *>(p.y) + un.at;
    for (int g = r0; g < r1; g += kGroup) {
        if (!early || g > r0) fetch(g);
        if (p.states && un.live) store(p.states + (int64_t)(g / kGroup) * p.H + un.at, h);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
            const int r = g + i;
            if (r < r1) {
                if (r == bound && s + 1 < p.nseq) {
                    do ++s;
                    while (s + 1 < p.nseq && starts.at(s + 1) <= r);
                    bound = starts.at(s + 1);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) h[j] = 0.f;
                    if (p.h0) take<VEC>(p.h0 + s * p.H + un.at, h);
                }
                float zu[VEC], zc[VEC], zv[VEC], out[VEC];
                unpack(u.r[i], zu);
                unpack(c.r[i], zc);
                unpack(v.r[i], zv);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    float f, k;
                    gate(__builtin_fmaf(zu[j], -kLog2e, bias.u[j]), f, k);
                    h[j] = __builtin_fmaf(f, h[j], k * (zc[j] + bias.c[j]));
                    out[j] = open(__builtin_fmaf(zv[j], -kLog2e, bias.v[j])) * h[j];
                }
                if (un.live) {
                    store<PAST>(y + (int64_t)r * p.ldy, out);
                    if (p.h_last && s >= 0 && r + 1 == bound) store(p.h_last + s * p.H + un.at, h);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- backward
template <typename T, int VEC, bool ALONE, bool PAST>
__global__ void __launch_bounds__(64 * kWaves, waves_backward<VEC>()) glr_backward(GlrParams p) {
    __shared__ float maps[kWaves][2][64 * VEC];
    __shared__ float sums[3][64 * VEC];
    const Starts starts(p);
    const Place<true> here(p);
    const int set = ALONE ? 0 : here.set;
    if (set >= p.sets) return;
    const Units<VEC> un(ALONE ? (int)blockIdx.x : here.tile, p.H);
    Bias<VEC> bias(p, un.at);
    const Chunk ch(p, set);
    float R[VEC];
    if (ALONE) {
        float a[VEC], b[VEC], A[VEC], SA[VEC], SB[VEC];
        backward_map<T, VEC>(p, starts, un, bias, ch.r0, ch.r1, a, b);
        compose_chunks<VEC>(maps, kWaves - 1 - ch.wave, a, b, A, R, SA, SB);
    } else {
        entering<VEC>(p, maps, un, ch, set, p.sets - 1, -1, p.sets - 1 - set, R);
        bias.scale();
    }
    if (p.dh0)
        for (int s = ch.index; s < p.nseq; s += p.sets * kWaves)
            if (starts.at(s) == starts.at(s + 1) && un.live) {
                float v[VEC] = {};
                if (p.dh_last) take<VEC>(p.dh_last + s * p.H + un.at, v);
                store(p.dh0 + s * p.H + un.at, v);
            }
    float bu[VEC], bc[VEC], bv[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) bu[j] = bc[j] = bv[j] = 0.f;
    const int r0 = ch.r0, r1 = ch.r1;
    if (r0 < r1) {
        int s = starts.below(r1) - 1;                           // the sequence of the row in hand, its first row and its end
        int begin = s >= 0 ? starts.at(s) : 0, end = s >= 0 ? starts.at(s + 1) : -1;
        for (int g = r0 + (r1 - 1 - r0) / kGroup * kGroup; g >= r0; g -= kGroup) {
            const int have = min(r1 - g, kGroup);
            Rows<T, VEC> u, c, v, d;
            u.fetch(p.gates, p.ldg, un.at, g, have);
            c.fetch(p.gates, p.ldg, p.H + un.at, g, have);
            v.fetch(p.gates, p.ldg, 2 * p.H + un.at, g, have);
            d.fetch(p.dy, p.lddy, un.at, g, have);
            float before[VEC];                                  // the state in front of the row
            take<VEC>(p.states + (int64_t)(g / kGroup) * p.H + un.at, before);
            // the group's states again, and its gates; `first` marks the rows that begin a sequence
            float h[kGroup][VEC], f[kGroup][VEC], k[kGroup][VEC];
            unsigned first = 0;
            int q = s, next = -1;                               // (no start inside: nothing to look for)
            if (begin >= g) {
                q = starts.below(g) - 1;
                next = starts.at(q + 1);
            }
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {
                if (i < have) {
                    if (g + i == next && q + 1 < p.nseq) {
                        do ++q;
                        while (q + 1 < p.nseq && starts.at(q + 1) <= g + i);
                        next = starts.at(q + 1);
                        first |= 1u << i;
#pragma unroll
                        for (int j = 0; j < VEC; ++j) before[j] = 0.f;
                        if (p.h0) take<VEC>(p.h0 + q * p.H + un.at, before);
                    }
                    float zu[VEC], zc[VEC];
                    unpack(u.r[i], zu);
                    unpack(c.r[i], zc);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        gate(__builtin_fmaf(zu[j], -kLog2e, bias.u[j]), f[i][j], k[i][j]);
                        h[i][j] = before[j];
                        before[j] = __builtin_fmaf(f[i][j], before[j], k[i][j] * (zc[j] + bias.c[j]));
                    }
                }
            }
#pragma unroll
            for (int i = kGroup - 1; i >= 0; --i) {
                if (i < have) {
                    const int r = g + i;
                    if (r < begin && s > 0) {
                        do --s;
                        while (s > 0 && starts.at(s) > r);
                        end = starts.at(s + 1), begin = starts.at(s);
                    }
                    if (r + 1 == end) {
#pragma unroll
                        for (int j = 0; j < VEC; ++j) R[j] = 0.f;
                        if (p.dh_last) take<VEC>(p.dh_last + s * p.H + un.at, R);
                    }
                    float zc[VEC], zv[VEC], dy[VEC], du[VEC], dc[VEC], dv[VEC];
                    unpack(c.r[i], zc);
                    unpack(v.r[i], zv);
                    unpack(d.r[i], dy);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        float o, ko;
                        gate(__builtin_fmaf(zv[j], -kLog2e, bias.v[j]), o, ko);
                        const float cc = zc[j] + bias.c[j];
                        const float dyo = dy[j] * o, G = dyo + R[j];
                        const float hh = __builtin_fmaf(f[i][j], h[i][j], k[i][j] * cc);
                        dc[j] = G * k[i][j];
                        R[j] = G * f[i][j];
                        du[j] = dc[j] * f[i][j] * (h[i][j] - cc);
                        dv[j] = dyo * ko * hh;
                        bu[j] += du[j], bc[j] += dc[j], bv[j] += dv[j];
                    }
                    if (un.live) {
                        T *out = static_cast<T *>(p.dgates) + (int64_t)r * p.lddg + un.at;
                        store<PAST>(out, du);
                        store<PAST>(out + p.H, dc);
                        store<PAST>(out + 2 * p.H, dv);
                        if (p.dh0 && s >= 0 && (first >> i & 1)) store(p.dh0 + s * p.H + un.at, R);
                    }
                }
            }
        }
    }
    if (!p.dbias_part) return;
    const int lane = threadIdx.x & 63;
    for (int w = 0; w < kWaves; ++w) {                          // the waves' sums, in the order of the waves
        if (ch.wave == w) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int at = lane * VEC + j;
                sums[0][at] = w ? sums[0][at] + bu[j] : bu[j];
                sums[1][at] = w ? sums[1][at] + bc[j] : bc[j];
                sums[2][at] = w ? sums[2][at] + bv[j] : bv[j];
            }
        }
        __syncthreads();
    }
    if (ch.wave < 3 && un.live) {
        float out[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) out[j] = sums[ch.wave][lane * VEC + j];
        store(p.dbias_part + ((int64_t)set * 3 + ch.wave) * p.H + un.at, out);
    }
}

// ---------------------------------------------------------------------------------------------- one token
struct GlrStepParams {
    const float *gates, *bias, *h;
    float *h_new;
    void *y;
    int64_t ldg, ldh, ldh_new, ldy, H;
    int32_t batch;
};

template <typename T>
__global__ void __launch_bounds__(256) glr_step_kernel(GlrStepParams p) {
    const uint32_t e = blockIdx.x * 256 + threadIdx.x;          // (all of a launch's threads count in 32 bits)
    if (e >= p.H * p.batch) return;
    const int64_t r = e / (uint32_t)p.batch, b = e % (uint32_t)p.batch;
    float zu = p.gates[r * p.ldg + b], zc = p.gates[(p.H + r) * p.ldg + b], zv = p.gates[(2 * p.H + r) * p.ldg + b];
    if (p.bias) zu += p.bias[r], zc += p.bias[p.H + r], zv += p.bias[2 * p.H + r];
    float f, k;
    gate(zu * -kLog2e, f, k);
    const float h = __builtin_fmaf(f, p.h[r * p.ldh + b], k * zc);
    p.h_new[r * p.ldh_new + b] = h;
    if (p.y) static_cast<T *>(p.y)[r * p.ldy + b] = (T)(open(zv * -kLog2e) * h);
}

// ---------------------------------------------------------------------------------------------- launches
// How the rows are cut.
struct Cut {
    int vec, last;              // units of a lane, and in the second launch
    bool past;
    int32_t L, sets, tiles;
};

inline Cut cut_rows(int64_t N, int64_t H, bool fp32, bool back) {
    Cut c;
    const int wide_one = fp32 ? wide<float>() : wide<f16>();
    // one unit a lane where more would leave compute units without work (1024 x 1024 bf16 24 against 27 us, 2048 x 1024 31 against 30)
    c.vec = H >= 256 && N * H >= (int64_t)1 << 21 ? wide_one : 1;
    c.past = past_caches((back ? 7 : 4) * N * H * (fp32 ? 4 : 2));
    // Eight bytes of a row where the outputs go past the caches, if three or more column blocks remain (bf16 forward 65536 x 1000 183 against
    // 194 us, as long with H = 1024); backward, where a compute unit then holds one workgroup instead of two, only with more than one
    // round of them (26 M units: 65536 x 1000 322 against 377 us, 65536 x 1024 285 against 297; 16384 x 1024 74 against 66).
    c.last = c.past && c.vec == 2 && H >= 768 && (!back || N * H >= (int64_t)26 << 20) ? 4 : c.vec;
    c.tiles = (int32_t)((H + 64 * c.vec - 1) / (64 * c.vec));
    // Chunks so short that the workgroups fill the compute units once (the second launch of the backward pass has room for 512,
    // the others for 1024), but no shorter than keep the maps of the sets, all of which a workgroup may have to read, within its own
    // rows' size: rows^2 = N / 64.  (bf16, both directions: 64000 x 128 81 us in 250 sets of 32 rows a wave, 94 in 334, 97
    // in 125; 20863 x 192 52 in 163 sets of 16, 61 in 109, 65 in 327.)
    const int64_t room = kWaves * (back && c.last < 4 ? 512 : 1024);
    const int64_t even = (N * c.tiles + room - 1) / room;
    const int64_t square = ((int64_t)__builtin_sqrt((double)N / 64.0) + kGroup / 2) / kGroup * kGroup;
    int64_t L = even > square ? even : square;
    L = L < N ? L : N;
    L = (L + kGroup - 1) / kGroup * kGroup;                     // (up to 64 rows: one set, one launch)
    c.L = (int32_t)(L < kGroup ? kGroup : L);
    const int64_t rows = (int64_t)c.L * kWaves;
    c.sets = N > 0 ? (int32_t)((N + rows - 1) / rows) : 1;
    return c;
}

inline int64_t map_floats(const Cut &c, int64_t H) { return ((int64_t)c.sets * (kWaves + 1)) * 2 * H; }

template <typename T, int VEC>
grim_status glr_launch(const GlrParams &p, const Cut &c, bool back, hipStream_t stream) {
    const dim3 grid(c.sets == 1 ? (unsigned)p.tiles : workgroups(p)), block(64 * kWaves);
    if (c.sets == 1) {
        if (back) hipLaunchKernelGGL((glr_backward<T, VEC, true, false>), grid, block, 0, stream, p);
        else hipLaunchKernelGGL((glr_forward<T, VEC, true, false>), grid, block, 0, stream, p);
        return launched();
    }
    if (back) hipLaunchKernelGGL((glr_maps<T, VEC, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((glr_maps<T, VEC, false>), grid, block, 0, stream, p);
    const grim_status st = launched();
    if (st != GRIM_OK) return st;
    constexpr int W = VEC == 2 ? 4 : VEC;
    GlrParams q = p;
    q.tiles = (int32_t)((p.H + 64 * c.last - 1) / (64 * c.last));
    const dim3 last(workgroups(q));
    if (c.last == 4) {
        if (back) hipLaunchKernelGGL((glr_backward<T, W, false, true>), last, block, 0, stream, q);
        else hipLaunchKernelGGL((glr_forward<T, W, false, true>), last, block, 0, stream, q);
    } else if (c.past) {
        if (back) hipLaunchKernelGGL((glr_backward<T, VEC, false, true>), last, block, 0, stream, q);
        else hipLaunchKernelGGL((glr_forward<T, VEC, false, true>), last, block, 0, stream, q);
    } else {
        if (back) hipLaunchKernelGGL((glr_backward<T, VEC, false, false>), last, block, 0, stream, q);
        else hipLaunchKernelGGL((glr_forward<T, VEC, false, false>), last, block, 0, stream, q);
    }
    return launched();
}

grim_status glr_run(GlrParams p, grim_dtype dt, bool back, hipStream_t stream) {
    const Cut c = cut_rows(p.N, p.H, dt == GRIM_F32, back);
    p.L = c.L, p.sets = c.sets, p.tiles = c.tiles;
    const int64_t e = bytes_of(dt);
    const auto whole = [&](const void *at, int64_t ld) { return !at || ((uintptr_t)at | (uintptr_t)(ld * e)) % 128 == 0; };
    p.torn = !(p.H * e % 128 == 0 && whole(p.gates, p.ldg) && whole(p.y, p.ldy) && whole(p.dy, p.lddy) && whole(p.dgates, p.lddg));
    p.set_maps = p.chunk_maps + (int64_t)c.sets * kWaves * 2 * p.H;
    switch (dt) {
        case GRIM_F32: return c.vec > 1 ? glr_launch<float, wide<float>()>(p, c, back, stream) : glr_launch<float, 1>(p, c, back, stream);
        case GRIM_F16: return c.vec > 1 ? glr_launch<f16, wide<f16>()>(p, c, back, stream) : glr_launch<f16, 1>(p, c, back, stream);
        default: return c.vec > 1 ? glr_launch<bf16, wide<bf16>()>(p, c, back, stream) : glr_launch<bf16, 1>(p, c, back, stream);
    }
}

inline bool glr_sizes(int64_t N, int64_t H, int32_t nseq, const int32_t *seq) {
    // (row numbers in 32 bits with room for a group more; cut_rows leaves some 1024 workgroups, or eight rows of up to 2^15 column blocks:
    // few enough threads for a launch)
    return N >= 0 && N <= (int64_t)1 << 30 && H >= 1 && H <= (int64_t)1 << 21 && nseq >= 1 && (seq || nseq == 1);
}

}  // namespace lm
}  // namespace grim

extern "C" {

int64_t grim_glr_states(int64_t N, int64_t H) {
    using namespace grim::lm;
    return glr_sizes(N, H, 1, nullptr) ? (N + kGroup - 1) / kGroup * H * (int64_t)sizeof(float) : 0;
}

int64_t grim_glr_workspace(int64_t N, int64_t H) {
    using namespace grim::lm;
    if (!glr_sizes(N, H, 1, nullptr)) return 0;
    int64_t most = 0;                                           // (whichever type and direction come)
    for (int way = 0; way < 4; ++way) {
        const Cut c = cut_rows(N, H, way & 1, way & 2);
        const int64_t floats = map_floats(c, H) + (int64_t)c.sets * 3 * H;
        most = floats > most ? floats : most;
    }
    return most * (int64_t)sizeof(float);
}

grim_status grim_glr_sequence(const void *gates_dev, grim_dtype dt, int64_t ldg, const float *bias_dev, const float *h0_dev,
                              const int32_t *seq_start_dev, int32_t nseq, int64_t N, int64_t H, void *y_dev, int64_t ldy,
                              float *h_last_dev, void *states_dev, void *workspace, int64_t workspace_bytes,
                              void *hip_stream) {
    using namespace grim::lm;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if (!glr_sizes(N, H, nseq, seq_start_dev) || ldg < 3 * H || ldy < H || !fits(N, ldg) || !fits(N, ldy)) return GRIM_ERR_SHAPE;
    if ((N > 0 && (!gates_dev || !y_dev)) || !workspace) return GRIM_ERR_NULL;
    if (workspace_bytes < grim_glr_workspace(N, H)) return GRIM_ERR_SHAPE;
    // (the wave that ends a sequence may be done before the one that starts it reads its state)
    if (overlap(h0_dev, h_last_dev, nseq * H * (int64_t)sizeof(float))) return GRIM_ERR_UNSUPPORTED;
    GlrParams p{};
    p.gates = gates_dev, p.bias = bias_dev, p.h0 = h0_dev, p.seq = seq_start_dev, p.nseq = nseq;
    p.y = y_dev, p.h_last = h_last_dev, p.states = static_cast<float *>(states_dev);
    p.chunk_maps = static_cast<float *>(workspace);
    p.ldg = ldg, p.ldy = ldy, p.N = N, p.H = H;
    return glr_run(p, dt, false, static_cast<hipStream_t>(hip_stream));
}

grim_status grim_glr_sequence_backward(const void *gates_dev, grim_dtype dt, int64_t ldg, const float *bias_dev,
                                       const float *h0_dev, const int32_t *seq_start_dev, int32_t nseq, int64_t N, int64_t H,
                                       const void *states_dev, const void *dy_dev, int64_t lddy, const float *dh_last_dev,
                                       void *dgates_dev, int64_t lddg, float *dbias_dev, float *dh0_dev, void *workspace,
                                       int64_t workspace_bytes, void *hip_stream) {
    using namespace grim::lm;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if (!glr_sizes(N, H, nseq, seq_start_dev) || ldg < 3 * H || lddy < H || lddg < 3 * H || !fits(N, ldg) || !fits(N, lddy) ||
        !fits(N, lddg))
        return GRIM_ERR_SHAPE;
    if ((N > 0 && (!gates_dev || !states_dev || !dy_dev || !dgates_dev)) || !workspace) return GRIM_ERR_NULL;
    if (workspace_bytes < grim_glr_workspace(N, H)) return GRIM_ERR_SHAPE;
    if (overlap(dh_last_dev, dh0_dev, nseq * H * (int64_t)sizeof(float))) return GRIM_ERR_UNSUPPORTED;
    const Cut c = cut_rows(N, H, dt == GRIM_F32, true);
    GlrParams p{};
    p.gates = gates_dev, p.bias = bias_dev, p.h0 = h0_dev, p.seq = seq_start_dev, p.nseq = nseq;
    p.states = static_cast<float *>(const_cast<void *>(states_dev));
    p.dy = dy_dev, p.dh_last = dh_last_dev, p.dgates = dgates_dev, p.dh0 = dh0_dev;
    p.chunk_maps = static_cast<float *>(workspace);
    p.dbias_part = dbias_dev ? p.chunk_maps + map_floats(c, H) : nullptr;
    p.ldg = ldg, p.lddy = lddy, p.lddg = lddg, p.N = N, p.H = H;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const grim_status st = glr_run(p, dt, true, stream);
    if (st != GRIM_OK || !dbias_dev) return st;
    return join_columns(p.dbias_part, c.sets, 3 * H, dbias_dev, 0, nullptr, stream);
}

grim_status grim_glr_step(const float *gates_dev, int64_t ldg, const float *bias_dev, const float *h_dev, int64_t ldh,
                          float *h_new_dev, int64_t ldh_new, void *y_dev, grim_dtype dt, int64_t ldy, int64_t H,
                          int32_t batch, void *hip_stream) {
    using namespace grim::lm;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if (H < 1 || batch < 0 || ldg < batch || ldh < batch || ldh_new < batch || (y_dev && ldy < batch) || H > (int64_t)1 << 32 ||
        !fits(3 * H, ldg) || !fits(H, ldh) || !fits(H, ldh_new) || (y_dev && !fits(H, ldy)))
        return GRIM_ERR_SHAPE;
    if (batch == 0) return GRIM_OK;
    if (!gates_dev || !h_dev || !h_new_dev) return GRIM_ERR_NULL;
    if (moves(h_dev, ldh, h_new_dev, ldh_new, H)) return GRIM_ERR_SHAPE;
    if (H > most_groups(256) * 256 / batch) return GRIM_ERR_SHAPE;
    const GlrStepParams p{gates_dev, bias_dev, h_dev, h_new_dev, y_dev, ldg, ldh, ldh_new, ldy, H, batch};
    const dim3 grid((unsigned)((H * batch + 255) / 256)), block(256);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dt == GRIM_F32) hipLaunchKernelGGL(glr_step_kernel<float>, grid, block, 0, stream, p);
    else if (dt == GRIM_F16) hipLaunchKernelGGL(glr_step_kernel<f16>, grid, block, 0, stream, p);
    else hipLaunchKernelGGL(glr_step_kernel<bf16>, grid, block, 0, stream, p);
    return launched();
}

}  // extern "C"
