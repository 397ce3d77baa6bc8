// The gated delta rule over packed sequences, backward: from chunk to chunk.
//
// In the notation of lm_gdr.hip, with dy, and A the gradient of the states behind a chunk:
//     dU = P' dy + exp(G_end - G) K A        P_ij = w_ij q_i . k_j scale (i >= j)
//     F = dU - M' beta dU                    the gradient of U less what comes back through later tokens of the chunk
//     Y = beta F = dX = dV                   dbeta = F . E
//     dS = exp(G_end) A + exp(G) Q' dy - exp(G) K' Y
// (E = X - M beta X and U = beta E, so dX = dE - beta M' dE with dE = beta dU.)  As in the forward pass all of this stays in its column of the states, and A goes from chunk to
// chunk in registers.  A and F are kept for the gradients that mix columns (lm_gdr_grad.hip).
#include "lm_gdr.hpp"

namespace grim {
namespace lm {

// What a workgroup keeps in LDS.
template <typename T, int DK, int COLS>
struct BackRoom {
    static constexpr int C = Gdr<T>::chunk, PD = Gdr<T>::data, PC = Gdr<T>::comp;
    using Keys = Tile<PD, C, DK>;
    using Square = Triangle<PC, C, PAIRED, true>;           // P transposed
    using Matrix = Triangle<PC, C, TURNED>;
    using Vals = Values<T, C, COLS>;
    static constexpr int keys = 0, queries = keys + Keys::bytes, values = queries + Keys::bytes, M = values + Vals::bytes, P = M + Matrix::bytes, G = P + Square::bytes,
                         tokens = G + C * 8, bytes = tokens + C * 24;
    static_assert(bytes <= 160 * 1024, "LDS");
};

// A workgroup takes 16 W columns of the states of a run of a sequence's head, its chunks from the last to the first.
// MAPS: what every run but a sequence's first adds to the gradient of the states in front of it, from a gradient of zeros behind it (of the last run, whose end
// is known, this is the gradient itself); what it makes of the gradient behind it is its map of the forward pass, transposed.
// Bound as the forward walk is: 4096 chunks of 128 x 128 heads in bf16 169 us (0.73 GB), the runs' parts 141; 64 x 64 heads, 6000 chunks, 163 and 82.
// HELP: the second half of the waves has no columns; they form P.
template <typename T, int DK, int W, bool WHOLE, bool MAPS, bool HELP>
__global__ void __launch_bounds__(64 * W, 2) walk_back(GdrBack b) {
    constexpr int C = Gdr<T>::chunk, PD = Gdr<T>::data, PC = Gdr<T>::comp, THREADS = 64 * W, COLS = 16 * W;
    constexpr int TT = C / 16, SS = C / 32, DT = DK / 16, DS = DK / 32;
    using Room = BackRoom<T, DK, COLS>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const GdrParams &p = b.p;
    const typename Room::Keys K{reinterpret_cast<uint16_t *>(lds + Room::keys)}, Q{reinterpret_cast<uint16_t *>(lds + Room::queries)};
    typename Room::Matrix M;
    typename Room::Square P;
    M.put(lds + Room::M), P.put(lds + Room::P);
    const typename Room::Vals V{reinterpret_cast<T *>(lds + Room::values)};
    double *G = reinterpret_cast<double *>(lds + Room::G);
    float *tokens = reinterpret_cast<float *>(lds + Room::tokens);
    const float *beta = tokens, *fk = tokens + C, *fu = tokens + 2 * C, *fq = tokens + 3 * C, *rk = tokens + 4 * C, *rq = tokens + 5 * C;

    const uint32_t blocks = (p.tiles + W - 1) / W, heads = (uint32_t)p.heads;
    const int block = (int)(blockIdx.x % blocks), h = (int)(blockIdx.x / blocks % heads);
    const uint32_t run = blockIdx.x / blocks / heads;
    const int s = sequence_of(p.seq_start, p.nseq, p.N, p.size, run);
    const Span span(p.seq_start, s, p.N);
    const uint32_t r = run - place_of(span, s, p.size);
    const int64_t from = span.first + (int64_t)r * p.size, to = min(span.end, from + p.size);
    if (from >= to && (MAPS || r > 0) || MAPS && r == 0) return;            // (an empty sequence has its first run for the gradient of its first states)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15, g4 = (lane >> 4) * 4, own = l15 * 16 + g4;
    const int tile = block * W + wave, col0 = block * COLS;
    const bool idle = tile >= p.tiles;
    const T *q = static_cast<const T *>(p.q) + (int64_t)(h / p.group) * p.dk, *k = static_cast<const T *>(p.k) + (int64_t)(h / p.group) * p.dk;
    const T *dy = static_cast<const T *>(b.dy) + (int64_t)h * p.dv + col0;
    T *dv = static_cast<T *>(b.dv) + (int64_t)h * p.dv;

    f32x4 state[DT];                                        // A: rows 16 n + g4 .. + 3, column 16 tile + l15
    const int64_t head = ((int64_t)s * p.heads + h) * p.dk;
    const bool last = to >= span.end;
#pragma unroll
    for (int n = 0; n < DT; ++n) {
        const int d = 16 * n + g4, col = 16 * tile + l15;
        state[n] = f32x4{};
        if (last) {
            if (b.ds_last)
#pragma unroll
                for (int e = 0; e < 4; ++e) state[n][e] = b.ds_last[(head + min(d + e, p.dk - 1)) * p.dv + min(col, p.dv - 1)];
        } else if (!MAPS && !idle) {
            state[n] = *reinterpret_cast<const f32x4 *>(p.starts + ((((int64_t)run * p.heads + h) * p.tiles + tile) * DT + n) * 256 + own);
        }
    }
#pragma unroll
    for (int n = 0; n < DT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            asm volatile("" : "+v"(state[n][e]));           // (all are asked for before any is looked at)
            if (16 * n + g4 + e >= p.dk || 16 * tile + l15 >= p.dv) state[n][e] = 0.f;
        }

    // ones on the diagonal, as the second operand of a sum over 32 rows of which it takes 16: a product with it turns a result over
    s16x8 unit[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const short one = g4 + i % 4 == l15 ? 0x3f80 : 0;
        unit[0][i] = i < 4 ? one : 0, unit[1][i] = i < 4 ? 0 : one;
    }

    Rows<WHOLE, T, THREADS, C, DK> kn, qn;
    Rows<WHOLE, T, THREADS, C, COLS> yn;
    constexpr int pieces = PC * Saved<T>::part / 8, MP = (pieces + THREADS - 1) / THREADS, TP = (6 * C + THREADS - 1) / THREADS;
    u32x4 mn[MP];
    double Gn = 0.;
    float tn[TP];
    const int64_t place = place_of(span, s, C) + r * (p.size / C);
    const auto fetch = [&](int64_t n) {
        const int64_t first = from + n * C;
        const int rows = __builtin_amdgcn_readfirstlane((int)min((int64_t)C, to - first));
        kn.fetch(k + first * p.ldk, p.ldk, rows, p.dk);
        qn.fetch(q + first * p.ldq, p.ldq, rows, p.dk);
        yn.fetch(dy + first * b.lddy, b.lddy, rows, p.dv - col0);
        const Saved<T> saved(p, place + n, h);
#pragma unroll
        for (int i = 0; i < MP; ++i) mn[i] = reinterpret_cast<const u32x4 *>(saved.M())[min(i * THREADS + (int)threadIdx.x, pieces - 1)];
        Gn = saved.G()[threadIdx.x % C];
#pragma unroll
        for (int i = 0; i < TP; ++i) tn[i] = saved.tokens()[min(i * THREADS + (int)threadIdx.x, 6 * C - 1)];
    };
    const int64_t chunks = (to - from + C - 1) / C;
    if (chunks > 0) fetch(chunks - 1);
    for (int64_t n = chunks - 1; n >= 0; --n) {
        const int64_t first = from + n * C;
        const int rows = __builtin_amdgcn_readfirstlane((int)min((int64_t)C, to - first));
        kn.place(K, rows, p.dk);
        qn.place(Q, rows, p.dk);
        yn.keep(V.at, V.ld, rows, p.dv - col0);
#pragma unroll
        for (int i = 0; i < MP; ++i) {                      // (from the paired order back into the columns' own)
            const int piece = i * THREADS + (int)threadIdx.x;
            if (piece < pieces) {
                const s16x8 w = __builtin_bit_cast(s16x8, mn[i]);
                uint16_t *at = M.piece(piece) - piece % 4 * 4;
                *reinterpret_cast<s16x4 *>(at) = __builtin_shufflevector(w, w, 0, 1, 2, 3);
                *reinterpret_cast<s16x4 *>(at + 16) = __builtin_shufflevector(w, w, 4, 5, 6, 7);
            }
        }
        if (threadIdx.x < C) G[threadIdx.x] = Gn;
#pragma unroll
        for (int i = 0; i < TP; ++i)
            if (i * THREADS + (int)threadIdx.x < 6 * C) tokens[i * THREADS + threadIdx.x] = tn[i];
        if (n > 0) fetch(n - 1);
        __syncthreads();
        constexpr int WORK = HELP ? W / 2 : W, EACH = (Lower<C>::count + WORK - 1) / WORK;
#pragma unroll 1
        for (int n = 0; n < EACH; ++n) {                    // P
            const int pair = n * WORK + wave - (W - WORK);
            if (pair < 0 || pair >= Lower<C>::count) break;
            int i, j;
            Lower<C>::get(pair, i, j);
            f32x4 acc = {};
#pragma unroll
            for (int d = 0; d < DS; ++d) acc = multiply(along(Q, 16 * i, 32 * d), along(K, 16 * j, 32 * d), acc);
            i = 16 * i + g4, j = 16 * j + l15;
            const double Gj = G[j];
            const float kj = rk[j];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = i + e >= j ? decay_of(G[i + e] - Gj) * (rq[i + e] * kj) * acc[e] : 0.f;
            put4(P, j, i, acc);
        }
        f32x4 x[TT] = {};
        Frag<PC> u[SS];
        Frag<PD> raw[SS];
        if (!idle) {
            {
                Frag<PC> S[DS];
#pragma unroll
                for (int d = 0; d < DS; ++d) S[d] = operand<PC>(state[2 * d], state[2 * d + 1]);
                if (!MAPS)
#pragma unroll
                    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4 *>(b.A + ((((place + n) * p.heads + h) * p.tiles + tile) * DT + d) * 256 + own) = state[d];
#pragma unroll
                for (int d = 0; d < DS; ++d)
#pragma unroll
                    for (int t = 0; t < TT; ++t) x[t] = multiply(along(K, 16 * t, 32 * d), S[d], x[t]);
            }
#pragma unroll
            for (int t = 0; t < TT; ++t) x[t] *= *reinterpret_cast<const f32x4 *>(fu + 16 * t + g4);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < SS; ++t) {
                const f32x4 lo = V.get(32 * t, 16 * wave), hi = V.get(32 * t + 16, 16 * wave);
                raw[t] = operand<PD>(lo, hi);
                u[t] = operand<PC>(lo * *reinterpret_cast<const f32x4 *>(fq + 32 * t + g4), hi * *reinterpret_cast<const f32x4 *>(fq + 32 * t + 16 + g4));
            }
            const float whole = decay_of(G[C - 1]);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                state[d] *= whole;
#pragma unroll
                for (int j = 0; j < SS; ++j) state[d] = multiply(across(Q, 16 * d, 32 * j), u[j], state[d]);
            }
        }
        __syncthreads();                                    // (P is there)
        if (!idle) {
            const auto by = [&](const float *factor, float sign) {
#pragma unroll
                for (int t = 0; t < SS; ++t) {
                    const f32x4 lo = *reinterpret_cast<const f32x4 *>(factor + 32 * t + g4), hi = *reinterpret_cast<const f32x4 *>(factor + 32 * t + 16 + g4);
                    u[t] = operand<PC>(x[2 * t] * lo * sign, x[2 * t + 1] * hi * sign);
                }
            };
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int i = t / 2; i < SS; ++i) x[t] = multiply(along(P, 16 * t, 32 * i), raw[i], x[t]);          // dU
            by(beta, 1.f);
            f32x4 less[TT] = {};
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int i = t / 2; i < SS; ++i) less[t] = multiply(across(M, 16 * t, 32 * i), u[i], less[t]);
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                x[t] -= less[t];
                if (!MAPS) *reinterpret_cast<f32x4 *>(b.F + ((((place + n) * p.heads + h) * p.tiles + tile) * TT + t) * 256 + own) = x[t];
                x[t] *= *reinterpret_cast<const f32x4 *>(beta + 16 * t + g4);       // Y
            }
            if (!MAPS) {
#pragma unroll
                for (int t = 0; t < SS; ++t) u[t] = operand<PC>(x[2 * t], x[2 * t + 1]);
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    f32x4 out = {};
#pragma unroll
                    for (int i = PC - 1; i >= 0; --i)
                        out = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, u[t / 2].part[i]), __builtin_bit_cast(b16x8, unit[t % 2]), out, 0, 0, 0);
                    const int i = 16 * t + l15;
                    if (i < rows) leave<WHOLE>(dv + (first + i) * b.lddv, 16 * tile + g4, p.dv, out);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            by(fk, -1.f);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < SS; ++j) state[d] = multiply(across(K, 16 * d, 32 * j), u[j], state[d]);
        }
        __syncthreads();
    }
    if (idle) return;
    if (MAPS) {
#pragma unroll
        for (int n = 0; n < DT; ++n)
            *reinterpret_cast<f32x4 *>(p.starts + ((((int64_t)(run - 1) * p.heads + h) * p.tiles + tile) * DT + n) * 256 + own) = state[n];
        return;
    }
    if (!b.ds0 || r > 0) return;
#pragma unroll
    for (int n = 0; n < DT; ++n) {
        const int d = 16 * n + g4, col = 16 * tile + l15;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < p.dk && col < p.dv) b.ds0[(head + d + e) * p.dv + col] = state[n][e];
    }
}

// ---------------------------------------------------------------------------------------------------- launches
template <typename T, int DK, int W, bool WHOLE, bool MAPS, bool HELP = false>
grim_status back_launch(const GdrBack &b, hipStream_t stream) {
    constexpr int bytes = BackRoom<T, DK, 16 * W>::bytes;
    const auto kernel = walk_back<T, DK, W, WHOLE, MAPS, HELP>;
    static std::atomic<bool> grown{false};
    if (!lds_of(reinterpret_cast<const void *>(kernel), bytes, grown)) return GRIM_ERR_DEVICE;
    const int64_t groups = runs_of(b.p.N, b.p.nseq, b.p.size) * b.p.heads * ((b.p.tiles + W - 1) / W);
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * W), bytes, stream, b);
    return launched();
}

template <typename T, int DK, bool WHOLE, bool MAPS>
grim_status back_walk(const GdrBack &b, hipStream_t stream) {
    if (b.p.tiles > 4) return back_launch<T, DK, 8, WHOLE, MAPS>(b, stream);
    if constexpr (DK == 64)                                 // (as in the forward pass)
        if (runs_of(b.p.N, b.p.nseq, b.p.size) * b.p.heads > kComputeUnits) return back_launch<T, DK, 4, WHOLE, MAPS>(b, stream);
    return back_launch<T, DK, 8, WHOLE, MAPS, true>(b, stream);
}

template <typename T, int DK, bool WHOLE>
grim_status back_all(const GdrBack &b, hipStream_t stream) {
    const GdrParams &p = b.p;
    if (p.N > 0 && p.size < (uint32_t)p.N) {
        grim_status st = back_walk<T, DK, WHOLE, true>(b, stream);
        if (st != GRIM_OK) return st;
        st = join_runs<T, DK, true>(p, stream);
        if (st != GRIM_OK) return st;
    }
    const grim_status st = back_walk<T, DK, WHOLE, false>(b, stream);
    if (st != GRIM_OK || p.N == 0) return st;
    return gdr_gradients<T, DK, WHOLE>(b, stream);
}

template <typename T>
grim_status back_typed(GdrBack b, const void *states, void *workspace, hipStream_t stream) {
    GdrParams &p = b.p;
    p.size = run_of<T>(p.N, p.nseq, p.heads, p.dv);
    const GdrRoom<T> room(p.N, p.nseq, p.heads, p.dk, p.dv);
    char *kept = static_cast<char *>(const_cast<void *>(states)), *at = static_cast<char *>(workspace);      // (read only)
    p.saved = kept;
    p.maps = reinterpret_cast<float *>(kept + room.saved);
    p.states = reinterpret_cast<float *>(kept + room.saved + room.maps);
    p.E = reinterpret_cast<float *>(kept + room.saved + room.maps + room.states);
    p.starts = reinterpret_cast<float *>(at);
    b.A = reinterpret_cast<float *>(at + room.starts);
    b.F = reinterpret_cast<float *>(at + room.starts + room.states);
    if (p.dk % 8 == 0 && p.dv % 8 == 0) return p.dk <= 64 ? back_all<T, 64, true>(b, stream) : back_all<T, 128, true>(b, stream);
    return p.dk <= 64 ? back_all<T, 64, false>(b, stream) : back_all<T, 128, false>(b, stream);
}

}  // namespace lm
}  // namespace grim

extern "C" grim_status grim_gdr_sequence_backward(const void *q_dev, const void *k_dev, const void *v_dev, grim_dtype dt, int64_t ldq, int64_t ldk, int64_t ldv,
                                                  const float *decay_dev, const float *beta_dev, int64_t ldg, const float *s0_dev,
                                                  const int32_t *seq_start_dev, int32_t nseq, int64_t N, int32_t heads, int32_t key_heads, int32_t dk,
                                                  int32_t dv, float scale, float norm_eps, const void *states_dev, const void *dy_dev, int64_t lddy,
                                                  const float *ds_last_dev, void *dq_dev, int64_t lddq, void *dk_dev, int64_t lddk, void *dv_dev,
                                                  int64_t lddv, float *ddecay_dev, float *dbeta_dev, int64_t lddg, float *ds0_dev, void *workspace,
                                                  int64_t workspace_bytes, void *hip_stream) {
    using namespace grim::lm;
    const int64_t keys = (int64_t)key_heads * dk, values = (int64_t)heads * dv;
    const grim_status st = gdr_check(dt, N, nseq, seq_start_dev != nullptr, heads, key_heads, dk, dv, scale, norm_eps);
    if (st != GRIM_OK) return st;
    const struct { int64_t ld, width; } all[] = {{ldq, keys}, {ldk, keys}, {ldv, values}, {ldg, heads}, {lddy, values}, {lddq, keys}, {lddk, keys}, {lddv, values}, {lddg, heads}};
    for (const auto &a : all)
        if (a.ld < a.width || !fits(N, a.ld)) return GRIM_ERR_SHAPE;
    if (N > 0 && (!q_dev || !k_dev || !v_dev || !decay_dev || !beta_dev || !states_dev || !dy_dev || !dq_dev || !dk_dev || !dv_dev || !ddecay_dev || !dbeta_dev || !workspace))
        return GRIM_ERR_NULL;
    if (workspace_bytes < grim_gdr_workspace(N, nseq, heads, key_heads, dk, dv) && N > 0) return GRIM_ERR_SHAPE;
    if (N == 0 && !ds0_dev) return GRIM_OK;
    if (ds_last_dev && ds0_dev && overlap(ds_last_dev, ds0_dev, (int64_t)nseq * heads * dk * dv * 4)) return GRIM_ERR_UNSUPPORTED;
    (void)s0_dev;                                           // (the states in front of the first chunks are kept)
    GdrBack b{};
    GdrParams &p = b.p;
    p.q = q_dev, p.k = k_dev, p.v = v_dev, p.decay = decay_dev, p.beta = beta_dev, p.seq_start = seq_start_dev;
    p.ldq = ldq, p.ldk = ldk, p.ldv = ldv, p.ldg = ldg, p.N = N, p.nseq = nseq, p.heads = heads, p.group = heads / key_heads, p.dk = dk, p.dv = dv;
    p.tiles = tiles_of(dv), p.scale = scale, p.norm_eps = norm_eps;
    b.dy = dy_dev, b.ds_last = ds_last_dev, b.dq = dq_dev, b.dk = dk_dev, b.dv = dv_dev, b.ddecay = ddecay_dev, b.dbeta = dbeta_dev, b.ds0 = ds0_dev;
    b.lddy = lddy, b.lddq = lddq, b.lddk = lddk, b.lddv = lddv, b.lddg = lddg, b.key_heads = key_heads;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dt == GRIM_F32   ? back_typed<float>(b, states_dev, workspace, stream)
           : dt == GRIM_F16 ? back_typed<f16>(b, states_dev, workspace, stream)
                            : back_typed<bf16>(b, states_dev, workspace, stream);
}
