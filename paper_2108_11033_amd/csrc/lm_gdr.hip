// The gated delta rule over packed sequences, forward.
//
//     D_t = exp(g_t) S_(t-1)     e_t = v_t - D_t' k_t     S_t = D_t + beta_t k_t e_t'     y_t = scale S_t' q_t
//
// Tokens in chunks of one sequence.  With G the running sums of g in a chunk, S the states in front of it, and w_ij = exp(G_i - G_j),
//     X_i = v_i - exp(G_i) S' k_i        L_ij = w_ij k_i . k_j (i > j)        E = X - L beta E        U = beta E
//     y_i = scale (exp(G_i) S' q_i + sum over j <= i of w_ij (q_i . k_j) U_j)
//     S_next = exp(G_end) S + sum over j of exp(G_end - G_j) k_j U_j'
// so that all but the states' way from chunk to chunk are products of matrices.  E = X - M beta X with the strictly lower matrix M = L - L beta M, which takes
// keys and gates alone: one launch forms it for all chunks, the second walks over the chunks.  Keys and queries that count divided by their lengths
// enter the products as they are, their lengths scale the results (so that 16-bit operands stay exact).  G is summed in fp64: differences of large sums
// (a decay of -10000 that forgets all, among others near 0) keep their digits.
#include "lm_gdr.hpp"

namespace grim {
namespace lm {

// M of every chunk and head, and G: a workgroup each.  L by the matrix cores, M by forward substitution: blocks of 16 x 16, those on the diagonal a column a lane, then
// block by block away from it, M_IJ = Z - M_II beta Z with Z = L_IJ - sum over J <= K < I of L_IK beta M_KJ, in fp32 on the matrix cores.
// Bound by the vector ALUs (two thirds of its time: lengths, decays, substitution, splitting): 4096 chunks of 128-wide heads 56 us, 6640 of 64-wide ones 72.
template <typename T, int DK, bool WHOLE>
__global__ void __launch_bounds__(kMatrixThreads) chunk_matrices(GdrParams p) {
    constexpr int C = Gdr<T>::chunk, PD = Gdr<T>::data, PC = Gdr<T>::comp, TT = C / 32, B = C / 16, LD = C + 4;
    using Keys = Tile<PD, C, DK, PAIRED>;
    constexpr int square = C * LD * 4;
    __shared__ __attribute__((aligned(16))) char lds[square + (Keys::bytes > square ? Keys::bytes : square)];
    __shared__ double G[C];
    __shared__ float tokens[3 * C];                          // beta, what keys and queries count with
    float *beta = tokens, *rk = tokens + C, *rq = tokens + 2 * C;
    float *L = reinterpret_cast<float *>(lds), *M = reinterpret_cast<float *>(lds + square);        // (M after the keys are done with)
    const Keys keys{reinterpret_cast<uint16_t *>(lds + square)};
    const uint32_t place = blockIdx.x / (uint32_t)p.heads;
    const int h = (int)(blockIdx.x % (uint32_t)p.heads);
    const int s = sequence_of(p.seq_start, p.nseq, p.N, C, place);
    const Span span(p.seq_start, s, p.N);
    const int64_t first = span.first + (int64_t)(place - place_of(span, s, C)) * C;
    if (first >= span.end) return;
    const int rows = (int)min((int64_t)C, span.end - first);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15, lq = lane >> 4;
    Rows<WHOLE, T, kMatrixThreads, C, DK> k, q;
    q.fetch(static_cast<const T *>(p.q) + first * p.ldq + (int64_t)(h / p.group) * p.dk, p.ldq, rows, p.dk);
    k.fetch(static_cast<const T *>(p.k) + first * p.ldk + (int64_t)(h / p.group) * p.dk, p.ldk, rows, p.dk);
    if (wave == 0) {
        const float g = lane < rows ? p.decay[(first + lane) * p.ldg + h] : 0.f;
        double sum = (g < kLeastDecay ? kLeastDecay : (double)g) * 1.44269504088896340736;
#pragma unroll
        for (int n = 1; n < C; n *= 2) {
            const double before = __shfl_up(sum, n, 64);
            if (lane >= n) sum += before;
        }
        if (lane < C) G[lane] = sum, beta[lane] = lane < rows ? p.beta[(first + lane) * p.ldg + h] : 0.f;
    }
    k.place(keys, rows, p.dk);
    k.lengths(rows, p.dk, rk, p.norm_eps, 1.f);
    q.lengths(rows, p.dk, rq, p.norm_eps, p.scale);
    __syncthreads();
    {
        const int j0 = (wave >> 1) * (C / 2), i0 = (wave & 1) * (C / 2);
        f32x4 acc[TT][TT] = {};
        if (j0 <= i0)
            for (int ks = 0; ks < DK; ks += 32) {
                Frag<PD> a[TT], b[TT];
#pragma unroll
                for (int t = 0; t < TT; ++t) a[t] = along(keys, j0 + 16 * t, ks), b[t] = along(keys, i0 + 16 * t, ks);
#pragma unroll
                for (int x = 0; x < TT; ++x)
#pragma unroll
                    for (int y = 0; y < TT; ++y) acc[x][y] = multiply(a[x], b[y], acc[x][y]);
            }
#pragma unroll
        for (int x = 0; x < TT; ++x)
#pragma unroll
            for (int y = 0; y < TT; ++y) {
                const int j = j0 + 16 * x + lq * 4, i = i0 + 16 * y + l15;
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = i > j + e ? decay_of(G[i] - G[j + e]) * rk[i] * rk[j + e] * acc[x][y][e] : 0.f;
                *reinterpret_cast<f32x4 *>(L + i * LD + j) = v;
            }
    }
    __syncthreads();
    if (wave < B) {
        const int at = wave * 16;
        float m[16];                                        // beta M, down the lane's column
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float *row = L + (at + r) * LD + at;
            float x = row[l15];
#pragma unroll
            for (int t = 0; t < r; ++t) x = __builtin_fmaf(-row[t], m[t], x);
            m[r] = beta[at + r] * x;
            if (lane < 16) M[(at + r) * LD + at + l15] = x;
        }
    }
    __syncthreads();
#pragma unroll
    for (int d = 1; d < B; ++d) {
        const int I = d + wave, J = wave;
        if (I < B) {
            f32x4 acc = {};
            for (int K = J; K < I; ++K)
#pragma unroll
                for (int t = 0; t < 16; t += 4) {
                    const int n = K * 16 + t + lq;
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(L[(I * 16 + l15) * LD + n] * beta[n], M[n * LD + J * 16 + l15], acc, 0, 0, 0);
                }
            f32x4 z;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                z[e] = L[(I * 16 + lq * 4 + e) * LD + J * 16 + l15] - acc[e];
                M[(I * 16 + lq * 4 + e) * LD + J * 16 + l15] = z[e];
            }
            __threadfence_block();
            acc = {};
#pragma unroll
            for (int t = 0; t < 16; t += 4) {
                const int n = I * 16 + t + lq;
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(M[(I * 16 + l15) * LD + n] * beta[n], M[n * LD + J * 16 + l15], acc, 0, 0, 0);
            }
            __threadfence_block();
#pragma unroll
            for (int e = 0; e < 4; ++e) M[(I * 16 + lq * 4 + e) * LD + J * 16 + l15] = z[e] - acc[e];
        }
        __syncthreads();
    }
    const Saved<T> saved(p, place, h);
    if (threadIdx.x < C) saved.G()[threadIdx.x] = G[threadIdx.x];
    if (threadIdx.x < C) {
        const int i = threadIdx.x;
        float *to = saved.tokens() + i;
        const float since = decay_of(G[i]);
        to[0] = beta[i], to[C] = since * rk[i], to[2 * C] = decay_of(G[C - 1] - G[i]) * rk[i], to[3 * C] = since * rq[i], to[4 * C] = rk[i], to[5 * C] = rq[i];
    }
    for (int q = threadIdx.x; q < Saved<T>::part / 8; q += kMatrixThreads) {          // four pieces of 8 to a row of 32; first the tall block, then the rest
        const int i = q < C * 4 ? q / 4 : q / 4 - C + 32, c = (q < C * 4 ? 0 : 32) + q % 4 * 4;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = c + j % 4 + j / 4 * 16;
            v[j] = at / 16 > i / 16 ? 0.f : M[i * LD + at];
        }
#pragma unroll
        for (int t = 0; t < PC; ++t) {
            bf16 part[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) part[j] = (bf16)v[j], v[j] -= (float)part[j];
            __builtin_memcpy(saved.M() + t * Saved<T>::part + q * 8, part, 16);
        }
    }
}

// ---------------------------------------------------------------------------------------------------- from chunk to chunk
// What a workgroup of the walk keeps in LDS (MAPS: without queries and what is made of them).
template <typename T, int DK, int COLS, bool MAPS>
struct WalkRoom {
    static constexpr int C = Gdr<T>::chunk, PD = Gdr<T>::data, PC = Gdr<T>::comp;
    using Keys = Tile<PD, C, DK>;
    using Queries = Tile<PD, C, DK, PAIRED>;
    using Square = Triangle<PC, C, PAIRED>;
    using Vals = Values<T, C, COLS>;
    static constexpr int keys = 0, values = keys + Keys::bytes, matrix = values + Vals::bytes, decays = matrix + Square::bytes, factors = decays + C * 8, queries = factors + C * 24,
                         products = queries + Queries::bytes, bytes = MAPS ? queries : products + Square::bytes;
    static_assert(bytes <= 160 * 1024, "LDS");
    Keys K;
    Queries Q;
    Square M, P;
    Vals V;
    double *G;
    float *tokens;
    const float *beta, *fk, *fu, *fq, *rk, *rq;
    __device__ __forceinline__ explicit WalkRoom(char *at) {
        K.at = reinterpret_cast<uint16_t *>(at + keys), Q.at = reinterpret_cast<uint16_t *>(at + queries);
        M.put(at + matrix), P.put(at + products);
        V.at = reinterpret_cast<T *>(at + values), G = reinterpret_cast<double *>(at + decays), tokens = reinterpret_cast<float *>(at + factors);
        beta = tokens, fk = tokens + C, fu = tokens + 2 * C, fq = tokens + 3 * C, rk = tokens + 4 * C, rq = tokens + 5 * C;
    }
};

// A workgroup takes 16 W columns of the states of a run of chunks of a sequence's head.  All that a chunk does to a column of the states stays in that column, so each of its W waves
// has 16 columns to itself from chunk to chunk, in registers: results that are sums over tokens or keys are the next product's operands.  The waves meet only where keys, queries,
// values and M are placed in LDS and where the products of queries and keys, which all need, are formed.
// A chunk is six phases between barriers, of fetches, LDS reads, matrix and vector work in turn, none of which takes half the time (matrix cores 33 %, vector ALUs 40 %, LDS 40 % of it).  4096
// chunks of 128 x 128 heads in bf16 with all that the backward pass needs 165 us, 0.73 GB moved at 4.4 TB/s; the maps of their 31 runs 170 us; 64 x 64 heads, 6000 chunks, 163 and 64.
// MAPS: no outputs; what every run but a sequence's last does to the states, as S -> A S + B: B's columns (into the places of the states in front of the next run; of a sequence's
// first run, whose start is known, these are the states themselves) come from a start of zeros, A's from the columns of 1 and values of zero.
// HELP: the second half of the waves has no columns; they form the products of queries and keys.
template <typename T, int DK, int W, bool WHOLE, bool MAPS, bool HELP>
__global__ void __launch_bounds__(64 * W, 2) walk(GdrParams p) {
    constexpr int C = Gdr<T>::chunk, PD = Gdr<T>::data, PC = Gdr<T>::comp, THREADS = 64 * W, COLS = 16 * W;
    constexpr int TT = C / 16, SS = C / 32, DT = DK / 16, DS = DK / 32;     // tiles of tokens, sums over them; of the states' rows
    using Room = WalkRoom<T, DK, COLS, MAPS>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const Room m(lds);

    // (the workgroups of a run, whose heads read the same rows, lie together)
    const uint32_t value_blocks = (p.tiles + W - 1) / W, blocks = value_blocks + (MAPS ? (DT + W - 1) / W : 0), heads = (uint32_t)p.heads;
    const int block = (int)(blockIdx.x % blocks), h = (int)(blockIdx.x / blocks % heads);
    const uint32_t run = blockIdx.x / blocks / heads;
    const int s = sequence_of(p.seq_start, p.nseq, p.N, p.size, run);
    const Span span(p.seq_start, s, p.N);
    const uint32_t r = run - place_of(span, s, p.size);     // of the sequence's runs
    const int64_t from = span.first + (int64_t)r * p.size, to = min(span.end, from + p.size);
    if (MAPS ? to >= span.end : from >= to && r > 0) return;            // (an empty sequence has its first run for its last states)
    const bool map = MAPS && block >= (int)value_blocks;
    if (map && r == 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15, g4 = (lane >> 4) * 4, own = l15 * 16 + g4;
    const int tile = (map ? block - (int)value_blocks : block) * W + wave, tiles = map ? DT : p.tiles, col0 = map ? 0 : block * COLS;
    const bool idle = tile >= tiles;
    const T *q = static_cast<const T *>(p.q) + (int64_t)(h / p.group) * p.dk, *k = static_cast<const T *>(p.k) + (int64_t)(h / p.group) * p.dk;
    const T *v = static_cast<const T *>(p.v) + (int64_t)h * p.dv + col0;
    T *y = static_cast<T *>(p.y) + (int64_t)h * p.dv;

    f32x4 state[DT];                                        // rows 16 n + g4 .. + 3, column 16 tile + l15
    const int64_t head = ((int64_t)s * p.heads + h) * p.dk;
#pragma unroll
    for (int n = 0; n < DT; ++n) {
        const int d = 16 * n + g4, col = 16 * tile + l15;
        state[n] = f32x4{};
        if (MAPS && r > 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) state[n][e] = map && d + e == col ? 1.f : 0.f;
        } else if (r > 0) {
            if (tile < p.tiles) state[n] = *reinterpret_cast<const f32x4 *>(p.starts + ((((int64_t)run * p.heads + h) * p.tiles + tile) * DT + n) * 256 + own);
        } else if (p.s0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) state[n][e] = p.s0[(head + min(d + e, p.dk - 1)) * p.dv + min(col, p.dv - 1)];
        }
    }
#pragma unroll
    for (int n = 0; n < DT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            asm volatile("" : "+v"(state[n][e]));           // (all are asked for before any is looked at)
            if (16 * n + g4 + e >= p.dk || 16 * tile + l15 >= (map ? p.dk : p.dv)) state[n][e] = 0.f;
        }

    // what the next chunk brings
    Rows<WHOLE, T, THREADS, C, DK> kn, qn;
    Rows<WHOLE, T, THREADS, C, COLS> vn;
    constexpr int pieces = PC * Saved<T>::part / 8, MP = (pieces + THREADS - 1) / THREADS, TP = (6 * C + THREADS - 1) / THREADS;
    u32x4 mn[MP];
    double Gn = 0.;
    float tn[TP];
    const int64_t place = place_of(span, s, C) + r * (p.size / C);
    const auto fetch = [&](int64_t n, int64_t first) {
        const int rows = __builtin_amdgcn_readfirstlane((int)min((int64_t)C, to - first));
        kn.fetch(k + first * p.ldk, p.ldk, rows, p.dk);
        if (!MAPS) qn.fetch(q + first * p.ldq, p.ldq, rows, p.dk);
        vn.fetch(v + first * p.ldv, p.ldv, rows, p.dv - col0);
        const Saved<T> saved(p, place + n, h);
#pragma unroll
        for (int i = 0; i < MP; ++i) mn[i] = reinterpret_cast<const u32x4 *>(saved.M())[min(i * THREADS + threadIdx.x, pieces - 1u)];
        Gn = saved.G()[threadIdx.x % C];
#pragma unroll
        for (int i = 0; i < TP; ++i) tn[i] = saved.tokens()[min(i * THREADS + threadIdx.x, 6 * C - 1u)];
    };
    if (from < to) fetch(0, from);
    for (int64_t n = 0, first = from; first < to; ++n, first += C) {
        const int rows = __builtin_amdgcn_readfirstlane((int)min((int64_t)C, to - first));
        kn.place(m.K, rows, p.dk);
        if (!MAPS) qn.place(m.Q, rows, p.dk);
        vn.keep(m.V.at, m.V.ld, map ? 0 : rows, p.dv - col0);
#pragma unroll
        for (int i = 0; i < MP; ++i) {
            const int piece = i * THREADS + (int)threadIdx.x;
            if (piece < pieces) *reinterpret_cast<u32x4 *>(m.M.piece(piece)) = mn[i];
        }
        if (threadIdx.x < C) m.G[threadIdx.x] = Gn;
#pragma unroll
        for (int i = 0; i < TP; ++i)
            if (i * THREADS + (int)threadIdx.x < 6 * C) m.tokens[i * THREADS + threadIdx.x] = tn[i];
        if (first + C < to) fetch(n + 1, first + C);
        __syncthreads();
        if (!MAPS) {                                        // the products of queries and keys
            constexpr int WORK = HELP ? W / 2 : W, EACH = (Lower<C>::count + WORK - 1) / WORK;
#pragma unroll 1
            for (int n = 0; n < EACH; ++n) {
                const int pair = n * WORK + wave - (W - WORK);
                if (pair < 0 || pair >= Lower<C>::count) break;
                int i, j;
                Lower<C>::get(pair, i, j);
                f32x4 acc = {};
#pragma unroll
                for (int d = 0; d < DS; ++d) acc = multiply(along(m.K, 16 * j, 32 * d), along(m.Q, 16 * i, 32 * d), acc);
                i = 16 * i + l15, j = 16 * j + g4;
                const double Gi = m.G[i];
                const float qi = m.rq[i];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = i >= j + e ? decay_of(Gi - m.G[j + e]) * (qi * m.rk[j + e]) * acc[e] : 0.f;
                put4(m.P, i, j, acc);
            }
        }
        f32x4 x[TT] = {}, out[TT] = {};                     // tokens x columns, columns x tokens
        Frag<PC> u[SS];
        if (!idle) {
        {
            if (!MAPS && p.states)
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    *reinterpret_cast<f32x4 *>(p.states + ((((place + n) * p.heads + h) * p.tiles + tile) * DT + d) * 256 + own) = state[d];
#pragma unroll
            for (int d = 0; d < DS; ++d) {
                const Frag<PC> S = operand<PC>(state[2 * d], state[2 * d + 1]);
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    const Frag<PD> a = along(m.K, 16 * t, 32 * d);
                    x[t] = multiply(a, S, x[t]);
                    if (MAPS) continue;
                    const Frag<PD> e = along(m.Q, 16 * t, 32 * d);
                    out[t] = multiply(S, e, out[t]);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const f32x4 f = *reinterpret_cast<const f32x4 *>(m.fk + 16 * t + g4);
            const float fo = m.fq[16 * t + l15];
            x[t] = m.V.get(16 * t, 16 * wave) - f * x[t], out[t] *= fo;
        }
        const auto by = [&](const float *factor, f32x4 (&a)[TT]) {
#pragma unroll
            for (int t = 0; t < SS; ++t) {
                const f32x4 lo = *reinterpret_cast<const f32x4 *>(factor + 32 * t + g4), hi = *reinterpret_cast<const f32x4 *>(factor + 32 * t + 16 + g4);
                u[t] = operand<PC>(a[2 * t] * lo, a[2 * t + 1] * hi);
            }
        };
        by(m.beta, x);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            f32x4 less = {};
#pragma unroll
            for (int j = 0; j <= t / 2; ++j) {
                const Frag<PC> a = along(m.M, 16 * t, 32 * j);
                less = multiply(a, u[j], less);
            }
            const f32x4 bt = *reinterpret_cast<const f32x4 *>(m.beta + 16 * t + g4);
            x[t] -= less;
            if (!MAPS && p.states)
                *reinterpret_cast<f32x4 *>(p.E + ((((place + n) * p.heads + h) * p.tiles + tile) * TT + t) * 256 + own) = x[t];
            x[t] *= bt;                                     // U
        }
        __builtin_amdgcn_sched_barrier(0);
        by(m.fu, x);
        const float whole = decay_of(m.G[C - 1]);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            state[d] *= whole;
#pragma unroll
            for (int j = 0; j < SS; ++j) {
                const Frag<PD> a = across(m.K, 16 * d, 32 * j);
                state[d] = multiply(a, u[j], state[d]);
            }
        }
        if (!MAPS)
#pragma unroll
            for (int t = 0; t < SS; ++t) u[t] = operand<PC>(x[2 * t], x[2 * t + 1]);
        }
        __syncthreads();                                    // (the products of queries and keys are there)
        if (MAPS || idle) {
            if (!MAPS) __syncthreads();
            continue;
        }
#pragma unroll
        for (int t = 0; t < TT; ++t) {
#pragma unroll
            for (int j = 0; j <= t / 2; ++j) {
                const Frag<PC> a = along(m.P, 16 * t, 32 * j);
                out[t] = multiply(u[j], a, out[t]);
            }
            const int i = 16 * t + l15;
            if (i < rows) leave<WHOLE>(y + (first + i) * p.ldy, 16 * tile + g4, p.dv, out[t]);
        }
        __syncthreads();
    }
    if (idle) return;
    if (MAPS) {
#pragma unroll
        for (int n = 0; n < DT; ++n) {
            if (!map) *reinterpret_cast<f32x4 *>(p.starts + ((((int64_t)(run + 1) * p.heads + h) * p.tiles + tile) * DT + n) * 256 + own) = state[n];
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) p.maps[(((int64_t)run * p.heads + h) * DK + 16 * n + g4 + e) * DK + 16 * tile + l15] = state[n][e];
        }
        return;
    }
    if (!p.s_last || to < span.end) return;
#pragma unroll
    for (int n = 0; n < DT; ++n) {
        const int d = 16 * n + g4, col = 16 * tile + l15;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < p.dk && col < p.dv) p.s_last[(head + d + e) * p.dv + col] = state[n][e];
    }
}

// ---------------------------------------------------------------------------------------------------- launches
template <typename T, int DK, int W, bool WHOLE, bool MAPS, bool HELP = false>
grim_status walk_launch(const GdrParams &p, hipStream_t stream) {
    constexpr int bytes = WalkRoom<T, DK, 16 * W, MAPS>::bytes;
    const auto kernel = walk<T, DK, W, WHOLE, MAPS, HELP>;
    static std::atomic<bool> grown{false};
    if (!lds_of(reinterpret_cast<const void *>(kernel), bytes, grown)) return GRIM_ERR_DEVICE;
    const int64_t blocks = (p.tiles + W - 1) / W + (MAPS ? (DK / 16 + W - 1) / W : 0), groups = runs_of(p.N, p.nseq, p.size) * p.heads * blocks;
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * W), bytes, stream, p);
    return launched();
}

template <typename T, int DK, bool WHOLE>
grim_status gdr_launch(const GdrParams &p, hipStream_t stream) {
    if (p.N > 0) {
        const int64_t places = places_of<T>(p.N, p.nseq);
        hipLaunchKernelGGL((chunk_matrices<T, DK, WHOLE>), dim3((unsigned)(places * p.heads)), dim3(kMatrixThreads), 0, stream, p);
        grim_status st = launched();
        if (st != GRIM_OK) return st;
        if (p.size < (uint32_t)p.N) {
            st = walk_launch<T, DK, 4, WHOLE, true>(p, stream);
            if (st != GRIM_OK) return st;
            st = join_runs<T, DK, false>(p, stream);
            if (st != GRIM_OK) return st;
        }
    }
    if (p.tiles > 4) return walk_launch<T, DK, 8, WHOLE, false>(p, stream);
    // 64 columns: four waves, two such workgroups to a compute unit, or where there are not enough of them (or for keys of 128, which are too much for the registers of four
    // waves) another four that help: 512 tokens in 8 sequences, 16 heads of 64 x 64 in fp16, 42.1 us with four and 36.1 with eight (with chunk_matrices); 24007 in 40 sequences, in bf16,
    // both directions, 759 with four and 775 with eight.
    if constexpr (DK == 64)
        if (runs_of(p.N, p.nseq, p.size) * p.heads > kComputeUnits) return walk_launch<T, DK, 4, WHOLE, false>(p, stream);
    return walk_launch<T, DK, 8, WHOLE, false, true>(p, stream);
}

template <typename T>
grim_status gdr_typed(GdrParams p, void *states, void *workspace, hipStream_t stream) {
    p.size = run_of<T>(p.N, p.nseq, p.heads, p.dv);
    const GdrRoom<T> room(p.N, p.nseq, p.heads, p.dk, p.dv);
    char *at = static_cast<char *>(states ? states : workspace);
    p.saved = at;
    p.maps = reinterpret_cast<float *>(at + room.saved);
    if (states) {
        p.states = reinterpret_cast<float *>(at + room.saved + room.maps);
        p.E = reinterpret_cast<float *>(at + room.saved + room.maps + room.states);
        p.starts = static_cast<float *>(workspace);
    } else {
        p.starts = reinterpret_cast<float *>(at + room.saved + room.maps);
    }
    if (p.dk % 8 == 0 && p.dv % 8 == 0) return p.dk <= 64 ? gdr_launch<T, 64, true>(p, stream) : gdr_launch<T, 128, true>(p, stream);
    return p.dk <= 64 ? gdr_launch<T, 64, false>(p, stream) : gdr_launch<T, 128, false>(p, stream);
}

}  // namespace lm
}  // namespace grim

extern "C" {

int64_t grim_gdr_states(int64_t N, int32_t nseq, int32_t heads, int32_t dk, int32_t dv) {
    using namespace grim::lm;
    if (gdr_check(N, nseq, heads, 1, dk, dv) != GRIM_OK) return 0;
    const int64_t a = GdrRoom<float>(N, nseq, heads, dk, dv).kept(), b = GdrRoom<f16>(N, nseq, heads, dk, dv).kept();
    return a > b ? a : b;
}

int64_t grim_gdr_workspace(int64_t N, int32_t nseq, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv) {
    using namespace grim::lm;
    if (gdr_check(N, nseq, heads, key_heads, dk, dv) != GRIM_OK) return 0;
    const int64_t a = GdrRoom<float>(N, nseq, heads, dk, dv).scratch(), b = GdrRoom<f16>(N, nseq, heads, dk, dv).scratch();
    return a > b ? a : b;
}

grim_status grim_gdr_sequence(const void *q_dev, const void *k_dev, const void *v_dev, grim_dtype dt, int64_t ldq, int64_t ldk, int64_t ldv,
                              const float *decay_dev, const float *beta_dev, int64_t ldg, const float *s0_dev, const int32_t *seq_start_dev,
                              int32_t nseq, int64_t N, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv, float scale, float norm_eps,
                              void *y_dev, int64_t ldy, float *s_last_dev, void *states_dev, void *workspace, int64_t workspace_bytes,
                              void *hip_stream) {
    using namespace grim::lm;
    const int64_t keys = (int64_t)key_heads * dk, values = (int64_t)heads * dv;
    const grim_status st = gdr_check(dt, N, nseq, seq_start_dev != nullptr, heads, key_heads, dk, dv, scale, norm_eps);
    if (st != GRIM_OK) return st;
    if (ldq < keys || ldk < keys || ldv < values || ldy < values || ldg < heads || !fits(N, ldq) || !fits(N, ldk) || !fits(N, ldv) || !fits(N, ldy) ||
        !fits(N, ldg))
        return GRIM_ERR_SHAPE;
    if (N > 0 && (!q_dev || !k_dev || !v_dev || !decay_dev || !beta_dev || !y_dev || !workspace)) return GRIM_ERR_NULL;
    if (workspace_bytes < grim_gdr_workspace(N, nseq, heads, key_heads, dk, dv) && N > 0) return GRIM_ERR_SHAPE;
    if (N == 0 && !s_last_dev) return GRIM_OK;
    if (s_last_dev && s0_dev && overlap(s0_dev, s_last_dev, (int64_t)nseq * heads * dk * dv * 4)) return GRIM_ERR_UNSUPPORTED;
    GdrParams p{};
    p.q = q_dev, p.k = k_dev, p.v = v_dev, p.decay = decay_dev, p.beta = beta_dev, p.s0 = s0_dev, p.seq_start = seq_start_dev, p.y = y_dev, p.s_last = s_last_dev;
    p.ldq = ldq, p.ldk = ldk, p.ldv = ldv, p.ldg = ldg, p.ldy = ldy, p.N = N, p.nseq = nseq, p.heads = heads, p.group = heads / key_heads, p.dk = dk, p.dv = dv;
    p.tiles = tiles_of(dv), p.scale = scale, p.norm_eps = norm_eps;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dt == GRIM_F32   ? gdr_typed<float>(p, states_dev, workspace, stream)
           : dt == GRIM_F16 ? gdr_typed<f16>(p, states_dev, workspace, stream)
                            : gdr_typed<bf16>(p, states_dev, workspace, stream);
}

}  // extern "C"
