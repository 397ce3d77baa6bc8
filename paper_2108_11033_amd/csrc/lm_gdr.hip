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
template <typename T, int DK>
__global__ void __launch_bounds__(kGdrThreads) chunk_matrices(GdrParams p) {
    constexpr int C = Gdr<T>::chunk, PD = Gdr<T>::data, PC = Gdr<T>::comp, TT = C / 32, B = C / 16, LD = C + 4;
    using Keys = Tile<PD, C, DK>;
    constexpr int square = C * LD * 4;
    __shared__ __attribute__((aligned(16))) char lds[square + (Keys::bytes > square ? Keys::bytes : square)];
    __shared__ double G[C];
    __shared__ float beta[C], rk[C];
    float *L = reinterpret_cast<float *>(lds), *M = reinterpret_cast<float *>(lds + square);        // (M after the keys are done with)
    const Keys keys{reinterpret_cast<uint16_t *>(lds + square)};
    const int64_t place = blockIdx.x / p.heads;
    const int h = (int)(blockIdx.x % p.heads);
    const int s = sequence_of<C>(p.seq_start, p.nseq, p.N, place);
    const Span span(p.seq_start, s, p.N);
    const int64_t first = span.first + (place - (span.first / C + s)) * C;
    const int rows = (int)min((int64_t)C, span.end - first);
    if (rows <= 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15, lq = lane >> 4;
    Rows<T, C, DK> k;
    k.fetch(static_cast<const T *>(p.k) + first * p.ldk + (int64_t)(h / p.group) * p.dk, p.ldk, rows, p.dk);
    if (wave == 0) {
        const float g = lane < rows ? p.decay[(first + lane) * p.ldg + h] : 0.f;
        double sum = g < kLeastDecay ? kLeastDecay : (double)g;
#pragma unroll
        for (int n = 1; n < C; n *= 2) {
            const double before = __shfl_up(sum, n, 64);
            if (lane >= n) sum += before;
        }
        if (lane < C) G[lane] = sum, beta[lane] = lane < rows ? p.beta[(first + lane) * p.ldg + h] : 0.f;
    }
    k.place(keys, rk, p.norm_eps, 1.f);
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
                f32x4 v = {};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i > j + e) v[e] = expf((float)(G[i] - G[j + e])) * rk[i] * rk[j + e] * acc[x][y][e];
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
    for (int q = threadIdx.x; q < C * C / 8; q += kGdrThreads) {
        const int i = q / (C / 8), c = q % (C / 8) * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c / 16 > i / 16 ? 0.f : M[i * LD + c + j];
#pragma unroll
        for (int t = 0; t < PC; ++t) {
            bf16 part[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) part[j] = (bf16)v[j], v[j] -= (float)part[j];
            __builtin_memcpy(saved.M() + t * C * C + q * 8, part, 16);
        }
    }
}

// ---------------------------------------------------------------------------------------------------- from chunk to chunk
// What a workgroup of the walk keeps in LDS.
template <typename T, int DK>
struct WalkRoom {
    static constexpr int C = Gdr<T>::chunk, PD = Gdr<T>::data, PC = Gdr<T>::comp;
    using Keys = Tile<PD, C, DK>;
    using States = Tile<PC, DK, kGdrColumns>;
    using Square = Tile<PC, C, C>;
    using Columns = Tile<PC, C, kGdrColumns>;
    static constexpr int keys = 0, queries = keys + Keys::bytes, states = queries + Keys::bytes, square = states + States::bytes,
                         x = square + Square::bytes, u = x + Columns::bytes, G = u + Columns::bytes, beta = G + C * 8, rk = beta + C * 4, rq = rk + C * 4,
                         bytes = rq + C * 4;
    static_assert(bytes <= 160 * 1024, "LDS");
};

// Four elements of a head's row of values from column c; zeros behind its width.
template <typename T>
__device__ __forceinline__ Pack<T, 4> fetch4(const T *row, int c, int width) {
    if (c + 4 <= width) return load<4>(row + c);
    Pack<T, 4> r;
#pragma unroll
    for (int j = 0; j < 4; ++j) put(r, j, c + j < width ? row[c + j] : (T)0.f);
    return r;
}

template <typename T>
__device__ __forceinline__ void store4(T *row, int c, int width, f32x4 v) {
    if (c + 4 <= width) {
        const float t[4] = {v[0], v[1], v[2], v[3]};
        store(row + c, t);
    } else
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < width) row[c + j] = (T)v[j];
}

// A workgroup takes 64 columns of the states of a sequence's head.  Its four waves have a half of the columns and a half of the tokens (of the rows of the states) each.
// Columns of the states are rows of the results of the products: lanes then have four columns of a token, which lie together in memory and in LDS.
template <typename T, int DK>
__global__ void __launch_bounds__(kGdrThreads) walk(GdrParams p) {
    constexpr int C = Gdr<T>::chunk, PD = Gdr<T>::data, PC = Gdr<T>::comp, TT = C / 32, TD = DK / 32;
    using Room = WalkRoom<T, DK>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const auto tile = [&](int at) { return reinterpret_cast<uint16_t *>(lds + at); };
    const typename Room::Keys K{tile(Room::keys)}, Q{tile(Room::queries)};
    const typename Room::States S{tile(Room::states)};
    const typename Room::Square M{tile(Room::square)};      // then the products of queries and keys
    const typename Room::Columns X{tile(Room::x)}, U{tile(Room::u)};
    double *G = reinterpret_cast<double *>(lds + Room::G);
    float *beta = reinterpret_cast<float *>(lds + Room::beta), *rk = reinterpret_cast<float *>(lds + Room::rk), *rq = reinterpret_cast<float *>(lds + Room::rq);

    int64_t b = blockIdx.x;
    const int block = (int)(b % p.blocks);
    b /= p.blocks;
    const int h = (int)(b % p.heads), s = (int)(b / p.heads);
    const Span span(p.seq_start, s, p.N);
    const int64_t place = span.first / C + s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15, lq = lane >> 4;
    const int v0 = (wave >> 1) * 32, t0 = (wave & 1) * (C / 2), d0 = (wave & 1) * (DK / 2), j0 = (wave >> 1) * (C / 2);
    const int col = block * kGdrColumns + v0 + lq * 4;      // of the lane's first value
    const T *q = static_cast<const T *>(p.q) + (int64_t)(h / p.group) * p.dk, *k = static_cast<const T *>(p.k) + (int64_t)(h / p.group) * p.dk;
    const T *v = static_cast<const T *>(p.v) + (int64_t)h * p.dv;
    T *y = static_cast<T *>(p.y) + (int64_t)h * p.dv;

    f32x4 state[2][TD];
    const int64_t head = ((int64_t)s * p.heads + h) * p.dk;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int n = 0; n < TD; ++n) {
            const int d = d0 + 16 * n + l15;
            state[x][n] = f32x4{};
            if (p.s0 && d < p.dk) {
                float t[4];
                unpack(fetch4(p.s0 + (head + d) * p.dv, col + 16 * x, p.dv), t);
#pragma unroll
                for (int e = 0; e < 4; ++e) state[x][n][e] = t[e];
            }
            put4(S, d, v0 + 16 * x + lq * 4, state[x][n]);
        }

    // what the next chunk brings
    Rows<T, C, DK> kn, qn;
    Pack<T, 4> vn[2][TT];
    constexpr int pieces = PC * C * C / 8, MP = (pieces + kGdrThreads - 1) / kGdrThreads;
    uint4 mn[MP];
    double Gn = 0.;
    float bn = 0.f;
    const auto fetch = [&](int64_t n, int64_t first) {
        const int rows = (int)min((int64_t)C, span.end - first);
        kn.fetch(k + first * p.ldk, p.ldk, rows, p.dk);
        qn.fetch(q + first * p.ldq, p.ldq, rows, p.dk);
        const Saved<T> saved(p, place + n, h);
#pragma unroll
        for (int i = 0; i < MP; ++i) {
            const int piece = i * kGdrThreads + (int)threadIdx.x;
            if (piece < pieces) mn[i] = reinterpret_cast<const uint4 *>(saved.M())[piece];
        }
        if (threadIdx.x < C) {
            Gn = saved.G()[threadIdx.x];
            bn = (int)threadIdx.x < rows ? p.beta[(first + threadIdx.x) * p.ldg + h] : 0.f;
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const int token = t0 + 16 * t + l15;
                if (token < rows) vn[x][t] = fetch4(v + (first + token) * p.ldv, col + 16 * x, p.dv);
                else
#pragma unroll
                    for (int i = 0; i < vn[x][t].W; ++i) vn[x][t].w[i] = 0;
            }
    };
    if (span.first < span.end) fetch(0, span.first);
    for (int64_t n = 0, first = span.first; first < span.end; ++n, first += C) {
        const int rows = (int)min((int64_t)C, span.end - first);
        kn.place(K, rk, p.norm_eps, 1.f);
        qn.place(Q, rq, p.norm_eps, p.scale);
#pragma unroll
        for (int i = 0; i < MP; ++i) {
            const int piece = i * kGdrThreads + (int)threadIdx.x, e = piece % (C * C / 8) * 8;
            if (piece < pieces) *reinterpret_cast<uint4 *>(M.at + piece / (C * C / 8) * M.part + e / C * M.ld + e % C) = mn[i];
        }
        if (threadIdx.x < C) G[threadIdx.x] = Gn, beta[threadIdx.x] = bn;
        f32x4 value[2][TT];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                float u[4];
                unpack(vn[x][t], u);
#pragma unroll
                for (int e = 0; e < 4; ++e) value[x][t][e] = u[e];
            }
        if (first + C < span.end) fetch(n + 1, first + C);
        if (p.states) {
            float *to = p.states + (((place + n) * p.heads + h) * p.blocks + block) * (DK * kGdrColumns);
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int m = 0; m < TD; ++m) *reinterpret_cast<f32x4 *>(to + (d0 + 16 * m + l15) * kGdrColumns + v0 + 16 * x + lq * 4) = state[x][m];
        }
        __syncthreads();
        f32x4 ks[2][TT] = {}, out[2][TT] = {}, pr[TT][TT] = {};
#pragma unroll
        for (int d = 0; d < DK; d += 32) {
            Frag<PC> a[2];
            Frag<PD> bk[TT], bq[TT], aj[TT];
#pragma unroll
            for (int x = 0; x < 2; ++x) a[x] = across(S, v0 + 16 * x, d);
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                bk[t] = along(K, t0 + 16 * t, d), bq[t] = along(Q, t0 + 16 * t, d);
                if (j0 <= t0) aj[t] = along(K, j0 + 16 * t, d);
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int t = 0; t < TT; ++t) ks[x][t] = multiply(a[x], bk[t], ks[x][t]), out[x][t] = multiply(a[x], bq[t], out[x][t]);
            if (j0 <= t0)
#pragma unroll
                for (int x = 0; x < TT; ++x)
#pragma unroll
                    for (int t = 0; t < TT; ++t) pr[x][t] = multiply(aj[x], bq[t], pr[x][t]);
        }
        float bt[TT], until[TT];
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const int i = t0 + 16 * t + l15;
            const float since = expf((float)G[i]);
            bt[t] = beta[i];
            until[t] = expf((float)(G[C - 1] - G[i])) * rk[i];
            const float fk = since * rk[i], fq = since * rq[i];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int e = 0; e < 4; ++e) value[x][t][e] -= fk * ks[x][t][e], out[x][t][e] *= fq;
                put4(X, i, v0 + 16 * x + lq * 4, value[x][t] * bt[t]);
            }
        }
        __syncthreads();
        f32x4 less[2][TT] = {};
#pragma unroll
        for (int j = 0; j < C; j += 32) {
            if (j >= t0 + C / 2) continue;                  // M is lower
            Frag<PC> a[2], m[TT];
#pragma unroll
            for (int x = 0; x < 2; ++x) a[x] = across(X, v0 + 16 * x, j);
#pragma unroll
            for (int t = 0; t < TT; ++t) m[t] = along(M, t0 + 16 * t, j);
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int t = 0; t < TT; ++t) less[x][t] = multiply(a[x], m[t], less[x][t]);
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const int i = t0 + 16 * t + l15;
                const f32x4 u = (value[x][t] - less[x][t]) * bt[t];
                put4(X, i, v0 + 16 * x + lq * 4, u);
                put4(U, i, v0 + 16 * x + lq * 4, u * until[t]);
            }
        if (j0 <= t0)
#pragma unroll
            for (int x = 0; x < TT; ++x)
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    const int j = j0 + 16 * x + lq * 4, i = t0 + 16 * t + l15;
                    f32x4 w = {};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i >= j + e) w[e] = expf((float)(G[i] - G[j + e])) * rq[i] * rk[j + e] * pr[x][t][e];
                    put4(M, i, j, w);
                }
        const float whole = expf((float)G[C - 1]);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < C; j += 32) {
            if (j >= t0 + C / 2) continue;
            Frag<PC> a[2], m[TT];
#pragma unroll
            for (int x = 0; x < 2; ++x) a[x] = across(X, v0 + 16 * x, j);
#pragma unroll
            for (int t = 0; t < TT; ++t) m[t] = along(M, t0 + 16 * t, j);
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int t = 0; t < TT; ++t) out[x][t] = multiply(a[x], m[t], out[x][t]);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int m = 0; m < TD; ++m) state[x][m] *= whole;
#pragma unroll
        for (int j = 0; j < C; j += 32) {
            Frag<PC> a[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) a[x] = across(U, v0 + 16 * x, j);
#pragma unroll
            for (int m = 0; m < TD; ++m) {
                const Frag<PD> f = across(K, d0 + 16 * m, j);
#pragma unroll
                for (int x = 0; x < 2; ++x) state[x][m] = multiply(a[x], f, state[x][m]);
            }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const int i = t0 + 16 * t + l15;
                if (i < rows) store4(y + (first + i) * p.ldy, col + 16 * x, p.dv, out[x][t]);
            }
#pragma unroll
            for (int m = 0; m < TD; ++m) put4(S, d0 + 16 * m + l15, v0 + 16 * x + lq * 4, state[x][m]);
        }
        __syncthreads();
    }
    if (!p.s_last) return;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int n = 0; n < TD; ++n) {
            const int d = d0 + 16 * n + l15;
            if (d < p.dk) store4(p.s_last + (head + d) * p.dv, col + 16 * x, p.dv, state[x][n]);
        }
}

// ---------------------------------------------------------------------------------------------------- launches
template <typename T>
int64_t places_of(int64_t N, int32_t nseq) { return N / Gdr<T>::chunk + nseq; }

inline int padded(int dk) { return dk <= 64 ? 64 : 128; }
inline int blocks_of(int dv) { return (dv + kGdrColumns - 1) / kGdrColumns; }

// Bytes of what is kept of the chunks: their matrices, and the states in front of them.
template <typename T>
int64_t saved_bytes(int64_t N, int32_t nseq, int32_t heads) { return (places_of<T>(N, nseq) * heads * Saved<T>::bytes + 15) / 16 * 16; }
template <typename T>
int64_t states_bytes(int64_t N, int32_t nseq, int32_t heads, int32_t dk, int32_t dv) {
    return places_of<T>(N, nseq) * heads * blocks_of(dv) * padded(dk) * kGdrColumns * 4;
}

inline bool gdr_shape(int64_t N, int32_t nseq, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv) {
    return N >= 0 && N <= (int64_t)1 << 30 && nseq >= 1 && heads >= 1 && heads <= kMostHeads && key_heads >= 1 && heads % key_heads == 0 && dk >= 1 && dv >= 1;
}

template <typename T, int DK>
grim_status gdr_launch(const GdrParams &p, hipStream_t stream) {
    const int64_t places = places_of<T>(p.N, p.nseq);
    if (p.N > 0) {
        const int64_t each = most_groups(kGdrThreads) / p.heads;
        if (places > each) return GRIM_ERR_UNSUPPORTED;
        hipLaunchKernelGGL((chunk_matrices<T, DK>), dim3((unsigned)(places * p.heads)), dim3(kGdrThreads), 0, stream, p);
        const grim_status st = launched();
        if (st != GRIM_OK) return st;
    }
    constexpr int bytes = WalkRoom<T, DK>::bytes;
    static const hipError_t grown = hipFuncSetAttribute(reinterpret_cast<const void *>(&walk<T, DK>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (grown != hipSuccess) return GRIM_ERR_DEVICE;
    hipLaunchKernelGGL((walk<T, DK>), dim3((unsigned)((int64_t)p.nseq * p.heads * p.blocks)), dim3(kGdrThreads), bytes, stream, p);
    return launched();
}

template <typename T>
grim_status gdr_typed(GdrParams p, void *states, void *workspace, hipStream_t stream) {
    p.saved = static_cast<char *>(states ? states : workspace);
    if (states) p.states = reinterpret_cast<float *>(p.saved + saved_bytes<T>(p.N, p.nseq, p.heads));
    return p.dk <= 64 ? gdr_launch<T, 64>(p, stream) : gdr_launch<T, 128>(p, stream);
}

}  // namespace lm
}  // namespace grim

extern "C" {

int64_t grim_gdr_states(int64_t N, int32_t nseq, int32_t heads, int32_t dk, int32_t dv) {
    using namespace grim::lm;
    if (!gdr_shape(N, nseq, heads, 1, dk, dv) || dk > kMostHeadSize || dv > kMostHeadSize) return 0;
    const int64_t a = saved_bytes<float>(N, nseq, heads) + states_bytes<float>(N, nseq, heads, dk, dv);
    const int64_t b = saved_bytes<f16>(N, nseq, heads) + states_bytes<f16>(N, nseq, heads, dk, dv);
    return a > b ? a : b;
}

int64_t grim_gdr_workspace(int64_t N, int32_t nseq, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv) {
    using namespace grim::lm;
    if (!gdr_shape(N, nseq, heads, key_heads, dk, dv) || dk > kMostHeadSize || dv > kMostHeadSize) return 0;
    const int64_t a = saved_bytes<float>(N, nseq, heads), b = saved_bytes<f16>(N, nseq, heads);
    return a > b ? a : b;
}

grim_status grim_gdr_sequence(const void *q_dev, const void *k_dev, const void *v_dev, grim_dtype dt, int64_t ldq, int64_t ldk, int64_t ldv,
                              const float *decay_dev, const float *beta_dev, int64_t ldg, const float *s0_dev, const int32_t *seq_start_dev,
                              int32_t nseq, int64_t N, int32_t heads, int32_t key_heads, int32_t dk, int32_t dv, float scale, float norm_eps,
                              void *y_dev, int64_t ldy, float *s_last_dev, void *states_dev, void *workspace, int64_t workspace_bytes,
                              void *hip_stream) {
    using namespace grim::lm;
    if (!known(dt)) return GRIM_ERR_DTYPE;
    if (!gdr_shape(N, nseq, heads, key_heads, dk, dv) || (nseq > 1 && !seq_start_dev) || !(fabsf(scale) < INFINITY) || !(norm_eps >= 0.f) || norm_eps > 3.4e38f)
        return GRIM_ERR_SHAPE;
    if (dk > kMostHeadSize || dv > kMostHeadSize) return GRIM_ERR_UNSUPPORTED;
    const int64_t keys = (int64_t)key_heads * dk, values = (int64_t)heads * dv;
    if (ldq < keys || ldk < keys || ldv < values || ldy < values || ldg < heads || !fits(N, ldq) || !fits(N, ldk) || !fits(N, ldv) || !fits(N, ldy) ||
        !fits(N, ldg))
        return GRIM_ERR_SHAPE;
    if ((int64_t)nseq * heads > (int64_t)1 << 23) return GRIM_ERR_UNSUPPORTED;
    if (N > 0 && (!q_dev || !k_dev || !v_dev || !decay_dev || !beta_dev || !y_dev || !workspace)) return GRIM_ERR_NULL;
    if (workspace_bytes < grim_gdr_workspace(N, nseq, heads, key_heads, dk, dv) && N > 0) return GRIM_ERR_SHAPE;
    if (N == 0 && !s_last_dev) return GRIM_OK;
    if (s_last_dev && s0_dev && overlap(s0_dev, s_last_dev, (int64_t)nseq * heads * dk * dv * 4)) return GRIM_ERR_UNSUPPORTED;
    const GdrParams p{q_dev, k_dev, v_dev, decay_dev, beta_dev, s0_dev, seq_start_dev, y_dev, s_last_dev, nullptr, nullptr, ldq, ldk, ldv, ldg, ldy, N, nseq,
                      heads, heads / key_heads, dk, dv, blocks_of(dv), scale, norm_eps};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dt == GRIM_F32   ? gdr_typed<float>(p, states_dev, workspace, stream)
           : dt == GRIM_F16 ? gdr_typed<f16>(p, states_dev, workspace, stream)
                            : gdr_typed<bf16>(p, states_dev, workspace, stream);
}

}  // extern "C"
