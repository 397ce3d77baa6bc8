// The gated delta rule over packed sequences, backward: the gradients that mix columns of the states.
//
// In the notation of lm_gdr.hip and lm_gdr_back.hip, for every chunk by itself, with keys and queries as they count (r the factor of the raw ones):
//     dQ   = exp(G) dy S' + dP K          dP_ij =   w_ij dy_i . U_j (i >= j)
//     dK_r = -exp(G) Y S' + dL K          dL_ij = - w_ij  Y_i . U_j (i > j)
//     dK_c = dP' Q + dL' K,    dK_e = exp(G_end - G) U A'           dK = dK_r + dK_c + dK_e
//     dg_i = exp(G_end) <S, A> + sum over j >= i of (dQ . Q + dK_r . K - dK_c . K)_j + sum over j < i of (dK_e . K)_j        dbeta = F . E
// and back through the division by the lengths.  A workgroup takes a chunk and a key head and goes through the heads that read it, so that
// their sums need no atomics; a wave has 16 rows of the states (16 elements of keys and queries), whose states come from memory straight into its operands.
// A chunk of a 128 x 128 head in bf16 is 270 KB, which a compute unit that has one workgroup fetches in 10 of its 24 us (2.3 us for 32 columns, the next ones on their way); the products of dP and
// dL with keys and queries, bound by LDS, and the sums over elements take the rest: 4096 of them 430 us.  Two workgroups would fetch through each other's ends, but the sums that a wave keeps do not
// fit half the registers (with spills 550 us).  64 x 64 heads, 6000 chunks, two workgroups: 226 us.
#include "lm_gdr.hpp"

namespace grim {
namespace lm {

// What a workgroup keeps in LDS: columns of the values VB at a time; dP and dL, in parts and with all factors, come where U, Y and dy were.
template <typename T, int DK>
struct GradRoom {
    static constexpr int C = Gdr<T>::chunk, PD = Gdr<T>::data, PC = Gdr<T>::comp, VB = 32, W = DK / 16;
    using Keys = Tile<PD, C, DK, TURNED>;
    using Values_ = Tile<PD, C, VB, PAIRED>;
    using Cols = Tile<PC, VB, C, TURNED>;                   // U and Y, a column's tokens in a row
    using Square = Triangle<PC, C, TURNED>;
    static constexpr int keys = 0, queries = keys + Keys::bytes, dy = queries + Keys::bytes, U = dy + Values_::bytes, Y = U + Cols::bytes, end1 = Y + Cols::bytes;
    static constexpr int P = dy, L = P + Square::bytes, end2 = L + Square::bytes, G = end1 > end2 ? end1 : end2, tokens = G + C * 8, sums = tokens + C * 24,
                         betas = sums + 2 * W * C * 4, bytes = betas + W * 16 * 4;
    static_assert(bytes <= 160 * 1024, "LDS");
};

template <typename T, int DK>
struct GradTiles {
    using Room = GradRoom<T, DK>;
    typename Room::Keys K, Q;
    typename Room::Values_ dY;
    typename Room::Cols U, Y;
    typename Room::Square dP, dL;
    double *G;
    float *tokens, *sums, *betas;
    const float *beta, *fk, *fu, *fq, *rk, *rq;
    // (The compiler is kept from seeing that the addresses are the same every time: it holds dozens of them in registers across the loops otherwise, and spills.)
    __device__ __forceinline__ GradTiles(char *lds) {
        int again = 0;
        asm volatile("" : "+s"(again));
        const auto tile = [&](int at) { return reinterpret_cast<uint16_t *>(lds + again + at); };
        K.at = tile(Room::keys), Q.at = tile(Room::queries), dY.at = tile(Room::dy), U.at = tile(Room::U), Y.at = tile(Room::Y), dP.put(lds + again + Room::P), dL.put(lds + again + Room::L);
        const auto floats = [&](int at) { return reinterpret_cast<float *>(lds + again + at); };
        G = reinterpret_cast<double *>(lds + again + Room::G), tokens = floats(Room::tokens), sums = floats(Room::sums), betas = floats(Room::betas);
        constexpr int C = Room::C;
        beta = tokens, fk = tokens + C, fu = tokens + 2 * C, fq = tokens + 3 * C, rk = tokens + 4 * C, rq = tokens + 5 * C;
    }
};

// Rows r + lane % 16, elements c + (lane / 16) 4 .. + 3, the parts added up again (exact for 16-bit elements, to 2^-25 in fp32).
template <int P, int R, int C, int ORDER>
__device__ __forceinline__ f32x4 elements(const Tile<P, R, C, ORDER> &m, int r, int c) {
    static_assert(ORDER != PAIRED, "columns in their own order");
    const int lane = threadIdx.x & 63;
    f32x4 v = {};
#pragma unroll
    for (int p = P - 1; p >= 0; --p) {
        const s16x4 w = *reinterpret_cast<const s16x4 *>(m.at + p * m.part + (r + (lane & 15)) * m.ld + c + (lane >> 4) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += __builtin_bit_cast(float, (uint32_t)(uint16_t)w[e] << 16);
    }
    return v;
}

template <typename T, int DK, bool WHOLE>
__global__ void __launch_bounds__(DK * 4, 2) gradients(GdrBack b) {
    using Room = GradRoom<T, DK>;
    constexpr int C = Room::C, PD = Room::PD, PC = Room::PC, VB = Room::VB, W = Room::W, THREADS = 64 * W, TT = C / 16, SS = C / 32, DT = DK / 16, VT = VB / 16;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const GdrParams &p = b.p;

    const int kh = (int)(blockIdx.x % (uint32_t)b.key_heads), head0 = kh * p.group, head1 = head0 + p.group;
    const uint32_t place = blockIdx.x / (uint32_t)b.key_heads;
    const int s = sequence_of(p.seq_start, p.nseq, p.N, C, place);
    const Span span(p.seq_start, s, p.N);
    const int64_t first = span.first + (int64_t)(place - place_of(span, s, C)) * C;
    if (first >= span.end) return;
    const int rows = (int)min((int64_t)C, span.end - first);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15, g4 = (lane >> 4) * 4, d0 = 16 * wave;
    const uint32_t own = l15 * 16 + g4, turned_own = g4 * 16 + l15;

    // what the next VB columns bring (operands of the states: row d0 + l15, columns g4 .. + 3 of a tile), and the next head
    constexpr int EACH = (VT * TT + W - 1) / W, TP = (6 * C + THREADS - 1) / THREADS;
    static_assert(W % TT == 0, "a wave has the same tokens of all its tiles of U");
    const int own_t = wave % TT;
    f32x4 S[VT], A[VT], e[EACH], f[EACH], bt;
    Rows<WHOLE, T, THREADS, C, VB> y;
    float tn[TP];
    double Gn;
    float gn;
    const auto fetch = [&](int h, int v0) {
        const int64_t chunk = (int64_t)place * p.heads + h;
        const int tile0 = v0 / 16, there = p.tiles - tile0;
#pragma unroll
        for (int v = 0; v < VT; ++v) {
            const int64_t at = ((chunk * p.tiles + tile0 + min(v, there - 1)) * DT + wave) * 256;
            const float *from_s = p.states + at, *from_a = b.A + at;
#pragma unroll
            for (int i = 0; i < 4; ++i) S[v][i] = from_s[turned_own + 16 * i], A[v][i] = from_a[turned_own + 16 * i];
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int64_t at = ((chunk * p.tiles + tile0 + min((i * W + wave) / TT, min(VT, there) - 1)) * TT + own_t) * 256;
            const float *from_e = p.E + at, *from_f = b.F + at;
            e[i] = *reinterpret_cast<const f32x4 *>(from_e + own), f[i] = *reinterpret_cast<const f32x4 *>(from_f + own);
        }
        y.fetch(static_cast<const T *>(b.dy) + first * b.lddy + (int64_t)h * p.dv + v0, b.lddy, rows, p.dv - v0);
        const Saved<T> saved(p, place, h);                  // (for all columns, which keeps the loads in one line)
#pragma unroll
        for (int i = 0; i < TP; ++i) tn[i] = saved.tokens()[min(i * THREADS + (int)threadIdx.x, 6 * C - 1)];
        Gn = saved.G()[threadIdx.x % C];
        gn = p.decay[(first + min(lane, rows - 1)) * p.ldg + h];
        bt = *reinterpret_cast<const f32x4 *>(saved.tokens() + 16 * own_t + g4);
    };
    {
        Rows<WHOLE, T, THREADS, C, DK> k, q;
        k.fetch(static_cast<const T *>(p.k) + first * p.ldk + (int64_t)kh * p.dk, p.ldk, rows, p.dk);
        q.fetch(static_cast<const T *>(p.q) + first * p.ldq + (int64_t)kh * p.dk, p.ldq, rows, p.dk);
        fetch(head0, 0);
        const GradTiles<T, DK> m(lds);
        k.place(m.K, rows, p.dk);
        q.place(m.Q, rows, p.dk);
    }
    f32x4 dq[TT] = {}, dk[TT] = {};                         // elements d0 + g4 .. + 3 of token 16 t + l15, sums over the heads
    constexpr int PP = (Lower<C>::count + W - 1) / W;       // of 16 x 16 of dP and dL
    const auto pair = [&](int i, int &t, int &j) {
        Lower<C>::get(i * W + wave, t, j);
        return i * W + wave < Lower<C>::count;
    };
    f32x4 q[TT] = {}, kr[TT] = {}, ke[TT] = {}, gp[PP] = {}, gl[PP] = {}, db = {};
    float sa = 0.f, g = 0.f;
    for (int h = head0, v0 = 0; h < head1;) {
        const bool done = v0 + VB >= p.dv;                  // with the head
        {
            const int there = min(VT, p.tiles - v0 / 16);
            g = gn;
            const GradTiles<T, DK> m(lds);
            __syncthreads();                                // (the columns and the head before are done with)
#pragma unroll
            for (int i = 0; i < TP; ++i)
                if (i * THREADS + (int)threadIdx.x < 6 * C) m.tokens[i * THREADS + threadIdx.x] = tn[i];
            if (threadIdx.x < C) m.G[threadIdx.x] = Gn;
            y.place(m.dY, rows, p.dv - v0);
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int v = (i * W + wave) / TT;
                if (v >= VT) continue;
                const float in = v < there ? 1.f : 0.f;     // (what is read twice is finite or hurts the head anyway)
                db += e[i] * f[i] * in;
                put4(m.U, 16 * v + l15, 16 * own_t + g4, e[i] * (bt * in));
                put4(m.Y, 16 * v + l15, 16 * own_t + g4, f[i] * (bt * in));
            }
            if (there < VT) S[1] = A[1] = f32x4{};
#pragma unroll
            for (int v = 0; v < VT; ++v) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sa = __builtin_fmaf(S[v][i], A[v][i], sa);
            }
            const Frag<PC> fs = operand<PC>(S[0], S[1]), fa = operand<PC>(A[0], A[1]);
            __builtin_amdgcn_sched_barrier(0);
            if (!done || h + 1 < head1) fetch(done ? h + 1 : h, done ? 0 : v0 + VB);
            __syncthreads();
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                __builtin_amdgcn_sched_barrier(0);
                q[t] = multiply(fs, along(m.dY, 16 * t, 0), q[t]);
                kr[t] = multiply(fs, across(m.Y, 16 * t, 0), kr[t]);
                ke[t] = multiply(fa, across(m.U, 16 * t, 0), ke[t]);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < PP; ++i) {
                int t, j;
                if (!pair(i, t, j)) continue;
                const Frag<PC> u = across(m.U, 16 * j, 0);
                gp[i] = multiply(u, along(m.dY, 16 * t, 0), gp[i]);
                gl[i] = multiply(u, across(m.Y, 16 * t, 0), gl[i]);
            }
        }
        v0 += VB;
        if (!done) continue;
        const GradTiles<T, DK> m(lds);
        int l15 = threadIdx.x & 15, g4 = (threadIdx.x & 63) / 16 * 4;
        asm volatile("" : "+v"(l15), "+v"(g4));             // (for the same reason: comparisons too would be kept)
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PP; ++i) {
            int t, j;
            if (!pair(i, t, j)) continue;
            t = 16 * t + l15, j = 16 * j + g4;
            const double Gt = m.G[t];
            const float kt = m.rk[t], qt = m.rq[t];
            f32x4 a, c;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float w = t >= j + e ? decay_of(Gt - m.G[j + e]) * m.rk[j + e] : 0.f;
                a[e] = t >= j + e ? w * qt * gp[i][e] : 0.f, c[e] = t > j + e ? -w * kt * gl[i][e] : 0.f;
            }
            put4(m.dP, t, j, a);
            put4(m.dL, t, j, c);
        }
        __syncthreads();
        f32x4 kc[TT] = {};
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            q[t] *= m.fq[16 * t + l15], kr[t] *= -m.fk[16 * t + l15], ke[t] *= m.fu[16 * t + l15];
        }
#pragma unroll
        for (int x = 0; x < SS; ++x) {
            __builtin_amdgcn_sched_barrier(0);
            const Frag<PD> fk_ = across(m.K, d0, 32 * x), fq_ = across(m.Q, d0, 32 * x);
#pragma unroll
            for (int t = 2 * x; t < TT; ++t) {              // (sums over j, 32 of them from 32 x, for the tokens from there on)
                q[t] = multiply(fk_, along(m.dP, 16 * t, 32 * x), q[t]);
                kr[t] = multiply(fk_, along(m.dL, 16 * t, 32 * x), kr[t]);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 2 * x + 2; ++j) {           // (sums over t)
                __builtin_amdgcn_sched_barrier(0);
                kc[j] = multiply(fq_, across(m.dP, 16 * j, 32 * x), kc[j]);
                kc[j] = multiply(fk_, across(m.dL, 16 * j, 32 * x), kc[j]);
            }
        }
        // what the decays get of it; the last token also exp(G_end) <S, A>, which all get
        const float all = wave_sum(sa) * decay_of(m.G[C - 1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const f32x4 kv = elements(m.K, 16 * t, d0), qv = elements(m.Q, 16 * t, d0);
            const f32x4 here = q[t] * qv + (kr[t] - kc[t]) * kv, n = ke[t] * kv;
            float from_here = across_rows(here[0] + here[1] + (here[2] + here[3]), Add());
            const float before = across_rows(n[0] + n[1] + (n[2] + n[3]), Add());
            if (16 * t + l15 == C - 1) from_here += all;
            if (lane < 16) m.sums[wave * C + 16 * t + l15] = from_here, m.sums[(W + wave) * C + 16 * t + l15] = before;
            dq[t] += q[t];
            dk[t] += kr[t] + kc[t] + ke[t];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float one = row_join(db[e], Add());
            if (l15 == 0) m.betas[wave * 16 + g4 + e] = one;
        }
        __syncthreads();
        if (wave == 0) {
            float a = 0.f, before = 0.f, d = 0.f;
            const int at = lane % C;
#pragma unroll
            for (int w = 0; w < W; ++w) a += m.sums[w * C + at], before += m.sums[(W + w) * C + at];
#pragma unroll
            for (int w = 0; w < W / TT; ++w) d += m.betas[(w * TT + at / 16) * 16 + at % 16];
#pragma unroll
            for (int x = 1; x < C; x *= 2) {
                const float after = __shfl_down(a, x, C), less = __shfl_up(before, x, C);
                if (at + x < C) a += after;
                if (at >= x) before += less;
            }
            before = __shfl_up(before, 1, C);
            if (at == 0) before = 0.f;
            if (lane < rows) {
                const int64_t t = first + lane;
                b.ddecay[t * b.lddg + h] = g < kLeastDecay ? 0.f : a + before;
                b.dbeta[t * b.lddg + h] = d;
            }
        }
#pragma unroll
        for (int t = 0; t < TT; ++t) q[t] = kr[t] = ke[t] = f32x4{};
#pragma unroll
        for (int i = 0; i < PP; ++i) gp[i] = gl[i] = f32x4{};
        db = f32x4{}, sa = 0.f, v0 = 0, ++h;
    }
    // through the division by the lengths: d(x / |x|) = (dx - x (x . dx) / |x|^2) / |x|, of which the last division is made already
    const GradTiles<T, DK> m(lds);
    if (p.norm_eps > 0.f) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const f32x4 l = dq[t] * elements(m.Q, 16 * t, d0), n = dk[t] * elements(m.K, 16 * t, d0);
            const float mq = across_rows(l[0] + l[1] + (l[2] + l[3]), Add()), mk = across_rows(n[0] + n[1] + (n[2] + n[3]), Add());
            if (lane < 16) m.sums[wave * C + 16 * t + l15] = mq, m.sums[(W + wave) * C + 16 * t + l15] = mk;
        }
        __syncthreads();
        const float unscale = p.scale != 0.f ? 1.f / p.scale : 0.f;
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const int i = 16 * t + l15;
            float mq = 0.f, mk = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) mq += m.sums[w * C + i], mk += m.sums[(W + w) * C + i];
            const float iq = m.rq[i] * unscale, ik = m.rk[i];
            dq[t] -= elements(m.Q, 16 * t, d0) * iq * (iq * mq);
            dk[t] -= elements(m.K, 16 * t, d0) * ik * (ik * mk);
        }
    }
    T *q_to = static_cast<T *>(b.dq) + first * b.lddq + (int64_t)kh * p.dk, *k_to = static_cast<T *>(b.dk) + first * b.lddk + (int64_t)kh * p.dk;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const int i = 16 * t + l15;
        if (i >= rows) continue;
        leave<WHOLE>(q_to + i * b.lddq, d0 + g4, p.dk, dq[t]);
        leave<WHOLE>(k_to + i * b.lddk, d0 + g4, p.dk, dk[t]);
    }
}

template <typename T, int DK, bool WHOLE>
grim_status gdr_gradients(const GdrBack &b, hipStream_t stream) {
    constexpr int bytes = GradRoom<T, DK>::bytes;
    const auto kernel = gradients<T, DK, WHOLE>;
    static std::atomic<bool> grown{false};
    if (!lds_of(reinterpret_cast<const void *>(kernel), bytes, grown)) return GRIM_ERR_DEVICE;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(places_of<T>(b.p.N, b.p.nseq) * b.key_heads)), dim3(DK * 4), bytes, stream, b);
    return launched();
}

#define GRADIENTS(T)                                                                    \
    template grim_status gdr_gradients<T, 64, false>(const GdrBack &, hipStream_t);     \
    template grim_status gdr_gradients<T, 64, true>(const GdrBack &, hipStream_t);      \
    template grim_status gdr_gradients<T, 128, false>(const GdrBack &, hipStream_t);    \
    template grim_status gdr_gradients<T, 128, true>(const GdrBack &, hipStream_t);
GRADIENTS(float)
GRADIENTS(f16)
GRADIENTS(bf16)

}  // namespace lm
}  // namespace grim
