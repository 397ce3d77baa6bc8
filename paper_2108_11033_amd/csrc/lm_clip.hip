// The norm of all gradients of a model, and their clipping by it.
//
//     norm = |unscale| sqrt(sum over all tensors of g^2)        out = g unscale min(1, max_norm / norm)
//
// Bound by memory: the gradients are read once for the norm and once more to be scaled, the outputs written once.  (Models of up to some 100 MB of gradients would fit the compute units'
// registers in between, in one launch whose workgroups wait for each other: not built.)  Squares are summed in fp64, where those of any fp32 number neither overflow nor vanish; of fp16, whose squares are exact in fp32, eight at a
// time in fp32 first.  A workgroup takes runs of a tensor (below) in turn and leaves one sum; the scaling workgroups join these sums themselves, each in the same
// order, so that no launch stands between, and walk the runs from the last one back: what was read last is still in the last-level cache.
// Tensors travel as launch arguments: no table on the device has to be written before, and a captured call keeps its own.
// 168 M bf16 gradients to fp32: 240 us (1.3 GB from and to memory at 5.6 TB/s); 18 M of fp16 in odd tensors: 25 us; a few small tensors: 8.9 us, two launches.
#include <algorithm>
#include <new>
#include <vector>

#include "lm_common.hpp"

struct grim_grad_list {
    std::vector<grim_grad> tensors;         // none of them empty
    std::vector<int64_t> last_run;          // of every tensor, in its launch's numbers: one past its last run
    int64_t workgroups = 0;                 // over all launches
};

namespace grim {
namespace lm {

constexpr int kRun = 8192;                  // elements of a run: 256 threads, 32 each
constexpr int kTable = 100;                 // tensors of a launch: their table is 3.2 KB of arguments
constexpr int kMostGroups = 1024;           // workgroups of a launch (1536 and 2048, and runs of 4096: the same times within 2 %)

struct TensorArgs {
    const void *grad;
    void *out;
    int64_t count;
    uint32_t last_run;
    uint16_t dt, out_dt;
};

struct ClipParams {
    double *sums;                           // one of every workgroup of every launch of the norm
    float *norm;
    int64_t groups;                         // of all launches
    double unscale, max_norm;
    uint32_t runs, first_group;
    int32_t tensors;
    TensorArgs t[kTable];
};
static_assert(sizeof(ClipParams) <= 4096, "launch arguments");

// The tensor that run r belongs to.
__device__ __forceinline__ int tensor_of(const ClipParams &p, uint32_t r) {
    int lo = 0, hi = p.tensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (r < p.t[mid].last_run) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// f(type) for an element type
template <typename F>
__device__ __forceinline__ void with_type(int dt, F f) {
    if (dt == GRIM_F32) f(float());
    else if (dt == GRIM_F16) f(f16());
    else f(bf16());
}

template <typename T>
__device__ __forceinline__ double squares(const T *g, int64_t left) {
    constexpr int V = 8, PER = kRun / 256 / V;
    double sum = 0.;
    auto add = [&](const float (&v)[V]) {
        if constexpr (__is_same(T, f16)) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) s = __builtin_fmaf(v[j], v[j], s);
            sum += (double)s;
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) sum = __builtin_fma((double)v[j], (double)v[j], sum);
        }
    };
    if (left >= kRun) {
        Pack<T, V> raw[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) raw[k] = load<V>(g + (k * 256 + threadIdx.x) * V);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            float v[V];
            unpack(raw[k], v);
            add(v);
        }
    } else {
        for (int64_t c = threadIdx.x * V; c < left; c += 256 * V) {
            float v[V];
            if (c + V <= left) unpack(load<V>(g + c), v);
            else
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = c + j < left ? (float)g[c + j] : 0.f;
            add(v);
        }
    }
    return sum;
}

// The sum over a workgroup of 256 threads, in a fixed order; all threads get it.
__device__ __forceinline__ double join(double v, double *room) {
    room[threadIdx.x] = v;
    __syncthreads();
#pragma unroll
    for (int n = 128; n >= 1; n /= 2) {
        if ((int)threadIdx.x < n) room[threadIdx.x] += room[threadIdx.x + n];
        __syncthreads();
    }
    return room[0];
}

__global__ void __launch_bounds__(256) sum_squares(const ClipParams p) {
    __shared__ double room[256];
    double sum = 0.;
    for (uint32_t r = blockIdx.x; r < p.runs; r += gridDim.x) {
        const int i = tensor_of(p, r);
        const uint32_t first = i ? p.t[i - 1].last_run : 0;
        const int64_t at = (int64_t)(r - first) * kRun;
        with_type(p.t[i].dt, [&](auto type) {
            using T = decltype(type);
            sum += squares(static_cast<const T *>(p.t[i].grad) + at, p.t[i].count - at);
        });
    }
    sum = join(sum, room);
    if (threadIdx.x == 0) p.sums[p.first_group + blockIdx.x] = sum;
}

// A factor as the product of two numbers, so that one that fp32 does not hold (1e-3 of a norm of 1e38) keeps its digits: below 2^-100 each takes half of its exponent, above the second is 1.
// (What the first product loses then, at its end, is nothing after the second.)
struct Factor {
    float first, second;
    __device__ __forceinline__ explicit Factor(double f) {
        const int half = f != 0. && fabs(f) < 0x1p-100 ? ilogb(f) / 2 : 0;
        first = (float)ldexp(f, -half), second = ldexpf(1.f, half);
    }
    __device__ __forceinline__ float times(float v) const { return v * first * second; }
};

// out = g * factor for a run; a thread reads what it writes, so that out may be g.
template <typename T, typename O, bool PAST>
__device__ __forceinline__ void scale_run(const T *g, O *out, int64_t left, Factor factor) {
    // 16 bytes of the wider type, so that an access of a wave is one piece of memory (two halves of 32 bytes a lane instead, bf16 into fp32, 168 M: 265 us)
    constexpr int V = 16 / (int)(sizeof(T) > sizeof(O) ? sizeof(T) : sizeof(O)), PER = kRun / 256 / V;
    if (left >= kRun) {
        Pack<T, V> raw[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) raw[k] = load<V>(g + (k * 256 + threadIdx.x) * V);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            float v[V];
            unpack(raw[k], v);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = factor.times(v[j]);
            store<PAST>(out + (k * 256 + threadIdx.x) * V, v);
        }
    } else {
        for (int64_t c = threadIdx.x * V; c < left; c += 256 * V) {
            float v[V];
            if (c + V <= left) {
                unpack(load<V>(g + c), v);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = factor.times(v[j]);
                store(out + c, v);
            } else {
                for (int j = 0; c + j < left; ++j) out[c + j] = (O)factor.times((float)g[c + j]);
            }
        }
    }
}

__device__ __forceinline__ double norm_of(const ClipParams &p, double *room) {
    double sum = 0.;
    for (int64_t i = threadIdx.x; i < p.groups; i += 256) sum += p.sums[i];
    return fabs(p.unscale) * sqrt(join(sum, room));
}

__global__ void __launch_bounds__(256) write_norm(const ClipParams p) {
    __shared__ double room[256];
    const double norm = norm_of(p, room);
    if (threadIdx.x == 0) p.norm[0] = (float)norm;
}

template <bool PAST>
__global__ void __launch_bounds__(256) scale_grads(const ClipParams p) {
    __shared__ double room[256];
    const double norm = norm_of(p, room);
    if (threadIdx.x == 0 && blockIdx.x == 0 && p.first_group == 0) p.norm[0] = (float)norm;
    // (a norm that is none, as it is read in fp32, leaves the gradients unclipped: whoever reads it can skip the step)
    const Factor factor(norm > p.max_norm && (float)norm < INFINITY ? p.unscale * (p.max_norm / norm) : p.unscale);
    for (uint32_t b = blockIdx.x; b < p.runs; b += gridDim.x) {
        const uint32_t r = p.runs - 1 - b;
        const int i = tensor_of(p, r);
        if (factor.first == 1.f && p.t[i].out == p.t[i].grad) continue;
        const uint32_t first = i ? p.t[i - 1].last_run : 0;
        const int64_t at = (int64_t)(r - first) * kRun;
        with_type(p.t[i].dt, [&](auto type) {
            using T = decltype(type);
            with_type(p.t[i].out_dt, [&](auto out_type) {
                using O = decltype(out_type);
                scale_run<T, O, PAST>(static_cast<const T *>(p.t[i].grad) + at, static_cast<O *>(p.t[i].out) + at, p.t[i].count - at, factor);
            });
        });
    }
}

inline int64_t runs_of(int64_t count) { return (count + kRun - 1) / kRun; }
inline int64_t groups_of(int64_t runs) { return runs < kMostGroups ? runs : kMostGroups; }

// The tensors of launch l.
ClipParams launch_of(const grim_grad_list &list, int64_t l) {
    ClipParams p{};
    const int64_t first = l * kTable, n = (int64_t)list.tensors.size() - first;
    p.tensors = (int32_t)(n < kTable ? n : kTable);
    for (int i = 0; i < p.tensors; ++i) {
        const grim_grad &t = list.tensors[first + i];
        p.t[i] = TensorArgs{t.grad, t.out, t.count, (uint32_t)list.last_run[first + i], (uint16_t)t.dt, (uint16_t)t.out_dt};
    }
    p.runs = p.t[p.tensors - 1].last_run;
    return p;
}

grim_status clip(const grim_grad_list *list, bool scales, float max_norm, float unscale, float *norm_dev, void *workspace, int64_t workspace_bytes,
                 void *hip_stream) {
    if (!list || !norm_dev || !workspace) return GRIM_ERR_NULL;
    if (!(max_norm >= 0.f) || !(fabsf(unscale) < INFINITY) || workspace_bytes < grim_grad_workspace(list)) return GRIM_ERR_SHAPE;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const int64_t launches = ((int64_t)list->tensors.size() + kTable - 1) / kTable;
    int64_t bytes = 0;
    for (const grim_grad &t : list->tensors) bytes += t.count * (bytes_of((grim_dtype)t.dt) + (scales ? bytes_of((grim_dtype)t.out_dt) : 0));
    uint32_t group = 0;
    const auto each = [&](auto launch) {
        group = 0;
        for (int64_t l = 0; l < launches; ++l) {
            ClipParams p = launch_of(*list, l);
            p.sums = static_cast<double *>(workspace), p.norm = norm_dev, p.groups = list->workgroups;
            p.unscale = unscale, p.max_norm = max_norm, p.first_group = group;
            const int64_t groups = groups_of(p.runs);
            launch(p, dim3((unsigned)groups));
            const grim_status st = launched();
            if (st != GRIM_OK) return st;
            group += (uint32_t)groups;
        }
        return GRIM_OK;
    };
    const grim_status st = each([&](const ClipParams &p, dim3 g) { hipLaunchKernelGGL(sum_squares, g, dim3(256), 0, stream, p); });
    if (st != GRIM_OK) return st;
    if (!scales || launches == 0) {
        ClipParams p{};
        p.sums = static_cast<double *>(workspace), p.norm = norm_dev, p.groups = list->workgroups, p.unscale = unscale;
        hipLaunchKernelGGL(write_norm, dim3(1), dim3(256), 0, stream, p);
        return launched();
    }
    return each([&](const ClipParams &p, dim3 g) {
        if (past_caches(bytes)) hipLaunchKernelGGL(scale_grads<true>, g, dim3(256), 0, stream, p);
        else hipLaunchKernelGGL(scale_grads<false>, g, dim3(256), 0, stream, p);
    });
}

// [address, end) of a tensor's gradients or outputs
struct Extent {
    uintptr_t lo, hi;
    size_t who;
};

}  // namespace lm
}  // namespace grim

extern "C" {

grim_status grim_grad_list_create(const grim_grad *grads, int32_t count, grim_grad_list **out) {
    using namespace grim::lm;
    if (!out) return GRIM_ERR_NULL;
    *out = nullptr;
    if (count < 0 || count > (1 << 20)) return GRIM_ERR_SHAPE;
    if (count > 0 && !grads) return GRIM_ERR_NULL;
    for (int32_t i = 0; i < count; ++i) {
        const grim_grad &t = grads[i];
        if (!known((grim_dtype)t.dt) || (t.out && !known((grim_dtype)t.out_dt))) return GRIM_ERR_DTYPE;
        if (t.count < 0 || t.count > (int64_t)1 << 40) return GRIM_ERR_SHAPE;
        if (t.count > 0 && !t.grad) return GRIM_ERR_NULL;
    }
    try {
        grim_grad_list list;
        std::vector<Extent> written;
        int64_t runs = 0;
        for (int32_t i = 0; i < count; ++i) {
            if (grads[i].count == 0) continue;
            if (list.tensors.size() % kTable == 0) list.workgroups += groups_of(runs), runs = 0;
            runs += runs_of(grads[i].count);
            if (runs >= (int64_t)1 << 31) return GRIM_ERR_SHAPE;
            list.tensors.push_back(grads[i]);
            list.last_run.push_back(runs);
            if (grads[i].out) {
                const uintptr_t at = (uintptr_t)grads[i].out;
                written.push_back({at, at + (uintptr_t)(grads[i].count * bytes_of((grim_dtype)grads[i].out_dt)), list.tensors.size() - 1});
            }
        }
        list.workgroups += groups_of(runs);
        // Outputs overlap nothing but the gradient that they replace.
        std::sort(written.begin(), written.end(), [](const Extent &a, const Extent &b) { return a.lo < b.lo; });
        for (size_t i = 1; i < written.size(); ++i)
            if (written[i].lo < written[i - 1].hi) return GRIM_ERR_SHAPE;
        for (size_t i = 0; i < list.tensors.size(); ++i) {
            const grim_grad &t = list.tensors[i];
            const uintptr_t lo = (uintptr_t)t.grad, hi = lo + (uintptr_t)(t.count * bytes_of((grim_dtype)t.dt));
            // (the outputs are in order and apart: the first one that ends behind lo)
            auto w = std::partition_point(written.begin(), written.end(), [&](const Extent &e) { return e.hi <= lo; });
            for (; w != written.end() && w->lo < hi; ++w)
                if (w->who != i || w->lo != lo || t.dt != t.out_dt) return GRIM_ERR_SHAPE;
        }
        grim_grad_list *kept = new (std::nothrow) grim_grad_list;
        if (!kept) return GRIM_ERR_ALLOC;
        std::swap(*kept, list);
        *out = kept;
        return GRIM_OK;
    } catch (...) {
        return GRIM_ERR_ALLOC;
    }
}

void grim_grad_list_free(grim_grad_list *list) { delete list; }

int64_t grim_grad_workspace(const grim_grad_list *list) { return list ? (list->workgroups > 0 ? list->workgroups : 1) * (int64_t)sizeof(double) : 0; }

grim_status grim_grad_norm(const grim_grad_list *list, float unscale, float *norm_dev, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    return grim::lm::clip(list, false, 0.f, unscale, norm_dev, workspace, workspace_bytes, hip_stream);
}

grim_status grim_grad_clip(const grim_grad_list *list, float max_norm, float unscale, float *norm_dev, void *workspace, int64_t workspace_bytes,
                           void *hip_stream) {
    if (list)
        for (const grim_grad &t : list->tensors)
            if (!t.out) return GRIM_ERR_NULL;
    return grim::lm::clip(list, true, max_norm, unscale, norm_dev, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
