// Global norm of many gradients with clipping, and the AdamW update that takes the clip's coefficient on the device.
//   norm = sqrt(sum over all tensors of g^2), coef = min(1, max_norm / (norm + eps)), g <- coef g
//   g = coef grad; m <- b1 m + (1 - b1) g; v <- b2 v + (1 - b2) g^2
//   p <- p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// A list of tensors is passed in the kernels' arguments, up to UP_CLIP / UP_ADAM of them per launch, so that nothing is copied to
// the device and a captured launch keeps its list.
#include "sol_internal.h"

namespace sol {

constexpr int UP_BLOCK = 256;
constexpr int UP_PARTS = 2048;                                      // workgroups of the norm per launch at most, each with a partial sum
constexpr uint64_t UP_STEPS = 0xffffff;                             // steps of a launch at most: 2^32 threads
constexpr int UP_VECS = 4;                                          // accesses of 16 bytes in flight per thread, for norm and scaling
constexpr int UP_STEP = 1024;                                       // elements of one step of an update's workgroup: four per thread
// elements of one step of a norm's or scaling's workgroup
template <class T> constexpr int clip_step() { return UP_BLOCK * UP_VECS * Vec16<T>::N; }
constexpr int UP_CLIP = 240, UP_ADAM = 80;                          // tensors per launch (arguments of at most 4 KB)
constexpr int64_t UP_LONGEST = (int64_t)1 << 31;                    // a longer tensor takes several places of a list

// first[i]: steps before tensor i
struct ClipList { int count; uint32_t first[UP_CLIP + 1]; void *g[UP_CLIP]; uint32_t n[UP_CLIP]; };
struct AdamList {
    int count; uint32_t first[UP_ADAM + 1];
    float *p[UP_ADAM], *m[UP_ADAM], *v[UP_ADAM]; const void *g[UP_ADAM]; bf16_t *copy[UP_ADAM]; uint32_t n[UP_ADAM];
};
static_assert(sizeof(ClipList) + 64 <= 4096 && sizeof(AdamList) + 128 <= 4096, "kernel arguments");

// f(tensor, first element, elements) for the steps blockIdx.x, blockIdx.x + gridDim.x, .. of a list, from its end to its beginning
// where BACK: what the pass before read last is then still in the caches.
template <bool BACK, int STEP, class L, class F> __device__ __forceinline__ void each_step(const L &l, F f)
{
    const uint32_t steps = l.first[l.count];
    int lo = 0, hi = l.count;                                       // first[lo] <= step < first[hi]
    for (uint32_t k = blockIdx.x; k < steps; k += gridDim.x) {
        const uint32_t c = BACK ? steps - 1 - k : k;
        if (BACK) lo = 0; else hi = l.count;                        // steps come in order: one end of the bracket stays
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (l.first[mid] <= c) lo = mid; else hi = mid;
        }
        const int64_t at = (int64_t)(c - l.first[lo]) * STEP, left = (int64_t)l.n[lo] - at;
        f(lo, at, (int)(left < STEP ? left : STEP));
    }
}

// Four consecutive elements of a thread. A pointer's phase is its distance from a boundary of N elements: where all streams of a tensor
// have one, its elements are taken from the boundaries on in single accesses of 8 or 16 bytes, else one by one.
template <class T> struct Four;
template <> struct Four<float> {
    static __device__ __forceinline__ void load(const float *p, float (&f)[4]) { const float4 v = *(const float4 *)p; f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
    static __device__ __forceinline__ void store(float *p, const float (&f)[4]) { *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]); }
};
template <> struct Four<bf16_t> {
    static __device__ __forceinline__ void load(const bf16_t *p, float (&f)[4])
    {
        const uint2 v = *(const uint2 *)p;
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
    static __device__ __forceinline__ void store(bf16_t *p, const float (&f)[4]) { *(uint2 *)p = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])); }
};
template <int N, class T> __device__ __forceinline__ int phase(const T *p) { return (int)((uintptr_t)p / sizeof(T) & (N - 1)); }

// A step's last `ph` elements lie behind its last thread's: the one that this thread takes, -1 if none
template <int STEP> __device__ __forceinline__ int last_ones(int ph, int n)
{
    const int e = STEP - ph + (int)threadIdx.x;
    return (int)threadIdx.x < ph && e < n ? e : -1;
}

// One step of one stream, UP_VECS accesses of 16 bytes per thread: whole(vector index, element) for those that lie inside, single(element)
// for the elements of the others
template <class T, class W, class S> __device__ __forceinline__ void stream_step(int ph, int n, W whole, S single)
{
    constexpr int V = Vec16<T>::N;
    const int j0 = (int)threadIdx.x * V - ph;
    static_for<UP_VECS>([&](auto v) {
        const int j = j0 + (int)v * UP_BLOCK * V;
        if (j >= 0 && j + V <= n) whole(v, j);
    });
#pragma unroll 1
    for (int v = 0; v < UP_VECS; ++v) {
        const int j = j0 + v * UP_BLOCK * V;
        if (j < n && (j < 0 || j + V > n))
            for (int e = 0; e < V; ++e) if (j + e >= 0 && j + e < n) single(j + e);
    }
    if (const int e = last_ones<clip_step<T>()>(ph, n); e >= 0) single(e);
}

template <int BLOCK> __device__ __forceinline__ double up_block_sum(double v, double *red)
{
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < BLOCK / 64; ++i) t += red[i];
    __syncthreads();
    return t;
}

// Squares are summed in 64 bits: neither do they overflow, nor does the number of elements show. Bound by reading the gradients once: 1.24 G
// bf16 elements 415 us, 5.9 TB/s (one 8-byte load in flight per thread: 1096).
template <class T>
__global__ void __launch_bounds__(UP_BLOCK) k_grad_squares(ClipList l, double *__restrict__ partial)
{
    __shared__ double red[UP_BLOCK / 64];
    double s = 0.0;
    each_step<false, clip_step<T>()>(l, [&](int i, int64_t at, int n) {
        const T *const g = (const T *)l.g[i] + at;
        Vec16<T> x[UP_VECS];
#pragma unroll
        for (int v = 0; v < UP_VECS; ++v) x[v].raw = {};
        stream_step<T>(phase<Vec16<T>::N>(g), n, [&](auto v, int j) { x[v].load(g + j); },
                       [&](int j) { const double f = (double)ld(g + j); s = __builtin_fma(f, f, s); });
#pragma unroll
        for (int v = 0; v < UP_VECS; ++v) {
            float f[Vec16<T>::N];
            x[v].unpack(f);
#pragma unroll
            for (int e = 0; e < Vec16<T>::N; ++e) s = __builtin_fma((double)f[e], (double)f[e], s);
        }
    });
    s = up_block_sum<UP_BLOCK>(s, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// coef is NaN where the norm is not finite: scaling and update then leave everything as it is
__global__ void __launch_bounds__(1024)
k_grad_norm(const double *__restrict__ partial, int64_t n, double max_norm, double eps, float *__restrict__ norm, float *__restrict__ coef)
{
    __shared__ double red[1024 / 64];
    double s = 0.0;
#pragma unroll 2
    for (int64_t i = threadIdx.x; i < n; i += 1024) s += partial[i];
    s = sqrt(up_block_sum<1024>(s, red));
    if (threadIdx.x == 0) {
        const double c = max_norm / (s + eps);
        *norm = (float)s;
        *coef = !((float)s < INFINITY) ? NAN : c < 1.0 ? (float)c : 1.f;
    }
}

// Every gradient read and written once more: 1.24 G bf16 elements 880 us, 5.6 TB/s with what the norm has left in the memory-side cache (2048
// looping workgroups 1110).
template <class T>
__global__ void __launch_bounds__(UP_BLOCK) k_grad_scale(ClipList l, const float *__restrict__ coef)
{
    const float f = *coef;
    if (!(f < 1.f)) return;
    each_step<true, clip_step<T>()>(l, [&](int i, int64_t at, int n) {
        T *const g = (T *)l.g[i] + at;
        Vec16<T> x[UP_VECS];
        const int ph = phase<Vec16<T>::N>(g);
        stream_step<T>(ph, n, [&](auto v, int j) { x[v].load(g + j); }, [&](int j) { st(g + j, ld(g + j) * f); });
        const int j0 = (int)threadIdx.x * Vec16<T>::N - ph;
#pragma unroll
        for (int v = 0; v < UP_VECS; ++v) {
            const int j = j0 + v * UP_BLOCK * Vec16<T>::N;
            if (j >= 0 && j + Vec16<T>::N <= n) {
                float y[Vec16<T>::N];
                x[v].unpack(y);
#pragma unroll
                for (int e = 0; e < Vec16<T>::N; ++e) y[e] *= f;
                x[v].pack(y);
                x[v].store(g + j);
            }
        }
    });
}

// b^t by squaring
__device__ __forceinline__ double pow_int(double b, int t)
{
    double r = 1.0;
    for (; t > 0; t >>= 1, b *= b) if (t & 1) r *= b;
    return r;
}

// All streams once, 28 bytes per element: 243 M elements with bf16 gradients and copies 1200 us, 5.7 TB/s (16384 looping workgroups 1455).
// Roundings: the moments and the parameter to 32 bits, the copy to bf16 from the rounded parameter.
template <class T>
__global__ void __launch_bounds__(UP_BLOCK)
k_adamw(AdamList l, AdamCfg a, const int32_t *__restrict__ step, const float *__restrict__ lr_dev, const float *__restrict__ coef, int *flags)
{
    const int t = *step;
    const float scale = coef ? *coef : 1.f;
    if (t < 1) { if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(flags, FLAG_BAD_STEP); return; }
    if (!(scale == scale)) return;
    const double lr = lr_dev ? (double)*lr_dev : a.lr;
    const float b1 = (float)a.beta1, c1 = (float)(1.0 - a.beta1), b2 = (float)a.beta2, c2 = (float)(1.0 - a.beta2);
    const float keep = (float)(1.0 - lr * a.weight_decay), rate = (float)(lr / (1.0 - pow_int(a.beta1, t)));
    const float corr = (float)(1.0 / (1.0 - pow_int(a.beta2, t))), eps = (float)a.eps;
    auto one = [&](float x, float &p, float &m, float &v) {
        x *= scale;
        m = b1 * m + c1 * x;
        v = b2 * v + c2 * x * x;
        p = p * keep - rate * m / (sqrtf(v * corr) + eps);
    };
    each_step<true, UP_STEP>(l, [&](int i, int64_t at, int n) {
        float *const p = l.p[i] + at, *const m = l.m[i] + at, *const v = l.v[i] + at;
        const T *const g = (const T *)l.g[i] + at;
        bf16_t *const copy = l.copy[i] ? l.copy[i] + at : nullptr;
        const int ph = phase<4>(p);
        auto single = [&](int j) {
            float pj = p[j], mj = m[j], vj = v[j];
            one(ld(g + j), pj, mj, vj);
            p[j] = pj; m[j] = mj; v[j] = vj;
            if (copy) copy[j] = f32_to_bf16(pj);
        };
        if (phase<4>(m) == ph && phase<4>(v) == ph && phase<4>(g) == ph && (!copy || phase<4>(copy) == ph)) {
            const int j = (int)threadIdx.x * 4 - ph;
            if (j >= 0 && j + 4 <= n) {
                float pf[4], mf[4], vf[4], gf[4];
                Four<float>::load(p + j, pf); Four<float>::load(m + j, mf); Four<float>::load(v + j, vf); Four<T>::load(g + j, gf);
#pragma unroll
                for (int e = 0; e < 4; ++e) one(gf[e], pf[e], mf[e], vf[e]);
                Four<float>::store(m + j, mf); Four<float>::store(v + j, vf); Four<float>::store(p + j, pf);
                if (copy) Four<bf16_t>::store(copy + j, pf);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) if (j + e >= 0 && j + e < n) single(j + e);
            }
            if (const int e = last_ones<UP_STEP>(ph, n); e >= 0) single(e);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) if (const int j = (int)threadIdx.x + e * UP_BLOCK; j < n) single(j);
        }
    });
}

// The list in parts of at most CAP places of one type: put(part, place, tensor, first element, elements), then f(type, part, its steps).
template <class List, int CAP, class Item, class Step, class Put, class F>
static void in_parts(const Item *items, int count, Step step, Put put, F f)
{
    for (int dtype = 0; dtype < 2; ++dtype) {
        List l;
        l.count = 0;
        uint64_t steps = 0;
        auto flush = [&] {
            if (l.count) { l.first[l.count] = (uint32_t)steps; f(dtype, l, (int)steps); }
            l.count = 0; steps = 0;
        };
        for (int i = 0; i < count; ++i) {
            if (items[i].dtype != dtype) continue;
            for (int64_t at = 0; at < items[i].n; at += UP_LONGEST) {
                const int64_t n = items[i].n - at < UP_LONGEST ? items[i].n - at : UP_LONGEST, c = (n + step(dtype) - 1) / step(dtype);
                if (l.count == CAP || steps + (uint64_t)c > UP_STEPS) flush();
                l.first[l.count] = (uint32_t)steps;
                put(l, l.count, items[i], at, (uint32_t)n);
                steps += (uint64_t)c; ++l.count;
            }
        }
        flush();
    }
}

// Partial sums of as many launches as `count` tensors of CLIP_MOST elements in all can take: UP_CLIP places each, one launch more per type
// (2), the 64 further places of tensors of over 2^31 elements (1), launches that end at UP_STEPS steps (2).
size_t clip_scratch_bytes(int count) { return ((size_t)count / UP_CLIP + 5) * UP_PARTS * sizeof(double); }
static_assert(CLIP_MOST / UP_LONGEST < UP_CLIP && CLIP_MOST / clip_step<float>() <= 3 * UP_STEPS, "launches of the norm");

void launch_grad_clip(const GradItem *items, int count, double max_norm, double eps, bool scale, float *norm, float *coef, void *scratch,
                      hipStream_t st)
{
    double *const partial = (double *)scratch;
    int64_t used = 0;
    auto step = [](int dtype) { return dtype == 1 ? clip_step<bf16_t>() : clip_step<float>(); };
    auto put = [](ClipList &l, int i, const GradItem &t, int64_t at, uint32_t n) { l.g[i] = (char *)t.g + at * (t.dtype == 1 ? 2 : 4); l.n[i] = n; };
    in_parts<ClipList, UP_CLIP>(items, count, step, put, [&](int dtype, const ClipList &l, int steps) {
        const int grid = steps < UP_PARTS ? steps : UP_PARTS;
        if (dtype == 1) hipLaunchKernelGGL(k_grad_squares<bf16_t>, dim3(grid), dim3(UP_BLOCK), 0, st, l, partial + used);
        else hipLaunchKernelGGL(k_grad_squares<float>, dim3(grid), dim3(UP_BLOCK), 0, st, l, partial + used);
        used += grid;
    });
    hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(1024), 0, st, partial, used, max_norm, eps, norm, coef);
    if (scale)
        in_parts<ClipList, UP_CLIP>(items, count, step, put, [&](int dtype, const ClipList &l, int steps) {
            if (dtype == 1) hipLaunchKernelGGL(k_grad_scale<bf16_t>, dim3(steps), dim3(UP_BLOCK), 0, st, l, coef);
            else hipLaunchKernelGGL(k_grad_scale<float>, dim3(steps), dim3(UP_BLOCK), 0, st, l, coef);
        });
}

void launch_adamw(const AdamItem *items, int count, const AdamCfg &a, const int32_t *step, const float *lr_dev, const float *coef,
                  int *flags, hipStream_t st)
{
    auto put = [](AdamList &l, int i, const AdamItem &t, int64_t at, uint32_t n) {
        l.p[i] = t.p + at; l.m[i] = t.m + at; l.v[i] = t.v + at; l.n[i] = n;
        l.g[i] = (const char *)t.g + at * (t.dtype == 1 ? 2 : 4);
        l.copy[i] = t.copy ? (bf16_t *)t.copy + at : nullptr;
    };
    in_parts<AdamList, UP_ADAM>(items, count, [](int) { return UP_STEP; }, put, [&](int dtype, const AdamList &l, int steps) {
        if (dtype == 1) hipLaunchKernelGGL(k_adamw<bf16_t>, dim3(steps), dim3(UP_BLOCK), 0, st, l, a, step, lr_dev, coef, flags);
        else hipLaunchKernelGGL(k_adamw<float>, dim3(steps), dim3(UP_BLOCK), 0, st, l, a, step, lr_dev, coef, flags);
    });
}

}  // namespace sol
