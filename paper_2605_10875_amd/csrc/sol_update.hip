// Global norm of many gradients with clipping, and the AdamW update that takes the clip's coefficient on the device.
//   norm = sqrt(sum over all tensors of g^2), coef = min(1, max_norm / (norm + eps)), g <- coef g
//   g = coef grad; m <- b1 m + (1 - b1) g; v <- b2 v + (1 - b2) g^2
//   p <- p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// A list of tensors is passed in the kernels' arguments, up to UP_CLIP / UP_ADAM of them per launch, so that nothing is copied to
// the device and a captured launch keeps its list.
#include "sol_internal.h"

namespace sol {

constexpr int UP_BLOCK = 256;
constexpr int UP_GRID = 2048;                                       // workgroups per launch at most
constexpr int UP_CHUNK = 4096;                                      // elements of one step of a workgroup
constexpr int UP_CLIP = 160, UP_ADAM = 56;                          // tensors per launch (arguments of at most 4 KB)

// first[i]: chunks before tensor i
struct ClipList { int count; uint32_t first[UP_CLIP + 1]; void *g[UP_CLIP]; int64_t n[UP_CLIP]; };
struct AdamList {
    int count; uint32_t first[UP_ADAM + 1];
    float *p[UP_ADAM], *m[UP_ADAM], *v[UP_ADAM]; const void *g[UP_ADAM]; bf16_t *copy[UP_ADAM]; int64_t n[UP_ADAM];
};
static_assert(sizeof(ClipList) <= 3600 && sizeof(AdamList) <= 3600, "kernel arguments");

template <class L> __device__ __forceinline__ int tensor_of(const L &l, uint32_t chunk)
{
    int lo = 0, hi = l.count;                                       // first[lo] <= chunk < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= chunk) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double up_block_sum(double v, double *red)
{
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < UP_BLOCK / 64; ++i) t += red[i];
    __syncthreads();
    return t;
}

// Squares are summed in 64 bits: neither do they overflow, nor does the number of elements show.
template <class T>
__global__ void __launch_bounds__(UP_BLOCK) k_grad_squares(ClipList l, double *__restrict__ partial)
{
    __shared__ double red[UP_BLOCK / 64];
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < l.first[l.count]; c += gridDim.x) {
        const int i = tensor_of(l, c);
        const T *const g = (const T *)l.g[i];
        const int64_t at = (int64_t)(c - l.first[i]) * UP_CHUNK, end = at + UP_CHUNK < l.n[i] ? at + UP_CHUNK : l.n[i];
        for (int64_t j = at + threadIdx.x; j < end; j += UP_BLOCK) { const double x = (double)ld(g + j); s += x * x; }
    }
    s = up_block_sum(s, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// coef is NaN where the norm is not finite: scaling and update then leave everything as it is
__global__ void __launch_bounds__(UP_BLOCK)
k_grad_norm(const double *__restrict__ partial, int64_t n, double max_norm, double eps, float *__restrict__ norm, float *__restrict__ coef)
{
    __shared__ double red[UP_BLOCK / 64];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += UP_BLOCK) s += partial[i];
    s = sqrt(up_block_sum(s, red));
    if (threadIdx.x == 0) {
        *norm = (float)s;
        const double c = max_norm / (s + eps);
        *coef = !(s < INFINITY) ? NAN : c < 1.0 ? (float)c : 1.f;
    }
}

template <class T>
__global__ void __launch_bounds__(UP_BLOCK) k_grad_scale(ClipList l, const float *__restrict__ coef)
{
    const float f = *coef;
    if (!(f < 1.f)) return;
    for (uint32_t c = blockIdx.x; c < l.first[l.count]; c += gridDim.x) {
        const int i = tensor_of(l, c);
        T *const g = (T *)l.g[i];
        const int64_t at = (int64_t)(c - l.first[i]) * UP_CHUNK, end = at + UP_CHUNK < l.n[i] ? at + UP_CHUNK : l.n[i];
        for (int64_t j = at + threadIdx.x; j < end; j += UP_BLOCK) st(g + j, ld(g + j) * f);
    }
}

// b^t by squaring
__device__ __forceinline__ double pow_int(double b, int t)
{
    double r = 1.0;
    for (; t > 0; t >>= 1, b *= b) if (t & 1) r *= b;
    return r;
}

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
    for (uint32_t c = blockIdx.x; c < l.first[l.count]; c += gridDim.x) {
        const int i = tensor_of(l, c);
        float *const p = l.p[i], *const m = l.m[i], *const v = l.v[i];
        const T *const g = (const T *)l.g[i];
        bf16_t *const copy = l.copy[i];
        const int64_t at = (int64_t)(c - l.first[i]) * UP_CHUNK, end = at + UP_CHUNK < l.n[i] ? at + UP_CHUNK : l.n[i];
        for (int64_t j = at + threadIdx.x; j < end; j += UP_BLOCK) {
            const float x = ld(g + j) * scale;
            const float mn = b1 * m[j] + c1 * x, vn = b2 * v[j] + c2 * x * x;
            const float pn = p[j] * keep - rate * mn / (sqrtf(vn * corr) + eps);
            m[j] = mn; v[j] = vn; p[j] = pn;
            if (copy) copy[j] = f32_to_bf16(pn);
        }
    }
}

// The list in parts of at most CAP tensors of one type: f(type, part, workgroups).
template <class List, int CAP, class Item, class Put, class F>
static void in_parts(const Item *items, int count, Put put, F f)
{
    for (int dtype = 0; dtype < 2; ++dtype) {
        List l;
        l.count = 0;
        uint64_t chunks = 0;
        auto flush = [&] {
            if (l.count) { l.first[l.count] = (uint32_t)chunks; f(dtype, l, (int)(chunks < UP_GRID ? chunks : UP_GRID)); }
            l.count = 0; chunks = 0;
        };
        for (int i = 0; i < count; ++i) {
            if (items[i].dtype != dtype || items[i].n == 0) continue;
            const uint64_t c = (uint64_t)((items[i].n + UP_CHUNK - 1) / UP_CHUNK);
            if (l.count == CAP || chunks + c > 0x7fffffffu) flush();
            l.first[l.count] = (uint32_t)chunks;
            put(l, l.count, items[i]);
            chunks += c; ++l.count;
        }
        flush();
    }
}

size_t clip_scratch_bytes(int count) { return ((size_t)count / UP_CLIP + 3) * UP_GRID * sizeof(double); }

void launch_grad_clip(const GradItem *items, int count, double max_norm, double eps, bool scale, float *norm, float *coef, void *scratch,
                      hipStream_t st)
{
    double *const partial = (double *)scratch;
    int64_t used = 0;
    auto put = [](ClipList &l, int i, const GradItem &t) { l.g[i] = t.g; l.n[i] = t.n; };
    in_parts<ClipList, UP_CLIP>(items, count, put, [&](int dtype, const ClipList &l, int grid) {
        if (dtype == 1) hipLaunchKernelGGL(k_grad_squares<bf16_t>, dim3(grid), dim3(UP_BLOCK), 0, st, l, partial + used);
        else hipLaunchKernelGGL(k_grad_squares<float>, dim3(grid), dim3(UP_BLOCK), 0, st, l, partial + used);
        used += grid;
    });
    hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(UP_BLOCK), 0, st, partial, used, max_norm, eps, norm, coef);
    if (scale)
        in_parts<ClipList, UP_CLIP>(items, count, put, [&](int dtype, const ClipList &l, int grid) {
            if (dtype == 1) hipLaunchKernelGGL(k_grad_scale<bf16_t>, dim3(grid), dim3(UP_BLOCK), 0, st, l, coef);
            else hipLaunchKernelGGL(k_grad_scale<float>, dim3(grid), dim3(UP_BLOCK), 0, st, l, coef);
        });
}

void launch_adamw(const AdamItem *items, int count, const AdamCfg &a, const int32_t *step, const float *lr_dev, const float *coef,
                  int *flags, hipStream_t st)
{
    auto put = [](AdamList &l, int i, const AdamItem &t) {
        l.p[i] = t.p; l.m[i] = t.m; l.v[i] = t.v; l.g[i] = t.g; l.copy[i] = (bf16_t *)t.copy; l.n[i] = t.n;
    };
    in_parts<AdamList, UP_ADAM>(items, count, put, [&](int dtype, const AdamList &l, int grid) {
        if (dtype == 1) hipLaunchKernelGGL(k_adamw<bf16_t>, dim3(grid), dim3(UP_BLOCK), 0, st, l, a, step, lr_dev, coef, flags);
        else hipLaunchKernelGGL(k_adamw<float>, dim3(grid), dim3(UP_BLOCK), 0, st, l, a, step, lr_dev, coef, flags);
    });
}

}  // namespace sol
