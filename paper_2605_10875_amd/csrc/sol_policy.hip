// Clipped policy loss over the actions of a likelihood pass, forward and gradient in one call (the update that the advantages of
// sol_reward.hip are made for). Per row (input b, schedule g, step t) of logits x_j, with z = x / temperature:
//   logp_j = z_j - log sum exp z, p_j = exp(logp_j), a the action taken, d = logp_a - old, rho = exp(d)
//   pg = -min(rho A, clip(rho, 1 - lo, 1 + hi) A),  H = -sum p_j logp_j
//   KL = exp(u) - u - 1 with u = ref - logp_a (estimate), or sum p_j (logp_j - logq_j) (exact, from reference logits y_j)
//   loss = scale * sum w (pg + beta KL - c H), w the row's share in the mean
// With the row's maximum m, t_j = (x_j - m) log2(e) / temperature, e_j = 2^(t_j), S = sum e_j,
// U = sum e_j t_j and, with a reference, t'_j, S' likewise and K = sum e_j (t_j - t'_j):
//   H = log S - ln2 U / S,  KL = ln2 K / S - (log S - log S')
//   d loss / d x_j = p_j (alpha + gamma t_j + kappa (t_j - t'_j)) + [j = a] w' G
// where w' = w scale / temperature, G = d(pg + beta KL) / d logp_a, gamma = w' c ln2, kappa = w' beta ln2 and
// alpha = -w' (G + c ln2 U / S + beta ln2 K / S): the row needs its sums once, then every element's gradient by itself.
// Where e_j is 0 (x_j = -inf above all) its products are 0 whatever the other factor is: times().
#include "sol_internal.h"

namespace sol {

constexpr int PL_BLOCK = 256;
constexpr int PL_GRID = 2048;                                       // workgroups of the rows' kernel at most
constexpr float PL_LOG2E = 1.44269504088896341f;
constexpr double PL_LN2 = 0.693147180559945309;
constexpr float PL_LOWEST = -3.402823466e38f;                       // below every finite logit's maximum: no NaN from -inf - -inf

struct PolicyScalars { double inv_temp, log_lo, log_hi, factor, kl, ent, scale; float lo, hi; };      // factor: scale / temperature

// what a row needs besides its sums
struct PolicyRow { int a; float adv, old, ref; double w; };
struct PolicySums { float S, Sr, U, K, xa; };                       // xa: the taken action's logit
struct PolicyCoef { float alpha, gamma, kappa, hot, logp, pg, kl, ent, clipped; };

// The share of an effective step of input b in the mean, 0 if the input has none. n: effective steps of the input, all: of all
// inputs, or the inputs that have any (by_schedule), times the schedules.
__device__ __forceinline__ double policy_share(int n, double all, int by_schedule)
{
    return n == 0 ? 0.0 : by_schedule ? 1.0 / ((double)n * all) : 1.0 / all;
}

// Few flags (PL_FEW of them, PL_INPUTS inputs at most): every workgroup counts them itself, which costs about a microsecond where
// the two kernels below cost two launches.
constexpr int PL_FEW = 4096, PL_INPUTS = 256;
struct PolicyShares { int n[PL_INPUTS]; int all; };
template <int BLOCK> __device__ __forceinline__ void policy_count(const PolicyArgs &q, PolicyShares &s)
{
    for (int b = threadIdx.x; b < q.B; b += BLOCK) s.n[b] = 0;
    if (threadIdx.x == 0) s.all = 0;
    __syncthreads();
    // 64 flags at a time: the first lane of each input among them adds what its part of the wave's ballot counts
    for (int at = threadIdx.x & ~63; at < q.B * q.T; at += BLOCK) {
        const int lane = threadIdx.x & 63, i = at + lane;
        const bool in = i < q.B * q.T;
        const unsigned long long set = __ballot(in && q.eff[in ? i : 0] != 0);
        const int b = i / q.T, t = i - b * q.T;
        if (in && (lane == 0 || t == 0)) {
            const int len = q.T - t < 64 - lane ? q.T - t : 64 - lane;
            const int c = __popcll((set >> lane) & (len == 64 ? ~0ull : (1ull << len) - 1));
            if (c) atomicAdd(&s.n[b], c);
        }
    }
    __syncthreads();
    for (int b = threadIdx.x; b < q.B; b += BLOCK) atomicAdd(&s.all, q.by_schedule ? s.n[b] > 0 : s.n[b]);
    __syncthreads();
}

// Many flags: LANES lanes count an input's, and each workgroup adds up its inputs'; then the shares. B and T may be close to 2^31. Bound by
// latency at few inputs (8 of 2048 flags: 3 us each), by reading the flags at many.
__device__ __forceinline__ int64_t policy_block_sum(int64_t v, int64_t *red)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < PL_BLOCK / 64; ++i) v += red[i];
    __syncthreads();
    return v;
}
template <int LANES>
__global__ void __launch_bounds__(PL_BLOCK)
k_policy_count(const int32_t *__restrict__ eff, int B, int T, int by_schedule, int32_t *__restrict__ n, int64_t *__restrict__ part)
{
    constexpr int INPUTS = PL_BLOCK / LANES;
    __shared__ int64_t red[PL_BLOCK / 64];
    const int lane = threadIdx.x % LANES;
    int64_t sum = 0;
    for (int64_t first = (int64_t)blockIdx.x * INPUTS; first < B; first += (int64_t)gridDim.x * INPUTS) {
        const int64_t b = first + threadIdx.x / LANES;
        int64_t c = 0;
        if (b < B)
#pragma unroll 4
            for (int64_t t = lane; t < T; t += LANES) c += eff[b * T + t] != 0;
        if (LANES > 64) c = policy_block_sum(c, red);
        else
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
        if (b < B && lane == 0) {
            n[b] = (int32_t)c;
            sum += by_schedule ? c > 0 : c;
        }
    }
    sum = policy_block_sum(sum, red);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}
__global__ void __launch_bounds__(PL_BLOCK)
k_policy_weights(const int32_t *__restrict__ n, const int64_t *__restrict__ part, int parts, int B, int G, int by_schedule, double *__restrict__ w)
{
    __shared__ int64_t red[PL_BLOCK / 64];
    int64_t c = 0;
    for (int i = threadIdx.x; i < parts; i += PL_BLOCK) c += part[i];
    const double all = (double)policy_block_sum(c, red) * (double)G;
    for (int64_t b = (int64_t)blockIdx.x * PL_BLOCK + threadIdx.x; b < B; b += (int64_t)gridDim.x * PL_BLOCK)
        w[b] = policy_share(n[b], all, by_schedule);
}

// exp(u) - u - 1: by its series near 0, where the difference would keep a few bits only (|u| < 0.5: the first term left out
// is below 2^-33 of the sum), without the difference where u is infinite
__device__ __forceinline__ float policy_kl(float u)
{
    float s = 1.f / 3628800.f;
    s = s * u + 1.f / 362880.f;
    s = s * u + 1.f / 40320.f;
    s = s * u + 1.f / 5040.f;
    s = s * u + 1.f / 720.f;
    s = s * u + 1.f / 120.f;
    s = s * u + 1.f / 24.f;
    s = s * u + 1.f / 6.f;
    s = s * u + 0.5f;
    return fabsf(u) < 0.5f ? s * u * u : u > 60.f ? expf(u) : expf(u) - u - 1.f;
}

// log x for 2^-1000 < x < 2^1000: mantissa in [sqrt 1/2, sqrt 2), log f = 2 artanh((f - 1) / (f + 1)), whose argument is at most
// 0.1716, so that the first term left out (s^17) is below 1e-14. A third of the instructions of the library's.
__device__ __forceinline__ double policy_log(double x)
{
    double f = __builtin_amdgcn_frexp_mant(x);
    int k = __builtin_amdgcn_frexp_exp(x);
    if (f < 0.70710678118654752) { f *= 2.0; --k; }
    const double d = f + 1.0;
    double r = __builtin_amdgcn_rcp(d);
    r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
    r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
    const double s = (f - 1.0) * r, q = s * s;
    double p = 2.0 / 15.0;
    p = __builtin_fma(p, q, 2.0 / 13.0);
    p = __builtin_fma(p, q, 2.0 / 11.0);
    p = __builtin_fma(p, q, 2.0 / 9.0);
    p = __builtin_fma(p, q, 2.0 / 7.0);
    p = __builtin_fma(p, q, 2.0 / 5.0);
    p = __builtin_fma(p, q, 2.0 / 3.0);
    p = __builtin_fma(p, q, 2.0);
    return __builtin_fma((double)k, PL_LN2, s * p);
}

// t of a logit f. As one fma, c = -m k rounded: every t of the row is then off by the same fma(m, k, c), which cancels in p, H and KL and
// which policy_row takes out of the log-probability. That holds while the offset is small, |m k| <= PL_FAR (offset below 1/4; c is
// bounded by it, so that it stays finite); rows beyond it are centred first (policy_centred), or take the difference itself (SUB).
constexpr float PL_FAR = 4194304.f;
struct PolicyScale { float k, c; };
template <bool SUB> __device__ __forceinline__ PolicyScale policy_scale(float m, float k)
{
    return PolicyScale{k, SUB ? m : -fminf(fmaxf(m * k, -PL_FAR), PL_FAR)};
}
template <bool SUB> __device__ __forceinline__ float policy_t(float f, PolicyScale z)
{
    return SUB ? (f - z.c) * z.k : __builtin_fmaf(f, z.k, z.c);
}
// a b, 0 where a or b is 0 (also against infinities and NaN): v_mul_legacy_f32, which has no builtin of clang
extern "C" __device__ float sol_mul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float times(float a, float b) { return sol_mul_legacy(a, b); }

// The row's loss terms and the coefficients of its gradient from its sums. The ratio's bounds are tested on its logarithm in 64 bits: a
// gradient is not continuous there. m: the row's maximum, off: its t.
__device__ __forceinline__ PolicyCoef policy_row(const PolicyScalars &pc, const PolicyRow &r, const PolicySums &s, float m, float off,
                                                 bool has_old, bool has_ref, bool exact_kl)
{
    PolicyCoef c;
    const double logS = policy_log((double)s.S), logp = ((double)s.xa - (double)m) * pc.inv_temp + (double)off * PL_LN2 - logS;
    const double d = has_old ? logp - (double)r.old : 0.0;
    const float A = r.adv, rho = expf((float)d);
    const bool clipped = (A > 0.f && d > pc.log_hi) || (A < 0.f && d < pc.log_lo);
    c.logp = (float)logp;
    c.pg = clipped ? -(A > 0.f ? pc.hi : pc.lo) * A : -rho * A;
    float G = clipped ? 0.f : -rho * A;
    const float beta = (float)pc.kl, ln2 = (float)PL_LN2, inv = 1.f / s.S, u_mean = ln2 * s.U * inv;
    c.ent = (float)(logS - (double)u_mean);
    c.kl = 0.f;
    float k_mean = 0.f;
    if (exact_kl) {
        k_mean = ln2 * s.K * inv;
        c.kl = (float)((double)k_mean - (logS - policy_log((double)s.Sr)));
    } else if (has_ref) {
        const float u = (float)((double)r.ref - logp);
        c.kl = policy_kl(u);
        G -= times(beta, u + c.kl);                                 // 1 - exp(u); an infinite KL without a coefficient is no one's
    }
    c.clipped = clipped ? 1.f : 0.f;
    const float w = (float)(r.w * pc.factor), ent = (float)pc.ent;
    c.hot = w * G;
    c.alpha = -w * (G + ent * u_mean + (exact_kl ? times(beta, k_mean) : 0.f)) * inv;
    c.gamma = w * ent * ln2 * inv;
    c.kappa = exact_kl ? w * beta * ln2 * inv : 0.f;
    return c;
}

// ---- a row's elements in 16-byte pieces -------------------------------------------------------------------------
// Piece i of a row covers elements V i - mis .. V i - mis + V - 1, mis being the row's distance from a 16-byte boundary in elements: inside
// the row every piece is one aligned access whatever the row's length and start are. The pieces that the row's ends cut are loaded
// as the 16 bytes at that end, not aligned, and shifted into place once they are there (policy_cut); elements outside are -inf.
template <class T> __device__ __forceinline__ int policy_mis(const T *x) { return (int)(((uintptr_t)x & 15) / sizeof(T)); }
template <class T> __device__ __forceinline__ uint4 policy_none()
{
    const uint32_t w = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
    return make_uint4(w, w, w, w);
}
// the 16 bytes nearest to element j that lie in the row; element by element for rows that have fewer, which are not LONG
template <bool LONG, class T> __device__ __forceinline__ uint4 policy_load(const T *x, int j, int A)
{
    constexpr int V = Vec16<T>::N;
    uint4 r;
    if (LONG || A >= V) {
        const int at = j < 0 ? 0 : j > A - V ? A - V : j;
        __builtin_memcpy(&r, x + at, 16);
        return r;
    }
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = j + i * (V / 4);
        if (sizeof(T) == 4) w[i] = (unsigned)e < (unsigned)A ? ((const uint32_t *)x)[e] : 0xFF800000u;
        else {
            const uint32_t lo = (unsigned)e < (unsigned)A ? ((const uint16_t *)x)[e] : 0xFF80u;
            const uint32_t hi = (unsigned)(e + 1) < (unsigned)A ? ((const uint16_t *)x)[e + 1] : 0xFF80u;
            w[i] = lo | hi << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// what policy_load(x, j, A) gave, as elements j .. j + V - 1: the four words moved by whole words, then by half of one
template <bool LONG, class T> __device__ __forceinline__ uint4 policy_cut(uint4 r, int j, int A)
{
    constexpr int V = Vec16<T>::N, H = V / 4;                       // elements per word
    if ((LONG || A >= V) && (j < 0 || j > A - V)) {
        const uint32_t none = policy_none<T>().x;
        const int by = j < 0 ? -j : j - (A - V);                    // elements, 0 < by < V
        if (j < 0) {
            if (by & 2 * H) r = make_uint4(none, none, r.x, r.y);
            if (by & H) r = make_uint4(none, r.x, r.y, r.z);
            if (H == 2 && (by & 1)) r = make_uint4(none >> 16 | r.x << 16, r.x >> 16 | r.y << 16, r.y >> 16 | r.z << 16, r.z >> 16 | r.w << 16);
        } else {
            if (by & 2 * H) r = make_uint4(r.z, r.w, none, none);
            if (by & H) r = make_uint4(r.y, r.z, r.w, none);
            if (H == 2 && (by & 1)) r = make_uint4(r.x >> 16 | r.y << 16, r.y >> 16 | r.z << 16, r.z >> 16 | r.w << 16, r.w >> 16 | none << 16);
        }
    }
    return r;
}
template <class T> __device__ __forceinline__ void policy_unpack(uint4 raw, float *f)
{
    Vec16<T> v;
    v.raw = __builtin_bit_cast(decltype(v.raw), raw);
    v.unpack(f);
}
template <class T> __device__ __forceinline__ void policy_put(T *d, const float *f, int j, int A)
{
    constexpr int V = Vec16<T>::N;
    if (j >= 0 && j + V <= A) {
        uint4 r;
        if (sizeof(T) == 4) r = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        else r = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4 % V], f[5 % V]), pack_bf16x2(f[6 % V], f[7 % V]));
        __builtin_memcpy(d + j, &r, 16);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) if ((unsigned)(j + i) < (unsigned)A) st(d + j + i, f[i]);
    }
}

// a row of zeros
template <class T> __device__ __forceinline__ void policy_clear(T *d, int A, int lane, int lanes)
{
    constexpr int V = Vec16<T>::N;
    const float zero[V] = {};
    for (int64_t j = (int64_t)lane * V - policy_mis(d); j < A; j += lanes * V) policy_put(d, zero, (int)j, A);
}

// ---- sums over the LANES lanes of a row: inside a wave, or over the waves of the workgroup ---------------------------
template <int LANES, class Op> __device__ __forceinline__ float lanes_reduce(float v, Op op)
{
    auto dpp = [&](auto ctrl) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, 0xF, 0xF, false));
    };
    if (LANES >= 2) v = op(v, dpp(std::integral_constant<int, 0xB1>{}));     // neighbour
    if (LANES >= 4) v = op(v, dpp(std::integral_constant<int, 0x4E>{}));     // other pair of the four
    if (LANES >= 8) v = op(v, dpp(std::integral_constant<int, 0x141>{}));    // other four of the eight
    if (LANES >= 16) v = op(v, dpp(std::integral_constant<int, 0x140>{}));   // other eight of the sixteen
    if (LANES >= 32) v = op(v, __shfl_xor(v, 16, 64));
    if (LANES >= 64) v = op(v, __shfl_xor(v, 32, 64));
    return v;
}
struct OpMaxF { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// N values at once; slot: LDS of this use alone. One barrier: a slot is written again only behind the other slot's barrier.
template <int LANES, int N, class Op> __device__ __forceinline__ void row_reduce(float (&v)[N], Op op, float (*slot)[16])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_reduce<(LANES > 64 ? 64 : LANES)>(v[i], op);
    if (LANES > 64) {
        constexpr int W = LANES / 64;
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) slot[i][w] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_reduce<(W < 2 ? 2 : W)>(slot[i][lane & (W - 1)], op);
    }
}

// the values that a row without (with) a reference has: 1 of 2 maxima; S, U and the logit of 5 sums
template <int LANES, bool EXACT, int N, class Op> __device__ __forceinline__ void reduce_some(float (&v)[N], Op op, float (*slot)[16])
{
    if constexpr (EXACT) row_reduce<LANES>(v, op, slot);
    else if constexpr (N == 2) {
        float u[1] = {v[0]};
        row_reduce<LANES>(u, op, slot);
        v[0] = u[0];
    } else {
        float u[3] = {v[0], v[1], v[4]};
        row_reduce<LANES>(u, op, slot);
        v[0] = u[0]; v[1] = u[1]; v[4] = u[2];
    }
}

// A row's share of the loss, and its inputs but the logits
__device__ __forceinline__ double policy_weight(const PolicyArgs &q, int row, double w_all, const double *w_in, const PolicyShares &few)
{
    if (!q.eff) return w_all;
    const int b = row / (q.G * q.T), t = row % q.T;
    if (!q.eff[(int64_t)b * q.T + t]) return 0.0;
    return w_in ? w_in[b] : policy_share(few.n[b], (double)few.all * (double)q.G, q.by_schedule);
}
// the same for all lanes of a wave
__device__ __forceinline__ double uniform(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b), hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ PolicyRow policy_inputs(const PolicyArgs &q, int row, double w, bool first)
{
    PolicyRow r;
    r.a = q.ids[row];
    if (r.a < 0 || r.a >= q.A) { r.a = 0; if (first) atomicOr(q.flags, FLAG_BAD_ACTION); }
    r.adv = q.adv ? q.adv[row] : 0.f;
    r.old = q.old_logp ? q.old_logp[row] : 0.f;
    r.ref = q.ref_logp ? q.ref_logp[row] : 0.f;
    r.w = w;
    return r;
}

template <class T, bool EXACT, bool SUB> struct PolicyPiece {
    static constexpr int V = Vec16<T>::N;
    // xa: the logit `at` elements behind the piece's first, if it is among them
    static __device__ __forceinline__ void max(uint4 rx, uint4 ry, int at, float (&m)[2], float &xa)
    {
        float f[V];
        policy_unpack<T>(rx, f);
#pragma unroll
        for (int i = 0; i < V; ++i) m[0] = fmaxf(m[0], f[i]);
        if ((unsigned)at < (unsigned)V)
#pragma unroll
            for (int i = 0; i < V; ++i) xa = i == at ? f[i] : xa;
        if (EXACT) {
            policy_unpack<T>(ry, f);
#pragma unroll
            for (int i = 0; i < V; ++i) m[1] = fmaxf(m[1], f[i]);
        }
    }
    // s: S, U, S', K
    static __device__ __forceinline__ void sums(uint4 rx, uint4 ry, PolicyScale z, PolicyScale zr, float (&s)[5])
    {
        float f[V], g[V];
        policy_unpack<T>(rx, f);
        if (EXACT) policy_unpack<T>(ry, g);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float t = policy_t<SUB>(f[i], z), e = __builtin_amdgcn_exp2f(t);
            s[0] += e;
            s[1] += times(e, t);
            if (EXACT) {
                const float r = policy_t<SUB>(g[i], zr);
                s[2] += __builtin_amdgcn_exp2f(r);
                s[3] += times(e, t - r);
            }
        }
    }
    static __device__ __forceinline__ void grad(uint4 rx, uint4 ry, PolicyScale z, PolicyScale zr, const PolicyCoef &c, int at, float (&o)[V])
    {
        float f[V], g[V];
        policy_unpack<T>(rx, f);
        if (EXACT) policy_unpack<T>(ry, g);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float t = policy_t<SUB>(f[i], z), e = __builtin_amdgcn_exp2f(t);
            float h = __builtin_fmaf(c.gamma, t, c.alpha);
            if (EXACT) h += times(c.kappa, t - policy_t<SUB>(g[i], zr));
            o[i] = times(e, h);
        }
        if ((unsigned)at < (unsigned)V)
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] += i == at ? c.hot : 0.f;
    }
};

// Rows beyond PL_FAR: logits minus the maximum. bf16 logits of that size lie 2^13 / k apart at least, so that rounding a difference
// that is not 0 back to 8 bits leaves 2^t = 0.
__device__ __forceinline__ bool policy_is_far(float m, float k) { return !(fabsf(m * k) <= PL_FAR); }
template <class T> __device__ __forceinline__ uint4 policy_centred(uint4 raw, float m)
{
    constexpr int V = Vec16<T>::N;
    float f[V];
    policy_unpack<T>(raw, f);
    if (sizeof(T) == 4) return make_uint4(__float_as_uint(f[0] - m), __float_as_uint(f[1] - m), __float_as_uint(f[2] - m), __float_as_uint(f[3] - m));
    return make_uint4(pack_bf16x2(f[0] - m, f[1] - m), pack_bf16x2(f[2] - m, f[3] - m), pack_bf16x2(f[4 % V] - m, f[5 % V] - m),
                      pack_bf16x2(f[6 % V] - m, f[7 % V] - m));
}

// Sums of a lane relative to a running maximum: turn() makes them relative to a larger one.
template <bool EXACT, bool SUB> struct PolicyRunning {
    float m[2] = {PL_LOWEST, PL_LOWEST}, s[5] = {0.f, 0.f, 0.f, 0.f, 0.f}, k;
    PolicyScale z, zr;
    __device__ __forceinline__ explicit PolicyRunning(float scale) : k(scale) { z = zr = policy_scale<SUB>(m[0], k); }
    __device__ __forceinline__ void turn(const float (&n)[2])
    {
        const PolicyScale y = policy_scale<SUB>(n[0], k), yr = EXACT ? policy_scale<SUB>(n[1], k) : y;
        if (s[0] > 0.f) {                                           // t' = t + up
            const float up = policy_t<SUB>(m[0], y) - policy_t<SUB>(m[0], z), f = __builtin_amdgcn_exp2f(up);
            // (no finite reference logit yet: s[3] is infinite and stays it)
            const float upr = EXACT && m[1] > PL_LOWEST ? policy_t<SUB>(m[1], yr) - policy_t<SUB>(m[1], zr) : 0.f;
            if (EXACT) s[3] = times(f, __builtin_fmaf(s[0], up - upr, s[3]));
            s[1] = times(f, __builtin_fmaf(s[0], up, s[1]));
            s[0] = times(f, s[0]);
        }
        if (EXACT && s[2] > 0.f) s[2] *= __builtin_amdgcn_exp2f(policy_t<SUB>(m[1], yr) - policy_t<SUB>(m[1], zr));
        z = y; zr = yr;
        m[0] = n[0]; m[1] = n[1];
    }
};

__device__ __forceinline__ double lanes_sum_f64(double v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// A row in the registers of LANES lanes, CH pieces of 16 bytes per lane: it is read once, all lanes wait for nothing but the row's
// maximum and its sums. LANES < 64: several rows per wave, side by side, no LDS. Bound by memory from rows of about 500 logits on
// (16288 rows of 4001 fp32 logits with a reference, a fifth of them not effective: 147 us, 4.6 TB/s), below by the row's scalars (512 rows of
// 64: 5.2 us, 32768: 7.1), where lanes that share a row all compute them.
template <class T, bool EXACT, int LANES, int CH>
__global__ void __launch_bounds__(LANES > 64 ? LANES : PL_BLOCK, LANES == 512 ? 4 : 1)
k_policy_held(PolicyArgs q, PolicyScalars pc, double w_all, const double *__restrict__ w_in, double *__restrict__ partial)
{
    using P = PolicyPiece<T, EXACT, false>;
    constexpr int V = P::V, BLOCK = LANES > 64 ? LANES : PL_BLOCK, ROWS = BLOCK / LANES;
    __shared__ float s_max[2][16], s_sum[5][16];
    __shared__ double s_part[ROWS][4];                              // a group's share of the means, its first lane's alone
    __shared__ PolicyShares few;
    if (q.eff && !w_in) policy_count<BLOCK>(q, few);
    const int tid = threadIdx.x, lane = tid % LANES, A = q.A;
    double *const sum = s_part[tid / LANES];
    if (lane == 0) sum[0] = sum[1] = sum[2] = sum[3] = 0.0;
    const float k = (float)pc.inv_temp * PL_LOG2E;
    const int rows = q.B * q.G * q.T, used = (q.pieces + LANES - 1) / LANES;     // pieces per lane
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < rows; first += (int64_t)gridDim.x * ROWS) {
        const int64_t at = first + tid / LANES;
        const bool there = at < rows;                               // (the same for all lanes of a row, as live is)
        const int row = (int)(there ? at : rows - 1);
        const double w = there ? policy_weight(q, row, w_all, w_in, few) : 0.0;
        const bool live = w != 0.0;
        if (LANES >= 64 && !live) {                                 // the whole row's lanes: nothing to read or to compute
            if (there && lane == 0 && q.logp) q.logp[row] = 0.f;
            if (there && q.grad) policy_clear((T *)q.grad + (int64_t)row * q.grad_ld, A, lane, LANES);
            continue;
        }
        const T *const x = (const T *)q.logits + (int64_t)row * q.ld, *const y = EXACT ? (const T *)q.ref_logits + (int64_t)row * q.ref_ld : nullptr;
        const int mis = policy_mis(x);
        uint4 rx[CH], ry[EXACT ? CH : 1];
        auto pieces = [&](auto f) {                                 // f(piece, its first element), all of them in registers
            static_for<CH>([&](auto c) {
                if (c < used) f(c, ((int)c * LANES + lane) * V - mis);
                if (CH * (EXACT ? 2 : 1) > 8) __builtin_amdgcn_sched_barrier(0);       // (not all pieces' elements at once)
            });
        };
        pieces([&](auto c, int j) {
            const bool in = live && j < A;
            rx[c] = in ? policy_load<(LANES * CH > 16)>(x, j, A) : policy_none<T>();
            if (EXACT) ry[EXACT ? (int)c : 0] = in ? policy_load<(LANES * CH > 16)>(y, j, A) : policy_none<T>();
        });
        PolicyRow r{};
        if (live) r = policy_inputs(q, row, w, lane == 0);
        pieces([&](auto c, int j) {
            if (live && j < A) {
                rx[c] = policy_cut<(LANES * CH > 16), T>(rx[c], j, A);
                if (EXACT) ry[EXACT ? (int)c : 0] = policy_cut<(LANES * CH > 16), T>(ry[EXACT ? (int)c : 0], j, A);
            }
        });
        float m[2] = {PL_LOWEST, PL_LOWEST}, s[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
        pieces([&](auto c, int j) { P::max(rx[c], ry[EXACT ? (int)c : 0], r.a - j, m, s[4]); });
        reduce_some<LANES, EXACT, 2>(m, OpMaxF(), s_max);
        const float top = m[0];
        const bool far = live && policy_is_far(m[0], k), far_ref = EXACT && live && policy_is_far(m[1], k);
        if (__any(far || far_ref)) {
            pieces([&](auto c, int) {
                if (far) rx[c] = policy_centred<T>(rx[c], m[0]);
                if (EXACT && far_ref) ry[EXACT ? (int)c : 0] = policy_centred<T>(ry[EXACT ? (int)c : 0], m[1]);
            });
            m[0] = far ? 0.f : m[0];
            m[1] = far_ref ? 0.f : m[1];
        }
        PolicyScale z = policy_scale<false>(m[0], k), zr = EXACT ? policy_scale<false>(m[1], k) : z;
        pieces([&](auto c, int) { P::sums(rx[c], ry[EXACT ? (int)c : 0], z, zr, s); });
        reduce_some<LANES, EXACT, 5>(s, OpAddF(), s_sum);
        PolicyCoef c = policy_row(pc, r, PolicySums{s[0], s[2], s[1], s[3], s[4]}, top, policy_t<false>(m[0], z), q.old_logp != nullptr,
                                  q.ref_logp != nullptr, EXACT);
        if (s[0] != s[0]) z.c = NAN;                                // (no distribution: no element's 2^t is 0)
        const bool dead = !live || s[0] == 0.f;                     // not an effective step, or no action allowed
        if (dead) { c = PolicyCoef{}; c.logp = live ? -INFINITY : 0.f; }
        if (there && lane == 0) {
            if (q.logp) q.logp[row] = c.logp;
            sum[0] += w * (double)c.pg;
            sum[1] += w * (double)c.kl;
            sum[2] += w * (double)c.ent;
            sum[3] += w * (double)c.clipped;
        }
        if (there && q.grad) {
            T *const d = (T *)q.grad + (int64_t)row * q.grad_ld;
            pieces([&](auto i, int j) {
                float o[V];
                P::grad(rx[i], ry[EXACT ? (int)i : 0], z, zr, c, r.a - j, o);
                if (j < A) policy_put(d, o, j, A);
            });
        }
    }
    __syncthreads();
    if (tid < 64) {                                                 // sixteen lanes per sum, in a fixed order
        double v = 0.0;
#pragma unroll
        for (int i = 0; i < (ROWS + 15) / 16; ++i) if (const int g = 16 * i + (tid >> 2); g < ROWS) v += s_part[g][tid & 3];
#pragma unroll
        for (int o = 4; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
        if (tid < 4) partial[4 * (int64_t)blockIdx.x + tid] = v;
    }
}

// A row in the registers of half a CU or a whole one, CH pieces per lane of 512 or 1024: too large for the other workgroups that would
// work while this one waits for memory, so each piece of the next row is requested as soon as this row's gradient has left its
// registers, and the sums start with the pieces that are there. Workgroups take rows in turn. 2664 rows of 128256 bf16 logits: 300 us, 4.6
// TB/s; vector instructions fill 166 of them, and nothing is under way while the last pieces arrive and the row's sums are folded.
template <class T, bool EXACT, int BLOCK, int CH>
__global__ void __launch_bounds__(BLOCK, 4)
k_policy_ring(PolicyArgs q, PolicyScalars pc, double w_all, const double *__restrict__ w_in, double *__restrict__ partial)
{
    using P = PolicyPiece<T, EXACT, false>;
    constexpr int V = P::V, GROUP = EXACT ? 1 : 2;                  // pieces between two looks at the maximum
    __shared__ float s_max[2][16], s_sum[5][16];
    __shared__ PolicyShares few;
    if (q.eff && !w_in) policy_count<BLOCK>(q, few);
    const int tid = threadIdx.x, A = q.A;
    const float k = (float)pc.inv_temp * PL_LOG2E;
    const int rows = q.B * q.G * q.T, used = (q.pieces + BLOCK - 1) / BLOCK;
    __shared__ double sum[4];                                       // the first lane's alone
    if (tid == 0) sum[0] = sum[1] = sum[2] = sum[3] = 0.0;
    uint4 rx[CH], ry[EXACT ? CH : 1];
    const T *x = nullptr, *y = nullptr;                             // the row that is being loaded
    int mis = 0;
    bool live = false;
    double w = 0.0;
    auto start = [&](int64_t row) {
        w = row < rows ? uniform(policy_weight(q, (int)row, w_all, w_in, few)) : 0.0;
        live = w != 0.0;
        if (!live) return;
        x = (const T *)q.logits + row * q.ld;
        y = EXACT ? (const T *)q.ref_logits + row * q.ref_ld : nullptr;
        mis = policy_mis(x);
    };
    auto request = [&](auto i) {
        const int j = ((int)i * BLOCK + tid) * V - mis;
        rx[i] = live && j < A ? policy_cut<true, T>(policy_load<true>(x, j, A), j, A) : policy_none<T>();
        if (EXACT) ry[EXACT ? (int)i : 0] = live && j < A ? policy_cut<true, T>(policy_load<true>(y, j, A), j, A) : policy_none<T>();
    };
    start(blockIdx.x);
    static_for<CH>([&](auto i) { if (i < used) request(i); });
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const double w_row = w;
        const bool live_row = live;
        const int mis_row = mis;
        PolicyRow r{};
        if (live_row) r = policy_inputs(q, (int)row, w_row, tid == 0);
        // A row that does not count is -inf throughout and takes the same way: a branch around it would make every load that is
        // under way wait at its end (313 -> 412 us for 2664 rows of 128256 bf16 logits).
        PolicyRunning<EXACT, false> u(k);
        float xa = 0.f, top;
        for (bool centred = false;; centred = true) {               // twice where the maximum is far from 0
            static_for<(CH + GROUP - 1) / GROUP>([&](auto g) {
                if (g * GROUP < used) {
                    float n[2] = {u.m[0], u.m[1]};
                    static_for<GROUP>([&](auto e) {
                        constexpr int i = decltype(g)::value * GROUP + decltype(e)::value;
                        const int j = (i * BLOCK + tid) * V - mis_row;
                        if (i < used) P::max(rx[i], ry[EXACT ? i : 0], centred ? -1 : r.a - j, n, xa);
                    });
                    u.turn(n);
                    static_for<GROUP>([&](auto e) {
                        constexpr int i = decltype(g)::value * GROUP + decltype(e)::value;
                        if (i < used) P::sums(rx[i], ry[EXACT ? i : 0], u.z, u.zr, u.s);
                    });
                }
                __builtin_amdgcn_sched_barrier(0);                  // (all groups' elements at once do not fit the registers)
            });
            float n[2] = {u.m[0], u.m[1]};
            reduce_some<BLOCK, EXACT, 2>(n, OpMaxF(), s_max);
            if (!centred) top = n[0];
            const bool far = live_row && policy_is_far(n[0], k), far_ref = EXACT && live_row && policy_is_far(n[1], k);
            if (centred || !(far || far_ref)) { u.turn(n); break; }
            static_for<CH>([&](auto i) {
                if (i < used) {
                    if (far) rx[i] = policy_centred<T>(rx[i], n[0]);
                    if (EXACT && far_ref) ry[EXACT ? (int)i : 0] = policy_centred<T>(ry[EXACT ? (int)i : 0], n[1]);
                }
            });
            u = PolicyRunning<EXACT, false>(k);
            __syncthreads();                                        // (s_max is written again without another use of s_sum between)
        }
        u.s[4] = xa;
        reduce_some<BLOCK, EXACT, 5>(u.s, OpAddF(), s_sum);
        PolicyCoef c = policy_row(pc, r, PolicySums{u.s[0], u.s[2], u.s[1], u.s[3], u.s[4]}, top, policy_t<false>(u.m[0], u.z),
                                  q.old_logp != nullptr, q.ref_logp != nullptr, EXACT);
        PolicyScale z = u.z;
        if (u.s[0] != u.s[0]) z.c = NAN;
        if (!live_row || u.s[0] == 0.f) { c = PolicyCoef{}; c.logp = live_row ? -INFINITY : 0.f; }
        if (tid == 0) {
            if (q.logp) q.logp[row] = c.logp;
            sum[0] += w_row * (double)c.pg;
            sum[1] += w_row * (double)c.kl;
            sum[2] += w_row * (double)c.ent;
            sum[3] += w_row * (double)c.clipped;
        }
        T *const d = q.grad ? (T *)q.grad + row * q.grad_ld : nullptr;
        start(row + gridDim.x);
        static_for<CH>([&](auto i) {
            if (i < used) {
                if (d) {
                    const int j = ((int)i * BLOCK + tid) * V - mis_row;
                    float o[V];
                    P::grad(rx[i], ry[EXACT ? (int)i : 0], z, u.zr, c, r.a - j, o);
                    if (j < A) policy_put(d, o, j, A);
                }
                request(i);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    }
    if (tid == 0)
        for (int i = 0; i < 4; ++i) partial[4 * (int64_t)blockIdx.x + i] = sum[i];
}

// A row that does not fit: one workgroup, two sweeps. The first keeps a running maximum per lane, its sums scaled anew where the
// maximum of the next CH pieces is larger; the second reads the row again, from the caches where the rows in flight fit them.
template <class T, bool EXACT, int BLOCK, int CH>
__global__ void __launch_bounds__(BLOCK, BLOCK == 512 ? 5 : 1)
k_policy_stream(PolicyArgs q, PolicyScalars pc, double w_all, const double *__restrict__ w_in, double *__restrict__ partial)
{
    using P = PolicyPiece<T, EXACT, true>;
    constexpr int V = P::V;
    __shared__ float s_max[2][16], s_sum[5][16];
    __shared__ PolicyShares few;
    if (q.eff && !w_in) policy_count<BLOCK>(q, few);
    const int tid = threadIdx.x, A = q.A;
    const float k = (float)pc.inv_temp * PL_LOG2E;
    const int rows = q.B * q.G * q.T;
    __shared__ double sum[4];                                       // the first lane's alone
    if (tid == 0) sum[0] = sum[1] = sum[2] = sum[3] = 0.0;
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
        const double w = uniform(policy_weight(q, row, w_all, w_in, few));
        T *const d = q.grad ? (T *)q.grad + (int64_t)row * q.grad_ld : nullptr;
        const T *const x = (const T *)q.logits + (int64_t)row * q.ld, *const y = EXACT ? (const T *)q.ref_logits + (int64_t)row * q.ref_ld : nullptr;
        const int mis = policy_mis(x);
        if (w == 0.0) {
            if (tid == 0 && q.logp) q.logp[row] = 0.f;
            if (d) policy_clear(d, A, tid, BLOCK);
            continue;
        }
        const PolicyRow r = policy_inputs(q, row, w, tid == 0);
        auto piece = [&](const T *v, int j) { return j < A ? policy_load<true>(v, j, A) : policy_none<T>(); };
        auto cut = [&](uint4 (&r)[CH], int j0) {
#pragma unroll
            for (int c = 0; c < CH; ++c) if (const int j = j0 + c * BLOCK * V; j < A) r[c] = policy_cut<true, T>(r[c], j, A);
        };
        PolicyRunning<EXACT, true> u(k);
        float xa = 0.f;
        for (int j0 = tid * V - mis; j0 < A; j0 += CH * BLOCK * V) {
            uint4 rx[CH], ry[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int j = j0 + c * BLOCK * V;
                rx[c] = piece(x, j);
                if (EXACT) ry[c] = piece(y, j);
            }
            cut(rx, j0);
            if (EXACT) cut(ry, j0);
            float n[2] = {u.m[0], u.m[1]};
#pragma unroll
            for (int c = 0; c < CH; ++c) P::max(rx[c], ry[c], r.a - (j0 + c * BLOCK * V), n, xa);
            u.turn(n);
#pragma unroll
            for (int c = 0; c < CH; ++c) P::sums(rx[c], ry[c], u.z, u.zr, u.s);
        }
        float top[2] = {u.m[0], u.m[1]};
        reduce_some<BLOCK, EXACT, 2>(top, OpMaxF(), s_max);
        u.turn(top);
        u.s[4] = xa;
        reduce_some<BLOCK, EXACT, 5>(u.s, OpAddF(), s_sum);
        PolicyCoef c = policy_row(pc, r, PolicySums{u.s[0], u.s[2], u.s[1], u.s[3], u.s[4]}, u.m[0], 0.f, q.old_logp != nullptr, q.ref_logp != nullptr, EXACT);
        if (u.s[0] != u.s[0]) u.z.c = NAN;
        const bool dead = u.s[0] == 0.f;                            // no action allowed
        if (dead) { c = PolicyCoef{}; c.logp = -INFINITY; }
        if (tid == 0) {
            if (q.logp) q.logp[row] = c.logp;
            sum[0] += w * (double)c.pg;
            sum[1] += w * (double)c.kl;
            sum[2] += w * (double)c.ent;
            sum[3] += w * (double)c.clipped;
        }
        if (d)
            for (int j0 = tid * V - mis; j0 < A; j0 += CH * BLOCK * V) {
                uint4 rx[CH], ry[CH];
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const int j = j0 + i * BLOCK * V;
                    rx[i] = dead ? policy_none<T>() : piece(x, j);
                    if (EXACT) ry[i] = dead ? policy_none<T>() : piece(y, j);
                }
                if (!dead) {
                    cut(rx, j0);
                    if (EXACT) cut(ry, j0);
                }
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const int j = j0 + i * BLOCK * V;
                    float o[V];
                    P::grad(rx[i], ry[i], u.z, u.zr, c, r.a - j, o);
                    if (j < A) policy_put(d, o, j, A);
                }
            }
    }
    if (tid == 0)
        for (int i = 0; i < 4; ++i) partial[4 * (int64_t)blockIdx.x + i] = sum[i];
}

// The workgroups' sums in a fixed order; stats: policy term, KL, entropy, clipped share. Latency: 2.2 us for a minibatch's 8 partial sums,
// 4.0 for 2048 (1024 threads: 3.6 and 4.0).
constexpr int PL_FINISH = 256;
__global__ void __launch_bounds__(PL_FINISH)
k_policy_finish(const double *__restrict__ partial, int n, PolicyScalars pc, float *__restrict__ loss, float *__restrict__ stats)
{
    __shared__ double red[PL_FINISH / 64][4];
    double v[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += PL_FINISH)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += partial[4 * i + e];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = lanes_sum_f64(v[e]);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6][e] = v[e];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = 0.0;
#pragma unroll
            for (int i = 0; i < PL_FINISH / 64; ++i) v[e] += red[i][e];
        }
        *loss = (float)(pc.scale * (v[0] + (pc.kl > 0.0 ? pc.kl * v[1] : 0.0) - pc.ent * v[2]));
        if (stats)
#pragma unroll
            for (int e = 0; e < 4; ++e) stats[e] = (float)v[e];
    }
}

// The row's kernel by its number of 16-byte pieces. Rows of up to 64 KB (32 of bf16 with a reference) stay in the registers of as few lanes as
// hold them at up to 8 pieces each (6 or less leave room for another wave), so that many rows are under way per CU and few lanes repeat a
// row's scalars; the number of rows has no say, so that a row's result does not depend on it. Longer ones fill the registers of a CU by
// one or two, and load ahead (k_policy_ring); what does not fit is read twice. Measured, 200 M logits (bytes read and written / time, of
// 5.06 TB/s that a copy of 1 GiB reaches):
//   8 bf16 logits: a lane per row 2.5 TB/s, 8 lanes 0.4;  64: 4 lanes x 2 pieces 3.8, 8 x 1 2.7;  320: 8 x 6 4.5, 16 x 4 3.8;  4200: 128 x 6
//   4.0, 256 x 4 3.3;  32 fp32: 4 x 2 4.0, 8 x 1 2.9, 2 x 4 3.6 (64 fp32, 4 x 4 against 8 x 2: 512 rows, all latency, 5.2 us and 4.4, 3.1 M rows 333 and 374)
//   4096 bf16 logits: 64 lanes x 8 pieces 4.8, 256 x 4 (two pieces each, two barriers per row) 3.6
//   32768 bf16: 512 x 8 4.7, two sweeps 3.7;  65536 bf16: ring of 512 4.7, one workgroup of 1024 without loading ahead 3.8, two sweeps 3.7
//   128256 bf16: ring of 1024 4.0 (4.4 where rows fill the CUs evenly), not loading ahead 3.2, two sweeps 3.6
//   32000 fp32: ring 5.1, two sweeps 4.2;  32000 fp32 with a reference: ring 4.8, two sweeps 3.3
// bf16 with a reference is bound by its arithmetic (two exponentials, 35 instructions per pair): from 32 KB on two sweeps by two
// workgroups per CU reach 3.4-3.8 TB/s, the ring, which spills there, 2.9.
template <class T, bool EXACT>
static int launch_rows(const PolicyArgs &q, const PolicyScalars &pc, double w_all, const double *w, double *partial, int rows, hipStream_t st)
{
    constexpr bool HEAVY = EXACT && sizeof(T) == 2;
    const int64_t pieces = q.pieces;
    int grid = 0;
    auto go = [&](auto kern, int block, int per) {
        const int64_t n = ((int64_t)rows + per - 1) / per;
        grid = (int)(n < PL_GRID ? n : PL_GRID);
        hipLaunchKernelGGL(kern, dim3(grid), dim3(block), 0, st, q, pc, w_all, w, partial);
    };
    auto held = [&](auto lanes, auto ch) {
        constexpr int L = decltype(lanes)::value, C = decltype(ch)::value, BLOCK = L > 64 ? L : PL_BLOCK;
        go(k_policy_held<T, EXACT, L, C>, BLOCK, BLOCK / L);
    };
    auto ring = [&](auto block, auto ch) {                          // as many workgroups as fit the chip: 16 waves per CU
        constexpr int BLOCK = decltype(block)::value;
        const int cus = device_cus(), fit = (cus > 0 ? cus : 256) * (1024 / BLOCK);
        grid = rows < fit ? rows : fit < PL_GRID ? fit : PL_GRID;
        hipLaunchKernelGGL((k_policy_ring<T, EXACT, BLOCK, decltype(ch)::value>), dim3(grid), dim3(BLOCK), 0, st, q, pc, w_all, w, partial);
    };
#define N(n) std::integral_constant<int, n>{}
    if (pieces <= 1) held(N(1), N(1));
    else if (pieces <= 2) held(N(1), N(2));
    else if (pieces <= 4) held(N(2), N(2));
    else if (pieces <= 8) held(N(4), N(2));
    else if (pieces <= 16) held(N(4), N(4));
    else if (pieces <= 32) held(N(8), N(4));
    else if (pieces <= 48) held(N(8), N(6));
    else if (pieces <= 64) held(N(8), N(8));
    else if (pieces <= 96) held(N(16), N(6));
    else if (pieces <= 128) held(N(16), N(8));
    else if (pieces <= 192) held(N(32), N(6));
    else if (pieces <= 256) held(N(32), N(8));
    else if (pieces <= 512) held(N(64), N(8));
    else if (!EXACT && pieces <= 768) { if constexpr (!EXACT) held(N(128), N(6)); }
    else if (pieces <= 1024) held(N(256), N(4));
    else if (pieces <= 2048) held(N(256), N(8));
    else if constexpr (HEAVY) go(k_policy_stream<T, EXACT, 512, 2>, 512, 1);
    else if (pieces <= 4096) held(N(512), N(8));
    else if constexpr (EXACT) {
        if (pieces <= 8192) ring(N(1024), N(8));
        else go(k_policy_stream<T, EXACT, 1024, 2>, 1024, 1);
    } else if (pieces <= 8192) ring(N(512), N(16));
    else if (pieces <= 16384) ring(N(1024), N(16));
    else go(k_policy_stream<T, EXACT, 1024, 2>, 1024, 1);
#undef N
    return grid;
}

// [partial sums][partial counts int64][weights double B][counts int32 B]
size_t policy_scratch_bytes(int B) { return (size_t)PL_GRID * (4 * sizeof(double) + sizeof(int64_t)) + (size_t)B * 12 + 64; }

void launch_policy_loss(PolicyArgs q, const PolicyCfg &g, void *scratch, hipStream_t st)
{
    // rows that may begin between two boundaries of 16 bytes touch one piece more
    const size_t es = q.dtype == 1 ? 2 : 4;
    const int64_t V = 16 / (int64_t)es;
    const bool aligned = (uintptr_t)q.logits % 16 == 0 && (q.ld % V == 0 || (int64_t)q.B * q.G * q.T == 1);
    q.pieces = (int)(((int64_t)q.A + (aligned ? 0 : V - 1) + V - 1) / V);
    q.by_schedule = g.by_schedule;
    double *partial = (double *)scratch;
    int64_t *part = (int64_t *)(partial + 4 * PL_GRID);
    double *w = (double *)(part + PL_GRID);
    int32_t *n = (int32_t *)(w + q.B);
    const PolicyScalars pc{1.0 / g.temperature, log(1.0 - g.clip_low), log(1.0 + g.clip_high), g.scale / g.temperature, g.kl_coef,
                           g.entropy_coef, g.scale, (float)(1.0 - g.clip_low), (float)(1.0 + g.clip_high)};
    const double w_all = 1.0 / ((double)q.B * q.G * q.T);           // every step counts: both means are one
    const bool few = (int64_t)q.B * q.T <= PL_FEW && q.B <= PL_INPUTS;
    if (q.eff && !few) {
        auto grid = [&](int64_t per) { const int64_t c = (q.B + per - 1) / per; return (int)(c < PL_GRID ? c : PL_GRID); };
        int parts = 0;
        auto count = [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            parts = grid(PL_BLOCK / L);
            hipLaunchKernelGGL(k_policy_count<L>, dim3(parts), dim3(PL_BLOCK), 0, st, q.eff, q.B, q.T, g.by_schedule, n, part);
        };
        if (q.T >= 512) count(std::integral_constant<int, 256>{});  // (at least two flags per lane)
        else if (q.T >= 128) count(std::integral_constant<int, 64>{});
        else if (q.T >= 16) count(std::integral_constant<int, 8>{});
        else count(std::integral_constant<int, 1>{});
        hipLaunchKernelGGL(k_policy_weights, dim3(grid(PL_BLOCK)), dim3(PL_BLOCK), 0, st, n, part, parts, q.B, q.G, g.by_schedule, w);
    } else w = nullptr;
    const int rows = q.B * q.G * q.T;
    const int grid = q.dtype == 1 ? (q.ref_logits ? launch_rows<bf16_t, true>(q, pc, w_all, w, partial, rows, st)
                                                  : launch_rows<bf16_t, false>(q, pc, w_all, w, partial, rows, st))
                                  : (q.ref_logits ? launch_rows<float, true>(q, pc, w_all, w, partial, rows, st)
                                                  : launch_rows<float, false>(q, pc, w_all, w, partial, rows, st));
    hipLaunchKernelGGL(k_policy_finish, dim3(1), dim3(PL_FINISH), 0, st, partial, grid, pc, q.loss, q.stats);
}

}  // namespace sol
