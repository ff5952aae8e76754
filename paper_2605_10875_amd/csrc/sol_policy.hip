// Clipped policy loss over the actions of a likelihood pass, forward and gradient in one call (the update that the advantages of
// sol_reward.hip are made for). Per row (input b, schedule g, step t) of logits x_j, with z = x / temperature:
//   logp_j = z_j - log sum exp z, p_j = exp(logp_j), a the action taken, d = logp_a - old, rho = exp(d)
//   pg = -min(rho A, clip(rho, 1 - lo, 1 + hi) A),  H = -sum p_j logp_j
//   KL = exp(u) - u - 1 with u = ref - logp_a (estimate), or sum p_j (logp_j - logq_j) (exact, from reference logits y_j)
//   loss = scale * sum w (pg + beta KL - c H), w the row's share in the mean
// With the row's maximum m, e_j = 2^(t_j), t_j = (x_j - m) log2(e) / temperature, S = sum e_j, U = sum e_j t_j and, with a
// reference, t'_j, S' likewise and K = sum e_j (t_j - t'_j):
//   H = log S - ln2 U / S,  KL = ln2 K / S - (log S - log S')
//   d loss / d x_j = p_j (alpha + gamma t_j + kappa (t_j - t'_j)) + [j = a] w' G
// where w' = w scale / temperature, G = d(pg + beta KL) / d logp_a, gamma = w' c ln2, kappa = w' beta ln2 and
// alpha = -w' (G + c ln2 U / S + beta ln2 K / S): the row needs its sums once, then every element's gradient by itself.
#include "sol_internal.h"

namespace sol {

constexpr int PL_BLOCK = 256;
constexpr int PL_GRID = 2048;                                       // workgroups of the rows' kernel at most
constexpr float PL_LOG2E = 1.44269504088896341f;
constexpr double PL_LN2 = 0.693147180559945309;

struct PolicyScalars { double inv_temp, log_lo, log_hi, lo, hi, kl, ent, scale; };

// what a row needs besides its sums
struct PolicyRow { int a; float adv, old, ref; double w; };
struct PolicySums { double S, Sr; float U, K, ln_diff; };
struct PolicyCoef { float alpha, gamma, kappa, hot, logp, pg, kl, ent, clipped; };

// w[b] = share of an effective step of input b in the mean (0: the input has none)
__global__ void __launch_bounds__(PL_BLOCK)
k_policy_count(const int32_t *__restrict__ eff, int T, int32_t *__restrict__ n)
{
    const int lane = threadIdx.x & 63, b = blockIdx.x;
    __shared__ int red[PL_BLOCK / 64];
    int c = 0;
    for (int t = threadIdx.x; t < T; t += PL_BLOCK) c += eff[(int64_t)b * T + t] != 0;
    c = wave_sum_i(c);
    if (lane == 0) red[threadIdx.x >> 6] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < PL_BLOCK / 64; ++i) c += red[i];
        n[b] = c;
    }
}
__global__ void __launch_bounds__(PL_BLOCK)
k_policy_weights(const int32_t *__restrict__ n, int B, int G, int by_schedule, double *__restrict__ w)
{
    __shared__ int64_t red[PL_BLOCK];
    int64_t c = 0;
    for (int b = threadIdx.x; b < B; b += PL_BLOCK) c += by_schedule ? n[b] > 0 : n[b];
    red[threadIdx.x] = c;
    __syncthreads();
    for (int o = PL_BLOCK / 2; o > 0; o >>= 1) {
        if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
        __syncthreads();
    }
    const double all = (double)red[0] * (double)G;
    for (int b = threadIdx.x; b < B; b += PL_BLOCK)
        w[b] = n[b] == 0 ? 0.0 : by_schedule ? 1.0 / ((double)n[b] * all) : 1.0 / all;
}

// exp(u) - u - 1: by its series near 0, where the difference would keep a few bits only (|u| < 0.5: the first term left out
// is below 2^-33 of the sum)
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
    return fabsf(u) < 0.5f ? s * u * u : expf(u) - u - 1.f;
}

// The row's loss terms and the coefficients of its gradient from its sums. xa: the taken action's logit minus the maximum.
// The ratio's bounds are tested on the logarithm in 64 bits: a gradient is not continuous there.
__device__ __forceinline__ PolicyCoef policy_row(const PolicyScalars &pc, const PolicyRow &r, const PolicySums &s, float xa,
                                                 bool has_old, bool has_ref, bool exact_kl)
{
    PolicyCoef c;
    const double logS = log(s.S), logp = (double)xa * pc.inv_temp - logS;
    const double d = has_old ? logp - (double)r.old : 0.0;
    const float A = r.adv, rho = expf((float)d);
    const bool clipped = (A > 0.f && d > pc.log_hi) || (A < 0.f && d < pc.log_lo);
    c.logp = (float)logp;
    c.pg = clipped ? -(A > 0.f ? (float)pc.hi : (float)pc.lo) * A : -rho * A;
    float G = clipped ? 0.f : -rho * A;
    const float beta = (float)pc.kl, ln2 = (float)PL_LN2, inv = (float)(1.0 / s.S), u_mean = ln2 * s.U * inv;
    c.ent = (float)(logS - (double)u_mean);
    c.kl = 0.f;
    float k_mean = 0.f;
    if (exact_kl) {
        k_mean = ln2 * s.K * inv;
        c.kl = (float)((double)k_mean - (logS - log(s.Sr)));
    } else if (has_ref) {
        const float u = (float)((double)r.ref - logp);
        c.kl = policy_kl(u);
        G -= beta * (u + c.kl);                                     // 1 - exp(u)
    }
    c.clipped = clipped ? 1.f : 0.f;
    const double wt = r.w * pc.scale * pc.inv_temp;
    const float w = (float)wt, ent = (float)pc.ent;
    c.hot = w * G;
    c.alpha = -w * (G + ent * u_mean + (exact_kl ? beta * k_mean : 0.f)) * inv;
    c.gamma = w * ent * ln2 * inv;
    c.kappa = exact_kl ? w * beta * ln2 * inv : 0.f;
    return c;
}

// One workgroup per row, rows strided over the grid. Three passes over the row: maximum, sums, gradient.
template <class T, bool EXACT>
__global__ void __launch_bounds__(PL_BLOCK)
k_policy_rows(PolicyArgs q, PolicyScalars pc, double w_all, const double *__restrict__ w_in, double *__restrict__ partial)
{
    __shared__ float red[PL_BLOCK / 64];
    const T *const X = (const T *)q.logits, *const Y = (const T *)q.ref_logits;
    T *const D = (T *)q.grad;
    const int tid = threadIdx.x, A = q.A;
    const float k = (float)(pc.inv_temp) * PL_LOG2E;
    const int rows = q.B * q.G * q.T;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
        const int b = row / (q.G * q.T), t = row % q.T;
        const double w = !q.eff ? w_all : q.eff[(int64_t)b * q.T + t] ? w_in[b] : 0.0;
        T *const dst = D ? D + (int64_t)row * q.grad_ld : nullptr;
        if (w == 0.0) {                                             // not an effective step: the row is not read
            if (dst) for (int j = tid; j < A; j += PL_BLOCK) st(dst + j, 0.f);
            if (tid == 0 && q.logp) q.logp[row] = 0.f;
            continue;
        }
        const T *const x = X + (int64_t)row * q.ld, *const y = EXACT ? Y + (int64_t)row * q.ref_ld : nullptr;
        float m = -3.402823466e38f, mr = -3.402823466e38f;
        for (int j = tid; j < A; j += PL_BLOCK) {
            m = fmaxf(m, ld(x + j));
            if (EXACT) mr = fmaxf(mr, ld(y + j));
        }
        m = block_max<PL_BLOCK>(m, red);
        if (EXACT) mr = block_max<PL_BLOCK>(mr, red);
        float S = 0.f, U = 0.f, Sr = 0.f, K = 0.f;
        for (int j = tid; j < A; j += PL_BLOCK) {
            const float tj = (ld(x + j) - m) * k, e = exp2f(tj);
            S += e;
            U += e * fmaxf(tj, -1e4f);                              // 0 log 0 = 0
            if (EXACT) {
                const float rj = (ld(y + j) - mr) * k;
                Sr += exp2f(rj);
                K += e > 0.f ? e * (tj - rj) : 0.f;
            }
        }
        PolicySums s;
        s.S = (double)block_sum<PL_BLOCK>(S, red);
        s.U = block_sum<PL_BLOCK>(U, red);
        s.Sr = EXACT ? (double)block_sum<PL_BLOCK>(Sr, red) : 1.0;
        s.K = EXACT ? block_sum<PL_BLOCK>(K, red) : 0.f;
        if (s.S == 0.0) {                                           // no action is allowed
            if (dst) for (int j = tid; j < A; j += PL_BLOCK) st(dst + j, 0.f);
            if (tid == 0 && q.logp) q.logp[row] = -INFINITY;
            continue;
        }
        PolicyRow r;
        r.a = q.ids[row];
        if (r.a < 0 || r.a >= A) { r.a = 0; if (tid == 0) atomicOr(q.flags, FLAG_BAD_ACTION); }
        r.adv = q.adv ? q.adv[row] : 0.f;
        r.old = q.old_logp ? q.old_logp[row] : 0.f;
        r.ref = q.ref_logp ? q.ref_logp[row] : 0.f;
        r.w = w;
        const PolicyCoef c = policy_row(pc, r, s, ld(x + r.a) - m, q.old_logp != nullptr, q.ref_logp != nullptr, EXACT);
        if (tid == 0) {
            if (q.logp) q.logp[row] = c.logp;
            sum[0] += w * (double)c.pg;
            sum[1] += w * (double)c.kl;
            sum[2] += w * (double)c.ent;
            sum[3] += w * (double)c.clipped;
        }
        if (dst) {
            __syncthreads();                                        // the gradient may replace the logits: x[a] has been read
            for (int j = tid; j < A; j += PL_BLOCK) {
                const float tj = (ld(x + j) - m) * k, e = exp2f(tj);
                float f = c.alpha + c.gamma * fmaxf(tj, -1e4f);
                if (EXACT) f += e > 0.f ? c.kappa * (tj - (ld(y + j) - mr) * k) : 0.f;
                st(dst + j, e * f + (j == r.a ? c.hot : 0.f));
            }
        }
    }
    if (tid == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) partial[4 * (int64_t)blockIdx.x + i] = sum[i];
}

// the workgroups' sums in a fixed order; out: policy term, KL, entropy, clipped share
__global__ void __launch_bounds__(PL_BLOCK)
k_policy_finish(const double *__restrict__ partial, int n, PolicyScalars pc, float *__restrict__ loss, float *__restrict__ stats)
{
    __shared__ double red[PL_BLOCK][4];
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    for (int i = threadIdx.x; i < n; i += PL_BLOCK)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += partial[4 * i + e];
#pragma unroll
    for (int e = 0; e < 4; ++e) red[threadIdx.x][e] = v[e];
    __syncthreads();
    for (int o = PL_BLOCK / 2; o > 0; o >>= 1) {
        if ((int)threadIdx.x < o)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[threadIdx.x][e] += red[threadIdx.x + o][e];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        *loss = (float)(pc.scale * (red[0][0] + pc.kl * red[0][1] - pc.ent * red[0][2]));
        if (stats)
#pragma unroll
            for (int e = 0; e < 4; ++e) stats[e] = (float)red[0][e];
    }
}

// [partial sums][counts int32 B][weights double B]
size_t policy_scratch_bytes(int B) { return (size_t)PL_GRID * 4 * sizeof(double) + (size_t)B * 16 + 64; }

void launch_policy_loss(const PolicyArgs &q, const PolicyCfg &g, void *scratch, hipStream_t st)
{
    double *partial = (double *)scratch, *w = partial + 4 * PL_GRID;
    int32_t *n = (int32_t *)(w + q.B);
    const PolicyScalars pc{1.0 / g.temperature, log(1.0 - g.clip_low), log(1.0 + g.clip_high), 1.0 - g.clip_low, 1.0 + g.clip_high,
                           g.kl_coef, g.entropy_coef, g.scale};
    const double w_all = 1.0 / ((double)q.B * q.G * q.T);           // every step counts: both means are one
    if (q.eff) {
        hipLaunchKernelGGL(k_policy_count, dim3(q.B), dim3(PL_BLOCK), 0, st, q.eff, q.T, n);
        hipLaunchKernelGGL(k_policy_weights, dim3(1), dim3(PL_BLOCK), 0, st, n, q.B, q.G, g.by_schedule, w);
    }
    const int rows = q.B * q.G * q.T, grid = rows < PL_GRID ? rows : PL_GRID;
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(grid), dim3(PL_BLOCK), 0, st, q, pc, w_all, w, partial); };
    if (q.dtype == 1) { if (q.ref_logits) go(k_policy_rows<bf16_t, true>); else go(k_policy_rows<bf16_t, false>); }
    else { if (q.ref_logits) go(k_policy_rows<float, true>); else go(k_policy_rows<float, false>); }
    hipLaunchKernelGGL(k_policy_finish, dim3(1), dim3(PL_BLOCK), 0, st, partial, grid, pc, q.loss, q.stats);
}

}  // namespace sol
