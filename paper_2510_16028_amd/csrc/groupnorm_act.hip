// tao_bound_groupnorm_act, tao_bound_check_groupnorm_act: GroupNorm with an activation on channels-last features
// x[sample][pixel][channel] (operators of App. A.3), re-executed and bounded in one call.  A (sample, group) is one row of n = pixels x
// channels per group elements of the LayerNorm chain (tao_rows.hpp), which gives the mean mu, the inverse root r and coefficients with
//     |p^ - p| <= E = E_p + u (|p| + E_p),   E_p = |gamma| (K1 |d| + K0),   d = x - mu,   p = d r gamma + beta.
// The activation then moves an error of its argument by at most (second order closed: |s''| <= 1/2, |s'| <= 1.1 for SiLU s)
//     none E,   ReLU max(0, min(E, p + E)),   SiLU B = min(|s'(p)| E + E^2/4, 1.1 E), and its own roundings k (|s(p)| + B).
//
// Channels last, so a thread keeps its channels (four of them, one 16-byte load) and walks the pixels of a part of the sample: its
// sums are per channel, whatever the number of channels per group, and reach their groups in LDS.  Three passes over x, as the mean
// has to be known before the deviations: (a) sum x, sum |x|, (b) sum |d|, sum d^2, (c) the outputs; every workgroup of (b) and (c)
// adds up the parts of its groups in the same order.  Bound by the memory's rate.
#include "tao_check.hpp"
#include "tao_device.hpp"
#include "tao_host.hpp"
#include "tao_rows.hpp"

namespace tao {

struct NormArgs {
    const float* x; const float* gamma; const float* beta;
    float* y; float* tau;
    const float* y_ref; const float* claimed;
    double* part;                    // [sample][part][group][4]: sum x, sum |x|, sum |d|, sum d^2
    long positions, channels, groups, per, ldx, ldy, batch;
    long nparts;                     // of a sample: pixel parts x column blocks
    long pixels;                     // of a part of the sums
    RowConsts k;
    double silu_k;                   // silu_f / (1 - silu_f)
};
constexpr int kNormThreads = 256;

// A workgroup takes columns of at most this many vectors (512 channels, or 256 where they come one by one): the coefficients of their
// groups then fit LDS beside the check's histogram, and the workgroup's pixels lie 2 KB of contiguous memory each.
template <int VEC> constexpr int kColumns = VEC == 4 ? 128 : 256;

// A workgroup's place: column block `cb` of the channels, thread (tx, ty) = vector of the block, first pixel.
template <int THREADS, int VEC>
struct Place {
    int TX, TY, tx, ty;
    long c0, c_lo, c_hi, g_lo, g_hi;
    bool active;
    __device__ __forceinline__ Place(const NormArgs& p, long cb) {
        const long cv = p.channels / VEC, first = cb * kColumns<VEC>;
        TX = (int)min((long)kColumns<VEC>, cv - first);
        TY = THREADS / TX;
        ty = threadIdx.x / TX; tx = threadIdx.x - ty * TX;
        active = ty < TY;
        c_lo = first * VEC; c_hi = c_lo + (long)TX * VEC;
        c0 = c_lo + (long)tx * VEC;
        g_lo = c_lo / p.per; g_hi = (c_hi - 1) / p.per + 1;
    }
};
template <int VEC>
__host__ __device__ inline long column_blocks(long channels) { return (channels / VEC + kColumns<VEC> - 1) / kColumns<VEC>; }

template <int VEC>
__device__ __forceinline__ void load_channels(const float* __restrict__ p, float (&v)[VEC]) {
    if constexpr (VEC == 4) {
        const float4 t = *reinterpret_cast<const float4*>(p);
        v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
    } else {
        v[0] = *p;
    }
}

// Sums of the block's channels (two per channel, v[c][i] of this thread) to sums of its groups, into two of the four values that each
// group has of this part; groups without a channel here get 0.  smem: 2 THREADS VEC doubles.
template <int THREADS, int VEC, int LANES>
__device__ __forceinline__ void store_groups(const NormArgs& p, const Place<THREADS, VEC>& at, const double* smem, double* out) {
    constexpr int STEPS = LANES == 1 ? 0 : LANES == 4 ? 2 : LANES == 16 ? 4 : 6;
    const int sub = threadIdx.x % LANES;
    const long trips = (p.groups + THREADS / LANES - 1) / (THREADS / LANES);
    for (long t = 0; t < trips; ++t) {
        const long g = t * (THREADS / LANES) + threadIdx.x / LANES;
        const long lo = max(g * p.per, at.c_lo), hi = min((g + 1) * p.per, at.c_hi);
        double s[2] = {0.0, 0.0};
        for (long c = lo + sub; c < hi; c += LANES) { s[0] += smem[(c - at.c_lo) * 2]; s[1] += smem[(c - at.c_lo) * 2 + 1]; }
        if constexpr (LANES > 1) {
#pragma unroll
            for (int i = 0; i < 2; ++i) s[i] = wave_all<0, STEPS>(s[i], [](double a, double b) { return a + b; });
        }
        if (sub == 0 && g < p.groups) { out[g * 4] = s[0]; out[g * 4 + 1] = s[1]; }
    }
}
template <int THREADS, int VEC>
__device__ __forceinline__ void channel_sums(const NormArgs& p, const Place<THREADS, VEC>& at, const double (&v)[VEC][2], double* smem, double* out) {
    const int width = at.TX * VEC;                           // [ty][channel][2]
    if (at.active) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
            double* o = smem + ((long)at.ty * width + at.tx * VEC + c) * 2;
            o[0] = v[c][0]; o[1] = v[c][1];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * width; i += THREADS) {
        double s = smem[i];
        for (int t = 1; t < at.TY; ++t) s += smem[(long)t * 2 * width + i];
        smem[i] = s;
    }
    __syncthreads();
    if (p.per <= 8)        store_groups<THREADS, VEC, 1>(p, at, smem, out);
    else if (p.per <= 32)  store_groups<THREADS, VEC, 4>(p, at, smem, out);
    else if (p.per <= 128) store_groups<THREADS, VEC, 16>(p, at, smem, out);
    else                   store_groups<THREADS, VEC, 64>(p, at, smem, out);
}
// Totals over a sample's parts of values FIRST .. FIRST + COUNT - 1 of the block's groups, handed to use(group, totals) by one thread
// each (kNormThreads threads at most take part).  smem: kNormThreads COUNT doubles.
template <int COUNT, class Use>
__device__ __forceinline__ void group_totals(const NormArgs& p, long s, long g_lo, long g_hi, double* smem, Use&& use) {
    const long ng = g_hi - g_lo;
    const double* part = p.part + s * p.nparts * p.groups * 4;
    const int width = (int)min(ng, (long)kNormThreads), slices = kNormThreads / width;
    const int slice = threadIdx.x / width, col = threadIdx.x - slice * width;
    for (long base = 0; base < ng; base += width) {
        const bool mine = slice < slices && base + col < ng;
        double t[COUNT] = {};
        if (mine) {
            for (long i = slice; i < p.nparts; i += slices) {
                const double* v = part + (i * p.groups + g_lo + base + col) * 4;
#pragma unroll
                for (int j = 0; j < COUNT; ++j) t[j] += v[j];
            }
#pragma unroll
            for (int j = 0; j < COUNT; ++j) smem[(slice * width + col) * COUNT + j] = t[j];
        }
        __syncthreads();
        if (slice == 0 && mine) {
            for (int i = 1; i < slices; ++i)
#pragma unroll
                for (int j = 0; j < COUNT; ++j) t[j] += smem[(i * width + col) * COUNT + j];
            use(base + col, t);
        }
        __syncthreads();
    }
}

// (a) sum x, sum |x| of a part
template <int VEC>
__global__ __launch_bounds__(kNormThreads) void norm_sums_a(NormArgs p) {
    __shared__ double smem[2 * kNormThreads * VEC];
    const long ncb = column_blocks<VEC>(p.channels);
    const long s = blockIdx.x / p.nparts, part = blockIdx.x - s * p.nparts;
    const Place<kNormThreads, VEC> at(p, part % ncb);
    const long p0 = part / ncb * p.pixels, p1 = min(p0 + p.pixels, p.positions);
    double v[VEC][2] = {};
    if (at.active) {
        const float* x = p.x + s * p.positions * p.ldx + at.c0;
#pragma unroll 4
        for (long i = p0 + at.ty; i < p1; i += at.TY) {
            float e[VEC];
            load_channels(x + i * p.ldx, e);
#pragma unroll
            for (int c = 0; c < VEC; ++c) { v[c][0] += (double)e[c]; v[c][1] += (double)fabsf(e[c]); }
        }
    }
    channel_sums<kNormThreads, VEC>(p, at, v, smem, p.part + (s * p.nparts + part) * p.groups * 4);
}
// (b) the means from the parts of (a), then sum |d|, sum d^2
template <int VEC>
__global__ __launch_bounds__(kNormThreads) void norm_sums_b(NormArgs p) {
    __shared__ double smem[2 * kNormThreads * VEC];
    extern __shared__ double mean[];                         // of the block's groups
    const long ncb = column_blocks<VEC>(p.channels);
    const long s = blockIdx.x / p.nparts, part = blockIdx.x - s * p.nparts;
    const Place<kNormThreads, VEC> at(p, part % ncb);
    group_totals<1>(p, s, at.g_lo, at.g_hi, smem, [&](long g, const double (&t)[1]) { mean[g] = t[0] * p.k.inv_n; });
    const long p0 = part / ncb * p.pixels, p1 = min(p0 + p.pixels, p.positions);
    double v[VEC][2] = {};
    if (at.active) {
        double mu[VEC];
#pragma unroll
        for (int c = 0; c < VEC; ++c) mu[c] = mean[(at.c0 + c) / p.per - at.g_lo];
        const float* x = p.x + s * p.positions * p.ldx + at.c0;
#pragma unroll 4
        for (long i = p0 + at.ty; i < p1; i += at.TY) {
            float e[VEC];
            load_channels(x + i * p.ldx, e);
#pragma unroll
            for (int c = 0; c < VEC; ++c) {
                const double d = (double)e[c] - mu[c];
                v[c][0] += fabs(d); v[c][1] = fma(d, d, v[c][1]);
            }
        }
    }
    channel_sums<kNormThreads, VEC>(p, at, v, smem, p.part + (s * p.nparts + part) * p.groups * 4 + 2);
}

// What an element's bound takes of its group.
struct GroupCoef { double mu, r, K1, K0, m; };
__device__ __forceinline__ GroupCoef group_coef(const RowConsts& k, double n, const double (&t)[4]) {
    GroupCoef c;
    c.mu = t[0] * k.inv_n;
    const double E_mu = ((k.G * t[1]) * k.inv_n + k.cd_u * fabs(c.mu)) * k.inv1mcd;
    double amp;
    layernorm_tail(E_mu, t[2], t[3], n, k, c.K1, c.K0, amp, &c.r);
    c.m = amp > 0.0 && amp < INFINITY ? k.m * (1.0 + 2.0 * amp) : 0.0;      // (else K0 is NaN, and so is the bound)
    return c;
}
// ... and of its channel: p = d rg + b, E_p = k1 |d| + k0
struct ChannelCoef { double mu, rg, b, k1, k0; };

// Output and bound of one element.  The slacks keep an evaluation in round-to-nearest binary64 at or above the formula's value: near
// a zero of s' its relative error is large, but 2^-36 (the exponential's error many times over) of E is far below 1e-6 of the other terms.
template <int ACT>
__device__ __forceinline__ void norm_element(float x, const ChannelCoef& c, double u, double silu_k, double mul, double sub, float& y, float& tau) {
    const double d = (double)x - c.mu;
    const double p = fma(d, c.rg, c.b);
    const double ep = fma(c.k1, fabs(d), c.k0);
    const double E = fma(u, fabs(p) + ep, ep);
    if constexpr (ACT == TAO_ACT_SILU) {
        const double e = exp_neg(fabs(p));
        const double inv = 1.0 / (1.0 + e), small = e * inv;
        const double sig = p < 0.0 ? small : inv, rest = p < 0.0 ? inv : small;      // sigmoid(p), 1 - sigmoid(p)
        const double s = p * sig;
        const double slope = fabs(sig * fma(p, rest, 1.0)) + 0x1p-36;
        const double B = fmin(E * fma(0.25 + 0x1p-23, E, slope), 1.1 * E);
        y = (float)s;
        tau = up32g(E == E ? fma(silu_k, fabs(s) + B, B) : E, mul, sub);
    } else if constexpr (ACT == TAO_ACT_RELU) {
        y = p <= 0.0 ? 0.f : (float)p;
        const double t = fmin(E, fma(E, 1.0 + 0x1p-24, p));
        tau = E == E ? (t > 0.0 ? up32g(t, mul, sub) : 0.f) : (float)E;
    } else {
        y = (float)p;
        tau = up32g(E, mul, sub);
    }
}

// The prologue of the last pass: coefficients of this thread's channels, from the totals of its groups.
template <int THREADS, int VEC>
struct Channels {
    ChannelCoef c[VEC];
    double mul, sub;
    __device__ __forceinline__ Channels(const NormArgs& p, long s, const Place<THREADS, VEC>& at, GroupCoef* coef, double* smem) {
        const double n = (double)(p.per * p.positions);
        group_totals<4>(p, s, at.g_lo, at.g_hi, smem, [&](long g, const double (&t)[4]) { coef[g] = group_coef(p.k, n, t); });
        if (!at.active) return;
        double m = 0.0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const GroupCoef g = coef[(at.c0 + i) / p.per - at.g_lo];
            const double gamma = p.gamma ? (double)p.gamma[at.c0 + i] : 1.0;
            c[i] = ChannelCoef{g.mu, g.r * gamma, p.beta ? (double)p.beta[at.c0 + i] : 0.0, fabs(gamma) * g.K1, fabs(gamma) * g.K0};
            m = fmax(m, g.m);
        }
        const UpFactors up(m);
        mul = up.mul; sub = up.sub;
    }
};

// (c) outputs and bounds
template <int ACT, int VEC>
__global__ __launch_bounds__(kNormThreads) void norm_apply(NormArgs p) {
    __shared__ double smem[4 * kNormThreads];
    extern __shared__ GroupCoef coef[];
    const long ncb = column_blocks<VEC>(p.channels);
    const long s = blockIdx.x / p.nparts, part = blockIdx.x - s * p.nparts;
    const Place<kNormThreads, VEC> at(p, part % ncb);
    const Channels<kNormThreads, VEC> ch(p, s, at, coef, smem);
    if (!at.active) return;
    const long p0 = part / ncb * p.pixels, p1 = min(p0 + p.pixels, p.positions);
    const float* x = p.x + s * p.positions * p.ldx + at.c0;
    const long out = s * p.positions * p.ldy + at.c0;
#pragma unroll 2
    for (long i = p0 + at.ty; i < p1; i += at.TY) {
        float e[VEC], y[VEC], t[VEC];
        load_channels(x + i * p.ldx, e);
#pragma unroll
        for (int c = 0; c < VEC; ++c) norm_element<ACT>(e[c], ch.c[c], p.k.u, p.silu_k, ch.mul, ch.sub, y[c], t[c]);
        if constexpr (VEC == 4) {
            if (p.y) ntstore4(reinterpret_cast<float4*>(p.y + out + i * p.ldy), make_float4(y[0], y[1], y[2], y[3]));
            if (p.tau) ntstore4(reinterpret_cast<float4*>(p.tau + out + i * p.ldy), make_float4(t[0], t[1], t[2], t[3]));
        } else {
            if (p.y) p.y[out + i * p.ldy] = y[0];
            if (p.tau) p.tau[out + i * p.ldy] = t[0];
        }
    }
}
// (c) checked on the spot: workgroups of the streaming check, which take (sample, part) items of `pixels` pixels in turn
template <int ACT, int VEC>
__global__ __launch_bounds__(kCheckThreads) void norm_act_check(NormArgs p, long items, long per_sample, long pixels, double alpha, double eps_rel, PassOut pass) {
    __shared__ unsigned int hist[kBins * kReplicas];
    __shared__ unsigned int red[kRedWords];
    __shared__ double smem[4 * kNormThreads];
    extern __shared__ GroupCoef coef[];
    const int tid = threadIdx.x;
    for (int i = tid; i < kBins * kReplicas; i += kCheckThreads) hist[i] = 0;
    __syncthreads();
    ThreadAcc acc;
    const int rep = tid & (kReplicas - 1);
    const long ncb = column_blocks<VEC>(p.channels);
    for (long it = blockIdx.x; it < items; it += gridDim.x) {
        const long s = it / per_sample, part = it - s * per_sample;
        const Place<kCheckThreads, VEC> at(p, part % ncb);
        const Channels<kCheckThreads, VEC> ch(p, s, at, coef, smem);
        if (at.active) {
            const long p0 = part / ncb * pixels, p1 = min(p0 + pixels, p.positions);
            const float* x = p.x + s * p.positions * p.ldx + at.c0;
            const long out = s * p.positions * p.ldy + at.c0;
            for (long i = p0 + at.ty; i < p1; i += at.TY) {
                float e[VEC], y[VEC], t[VEC], c[VEC];
                load_channels(x + i * p.ldx, e);
                load_channels(p.claimed + out + i * p.ldy, c);
#pragma unroll
                for (int j = 0; j < VEC; ++j) norm_element<ACT>(e[j], ch.c[j], p.k.u, p.silu_k, ch.mul, ch.sub, y[j], t[j]);
                if (p.y_ref) load_channels(p.y_ref + out + i * p.ldy, y);
                if constexpr (VEC == 4) check_four(c, y, t, alpha, eps_rel, hist, rep, acc);
                else                    check_one(c[0], y[0], t[0], alpha, eps_rel, hist, rep, acc);
            }
        }
        __syncthreads();                                     // (the coefficients are replaced)
    }
    finish_pass(hist, acc, red, pass);
}

// Parts of a sample: pixel parts, each for every column block, so that about four workgroups a compute unit are at work, of eight or more trips
// of a workgroup over its pixels.
struct NormParts { long nparts, pixels; };
template <int THREADS, int VEC>
static NormParts norm_parts(long batch, long positions, long channels, long workgroups) {
    const long ncb = column_blocks<VEC>(channels);
    const long cv = channels / VEC, ty = THREADS / (cv < kColumns<VEC> ? cv : kColumns<VEC>);
    long want = (workgroups + batch * ncb - 1) / (batch * ncb);
    const long most = (positions + 8 * ty - 1) / (8 * ty);
    want = want < 1 ? 1 : want > most ? most : want;
    NormParts r;
    r.pixels = (positions + want - 1) / want;
    r.nparts = (positions + r.pixels - 1) / r.pixels * ncb;
    return r;
}
static NormParts sums_parts(long batch, long positions, long channels, bool vec) {
    return vec ? norm_parts<kNormThreads, 4>(batch, positions, channels, 1024) : norm_parts<kNormThreads, 1>(batch, positions, channels, 1024);
}
static bool norm_shape_ok(long batch, long positions, long channels, long groups) {
    if (batch < 0 || positions < 0 || channels < 0 || groups < 1 || channels % groups) return false;
    const long lim = 1L << 31;
    if (batch >= lim || positions >= lim || channels >= lim) return false;
    return (__int128)(channels / groups) * positions < lim && (__int128)batch * positions * channels < ((__int128)1 << 36);
}
// (a caller's tensors may or may not allow vectors, which decides the number of parts: the larger of the two)
static size_t sums_bytes(long batch, long positions, long channels, long groups) {
    if (!norm_shape_ok(batch, positions, channels, groups) || batch * positions * channels == 0) return 0;
    const long one = sums_parts(batch, positions, channels, false).nparts;
    const long four = channels % 4 == 0 ? sums_parts(batch, positions, channels, true).nparts : 0;
    return (size_t)batch * (size_t)(one > four ? one : four) * (size_t)groups * 4 * sizeof(double);
}

// Checks the arguments that the two entry points share and fills the kernels'.
static int norm_setup(int act, const float* x, const float* gamma, const float* beta, double eps, long batch, long positions, long channels,
                      long groups, long ldx, long ldy, const tao_fp_model* model, NormArgs* out) {
    tao_fp_model md;
    int rc = resolve_model(model, &md);
    if (rc != TAO_OK) return rc;
    if (act != TAO_ACT_EXACT && act != TAO_ACT_RELU && act != TAO_ACT_SILU) return TAO_ERR_KIND;
    if (!norm_shape_ok(batch, positions, channels, groups) || ldx < channels || ldy < channels) return TAO_ERR_SHAPE;
    if ((__int128)batch * positions * ldx >= ((__int128)1 << 60) || (__int128)batch * positions * ldy >= ((__int128)1 << 60)) return TAO_ERR_SHAPE;
    if (!(eps >= 0.0) || !std::isfinite(eps)) return TAO_ERR_SHAPE;
    if (batch * positions * channels > 0 && !x) return TAO_ERR_NULL;
    if (!aligned(x, 4) || !aligned(gamma, 4) || !aligned(beta, 4)) return TAO_ERR_ALIGN;
    NormArgs& p = *out;
    p = NormArgs();
    const long per = channels / groups, n = per * positions;
    rc = make_consts(md, n > 0 ? n : 1, eps, &p.k, true);
    if (rc != TAO_OK) return rc;
    const double f = silu_factor(md);
    if (!(f < 0.5)) return TAO_ERR_MODEL;
    p.silu_k = widen(f / (1.0 - f));
    p.x = x; p.gamma = gamma; p.beta = beta;
    p.batch = batch; p.positions = positions; p.channels = channels; p.groups = groups; p.per = per; p.ldx = ldx; p.ldy = ldy;
    return TAO_OK;
}
// Groups that a column block can touch: one a channel, or all there are.
static long block_groups(long groups, bool vec) {
    const long most = vec ? 4 * kColumns<4> : kColumns<1>;
    return groups < most ? groups : most;
}
// The sums of all groups, left in p.part.
static int norm_sums(NormArgs& p, bool vec, hipStream_t st) {
    const NormParts parts = sums_parts(p.batch, p.positions, p.channels, vec);
    p.nparts = parts.nparts; p.pixels = parts.pixels;
    if ((__int128)p.batch * p.nparts >= (1L << 24)) return TAO_ERR_SHAPE;
    const dim3 grid((unsigned)(p.batch * p.nparts)), blk(kNormThreads);
    const size_t lds = (size_t)block_groups(p.groups, vec) * sizeof(double);
    if (vec) {
        hipLaunchKernelGGL(norm_sums_a<4>, grid, blk, 0, st, p);
        hipLaunchKernelGGL(norm_sums_b<4>, grid, blk, lds, st, p);
    } else {
        hipLaunchKernelGGL(norm_sums_a<1>, grid, blk, 0, st, p);
        hipLaunchKernelGGL(norm_sums_b<1>, grid, blk, lds, st, p);
    }
    return TAO_OK;
}

}  // namespace tao

extern "C" {

size_t tao_groupnorm_act_workspace_bytes(long batch, long positions, long channels, long groups) {
    return tao::sums_bytes(batch, positions, channels, groups);
}

size_t tao_bound_check_groupnorm_act_workspace_bytes(long batch, long positions, long channels, long groups) {
    return tao::check_workspace_bytes() + tao::sums_bytes(batch, positions, channels, groups);
}

int tao_bound_groupnorm_act(int act, const float* x, const float* gamma, const float* beta, double eps, float* y, float* tau,
                            long batch, long positions, long channels, long groups, long ldx, long ldy,
                            const tao_fp_model* model, void* ws, size_t ws_bytes, void* stream) {
    using namespace tao;
    NormArgs p;
    int rc = norm_setup(act, x, gamma, beta, eps, batch, positions, channels, groups, ldx, ldy, model, &p);
    if (rc != TAO_OK) return rc;
    if (batch * positions * channels == 0) return TAO_OK;
    if (!y && !tau) return TAO_ERR_NULL;
    if (!aligned(y, 4) || !aligned(tau, 4)) return TAO_ERR_ALIGN;
    if (!ws || !aligned(ws, 256) || ws_bytes < sums_bytes(batch, positions, channels, groups)) return TAO_ERR_WORKSPACE;
    p.y = y; p.tau = tau; p.part = static_cast<double*>(ws);
    const bool vec = channels % 4 == 0 && ldx % 4 == 0 && ldy % 4 == 0 && aligned(x, 16) && aligned(y, 16) && aligned(tau, 16);
    hipStream_t st = (hipStream_t)stream;
    rc = norm_sums(p, vec, st);
    if (rc != TAO_OK) return rc;
    const dim3 grid((unsigned)(batch * p.nparts)), blk(kNormThreads);
    const size_t lds = (size_t)block_groups(groups, vec) * sizeof(GroupCoef);
#define TAO_NORM_APPLY(ACT) do { if (vec) hipLaunchKernelGGL((norm_apply<ACT, 4>), grid, blk, lds, st, p); \
                                 else hipLaunchKernelGGL((norm_apply<ACT, 1>), grid, blk, lds, st, p); } while (0)
    if (act == TAO_ACT_SILU)      TAO_NORM_APPLY(TAO_ACT_SILU);
    else if (act == TAO_ACT_RELU) TAO_NORM_APPLY(TAO_ACT_RELU);
    else                          TAO_NORM_APPLY(TAO_ACT_EXACT);
#undef TAO_NORM_APPLY
    return launch_status();
}

int tao_bound_check_groupnorm_act(int act, const float* x, const float* gamma, const float* beta, double eps, const float* y_ref,
                                  const float* claimed, long batch, long positions, long channels, long groups, long ldx, long ldy,
                                  double alpha, double eps_rel, const tao_fp_model* model, tao_profile* out,
                                  void* ws, size_t ws_bytes, void* stream) {
    using namespace tao;
    NormArgs p;
    int rc = norm_setup(act, x, gamma, beta, eps, batch, positions, channels, groups, ldx, ldy, model, &p);
    if (rc != TAO_OK) return rc;
    if (!out || !ws) return out ? TAO_ERR_WORKSPACE : TAO_ERR_NULL;
    if (!(alpha >= 0.0) || !std::isfinite(alpha) || !(eps_rel >= 0.0) || !std::isfinite(eps_rel)) return TAO_ERR_SHAPE;
    const long n = batch * positions * channels;
    if (n > 0 && !claimed) return TAO_ERR_NULL;
    if (!aligned(y_ref, 4) || !aligned(claimed, 4) || !aligned(out, 8)) return TAO_ERR_ALIGN;
    if (!aligned(ws, 256) || ws_bytes < check_workspace_bytes() + sums_bytes(batch, positions, channels, groups)) return TAO_ERR_WORKSPACE;
    p.y_ref = y_ref; p.claimed = claimed;
    p.part = reinterpret_cast<double*>(static_cast<char*>(ws) + check_workspace_bytes());
    const bool vec = channels % 4 == 0 && ldx % 4 == 0 && ldy % 4 == 0 && aligned(x, 16) && aligned(y_ref, 16) && aligned(claimed, 16);
    hipStream_t st = (hipStream_t)stream;
    const CheckWorkspace w = carve_check_workspace(ws);
    long items = 0;
    NormParts parts{1, 1};
    if (n > 0) {
        rc = norm_sums(p, vec, st);
        if (rc != TAO_OK) return rc;
        parts = vec ? norm_parts<kCheckThreads, 4>(batch, positions, channels, kMaxCheckBlocks) : norm_parts<kCheckThreads, 1>(batch, positions, channels, kMaxCheckBlocks);
        items = batch * parts.nparts;
    } else {
        p.channels = p.groups = p.per = 4;                   // (no item is taken)
    }
    const int nblocks = (int)(items < 1 ? 1 : items < kMaxCheckBlocks ? items : kMaxCheckBlocks);
    const size_t lds = (size_t)block_groups(groups, vec) * sizeof(GroupCoef);
#define TAO_NORM_CHECK_V(ACT, VEC) hipLaunchKernelGGL((norm_act_check<ACT, VEC>), dim3(nblocks), dim3(kCheckThreads), lds, st, p, items, parts.nparts, \
                                                      parts.pixels, alpha, eps_rel, pass_out(w, nblocks, n, out))
#define TAO_NORM_CHECK(ACT) do { if (vec) TAO_NORM_CHECK_V(ACT, 4); else TAO_NORM_CHECK_V(ACT, 1); } while (0)
    if (act == TAO_ACT_SILU)      TAO_NORM_CHECK(TAO_ACT_SILU);
    else if (act == TAO_ACT_RELU) TAO_NORM_CHECK(TAO_ACT_RELU);
    else                          TAO_NORM_CHECK(TAO_ACT_EXACT);
#undef TAO_NORM_CHECK
#undef TAO_NORM_CHECK_V
    launch_finish(w, nblocks, n, out, st);
    return launch_status();
}

}  // extern "C"
