// tao_bound_groupnorm_act, tao_bound_check_groupnorm_act: GroupNorm with an activation on channels-last features
// x[sample][pixel][channel] (operators of App. A.3), re-executed and bounded in one call.  A (sample, group) is one row of n = pixels x
// channels per group elements of the LayerNorm chain (tao_rows.hpp), which gives the mean mu, the inverse root r and coefficients with
//     |p^ - p| <= E = E_p + u (|p| + E_p),   E_p = |gamma| (K1 |d| + K0),   d = x - mu,   p = d r gamma + beta.
// The activation then moves an error of its argument by at most (second order closed: |s''| <= 1/2, |s'| <= 1.1 for SiLU s)
//     none E,   ReLU max(0, min(E, p + E)),   SiLU B = min(|s'(p)| E + E^2/4, 1.1 E), and its own roundings k (|s(p)| + B).
//
// Two ways.  Few groups that a workgroup's registers hold (norm_rows): one workgroup a (sample, group), one launch.
// Others: a thread keeps its channels (four of them, one 16-byte load) and walks the pixels of a part of the sample, so its sums are
// per channel, whatever the number of channels per group, and reach their groups in LDS.  Three passes over x, as the mean has to
// be known before the deviations, and sum |d| with it: (a) sum x, sum |x|, (b) sum |d|, sum d^2, (c) the outputs; every workgroup of (b) and (c) adds up
// the parts of its groups in the same order.  4 x 16384 x 512 SiLU: 24 + 24 + 70 us (134 MB read at 5.5 TB/s twice, 402 MB moved at 5.7 TB/s); the check in place
// of (c) 80 us, next to its instructions (about 72 an element, 35 of them binary64, four cycles each).
#include <algorithm>
#include <type_traits>
#include "tao_check.hpp"
#include "tao_device.hpp"
#include "tao_host.hpp"
#include "tao_rows.hpp"

namespace tao {

struct NormArgs {
    const float* x; const float* gamma; const float* beta;
    float* y; float* tau;
    const float* y_ref; const float* claimed;
    double2* part;                   // [sample][2][group][column block of the group, pixel part]: (sum x, sum |x|), (sum |d|, sum d^2)
    long positions, ldx, ldy, batch;
    int channels, groups, per;
    int ncb, pixel_parts;            // of a sample: column blocks, parts of its pixels
    int span;                        // column blocks that a group lies in, at most
    long pixels;                     // of a part
    RowConsts k;
    // of norm_element, with the final upper rounding's factor in them, and SiLU's 1 + silu_f / (1 - silu_f) in the first two
    double grow_ep, grow_p;          // of E: (1 + u) E_p, u |p|
    double quarter, silu_k;          // of SiLU: of E^2 without the factors, silu_f / (1 - silu_f)
    double n;
};
// ... of a check: items are rows, or parts of all samples
struct NormCheckArgs { NormArgs p; long items; double alpha, eps_rel; PassOut pass; };
constexpr int kNormThreads = kCheckThreads;

// A vector of VEC floats needs the alignment of one.
template <int VEC> struct Floats { typedef float type __attribute__((ext_vector_type(VEC), aligned(4))); };
template <> struct Floats<1> { typedef float type; };
template <int VEC, bool STREAM>
__device__ __forceinline__ void load_floats(const float* __restrict__ p, float (&v)[VEC]) {
    typedef typename Floats<VEC>::type T;
    T t;
    if constexpr (STREAM) t = __builtin_nontemporal_load(reinterpret_cast<const T*>(p)); else t = *reinterpret_cast<const T*>(p);
    if constexpr (VEC == 1) v[0] = t;
    else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = t[i];
    }
}
template <int VEC>
__device__ __forceinline__ void store_floats(float* __restrict__ p, const float (&v)[VEC]) {
    typedef typename Floats<VEC>::type T;
    T t;
    if constexpr (VEC == 1) t = v[0];
    else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) t[i] = v[i];
    }
    __builtin_nontemporal_store(t, reinterpret_cast<T*>(p));
}

// ---- one element

// What an element's bound takes of its group.
struct GroupCoef { double mu, r, K1, K0; };
// The thread's number, of which nothing is formed ahead: in loops over rows or items the compiler else keeps what follows from it from trip to trip, in registers that
// the loops over pixels then lack.
__device__ __forceinline__ int thread_here() {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    return tid;
}
// ... and the arguments of a kernel that has one, read from its segment anew: kept from the start they take the scalar registers that the loops need for constants.
template <class T> __device__ __forceinline__ const T& args_here() {
    auto* args = (const __attribute__((address_space(4))) T*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    return *(const T*)args;
}
// A value as it is, not as a branch around the loads that use it.
__device__ __forceinline__ long plain(long v) {
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ GroupCoef group_coef(const RowConsts& k, double n, double s_x, double s_ax, double s_ad, double s_d2) {
    GroupCoef c;
    c.mu = s_x * k.inv_n;
    const double E_mu = ((k.G * s_ax) * k.inv_n + k.cd_u * fabs(c.mu)) * k.inv1mcd;
    double amp;
    layernorm_tail(E_mu, s_ad, s_d2, n, k, c.K1, c.K0, amp, &c.r);
    // the group's own rounding margin goes into its E_p, which everything after it grows with: neighbours in a thread may be of another group
    const double m = amp > 0.0 && amp < INFINITY ? k.m * (1.0 + 2.0 * amp) : 0.0;      // (else K0 is NaN, and so is the bound)
    c.K1 *= 1.0 + 2.0 * m; c.K0 *= 1.0 + 2.0 * m;
    return c;
}
// ... and of its channel: p = d rg + b, grow_ep E_p = k1 |d| + k0 (NaN where gamma or beta is infinite: such a bound would admit every finite claim)
struct ChannelCoef { double mu, rg, b, k1, k0; };
__device__ __forceinline__ ChannelCoef channel_coef(const NormArgs& p, const GroupCoef& g, int channel) {
    const float gamma = p.gamma ? p.gamma[channel] : 1.f, beta = p.beta ? p.beta[channel] : 0.f;
    const double w = (double)gamma, grown = fabs(w) * p.grow_ep;
    return ChannelCoef{g.mu, g.r * w, (double)beta, grown * g.K1, fma(grown, g.K0, (double)(gamma * 0.f + beta * 0.f))};
}

// 1 / (1 + exp(-p)) and 1 minus it, to 2^-39, for |p| <= 700 (beyond, those of 700 with p's sign: where |p| 2^-1009 stands for |p| exp(-|p|)).
// exp(r) on |r| <= ln2 / 2 as a polynomial of degree 8 whose relative error, 2^-40.2, is the least possible (found by exchange of its extrema);
// the quotient from v_rcp_f64 (2^-23) and one Newton step.  18 instructions of binary64, where exp_neg and a division take twice that:
// the outputs of 512 x 512 x 128 in 74 us instead of 129.
__device__ __forceinline__ double sigmoid(double p, double& rest) {
    const double s = fmin(fmax(p, -700.0), 700.0);
    const double magic = 0x1.8p52, t = fma(s, -0x1.71547652b82fep+0, magic);     // its low word: round(-s / ln 2)
    const double kf = t - magic;
    const double r = fma(kf, -0x1.62e42fefa39efp-1, -s);                          // (|kf| <= 1010: rounded once, to 2^-44)
    double e = 0x1.9eda8535decb2p-16;
    e = fma(e, r, 0x1.a1a82ff78d480p-13);
    e = fma(e, r, 0x1.6c18b36b04275p-10);
    e = fma(e, r, 0x1.111082a0f01e3p-7);
    e = fma(e, r, 0x1.55555404defd4p-5);
    e = fma(e, r, 0x1.555555a08cff3p-3);
    e = fma(e, r, 0x1.00000000880efp-1);
    e = fma(e, r, 0x1.ffffffffd55b1p-1);
    e = fma(e, r, 0x1.ffffffffff7a1p-1);
    e = __hiloint2double(__double2hiint(e) + (__double2loint(t) << 20), __double2loint(e));      // (the exponent stays within +-1012)
    const double a = 1.0 + e;
    double q = __builtin_amdgcn_rcp(a);
    q = fma(q, fma(-a, q, 1.0), q);
    rest = e * q;
    return q;
}

// Output and bound of one element.  E comes with the factor of the final upper rounding (kUp: 2^-24 for it, 2^-32 for the few roundings before it) and, for
// SiLU, with that of its own roundings, so both cost nothing here.  The slacks keep an evaluation in round-to-nearest binary64 at or above the formula's
// value.  s' = q (1 + p rest) is formed from q and rest = e q, e = exp(-p): a relative error of e (2^-40) reaches it as at most 2^-40 |s'| +
// 2^-41 q, as |p| q rest < 0.28, and one of q (2^-46, the reciprocal's) as 2^-46 (|s'| + |p| q rest), at most 2^-45 |s'| + 2^-46 q.  kUp has the parts of |s'|, and 2^-39 q those of q.
// That vanishes where s' does far below 0; about its zero at -1.278, where q = 0.22, it is 4e-13 E, far below 1e-6 of E^2/4 and the own roundings, 0.28 silu_f, together
// (for unit roundoffs from 2^-40 on).
constexpr double kUp = 1.0 + 0x1p-24 + 0x1p-32;
__device__ __forceinline__ float rounded_up(double v) {      // (v holds kUp)
    float f = (float)v;
    if (f < 0x1p-126f && (double)f < v) f = __uint_as_float(__float_as_uint(f) + 1u);
    return f;
}
template <int ACT>
__device__ __forceinline__ void norm_element(float x, const ChannelCoef& c, const NormArgs& a, float& y, float& tau) {
    const double d = (double)x - c.mu;
    const double p = fma(d, c.rg, c.b);
    const double E = fma(a.grow_p, fabs(p), fma(c.k1, fabs(d), c.k0));
    if constexpr (ACT == TAO_ACT_SILU) {
        double rest;
        const double sig = sigmoid(p, rest), s = p * sig;
        const double slope = fma(0x1p-39, sig, fabs(fma(s, rest, sig)));
        const double B = E * fmin(fma(a.quarter, E, slope), 1.1);
        y = (float)s;
        tau = rounded_up(fma(a.silu_k, fabs(s), B));         // (a minimum leaves a NaN out, but E times 1.1 is one)
    } else if constexpr (ACT == TAO_ACT_RELU) {
        y = p <= 0.0 ? 0.f : (float)p;
        const double t = fmin(E, fma(E, 1.0 + 0x1p-24, p));
        tau = E == E ? (t > 0.0 ? rounded_up(t) : 0.f) : (float)E;
    } else {
        y = (float)p;
        tau = rounded_up(E);
    }
}

// Four elements are taken at a time, 4 / VEC pixels of VEC neighbouring channels each (element 4 / VEC vectors, one after the other), and stored or checked; at(j)
// is the index of pixel j's first element, and the last four of a thread have `vectors` pixels.
template <int VEC> constexpr int kPixels = 4 / VEC;
template <int VEC, bool STREAM, class At>
__device__ __forceinline__ void load_quad(const float* __restrict__ p, At&& at, float (&q)[4]) {
#pragma unroll
    for (int j = 0; j < kPixels<VEC>; ++j) {
        float v[VEC];
        load_floats<VEC, STREAM>(p + at(j), v);
#pragma unroll
        for (int c = 0; c < VEC; ++c) q[j * VEC + c] = v[c];
    }
}
struct NormStore {
    float* y; float* tau;
    template <int VEC, class At> __device__ __forceinline__ void request(At&&, float (&)[4]) const {}
    template <int VEC, class At> __device__ __forceinline__ void reference(At&&, float (&)[4]) const {}
    template <int VEC, class At> __device__ __forceinline__ void put(At&& at, int vectors, const float (&yv)[4], const float (&tv)[4], const float (&)[4], const float (&)[4]) {
#pragma unroll
        for (int j = 0; j < kPixels<VEC>; ++j) {
            float a[VEC], b[VEC];
#pragma unroll
            for (int c = 0; c < VEC; ++c) { a[c] = yv[j * VEC + c]; b[c] = tv[j * VEC + c]; }
            if (j < vectors && y) store_floats<VEC>(y + at(j), a);
            if (j < vectors && tau) store_floats<VEC>(tau + at(j), b);
        }
    }
};
// REF: against the verifier's own outputs.  (No branch around their loads, behind which they would be waited for.)
template <bool REF>
struct NormCheck {
    const float* y_ref; const float* claimed; double alpha, eps_rel; QuickCheck q; bool ordinary;
    unsigned int* hist; unsigned int* largest; int rep;
    ThreadAcc acc; unsigned int zeros = 0; Farthest top;
    __device__ __forceinline__ NormCheck(const NormCheckArgs& a, unsigned int* hist_, unsigned int* largest_)
        : y_ref(a.p.y_ref), claimed(a.p.claimed), alpha(a.alpha), eps_rel(a.eps_rel), q(a.p.k.quick_alpha, a.eps_rel), hist(hist_), largest(largest_), rep(threadIdx.x & (kReplicas - 1)) {
        ordinary = q.eps < INFINITY && q.alpha > 0.f;
    }
    template <int VEC, class At> __device__ __forceinline__ void request(At&& at, float (&c)[4]) const { load_quad<VEC, true>(claimed, at, c); }
    template <int VEC, class At> __device__ __forceinline__ void reference(At&& at, float (&r)[4]) const { if constexpr (REF) load_quad<VEC, true>(y_ref, at, r); }
    template <int VEC, class At> __device__ __forceinline__ void put(At&&, int vectors, const float (&yv)[4], const float (&tv)[4], const float (&c)[4], const float (&rv)[4]) {
        floatv4 r, t, k;
#pragma unroll
        for (int e = 0; e < 4; ++e) { r[e] = REF ? rv[e] : yv[e]; t[e] = tv[e]; k[e] = c[e]; }
        // (a NaN among them shows in the error)
        const float most = fmaxf(fmaxf(fabsf(r[0]), fabsf(r[1])), fmaxf(fabsf(r[2]), fabsf(r[3])));
        if (settle_four<true, true>(k, r, t, q, top, largest, newest(largest), ordinary && most <= 0x1p90f && vectors >= kPixels<VEC>, acc, zeros,
                        [&](unsigned bin) __attribute__((always_inline)) { atomicAdd(&hist[bin * kReplicas + rep], 1u); })) return;
        // (one at a time, in registers that move down: about one four in a thousand, and their divisions side by side take the registers of everything else)
        const int n = min(vectors * VEC, 4);
#pragma unroll 1
        for (int e = 0; e < n; ++e) {
            check_one(k[0], r[0], t[0], alpha, eps_rel, hist, rep, acc);
            k = k.yzww; r = r.yzww; t = t.yzww;
        }
    }
    __device__ __forceinline__ void finish() {
        if (zeros) atomicAdd(&hist[rep], zeros);
        settled(top, alpha, eps_rel, acc);
    }
};
// The check's LDS, in kernels of kCheckThreads threads.
struct CheckShared { unsigned int hist[kBins * kReplicas], red[kRedWords], largest; };
__device__ __forceinline__ void clear_check(CheckShared& c) {
    for (int i = threadIdx.x; i < kBins * kReplicas; i += kCheckThreads) c.hist[i] = 0;
    if (threadIdx.x == 0) c.largest = 0;
    __syncthreads();
}

// ---- groups that a workgroup's registers hold: V vectors a thread
constexpr int kRowVectors = 2;                               // of the largest workgroups

// Vector v THREADS + tid of a group is vector c of pixel pix; the next one of this thread lies a fixed number of pixels and vectors on.
struct RowWalk {
    unsigned per_pixel, pix, c, dpix, dc;
    __device__ __forceinline__ RowWalk(unsigned per_pixel_, unsigned tid, unsigned threads) : per_pixel(per_pixel_) {
        pix = tid / per_pixel; c = tid - pix * per_pixel;
        dpix = threads / per_pixel; dc = threads - dpix * per_pixel;
    }
    __device__ __forceinline__ void next() {
        pix += dpix; c += dc;
        if (c >= per_pixel) { c -= per_pixel; ++pix; }
    }
};
// Sums over the LANES lanes of a group of lanes, in every one of them.
template <int LANES>
__device__ __forceinline__ double lanes_sum(double v) {
    constexpr int STEPS = LANES == 1 ? 0 : LANES == 4 ? 2 : LANES == 16 ? 4 : 6;
    return wave_all<0, STEPS>(v, [](double a, double b) { return a + b; });
}
template <int THREADS>
__device__ __forceinline__ void block_sums(double (&v)[2], double* smem) {
    const int tid = thread_here(), wave = tid / kWave, lane = tid & (kWave - 1);
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = wave_sum(v[i]);
    if (lane == 0) { smem[wave * 2] = v[0]; smem[wave * 2 + 1] = v[1]; }
    __syncthreads();
    constexpr int WAVES = THREADS / kWave;
    v[0] = lanes_sum<WAVES>(smem[lane % WAVES * 2]); v[1] = lanes_sum<WAVES>(smem[lane % WAVES * 2 + 1]);
}
template <int ACT, int VEC, int V, int THREADS, class Sink>
__device__ __forceinline__ void norm_row(const NormArgs& p, long row, double* smem, Sink& sink) {
    const unsigned tid = thread_here();
    const long s = row / p.groups;
    const int g = (int)(row - s * p.groups);
    const unsigned per_pixel = (unsigned)(p.per / VEC), vectors = per_pixel * (unsigned)p.positions;
    const float* x = p.x + s * p.positions * p.ldx + (long)g * p.per;
    const RowWalk start(per_pixel, tid, THREADS);
    float e[V][VEC];
    double a[2] = {0.0, 0.0};
    RowWalk w = start;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const bool in = v * THREADS + tid < vectors;
#pragma unroll
        for (int c = 0; c < VEC; ++c) e[v][c] = 0.f;
        if (in) load_floats<VEC, false>(x + w.pix * p.ldx + w.c * VEC, e[v]);
        w.next();
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int c = 0; c < VEC; ++c) { a[0] += (double)e[v][c]; a[1] += (double)fabsf(e[v][c]); }
    block_sums<THREADS>(a, smem);
    const double mu = a[0] * p.k.inv_n;
    double b[2] = {0.0, 0.0};
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const bool in = v * THREADS + tid < vectors;
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
            const double d = in ? (double)e[v][c] - mu : 0.0;
            b[0] += fabs(d); b[1] = fma(d, d, b[1]);
        }
    }
    block_sums<THREADS>(b, smem + 2 * (THREADS / kWave));
    const GroupCoef coef = group_coef(p.k, p.n, a[0], a[1], b[0], b[1]);
    const long out = s * p.positions * p.ldy + (long)g * p.per;
    // (a loop that reads x again, from the caches, and the next four elements while four are computed: unrolled over the registers it would take several times the
    // code, and registers that spill)
    constexpr int PIX = kPixels<VEC>;
    RowWalk ahead = start;
    float xn[4], cn[4];
    auto request = [&](unsigned first) __attribute__((always_inline)) {
        long ix[PIX], iy[PIX];
#pragma unroll
        for (int j = 0; j < PIX; ++j) {
            const bool in = first + j * THREADS < vectors;
            ix[j] = plain(in ? ahead.pix * p.ldx + ahead.c * VEC : 0);
            iy[j] = plain(in ? out + ahead.pix * p.ldy + ahead.c * VEC : out);
            ahead.next();
        }
        load_quad<VEC, true>(x, [&](int j) { return ix[j]; }, xn);
        sink.template request<VEC>([&](int j) { return iy[j]; }, cn);
    };
    w = start;
    request(tid);
#pragma unroll 1
    for (unsigned at = tid; at < vectors; at += PIX * THREADS) {
        float xv[4], claims[4], ref[4], y[4], t[4];
        long index[PIX];
        unsigned channel[PIX];
#pragma unroll
        for (int j = 0; j < PIX; ++j) {
            const bool in = at + j * THREADS < vectors;
            index[j] = plain(in ? out + w.pix * p.ldy + w.c * VEC : out);
            channel[j] = (in ? w.c : 0u) * VEC;
            w.next();
        }
        const auto place = [&](int j) { return index[j]; };
#pragma unroll
        for (int c = 0; c < 4; ++c) { xv[c] = xn[c]; claims[c] = cn[c]; }
        sink.template reference<VEC>(place, ref);
        request(at + PIX * THREADS);
        // (one at a time, through registers that move round: a workgroup runs this code once or a few times, so its length costs as much as its operations)
        unsigned of[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) of[e] = g * p.per + channel[e / VEC] + e % VEC;
#pragma unroll 1
        for (int e = 0; e < 4; ++e) {
            float y1, t1;
            norm_element<ACT>(xv[0], channel_coef(p, coef, (int)of[0]), p, y1, t1);
#pragma unroll
            for (int i = 0; i < 3; ++i) { xv[i] = xv[i + 1]; of[i] = of[i + 1]; y[i] = y[i + 1]; t[i] = t[i + 1]; }
            y[3] = y1; t[3] = t1;
        }
        sink.template put<VEC>(place, (int)((vectors - at + THREADS - 1) / THREADS), y, t, claims, ref);
    }
}
// Workgroup b of n takes rows b, b + n, ... of an order in which the workgroups of an XCD (b modulo 8) have rows that follow each other: groups of a pixel that
// share a line of memory are then read through one L2.
struct RowOrder {
    long share, n, at, step, base;
    __device__ __forceinline__ RowOrder(long rows) {
        const long xcd = blockIdx.x & 7;
        share = (rows + 7) / 8; base = xcd * share; n = min(share, rows - base);
        at = blockIdx.x >> 3; step = (gridDim.x - xcd + 7) / 8;
    }
};
template <int ACT, int VEC, int V, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_rows(NormArgs p) {
    __shared__ double smem[4 * (THREADS / kWave)];
    NormStore sink{p.y, p.tau};
    const RowOrder o(p.batch * p.groups);
    if (o.at < o.n) norm_row<ACT, VEC, V, THREADS>(p, o.base + o.at, smem, sink);
}
template <int ACT, int VEC, bool REF>
__global__ __launch_bounds__(kCheckThreads) void norm_rows_check(NormCheckArgs) {
    __shared__ CheckShared chk;
    __shared__ double smem[4 * (kCheckThreads / kWave)];
    clear_check(chk);
    const NormCheckArgs& a = args_here<NormCheckArgs>();
    NormCheck<REF> sink(a, chk.hist, &chk.largest);
    const RowOrder o(a.items);
    for (long i = o.at; i < o.n; i += o.step) {
        norm_row<ACT, VEC, kRowVectors, kCheckThreads>(args_here<NormCheckArgs>().p, o.base + i, smem, sink);
        __syncthreads();                                     // (the sums are the next row's)
    }
    sink.finish();
    __syncthreads();
    finish_pass(chk.hist, sink.acc, chk.red, args_here<NormCheckArgs>().pass);
}

// ---- larger groups

// A workgroup takes columns of at most this many channels: the coefficients of their groups then fit LDS beside the check's histogram, and the
// workgroup's pixels lie 2 KB of contiguous memory each.
constexpr int kColumns = 512;
// A workgroup's place: sample, part of its pixels, column block; thread (tx, ty) = vector of the block, first pixel.
template <int VEC>
struct Place {
    long s, p0, p1;
    int cb, part, TX, TY, tx, ty, c0, c_lo, c_hi, g_lo, g_hi;
    bool active;
    __device__ __forceinline__ Place(const NormArgs& p, long item) {
        const int tid = thread_here();
        const long of_sample = (long)p.pixel_parts * p.ncb;
        s = item / of_sample;
        const int in = (int)(item - s * of_sample);
        part = in / p.ncb; cb = in - part * p.ncb;
        p0 = part * p.pixels; p1 = min(p0 + p.pixels, p.positions);
        c_lo = cb * kColumns;
        TX = min(kColumns, p.channels - c_lo) / VEC;
        TY = kNormThreads / TX;
        ty = tid / TX; tx = tid - ty * TX;
        active = ty < TY;
        c_hi = c_lo + TX * VEC;
        c0 = c_lo + tx * VEC;
        g_lo = c_lo / p.per; g_hi = (c_hi - 1) / p.per + 1;
    }
};
__device__ __forceinline__ double2* parts_of(const NormArgs& p, long s, int which, int g) { return p.part + ((s * 2 + which) * p.groups + g) * p.span * p.pixel_parts; }
__device__ __forceinline__ int first_block(const NormArgs& p, int g) { return g * p.per / kColumns; }
__device__ __forceinline__ int parts_in(const NormArgs& p, int g) { return (((g + 1) * p.per - 1) / kColumns - first_block(p, g) + 1) * p.pixel_parts; }

// A number of lanes for `items` items: enough that each has few.
template <class Use> __device__ __forceinline__ void with_lanes(int items, Use&& use) {
    if (items <= 4)       use(std::integral_constant<int, 1>());
    else if (items <= 16) use(std::integral_constant<int, 4>());
    else if (items <= 64) use(std::integral_constant<int, 16>());
    else                  use(std::integral_constant<int, 64>());
}

// The threads' sums v[channel][i] to those of the block's groups, this part's entry of each.  Where a thread's channels are of
// one group, the thread leaves one entry, else one a channel; the lanes of a group then take its entries of all rows of threads, so the number of threads
// that add does not depend on the number of channels.  smem: 2 kNormThreads VEC doubles.
template <int VEC>
__device__ __forceinline__ void channel_sums(const NormArgs& p, const Place<VEC>& at, const double (&v)[VEC][2], double* smem, int which) {
    const bool joined = p.per % VEC == 0;
    const int each = joined ? VEC : 1, width = at.TX * (VEC / each), per = p.per / each, lo_c = at.c_lo / each, hi_c = at.c_hi / each;
    double2* entry = reinterpret_cast<double2*>(smem);       // [ty][channel, or four of them]
    if (at.active) {
        if (joined) {
            double2 s = make_double2(v[0][0], v[0][1]);
#pragma unroll
            for (int c = 1; c < VEC; ++c) { s.x += v[c][0]; s.y += v[c][1]; }
            entry[at.ty * width + at.tx] = s;
        } else {
#pragma unroll
            for (int c = 0; c < VEC; ++c) entry[at.ty * width + at.tx * VEC + c] = make_double2(v[c][0], v[c][1]);
        }
    }
    __syncthreads();
    with_lanes(kNormThreads / (at.g_hi - at.g_lo), [&](auto lanes) __attribute__((always_inline)) {
        constexpr int LANES = decltype(lanes)::value, AT_ONCE = kNormThreads / LANES;
        const int sub = threadIdx.x % LANES;
        for (int first = at.g_lo; first < at.g_hi; first += AT_ONCE) {       // (the same number of trips for all lanes)
            const int g = first + threadIdx.x / LANES;
            const int lo = max(g * per, lo_c), n = g < at.g_hi ? min((g + 1) * per, hi_c) - lo : 0;
            double2 s = make_double2(0.0, 0.0);
            // the lanes side by side on a row's entries where it has as many, on several rows where it has fewer
            const int rows = n >= LANES ? 1 : n > 0 ? LANES / n : 1, row = n >= LANES ? 0 : n > 0 ? sub / n : rows, first_c = n >= LANES ? sub : n > 0 ? sub % n : 0;
            if (row < rows)
                for (int t = row; t < at.TY; t += rows)
                    for (int c = first_c; c < n; c += LANES) { const double2 q = entry[t * width + lo - lo_c + c]; s.x += q.x; s.y += q.y; }
            s.x = lanes_sum<LANES>(s.x); s.y = lanes_sum<LANES>(s.y);
            if (sub == 0 && g < at.g_hi) parts_of(p, at.s, which, g)[(at.cb - first_block(p, g)) * p.pixel_parts + at.part] = s;
        }
    });
}
// Totals over a sample's parts of the block's groups, handed to use(group - g_lo, first totals, second totals) by one lane each; BOTH: of the deviations too.
// (The parts come from other XCDs, through memory: four of each sum are requested at a time.)
template <bool BOTH, int VEC, class Use>
__device__ __forceinline__ void group_totals(const NormArgs& p, const Place<VEC>& at, Use&& use) {
    with_lanes(p.span * p.pixel_parts, [&](auto lanes) __attribute__((always_inline)) {
        constexpr int LANES = decltype(lanes)::value, AT_ONCE = kNormThreads / LANES, SUMS = BOTH ? 2 : 1;
        const int tid = thread_here();
        const int sub = tid % LANES;
        for (int first = at.g_lo; first < at.g_hi; first += AT_ONCE) {
            const int g = first + tid / LANES;
            double2 t[2] = {};
            if (g < at.g_hi) {
                const double2* v = parts_of(p, at.s, 0, g);
                const long second = (long)p.groups * p.span * p.pixel_parts;
                const int parts = parts_in(p, g);
                for (int i = sub; i < parts; i += 4 * LANES) {
                    double2 q[4][SUMS];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int w = 0; w < SUMS; ++w) q[k][w] = v[min(i + k * LANES, parts - 1) + w * second];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int w = 0; w < SUMS; ++w) {
                            const bool in = i + k * LANES < parts;
                            t[w].x += in ? q[k][w].x : 0.0; t[w].y += in ? q[k][w].y : 0.0;
                        }
                }
            }
#pragma unroll
            for (int w = 0; w < SUMS; ++w) { t[w].x = lanes_sum<LANES>(t[w].x); t[w].y = lanes_sum<LANES>(t[w].y); }
            if (sub == 0 && g < at.g_hi) use(g - at.g_lo, t[0], t[1]);
        }
    });
}

// (a) sum x, sum |x| of a part; DEVIATIONS: (b) the means from the parts of (a), then sum |d|, sum d^2
template <int VEC, bool DEVIATIONS>
__global__ __launch_bounds__(kNormThreads) void norm_sums(NormArgs p) {
    __shared__ __align__(16) double smem[2 * kNormThreads * VEC];
    double* mean = smem;                                     // of the block's groups, read before the sums are left there
    const Place<VEC> at(p, blockIdx.x);
    const float* x = p.x + at.s * p.positions * p.ldx + at.c0;
    const long end = at.active ? at.p1 : 0;
    double mu[VEC] = {}, v[VEC][2] = {};
    // (the first pixels are on their way while the means are added up)
    constexpr int AHEAD = 4;
    float e[AHEAD][VEC];
    long i = at.p0 + at.ty;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) e[k][c] = 0.f;
        if (i + k * at.TY < end) load_floats<VEC, false>(x + (i + k * at.TY) * p.ldx, e[k]);
    }
    if constexpr (DEVIATIONS) {
        group_totals<false>(p, at, [&](int g, const double2& t, const double2&) __attribute__((always_inline)) { mean[g] = t.x * p.k.inv_n; });
        __syncthreads();
        if (at.active) {
#pragma unroll
            for (int c = 0; c < VEC; ++c) mu[c] = mean[(at.c0 + c) / p.per - at.g_lo];
        }
        __syncthreads();
    }
    auto add = [&](const float (&f)[VEC]) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
            const double d = DEVIATIONS ? (double)f[c] - mu[c] : (double)f[c];
            if constexpr (DEVIATIONS) { v[c][0] += fabs(d); v[c][1] = fma(d, d, v[c][1]); }
            else                      { v[c][0] += d; v[c][1] += fabs(d); }
        }
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        if (i + k * at.TY < end) add(e[k]);
    i += AHEAD * at.TY;
#pragma unroll 4
    for (; i < end; i += at.TY) {
        float f[VEC];
        load_floats<VEC, false>(x + i * p.ldx, f);
        add(f);
    }
    channel_sums<VEC>(p, at, v, smem, DEVIATIONS ? 1 : 0);
}

// (c) the outputs of a part
template <int ACT, int VEC, class Sink>
__device__ __forceinline__ void norm_part(const NormArgs& p, long item, GroupCoef* coef, Sink& sink) {
    const Place<VEC> at(p, item);
    // (the next four elements are requested while four are computed, the first while the totals are added up; left: pixels from the thread's next one to the part's end)
    constexpr int PIX = kPixels<VEC>;
    const long step_x = at.TY * p.ldx, step_y = at.TY * p.ldy, pixel = at.s * p.positions + at.p0 + at.ty;
    const float* x = p.x + pixel * p.ldx + at.c0;
    long out = pixel * p.ldy + at.c0;
    int left = at.active ? (int)(at.p1 - at.p0) - at.ty : 0;
    float e1[4], claims1[4];
    const auto request = [&]() __attribute__((always_inline)) {
        load_quad<VEC, true>(x, [&](int j) { return j == 0 ? 0 : plain(j * at.TY < left ? j * step_x : 0); }, e1);
        sink.template request<VEC>([&](int j) { return j == 0 ? out : plain(j * at.TY < left ? out + j * step_y : out); }, claims1);
    };
    if (left > 0) request();
    // (totals first, then a thread a group: a chain of dependent operations, run once for all groups)
    group_totals<true>(p, at, [&](int g, const double2& t, const double2& d) __attribute__((always_inline)) { coef[g].mu = t.x; coef[g].r = t.y; coef[g].K1 = d.x; coef[g].K0 = d.y; });
    __syncthreads();
    for (int g = thread_here(); g < at.g_hi - at.g_lo; g += kNormThreads) {
        const GroupCoef t = coef[g];
        coef[g] = group_coef(p.k, p.n, t.mu, t.r, t.K1, t.K0);
    }
    __syncthreads();
    if (!at.active) return;
    ChannelCoef ch[VEC];
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
        const GroupCoef g = coef[(at.c0 + c) / p.per - at.g_lo];
        ch[c] = channel_coef(p, g, at.c0 + c);
    }
    while (left > 0) {
        float e[4], claims[4], ref[4], y[4], t[4];
        const long here = out;
        const int now = left;
        const auto place = [&](int j) { return j == 0 ? here : plain(j * at.TY < now ? here + j * step_y : here); };
#pragma unroll
        for (int c = 0; c < 4; ++c) { e[c] = e1[c]; claims[c] = claims1[c]; }
        sink.template reference<VEC>(place, ref);
        left -= PIX * at.TY; x += PIX * step_x; out += PIX * step_y;
        if (left > 0) request();
#pragma unroll
        for (int c = 0; c < 4; ++c) norm_element<ACT>(e[c], ch[c % VEC], p, y[c], t[c]);
        const int vectors = now > (PIX - 1) * at.TY ? PIX : (now + at.TY - 1) / at.TY;
        sink.template put<VEC>(place, vectors, y, t, claims, ref);
    }
}
template <int ACT, int VEC>
__global__ __launch_bounds__(kNormThreads) void norm_apply(NormArgs p) {
    extern __shared__ GroupCoef coef[];
    NormStore sink{p.y, p.tau};
    norm_part<ACT, VEC>(p, blockIdx.x, coef, sink);
}
// checked on the spot: workgroups of the streaming check, which take the parts in turn
template <int ACT, int VEC, bool REF>
__global__ __launch_bounds__(kCheckThreads) void norm_act_check(NormCheckArgs) {
    __shared__ CheckShared chk;
    extern __shared__ GroupCoef coef[];
    clear_check(chk);
    const NormCheckArgs& a = args_here<NormCheckArgs>();
    NormCheck<REF> sink(a, chk.hist, &chk.largest);
    for (long it = blockIdx.x; it < a.items; it += gridDim.x) {
        norm_part<ACT, VEC>(args_here<NormCheckArgs>().p, it, coef, sink);
        __syncthreads();                                     // (the coefficients are replaced)
    }
    sink.finish();
    __syncthreads();
    finish_pass(chk.hist, sink.acc, chk.red, args_here<NormCheckArgs>().pass);
}

// Parts of a sample: pixel parts, each for every column block, as many as the chip's 256 compute units hold a workgroup each of in one round (from 129 column blocks of
// all samples on one part each, which leaves units idle up to 256); of two trips of a workgroup over its pixels at least (2 x 4096 x 320 with SiLU 28 us, of eight 33).  The
// number of units is written out: the parts decide the workspace, whose size is asked for where there may be no device, or another than that of the call.
struct NormParts { int ncb, pixel_parts, span; long pixels; };
static int channel_vec(long channels) { return channels % 4 == 0 ? 4 : channels % 2 == 0 ? 2 : 1; }
static NormParts norm_parts(long batch, long positions, long channels, long groups) {
    const int ncb = (int)((channels + kColumns - 1) / kColumns);
    const long ty = kNormThreads / ((channels < kColumns ? channels : kColumns) / channel_vec(channels)), cus = 256;
    long want = cus / (batch * ncb);
    const long most = (positions + 2 * ty - 1) / (2 * ty);
    want = want < 1 ? 1 : want > most ? most : want;
    NormParts r;
    r.ncb = ncb;
    r.pixels = (positions + want - 1) / want;
    r.pixel_parts = (int)((positions + r.pixels - 1) / r.pixels);
    r.span = (int)std::min<long>(ncb, (channels / groups + kColumns - 2) / kColumns + 1);      // (a group's first channel is the last of a block at worst)
    return r;
}
// Whether one workgroup a group does: groups of at most two vectors a thread; no more than two workgroups a compute unit, as each walks through its sums and its outputs on
// its own; and little work in all, or pixels of 64 bytes a group at least (lines that are not shared out).  GPU us, norm_rows / the three passes, bound and check: 2 x 64 x 1280 in
// 32 groups 7.4 / 19 and 13 / 26, 2 x 256 x 1024 11.5 / 19 and 18 / 26, 16 x 256 x 256 9.7 / 19 and 20 / 26, 16 x 256 x 1024 20 / 31 and 30 / 36; beyond,
// 2 x 256 x 2048 20 / 20 and 39 / 30, 16 x 1024 x 128 38 / 21 and 32 / 31, 64 x 16 x 256 in 64 14 / 16 and 78 / 22.
static bool holds_row(long batch, long positions, long channels, long groups) {
    const long per = channels / groups, vectors = per / channel_vec(per) * positions, rows = batch * groups;
    return vectors <= kRowVectors * kNormThreads && rows <= 512 && (rows * vectors <= 1 << 18 || per >= 16);
}
static bool norm_shape_ok(long batch, long positions, long channels, long groups) {
    if (batch < 0 || positions < 0 || channels < 0 || groups < 1 || channels % groups) return false;
    const long lim = 1L << 31;
    if (batch >= lim || positions >= lim || channels >= lim) return false;
    if ((__int128)batch * groups >= (1L << 22) || (__int128)batch * ((channels + kColumns - 1) / kColumns) >= (1L << 22)) return false;      // workgroups of a launch
    return (__int128)(channels / groups) * positions < lim && (__int128)batch * positions * channels < ((__int128)1 << 36);
}
static size_t sums_bytes(long batch, long positions, long channels, long groups) {
    if (!norm_shape_ok(batch, positions, channels, groups) || batch * positions * channels == 0 || holds_row(batch, positions, channels, groups)) return 0;
    const NormParts r = norm_parts(batch, positions, channels, groups);
    return (size_t)batch * (size_t)groups * (size_t)r.span * (size_t)r.pixel_parts * 2 * sizeof(double2);
}

// Checks the arguments that the two entry points share and fills the kernels'.
static int norm_setup(int act, const float* x, const float* gamma, const float* beta, double eps, long batch, long positions, long channels,
                      long groups, long ldx, long ldy, const tao_fp_model* model, tao_fp_model* md, NormArgs* out) {
    int rc = resolve_model(model, md);
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
    rc = make_consts(*md, n > 0 ? n : 1, eps, &p.k, true);
    if (rc != TAO_OK) return rc;
    const double f = silu_factor(*md);
    if (!(f < 0.5)) return TAO_ERR_MODEL;
    const double k = widen(f / (1.0 - f)), own = act == TAO_ACT_SILU ? 1.0 + k : 1.0;
    p.grow_ep = (1.0 + md->u) * own * kUp; p.grow_p = md->u * own * kUp;
    p.quarter = (0.25 + 0x1p-23) / own; p.silu_k = k * kUp;
    p.x = x; p.gamma = gamma; p.beta = beta;
    p.batch = batch; p.positions = positions; p.ldx = ldx; p.ldy = ldy;
    p.channels = (int)channels; p.groups = (int)groups; p.per = (int)per; p.n = (double)n;
    if (n > 0 && batch > 0) {
        const NormParts r = norm_parts(batch, positions, channels, groups);
        p.ncb = r.ncb; p.pixel_parts = r.pixel_parts; p.span = r.span; p.pixels = r.pixels;
    }
    return TAO_OK;
}
// LDS for what the last two passes keep of the groups that a column block can touch: one a channel, or all there are.
static size_t block_lds(const NormArgs& p, size_t each) {
    return (size_t)(p.groups < kColumns ? p.groups : kColumns) * each;
}
// The sums of all groups, left in p.part.
template <int VEC>
static void sums_launch(const NormArgs& p, hipStream_t st) {
    const dim3 grid((unsigned)(p.batch * p.pixel_parts * p.ncb)), blk(kNormThreads);
    hipLaunchKernelGGL((norm_sums<VEC, false>), grid, blk, 0, st, p);
    hipLaunchKernelGGL((norm_sums<VEC, true>), grid, blk, 0, st, p);
}
static void norm_sums_launch(const NormArgs& p, hipStream_t st) {
    const int vec = channel_vec(p.channels);
    if (vec == 4)      sums_launch<4>(p, st);
    else if (vec == 2) sums_launch<2>(p, st);
    else               sums_launch<1>(p, st);
}
template <int ACT, int VEC>
static void rows_launch(const NormArgs& p, hipStream_t st) {
    const dim3 grid((unsigned)((p.batch * p.groups + 7) / 8 * 8));
    const long vectors = (long)p.per / VEC * p.positions;
    // (320 vectors: 6.3 us with 256 threads, 6.5 with 1024; 640: 8.0 and 7.5)
    if (vectors <= 2 * 256)               hipLaunchKernelGGL((norm_rows<ACT, VEC, 2, 256>), grid, dim3(256), 0, st, p);
    else                                  hipLaunchKernelGGL((norm_rows<ACT, VEC, kRowVectors, kNormThreads>), grid, dim3(kNormThreads), 0, st, p);
}
template <int ACT>
static void norm_launch(const NormArgs& p, hipStream_t st) {
    if (holds_row(p.batch, p.positions, p.channels, p.groups)) {
        const int vec = channel_vec(p.per);
        if (vec == 4)      rows_launch<ACT, 4>(p, st);
        else if (vec == 2) rows_launch<ACT, 2>(p, st);
        else               rows_launch<ACT, 1>(p, st);
        return;
    }
    norm_sums_launch(p, st);
    const dim3 grid((unsigned)(p.batch * p.pixel_parts * p.ncb)), blk(kNormThreads);
    const size_t lds = block_lds(p, sizeof(GroupCoef));
    const int vec = channel_vec(p.channels);
    if (vec == 4)      hipLaunchKernelGGL((norm_apply<ACT, 4>), grid, blk, lds, st, p);
    else if (vec == 2) hipLaunchKernelGGL((norm_apply<ACT, 2>), grid, blk, lds, st, p);
    else               hipLaunchKernelGGL((norm_apply<ACT, 1>), grid, blk, lds, st, p);
}
template <int ACT, bool REF>
static int norm_check_launch(NormArgs& p, const CheckWorkspace& w, long n, double alpha, double eps_rel, tao_profile* out, hipStream_t st) {
    const bool rows = n == 0 || holds_row(p.batch, p.positions, p.channels, p.groups);
    const long items = n == 0 ? 0 : p.batch * (rows ? p.groups : (long)p.pixel_parts * p.ncb);
    const int nblocks = (int)(items < 1 ? 1 : items < kMaxCheckBlocks ? items : kMaxCheckBlocks);
    if (n == 0) p.batch = 0;                                 // (no row is taken)
    const NormCheckArgs a = {p, items, alpha, eps_rel, pass_out(w, nblocks, n, out)};
    const dim3 grid((unsigned)nblocks), blk(kCheckThreads);
    if (rows) {
        const int vec = channel_vec(p.per);
        if (vec == 4)      hipLaunchKernelGGL((norm_rows_check<ACT, 4, REF>), grid, blk, 0, st, a);
        else if (vec == 2) hipLaunchKernelGGL((norm_rows_check<ACT, 2, REF>), grid, blk, 0, st, a);
        else               hipLaunchKernelGGL((norm_rows_check<ACT, 1, REF>), grid, blk, 0, st, a);
    } else {
        norm_sums_launch(p, st);
        const size_t lds = block_lds(p, sizeof(GroupCoef));
        // (two channels a thread: the coefficients of four leave no registers for the check)
        if (p.channels % 2 == 0) hipLaunchKernelGGL((norm_act_check<ACT, 2, REF>), grid, blk, lds, st, a);
        else                     hipLaunchKernelGGL((norm_act_check<ACT, 1, REF>), grid, blk, lds, st, a);
    }
    return nblocks;
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
    tao_fp_model md;
    const int rc = norm_setup(act, x, gamma, beta, eps, batch, positions, channels, groups, ldx, ldy, model, &md, &p);
    if (rc != TAO_OK) return rc;
    if (batch * positions * channels == 0) return TAO_OK;
    if (!y && !tau) return TAO_ERR_NULL;
    if (!aligned(y, 4) || !aligned(tau, 4)) return TAO_ERR_ALIGN;
    const size_t need = sums_bytes(batch, positions, channels, groups);
    if (need > 0 && (!ws || !aligned(ws, 256) || ws_bytes < need)) return TAO_ERR_WORKSPACE;
    p.y = y; p.tau = tau; p.part = static_cast<double2*>(ws);
    hipStream_t st = (hipStream_t)stream;
    if (act == TAO_ACT_SILU)      norm_launch<TAO_ACT_SILU>(p, st);
    else if (act == TAO_ACT_RELU) norm_launch<TAO_ACT_RELU>(p, st);
    else                          norm_launch<TAO_ACT_EXACT>(p, st);
    return launch_status();
}

int tao_bound_check_groupnorm_act(int act, const float* x, const float* gamma, const float* beta, double eps, const float* y_ref,
                                  const float* claimed, long batch, long positions, long channels, long groups, long ldx, long ldy,
                                  double alpha, double eps_rel, const tao_fp_model* model, tao_profile* out,
                                  void* ws, size_t ws_bytes, void* stream) {
    using namespace tao;
    NormArgs p;
    tao_fp_model md;
    const int rc = norm_setup(act, x, gamma, beta, eps, batch, positions, channels, groups, ldx, ldy, model, &md, &p);
    if (rc != TAO_OK) return rc;
    if (!out || !ws) return out ? TAO_ERR_WORKSPACE : TAO_ERR_NULL;
    if (!(alpha >= 0.0) || !std::isfinite(alpha) || !(eps_rel >= 0.0) || !std::isfinite(eps_rel)) return TAO_ERR_SHAPE;
    const long n = batch * positions * channels;
    if (n > 0 && !claimed) return TAO_ERR_NULL;
    if (!aligned(y_ref, 4) || !aligned(claimed, 4) || !aligned(out, 8)) return TAO_ERR_ALIGN;
    if (!aligned(ws, 256) || ws_bytes < check_workspace_bytes() + sums_bytes(batch, positions, channels, groups)) return TAO_ERR_WORKSPACE;
    p.y_ref = y_ref; p.claimed = claimed;
    p.part = reinterpret_cast<double2*>(static_cast<char*>(ws) + check_workspace_bytes());
    p.k.quick_alpha = quick_alpha(alpha, md);
    hipStream_t st = (hipStream_t)stream;
    const CheckWorkspace w = carve_check_workspace(ws);
    const auto launch = [&](auto kind) { return y_ref ? norm_check_launch<decltype(kind)::value, true>(p, w, n, alpha, eps_rel, out, st)
                                                      : norm_check_launch<decltype(kind)::value, false>(p, w, n, alpha, eps_rel, out, st); };
    const int nblocks = act == TAO_ACT_SILU   ? launch(std::integral_constant<int, TAO_ACT_SILU>())
                        : act == TAO_ACT_RELU ? launch(std::integral_constant<int, TAO_ACT_RELU>())
                                              : launch(std::integral_constant<int, TAO_ACT_EXACT>());
    launch_finish(w, nblocks, n, out, st);
    return launch_status();
}

}  // extern "C"
