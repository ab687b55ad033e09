// tao_bound_rope_tables, tao_bound_norm_rope, tao_bound_check_norm_rope: the tables of the rotary embedding from positions and frequencies, and the
// RMS norm of every query and key head with the rotation of its first elements, re-executed and bounded in one call (operators of App. A.3; primitive
// rule of Sec. 3.1, Gamma(n-1) and Gamma(2) for the reductions).
#include <type_traits>
#include "tao_check.hpp"
#include "tao_device.hpp"
#include "tao_host.hpp"
#include "tao_rows.hpp"

namespace tao {

// ---- tables: c = m cos(p f), its bound K1 B + K2 |cos|, B = min(|sin| E + E^2/2, E, 1 + |cos|), E = Gamma(d)|p f|: what an angle off by E moves the
// function by, the function's own error and m's rounding in K1 and K2.
struct TableArgs {
    const int64_t* positions; const float* inv_freq;
    float* out[4];                   // cos, sin, their bounds; any may be null
    long npos; int half;
    double m, e1, e2, whole;         // Gamma(1), Gamma(2); positions up to `whole` are not rounded
    double k1[2], k2[2];             // of cos, of sin
    float q1[2], q2[2];              // the same in binary32
    float near;                      // E up to which bounds are formed from those: Gamma(1) 2^45, or 0
};

// cos and sin of t + lost, |t| < 2^50, lost what t's own rounding left off: t less the nearest multiple k of pi/2 (two parts of pi/2 in fused steps: the first difference is exact, as t
// and k times the first part are multiples of 2^-52 where k is not 0), then lost, which next to a multiple of pi/2 may be most of what remains; then polynomials on |r| <= pi/4 of degree 11 and 12,
// for (sin r / r - 1) / r^2 and (cos r - 1 + r^2/2) / r^4 fitted in extended precision at 400 Chebyshev points of r^2 with weights that even out the largest errors: 2^-45 relatively
// (Taylor's of that degree 2^-37; two terms more took 1 us of 28 at 131072 x 64).  k is the nearest to t (1 + 2^-53.8) / (pi/2), and lost lies outside: |r| <= pi/4 + 2^-53.8 |t| + |lost|, below 0.8
// up to angles of 2^45 (2^-43.7 there) and 1.05 at 2^50 (2^-34).
__device__ __forceinline__ void cos_sin(double t, double lost, double& c, double& s) {
    const double at = fma(t, 0x1.45f306dc9c883p-1, 0x1.8p52), k = at - 0x1.8p52;         // (k in the last bits of the sum)
    const double r = fma(-k, 0x1.1a62633145c07p-54, fma(-k, 0x1.921fb54442d18p+0, t)) + lost, z = r * r;
    double ps = -0x1.aa288026d8c33p-26, pc = 0x1.1c81d7955fe06p-29;
    ps = fma(ps, z, 0x1.71d9aa58557b2p-19);   pc = fma(pc, z, -0x1.27e25f7db439cp-22);
    ps = fma(ps, z, -0x1.a019fd9bd07dap-13);  pc = fma(pc, z, 0x1.a019ff53f3bf3p-16);
    ps = fma(ps, z, 0x1.1111110fd4207p-7);    pc = fma(pc, z, -0x1.6c16c16b6175dp-10);
    ps = fma(ps, z, -0x1.555555555516dp-3);   pc = fma(pc, z, 0x1.5555555555437p-5);
    const double sr = fma(ps * z, r, r);
    const double cr = fma(fma(pc, z, -0.5), z, 1.0);
    const int q = __double2loint(at) & 3;
    s = q & 1 ? cr : sr; c = q & 1 ? sr : cr;
    if (q & 2) s = -s;
    if ((q + 1) & 2) c = -c;
}
// An element from the angle t = p f, with bounds in binary32, whose operations take half the time of binary64's: from E, c and s, an u each off, the sums of positive terms are 6u off at most; (1 + 8u)
// above them they are at or above their formulas and less than 16u < 1e-6 from them (131072 x 64: 26 us, 32.6 in binary64 with the argument's multiple of pi/2 converted to a whole number).
// False where that does not hold, and table_element has to form the element:
//  - bounds below 2^-60 (angles next to 0 where c_cos or c_sin is 0 or u or m small): what is lost below 2^-126 on the way is less than 2^-28 of the others (factors up to 2^60);
//  - positions from 2^29 on: below, p f has 53 bits at most and is exact; there what the product leaves off, 2^-53 |t|, moves tables, bounds of 1 + |cos| or 1 + |sin|, and those next to a multiple of pi/2;
//  - angles from about 2^45 on, which may be none (2^50).
__device__ __forceinline__ bool table_element_near(const TableArgs& a, int64_t n, double f, float (&v)[4]) {
    const double p = (double)n, t = p * f, e = (fabs(p) > a.whole ? a.e2 : a.e1) * fabs(t);
    double c, s;
    cos_sin(t, 0.0, c, s);
    v[0] = (float)(a.m * c); v[1] = (float)(a.m * s);
    const float ac = fabsf((float)c), as = fabsf((float)s), E = (float)e, e2 = 0.5f * E * E;
    const float bc = fminf(fminf(fmaf(as, E, e2), E), 1.f + ac), bs = fminf(fminf(fmaf(ac, E, e2), E), 1.f + as);
    v[2] = fmaf(a.q1[0], bc, a.q2[0] * ac) * (1.f + 0x1p-21f); v[3] = fmaf(a.q1[1], bs, a.q2[1] * as) * (1.f + 0x1p-21f);
    return fminf(v[2], v[3]) >= 0x1p-60f && E < a.near && fabs(p) < 0x1p29;
}
__device__ __forceinline__ void table_element(const TableArgs& a, int64_t n, double f, float (&v)[4]) {
    double p = (double)n, low = 0.0;                         // the position is p + low exactly
    if (fabs(p) >= 0x1p53) {
        if (p >= 0x1p63) p = 0x1.fffffffffffffp62;           // (2^63 is no int64)
        low = (double)(n - (int64_t)p);
    }
    const double t = p * f, e = (fabs(p) > a.whole || (fabs(p) == a.whole && p * low > 0.0) ? a.e2 : a.e1) * fabs(t);
    double c, s;
    cos_sin(t, fma(low, f, fma(p, f, -t)), c, s);
    const double ac = fabs(c), as = fabs(s), e2 = 0.5 * e * e;
    const double bc = fmin(fmin(fma(as, e, e2), e), 1.0 + ac), bs = fmin(fmin(fma(ac, e, e2), e), 1.0 + as);
    v[0] = (float)(a.m * c); v[1] = (float)(a.m * s);
    v[2] = up32g(fma(a.k1[0], bc, a.k2[0] * ac)); v[3] = up32g(fma(a.k1[1], bs, a.k2[1] * as));
    if (!(fabs(t) < 0x1p50)) { v[0] = v[1] = v[2] = v[3] = NAN; }
}
// The elements whose bits are set in `left` of VEC, one after the other (in line for each, they cost the common way registers: 2^20 x 16 48.6 us, 42.7 so); at(e, n, f): element e's position and frequency.
template <int VEC, class At>
__device__ __forceinline__ void table_elements_left(const TableArgs& a, unsigned left, float (&v)[VEC][4], At&& at) {
#pragma unroll 1
    while (left) {
        const int e = __builtin_ctz(left);
        left &= left - 1;
        int64_t n;
        double f;
        at(e, n, f);
        float w[4];
        table_element(a, n, f, w);
#pragma unroll
        for (int k = 0; k < VEC; ++k)
#pragma unroll
            for (int o = 0; o < 4; ++o) v[k][o] = k == e ? w[o] : v[k][o];
    }
}
// A thread has VEC neighbouring frequencies of a position: 16-byte stores where rows are whole vectors.  What bounds long tables: their bytes (16 an element)
// and, hardly less, 35 binary64 operations an element: 131072 x 64 in 26 us, 5.2 TB/s; one frequency a thread 46.
template <int VEC>
__global__ __launch_bounds__(256) void rope_tables(TableArgs a) {
    const unsigned per = (unsigned)a.half / VEC;
    const long n = a.npos * per, stride = (long)gridDim.x * 256;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += stride) {
        const long r = n < (1L << 32) ? (long)((unsigned)i / per) : i / per;
        const int j = (int)(i - r * per) * VEC;
        const int64_t p = a.positions ? a.positions[r] : r;
        float v[VEC][4];
        unsigned left = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) left |= table_element_near(a, p, (double)a.inv_freq[j + e], v[e]) ? 0u : 1u << e;
        table_elements_left<VEC>(a, left, v, [&](int e, int64_t& at, double& f) __attribute__((always_inline)) { at = p; f = (double)a.inv_freq[j + e]; });
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            if (!a.out[o]) continue;
            if constexpr (VEC == 4) ntstore4(reinterpret_cast<float4*>(a.out[o] + i * 4), make_float4(v[0][o], v[1][o], v[2][o], v[3][o]));
            else a.out[o][i] = v[0][o];
        }
    }
}
// Rows of other lengths: four neighbouring elements of the whole table a thread, over the ends of rows (131072 x 63 25.3 us; one element a thread 35.7 where this took 29.0, 2^23 x 1 39.2 and 34.4).
__global__ __launch_bounds__(256) void rope_tables_flat(TableArgs a) {
    const long n = a.npos * a.half, stride = (long)gridDim.x * 1024;
    for (long i = ((long)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += stride) {
        long r = n < (1L << 32) ? (long)((unsigned)i / (unsigned)a.half) : i / a.half;
        int j = (int)(i - r * a.half);
        int64_t p = a.positions ? a.positions[r] : r;
        float v[4][4];
        unsigned left = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e > 0 && ++j == a.half) {
                j = 0;
                ++r;
                if (r < a.npos) p = a.positions ? a.positions[r] : r;             // (what lies behind the last row is not stored)
            }
            left |= table_element_near(a, p, (double)a.inv_freq[j], v[e]) ? 0u : 1u << e;
        }
        table_elements_left<4>(a, left, v, [&](int e, int64_t& at, double& f) __attribute__((always_inline)) {
            const long k = i + e < n ? i + e : 0, row = k / a.half;
            at = a.positions ? a.positions[row] : row;
            f = (double)a.inv_freq[k - row * a.half];
        });
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            if (!a.out[o]) continue;
            if (i + 4 <= n) {
                ntstore4(reinterpret_cast<float4*>(a.out[o] + i), make_float4(v[0][o], v[1][o], v[2][o], v[3][o]));
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (i + e < n) a.out[o][i + e] = v[e][o];
            }
        }
    }
}

// ---- norm and rotation of heads
struct HeadArgs {
    const float* x; const float* gain[2];
    const float* c; const float* s; const float* tc; const float* ts;
    const int64_t* positions;
    float* y; float* tau;
    const float* y_ref; const float* claimed;
    long tokens, npos, ldt, ldh, ldyt, ldyh;
    int heads_q, heads, d, rot;
    bool interleaved, norm;
    RowConsts k;
    double g2, uflow;                // Gamma(2), 2 2^-149 or 0
    double norm_fy;                  // u (1 + u)^2
};
// What a head's sum of squares gives: r, F (an element's error is F |x g|), k of the rotation, and the factors of the final rounding.  The chain of rsqrt_tail with inverse roots from
// v_rsq_f64 (2^-24) and two Newton steps in place of its roots and divisions (a few 2^-53, far inside the margin): it is run for every head by all lanes that have one.
struct HeadCoef { double r, F, k, mul, sub; };
__device__ __forceinline__ double inverse_root(double w) {
    double r = __builtin_amdgcn_rsq(w);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = fma(r * 0.5, fma(-w * r, r, 1.0), r);
    return r;
}
__device__ __forceinline__ HeadCoef head_coef(const HeadArgs& a, double squares) {
    HeadCoef h{1.0, 0.0, a.g2, kUpMul, 1.0 + 0x1p-46};
    if (a.norm) {
        const RowConsts& k = a.k;
        const double E_t = (k.G * (1.0 + k.u) + k.u) * squares, vstar = squares * k.inv_n;
        const double E_v = (E_t * k.inv_n + k.cd_u * vstar) * k.inv1mcd;
        const double w = vstar + k.eps, E_w = (E_v + k.u * w) * k.inv1mu, w_lo = w - E_w, s = inverse_root(w_lo);
        const double E_r = fma(0.5 * E_w, s * s * s, k.cr_u * s), amp = (w + E_w) * s * s;
        h.r = inverse_root(w);
        const double R = h.r + E_r;
        h.F = w_lo > 0.0 ? E_r + k.u * R + a.norm_fy * R : NAN;
        h.k = fma(a.g2, h.r + h.F, h.F);
        const UpFactors up(k.m * (1.0 + 2.0 * amp));
        h.mul = up.mul; h.sub = up.sub;
    }
    return h;
}
// (a bound that is infinite in binary64 comes of an infinite operand: it would admit every finite claim)
__device__ __forceinline__ float head_bound(double e, const HeadCoef& h) {
    float f = (float)(e * h.mul);
    if (!(f >= 0x1p-126f && f < INFINITY)) f = e < INFINITY ? up32g(e, h.mul, h.sub) : NAN;
    return f;
}
// The two elements of a pair: ha, hb are x g.
template <bool ERRORS>
__device__ __forceinline__ void rotate_pair(const HeadArgs& a, const HeadCoef& h, double ha, double hb, float c, float s, float tc, float ts,
                                            float& ya, float& yb, float& ta, float& tb) {
    const double C = (double)c, S = (double)s;
    double kc = h.k * fabs(C), ks = h.k * fabs(S);
    if constexpr (ERRORS) {
        const double ec = fabs((double)tc), es = fabs((double)ts), more = h.k + h.r;
        kc = fma(more, ec, kc); ks = fma(more, es, ks);
    }
    ya = (float)(h.r * fma(ha, C, -(hb * S))); yb = (float)(h.r * fma(hb, C, ha * S));
    ta = head_bound(fma(fabs(ha), kc, fabs(hb) * ks) + a.uflow, h);
    tb = head_bound(fma(fabs(hb), kc, fabs(ha) * ks) + a.uflow, h);
}
// (without a norm F is 0, and what is not finite has NaN for its bound)
__device__ __forceinline__ void plain_element(const HeadCoef& h, double hx, float& y, float& t) {
    y = (float)(h.r * hx);
    t = head_bound(h.F * fabs(hx), h);
}
// Sums over TEAM lanes, in every one of them.
template <int TEAM>
__device__ __forceinline__ double team_sum(double v) {
    constexpr int STEPS = TEAM == 4 ? 2 : TEAM == 8 ? 3 : TEAM == 16 ? 4 : TEAM == 32 ? 5 : 6;
    return wave_all<0, STEPS>(v, [](double p, double q) { return p + q; });
}

struct HeadStore {
    float* y; float* tau;
    __device__ __forceinline__ void put1(long i, float yv, float tv) {
        if (y) y[i] = yv;
        if (tau) tau[i] = tv;
    }
};
struct HeadCheck {
    const float* y_ref; const float* claimed; double alpha, eps_rel; unsigned int* hist; int rep; ThreadAcc acc;
    __device__ __forceinline__ void put1(long i, float yv, float tv) { check_one(claimed[i], y_ref ? y_ref[i] : yv, tv, alpha, eps_rel, hist, rep, acc); }
};
// Any size, stride and layout: a wavefront a head, element by element, x read twice.  (For heads of more than 512 elements, and 2^31 heads and more.)
template <class Sink>
__device__ __forceinline__ void head_any(const HeadArgs& a, long row, Sink& sink) {
    const int lane = threadIdx.x & (kWave - 1), half = a.rot >> 1;
    const long t = row / a.heads;
    const int head = (int)(row - t * a.heads);
    const float* x = a.x + t * a.ldt + head * a.ldh;
    const float* g = a.gain[head >= a.heads_q];
    const long out = t * a.ldyt + head * a.ldyh;
    double sum = 0.0;
    if (a.norm) {
        for (int j = lane; j < a.d; j += kWave) sum = fma((double)x[j], (double)x[j], sum);
        sum = team_sum<64>(sum);
    }
    const HeadCoef h = head_coef(a, sum);
    auto at = [&](int j) __attribute__((always_inline)) { return (double)x[j] * (g ? (double)g[j] : 1.0); };
    const long p = a.positions ? a.positions[t] : a.npos > 0 ? t % a.npos : 0;
    const bool inside = p >= 0 && p < a.npos;
    for (int j = lane; j < half; j += kWave) {
        const int ja = a.interleaved ? 2 * j : j, jb = a.interleaved ? 2 * j + 1 : j + half;
        const long e = p * half + j;
        float ya, yb, ta, tb;
        rotate_pair<true>(a, h, at(ja), at(jb), inside ? a.c[e] : NAN, inside ? a.s[e] : NAN, inside && a.tc ? a.tc[e] : 0.f, inside && a.ts ? a.ts[e] : 0.f, ya, yb, ta, tb);
        sink.put1(out + ja, ya, ta);
        sink.put1(out + jb, yb, tb);
    }
    for (int j = a.rot + lane; j < a.d; j += kWave) {
        float y, tau;
        plain_element(h, at(j), y, tau);
        sink.put1(out + j, y, tau);
    }
}
__global__ __launch_bounds__(256) void heads_any(HeadArgs a) {
    HeadStore sink{a.y, a.tau};
    const long rows = a.tokens * a.heads;
    for (long row = (long)blockIdx.x * 4 + threadIdx.x / kWave; row < rows; row += (long)gridDim.x * 4) head_any(a, row, sink);
}
__global__ __launch_bounds__(kCheckThreads) void heads_any_check(HeadArgs a, double alpha, double eps_rel, PassOut pass) {
    __shared__ unsigned int hist[kBins * kReplicas];
    __shared__ unsigned int red[kRedWords];
    for (int i = threadIdx.x; i < kBins * kReplicas; i += kCheckThreads) hist[i] = 0;
    __syncthreads();
    HeadCheck sink{a.y_ref, a.claimed, alpha, eps_rel, hist, (int)(threadIdx.x & (kReplicas - 1)), ThreadAcc()};
    const long rows = a.tokens * a.heads;
    constexpr int WAVES = kCheckThreads / kWave;
    for (long row = (long)blockIdx.x * WAVES + threadIdx.x / kWave; row < rows; row += (long)gridDim.x * WAVES) head_any(a, row, sink);
    finish_pass(hist, sink.acc, red, pass);
}

// ---- heads of whole vectors: d and rot multiples of 8, on 16-byte addresses, up to 512 elements.  TEAM lanes a head; lane j has two vectors of four elements: those from 4 j and from rot / 2 + 4 j on
// of the rotated ones, with entries 4 j of the tables; lanes from rot / 8 on have those of the two halves of the rest.  Where pairs are neighbours any vectors do: those of the head's two halves.  So
// neighbouring lanes have neighbouring vectors (two vectors of one lane next to each other, every store fills half a line: 2048 x 40 heads of 128 with neighbouring pairs 45 us, 23 so).  A head stays in registers, so x is read once.
// What bounds it: HBM for many heads (12 bytes an element), launches for few.
struct HeadPlace { const float* x; const float* g; long out, table; bool inside; };
__device__ __forceinline__ HeadPlace head_place(const HeadArgs& a, unsigned row) {
    const unsigned t = row / (unsigned)a.heads, head = row - t * (unsigned)a.heads;
    const long p = a.positions ? a.positions[t] : a.npos > 0x7fffffffL ? (long)t : (long)(t % (unsigned)a.npos);
    const bool inside = p >= 0 && p < a.npos;
    return HeadPlace{a.x + t * a.ldt + head * a.ldh, a.gain[head >= (unsigned)a.heads_q], t * a.ldyt + head * a.ldyh, inside ? p * (a.rot >> 1) : 0, inside};
}
template <bool INTER>
__device__ __forceinline__ void item_offsets(const HeadArgs& a, int j, int& first, int& second) {
    const int plain = a.d - a.rot;
    if (INTER)              { first = 4 * j; second = first + (a.d >> 1); }
    else if (8 * j < a.rot) { first = 4 * j; second = first + (a.rot >> 1); }
    else                    { first = (a.rot >> 1) + 4 * j; second = first + (plain >> 1); }
}
__device__ __forceinline__ floatv4 vector_at(const float* p) { return *reinterpret_cast<const floatv4*>(p); }
typedef float floatv2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ floatv2 two_at(const float* p) { return *reinterpret_cast<const floatv2*>(p); }
__device__ __forceinline__ floatv4 stream_at(const float* p) { return __builtin_nontemporal_load(reinterpret_cast<const floatv4*>(p)); }
// One item's outputs and bounds from its elements (x) and what it looks up.
template <bool INTER, bool ERRORS>
__device__ __forceinline__ void head_item(const HeadArgs& a, const HeadCoef& h, const HeadPlace& at, int j, const int (&o)[2], const floatv4 (&x)[2], floatv4 (&y)[2], floatv4 (&t)[2]) {
    double hx[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        floatv4 g = {1.f, 1.f, 1.f, 1.f};
        if (at.g) g = vector_at(at.g + o[k]);
#pragma unroll
        for (int e = 0; e < 4; ++e) hx[k][e] = (double)x[k][e] * (double)g[e];
    }
    auto plain = [&](int k) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float yv, tv;
            plain_element(h, hx[k][e], yv, tv);
            y[k][e] = yv; t[k][e] = tv;
        }
    };
    auto turn = [&](int ka, int ea, int kb, int eb, float c, float s, float tc, float ts) __attribute__((always_inline)) {
        float ya, yb, ta, tb;
        rotate_pair<ERRORS>(a, h, hx[ka][ea], hx[kb][eb], c, s, tc, ts, ya, yb, ta, tb);
        y[ka][ea] = ya; y[kb][eb] = yb; t[ka][ea] = ta; t[kb][eb] = tb;
    };
    if constexpr (INTER) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (o[k] >= a.rot) { plain(k); continue; }
            const long entry = at.table + (o[k] >> 1);
            floatv2 c = {NAN, NAN}, s = c, tc = {0.f, 0.f}, ts = tc;
            if (at.inside) {
                c = two_at(a.c + entry); s = two_at(a.s + entry);
                if (ERRORS) { tc = two_at(a.tc + entry); ts = two_at(a.ts + entry); }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) turn(k, 2 * e, k, 2 * e + 1, c[e], s[e], tc[e], ts[e]);
        }
    } else if (8 * j < a.rot) {
        const floatv4 none = {0.f, 0.f, 0.f, 0.f}, bad = {NAN, NAN, NAN, NAN};
        floatv4 c = bad, s = bad, tc = none, ts = none;
        if (at.inside) {
            c = vector_at(a.c + at.table + 4 * j); s = vector_at(a.s + at.table + 4 * j);
            if (ERRORS) { tc = vector_at(a.tc + at.table + 4 * j); ts = vector_at(a.ts + at.table + 4 * j); }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) turn(0, e, 1, e, c[e], s[e], tc[e], ts[e]);
    } else {
        plain(0); plain(1);
    }
}
template <int TEAM>
__device__ __forceinline__ HeadCoef head_chain(const HeadArgs& a, const floatv4 (&x)[2]) {
    double sum = 0.0;
    if (a.norm) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fma((double)x[k][e], (double)x[k][e], sum);
        sum = team_sum<TEAM>(sum);
    }
    return head_coef(a, sum);
}
template <int TEAM, bool INTER, bool ERRORS>
__global__ __launch_bounds__(256) void heads_rows(HeadArgs a) {
    constexpr int TEAMS = 256 / TEAM;
    const int j = threadIdx.x % TEAM;
    const bool mine = 8 * j < a.d;
    const unsigned rows = (unsigned)(a.tokens * a.heads);
    int o[2];
    item_offsets<INTER>(a, j, o[0], o[1]);
    for (unsigned row = blockIdx.x * TEAMS + threadIdx.x / TEAM; row < rows; row += gridDim.x * TEAMS) {
        const HeadPlace at = head_place(a, row);
        floatv4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        if (mine) { x[0] = stream_at(at.x + o[0]); x[1] = stream_at(at.x + o[1]); }
        const HeadCoef h = head_chain<TEAM>(a, x);
        if (!mine) continue;
        floatv4 y[2], t[2];
        head_item<INTER, ERRORS>(a, h, at, j, o, x, y, t);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (a.y) __builtin_nontemporal_store(y[k], reinterpret_cast<floatv4*>(a.y + at.out + o[k]));
            if (a.tau) __builtin_nontemporal_store(t[k], reinterpret_cast<floatv4*>(a.tau + at.out + o[k]));
        }
    }
}
// ... checked on the spot: fours of claims settled in binary32 where that is clear (settle_four).
struct HeadCheckArgs { HeadArgs a; double alpha, eps_rel; float quick; PassOut pass; };
template <int TEAM, bool INTER, bool ERRORS, bool REF>
__global__ __launch_bounds__(kCheckThreads) void heads_rows_check(HeadCheckArgs g) {
    __shared__ unsigned int hist[kBins * kReplicas];
    __shared__ unsigned int red[kRedWords];
    __shared__ unsigned int largest;
    for (int i = threadIdx.x; i < kBins * kReplicas; i += kCheckThreads) hist[i] = 0;
    if (threadIdx.x == 0) largest = 0;
    __syncthreads();
    const HeadArgs& a = g.a;
    const QuickCheck q(g.quick, g.eps_rel);
    const bool ordinary = q.eps < INFINITY && q.alpha > 0.f;
    ThreadAcc acc;
    Farthest top;
    unsigned int zeros = 0;
    const int rep = threadIdx.x & (kReplicas - 1);
    constexpr int TEAMS = kCheckThreads / TEAM;
    const int j = threadIdx.x % TEAM;
    const bool mine = 8 * j < a.d;
    const unsigned rows = (unsigned)(a.tokens * a.heads);
    int o[2];
    item_offsets<INTER>(a, j, o[0], o[1]);
    for (unsigned row = blockIdx.x * TEAMS + threadIdx.x / TEAM; row < rows; row += gridDim.x * TEAMS) {
        const HeadPlace at = head_place(a, row);
        floatv4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, c[2], r[2];
        if (mine) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                x[k] = stream_at(at.x + o[k]);
                c[k] = stream_at(a.claimed + at.out + o[k]);
                if (REF) r[k] = stream_at(a.y_ref + at.out + o[k]);
            }
        }
        const HeadCoef h = head_chain<TEAM>(a, x);
        if (!mine) continue;
        floatv4 y[2], t[2];
        head_item<INTER, ERRORS>(a, h, at, j, o, x, y, t);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            floatv4 claim = c[k], ref = REF ? r[k] : y[k], bound = t[k];
            const float most = fmaxf(fmaxf(fabsf(ref[0]), fabsf(ref[1])), fmaxf(fabsf(ref[2]), fabsf(ref[3])));      // (a NaN among them shows in the error)
            if (settle_four<true, true>(claim, ref, bound, q, top, &largest, newest(&largest), ordinary && most <= 0x1p90f, acc, zeros,
                                        [&](unsigned bin) __attribute__((always_inline)) { atomicAdd(&hist[bin * kReplicas + rep], 1u); })) continue;
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {
                check_one(claim[0], ref[0], bound[0], g.alpha, g.eps_rel, hist, rep, acc);
                claim = claim.yzww; ref = ref.yzww; bound = bound.yzww;
            }
        }
    }
    if (zeros) atomicAdd(&hist[rep], zeros);
    settled(top, g.alpha, g.eps_rel, acc);
    __syncthreads();
    finish_pass(hist, acc, red, g.pass);
}
// ---- heads of up to 512 elements of any kind, stride and address: TEAM lanes a head, each with up to PAIRS pairs of elements (two; four pairs and half the lanes 44 us for 40 at 2048 x 40 heads of 126), TEAM apart: those of the rotation, then those of the two halves of the rest.
// All of a head is requested before the first of it is used, and stays in registers.  (A wavefront a head, x read twice: 2048 x 40 heads of 126 51 us, 40 so, checked 87 and 53; 8000 x 40 of 18 149 and 36.)
template <int TEAM, int PAIRS>
struct HeadPairs {
    int ja[PAIRS], jb[PAIRS], entry[PAIRS];                  // places, -1 where there is none; entry of the tables, -1 where the pair is not rotated
    float x[PAIRS][2];
    __device__ __forceinline__ HeadPairs(const HeadArgs& a, int lane) {
        const int half = a.rot >> 1, rest = (a.d - a.rot + 1) >> 1;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const int j = lane + i * TEAM, k = j - half;
            entry[i] = k < 0 ? j : -1;
            ja[i] = k < 0 ? (a.interleaved ? 2 * j : j) : k < rest ? a.rot + k : -1;
            jb[i] = k < 0 ? (a.interleaved ? 2 * j + 1 : j + half) : k < rest && a.rot + rest + k < a.d ? a.rot + rest + k : -1;
        }
    }
    // One head's outputs and bounds.
    __device__ __forceinline__ void head(const HeadArgs& a, const HeadPlace& at, float (&y)[PAIRS][2], float (&t)[PAIRS][2]) {
        float g[PAIRS][2], c[PAIRS], s[PAIRS], tc[PAIRS], ts[PAIRS];
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            x[i][0] = ja[i] >= 0 ? at.x[ja[i]] : 0.f; x[i][1] = jb[i] >= 0 ? at.x[jb[i]] : 0.f;
            g[i][0] = at.g && ja[i] >= 0 ? at.g[ja[i]] : 1.f; g[i][1] = at.g && jb[i] >= 0 ? at.g[jb[i]] : 1.f;
            const bool turned = entry[i] >= 0 && at.inside;
            const long e = at.table + entry[i];
            c[i] = turned ? a.c[e] : NAN; s[i] = turned ? a.s[e] : NAN;
            tc[i] = turned && a.tc ? a.tc[e] : 0.f; ts[i] = turned && a.tc ? a.ts[e] : 0.f;
        }
        if (a.norm) {
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) sum = fma((double)x[i][1], (double)x[i][1], fma((double)x[i][0], (double)x[i][0], sum));
            sum = team_sum<TEAM>(sum);
        }
        const HeadCoef h = head_coef(a, sum);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const double ha = (double)x[i][0] * (double)g[i][0], hb = (double)x[i][1] * (double)g[i][1];
            if (entry[i] >= 0) {
                rotate_pair<true>(a, h, ha, hb, c[i], s[i], tc[i], ts[i], y[i][0], y[i][1], t[i][0], t[i][1]);
            } else {
                plain_element(h, ha, y[i][0], t[i][0]);
                plain_element(h, hb, y[i][1], t[i][1]);
            }
        }
    }
};
template <int TEAM, int PAIRS>
__global__ __launch_bounds__(256) void heads_pairs(HeadArgs a) {
    constexpr int TEAMS = 256 / TEAM;
    HeadPairs<TEAM, PAIRS> p(a, threadIdx.x % TEAM);
    const unsigned rows = (unsigned)(a.tokens * a.heads);
    for (unsigned row = blockIdx.x * TEAMS + threadIdx.x / TEAM; row < rows; row += gridDim.x * TEAMS) {
        const HeadPlace at = head_place(a, row);
        float y[PAIRS][2], t[PAIRS][2];
        p.head(a, at, y, t);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            if (p.ja[i] >= 0) {
                if (a.y) a.y[at.out + p.ja[i]] = y[i][0];
                if (a.tau) a.tau[at.out + p.ja[i]] = t[i][0];
            }
            if (p.jb[i] >= 0) {
                if (a.y) a.y[at.out + p.jb[i]] = y[i][1];
                if (a.tau) a.tau[at.out + p.jb[i]] = t[i][1];
            }
        }
    }
}
template <int TEAM, int PAIRS, bool REF>
__global__ __launch_bounds__(kCheckThreads) void heads_pairs_check(HeadCheckArgs g) {
    __shared__ unsigned int hist[kBins * kReplicas];
    __shared__ unsigned int red[kRedWords];
    __shared__ unsigned int largest;
    for (int i = threadIdx.x; i < kBins * kReplicas; i += kCheckThreads) hist[i] = 0;
    if (threadIdx.x == 0) largest = 0;
    __syncthreads();
    const HeadArgs& a = g.a;
    const QuickCheck q(g.quick, g.eps_rel);
    const bool ordinary = q.eps < INFINITY && q.alpha > 0.f;
    ThreadAcc acc;
    Farthest top;
    unsigned int zeros = 0;
    const int rep = threadIdx.x & (kReplicas - 1);
    constexpr int TEAMS = kCheckThreads / TEAM;
    HeadPairs<TEAM, PAIRS> p(a, threadIdx.x % TEAM);
    const unsigned rows = (unsigned)(a.tokens * a.heads);
    for (unsigned row = blockIdx.x * TEAMS + threadIdx.x / TEAM; row < rows; row += gridDim.x * TEAMS) {
        const HeadPlace at = head_place(a, row);
        float y[PAIRS][2], t[PAIRS][2], c[PAIRS][2], f[PAIRS][2];
        // (what does not exist: a claim of 1 for an output of 1, taken out of the count again)
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            c[i][0] = p.ja[i] >= 0 ? a.claimed[at.out + p.ja[i]] : 1.f; c[i][1] = p.jb[i] >= 0 ? a.claimed[at.out + p.jb[i]] : 1.f;
            if (REF) { f[i][0] = p.ja[i] >= 0 ? a.y_ref[at.out + p.ja[i]] : 1.f; f[i][1] = p.jb[i] >= 0 ? a.y_ref[at.out + p.jb[i]] : 1.f; }
        }
        p.head(a, at, y, t);
#pragma unroll
        for (int k = 0; k < PAIRS; k += 2) {
            floatv4 claim, ref, bound;
            unsigned none = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = k + e / 2;
                const bool there = (e & 1 ? p.jb[i] : p.ja[i]) >= 0;
                claim[e] = c[i][e & 1];
                ref[e] = REF ? f[i][e & 1] : there ? y[i][e & 1] : 1.f;
                bound[e] = there ? t[i][e & 1] : 0.f;
                none += there ? 0u : 1u << (8 * e);
            }
            if (p.ja[k] < 0) continue;
            const float most = fmaxf(fmaxf(fabsf(ref[0]), fabsf(ref[1])), fmaxf(fabsf(ref[2]), fabsf(ref[3])));      // (a NaN among them shows in the error)
            if (settle_four<true, true>(claim, ref, bound, q, top, &largest, newest(&largest), ordinary && most <= 0x1p90f, acc, zeros,
                                        [&](unsigned bin) __attribute__((always_inline)) { atomicAdd(&hist[bin * kReplicas + rep], 1u); })) {
                zeros -= __popc(none);
                continue;
            }
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {
                if (!(none & 1u)) check_one(claim[0], ref[0], bound[0], g.alpha, g.eps_rel, hist, rep, acc);
                claim = claim.yzww; ref = ref.yzww; bound = bound.yzww;
                none >>= 8;
            }
        }
    }
    if (zeros) atomicAdd(&hist[rep], zeros);
    settled(top, g.alpha, g.eps_rel, acc);
    __syncthreads();
    finish_pass(hist, acc, red, g.pass);
}
// Lanes of a head in those kernels, or 0 for the ones of any size.
static int pairs_team(const HeadArgs& a) {
    return a.d > 512 || a.tokens * a.heads >= (1L << 31) ? 0 : a.d <= 16 ? 4 : a.d <= 32 ? 8 : a.d <= 64 ? 16 : a.d <= 128 ? 32 : 64;
}
// f(team, pairs) with the constants of a launch
template <class F> static void pairs_dispatch(const HeadArgs& a, int team, F&& f) {
    using std::integral_constant;
    const integral_constant<int, 2> two;
    switch (team) {
        case 4:  f(integral_constant<int, 4>(), two); break;
        case 8:  f(integral_constant<int, 8>(), two); break;
        case 16: f(integral_constant<int, 16>(), two); break;
        case 32: f(integral_constant<int, 32>(), two); break;
        default: if (a.d <= 256) f(integral_constant<int, 64>(), two); else f(integral_constant<int, 64>(), integral_constant<int, 4>()); break;
    }
}
// Lanes of a head of whole vectors, or 0.  y, tau: the claims' or outputs' addresses
static int heads_team(const HeadArgs& a, const void* y, const void* tau) {
    const bool vec = a.d % 8 == 0 && a.rot % 8 == 0 && a.d <= 512 && a.tokens * a.heads < (1L << 31) && aligned(a.x, 16) && aligned(a.gain[0], 16) && aligned(a.gain[1], 16) &&
                     aligned(a.c, 16) && aligned(a.s, 16) && aligned(a.tc, 16) && aligned(a.ts, 16) && aligned(y, 16) && aligned(tau, 16) &&
                     a.ldt % 4 == 0 && a.ldh % 4 == 0 && a.ldyt % 4 == 0 && a.ldyh % 4 == 0;
    return !vec ? 0 : a.d <= 32 ? 4 : a.d <= 64 ? 8 : a.d <= 128 ? 16 : a.d <= 256 ? 32 : 64;
}
template <int TEAM, bool INTER, bool ERRORS>
static void heads_launch(const HeadArgs& a, hipStream_t st) {
    const long blocks = (a.tokens * a.heads + 256 / TEAM - 1) / (256 / TEAM);
    hipLaunchKernelGGL((heads_rows<TEAM, INTER, ERRORS>), dim3((unsigned)(blocks < 256L * 64 ? blocks : 256L * 64)), dim3(256), 0, st, a);
}
template <int TEAM, bool INTER, bool ERRORS>
static void heads_launch_check(const HeadCheckArgs& g, int nblocks, hipStream_t st) {
    if (g.a.y_ref) hipLaunchKernelGGL((heads_rows_check<TEAM, INTER, ERRORS, true>), dim3(nblocks), dim3(kCheckThreads), 0, st, g);
    else           hipLaunchKernelGGL((heads_rows_check<TEAM, INTER, ERRORS, false>), dim3(nblocks), dim3(kCheckThreads), 0, st, g);
}
// f(team, interleaved, errors) with the constants of a launch
template <class F> static void heads_dispatch(const HeadArgs& a, int team, F&& f) {
    using std::integral_constant;
    using std::bool_constant;
    auto rest = [&](auto t) {
        if (a.interleaved) { if (a.tc) f(t, bool_constant<true>(), bool_constant<true>()); else f(t, bool_constant<true>(), bool_constant<false>()); }
        else               { if (a.tc) f(t, bool_constant<false>(), bool_constant<true>()); else f(t, bool_constant<false>(), bool_constant<false>()); }
    };
    switch (team) {
        case 4:  rest(integral_constant<int, 4>()); break;
        case 8:  rest(integral_constant<int, 8>()); break;
        case 16: rest(integral_constant<int, 16>()); break;
        case 32: rest(integral_constant<int, 32>()); break;
        default: rest(integral_constant<int, 64>()); break;
    }
}

// Checks the arguments that the two entry points share and fills the kernels'.
static int heads_setup(int norm, const float* x, const float* gamma_q, const float* gamma_k, double eps, const float* cos_table, const float* sin_table,
                       const float* tau_cos, const float* tau_sin, const int64_t* positions, long tokens, long heads_q, long heads_k, long d, long rot, long npos,
                       long ldt, long ldh, long ldyt, long ldyh, int interleaved, const tao_fp_model* model, tao_fp_model* md, HeadArgs* out) {
    int rc = resolve_model(model, md);
    if (rc != TAO_OK) return rc;
    if ((norm != TAO_NORM_RMSNORM && norm != TAO_NORM_NONE) || (norm == TAO_NORM_NONE && (gamma_q || gamma_k))) return TAO_ERR_KIND;
    if (tokens < 0 || heads_q < 0 || heads_k < 0 || d < 0 || d >= (1L << 30) || rot < 0 || (rot & 1) || rot > d || npos < 1) return TAO_ERR_SHAPE;
    if (ldt < 0 || ldh < 0 || ldyt < 0 || ldyh < 0 || !(eps >= 0.0) || !std::isfinite(eps)) return TAO_ERR_SHAPE;
    const __int128 heads = (__int128)heads_q + heads_k, lim = (__int128)1 << 60;
    if (heads >= (1L << 30) || tokens >= (1L << 40) || (__int128)tokens * heads * d >= ((__int128)1 << 36) || (__int128)tokens * heads >= ((__int128)1 << 36)) return TAO_ERR_SHAPE;
    if ((__int128)tokens * ldt + heads * ldh >= lim || (__int128)tokens * ldyt + heads * ldyh >= lim || (__int128)npos * rot >= lim) return TAO_ERR_SHAPE;
    const bool some = tokens > 0 && heads > 0 && d > 0;
    if (some) {
        // outputs: heads inside a token's stride, or tokens inside a head's
        const bool by_token = (heads == 1 || ldyh >= d) && (tokens == 1 || ldyt >= (heads - 1) * ldyh + d);
        const bool by_head = (tokens == 1 || ldyt >= d) && (heads == 1 || ldyh >= (__int128)(tokens - 1) * ldyt + d);
        if (!by_token && !by_head) return TAO_ERR_SHAPE;
        if (!x || (rot > 0 && (!cos_table || !sin_table)) || (!tau_cos != !tau_sin)) return TAO_ERR_NULL;
    }
    if (!aligned(x, 4) || !aligned(gamma_q, 4) || !aligned(gamma_k, 4) || !aligned(cos_table, 4) || !aligned(sin_table, 4) || !aligned(tau_cos, 4) ||
        !aligned(tau_sin, 4) || !aligned(positions, 8)) return TAO_ERR_ALIGN;
    HeadArgs& a = *out;
    a = HeadArgs();
    rc = make_consts(*md, d > 0 ? d : 1, eps, &a.k, norm == TAO_NORM_RMSNORM);
    if (rc != TAO_OK) return rc;
    a.g2 = gamma_up(2, *md);
    if (!(a.g2 == a.g2)) return TAO_ERR_K_RANGE;
    a.uflow = (md->flags & TAO_FLAG_UNDERFLOW_TERMS) ? 2.0 * 0x1p-149 : 0.0;
    a.norm_fy = widen(md->u * (1.0 + md->u) * (1.0 + md->u));
    a.x = x; a.gain[0] = gamma_q; a.gain[1] = gamma_k;
    a.c = cos_table; a.s = sin_table; a.tc = tau_cos; a.ts = tau_sin; a.positions = positions;
    a.tokens = tokens; a.npos = npos; a.ldt = ldt; a.ldh = ldh; a.ldyt = ldyt; a.ldyh = ldyh;
    a.heads_q = (int)heads_q; a.heads = (int)heads; a.d = (int)d; a.rot = (int)rot; a.interleaved = interleaved != 0; a.norm = norm == TAO_NORM_RMSNORM;
    return TAO_OK;
}

}  // namespace tao

extern "C" {

int tao_bound_rope_tables(const int64_t* positions, const float* inv_freq, double scale, float* cos_table, float* sin_table,
                          float* tau_cos, float* tau_sin, long npos, long half, const tao_fp_model* model, void* stream) {
    using namespace tao;
    tao_fp_model md;
    const int rc = resolve_model(model, &md);
    if (rc != TAO_OK) return rc;
    const long lim = 1L << 31;
    if (npos < 0 || half < 0 || npos >= lim || half >= lim || (__int128)npos * half >= ((__int128)1 << 40)) return TAO_ERR_SHAPE;
    if (!std::isfinite(scale) || !std::isfinite((float)scale)) return TAO_ERR_SHAPE;
    TableArgs a;
    a.e1 = gamma_up(1, md); a.e2 = gamma_up(2, md);
    if (!(a.e1 == a.e1) || !(a.e2 == a.e2)) return TAO_ERR_K_RANGE;
    if (npos == 0 || half == 0) return TAO_OK;
    if (!inv_freq || (!cos_table && !sin_table && !tau_cos && !tau_sin)) return TAO_ERR_NULL;
    if (!aligned(positions, 8) || !aligned(inv_freq, 4) || !aligned(cos_table, 4) || !aligned(sin_table, 4) || !aligned(tau_cos, 4) || !aligned(tau_sin, 4)) return TAO_ERR_ALIGN;
    a.positions = positions; a.inv_freq = inv_freq;
    a.out[0] = cos_table; a.out[1] = sin_table; a.out[2] = tau_cos; a.out[3] = tau_sin;
    a.npos = npos; a.half = (int)half;
    a.m = (double)(float)scale;
    a.whole = 1.0 / md.u;
    const double u = md.u, c_lib[2] = {md.c_cos, md.c_sin}, m = std::fabs(a.m);
    for (int i = 0; i < 2; ++i) {                            // B' = (1 + c u) B + c u |v|;  with m's rounding (1 + u) B' + u |v|
        const double cu = c_lib[i] * u;
        a.k1[i] = widen(m * (a.m == 1.0 ? 1.0 + cu : (1.0 + u) * (1.0 + cu)));
        a.k2[i] = widen(m * (a.m == 1.0 ? cu : (1.0 + u) * cu + u));
    }
    bool quick = true;
    for (int i = 0; i < 2; ++i) {
        a.q1[i] = (float)a.k1[i]; a.q2[i] = (float)a.k2[i];
        quick = quick && a.k1[i] <= 0x1p60 && a.k2[i] <= 0x1p60;
    }
    a.near = quick ? (float)a.e1 * 0x1p45f : 0.f;
    // (tables of less than one element for each of the chip's threads: one a thread; 16640 x 63 8.9 us, four a thread 8.4, 2080 x 63 3.5 and 4.7)
    const bool vec = (half % 4 == 0 || npos * half >= 1L << 19) && aligned(cos_table, 16) && aligned(sin_table, 16) && aligned(tau_cos, 16) && aligned(tau_sin, 16);
    const long blocks = ((vec ? (npos * half + 3) / 4 : npos * half) + 255) / 256;
    const dim3 grid((unsigned)(blocks < 256L * 64 ? blocks : 256L * 64)), blk(256);
    if (vec && half % 4 == 0) hipLaunchKernelGGL(rope_tables<4>, grid, blk, 0, (hipStream_t)stream, a);
    else if (vec)             hipLaunchKernelGGL(rope_tables_flat, grid, blk, 0, (hipStream_t)stream, a);
    else                      hipLaunchKernelGGL(rope_tables<1>, grid, blk, 0, (hipStream_t)stream, a);
    return launch_status();
}

int tao_bound_norm_rope(int norm, const float* x, const float* gamma_q, const float* gamma_k, double eps,
                        const float* cos_table, const float* sin_table, const float* tau_cos, const float* tau_sin,
                        const int64_t* positions, float* y, float* tau, long tokens, long heads_q, long heads_k, long d, long rot, long npos,
                        long ldt, long ldh, long ldyt, long ldyh, int interleaved, const tao_fp_model* model, void* stream) {
    using namespace tao;
    tao_fp_model md;
    HeadArgs a;
    const int rc = heads_setup(norm, x, gamma_q, gamma_k, eps, cos_table, sin_table, tau_cos, tau_sin, positions, tokens, heads_q, heads_k, d, rot, npos, ldt, ldh, ldyt, ldyh,
                               interleaved, model, &md, &a);
    if (rc != TAO_OK) return rc;
    const long rows = tokens * (heads_q + heads_k);
    if (rows == 0 || d == 0) return TAO_OK;
    if (!y && !tau) return TAO_ERR_NULL;
    if (!aligned(y, 4) || !aligned(tau, 4)) return TAO_ERR_ALIGN;
    a.y = y; a.tau = tau;
    hipStream_t st = (hipStream_t)stream;
    if (const int team = heads_team(a, y, tau)) {
        heads_dispatch(a, team, [&](auto t, auto inter, auto errors) { heads_launch<t(), inter(), errors()>(a, st); });
        return launch_status();
    }
    if (const int team = pairs_team(a)) {
        const long blocks = (rows + 256 / team - 1) / (256 / team);
        pairs_dispatch(a, team, [&](auto t, auto pairs) { hipLaunchKernelGGL((heads_pairs<t(), pairs()>), dim3((unsigned)(blocks < 256L * 64 ? blocks : 256L * 64)), dim3(256), 0, st, a); });
        return launch_status();
    }
    const long blocks = (rows + 3) / 4;
    hipLaunchKernelGGL(heads_any, dim3((unsigned)(blocks < 256L * 64 ? blocks : 256L * 64)), dim3(256), 0, st, a);
    return launch_status();
}

int tao_bound_check_norm_rope(int norm, const float* x, const float* gamma_q, const float* gamma_k, double eps,
                              const float* cos_table, const float* sin_table, const float* tau_cos, const float* tau_sin,
                              const int64_t* positions, const float* y_ref, const float* claimed,
                              long tokens, long heads_q, long heads_k, long d, long rot, long npos,
                              long ldt, long ldh, long ldyt, long ldyh, int interleaved, double alpha, double eps_rel,
                              const tao_fp_model* model, tao_profile* out, void* ws, size_t ws_bytes, void* stream) {
    using namespace tao;
    tao_fp_model md;
    HeadArgs a;
    const int rc = heads_setup(norm, x, gamma_q, gamma_k, eps, cos_table, sin_table, tau_cos, tau_sin, positions, tokens, heads_q, heads_k, d, rot, npos, ldt, ldh, ldyt, ldyh,
                               interleaved, model, &md, &a);
    if (rc != TAO_OK) return rc;
    if (!out || !ws) return out ? TAO_ERR_WORKSPACE : TAO_ERR_NULL;
    if (!(alpha >= 0.0) || !std::isfinite(alpha) || !(eps_rel >= 0.0) || !std::isfinite(eps_rel)) return TAO_ERR_SHAPE;
    const long rows = d > 0 ? tokens * (heads_q + heads_k) : 0, n = rows * d;
    if (n > 0 && !claimed) return TAO_ERR_NULL;
    if (!aligned(y_ref, 4) || !aligned(claimed, 4) || !aligned(out, 8)) return TAO_ERR_ALIGN;
    if (!aligned(ws, 256) || ws_bytes < check_workspace_bytes()) return TAO_ERR_WORKSPACE;
    a.y_ref = y_ref; a.claimed = claimed;
    hipStream_t st = (hipStream_t)stream;
    const CheckWorkspace w = carve_check_workspace(ws);
    a.tokens = d > 0 ? tokens : 0;
    const int team = heads_team(a, y_ref, claimed), pairs = team ? 0 : pairs_team(a), lanes = team ? team : pairs ? pairs : kWave;
    const long want = (rows + kCheckThreads / lanes - 1) / (kCheckThreads / lanes);
    const int nblocks = (int)(want < 1 || n <= kAloneElements ? 1 : want > kMaxCheckBlocks ? kMaxCheckBlocks : want);
    const PassOut pass = pass_out(w, nblocks, n, out);
    const HeadCheckArgs g{a, alpha, eps_rel, quick_alpha(alpha, md), pass};
    if (team) {
        heads_dispatch(a, team, [&](auto t, auto inter, auto errors) { heads_launch_check<t(), inter(), errors()>(g, nblocks, st); });
    } else if (pairs) {
        pairs_dispatch(a, pairs, [&](auto t, auto n) {
            if (y_ref) hipLaunchKernelGGL((heads_pairs_check<t(), n(), true>), dim3(nblocks), dim3(kCheckThreads), 0, st, g);
            else       hipLaunchKernelGGL((heads_pairs_check<t(), n(), false>), dim3(nblocks), dim3(kCheckThreads), 0, st, g);
        });
    } else {
        hipLaunchKernelGGL(heads_any_check, dim3(nblocks), dim3(kCheckThreads), 0, st, a, alpha, eps_rel, pass);
    }
    launch_finish(w, nblocks, n, out, st);
    return launch_status();
}

}  // extern "C"
