// tao_bound_rope_tables, tao_bound_norm_rope, tao_bound_check_norm_rope: the tables of the rotary embedding from positions and frequencies, and the
// RMS norm of every query and key head with the rotation of its first elements, re-executed and bounded in one call (operators of App. A.3; primitive
// rule of Sec. 3.1, Gamma(n-1) and Gamma(2) for the reductions).
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
};

// cos and sin of |t| < 2^50: t less the nearest multiple k of pi/2 (two parts of pi/2 in fused steps: the first difference is exact, as t and k times the
// first part are multiples of 2^-52 where k is not 0, the second rounds once: 2^-53 absolutely), then Taylor polynomials on |r| <= pi/4 of degree 13 and 14,
// whose remainders are below 2^-45 relatively.
__device__ __forceinline__ void cos_sin(double t, double& c, double& s) {
    const double k = rint(t * 0x1.45f306dc9c883p-1);
    const double r = fma(-k, 0x1.1a62633145c07p-54, fma(-k, 0x1.921fb54442d18p+0, t)), z = r * r;
    double ps = 1.0 / 6227020800.0, pc = -1.0 / 87178291200.0;
    ps = fma(ps, z, -1.0 / 39916800.0);  pc = fma(pc, z, 1.0 / 479001600.0);
    ps = fma(ps, z, 1.0 / 362880.0);     pc = fma(pc, z, -1.0 / 3628800.0);
    ps = fma(ps, z, -1.0 / 5040.0);      pc = fma(pc, z, 1.0 / 40320.0);
    ps = fma(ps, z, 1.0 / 120.0);        pc = fma(pc, z, -1.0 / 720.0);
    ps = fma(ps, z, -1.0 / 6.0);         pc = fma(pc, z, 1.0 / 24.0);
    const double sr = fma(ps * z, r, r);
    const double cr = fma(fma(pc, z, -0.5), z, 1.0);
    const int q = (int)(long long)k & 3;
    s = q & 1 ? cr : sr; c = q & 1 ? sr : cr;
    if (q & 2) s = -s;
    if ((q + 1) & 2) c = -c;
}
__device__ __forceinline__ void table_element(const TableArgs& a, double p, double f, float (&v)[4]) {
    const double t = p * f, e = (fabs(p) > a.whole ? a.e2 : a.e1) * fabs(t);
    double c, s;
    cos_sin(t, c, s);
    const double ac = fabs(c), as = fabs(s), e2 = 0.5 * e * e;
    const double bc = fmin(fmin(fma(as, e, e2), e), 1.0 + ac), bs = fmin(fmin(fma(ac, e, e2), e), 1.0 + as);
    v[0] = (float)(a.m * c); v[1] = (float)(a.m * s);
    v[2] = up32g(fma(a.k1[0], bc, a.k2[0] * ac)); v[3] = up32g(fma(a.k1[1], bs, a.k2[1] * as));
    if (!(fabs(t) < 0x1p50)) { v[0] = v[1] = v[2] = v[3] = NAN; }
}
__global__ __launch_bounds__(256) void rope_tables(TableArgs a) {
    const long n = a.npos * a.half, stride = (long)gridDim.x * 256;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += stride) {
        const long r = i / a.half;
        const int j = (int)(i - r * a.half);
        float v[4];
        table_element(a, (double)(a.positions ? a.positions[r] : r), (double)a.inv_freq[j], v);
#pragma unroll
        for (int o = 0; o < 4; ++o) if (a.out[o]) a.out[o][i] = v[o];
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
    bool interleaved;
    RowConsts k;
    double g2, uflow;                // Gamma(2), 2 2^-149 or 0
    double norm_fy;                  // u (1 + u)^2
};
// What a head's sum of squares gives: r, F (an element's error is F |x g|), k of the rotation, and the factors of the final rounding.
struct HeadCoef { double r, F, k, mul, sub; };
template <bool NORM>
__device__ __forceinline__ HeadCoef head_coef(const HeadArgs& a, double squares) {
    HeadCoef h{1.0, 0.0, a.g2, kUpMul, 1.0 + 0x1p-46};
    if constexpr (NORM) {
        const RowConsts& k = a.k;
        const double E_t = (k.G * (1.0 + k.u) + k.u) * squares, vstar = squares * k.inv_n;
        const double E_v = (E_t * k.inv_n + k.cd_u * vstar) * k.inv1mcd;
        double E_r, R, amp;
        const bool ok = rsqrt_tail(vstar, E_v, k, h.r, E_r, R, amp);
        h.F = ok ? E_r + k.u * R + a.norm_fy * R : NAN;
        h.k = fma(a.g2, h.r + h.F, h.F);
        const UpFactors up(k.m * (1.0 + 2.0 * amp));
        h.mul = up.mul; h.sub = up.sub;
    }
    return h;
}
// (a bound that is infinite in binary64 comes of an infinite operand: it would admit every finite claim)
__device__ __forceinline__ float head_bound(double e, const HeadCoef& h) { return e < INFINITY ? up32g(e, h.mul, h.sub) : NAN; }
// The two elements of a pair: ha, hb are x g.
__device__ __forceinline__ void rotate_pair(const HeadArgs& a, const HeadCoef& h, double ha, double hb, float c, float s, float tc, float ts,
                                            float& ya, float& yb, float& ta, float& tb) {
    const double C = (double)c, S = (double)s, ec = fabs((double)tc), es = fabs((double)ts);
    const double kc = fma(h.k, fabs(C) + ec, h.r * ec), ks = fma(h.k, fabs(S) + es, h.r * es);
    ya = (float)(h.r * (ha * C - hb * S)); yb = (float)(h.r * (hb * C + ha * S));
    ta = head_bound(fma(fabs(ha), kc, fabs(hb) * ks) + a.uflow, h);
    tb = head_bound(fma(fabs(hb), kc, fabs(ha) * ks) + a.uflow, h);
}
template <bool NORM>
__device__ __forceinline__ void plain_element(const HeadCoef& h, double hx, float& y, float& t) {
    y = (float)(h.r * hx);
    t = head_bound(NORM ? h.F * fabs(hx) : hx * 0.0, h);
}
// Sums over TEAM lanes, in every one of them.
template <int TEAM>
__device__ __forceinline__ double team_sum(double v) {
    constexpr int STEPS = TEAM == 8 ? 3 : TEAM == 16 ? 4 : TEAM == 32 ? 5 : 6;
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
// Any size, stride and layout: a wavefront a head, element by element, x read twice.
template <bool NORM, class Sink>
__device__ __forceinline__ void head_any(const HeadArgs& a, long row, Sink& sink) {
    const int lane = threadIdx.x & (kWave - 1), half = a.rot >> 1;
    const long t = row / a.heads;
    const int head = (int)(row - t * a.heads);
    const float* x = a.x + t * a.ldt + head * a.ldh;
    const float* g = a.gain[head >= a.heads_q];
    const long out = t * a.ldyt + head * a.ldyh;
    double sum = 0.0;
    if constexpr (NORM) {
        for (int j = lane; j < a.d; j += kWave) sum = fma((double)x[j], (double)x[j], sum);
        sum = team_sum<64>(sum);
    }
    const HeadCoef h = head_coef<NORM>(a, sum);
    auto at = [&](int j) __attribute__((always_inline)) { return (double)x[j] * (g ? (double)g[j] : 1.0); };
    const long p = a.positions ? a.positions[t] : a.npos > 0 ? t % a.npos : 0;
    const bool inside = p >= 0 && p < a.npos;
    for (int j = lane; j < half; j += kWave) {
        const int ja = a.interleaved ? 2 * j : j, jb = a.interleaved ? 2 * j + 1 : j + half;
        const long e = p * half + j;
        float ya, yb, ta, tb;
        rotate_pair(a, h, at(ja), at(jb), inside ? a.c[e] : NAN, inside ? a.s[e] : NAN, inside && a.tc ? a.tc[e] : 0.f, inside && a.ts ? a.ts[e] : 0.f, ya, yb, ta, tb);
        sink.put1(out + ja, ya, ta);
        sink.put1(out + jb, yb, tb);
    }
    for (int j = a.rot + lane; j < a.d; j += kWave) {
        float y, tau;
        plain_element<NORM>(h, at(j), y, tau);
        sink.put1(out + j, y, tau);
    }
}
template <bool NORM>
__global__ __launch_bounds__(256) void heads_any(HeadArgs a) {
    HeadStore sink{a.y, a.tau};
    const long rows = a.tokens * a.heads;
    for (long row = (long)blockIdx.x * 4 + threadIdx.x / kWave; row < rows; row += (long)gridDim.x * 4) head_any<NORM>(a, row, sink);
}
template <bool NORM>
__global__ __launch_bounds__(kCheckThreads) void heads_any_check(HeadArgs a, double alpha, double eps_rel, PassOut pass) {
    __shared__ unsigned int hist[kBins * kReplicas];
    __shared__ unsigned int red[kRedWords];
    for (int i = threadIdx.x; i < kBins * kReplicas; i += kCheckThreads) hist[i] = 0;
    __syncthreads();
    HeadCheck sink{a.y_ref, a.claimed, alpha, eps_rel, hist, (int)(threadIdx.x & (kReplicas - 1)), ThreadAcc()};
    const long rows = a.tokens * a.heads;
    constexpr int WAVES = kCheckThreads / kWave;
    for (long row = (long)blockIdx.x * WAVES + threadIdx.x / kWave; row < rows; row += (long)gridDim.x * WAVES) head_any<NORM>(a, row, sink);
    finish_pass(hist, sink.acc, red, pass);
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
    a.heads_q = (int)heads_q; a.heads = (int)heads; a.d = (int)d; a.rot = (int)rot; a.interleaved = interleaved != 0;
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
    const long blocks = (npos * half + 255) / 256;
    hipLaunchKernelGGL(rope_tables, dim3((unsigned)(blocks < 256L * 64 ? blocks : 256L * 64)), dim3(256), 0, (hipStream_t)stream, a);
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
    const long blocks = (rows + 3) / 4;
    const dim3 grid((unsigned)(blocks < 256L * 64 ? blocks : 256L * 64)), blk(256);
    if (norm == TAO_NORM_RMSNORM) hipLaunchKernelGGL(heads_any<true>, grid, blk, 0, st, a);
    else                          hipLaunchKernelGGL(heads_any<false>, grid, blk, 0, st, a);
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
    const long want = (rows + kCheckThreads / kWave - 1) / (kCheckThreads / kWave);
    const int nblocks = (int)(want < 1 || n <= kAloneElements ? 1 : want > kMaxCheckBlocks ? kMaxCheckBlocks : want);
    const PassOut pass = pass_out(w, nblocks, n, out);
    a.tokens = d > 0 ? tokens : 0;
    if (norm == TAO_NORM_RMSNORM) hipLaunchKernelGGL(heads_any_check<true>, dim3(nblocks), dim3(kCheckThreads), 0, st, a, alpha, eps_rel, pass);
    else                          hipLaunchKernelGGL(heads_any_check<false>, dim3(nblocks), dim3(kCheckThreads), 0, st, a, alpha, eps_rel, pass);
    launch_finish(w, nblocks, n, out, st);
    return launch_status();
}

}  // extern "C"
