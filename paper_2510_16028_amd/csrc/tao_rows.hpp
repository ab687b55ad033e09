// What the bounds of row-wise operators share: the constants of a row length, the final upper rounding, and the chain of the
// normalisations from the row's sums to the coefficients of an element's bound (operators of App. A.3, primitive rule of
// Sec. 3.1, Gamma(n-1) for the reductions).
#pragma once
#include "tao_device.hpp"
#include "tao_host.hpp"

namespace tao {

struct RowConsts {
    double u;          // unit roundoff
    double G;          // Gamma(cols - 1), upper
    double inv1mu;     // >= 1/(1-u)
    double ce_u;       // c_exp * u
    double inv1mce;    // >= 1/(1 - c_exp u)
    double cd_u;       // c_div * u
    double inv1mcd;    // >= 1/(1 - c_div u)
    double cr_u;       // c_rsqrt * u
    double eps;        // (double)(float)eps
    double inv_n;      // 1/cols (nearest; covered by the guard factor)
    double mean_f;     // c_div u / (1 - c_div u), upper
    double m;          // rounding margin of a bound of this row length (see make_consts)
    float quick_alpha; // the one-pass checks: alpha of the estimates
    int apart;         // ... and rows between those of neighbouring row groups of a workgroup (row_blocks)
};

// Factors of the final upper rounding (up32g) for a rounding margin m.
struct UpFactors {
    double mul, sub;
    __device__ __forceinline__ explicit UpFactors(double m) : mul(1.0 + 0x1p-24 + fmax(0x1p-32, 2.0 * m)), sub(1.0 + m) {}
};

// tail shared by LayerNorm and RMSNorm: from v*, E_v to (r*, E_r, R); ok = finite bound
// amp: how much a relative error of the row sums is amplified on its way into E_r (the sums enter
// through the difference w_lo = w - E_w, and E_r falls with w_lo at most like its power -3/2)
__device__ __forceinline__ bool rsqrt_tail(double vstar, double E_v, const RowConsts& k,
                                           double& rs, double& E_r, double& R, double& amp) {
    const double w = vstar + k.eps;
    const double E_w = (E_v + k.u * w) * k.inv1mu;
    const double w_lo = w - E_w;
    const bool ok = w_lo > 0.0;
    amp = (w + E_w) / w_lo;
    const double inv_s = 1.0 / sqrt(w_lo);
    const double inv_s3 = inv_s / w_lo;
    E_r = 0.5 * E_w * inv_s3 + k.cr_u * inv_s;
    rs = 1.0 / sqrt(w);
    R = rs + E_r;
    return ok;
}

// Chain of the template (E_s, E_mu, E_d, D, E_q, Q, E_t, E_v, E_w, w_lo, E_r, R, E_h, H, E_p).
// Per element only |d| = |x - mu| varies, and everything downstream is a polynomial in it with
// non-negative coefficients:
//   E_d = u' |d| + E'      (u' = u/(1-u), E' = E_mu/(1-u));   D = |d| + E_d = (1+u')|d| + E'
// so the two sums the variance bound needs,
//   sum Q   = (1+u) sum D^2,   sum E_q = sum E_d(|d| + D) + u sum D^2,
// follow from n, sum|d| and sum d^2, and the per-element tail
//   E_p/|g| = (1+u) E_h + u r|d|,  E_h = D (E_r + u R) + r E_d
// collapses to K1 |d| + K0.  Same real-number formula as the step-by-step chain; the different
// binary64 rounding (a few 2^-53) is covered by the rounding margin of up32g.
// From E_mu, sum|d|, sum d^2 to the per-element coefficients: E_p/|g| = K1 |d| + K0.
__device__ __forceinline__ void layernorm_tail(double E_mu, double s_ad, double s_d2, double n, const RowConsts& k,
                                               double& K1, double& K0, double& amp, double* rs_out = nullptr) {
    const double up = k.u * k.inv1mu, Ep = E_mu * k.inv1mu;       // u', E'
    const double c1 = 1.0 + up;
    const double sD2 = c1 * c1 * s_d2 + 2.0 * c1 * Ep * s_ad + n * Ep * Ep;           // sum D^2
    const double sEdD = up * (1.0 + c1) * s_d2 + Ep * (up + 1.0 + c1) * s_ad + n * Ep * Ep;  // sum E_d(|d|+D)
    const double E_t = k.G * (1.0 + k.u) * sD2 + sEdD + k.u * sD2;
    const double vstar = s_d2 * k.inv_n;
    const double E_v = (E_t * k.inv_n + k.cd_u * vstar) * k.inv1mcd;
    double rs, E_r, R;
    const bool ok = rsqrt_tail(vstar, E_v, k, rs, E_r, R, amp);
    const double hc = E_r + k.u * R;                              // E_h = D hc + r E_d
    K1 = (1.0 + k.u) * (c1 * hc + rs * up) + k.u * rs;
    K0 = ok ? (1.0 + k.u) * Ep * (hc + rs) : NAN;                 // NaN row when the bound is not finite
    if (rs_out) *rs_out = rs;
}

// variance: the operator divides by a computed variance (LayerNorm, RMSNorm, GroupNorm).  Its
// template subtracts the variance's own error bound, about Gamma(n-1) times the variance, from the
// variance: beyond Gamma(n-1) = 1/2 the difference has lost its relative accuracy (and soon its
// sign), so such rows are refused rather than bounded by noise.
inline int make_consts(const tao_fp_model& md, long cols, double eps, RowConsts* k, bool variance = false) {
    const double G = gamma_up(cols - 1, md);
    if (!(G == G) || (variance && G > 0.5)) return TAO_ERR_K_RANGE;
    const double u = md.u;
    k->u = u; k->G = G;
    k->inv1mu = widen(1.0 / (1.0 - u));
    k->ce_u = md.c_exp * u;
    k->inv1mce = widen(1.0 / (1.0 - md.c_exp * u));
    k->cd_u = md.c_div * u;
    k->inv1mcd = widen(1.0 / (1.0 - md.c_div * u));
    k->cr_u = md.c_rsqrt * u;
    k->eps = (double)(float)eps;
    k->inv_n = 1.0 / (double)cols;
    k->mean_f = widen(k->cd_u * k->inv1mcd);
    // Rounding margin of the emitted bound.  The row sums are formed here in round-to-nearest
    // binary64 (each thread a sequential part, then a tree: at most cols 2^-53 below the real sum),
    // and a reference that adds the row sequentially with upward rounding sits up to cols 2^-52
    // above it; the scalar chain after the sums adds a few dozen roundings.  m covers both for a
    // bound that depends on the sums with unit sensitivity; the kernels scale it where a sum enters
    // through a difference (1 - sigma of the softmax, the lower end w_lo of the variance).
    k->m = ((double)cols + 130.0) * 0x1p-51;
    k->quick_alpha = NAN;
    k->apart = 1;                                            // (no launch leaves it open, one of no rows either: row_blocks chooses for the others)
    if (!(md.c_exp * u < 0.5) || !(md.c_div * u < 0.5)) return TAO_ERR_MODEL;
    return TAO_OK;
}

}  // namespace tao
