// tao_bound_linear_int4, tao_bound_check_linear_int4: binary32 activations times weights in 4 bits with a scale, and possibly a zero point, for each group,
//     w_jk = (q_jk - z_jg) s_jg,    y_ij = sum_k a_ik w_jk + b_j,    tau_ij = Gamma(K') (sum_k |a_ik||w_jk| + |b_j|),
// a reduction of K products (Sec. 3.1) whose terms are rounded once more for the scale: K' = K + 1, or K + 2 with a bias.
#include "tao_check.hpp"
#include "tao_device.hpp"
#include "tao_host.hpp"

namespace tao {

struct Int4Args {
    const float* A; const unsigned char* W;
    const float* scale; const unsigned char* zero;           // [N][groups], zero may be null
    const float* bias;
    float* y; float* tau;
    long M, N, K, lda, ldw, ldy;
    long group; int groups;
    double gamma;                    // Gamma(K'), with the margins of the sums' roundings
    double uflow, terms;             // 2^-149 or 0, K'
};
// The bound from the sum of magnitudes, rounded up.  NaN where an operand is not finite, as an infinite bound would admit every finite claim (sums of finite operands
// stay inside the binary64 range).
__device__ __forceinline__ float int4_bound(const Int4Args& p, double size, double b, double uflow) {
    const double e = fma(p.gamma, size + fabs(b), uflow);
    return e < INFINITY ? up32(e) : NAN;
}

// Any size, in binary64: a wavefront an output, lanes along the bytes of its row.
__device__ __forceinline__ void int4_wave_sums(const Int4Args& p, long i, long j, int lane, double& sum, double& size, double& extra) {
    const float* a = p.A + i * p.lda;
    const unsigned char* w = p.W + j * p.ldw;
    sum = 0.0; size = 0.0; extra = 0.0;
    for (long k = 2 * lane; k < p.K; k += 2 * kWave) {
        const unsigned byte = w[k >> 1];
        const long g = j * p.groups + k / p.group;           // (groups of more than one begin at even columns)
        const double s = (double)p.scale[g], z = p.zero ? (double)p.zero[g] : 8.0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (k + e >= p.K) break;
            const double v = (double)a[k + e], q = ((double)(byte >> (4 * e) & 15u) - z) * s;
            sum = fma(v, q, sum);
            size = fma(fabs(v), fabs(q), size);
            if (p.uflow != 0.0) extra += fabs(v) + fabs(s);
        }
    }
    sum = wave_sum(sum); size = wave_sum(size);
    if (p.uflow != 0.0) extra = wave_sum(extra);
}
__global__ __launch_bounds__(256) void int4_any(Int4Args p) {
    const long n = p.M * p.N;
    const int lane = threadIdx.x & (kWave - 1);
    for (long at = (long)blockIdx.x * 4 + threadIdx.x / kWave; at < n; at += (long)gridDim.x * 4) {
        const long j = at / p.M, i = at - j * p.M;
        double sum, size, extra;
        int4_wave_sums(p, i, j, lane, sum, size, extra);
        if (lane == 0) {
            const double b = p.bias ? (double)p.bias[j] : 0.0;
            if (p.y) p.y[i * p.ldy + j] = (float)(sum + b);
            if (p.tau) p.tau[i * p.ldy + j] = int4_bound(p, size, b, p.uflow * (p.terms + extra));
        }
    }
}

// The check of stored outputs (contiguous) and bounds against claims of another row stride.
struct Int4CheckArgs { const float* y; const float* tau; const float* claimed; long N, ldr, ldy; double alpha, eps_rel; PassOut pass; };
__global__ __launch_bounds__(kCheckThreads) void int4_check(Int4CheckArgs a, long n) {
    __shared__ unsigned int hist[kBins * kReplicas];
    __shared__ unsigned int red[kRedWords];
    for (int i = threadIdx.x; i < kBins * kReplicas; i += kCheckThreads) hist[i] = 0;
    __syncthreads();
    ThreadAcc acc;
    const int rep = threadIdx.x & (kReplicas - 1);
    for (long i = (long)blockIdx.x * kCheckThreads + threadIdx.x; i < n; i += (long)gridDim.x * kCheckThreads) {
        const long row = i / a.N, col = i - row * a.N;
        check_one(a.claimed[row * a.ldy + col], a.y[row * a.ldr + col], a.tau[i], a.alpha, a.eps_rel, hist, rep, acc);
    }
    finish_pass(hist, acc, red, a.pass);
}

// Checks the arguments that the two entry points share and fills the kernels'.
static int int4_setup(const float* A, const uint8_t* W, const float* scale, const uint8_t* zero, long group, const float* bias, long M, long N, long K,
                      long lda, long ldw, long ldy, const tao_fp_model* model, tao_fp_model* md, Int4Args* out) {
    const int rc = resolve_model(model, md);
    if (rc != TAO_OK) return rc;
    const long most = 1L << 31;
    if (M < 0 || N < 0 || K < 0 || M >= most || N >= most || K >= most || (__int128)M * N >= ((__int128)1 << 36)) return TAO_ERR_SHAPE;
    if (lda < K || ldw < (K + 1) / 2 || ldy < N || group < 1 || (group % 32 != 0 && group < K)) return TAO_ERR_SHAPE;
    const __int128 room = (__int128)1 << 60;
    if ((__int128)M * lda >= room || (__int128)N * ldw >= room || (__int128)M * ldy >= room) return TAO_ERR_SHAPE;
    const long steps = K + (bias ? 2 : 1);
    const double g = gamma_up(steps, *md);
    if (!(g == g)) return TAO_ERR_K_RANGE;
    if (M > 0 && N > 0) {
        if (K > 0 && (!A || !W || !scale)) return TAO_ERR_NULL;
        if (!aligned(A, 4) || !aligned(scale, 4) || !aligned(bias, 4)) return TAO_ERR_ALIGN;
    }
    Int4Args& p = *out;
    p.A = A; p.W = W; p.scale = scale; p.zero = zero; p.bias = bias; p.y = nullptr; p.tau = nullptr;
    p.M = M; p.N = N; p.K = K; p.lda = lda; p.ldw = ldw; p.ldy = ldy;
    p.group = group < K || K == 0 ? group : K + (K & 1);     // (one group: its end at an even column)
    p.groups = (int)((K + p.group - 1) / p.group);
    p.gamma = g * (1.0 + ((double)K + 64.0) * 0x1p-52) * kGuard;
    p.uflow = (md->flags & TAO_FLAG_UNDERFLOW_TERMS) ? 0x1p-149 * kGuard : 0.0;
    p.terms = (double)steps;
    return TAO_OK;
}
static int int4_launch(const Int4Args& p, hipStream_t st) {
    const long blocks = (p.M * p.N + 3) / 4;
    hipLaunchKernelGGL(int4_any, dim3((unsigned)(blocks < 256L * 256 ? blocks : 256L * 256)), dim3(256), 0, st, p);
    return launch_status();
}
static size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace tao

extern "C" {

size_t tao_linear_int4_workspace_bytes(long M, long N, long K) {
    (void)M; (void)N; (void)K;
    return 0;
}

size_t tao_bound_check_linear_int4_workspace_bytes(long M, long N, long K) {
    using namespace tao;
    if (M < 0 || N < 0 || (__int128)M * N >= ((__int128)1 << 36)) return 0;
    return tao_linear_int4_workspace_bytes(M, N, K) + padded(check_workspace_bytes()) + 2 * padded((size_t)(M * N) * sizeof(float));
}

int tao_bound_linear_int4(const float* A, const uint8_t* W, const float* scale, const uint8_t* zero, long group, const float* bias,
                          float* y, float* tau, long M, long N, long K, long lda, long ldw, long ldy,
                          const tao_fp_model* model, void* ws, size_t ws_bytes, void* stream) {
    using namespace tao;
    tao_fp_model md;
    Int4Args p;
    const int rc = int4_setup(A, W, scale, zero, group, bias, M, N, K, lda, ldw, ldy, model, &md, &p);
    if (rc != TAO_OK) return rc;
    if (M == 0 || N == 0) return TAO_OK;
    if (!y && !tau) return TAO_ERR_NULL;
    if (!aligned(y, 4) || !aligned(tau, 4)) return TAO_ERR_ALIGN;
    const size_t need = tao_linear_int4_workspace_bytes(M, N, K);
    if (need > 0 && (!ws || !aligned(ws, 256) || ws_bytes < need)) return TAO_ERR_WORKSPACE;
    p.y = y; p.tau = tau;
    return int4_launch(p, (hipStream_t)stream);
}

int tao_bound_check_linear_int4(const float* A, const uint8_t* W, const float* scale, const uint8_t* zero, long group, const float* bias,
                                const float* y_ref, const float* claimed, long M, long N, long K, long lda, long ldw, long ldy,
                                double alpha, double eps_rel, const tao_fp_model* model, tao_profile* out,
                                void* ws, size_t ws_bytes, void* stream) {
    using namespace tao;
    tao_fp_model md;
    Int4Args p;
    const int rc = int4_setup(A, W, scale, zero, group, bias, M, N, K, lda, ldw, ldy, model, &md, &p);
    if (rc != TAO_OK) return rc;
    if (!out || !ws) return out ? TAO_ERR_WORKSPACE : TAO_ERR_NULL;
    if (!(alpha >= 0.0) || !std::isfinite(alpha) || !(eps_rel >= 0.0) || !std::isfinite(eps_rel)) return TAO_ERR_SHAPE;
    const long n = M * N;
    if (n > 0 && !claimed) return TAO_ERR_NULL;
    if (!aligned(y_ref, 4) || !aligned(claimed, 4) || !aligned(out, 8)) return TAO_ERR_ALIGN;
    if (!aligned(ws, 256) || ws_bytes < tao_bound_check_linear_int4_workspace_bytes(M, N, K)) return TAO_ERR_WORKSPACE;
    const CheckWorkspace w = carve_check_workspace(ws);
    float* stored = (float*)((char*)ws + padded(check_workspace_bytes()));
    hipStream_t st = (hipStream_t)stream;
    if (n > 0) {
        p.tau = stored;
        if (!y_ref) p.y = (float*)((char*)stored + padded((size_t)n * sizeof(float)));
        p.ldy = N;
        const int rc = int4_launch(p, st);
        if (rc != TAO_OK) return rc;
    }
    const long want = (n + kCheckThreads - 1) / kCheckThreads;
    const int nblocks = (int)(want < 1 || n <= kAloneElements ? 1 : want > kMaxCheckBlocks ? kMaxCheckBlocks : want);
    const Int4CheckArgs c{y_ref ? y_ref : p.y, p.tau, claimed, N, y_ref ? ldy : N, ldy, alpha, eps_rel, pass_out(w, nblocks, n, out)};
    hipLaunchKernelGGL(int4_check, dim3(nblocks), dim3(kCheckThreads), 0, st, c, n);
    launch_finish(w, nblocks, n, out, st);
    return launch_status();
}

}  // extern "C"
