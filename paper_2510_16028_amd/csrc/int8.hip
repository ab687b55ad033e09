// tao_quantize_rows, tao_bound_linear_int8, tao_bound_check_linear_int8: a matrix product in 8-bit whole numbers with a scale for
// each token (row of A) and each channel (row of W),
//     S_ij = sum_k A_ik W_jk,    y_ij = fl(fl(fl(fl(S_ij) sa_i) sw_j) + b_j).
// S is exact in 32 bits in any order (|S| <= K 2^14 < 2^31), so the re-executed output is the same bit for bit whatever tile, split
// or order forms it, and the bound is the few roundings behind the sum (Sec. 3.1, primitive rule):
//     tau = Gamma(d) |S sa sw|  [+ u (|S sa sw + b| + Gamma(d) |S sa sw|)],   d = 2, or 3 where the conversion of S rounds too.
#include "tao_check.hpp"
#include "tao_device.hpp"
#include "tao_host.hpp"

namespace tao {

typedef int intx4 __attribute__((ext_vector_type(4)));

struct Int8Args {
    const signed char* A; const float* sa;      // [batch][M][K], [batch][M]
    const signed char* W; const float* sw;      // [batch or 1][N][K], [batch or 1][N]
    const float* bias;                          // [N] or null
    float* y; float* tau;                       // [batch][M][N], either may be null
    long M, N, K, lda, ldw, ldy, batch, strideA, strideW, strideY;
    double g2, g3, u, limit, uflow;             // Gamma(2), Gamma(3); whole numbers up to limit are exact in binary32
};

// The operator's last steps on one sum, and their bound.  Binary64 holds S sa exactly to a rounding of 2^-53, far inside the margin
// of the final upper rounding; the sum with the bias may cancel, but its rounding is relative to terms that the bound itself carries.
__device__ __forceinline__ float int8_value(int S, float sa, float sw, float b, bool has_bias) {
    const float v = ((float)S * sa) * sw;
    return has_bias ? v + b : v;
}
__device__ __forceinline__ float int8_bound(int S, float sa, float sw, float b, bool has_bias, const Int8Args& p) {
    const double s = (double)S, v = s * (double)sa * (double)sw;
    double e = (fabs(s) > p.limit ? p.g3 : p.g2) * fabs(v);
    if (has_bias) e = fma(p.u, fabs(v + (double)b) + e, e);
    e = fma(p.uflow, fabs(s) + fabs((double)sa) + fabs((double)sw) + 1.0, e);
    return up32g(e);
}

// 16 bytes of a row from column k on; columns from K on read as 0 (nothing beyond the row's K columns is touched).
__device__ __forceinline__ intx4 row16(const signed char* __restrict__ row, long k, long K) {
    intx4 r = {0, 0, 0, 0};
    if (k + 16 <= K) {
        __builtin_memcpy(&r, row + k, 16);
    } else {
        for (int i = 0; i < 16 && k + i < K; ++i) r[i >> 2] |= (int)(unsigned)(unsigned char)row[k + i] << (8 * (i & 3));
    }
    return r;
}

// What becomes of an output: stored with its bound, or checked against the claim.
struct Int8Store {
    __device__ __forceinline__ void put(const Int8Args& p, long i, int S, float sa, float sw, float b) {
        const bool has_bias = p.bias != nullptr;
        if (p.y) p.y[i] = int8_value(S, sa, sw, b, has_bias);
        if (p.tau) p.tau[i] = int8_bound(S, sa, sw, b, has_bias, p);
    }
};
struct Int8Check {
    const float* y_ref; const float* claimed; double alpha, eps_rel;
    unsigned int* hist; int rep; ThreadAcc acc;
    __device__ __forceinline__ void put(const Int8Args& p, long i, int S, float sa, float sw, float b) {
        const bool has_bias = p.bias != nullptr;
        const float r = y_ref ? y_ref[i] : int8_value(S, sa, sw, b, has_bias);
        check_one(claimed[i], r, int8_bound(S, sa, sw, b, has_bias, p), alpha, eps_rel, hist, rep, acc);
    }
};

// ---- few rows: a workgroup of 16 wavefronts takes all of up to 16 MT rows of A with 16 NT rows of W; the wavefronts share out the
// reduction in chunks of 64 columns and add their sums in LDS, in whole numbers, so in any order.  Operands go from memory to
// registers in the layout of v_mfma_i32_16x16x64_i8 (lane: row lane % 16, columns 16 (lane / 16) on); the order of the columns inside
// a chunk does not matter, as both operands have the same.
constexpr int kInt8Threads = kCheckThreads;
template <int MT, int NT>
struct Int8Tile {
    static constexpr int ROWS = 16 * MT, COLS = 16 * NT;
    int sums[ROWS * COLS];
};
template <int MT, int NT>
__device__ __forceinline__ void int8_sums(const Int8Args& p, Int8Tile<MT, NT>& t, long z, long m0, long n0) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    constexpr int WAVES = kInt8Threads / kWave;
    for (int i = tid; i < t.ROWS * t.COLS; i += kInt8Threads) t.sums[i] = 0;
    __syncthreads();
    const signed char* a[MT];
    const signed char* w[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a[i] = p.A + z * p.strideA + min(m0 + i * 16 + (lane & 15), p.M - 1) * p.lda;
#pragma unroll
    for (int j = 0; j < NT; ++j) w[j] = p.W + z * p.strideW + min(n0 + j * 16 + (lane & 15), p.N - 1) * p.ldw;
    intx4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = intx4{0, 0, 0, 0};
    for (long c = wave; c * 64 < p.K; c += WAVES) {
        const long k = c * 64 + (lane >> 4) * 16;
        intx4 av[MT], wv[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) av[i] = row16(a[i], k, p.K);
#pragma unroll
        for (int j = 0; j < NT; ++j) wv[j] = row16(w[j], k, p.K);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(av[i], wv[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) atomicAdd(&t.sums[(i * 16 + (lane >> 4) * 4 + v) * t.COLS + j * 16 + (lane & 15)], acc[i][j][v]);
    __syncthreads();
}
template <int MT, int NT, class Sink>
__device__ __forceinline__ void int8_few_body(const Int8Args& p, Sink& sink, Int8Tile<MT, NT>& t) {
    const long tm = (p.M + t.ROWS - 1) / t.ROWS, tn = (p.N + t.COLS - 1) / t.COLS, tiles = tm * tn * p.batch;
    for (long at = blockIdx.x; at < tiles; at += gridDim.x) {
        const long z = at / (tm * tn), in = at - z * (tm * tn), m0 = in % tm * t.ROWS, n0 = in / tm * t.COLS;
        int8_sums(p, t, z, m0, n0);
        const float* sa = p.sa + z * p.M;
        const float* sw = p.sw + (p.strideW ? z * p.N : 0);
        for (int e = threadIdx.x; e < t.ROWS * t.COLS; e += kInt8Threads) {
            const long m = m0 + e / t.COLS, n = n0 + e % t.COLS;
            if (m < p.M && n < p.N) sink.put(p, z * p.strideY + m * p.ldy + n, t.sums[e], sa[m], sw[n], p.bias ? p.bias[n] : 0.f);
        }
        __syncthreads();
    }
}
template <int MT, int NT>
__global__ __launch_bounds__(kInt8Threads) void int8_few(Int8Args p) {
    __shared__ Int8Tile<MT, NT> t;
    Int8Store sink;
    int8_few_body(p, sink, t);
}
template <int MT, int NT>
__global__ __launch_bounds__(kInt8Threads) void int8_few_check(Int8Args p, const float* y_ref, const float* claimed, double alpha, double eps_rel, PassOut pass) {
    __shared__ Int8Tile<MT, NT> t;
    __shared__ unsigned int hist[kBins * kReplicas];
    __shared__ unsigned int red[kRedWords];
    for (int i = threadIdx.x; i < kBins * kReplicas; i += kInt8Threads) hist[i] = 0;
    Int8Check sink{y_ref, claimed, alpha, eps_rel, hist, (int)threadIdx.x & (kReplicas - 1), ThreadAcc()};
    int8_few_body(p, sink, t);
    __syncthreads();
    finish_pass(hist, sink.acc, red, pass);
}

// ---- quantisation of rows: scale = fl(max|x| / 127), q = round(fl(x / scale)), ties to even.  A row that is not finite has scale NaN
// and q = 0 (so the product is NaN, which no check admits); a row of zeros, or one so small that its scale rounds to 0, scale 0 and q = 0.
__global__ __launch_bounds__(256) void quantize_rows(const float* __restrict__ x, signed char* __restrict__ q, float* __restrict__ scale,
                                                     long rows, long cols, long ld, long ldq) {
    __shared__ float most[4];
    const int tid = threadIdx.x;
    for (long r = blockIdx.x; r < rows; r += gridDim.x) {
        const float* xr = x + r * ld;
        float m = 0.f;
        int bad = 0;
        for (long c = tid; c < cols; c += 256) { const float a = fabsf(xr[c]); bad |= !(a < INFINITY); m = fmaxf(m, a); }
        m = wave_max(bad ? INFINITY : m);
        if ((tid & (kWave - 1)) == 0) most[tid / kWave] = m;
        __syncthreads();
        m = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
        const float s = m < INFINITY ? m / 127.f : NAN;
        for (long c = tid; c < cols; c += 256)
            q[r * ldq + c] = s > 0.f ? (signed char)(int)fminf(fmaxf(rintf(xr[c] / s), -127.f), 127.f) : (signed char)0;
        if (tid == 0) scale[r] = s;
        __syncthreads();
    }
}

// Checks the arguments that the two entry points share and fills the kernels'.
static int int8_setup(const int8_t* A, const float* scale_a, const int8_t* W, const float* scale_w, const float* bias,
                      long M, long N, long K, long lda, long ldw, long ldy, long batch, long strideA, long strideW, long strideY,
                      const tao_fp_model* model, Int8Args* out) {
    tao_fp_model md;
    const int rc = resolve_model(model, &md);
    if (rc != TAO_OK) return rc;
    if (M < 0 || N < 0 || K < 0 || batch < 0) return TAO_ERR_SHAPE;
    if (lda < K || ldw < K || ldy < N) return TAO_ERR_SHAPE;
    if (strideA < 0 || strideW < 0 || strideY < 0) return TAO_ERR_SHAPE;
    const long most = 1L << 31;                                   // sizes; extents of the memory up to 2^60 elements
    if (M >= most || N >= most || batch >= most) return TAO_ERR_SHAPE;
    if (K > TAO_INT8_MAX_K) return TAO_ERR_K_RANGE;               // the sum may leave 32 bits
    auto extent = [&](long rows, long ld, long stride) { return (__int128)rows * ld + (__int128)batch * stride; };
    const __int128 room = (__int128)1 << 60;
    if (extent(M, lda, strideA) >= room || extent(N, ldw, strideW) >= room || extent(M, ldy, strideY) >= room) return TAO_ERR_SHAPE;
    if (batch > 1 && M > 0 && strideY < M * ldy - (ldy - N)) return TAO_ERR_SHAPE;      // outputs would overlap
    if ((__int128)M * N * batch >= ((__int128)1 << 36)) return TAO_ERR_SHAPE;
    if (M > 0 && N > 0 && batch > 0) {
        if (!scale_a || !scale_w || (K > 0 && (!A || !W))) return TAO_ERR_NULL;
        if (!aligned(scale_a, 4) || !aligned(scale_w, 4) || !aligned(bias, 4)) return TAO_ERR_ALIGN;
    }
    Int8Args& p = *out;
    p.A = (const signed char*)A; p.sa = scale_a; p.W = (const signed char*)W; p.sw = scale_w; p.bias = bias;
    p.y = nullptr; p.tau = nullptr;
    p.M = M; p.N = N; p.K = K; p.lda = lda; p.ldw = ldw; p.ldy = ldy;
    p.batch = batch; p.strideA = strideA; p.strideW = strideW; p.strideY = strideY;
    p.g2 = gamma_up(2, md); p.g3 = gamma_up(3, md); p.u = md.u; p.limit = 1.0 / md.u;
    if (!(p.g2 == p.g2) || !(p.g3 == p.g3)) return TAO_ERR_K_RANGE;
    p.uflow = (md.flags & TAO_FLAG_UNDERFLOW_TERMS) ? 0x1p-149 : 0.0;
    return TAO_OK;
}

}  // namespace tao

extern "C" {

int tao_quantize_rows(const float* x, int8_t* q, float* scale, long rows, long cols, long ld, long ldq, void* stream) {
    using namespace tao;
    if (rows < 0 || cols < 0 || ld < cols || ldq < cols) return TAO_ERR_SHAPE;
    if ((__int128)rows * ld >= ((__int128)1 << 60) || (__int128)rows * ldq >= ((__int128)1 << 60)) return TAO_ERR_SHAPE;
    if (rows == 0) return TAO_OK;
    if (!scale || (cols > 0 && (!x || !q))) return TAO_ERR_NULL;
    if (!aligned(x, 4) || !aligned(scale, 4)) return TAO_ERR_ALIGN;
    const long blocks = rows < 256L * 64 ? rows : 256L * 64;
    hipLaunchKernelGGL(quantize_rows, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, x, (signed char*)q, scale, rows, cols, ld, ldq);
    return launch_status();
}

int tao_bound_linear_int8(const int8_t* A, const float* scale_a, const int8_t* W, const float* scale_w, const float* bias,
                          float* y, float* tau, long M, long N, long K, long lda, long ldw, long ldy,
                          long batch, long strideA, long strideW, long strideY, const tao_fp_model* model, void* stream) {
    using namespace tao;
    Int8Args p;
    const int rc = int8_setup(A, scale_a, W, scale_w, bias, M, N, K, lda, ldw, ldy, batch, strideA, strideW, strideY, model, &p);
    if (rc != TAO_OK) return rc;
    if (M == 0 || N == 0 || batch == 0) return TAO_OK;
    if (!y && !tau) return TAO_ERR_NULL;
    if (!aligned(y, 4) || !aligned(tau, 4)) return TAO_ERR_ALIGN;
    p.y = y; p.tau = tau;
    const __int128 tiles = (__int128)((M + 63) / 64) * ((N + 15) / 16) * batch;
    const unsigned grid = tiles < (1 << 20) ? (unsigned)tiles : 1u << 20;
    hipStream_t st = (hipStream_t)stream;
    if (M <= 16) hipLaunchKernelGGL((int8_few<1, 1>), dim3(grid), dim3(kInt8Threads), 0, st, p);
    else         hipLaunchKernelGGL((int8_few<4, 1>), dim3(grid), dim3(kInt8Threads), 0, st, p);
    return launch_status();
}

int tao_bound_check_linear_int8(const int8_t* A, const float* scale_a, const int8_t* W, const float* scale_w, const float* bias,
                                const float* y_ref, const float* claimed, long M, long N, long K, long lda, long ldw, long ldy,
                                long batch, long strideA, long strideW, long strideY, double alpha, double eps_rel,
                                const tao_fp_model* model, tao_profile* out, void* ws, size_t ws_bytes, void* stream) {
    using namespace tao;
    Int8Args p;
    const int rc = int8_setup(A, scale_a, W, scale_w, bias, M, N, K, lda, ldw, ldy, batch, strideA, strideW, strideY, model, &p);
    if (rc != TAO_OK) return rc;
    if (!out || !ws) return out ? TAO_ERR_WORKSPACE : TAO_ERR_NULL;
    if (!(alpha >= 0.0) || !std::isfinite(alpha) || !(eps_rel >= 0.0) || !std::isfinite(eps_rel)) return TAO_ERR_SHAPE;
    const long n = M * N * batch;
    if (n > 0 && !claimed) return TAO_ERR_NULL;
    if (!aligned(y_ref, 4) || !aligned(claimed, 4) || !aligned(out, 8)) return TAO_ERR_ALIGN;
    if (!aligned(ws, 256) || ws_bytes < check_workspace_bytes()) return TAO_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const CheckWorkspace w = carve_check_workspace(ws);
    const long tiles = n > 0 ? ((M + 63) / 64) * ((N + 15) / 16) * batch : 1;
    const int nblocks = (int)(tiles < kMaxCheckBlocks ? tiles : kMaxCheckBlocks);
    if (M <= 16) hipLaunchKernelGGL((int8_few_check<1, 1>), dim3(nblocks), dim3(kInt8Threads), 0, st, p, y_ref, claimed, alpha, eps_rel, pass_out(w, nblocks, n, out));
    else         hipLaunchKernelGGL((int8_few_check<4, 1>), dim3(nblocks), dim3(kInt8Threads), 0, st, p, y_ref, claimed, alpha, eps_rel, pass_out(w, nblocks, n, out));
    launch_finish(w, nblocks, n, out, st);
    return launch_status();
}

}  // extern "C"
