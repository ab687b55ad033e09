// tao_quantize_rows, tao_bound_linear_int8, tao_bound_check_linear_int8: a matrix product in 8-bit whole numbers with a scale for
// each token (row of A) and each channel (row of W),
//     S_ij = sum_k A_ik W_jk,    y_ij = fl(fl(fl(fl(S_ij) sa_i) sw_j) + b_j).
// S is exact in 32 bits in any order (|S| <= K 2^14 < 2^31), so the re-executed output is the same bit for bit whatever tile, split
// or order forms it, and the bound is the few roundings behind the sum (Sec. 3.1, primitive rule):
//     tau = Gamma(d) |S sa sw|  [+ u (|S sa sw + b| + Gamma(d) |S sa sw|)],   d = 2, or 3 where the conversion of S rounds too.
#include <type_traits>
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
    double g2, g3, u, uflow;                    // Gamma(2), Gamma(3), unit roundoff; 2^-149 or 0
    int vec;                                    // rows of outputs and claims are on 16-byte addresses
    int limit;                                  // whole numbers of larger magnitude round in the conversion
    float c2, c3, cu, least;                    // the bound in binary32 (int8_output), for |v| from `least` on
};

// The bound of one sum in binary64.  Binary64 holds S sa exactly to a rounding of 2^-53, far inside the margin of the final upper
// rounding; the sum with the bias may cancel, but its rounding is relative to terms that the bound itself carries.
__device__ __forceinline__ float int8_bound(int S, float sa, float sw, float b, bool has_bias, const Int8Args& p) {
    const double s = (double)S, v = s * (double)sa * (double)sw;
    double e = (abs(S) > p.limit ? p.g3 : p.g2) * fabs(v);
    if (has_bias) e = fma(p.u, fabs(v + (double)b) + e, e);
    e = fma(p.uflow, fabs(s) + fabs((double)sa) + fabs((double)sw) + 1.0, e);
    return up32g(e);
}
// Output and bound of one sum.  The bound takes binary32 where that is accurate enough (eight binary64 instructions and three
// conversions less).  With h = 2^-24: v32, of three roundings, is within 3h of v (a product with S is exact where it is subnormal, so only the
// last can underflow: |v32| >= least excludes it).
//   Without a bias, e32 = fl(|v32| c) with c >= Gamma (1 + 4.2 h), its successor at most, lies in [1, 1 + 10.4 h] Gamma|v|.
//   With one, y32 = fl(v32 + b) is within h|y32| + 3h|v| of v + b, and 3h u|v| <= 1.5 h Gamma|v|; with c >= Gamma (1 + 6.8 h) and
//   cu >= u (1 + 3.2 h), fma(cu, |y32| + e32, e32) lies in [1, 1 + 15.4 h] tau.
// 15.4 h = 9.2e-7; what is left out is of the order h^2.  A NaN, an infinity, a small or zero v go the binary64 way.
// Returns whether binary32 was enough; otherwise tau is left to int8_bound.
__device__ __forceinline__ bool int8_output(int S, float sa, float sw, float b, bool has_bias, const Int8Args& p, float& y, float& tau) {
    const float v = ((float)S * sa) * sw;
    y = has_bias ? v + b : v;
    const float e = fabsf(v) * (abs(S) > p.limit ? p.c3 : p.c2);
    tau = has_bias ? fmaf(p.cu, fabsf(y) + e, e) : e;
    return fabsf(v) >= p.least && fmaxf(fabsf(y), fabsf(v)) <= 0x1p120f;
}

// 16 bytes of a row from column k on; columns from K on read as 0 (nothing beyond the row's K columns is touched).
__device__ __forceinline__ intx4 row16(const signed char* __restrict__ row, long k, long K) {
    intx4 r = {0, 0, 0, 0};
    if (k + 16 <= K) {
        __builtin_memcpy(&r, row + k, 16);
    } else {
        unsigned long long lo = 0, hi = 0;
#pragma unroll 1
        for (long i = K - 1; i >= k; --i) {                  // (at most 15 bytes, the last one first)
            hi = hi << 8 | lo >> 56;
            lo = lo << 8 | (unsigned char)row[i];
        }
        r = intx4{(int)(unsigned)lo, (int)(unsigned)(lo >> 32), (int)(unsigned)hi, (int)(unsigned)(hi >> 32)};
    }
    return r;
}

// What becomes of four neighbouring outputs of one row, from index i on (cols: how many there are; vec: as one vector): stored with
// their bounds, or checked against the claims, which are requested ahead.
__device__ __forceinline__ floatv4 quad_load(const float* __restrict__ src, long i, int cols, bool vec) {
    floatv4 v = {0.f, 0.f, 0.f, 0.f};
    if (vec) {
        v = __builtin_nontemporal_load(reinterpret_cast<const floatv4*>(src + i));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (e < cols) v[e] = src[i + e];
    }
    return v;
}
__device__ __forceinline__ void quad_store(float* __restrict__ dst, long i, int cols, bool vec, floatv4 v) {
    if (vec) {
        __builtin_nontemporal_store(v, reinterpret_cast<floatv4*>(dst + i));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (e < cols) dst[i + e] = v[e];
    }
}
struct Int8Store {
    static constexpr int AHEAD = 1, UNROLL = 4;
    struct Ahead {};
    __device__ __forceinline__ Ahead request(long, int, bool) const { return Ahead(); }
    template <bool BIAS>
    __device__ __forceinline__ void put(const Int8Args& p, long i, int cols, bool vec, intx4 S, float sa, floatv4 sw, floatv4 b, const Ahead&) {
        floatv4 y, t;
        bool ok = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float ye, te;
            ok &= int8_output(S[e], sa, sw[e], b[e], BIAS, p, ye, te);
            y[e] = ye; t[e] = te;
        }
        if (!ok) {
#pragma unroll 1
            for (int e = 0; e < 4; ++e) t[e] = int8_bound(S[e], sa, sw[e], b[e], BIAS, p);
        }
        if (p.y) quad_store(p.y, i, cols, vec, y);
        if (p.tau) quad_store(p.tau, i, cols, vec, t);
    }
};
// (R copies of every bin; errors of 0, which most claims have, are counted in a register: the lanes of a wavefront would queue for one word of LDS)
template <int R>
struct Int8Check {
    const float* y_ref; const float* claimed; double alpha, eps_rel;
    unsigned int* hist; unsigned int* largest; QuickCheck q;
    ThreadAcc acc; unsigned int zeros = 0, known = 0;
    static constexpr int AHEAD = 6, UNROLL = 1;
    struct Ahead { floatv4 c; };
    __device__ __forceinline__ Int8Check(const float* y_ref_, const float* claimed_, double alpha_, double eps_rel_, float quick, unsigned int* hist_, unsigned int* largest_)
        : y_ref(y_ref_), claimed(claimed_), alpha(alpha_), eps_rel(eps_rel_), hist(hist_), largest(largest_), q(quick, eps_rel_) {}
    __device__ __forceinline__ Ahead request(long i, int cols, bool vec) const {
        Ahead a;
        a.c = quad_load(claimed, i, cols, vec);
        return a;
    }
    template <bool BIAS>
    __device__ __forceinline__ void put(const Int8Args& p, long i, int cols, bool vec, intx4 S, float sa, floatv4 sw, floatv4 b, const Ahead& a) {
        floatv4 r;
        if (y_ref) r = quad_load(y_ref, i, cols, vec);
        unsigned int bin[4];
        bool ok = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float ye, te;
            const bool accurate = int8_output(S[e], sa, sw[e], b[e], BIAS, p, ye, te);
            if (!y_ref) r[e] = ye;
            ok &= e >= cols || (accurate && quick_settled(a.c[e], r[e], te * q.alpha, q, known, bin[e]));
        }
        const int rep = threadIdx.x & (R - 1);
        if (ok) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (e >= cols) continue;
                if (bin[e] == 0) ++zeros; else atomicAdd(&hist[bin[e] * R + rep], 1u);
            }
            return;
        }
#pragma unroll 1
        for (int e = 0; e < 4; ++e) {
            float ye, te;
            if (!int8_output(S[e], sa, sw[e], b[e], BIAS, p, ye, te)) te = int8_bound(S[e], sa, sw[e], b[e], BIAS, p);
            if (e < cols) check_one<R>(a.c[e], r[e], te, alpha, eps_rel, hist, rep, acc);
        }
        if (acc.max_bits > known) atomicMax(largest, acc.max_bits);
        known = max(newest(largest), acc.max_bits);
    }
    // (before the histogram is read, with a barrier behind)
    __device__ __forceinline__ void finish() { if (zeros) atomicAdd(&hist[threadIdx.x & (R - 1)], zeros); }
};

// ---- few rows: a workgroup of 16 wavefronts takes all of up to 16 MT rows of A with 16 NT rows of W; the wavefronts share out the
// reduction in chunks of 64 columns and add their sums in LDS, in whole numbers, so in any order.  Operands go from memory to
// registers in the layout of v_mfma_i32_16x16x64_i8 (lane: row lane % 16, columns 16 (lane / 16) on); the order of the columns inside
// a chunk does not matter, as both operands have the same.
constexpr int kInt8Threads = kCheckThreads;
template <int MT, int NT>
struct Int8Tile {
    static constexpr int ROWS = 16 * MT, COLS = 16 * NT;
    __align__(16) int sums[ROWS * COLS];
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
        for (int e = threadIdx.x; e < t.ROWS * t.COLS / 4; e += kInt8Threads) {
            const int row = e / (t.COLS / 4), col = e % (t.COLS / 4) * 4;
            const long m = m0 + row, n = n0 + col, left = p.N - n;
            if (m >= p.M || left <= 0) continue;
            const int cols = left < 4 ? (int)left : 4;
            const bool vec = p.vec && cols == 4;
            const long i = z * p.strideY + m * p.ldy + n;
            const auto ahead = sink.request(i, cols, vec);
            floatv4 w4, b4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                w4[c] = sw[min(n + c, p.N - 1)];
                if (p.bias) b4[c] = p.bias[min(n + c, p.N - 1)];
            }
            const intx4 S = *reinterpret_cast<const intx4*>(&t.sums[row * t.COLS + col]);
            if (p.bias) sink.template put<true>(p, i, cols, vec, S, sa[m], w4, b4, ahead);
            else        sink.template put<false>(p, i, cols, vec, S, sa[m], w4, b4, ahead);
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
__global__ __launch_bounds__(kInt8Threads) void int8_few_check(Int8Args p, const float* y_ref, const float* claimed, double alpha, double eps_rel, float quick, PassOut pass) {
    __shared__ Int8Tile<MT, NT> t;
    __shared__ unsigned int hist[kBins * kReplicas];
    __shared__ unsigned int red[kRedWords];
    __shared__ unsigned int largest;
    for (int i = threadIdx.x; i < kBins * kReplicas; i += kInt8Threads) hist[i] = 0;
    if (threadIdx.x == 0) largest = 0;
    Int8Check<kReplicas> sink(y_ref, claimed, alpha, eps_rel, quick, hist, &largest);
    int8_few_body(p, sink, t);
    sink.finish();
    __syncthreads();
    finish_pass(hist, sink.acc, red, pass);
}

// ---- many rows: a workgroup of 8 wavefronts takes BM x BN outputs, 128 columns of the reduction a stage, two stages in LDS: one is
// multiplied by v_mfma_i32_32x32x32_i8 while the next is on its way.  A stage holds rows of 128 bytes, whose 16-byte units lie at
// place unit ^ (row & 7): the eight rows that a read of a fragment touches at a time then lie in different banks.
// A wavefront takes WM x WN outputs, so that a fragment read from LDS serves WN / 32 or WM / 32 instructions.
// DIRECT: rows of whole units on 16-byte addresses go from memory to LDS without a stop in registers (global_load_lds_dwordx4: lane i's 16 bytes
// land at the wavefront's place + 16 i; an address in scalar registers and a 32-bit offset, as 64-bit addresses per lane stall the SIMD next
// to matrix instructions).  Otherwise they are read from any address into registers while the previous stage is multiplied, then written to LDS.
typedef int intx16 __attribute__((ext_vector_type(16)));
constexpr int kSlabK = 128;
static __device__ __align__(16) const int zero_unit[4] = {0, 0, 0, 0};

template <int BM_, int BN_, int WM_, int WN_>
struct Int8Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, RM = WM / 32, RN = WN / 32;
    static constexpr int WAVES = (BM / WM) * (BN / WN), THREADS = WAVES * kWave;
    static constexpr int NA = BM / 8 / WAVES, NW = BN / 8 / WAVES;           // pieces of 8 rows that a wavefront copies
    static constexpr int STAGE = (BM + BN) * kSlabK;
    static constexpr int SCALES = (BM + 2 * BN) * 4;                         // of the tile's rows and columns, and the bias
};

// Tiles in the order in which workgroups take them: the eight dies (workgroup modulo 8) have consecutive shares, inside which four
// tile rows go along together, so that what one die reads at a time shares rows of A and W in its L2.
struct Int8Grid { unsigned tm, tn, batch, tiles, share; };
__device__ __forceinline__ bool locate(const Int8Grid& g, unsigned t, unsigned& m, unsigned& n, unsigned& z) {
    unsigned at = (t & 7) * g.share + (t >> 3);
    if (at >= g.tiles) return false;
    const unsigned per = g.tm * g.tn;
    z = at / per; at -= z * per;
    const unsigned group = at / (4 * g.tn), first = group * 4, rows = min(4u, g.tm - first), in = at - group * 4 * g.tn;
    n = in / rows; m = first + in - n * rows;
    return true;
}

template <class SH, bool DIRECT>
struct Int8Walk {
    const Int8Args& p;
    char* lds;
    int lane, wave;
    // of the tile: operand rows of this lane's pieces
    const signed char* A; const signed char* W;              // first rows of the tile (scalar)
    unsigned offA[SH::NA], offW[SH::NW];                     // DIRECT: byte offsets of this lane's unit from there
    long rowA[SH::NA], rowW[SH::NW];                         // otherwise the rows' offsets
    int unit;                                                // this lane's unit of a row
    intx4 held[DIRECT ? 1 : SH::NA + SH::NW];

    __device__ __forceinline__ Int8Walk(const Int8Args& p_, char* lds_) : p(p_), lds(lds_) {
        const int tid = threadIdx.x;
        lane = tid & (kWave - 1);
        wave = __builtin_amdgcn_readfirstlane(tid / kWave);
        unit = (lane & 7) ^ (lane >> 3);                     // (row & 7 is lane / 8 in every piece)
    }
    __device__ __forceinline__ void start(long z, long m0, long n0) {
        A = p.A + z * p.strideA + m0 * p.lda;
        W = p.W + z * p.strideW + n0 * p.ldw;
#pragma unroll
        for (int i = 0; i < SH::NA; ++i) {
            const long r = min((long)((wave + i * SH::WAVES) * 8 + (lane >> 3)), p.M - 1 - m0);       // (rows beyond the last repeat it)
            if (DIRECT) offA[i] = (unsigned)(r * p.lda) + unit * 16; else rowA[i] = r * p.lda;
        }
#pragma unroll
        for (int i = 0; i < SH::NW; ++i) {
            const long r = min((long)((wave + i * SH::WAVES) * 8 + (lane >> 3)), p.N - 1 - n0);
            if (DIRECT) offW[i] = (unsigned)(r * p.ldw) + unit * 16; else rowW[i] = r * p.ldw;
        }
    }
    __device__ __forceinline__ unsigned place(int stage, int piece) const {
        return (unsigned)(size_t)(__attribute__((address_space(3))) char*)lds + (unsigned)(stage * SH::STAGE + piece * 1024);
    }
    // columns k .. k + 127 into stage `stage`; units from column K on become 0
    __device__ __forceinline__ void request(int stage, long k) {
        if constexpr (DIRECT) {
            // (written as assembly: the compiler would wait for these copies before every barrier; the waits are the explicit ones in the loop)
            if (k + kSlabK <= p.K) {
                const signed char* a = A + k;
                const signed char* w = W + k;
#pragma unroll
                for (int i = 0; i < SH::NA; ++i)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(place(stage, wave + i * SH::WAVES)), "v"(offA[i]), "s"(a) : "memory");
#pragma unroll
                for (int i = 0; i < SH::NW; ++i)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(place(stage, SH::BM / 8 + wave + i * SH::WAVES)), "v"(offW[i]), "s"(w) : "memory");
            } else {
                const bool in = k + unit * 16 < p.K;         // (K is a whole number of units)
                const char* zero = reinterpret_cast<const char*>(zero_unit);
#pragma unroll
                for (int i = 0; i < SH::NA; ++i)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                                 :: "s"(place(stage, wave + i * SH::WAVES)), "v"(in ? reinterpret_cast<const char*>(A + k) + offA[i] : zero) : "memory");
#pragma unroll
                for (int i = 0; i < SH::NW; ++i)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                                 :: "s"(place(stage, SH::BM / 8 + wave + i * SH::WAVES)), "v"(in ? reinterpret_cast<const char*>(W + k) + offW[i] : zero) : "memory");
            }
        } else {
#pragma unroll
            for (int i = 0; i < SH::NA; ++i) held[i] = row16(A + rowA[i], k + unit * 16, p.K);
#pragma unroll
            for (int i = 0; i < SH::NW; ++i) held[SH::NA + i] = row16(W + rowW[i], k + unit * 16, p.K);
        }
    }
    // DIRECT: what was requested has landed (of this wavefront); otherwise it is written
    __device__ __forceinline__ void commit(int stage) {
        if constexpr (DIRECT) {
            __builtin_amdgcn_s_waitcnt(0x0F70);              // vmcnt(0)
        } else {
#pragma unroll
            for (int i = 0; i < SH::NA; ++i) *reinterpret_cast<intx4*>(lds + stage * SH::STAGE + (wave + i * SH::WAVES) * 1024 + lane * 16) = held[i];
#pragma unroll
            for (int i = 0; i < SH::NW; ++i)
                *reinterpret_cast<intx4*>(lds + stage * SH::STAGE + (SH::BM / 8 + wave + i * SH::WAVES) * 1024 + lane * 16) = held[SH::NA + i];
        }
    }
    __device__ __forceinline__ void multiply(int stage, intx16 (&acc)[SH::RM][SH::RN]) const {
        constexpr int WC = SH::BN / SH::WN;
        const char* a = lds + stage * SH::STAGE + ((wave / WC) * SH::WM + (lane & 31)) * kSlabK;
        const char* w = lds + stage * SH::STAGE + (SH::BM + (wave % WC) * SH::WN + (lane & 31)) * kSlabK;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int at = ((2 * s + (lane >> 5)) ^ (lane & 7)) * 16;
            intx4 av[SH::RM], wv[SH::RN];
#pragma unroll
            for (int i = 0; i < SH::RM; ++i) av[i] = *reinterpret_cast<const intx4*>(a + i * 32 * kSlabK + at);
#pragma unroll
            for (int j = 0; j < SH::RN; ++j) wv[j] = *reinterpret_cast<const intx4*>(w + j * 32 * kSlabK + at);
#pragma unroll
            for (int i = 0; i < SH::RM; ++i)
#pragma unroll
                for (int j = 0; j < SH::RN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(av[i], wv[j], acc[i][j], 0, 0, 0);
        }
    }
};
// The sums of a tile by way of LDS (the stages' memory, a half of the rows at a time where that is what fits) to threads that have four
// neighbouring columns each, so that outputs and claims move as vectors; claims are requested AHEAD rows of a thread before they are needed.
template <class SH, bool BIAS, class Sink>
__device__ __forceinline__ void int8_outputs(const Int8Args& p, const intx16 (&acc)[SH::RM][SH::RN], int lane, int wave, long z, long m0, long n0,
                                             char* lds, const float* scales, Sink& sink) {
    constexpr int WC = SH::BN / SH::WN, PARTS = SH::BM * SH::BN * 4 / (2 * SH::STAGE), RP = SH::RM / PARTS, BAND = SH::WM / PARTS;
    constexpr int QUADS = SH::BN / 4, STEP = SH::THREADS / QUADS, TRIPS = SH::BM / PARTS / STEP, AHEAD = Sink::AHEAD;
    static_assert(PARTS * 2 * SH::STAGE == SH::BM * SH::BN * 4, "a part of the tile fills the stages");
    int* sums = reinterpret_cast<int*>(lds);
    const int col = threadIdx.x % QUADS * 4, row0 = threadIdx.x / QUADS;
    const long left = p.N - n0 - col;
    const int cols = (int)max(min(left, 4L), 0L);
    const bool vec = p.vec && cols == 4;
    const floatv4 sw = *reinterpret_cast<const floatv4*>(scales + SH::BM + col), b = *reinterpret_cast<const floatv4*>(scales + SH::BM + SH::BN + col);
    const long base = z * p.strideY + m0 * p.ldy + n0 + col;
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
        // row of the tile that row r of the part is: every wavefront's rows fall into PARTS bands
        auto row_of = [&](int r) __attribute__((always_inline)) { return r / BAND * SH::WM + part * BAND + r % BAND; };
        __syncthreads();                                     // (nobody reads what lies there any more)
#pragma unroll
        for (int i = 0; i < RP; ++i)
#pragma unroll
            for (int j = 0; j < SH::RN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    sums[((wave / WC) * BAND + i * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * SH::BN + (wave % WC) * SH::WN + j * 32 + (lane & 31)] = acc[part * RP + i][j][v];
        __syncthreads();
        typename Sink::Ahead ahead[AHEAD];
        auto ask = [&](int trip) __attribute__((always_inline)) {
            const int row = row_of(row0 + trip * STEP);
            const bool inside = trip < TRIPS && m0 + row < p.M;
            return sink.request(inside ? base + row * p.ldy : 0, inside ? cols : 0, inside && vec);
        };
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) ahead[a] = ask(a);
#pragma unroll Sink::UNROLL
        for (int trip = 0; trip < TRIPS; ++trip) {
            const typename Sink::Ahead mine = ahead[0];
#pragma unroll
            for (int a = 0; a + 1 < AHEAD; ++a) ahead[a] = ahead[a + 1];
            ahead[AHEAD - 1] = ask(trip + AHEAD);
            const int r = row0 + trip * STEP, row = row_of(r);
            if (m0 + row >= p.M || cols == 0) continue;
            sink.template put<BIAS>(p, base + row * p.ldy, cols, vec, *reinterpret_cast<const intx4*>(sums + r * SH::BN + col), scales[row], sw, b, mine);
        }
    }
}
template <class SH, bool DIRECT, class Sink>
__device__ __forceinline__ void int8_tiles_body(const Int8Args& p, const Int8Grid& grid, Sink& sink, char* lds) {
    Int8Walk<SH, DIRECT> walk(p, lds);
    float* scales = reinterpret_cast<float*>(lds + 2 * SH::STAGE);           // [BM], [BN], bias [BN]
    const int slabs = (int)((p.K + kSlabK - 1) / kSlabK);
    for (unsigned t = blockIdx.x; (t >> 3) < grid.share; t += gridDim.x) {
        unsigned tm, tn, z;
        if (!locate(grid, t, tm, tn, z)) continue;
        const long m0 = (long)tm * SH::BM, n0 = (long)tn * SH::BN;
        walk.start(z, m0, n0);
        intx16 acc[SH::RM][SH::RN];
#pragma unroll
        for (int i = 0; i < SH::RM; ++i)
#pragma unroll
            for (int j = 0; j < SH::RN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
        if (slabs > 0) walk.request(0, 0);
        for (int i = threadIdx.x; i < SH::BM; i += SH::THREADS) scales[i] = p.sa[z * p.M + min(m0 + i, p.M - 1)];
        for (int i = threadIdx.x; i < SH::BN; i += SH::THREADS) {
            const long n = min(n0 + i, p.N - 1);
            scales[SH::BM + i] = p.sw[(p.strideW ? z * p.N : 0) + n];
            scales[SH::BM + SH::BN + i] = p.bias ? p.bias[n] : 0.f;
        }
        for (int g = 0; g < slabs; ++g) {
            if (DIRECT || g == 0) walk.commit(g & 1);
            __syncthreads();                                 // stage g is whole, and nobody reads the other one any more
            if (g + 1 < slabs) walk.request((g + 1) & 1, (long)(g + 1) * kSlabK);
            walk.multiply(g & 1, acc);
            if (!DIRECT && g + 1 < slabs) walk.commit((g + 1) & 1);
        }
        if (slabs == 0) __syncthreads();                     // (the scales are in place)
        if (p.bias) int8_outputs<SH, true>(p, acc, walk.lane, walk.wave, z, m0, n0, lds, scales, sink);
        else        int8_outputs<SH, false>(p, acc, walk.lane, walk.wave, z, m0, n0, lds, scales, sink);
        __syncthreads();                                     // (the scales and the stages are the next tile's)
    }
}
template <class SH, bool DIRECT>
__global__ __launch_bounds__(SH::THREADS) void int8_tiles(Int8Args p, Int8Grid grid) {
    extern __shared__ __align__(16) char lds[];
    Int8Store sink;
    int8_tiles_body<SH, DIRECT>(p, grid, sink, lds);
}
constexpr int kTileReplicas = 2;
template <class SH, bool DIRECT>
__global__ __launch_bounds__(SH::THREADS) void int8_tiles_check(Int8Args p, Int8Grid grid, const float* y_ref, const float* claimed, double alpha, double eps_rel,
                                                                float quick, CheckWorkspace w) {
    extern __shared__ __align__(16) char lds[];
    unsigned int* hist = reinterpret_cast<unsigned int*>(lds + 2 * SH::STAGE + SH::SCALES);
    unsigned int* rest = hist + kBins * kTileReplicas;       // largest error, three counters of every wavefront
    const int tid = threadIdx.x, wave = tid / kWave;
    for (int i = tid; i < kBins * kTileReplicas; i += SH::THREADS) hist[i] = 0;
    if (tid == 0) rest[0] = 0;
    __syncthreads();
    Int8Check<kTileReplicas> sink(y_ref, claimed, alpha, eps_rel, quick, hist, rest);
    int8_tiles_body<SH, DIRECT>(p, grid, sink, lds);
    sink.finish();
    const unsigned int v = wave_sum(sink.acc.violations), q = wave_sum(sink.acc.nans), m = wave_max(sink.acc.max_bits);
    if ((tid & (kWave - 1)) == 0) { rest[4 + wave * 3] = v; rest[4 + wave * 3 + 1] = q; rest[4 + wave * 3 + 2] = m; }
    __syncthreads();
    if (tid == 0) {
        unsigned long long vs = 0, qs = 0;
        unsigned int ms = 0;
        for (int i = 0; i < SH::WAVES; ++i) { vs += rest[4 + i * 3]; qs += rest[4 + i * 3 + 1]; ms = max(ms, rest[4 + i * 3 + 2]); }
        BlockStats& o = w.stats[blockIdx.x];
        o.violations = vs; o.nans = qs; o.max_bits = ms;
    }
    flush_histogram<kTileReplicas>(hist, w.hist + (size_t)blockIdx.x * kBins, w.coarse + blockIdx.x * kGroups);
}
template <class SH> constexpr int tile_lds(bool check) {
    return 2 * SH::STAGE + SH::SCALES + (check ? kBins * kTileReplicas * 4 + (4 + 3 * SH::WAVES) * 4 : 0);
}
typedef Int8Shape<256, 256, 128, 64> Int8Wide;
typedef Int8Shape<128, 128, 64, 32> Int8Mid;
static_assert(Int8Wide::THREADS == 512 && Int8Mid::THREADS == 512 && tile_lds<Int8Wide>(true) <= 160 * 1024, "one workgroup a compute unit");

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
    p.g2 = gamma_up(2, md); p.g3 = gamma_up(3, md); p.u = md.u;
    if (!(p.g2 == p.g2) || !(p.g3 == p.g3)) return TAO_ERR_K_RANGE;
    p.limit = 1.0 / md.u >= 2147483647.0 ? 2147483647 : (int)std::floor(1.0 / md.u);
    p.vec = ldy % 4 == 0 && strideY % 4 == 0;                // (and the tensors' addresses, below)
    p.uflow = (md.flags & TAO_FLAG_UNDERFLOW_TERMS) ? 0x1p-149 : 0.0;
    auto up = [](double v) { const float f = (float)v; return (double)f < v ? std::nextafterf(f, INFINITY) : f; };
    const double h = 0x1p-24, k = bias ? 6.8 : 4.2;
    p.c2 = up(p.g2 * (1.0 + k * h)); p.c3 = up(p.g3 * (1.0 + k * h)); p.cu = up(md.u * (1.0 + 3.2 * h));
    // (binary32 results stay normal from 2^-100 on for an ordinary unit roundoff; Gamma(2) >= 2u is what the derivation with a bias uses)
    p.least = md.u >= 0x1p-25 && p.g2 >= 2.0 * md.u && p.uflow == 0.0 ? 0x1p-100f : INFINITY;
    return TAO_OK;
}

// Which kernel: `few` where the rows are few or the outputs too few to give every compute unit a tile of 128 x 128; of the tiles the large ones
// where there are enough of them.
enum { kFewTiny, kFewTall, kFewSquare, kMidTiles, kWideTiles };
static int int8_kind(const Int8Args& p) {
    auto tiles = [&](long bm, long bn) { return (double)((p.M + bm - 1) / bm) * (double)((p.N + bn - 1) / bn) * (double)p.batch; };
    if (p.M <= 16) return kFewTiny;
    if (p.M <= 64) return kFewTall;
    const int cus = device_cus();
    if (tiles(256, 256) >= cus / 2) return kWideTiles;
    if (tiles(128, 128) >= cus / 2) return kMidTiles;
    return tiles(64, 64) >= cus / 2 ? kFewSquare : kFewTall;
}
template <class SH> static bool int8_grid(const Int8Args& p, Int8Grid* g) {
    const long tm = (p.M + SH::BM - 1) / SH::BM, tn = (p.N + SH::BN - 1) / SH::BN;
    const __int128 tiles = (__int128)tm * tn * p.batch;
    if (tiles >= (1L << 31) - 8) return false;
    g->tm = (unsigned)tm; g->tn = (unsigned)tn; g->batch = (unsigned)p.batch; g->tiles = (unsigned)tiles; g->share = (unsigned)((tiles + 7) / 8);
    return true;
}
// (a lane's offset inside the tile has 32 bits)
static bool int8_direct(const Int8Args& p, int rows) {
    return p.K % 16 == 0 && p.lda % 16 == 0 && p.ldw % 16 == 0 && p.strideA % 16 == 0 && p.strideW % 16 == 0 && aligned(p.A, 16) && aligned(p.W, 16) &&
           (p.lda + kSlabK) * rows < (1L << 31) && (p.ldw + kSlabK) * rows < (1L << 31);
}
template <class K> static hipError_t allow_lds(K kernel, int bytes) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <class SH> static int int8_launch_tiles(const Int8Args& p, const Int8Grid& g, hipStream_t st) {
    static OncePerDevice once;
    const hipError_t e = once.run([] {
        const hipError_t e = allow_lds(int8_tiles<SH, true>, tile_lds<SH>(false));
        return e != hipSuccess ? e : allow_lds(int8_tiles<SH, false>, tile_lds<SH>(false));
    });
    if (e != hipSuccess) { g_last_hip_error = (int)e; return TAO_ERR_LAUNCH; }
    const dim3 grid(g.share * 8 < (1u << 22) ? g.share * 8 : 1u << 22), blk(SH::THREADS);
    if (int8_direct(p, SH::BM)) hipLaunchKernelGGL((int8_tiles<SH, true>), grid, blk, tile_lds<SH>(false), st, p, g);
    else                        hipLaunchKernelGGL((int8_tiles<SH, false>), grid, blk, tile_lds<SH>(false), st, p, g);
    return launch_status();
}
template <class SH> static int int8_launch_check(const Int8Args& p, const Int8Grid& g, int nblocks, const float* y_ref, const float* claimed, double alpha, double eps_rel,
                                                 float quick, const CheckWorkspace& w, hipStream_t st) {
    static OncePerDevice once;
    const hipError_t e = once.run([] {
        const hipError_t e = allow_lds(int8_tiles_check<SH, true>, tile_lds<SH>(true));
        return e != hipSuccess ? e : allow_lds(int8_tiles_check<SH, false>, tile_lds<SH>(true));
    });
    if (e != hipSuccess) { g_last_hip_error = (int)e; return TAO_ERR_LAUNCH; }
    const dim3 grid(nblocks), blk(SH::THREADS);
    if (int8_direct(p, SH::BM)) hipLaunchKernelGGL((int8_tiles_check<SH, true>), grid, blk, tile_lds<SH>(true), st, p, g, y_ref, claimed, alpha, eps_rel, quick, w);
    else                        hipLaunchKernelGGL((int8_tiles_check<SH, false>), grid, blk, tile_lds<SH>(true), st, p, g, y_ref, claimed, alpha, eps_rel, quick, w);
    return launch_status();
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
    p.vec = p.vec && aligned(y, 16) && aligned(tau, 16);
    hipStream_t st = (hipStream_t)stream;
    int kind = int8_kind(p);
    Int8Grid g;
    if (kind == kWideTiles && int8_grid<Int8Wide>(p, &g)) return int8_launch_tiles<Int8Wide>(p, g, st);
    if (kind == kMidTiles && int8_grid<Int8Mid>(p, &g)) return int8_launch_tiles<Int8Mid>(p, g, st);
    auto few = [&](auto kernel, long rows, long cols) {
        const __int128 tiles = (__int128)((M + rows - 1) / rows) * ((N + cols - 1) / cols) * batch;
        hipLaunchKernelGGL(kernel, dim3(tiles < (1 << 20) ? (unsigned)tiles : 1u << 20), dim3(kInt8Threads), 0, st, p);
    };
    if (kind == kFewTiny)      few(int8_few<1, 1>, 16, 16);
    else if (kind == kFewTall) few(int8_few<4, 1>, 64, 16);
    else                       few(int8_few<4, 4>, 64, 64);
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
    p.vec = p.vec && aligned(claimed, 16) && aligned(y_ref, 16);
    tao_fp_model md;
    resolve_model(model, &md);                               // (validated above)
    const float quick = quick_alpha(alpha, md);
    int kind = int8_kind(p), nblocks = 1;
    Int8Grid g;
    if ((kind == kWideTiles && int8_grid<Int8Wide>(p, &g)) || (kind == kMidTiles && int8_grid<Int8Mid>(p, &g))) {
        nblocks = g.share * 8 < kMaxCheckBlocks ? g.share * 8 : kMaxCheckBlocks;
        const int rc = kind == kWideTiles ? int8_launch_check<Int8Wide>(p, g, nblocks, y_ref, claimed, alpha, eps_rel, quick, w, st)
                                          : int8_launch_check<Int8Mid>(p, g, nblocks, y_ref, claimed, alpha, eps_rel, quick, w, st);
        if (rc != TAO_OK) return rc;
        launch_profile_reduce(w, nblocks, (unsigned long long)n, out, st);
        return launch_status();
    }
    auto few = [&](auto kernel, long rows, long cols) {
        const long tiles = n > 0 ? ((M + rows - 1) / rows) * ((N + cols - 1) / cols) * batch : 1;
        nblocks = (int)(tiles < kMaxCheckBlocks ? tiles : kMaxCheckBlocks);
        hipLaunchKernelGGL(kernel, dim3(nblocks), dim3(kInt8Threads), 0, st, p, y_ref, claimed, alpha, eps_rel, quick, pass_out(w, nblocks, n, out));
    };
    if (kind == kFewTiny)      few(int8_few_check<1, 1>, 16, 16);
    else if (kind == kFewTall) few(int8_few_check<4, 1>, 64, 16);
    else                       few(int8_few_check<4, 4>, 64, 64);
    launch_finish(w, nblocks, n, out, st);
    return launch_status();
}

}  // extern "C"
