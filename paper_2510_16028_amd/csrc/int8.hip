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
    double e2, e3, eu, uflow;                   // the bound in binary64 (int8_bound)
    unsigned limit;                             // whole numbers of larger magnitude (beyond_limit) round in the conversion
    float flimit;                               // ... binary32 ones below it do not
    float c2, c3, cu, least;                    // its estimate in binary32 (int8_quad), for |v| from `least` on
};

__device__ __forceinline__ bool beyond_limit(int S, const Int8Args& p) { return (unsigned)S + p.limit > 2u * p.limit; }     // |S| > limit

// The bound of one sum in binary64, with the factor of its upper rounding to binary32 (kUpMul) in the constants: e2 and e3 are Gamma(2) and Gamma(3), times 1 + u where there
// is a bias, eu is u and uflow 2^-149 or 0.  Binary64 holds S sa exactly to a rounding of 2^-53, far inside the margin of that rounding; the sum with the bias may
// cancel, but its rounding is relative to terms that the bound itself carries.  The bound is 6e-8 above its formula on average; in binary32 with a guard for its roundings it was
// 3.9e-7 above and the kernels that store it up to 4 % faster (us, 8192^3 516 against 524, 1536 x 4096 x 4096 37.3 / 39.0, 512 x 768 x 2304 with a bias 8.15 both).
// own: e2, or e3 beyond the limit.
__device__ __forceinline__ double int8_own(int S, const Int8Args& p) { return beyond_limit(S, p) ? p.e3 : p.e2; }
template <bool BIAS>
__device__ __forceinline__ double int8_bound(int S, float sa, float sw, float b, double own, const Int8Args& p) {
    const double s = (double)S;
    double e;
    if constexpr (BIAS) {
        const double v = s * (double)sa * (double)sw;
        e = fma(p.eu, fabs(v + (double)b), own * fabs(v));
    } else {
        e = fabs(s * ((double)sa * own) * (double)sw);       // (neighbours of a row share sa own)
    }
    if (p.uflow != 0.0) e = fma(p.uflow, fabs(s) + fabs((double)sa) + fabs((double)sw) + 1.0, e);
    return e;
}
// ... rounded: below the normal range a step up where the conversion went down; NaN where an operand is not finite, as an infinite bound would admit every finite claim
// (finite ones stay far inside the binary64 range, so a bound that is infinite there comes of an infinite operand).
__device__ __forceinline__ float int8_rounded(double e) {
    float f = (float)e;
    if (f < 0x1p-126f && (double)f < e) f = __uint_as_float(__float_as_uint(f) + 1u);
    return e < INFINITY ? f : NAN;
}
__device__ __forceinline__ float most_of(floatv4 v) { return fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3]))); }
__device__ __forceinline__ float least_of(floatv4 v) { return fminf(fminf(fabsf(v[0]), fabsf(v[1])), fminf(fabsf(v[2]), fabsf(v[3]))); }
// The outputs of four sums of a row: each step rounded.
template <bool BIAS>
__device__ __forceinline__ void int8_outputs(intx4 S, float sa, floatv4 sw, floatv4 b, floatv4& f, floatv4& v, floatv4& y) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { f[e] = (float)S[e]; v[e] = (f[e] * sa) * sw[e]; y[e] = BIAS ? v[e] + b[e] : v[e]; }
}
// ... and estimates of their bounds in binary32, for checks, which need the bound itself only where an estimate leaves a comparison open.  With h = 2^-24: v, of three
// roundings, is within 3h of its value (a product with S is exact where it is subnormal, so only the last can underflow: |v| >= least excludes it), and u times the 3h |v| that
// y has of it is at most 1.5 h Gamma|v|: the estimate is within 8h of the bound.  Returns whether that holds for all four (a NaN, which the tests leave out, has a NaN for
// its estimate) and they are no larger than 2^90 (alpha times a bound is then an ordinary number).
template <bool BIAS>
__device__ __forceinline__ bool int8_quad(const Int8Args& p, intx4 S, float sa, floatv4 sw, floatv4 b, floatv4& y, floatv4& tau) {
    floatv4 f, v;
    int8_outputs<BIAS>(S, sa, sw, b, f, v, y);
    floatv4 c = {p.c2, p.c2, p.c2, p.c2};
    if (!(most_of(f) < p.flimit)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = beyond_limit(S[e], p) ? p.c3 : p.c2;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float t = fabsf(v[e]) * c[e];
        tau[e] = BIAS ? fmaf(p.cu, fabsf(y[e]), t) : t;
    }
    bool ok = least_of(v) >= p.least && most_of(v) <= 0x1p90f;
    if (BIAS) ok = ok && most_of(y) <= 0x1p90f;
    return ok;
}

// 16 bytes of a row from column k on; columns from K on read as 0 (nothing beyond the row's K columns is touched): at the row's end its last
// 16 bytes, moved down.
__device__ __forceinline__ intx4 row16(const signed char* __restrict__ row, long k, long K) {
    intx4 r = {0, 0, 0, 0};
    if (k + 16 <= K) {
        __builtin_memcpy(&r, row + k, 16);
    } else if (k < K) {
        unsigned long long w[2] = {0, 0};
        if (K >= 16) {
            __builtin_memcpy(w, row + K - 16, 16);
            const int beyond = (int)(k + 16 - K) * 8;        // 8 .. 120
            w[0] = beyond >= 64 ? w[1] >> (beyond - 64) : w[0] >> beyond | w[1] << (64 - beyond);
            w[1] = beyond >= 64 ? 0 : w[1] >> beyond;
        } else {
#pragma unroll 1
            for (int i = (int)K - 1; i >= 0; --i) {          // (k is 0)
                w[1] = w[1] << 8 | w[0] >> 56;
                w[0] = w[0] << 8 | (unsigned char)row[i];
            }
        }
        r = intx4{(int)(unsigned)w[0], (int)(unsigned)(w[0] >> 32), (int)(unsigned)w[1], (int)(unsigned)(w[1] >> 32)};
    }
    return r;
}

// What becomes of four neighbouring outputs of one row, from index i on (cols: how many there are): stored with their bounds, or checked
// against the claims, which are requested ahead.  (A vector of four needs the alignment of one: rows of any stride, on any address.)
typedef float floatv4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ floatv4 quad_load(const float* __restrict__ src, long i, int cols) {
    floatv4 v = {0.f, 0.f, 0.f, 0.f};
    if (cols == 4) {
        v = __builtin_nontemporal_load(reinterpret_cast<const floatv4_any*>(src + i));
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e) if (e < cols) v[e] = src[i + e];
    }
    return v;
}
__device__ __forceinline__ void quad_store(float* __restrict__ dst, long i, int cols, floatv4 v) {
    if (cols == 4) {
        __builtin_nontemporal_store(v, reinterpret_cast<floatv4_any*>(dst + i));
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e) if (e < cols) dst[i + e] = v[e];
    }
}
struct Int8Store {
    static constexpr int AHEAD = 1, UNROLL = 4;
    struct Ahead {};
    __device__ __forceinline__ Ahead request(long, int) const { return Ahead(); }
    template <bool BIAS>
    __device__ __forceinline__ void put(const Int8Args& p, long i, int cols, intx4 S, float sa, floatv4 sw, floatv4 b, const Ahead&) {
        floatv4 f, v, y, t;
        int8_outputs<BIAS>(S, sa, sw, b, f, v, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = (float)int8_bound<BIAS>(S[e], sa, sw[e], b[e], p.e2, p);
        if (!(most_of(f) < p.flimit && least_of(t) >= 0x1p-126f && most_of(t) < INFINITY)) {
#pragma unroll 1
            for (int e = 0; e < 4; ++e) t[e] = int8_rounded(int8_bound<BIAS>(S[e], sa, sw[e], b[e], int8_own(S[e], p), p));
        }
        if (p.y) quad_store(p.y, i, cols, y);
        if (p.tau) quad_store(p.tau, i, cols, t);
    }
};
// The histogram of a workgroup: all bins once, and those of errors from 2^-32 to 1, where claims of binary32 outputs mostly fall, four times more:
// a wavefront's errors of one or two steps share a few bins, and lanes that add to one word of LDS queue for it.  Errors of 0 are counted in a register.
struct Int8Bins {
    static constexpr unsigned NEAR = 760, NEARS = 256, COPIES = 4;
    static constexpr int WORDS = kBins + NEARS * COPIES;
    static __device__ __forceinline__ void add(unsigned int* hist, unsigned bin) {
        const unsigned near = bin - NEAR;
        atomicAdd(&hist[near < NEARS ? kBins + near * COPIES + (threadIdx.x & (COPIES - 1)) : bin], 1u);
    }
    static __device__ __forceinline__ unsigned int total(const unsigned int* hist, unsigned bin) {
        unsigned int c = hist[bin];
        const unsigned near = bin - NEAR;
        if (near < NEARS) {
#pragma unroll
            for (unsigned i = 0; i < COPIES; ++i) c += hist[kBins + near * COPIES + i];
        }
        return c;
    }
};
// ROOM: the kernel has registers to spare (one workgroup a compute unit): two rows under way, and the element of the largest error kept.
template <bool ROOM>
struct Int8Check {
    const float* y_ref; const float* claimed; double alpha, eps_rel;
    unsigned int* hist; unsigned int* largest; QuickCheck q; bool ordinary;
    ThreadAcc acc; unsigned int zeros = 0; Farthest top;
    static constexpr int AHEAD = 4, UNROLL = ROOM ? 2 : 1;
    struct Ahead { floatv4 c; };
    __device__ __forceinline__ Int8Check(const float* y_ref_, const float* claimed_, double alpha_, double eps_rel_, float quick, unsigned int* hist_, unsigned int* largest_)
        : y_ref(y_ref_), claimed(claimed_), alpha(alpha_), eps_rel(eps_rel_), hist(hist_), largest(largest_), q(quick, eps_rel_) { ordinary = q.eps < INFINITY && q.alpha > 0.f; }
    __device__ __forceinline__ Ahead request(long i, int cols) const {
        Ahead a;
        a.c = quad_load(claimed, i, cols);
        return a;
    }
    template <bool BIAS>
    __device__ __forceinline__ void put(const Int8Args& p, long i, int cols, intx4 S, float sa, floatv4 sw, floatv4 b, const Ahead& a) {
        floatv4 y, t;
        const bool estimated = int8_quad<BIAS>(p, S, sa, sw, b, y, t);
        // four claims equal to their outputs: errors of 0 inside any bounds that are numbers, as they are where the outputs are (outputs and bounds of 0, of padded rows, too)
        bool same = most_of(y) < INFINITY && !y_ref && cols == 4 && ordinary;
#pragma unroll
        for (int e = 0; e < 4; ++e) same &= a.c[e] == y[e];
        if (same) {
            zeros += 4;
            return;
        }
        if (y_ref) y = quad_load(y_ref, i, cols);
        const unsigned int published = newest(largest);
        bool ok = estimated && cols == 4 && ordinary;
        if (y_ref) ok = ok && most_of(y) <= 0x1p100f;
        if (settle_four<ROOM, false>(a.c, y, t, q, top, largest, published, ok, acc, zeros, [&](unsigned bin) __attribute__((always_inline)) { Int8Bins::add(hist, bin); })) return;
#pragma unroll 1
        for (int e = 0; e < cols; ++e)
            check_one<1>(a.c[e], y[e], int8_rounded(int8_bound<BIAS>(S[e], sa, sw[e], b[e], int8_own(S[e], p), p)), alpha, eps_rel, hist, 0, acc);
        if (!ROOM && acc.max_bits > published) atomicMax(largest, acc.max_bits);
    }
    // (before the histogram is read, with a barrier behind)
    __device__ __forceinline__ void finish() {
        if (zeros) atomicAdd(&hist[0], zeros);
        if (ROOM) settled(top, alpha, eps_rel, acc);
    }
};

// ---- the product: a workgroup takes BM x BN outputs and walks the reduction in slabs of KB columns, of which STAGES lie in LDS: one is
// multiplied by v_mfma_i32_32x32x32_i8 while the next ones are on their way.  A slab holds rows of KB bytes, whose 16-byte units are
// permuted by the row (unit ^ row & 7, or unit ^ row / 2 & 3 for rows of four units): the eight rows that a read of a fragment touches at
// a time then lie in different banks.  A wavefront takes WM x WN outputs, so that a fragment serves WN / 32 or WM / 32 instructions, and reads
// the fragments of one step while it multiplies those of the one before, across the slabs' borders too: the barrier of a slab stands before
// its last step, when all its fragments are in registers and the slab behind it has landed.
// GROUPS: where there are fewer tiles than compute units, several groups of wavefronts of a workgroup share out the reduction, each with
// stages of its own, and their sums are added at the end.
// DIRECT: rows of whole units on 16-byte addresses go from memory to LDS without a stop in registers (global_load_lds_dwordx4: lane i's 16 bytes
// land at the wavefront's place + 16 i; an address in scalar registers and a 32-bit offset, as 64-bit addresses per lane stall the SIMD next
// to matrix instructions).  Otherwise they are read from any address into registers while a slab is multiplied, then written to LDS.
typedef int intx16 __attribute__((ext_vector_type(16)));
static __device__ __align__(16) const int zero_unit[4] = {0, 0, 0, 0};

template <int BM_, int BN_, int WM_, int WN_, int KB_, int STAGES_, int GROUPS_ = 1>
struct Int8Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KB = KB_, STAGES = STAGES_, GROUPS = GROUPS_, RM = WM / 32, RN = WN / 32;
    static constexpr int WAVES = (BM / WM) * (BN / WN), THREADS = WAVES * GROUPS * kWave;      // of a group, of the workgroup
    static constexpr int UNITS = KB / 16, STEPS = KB / 32, PIECE = kWave / UNITS;      // units of a row, matrix steps of a slab, rows that a wavefront copies at a time
    static constexpr int NA = BM / PIECE / WAVES, NW = BN / PIECE / WAVES;
    static constexpr int STAGE = (BM + BN) * KB, LDS = STAGES * STAGE * GROUPS;
    static constexpr int SCALES = (BM + 2 * BN) * 4;                         // of the tile's rows and columns, and the bias
    static constexpr bool TWO = LDS <= 64 * 1024;                            // two workgroups a compute unit
    static_assert(NA * PIECE * WAVES == BM && NW * PIECE * WAVES == BN && (UNITS == 4 || UNITS == 8), "whole pieces");
};

// Tiles in the order in which workgroups take them: the eight dies (workgroup modulo 8) have consecutive shares, inside which four
// tile rows go along together, so that what one die reads at a time shares rows of A and W in its L2.
struct Int8Grid { unsigned tm, tn, tiles, share; };
__device__ __forceinline__ bool locate(const Int8Grid& g, unsigned t, unsigned& m, unsigned& n, unsigned& z) {
    unsigned at = (t & 7) * g.share + (t >> 3);
    if (at >= g.tiles) return false;
    const unsigned per = g.tm * g.tn;
    z = at / per; at -= z * per;
    const unsigned group = at / (4 * g.tn), first = group * 4, rows = min(4u, g.tm - first), in = at - group * 4 * g.tn;
    n = in / rows; m = first + in - n * rows;
    return true;
}

// s_waitcnt: at most n copies from memory on their way, and no access to LDS
__device__ __forceinline__ constexpr int at_most(int n) { return 0x0070 | (n & 15) | (n >> 4 << 14); }
template <class SH, bool DIRECT>
struct Int8Walk {
    const Int8Args& p;
    char* lds;                                               // the group's stages
    int lane, wave, group;                                   // (wavefront of the group)
    // of the tile: operand rows of this lane's pieces
    const signed char* A; const signed char* W;              // first rows of the tile (scalar)
    unsigned offA[SH::NA], offW[SH::NW];                     // DIRECT: byte offsets of this lane's unit from there
    long rowA[SH::NA], rowW[SH::NW];                         // otherwise the rows' offsets
    int unit;                                                // this lane's unit of a row
    intx4 held[DIRECT ? 1 : SH::NA + SH::NW];
    struct Fragments { intx4 a[SH::RM], w[SH::RN]; };

    static __device__ __forceinline__ int turn(int row) { return SH::UNITS == 8 ? row & 7 : row >> 1 & 3; }
    __device__ __forceinline__ Int8Walk(const Int8Args& p_, char* lds_, int tid) : p(p_) {
        lane = tid & (kWave - 1);
        wave = __builtin_amdgcn_readfirstlane(tid / kWave);
        group = wave / SH::WAVES;
        wave -= group * SH::WAVES;
        lds = lds_ + group * SH::STAGES * SH::STAGE;
        unit = (lane % SH::UNITS) ^ turn(lane / SH::UNITS);  // (pieces begin at multiples of eight rows)
    }
    __device__ __forceinline__ void start(long z, long m0, long n0) {
        A = p.A + z * p.strideA + m0 * p.lda;
        W = p.W + z * p.strideW + n0 * p.ldw;
#pragma unroll
        for (int i = 0; i < SH::NA; ++i) {
            const long r = min((long)((wave + i * SH::WAVES) * SH::PIECE + lane / SH::UNITS), p.M - 1 - m0);       // (rows beyond the last repeat it)
            if (DIRECT) offA[i] = (unsigned)(r * p.lda) + unit * 16; else rowA[i] = r * p.lda;
        }
#pragma unroll
        for (int i = 0; i < SH::NW; ++i) {
            const long r = min((long)((wave + i * SH::WAVES) * SH::PIECE + lane / SH::UNITS), p.N - 1 - n0);
            if (DIRECT) offW[i] = (unsigned)(r * p.ldw) + unit * 16; else rowW[i] = r * p.ldw;
        }
    }
    __device__ __forceinline__ unsigned place(int stage, int piece) const {
        return (unsigned)(size_t)(__attribute__((address_space(3))) char*)lds + (unsigned)(stage * SH::STAGE + piece * 1024);
    }
    // columns k .. k + KB - 1 into stage `stage` (DIRECT) or into registers; units from column K on become 0
    __device__ __forceinline__ void request(int stage, int k) {
        if constexpr (DIRECT) {
            // (written as assembly: the compiler would wait for these copies before every barrier; the waits are the explicit ones in the loop.  m0 is a reserved register, which
            // the compiler sets itself right before it needs it: it is not named as overwritten, which the compiler warns of.)
            if (k + SH::KB <= p.K) {
                const signed char* a = A + k;
                const signed char* w = W + k;
#pragma unroll
                for (int i = 0; i < SH::NA; ++i)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(place(stage, wave + i * SH::WAVES)), "v"(offA[i]), "s"(a) : "memory");
#pragma unroll
                for (int i = 0; i < SH::NW; ++i)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(place(stage, SH::BM / SH::PIECE + wave + i * SH::WAVES)), "v"(offW[i]), "s"(w) : "memory");
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
                                 :: "s"(place(stage, SH::BM / SH::PIECE + wave + i * SH::WAVES)), "v"(in ? reinterpret_cast<const char*>(W + k) + offW[i] : zero) : "memory");
            }
        } else {
#pragma unroll
            for (int i = 0; i < SH::NA; ++i) held[i] = row16(A + rowA[i], k + unit * 16, p.K);
#pragma unroll
            for (int i = 0; i < SH::NW; ++i) held[SH::NA + i] = row16(W + rowW[i], k + unit * 16, p.K);
        }
    }
    __device__ __forceinline__ void write(int stage) const {
#pragma unroll
        for (int i = 0; i < SH::NA; ++i) *reinterpret_cast<intx4*>(lds + stage * SH::STAGE + (wave + i * SH::WAVES) * 1024 + lane * 16) = held[i];
#pragma unroll
        for (int i = 0; i < SH::NW; ++i)
            *reinterpret_cast<intx4*>(lds + stage * SH::STAGE + (SH::BM / SH::PIECE + wave + i * SH::WAVES) * 1024 + lane * 16) = held[SH::NA + i];
    }
    __device__ __forceinline__ void read(Fragments& f, int stage, int step) const {
        constexpr int WC = SH::BN / SH::WN;
        const int row = lane & 31, at = row * SH::KB + ((2 * step + (lane >> 5)) ^ turn(row)) * 16;
        const char* a = lds + stage * SH::STAGE + (wave / WC) * SH::WM * SH::KB + at;
        const char* w = lds + stage * SH::STAGE + (SH::BM + (wave % WC) * SH::WN) * SH::KB + at;
#pragma unroll
        for (int i = 0; i < SH::RM; ++i) f.a[i] = *reinterpret_cast<const intx4*>(a + i * 32 * SH::KB);
#pragma unroll
        for (int j = 0; j < SH::RN; ++j) f.w[j] = *reinterpret_cast<const intx4*>(w + j * 32 * SH::KB);
    }
    static __device__ __forceinline__ void multiply(const Fragments& f, intx16 (&acc)[SH::RM][SH::RN]) {
#pragma unroll
        for (int i = 0; i < SH::RM; ++i)
#pragma unroll
            for (int j = 0; j < SH::RN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.a[i], f.w[j], acc[i][j], 0, 0, 0);
    }
    // all of this wavefront's copies but those of the newest SLABS slabs have landed, and its reads of LDS have ended: behind a barrier everybody's
    template <int SLABS>
    static __device__ __forceinline__ void landed() { __builtin_amdgcn_s_waitcnt(at_most(SLABS * (SH::NA + SH::NW))); }
    // the group's share of the reduction: `slabs` slabs (the same number for every group, which meet at the barriers; beyond K all is 0)
    __device__ __forceinline__ void sums(intx16 (&acc)[SH::RM][SH::RN], int slabs) {
        constexpr int S = SH::STAGES;
        const int k0 = group * slabs * SH::KB;
        if constexpr (DIRECT) {
#pragma unroll
            for (int s = 0; s < S; ++s) if (s < slabs) request(s, k0 + s * SH::KB);
            if (slabs >= S) landed<S - 1>(); else landed<0>();
        } else {
            request(0, k0);
            write(0);
        }
        __syncthreads();
        Fragments f[2];
        read(f[0], 0, 0);
        int stage = 0;
        for (int g = 0; g < slabs; ++g) {
            const int next = stage + 1 == S ? 0 : stage + 1;
            if (!DIRECT && g + 1 < slabs) request(next, k0 + (g + 1) * SH::KB);
#pragma unroll
            for (int s = 0; s + 1 < SH::STEPS; ++s) {
                read(f[(s + 1) & 1], stage, s + 1);
                multiply(f[s & 1], acc);
            }
            __builtin_amdgcn_s_waitcnt(at_most(63));         // (on either way: else the last step would wait for the next slab's fragments)
            if (g + 1 < slabs) {
                if constexpr (DIRECT) {
                    if (g + S <= slabs) landed<S - 2>(); else landed<0>();
                } else {
                    write(next);
                }
                __syncthreads();                             // the next slab is whole; of this one all fragments are in registers
                if (DIRECT && g + S < slabs) request(stage, k0 + (g + S) * SH::KB);
                read(f[0], next, 0);
            }
            multiply(f[1], acc);
            stage = next;
        }
    }
};
// The sums of a tile go by way of LDS (the stages' memory, a half of the rows at a time where that is what fits) to threads that have four
// neighbouring columns each, so that outputs and claims move as vectors.  Claims are requested AHEAD rows of a thread before they are needed,
// the first ones with the tile's first slabs.
template <class SH, class Sink>
struct Int8Outputs {
    static constexpr int WC = SH::BN / SH::WN, PARTS = (SH::BM * SH::BN * 4 + SH::STAGES * SH::STAGE - 1) / (SH::STAGES * SH::STAGE), RP = SH::RM / PARTS, BAND = SH::WM / PARTS;
    static constexpr int QUADS = SH::BN / 4, STEP = SH::THREADS / QUADS, ROWS = SH::BM / PARTS, TRIPS = (ROWS + STEP - 1) / STEP, AHEAD = Sink::AHEAD;
    static_assert(SH::RM % PARTS == 0 && STEP > 0, "whole blocks a part, whole rows a trip");
    const Int8Args& p;
    Sink& sink;
    int col, row0, cols, rows;                               // this thread's columns (how many exist) and first row; rows of the tile that exist
    long base;
    typename Sink::Ahead ahead[AHEAD];

    // row of the tile that row r of part `part` is: every wavefront's rows fall into PARTS bands
    static __device__ __forceinline__ int row_of(int part, int r) { return r / BAND * SH::WM + part * BAND + r % BAND; }
    __device__ __forceinline__ typename Sink::Ahead ask(int part, int trip) const {
        const int r = row0 + trip * STEP, row = row_of(part, r);
        const bool inside = r < ROWS && row < rows;
        return sink.request(inside ? base + row * p.ldy : 0, inside ? cols : 0);
    }
    __device__ __forceinline__ Int8Outputs(const Int8Args& p_, Sink& sink_, long z, long m0, long n0, int tid) : p(p_), sink(sink_) {
        col = tid % QUADS * 4; row0 = tid / QUADS;
        cols = (int)max(min(p.N - n0 - col, 4L), 0L);
        rows = (int)min(p.M - m0, (long)SH::BM);
        base = z * p.strideY + m0 * p.ldy + n0 + col;
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) ahead[a] = ask(0, a);
    }
    template <bool BIAS, class Walk>
    __device__ __forceinline__ void put(const intx16 (&acc)[SH::RM][SH::RN], const Walk& walk, const char* lds, const float* scales) {
        const int lane = walk.lane, wave = walk.wave;
        const int* sums = reinterpret_cast<const int*>(lds);  // [group][row][column], a group's in its own stages
        int* mine = reinterpret_cast<int*>(walk.lds);
        const floatv4 sw = *reinterpret_cast<const floatv4*>(scales + SH::BM + col), b = *reinterpret_cast<const floatv4*>(scales + SH::BM + SH::BN + col);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            __syncthreads();                                 // (nobody reads what lies there any more)
#pragma unroll
            for (int i = 0; i < RP; ++i)
#pragma unroll
                for (int j = 0; j < SH::RN; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        mine[((wave / WC) * BAND + i * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * SH::BN + (wave % WC) * SH::WN + j * 32 + (lane & 31)] = acc[part * RP + i][j][v];
            if (part > 0) {
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) ahead[a] = ask(part, a);
            }
            __syncthreads();
#pragma unroll Sink::UNROLL
            for (int trip = 0; trip < TRIPS; ++trip) {
                const typename Sink::Ahead claims = ahead[0];
#pragma unroll
                for (int a = 0; a + 1 < AHEAD; ++a) ahead[a] = ahead[a + 1];
                ahead[AHEAD - 1] = ask(part, trip + AHEAD);
                const int r = row0 + trip * STEP, row = row_of(part, r);
                if (r >= ROWS || row >= rows || cols == 0) continue;
                intx4 S = *reinterpret_cast<const intx4*>(sums + r * SH::BN + col);
#pragma unroll
                for (int g = 1; g < SH::GROUPS; ++g) S += *reinterpret_cast<const intx4*>(sums + g * (SH::STAGES * SH::STAGE / 4) + r * SH::BN + col);
                sink.template put<BIAS>(p, base + row * p.ldy, cols, S, scales[row], sw, b, claims);
            }
        }
    }
};
template <class SH, bool DIRECT, class Sink>
__device__ __forceinline__ void int8_tiles_body(const Int8Args& p, const Int8Grid& grid, Sink& sink, char* lds) {
    float* scales = reinterpret_cast<float*>(lds + SH::LDS);              // [BM], [BN], bias [BN]
    const int slabs = (int)((p.K + SH::KB * SH::GROUPS - 1) / (SH::KB * SH::GROUPS));
    for (unsigned t = blockIdx.x; (t >> 3) < grid.share; t += gridDim.x) {
        unsigned tm, tn, z;
        if (!locate(grid, t, tm, tn, z)) continue;
        const long m0 = (long)tm * SH::BM, n0 = (long)tn * SH::BN;
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                        // (what is formed of it is formed anew for every tile: kept from tile to tile it would take the registers of the sums)
        Int8Walk<SH, DIRECT> walk(p, lds, tid);
        walk.start(z, m0, n0);
        Int8Outputs<SH, Sink> outputs(p, sink, z, m0, n0, tid);
        intx16 acc[SH::RM][SH::RN];
#pragma unroll
        for (int i = 0; i < SH::RM; ++i)
#pragma unroll
            for (int j = 0; j < SH::RN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
        for (int i = threadIdx.x; i < SH::BM; i += SH::THREADS) scales[i] = p.sa[z * p.M + min(m0 + i, p.M - 1)];
        for (int i = threadIdx.x; i < SH::BN; i += SH::THREADS) {
            const long n = min(n0 + i, p.N - 1);
            scales[SH::BM + i] = p.sw[(p.strideW ? z * p.N : 0) + n];
            scales[SH::BM + SH::BN + i] = p.bias ? p.bias[n] : 0.f;
        }
        if (slabs > 0) walk.sums(acc, slabs); else __syncthreads();          // (the scales are in place behind a barrier)
        asm volatile("" : "+v"(walk.lane), "+v"(outputs.col), "+v"(outputs.row0));
        if (p.bias) outputs.template put<true>(acc, walk, lds, scales);
        else        outputs.template put<false>(acc, walk, lds, scales);
        __syncthreads();                                     // (the scales and the stages are the next tile's)
    }
}
template <class SH, bool DIRECT>
__global__ __launch_bounds__(SH::THREADS) void int8_tiles(Int8Args p, Int8Grid grid) {
    extern __shared__ __align__(16) char lds[];
    Int8Store sink;
    int8_tiles_body<SH, DIRECT>(p, grid, sink, lds);
}
// More workgroups than partial results: several add to one of them, which the launch before has cleared (whole numbers, so in any order).
__global__ __launch_bounds__(kCheckThreads) void clear_partials(CheckWorkspace w) {
    const int tid = threadIdx.x;
    for (int i = tid; i < kBins; i += kCheckThreads) w.hist[(size_t)blockIdx.x * kBins + i] = 0;
    if (tid < kGroups) w.coarse[blockIdx.x * kGroups + tid] = 0;
    if (tid == 0) { BlockStats& o = w.stats[blockIdx.x]; o.violations = 0; o.nans = 0; o.max_bits = 0; }
}
// PAIR: two workgroups a compute unit, from two tiles for each on: one's checks go on under the other's products (2048 x 4096 x 12288 200 -> 165 us;
// with one tile each the registers are worth more, 2048 x 2048 x 2048 32 us against 39, and with 288 tiles a launch less, 512 x 768 x 2304 22 against 28).
template <class SH, bool DIRECT, bool PAIR>
__global__ __launch_bounds__(SH::THREADS, PAIR ? SH::THREADS * 2 / (4 * kWave) : 1) void int8_tiles_check(Int8Args p, Int8Grid grid, const float* y_ref, const float* claimed, double alpha, double eps_rel,
                                                                float quick, CheckWorkspace w) {
    extern __shared__ __align__(16) char lds[];
    unsigned int* hist = reinterpret_cast<unsigned int*>(lds + SH::LDS + SH::SCALES);
    unsigned int* rest = hist + Int8Bins::WORDS;       // largest estimate, three counters of every wavefront
    const int tid = threadIdx.x, wave = tid / kWave;
    for (int i = tid; i < Int8Bins::WORDS; i += SH::THREADS) hist[i] = 0;
    if (tid == 0) rest[0] = 0;
    __syncthreads();
    Int8Check<!PAIR && SH::BN < 256> sink(y_ref, claimed, alpha, eps_rel, quick, hist, rest);
    int8_tiles_body<SH, DIRECT>(p, grid, sink, lds);
    sink.finish();
    const unsigned int v = wave_sum(sink.acc.violations), q = wave_sum(sink.acc.nans), m = wave_max(sink.acc.max_bits);
    if ((tid & (kWave - 1)) == 0) { rest[4 + wave * 3] = v; rest[4 + wave * 3 + 1] = q; rest[4 + wave * 3 + 2] = m; }
    __syncthreads();
    const int slot = blockIdx.x % kMaxCheckBlocks;
    const bool shared = gridDim.x > kMaxCheckBlocks;
    if (tid == 0) {
        unsigned long long vs = 0, qs = 0;
        unsigned int ms = 0;
        for (int i = 0; i < SH::THREADS / kWave; ++i) { vs += rest[4 + i * 3]; qs += rest[4 + i * 3 + 1]; ms = max(ms, rest[4 + i * 3 + 2]); }
        BlockStats& o = w.stats[slot];
        if (shared) {
            if (vs) atomicAdd(&o.violations, vs);
            if (qs) atomicAdd(&o.nans, qs);
            if (ms) atomicMax(&o.max_bits, ms);
        } else {
            o.violations = vs; o.nans = qs; o.max_bits = ms;
        }
    }
    unsigned int* bins = w.hist + (size_t)slot * kBins;
    unsigned int* coarse = w.coarse + slot * kGroups;
    for (int b = tid; b < kBins; b += SH::THREADS) {         // (a wavefront covers a group of 64 bins)
        const unsigned int c = Int8Bins::total(hist, b), g = wave_sum(c);
        const bool first = (tid & (kWave - 1)) == 0;
        if (shared) {
            if (c) atomicAdd(&bins[b], c);
            if (first && g) atomicAdd(&coarse[b / kBinsPerReduceBlock], g);
        } else {
            bins[b] = c;
            if (first) coarse[b / kBinsPerReduceBlock] = g;
        }
    }
}
template <class SH> constexpr int tile_lds(bool check) {
    return SH::LDS + SH::SCALES + (check ? Int8Bins::WORDS * 4 + (4 + 3 * SH::THREADS / kWave) * 4 : 0);
}
typedef Int8Shape<32, 32, 32, 32, 128, 2, 8> Int8Tiny;                       // 136 KB of LDS
typedef Int8Shape<32, 64, 32, 32, 128, 3, 4> Int8Flat;                       // 144 KB
typedef Int8Shape<64, 64, 32, 32, 128, 2, 2> Int8Small;                      // 64 KB: two workgroups a compute unit
typedef Int8Shape<128, 128, 64, 32, 128, 2> Int8Mid;                         // 64 KB
typedef Int8Shape<256, 256, 128, 64, 128, 2> Int8Wide;                       // 128 KB
static_assert(tile_lds<Int8Tiny>(true) <= 160 * 1024 && tile_lds<Int8Flat>(true) <= 160 * 1024 &&
              tile_lds<Int8Wide>(true) <= 160 * 1024 && tile_lds<Int8Small>(true) <= 80 * 1024 && tile_lds<Int8Mid>(true) <= 80 * 1024, "a compute unit's LDS");

// ---- quantisation of rows: scale = fl(max|x| fl(1/127)), q = round(fl(x / scale)), ties to even.  A row that is not finite has scale NaN
// and q = 0 (so the product is NaN, which no check admits); a row of zeros, or one so small that its scale rounds to 0, scale 0 and q = 0.
// A team of lanes holds its row in registers, so x is read once: 16 lanes or a wavefront for the short rows (several to a workgroup, no barrier), a
// workgroup for the long ones, which reads what goes beyond its registers again.  A row is taken in fours at any alignment, the last of
// them moved back to the row's end (the elements that two lanes then write are the same).  GPU us of 8 x 4096 2.8 (6.7 element by
// element), 2048 x 12288 21 (41), 5.9 TB/s, 100000 x 64 6.1 (47): the memory and, below 100 rows, one read of it.
struct QuantizeArgs { const float* x; signed char* q; float* scale; long rows, cols, ld, ldq; };
typedef float rowfloats __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned rowbytes __attribute__((aligned(1)));
__device__ __forceinline__ floatv4 four_of(const float* x) { return *reinterpret_cast<const rowfloats*>(x); }
// One quotient, as its definition.
__device__ __forceinline__ int quantized(float x, float s) { return s > 0.f ? (int)fminf(fmaxf(rintf(x / s), -127.f), 127.f) : 0; }
// Four.  x / s by v_rcp_f32 is within 127 (2^-22 + 2^-24) < 2^-14 of the rounded quotient, so whole numbers that it is not within 2^-13 of the middle of
// are those of the quotient, which is below 127.5; adding 3 2^22 rounds them and leaves them in the low byte.  The other fours (about one in two thousand), and
// rows whose scale is as small as its reciprocal is large, are divided.
__device__ __forceinline__ unsigned quantized_four(const floatv4& x, float s, float r) {
    unsigned b[4];
    float off = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float t = x[e] * r, w = t + 0x1.8p23f;
        b[e] = __float_as_uint(w);
        off = fmaxf(off, fabsf(t - (w - 0x1.8p23f)));
    }
    if (!(s >= 0x1p-100f && off <= 0.5f - 0x1p-13f)) {
        floatv4 v = x;
        unsigned word = 0;
#pragma unroll 1
        for (int e = 0; e < 4; ++e) { word = word >> 8 | (unsigned)quantized(v[0], s) << 24; v = v.yzww; }
        return word;
    }
    return __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u) | __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
}
__device__ __forceinline__ unsigned magnitude(const floatv4& v) {       // (as a whole number, so a NaN is the largest)
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
    return m;
}
// LANES lanes, of THREADS, a row, V fours each; REST: longer rows.
template <int LANES, int V, int THREADS, bool REST>
__global__ __launch_bounds__(THREADS) void quantize_rows(QuantizeArgs p) {
    constexpr int TEAMS = THREADS / LANES, WAVES = LANES / kWave;
    __shared__ unsigned most[WAVES > 1 ? WAVES : 1];
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    const long fours = (p.cols + 3) / 4;
    for (long r = (long)blockIdx.x * TEAMS + team; r < p.rows; r += (long)gridDim.x * TEAMS) {
        const float* x = p.x + r * p.ld;
        signed char* q = p.q + r * p.ldq;
        floatv4 v[V];
        unsigned m = 0;
        auto at = [&](long i) __attribute__((always_inline)) { return min(i * 4, p.cols - 4); };
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const long i = k * LANES + lane;
            v[k] = floatv4{0.f, 0.f, 0.f, 0.f};
            if (i < fours) v[k] = four_of(x + at(i));
        }
#pragma unroll
        for (int k = 0; k < V; ++k) m = max(m, magnitude(v[k]));
        if constexpr (REST)
            for (long i = V * LANES + lane; i < fours; i += LANES) m = max(m, magnitude(four_of(x + at(i))));
        constexpr int STEPS = LANES == 16 ? 4 : 6;
        m = wave_all<0, STEPS>(m, [](unsigned a, unsigned b) { return max(a, b); });
        if constexpr (WAVES > 1) {
            if (lane % kWave == 0) most[lane / kWave] = m;
            __syncthreads();
            m = most[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) m = max(m, most[w]);
            __syncthreads();                                 // (the next row's)
        }
        const float s = m < 0x7f800000u ? __uint_as_float(m) * (1.f / 127.f) : NAN, inverse = __builtin_amdgcn_rcpf(s);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const long i = k * LANES + lane;
            if (i < fours) *reinterpret_cast<rowbytes*>(q + at(i)) = quantized_four(v[k], s, inverse);
        }
        if constexpr (REST)
            for (long i = V * LANES + lane; i < fours; i += LANES)
                *reinterpret_cast<rowbytes*>(q + at(i)) = quantized_four(four_of(x + at(i)), s, inverse);
        if (lane == 0) p.scale[r] = s;
    }
}
// Rows of less than four elements: a thread each.
__global__ __launch_bounds__(256) void quantize_short_rows(QuantizeArgs p) {
    for (long r = (long)blockIdx.x * 256 + threadIdx.x; r < p.rows; r += (long)gridDim.x * 256) {
        unsigned m = 0;
        for (long c = 0; c < p.cols; ++c) m = max(m, __float_as_uint(p.x[r * p.ld + c]) & 0x7fffffffu);
        const float s = m < 0x7f800000u ? __uint_as_float(m) * (1.f / 127.f) : NAN;
        for (long c = 0; c < p.cols; ++c) p.q[r * p.ldq + c] = (signed char)quantized(p.x[r * p.ld + c], s);
        p.scale[r] = s;
    }
}
template <int LANES, int V, int THREADS, bool REST>
static void quantize_launch(const QuantizeArgs& p, hipStream_t st) {
    const long teams = THREADS / LANES, blocks = (p.rows + teams - 1) / teams, most = 256L * 64;
    hipLaunchKernelGGL((quantize_rows<LANES, V, THREADS, REST>), dim3((unsigned)(blocks < most ? blocks : most)), dim3(THREADS), 0, st, p);
}
static void quantize_launch(const QuantizeArgs& p, hipStream_t st) {
    const long fours = (p.cols + 3) / 4;
    if (p.cols < 4) {
        const long blocks = (p.rows + 255) / 256;
        hipLaunchKernelGGL(quantize_short_rows, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, p);
    }
    else if (fours <= 16)        quantize_launch<16, 1, 256, false>(p, st);
    else if (fours <= 16 * 4)    quantize_launch<16, 4, 256, false>(p, st);
    else if (fours <= 64 * 4)    quantize_launch<64, 4, 256, false>(p, st);
    else if (fours <= 256 * 4)   quantize_launch<256, 4, 256, false>(p, st);
    else if (fours <= 256 * 16)  quantize_launch<256, 16, 256, false>(p, st);
    else                         quantize_launch<1024, 8, 1024, true>(p, st);
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
    const double g2 = gamma_up(2, md), g3 = gamma_up(3, md), own = (bias ? 1.0 + md.u : 1.0) * kUpMul;
    if (!(g2 == g2) || !(g3 == g3)) return TAO_ERR_K_RANGE;
    p.e2 = g2 * own; p.e3 = g3 * own; p.eu = md.u * kUpMul;
    p.uflow = (md.flags & TAO_FLAG_UNDERFLOW_TERMS) ? 0x1p-149 * kUpMul : 0.0;
    p.limit = 1.0 / md.u >= 2147483647.0 ? 2147483647u : (unsigned)std::floor(1.0 / md.u);
    p.flimit = (float)p.limit > 0x1p24f ? 0x1p24f : (float)p.limit;      // (those below 2^24 are the whole numbers themselves)
    p.c2 = (float)p.e2; p.c3 = (float)p.e3; p.cu = (float)p.eu;
    // (binary32 results stay normal from 2^-100 on for an ordinary unit roundoff; Gamma(2) >= 2u is what the estimate with a bias uses)
    p.least = md.u >= 0x1p-25 && g2 >= 2.0 * md.u && p.uflow == 0.0 ? 0x1p-100f : INFINITY;
    return TAO_OK;
}

// Which tiles: the smallest ones that one round of the compute units takes, their groups sharing out the reduction; 64 x 64 from there on, 128 x 128
// from three quarters of a round of those on, 256 x 256 where its whole rounds are less than those of 128 x 128 (a tile of four times the size in about
// 3.5 times the time).  Measured on 256 units, us, output and bound stored: 64 x 4096 x 4096 (M x K x N) 32 x 32 6.6, 32 x 64 7.8, 64 x 64 10.2, 128 x 128 20.8;
// 8 x 4096 x 12288 13.8, 11.1, 13.6, 22.8; 128 x 4096 x 4096 11.4, 8.3, 10.5, 22.1; 64 x 4096 x 12288 19.0, 16.1, 14.6, 24.1; 512 x 4096 x 4096 43.5, 30.1,
// 18.0, 24.0; 1536 x 4096 x 4096 64 x 64 51.0, 128 x 128 39.8, 256 x 256 60.9; 4096 x 4096 x 4096 128 x 128 91, 256 x 256 80;
// 2048 x 4096 x 12288 132, 141; 8192 x 8192 x 8192 637, 542.
enum { kTinyTiles, kFlatTiles, kSmallTiles, kMidTiles, kWideTiles };
static int int8_kind(const Int8Args& p) {
    auto tiles = [&](long bm, long bn) { return (double)((p.M + bm - 1) / bm) * (double)((p.N + bn - 1) / bn) * (double)p.batch; };
    const double cus = device_cus();
    if (tiles(32, 32) <= cus) return kTinyTiles;
    if (tiles(32, 64) <= cus) return kFlatTiles;
    if (tiles(128, 128) < 0.75 * cus) return kSmallTiles;
    return std::ceil(tiles(256, 256) / cus) * 3.5 < tiles(128, 128) / cus ? kWideTiles : kMidTiles;
}
template <class SH> static bool int8_grid(const Int8Args& p, Int8Grid* g) {
    const long tm = (p.M + SH::BM - 1) / SH::BM, tn = (p.N + SH::BN - 1) / SH::BN;
    const __int128 tiles = (__int128)tm * tn * p.batch;
    if (tiles >= (1L << 31) - 8) return false;
    g->tm = (unsigned)tm; g->tn = (unsigned)tn; g->tiles = (unsigned)tiles; g->share = (unsigned)((tiles + 7) / 8);
    return true;
}
// (a lane's offset inside the tile has 32 bits)
static bool int8_direct(const Int8Args& p, int rows) {
    return p.K % 16 == 0 && p.lda % 16 == 0 && p.ldw % 16 == 0 && p.strideA % 16 == 0 && p.strideW % 16 == 0 && aligned(p.A, 16) && aligned(p.W, 16) &&
           (p.lda + 128) * rows < (1L << 31) && (p.ldw + 128) * rows < (1L << 31);
}
template <class K> static hipError_t allow_lds(K kernel, int bytes) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <class SH> static int int8_launch_tiles(const Int8Args& p, hipStream_t st) {
    Int8Grid g;
    if (!int8_grid<SH>(p, &g)) return TAO_ERR_SHAPE;
    static OncePerDevice once;
    const hipError_t e = once.run([] {
        const hipError_t e = allow_lds(int8_tiles<SH, true>, tile_lds<SH>(false));
        return e != hipSuccess ? e : allow_lds(int8_tiles<SH, false>, tile_lds<SH>(false));
    });
    if (e != hipSuccess) { g_last_hip_error = (int)e; return TAO_ERR_LAUNCH; }
    const dim3 grid(g.share * 8 < (1u << 22) ? g.share * 8 : 1u << 22), blk(SH::THREADS);
    if (int8_direct(p, SH::BM > SH::BN ? SH::BM : SH::BN)) hipLaunchKernelGGL((int8_tiles<SH, true>), grid, blk, tile_lds<SH>(false), st, p, g);
    else hipLaunchKernelGGL((int8_tiles<SH, false>), grid, blk, tile_lds<SH>(false), st, p, g);
    return launch_status();
}
struct Int8CheckArgs { const float* y_ref; const float* claimed; double alpha, eps_rel; float quick; CheckWorkspace w; long n; tao_profile* out; };
template <class SH, bool PAIR> static int int8_launch_check(const Int8Args& p, const Int8Grid& g, const Int8CheckArgs& c, hipStream_t st) {
    static OncePerDevice once;
    const hipError_t e = once.run([] {
        const hipError_t e = allow_lds(int8_tiles_check<SH, true, PAIR>, tile_lds<SH>(true));
        return e != hipSuccess ? e : allow_lds(int8_tiles_check<SH, false, PAIR>, tile_lds<SH>(true));
    });
    if (e != hipSuccess) { g_last_hip_error = (int)e; return TAO_ERR_LAUNCH; }
    const long places = PAIR ? 2 * kMaxCheckBlocks : kMaxCheckBlocks;
    const int nblocks = g.share == 0 ? 1 : (int)((long)g.share * 8 < places ? g.share * 8 : places), partials = nblocks < kMaxCheckBlocks ? nblocks : kMaxCheckBlocks;
    const dim3 grid(nblocks), blk(SH::THREADS);
    if (nblocks > kMaxCheckBlocks) hipLaunchKernelGGL(clear_partials, dim3(kMaxCheckBlocks), dim3(kCheckThreads), 0, st, c.w);
    if (int8_direct(p, SH::BM > SH::BN ? SH::BM : SH::BN))
        hipLaunchKernelGGL((int8_tiles_check<SH, true, PAIR>), grid, blk, tile_lds<SH>(true), st, p, g, c.y_ref, c.claimed, c.alpha, c.eps_rel, c.quick, c.w);
    else
        hipLaunchKernelGGL((int8_tiles_check<SH, false, PAIR>), grid, blk, tile_lds<SH>(true), st, p, g, c.y_ref, c.claimed, c.alpha, c.eps_rel, c.quick, c.w);
    launch_profile_reduce(c.w, partials, (unsigned long long)c.n, c.out, st);
    return launch_status();
}
template <class SH> static int int8_launch_check(const Int8Args& p, const Int8CheckArgs& c, hipStream_t st) {
    Int8Grid g;
    if (!int8_grid<SH>(p, &g)) return TAO_ERR_SHAPE;
    if constexpr (SH::TWO) {
        if (g.tiles >= 2u * kMaxCheckBlocks) return int8_launch_check<SH, true>(p, g, c, st);
    }
    return int8_launch_check<SH, false>(p, g, c, st);
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
    quantize_launch(QuantizeArgs{x, (signed char*)q, scale, rows, cols, ld, ldq}, (hipStream_t)stream);
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
    hipStream_t st = (hipStream_t)stream;
    switch (int8_kind(p)) {
        case kTinyTiles:  return int8_launch_tiles<Int8Tiny>(p, st);
        case kFlatTiles:  return int8_launch_tiles<Int8Flat>(p, st);
        case kSmallTiles: return int8_launch_tiles<Int8Small>(p, st);
        case kMidTiles:   return int8_launch_tiles<Int8Mid>(p, st);
        default:          return int8_launch_tiles<Int8Wide>(p, st);
    }
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
    tao_fp_model md;
    resolve_model(model, &md);                               // (validated above)
    const Int8CheckArgs c{y_ref, claimed, alpha, eps_rel, quick_alpha(alpha, md), w, n, out};
    switch (int8_kind(p)) {
        case kTinyTiles:  return int8_launch_check<Int8Tiny>(p, c, st);
        case kFlatTiles:  return int8_launch_check<Int8Flat>(p, c, st);
        case kSmallTiles: return int8_launch_check<Int8Small>(p, c, st);
        case kMidTiles:   return int8_launch_check<Int8Mid>(p, c, st);
        default:          return int8_launch_check<Int8Wide>(p, c, st);
    }
}

}  // extern "C"
