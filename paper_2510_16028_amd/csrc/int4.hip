// tao_bound_linear_int4, tao_bound_check_linear_int4: binary32 activations times weights in 4 bits with a scale, and possibly a zero point, for each group,
//     w_jk = (q_jk - z_jg) s_jg,    y_ij = sum_k a_ik w_jk + b_j,    tau_ij = Gamma(K') (sum_k |a_ik||w_jk| + |b_j|),
// a reduction of K products (Sec. 3.1) whose terms are rounded once more for the scale: K' = K + 1, or K + 2 with a bias.
#include <algorithm>
#include "tao_check.hpp"
#include "tao_device.hpp"
#include "tao_host.hpp"

namespace tao {

typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));

// The two sums of an output, and how far a tile's may be off (0 for those of binary64).
struct Int4Sums { double sum, size, err; };
// Tiles of columns and of tokens, whole blocks of the reduction and those of a group of wavefronts, and the last part if a block that is not whole follows (else -1), first workgroup
// of the launch (a grid has fewer than 2^32 threads).
struct Int4Grid { unsigned tiles, token_blocks; int blocks, share, tail; unsigned from; };
// ... relative to the size, for the output to be taken: 14u at most, so that bounds stay within 1e-6; and never so much that the output, rounded, could lie farther off than tau (probabilistic
// models of small lambda, and those of small u).  Models that leave less than kInt4Least, which ordinary tokens' err may reach, take the kernel of any size.
constexpr double kInt4Spare = 14.0 * 0x1p-24, kInt4Least = 2.0 * 0x1p-24;

struct Int4Args {
    const float* A; const unsigned char* W;
    const float* scale; const unsigned char* zero;           // [N][groups], zero may be null
    const float* bias;
    float* y; float* tau;
    Int4Sums* part;                                          // [part][M][N], where the reduction is cut into parts or the outputs are checked
    long part_stride;                                        // outputs of all tokens (a launch may have some of them)
    long M, N, K, lda, ldw, ldy;
    long group; int groups;
    unsigned long per_group;                                 // column / 32 times this over 2^32 is its group (0 for one group; exact up to 2^20 columns)
    double gamma;                    // Gamma(K'), with the margins of the sums' roundings
    double uflow, terms;             // 2^-149 over Gamma(K') or 0, K'
    double spare;                    // how much of its size an output of the tiles may be off before it is rounded
};
// The bound from the sum of magnitudes, rounded up.  NaN where an operand is not finite, as an infinite bound would admit every finite claim (sums of finite operands
// stay inside the binary64 range).
__device__ __forceinline__ float int4_bound(const Int4Args& p, double size, double b) {
    const double e = p.gamma * (size + fabs(b));
    return e < INFINITY ? up32(e) : NAN;
}

// Any size, in binary64: a wavefront an output; the sums in every lane.  A lane has eight neighbouring columns (of one group) at a time, so that a row's loads are few and on their way together.
// (Outputs that tiles leave open come one after the other: 16 x 4096 over 12288 with activations of 10^4 in a third of the blocks take 59 us, 25 without those; two columns at a time 122.  A token that is no number, 1 x 4096 over 4096: 51, 143.)
__device__ __forceinline__ void int4_wave_sums(const Int4Args& p, long i, long j, int lane, double& sum, double& size) {
    const float* a = p.A + i * p.lda;
    const unsigned char* w = p.W + j * p.ldw;
    const bool terms = p.uflow != 0.0;
    double extra = 0.0;
    sum = 0.0; size = 0.0;
    auto add = [&](float v, unsigned code, double s, double z) __attribute__((always_inline)) {
        const double q = ((double)code - z) * s;
        sum = fma((double)v, q, sum);
        size = fma(fabs((double)v), fabs(q), size);
        if (terms) extra += fabs((double)v) + fabs(s);
    };
    for (long k = 8 * lane; k + 8 <= p.K; k += 8 * kWave) {
        const long g = j * p.groups + k / p.group;           // (groups of more than one begin at multiples of 32 columns)
        const double s = (double)p.scale[g], z = p.zero ? (double)p.zero[g] : 8.0;
        unsigned word;
        __builtin_memcpy(&word, w + (k >> 1), 4);
        const floatx4_any lo = *reinterpret_cast<const floatx4_any*>(a + k), hi = *reinterpret_cast<const floatx4_any*>(a + k + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) add(e < 4 ? lo[e & 3] : hi[e & 3], word >> (4 * e) & 15u, s, z);
    }
    const long k = (p.K & ~7L) + lane;                       // the columns behind the last eight
    if (k < p.K) {
        const long g = j * p.groups + k / p.group;
        add(a[k], (unsigned)w[k >> 1] >> (4 * (k & 1)) & 15u, (double)p.scale[g], p.zero ? (double)p.zero[g] : 8.0);
    }
    sum = wave_sum(sum); size = wave_sum(size);
    if (terms) size += p.uflow * (p.terms + wave_sum(extra));
}
// Output and bound from the two sums.
__device__ __forceinline__ void int4_values(const Int4Args& p, long j, const Int4Sums& v, float& y, float& tau) {
    const double b = p.bias ? (double)p.bias[j] : 0.0;
    y = (float)(v.sum + b);
    tau = int4_bound(p, v.size, b);
}
__global__ __launch_bounds__(256) void int4_any(Int4Args p) {
    const long n = p.M * p.N;
    const int lane = threadIdx.x & (kWave - 1);
    for (long at = (long)blockIdx.x * 4 + threadIdx.x / kWave; at < n; at += (long)gridDim.x * 4) {
        const long i = at % p.M, j = at / p.M;
        Int4Sums v;
        int4_wave_sums(p, i, j, lane, v.sum, v.size);
        v.err = 0.0;
        if (lane == 0) {
            if (p.part) { p.part[i * p.N + j] = v; continue; }
            float y, tau;
            int4_values(p, j, v, y, tau);
            if (p.y) p.y[i * p.ldy + j] = y;
            if (p.tau) p.tau[i * p.ldy + j] = tau;
        }
    }
}
// Whether a tile's sums are not exact enough, or no numbers.  (A size of 0 is exact: blocks of zeros and scales of 0 add nothing to either, all others add to both; so a column
// whose codes all equal their zero points has a size of err alone, and is open: 16 x 4096 over 12288 with 64 such columns together 552 us, 26 without, with every sixteenth 61.)
__device__ __forceinline__ bool int4_open(const Int4Args& p, const Int4Sums& v) { return !(v.size < INFINITY) || (v.size > 0.0 && v.err > p.spare * v.size); }
// The wavefront forms those anew, one lane's after the other's.
__device__ __forceinline__ void int4_settle(const Int4Args& p, bool mine, int i, int j, Int4Sums& v) {
    const int lane = threadIdx.x & (kWave - 1);
    unsigned long long open = __ballot(mine && int4_open(p, v));
    while (open) {
        const int l = __builtin_ctzll(open);
        open &= open - 1;
        double sum, size;
        int4_wave_sums(p, __builtin_amdgcn_readlane(i, l), __builtin_amdgcn_readlane(j, l), lane, sum, size);
        if (lane == l) { v.sum = sum; v.size = size; }
    }
}

// ---- tiles in whole numbers.  Both sums go through v_mfma_i32_16x16x64_i8, which is exact: a weight's q - z and |q - z| are bytes (z up to 127; other columns are formed
// in binary64), and 128 activations of a token become whole numbers X = trunc(a 2^(29 - E)), E the exponent of the largest of them, in four digits of base 256 from -128 to
// 127, of X for the output and of |X| for the bound.  A digit is a row of its own (4 t + digit), so that a lane finds a token's digits in neighbouring registers.  Sums of 128
// products of a digit stay below 2^21; the digits are put together and scaled in binary64.
// What truncation leaves off: at most one unit of every X, so with dmax >= |q - z| the sum of |X||q - z| lies within [exact - 128 dmax, exact] units: the bound takes the upper end, and
//     err = sum over the blocks of |s| 2^(E - 29) 128 dmax
// is how far it may lie above, and how far y may be off.  An output with err <= spare size <= 14u size has exact <= size <= exact (1 + 14u), so tau, rounded up, is within 16.1u < 1e-6 of its formula, and
// y, rounded once, within 15u, and Gamma(K'), of the sum of magnitudes; others (blocks whose largest activation is hundreds of times the usual one, while its weight is 0) are formed in binary64.
// For ordinary tokens err is about 0.5u size (largest activation of 128 about 3.5 times the mean, dmax twice the mean of |q - z|).
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
constexpr int kInt4Block = 128;                              // columns of a block
constexpr int kInt4Codes = kInt4Block / 2 + 16;              // bytes of a column's codes of a block in LDS
constexpr unsigned kInt4Row = kInt4Block + 16;               // bytes of a digit's row in LDS (16 more: the eight rows that are read at a time lie in different banks)

// Few tiles of up to eight tokens: a workgroup has 16 columns, its KW wavefronts share out the reduction, and each forms the digits of its blocks by itself.  A wavefront has the tokens in RT row tiles
// of four; fewer tokens are there again in the other rows.
template <int TOKENS_, int WAVES_>
struct Int4Shape {
    static constexpr int TOKENS = TOKENS_, CT = 1, NW = 1, KW = 8, WAVES = WAVES_, THREADS = KW * kWave, COLUMNS = 16;
    static constexpr int RT = (TOKENS + 3) / 4, ALIKE = TOKENS < 4 ? TOKENS : 4, SLOTS = RT;       // ALIKE: tokens of a row tile, SLOTS: outputs of a lane
    static constexpr int PIECES = TOKENS * kInt4Block / 8;   // of eight activations, in a block
    static constexpr int BLOCKS = PIECES < kWave ? kWave / PIECES : 1, UNITS = BLOCKS * PIECES / kWave;      // blocks of a chunk, pieces that a lane brings
    static constexpr int SET = TOKENS * 4 * kInt4Row, BLOCK = 2 * SET, DIGITS = BLOCKS * (BLOCK + 8 * TOKENS);     // bytes: digits of X, and of |X|; their units behind them
    static constexpr int CODES = 16 * kInt4Codes;            // of a wavefront
    static constexpr int SUMS = KW * SLOTS * kWave * (int)sizeof(Int4Sums);
    static constexpr int STAGES = KW * (DIGITS + CODES), LDS = STAGES > SUMS ? STAGES : SUMS;
    static_assert(BLOCKS * PIECES == UNITS * kWave && DIGITS % 16 == 0, "whole blocks a chunk");
    static_assert(LDS <= 160 * 1024, "a compute unit's");
};

// 16 bytes of a row of weights from byte `at` on; bytes from `bytes` on are not touched (the activations there are 0): at the row's end its last 16 bytes, moved down.
__device__ __forceinline__ uintx4 int4_bytes(const unsigned char* __restrict__ row, int at, int bytes) {
    uintx4 r = {0, 0, 0, 0};
    if (at + 16 <= bytes) {
        __builtin_memcpy(&r, row + at, 16);
    } else if (at < bytes) {
        unsigned long long w[2] = {0, 0};
        if (bytes >= 16) {
            __builtin_memcpy(w, row + bytes - 16, 16);
            const int beyond = (at + 16 - bytes) * 8;        // 8 .. 120
            w[0] = beyond >= 64 ? w[1] >> (beyond - 64) : w[0] >> beyond | w[1] << (64 - beyond);
            w[1] = beyond >= 64 ? 0 : w[1] >> beyond;
        } else {
#pragma unroll 1
            for (int i = bytes - at - 1; i >= 0; --i) {
                w[1] = w[1] << 8 | w[0] >> 56;
                w[0] = w[0] << 8 | row[at + i];
            }
        }
        r = uintx4{(unsigned)w[0], (unsigned)(w[0] >> 32), (unsigned)w[1], (unsigned)(w[1] >> 32)};
    }
    return r;
}
// Eight codes less their zero point and the magnitudes of that, as bytes: the even ones, then the odd ones.  biased: 127 + z in every byte, so that v = biased - q
// has its top bit where q < z, is 127 - d elsewhere and 128 + (|d| - 1) there.  (No byte borrows from the next.  Additions, shifts and bitwise operations of two operands take a SIMD half
// the time of the others here: 2.6 cycles, 4.6.)
__device__ __forceinline__ void int4_codes(unsigned w, unsigned biased, int* d, int* m) {
    const unsigned half[2] = {w & 0x0f0f0f0fu, w >> 4 & 0x0f0f0f0fu};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const unsigned v = biased - half[i], n = v >> 7 & 0x01010101u;
        d[i] = (int)(v ^ 0x7f7f7f7fu);
        m[i] = (int)((v ^ (n + 0x7f7f7f7fu)) + n);
    }
}
// A tile of 16 digits' rows by 16 columns, over 64 columns of the reduction or 32 (WORDS 2 or 1): a lane has 16 or 8 bytes of a row and of a column.
template <int WORDS>
__device__ __forceinline__ intx4 int4_product(const char* row, const int* d, intx4 sum) {
    if constexpr (WORDS == 2) return __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const intx4*>(row), intx4{d[0], d[1], d[2], d[3]}, sum, 0, 0, 0);
    else return __builtin_amdgcn_mfma_i32_16x16x32_i8(*reinterpret_cast<const long*>(row), (long)((unsigned long)(unsigned)d[1] << 32 | (unsigned)d[0]), sum, 0, 0, 0);
}
// byte j of four words
__device__ __forceinline__ void int4_transpose(const unsigned (&w)[4], unsigned (&digit)[4]) {
    const unsigned a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);      // bytes 0 and 1 of two words
    const unsigned c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), e = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);      // ... 2 and 3
    digit[0] = __builtin_amdgcn_perm(b, a, 0x05040100u); digit[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    digit[2] = __builtin_amdgcn_perm(e, c, 0x05040100u); digit[3] = __builtin_amdgcn_perm(e, c, 0x07060302u);
}
// Sums over `columns` columns of a column's scale and biased zero point and a token's unit, from the products of their digits.  (The size comes without err, which the end adds.)
__device__ __forceinline__ void int4_fold(const intx4& y, const intx4& t, float scale, unsigned biased, int columns, double unit, Int4Sums& v) {
    const int z = (int)(biased & 255u) - 127;
    const double by = (double)scale * unit, size = fabs(by);
    v.sum = fma(by, fma((double)(y[2] + (y[3] << 8)), 65536.0, (double)(y[0] + (y[1] << 8))), v.sum);
    v.size = fma(size, fma((double)(t[2] + (t[3] << 8)), 65536.0, (double)(t[0] + (t[1] << 8))), v.size);
    v.err = fma(size, (double)(max(z, 15 - z) * columns), v.err);              // (units that truncation may have left off)
}
// Eight activations as digits, with the unit of their block (a row of 16 lanes has a block of a token): four times (even ones, odd ones) for X, then for |X|.
__device__ __forceinline__ double int4_digits_of(const float (&a)[8], uint2 (&digit)[2][4]) {
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(a[i]) & 0x7fffffffu);
    most = wave_all<0, 4>(most, [](unsigned x, unsigned y) { return max(x, y); });
    const int E = max((int)(most >> 23), 1) - 127;
    unsigned x[2][2][4];                                     // [set][even or odd]
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned m = (unsigned)__builtin_amdgcn_ldexpf(fabsf(a[i]), 29 - E), sign = (unsigned)(__float_as_int(a[i]) >> 31);
        x[0][i & 1][i >> 1] = (((m ^ sign) - sign) + 0x00808080u) ^ 0x00808080u;
        x[1][i & 1][i >> 1] = (m + 0x00808080u) ^ 0x00808080u;
    }
#pragma unroll
    for (int set = 0; set < 2; ++set) {
        unsigned even[4], odd[4];
        int4_transpose(x[set][0], even);
        int4_transpose(x[set][1], odd);
#pragma unroll
        for (int j = 0; j < 4; ++j) digit[set][j] = make_uint2(even[j], odd[j]);
    }
    // (0 where all are 0, which is exact; NaN where one is not finite)
    return most == 0 ? 0.0 : most >= 0x7f800000u ? (double)NAN : ldexp(1.0, E - 29);
}
// The values of four rows of 16 lanes, each to all lanes of its column.
__device__ __forceinline__ void int4_spread(unsigned v, unsigned* to) {
    const auto pairs = __builtin_amdgcn_permlane32_swap(v, v, false, false);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto rows = __builtin_amdgcn_permlane16_swap(pairs[i], pairs[i], false, false);
        to[2 * i] = rows[0]; to[2 * i + 1] = rows[1];
    }
}
// A column's scale and biased zero point of four folds, or of two for two tiles of columns, from the rows of 16 lanes that read them.  (A column whose zero point does not fit the
// bytes gets NaN: its outputs are then formed in binary64.)
__device__ __forceinline__ void int4_factors(bool zeroed, float s, unsigned char own_z, unsigned* scale, unsigned* biased) {
    const unsigned z = zeroed ? own_z : 8u;
    int4_spread(__builtin_amdgcn_perm(0u, 127u + min(z, 127u), 0u), biased);
    int4_spread(z > 127u ? 0x7fc00000u : __float_as_uint(s), scale);
}
__device__ __forceinline__ int int4_group(const Int4Args& p, int column) { return min((int)((unsigned long)(column >> 5) * p.per_group >> 32), p.groups - 1); }
// Order between the lanes of a wavefront: LDS takes its accesses in order, so only the compiler has to keep it.
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The end of a workgroup: its groups' sums meet in LDS, where every wavefront takes some of the outputs: parts of the reduction, or outputs and bounds.
template <class SH>
__device__ __forceinline__ void int4_finish(const Int4Args& p, char* lds, const Int4Sums (&total)[SH::SLOTS], long m0, long n0) {
    constexpr int NW = SH::NW, KW = SH::KW, SLOTS = SH::SLOTS, CT = SH::CT;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    constexpr int OUT = SLOTS * kWave;                      // of a wavefront: [output of a lane][lane]
    __syncthreads();
    Int4Sums* sums = reinterpret_cast<Int4Sums*>(lds);       // [group][wavefront][output]
#pragma unroll
    for (int o = 0; o < SLOTS; ++o) sums[wave * OUT + o * kWave + lane] = total[o];
    __syncthreads();
#pragma unroll 1
    for (int o = threadIdx.x; o < NW * OUT; o += SH::THREADS) {
        Int4Sums v = sums[o];
#pragma unroll
        for (int k = 1; k < KW; ++k) {
            const Int4Sums& other = sums[k * NW * OUT + o];
            v.sum += other.sum; v.size += other.size; v.err += other.err;
        }
        v.size += v.err;
        const int slot = o / kWave % SLOTS, q = o >> 4 & 3, t = slot / CT * 4 + q, c = slot % CT;
        const long i = m0 + t, j = n0 + (o / OUT * CT + c) * 16 + (o & 15);
        const bool own = t < SH::TOKENS && i < p.M && j < p.N;
        if (p.part) {
            if (own) p.part[blockIdx.y * p.part_stride + i * p.N + j] = v;
            continue;
        }
        int4_settle(p, own, (int)i, (int)j, v);
        if (own) {
            const long to = i * p.ldy + j;
            float out, tau;
            int4_values(p, j, v, out, tau);
            if (p.y) p.y[to] = out;
            if (p.tau) p.tau[to] = tau;
        }
    }
}

// What a lane requests of a chunk: pieces of eight activations, of each block 16 bytes of weights, and of the scales and zero points of the chunk's folds every fourth for one column.
template <class SH, int FOLDS>
struct Int4Chunk {
    static constexpr int FACTORS = (SH::BLOCKS * FOLDS + 3) / 4;
    floatx4_any a[SH::UNITS][2];
    uintx4 raw[SH::BLOCKS];
    float s[FACTORS];
    unsigned char z[FACTORS];
};

// Weights are read in lines: four lanes a row's 64 bytes of a block, and handed to the lanes of their columns through LDS (a load whose lanes have a row each takes the address
// unit a cycle or two a lane: with 16 bytes a lane four times as long).
// FOLDS: how often a block's sums are scaled (1: groups of whole blocks, 2: of halves, 4: of 32 columns)
template <class SH, int FOLDS>
__global__ __launch_bounds__(SH::THREADS, SH::WAVES) void int4_tiles(Int4Args p, Int4Grid grid) {
    extern __shared__ __align__(16) char lds[];
    constexpr int RT = SH::RT, KW = SH::KW, SLOTS = SH::SLOTS, TOKENS = SH::TOKENS, BLOCKS = SH::BLOCKS;
    constexpr int STEP = FOLDS == 4 ? 32 : 64, STEPS = kInt4Block / STEP, WORDS = STEP / 32;       // columns of a matrix instruction, those of a block, words of a lane's codes for one
    using Chunk = Int4Chunk<SH, FOLDS>;
    // workgroups of one tile of columns on one die (workgroup modulo 8), whose cache then holds their weights
    const unsigned rest = (grid.from + blockIdx.x) >> 3, up = grid.token_blocks == 1 ? rest : rest / grid.token_blocks, tile = up * 8 + (blockIdx.x & 7);
    if (tile >= grid.tiles) return;
    const int lane = threadIdx.x & (kWave - 1), col = lane & 15, piece = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const long n0 = (long)tile * SH::COLUMNS, m0 = (long)(rest - up * grid.token_blocks) * SH::TOKENS;
    // whole blocks are shared out among the wavefronts of all parts
    const int blocks = grid.blocks, first = min((int)(blockIdx.y * KW + wave) * grid.share, blocks), last = min(first + grid.share, blocks);
    const unsigned char* row_w = p.W + min(n0 + lane / 4, p.N - 1) * p.ldw + lane % 4 * 16;
    const long n = min(n0 + col, p.N - 1);
    const float* scales = p.scale + n * p.groups;
    const bool zeroed = p.zero != nullptr;
    const unsigned char* zeros = zeroed ? p.zero + n * p.groups : reinterpret_cast<const unsigned char*>(scales);        // (bytes that are there, where there are none: a load all the same)
    const int zero_step = zeroed ? 1 : 0;
    // this lane's pieces of eight activations of a chunk
    const int at = lane / 16, own_block = at % BLOCKS, own_token = at / BLOCKS, unit = lane % 16;
    const float* a_row[SH::UNITS];
#pragma unroll
    for (int u = 0; u < SH::UNITS; ++u) a_row[u] = p.A + min(m0 + own_token + u * (4 / BLOCKS), p.M - 1) * p.lda + unit * 8;

    Int4Sums total[SLOTS];
#pragma unroll
    for (int o = 0; o < SLOTS; ++o) total[o] = Int4Sums{0.0, 0.0, 0.0};
    char* digits = lds + wave * SH::DIGITS;
    double* units = reinterpret_cast<double*>(digits + BLOCKS * SH::BLOCK);
    char* codes = lds + KW * SH::DIGITS + wave * SH::CODES;
    const int row = lane & (4 * SH::ALIKE - 1), token = piece & (SH::ALIKE - 1);     // a lane's row of a row tile, its token of the products'

    auto factors = [&](Chunk& w, int block) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < Chunk::FACTORS; ++i) {
            int g = 0;
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int of = int4_group(p, block * kInt4Block + (i * 4 + f) * (kInt4Block / FOLDS));
                g = f == 0 || lane >= f * 16 ? of : g;
            }
            w.s[i] = scales[g];
            w.z[i] = zeros[g * zero_step];
        }
    };
    // (nothing here branches, so that what is on its way is known where it is waited for: blocks behind the wavefront's last one repeat it)
    auto request = [&](Chunk& w, int block) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) __builtin_memcpy(&w.raw[i], row_w + min(block + i, last - 1) * (kInt4Block / 2), 16);
        const int first_column = min(block + own_block, last - 1) * kInt4Block;
#pragma unroll
        for (int u = 0; u < SH::UNITS; ++u) {
            const float* a = a_row[u] + first_column;
            w.a[u][0] = *reinterpret_cast<const floatx4_any*>(a); w.a[u][1] = *reinterpret_cast<const floatx4_any*>(a + 4);
        }
        factors(w, block);
    };
    // activations to digits in LDS
    auto write = [&](const floatx4_any (&a)[2], int token) __attribute__((always_inline)) {
        const float v[8] = {a[0][0], a[0][1], a[0][2], a[0][3], a[1][0], a[1][1], a[1][2], a[1][3]};
        uint2 digit[2][4];
        const double by = int4_digits_of(v, digit);
        char* to = digits + own_block * SH::BLOCK + token * 4 * kInt4Row + unit * 8;
#pragma unroll
        for (int set = 0; set < 2; ++set)
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<uint2*>(to + set * SH::SET + j * kInt4Row) = digit[set][j];
        if (unit == 0) units[own_block * SH::TOKENS + token] = by;
    };
    // block i of the chunk
    auto multiply = [&](const uintx4& raw, int i, const unsigned (&scale)[4 * Chunk::FACTORS], const unsigned (&biased)[4 * Chunk::FACTORS]) __attribute__((always_inline)) {
        wave_order();
        *reinterpret_cast<uintx4*>(codes + lane / 4 * kInt4Codes + lane % 4 * 16) = raw;
        wave_order();
        const char* from = codes + col * kInt4Codes + piece * (4 * WORDS);
        const char* rows = digits + i * SH::BLOCK + row * kInt4Row + piece * (8 * WORDS);
        intx4 y[RT], t[RT];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int f = i * FOLDS + s * FOLDS / STEPS;
            const bool fresh = s % (STEPS / FOLDS) == 0;
            int d[2 * WORDS], m[2 * WORDS];
#pragma unroll
            for (int w = 0; w < WORDS; ++w) int4_codes(*reinterpret_cast<const unsigned*>(from + s * (STEP / 2) + 4 * w), biased[f], d + 2 * w, m + 2 * w);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const intx4 none = {0, 0, 0, 0};
                y[r] = int4_product<WORDS>(rows + r * 16 * kInt4Row + s * STEP, d, fresh ? none : y[r]);
                t[r] = int4_product<WORDS>(rows + r * 16 * kInt4Row + s * STEP + SH::SET, m, fresh ? none : t[r]);
            }
            if ((s + 1) % (STEPS / FOLDS) != 0) continue;
#pragma unroll
            for (int r = 0; r < RT; ++r) int4_fold(y[r], t[r], __uint_as_float(scale[f]), biased[f], kInt4Block / FOLDS, units[i * TOKENS + r * 4 + token], total[r]);
        }
    };
    auto chunk = [&](const Chunk& now, int block, int limit) __attribute__((always_inline)) {
        wave_order();
#pragma unroll
        for (int u = 0; u < SH::UNITS; ++u) write(now.a[u], own_token + u * (4 / BLOCKS));
        unsigned scale[4 * Chunk::FACTORS], biased[4 * Chunk::FACTORS];          // of the folds
#pragma unroll
        for (int i = 0; i < Chunk::FACTORS; ++i) int4_factors(zeroed, now.s[i], now.z[i], scale + 4 * i, biased + 4 * i);
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
            if (block + i < limit) multiply(now.raw[i], i, scale, biased);
    };
    if (first < last) {
        Chunk now, next;
        request(now, first);
        for (int block = first;;) {
            if (block + BLOCKS < last) request(next, block + BLOCKS);
            chunk(now, block, last);
            block += BLOCKS;
            if (block >= last) break;
            now = next;
        }
    }
    if (grid.tail == (int)blockIdx.y && wave == KW - 1) {    // the last block, which is not whole, goes to the last wavefront (columns that do not exist have activations of 0)
        Chunk odd;
        const int columns = own_block == 0 ? (int)(p.K % kInt4Block) - unit * 8 : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int u = 0; u < SH::UNITS; ++u) odd.a[u][i >> 2][i & 3] = i < columns ? a_row[u][(long)blocks * kInt4Block + i] : 0.f;
        odd.raw[0] = int4_bytes(row_w - lane % 4 * 16, blocks * (kInt4Block / 2) + lane % 4 * 16, (int)((p.K + 1) / 2));
        factors(odd, blocks);
        chunk(odd, blocks, blocks + 1);
    }
    int4_finish<SH>(p, lds, total, m0, n0);
}

// ---- more tokens: digits are formed once, by a kernel of their own, and lie in the workspace as the products want them: of four tokens and a block
// X, then |X|, of each the steps' 16 rows in the order of the lanes (loads whose lanes have a row each take the address unit a cycle or two a lane: 49 us for 16 x 12288 x 4096).
constexpr int kInt4Tile = 2 * 16 * kInt4Block;               // bytes
__global__ __launch_bounds__(256) void int4_digits(Int4Args p, char* digits, double* units, int blocks, long pieces, int step) {
    const long at = (long)blockIdx.x * 256 + threadIdx.x;
    if (at >= pieces) return;
    const int unit = (int)(at & 15), token = (int)(at >> 4 & 3);
    const long tile = at >> 6, tokens = tile / blocks, block = tile - tokens * blocks, i = tokens * 4 + token, k = block * kInt4Block + unit * 8;
    float a[8];
    const float* from = p.A + i * p.lda + k;
    if (i < p.M && k + 8 <= p.K) {
        const floatx4_any lo = *reinterpret_cast<const floatx4_any*>(from), hi = *reinterpret_cast<const floatx4_any*>(from + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { a[e] = lo[e]; a[4 + e] = hi[e]; }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = i < p.M && k + e < p.K ? from[e] : 0.f;
    }
    uint2 digit[2][4];
    const double by = int4_digits_of(a, digit);
    const int lane = step == 64 ? (unit & 7) >> 1 : unit & 3, wide = step / 4, s = unit * 8 / step;             // (of row 0: the wavefront's row of 16 lanes)
    char* to = digits + tile * kInt4Tile + s * 16 * step + (lane * 16 + token * 4) * wide + (step == 64 ? (unit & 1) * 8 : 0);
#pragma unroll
    for (int set = 0; set < 2; ++set)
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<uint2*>(to + set * 16 * kInt4Block + j * wide) = digit[set][j];
    if (unit == 0) units[tile * 4 + token] = by;
}
template <int TOKENS_, int NW_, int KW_, int WAVES_>
struct Int4Rows {
    static constexpr int TOKENS = TOKENS_, CT = 2, NW = NW_, KW = KW_, WAVES = WAVES_, THREADS = NW * KW * kWave, COLUMNS = 16 * CT * NW, RT = TOKENS / 4, SLOTS = RT * CT;
    static constexpr int DIGITS = RT * kInt4Tile, COPIES = DIGITS / 1024 / NW;   // bytes of a block's digits; pieces of 1024 of them that a wavefront brings
    static constexpr int CODES = 16 * CT * kInt4Codes, STAGES = KW * 2 * DIGITS + NW * KW * CODES;
    static constexpr int SUMS = KW * NW * SLOTS * kWave * (int)sizeof(Int4Sums), LDS = STAGES > SUMS ? STAGES : SUMS;
    static_assert(COPIES * NW * 1024 == DIGITS && LDS <= 160 * 1024, "whole pieces; a compute unit's");
};
template <class SH, int FOLDS>
__global__ __launch_bounds__(SH::THREADS, SH::WAVES) void int4_rows(Int4Args p, Int4Grid grid, const char* __restrict__ digits, const double* __restrict__ units) {
    extern __shared__ __align__(16) char lds[];
    constexpr int RT = SH::RT, CT = SH::CT, NW = SH::NW, KW = SH::KW, SLOTS = SH::SLOTS;
    constexpr int STEP = FOLDS == 4 ? 32 : 64, STEPS = kInt4Block / STEP, WORDS = STEP / 32, FACTORS = (FOLDS * CT + 3) / 4;
    const unsigned rest = (grid.from + blockIdx.x) >> 3, up = grid.token_blocks == 1 ? rest : rest / grid.token_blocks, tile = up * 8 + (blockIdx.x & 7);
    if (tile >= grid.tiles) return;
    const int lane = threadIdx.x & (kWave - 1), col = lane & 15, piece = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), kg = wave / NW, nw = wave % NW;
    const long n0 = (long)tile * SH::COLUMNS + 16 * CT * nw, m0 = (long)(rest - up * grid.token_blocks) * SH::TOKENS;
    const int blocks = grid.blocks, every = blocks + (p.K % kInt4Block != 0);
    const int first = min((int)(blockIdx.y * KW + kg) * grid.share, blocks), last = min(first + grid.share, blocks);
    const int trips = min(grid.share, blocks), all = trips + (grid.tail == (int)blockIdx.y);       // (every group's, as they meet at barriers)
    // the group's block of a trip, or -1: the last one, which is not whole, goes to the last group
    auto block_of = [&](int trip) __attribute__((always_inline)) {
        return trip < trips ? (first + trip < last ? first + trip : -1) : trip < all && kg == KW - 1 ? blocks : -1;
    };
    const unsigned char* rows_w[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) rows_w[c] = p.W + min(n0 + lane / 4 + 16 * c, p.N - 1) * p.ldw + lane % 4 * 16;
    const long n = min(n0 + (lane & 31), p.N - 1);
    const float* scales = p.scale + n * p.groups;
    const bool zeroed = p.zero != nullptr;
    const unsigned char* zeros = zeroed ? p.zero + n * p.groups : reinterpret_cast<const unsigned char*>(scales);
    const int zero_step = zeroed ? 1 : 0;
    const char* mine = digits + m0 / 4 * every * kInt4Tile;
    const double* tokens = units + m0 / 4 * every * 4 + piece;

    Int4Sums total[SLOTS];
#pragma unroll
    for (int o = 0; o < SLOTS; ++o) total[o] = Int4Sums{0.0, 0.0, 0.0};
    char* stages = lds + kg * 2 * SH::DIGITS;
    char* codes = lds + KW * 2 * SH::DIGITS + wave * SH::CODES;
    const unsigned stages_at = __builtin_amdgcn_readfirstlane((unsigned)(unsigned long)(__attribute__((address_space(3))) char*)stages);
    uintx4 raw[CT];
    float s_own[FACTORS];
    unsigned char z_own[FACTORS];
    double unit[RT];
    auto factors = [&](int block) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < FACTORS; ++i) {
            const int g = int4_group(p, block * kInt4Block + (2 * i + lane / 32) * (kInt4Block / FOLDS));
            s_own[i] = scales[g];
            z_own[i] = zeros[g * zero_step];
        }
    };
    // what a block needs, requested a block ahead and waited for together: digits to LDS, the rest to registers
    auto fetch = [&](int block, int stage) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < SH::COPIES; ++i) {
            const int at = nw * SH::COPIES + i, r = at / (kInt4Tile / 1024), part = at % (kInt4Tile / 1024);
            const char* from = mine + ((long)r * every + block) * kInt4Tile + part * 1024;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(stages_at + stage * SH::DIGITS + at * 1024), "v"(lane * 16), "s"(from) : "memory");
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) __builtin_memcpy(&raw[c], rows_w[c] + (long)min(block, blocks - 1) * (kInt4Block / 2), 16);
        factors(block);
#pragma unroll
        for (int r = 0; r < RT; ++r) unit[r] = tokens[((long)r * every + block) * 4];
    };
    int block = block_of(0);
    if (block >= 0) fetch(block, 0);
    for (int trip = 0; trip < all; ++trip) {
        const int after = block_of(trip + 1);
        if (block == blocks) {
            const int from = blocks * (kInt4Block / 2) + lane % 4 * 16, bytes = (int)((p.K + 1) / 2);
#pragma unroll
            for (int c = 0; c < CT; ++c) raw[c] = int4_bytes(rows_w[c] - lane % 4 * 16, from, bytes);
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0)
        unsigned scale[4 * FACTORS], biased[4 * FACTORS];    // [fold][tile of columns]
#pragma unroll
        for (int i = 0; i < FACTORS; ++i) int4_factors(zeroed, s_own[i], z_own[i], scale + 4 * i, biased + 4 * i);
        double by[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) by[r] = unit[r];
        char* to = codes + lane / 4 * kInt4Codes + lane % 4 * 16;
#pragma unroll
        for (int c = 0; c < CT; ++c) *reinterpret_cast<uintx4*>(to + c * 16 * kInt4Codes) = raw[c];
        __syncthreads();                                     // (the group's digits are there, and nobody reads the stage before any more)
        if (after >= 0) fetch(after, (trip + 1) & 1);
        const int now = block;
        block = after;
        if (now < 0) continue;
        const char* rows = stages + (trip & 1) * SH::DIGITS + lane * (8 * WORDS);
        const char* from = codes + col * kInt4Codes + piece * (4 * WORDS);
        intx4 y[RT][CT], t[RT][CT];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int f = s * FOLDS / STEPS * CT;
            const bool fresh = s % (STEPS / FOLDS) == 0;
            int d[CT][2 * WORDS], m[CT][2 * WORDS];
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int w = 0; w < WORDS; ++w)
                    int4_codes(*reinterpret_cast<const unsigned*>(from + c * 16 * kInt4Codes + s * (STEP / 2) + 4 * w), biased[f + c], d[c] + 2 * w, m[c] + 2 * w);
            const intx4 none = {0, 0, 0, 0};
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    y[r][c] = int4_product<WORDS>(rows + r * kInt4Tile + s * 16 * STEP, d[c], fresh ? none : y[r][c]);
                    t[r][c] = int4_product<WORDS>(rows + r * kInt4Tile + 16 * kInt4Block + s * 16 * STEP, m[c], fresh ? none : t[r][c]);
                }
            if ((s + 1) % (STEPS / FOLDS) != 0) continue;
#pragma unroll
            for (int o = 0; o < SLOTS; ++o)
                int4_fold(y[o / CT][o % CT], t[o / CT][o % CT], __uint_as_float(scale[f + o % CT]), biased[f + o % CT], kInt4Block / FOLDS, by[o / CT], total[o]);
        }
    }
    int4_finish<SH>(p, lds, total, m0, (long)tile * SH::COLUMNS);
}
// The parts of the reduction added up, in order: outputs and bounds from them.
__device__ __forceinline__ void int4_joined(const Int4Args& p, int parts, bool own, long at, int& i, int& j, Int4Sums& v) {
    v = Int4Sums{0.0, 0.0, 0.0};
    i = 0; j = 0;
    if (own) {
        i = (int)(at / p.N); j = (int)(at - i * p.N);
        const long n = p.M * p.N;
        for (int k = 0; k < parts; ++k) {
            const Int4Sums o = p.part[k * n + at];
            v.sum += o.sum; v.size += o.size; v.err += o.err;
        }
    }
    int4_settle(p, own, i, j, v);
}
__global__ __launch_bounds__(256) void int4_join(Int4Args p, int parts) {
    const long n = p.M * p.N;
    for (long at0 = (long)blockIdx.x * 256; at0 < n; at0 += (long)gridDim.x * 256) {
        const long at = at0 + threadIdx.x;
        int i, j;
        Int4Sums v;
        int4_joined(p, parts, at < n, at, i, j, v);
        if (at < n) {
            float y, tau;
            int4_values(p, j, v, y, tau);
            if (p.y) p.y[i * p.ldy + j] = y;
            if (p.tau) p.tau[i * p.ldy + j] = tau;
        }
    }
}
// ... and checked.
struct Int4CheckArgs { const float* y_ref; const float* claimed; double alpha, eps_rel; PassOut pass; };
__global__ __launch_bounds__(kCheckThreads) void int4_join_check(Int4Args p, int parts, Int4CheckArgs a) {
    __shared__ unsigned int hist[kBins * kReplicas];
    __shared__ unsigned int red[kRedWords];
    for (int i = threadIdx.x; i < kBins * kReplicas; i += kCheckThreads) hist[i] = 0;
    __syncthreads();
    ThreadAcc acc;
    const int rep = threadIdx.x & (kReplicas - 1);
    const long n = p.M * p.N;
    for (long at0 = (long)blockIdx.x * kCheckThreads; at0 < n; at0 += (long)gridDim.x * kCheckThreads) {
        const long at = at0 + threadIdx.x;
        int i, j;
        Int4Sums v;
        int4_joined(p, parts, at < n, at, i, j, v);
        if (at < n) {
            float y, tau;
            int4_values(p, j, v, y, tau);
            const long place = i * p.ldy + j;
            check_one(a.claimed[place], a.y_ref ? a.y_ref[place] : y, tau, a.alpha, a.eps_rel, hist, rep, acc);
        }
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
    p.A = A; p.W = W; p.scale = scale; p.zero = zero; p.bias = bias; p.y = nullptr; p.tau = nullptr; p.part = nullptr;
    p.part_stride = M * N; p.M = M; p.N = N; p.K = K; p.lda = lda; p.ldw = ldw; p.ldy = ldy;
    p.group = group < K || K == 0 ? group : K + (K & 1);     // (one group: its end at an even column)
    p.groups = (int)((K + p.group - 1) / p.group);
    p.per_group = p.groups > 1 ? (1UL << 32) / (unsigned long)(p.group / 32) + 1 : 0;
    p.gamma = g * (1.0 + ((double)K + 64.0) * 0x1p-52) * kGuard;
    p.uflow = (md->flags & TAO_FLAG_UNDERFLOW_TERMS) ? 0x1p-149 * kGuard / p.gamma : 0.0;
    p.terms = (double)steps;
    p.spare = std::min(kInt4Spare, g * (1.0 - 0x1p-20) - 0x1p-24 * (1.0 + 0x1p-20));
    return TAO_OK;
}
// What a call launches: tiles of up to `tokens` tokens in `parts` parts of the reduction (tokens 0: the kernel of any size), with digits formed beforehand for `slab` tokens at a time
// (0: by the tiles themselves), and of those whether a workgroup has one wavefront's columns or two.
struct Int4Plan { int tokens, parts; long slab; int nw, kw; };
constexpr long kInt4Slab = 64L << 20;                        // bytes of digits that are kept at a time (a few tokens', where those are more)
static Int4Plan int4_plan(long M, long N, long K, bool exact) {
    // (short reductions: a wavefront's lanes are hardly used, and what truncation leaves off would show next to the few roundings that the bound holds)
    if (K <= 32 || K > (1L << 20) || exact) return {0, 1, 0, 1, 1};
    // (Digits formed anew by every tile of 16 columns and eight tokens, or once, by a launch of their own.  us: 8 x 1024 over 8192 7.7 and 8.7, 8 x 4096 over 4096 10.5 and 14.9, 16 x 1024 over 2048 4.8 and 8.7,
    // 16 x 512 over 4096 6.9 and 8.8; where there are more than two tiles a compute unit, 8 x 512 over 16384 10.9 and 7.3; more than one of long reductions, 8 x 4096 over 6144 19.2 and 15.6,
    // 16 x 4096 over 4096 19.3 and 16.4; in long enough ones, 5 x 12288 over 4096 25.5 and 20.5.  Four tokens and fewer by tiles of theirs: 4096 over 12288 15.5 and 18.3.)
    const long work = (N + 15) / 16 * ((M + 7) / 8);
    const bool rows = K >= kInt4Block && M > 4 && (work > 512 || (work > 256 && K > 2048) || work * K >= 1L << 21);
    const long sixteens = (M + 15) / 16;
    const int tokens = M <= 1 ? 1 : M <= 2 ? 2 : M <= 4 ? 4 : M <= 8 || !rows || (N + 63) / 64 * sixteens < 160 ? 8 : 16;
    const long token_blocks = (M + tokens - 1) / tokens, wide = (N + 127) / 128 * token_blocks;
    // columns and groups of a workgroup: the more columns, the fewer read the same digits; four wavefronts where there are two such workgroups a compute unit
    const int nw = !rows ? 1 : tokens == 16 && wide >= 256 ? 4 : 2, kw = !rows ? 8 : nw == 2 ? 4 : wide >= 512 ? 1 : 2;
    // parts until there is a workgroup for each of the chip's 256 compute units (written out: the workspace's size is asked for where there may be no device), of four blocks a group
    // at least, as their sums take a launch more
    const long columns = rows ? 32 * nw : 16;
    const long workgroups = (N + columns - 1) / columns * token_blocks, most = K / kInt4Block / (4 * kw);
    const long parts = std::max(1L, std::min(256 / std::max(workgroups, 1L), most));
    const long fit = kInt4Slab / ((K + kInt4Block - 1) / kInt4Block * kInt4Block * 8) / tokens;
    return {tokens, (int)parts, rows ? tokens * std::min(std::max(fit, 1L), token_blocks) : 0, nw, kw};
}
// Models whose bounds the tiles do not form, or whose tau does not cover what they may be off.
static bool int4_exact(const Int4Args& p) { return p.uflow != 0.0 || p.spare < kInt4Least; }
static size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }
static size_t part_bytes(long M, long N, const Int4Plan& plan) { return plan.parts > 1 ? padded((size_t)plan.parts * (size_t)(M * N) * sizeof(Int4Sums)) : 0; }
// Digits, then units.
static size_t digit_bytes(long K, const Int4Plan& plan) { return (size_t)(plan.slab / 4 * ((K + kInt4Block - 1) / kInt4Block)) * kInt4Tile; }
static size_t unit_bytes(long K, const Int4Plan& plan) { return padded((size_t)(plan.slab * ((K + kInt4Block - 1) / kInt4Block)) * sizeof(double)); }
// Shape SH of a kernel for groups of whole blocks, of halves, or of 32 columns and their multiples.
template <class SH, class... Rest>
static int int4_launch_shape(void (*whole)(Int4Args, Int4Grid, Rest...), void (*halves)(Int4Args, Int4Grid, Rest...), void (*quarters)(Int4Args, Int4Grid, Rest...),
                             const Int4Args& p, int parts, hipStream_t st, Rest... rest) {
    const long tiles = (p.N + SH::COLUMNS - 1) / SH::COLUMNS, token_blocks = (p.M + SH::TOKENS - 1) / SH::TOKENS;
    const __int128 grid = (__int128)((tiles + 7) / 8 * 8) * token_blocks;
    if (grid >= (1L << 32)) return TAO_ERR_SHAPE;            // (none that the arguments' checks let through: 2^31 at most, of one tile of columns)
    static OncePerDevice once;
    const hipError_t e = once.run([&] {
        for (const auto kernel : {whole, halves, quarters}) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
    if (e != hipSuccess) { g_last_hip_error = (int)e; return TAO_ERR_LAUNCH; }
    const long blocks = p.K / kInt4Block, sharers = (long)SH::KW * parts;
    Int4Grid g{(unsigned)tiles, (unsigned)token_blocks, (int)blocks, (int)((blocks + sharers - 1) / sharers), p.K % kInt4Block ? parts - 1 : -1, 0};
    const auto kernel = p.groups <= 1 || p.group % kInt4Block == 0 ? whole : p.group % (kInt4Block / 2) == 0 ? halves : quarters;
    constexpr long most = 1L << 22;                          // workgroups of a launch (whole eights, 2^31 threads)
    for (long from = 0; from < (long)grid; from += most) {
        g.from = (unsigned)from;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min((long)grid - from, most), (unsigned)parts), dim3(SH::THREADS), SH::LDS, st, p, g, rest...);
        const int rc = launch_status();
        if (rc != TAO_OK) return rc;
    }
    return TAO_OK;
}
template <class SH>
static int int4_launch_tiles(const Int4Args& p, int parts, hipStream_t st) {
    return int4_launch_shape<SH>(int4_tiles<SH, 1>, int4_tiles<SH, 2>, int4_tiles<SH, 4>, p, parts, st);
}
template <class SH>
static int int4_launch_rows(const Int4Args& p, int parts, const char* digits, const double* units, hipStream_t st) {
    return int4_launch_shape<SH>(int4_rows<SH, 1>, int4_rows<SH, 2>, int4_rows<SH, 4>, p, parts, st, digits, units);
}
// Slab by slab: digits, then the tiles that read them.
static int int4_launch_slabs(const Int4Args& p, const Int4Plan& plan, char* ws, hipStream_t st) {
    const long blocks = (p.K + kInt4Block - 1) / kInt4Block;
    const int step = p.groups <= 1 || p.group % 64 == 0 ? 64 : 32;         // columns of the products' steps
    double* units = reinterpret_cast<double*>(ws + digit_bytes(p.K, plan));
    for (long m = 0; m < p.M; m += plan.slab) {
        Int4Args q = p;
        q.M = std::min(plan.slab, p.M - m);
        q.A += m * p.lda;
        if (q.y) q.y += m * p.ldy;
        if (q.tau) q.tau += m * p.ldy;
        if (q.part) q.part += m * p.N;
        const long pieces = (q.M + plan.tokens - 1) / plan.tokens * plan.tokens * blocks * 16;
        hipLaunchKernelGGL(int4_digits, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, st, q, ws, units, (int)blocks, pieces, step);
        int rc = launch_status();
        if (rc != TAO_OK) return rc;
        if (plan.tokens == 8) rc = int4_launch_rows<Int4Rows<8, 2, 4, 2>>(q, plan.parts, ws, units, st);
        else if (plan.nw == 2) rc = int4_launch_rows<Int4Rows<16, 2, 4, 2>>(q, plan.parts, ws, units, st);
        else if (plan.kw == 2) rc = int4_launch_rows<Int4Rows<16, 4, 2, 2>>(q, plan.parts, ws, units, st);
        else rc = int4_launch_rows<Int4Rows<16, 4, 1, 2>>(q, plan.parts, ws, units, st);
        if (rc != TAO_OK) return rc;
    }
    return TAO_OK;
}
// The sums (p.part) or, with one part, the outputs.
static int int4_launch(const Int4Args& p, const Int4Plan& plan, char* ws, hipStream_t st) {
    if (plan.slab) return int4_launch_slabs(p, plan, ws, st);
    switch (plan.tokens) {
        case 1:  return int4_launch_tiles<Int4Shape<1, 2>>(p, plan.parts, st);
        case 2:  return int4_launch_tiles<Int4Shape<2, 4>>(p, plan.parts, st);
        case 4:  return int4_launch_tiles<Int4Shape<4, 4>>(p, plan.parts, st);
        case 8:  return int4_launch_tiles<Int4Shape<8, 2>>(p, plan.parts, st);
    }
    const long blocks = (p.M * p.N + 3) / 4;
    hipLaunchKernelGGL(int4_any, dim3((unsigned)(blocks < 256L * 256 ? blocks : 256L * 256)), dim3(256), 0, st, p);
    return launch_status();
}
static bool int4_sizes_ok(long M, long N, long K) {
    const long most = 1L << 31;
    return M >= 0 && N >= 0 && K >= 0 && M < most && N < most && K < most && (__int128)M * N < ((__int128)1 << 36);
}

}  // namespace tao

extern "C" {

size_t tao_linear_int4_workspace_bytes(long M, long N, long K) {
    using namespace tao;
    if (!int4_sizes_ok(M, N, K)) return 0;
    const Int4Plan plan = int4_plan(M, N, K, false);
    return part_bytes(M, N, plan) + digit_bytes(K, plan) + unit_bytes(K, plan);
}

size_t tao_bound_check_linear_int4_workspace_bytes(long M, long N, long K) {
    using namespace tao;
    if (!int4_sizes_ok(M, N, K)) return 0;
    const Int4Plan plan = int4_plan(M, N, K, false);
    return padded(check_workspace_bytes()) + std::max(part_bytes(M, N, plan), padded((size_t)(M * N) * sizeof(Int4Sums))) + digit_bytes(K, plan) + unit_bytes(K, plan);
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
    const Int4Plan plan = int4_plan(M, N, K, int4_exact(p));
    hipStream_t st = (hipStream_t)stream;
    p.y = y; p.tau = tau;
    char* rest = (char*)ws + part_bytes(M, N, plan);
    if (plan.parts == 1) return int4_launch(p, plan, rest, st);
    p.part = (Int4Sums*)ws;
    const int rc2 = int4_launch(p, plan, rest, st);
    if (rc2 != TAO_OK) return rc2;
    const long blocks = (M * N + 255) / 256;
    hipLaunchKernelGGL(int4_join, dim3((unsigned)(blocks < 256L * 64 ? blocks : 256L * 64)), dim3(256), 0, st, p, plan.parts);
    return launch_status();
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
    hipStream_t st = (hipStream_t)stream;
    const Int4Plan plan = int4_plan(M, N, K, int4_exact(p));
    p.part = (Int4Sums*)((char*)ws + padded(check_workspace_bytes()));
    if (n > 0) {
        const int rc2 = int4_launch(p, plan, (char*)p.part + std::max(part_bytes(M, N, plan), padded((size_t)n * sizeof(Int4Sums))), st);
        if (rc2 != TAO_OK) return rc2;
    }
    const long want = (n + kCheckThreads - 1) / kCheckThreads;
    const int nblocks = (int)(want < 1 || n <= kAloneElements ? 1 : want > kMaxCheckBlocks ? kMaxCheckBlocks : want);
    hipLaunchKernelGGL(int4_join_check, dim3(nblocks), dim3(kCheckThreads), 0, st, p, plan.parts, Int4CheckArgs{y_ref, claimed, alpha, eps_rel, pass_out(w, nblocks, n, out)});
    launch_finish(w, nblocks, n, out, st);
    return launch_status();
}

}  // extern "C"
