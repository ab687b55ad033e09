// tao_bound_linear_int4, tao_bound_check_linear_int4: binary32 activations times weights in 4 bits with a scale, and possibly a zero point, for each group,
//     w_jk = (q_jk - z_jg) s_jg,    y_ij = sum_k a_ik w_jk + b_j,    tau_ij = Gamma(K') (sum_k |a_ik||w_jk| + |b_j|),
// a reduction of K products (Sec. 3.1) whose terms are rounded once more for the scale: K' = K + 1, or K + 2 with a bias.
#include <algorithm>
#include "tao_check.hpp"
#include "tao_device.hpp"
#include "tao_host.hpp"

namespace tao {

// The two sums of an output, and how far a tile's may be off (0 for those of binary64).
struct Int4Sums { double sum, size, err; };
// Tiles of columns and of tokens, whole blocks of the reduction and those of a group of wavefronts, and the last part if a block that is not whole follows (else -1).
struct Int4Grid { unsigned tiles, token_blocks; int blocks, share, tail; };
constexpr double kInt4Spare = 14.0 * 0x1p-24;                // ... relative to the size, for the output to be taken

struct Int4Args {
    const float* A; const unsigned char* W;
    const float* scale; const unsigned char* zero;           // [N][groups], zero may be null
    const float* bias;
    float* y; float* tau;
    Int4Sums* part;                                          // [part][M][N], where the reduction is cut into parts or the outputs are checked
    long M, N, K, lda, ldw, ldy;
    long group; int groups;
    unsigned long per_group;                                 // column / 32 times this over 2^32 is its group (0 for one group; exact up to 2^20 columns)
    double gamma;                    // Gamma(K'), with the margins of the sums' roundings
    double uflow, terms;             // 2^-149 over Gamma(K') or 0, K'
};
// The bound from the sum of magnitudes, rounded up.  NaN where an operand is not finite, as an infinite bound would admit every finite claim (sums of finite operands
// stay inside the binary64 range).
__device__ __forceinline__ float int4_bound(const Int4Args& p, double size, double b) {
    const double e = p.gamma * (size + fabs(b));
    return e < INFINITY ? up32(e) : NAN;
}

// Any size, in binary64: a wavefront an output, lanes along the bytes of its row; the sums in every lane.
__device__ __forceinline__ void int4_wave_sums(const Int4Args& p, long i, long j, int lane, double& sum, double& size) {
    const float* a = p.A + i * p.lda;
    const unsigned char* w = p.W + j * p.ldw;
    double extra = 0.0;
    sum = 0.0; size = 0.0;
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
    if (p.uflow != 0.0) size += p.uflow * (p.terms + wave_sum(extra));
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
// Whether a tile's sums are not exact enough, or no numbers: a size of 0 is exact (the tiles see to that).
__device__ __forceinline__ bool int4_open(const Int4Sums& v) { return !(v.size < INFINITY) || (v.size > 0.0 && v.err > kInt4Spare * v.size); }
// The wavefront forms those anew, one lane's after the other's.
__device__ __forceinline__ void int4_settle(const Int4Args& p, bool mine, int i, int j, Int4Sums& v) {
    const int lane = threadIdx.x & (kWave - 1);
    unsigned long long open = __ballot(mine && int4_open(v));
    while (open) {
        const int l = __builtin_ctzll(open);
        open &= open - 1;
        double sum, size;
        int4_wave_sums(p, __builtin_amdgcn_readlane(i, l), __builtin_amdgcn_readlane(j, l), lane, sum, size);
        if (lane == l) { v.sum = sum; v.size = size; }
    }
}

// ---- tiles in whole numbers.  Both sums go through v_mfma_i32_32x32x32_i8, which is exact: a weight's q - z and |q - z| are bytes (z up to 127; other columns are formed
// in binary64), and 128 activations of a token become whole numbers X = trunc(a 2^(29 - E)), E the exponent of the largest of them, in four digits of base 256 from -128 to
// 127, of X for the output and of |X| for the bound.  A digit is a row of its own (4 t + digit), so that a lane finds a token's digits in neighbouring registers.  Sums of 128
// products of a digit stay below 2^21; the digits are put together and scaled in binary64.
// What truncation leaves off: at most one unit of every X, so with dmax >= |q - z| the sum of |X||q - z| lies within [exact - 128 dmax, exact] units: the bound takes the upper end, and
//     err = sum over the blocks of |s| 2^(E - 29) 128 dmax
// is how far it may lie above, and how far y may be off.  An output with err <= 14u size has exact <= size <= exact (1 + 14u), so tau, rounded up, is within 16.1u < 1e-6 of its formula, and
// y, rounded once, within 15u of the sum of magnitudes; others (blocks whose largest activation is hundreds of times the usual one, while its weight is 0) are formed in binary64.
// For ordinary tokens err is about 0.5u size (largest activation of 128 about 3.5 times the mean, dmax twice the mean of |q - z|).
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));
typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));
constexpr int kInt4Block = 128;                              // columns of a block
constexpr int kInt4Codes = kInt4Block / 2 + 16;              // bytes of a column's codes of a block in LDS
constexpr unsigned kInt4Row = kInt4Block + 16;               // bytes of a digit's row in LDS (16 more: the eight rows that are read at a time lie in different banks)

// KW groups of NW wavefronts: a wavefront has 32 columns and the tokens of RT row tiles of OWN each; the groups share out the reduction, their sums are added in LDS.
template <int OWN_, int RT_, int NW_, int KW_>
struct Int4Shape {
    static constexpr int OWN = OWN_, RT = RT_, NW = NW_, KW = KW_, THREADS = NW * KW * kWave, Q = (OWN + 1) / 2;      // Q: tokens of a lane in a row tile
    static constexpr int TOKENS = OWN * RT, COLUMNS = 32 * NW;
    static constexpr int BLOCKS = NW * kWave / (TOKENS * kInt4Block / 8);        // of a chunk: a lane brings eight activations
    static constexpr int SET = TOKENS * 4 * kInt4Row, BLOCK = 2 * SET, DIGITS = BLOCKS * (BLOCK + 4 * TOKENS);     // bytes: digits of X, and of |X|; exponents behind them
    static constexpr int CODES = 32 * kInt4Codes;            // of a wavefront
    static constexpr int SUMS = (KW - 1) * NW * RT * Q * kWave * (int)sizeof(Int4Sums);
    static constexpr int STAGES = KW * (DIGITS + NW * CODES), LDS = (STAGES > SUMS ? STAGES : SUMS) + 16 * ((TOKENS + 3) / 4);
    static_assert(BLOCKS >= 1 && NW * kWave % (TOKENS * kInt4Block / 8) == 0 && DIGITS % 16 == 0, "whole blocks a chunk");
    static_assert(LDS <= 80 * 1024, "two workgroups a compute unit");
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
// Sixteen codes less their zero point and the magnitudes of that, as bytes: of a word of eight the even ones, then the odd ones.  biased: 128 - z in every byte.  Additions, shifts and bitwise
// operations of two operands take a SIMD half the time of the others here (2.6 cycles, 4.6).
__device__ __forceinline__ void int4_codes(unsigned w0, unsigned w1, unsigned biased, intx4& d, intx4& m) {
    const unsigned half[4] = {w0 & 0x0f0f0f0fu, w0 >> 4 & 0x0f0f0f0fu, w1 & 0x0f0f0f0fu, w1 >> 4 & 0x0f0f0f0fu};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned v = (half[i] + biased) ^ 0x80808080u, sign = v & 0x80808080u, n = sign >> 7;       // (no byte carries into the next)
        d[i] = (int)v;
        m[i] = (int)((v ^ (sign | (sign - n))) + n);
    }
}
// Order between the lanes of a wavefront: LDS takes its accesses in order, so only the compiler has to keep it.
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// byte j of four words
__device__ __forceinline__ void int4_transpose(const unsigned (&w)[4], unsigned (&digit)[4]) {
    const unsigned a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);      // bytes 0 and 1 of two words
    const unsigned c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), e = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);      // ... 2 and 3
    digit[0] = __builtin_amdgcn_perm(b, a, 0x05040100u); digit[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    digit[2] = __builtin_amdgcn_perm(e, c, 0x05040100u); digit[3] = __builtin_amdgcn_perm(e, c, 0x07060302u);
}

// What a lane requests of a chunk: eight activations, of each block two times 16 bytes of weights, and for its column the scales and zero points of the chunk's folds, every other one
// (the lower half of the wavefront has the even ones).
template <class SH, int FOLDS>
struct Int4Chunk {
    static constexpr int PAIRS = (SH::BLOCKS * FOLDS + 1) / 2;
    floatx4_any a[2];
    uintx4 raw[SH::BLOCKS][2];
    float s[PAIRS];
    unsigned char z[PAIRS];
};

// Weights are read in lines: four lanes a row's 64 bytes of a block, and handed to the lanes of their columns through LDS (a load whose lanes have a row each takes the address
// unit a cycle or two a lane: with 16 bytes a lane four times as long).
// FOLDS: how often a block's sums are scaled (1: groups of whole blocks, 2: of halves, 4: of 32 columns)
template <class SH, int FOLDS>
__global__ __launch_bounds__(SH::THREADS, SH::RT == 1 ? 4 : 2) void int4_tiles(Int4Args p, Int4Grid grid) {
    extern __shared__ __align__(16) char lds[];
    constexpr int Q = SH::Q, RT = SH::RT, NW = SH::NW, KW = SH::KW, OWN = SH::OWN, BLOCKS = SH::BLOCKS, STEPS = 4 / FOLDS;
    using Chunk = Int4Chunk<SH, FOLDS>;
    unsigned* marks = reinterpret_cast<unsigned*>(lds + SH::LDS - 16 * ((SH::TOKENS + 3) / 4));       // of a token: 1 not a number, 2 an activation that became 0
    // workgroups of one tile of columns on one die (workgroup modulo 8), whose cache then holds their weights
    const unsigned rest = blockIdx.x >> 3, up = grid.token_blocks == 1 ? rest : rest / grid.token_blocks, tile = up * 8 + (blockIdx.x & 7);
    if (tile >= grid.tiles) return;
    const int lane = threadIdx.x & (kWave - 1), half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), kg = wave / NW, nw = wave % NW;
    const long n0 = (long)tile * SH::COLUMNS + 32 * nw, m0 = (long)(rest - up * grid.token_blocks) * SH::TOKENS;
    if (threadIdx.x < SH::TOKENS) marks[threadIdx.x] = 0;
    // whole blocks are shared out among the groups of all parts
    const int blocks = grid.blocks, first = min((int)(blockIdx.y * KW + kg) * grid.share, blocks), last = min(first + grid.share, blocks);
    const int trips = (min(grid.share, blocks) + BLOCKS - 1) / BLOCKS, all = trips + (grid.tail == (int)blockIdx.y);
    auto group_of = [&](int k) __attribute__((always_inline)) { return min((int)((unsigned long)(k >> 5) * p.per_group >> 32), p.groups - 1); };
    const unsigned char* row0 = p.W + min(n0 + lane / 4, p.N - 1) * p.ldw + lane % 4 * 16;
    const unsigned char* row1 = p.W + min(n0 + 16 + lane / 4, p.N - 1) * p.ldw + lane % 4 * 16;
    const long n = min(n0 + col, p.N - 1);
    const float* scales = p.scale + n * p.groups;
    const bool zeroed = p.zero != nullptr;
    const unsigned char* zeros = zeroed ? p.zero + n * p.groups : row0;      // (any bytes, where there are none: a load all the same)
    const int zero_step = zeroed ? 1 : 0;
    // this lane's eight activations of a chunk
    const int at = (nw * kWave + lane) / 16, own_block = at % BLOCKS, own_token = at / BLOCKS, unit = lane % 16;
    const float* a_row = p.A + min(m0 + own_token, p.M - 1) * p.lda + unit * 8;

    Int4Sums total[RT][Q];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int q = 0; q < Q; ++q) total[r][q] = Int4Sums{0.0, 0.0, 0.0};
    char* digits = lds + kg * SH::DIGITS;
    const int* exps = reinterpret_cast<const int*>(digits + BLOCKS * SH::BLOCK);
    char* codes = lds + KW * SH::DIGITS + wave * SH::CODES;
    const unsigned fragment = (((lane >> 2) & (OWN - 1) & 7) * 4 + (lane & 3)) * kInt4Row + half * 16;     // of this lane's row of a row tile

    auto meet = [&]() __attribute__((always_inline)) { if constexpr (NW > 1) __syncthreads(); else wave_order(); };
    auto factors = [&](Chunk& w, int block) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < Chunk::PAIRS; ++i) {
            const int g0 = group_of(block * kInt4Block + 2 * i * (kInt4Block / FOLDS)), g1 = group_of(block * kInt4Block + (2 * i + 1) * (kInt4Block / FOLDS)), g = half ? g1 : g0;
            w.s[i] = scales[g];
            w.z[i] = zeros[g * zero_step];
        }
    };
    // (nothing here branches, so that what is on its way is known where it is waited for: blocks behind the last one repeat it)
    auto request = [&](Chunk& w, int block) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            const int b = min(block + i, blocks - 1) * (kInt4Block / 2);
            __builtin_memcpy(&w.raw[i][0], row0 + b, 16);
            __builtin_memcpy(&w.raw[i][1], row1 + b, 16);
        }
        const float* a = a_row + min(block + own_block, blocks - 1) * kInt4Block;
        w.a[0] = *reinterpret_cast<const floatx4_any*>(a); w.a[1] = *reinterpret_cast<const floatx4_any*>(a + 4);
        factors(w, block);
    };
    // activations to digits in LDS, with the exponent of their block: a row of 16 lanes has a block of a token
    auto write = [&](const floatx4_any (&a)[2]) __attribute__((always_inline)) {
        unsigned most = 0, least = ~0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned size = __float_as_uint(a[i >> 2][i & 3]) & 0x7fffffffu;
            most = max(most, size); least = min(least, size - 1u);
        }
        most = wave_all<0, 4>(most, [](unsigned x, unsigned y) { return max(x, y); });
        const int E = max((int)(most >> 23), 1) - 127;
        const int unit_bits = E - 29 + 127;                  // of 2^(E - 29) as binary32 (where that is subnormal, any subnormal activation counts as gone)
        const bool gone = least != ~0u && (unit_bits > 0 ? least + 1u < (unsigned)unit_bits << 23 : least < 0x7fffffu);
        if (most >= 0x7f800000u || gone) atomicOr(&marks[own_token], most >= 0x7f800000u ? 1u : 2u);
        char* to = digits + own_block * SH::BLOCK + own_token * 4 * kInt4Row + unit * 8;
        unsigned x[2][2][4];                                 // [set][even or odd]
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = a[i >> 2][i & 3];
            const unsigned m = (unsigned)__builtin_amdgcn_ldexpf(fabsf(v), 29 - E), sign = (unsigned)(__float_as_int(v) >> 31);
            x[0][i & 1][i >> 1] = (((m ^ sign) - sign) + 0x00808080u) ^ 0x00808080u;
            x[1][i & 1][i >> 1] = (m + 0x00808080u) ^ 0x00808080u;
        }
#pragma unroll
        for (int set = 0; set < 2; ++set) {
            unsigned even[4], odd[4];
            int4_transpose(x[set][0], even);
            int4_transpose(x[set][1], odd);
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<uint2*>(to + set * SH::SET + j * kInt4Row) = make_uint2(even[j], odd[j]);
        }
        if (unit == 0) reinterpret_cast<int*>(digits + BLOCKS * SH::BLOCK)[own_block * SH::TOKENS + own_token] = E - 29;
    };
    // block i of the chunk, whose folds have these scales and biases
    auto multiply = [&](const uintx4 (&raw)[2], int i, const float* scale, const unsigned* biased) __attribute__((always_inline)) {
        wave_order();
        char* to = codes + lane / 4 * kInt4Codes + lane % 4 * 16;
        *reinterpret_cast<uintx4*>(to) = raw[0];
        *reinterpret_cast<uintx4*>(to + 16 * kInt4Codes) = raw[1];
        wave_order();
        const char* from = codes + col * kInt4Codes + half * 8;
        uint2 word[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) word[s] = *reinterpret_cast<const uint2*>(from + 16 * s);
        intx16 y[RT], t[RT];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int f = s / STEPS;
            intx4 d, m;
            int4_codes(word[s].x, word[s].y, biased[f], d, m);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const char* row = digits + i * SH::BLOCK + fragment + r * OWN * 4 * kInt4Row + s * 32;
                const intx16 none = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
                y[r] = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const intx4*>(row), d, s % STEPS ? y[r] : none, 0, 0, 0);
                t[r] = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const intx4*>(row + SH::SET), m, s % STEPS ? t[r] : none, 0, 0, 0);
            }
            if (s % STEPS == STEPS - 1) {
                const int z = 128 - (int)(biased[f] & 255u), left = max(z, 15 - z) * (32 * STEPS);      // units that truncation may have left off
                const double wide = (double)scale[f];
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int q = 0; q < Q; ++q) {
                        Int4Sums& v = total[r][q];
                        const double by = ldexp(wide, exps[i * SH::TOKENS + r * OWN + (OWN > 1 ? 2 * q + half : 0)]), size = fabs(by);
                        const int e = 4 * q;
                        v.sum = fma(by, fma((double)(y[r][e + 2] + (y[r][e + 3] << 8)), 65536.0, (double)(y[r][e] + (y[r][e + 1] << 8))), v.sum);
                        v.size = fma(size, fma((double)(t[r][e + 2] + (t[r][e + 3] << 8)), 65536.0, (double)(t[r][e] + (t[r][e + 1] << 8) + left)), v.size);
                        v.err = fma(size, (double)left, v.err);
                    }
            }
        }
    };
    Chunk now, next;
    if (trips > 0) request(now, first);
    __syncthreads();                                         // (the marks)
    for (int trip = 0; trip < all; ++trip) {
        const bool odd = trip == trips;                      // the last block, which is not whole, goes to the last group
        const int block = odd ? blocks : first + trip * BLOCKS, limit = !odd ? last : kg == KW - 1 ? blocks + 1 : 0;
        if (odd) {                                           // (columns that do not exist have activations of 0)
            const int columns = own_block == 0 ? (int)(p.K % kInt4Block) - unit * 8 : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) now.a[i >> 2][i & 3] = i < columns ? a_row[(long)blocks * kInt4Block + i] : 0.f;
            const int from = blocks * (kInt4Block / 2) + lane % 4 * 16, bytes = (int)((p.K + 1) / 2);
            now.raw[0][0] = int4_bytes(row0 - lane % 4 * 16, from, bytes);
            now.raw[0][1] = int4_bytes(row1 - lane % 4 * 16, from, bytes);
            factors(now, block);
        } else if (trip + 1 < trips) {
            request(next, block + BLOCKS);
        }
        meet();
        write(now.a);
        meet();
        // (a column whose zero point does not fit the bytes gets NaN: its outputs are then formed in binary64)
        float scale[2 * Chunk::PAIRS];
        unsigned biased[2 * Chunk::PAIRS];
#pragma unroll
        for (int i = 0; i < Chunk::PAIRS; ++i) {
            const unsigned z = zeroed ? now.z[i] : 8u, b = (128u - min(z, 127u)) * 0x01010101u, s = z > 127u ? 0x7fc00000u : __float_as_uint(now.s[i]);
            const auto bs = __builtin_amdgcn_permlane32_swap(b, b, false, false), ss = __builtin_amdgcn_permlane32_swap(s, s, false, false);
            biased[2 * i] = bs[0]; biased[2 * i + 1] = bs[1];
            scale[2 * i] = __uint_as_float(ss[0]); scale[2 * i + 1] = __uint_as_float(ss[1]);
        }
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
            if (block + i < limit) multiply(now.raw[i], i, scale + i * FOLDS, biased + i * FOLDS);
        now = next;
    }
    __syncthreads();                                         // (the stages' memory is that of the sums)
    Int4Sums* others = reinterpret_cast<Int4Sums*>(lds);     // [group - 1][wavefront][output of a lane][lane]
    if (kg > 0) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int q = 0; q < Q; ++q) others[(((kg - 1) * NW + nw) * RT * Q + r * Q + q) * kWave + lane] = total[r][q];
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            Int4Sums v = total[r][q];
#pragma unroll
            for (int k = 1; k < KW; ++k) {
                const Int4Sums& o = others[(((k - 1) * NW + nw) * RT * Q + r * Q + q) * kWave + lane];
                v.sum += o.sum; v.size += o.size; v.err += o.err;
            }
            const int t = r * OWN + 2 * q + half;
            const unsigned mark = marks[min(t, SH::TOKENS - 1)];
            if (mark & 1u) v.size = NAN;
            if (mark & 2u) v.size += 0x1p-900;               // (not the 0 that int4_open takes for exact)
            const bool own = (OWN > 1 || half == 0) && m0 + t < p.M && n0 + col < p.N;
            if (p.part) {
                if (own) p.part[((long)blockIdx.y * p.M + m0 + t) * p.N + n0 + col] = v;
                continue;
            }
            int4_settle(p, own, (int)m0 + t, (int)n0 + col, v);
            if (own) {
                const long to = (m0 + t) * p.ldy + n0 + col;
                float out, tau;
                int4_values(p, n0 + col, v, out, tau);
                if (p.y) p.y[to] = out;
                if (p.tau) p.tau[to] = tau;
            }
        }
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
    p.M = M; p.N = N; p.K = K; p.lda = lda; p.ldw = ldw; p.ldy = ldy;
    p.group = group < K || K == 0 ? group : K + (K & 1);     // (one group: its end at an even column)
    p.groups = (int)((K + p.group - 1) / p.group);
    p.per_group = p.groups > 1 ? (1UL << 32) / (unsigned long)(p.group / 32) + 1 : 0;
    p.gamma = g * (1.0 + ((double)K + 64.0) * 0x1p-52) * kGuard;
    p.uflow = (md->flags & TAO_FLAG_UNDERFLOW_TERMS) ? 0x1p-149 * kGuard / p.gamma : 0.0;
    p.terms = (double)steps;
    return TAO_OK;
}
// What a launch does: tiles of up to `tokens` tokens in `parts` parts of the reduction, or the kernel of any size (tokens 0).
struct Int4Plan { int tokens, parts; };
static Int4Plan int4_plan(long M, long N, long K, bool terms) {
    // (short reductions: a wavefront's lanes are hardly used, and what truncation leaves off would show next to the few roundings that the bound holds)
    if (K <= 32 || K > (1L << 20) || terms) return {0, 1};
    const int tokens = M <= 2 ? 2 : M <= 4 ? 4 : M <= 8 ? 8 : 16;
    // parts until there is a workgroup for each of the chip's 256 compute units (written out: the workspace's size is asked for where there may be no device), of four blocks a group
    // at least, as their sums take a launch more
    const long columns = tokens <= 4 ? 32 : tokens == 8 ? 64 : 128, groups = tokens <= 4 ? 8 : tokens == 8 ? 4 : 2;
    const long workgroups = (N + columns - 1) / columns * ((M + tokens - 1) / tokens), most = K / kInt4Block / (4 * groups);
    const long parts = std::max(1L, std::min(256 / std::max(workgroups, 1L), most));
    return {tokens, (int)parts};
}
template <class SH, int FOLDS>
static int int4_launch_tiles(const Int4Args& p, int parts, hipStream_t st) {
    const long tiles = (p.N + SH::COLUMNS - 1) / SH::COLUMNS, token_blocks = (p.M + SH::TOKENS - 1) / SH::TOKENS;
    const __int128 grid = (__int128)((tiles + 7) / 8 * 8) * token_blocks;
    if (grid >= (1L << 31)) return TAO_ERR_SHAPE;
    static OncePerDevice once;
    const hipError_t e = once.run([] { return hipFuncSetAttribute(reinterpret_cast<const void*>(int4_tiles<SH, FOLDS>), hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS); });
    if (e != hipSuccess) { g_last_hip_error = (int)e; return TAO_ERR_LAUNCH; }
    const long blocks = p.K / kInt4Block, sharers = (long)SH::KW * parts;
    const Int4Grid g{(unsigned)tiles, (unsigned)token_blocks, (int)blocks, (int)((blocks + sharers - 1) / sharers), p.K % kInt4Block ? parts - 1 : -1};
    hipLaunchKernelGGL((int4_tiles<SH, FOLDS>), dim3((unsigned)grid, (unsigned)parts), dim3(SH::THREADS), SH::LDS, st, p, g);
    return launch_status();
}
template <class SH>
static int int4_launch_tiles(const Int4Args& p, int parts, hipStream_t st) {
    if (p.groups <= 1 || p.group % kInt4Block == 0) return int4_launch_tiles<SH, 1>(p, parts, st);
    if (p.group % (kInt4Block / 2) == 0) return int4_launch_tiles<SH, 2>(p, parts, st);
    return int4_launch_tiles<SH, 4>(p, parts, st);
}
// The sums (p.part) or, with one part, the outputs.
static int int4_launch(const Int4Args& p, const Int4Plan& plan, hipStream_t st) {
    switch (plan.tokens) {
        case 2:  return int4_launch_tiles<Int4Shape<2, 1, 1, 8>>(p, plan.parts, st);
        case 4:  return int4_launch_tiles<Int4Shape<4, 1, 1, 8>>(p, plan.parts, st);
        case 8:  return int4_launch_tiles<Int4Shape<8, 1, 2, 4>>(p, plan.parts, st);
        case 16: return int4_launch_tiles<Int4Shape<8, 2, 4, 2>>(p, plan.parts, st);
    }
    const long blocks = (p.M * p.N + 3) / 4;
    hipLaunchKernelGGL(int4_any, dim3((unsigned)(blocks < 256L * 256 ? blocks : 256L * 256)), dim3(256), 0, st, p);
    return launch_status();
}
static size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }
static bool int4_sizes_ok(long M, long N, long K) {
    const long most = 1L << 31;
    return M >= 0 && N >= 0 && K >= 0 && M < most && N < most && K < most && (__int128)M * N < ((__int128)1 << 36);
}
static size_t part_bytes(long M, long N, int parts) { return padded((size_t)parts * (size_t)(M * N) * sizeof(Int4Sums)); }

}  // namespace tao

extern "C" {

size_t tao_linear_int4_workspace_bytes(long M, long N, long K) {
    using namespace tao;
    if (!int4_sizes_ok(M, N, K)) return 0;
    const Int4Plan plan = int4_plan(M, N, K, false);
    return plan.parts > 1 ? part_bytes(M, N, plan.parts) : 0;
}

size_t tao_bound_check_linear_int4_workspace_bytes(long M, long N, long K) {
    using namespace tao;
    if (!int4_sizes_ok(M, N, K)) return 0;
    return padded(check_workspace_bytes()) + part_bytes(M, N, int4_plan(M, N, K, false).parts);
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
    const Int4Plan plan = int4_plan(M, N, K, p.uflow != 0.0);
    hipStream_t st = (hipStream_t)stream;
    p.y = y; p.tau = tau;
    if (plan.parts == 1) return int4_launch(p, plan, st);
    p.part = (Int4Sums*)ws;
    const int rc2 = int4_launch(p, plan, st);
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
    const Int4Plan plan = int4_plan(M, N, K, p.uflow != 0.0);
    p.part = (Int4Sums*)((char*)ws + padded(check_workspace_bytes()));
    if (n > 0) {
        const int rc2 = int4_launch(p, plan, st);
        if (rc2 != TAO_OK) return rc2;
    }
    const long want = (n + kCheckThreads - 1) / kCheckThreads;
    const int nblocks = (int)(want < 1 || n <= kAloneElements ? 1 : want > kMaxCheckBlocks ? kMaxCheckBlocks : want);
    hipLaunchKernelGGL(int4_join_check, dim3(nblocks), dim3(kCheckThreads), 0, st, p, plan.parts, Int4CheckArgs{y_ref, claimed, alpha, eps_rel, pass_out(w, nblocks, n, out)});
    launch_finish(w, nblocks, n, out, st);
    return launch_status();
}

}  // extern "C"
