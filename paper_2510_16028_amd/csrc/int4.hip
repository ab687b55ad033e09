// tao_bound_linear_int4, tao_bound_check_linear_int4: binary32 activations times weights in 4 bits with a scale, and possibly a zero point, for each group,
//     w_jk = (q_jk - z_jg) s_jg,    y_ij = sum_k a_ik w_jk + b_j,    tau_ij = Gamma(K') (sum_k |a_ik||w_jk| + |b_j|),
// a reduction of K products (Sec. 3.1) whose terms are rounded once more for the scale: K' = K + 1, or K + 2 with a bias.
#include "tao_check.hpp"
#include "tao_device.hpp"
#include "tao_host.hpp"

namespace tao {

constexpr double kInt4Inflation = 1.0 / (1.0 - 11.2 * 0x1p-24);      // of the tiles' sums of magnitudes

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
__device__ __forceinline__ void int4_output(const Int4Args& p, long i, long j, int lane) {
    double sum, size, extra;
    int4_wave_sums(p, i, j, lane, sum, size, extra);
    if (lane == 0) {
        const double b = p.bias ? (double)p.bias[j] : 0.0;
        if (p.y) p.y[i * p.ldy + j] = (float)(sum + b);
        if (p.tau) p.tau[i * p.ldy + j] = int4_bound(p, size, b, p.uflow * (p.terms + extra));
    }
}
__global__ __launch_bounds__(256) void int4_any(Int4Args p) {
    const long n = p.M * p.N;
    for (long at = (long)blockIdx.x * 4 + threadIdx.x / kWave; at < n; at += (long)gridDim.x * 4)
        int4_output(p, at % p.M, at / p.M, threadIdx.x & (kWave - 1));
}

// ---- tiles: a wavefront takes 32 columns and a share of the reduction, a workgroup of KW wavefronts 32 columns and up to 2 Q RT tokens; the wavefronts' sums are added in LDS.
// Both sums go through v_mfma_f32_32x32x16_bf16, whose products are exact here: a weight's whole number q - z has 8 bits, and an activation is cut into three pieces of 8 bits
// each by masking, a = h + m + l, all of its sign, with |m| < 2^-7 |a| and |l| < 2^-15 |a|.  The pieces of a token are rows of their own (4 t + piece, the fourth unused), so
// that a lane finds a token's three sums in neighbouring registers.  y multiplies the pieces by q - z, the bound their magnitudes by |q - z|.
// Errors (the instruction's model is that of linear_split.hip; u = 2^-24): an instruction from a zero accumulator gives a sum S of terms of one sign within [S(1 - 10u), S(1 + 2u)].  The
// sums of h of two instructions are added in binary32 (1u) and then, times the scale, in binary64; those of m and l, which are 2^-7 of it, over four instructions in binary32:
// [1 - 11.2u, 1 + 3.2u] in all, so the bound is multiplied by 1 / (1 - 11.2u): exact <= tau <= exact (1 + 14.4u + 2u for the last rounding) < exact (1 + 1e-6).
// y lets four instructions (64 columns) run in one accumulator: 7u of every step's magnitudes and 2u of all so far for 8 steps, 23.3u with the pieces' 2^-7, 1u for h + (m + l)
// and 1u for the last rounding: 25.3u of the sum of magnitudes.
// Operands for which that does not hold -- magnitudes below 2^-100, whose pieces are next to BF16's subnormal range, from 2^110 on, whose sums may overflow, and what is no number -- mark their
// token, whose outputs are then formed in binary64 (int4_wave_sums).
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
constexpr int kInt4Block = 64, kInt4Ahead = 4;               // columns of a block; blocks of weights that are requested together (128 bytes of a row)
constexpr unsigned kInt4Row = 2 * kInt4Block + 16;           // bytes of a piece's row in LDS (16 more: the eight rows that are read at a time lie in different banks)

template <int Q_, int RT_, int KW_>
struct Int4Shape {
    static constexpr int Q = Q_, RT = RT_, KW = KW_, THREADS = KW * kWave;
    static constexpr int OWN = 2 * Q, TOKENS = OWN * RT;     // tokens of a row tile, of a workgroup
    static constexpr int STAGE = TOKENS * 3 * kInt4Row, SUMS = TOKENS * 32 * 16;      // bytes of a wavefront
    static constexpr int LDS = KW * (2 * STAGE > SUMS ? 2 * STAGE : SUMS) + 4 * TOKENS;
};

// 16 bytes of a row of weights from byte `at` on; bytes from `bytes` on are not touched and read as 0 (the activations there are 0).
__device__ __forceinline__ uintx4 int4_bytes(const unsigned char* __restrict__ row, int at, int bytes) {
    uintx4 r = {0, 0, 0, 0};
    if (at + 16 <= bytes) {
        __builtin_memcpy(&r, row + at, 16);
    } else {
#pragma unroll 1
        for (int i = min(bytes - at, 16) - 1; i >= 0; --i) {
            r = uintx4{r[0] << 8, r[1] << 8 | r[0] >> 24, r[2] << 8 | r[1] >> 24, r[3] << 8 | r[2] >> 24};
            r[0] |= row[at + i];
        }
    }
    return r;
}
// Eight codes less their zero point as BF16: codes i and i + 4 of a word become two binary16 numbers 1024 + q, whose difference to 1024 + z binary32 holds exactly, and so does BF16.
// offset: -(1024 + z).
__device__ __forceinline__ uintx4 int4_codes(unsigned word, float offset, float one) {
    uintx4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const halfx2 h = __builtin_bit_cast(halfx2, (word >> 4 * i & 0x000f000fu) | 0x64006400u);
        const float lo = fmaf((float)h[0], one, offset), hi = fmaf((float)h[1], one, offset);
        r[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    }
    return r;
}
__device__ __forceinline__ bf16x8 as_bf16(uintx4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ bf16x8 as_magnitudes(uintx4 v) { return __builtin_bit_cast(bf16x8, v & 0x7fff7fffu); }

// Activations on their way to LDS: of a block, a lane has 2 Q columns of a token of every row tile (codes i and i + 4 of a word are neighbours, so columns i and i + 4 are).
template <class SH>
struct Int4Stage {
    static constexpr int Q = SH::Q, PER = 32 / Q;            // lanes of a token
    const float* row[SH::RT];
    int at, limit;                                           // first column in a block, K
    unsigned place;                                          // of its first piece in LDS
    float v[SH::RT][2 * Q];
    unsigned most, least;                                    // of the bits of all magnitudes (less one: zeros do not count)
    __device__ __forceinline__ Int4Stage(const Int4Args& p, long m0, int lane) {
        const int t = lane / PER, rest = lane % PER;
#pragma unroll
        for (int r = 0; r < SH::RT; ++r) row[r] = p.A + min(m0 + r * SH::OWN + t, p.M - 1) * p.lda;
        at = rest / (4 / Q) * 8 + rest % (4 / Q) * Q;
        limit = (int)p.K;
        place = t * 3 * kInt4Row + rest / (4 / Q) * 16 + rest % (4 / Q) * Q * 4;
        most = 0; least = ~0u;
    }
    __device__ __forceinline__ void request(int block) {
        const int k = block * kInt4Block + at;
        typedef float run __attribute__((ext_vector_type(Q == 1 ? 2 : Q), aligned(4)));
#pragma unroll
        for (int r = 0; r < SH::RT; ++r) {
            if (k + 4 + Q <= limit) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if constexpr (Q == 1) {
                        v[r][half] = row[r][k + 4 * half];
                    } else {
                        const run x = *reinterpret_cast<const run*>(row[r] + k + 4 * half);
#pragma unroll
                        for (int i = 0; i < Q; ++i) v[r][half * Q + i] = x[i];
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2 * Q; ++i) {
                    const int c = k + (i / Q) * 4 + i % Q;
                    v[r][i] = c < limit ? row[r][c] : 0.f;
                }
            }
        }
    }
    __device__ __forceinline__ void write(char* buffer) {
#pragma unroll
        for (int r = 0; r < SH::RT; ++r) {
            unsigned piece[3][Q];
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                unsigned top[2][3];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float x = v[r][half * Q + i];
                    const unsigned bits = __float_as_uint(x), size = bits & 0x7fffffffu;
                    most = max(most, size); least = min(least, size - 1u);
                    const float m = x - __uint_as_float(bits & 0xffff0000u);
                    const float l = m - __uint_as_float(__float_as_uint(m) & 0xffff0000u);
                    top[half][0] = bits; top[half][1] = __float_as_uint(m); top[half][2] = __float_as_uint(l);
                }
#pragma unroll
                for (int j = 0; j < 3; ++j) piece[j][i] = __builtin_amdgcn_perm(top[1][j], top[0][j], 0x07060302u);
            }
            char* to = buffer + r * SH::OWN * 3 * kInt4Row + place;
#pragma unroll
            for (int j = 0; j < 3; ++j) {
                if constexpr (Q == 4)      *reinterpret_cast<uintx4*>(to + j * kInt4Row) = uintx4{piece[j][0], piece[j][1], piece[j][2], piece[j][3]};
                else if constexpr (Q == 2) *reinterpret_cast<uint2*>(to + j * kInt4Row) = make_uint2(piece[j][0], piece[j][1]);
                else                       *reinterpret_cast<unsigned*>(to + j * kInt4Row) = piece[j][0];
            }
        }
    }
    __device__ __forceinline__ bool marked() const { return most >= (127u + 110u) << 23 || least < ((127u - 100u) << 23) - 1u; }
};
// Order between the lanes of a wavefront: LDS takes its accesses in order, so only the compiler has to keep it.
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Blocks of weights with the scale and zero point of each half (32 columns) of a block.
struct Int4Weights { uintx4 raw[kInt4Ahead]; float s[kInt4Ahead][2], z[kInt4Ahead][2]; };

// FINE: groups may end in the middle of a block.
template <class SH, bool FINE>
__global__ __launch_bounds__(SH::THREADS) void int4_tiles(Int4Args p, unsigned tiles, unsigned token_blocks) {
    extern __shared__ __align__(16) char lds[];
    constexpr int Q = SH::Q, RT = SH::RT, KW = SH::KW;
    unsigned* marks = reinterpret_cast<unsigned*>(lds + SH::LDS - 4 * SH::TOKENS);
    // workgroups of one tile of columns on one die (workgroup modulo 8), whose cache then holds their weights
    const unsigned rest = blockIdx.x >> 3, tile = rest / token_blocks * 8 + (blockIdx.x & 7);
    if (tile >= tiles) return;
    const long n0 = (long)tile * 32, m0 = (long)(rest % token_blocks) * SH::TOKENS;
    const int lane = threadIdx.x & (kWave - 1), half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (threadIdx.x < SH::TOKENS) marks[threadIdx.x] = 0;
    __syncthreads();
    const int blocks = (int)((p.K + kInt4Block - 1) / kInt4Block), share = (blocks + KW - 1) / KW;
    const int first = min(wave * share, blocks), last = min(first + share, blocks);
    const long n = min(n0 + col, p.N - 1);
    const unsigned char* row = p.W + n * p.ldw;
    const float* scales = p.scale + n * p.groups;
    const unsigned char* zeros = p.zero + (p.zero ? n * p.groups : 0);
    const int bytes = (int)((p.K + 1) / 2), group = (int)min(p.group, 0x7fffffffL);
    auto request = [&](Int4Weights& w, int block) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kInt4Ahead; ++i) {
            if (block + i >= last) break;
            w.raw[i] = int4_bytes(row, (block + i) * 32 + half * 16, bytes);
#pragma unroll
            for (int j = 0; j < (FINE ? 2 : 1); ++j) {
                const int g = min(((block + i) * kInt4Block + 32 * j) / group, p.groups - 1);
                w.s[i][j] = scales[g];
                w.z[i][j] = p.zero ? (float)zeros[g] : 8.f;
            }
        }
    };
    double ty[RT][Q], tt[RT][Q];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int q = 0; q < Q; ++q) ty[r][q] = tt[r][q] = 0.0;
    char* mine = lds + wave * 2 * SH::STAGE;
    // this lane's row of a row tile: piece of a token (the fourth one's sums are not used)
    const char* fragment = mine + (((lane >> 2) & (SH::OWN - 1) & 7) * 3 + min(lane & 3, 2)) * kInt4Row + half * 16;
    float one = 1.f;
    asm volatile("" : "+v"(one));                            // (a product with 1 that the compiler knows becomes a conversion and an addition)
    Int4Stage<SH> stage(p, m0, lane);
    Int4Weights now, next;
    if (first < last) {
        request(now, first);
        stage.request(first);
        stage.write(mine + (first & 1) * SH::STAGE);
        stage.request(first + 1);
    }
    for (int block = first; block < last; block += kInt4Ahead) {
        request(next, block + kInt4Ahead);
#pragma unroll
        for (int i = 0; i < kInt4Ahead; ++i) {
            const int b = block + i;
            if (b >= last) break;
            wave_order();
            if (b + 1 < last) {                              // (the one after the last belongs to another wavefront, or lies behind the row's end)
                stage.write(mine + ((b + 1) & 1) * SH::STAGE);
                stage.request(b + 2);
            }
            wave_order();
            // a lane has 32 columns of a row's 64: words of 8 columns 0-3 in the lower half of the wavefront, 4-7 in the upper; an instruction takes words 2 s and 2 s + 1
            unsigned word[4];
            {
                const auto a = __builtin_amdgcn_permlane32_swap(now.raw[i][0], now.raw[i][1], false, false), c = __builtin_amdgcn_permlane32_swap(now.raw[i][2], now.raw[i][3], false, false);
                word[0] = a[0]; word[2] = a[1]; word[1] = c[0]; word[3] = c[1];
            }
            floatx16 y[RT];
            float hp[RT][Q], ml[RT][Q];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int part = FINE ? s >> 1 : 0;
                const bool fresh = s == 0 || (FINE && s == 2), ends = s == 3 || (FINE && s == 1);
                const uintx4 codes = int4_codes(word[s], -1024.f - now.z[i][part], one);
                const double scale = (double)now.s[i][part], size = fabs(scale);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const uintx4 a = *reinterpret_cast<const uintx4*>(fragment + (b & 1) * SH::STAGE + r * SH::OWN * 3 * kInt4Row + s * 32);
                    const floatx16 none = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    y[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(a), as_bf16(codes), fresh ? none : y[r], 0, 0, 0);
                    const floatx16 t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_magnitudes(a), as_magnitudes(codes), none, 0, 0, 0);
#pragma unroll
                    for (int q = 0; q < Q; ++q) {
                        const float small = t[4 * q + 1] + t[4 * q + 2];
                        ml[r][q] = fresh ? small : ml[r][q] + small;
                        if (s & 1) tt[r][q] = fma(size, (double)(hp[r][q] + t[4 * q]), tt[r][q]);
                        else       hp[r][q] = t[4 * q];
                        if (ends) {
                            tt[r][q] = fma(size, (double)ml[r][q], tt[r][q]);
                            ty[r][q] = fma(scale, (double)(y[r][4 * q] + (y[r][4 * q + 1] + y[r][4 * q + 2])), ty[r][q]);
                        }
                    }
                }
            }
        }
        now = next;
    }
    if (first < last && stage.marked()) {
#pragma unroll
        for (int r = 0; r < RT; ++r) marks[r * SH::OWN + lane / Int4Stage<SH>::PER] = 1;      // (all tiles' tokens of the lane: what they lose is time)
    }
    __syncthreads();                                         // (the stages' memory is that of the sums)
    double2* sums = reinterpret_cast<double2*>(lds);         // [wavefront][token][column]
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int q = 0; q < Q; ++q) sums[(wave * SH::TOKENS + r * SH::OWN + 2 * q + half) * 32 + col] = make_double2(ty[r][q], tt[r][q]);
    __syncthreads();
    const int tokens = (int)min(p.M - m0, (long)SH::TOKENS), cols = (int)min(p.N - n0, 32L);
    for (int i = threadIdx.x; i < tokens * 32; i += SH::THREADS) {
        const int t = i >> 5, c = i & 31;
        if (c >= cols || marks[t]) continue;
        double sum = 0.0, size = 0.0;
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            const double2 v = sums[w * SH::TOKENS * 32 + i];
            sum += v.x; size += v.y;
        }
        const double b = p.bias ? (double)p.bias[n0 + c] : 0.0;
        const long at = (m0 + t) * p.ldy + n0 + c;
        if (p.y) p.y[at] = (float)(sum + b);
        if (p.tau) p.tau[at] = int4_bound(p, size * kInt4Inflation, b, 0.0);
    }
    for (int t = 0; t < tokens; ++t) {
        if (!marks[t]) continue;
        for (int c = wave; c < cols; c += KW) int4_output(p, m0 + t, n0 + c, lane);
    }
}
template <class SH>
static int int4_launch_tiles(const Int4Args& p, hipStream_t st) {
    const long tiles = (p.N + 31) / 32, token_blocks = (p.M + SH::TOKENS - 1) / SH::TOKENS;
    const __int128 grid = (__int128)((tiles + 7) / 8 * 8) * token_blocks;
    if (grid >= (1L << 31)) return TAO_ERR_SHAPE;
    static OncePerDevice once;
    const hipError_t e = once.run([] {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(int4_tiles<SH, false>), hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS);
        return e != hipSuccess ? e : hipFuncSetAttribute(reinterpret_cast<const void*>(int4_tiles<SH, true>), hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS);
    });
    if (e != hipSuccess) { g_last_hip_error = (int)e; return TAO_ERR_LAUNCH; }
    const dim3 blocks((unsigned)grid), threads(SH::THREADS);
    if (p.group % kInt4Block && p.groups > 1) hipLaunchKernelGGL((int4_tiles<SH, true>), blocks, threads, SH::LDS, st, p, (unsigned)tiles, (unsigned)token_blocks);
    else                                      hipLaunchKernelGGL((int4_tiles<SH, false>), blocks, threads, SH::LDS, st, p, (unsigned)tiles, (unsigned)token_blocks);
    return launch_status();
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
    // (short reductions: the wavefront's lanes are hardly used, but the tiles' errors would show next to the few roundings that the bound holds)
    if (p.K > 32 && p.K < (1L << 30) && p.uflow == 0.0) {
        if (p.M <= 2)  return int4_launch_tiles<Int4Shape<1, 1, 8>>(p, st);
        if (p.M <= 4)  return int4_launch_tiles<Int4Shape<2, 1, 8>>(p, st);
        if (p.M <= 8)  return int4_launch_tiles<Int4Shape<4, 1, 8>>(p, st);
        if (p.M <= 16) return int4_launch_tiles<Int4Shape<4, 2, 8>>(p, st);
        return int4_launch_tiles<Int4Shape<4, 4, 4>>(p, st);
    }
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
