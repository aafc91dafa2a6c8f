// FP8 linear layer with a scale for every block of 128 along the contraction:
//   Y_ik = sum_b s_x[b][i] s_w[k / 128][b] P_b,   P_b = sum over the 128 channels of block b of cx_ij cw_kj
//
// One v_mfma_f32_16x16x128_f8f6f4 is one block of the contraction: it starts from zero and leaves P_b, which is added to the
// binary32 total times its scale by the vector unit (the product of the two scales once a token tile, one fused multiply-add an
// output and block).  The weights are the instruction's first operand, so that a lane holds outputs of one token only (lane l:
// token l & 15 of the tile, channels 4 (l >> 4) + register) and needs one scale a tile.
//
// A block's 8 waves are WM x WN wave tiles of 16 MT tokens x 16 NT channels times WK shares of the contraction; a step is WK
// blocks of 128, wave share wk multiplies the wk-th.  Steps go through a ring of S slots in LDS ([wk][TM + TN rows][128
// bytes], then [wk][TM] scales), filled by requests that bypass the registers: step k + S is requested while step k is multiplied.
// Within a slot 16-byte chunk c of row R sits at chunk c ^ ((R >> 1) & 7), so that the 16 rows a fragment read covers fall on
// distinct banks.  A lane reads chunks g and g + 4 of its row (g = lane >> 4): which K positions those take inside the
// instruction does not matter, as long as both operands are read the same way.
// The instruction sums 8 neighbouring products (bytes 8 n .. 8 n + 7 of a lane) with 13 bits below the exponent of the largest,
// dropping the rest, and only those sums with 24 bits; the older 16 x 16 x 32 form does the same at half the rate.  On normally
// distributed operands that is a relative 1e-5 of the result, a twentieth of binary16's rounding.
// LDS row 16 ni + i of a wave's weight rows holds its channel 4 NT (i >> 2) + 4 ni + (i & 3): a lane's 4 NT outputs of a token
// are neighbours in Y.
#include <algorithm>
#include <type_traits>

#include "cq_gemm_common.h"

namespace cq {
namespace {

__device__ __forceinline__ v4f product128(const v8i& w, const v8i& x) {
    // formats 0 = e4m3; scale operands 0 select the unscaled instruction
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, v4f{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}

// a wave-uniform pointer, in scalar registers whatever the compiler made of it
__device__ __forceinline__ const void* in_scalar(const void* p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);      // (the builtin's int would extend its sign)
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
    return reinterpret_cast<const void*>((uint64_t)hi << 32 | lo);
}
// request_1k and request_words from a scalar base and a lane's 32-bit offset
__device__ __forceinline__ void request_1k_from(const void* base, uint32_t off, const int8_t* dst) {
    const uint32_t lds_off = (uint32_t)(uintptr_t)((lptr_t)dst);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 sc0" : : "v"(off), "s"(in_scalar(base)), "s"(lds_off) : "m0");
}
__device__ __forceinline__ void request_words_from(const void* base, uint32_t off, const int8_t* dst) {
    const uint32_t lds_off = (uint32_t)(uintptr_t)((lptr_t)dst);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(off), "s"(in_scalar(base)), "s"(lds_off) : "m0");
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
    if (!BF16) return pack_half2(a, b);
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// 4 or 8 neighbouring outputs of a token as one store, wherever they lie (2-byte aligned: what a row of an odd pitch is); those past O
// are left out.  (509 x 2816 x 4090, rows of 8180 bytes: 2 bytes at a time 19.1 us, so 13.5; 2000 x 2816 x
// 4091 42 and 30)
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
template <typename P>
__device__ __forceinline__ void store_row(uint16_t* __restrict__ row, int col, int O, const P& p) {
    constexpr int kCount = sizeof(P) / 2;
    if (col + kCount <= O) {
        __builtin_memcpy(row + col, &p, sizeof(P));
    } else {
#pragma unroll
        for (int e = 0; e < kCount; ++e)
            if (col + e < O) row[col + e] = (uint16_t)(e & 1 ? p[e / 2] >> 16 : p[e / 2]);
    }
}
template <bool BF16>
__device__ __forceinline__ v2u pack4(const v4f& y) { return v2u{pack_pair<BF16>(y[0], y[1]), pack_pair<BF16>(y[2], y[3])}; }
template <bool BF16>
__device__ __forceinline__ v4u pack8(const v4f& a, const v4f& b) {
    return v4u{pack_pair<BF16>(a[0], a[1]), pack_pair<BF16>(a[2], a[3]), pack_pair<BF16>(b[0], b[1]), pack_pair<BF16>(b[2], b[3])};
}

template <int MT, int NT, int WM, int WN, int WK, int S>
struct Fp8Tile {
    static_assert(WM * WN * WK == kSplitWaves, "8 waves");
    static constexpr int TM = 16 * MT * WM, TN = 16 * NT * WN, kRows = TM + TN;
    static constexpr int kData = kRows * 128 * WK, kSlot = kData + TM * WK * 4;
    static constexpr int N = kData / 1024 / kSplitWaves;                     // 1 KiB requests per wave and step
    static constexpr int kScaleLanes = TM * WK / kSplitWaves;                // scales each wave requests per step
    static constexpr int kParts = WM * WN * MT * NT * (WK - 1) * 64 * 16;    // partial sums that change hands
    static constexpr int kLds = std::max(S * kSlot, kParts);
    static_assert(N * 1024 * kSplitWaves == kData && kScaleLanes * kSplitWaves == TM * WK && kScaleLanes <= 64, "shared evenly");
    static_assert(TN <= 128 ? 128 % TN == 0 : TN % 128 == 0, "a wave's channels lie in one block of 128");
    static_assert(kLds <= 160 * 1024, "LDS of a CU");
};

// ONCE: the weights' requests are non-temporal.
template <int MT, int NT, int WM, int WN, int WK, int S, bool ONCE, bool BF16>
__global__ void __launch_bounds__(64 * kSplitWaves)
gemm_fp8_kernel(const int8_t* __restrict__ qx, const float* __restrict__ x_scale, const int8_t* __restrict__ qw,
                const float* __restrict__ w_scale, int T, int nk, int O, uint16_t* __restrict__ Y, int64_t ldy, int tiles_m,
                int tiles_n) {
    using P = Fp8Tile<MT, NT, WM, WN, WK, S>;
    constexpr int TM = P::TM, kRows = P::kRows, kSlot = P::kSlot, N = P::N;
    extern __shared__ __align__(16) int8_t lds[];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int w = wave % (WM * WN), wk = wave / (WM * WN);
    const int wm = w / WN, wn = w % WN;
    const int fr = lane & 15, grp = lane >> 4;
    const int steps = (nk + WK - 1) / WK;
    const int64_t K = (int64_t)nk * 128;

    int tile_m, tile_n;
    if (!tile_of_block(blockIdx.x, tiles_m, tiles_n, tile_m, tile_n)) return;
    const int m0 = tile_m * TM, n0 = tile_n * P::TN;

    // Request n of this wave fills the 8 LDS rows (wave N + n) 8 + (lane >> 3) of a slot; the lane's 16 bytes are physical chunk
    // lane & 7 of its row.  Rows past T or O take the last one's bytes: they feed outputs that are not stored.
    const int8_t* src[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int R = (8 * (wave * N + n) + (lane >> 3)) % kRows;
        const int8_t* row;
        if (R < TM) {
            row = qx + (int64_t)min(m0 + R, T - 1) * K;
        } else {
            const int b = R - TM, in = b % (16 * NT), i = in & 15;
            row = qw + (int64_t)min(n0 + b - in + 4 * NT * (i >> 2) + 4 * (in >> 4) + (i & 3), O - 1) * K;
        }
        src[n] = row + ((lane & 7) ^ ((R >> 1) & 7)) * 16;
    }
    const int e = wave * P::kScaleLanes + min(lane, P::kScaleLanes - 1);     // this lane's scale: slab, token
    const int e_slab = e / TM, e_tok = min(m0 + e % TM, T - 1);
    auto request = [&](int kt, int slot) {
        int8_t* dst = lds + slot * kSlot;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int slab = 8 * (wave * N + n) / kRows;                      // (scalar)
            const int8_t* from = src[n] + (int64_t)min(kt * WK + slab, nk - 1) * 128;
            if (ONCE && 8 * (wave * N + n) % kRows >= TM) request_1k<true>(from, dst + (wave * N + n) * 1024);     // (scalar)
            else request_1k(from, dst + (wave * N + n) * 1024);
        }
        if (lane < P::kScaleLanes)
            request_words(x_scale + (int64_t)min(kt * WK + e_slab, nk - 1) * T + e_tok, dst + P::kData + wave * P::kScaleLanes * 4);
    };

    v4f acc[MT][NT];
#pragma unroll
    for (int mi = 0; mi < MT; ++mi)
#pragma unroll
        for (int ni = 0; ni < NT; ++ni) acc[mi][ni] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    // weight scales of 64 steps at a time, one a lane
    const float* ws_row = n0 + wn * 16 * NT < O ? w_scale + (int64_t)((n0 + wn * 16 * NT) / 128) * nk : w_scale;
    float ws_all = ws_row[min(lane * WK + wk, nk - 1)];

#pragma unroll
    for (int s = 0; s < S; ++s)
        if (s < steps) request(s, s);
    if (steps >= S) __builtin_amdgcn_s_waitcnt(waitcnt_imm((S - 1) * (N + 1), 0));       // step 0 has landed
    else __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
    step_barrier();

    const int a_off = wk * kRows * 128 + (wm * 16 * MT + fr) * 128, b_off = wk * kRows * 128 + (TM + wn * 16 * NT + fr) * 128;
    const int sw0 = (grp ^ ((fr >> 1) & 7)) * 16, sw1 = sw0 ^ 64;
    const int s_off = P::kData + (wk * TM + wm * 16 * MT + fr) * 4;
    struct Frags {
        v8i a[MT], b[NT];
        float s[MT];
    };
    auto read = [&](Frags& f, int slot) {
        const int8_t* base = lds + slot * kSlot;
        auto two = [](const int8_t* lo, const int8_t* hi) {
            return __builtin_shufflevector(*reinterpret_cast<const v4i*>(lo), *reinterpret_cast<const v4i*>(hi), 0, 1, 2, 3, 4, 5, 6, 7);
        };
#pragma unroll
        for (int ni = 0; ni < NT; ++ni) f.b[ni] = two(base + b_off + sw0 + ni * 2048, base + b_off + sw1 + ni * 2048);
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) {
            f.a[mi] = two(base + a_off + sw0 + mi * 2048, base + a_off + sw1 + mi * 2048);
            f.s[mi] = *reinterpret_cast<const float*>(base + s_off + mi * 64);
        }
    };
    // Step kt: its fragments are in registers; behind the barrier its slot is free (step kt + S is requested into it) and step
    // kt + 1 has landed (its fragments are read while kt is multiplied).  A request holds its wave for some 100 clocks: waves 0-3,
    // one of every SIMD, make theirs before they multiply, waves 4-7 after.
    Frags f0, f1;
    read(f0, 0);
    int slot = 0;
    auto step = [&](auto full_c, int kt, Frags& cur, Frags& nxt) {       // full_c: steps kt + 1 and kt + S exist
        constexpr bool kFull = decltype(full_c)::value;
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(kFull ? (S - 2) * (N + 1) : 0, 0));
        step_barrier();
        if (kFull && wave < 4) request(kt + S, slot);
        const int next_slot = slot + 1 == S ? 0 : slot + 1;
        if (kFull || kt + 1 < steps) read(nxt, next_slot);
        __builtin_amdgcn_sched_barrier(0);
        const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ws_all), kt & 63));
        if (WK == 1 || kt * WK + wk < nk) {                   // the last step may have fewer than WK blocks (wave-uniform)
            v4f p[2][NT];
#pragma unroll
            for (int mi = 0; mi <= MT; ++mi) {
#pragma unroll
                for (int ni = 0; ni < NT; ++ni) {
                    if (mi < MT) p[mi & 1][ni] = product128(cur.b[ni], cur.a[mi]);
                    if (mi > 0) {
                        const float s = cur.s[mi - 1] * ws;
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[mi - 1][ni][r] = __builtin_fmaf(p[(mi - 1) & 1][ni][r], s, acc[mi - 1][ni][r]);
                    }
                }
            }
        }
        if (kFull && wave >= 4) {
            __builtin_amdgcn_sched_barrier(0);
            request(kt + S, slot);
        }
        if ((kt & 63) == 63) ws_all = ws_row[min((kt + 1 + lane) * WK + wk, nk - 1)];
        slot = next_slot;
    };
    int kt = 0;
    for (; kt + S + 1 < steps; kt += 2) {                     // two steps a turn: the fragments' registers change places
        step(std::true_type(), kt, f0, f1);
        step(std::true_type(), kt + 1, f1, f0);
    }
    for (; kt < steps; kt += 2) {
        if (kt + S < steps) step(std::true_type(), kt, f0, f1);
        else step(std::false_type(), kt, f0, f1);
        if (kt + 1 < steps) step(std::false_type(), kt + 1, f1, f0);
    }

    // Outputs are stored G neighbouring weight tiles at a time, 8 or 16 bytes a lane.
    constexpr int G = NT % 2 == 0 && MT * NT / 2 >= WK ? 2 : 1, kGroups = MT * NT / G;
    const int col0 = n0 + wn * 16 * NT + 4 * NT * grp, row0 = m0 + wm * 16 * MT + fr;
    auto store = [&](int first, const v4f* y) {               // tiles first .. first + G - 1 of mi NT + ni
        const int row = row0 + 16 * (first / NT), col = col0 + 4 * (first % NT);
        if (row >= T) return;
        uint16_t* at = Y + (int64_t)row * ldy;
        if (G == 2) store_row(at, col, O, pack8<BF16>(y[0], y[G - 1]));
        else store_row(at, col, O, pack4<BF16>(y[0]));
    };
    if (WK == 1) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            v4f y[G];
#pragma unroll
            for (int i = 0; i < G; ++i) y[i] = acc[(g * G + i) / NT][(g * G + i) % NT];
            store(g * G, y);
        }
        return;
    }
    // The WK shares of a wave tile meet in LDS: group g of its tiles is summed and stored by share g % WK, the others hand theirs over;
    // always summed in the order of the shares.
    __syncthreads();                                         // the last step's reads are done
    v4f* parts = reinterpret_cast<v4f*>(lds) + w * (MT * NT * (WK - 1) * 64) + lane;
#pragma unroll
    for (int u = 0; u < MT * NT; ++u) {
        const int owner = u / G % WK;
        if (wk != owner) parts[(u * (WK - 1) + (wk < owner ? wk : wk - 1)) * 64] = acc[u / NT][u % NT];
    }
    __syncthreads();
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int owner = g % WK;
        if (wk != owner) continue;
        v4f sum[G];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int u = g * G + i;
            sum[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int p = 0; p < WK; ++p) {
                const v4f v = p == owner ? acc[u / NT][u % NT] : parts[(u * (WK - 1) + (p < owner ? p : p - 1)) * 64];
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[i][r] += v[r];
            }
        }
        store(g * G, sum);
    }
}

// Large layers: 256 x 256 tiles, one share of the contraction, held to a schedule by hand.
//
// A wave's 128 tokens x 64 channels are multiplied token tile by token tile.  While the four products of tile mi run, those of tile
// mi - 1 are added to their totals (the vector unit needs half the matrix unit's time for that) and the fragment of tile mi + 3 is
// read.  A step's one barrier stands before its last three tiles: by then every wave has read all it needs of this step, so its place
// in LDS is free, and what the next step needs has to have landed.  The last tile's products cover, weight tile by weight tile as
// they are done with, the reads of the next step's weight fragments.
//
// What costs time beside the matrix unit are the requests: a wave stands still while its own wait for the CU's vector memory unit
// (some 100 clocks each), and a SIMD's other wave has its matrix unit meanwhile.  So the two waves of a SIMD request at different
// times: waves 0-3 the weights (two steps ahead) and the token scales behind the barrier, waves 4-7 the activations, half a step's at
// tile 0 and half at tile 3.  LDS holds
//   weights: two slots of 32 KiB;
//   activations: five slots of 16 KiB, half a step each: half h of step k is in slot (2 k + h) mod 5.  The second half of step k + 1
//     and the first of step k + 2 are requested in step k, into the place that step k - 1 left and the one that was free;
//   token scales: three slots of 1 KiB.
// Measured (4096 x 8192 x 28672): all requests of a step at once behind the barrier, two whole slots 988 us; two a product, by all
// waves, 857; this form 790 to 810, with whole-line stores 777 to 806 over cards, 2.39 to 2.47 PFLOP/s.  With operands of zeros it took 690: the difference is the
// clock under power, 1.8 GHz.  Without the requests of all steps but the first it would take 666 (zeros: 568), without the additions 723.
// Matrix instructions alone from registers reach 4.5 PFLOP/s; what remains are the instructions a wave has to issue between
// them (reads of fragments, additions, requests).
//
// NT = 2 is half a tile, 256 x 128 (128 x 32 a wave, half the weight requests): outputs of less than a round of the CUs, and the last
// round of others, are covered by such where that leaves fewer CUs idle (launch_fp8_ring).
constexpr int kRingTile = 256, kHalf = 128 * 128;
constexpr int kRingB = 5 * kHalf, kRingScales = kRingB + 2 * 2 * kHalf, kRingLds = kRingScales + 3 * 1024;
static_assert(kRingLds <= 160 * 1024, "LDS of a CU");

template <int NT, bool BF16>
__device__ __forceinline__ void ring_tile(const int8_t* __restrict__ qx, const float* __restrict__ x_scale,
                                          const int8_t* __restrict__ qw, const float* __restrict__ w_scale, int T, int nk, int O,
                                          uint16_t* __restrict__ Y, int64_t ldy, int8_t* lds, int m0, int n0) {
    constexpr int MT = 8, WN = 4, WTN = 16 * NT, kMidAt = 0, kLateAt = 3, kEarlyAt = 1, kAhead = 3;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int fr = lane & 15, grp = lane >> 4;
    const int64_t K = (int64_t)nk * 128;

    // ---- requests.  A lane's offsets from the tile's first row of the operand: below 2^32 (256 rows of fewer than 2^24 bytes).
    const int8_t* const a_base = qx + (int64_t)m0 * K;
    const int8_t* const b_base = qw + (int64_t)n0 * K;
    // waves 0-3 ("front") request the weights and the scales, waves 4-7 the activations: eight pieces a step each
    const bool front = wave < 4;
    uint32_t from[8];                                         // waves 4-7: four pieces of either half
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int w = wave & 3, R = (front ? WTN * w + 8 * i : 128 * (i >> 2) + 32 * w + 8 * (i & 3)) + (lane >> 3);
        const int in = R % WTN, j = in & 15;
        const uint32_t row = (uint32_t)(front ? min(R - in + 4 * NT * (j >> 2) + 4 * (in >> 4) + (j & 3), O - 1 - n0) : min(R, T - 1 - m0));
        from[i] = row * (uint32_t)K + ((lane & 7) ^ ((R >> 1) & 7)) * 16;
    }
    // the scales of 64 tokens a front wave: word 8 f + mi of a 128-token half is the one of its token 16 mi + f (one past the last
    // token reads the last one's)
    const uint32_t s_from = (uint32_t)min(128 * ((wave & 3) >> 1) + 16 * (lane & 7) + 8 * (wave & 1) + (lane >> 3), T - 1 - m0) * 4;
    auto request_a = [&](int half, int k, int slot) {         // half of the activations of step k
#pragma unroll
        for (int i = 0; i < 4; ++i)
            request_1k_from(a_base + (int64_t)k * 128, from[4 * half + i], lds + slot * kHalf + (4 * (wave & 3) + i) * 1024);
    };
    auto request_b = [&](int k) {
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i)
            request_1k_from(b_base + (int64_t)k * 128, from[i], lds + kRingB + (k & 1) * 2 * kHalf + (2 * NT * (wave & 3) + i) * 1024);
    };
    auto request_scales = [&](int k, int slot) {
        request_words_from(x_scale + m0 + (int64_t)min(k, nk - 1) * T, s_from, lds + kRingScales + slot * 1024 + (wave & 3) * 256);
    };

    v4f acc[MT][NT];
#pragma unroll
    for (int mi = 0; mi < MT; ++mi)
#pragma unroll
        for (int ni = 0; ni < NT; ++ni) acc[mi][ni] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    const float* ws_row = n0 + wn * WTN < O ? w_scale + (int64_t)((n0 + wn * WTN) / 128) * nk : w_scale;
    float ws_all = ws_row[min(lane, nk - 1)];                 // the weight block's scales of 64 steps

    // step 0, then what earlier steps would have requested
    if (front) {
        request_scales(0, 0);
        request_b(0);
        if (nk > 1) {
            request_scales(1, 1);
            request_scales(2, 2);
            request_b(1);
            __builtin_amdgcn_s_waitcnt(waitcnt_imm(2 * NT + 2, 0));
        } else {
            __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
        }
    } else {
        request_a(0, 0, 0);
        request_a(1, 0, 1);
        if (nk > 1) {
            request_a(0, 1, 2);
            __builtin_amdgcn_s_waitcnt(waitcnt_imm(4, 0));
        } else {
            __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
        }
    }
    step_barrier();

    const int sw = (grp ^ ((fr >> 1) & 7)) * 16;
    const int8_t* a_lo = lds + wm * kHalf + fr * 128 + sw;
    const int8_t* a_hi = lds + wm * kHalf + fr * 128 + (sw ^ 64);
    const int8_t* b_lo = lds + kRingB + (wn * WTN + fr) * 128 + sw;
    const int8_t* b_hi = lds + kRingB + (wn * WTN + fr) * 128 + (sw ^ 64);
    const int8_t* s_at = lds + kRingScales + wm * 512 + fr * 32;
    int b_turn = 2 * kHalf;                                   // to the other slot
    int slot_a = wm;                                          // the wave's half of the step whose fragments are read: 2 k + wm mod 5
    int slot_next = 3;                                        // 2 k + 3 mod 5: the second half of step k + 1
    int slot_s = 0;
    auto two = [](const int8_t* lo, const int8_t* hi) {
        return __builtin_shufflevector(*reinterpret_cast<const v4i*>(lo), *reinterpret_cast<const v4i*>(hi), 0, 1, 2, 3, 4, 5, 6, 7);
    };

    v8i b[NT], a[4];
    v4f p[4], s[2], s_next[2];                                // (scales of the step's eight token tiles, and the next step's)
#pragma unroll
    for (int ni = 0; ni < NT; ++ni) b[ni] = two(b_lo + ni * 2048, b_hi + ni * 2048);
#pragma unroll
    for (int mi = 0; mi < kAhead; ++mi) a[mi] = two(a_lo + mi * 2048, a_hi + mi * 2048);
#pragma unroll
    for (int i = 0; i < 2; ++i) s_next[i] = s[i] = *reinterpret_cast<const v4f*>(s_at + i * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ws_all), 0));
    float s_old = 0.0f;                                       // scale of the products of the tile before

    // next_c: there is a step after k; more_c: and one after that
    auto step = [&](auto next_c, auto more_c, int k) {
        constexpr bool kNext = decltype(next_c)::value, kMore = decltype(more_c)::value;
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) {
            if (mi == MT - kAhead) {
                // all of step k + 1 has landed (waves 4-7: all but the four latest requests, for step k + 2), and nobody reads step k
                // any more
                if (kMore && !front) __builtin_amdgcn_s_waitcnt(waitcnt_imm(4, 0));
                else __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
                step_barrier();
                const int turn_a = slot_a >= 3 ? -3 * kHalf : 2 * kHalf;
                slot_a += slot_a >= 3 ? -3 : 2;
                a_lo += turn_a;
                a_hi += turn_a;
                b_lo += b_turn;
                b_hi += b_turn;
                b_turn = -b_turn;
                const int turn_s = slot_s == 2 ? -2048 : 1024;
                s_at += turn_s;
#pragma unroll
                for (int i = 0; i < 2; ++i) s_next[i] = *reinterpret_cast<const v4f*>(s_at + i * 16);
            }
            // the fragment after the next one (past the last step: what is there, not used)
            constexpr int kTile = 16 * 128;
            const int ahead = (mi + kAhead) % MT;
            a[(mi + kAhead) & 3] = two(a_lo + ahead * kTile, a_hi + ahead * kTile);
            const float s_now = s[mi >> 2][mi & 3] * ws;
#pragma unroll
            for (int ni = 0; ni < NT; ++ni) {
                // the products of the tile before go to their totals, this tile's take their registers
                const int mo = mi == 0 ? MT - 1 : mi - 1;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[mo][ni][r] = __builtin_fmaf(p[ni][r], s_old, acc[mo][ni][r]);
                asm volatile("" : "+v"(acc[mo][ni]));         // (the compiler would move all additions to the step's end)
                p[ni] = product128(b[ni], a[mi & 3]);
                if (mi == MT - 1) b[ni] = two(b_lo + ni * 2048, b_hi + ni * 2048);
                __builtin_amdgcn_sched_barrier(0);
                if (mi == kMidAt && ni == 0 && kNext && !front) request_a(1, k + 1, slot_next);
                if (mi == kLateAt && ni == 0 && kMore && !front) request_a(0, k + 2, slot_next == 4 ? 0 : slot_next + 1);
                if (mi == MT - kAhead && ni == kEarlyAt && kMore && front) {
                    request_scales(k + 3, slot_s);            // step k's place
                    request_b(k + 2);
                }
                if ((mi == kMidAt && ni == 0) || (mi == kLateAt && ni == 0) || (mi == MT - kAhead && ni == kEarlyAt)) __builtin_amdgcn_sched_barrier(0);
            }
            s_old = s_now;
        }
        slot_s = slot_s == 2 ? 0 : slot_s + 1;
        slot_next += slot_next >= 3 ? -3 : 2;
#pragma unroll
        for (int i = 0; i < 2; ++i) s[i] = s_next[i];
        const int nx = (k + 1) & 63;
        if (nx == 0) ws_all = ws_row[min(k + 1 + lane, nk - 1)];
        ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ws_all), nx));
    };
    for (int k = 0; k < nk - 2; ++k) step(std::true_type(), std::true_type(), k);
    if (nk > 1) step(std::true_type(), std::false_type(), nk - 2);
    step(std::false_type(), std::false_type(), nk - 1);       // (waits for every request: none outlives the block)
#pragma unroll
    for (int ni = 0; ni < NT; ++ni)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[MT - 1][ni][r] = __builtin_fmaf(p[ni][r], s_old, acc[MT - 1][ni][r]);

    const int col0 = n0 + wn * WTN + 4 * NT * grp, row0 = m0 + wm * 128 + fr;
    // Outputs leave 16 bytes a lane, and whole lines of 128 bytes an instruction: of its 32 bytes of a token (NT = 4) a lane keeps one
    // half and trades the other for the same half of its neighbour's token.  (4096 x 4096 x 4096: 8 bytes a lane 63.4 us, 16 of its own
    // token 59.0, 57.4 so)
    const int odd = lane & 1;
#pragma unroll
    for (int mi = 0; mi < MT; ++mi) {
        const int row = row0 + 16 * mi;
        if (NT == 2) {
            if (row < T) store_row(Y + (int64_t)row * ldy, col0, O, pack8<BF16>(acc[mi][0], acc[mi][1]));
        } else {
            const v4u lo = pack8<BF16>(acc[mi][0], acc[mi][1]), hi = pack8<BF16>(acc[mi][NT - 2], acc[mi][NT - 1]);
            v4u even, next;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(odd ? lo[i] : hi[i]), 0xB1, 0xF, 0xF, true);     // lane ^ 1
                even[i] = odd ? other : lo[i];
                next[i] = odd ? hi[i] : other;
            }
            uint16_t* y = Y + (int64_t)(row - odd) * ldy;
            if (row - odd < T) store_row(y, col0 + 8 * odd, O, even);
            if (row - odd + 1 < T) store_row(y + ldy, col0 + 8 * odd, O, next);
        }
    }
}

// The first n_whole tiles of the walk are whole (a multiple of 8, or all there are), the others two halves each, on blocks behind theirs.
template <bool BF16>
__global__ void __launch_bounds__(64 * kSplitWaves, 2)
gemm_fp8_ring_kernel(const int8_t* __restrict__ qx, const float* __restrict__ x_scale, const int8_t* __restrict__ qw,
                     const float* __restrict__ w_scale, int T, int nk, int O, uint16_t* __restrict__ Y, int64_t ldy, int tiles_m,
                     int tiles_n, int n_whole) {
    extern __shared__ __align__(16) int8_t lds[];
    const int whole_blocks = (n_whole + kXcds - 1) / kXcds * kXcds;
    const bool whole = (int)blockIdx.x < whole_blocks;
    const int block = whole ? blockIdx.x : blockIdx.x - whole_blocks, n = whole ? n_whole : 2 * (tiles_m * tiles_n - n_whole);
    const int per_xcd = (n + kXcds - 1) / kXcds, at = (block % kXcds) * per_xcd + block / kXcds;    // (see tile_of_block)
    if (at >= n || block / kXcds >= per_xcd) return;
    int tile_m, tile_n;
    tile_of_index(whole ? at : n_whole + at / 2, tiles_m, tiles_n, tile_m, tile_n);
    const int m0 = tile_m * kRingTile, n0 = tile_n * kRingTile + (whole ? 0 : at % 2 * (kRingTile / 2));
    if (n0 >= O) return;                                      // the right half of a last tile may have no channel
    if (whole) ring_tile<4, BF16>(qx, x_scale, qw, w_scale, T, nk, O, Y, ldy, lds, m0, n0);
    else ring_tile<2, BF16>(qx, x_scale, qw, w_scale, T, nk, O, Y, ldy, lds, m0, n0);
}

hipError_t go_ring(const int8_t* qx, const float* xs, const int8_t* qw, const float* ws, int T, int nk, int O, uint16_t* Y, bool bf16,
                   int64_t ldy, int n_cu, hipStream_t stream) {
    const int tiles_m = (T + kRingTile - 1) / kRingTile, tiles_n = (O + kRingTile - 1) / kRingTile;
    const int64_t total = (int64_t)tiles_m * tiles_n, rest = total % n_cu;
    const int64_t n_whole = 2 * rest <= n_cu ? total - rest : total, halves = 2 * (total - n_whole);
    auto padded = [](int64_t n) { return (n + kXcds - 1) / kXcds * kXcds; };
    const int64_t blocks = padded(n_whole) + padded(halves);
    if (!grid_fits(blocks, 64 * kSplitWaves)) return hipErrorInvalidValue;
    static std::atomic<uint64_t> done[2];
    auto launch = [&](auto k, std::atomic<uint64_t>& d) {
        if (hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(k), kRingLds, d); e != hipSuccess) return e;
        k<<<(unsigned)blocks, 64 * kSplitWaves, kRingLds, stream>>>(qx, xs, qw, ws, T, nk, O, Y, ldy, tiles_m, tiles_n, (int)n_whole);
        return hipGetLastError();
    };
    return bf16 ? launch(gemm_fp8_ring_kernel<true>, done[1]) : launch(gemm_fp8_ring_kernel<false>, done[0]);
}

template <int MT, int NT, int WM, int WN, int WK, int S, bool ONCE = false>
hipError_t go(const int8_t* qx, const float* xs, const int8_t* qw, const float* ws, int T, int nk, int O, uint16_t* Y, bool bf16,
              int64_t ldy, hipStream_t stream) {
    using P = Fp8Tile<MT, NT, WM, WN, WK, S>;
    const int tiles_m = (T + P::TM - 1) / P::TM, tiles_n = (O + P::TN - 1) / P::TN;
    const int64_t total = (int64_t)tiles_m * tiles_n, blocks = (total + kXcds - 1) / kXcds * kXcds;
    if (!grid_fits(blocks, 64 * kSplitWaves)) return hipErrorInvalidValue;
    static std::atomic<uint64_t> done[2];
    const void* kernel = bf16 ? reinterpret_cast<const void*>(gemm_fp8_kernel<MT, NT, WM, WN, WK, S, ONCE, true>)
                              : reinterpret_cast<const void*>(gemm_fp8_kernel<MT, NT, WM, WN, WK, S, ONCE, false>);
    if (hipError_t e = allow_dynamic_lds(kernel, P::kLds, done[bf16]); e != hipSuccess) return e;
    auto launch = [&](auto k) {
        k<<<(unsigned)blocks, 64 * kSplitWaves, P::kLds, stream>>>(qx, xs, qw, ws, T, nk, O, Y, ldy, tiles_m, tiles_n);
    };
    if (bf16) launch(gemm_fp8_kernel<MT, NT, WM, WN, WK, S, ONCE, true>);
    else launch(gemm_fp8_kernel<MT, NT, WM, WN, WK, S, ONCE, false>);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_fp8_linear(const void* qx, const float* x_scale, const void* qw, const float* w_scale, int T, int I, int O,
                             uint16_t* Y, bool bf16, int64_t ldy, hipStream_t stream) {
    const int8_t* x = static_cast<const int8_t*>(qx);
    const int8_t* w = static_cast<const int8_t*>(qw);
    const int nk = I / 128;
    int n_cu = 0, dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n_cu < 1)
        n_cu = 256;
    // The tile: the form whose estimated time is least.  A round of `at_once` tiles takes `ns` for each 128 channels of the
    // contraction, in whole steps, and `fixed` is a launch's and a tile's beginning and end (us, all measured on one card; us for 512 x
    // 4096 x 4096 by form: 16 x 32 49, 32 x 32 46, 32 x 64 32, 64 x 64 23.5, 64 x 128 17.4, 128 x 128 25.0, 256 x 128 32.8; for 4096 x 4096 x
    // 4096: 128 x 128 117, 256 x 256 66).  Small tiles have more CUs at work, large ones take in less for each product.
    struct Form {
        int tm, tn, wk, per_cu, ns, fixed;
    };
    constexpr Form kForms[] = {{16, 16, 8, 1, 117, 2300}, {16, 32, 4, 2, 180, 2300}, {32, 32, 4, 1, 172, 2200},
                               {32, 64, 4, 1, 235, 2200}, {64, 64, 2, 1, 350, 2300}, {64, 128, 2, 1, 580, 2300}, {128, 128, 1, 1, 850, 2300}};
    auto tiles = [&](int tm, int tn) { return (int64_t)((T + tm - 1) / tm) * ((O + tn - 1) / tn); };
    const int64_t whole = tiles(256, 256), rest = whole % n_cu;
    // a round of whole tiles 1950, of half tiles 1330
    int64_t best = (whole / n_cu * 1950 + (rest == 0 ? 0 : 2 * rest <= n_cu ? 1330 : 1950)) * nk + 4000;
    int form = -1;
    for (int i = 0; i < (int)(sizeof(kForms) / sizeof(kForms[0])); ++i) {
        const Form& f = kForms[i];
        const int64_t at_once = (int64_t)n_cu * f.per_cu, rounds = (tiles(f.tm, f.tn) + at_once - 1) / at_once;
        const int64_t time = rounds * ((nk + f.wk - 1) / f.wk * f.wk) * f.ns + f.fixed;
        if (time < best) {
            best = time;
            form = i;
        }
    }
    // Weights that one row of tiles reads once and that no cache keeps are requested non-temporally: 16 x 8192 x 28672 45.4 -> 41.5 us,
    // 128 x 8192 x 28672 66.3 -> 61.9, 1 x 65536 x 4096 56 -> 50, 8 x 53248 x 4096 49 -> 46; three weights of 64 MiB in turn, which the
    // memory-side cache holds, 12.6 -> 15.1.
    const bool once = form >= 0 && T <= kForms[form].tm && (int64_t)I * O > (int64_t)128 << 20;
    switch (form) {
        case 0: return once ? go<1, 1, 1, 1, 8, 4, true>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream) : go<1, 1, 1, 1, 8, 4>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream);
        case 1: return once ? go<1, 1, 1, 2, 4, 3, true>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream) : go<1, 1, 1, 2, 4, 3>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream);
        case 2: return once ? go<2, 1, 1, 2, 4, 4, true>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream) : go<2, 1, 1, 2, 4, 4>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream);
        case 3: return once ? go<2, 2, 1, 2, 4, 3, true>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream) : go<2, 2, 1, 2, 4, 3>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream);
        case 4: return once ? go<2, 2, 2, 2, 2, 4, true>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream) : go<2, 2, 2, 2, 2, 4>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream);
        case 5: return once ? go<2, 4, 2, 2, 2, 3, true>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream) : go<2, 4, 2, 2, 2, 3>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream);
        case 6: return once ? go<4, 2, 2, 4, 1, 4, true>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream) : go<4, 2, 2, 4, 1, 4>(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, stream);
        default: return go_ring(x, x_scale, w, w_scale, T, nk, O, Y, bf16, ldy, n_cu, stream);
    }
}

}  // namespace cq
