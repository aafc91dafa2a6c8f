// Attention of a decode step over the quantized key/value cache, in one pass over the codes.
//
//   z_p = scale log2(e) q . k_p,  k_p = a_p (code * b);   out = sum_p 2^(z_p - m) v_p / sum_p 2^(z_p - m),  m = max z_p
// A block takes 16 MR rows (tokens x query heads that share a key/value head) and a stretch of one sequence, its four waves every
// fourth tile of 32 positions; each wave keeps a running maximum, sum and output of its own, which meet at the end.  When a
// sequence is split over blocks, a second kernel joins their results.
//
// Scores: the column factors go into the query, q' = q b, and the codes into the INT8 matrix instruction as they are.  The other
// operand is q' as 16-bit fixed-point number relative to the row's largest |q'|: two signed digits, two products, an exact 32-bit
// sum (256 high + low: at most 256 * 127 * 32512 < 2^31), off by at most 1.6e-5 (half of 1 / 32512) of that largest.  Against codes turned into
// binary16: no conversion of K at all, at the same matrix time.  INT4 codes enter as 16 times their value (a mask or a shift).
// Values: weights w_p = 2^(z_p - m) a_p become binary16 relative to the largest a so far (a power of two R, 2^14 / R; the sums are
// rescaled when R grows, as for m), which leaves 38 binades below the largest weight; codes become binary16 exactly (0x6400 | u is
// 1024 + u).  Sums, m and the sum of 2^(z - m) are binary32.
//
// No operand passes through LDS.  The score tile is keys x rows, so that a lane holds scores of one row (lane & 15) for the positions
// 4 (lane >> 4) + r of a subtile of 16: just the contraction elements that the product with the values wants from it, in a
// position order that the loads of V follow.  A lane loads V for neighbouring channels of those positions and sorts the bytes.
// Bound by the cache's way from memory: 32 positions are requested while the 32 before are worked on.
#include <algorithm>
#include <type_traits>

#include "cq_gemm_common.h"

namespace cq {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kTile = 32;                                  // positions of a wave's step
constexpr int kBlockStep = kWaves * kTile;
constexpr float kDigits = 32512.0f;                        // 127 * 256
constexpr float kWeightTop = 16384.0f;                     // 2^14
constexpr float kSmallest = 7.888609052210118e-31f;        // 2^-100: queries and scales below count as zero

struct Args {
    const uint16_t* Q;
    int64_t q_batch, q_token, q_head;
    const uint8_t *k_codes, *v_codes;
    const float *k_scale, *v_scale, *k_col, *v_col;
    const int32_t *table, *lengths;
    int64_t table_width, pages;
    uint16_t* out;
    float* partial;                                        // [pair][split][rows][dim] sums, then [pair][split][rows][2] (m, l)
    int64_t n_partials;
    int heads, group, S, row_tiles, splits, chunk, page_shift, max_length;
    float scale;
    bool bf16;
};

// positions that token s of a sequence of n positions sees
__device__ __forceinline__ int visible(const Args& a, int n, int s) { return min(max(n - (a.S - 1 - s), 0), a.max_length); }

__device__ __forceinline__ float max_groups(float v) {     // over the four lanes that share a row
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_groups(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// N bytes per lane, N = 2 .. 32
template <int N>
struct Bytes {
    static constexpr int kWords = N < 4 ? 1 : N / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const uint8_t* p) {
        if (N == 2) {
            w[0] = *reinterpret_cast<const uint16_t*>(p);
        } else {
            __builtin_memcpy(w, __builtin_assume_aligned(p, N < 16 ? N : 16), N);
        }
    }
};

// The element of a row of `DIM` channels that byte e of fragment f holds for lane group g
template <int DIM, int BITS>
__device__ __forceinline__ constexpr int key_channel(int f, int e, int g) {
    return BITS == 8 ? 64 * f + 16 * g + e : DIM == 64 ? 16 * g + 2 * (e & 7) + (e >> 3) : 128 * (f >> 1) + 32 * g + 2 * e + (f & 1);
}

template <int DIM, int BITS>
struct Step {                                              // 32 positions: two subtiles of 16
    static constexpr int kKeyPiece = BITS == 4 && DIM == 64 ? 8 : 16, kKeyPieces = DIM * BITS / 8 / 4 / kKeyPiece;
    static constexpr int kValuePiece = DIM / 16 * BITS / 8;
    Bytes<kKeyPiece> k[2][kKeyPieces];
    Bytes<kValuePiece> v[2][4];
    float ka[2][4], va[2][4];
};

template <int DIM, int BITS, int MR>
__global__ void __launch_bounds__(64 * kWaves, 2)
attention_kernel(Args a) {
    constexpr int kFrags = DIM / 64, kOut = DIM / 16, kRowBytes = DIM * BITS / 8;
    constexpr int kPitch = DIM + 4;                        // floats; 16 rows 4 banks apart
    using StepT = Step<DIM, BITS>;
    __shared__ __align__(16) float sh_o[kWaves][16][kPitch];
    __shared__ float sh_ml[kWaves][16][2];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int fr = lane & 15, grp = lane >> 4;
    const int split = blockIdx.x % a.splits;
    const int64_t pair = blockIdx.x / a.splits;            // (sequence, head, row tile)
    const int rt = (int)(pair % a.row_tiles), head = (int)(pair / a.row_tiles % a.heads);
    const int64_t seq = pair / a.row_tiles / a.heads;
    const int rows = a.S * a.group, row0 = rt * 16 * MR, tile_rows = min(16 * MR, rows - row0);
    const int n = a.lengths[seq];
    const int s_first = row0 / a.group, s_last = (row0 + tile_rows - 1) / a.group;
    const int see_min = visible(a, n, s_first), see_max = visible(a, n, s_last);
    const int begin = split * a.chunk, end = min(begin + a.chunk, see_max);
    if (begin >= see_max && a.splits > 1) return;          // (the joining kernel knows)

    // ---- the rows' queries as two digits
    v4i q_hi[MR][kFrags], q_lo[MR][kFrags];
    float row_factor[MR], m[MR], l[MR];
    int see[MR];
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) {
        const int row = min(row0 + 16 * mr + fr, rows - 1), s = row / a.group, h = head * a.group + row % a.group;
        see[mr] = visible(a, n, s);
        const uint16_t* q = a.Q + seq * a.q_batch + s * a.q_token + h * a.q_head;
        float x[kFrags][16], top = 0.0f, bad = 0.0f;
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int d = key_channel<DIM, BITS>(f, e, grp);
                const uint32_t raw = q[d];
                float v = a.bf16 ? __uint_as_float(raw << 16) : h2f(raw);
                if (a.k_col) v *= a.k_col[head * DIM + d];
                x[f][e] = v;
                top = fmaxf(top, fabsf(v));
                bad += v * 0.0f;                           // NaN where q is no number
            }
        top = max_groups(top);
        bad = sum_groups(bad);
        const bool live = top >= kSmallest;                // kDigits / top stays in range
        const float inv = live ? kDigits / top : 0.0f;
        // codes of 4 bits enter as 16 times their value
        row_factor[mr] = (live ? top / kDigits : 0.0f) * (a.scale * 1.4426950408889634f * (BITS == 4 ? 0.0625f : 1.0f)) + bad;
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t hi = 0, lo = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int v = (int)__builtin_rintf(x[f][4 * w + b] * inv), h8 = (v + 128) >> 8;
                    hi |= (uint32_t)(h8 & 255) << (8 * b);
                    lo |= (uint32_t)(v & 255) << (8 * b);
                }
                q_hi[mr][f][w] = (int)hi;
                q_lo[mr][f][w] = (int)lo;
            }
        m[mr] = -INFINITY;
        l[mr] = 0.0f;
    }
    v4f o[MR][kOut];
#pragma unroll
    for (int mr = 0; mr < MR; ++mr)
#pragma unroll
        for (int i = 0; i < kOut; ++i) o[mr][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float R = kSmallest;                                   // the power of two above every a of V so far (from 2^-100)

    // ---- loads of 32 positions from `pos`.  Positions on no page read page 0 and are masked by their scale's place in `off`.
    const int32_t* table = a.table + seq * a.table_width;
    const int page_mask = (1 << a.page_shift) - 1, last_page = see_max > 0 ? (see_max - 1) >> a.page_shift : 0;
    auto load = [&](StepT& st, bool (&off)[2], int pos) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int p = pos + 16 * t;                    // wave-uniform; a subtile lies within a page
            int page = -1;
            if (p < see_max) page = table[min(p >> a.page_shift, last_page)];
            off[t] = page < 0 || page >= a.pages;
            const int64_t row = off[t] ? 0 : (((int64_t)page * a.heads + head) << a.page_shift) + (p & page_mask);
            const uint8_t* kp = a.k_codes + row * kRowBytes;
            const uint8_t* vp = a.v_codes + row * kRowBytes;
#pragma unroll
            for (int c = 0; c < StepT::kKeyPieces; ++c)
                st.k[t][c].load(kp + fr * kRowBytes + c * 4 * StepT::kKeyPiece + grp * StepT::kKeyPiece);
            const float4 ka = *reinterpret_cast<const float4*>(a.k_scale + row + 4 * grp);
            st.ka[t][0] = ka.x; st.ka[t][1] = ka.y; st.ka[t][2] = ka.z; st.ka[t][3] = ka.w;
#pragma unroll
            for (int r = 0; r < 4; ++r) st.v[t][r].load(vp + (4 * grp + r) * kRowBytes + fr * StepT::kValuePiece);
            const float4 va = *reinterpret_cast<const float4*>(a.v_scale + row + 4 * grp);
            st.va[t][0] = va.x; st.va[t][1] = va.y; st.va[t][2] = va.z; st.va[t][3] = va.w;
        }
    };

    auto work = [&](StepT& st, const bool (&off)[2], int pos) {
        const bool masked = pos + kTile > see_min || off[0] || off[1];       // (scalar)
        // keys: fragments of one position a lane
        v4i kf[2][kFrags];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int f = 0; f < kFrags; ++f)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t u;
                    if constexpr (BITS == 8) {
                        u = st.k[t][f].w[w];
                    } else if constexpr (DIM == 64) {
                        const uint32_t c = st.k[t][0].w[w & 1];
                        u = (w < 2 ? c << 4 : c) & 0xF0F0F0F0u;
                    } else {
                        const uint32_t c = st.k[t][f >> 1].w[w];
                        u = (f & 1 ? c : c << 4) & 0xF0F0F0F0u;
                    }
                    kf[t][f][w] = (int)u;
                }
        // the scale of V's weights
        float va_top = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (masked && (off[t] || pos + 16 * t + 4 * grp + r >= see_max)) st.va[t][r] = 0.0f;
                va_top = fmaxf(va_top, st.va[t][r]);
            }
        va_top = max_groups(va_top);
        const float R_new = fmaxf(R, __uint_as_float((__float_as_uint(va_top) & 0x7F800000u) + 0x00800000u));
        const float shrink = R / R_new;                    // powers of two
        R = R_new;
        const float to_weight = kWeightTop / R_new;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) st.va[t][r] *= to_weight;

        v8h p[MR];
#pragma unroll
        for (int mr = 0; mr < MR; ++mr) {
            float z[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                v4i hi = v4i{0, 0, 0, 0}, lo = v4i{0, 0, 0, 0};
#pragma unroll
                for (int f = 0; f < kFrags; ++f) {
                    hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[t][f], q_hi[mr][f], hi, 0, 0, 0);
                    lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[t][f], q_lo[mr][f], lo, 0, 0, 0);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    z[t][r] = (float)((hi[r] << 8) + lo[r]) * (row_factor[mr] * st.ka[t][r]);
                    if (masked && (off[t] || pos + 16 * t + 4 * grp + r >= see[mr])) z[t][r] = -INFINITY;
                }
            }
            float top = m[mr];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, z[t][r]);
            top = max_groups(top);
            const float ref = top == -INFINITY ? 0.0f : top;
            const float keep = __builtin_amdgcn_exp2f(m[mr] - ref);
            m[mr] = top;
            l[mr] *= keep;
            const float factor = keep * shrink;
            if (__any(factor != 1.0f)) {
#pragma unroll
                for (int i = 0; i < kOut; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[mr][i][r] *= factor;
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = __builtin_amdgcn_exp2f(z[t][r] - ref);
                    l[mr] += e;
                    float w = e * st.va[t][r];
                    if (masked && z[t][r] == -INFINITY) w = 0.0f;      // an unseen position's scale may be anything
                    p[mr][4 * t + r] = (_Float16)w;
                }
        }
        // values: channel kOut fr + i of the positions, i a tile of the product
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            v8h vf;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // code i of positions 2 h, 2 h + 1 as unsigned numbers in the low bytes of two halves
                    const int word = BITS == 8 ? i / 4 : i / 8, byte = BITS == 8 ? i % 4 : i % 8 / 2;
                    uint32_t x0 = st.v[t][2 * h].w[word], x1 = st.v[t][2 * h + 1].w[word];
                    if (BITS == 8) {
                        x0 ^= 0x80808080u;
                        x1 ^= 0x80808080u;
                    } else {
                        x0 = ((x0 ^ 0x88888888u) >> (i & 1 ? 4 : 0)) & 0x0F0F0F0Fu;
                        x1 = ((x1 ^ 0x88888888u) >> (i & 1 ? 4 : 0)) & 0x0F0F0F0Fu;
                    }
                    const uint32_t u = __builtin_amdgcn_perm(x1, x0, 0x0C040C00u + 0x00010001u * byte) | 0x64006400u;
                    const v2h c = __builtin_bit_cast(v2h, u) - (v2h)(_Float16)(BITS == 8 ? 1152.0f : 1032.0f);
                    vf[4 * t + 2 * h] = c[0];
                    vf[4 * t + 2 * h + 1] = c[1];
                }
#pragma unroll
            for (int mr = 0; mr < MR; ++mr) o[mr][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p[mr], o[mr][i], 0, 0, 0);
        }
    };

    {
        StepT st[2];
        bool off[2][2];
        int pos = begin + wave * kTile;
        if (pos < end) load(st[0], off[0], pos);
        while (pos < end) {
            if (pos + kBlockStep < end) load(st[1], off[1], pos + kBlockStep);
            work(st[0], off[0], pos);
            pos += kBlockStep;
            if (pos >= end) break;
            if (pos + kBlockStep < end) load(st[0], off[0], pos + kBlockStep);
            work(st[1], off[1], pos);
            pos += kBlockStep;
        }
    }

    // ---- the waves' results meet: 16 rows at a time
    const float unit = R / kWeightTop;
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) {
        if (mr > 0) __syncthreads();
        const float sum = sum_groups(l[mr]);
        if (grp == 0) {
            sh_ml[wave][fr][0] = m[mr];
            sh_ml[wave][fr][1] = sum;
        }
        // lane: channels kOut (4 grp + r) + i of row fr
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < kOut; i += 4)
                *reinterpret_cast<float4*>(&sh_o[wave][fr][kOut * (4 * grp + r) + i]) =
                    make_float4(o[mr][i][r] * unit, o[mr][i + 1][r] * unit, o[mr][i + 2][r] * unit, o[mr][i + 3][r] * unit);
        __syncthreads();
        constexpr int kCols = DIM / 16;                    // channels a thread joins
        const int row = threadIdx.x / 16, d0 = threadIdx.x % 16 * kCols, in_tile = 16 * mr + row;
        if (in_tile >= tile_rows) continue;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh_ml[w][row][0]);
        const float ref = top == -INFINITY ? 0.0f : top;
        float total = 0.0f, acc[kCols];
#pragma unroll
        for (int c = 0; c < kCols; ++c) acc[c] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(sh_ml[w][row][0] - ref);
            total = __builtin_fmaf(f, sh_ml[w][row][1], total);
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[c] = __builtin_fmaf(f, sh_o[w][row][d0 + c], acc[c]);
        }
        if (a.v_col) {
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[c] *= a.v_col[head * DIM + d0 + c];
        }
        if (a.splits == 1) {
            const int rr = row0 + in_tile, s = rr / a.group, h = head * a.group + rr % a.group;
            uint16_t* y = a.out + ((seq * a.S + s) * (int64_t)(a.heads * a.group) + h) * DIM + d0;
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const float v = total == 0.0f ? 0.0f : acc[c] / total;
                y[c] = a.bf16 ? __builtin_bit_cast(uint16_t, (__bf16)v) : (uint16_t)f2h(v);
            }
        } else {
            const int64_t at = (pair * a.splits + split) * min(16 * MR, rows) + in_tile;
#pragma unroll
            for (int c = 0; c < kCols; ++c) a.partial[at * DIM + d0 + c] = acc[c];
            if (d0 == 0) {
                float* ml = a.partial + a.n_partials * DIM + at * 2;
                ml[0] = top;
                ml[1] = total;
            }
        }
    }
}

// One block a row: dim / 4 lanes for the channels, the others share the splits.
template <int DIM>
__global__ void __launch_bounds__(256)
attention_join_kernel(Args a, int rows_per_tile) {
    constexpr int kLanesPerSplit = DIM / 4, kShares = 256 / kLanesPerSplit;
    __shared__ float4 sh[kShares][kLanesPerSplit];
    __shared__ float sh_l[kShares];
    const int rows = a.S * a.group;
    const int row = blockIdx.x % rows;
    const int64_t sh_pair = blockIdx.x / rows;             // (sequence, head)
    const int head = (int)(sh_pair % a.heads);
    const int64_t seq = sh_pair / a.heads;
    const int rt = row / rows_per_tile, in_tile = row - rt * rows_per_tile;
    const int s_last = min((rt + 1) * rows_per_tile, rows) - 1;
    const int see = visible(a, a.lengths[seq], s_last / a.group);
    const int used = (see + a.chunk - 1) / a.chunk;
    const int64_t first = (sh_pair * a.row_tiles + rt) * a.splits;
    const int share = threadIdx.x / kLanesPerSplit, c = threadIdx.x % kLanesPerSplit;
    const int per = min(rows_per_tile, rows);
    const float* ml = a.partial + a.n_partials * DIM;
    float top = -INFINITY;
    for (int k = 0; k < used; ++k) top = fmaxf(top, ml[((first + k) * per + in_tile) * 2]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float total = 0.0f;
    for (int k = share; k < used; k += kShares) {
        const int64_t at = (first + k) * per + in_tile;
        const float f = __builtin_amdgcn_exp2f(ml[at * 2] - ref);
        const float4 v = *reinterpret_cast<const float4*>(a.partial + at * DIM + 4 * c);
        total = __builtin_fmaf(f, ml[at * 2 + 1], total);
        acc.x = __builtin_fmaf(f, v.x, acc.x);
        acc.y = __builtin_fmaf(f, v.y, acc.y);
        acc.z = __builtin_fmaf(f, v.z, acc.z);
        acc.w = __builtin_fmaf(f, v.w, acc.w);
    }
    sh[share][c] = acc;
    if (c == 0) sh_l[share] = total;
    __syncthreads();
    if (share != 0) return;
#pragma unroll
    for (int k = 1; k < kShares; ++k) {
        const float4 v = sh[k][c];
        acc.x += v.x;
        acc.y += v.y;
        acc.z += v.z;
        acc.w += v.w;
        total += sh_l[k];
    }
    const float f[4] = {acc.x, acc.y, acc.z, acc.w};
    uint16_t* y = a.out + ((seq * a.S + row / a.group) * (int64_t)(a.heads * a.group) + head * a.group + row % a.group) * DIM + 4 * c;
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float v = total == 0.0f ? 0.0f : f[i] / total;
        q[i] = a.bf16 ? __builtin_bit_cast(uint16_t, (__bf16)v) : f2h(v);
    }
    *reinterpret_cast<uint2*>(y) = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
}

// How a call is cut: 16 or 32 rows a block, and sequences into stretches of `chunk` positions so that some kBlocks blocks come
// out (a CU holds two or three), but none of fewer than one step of its four waves.
constexpr int kBlocks = 1024;
struct Plan {
    int mr, row_tiles, splits, chunk;
    int64_t pairs;
};
Plan plan(const CacheView& c, const AttentionShape& s) {
    Plan p;
    const int rows = s.S * (s.q_heads / c.heads);
    p.mr = rows > 16 && c.dim < 256 ? 2 : 1;
    p.row_tiles = (rows + 16 * p.mr - 1) / (16 * p.mr);
    p.pairs = s.B * c.heads * p.row_tiles;
    const int64_t want = (kBlocks + p.pairs - 1) / p.pairs, steps = (s.max_length + kBlockStep - 1) / kBlockStep;
    const int64_t per = (steps + std::min(want, steps) - 1) / std::min(want, steps);        // steps of a block
    p.chunk = (int)(per * kBlockStep);
    p.splits = (int)((steps + per - 1) / per);
    return p;
}
int64_t partials(const CacheView& c, const AttentionShape& s, const Plan& p) {
    return p.splits > 1 ? p.pairs * p.splits * std::min(16 * p.mr, s.S * (s.q_heads / c.heads)) : 0;
}

}  // namespace

int64_t cache_attention_workspace(const CacheView& c, const AttentionShape& s) {
    return partials(c, s, plan(c, s)) * (c.dim + 2) * 4;
}

hipError_t launch_cache_attention(const CacheView& c, const AttentionShape& s, const uint16_t* Q, int64_t q_batch, int64_t q_token,
                                  int64_t q_head, bool bf16, const int32_t* table, int64_t table_width, const int32_t* lengths,
                                  float scale, uint16_t* out, float* workspace, hipStream_t stream) {
    const Plan p = plan(c, s);
    const int group = s.q_heads / c.heads;
    const int64_t blocks = p.pairs * p.splits, rows = s.B * c.heads * s.S * group;
    if (!grid_fits(blocks, 64 * kWaves) || !grid_fits(rows, 256)) return hipErrorInvalidValue;
    Args a;
    a.Q = Q; a.q_batch = q_batch; a.q_token = q_token; a.q_head = q_head;
    a.k_codes = c.k_codes; a.v_codes = c.v_codes; a.k_scale = c.k_scale; a.v_scale = c.v_scale; a.k_col = c.k_col; a.v_col = c.v_col;
    a.table = table; a.lengths = lengths; a.table_width = table_width; a.pages = c.pages;
    a.out = out; a.partial = workspace; a.n_partials = partials(c, s, p);
    a.heads = c.heads; a.group = group; a.S = s.S; a.row_tiles = p.row_tiles; a.splits = p.splits; a.chunk = p.chunk;
    a.page_shift = c.page_shift; a.max_length = s.max_length; a.scale = scale; a.bf16 = bf16;
    auto go = [&](auto kernel) { kernel<<<(unsigned)blocks, 64 * kWaves, 0, stream>>>(a); };
    if (c.bits == 8) {
        if (c.dim == 64) p.mr == 2 ? go(attention_kernel<64, 8, 2>) : go(attention_kernel<64, 8, 1>);
        else if (c.dim == 128) p.mr == 2 ? go(attention_kernel<128, 8, 2>) : go(attention_kernel<128, 8, 1>);
        else go(attention_kernel<256, 8, 1>);
    } else {
        if (c.dim == 64) p.mr == 2 ? go(attention_kernel<64, 4, 2>) : go(attention_kernel<64, 4, 1>);
        else if (c.dim == 128) p.mr == 2 ? go(attention_kernel<128, 4, 2>) : go(attention_kernel<128, 4, 1>);
        else go(attention_kernel<256, 4, 1>);
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess || p.splits == 1) return e;
    auto join = [&](auto kernel) { kernel<<<(unsigned)rows, 256, 0, stream>>>(a, 16 * p.mr); };
    if (c.dim == 64) join(attention_join_kernel<64>);
    else if (c.dim == 128) join(attention_join_kernel<128>);
    else join(attention_join_kernel<256>);
    return hipGetLastError();
}

}  // namespace cq
