// Attention of a decode step over the quantized key/value cache, in one pass over the codes.
//
//   z_p = scale log2(e) q . k_p,  k_p = a_p (code * b);   out = sum_p 2^(z_p - m) v_p / sum_p 2^(z_p - m),  m = max z_p
// A pair is a sequence, a key/value head and 16 MR rows (tokens x query heads that share the head); its unit of work is one step of a block, 128 positions.  All
// units in a row, pair after pair, are cut into equal stretches, one for each block that the chip holds at once: each block adds up the lengths
// for itself to find where its stretch starts.  A block works through the pieces of pairs in its stretch, its four waves every
// fourth tile of 32 positions, each with a running maximum, sum and output of its own, which meet at the piece's end.  A pair that lies in one
// stretch is done then; pieces of others go to the workspace and a second kernel joins them.
// (64 sequences of 1024 to 8192 positions, 512 pairs: with the pairs' maximum length cut into a fixed number of blocks 175 us at best, 135 so; with
// what came later 125, 5.1 TB/s; 2 sequences of 73728 and 131072 positions, INT4, 8 heads: 57 to 60 us, 3.7 to 3.9 TB/s.)
//
// Scores: the column factors go into the query, q' = q b, and the codes into the INT8 matrix instruction as they are.  The other
// operand is q' as 16-bit fixed-point number relative to the row's largest |q'|: two signed digits, two products, an exact 32-bit
// sum (256 high + low: at most 256 * 127 * 32512 < 2^31), off by at most 1.6e-5 (half of 1 / 32512) of that largest.  Against codes turned into
// binary16: no conversion of K at all, at the same matrix time.  INT4 codes enter as 16 times their value (a mask or a shift).
// Values: weights w_p = 2^(z_p - m) a_p become two binary16 numbers (rounded, and what is left: 22 bits) in units of R / 65504, R the
// row's largest w so far up to a power of two and two binades.  R shrinks with the weights as m grows, so that the sums, in units of it
// too, need no rescaling then; a larger w takes a new R and rescales them.  The 22 bits reach 16 binades below the largest w, the units of
// the second number 38.  (With R from the largest a, whatever its position's score, a value 2^30 times the others that no query attends to
// took all but 8 bits of them.  Without the two binades some row of a wave takes a new R in most tiles of a stretch: 2 x 131072 INT4
// 62 us, with them 60.3; 64 x 1024-8192, INT4, 86.2 and 85.6.)
// Codes become binary16 exactly (as subnormal numbers, and from there in one fused step).  With one number a weight the result was off by sqrt(2) times what its
// own rounding to binary16 costs; the second product is in the shadow of the loads.  Sums, m and the sum of 2^(z - m) are binary32.
//
// No operand passes through LDS.  The score tile is keys x rows, so that a lane holds scores of one row (lane & 15) for the positions
// 4 (lane >> 4) + r of a subtile of 16: just the contraction elements that the product with the values wants from it, in a
// position order that the loads of V follow.  A lane loads V for neighbouring channels of those positions and sorts the bytes.
// Bound by the cache's way from memory.
#include <algorithm>
#include <type_traits>

#include "cq_gemm_common.h"

namespace cq {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kSub = 2;                                    // subtiles of 16 positions that a wave works on at a time
constexpr int kTile = 16 * kSub, kBlockStep = kWaves * kTile;
constexpr float kDigits = 32512.0f;                        // 127 * 256
constexpr float kWeightTop = 65504.0f;                     // binary16's largest
constexpr uint32_t kHeadroom = 2;                          // binades that R leaves above the product it is taken from
constexpr float kSmallest = 7.888609052210118e-31f;        // 2^-100: queries below count as zero, and R is no smaller

struct Args {
    const uint16_t* Q;
    int64_t q_batch, q_token, q_head;
    const uint8_t *k_codes, *v_codes;
    const float *k_scale, *v_scale, *k_col, *v_col;
    const int32_t *table, *lengths;
    int64_t table_width, pages;
    uint16_t* out;
    // pieces of pairs, two a block: [piece][rows][dim] sums, [piece][rows][2] (m, l); then for each pair its first and last block
    float* partial;
    int64_t n_partials, n_sequences;
    int heads, group, S, row_tiles, n_blocks, page_shift, max_length;     // n_blocks 0: a block a pair, no pieces
    float scale;
    bool bf16;
};

// positions that token s of a sequence of n positions sees (n from memory: anything)
__device__ __forceinline__ int visible(const Args& a, int n, int s) { return min(max(max(n, 0) - (a.S - 1 - s), 0), a.max_length); }

// over the four lanes that share a row: the swap leaves one row of 16 (half of 32) lanes twice in the first and the other twice in
// the second register
__device__ __forceinline__ float max_groups(float v) {
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float sum_groups(float v) {
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
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
    // the same for bytes that no other load asks for and no cache keeps
    __device__ __forceinline__ void load_once(const uint8_t* p) {
        if (N == 2) return load(p);
        typedef uint32_t V __attribute__((ext_vector_type(N < 4 ? 1 : N < 16 ? N / 4 : 4)));
#pragma unroll
        for (int i = 0; i < (N + 15) / 16; ++i) {
            const V v = __builtin_nontemporal_load(reinterpret_cast<const V*>(p) + i);
            __builtin_memcpy(w + 4 * i, &v, sizeof(v));
        }
    }
};

// Which of a lane's channels (neighbours, 16 or 32 at a time, see the queries' part) byte e of fragment f holds.  8 bits: fragment f is
// a piece of 16 bytes.  4 bits: a piece's low nibbles are its even channels, its high ones the odd; a piece makes two fragments, or one
// where it has 8 bytes only.
template <int DIM, int BITS>
__device__ __forceinline__ constexpr int key_run(int f, int e) {
    return BITS == 8 ? 16 * f + e : DIM == 64 ? 2 * (e & 7) + (e >> 3) : 32 * (f >> 1) + 2 * e + (f & 1);
}

template <int DIM, int BITS>
struct Keys {                                              // of a wave's subtiles
    static constexpr int kPiece = BITS == 4 && DIM == 64 ? 8 : 16, kPieces = DIM * BITS / 8 / 4 / kPiece;
    Bytes<kPiece> c[kSub][kPieces];
    float a[kSub][4];
    int64_t row[kSub];                                     // the subtiles' first rows
    bool off[kSub];                                        // on no page
};
template <int DIM, int BITS>
struct Values {
    static constexpr int kPiece = DIM / 16 * BITS / 8;
    Bytes<kPiece> c[kSub][4];
    float a[kSub][4];
};

// units of a sequence of n positions, in every one of its pairs
__device__ __forceinline__ int units_of(const Args& a, int n) { return (visible(a, n, a.S - 1) + kBlockStep - 1) / kBlockStep; }

// x / n for x >= 0, n > 0 (a division of 64 bits takes several times as long)
__device__ __forceinline__ int64_t divide(int64_t x, int n) { return x >> 32 == 0 ? (int64_t)((uint32_t)x / (uint32_t)n) : x / n; }

// `total` units cut for n blocks: block i's stretch is [i q + min(i, r), ...), q = total / n, r = total % n
struct Cut {
    int64_t q, r;
    __device__ __forceinline__ Cut(int64_t total, int n) : q(divide(total, n)), r(total - q * n) {}
    __device__ __forceinline__ int64_t first(int64_t i) const { return i * q + min(i, r); }
    __device__ __forceinline__ int block_of(int64_t unit) const {
        const int64_t longer = r * (q + 1);                // units in the stretches of q + 1
        return (int)(unit < longer ? divide(unit, (int)q + 1) : r + divide(unit - longer, (int)q));
    }
};

// inclusive sums over the wave's lanes
__device__ __forceinline__ int prefix_sum(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);        // from the lanes 1, 2, 4, 8 before in a row of 16
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);        // the row before's last lane, to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);        // lane 31, to rows 2 and 3
    return v;
}

// a wave-uniform value in scalar registers: what comes out of LDS would make vector work of all that follows from it
__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t scalar(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)scalar((int)(v >> 32)) << 32 | (uint32_t)scalar((int)v));
}

template <int DIM, int W>
struct Shared {
    float o[W][16][DIM + 4];                               // 16 rows 4 banks apart
    float ml[W][16][2];
};

// Units [unit0, unit0 + count) of a pair.  piece < 0: that is all of it, and the result is written; otherwise where it goes.
// ONCE: the values' loads are non-temporal.  W: waves of the block (a unit is W tiles of positions).
template <int DIM, int BITS, int MR, bool ONCE, int W>
__device__ __forceinline__ void attention_piece(const Args& a, Shared<DIM, W>& sh, int64_t seq, int head, int rt, int n, int unit0, int count,
                                                int piece) {
    constexpr int kFrags = DIM / 64, kOut = DIM / 16, kRowBytes = DIM * BITS / 8, kStep = W * kTile;
    using KeysT = Keys<DIM, BITS>;
    using ValuesT = Values<DIM, BITS>;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int fr = lane & 15, grp = lane >> 4;
    const int rows = a.S * a.group, row0 = rt * 16 * MR, tile_rows = min(16 * MR, rows - row0);
    const int s_first = row0 / a.group, s_last = (row0 + tile_rows - 1) / a.group;
    const int see_min = visible(a, n, s_first), see_max = visible(a, n, s_last);
    const int begin = unit0 * kStep, end = min(begin + count * kStep, see_max);

    // ---- loads of a tile's positions from `pos`.  Positions on no page read page 0 and are masked.
    const int32_t* table = a.table + seq * a.table_width;
    const int page_mask = (1 << a.page_shift) - 1, last_page = see_max > 0 ? (see_max - 1) >> a.page_shift : 0;
    // A tile's page numbers come from a register that holds those of the wave's next 32 tiles: asked of the table tile by tile they
    // would stand in front of every tile's loads.
    static_assert(kSub == 2, "two lanes a tile");
    int pages = -1;
    auto load_pages = [&](int pos) {                       // of the tiles at pos, pos + kStep, ..
        const int64_t p = pos + (int64_t)(lane >> 1) * kStep + 16 * (lane & 1);
        pages = p < see_max ? table[min((int)(p >> a.page_shift), last_page)] : -1;
    };
    auto load_keys = [&](KeysT& k, int pos, int tile) {
#pragma unroll
        for (int t = 0; t < kSub; ++t) {
            const int p = pos + 16 * t;                    // wave-uniform; a subtile lies within a page
            const int page = __builtin_amdgcn_readlane(pages, (2 * tile + t) & 63);
            k.off[t] = page < 0 || page >= a.pages;
            k.row[t] = k.off[t] ? 0 : (((int64_t)page * a.heads + head) << a.page_shift) + (p & page_mask);
            const uint8_t* kp = a.k_codes + k.row[t] * kRowBytes;
#pragma unroll
            for (int c = 0; c < KeysT::kPieces; ++c)
                k.c[t][c].load(kp + fr * kRowBytes + c * 4 * KeysT::kPiece + grp * KeysT::kPiece);
            const float4 f = *reinterpret_cast<const float4*>(a.k_scale + k.row[t] + 4 * grp);
            k.a[t][0] = f.x; k.a[t][1] = f.y; k.a[t][2] = f.z; k.a[t][3] = f.w;
        }
    };
    auto load_values = [&](ValuesT& v, const KeysT& k) {
#pragma unroll
        for (int t = 0; t < kSub; ++t) {
            const uint8_t* vp = a.v_codes + k.row[t] * kRowBytes;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint8_t* at = vp + (4 * grp + r) * kRowBytes + fr * ValuesT::kPiece;
                if (ONCE) v.c[t][r].load_once(at);
                else v.c[t][r].load(at);
            }
            const float4 f = *reinterpret_cast<const float4*>(a.v_scale + k.row[t] + 4 * grp);
            v.a[t][0] = f.x; v.a[t][1] = f.y; v.a[t][2] = f.z; v.a[t][3] = f.w;
        }
    };
    KeysT k;
    ValuesT v;
    int pos = begin + wave * kTile, tile = 0;
    load_pages(pos);
    load_keys(k, pos, 0);                                     // (before the queries are worked on; past the end nothing is seen)
    load_values(v, k);

    // ---- the rows' queries as two digits
    v4i q_hi[MR][kFrags], q_lo[MR][kFrags];
    float row_factor[MR], m[MR], l[MR];
    int see[MR];
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) {
        const int row = min(row0 + 16 * mr + fr, rows - 1), s = row / a.group, h = head * a.group + row % a.group;
        see[mr] = visible(a, n, s);
        const uint16_t* q = a.Q + seq * a.q_batch + s * a.q_token + h * a.q_head;
        // the lane's channels are runs of kRun neighbours
        constexpr int kRun = BITS == 4 && DIM > 64 ? 32 : 16, kRuns = DIM / 4 / kRun;
        float x[kRuns * kRun], top = 0.0f, bad = 0.0f;
#pragma unroll
        for (int c = 0; c < kRuns * kRun; c += 8) {
            const int d = c / kRun * 4 * kRun + grp * kRun + c % kRun;
            const uint4 raw = *reinterpret_cast<const uint4*>(q + d);
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t h = e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xFFFFu;
                x[c + e] = a.bf16 ? __uint_as_float(h << 16) : h2f(h);
            }
            if (a.k_col) {
                const float4 lo = *reinterpret_cast<const float4*>(a.k_col + (int64_t)head * DIM + d);
                const float4 hi = *reinterpret_cast<const float4*>(a.k_col + (int64_t)head * DIM + d + 4);
                const float b[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) x[c + e] *= b[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                top = fmaxf(top, fabsf(x[c + e]));
                bad += x[c + e] * 0.0f;                    // NaN where q is no number
            }
        }
        top = max_groups(top);
        bad = sum_groups(bad);
        // A row whose query holds no number: digits of zero and an infinite factor, so that a score is 0 * infinity = NaN where the row
        // sees the position and -infinity where it does not (a row that sees none stays zero).
        const bool none = bad != 0.0f;
        if (__any(none)) {
            asm volatile("");                              // (a branch: seldom)
#pragma unroll
            for (int e = 0; e < kRuns * kRun; ++e) x[e] = none ? 0.0f : x[e];
        }
        const bool live = top >= kSmallest && !none;       // kDigits / top stays in range
        // (the digits take the scale's sign)
        const float inv = live ? (a.scale < 0.0f ? -kDigits : kDigits) / top : 0.0f;
        // (codes of 4 bits enter as 16 times their value)
        const float f = (live ? top / kDigits : 0.0f) * (fabsf(a.scale) * 1.4426950408889634f * (BITS == 4 ? 0.0625f : 1.0f));
        row_factor[mr] = none ? INFINITY : f;
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t hi = 0, lo = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    // byte e of fragment f: see key_run
                    const int v = (int)__builtin_rintf(x[key_run<DIM, BITS>(f, 4 * w + b)] * inv), h8 = (v + 128) >> 8;
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
    float R[MR];                                           // above every product 2^(z - m) a of the row so far; o is in units of it
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) R[mr] = 0.0f;
    // codes leave the subnormal numbers times 2^10 and without what was added to them: q 2^-14
    const v2h code_unit = (v2h)(_Float16)1024.0f, code_zero = (v2h)(_Float16)(BITS == 8 ? -0.0078125f : -0.00048828125f);

    // Keys are requested for the next positions as soon as the scores are out, values as soon as they are summed: one set of registers
    // each, and always something on its way.
    while (pos < end) {
        const int next = pos + kStep;
        bool off[kSub], masked = pos + kTile > see_min;        // (scalar)
#pragma unroll
        for (int t = 0; t < kSub; ++t) {
            off[t] = k.off[t];
            masked = masked || off[t];
        }
        float z[MR][kSub][4];
#pragma unroll
        for (int t = 0; t < kSub; ++t) {
            v4i kf[kFrags];                                // fragments of one position a lane
#pragma unroll
            for (int f = 0; f < kFrags; ++f)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t u;
                    if constexpr (BITS == 8) {
                        u = k.c[t][f].w[w];
                    } else if constexpr (DIM == 64) {
                        const uint32_t c = k.c[t][0].w[w & 1];
                        u = (w < 2 ? c << 4 : c) & 0xF0F0F0F0u;
                    } else {
                        const uint32_t c = k.c[t][f >> 1].w[w];
                        u = (f & 1 ? c : c << 4) & 0xF0F0F0F0u;
                    }
                    kf[f][w] = (int)u;
                }
#pragma unroll
            for (int mr = 0; mr < MR; ++mr) {
                v4i hi = v4i{0, 0, 0, 0}, lo = v4i{0, 0, 0, 0};
#pragma unroll
                for (int f = 0; f < kFrags; ++f) {
                    hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[f], q_hi[mr][f], hi, 0, 0, 0);
                    lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[f], q_lo[mr][f], lo, 0, 0, 0);
                }
                // The two factors first: no part leaves binary32 where the score does not.  And rounded before the maximum is taken from it: with
                // a rounded maximum against products inside a fused step, equal scores of more than 2^32 gave NaN.
#pragma unroll
                for (int r = 0; r < 4; ++r) z[mr][t][r] = (float)((hi[r] << 8) + lo[r]) * (k.a[t][r] * row_factor[mr]);
            }
        }
        if (masked) {
            asm volatile("");                              // (a branch: as selects it would cost every tile 40 instructions)
#pragma unroll
            for (int t = 0; t < kSub; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = pos + 16 * t + 4 * grp + r;
                    bool any = false;
#pragma unroll
                    for (int mr = 0; mr < MR; ++mr) {
                        const bool seen = !off[t] && at < see[mr];
                        any = any || seen;
                        if (!seen) z[mr][t][r] = -INFINITY;
                    }
                    if (!any) v.a[t][r] = 0.0f;            // an unseen position's scale may be anything
                }
        }
        if (next < end) {
            if ((++tile & 31) == 0) load_pages(next);
            load_keys(k, next, tile);
        }
        v8h p[MR][kSub / 2], p_rest[MR][kSub / 2];
#pragma unroll
        for (int mr = 0; mr < MR; ++mr) {
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < kSub; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, z[mr][t][r]);
            top = fmaxf(m[mr], max_groups(top));
            const float ref = top == -INFINITY ? 0.0f : top;
            const float keep = __builtin_amdgcn_exp2f(m[mr] - ref);
            m[mr] = top;
            l[mr] *= keep;
            float w[kSub][4], w_top = kSmallest;
#pragma unroll
            for (int t = 0; t < kSub; ++t)
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    const float e0 = __builtin_amdgcn_exp2f(z[mr][t][r] - ref);
                    const float e1 = __builtin_amdgcn_exp2f(z[mr][t][r + 1] - ref);
                    l[mr] += e0 + e1;
                    w[t][r] = e0 * v.a[t][r];
                    w[t][r + 1] = e1 * v.a[t][r + 1];
                    // (of two rows one may see a position whose scale is no number, and the other not: by the score, as a weight that
                    // is 0 in binary32 does not hide it)
                    if (MR > 1 && masked) {
                        if (z[mr][t][r] == -INFINITY) w[t][r] = 0.0f;
                        if (z[mr][t][r + 1] == -INFINITY) w[t][r + 1] = 0.0f;
                    }
                    w_top = fmaxf(w_top, fmaxf(w[t][r], w[t][r + 1]));
                }
            // Sums so far shrink with R as m grows; a larger product (or an R below 2^-100) takes a new power of two.
            R[mr] *= keep;
            if (__any(w_top >= R[mr])) {
                w_top = max_groups(w_top);
                const bool more = w_top >= R[mr];
                // (2^126 at most, which is above every factor that a row of numbers can have)
                const uint32_t R_bits = min((__float_as_uint(w_top) & 0x7F800000u) + (kHeadroom + 1) * 0x00800000u, 0x7E800000u);
                const float shrink = more ? R[mr] * __uint_as_float(0x7F000000u - R_bits) : 1.0f;     // (times 1 / R_new)
#pragma unroll
                for (int i = 0; i < kOut; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[mr][i][r] *= shrink;
                R[mr] = more ? __uint_as_float(R_bits) : R[mr];
            }
            const float to_weight = kWeightTop * __builtin_amdgcn_rcpf(R[mr]);
#pragma unroll
            for (int t = 0; t < kSub; ++t)
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    typedef float v2f __attribute__((ext_vector_type(2)));
                    const v2f u = {w[t][r] * to_weight, w[t][r + 1] * to_weight};
                    const v2h w16 = __builtin_convertvector(u, v2h);
                    const v2f rest = {__builtin_fmaf((float)w16[0], -1.0f, u[0]), __builtin_fmaf((float)w16[1], -1.0f, u[1])};
                    const v2h rest16 = __builtin_convertvector(rest, v2h);
                    const int at = 4 * (t & 1) + r;
                    p[mr][t / 2][at] = w16[0];
                    p[mr][t / 2][at + 1] = w16[1];
                    p_rest[mr][t / 2][at] = rest16[0];
                    p_rest[mr][t / 2][at + 1] = rest16[1];
                }
        }
        // values: channel kOut fr + i of the positions, i a tile of the product
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            v8h vf[kSub / 2];
#pragma unroll
            for (int t = 0; t < kSub; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // code i of positions 2 h, 2 h + 1 plus 128 (8) as the low bytes of two halves: subnormal numbers of 2^-24
                    const int word = BITS == 8 ? i / 4 : i / 8, byte = BITS == 8 ? i % 4 : i % 8 / 2;
                    uint32_t x0 = v.c[t][2 * h].w[word], x1 = v.c[t][2 * h + 1].w[word];
                    if (BITS == 8) {
                        x0 ^= 0x80808080u;
                        x1 ^= 0x80808080u;
                    } else {
                        x0 = ((x0 ^ 0x88888888u) >> (i & 1 ? 4 : 0)) & 0x0F0F0F0Fu;
                        x1 = ((x1 ^ 0x88888888u) >> (i & 1 ? 4 : 0)) & 0x0F0F0F0Fu;
                    }
                    const uint32_t u = __builtin_amdgcn_perm(x1, x0, 0x0C040C00u + 0x00010001u * byte);
                    const v2h c = __builtin_elementwise_fma(__builtin_bit_cast(v2h, u), code_unit, code_zero);
                    vf[t / 2][4 * (t & 1) + 2 * h] = c[0];
                    vf[t / 2][4 * (t & 1) + 2 * h + 1] = c[1];
                }
#pragma unroll
            for (int mr = 0; mr < MR; ++mr)
#pragma unroll
                for (int c = 0; c < kSub / 2; ++c) {
                    o[mr][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[c], p[mr][c], o[mr][i], 0, 0, 0);
                    o[mr][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[c], p_rest[mr][c], o[mr][i], 0, 0, 0);
                }
        }
        if (next < end) load_values(v, k);
        pos = next;
    }

    // ---- the waves' results meet: 16 rows at a time
#pragma unroll
    for (int mr = 0; mr < MR; ++mr) {
        __syncthreads();                                   // (what the last piece or rows left has been read)
        const float sum = sum_groups(l[mr]), unit = R[mr] * (16384.0f / kWeightTop);          // (2^-14 a code)
        if (grp == 0) {
            sh.ml[wave][fr][0] = m[mr];
            sh.ml[wave][fr][1] = sum;
        }
        // lane: channels kOut (4 grp + r) + i of row fr
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < kOut; i += 4)
                *reinterpret_cast<float4*>(&sh.o[wave][fr][kOut * (4 * grp + r) + i]) =
                    make_float4(o[mr][i][r] * unit, o[mr][i + 1][r] * unit, o[mr][i + 2][r] * unit, o[mr][i + 3][r] * unit);
        __syncthreads();
        constexpr int kCols = DIM / 16;                    // channels a thread joins
        const int row = threadIdx.x / 16, d0 = threadIdx.x % 16 * kCols, in_tile = 16 * mr + row;
        if (in_tile >= tile_rows || row >= 16) continue;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, sh.ml[w][row][0]);
        const float ref = top == -INFINITY ? 0.0f : top;
        float total = 0.0f, acc[kCols];
#pragma unroll
        for (int c = 0; c < kCols; ++c) acc[c] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = __builtin_amdgcn_exp2f(sh.ml[w][row][0] - ref);
            total = __builtin_fmaf(f, sh.ml[w][row][1], total);
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[c] = __builtin_fmaf(f, sh.o[w][row][d0 + c], acc[c]);
        }
        if (a.v_col) {
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[c] *= a.v_col[(int64_t)head * DIM + d0 + c];
        }
        if (piece < 0) {
            const int rr = row0 + in_tile, s = rr / a.group, h = head * a.group + rr % a.group;
            uint16_t* y = a.out + ((seq * a.S + s) * (int64_t)(a.heads * a.group) + h) * DIM + d0;
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const float v = total == 0.0f ? 0.0f : acc[c] / total;
                y[c] = a.bf16 ? __builtin_bit_cast(uint16_t, (__bf16)v) : (uint16_t)f2h(v);
            }
        } else {
            const int64_t at = (int64_t)piece * min(16 * MR, rows) + in_tile;
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

// W = 8: a block a pair only.
template <int DIM, int BITS, int MR, bool ONCE, int W>
__global__ void __launch_bounds__(64 * W, MR == 1 ? DIM == 64 ? 4 : DIM == 128 ? 3 : 2 : 2)
attention_kernel(Args a) {
    __shared__ __align__(16) Shared<DIM, W> sh;
    __shared__ int64_t sh_sum[kWaves], sh_at[2];
    const int per_seq = a.heads * a.row_tiles, tid = threadIdx.x;          // pairs of a sequence
    int64_t total = 0, at = 0, end = 0;
    int seq, j, unit, n, u;
    if (W != kWaves || a.n_blocks == 0) {
        seq = blockIdx.x / per_seq;
        j = blockIdx.x - seq * per_seq;
        unit = 0;
        n = scalar(a.lengths[seq]);
        u = units_of(a, n);
        end = u;
    } else if (a.n_sequences <= 64) {
        // where this block's stretch starts: each wave for itself, a lane a sequence (at most 2^24 units each)
        const int q = tid & 63, n_q = q < a.n_sequences ? a.lengths[q] : 0, u_q = q < a.n_sequences ? units_of(a, n_q) : 0, upto = prefix_sum(u_q);
        total = (int64_t)__builtin_amdgcn_readlane(upto, 63) * per_seq;
        const Cut cut(total, a.n_blocks);
        at = cut.first(blockIdx.x);
        end = cut.first(blockIdx.x + 1);
        if (at >= end) return;
        seq = __builtin_ctzll(__ballot((int64_t)upto * per_seq > at));
        n = __builtin_amdgcn_readlane(n_q, seq);
        u = __builtin_amdgcn_readlane(u_q, seq);
        const int64_t in_seq = at - (int64_t)(__builtin_amdgcn_readlane(upto, seq) - u) * per_seq;
        j = (int)divide(in_seq, u);
        unit = (int)(in_seq - (int64_t)j * u);
    } else {
        // the same for more: a thread adds up neighbouring sequences
        const int64_t each = (a.n_sequences + 64 * kWaves - 1) / (64 * kWaves), s0 = min(tid * each, a.n_sequences), s1 = min(s0 + each, a.n_sequences);
        int64_t mine = 0;
        for (int64_t q = s0; q < s1; ++q) mine += units_of(a, a.lengths[q]);
        int64_t upto = mine;                                   // inclusive sums over the wave
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int64_t v = __shfl_up((long long)upto, d, 64);
            if ((tid & 63) >= d) upto += v;
        }
        if ((tid & 63) == 63) sh_sum[tid >> 6] = upto;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < tid >> 6) upto += sh_sum[w];
            total += sh_sum[w];
        }
        total = scalar(total * per_seq);
        const Cut cut(total, a.n_blocks);
        at = scalar(cut.first(blockIdx.x));
        end = scalar(cut.first(blockIdx.x + 1));
        if (at >= end) return;                                 // (block-uniform)
        if ((upto - mine) * per_seq <= at && at < upto * per_seq) {
            int64_t before = upto - mine;
            for (int64_t q = s0; q < s1; ++q) {
                const int u = units_of(a, a.lengths[q]);
                if (at < (before + u) * per_seq) {
                    sh_at[0] = q;
                    sh_at[1] = before;
                    break;
                }
                before += u;
            }
        }
        __syncthreads();
        seq = scalar((int)sh_at[0]);
        n = scalar(a.lengths[seq]);
        u = units_of(a, n);
        const int64_t in_seq = at - scalar(sh_at[1]) * per_seq;
        j = scalar((int)divide(in_seq, u));
        unit = scalar((int)(in_seq - (int64_t)j * u));
    }
    int* ends = reinterpret_cast<int*>(a.partial + a.n_partials * (DIM + 2));
    while (true) {
        const int count = (int)min((int64_t)(u - unit), end - at);
        if (a.n_blocks != 0 && unit == 0 && tid == 0) {
            const int64_t pair = (int64_t)seq * per_seq + j;
            ends[2 * pair] = blockIdx.x;
            ends[2 * pair + 1] = count == u ? blockIdx.x : Cut(total, a.n_blocks).block_of(at + u - 1);
        }
        // a stretch has at most one piece that continues a pair and one that only begins one
        attention_piece<DIM, BITS, MR, ONCE, W>(a, sh, seq, j / a.row_tiles, j % a.row_tiles, n, unit, count,
                                       count == u ? -1 : 2 * blockIdx.x + (unit == 0 ? 1 : 0));
        at += count;
        if (at >= end) break;
        unit = 0;
        if (++j == per_seq) {                              // a unit is left, so there is a sequence with one
            j = 0;
            do {
                n = scalar(a.lengths[++seq]);
                u = units_of(a, n);
            } while (u == 0);
        }
    }
}

// A row that has pieces in several blocks (none that lies in one is worked on again): where they are, and where it goes.
struct JoinRow {
    int first, used, per, in_tile;                         // blocks first .. first + used - 1; used 0: no position at all, the row is zero
    uint16_t* out;
    // the pair's first block left its piece in the second of its places, the others in their first
    __device__ __forceinline__ int64_t row_of(int k) const { return ((int64_t)2 * (first + k) + (k == 0 ? 1 : 0)) * per + in_tile; }
};
template <int DIM>
__device__ __forceinline__ JoinRow join_row(const Args& a, int64_t id, int rows_per_tile) {
    JoinRow j;
    const int rows = a.S * a.group, row = (int)(id % rows);
    const int64_t sh_pair = id / rows, seq = sh_pair / a.heads;            // (sequence, head)
    const int head = (int)(sh_pair - seq * a.heads), rt = row / rows_per_tile;
    j.in_tile = row - rt * rows_per_tile;
    j.per = min(rows_per_tile, rows);
    const int* ends = reinterpret_cast<const int*>(a.partial + a.n_partials * (DIM + 2)) + 2 * (sh_pair * a.row_tiles + rt);
    const int first = ends[0], last = ends[1];             // (asked for before the length says whether they mean anything)
    const bool any = units_of(a, a.lengths[seq]) > 0;
    j.first = any ? first : 0;
    j.used = any ? last - first + 1 : 0;
    j.out = a.out + ((seq * a.S + row / a.group) * (int64_t)(a.heads * a.group) + head * a.group + row % a.group) * DIM;
    return j;
}
__device__ __forceinline__ uint32_t rounded_pair(const Args& a, float x, float y, float total) {
    const float u = total == 0.0f ? 0.0f : x / total, v = total == 0.0f ? 0.0f : y / total;
    if (!a.bf16) return pack_half2(u, v);
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)u) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v) << 16;
}

// Many rows, few pieces each: half a wave a row.  (64 sequences of 8 heads x 8 rows, most of them whole: a block a row took 10.8 us, 6.7 so.)
template <int DIM>
__global__ void __launch_bounds__(256)
attention_join_rows_kernel(Args a, int rows_per_tile, int64_t total_rows) {
    constexpr int kEach = DIM / 32;                        // channels a lane
    const int g = threadIdx.x & 31;
    const int64_t id = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    const JoinRow j = join_row<DIM>(a, min(id, total_rows - 1), rows_per_tile);
    const int used = id >= total_rows || j.used == 1 ? 0 : j.used;         // (half waves differ: loops run for the longer)
    const float* ml = a.partial + a.n_partials * DIM;
    const int most = max(used, __shfl_xor(used, 32, 64));
    auto load = [&](int k) { return k < used ? *reinterpret_cast<const float2*>(ml + j.row_of(k) * 2) : make_float2(-INFINITY, 0.0f); };
    const float2 first = load(g);                          // (m, l) of the first 32 pieces
    float top = first.x;
    for (int k = 32 + g; k < used; k += 32) top = fmaxf(top, load(k).x);
#pragma unroll
    for (int d = 1; d < 32; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float ref = top == -INFINITY ? 0.0f : top;
    float acc[kEach], total = 0.0f;
#pragma unroll
    for (int c = 0; c < kEach; ++c) acc[c] = 0.0f;
    for (int k0 = 0; k0 < most; k0 += 32) {
        const float2 v = k0 == 0 ? first : load(k0 + g);
        const float f = __builtin_amdgcn_exp2f(v.x - ref);
        total = __builtin_fmaf(f, v.y, total);
        for (int k = 0; k < min(32, most - k0); k += 2) {   // two pieces at a time; past the last one that one again, not used
            float o[2][kEach];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float* at = a.partial + j.row_of(max(min(k0 + k + i, used - 1), 0)) * DIM + kEach * g;
                __builtin_memcpy(o[i], at, sizeof(o[i]));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float fk = __shfl(f, k + i, 32);
                if (k0 + k + i >= used) continue;
#pragma unroll
                for (int c = 0; c < kEach; ++c) acc[c] = __builtin_fmaf(fk, o[i][c], acc[c]);
            }
        }
    }
#pragma unroll
    for (int d = 1; d < 32; d *= 2) total += __shfl_xor(total, d, 64);
    if (id >= total_rows || j.used == 1) return;
#pragma unroll
    for (int c = 0; c < kEach; c += 2) *reinterpret_cast<uint32_t*>(j.out + kEach * g + c) = rounded_pair(a, acc[c], acc[c + 1], total);
}

// Few rows, perhaps of many pieces: a block a row, dim / 4 lanes for the channels, the others share the pieces, whose (m, l) the
// threads read side by side (one after the other, 512 pieces cost 100 us).
template <int DIM>
__global__ void __launch_bounds__(256)
attention_join_kernel(Args a, int rows_per_tile) {
    constexpr int kLanes = DIM / 4, kShares = 256 / kLanes;
    __shared__ float4 sh[kShares][kLanes];
    __shared__ float sh_f[256], sh_top[4], sh_l[4];
    const int tid = threadIdx.x;
    const JoinRow j = join_row<DIM>(a, blockIdx.x, rows_per_tile);
    const int used = j.used;
    if (used == 1) return;
    const float* ml = a.partial + a.n_partials * DIM;
    const int share = tid / kLanes, c = tid % kLanes;
    float4 first = make_float4(0.0f, 0.0f, 0.0f, 0.0f);      // (asked for before its factor is known)
    if (share < used) first = *reinterpret_cast<const float4*>(a.partial + j.row_of(share) * DIM + 4 * c);
    float top = -INFINITY;
    for (int k = tid; k < used; k += 256) top = fmaxf(top, ml[j.row_of(k) * 2]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    if ((tid & 63) == 0) sh_top[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(sh_top[0], sh_top[1]), fmaxf(sh_top[2], sh_top[3]));
    const float ref = top == -INFINITY ? 0.0f : top;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float total = 0.0f;
    for (int k0 = 0; k0 < used; k0 += 256) {
        const int n = min(256, used - k0);
        __syncthreads();
        if (tid < n) {
            const float2 v = *reinterpret_cast<const float2*>(ml + j.row_of(k0 + tid) * 2);
            const float f = __builtin_amdgcn_exp2f(v.x - ref);
            sh_f[tid] = f;
            total = __builtin_fmaf(f, v.y, total);
        }
        __syncthreads();
#pragma unroll 4
        for (int k = share; k < n; k += kShares) {
            const float4 v = k0 + k == share ? first : *reinterpret_cast<const float4*>(a.partial + j.row_of(k0 + k) * DIM + 4 * c);
            const float f = sh_f[k];
            acc.x = __builtin_fmaf(f, v.x, acc.x);
            acc.y = __builtin_fmaf(f, v.y, acc.y);
            acc.z = __builtin_fmaf(f, v.z, acc.z);
            acc.w = __builtin_fmaf(f, v.w, acc.w);
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d, 64);
    if ((tid & 63) == 0) sh_l[tid >> 6] = total;
    sh[share][c] = acc;
    __syncthreads();
    if (share != 0) return;
    total = (sh_l[0] + sh_l[1]) + (sh_l[2] + sh_l[3]);
#pragma unroll
    for (int k = 1; k < kShares; ++k) {
        const float4 v = sh[k][c];
        acc.x += v.x;
        acc.y += v.y;
        acc.z += v.z;
        acc.w += v.w;
    }
    *reinterpret_cast<uint2*>(j.out + 4 * c) = make_uint2(rounded_pair(a, acc.x, acc.y, total), rounded_pair(a, acc.z, acc.w, total));
}

// How a call is cut: 16 or 32 rows a block; as many blocks as the chip holds at once (two to four a CU), or a block a pair, which
// needs no second kernel.  A unit that follows another in a block takes some 1 us, the second kernel and finding the stretches 4, so
// a block a pair is for pairs of at most
// - four units: one sequence (8 pairs) of 256 (500) positions 8.4 (10.5) us so, 11.6 (11.7) in stretches, 640 positions 11.4 and 11.8;
// - sixteen where they keep half the CUs busy: of up to 1024 positions, 100 sequences 31 and 40, 200 67 and 77; of up to 2048, 60
//   37 and 40, 100 62 and 68, 400 211 and 224;
// - what each of the chip's places gets of them where that is more still (and never for 2^24 pairs and more, which no launch holds).
// Pairs of more than four units that do not fill the CUs twice have blocks of eight waves, half the steps: 16 sequences of up to 1024
// (2048) positions 14.9 (21.3) us, with four waves 16.9, in stretches 18.8 (24.2); 30: 15.9 (22.7), 17.5, (29.4).  With four units the
// longer way to one result costs as much: 10.7 and 10.5; with more pairs eight waves are in each other's way: 48 of 1024 24.6 and 21.3.
// Lengths are known on the GPU only: longer ones could keep all others waiting (1024 sequences of 4096 positions, INT4, of about one
// length: 578 and 607).
struct Plan {
    int mr, row_tiles, n_blocks;
    int64_t pairs;
    bool wide;                                             // eight waves a block
};
Plan plan(const CacheView& c, const AttentionShape& s) {
    Plan p;
    const int rows = s.S * (s.q_heads / c.heads);
    p.mr = rows > 16 && c.dim < 256 ? 2 : 1;
    p.row_tiles = (rows + 16 * p.mr - 1) / (16 * p.mr);
    p.pairs = s.B * c.heads * p.row_tiles;
    p.n_blocks = p.mr > 1 || c.dim == 256 ? 512 : c.dim == 128 ? 768 : 1024;
    const int64_t longest = (s.max_length + (int64_t)kBlockStep - 1) / kBlockStep;
    if (grid_fits(p.pairs, 64 * kWaves) && longest <= (p.pairs < 128 ? 4 : std::max<int64_t>(16, p.pairs / p.n_blocks))) p.n_blocks = 0;
    p.wide = p.n_blocks == 0 && longest > 4 && p.pairs <= 256;
    return p;
}
int64_t partials(const CacheView& c, const AttentionShape& s, const Plan& p) {
    return (int64_t)2 * p.n_blocks * std::min(16 * p.mr, s.S * (s.q_heads / c.heads));
}

}  // namespace

int64_t cache_attention_workspace(const CacheView& c, const AttentionShape& s) {
    const Plan p = plan(c, s);
    return p.n_blocks ? partials(c, s, p) * (c.dim + 2) * 4 + p.pairs * 8 : 0;
}

hipError_t launch_cache_attention(const CacheView& c, const AttentionShape& s, const uint16_t* Q, int64_t q_batch, int64_t q_token,
                                  int64_t q_head, bool bf16, const int32_t* table, int64_t table_width, const int32_t* lengths,
                                  float scale, uint16_t* out, float* workspace, hipStream_t stream) {
    const Plan p = plan(c, s);
    const int group = s.q_heads / c.heads;
    const int64_t blocks = p.n_blocks ? p.n_blocks : p.pairs, rows = s.B * c.heads * s.S * group, join_blocks = rows >= 1024 ? (rows + 7) / 8 : rows;
    if (!grid_fits(blocks, p.wide ? 64 * 8 : 64 * kWaves) || (p.n_blocks && !grid_fits(join_blocks, 256))) return hipErrorInvalidValue;
    Args a;
    a.Q = Q; a.q_batch = q_batch; a.q_token = q_token; a.q_head = q_head;
    a.k_codes = c.k_codes; a.v_codes = c.v_codes; a.k_scale = c.k_scale; a.v_scale = c.v_scale; a.k_col = c.k_col; a.v_col = c.v_col;
    a.table = table; a.lengths = lengths; a.table_width = table_width; a.pages = c.pages;
    a.out = out; a.partial = workspace; a.n_partials = partials(c, s, p);
    a.heads = c.heads; a.group = group; a.S = s.S; a.row_tiles = p.row_tiles; a.n_blocks = p.n_blocks; a.n_sequences = s.B;
    a.page_shift = c.page_shift; a.max_length = s.max_length; a.scale = scale; a.bf16 = bf16;
    // What the memory-side cache (256 MiB) cannot keep for the next call, beside another layer's, is not put there, as far as values go: a
    // value row is loaded by one instruction, a key row by several.  64 x 1024-8192 133 -> 125 us, 2 x 131072 INT4 64.4 -> 59.8, 100
    // sequences of 2048 62 -> 53, 32 of 4096 (16 heads of 64, 150 MiB) 45 -> 41; two caches of 127 MiB in turn, which stay there, 31.5 -> 33.
    // (keys too: 128 us, 65, 62, 47)
    const int64_t positions = std::min(s.B * (int64_t)s.max_length, c.pages << c.page_shift);
    const bool once = positions * c.heads * 2 * (c.dim * c.bits / 8 + 4) > (int64_t)128 << 20;
    auto go = [&](auto dim, auto bits, auto mr) {
        constexpr int kDim = decltype(dim)::value, kBits = decltype(bits)::value, kMr = decltype(mr)::value;
        if (p.wide) attention_kernel<kDim, kBits, kMr, false, 8><<<(unsigned)blocks, 64 * 8, 0, stream>>>(a);
        else if (once) attention_kernel<kDim, kBits, kMr, true, kWaves><<<(unsigned)blocks, 64 * kWaves, 0, stream>>>(a);
        else attention_kernel<kDim, kBits, kMr, false, kWaves><<<(unsigned)blocks, 64 * kWaves, 0, stream>>>(a);
    };
    auto with_bits = [&](auto bits) {
        using One = std::integral_constant<int, 1>;
        using Two = std::integral_constant<int, 2>;
        if (c.dim == 64) p.mr == 2 ? go(std::integral_constant<int, 64>(), bits, Two()) : go(std::integral_constant<int, 64>(), bits, One());
        else if (c.dim == 128) p.mr == 2 ? go(std::integral_constant<int, 128>(), bits, Two()) : go(std::integral_constant<int, 128>(), bits, One());
        else go(std::integral_constant<int, 256>(), bits, One());
    };
    if (c.bits == 8) with_bits(std::integral_constant<int, 8>());
    else with_bits(std::integral_constant<int, 4>());
    if (hipError_t e = hipGetLastError(); e != hipSuccess || p.n_blocks == 0) return e;
    auto join = [&](auto many, auto few) {
        if (rows >= 1024) many<<<(unsigned)join_blocks, 256, 0, stream>>>(a, 16 * p.mr, rows);
        else few<<<(unsigned)join_blocks, 256, 0, stream>>>(a, 16 * p.mr);
    };
    if (c.dim == 64) join(attention_join_rows_kernel<64>, attention_join_kernel<64>);
    else if (c.dim == 128) join(attention_join_rows_kernel<128>, attention_join_kernel<128>);
    else join(attention_join_rows_kernel<256>, attention_join_kernel<256>);
    return hipGetLastError();
}

}  // namespace cq
