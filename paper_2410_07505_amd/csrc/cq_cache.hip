// Key/value cache in CrossQuant codes: quantized row by row as it is written, and read back.
//
//   a row is the `dim` channels of one token and head: t = max |x|, a = fl32(t^alpha / q_max), D_j = fl32(a b_j),
//   q_j = D_j == 0 ? 0 : clamp(rne(fl32(x_j / D_j)), +-q_max);  read back: fl32(q_j D_j), rounded to the type asked for;
//   a = NaN for a row that holds an infinity or NaN
// with the column factors b_j calibrated beforehand.  dim / 8 lanes take a row, 16 bytes of activations a lane.
// For a prompt's worth of rows the read is bound by memory and the write by its vector instructions (16384 tokens of 2 x 8 heads, INT4: 47 of
// the 49 thousand cycles that a CU is busy, 3.2 TB/s); for a decode step's both by the latency of two dependent reads (slot, row).
#include "cq_device.h"

namespace cq {
namespace {

// maximum over the N lanes (8, 16 or 32, aligned) that share a row, in all of them
template <int N>
__device__ __forceinline__ uint32_t max_lanes(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));     // lane ^ 1
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));     // lane ^ 2
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xF, 0xF, true));    // mirrored in 8 lanes
    if (N >= 16) m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xF, 0xF, true));   // mirrored in 16
    if (N >= 32) m = max(m, shx(m, 16));
    return m;
}

template <bool BF16>
__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = BF16 ? __uint_as_float(w[i] << 16) : h2f(w[i] & 0xFFFFu);
        f[2 * i + 1] = BF16 ? __uint_as_float(w[i] & 0xFFFF0000u) : h2f(w[i] >> 16);
    }
}

__device__ __forceinline__ void load_col(const float* __restrict__ col, int64_t at, float (&b)[8]) {
    const float4 lo = col ? *reinterpret_cast<const float4*>(col + at) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
    const float4 hi = col ? *reinterpret_cast<const float4*>(col + at + 4) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
    b[0] = lo.x; b[1] = lo.y; b[2] = lo.z; b[3] = lo.w;
    b[4] = hi.x; b[5] = hi.y; b[6] = hi.z; b[7] = hi.w;
}

struct Side {
    uint8_t* codes;
    float* scale;
    const float* col;
};
struct Source {
    const uint16_t* x;
    int64_t token_stride, head_stride;
};

// a factor whose reciprocal, and whose products with another one, are normal numbers
__device__ __forceinline__ bool plain_factor(float f) { return (f >= kTinyFactor) & (f <= 1.0f / kTinyFactor); }

// q_e = clamp(rne(fl32(x_e / fl32(a b_e))), +-QMAX), a NaN to -QMAX, as whole numbers in the low bits.
// The same by a multiplication: x (1/a)(1/b) is within 2^-20 of the quotient (two reciprocals of 1 ulp, four roundings), so its
// nearest integer is the quotient's too unless it is that close to a tie (a quotient beyond QMAX + 1/4 is taken as that); a wave with
// an element within 2^-19 (|q| + 1) of one, or with a factor so small or large that a product could leave the normal range or no
// number in a row (!plain), divides.  (2048 tokens of 2 x 8 heads, INT4: 7.1 us with all eight divided, 6.3 so)
template <int QMAX>
__device__ __forceinline__ void row_codes(const float (&x)[8], float a, const float (&b)[8], const float (&rb)[8], bool plain,
                                          uint32_t (&q)[8]) {
    constexpr float kMax = (float)QMAX;
    const float ra = safe_rcp(a);
    float score = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_fmed3f(x[e] * (ra * rb[e]), -kMax - 0.25f, kMax + 0.25f);
        const float m = p + kMagic, n = m - kMagic;
        score = __builtin_fmaxf(score, __builtin_fmaf(__builtin_fabsf(n), kTieTol, __builtin_fabsf(p - n)));
        q[e] = __float_as_uint(m);                                   // (1.5 * 2^23 + n holds n in its low bits)
    }
    if (__any(!plain | !((a == 0.0f) | plain_factor(a)) | (score >= 0.5f - kTieTol))) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float step = a * b[e];
            const float r = step == 0.0f ? 0.0f : __builtin_rintf(x[e] / step);
            q[e] = (uint32_t)(int)fminf(fmaxf(r, -kMax), kMax);
        }
    }
}

// A block takes a stretch of R * kRows tokens of one head (blockIdx.x = stretch * heads + head; blockIdx.y = 0 keys, 1 values), so
// that consecutive slots fill whole lines of codes and scales, and the head's column factors serve all its rows: a thread's R rows
// are kRows tokens apart.  The powers in the rows' factors, in binary64 as long as the rest of a row, are formed by R of a row's
// lanes at once and handed to the others.
template <int DIM, int BITS, bool BF16, int R>
__global__ void __launch_bounds__(256)
cache_write_kernel(Side ks, Side vs, Source k, Source v, const int32_t* __restrict__ slots, int T, int heads, int page_shift,
                   int64_t places, double alpha) {
    constexpr int kLanesPerRow = DIM / 8, kRowBytes = DIM * BITS / 8, kRows = 256 / kLanesPerRow, kQmax = BITS == 8 ? 127 : 7;
    static_assert(R <= kLanesPerRow, "a lane a row");
    const Side side = blockIdx.y ? vs : ks;
    const Source in = blockIdx.y ? v : k;
    const int stretch = blockIdx.x / (uint32_t)heads, head = blockIdx.x - stretch * heads;
    const int mine = threadIdx.x % kLanesPerRow, at = mine * 8;
    const uint32_t first = (uint32_t)stretch * (R * kRows) + threadIdx.x / kLanesPerRow;
    int slot[R];
    uint4 raw[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const uint32_t token = first + i * kRows, t = min(token, (uint32_t)T - 1);
        slot[i] = slots[t];
        if (token >= (uint32_t)T || slot[i] >= places) slot[i] = -1;
        raw[i] = *reinterpret_cast<const uint4*>(in.x + (int64_t)t * in.token_stride + (int64_t)head * in.head_stride + at);
    }
    float b[8], rb[8];
    load_col(side.col, (int64_t)head * DIM + at, b);
    bool plain = true;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        rb[e] = safe_rcp(b[e]);
        plain = plain & ((b[e] == 0.0f) | plain_factor(__builtin_fabsf(b[e])));
    }
    uint32_t m_mine = 0, m_any = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const uint4& w = raw[i];
        const uint32_t m2 = pkmax(pkmax(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu), pkmax(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu));
        const uint32_t m = max_lanes<kLanesPerRow>(max(m2 & 0xFFFFu, m2 >> 16));
        m_any = max(m_any, m);
        if (R == 1 || mine == i) m_mine = m;
    }
    constexpr uint32_t kInfinity = BF16 ? 0x7F80u : 0x7C00u;
    plain = plain & (m_any < kInfinity);
    // (an infinite factor would let a score of one sign drop out of the softmax as if the position were not there)
    const float a_mine = m_mine < kInfinity ? row_factor(BF16 ? __uint_as_float(m_mine << 16) : h2f(m_mine), alpha, kQmax) : __builtin_nanf("");
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const float a = R == 1 ? a_mine : __shfl(a_mine, i, kLanesPerRow);
        if (slot[i] < 0) continue;
        float x[8];
        unpack8<BF16>(raw[i], x);
        uint32_t q[8];
        row_codes<kQmax>(x, a, b, rb, plain, q);
        const int64_t row = (((int64_t)(slot[i] >> page_shift) * heads + head) << page_shift) + (slot[i] & ((1 << page_shift) - 1));
        uint8_t* dst = side.codes + row * kRowBytes + at * BITS / 8;
        if (BITS == 8) {
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bytes(q[0], q[1], q[2], q[3]), pack_bytes(q[4], q[5], q[6], q[7]));
        } else {
            uint32_t c = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) c |= (q[e] & 15u) << (4 * e);
            *reinterpret_cast<uint32_t*>(dst) = c;
        }
        if (mine == 0) side.scale[row] = a;
    }
}

// R rows a thread, for whose slots, codes and scales it waits once.
template <int DIM, int BITS, bool BF16, int R>
__global__ void __launch_bounds__(256)
cache_read_kernel(Side ks, Side vs, const int32_t* __restrict__ slots, int T, int heads, int page_shift, int64_t places,
                  uint16_t* __restrict__ K, uint16_t* __restrict__ V) {
    constexpr int kLanesPerRow = DIM / 8, kRowBytes = DIM * BITS / 8, kRows = 256 / kLanesPerRow, kWords = BITS / 4;
    const Side side = blockIdx.y ? vs : ks;
    const int stretch = blockIdx.x / (uint32_t)heads, head = blockIdx.x - stretch * heads, at = (threadIdx.x % kLanesPerRow) * 8;
    const uint32_t first = (uint32_t)stretch * (R * kRows) + threadIdx.x / kLanesPerRow;
    int slot[R];
#pragma unroll
    for (int i = 0; i < R; ++i) slot[i] = slots[min(first + i * kRows, (uint32_t)T - 1)];
    uint32_t c[R][kWords];
    float a[R], b[8];
    load_col(side.col, (int64_t)head * DIM + at, b);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const bool live = slot[i] >= 0 && slot[i] < places;
        if (!live) slot[i] = -1;
        const int s = live ? slot[i] : 0;
        const int64_t row = (((int64_t)(s >> page_shift) * heads + head) << page_shift) + (s & ((1 << page_shift) - 1));
        __builtin_memcpy(c[i], __builtin_assume_aligned(side.codes + row * kRowBytes + at * BITS / 8, BITS), BITS);
        a[i] = side.scale[row];
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const uint32_t token = first + i * kRows;
        if (token >= (uint32_t)T) return;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float x[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int q = BITS == 8 ? (int)(int8_t)(c[i][(e + h) / 4 % kWords] >> (8 * ((e + h) & 3))) : (int)(c[i][0] << (28 - 4 * (e + h))) >> 28;
                x[h] = rounded_f32((float)q * rounded_f32(a[i] * b[e + h]));
            }
            if (BF16) {
                typedef float f32x2 __attribute__((ext_vector_type(2)));
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                w[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[0], x[1]}, bf16x2));
            } else {
                w[e / 2] = pack_half2(x[0], x[1]);
            }
        }
        const bool live = slot[i] >= 0;                      // the others' rows are zero
        *reinterpret_cast<uint4*>((blockIdx.y ? V : K) + ((int64_t)token * heads + head) * DIM + at) =
            live ? make_uint4(w[0], w[1], w[2], w[3]) : make_uint4(0u, 0u, 0u, 0u);
    }
}

Side side_k(const CacheView& c) { return {c.k_codes, c.k_scale, c.k_col}; }
Side side_v(const CacheView& c) { return {c.v_codes, c.v_scale, c.v_col}; }

// calls f(dim, bits, bf16) with the three as compile-time constants
template <typename F>
hipError_t dispatch(const CacheView& c, bool bf16, F f) {
    auto with_type = [&](auto dim, auto bits) {
        if (bf16) f(dim, bits, std::true_type());
        else f(dim, bits, std::false_type());
    };
    auto with_bits = [&](auto dim) {
        if (c.bits == 8) with_type(dim, std::integral_constant<int, 8>());
        else with_type(dim, std::integral_constant<int, 4>());
    };
    if (c.dim == 64) with_bits(std::integral_constant<int, 64>());
    else if (c.dim == 128) with_bits(std::integral_constant<int, 128>());
    else with_bits(std::integral_constant<int, 256>());
    return hipGetLastError();
}

// Rows a thread takes, and blocks for the keys of T tokens: `many` rows where that leaves `least` blocks, else one.  Several share a
// head's factors, a wait and, in the write, one power: INT4, 2 x 8 heads of 128, 16384 tokens are written in 24.5 us with eight, 27.6
// with four and 31.7 with one, and read in 14.9 with four (5.7 TB/s), 14.6 with eight and 16.5 with one (INT8, 8192 tokens: 9.4, 10.2
// and 10.3).  With fewer blocks one row a thread hides more of the latency (64 tokens, written: 3.0 us with one, 5.8 with four;
// from 2048 to 4096 tokens all are within 3 %).
struct Stretches {
    int rows;
    int64_t blocks;
};
Stretches stretches(const CacheView& c, int T, int many, int64_t least) {
    const int64_t kept = 256 / (c.dim / 8), blocks = (T + many * kept - 1) / (many * kept) * c.heads;
    if (blocks >= least) return {many, blocks};
    return {1, (T + kept - 1) / kept * c.heads};
}

}  // namespace

hipError_t launch_cache_write(const CacheView& c, const uint16_t* K, int64_t k_token, int64_t k_head, const uint16_t* V,
                              int64_t v_token, int64_t v_head, bool bf16, const int32_t* slots, int T, hipStream_t stream) {
    const Stretches g = stretches(c, T, 8, 512);
    if (!grid_fits(2 * g.blocks, 256)) return hipErrorInvalidValue;
    return dispatch(c, bf16, [&](auto dim, auto bits, auto bf) {
        auto go = [&](auto kernel) {
            kernel<<<dim3((unsigned)g.blocks, 2), 256, 0, stream>>>(side_k(c), side_v(c), Source{K, k_token, k_head}, Source{V, v_token, v_head},
                                                                    slots, T, c.heads, c.page_shift, c.pages << c.page_shift, c.alpha);
        };
        if (g.rows == 8) go(cache_write_kernel<dim(), bits(), bf(), 8>);
        else go(cache_write_kernel<dim(), bits(), bf(), 1>);
    });
}

hipError_t launch_cache_read(const CacheView& c, const int32_t* slots, int T, uint16_t* K, uint16_t* V, bool bf16,
                             hipStream_t stream) {
    const Stretches g = stretches(c, T, 4, 1024);
    if (!grid_fits(2 * g.blocks, 256)) return hipErrorInvalidValue;
    return dispatch(c, bf16, [&](auto dim, auto bits, auto bf) {
        auto go = [&](auto kernel) {
            kernel<<<dim3((unsigned)g.blocks, 2), 256, 0, stream>>>(side_k(c), side_v(c), slots, T, c.heads, c.page_shift,
                                                                    c.pages << c.page_shift, K, V);
        };
        if (g.rows == 4) go(cache_read_kernel<dim(), bits(), bf(), 4>);
        else go(cache_read_kernel<dim(), bits(), bf(), 1>);
    });
}

}  // namespace cq
