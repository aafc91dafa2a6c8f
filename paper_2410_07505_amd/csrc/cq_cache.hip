// Key/value cache in CrossQuant codes: quantized row by row as it is written, and read back.
//
//   a row is the `dim` channels of one token and head: t = max |x|, a = fl32(t^alpha / q_max), D_j = fl32(a b_j),
//   q_j = D_j == 0 ? 0 : clamp(rne(fl32(x_j / D_j)), +-q_max);  read back: fl32(q_j D_j), rounded to the type asked for
// with the column factors b_j calibrated beforehand.  dim / 8 lanes take a row, 16 bytes of activations a lane.
// Bound by memory for a prompt's worth of rows and by the latency of two dependent reads (slot, row) for a decode step's.
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

// unit = token * heads + head; blockIdx.y = 0 keys, 1 values
template <int DIM, int BITS, bool BF16>
__global__ void __launch_bounds__(256)
cache_write_kernel(Side ks, Side vs, Source k, Source v, const int32_t* __restrict__ slots, int64_t units, int heads,
                   int page_shift, int64_t places, double alpha) {
    constexpr int kLanesPerRow = DIM / 8, kRowBytes = DIM * BITS / 8;
    constexpr float kQmax = BITS == 8 ? 127.0f : 7.0f;
    const Side side = blockIdx.y ? vs : ks;
    const Source in = blockIdx.y ? v : k;
    const int64_t unit = (int64_t)blockIdx.x * (256 / kLanesPerRow) + threadIdx.x / kLanesPerRow;
    if (unit >= units) return;                               // whole rows leave
    const int64_t token = unit / heads;
    const int head = (int)(unit - token * heads), at = (threadIdx.x % kLanesPerRow) * 8;
    const int slot = slots[token];
    const uint4 raw = *reinterpret_cast<const uint4*>(in.x + token * in.token_stride + head * in.head_stride + at);
    float b[8], x[8];
    load_col(side.col, (int64_t)head * DIM + at, b);
    unpack8<BF16>(raw, x);
    const uint32_t m2 = pkmax(pkmax(raw.x & 0x7FFF7FFFu, raw.y & 0x7FFF7FFFu), pkmax(raw.z & 0x7FFF7FFFu, raw.w & 0x7FFF7FFFu));
    const uint32_t m = max_lanes<kLanesPerRow>(max(m2 & 0xFFFFu, m2 >> 16));
    if (slot < 0 || slot >= places) return;
    const float a = row_factor(BF16 ? __uint_as_float(m << 16) : h2f(m), alpha, (int)kQmax);
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float step = a * b[e];
        const float r = step == 0.0f ? 0.0f : __builtin_rintf(x[e] / step);
        q[e] = (uint32_t)(int)fminf(fmaxf(r, -kQmax), kQmax);
    }
    const int64_t row = (((int64_t)(slot >> page_shift) * heads + head) << page_shift) + (slot & ((1 << page_shift) - 1));
    uint8_t* dst = side.codes + row * kRowBytes + at * BITS / 8;
    if (BITS == 8) {
        *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bytes(q[0], q[1], q[2], q[3]), pack_bytes(q[4], q[5], q[6], q[7]));
    } else {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w |= (q[e] & 15u) << (4 * e);
        *reinterpret_cast<uint32_t*>(dst) = w;
    }
    if (at == 0) side.scale[row] = a;
}

template <int DIM, int BITS, bool BF16>
__global__ void __launch_bounds__(256)
cache_read_kernel(Side ks, Side vs, const int32_t* __restrict__ slots, int64_t units, int heads, int page_shift, int64_t places,
                  uint16_t* __restrict__ K, uint16_t* __restrict__ V) {
    constexpr int kLanesPerRow = DIM / 8, kRowBytes = DIM * BITS / 8;
    const Side side = blockIdx.y ? vs : ks;
    const int64_t unit = (int64_t)blockIdx.x * (256 / kLanesPerRow) + threadIdx.x / kLanesPerRow;
    if (unit >= units) return;
    const int64_t token = unit / heads;
    const int head = (int)(unit - token * heads), at = (threadIdx.x % kLanesPerRow) * 8;
    const int slot = slots[token];
    uint4 out = make_uint4(0u, 0u, 0u, 0u);
    if (slot >= 0 && slot < places) {
        const int64_t row = (((int64_t)(slot >> page_shift) * heads + head) << page_shift) + (slot & ((1 << page_shift) - 1));
        const uint8_t* src = side.codes + row * kRowBytes + at * BITS / 8;
        int q[8];
        if (BITS == 8) {
            const uint2 c = *reinterpret_cast<const uint2*>(src);
#pragma unroll
            for (int e = 0; e < 8; ++e) q[e] = (int8_t)((e < 4 ? c.x : c.y) >> (8 * (e & 3)));
        } else {
            const uint32_t c = *reinterpret_cast<const uint32_t*>(src);
#pragma unroll
            for (int e = 0; e < 8; ++e) q[e] = (int)(c << (28 - 4 * e)) >> 28;
        }
        const float a = side.scale[row];
        float b[8];
        load_col(side.col, (int64_t)head * DIM + at, b);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = rounded_f32((float)q[2 * i] * rounded_f32(a * b[2 * i]));
            const float hi = rounded_f32((float)q[2 * i + 1] * rounded_f32(a * b[2 * i + 1]));
            if (BF16) {
                typedef float f32x2 __attribute__((ext_vector_type(2)));
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
            } else {
                w[i] = pack_half2(lo, hi);
            }
        }
        out = make_uint4(w[0], w[1], w[2], w[3]);
    }
    *reinterpret_cast<uint4*>((blockIdx.y ? V : K) + unit * DIM + at) = out;
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

}  // namespace

hipError_t launch_cache_write(const CacheView& c, const uint16_t* K, int64_t k_token, int64_t k_head, const uint16_t* V,
                              int64_t v_token, int64_t v_head, bool bf16, const int32_t* slots, int T, hipStream_t stream) {
    const int64_t units = (int64_t)T * c.heads, per_block = 256 / (c.dim / 8), blocks = (units + per_block - 1) / per_block;
    if (!grid_fits(2 * blocks, 256)) return hipErrorInvalidValue;
    return dispatch(c, bf16, [&](auto dim, auto bits, auto bf) {
        cache_write_kernel<dim(), bits(), bf()><<<dim3((unsigned)blocks, 2), 256, 0, stream>>>(
            side_k(c), side_v(c), Source{K, k_token, k_head}, Source{V, v_token, v_head}, slots, units, c.heads, c.page_shift,
            c.pages << c.page_shift, c.alpha);
    });
}

hipError_t launch_cache_read(const CacheView& c, const int32_t* slots, int T, uint16_t* K, uint16_t* V, bool bf16,
                             hipStream_t stream) {
    const int64_t units = (int64_t)T * c.heads, per_block = 256 / (c.dim / 8), blocks = (units + per_block - 1) / per_block;
    if (!grid_fits(2 * blocks, 256)) return hipErrorInvalidValue;
    return dispatch(c, bf16, [&](auto dim, auto bits, auto bf) {
        cache_read_kernel<dim(), bits(), bf()><<<dim3((unsigned)blocks, 2), 256, 0, stream>>>(
            side_k(c), side_v(c), slots, units, c.heads, c.page_shift, c.pages << c.page_shift, K, V);
    });
}

}  // namespace cq
