// FP8 (e4m3) codes with a binary32 scale for every block of 128: the operands of crossquant_fp8_linear.
//
//   activations: a group is 128 consecutive channels of one token; weights: a block is 128 input x 128 output channels.
//   m = max |x| of the group;  m < 2^-100: s = r = 0, else s = fl32(m / 448), r = fl32(448 / m)
//   code = e4m3(fl32(x r))
// Two divisions for a group and one product for an element; 448 (1 + 2^-23) still rounds to 448, so no code needs clamping.
// Below 2^-100 r would leave binary32: such a group (bfloat16 reaches it) counts as zero.
// m is a maximum of the bit patterns without sign, which order like the magnitudes with infinities and NaN above all numbers: a
// group that holds one gets a scale that is not finite, and so shows in the outputs of its token.
// Bound by memory: 2 bytes read and 1 written per element.
#include "cq_device.h"

namespace cq {
namespace {

constexpr int kGroup = 128;
constexpr float kFp8Max = 448.0f;
constexpr float kSmallest = 7.888609052210118e-31f;      // 2^-100

template <bool BF16>
__device__ __forceinline__ float lo_f(uint32_t w) { return BF16 ? __uint_as_float(w << 16) : h2f(w & 0xFFFFu); }
template <bool BF16>
__device__ __forceinline__ float hi_f(uint32_t w) { return BF16 ? __uint_as_float(w & 0xFFFF0000u) : h2f(w >> 16); }
// magnitude pattern -> binary32
template <bool BF16>
__device__ __forceinline__ float magnitude(uint32_t m) { return BF16 ? __uint_as_float(m << 16) : h2f(m); }

__device__ __forceinline__ uint32_t absmax8(const uint4& v) {
    const uint32_t a = pkmax(pkmax(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), pkmax(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
    return max(a & 0xFFFFu, a >> 16);
}

// maximum over the 16 lanes of a row of lanes, in all of them
__device__ __forceinline__ uint32_t max16(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x128, 0xF, 0xF, true));    // row_ror 8
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x124, 0xF, 0xF, true));
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x122, 0xF, 0xF, true));
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x121, 0xF, 0xF, true));
    return m;
}

struct Scale {
    float s, r;
};
__device__ __forceinline__ Scale scale_of(float m) {
    if (m < kSmallest) return {0.0f, 0.0f};
    return {m / kFp8Max, kFp8Max / m};
}

__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// A wave takes 512 columns (four groups, 16 lanes each: one 16-byte load a lane and row) of R tokens.  The R scales of a group
// are neighbours in the output ([group][token]).
// VEC: X 16-byte aligned, ldx % 8 == 0, I % 8 == 0.  Other layouts load unaligned, and nothing outside a row.
template <bool BF16, bool VEC, int R>
__global__ void __launch_bounds__(256)
quantize_fp8_kernel(const uint16_t* __restrict__ X, int T, int I, int64_t ldx, int n_chunks, uint8_t* __restrict__ codes,
                    float* __restrict__ scale) {
    const int lane = threadIdx.x & 63;
    const int unit = (int)(blockIdx.x * 4 + (threadIdx.x >> 6));          // below 2^26: a launch has fewer than 2^32 threads
    const int chunk = unit % n_chunks, t0 = unit / n_chunks * R;
    const int j = chunk * 512 + lane * 8, Ip = (I + kGroup - 1) / kGroup * kGroup;
    if (t0 >= T || j >= Ip) return;                          // whole groups leave: 16 lanes share j / 128
    uint4 v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = load8<VEC>(X + (int64_t)min(t0 + r, T - 1) * ldx, j, I);
    float mine = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const Scale sc = scale_of(magnitude<BF16>(max16(absmax8(v[r]))));
        if ((lane & 15) == r) mine = sc.s;
        if (t0 + r < T) {
            const uint2 q = make_uint2(four_codes(lo_f<BF16>(v[r].x) * sc.r, hi_f<BF16>(v[r].x) * sc.r, lo_f<BF16>(v[r].y) * sc.r,
                                                  hi_f<BF16>(v[r].y) * sc.r),
                                       four_codes(lo_f<BF16>(v[r].z) * sc.r, hi_f<BF16>(v[r].z) * sc.r, lo_f<BF16>(v[r].w) * sc.r,
                                                  hi_f<BF16>(v[r].w) * sc.r));
            *reinterpret_cast<uint2*>(codes + (int64_t)(t0 + r) * Ip + j) = q;
        }
    }
    const int row = lane & 15;
    if (row < R && t0 + row < T) scale[(int64_t)(j / kGroup) * T + t0 + row] = mine;
}

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// One block of 256 threads for one 128 x 128 block of W [I][O]; the codes leave transposed, [O][Ip].
// A thread holds 8 rows x 8 columns, 16 lanes the 128 columns of the same rows: a load is 256 adjacent bytes of four rows.  The codes of a
// column's 8 rows, 8 bytes, pass through LDS ([column][16 chunks], chunk q of column group g at q ^ g, which spreads writes and reads over
// the banks), so that a column's 128 leave as a whole line, 16 bytes a lane, and past the caches: a weight is prepared long before it is
// used.  (4096 x 11008, 8192 x 28672, 4096 x 4096, 2750 x 4090: rows of 64 bytes loaded and 8 bytes a lane stored, without LDS 34.9,
// 147, 10.8 and 10.5 us; through LDS 32.8, 138, 11.1 and 10.9; past the caches too 25.6, 131, 9.3 and 9.8, 5.3 TB/s.)
template <bool BF16, bool VEC>
__global__ void __launch_bounds__(256)
weight_fp8_kernel(const uint16_t* __restrict__ W, int I, int O, int nb, uint8_t* __restrict__ qw, float* __restrict__ w_scale) {
    __shared__ uint32_t part[4];
    __shared__ __align__(16) uint2 tile[kGroup][16];
    const int b = blockIdx.x % nb, ob = blockIdx.x / nb;
    const int g = threadIdx.x & 15, q = threadIdx.x >> 4;
    const int i0 = b * kGroup + 8 * q, o0 = ob * kGroup + 8 * g;
    const int64_t Ip = (int64_t)nb * kGroup;
    uint4 v[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        v[r] = make_uint4(0u, 0u, 0u, 0u);
        if (i0 + r < I && o0 < O) v[r] = load8<VEC>(W + (int64_t)(i0 + r) * O, o0, O);
    }
    uint32_t m = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) m = max(m, absmax8(v[r]));
    m = max16(m);
    m = max(m, shx(m, 16));
    m = max(m, shx(m, 32));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    const Scale sc = scale_of(magnitude<BF16>(max(max(part[0], part[1]), max(part[2], part[3]))));
    if (threadIdx.x == 0) w_scale[(int64_t)ob * nb + b] = sc.s;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        float f[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const uint32_t w = c < 2 ? v[r].x : c < 4 ? v[r].y : c < 6 ? v[r].z : v[r].w;
            f[r] = (c & 1 ? hi_f<BF16>(w) : lo_f<BF16>(w)) * sc.r;
        }
        tile[8 * g + c][q ^ g] = make_uint2(four_codes(f[0], f[1], f[2], f[3]), four_codes(f[4], f[5], f[6], f[7]));
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int col = 32 * c + (threadIdx.x >> 3), o = ob * kGroup + col, h = 2 * (threadIdx.x & 7);
        const uint2 x = tile[col][h ^ (col >> 3)], y = tile[col][(h + 1) ^ (col >> 3)];
        if (o < O) __builtin_nontemporal_store(v4u{x.x, x.y, y.x, y.y}, reinterpret_cast<v4u*>(qw + (int64_t)o * Ip + b * kGroup + 8 * h));
    }
}

}  // namespace

hipError_t launch_quantize_fp8(const uint16_t* X, bool bf16, int T, int I, int64_t ldx, uint8_t* codes, float* scale,
                               hipStream_t stream) {
    const int n_chunks = (I + 511) / 512;
    const bool vec = reinterpret_cast<uintptr_t>(X) % 16 == 0 && ldx % 8 == 0 && I % 8 == 0;
    // (two rows a wave where there are more than 16 waves a SIMD: 4096 x 8192 19.3 us, with one 21.3, eight 21.5; 16384 x 8192 70.5, 73.8,
    // 78.7; 2048 x 4096, which has 16, 6.4 with two and 6.2 with one)
    const int rows = (int64_t)n_chunks * T > 16384 ? 2 : 1;
    const int64_t blocks = ((int64_t)n_chunks * ((T + rows - 1) / rows) + 3) / 4;
    if (!grid_fits(blocks, 256)) return hipErrorInvalidValue;
    auto go = [&](auto kernel) { kernel<<<(unsigned)blocks, 256, 0, stream>>>(X, T, I, ldx, n_chunks, codes, scale); };
    if (rows == 2) {
        if (bf16) vec ? go(quantize_fp8_kernel<true, true, 2>) : go(quantize_fp8_kernel<true, false, 2>);
        else vec ? go(quantize_fp8_kernel<false, true, 2>) : go(quantize_fp8_kernel<false, false, 2>);
    } else {
        if (bf16) vec ? go(quantize_fp8_kernel<true, true, 1>) : go(quantize_fp8_kernel<true, false, 1>);
        else vec ? go(quantize_fp8_kernel<false, true, 1>) : go(quantize_fp8_kernel<false, false, 1>);
    }
    return hipGetLastError();
}

hipError_t launch_weight_quantize_fp8(const uint16_t* W, bool bf16, int I, int O, uint8_t* qw, float* w_scale, hipStream_t stream) {
    const int nb = (I + kGroup - 1) / kGroup, ob = (O + kGroup - 1) / kGroup;
    const bool vec = reinterpret_cast<uintptr_t>(W) % 16 == 0 && O % 8 == 0;
    const int64_t blocks = (int64_t)nb * ob;
    if (!grid_fits(blocks, 256)) return hipErrorInvalidValue;
    auto go = [&](auto kernel) { kernel<<<(unsigned)blocks, 256, 0, stream>>>(W, I, O, nb, qw, w_scale); };
    if (bf16) vec ? go(weight_fp8_kernel<true, true>) : go(weight_fp8_kernel<true, false>);
    else vec ? go(weight_fp8_kernel<false, true>) : go(weight_fp8_kernel<false, false>);
    return hipGetLastError();
}

}  // namespace cq
