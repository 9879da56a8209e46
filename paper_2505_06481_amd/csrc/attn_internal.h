// Internal declarations of the attention half: projections with adapters, rotary positions, paged cache, attention.
#pragma once

#include <utility>

#include "mmoe_internal.h"

namespace mmoe {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

constexpr int kPage = MMOE_PAGE_TOKENS;
constexpr int kMaxAdapters = 1024;
constexpr int kMaxRank = 128;
constexpr int64_t kMaxRow = (int64_t)1 << 20;  // row strides of a projection: a tile's rows are addressed with 32 bits

// f(0) .. f(N - 1) with the numbers as constants: register arrays are indexed statically whatever the loop's size.
template <typename F, int... I>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F&& f)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f)
{
    each(std::make_integer_sequence<int, N>{}, f);
}

// Matrix products on 16-byte operand pieces.  Lane 16 g + r of a wavefront holds, of row r of the operand, the
// 16 bytes of group g: 8 bf16 of the 32 k of v_mfma_f32_16x16x32_bf16, or 4 fp32 of 16 k, which four
// v_mfma_f32_16x16x4f32 take one each (lane group g then brings k = 4 g + e to instruction e, in both operands).  The result's
// element e of lane 16 g + r is row 4 g + e, column r.
template <bool F32>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (F32) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
        return c;
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return (uint32_t)f32_to_bf16_bits(lo) | ((uint32_t)f32_to_bf16_bits(hi) << 16);
}
__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }

int check_project(const mmoe_project_shape* s);
int check_rotary(const mmoe_rotary_shape* s);
int check_cache(const mmoe_cache_shape* s);
int check_attend(const mmoe_attend_shape* s);

inline int padded_rank(const mmoe_project_shape& s)
{
    const int q = s.dtype == MMOE_BF16 ? 32 : 16;
    return (s.rank + q - 1) / q * q;
}
size_t project_need(const mmoe_project_shape& s);
size_t project_ws_bytes(const mmoe_project_shape& s);
int launch_pack_pieces(const void* in, void* out, int S, int K, int N, int Kp, int Np, int dtype, hipStream_t st);
int launch_project(const mmoe_project_shape& s, const void* X, const int32_t* aid, const void* Wp, const void* Ap,
                   const void* Bp, const float* scale, void* Y, void* ws, hipStream_t st);

int launch_rotary(const mmoe_rotary_shape& s, const void* X, const int32_t* pos, const uint64_t* steps, void* Y, hipStream_t st);
int launch_cache_append(const mmoe_cache_shape& s, const mmoe_cache_rows& rows, const void* K, const void* V,
                        const int32_t* places, const mmoe_rotary_shape* rotary, const int32_t* pos, const uint64_t* steps,
                        const mmoe_cache& cache, hipStream_t st);
int launch_cache_read(const mmoe_cache_shape& s, const mmoe_cache& cache, int R, const int32_t* places, void* K, void* V,
                      hipStream_t st);

bool attend_fits(const mmoe_attend_shape& s);
size_t attend_need(const mmoe_attend_shape& s);
size_t attend_ws_bytes(const mmoe_attend_shape& s);
int launch_attend(const mmoe_attend_shape& s, const void* Q, const int32_t* starts, const int32_t* ctx, const uint64_t* tree,
                  const int32_t* pages, const mmoe_cache& cache, void* out, float* lse, void* ws, hipStream_t st);

}  // namespace mmoe
