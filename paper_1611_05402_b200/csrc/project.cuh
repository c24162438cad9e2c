// What the kernels behind zipml_checkpoint_* and zipml_project* share: 16-bit loads, the pieces of a token tile, and the
// argument blocks of the three stages (reduction of the tokens onto the adapters' ranks, the projection, the gradients).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sgd_common.cuh"

namespace zipml {

constexpr int kMaxRank = 128;
constexpr int kShrinkRows = 16;                 // tokens of a shrink tile: one row block of the 16-bit matrix instruction
constexpr int kNoRequest = -2;                  // adapter index of a token that belongs to no request; -1: to one without an adapter

// The dense floating types of activations and adapters.
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// The two values of a 32-bit word of 16-bit ones.
template <typename T> __device__ __forceinline__ float2 unpack_pair(uint32_t w);
template <> __device__ __forceinline__ float2 unpack_pair<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack_pair<__half>(uint32_t w) {
    __half2 h;
    *reinterpret_cast<uint32_t*>(&h) = w;
    return __half22float2(h);
}
template <typename T> __device__ __forceinline__ uint32_t pack_pair(float a, float b);
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Two values as the sum of two pairs, the rounded values and the rounded rest of them: twice the type's bits.
template <typename T> __device__ __forceinline__ void split_pair(float a, float b, uint32_t& high, uint32_t& low) {
    high = pack_pair<T>(a, b);
    const float2 f = unpack_pair<T>(high);
    low = pack_pair<T>(a - f.x, b - f.y);
}

// Eight 16-bit values from p on, the first `count` of them (0 .. 8) there, the rest zero.  `wide`: p is 16-byte aligned.
__device__ __forceinline__ uint4 load8_16(const void* p, int count, bool wide) {
    if (wide && count >= 8) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0, 0, 0, 0};
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) w[i >> 1] |= (uint32_t)h[i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The same for a number of a row that scale_to_range has scaled: the high part a multiple of 2^5, 9 bits, the low one the rest in fp16's 11.  Codes
// have 8 bits, so the high parts' products are multiples of 2^5 below 2^21, and fp32 holds their sums exactly up to 2^29.
__device__ __forceinline__ void split_scaled(float a, float b, uint32_t& high, uint32_t& low) {
    constexpr float kMagic = 1.5f * (float)(1 << 28);                     // (numbers around it are 2^5 apart)
    const float x = __fsub_rn(__fadd_rn(a, kMagic), kMagic), y = __fsub_rn(__fadd_rn(b, kMagic), kMagic);
    high = pack_pair<__half>(x, y);
    low = pack_pair<__half>(a - x, b - y);
}

// Power of two that brings a value of magnitude `top` into [2^13, 2^14); 1 for zero and what is not finite.
__device__ __forceinline__ float scale_to_range(float top) {
    if (!(top > 0.0f) || !(top <= 3.402823466e38f)) return 1.0f;
    const int e = max((int)(__float_as_uint(top) >> 23), 1) - 127;        // (subnormal tops count as 2^-126)
    return __uint_as_float((uint32_t)(min(max(13 - e, -126), 126) + 127) << 23);
}

// Stage 1, over tokens x `columns` values z (the forward pass's inputs, the backward pass's output gradients):
//   hidden[t] = scale_i * (D_i z_t)   D_i: rank x columns, the adapter of token t
//   forward:  sum[t] = sum_j z_tj
//   backward: sum[t] = sum_j z_tj (lo_j + center step_j), scaled[t][j] + scaled[tokens + t][j] = z_tj step_j * 2^k with 2^-k in row_scale[t],
//             as split_scaled makes them
struct ShrinkArgs {
    const void* z;
    int64_t tokens, ldz;
    int columns;
    const void* down;            // adapters x rank x columns, or null
    const float* scale;          // per adapter, or null
    const int32_t *starts, *which;
    int requests, adapters, rank;
    float* hidden;               // tokens x rank
    int* ids;                    // adapter index of each token
    float *sum, *row_scale, *hidden_scale;
    const float *lo, *step;      // backward
    float center;
    __half* scaled;              // backward: 2 tokens x ld_scaled, the products' high parts and then their low ones
    int64_t ld_scaled;
    void* copy;                  // forward: z once more in rows that tensor copies can take, or null
    int64_t ld_copy;
    DeviceStatus* status;
};

// Stage 2: out[t][f] = alpha_f row_scale_t (codes_f - center) . u_t + beta_f sum_t + up_i[:, f] . hidden_t
struct ProjectArgs {
    int64_t tokens;
    int features, depth;         // rows of the product's result, length of its sums
    int bits;
    const float *lo, *step;      // per feature: alpha = step, beta = lo + center step; null: 1 and 1
    float center;
    const int* ids;
    const float *sum, *row_scale, *hidden_scale, *hidden;   // row_scale may be null
    const void* up;              // adapters x rank x features, or null
    int rank, requests;
    void* out;
    int64_t ldo;
    int out_bf16;
    int early;                   // launched so that it may start before stage 1 has ended
    DeviceStatus* status;
};

// Stage 3: grad_down[i][r][j] = sum over i's tokens of v_tr Q(x_t)_j, grad_up[i][r][o] = sum of hidden_tr dy_to
struct GradArgs {
    int64_t tokens;
    const int32_t *starts, *which;
    int requests, adapters, rank;
    const float *v, *hidden;     // tokens x rank
    const uint8_t* codes;        // tokens x code_stride
    int64_t code_stride;
    const float2* grids;         // tokens x groups of (lo, step)
    int inputs, group, groups;
    const void* dy;              // tokens x lddy
    int64_t lddy;
    int outputs, bf16;
    int dy_copied;               // dy's rows are aligned for tensor copies
    float *grad_down, *grad_up;  // either may be null
    int down_blocks, up_blocks;
    DeviceStatus* status;
};

// Tensor map of a matrix of `rows` rows (project.cu).
int encode_map(zipml_ctx* ctx, CUtensorMapDataType type, const void* base, int64_t inner, int64_t rows, int64_t stride_bytes, int box_inner, int box_rows,
               CUtensorMapSwizzle swizzle, CUtensorMap* out);

int launch_shrink(zipml_ctx* ctx, const ShrinkArgs& a, int dtype, bool backward);
int launch_project(zipml_ctx* ctx, const ProjectArgs& a, const void* tokens_operand, int64_t ld_operand, bool operand_bf16, const zipml_dataset* w,
                   bool backward);
int launch_project_grad(zipml_ctx* ctx, const GradArgs& a);
int launch_group_probe(zipml_ctx* ctx, int64_t limit_ns);
int launch_checkpoint_encode(zipml_ctx* ctx, const void* X, int dtype, int64_t m, int64_t n, int64_t ldx, uint64_t seed, const zipml_checkpoint* out);
int launch_checkpoint_decode(zipml_ctx* ctx, const zipml_checkpoint* cp, int dtype, void* X, int64_t ldx);

}  // namespace zipml
