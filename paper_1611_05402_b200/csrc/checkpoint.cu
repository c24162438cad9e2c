// Checkpoints of activations in 8 bits: one pass that finds each group's grid, rounds its values stochastically onto it
// (paper Section 2.1; the row scaling of the Supplement, group by group) and writes a byte each, and the way back.
#include "project.cuh"

namespace zipml {

// ---------------------------------------------------------------------------------------------
// A lane takes 8 neighbouring features (one block of random numbers, Philox4x32-10 of (block, row)), a warp 256 of one row, so a
// group of 32 .. 256 features is 4 .. 32 lanes and its range a butterfly among them; the values stay in registers between range and
// rounding and are read once.
//   t = (x - lo) * (255 / (hi - lo)), each operation one fp32 rounding; code = (ceil(2^16 t) + u16) >> 16: floor(t), or one more with
//   the probability of t's fraction (rounded up to 2^-16: the mean is off by at most 2^-16 of a step).
// ---------------------------------------------------------------------------------------------
constexpr int kEncodeWarps = 8;
constexpr uint32_t kCheckpointDraws = 8;        // the Philox counter's last word (the quantizers use others)

struct EncodeArgs {
    const void* x;
    int64_t m, ldx;
    int n, group, groups;
    uint64_t seed;
    uint8_t* codes;
    int64_t row_bytes;
    float2* grids;
    int segments;               // pieces of 256 features a row
    int wide;                   // rows and base are 16-byte aligned
    DeviceStatus* status;
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, int count, bool wide, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        if (wide && count >= 8) {
            const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < count ? p[i] : 0.0f;
        }
    } else {
        const uint4 w = load8_16(p, count, wide);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack_pair<T>(u[i]);
            v[2 * i] = f.x; v[2 * i + 1] = f.y;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(32 * kEncodeWarps) checkpoint_encode_kernel(EncodeArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t units = a.m * a.segments;
    const int lanes = a.group >> 3;
    bool bad = false;
    for (int64_t u = (int64_t)blockIdx.x * kEncodeWarps + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * kEncodeWarps) {
        const int64_t row = u / a.segments;
        const int j = (int)(u - row * a.segments) * 256 + lane * 8;
        const int count = min(max(a.n - j, 0), 8);
        float v[8];
        load8<T>(reinterpret_cast<const T*>(a.x) + row * a.ldx + j, count, a.wide != 0, v);
        float lo = INFINITY, hi = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) {
                lo = fminf(lo, v[i]);
                hi = fmaxf(hi, v[i]);
                bad |= !(fabsf(v[i]) <= 3.402823466e38f);
            }
        for (int o = 1; o < lanes; o <<= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        const float range = __fsub_rn(hi, lo);
        const float step = __fdiv_rn(range, 255.0f);
        const float inv = range > 0.0f ? fminf(__fdiv_rn(255.0f, range), 3.402823466e38f) : 0.0f;
        const Philox4 r = philox4x32_10((uint32_t)(j >> 3), (uint32_t)row, (uint32_t)((uint64_t)row >> 32), kCheckpointDraws, (uint32_t)a.seed,
                                        (uint32_t)(a.seed >> 32));
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = fminf(fmaxf(__fmul_rn(__fsub_rn(v[i], lo), inv), 0.0f), 255.0f);
            const uint32_t u16 = (r.v[i >> 1] >> (16 * (i & 1))) & 0xffffu;
            const uint32_t code = (__float2uint_ru(__fmul_rn(t, 65536.0f)) + u16) >> 16;
            if (i < count) w[i >> 2] |= code << (8 * (i & 3));
        }
        if (j < a.row_bytes) *reinterpret_cast<uint2*>(a.codes + row * a.row_bytes + j) = make_uint2(w[0], w[1]);
        if (count > 0 && (lane & (lanes - 1)) == 0) {
            a.grids[row * a.groups + j / a.group] = make_float2(lo, step);
            bad |= !(range <= 3.402823466e38f);
        }
    }
    if (bad) set_status(a.status, ZIPML_ERR_NONFINITE, 92);
}

template <typename T>
__global__ void __launch_bounds__(256) checkpoint_decode_kernel(const uint8_t* codes, int64_t row_bytes, const float2* grids, int groups, int group, int64_t m,
                                                                int n, int blocks, T* x, int64_t ldx, int wide) {
    const int64_t units = m * blocks;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
        const int64_t row = u / blocks;
        const int j = (int)(u - row * blocks) * 8;
        const uint2 w = *reinterpret_cast<const uint2*>(codes + row * row_bytes + j);
        const float2 g = grids[row * groups + j / group];
        const int count = min(n - j, 8);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fmaf_rn(byte_to_float(i < 4 ? w.x : w.y, i & 3), g.y, g.x);
        T* p = x + row * ldx + j;
        if (wide && count == 8) {
            if constexpr (sizeof(T) == 4) {
                *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                *reinterpret_cast<uint4*>(p) = make_uint4(pack_pair<T>(v[0], v[1]), pack_pair<T>(v[2], v[3]), pack_pair<T>(v[4], v[5]), pack_pair<T>(v[6], v[7]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) p[i] = from_float<T>(v[i]);
        }
    }
}

static int element_bytes(int dtype) { return dtype == ZIPML_F32 ? 4 : 2; }

int launch_checkpoint_encode(zipml_ctx* ctx, const void* X, int dtype, int64_t m, int64_t n, int64_t ldx, uint64_t seed, const zipml_checkpoint* out) {
    EncodeArgs a{};
    a.x = X; a.m = m; a.n = (int)n; a.ldx = ldx;
    a.group = out->group; a.groups = (int)((n + out->group - 1) / out->group);
    a.seed = seed; a.codes = const_cast<uint8_t*>(out->codes); a.row_bytes = out->row_bytes;
    a.grids = reinterpret_cast<float2*>(const_cast<float*>(out->grids));
    a.segments = (int)((out->row_bytes + 255) / 256);
    a.wide = (reinterpret_cast<uintptr_t>(X) % 16 == 0) && (ldx * element_bytes(dtype)) % 16 == 0;
    a.status = ctx->d_status;
    const int64_t units = m * a.segments;
    const int64_t want = (units + kEncodeWarps - 1) / kEncodeWarps;
    const int grid = (int)(want < (int64_t)ctx->sm_count * 32 ? want : (int64_t)ctx->sm_count * 32);
    if (dtype == ZIPML_F32) checkpoint_encode_kernel<float><<<grid, 32 * kEncodeWarps, 0, ctx->stream>>>(a);
    else if (dtype == ZIPML_BF16) checkpoint_encode_kernel<__nv_bfloat16><<<grid, 32 * kEncodeWarps, 0, ctx->stream>>>(a);
    else checkpoint_encode_kernel<__half><<<grid, 32 * kEncodeWarps, 0, ctx->stream>>>(a);
    ctx->launches += 1;
    return cuda_status(cudaGetLastError());
}

int launch_checkpoint_decode(zipml_ctx* ctx, const zipml_checkpoint* cp, int dtype, void* X, int64_t ldx) {
    const int n = (int)cp->n, groups = (n + cp->group - 1) / cp->group, blocks = (n + 7) / 8;
    const int wide = (reinterpret_cast<uintptr_t>(X) % 16 == 0) && (ldx * element_bytes(dtype)) % 16 == 0;
    const int64_t want = (cp->m * blocks + 255) / 256;
    const int grid = (int)(want < (int64_t)ctx->sm_count * 32 ? want : (int64_t)ctx->sm_count * 32);
    const float2* grids = reinterpret_cast<const float2*>(cp->grids);
    if (dtype == ZIPML_F32)
        checkpoint_decode_kernel<float><<<grid, 256, 0, ctx->stream>>>(cp->codes, cp->row_bytes, grids, groups, cp->group, cp->m, n, blocks, (float*)X, ldx, wide);
    else if (dtype == ZIPML_BF16)
        checkpoint_decode_kernel<__nv_bfloat16><<<grid, 256, 0, ctx->stream>>>(cp->codes, cp->row_bytes, grids, groups, cp->group, cp->m, n, blocks, (__nv_bfloat16*)X, ldx, wide);
    else
        checkpoint_decode_kernel<__half><<<grid, 256, 0, ctx->stream>>>(cp->codes, cp->row_bytes, grids, groups, cp->group, cp->m, n, blocks, (__half*)X, ldx, wide);
    ctx->launches += 1;
    return cuda_status(cudaGetLastError());
}

}  // namespace zipml
