// Checkpoints of activations in 8 bits: one pass that finds each group's grid, rounds its values stochastically onto it
// (paper Section 2.1; the row scaling of the Supplement, group by group) and writes a byte each, and the way back.
#include <type_traits>

#include "project.cuh"

namespace zipml {

// ---------------------------------------------------------------------------------------------
// A lane takes 16 neighbouring features (two blocks of random numbers, Philox4x32-10 of (block, row)), a warp 512 of one row, so a
// group of 32 .. 256 features is 2 .. 16 lanes and its range a butterfly among them; the values stay in registers between range and
// rounding and are read once.
//   t = (x - lo) * (255 / (hi - lo)), each operation one fp32 rounding; code = (ceil(2^16 t) + u16) >> 16: floor(t), or one more with
//   the probability of t's fraction (rounded up to 2^-16: the mean is off by at most 2^-16 of a step).
// Bound by instructions, the generator's 64-bit products first: 16 random bits a value instead of the quantizers' 24, the round keys
// from the host, minimum and maximum of 16-bit types in pairs, and 16 features a lane for one butterfly and two divisions.
// 16,384 x 8,192 bf16 137 us (3.0 TB/s in and out; 28 instructions a value, three quarters of the issue slots taken), 259 with 8 features a
// lane, keys worked out a round and ranges one by one; 2,047 x 4,096 fp16 11 us.
// ---------------------------------------------------------------------------------------------
constexpr int kEncodeWarps = 8;
constexpr int kLaneFeatures = 16;
constexpr int kWarpFeatures = 32 * kLaneFeatures;
constexpr uint32_t kCheckpointDraws = 8;        // the Philox counter's last word (zipml_quantize_draw's draw 8 has the same)
constexpr float kMostFloat = 3.402823466e38f;

struct EncodeArgs {
    const void* x;
    int64_t m, ldx;
    int n, group, groups;
    uint32_t keys[20];          // Philox's ten pairs of round keys
    uint8_t* codes;
    int64_t row_bytes;
    float2* grids;
    int segments;               // pieces of 512 features a row
    int wide;                   // rows and base are 16-byte aligned
    DeviceStatus* status;
};

// philox4x32_10 with its round keys given.
__device__ __forceinline__ Philox4 philox_keyed(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, const uint32_t (&keys)[20]) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ keys[2 * r];
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ keys[2 * r + 1];
        c3 = (uint32_t)p0;
    }
    Philox4 out;
    out.v[0] = c0; out.v[1] = c1; out.v[2] = c2; out.v[3] = c3;
    return out;
}

// Sixteen values from p on as 32-bit words; where fewer are there (`count`, at least one) the last one stands for the others.
template <typename T>
__device__ __forceinline__ void load_lane(const T* p, int count, bool wide, uint32_t (&w)[kLaneFeatures * sizeof(T) / 4]) {
    constexpr int N = kLaneFeatures * sizeof(T) / 16;
    if (wide && count == kLaneFeatures) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint4 u = reinterpret_cast<const uint4*>(p)[i];
            w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
        }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < kLaneFeatures; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[min(i, count - 1)];
    } else {
#pragma unroll
        for (int i = 0; i < kLaneFeatures; i += 2) {
            const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
            w[i / 2] = h[min(i, count - 1)] | (uint32_t)h[min(i + 1, count - 1)] << 16;
        }
    }
}

// Their least and largest; NaN where one of them is.
template <typename T>
__device__ __forceinline__ void lane_range(const uint32_t (&w)[kLaneFeatures * sizeof(T) / 4], float& lo, float& hi) {
    if constexpr (sizeof(T) == 4) {
        float nan = 0.0f;
        lo = hi = __uint_as_float(w[0]);
#pragma unroll
        for (int i = 0; i < kLaneFeatures; ++i) {
            const float v = __uint_as_float(w[i]);
            lo = fminf(lo, v);
            hi = fmaxf(hi, v);
            nan = fmaf(v, 0.0f, nan);
        }
        lo += nan;
    } else {
        using P = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        const P* v = reinterpret_cast<const P*>(w);
        P a = v[0], b = v[0];
#pragma unroll
        for (int i = 1; i < kLaneFeatures / 2; ++i) {
            a = __hmin2_nan(a, v[i]);
            b = __hmax2_nan(b, v[i]);
        }
        const float2 x = unpack_pair<T>(*reinterpret_cast<const uint32_t*>(&a)), y = unpack_pair<T>(*reinterpret_cast<const uint32_t*>(&b));
        lo = fminf(x.x, x.y) + (x.x - x.x) + (x.y - x.y);                             // (fminf drops a NaN)
        hi = fmaxf(y.x, y.y);
    }
}

// Unit u of `per` a row, u = first, first + stride, ...: its row and place there, without a division a turn.
struct RowUnits {
    int64_t row;
    int place, per, step_place;
    int64_t step_row;
    __device__ __forceinline__ RowUnits(int64_t first, int64_t stride, int per_row) : per(per_row) {
        row = first / per;
        place = (int)(first - row * per);
        step_row = stride / per;
        step_place = (int)(stride - step_row * per);
    }
    __device__ __forceinline__ void next() {
        row += step_row;
        place += step_place;
        if (place >= per) { place -= per; ++row; }
    }
};

template <typename T>
__global__ void __launch_bounds__(32 * kEncodeWarps) checkpoint_encode_kernel(const __grid_constant__ EncodeArgs a) {
    constexpr int W = kLaneFeatures * sizeof(T) / 4;
    const int lane = threadIdx.x & 31;
    const int lanes = a.group / kLaneFeatures;
    bool bad = false;
    for (RowUnits u((int64_t)blockIdx.x * kEncodeWarps + (threadIdx.x >> 5), (int64_t)gridDim.x * kEncodeWarps, a.segments); u.row < a.m; u.next()) {
        const int64_t row = u.row;
        const int j = u.place * kWarpFeatures + lane * kLaneFeatures;
        const int count = min(max(a.n - j, 0), kLaneFeatures);
        uint32_t w[W] = {};
        float lo = INFINITY, hi = -INFINITY;
        if (count > 0) {
            load_lane<T>(reinterpret_cast<const T*>(a.x) + row * a.ldx + j, count, a.wide != 0, w);
            lane_range<T>(w, lo, hi);
            bad |= !(hi - lo <= kMostFloat);
        }
        for (int o = 1; o < lanes; o <<= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        const float range = __fsub_rn(hi, lo);
        const float step = __fdiv_rn(range, 255.0f);
        const float inv = range > 0.0f ? fminf(__fdiv_rn(255.0f, range), kMostFloat) : 0.0f;
        uint32_t codes[4];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const Philox4 r = philox_keyed((uint32_t)(j >> 3) + b, (uint32_t)row, (uint32_t)((uint64_t)row >> 32), kCheckpointDraws, a.keys);
            uint32_t sum[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 v;
                if constexpr (sizeof(T) == 4) v = make_float2(__uint_as_float(w[8 * b + 2 * i]), __uint_as_float(w[8 * b + 2 * i + 1]));
                else v = unpack_pair<T>(w[4 * b + i]);
                const float s = fminf(__fmul_rn(__fsub_rn(v.x, lo), inv), 255.0f), t = fminf(__fmul_rn(__fsub_rn(v.y, lo), inv), 255.0f);
                sum[2 * i] = __float2uint_ru(__fmul_rn(s, 65536.0f)) + (r.v[i] & 0xffffu);
                sum[2 * i + 1] = __float2uint_ru(__fmul_rn(t, 65536.0f)) + (r.v[i] >> 16);
            }
            // (the code is a sum's third byte)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                codes[2 * b + i] = __byte_perm(__byte_perm(sum[4 * i], sum[4 * i + 1], 0x0062), __byte_perm(sum[4 * i + 2], sum[4 * i + 3], 0x0062), 0x5410);
        }
        if (count < kLaneFeatures) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int there = min(max(count - 4 * i, 0), 4);
                codes[i] &= there == 4 ? 0xffffffffu : (1u << (8 * there)) - 1u;
            }
        }
        if (j < a.row_bytes) *reinterpret_cast<uint4*>(a.codes + row * a.row_bytes + j) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
        if (count > 0 && (lane & (lanes - 1)) == 0) {
            // (the roundings of range and step may take the upper end past the largest number: a step's last place keeps it there)
            const bool past = !(__fmaf_rn(255.0f, step, lo) <= kMostFloat);
            a.grids[row * a.groups + j / a.group] = make_float2(lo, past ? __uint_as_float(__float_as_uint(step) - 1u) : step);
            bad |= !(range <= kMostFloat);
        }
    }
    if (bad) set_status(a.status, ZIPML_ERR_NONFINITE, 92);
}

// A thread takes 16 codes; bound by HBM: 16,384 x 8,192 to bf16 68 us, 6.0 TB/s.
template <typename T>
__global__ void __launch_bounds__(256) checkpoint_decode_kernel(const uint8_t* codes, int64_t row_bytes, const float2* grids, int groups, int group_shift, int64_t m,
                                                                int n, int blocks, T* x, int64_t ldx, int wide) {
    for (RowUnits u((int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, blocks); u.row < m; u.next()) {
        const int64_t row = u.row;
        const int j = u.place * kLaneFeatures;
        const uint4 c = *reinterpret_cast<const uint4*>(codes + row * row_bytes + j);
        const float2 g = grids[row * groups + (j >> group_shift)];
        const int count = min(n - j, kLaneFeatures);
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
        float v[kLaneFeatures];
#pragma unroll
        for (int i = 0; i < kLaneFeatures; ++i) v[i] = __fmaf_rn(byte_to_float(w[i >> 2], i & 3), g.y, g.x);
        T* p = x + row * ldx + j;
        if (wide && count == kLaneFeatures) {
#pragma unroll
            for (int i = 0; i < kLaneFeatures; i += 16 / (int)sizeof(T)) {
                if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                else
                    *reinterpret_cast<uint4*>(p + i) = make_uint4(pack_pair<T>(v[i], v[i + 1]), pack_pair<T>(v[i + 2], v[i + 3]), pack_pair<T>(v[i + 4], v[i + 5]),
                                                                  pack_pair<T>(v[i + 6], v[i + 7]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLaneFeatures; ++i)
                if (i < count) p[i] = from_float<T>(v[i]);
        }
    }
}

static int element_bytes(int dtype) { return dtype == ZIPML_F32 ? 4 : 2; }

int launch_checkpoint_encode(zipml_ctx* ctx, const void* X, int dtype, int64_t m, int64_t n, int64_t ldx, uint64_t seed, const zipml_checkpoint* out) {
    EncodeArgs a{};
    a.x = X; a.m = m; a.n = (int)n; a.ldx = ldx;
    a.group = out->group; a.groups = (int)((n + out->group - 1) / out->group);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
    for (int r = 0; r < 10; ++r, k0 += 0x9E3779B9u, k1 += 0xBB67AE85u) { a.keys[2 * r] = k0; a.keys[2 * r + 1] = k1; }
    a.codes = const_cast<uint8_t*>(out->codes); a.row_bytes = out->row_bytes;
    a.grids = reinterpret_cast<float2*>(const_cast<float*>(out->grids));
    a.segments = (int)((out->row_bytes + kWarpFeatures - 1) / kWarpFeatures);
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
    const int n = (int)cp->n, groups = (n + cp->group - 1) / cp->group, blocks = (n + kLaneFeatures - 1) / kLaneFeatures;
    const int shift = cp->group == 32 ? 5 : cp->group == 64 ? 6 : cp->group == 128 ? 7 : 8;
    const int wide = (reinterpret_cast<uintptr_t>(X) % 16 == 0) && (ldx * element_bytes(dtype)) % 16 == 0;
    const int64_t want = (cp->m * blocks + 255) / 256;
    const int grid = (int)(want < (int64_t)ctx->sm_count * 32 ? want : (int64_t)ctx->sm_count * 32);
    const float2* grids = reinterpret_cast<const float2*>(cp->grids);
    if (dtype == ZIPML_F32)
        checkpoint_decode_kernel<float><<<grid, 256, 0, ctx->stream>>>(cp->codes, cp->row_bytes, grids, groups, shift, cp->m, n, blocks, (float*)X, ldx, wide);
    else if (dtype == ZIPML_BF16)
        checkpoint_decode_kernel<__nv_bfloat16><<<grid, 256, 0, ctx->stream>>>(cp->codes, cp->row_bytes, grids, groups, shift, cp->m, n, blocks, (__nv_bfloat16*)X, ldx, wide);
    else
        checkpoint_decode_kernel<__half><<<grid, 256, 0, ctx->stream>>>(cp->codes, cp->row_bytes, grids, groups, shift, cp->m, n, blocks, (__half*)X, ldx, wide);
    ctx->launches += 1;
    return cuda_status(cudaGetLastError());
}

}  // namespace zipml
