// Third stage of a projection's backward pass: the gradients of the low-rank adapters, grad_down = sum v (x) Q(x) over the 8-bit
// checkpoints as they lie and grad_up = sum hidden (x) dy, each over the tokens of its adapter.
#include <cooperative_groups.h>

#include "project.cuh"

namespace zipml {

namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------------------------
// A cluster takes one adapter and one block of columns (128 codes or 64 values of dy: 128 bytes of each row), its CTAs' warps the
// adapter's tokens in turns of 8.  m16n8k8 products in tf32, ranks x columns x tokens: codes (code - 128) and 16-bit values are exact in
// its 11 bits, v step and hidden are split into two such parts, so a product keeps 22 bits.  A lane reads 16 consecutive bytes of
// the rows of two tokens; byte f of eight lanes is the f-th block of columns.  The lower ends' share, v . (lo + 128 step), is the same for a
// group's columns and is summed once per group.  Warps' and CTAs' sums are added in a fixed order.
// ---------------------------------------------------------------------------------------------
constexpr int kGradWarps = 8;

__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&x)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(b0), "r"(b1));
}
// x = high + low, both within tf32's 11 bits up to 2^-22 of x
__device__ __forceinline__ void split_tf32(float x, uint32_t& high, uint32_t& low) {
    high = __float_as_uint(x) & 0xffffe000u;
    low = __float_as_uint(x - __uint_as_float(high));
}

// MT: blocks of 16 ranks.  A pass takes at most kPassBlocks of them (registers), so higher ranks read the rows more than once.
template <bool CODES, int MT>
__device__ __forceinline__ void grad_pass(const GradArgs& a, int adapter, int block, int r0, float* sums, cg::cluster_group& cluster) {
    constexpr int NF = CODES ? 16 : 8;                     // columns of a lane's 16 bytes
    constexpr int GROUPS = CODES ? 4 : 1;                  // grids that 128 codes can lie in
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int ranks = (int)cluster.num_blocks(), crank = (int)cluster.block_rank();
    const int columns = CODES ? a.inputs : a.outputs;
    const int col0 = block * NF * 8, lane_col = col0 + g * NF;
    const float* left = CODES ? a.v : a.hidden;
    float acc[MT][NF][4] = {};
    float base[MT][GROUPS][2] = {};
    int turn = crank * kGradWarps + warp;                  // chunks of 8 tokens until this warp's next one
    for (int req = 0; req < a.requests; ++req) {
        if (a.which[req] != adapter) continue;
        const int64_t s = max((int64_t)a.starts[req], (int64_t)0), e = min((int64_t)a.starts[req + 1], a.tokens);
        if (e <= s) continue;
        const int64_t chunks = (e - s + 7) >> 3;
        int64_t c = turn;
        for (; c < chunks; c += ranks * kGradWarps) {
            const int64_t t0 = s + c * 8 + q, t1 = t0 + 4;
            const bool in0 = t0 < e, in1 = t1 < e;
            uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0;
            if constexpr (CODES) {
                if (lane_col < a.code_stride) {
                    if (in0) w0 = *reinterpret_cast<const uint4*>(a.codes + t0 * a.code_stride + lane_col);
                    if (in1) w1 = *reinterpret_cast<const uint4*>(a.codes + t1 * a.code_stride + lane_col);
                }
            } else {
                const uint16_t* dy = reinterpret_cast<const uint16_t*>(a.dy);
                const bool wide = ((reinterpret_cast<uintptr_t>(dy) | (uintptr_t)(a.lddy * 2)) & 15) == 0;
                const int count = min(max(columns - lane_col, 0), 8);
                if (in0) w0 = load8_16(dy + t0 * a.lddy + lane_col, count, wide);
                if (in1) w1 = load8_16(dy + t1 * a.lddy + lane_col, count, wide);
            }
            // the left factor of (rank g or g + 8 of each block, token t0 or t1)
            float v[MT][4];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int ra = r0 + m * 16 + g, rb = ra + 8;
                v[m][0] = in0 && ra < a.rank ? left[t0 * a.rank + ra] : 0.0f;
                v[m][1] = in0 && rb < a.rank ? left[t0 * a.rank + rb] : 0.0f;
                v[m][2] = in1 && ra < a.rank ? left[t1 * a.rank + ra] : 0.0f;
                v[m][3] = in1 && rb < a.rank ? left[t1 * a.rank + rb] : 0.0f;
            }
            const uint32_t u0[4] = {w0.x, w0.y, w0.z, w0.w}, u1[4] = {w1.x, w1.y, w1.z, w1.w};
            if constexpr (CODES) {
                // Where the block holds several groups, each takes a product of its own, with v times its step on the left and the other
                // groups' columns zero on the right.
                const int per = max(1, 128 / a.group);     // grids in the block: 1, 2 or 4
                for (int k = 0; k < per; ++k) {
                    const int grid = (col0 + k * a.group) / a.group;
                    if (col0 + k * a.group >= columns) break;
                    const float2 g0 = in0 ? a.grids[t0 * a.groups + grid] : make_float2(0.0f, 0.0f);
                    const float2 g1 = in1 ? a.grids[t1 * a.groups + grid] : make_float2(0.0f, 0.0f);
                    const float m0 = fmaf(128.0f, g0.y, g0.x), m1 = fmaf(128.0f, g1.y, g1.x);
                    const bool own = per == 1 || (g * NF) / a.group == k;
                    uint32_t hi[MT][4], lo[MT][4];
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        split_tf32(v[m][0] * g0.y, hi[m][0], lo[m][0]);
                        split_tf32(v[m][1] * g0.y, hi[m][1], lo[m][1]);
                        split_tf32(v[m][2] * g1.y, hi[m][2], lo[m][2]);
                        split_tf32(v[m][3] * g1.y, hi[m][3], lo[m][3]);
#pragma unroll
                        for (int kk = 0; kk < GROUPS; ++kk)
                            if (kk == k) {
                                base[m][kk][0] += fmaf(v[m][0], m0, v[m][2] * m1);
                                base[m][kk][1] += fmaf(v[m][1], m0, v[m][3] * m1);
                            }
                    }
#pragma unroll
                    for (int f = 0; f < NF; ++f) {
                        const float b0 = own ? byte_to_float(u0[f >> 2], f & 3) - 128.0f : 0.0f;
                        const float b1 = own ? byte_to_float(u1[f >> 2], f & 3) - 128.0f : 0.0f;
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            mma_tf32(acc[m][f], hi[m], __float_as_uint(b0), __float_as_uint(b1));
                            mma_tf32(acc[m][f], lo[m], __float_as_uint(b0), __float_as_uint(b1));
                        }
                    }
                }
            } else {
                uint32_t hi[MT][4], lo[MT][4];
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) split_tf32(v[m][i], hi[m][i], lo[m][i]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 b0 = a.bf16 ? unpack_pair<__nv_bfloat16>(u0[i]) : unpack_pair<__half>(u0[i]);
                    const float2 b1 = a.bf16 ? unpack_pair<__nv_bfloat16>(u1[i]) : unpack_pair<__half>(u1[i]);
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        mma_tf32(acc[m][2 * i], hi[m], __float_as_uint(b0.x), __float_as_uint(b1.x));
                        mma_tf32(acc[m][2 * i], lo[m], __float_as_uint(b0.x), __float_as_uint(b1.x));
                        mma_tf32(acc[m][2 * i + 1], hi[m], __float_as_uint(b0.y), __float_as_uint(b1.y));
                        mma_tf32(acc[m][2 * i + 1], lo[m], __float_as_uint(b0.y), __float_as_uint(b1.y));
                    }
                }
            }
        }
        turn = (int)(c - chunks);                          // (the next request's chunks go on where this one's ended)
    }
    if constexpr (CODES) {
        const int per = max(1, 128 / a.group);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
            for (int k = 0; k < GROUPS; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float s = base[m][k][i];
                    s += __shfl_xor_sync(0xffffffffu, s, 1);
                    s += __shfl_xor_sync(0xffffffffu, s, 2);
                    base[m][k][i] = s;
                }
            // column n of the product's blocks is lane n's 16 codes: columns 2 q and 2 q + 1 here
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int k = per == 1 ? 0 : ((2 * q + half) * NF) / a.group;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float s = k == 0 ? base[m][0][i] : k == 1 ? base[m][1][i] : k == 2 ? base[m][2][i] : base[m][3][i];
#pragma unroll
                    for (int f = 0; f < NF; ++f) acc[m][f][2 * i + half] += s;
                }
            }
        }
    }
    // Sums over the warps, then over the CTAs: [rank of the pass][column], one warp after the other
    constexpr int C = NF * 8;
    for (int w = 0; w < kGradWarps; ++w) {
        if (warp == w)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float* p = sums + (m * 16 + g + 8 * (i >> 1)) * C + (2 * q + (i & 1)) * NF + f;
                        *p = w == 0 ? acc[m][f][i] : *p + acc[m][f][i];
                    }
        __syncthreads();
    }
    cluster.sync();
    float* out = CODES ? a.grad_down : a.grad_up;
    const int most = min(MT * 16, a.rank - r0);
    for (int i = crank * blockDim.x + threadIdx.x; i < most * C; i += ranks * blockDim.x) {
        const int r = i / C, col = col0 + i % C;
        float s = 0.0f;
        for (int c = 0; c < ranks; ++c) s += cluster.map_shared_rank(sums, c)[i];
        if (col < columns) out[((int64_t)adapter * a.rank + r0 + r) * columns + col] = s;
    }
    cluster.sync();
}

template <int MT>
__global__ void __launch_bounds__(32 * kGradWarps) grad_kernel(GradArgs a) {
    extern __shared__ float sums[];
    cg::cluster_group cluster = cg::this_cluster();
    const int block = blockIdx.x / cluster.num_blocks(), adapter = blockIdx.y, r0 = blockIdx.z * MT * 16;
    if (block < a.down_blocks) grad_pass<true, MT>(a, adapter, block, r0, sums, cluster);
    else grad_pass<false, MT>(a, adapter, block - a.down_blocks, r0, sums, cluster);
}

template <int MT>
static int launch_grad_as(zipml_ctx* ctx, const GradArgs& a) {
    const int blocks = a.down_blocks + a.up_blocks, passes = (a.rank + MT * 16 - 1) / (MT * 16);
    const size_t smem = (size_t)MT * 16 * 128 * sizeof(float);
    int ranks = 1;
    while (ranks < 8 && (int64_t)blocks * a.adapters * passes * ranks < 2 * ctx->sm_count && (int64_t)ranks * kGradWarps * 8 < a.tokens) ranks *= 2;
    if (a.adapters > 65535 || (int64_t)blocks * ranks > 0x7fffffffLL) return ZIPML_ERR_WORKSPACE;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(blocks * ranks), (unsigned)a.adapters, (unsigned)passes);
    cfg.blockDim = dim3(32 * kGradWarps);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, &grad_kernel<MT>, a);
    ctx->launches += 1;
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError());
}

int launch_project_grad(zipml_ctx* ctx, const GradArgs& in) {
    GradArgs a = in;
    a.down_blocks = a.grad_down ? (a.inputs + 127) / 128 : 0;
    a.up_blocks = a.grad_up ? (a.outputs + 63) / 64 : 0;
    if (a.down_blocks + a.up_blocks == 0 || a.adapters == 0) return ZIPML_OK;
    return a.rank <= 16 ? launch_grad_as<1>(ctx, a) : launch_grad_as<2>(ctx, a);
}

}  // namespace zipml
