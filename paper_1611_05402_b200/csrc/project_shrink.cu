// First stage of a projection with low-rank adapters: every token onto the ranks of its own adapter (hidden = scale A x in the
// forward pass, scale B dy in the backward one), with the sums that the codes' grids need of a token, in one pass over the tokens.
#include <type_traits>

#include <cooperative_groups.h>

#include "project.cuh"

namespace zipml {

namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------------------------
// A cluster takes 16 tokens, its CTAs and their warps the columns in turns of 32.  m16n8k16 products (16-bit factors are exact, sums in
// fp32): a lane reads 16 consecutive bytes of a token's row and of the adapter's rows, 8 columns that both operands count as
// the same 8 places of two products' depth, so nothing passes through shared memory on the way.  Tokens of several adapters in a
// tile take a pass over the columns for each adapter and keep the rows that are theirs.  The warps' and CTAs' sums are added
// in a fixed order.
// ---------------------------------------------------------------------------------------------
constexpr int kShrinkWarps = 8;

struct ShrinkShared {
    int ids[kShrinkRows];
    int distinct[kShrinkRows];
    int count;
    float sum[kShrinkWarps][kShrinkRows];
    float top[kShrinkWarps][kShrinkRows];
    float cta_sum[kShrinkRows];
    float cta_top[kShrinkRows];
    float scale[kShrinkRows];
};

template <typename T>
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// RT: blocks of 8 ranks (0: no adapters).
template <typename T, bool BACK, int RT>
__global__ void __launch_bounds__(32 * kShrinkWarps) shrink_kernel(ShrinkArgs a) {
    // (the projection may start: what it does before it waits for this kernel's end does not depend on it)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    extern __shared__ float part[];                       // [warps][16][RT * 8], then its sum over the warps in [0]
    __shared__ ShrinkShared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int64_t t0 = (int64_t)(blockIdx.x / ranks) * kShrinkRows;
    const int slice = blockIdx.y, slices = gridDim.y;     // this cluster's share of the tile's adapters
    constexpr int R = RT * 8;

    if (threadIdx.x < kShrinkRows) {
        const int64_t t = t0 + threadIdx.x;
        sh.ids[threadIdx.x] = t < a.tokens ? adapter_of(a.starts, a.which, a.requests, a.adapters, t, a.status) : kNoRequest;
    }
    for (int i = threadIdx.x; i < kShrinkWarps * kShrinkRows * R; i += blockDim.x) part[i] = 0.0f;
    __syncthreads();
    if (threadIdx.x == 0) {
        int count = 0, seen = 0;
        for (int r = 0; r < kShrinkRows; ++r) {
            bool fresh = sh.ids[r] >= 0;
            for (int s = 0; s < r; ++s) fresh &= sh.ids[s] != sh.ids[r];
            if (fresh && seen++ % slices == slice) sh.distinct[count++] = sh.ids[r];
        }
        sh.count = count;
    }
    __syncthreads();

    const T* z = reinterpret_cast<const T*>(a.z);
    const int64_t tg = t0 + g, th = t0 + g + 8;
    const T* zg = z + tg * a.ldz;
    const T* zh = z + th * a.ldz;
    const bool wide_z = ((reinterpret_cast<uintptr_t>(z) | (uintptr_t)(a.ldz * 2)) & 15) == 0;
    const bool wide_d = ((reinterpret_cast<uintptr_t>(a.down) | (uintptr_t)((int64_t)a.columns * 2)) & 15) == 0;
    const bool use_g = sh.ids[g] != kNoRequest, use_h = sh.ids[g + 8] != kNoRequest;
    float sum_g = 0.0f, sum_h = 0.0f, top_g = 0.0f, top_h = 0.0f;
    const int passes = RT == 0 ? (slice == 0 ? 1 : 0) : max(sh.count, slice == 0 ? 1 : 0);
    for (int d = 0; d < passes; ++d) {
        const bool stats = d == 0 && slice == 0;
        const int adapter = RT > 0 && d < sh.count ? sh.distinct[d] : -1;
        float acc[RT > 0 ? RT : 1][4] = {};
        const T* down = reinterpret_cast<const T*>(a.down) + (adapter >= 0 ? (int64_t)adapter * a.rank * a.columns : 0);
        for (int j0 = (rank * kShrinkWarps + warp) * 32; j0 < a.columns; j0 += ranks * kShrinkWarps * 32) {
            const int j = j0 + q * 8, count = min(max(a.columns - j, 0), 8);
            const uint4 x0 = use_g ? load8_16(zg + j, count, wide_z) : make_uint4(0, 0, 0, 0);
            const uint4 x1 = use_h ? load8_16(zh + j, count, wide_z) : make_uint4(0, 0, 0, 0);
            if (stats) {
                const uint32_t w0[4] = {x0.x, x0.y, x0.z, x0.w}, w1[4] = {x1.x, x1.y, x1.z, x1.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f0 = unpack_pair<T>(w0[i]), f1 = unpack_pair<T>(w1[i]);
                    if constexpr (BACK) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int c = 2 * i + e;
                            if (c < count) {
                                const float step = a.step[j + c], mid = fmaf(a.center, step, a.lo[j + c]);
                                const float u0 = e ? f0.y : f0.x, u1 = e ? f1.y : f1.x;
                                sum_g = fmaf(u0, mid, sum_g);
                                sum_h = fmaf(u1, mid, sum_h);
                                top_g = fmaxf(top_g, fabsf(u0 * step));
                                top_h = fmaxf(top_h, fabsf(u1 * step));
                            }
                        }
                    } else {
                        sum_g += f0.x + f0.y;
                        sum_h += f1.x + f1.y;
                    }
                }
                if (!BACK && a.copy && count > 0) {
                    T* copy = reinterpret_cast<T*>(a.copy);                 // (rows padded to a multiple of 8: the zeros behind the last column fit)
                    if (tg < a.tokens) *reinterpret_cast<uint4*>(copy + tg * a.ld_copy + j) = x0;
                    if (th < a.tokens) *reinterpret_cast<uint4*>(copy + th * a.ld_copy + j) = x1;
                }
            }
            if constexpr (RT > 0) {
                if (adapter >= 0) {
#pragma unroll
                    for (int n = 0; n < RT; ++n) {
                        const int r = n * 8 + g;
                        const uint4 y = r < a.rank ? load8_16(down + (int64_t)r * a.columns + j, count, wide_d) : make_uint4(0, 0, 0, 0);
                        mma_16816<T>(acc[n], x0.x, x1.x, x0.y, x1.y, y.x, y.y);
                        mma_16816<T>(acc[n], x0.z, x1.z, x0.w, x1.w, y.z, y.w);
                    }
                }
            }
        }
        if constexpr (RT > 0) {
            if (adapter >= 0) {
                float* mine = part + warp * kShrinkRows * R;
#pragma unroll
                for (int n = 0; n < RT; ++n) {
                    if (sh.ids[g] == adapter) { mine[g * R + n * 8 + 2 * q] = acc[n][0]; mine[g * R + n * 8 + 2 * q + 1] = acc[n][1]; }
                    if (sh.ids[g + 8] == adapter) { mine[(g + 8) * R + n * 8 + 2 * q] = acc[n][2]; mine[(g + 8) * R + n * 8 + 2 * q + 1] = acc[n][3]; }
                }
            }
        }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        sum_g += __shfl_xor_sync(0xffffffffu, sum_g, o);
        sum_h += __shfl_xor_sync(0xffffffffu, sum_h, o);
        top_g = fmaxf(top_g, __shfl_xor_sync(0xffffffffu, top_g, o));
        top_h = fmaxf(top_h, __shfl_xor_sync(0xffffffffu, top_h, o));
    }
    if (q == 0) {
        sh.sum[warp][g] = sum_g; sh.sum[warp][g + 8] = sum_h;
        sh.top[warp][g] = top_g; sh.top[warp][g + 8] = top_h;
    }
    __syncthreads();
    // the CTA's sums
    for (int i = threadIdx.x; i < kShrinkRows * R; i += blockDim.x) {
        float s = part[i];
        for (int w = 1; w < kShrinkWarps; ++w) s += part[w * kShrinkRows * R + i];
        part[i] = s;
    }
    if (threadIdx.x < kShrinkRows) {
        float s = 0.0f, m = 0.0f;
        for (int w = 0; w < kShrinkWarps; ++w) {
            s += sh.sum[w][threadIdx.x];
            m = fmaxf(m, sh.top[w][threadIdx.x]);
        }
        sh.cta_sum[threadIdx.x] = s;
        sh.cta_top[threadIdx.x] = m;
    }
    cluster.sync();
    // the cluster's: row by row, CTA `rank` the rows rank, rank + ranks, ..., a warp each
    for (int row = rank + ranks * warp; row < kShrinkRows; row += ranks * kShrinkWarps) {
        const int64_t t = t0 + row;
        const int id = sh.ids[row];
        if (t >= a.tokens) continue;
        bool mine = slice == 0 && id < 0;
        for (int d = 0; d < sh.count; ++d) mine |= sh.distinct[d] == id;
        if constexpr (RT > 0) {
            if (mine && id != kNoRequest) {
                const float scale = id >= 0 ? (a.scale ? a.scale[id] : 1.0f) : 0.0f;
                float top = 0.0f;
                for (int r = lane; r < a.rank; r += 32) {
                    float s = 0.0f;
                    if (id >= 0) {
                        for (int c = 0; c < ranks; ++c) s += cluster.map_shared_rank(part, c)[row * R + r];
                        s *= scale;
                    }
                    a.hidden[t * a.rank + r] = s;
                    top = fmaxf(top, fabsf(s));
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                if (lane == 0) a.hidden_scale[t] = 1.0f / scale_to_range(top);
            }
        }
        if (slice == 0 && lane == 0) {
            a.ids[t] = id;
            float s = 0.0f;
            for (int c = 0; c < ranks; ++c) s += cluster.map_shared_rank(sh.cta_sum, c)[row];
            a.sum[t] = s;
        }
    }
    if constexpr (BACK) {
        if (slice == 0 && a.scaled) {
            // z step, scaled by a power of two of the row so that fp16's range holds it: fp16 keeps 11 bits where bf16 would keep 8, one rounding
            if (threadIdx.x < kShrinkRows) {
                float m = 0.0f;
                for (int c = 0; c < ranks; ++c) m = fmaxf(m, cluster.map_shared_rank(sh.cta_top, c)[threadIdx.x]);
                const float s = scale_to_range(m);
                sh.scale[threadIdx.x] = s;
                if (rank == 0 && t0 + (int)threadIdx.x < a.tokens) a.row_scale[t0 + threadIdx.x] = 1.0f / s;
            }
            __syncthreads();
            const float s0 = sh.scale[g], s1 = sh.scale[g + 8];
            for (int j0 = (rank * kShrinkWarps + warp) * 32; j0 < a.columns; j0 += ranks * kShrinkWarps * 32) {
                const int j = j0 + q * 8, count = min(max(a.columns - j, 0), 8);
                if (count == 0) continue;
                const uint4 x0 = use_g ? load8_16(zg + j, count, wide_z) : make_uint4(0, 0, 0, 0);
                const uint4 x1 = use_h ? load8_16(zh + j, count, wide_z) : make_uint4(0, 0, 0, 0);
                const uint32_t w0[4] = {x0.x, x0.y, x0.z, x0.w}, w1[4] = {x1.x, x1.y, x1.z, x1.w};
                uint32_t o0[4], o1[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f0 = unpack_pair<T>(w0[i]), f1 = unpack_pair<T>(w1[i]);
                    const float e0 = 2 * i < count ? a.step[j + 2 * i] : 0.0f, e1 = 2 * i + 1 < count ? a.step[j + 2 * i + 1] : 0.0f;
                    o0[i] = pack_pair<__half>(f0.x * e0 * s0, f0.y * e1 * s0);
                    o1[i] = pack_pair<__half>(f1.x * e0 * s1, f1.y * e1 * s1);
                }
                if (tg < a.tokens) *reinterpret_cast<uint4*>(a.scaled + tg * a.ld_scaled + j) = make_uint4(o0[0], o0[1], o0[2], o0[3]);
                if (th < a.tokens) *reinterpret_cast<uint4*>(a.scaled + th * a.ld_scaled + j) = make_uint4(o1[0], o1[1], o1[2], o1[3]);
            }
        }
    }
    cluster.sync();                                      // (no CTA leaves while another may still read its sums)
}

template <typename T, bool BACK, int RT>
static int launch_shrink_as(zipml_ctx* ctx, const ShrinkArgs& a) {
    const size_t smem = (size_t)kShrinkWarps * kShrinkRows * RT * 8 * sizeof(float);
    auto kernel = &shrink_kernel<T, BACK, RT>;
    if (smem > 40 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return cuda_status(e);
    }
    const int64_t tiles = (a.tokens + kShrinkRows - 1) / kShrinkRows;
    // Few tiles: the columns over the CTAs of a cluster, the tile's adapters over several clusters, until the GPU is about full.
    int ranks = 1, slices = 1;
    const int turns = (a.columns + 32 * kShrinkWarps - 1) / (32 * kShrinkWarps);
    while (ranks < 8 && tiles * ranks * 2 <= 2 * ctx->sm_count && ranks * 2 <= turns) ranks *= 2;
    const int most = a.requests < kShrinkRows ? a.requests : kShrinkRows;
    while (RT > 0 && slices * 2 <= most && tiles * ranks * slices * 2 <= 4 * ctx->sm_count) slices *= 2;
    if (tiles * ranks > 0x7fffffffLL) return ZIPML_ERR_WORKSPACE;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles * ranks), (unsigned)slices);
    cfg.blockDim = dim3(32 * kShrinkWarps);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
    ctx->launches += 1;
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError());
}

template <typename T, bool BACK>
static int launch_shrink_ranks(zipml_ctx* ctx, const ShrinkArgs& a) {
    if (!a.down) return launch_shrink_as<T, BACK, 0>(ctx, a);
    if (a.rank <= 8) return launch_shrink_as<T, BACK, 1>(ctx, a);
    if (a.rank <= 16) return launch_shrink_as<T, BACK, 2>(ctx, a);
    if (a.rank <= 32) return launch_shrink_as<T, BACK, 4>(ctx, a);
    if (a.rank <= 64) return launch_shrink_as<T, BACK, 8>(ctx, a);
    return launch_shrink_as<T, BACK, 16>(ctx, a);
}

int launch_shrink(zipml_ctx* ctx, const ShrinkArgs& a, int dtype, bool backward) {
    if (dtype == ZIPML_BF16) return backward ? launch_shrink_ranks<__nv_bfloat16, true>(ctx, a) : launch_shrink_ranks<__nv_bfloat16, false>(ctx, a);
    return backward ? launch_shrink_ranks<__half, true>(ctx, a) : launch_shrink_ranks<__half, false>(ctx, a);
}

}  // namespace zipml
