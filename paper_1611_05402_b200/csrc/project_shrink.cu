// First stage of a projection with low-rank adapters: every token onto the ranks of its own adapter (hidden = scale A x in the
// forward pass, scale B dy in the backward one), with the sums that the codes' grids need of a token, in one pass over the tokens.
#include <type_traits>

#include <cooperative_groups.h>

#include "project.cuh"
#include "tensor_core.cuh"

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

// The adapters of the tile's tokens, request by request: all threads of a block, which is synchronised at the end.  A token that no request
// holds has kNoRequest; an index past the adapters counts as none and is reported.
template <int ROWS>
__device__ __forceinline__ void find_adapters(const ShrinkArgs& a, int64_t t0, int* ids) {
    if (threadIdx.x < ROWS) ids[threadIdx.x] = !a.starts && t0 + threadIdx.x < a.tokens ? -1 : kNoRequest;
    __syncthreads();
    if (a.starts) {
        for (int q = threadIdx.x; q < a.requests; q += blockDim.x) {
            const int which = a.which[q];                                             // (loaded with the others, not after them)
            const int64_t s = max((int64_t)a.starts[q], t0), e = min(min((int64_t)a.starts[q + 1], a.tokens), t0 + ROWS);
            if (s >= e) continue;
            if (which >= a.adapters) set_status(a.status, ZIPML_ERR_INVALID_ARG, 91);
            const int id = which >= a.adapters ? -1 : max(which, -1);
            for (int64_t t = s; t < e; ++t) ids[t - t0] = id;
        }
        __syncthreads();
    }
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

    find_adapters<kShrinkRows>(a, t0, sh.ids);
    for (int i = threadIdx.x; i < kShrinkWarps * kShrinkRows * R; i += blockDim.x) part[i] = 0.0f;
    __syncthreads();
    if (warp == 0) {
        // the first token of each adapter, and of those every slices-th
        const int id = lane < kShrinkRows ? sh.ids[lane] : -1;
        const uint32_t same = __match_any_sync(0xffffffffu, id);
        const bool fresh = id >= 0 && (int)__ffs(same) - 1 == lane;
        const uint32_t firsts = __ballot_sync(0xffffffffu, fresh);
        const int nth = __popc(firsts & ((1u << lane) - 1u));
        if (fresh && nth % slices == slice) sh.distinct[nth / slices] = id;
        if (lane == 0) sh.count = (__popc(firsts) - slice + slices - 1) / slices;
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
            // z step, scaled by a power of two of the row so that fp16's range holds it, in two parts
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
                uint32_t high0[4], low0[4], high1[4], low1[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f0 = unpack_pair<T>(w0[i]), f1 = unpack_pair<T>(w1[i]);
                    const float e0 = 2 * i < count ? a.step[j + 2 * i] : 0.0f, e1 = 2 * i + 1 < count ? a.step[j + 2 * i + 1] : 0.0f;
                    split_scaled(f0.x * e0 * s0, f0.y * e1 * s0, high0[i], low0[i]);
                    split_scaled(f1.x * e0 * s1, f1.y * e1 * s1, high1[i], low1[i]);
                }
                if (tg < a.tokens) {
                    *reinterpret_cast<uint4*>(a.scaled + tg * a.ld_scaled + j) = make_uint4(high0[0], high0[1], high0[2], high0[3]);
                    *reinterpret_cast<uint4*>(a.scaled + (a.tokens + tg) * a.ld_scaled + j) = make_uint4(low0[0], low0[1], low0[2], low0[3]);
                }
                if (th < a.tokens) {
                    *reinterpret_cast<uint4*>(a.scaled + th * a.ld_scaled + j) = make_uint4(high1[0], high1[1], high1[2], high1[3]);
                    *reinterpret_cast<uint4*>(a.scaled + (a.tokens + th) * a.ld_scaled + j) = make_uint4(low1[0], low1[1], low1[2], low1[3]);
                }
            }
        }
    }
    cluster.sync();                                      // (no CTA leaves while another may still read its sums)
}

// ---------------------------------------------------------------------------------------------
// Many tokens: tiles of 128 on the tensor cores' rows, the adapters' ranks on the columns, both operands by tensor copies.  What counts is
// that the tokens' bytes keep coming (up to eight stages of 16 KB on their way), the products are next to nothing.  The forward pass's
// sums are one more column: 16 rows of ones lead the right operand.  A tile's adapters take `slots` at a time; a column that does not belong to
// a token's adapter, and ranks past the last that a copy's box brings along, are not read.  A cluster's CTAs divide the columns.  The
// tensor cores cut what they add to a sum where fp32 would round, always towards zero, so a long sum loses a few units of 2^-24 for
// every hundred products: the stages take up to eight sets of sums in turn, which are added in fp32 (8192 columns: 4.5e-6 of hidden off
// with one set, 0.7e-6 with them).
// 8192 tokens x 8192 x 32 ranks: 200 us with the kernel above (its 16-byte loads left most of each turn waiting).
// ---------------------------------------------------------------------------------------------
constexpr int kTallTokens = 128;
constexpr int kTallDepth = 64;
constexpr int kTallThreads = 256;
constexpr int kTallMostStages = 8;
constexpr uint32_t kTallLeftBytes = kTallTokens * kTallDepth * 2;

struct TallShared {
    uint64_t full[kTallMostStages], empty[kTallMostStages], done;
    uint32_t tmem;
    int gave_up;
    int ids[kTallTokens], distinct[kTallTokens], count;
    float sum[kTallTokens], scale[kTallTokens];
};

struct TallShape {
    int slots, ranks8, lead, rows, columns, stages;      // rows of the right operand; columns of tensor memory
    // columns of a pass with so many adapters, and sets of sums that tensor memory has room for
    __device__ __forceinline__ int pass_columns(int used) const { return (lead + used * ranks8 + 15) & ~15; }
    __device__ __forceinline__ int pass_sets(int used) const { return min(8, columns / max(pass_columns(used), 16)); }
};

template <bool BF16>
__global__ void __launch_bounds__(kTallThreads, 1) shrink_tall_kernel(ShrinkArgs a, TallShape f, const __grid_constant__ CUtensorMap z_map,
                                                                      const __grid_constant__ CUtensorMap down_map) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    extern __shared__ uint8_t raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t right_bytes = (uint32_t)f.rows * 128, stage_bytes = kTallLeftBytes + right_bytes;
    float* part = reinterpret_cast<float*>(ring + f.stages * stage_bytes);            // [token][rank], an odd stride
    const int stride = a.rank | 1;
    TallShared& sh = *reinterpret_cast<TallShared*>(part + kTallTokens * stride);
    cg::cluster_group cluster = cg::this_cluster();
    const int crank = (int)cluster.block_rank(), cranks = (int)cluster.num_blocks();
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // (known to be the same for a whole warp)
    const int64_t t0 = (int64_t)(blockIdx.x / cranks) * kTallTokens;
    const int all_steps = (a.columns + kTallDepth - 1) / kTallDepth, per = (all_steps + cranks - 1) / cranks;
    const int step0 = min(crank * per, all_steps), steps = min(per, all_steps - step0);
    volatile int* gave_up = &sh.gave_up;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kTallMostStages; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], 1);
        }
        mbar_init(&sh.done, 1);
        sh.gave_up = 0;
        mbar_fence_init();
    }
    if (warp == 2) {
        tc_alloc<false>(&sh.tmem, (uint32_t)f.columns);
        tc_fence_before();
    }
    if (threadIdx.x < kTallTokens) sh.sum[threadIdx.x] = 0.0f;
    for (int i = threadIdx.x; i < kTallTokens * stride; i += kTallThreads) part[i] = 0.0f;
    // ones: bf16 0x3F80, fp16 0x3C00
    for (int i = threadIdx.x; i < f.stages * f.lead * 8; i += kTallThreads) {
        const uint32_t one = BF16 ? 0x3F803F80u : 0x3C003C00u;
        *reinterpret_cast<uint4*>(ring + (i / (f.lead * 8)) * stage_bytes + kTallLeftBytes + (i % (f.lead * 8)) * 16) = make_uint4(one, one, one, one);
    }
    tc_publish();
    __syncthreads();
    tc_fence_after();
    find_adapters<kTallTokens>(a, t0, sh.ids);
    if (threadIdx.x < kTallTokens) {
        const int id = sh.ids[threadIdx.x];
        sh.scale[threadIdx.x] = id < 0 ? 0.0f : a.scale ? a.scale[id] : 1.0f;
    }
    if (warp == 0) {
        int mine[kTallTokens / 32], count = 0;
#pragma unroll
        for (int i = 0; i < kTallTokens / 32; ++i) mine[i] = f.slots > 0 ? sh.ids[lane + 32 * i] : -1;
        for (;;) {
            int least = 0x7fffffff;                                                   // (in the order of their numbers: every CTA of the cluster the same)
#pragma unroll
            for (int i = 0; i < kTallTokens / 32; ++i)
                if (mine[i] >= 0) least = min(least, mine[i]);
            least = __reduce_min_sync(0xffffffffu, least);
            if (least == 0x7fffffff) break;
#pragma unroll
            for (int i = 0; i < kTallTokens / 32; ++i)
                if (mine[i] == least) mine[i] = -1;
            if (lane == 0) sh.distinct[count] = least;
            ++count;
        }
        if (lane == 0) sh.count = count;
    }
    __syncthreads();
    const uint32_t tmem = sh.tmem;
    const int passes = max(f.slots > 0 ? (sh.count + f.slots - 1) / f.slots : 0, f.lead > 0 ? 1 : 0);

    if (warp == 0) {
        int n = 0;                                                                    // stages of all passes
        bool ok = true;
        const uint32_t first = smem_u32(ring);
        for (int p = 0; ok && p < passes; ++p) {
            const int used = max(min(f.slots, sh.count - p * f.slots), 0);
            for (int s = 0, slot = n % f.stages; s < steps; ++s, ++n, slot = slot + 1 == f.stages ? 0 : slot + 1) {
                if (n >= f.stages) ok = __all_sync(0xffffffffu, tc_wait(&sh.empty[slot], (n / f.stages - 1) & 1, gave_up, a.status, 110));
                if (!ok) break;
                const uint32_t at = first + slot * stage_bytes;
                if (tc_elect()) {
                    mbar_arrive_expect_tx(&sh.full[slot], kTallLeftBytes + (uint32_t)(used * f.ranks8 * 128));
                    tc_copy_2d(at, &z_map, (step0 + s) * kTallDepth, (int)t0, &sh.full[slot]);
                    for (int i = 0; i < used; ++i)
                        tc_copy_2d(at + kTallLeftBytes + (f.lead + i * f.ranks8) * 128, &down_map, (step0 + s) * kTallDepth, sh.distinct[p * f.slots + i] * a.rank, &sh.full[slot]);
                }
                __syncwarp();
            }
        }
    } else if (warp == 1) {
        int n = 0;
        bool ok = true;
        const uint64_t z_at = tc_operand(smem_u32(ring), 16, 1024), d_at = tc_operand(smem_u32(ring + kTallLeftBytes), 16, 1024);
        for (int p = 0; p < passes; ++p) {                                            // (every pass's barrier, whether or not a wait has given up)
            const int used = max(min(f.slots, sh.count - p * f.slots), 0);
            const int n16 = f.pass_columns(used), sets = f.pass_sets(used);
            const uint32_t kind = tc_kind(BF16, false, kTallTokens, n16);
            // (the pass before has to have been read out of tensor memory)
            if (p > 0) asm volatile("bar.sync 1, %0;" ::"n"(32 * 5) : "memory");
            tc_fence_after();
            for (int s = 0; ok && s < steps; ++s, ++n) {
                const int slot = n % f.stages;
                ok = __all_sync(0xffffffffu, tc_wait(&sh.full[slot], (n / f.stages) & 1, gave_up, a.status, 111));
                if (!ok) break;
                tc_fence_after();
                const uint64_t offset = (uint64_t)((uint32_t)slot * (stage_bytes / 16));
                if (tc_elect()) {
#pragma unroll
                    for (int k = 0; k < kTallDepth / 16; ++k) tc_mma<false>(tmem + (s % sets) * n16, z_at + offset + k * 2, d_at + offset + k * 2, kind, s >= sets || k > 0);
                    tc_commit<false>(&sh.empty[slot]);
                }
                __syncwarp();
            }
            if (tc_elect()) tc_commit<false>(&sh.done);
            __syncwarp();
        }
    } else if (warp >= 4) {
        const int quarter = warp - 4, row = quarter * 32 + lane, id = sh.ids[row];
        bool ok = true;
        for (int p = 0; p < passes; ++p) {
            const int used = max(min(f.slots, sh.count - p * f.slots), 0);
            ok = __all_sync(0xffffffffu, ok && tc_wait(&sh.done, p & 1, gave_up, a.status, 112));
            if (ok && steps > 0) {
                tc_fence_after();
                const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16);
                const int n16 = f.pass_columns(used), sets = min(f.pass_sets(used), steps);
                const auto add_sets = [&](int column, float (&y)[8]) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = 0.0f;
                    for (int set = 0; set < sets; ++set) {
                        uint32_t v[8];
                        tc_load8(at + set * n16 + column, v);
                        tc_load_wait();
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] += __uint_as_float(v[k]);
                    }
                };
                float y[8];
                if (f.lead > 0 && p == 0) {
                    add_sets(0, y);
                    sh.sum[row] = y[0];
                }
                for (int i = 0; i < used; ++i) {
                    const bool mine = sh.distinct[p * f.slots + i] == id;
                    for (int r = 0; r < f.ranks8; r += 8) {
                        add_sets(f.lead + i * f.ranks8 + r, y);
                        if (mine) {
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                if (r + k < a.rank) part[row * stride + r + k] = y[k];
                        }
                    }
                }
                tc_fence_before();
            }
            if (p + 1 < passes) asm volatile("bar.sync 1, %0;" ::"n"(32 * 5) : "memory");
        }
    }
    __syncthreads();
    if (*gave_up) tc_settle();
    if (warp == 2) {
        tc_fence_after();
        tc_free<false>(tmem, (uint32_t)f.columns);
    }
    cluster.sync();
    // The cluster's sums: every CTA a block of the tokens, a thread some ranks of one (what it needs of the others is on its way together), then
    // a thread a token.
    const int most = kTallTokens / cranks, row0 = crank * most;
    if (f.slots > 0) {
        // (a lane a rank, four of a warp's rows at a time)
        constexpr int N = 4, W = kTallThreads / 32;
        for (int r = lane; r < a.rank; r += 32)
            for (int first = row0 + warp; first < row0 + most; first += N * W) {
                float s[N] = {};
                for (int c = 0; c < cranks; ++c) {
                    const float* p = cluster.map_shared_rank(part, c) + r;
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        if (first + k * W < row0 + most) s[k] += p[(first + k * W) * stride];
                }
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const int row = first + k * W;
                    if (row >= row0 + most || sh.ids[row] == kNoRequest) continue;
                    const float y = s[k] * sh.scale[row];                             // (zero for tokens without an adapter)
                    a.hidden[(t0 + row) * a.rank + r] = y;
                    part[row * stride + r] = y;                                       // (no other CTA reads these)
                }
            }
        __syncthreads();
    }
    if ((int)threadIdx.x < most && t0 + row0 + (int)threadIdx.x < a.tokens) {
        const int row = row0 + (int)threadIdx.x, id = sh.ids[row];
        const int64_t t = t0 + row;
        a.ids[t] = id;
        if (f.slots > 0) {
            float top = 0.0f;
            for (int r = 0; r < a.rank; ++r) top = fmaxf(top, fabsf(part[row * stride + r]));
            a.hidden_scale[t] = 1.0f / scale_to_range(id == kNoRequest ? 0.0f : top);
        }
        if (f.lead > 0) {
            float s = 0.0f;
            for (int c = 0; c < cranks; ++c) s += cluster.map_shared_rank(sh.sum, c)[row];
            a.sum[t] = id == kNoRequest ? 0.0f : s;
        }
    }
    cluster.sync();
}

// ---------------------------------------------------------------------------------------------
// The backward pass's rows: sum z mid and the largest |z step| of a row, then z step 2^k in two parts (see split_scaled).  A CTA takes several
// rows, so that the grids' 8 bytes a column are read once for all of them; the second look at z finds it in L1 or L2.  Bound by HBM: z once
// in, twice out.  Nothing here needs what the kernel before it, which takes the same tokens onto their ranks, makes: it starts beside that
// one and ends after it, so that whoever waits for this kernel has waited for both.
// ---------------------------------------------------------------------------------------------
constexpr int kScaleRows = 4;
constexpr int kScaleThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kScaleThreads) scale_rows_kernel(ShrinkArgs a, int early) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ float sums[kScaleRows][kScaleThreads / 32], tops[kScaleRows][kScaleThreads / 32];
    const T* z = reinterpret_cast<const T*>(a.z);
    const int64_t t0 = (int64_t)blockIdx.x * kScaleRows;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool wide = ((reinterpret_cast<uintptr_t>(z) | (uintptr_t)(a.ldz * 2)) & 15) == 0;
    const bool wide_grid = ((reinterpret_cast<uintptr_t>(a.lo) | reinterpret_cast<uintptr_t>(a.step)) & 15) == 0;
    const auto load_grid = [&](const float* p, int j, int count, float (&v)[8]) {
        if (wide_grid && count == 8) {
            const float4 x = *reinterpret_cast<const float4*>(p + j), y = *reinterpret_cast<const float4*>(p + j + 4);
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < count ? p[j + i] : 0.0f;
        }
    };
    float sum[kScaleRows] = {}, top[kScaleRows] = {};
    for (int j = threadIdx.x * 8; j < a.columns; j += kScaleThreads * 8) {
        const int count = min(a.columns - j, 8);
        uint4 w[kScaleRows];
#pragma unroll
        for (int r = 0; r < kScaleRows; ++r) w[r] = t0 + r < a.tokens ? load8_16(z + (t0 + r) * a.ldz + j, count, wide) : make_uint4(0, 0, 0, 0);
        float lo[8], step[8];
        load_grid(a.lo, j, count, lo);
        load_grid(a.step, j, count, step);
#pragma unroll
        for (int i = 0; i < 8; ++i) lo[i] = fmaf(a.center, step[i], lo[i]);
#pragma unroll
        for (int r = 0; r < kScaleRows; ++r) {
            const uint32_t u[4] = {w[r].x, w[r].y, w[r].z, w[r].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 v = unpack_pair<T>(u[i]);
                sum[r] = fmaf(v.x, lo[2 * i], fmaf(v.y, lo[2 * i + 1], sum[r]));
                top[r] = fmaxf(top[r], fmaxf(fabsf(v.x * step[2 * i]), fabsf(v.y * step[2 * i + 1])));
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kScaleRows; ++r) {
        sum[r] = warp_sum(sum[r]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], o));
        if (lane == 0) { sums[r][warp] = sum[r]; tops[r][warp] = top[r]; }
    }
    __syncthreads();
    float scale[kScaleRows];
#pragma unroll
    for (int r = 0; r < kScaleRows; ++r) {
        float s = 0.0f, m = 0.0f;
#pragma unroll
        for (int w = 0; w < kScaleThreads / 32; ++w) { s += sums[r][w]; m = fmaxf(m, tops[r][w]); }
        scale[r] = scale_to_range(m);
        if (threadIdx.x == 0 && t0 + r < a.tokens) { a.sum[t0 + r] = s; a.row_scale[t0 + r] = 1.0f / scale[r]; }
    }
    for (int j = threadIdx.x * 8; j < a.columns; j += kScaleThreads * 8) {
        const int count = min(a.columns - j, 8);
        float step[8];
        load_grid(a.step, j, count, step);
#pragma unroll
        for (int r = 0; r < kScaleRows; ++r) {
            if (t0 + r >= a.tokens) break;
            const uint4 w = load8_16(z + (t0 + r) * a.ldz + j, count, wide);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
            uint32_t high[4], low[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 v = unpack_pair<T>(u[i]);
                split_scaled(v.x * step[2 * i] * scale[r], v.y * step[2 * i + 1] * scale[r], high[i], low[i]);
            }
            *reinterpret_cast<uint4*>(a.scaled + (t0 + r) * a.ld_scaled + j) = make_uint4(high[0], high[1], high[2], high[3]);
            *reinterpret_cast<uint4*>(a.scaled + (a.tokens + t0 + r) * a.ld_scaled + j) = make_uint4(low[0], low[1], low[2], low[3]);
        }
    }
    if (early) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Whether the kernel for many tokens takes them: rows that tensor copies can read, enough tokens to fill its tiles and few adapters in each.
static bool tall_takes(const ShrinkArgs& a) {
    if (a.tokens < 2 * kTallTokens || a.copy) return false;
    if ((reinterpret_cast<uintptr_t>(a.z) & 15) || a.ldz % 8) return false;
    if (a.down && ((reinterpret_cast<uintptr_t>(a.down) & 15) || a.columns % 8 || a.tokens < (int64_t)a.requests * 32)) return false;
    return true;
}

static int launch_tall(zipml_ctx* ctx, const ShrinkArgs& a, int dtype, bool sums) {
    TallShape f{};
    f.lead = sums ? 16 : 0;
    f.ranks8 = (a.rank + 7) / 8 * 8;
    if (a.down) {
        f.slots = 128 / f.ranks8;                        // (a tile that needs a second pass takes twice as long, and all wait for it)
        if (f.slots > a.adapters) f.slots = a.adapters;
        if (f.slots > a.requests) f.slots = a.requests;
    }
    f.rows = (f.lead + f.slots * f.ranks8 + 15) / 16 * 16;
    f.columns = f.rows > 0 ? 512 : 32;
    const size_t stage = kTallLeftBytes + (size_t)f.rows * 128, fixed = 1024 + sizeof(float) * kTallTokens * (a.rank | 1) + sizeof(TallShared);
    f.stages = (int)((200 * 1024 - fixed) / stage);
    if (f.stages > kTallMostStages) f.stages = kTallMostStages;
    const size_t smem = fixed + f.stages * stage;
    const int64_t tiles = (a.tokens + kTallTokens - 1) / kTallTokens;
    const int steps = (a.columns + kTallDepth - 1) / kTallDepth;
    int ranks = 1;
    while (ranks < 8 && tiles * ranks * 2 <= ctx->sm_count && steps / (ranks * 2) >= 4) ranks *= 2;
    CUtensorMap z_map{}, down_map{};
    const CUtensorMapDataType type = dtype == ZIPML_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    int rc = encode_map(ctx, type, a.z, a.columns, a.tokens, a.ldz * 2, kTallDepth, kTallTokens, CU_TENSOR_MAP_SWIZZLE_128B, &z_map);
    if (rc == ZIPML_OK && a.down)
        rc = encode_map(ctx, type, a.down, a.columns, (int64_t)a.adapters * a.rank, (int64_t)a.columns * 2, kTallDepth, f.ranks8, CU_TENSOR_MAP_SWIZZLE_128B, &down_map);
    if (rc != ZIPML_OK) return rc;
    auto kernel = dtype == ZIPML_BF16 ? &shrink_tall_kernel<true> : &shrink_tall_kernel<false>;
    rc = allow_shared(ctx, reinterpret_cast<const void*>(kernel), smem);
    if (rc != ZIPML_OK) return rc;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles * ranks));
    cfg.blockDim = dim3(kTallThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, f, z_map, down_map);
    ctx->launches += 1;
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError());
}

static int launch_scale_rows(zipml_ctx* ctx, const ShrinkArgs& a, int dtype) {
    const unsigned grid = (unsigned)((a.tokens + kScaleRows - 1) / kScaleRows);
    const int early = capturing(ctx) ? 0 : 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kScaleThreads);
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = (unsigned)early;
    const cudaError_t e = dtype == ZIPML_BF16 ? cudaLaunchKernelEx(&cfg, &scale_rows_kernel<__nv_bfloat16>, a, early)
                                              : cudaLaunchKernelEx(&cfg, &scale_rows_kernel<__half>, a, early);
    ctx->launches += 1;
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError());
}

template <typename T, bool BACK, int RT>
static int launch_shrink_as(zipml_ctx* ctx, const ShrinkArgs& a) {
    const size_t smem = (size_t)kShrinkWarps * kShrinkRows * RT * 8 * sizeof(float);
    auto kernel = &shrink_kernel<T, BACK, RT>;
    if (smem > 40 * 1024) {
        const int rc = allow_shared(ctx, reinterpret_cast<const void*>(kernel), smem);
        if (rc != ZIPML_OK) return rc;
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
    if (tall_takes(a)) {
        const int rc = launch_tall(ctx, a, dtype, !backward);
        return rc != ZIPML_OK || !backward || !a.scaled ? rc : launch_scale_rows(ctx, a, dtype);
    }
    if (dtype == ZIPML_BF16) return backward ? launch_shrink_ranks<__nv_bfloat16, true>(ctx, a) : launch_shrink_ranks<__nv_bfloat16, false>(ctx, a);
    return backward ? launch_shrink_ranks<__half, true>(ctx, a) : launch_shrink_ranks<__half, false>(ctx, a);
}

}  // namespace zipml
