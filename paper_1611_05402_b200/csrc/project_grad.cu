// Third stage of a projection's backward pass: the gradients of the low-rank adapters, grad_down = sum v (x) Q(x) over the 8-bit
// checkpoints as they lie and grad_up = sum hidden (x) dy, each over the tokens of its adapter.
#include <cooperative_groups.h>

#include "project.cuh"
#include "tensor_core.cuh"

namespace zipml {

namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------------------------
// A cluster takes one adapter and one block of columns (128 codes or 64 values of dy: 128 bytes of each row), its CTAs' warps the adapter's
// tokens in chunks of 32 in turn.  Every warp has slots of 4 KB of its own and keeps them on their way (tensor copies with the 128-byte
// swizzle; rows of dy that these cannot take are read straight from global memory): nothing is handed from warp to warp before the
// end.  m16n8k8 products in tf32, ranks x columns x tokens: codes (code - 128) and 16-bit values are exact in its 11 bits, v step and
// hidden are split into two such parts, so a product keeps 22 bits.  A lane reads 16 consecutive bytes of the rows of two tokens; byte f of
// eight lanes is the f-th block of columns.  The two tokens of a lane are neighbours, which with the swizzle is free of bank
// conflicts.  The lower ends' share, v . (lo + 128 step), is the same for a group's columns and is summed once per group.  Warps' and CTAs'
// sums are added in a fixed order.
// ---------------------------------------------------------------------------------------------
constexpr int kGradWarps = 8;
constexpr int kGradThreads = 32 * kGradWarps;
constexpr int kGradChunk = 32;                          // tokens
constexpr uint32_t kGradSlotBytes = kGradChunk * 128;
constexpr int kGradBatch = kGradThreads;                // requests that are looked at together
// Slots of a warp: two CTAs of an SM for up to 16 ranks, one (by its registers) for 32.
__host__ __device__ constexpr int grad_slots(int mt) { return mt == 1 ? 3 : 6; }
static_assert(3 * kGradSlotBytes >= 16 * 128 * sizeof(float) && 6 * kGradSlotBytes >= 32 * 128 * sizeof(float), "a warp's sums fit its slots");
constexpr int kGradMostSlots = 6;

struct GradShared {
    uint64_t full[kGradWarps][kGradMostSlots];
    int gave_up;
    int found[kGradWarps];
    int segments;
    int begin[kGradBatch], end[kGradBatch];             // this adapter's token ranges among the batch's requests
};

__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&x)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(b0), "r"(b1));
}
// The same with both parts of the left factor, (low + high) x b of 8 tokens from zero, which is then added in fp32: the tensor cores cut
// what they add to a sum where fp32 would round, always towards zero, and sums over thousands of tokens would show it.  (2048 tokens: 2.3e-6
// of the result off when the sums stayed in the tensor cores, 0.2e-6 so, for 8 % of the kernel's time.)
__device__ __forceinline__ void add_products(float (&d)[4], const uint32_t (&high)[4], const uint32_t (&low)[4], uint32_t b0, uint32_t b1) {
    float t[4];
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(t[0]), "=f"(t[1]), "=f"(t[2]), "=f"(t[3]) : "r"(low[0]), "r"(low[1]), "r"(low[2]), "r"(low[3]), "r"(b0), "r"(b1), "f"(0.0f));
    mma_tf32(t, high, b0, b1);
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] += t[i];
}
// The same where the right factor has two parts too (the product of the low ones is below what is kept).
__device__ __forceinline__ void add_products(float (&d)[4], const uint32_t (&high)[4], const uint32_t (&low)[4], float b0, float b1) {
    const uint32_t h0 = __float_as_uint(b0) & 0xffffe000u, h1 = __float_as_uint(b1) & 0xffffe000u;
    float t[4];
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(t[0]), "=f"(t[1]), "=f"(t[2]), "=f"(t[3]) : "r"(low[0]), "r"(low[1]), "r"(low[2]), "r"(low[3]), "r"(h0), "r"(h1), "f"(0.0f));
    mma_tf32(t, high, __float_as_uint(b0 - __uint_as_float(h0)), __float_as_uint(b1 - __uint_as_float(h1)));
    mma_tf32(t, high, h0, h1);
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] += t[i];
}
// byte i of a word, less 128 (see byte_to_float)
__device__ __forceinline__ float centred_code(uint32_t bytes, int i) { return __uint_as_float(__byte_perm(bytes, 0x4B000000u, 0x7650 + i)) - 8388736.0f; }
// x = high + low, both within tf32's 11 bits up to 2^-22 of x
__device__ __forceinline__ void split_tf32(float x, uint32_t& high, uint32_t& low) {
    high = __float_as_uint(x) & 0xffffe000u;
    low = __float_as_uint(x - __uint_as_float(high));
}

// What stands on the right: the values of dy; codes on one grid a token for the whole block (groups of 128 features and more), whose step goes to
// the left and whose lower end is summed apart; or codes of narrower groups, as the values they stand for.
enum GradRight { kDy = 0, kCodes = 1, kValues = 2 };

// The left factors of 8 tokens and their grids, as a lane needs them: ranks g and g + 8 of each block, tokens 2 q and 2 q + 1.
template <int MT>
struct GradLeft {
    float v[MT][4];
    float2 grid[2];
};

// MT: blocks of 16 ranks, 1 or 2 (registers); higher ranks read the rows once for each 32.
template <int RIGHT, int MT>
__device__ __forceinline__ void grad_pass(const GradArgs& a, const CUtensorMap* map, int adapter, int block, int r0, uint8_t* ring, GradShared& sh,
                                          cg::cluster_group& cluster) {
    constexpr bool CODES = RIGHT != kDy;
    constexpr int NF = CODES ? 16 : 8;                     // columns of a lane's 16 bytes
    constexpr int SLOTS = grad_slots(MT);
    using Left = GradLeft<MT>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int ranks = (int)cluster.num_blocks(), crank = (int)cluster.block_rank();
    const int columns = CODES ? a.inputs : a.outputs;
    const int col0 = block * NF * 8, lane_col = col0 + g * NF;
    const bool copied = CODES || a.dy_copied;
    const float* left = CODES ? a.v : a.hidden;
    const int grid_at = CODES ? (RIGHT == kValues ? min(lane_col, columns - 1) : col0) / a.group : 0;
    volatile int* gave_up = &sh.gave_up;
    uint8_t* slots = ring + warp * SLOTS * kGradSlotBytes;
    float acc[MT][NF][4] = {};
    float base[MT][2] = {};
    const int others = ranks * kGradWarps, me = crank * kGradWarps + warp; // (a power of two of warps take the chunks in turn)
    bool any = false;                                      // has this adapter tokens?
    bool lost = false;                                     // a copy of this warp's has not come: no further ones
    int turn = 0;                                          // chunks of the batches so far, of all warps
    uint32_t taken = 0, issued = 0;                        // of this one
    for (int first = 0; first < a.requests; first += kGradBatch) {
        // the batch's requests of this adapter, in order
        __syncthreads();
        {
            const int req = first + (int)threadIdx.x;
            int s = 0, e = 0;
            const int which = req < a.requests ? a.which[req] : -1;
            if (which == adapter || which >= a.adapters) {
                s = max(a.starts[req], 0);
                e = (int)min((int64_t)a.starts[req + 1], a.tokens);
            }
            if (which >= a.adapters) {                     // (the first stage reports it too, but a call that wants grad_up alone has none)
                if (e > s) set_status(a.status, ZIPML_ERR_INVALID_ARG, 91);
                e = s;
            }
            const uint32_t has = __ballot_sync(0xffffffffu, e > s);
            if (lane == 0) sh.found[warp] = __popc(has);
            __syncthreads();
            int at = __popc(has & ((1u << lane) - 1u));
            for (int w = 0; w < warp; ++w) at += sh.found[w];
            if (e > s) { sh.begin[at] = s; sh.end[at] = e; }
            if (threadIdx.x == kGradThreads - 1) sh.segments = at + (e > s);
        }
        __syncthreads();
        const int segments = sh.segments;
        any |= segments > 0;
        struct Cursor { int i, c, turn; };                 // chunk c of range i, the turn-th of all warps' chunks
        const auto settle = [&](Cursor& at) {              // on to the next chunk that is this warp's
            while (at.i < segments) {
                const int chunks = (sh.end[at.i] - sh.begin[at.i] + kGradChunk - 1) / kGradChunk;
                const int skip = (me - at.turn) & (others - 1);
                if (at.c + skip < chunks) { at.c += skip; at.turn += skip; return; }
                at.turn += chunks - at.c;
                ++at.i;
                at.c = 0;
            }
        };
        const auto step = [&](Cursor& at) { ++at.c; ++at.turn; settle(at); };
        Cursor ahead{0, 0, turn};
        const auto issue = [&] {                           // (into the slot that was read longest ago, by this warp)
            if (lost || ahead.i >= segments) return;
            const uint32_t slot = issued % SLOTS;
            if (tc_elect()) {
                mbar_arrive_expect_tx(&sh.full[warp][slot], kGradSlotBytes);
                tc_copy_2d(smem_u32(slots + slot * kGradSlotBytes), map, col0, sh.begin[ahead.i] + ahead.c * kGradChunk, &sh.full[warp][slot]);
            }
            __syncwarp();
            ++issued;
            step(ahead);
        };
        if (copied) {
            settle(ahead);
            for (int k = 0; k < SLOTS; ++k) issue();
        }
        const auto load_left = [&](Left& l, int t, int e) {
            const bool in0 = t < e, in1 = t + 1 < e;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int ra = r0 + m * 16 + g, rb = ra + 8;
                const float* p = left + (int64_t)t * a.rank;
                l.v[m][0] = in0 && ra < a.rank ? p[ra] : 0.0f;
                l.v[m][1] = in0 && rb < a.rank ? p[rb] : 0.0f;
                l.v[m][2] = in1 && ra < a.rank ? p[a.rank + ra] : 0.0f;
                l.v[m][3] = in1 && rb < a.rank ? p[a.rank + rb] : 0.0f;
            }
            if constexpr (CODES) {
                const float2 none = make_float2(0.0f, 0.0f);
                const float2* p = a.grids + (int64_t)t * a.groups + grid_at;
                l.grid[0] = in0 ? p[0] : none;
                l.grid[1] = in1 ? p[a.groups] : none;
            }
        };
        Left next;
        Cursor at{0, 0, turn};
        settle(at);
        if (at.i < segments) load_left(next, sh.begin[at.i] + at.c * kGradChunk + 2 * q, sh.end[at.i]);
        while (at.i < segments) {
            const int t0 = sh.begin[at.i] + at.c * kGradChunk, e = sh.end[at.i];
            step(at);
            const uint32_t slot = taken % SLOTS;
            lost = lost || (copied && !__all_sync(0xffffffffu, tc_wait(&sh.full[warp][slot], (taken / SLOTS) & 1, gave_up, a.status, 108)));
            if (lost) break;
#pragma unroll 1
            for (int tt = 0; tt < kGradChunk && t0 + tt < e; tt += 8) {
                const Left l = next;
                const int t = t0 + tt + 2 * q;
                const bool in0 = t < e, in1 = t + 1 < e;
                if (tt + 8 < kGradChunk && t0 + tt + 8 < e) load_left(next, t + 8, e);
                else if (at.i < segments) load_left(next, sh.begin[at.i] + at.c * kGradChunk + 2 * q, sh.end[at.i]);
                uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0;
                if (copied) {
                    const uint8_t* p = slots + slot * kGradSlotBytes + (tt + 2 * q) * 128;
                    w0 = *reinterpret_cast<const uint4*>(p + ((g ^ (2 * q)) << 4));
                    w1 = *reinterpret_cast<const uint4*>(p + 128 + ((g ^ (2 * q + 1)) << 4));
                } else {
                    const uint16_t* dy = reinterpret_cast<const uint16_t*>(a.dy) + (int64_t)t * a.lddy + lane_col;
                    const int count = min(max(columns - lane_col, 0), 8);
                    if (in0) w0 = load8_16(dy, count, false);
                    if (in1) w1 = load8_16(dy + a.lddy, count, false);
                }
                if (!CODES) {                              // (what lies behind the range belongs to others and need not be finite)
                    if (!in0) w0 = make_uint4(0, 0, 0, 0);
                    if (!in1) w1 = make_uint4(0, 0, 0, 0);
                }
                const uint32_t u0[4] = {w0.x, w0.y, w0.z, w0.w}, u1[4] = {w1.x, w1.y, w1.z, w1.w};
                if constexpr (CODES) {
                    const float2 g0 = l.grid[0], g1 = l.grid[1];
                    uint32_t hi[MT][4], lo[MT][4];
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const float s0 = RIGHT == kCodes ? g0.y : 1.0f, s1 = RIGHT == kCodes ? g1.y : 1.0f;
                        split_tf32(l.v[m][0] * s0, hi[m][0], lo[m][0]);
                        split_tf32(l.v[m][1] * s0, hi[m][1], lo[m][1]);
                        split_tf32(l.v[m][2] * s1, hi[m][2], lo[m][2]);
                        split_tf32(l.v[m][3] * s1, hi[m][3], lo[m][3]);
                        if constexpr (RIGHT == kCodes) {
                            const float m0 = fmaf(128.0f, g0.y, g0.x), m1 = fmaf(128.0f, g1.y, g1.x);
                            base[m][0] += fmaf(l.v[m][0], m0, l.v[m][2] * m1);
                            base[m][1] += fmaf(l.v[m][1], m0, l.v[m][3] * m1);
                        }
                    }
#pragma unroll
                    for (int f = 0; f < NF; ++f) {
                        if constexpr (RIGHT == kCodes) {
                            const uint32_t b0 = __float_as_uint(centred_code(u0[f >> 2], f & 3)), b1 = __float_as_uint(centred_code(u1[f >> 2], f & 3));
#pragma unroll
                            for (int m = 0; m < MT; ++m) add_products(acc[m][f], hi[m], lo[m], b0, b1);
                        } else {
                            const float b0 = fmaf(byte_to_float(u0[f >> 2], f & 3), g0.y, g0.x), b1 = fmaf(byte_to_float(u1[f >> 2], f & 3), g1.y, g1.x);
#pragma unroll
                            for (int m = 0; m < MT; ++m) add_products(acc[m][f], hi[m], lo[m], b0, b1);
                        }
                    }
                } else {
                    uint32_t hi[MT][4], lo[MT][4];
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int k = 0; k < 4; ++k) split_tf32(l.v[m][k], hi[m][k], lo[m][k]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 b0 = a.bf16 ? unpack_pair<__nv_bfloat16>(u0[k]) : unpack_pair<__half>(u0[k]);
                        const float2 b1 = a.bf16 ? unpack_pair<__nv_bfloat16>(u1[k]) : unpack_pair<__half>(u1[k]);
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            add_products(acc[m][2 * k], hi[m], lo[m], __float_as_uint(b0.x), __float_as_uint(b1.x));
                            add_products(acc[m][2 * k + 1], hi[m], lo[m], __float_as_uint(b0.y), __float_as_uint(b1.y));
                        }
                    }
                }
            }
            if (copied) {
                __syncwarp();
                ++taken;
                issue();
            }
        }
        turn = at.turn;
    }
    if constexpr (RIGHT == kCodes) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float s = base[m][i];
                s += __shfl_xor_sync(0xffffffffu, s, 1);
                s += __shfl_xor_sync(0xffffffffu, s, 2);
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    acc[m][f][2 * i] += s;
                    acc[m][f][2 * i + 1] += s;
                }
            }
    }
    constexpr int C = NF * 8;
    float* out = (CODES ? a.grad_down : a.grad_up) + ((int64_t)adapter * a.rank + r0) * columns + col0;
    const int most = min(16 * MT, a.rank - r0);
    if (!any) {                                            // (for all CTAs of the cluster)
        for (int i = crank * kGradThreads + threadIdx.x; i < most * C; i += ranks * kGradThreads)
            if (col0 + i % C < columns) out[(int64_t)(i / C) * columns + i % C] = 0.0f;
        return;
    }
    // Sums over the warps, then over the CTAs: [warp][rank][column] in the slots' place, 16 bytes at a position that the eight lanes of a
    // store share no bank in.
    float* sums = reinterpret_cast<float*>(ring);
    const auto place = [](int r, int col) { return r * C + (((col >> 2) ^ ((col >> (CODES ? 5 : 4)) & 3) ^ ((r & 1) << 2)) << 2) + (col & 3); };
    __syncthreads();                                       // (the slots have been read)
    if (*gave_up) tc_settle();
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int f = 0; f < NF; f += 4)
                *reinterpret_cast<float4*>(sums + warp * 16 * MT * C + place(m * 16 + g + 8 * (i >> 1), (2 * q + (i & 1)) * NF + f)) =
                    make_float4(acc[m][f][i], acc[m][f + 1][i], acc[m][f + 2][i], acc[m][f + 3][i]);
    __syncthreads();
    const auto of_warps = [&](int i) {
        float s = sums[i];
#pragma unroll
        for (int w = 1; w < kGradWarps; ++w) s += sums[w * 16 * MT * C + i];
        return s;
    };
    if (ranks == 1) {
        for (int i = threadIdx.x; i < most * C; i += kGradThreads)
            if (col0 + i % C < columns) out[(int64_t)(i / C) * columns + i % C] = of_warps(place(i / C, i % C));
        return;
    }
    for (int i = threadIdx.x; i < 16 * MT * C; i += kGradThreads) sums[i] = of_warps(i);
    cluster.sync();
    for (int i = crank * kGradThreads + threadIdx.x; i < most * C; i += ranks * kGradThreads) {
        float s = 0.0f;
        for (int c = 0; c < ranks; ++c) s += cluster.map_shared_rank(sums, c)[place(i / C, i % C)];
        if (col0 + i % C < columns) out[(int64_t)(i / C) * columns + i % C] = s;
    }
    cluster.sync();
}

template <int MT>
__global__ void __launch_bounds__(kGradThreads, MT == 1 ? 2 : 1) grad_kernel(GradArgs a, const __grid_constant__ CUtensorMap codes_map, const __grid_constant__ CUtensorMap dy_map) {
    extern __shared__ uint8_t raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    GradShared& sh = *reinterpret_cast<GradShared*>(ring + kGradWarps * grad_slots(MT) * kGradSlotBytes);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kGradWarps * kGradMostSlots; ++i) mbar_init(&sh.full[0][0] + i, 1);
        sh.gave_up = 0;
        mbar_fence_init();
    }
    cg::cluster_group cluster = cg::this_cluster();
    const int block = blockIdx.x / cluster.num_blocks(), adapter = blockIdx.y, r0 = blockIdx.z * MT * 16;
    if (block >= a.down_blocks) grad_pass<kDy, MT>(a, &dy_map, adapter, block - a.down_blocks, r0, ring, sh, cluster);
    else if (a.group >= 128) grad_pass<kCodes, MT>(a, &codes_map, adapter, block, r0, ring, sh, cluster);
    else grad_pass<kValues, MT>(a, &codes_map, adapter, block, r0, ring, sh, cluster);
}

template <int MT>
static int launch_grad_as(zipml_ctx* ctx, const GradArgs& a, const CUtensorMap& codes_map, const CUtensorMap& dy_map) {
    const int blocks = a.down_blocks + a.up_blocks, passes = (a.rank + MT * 16 - 1) / (MT * 16);
    const size_t smem = 1024 + kGradWarps * grad_slots(MT) * kGradSlotBytes + sizeof(GradShared);
    const int rc = allow_shared(ctx, reinterpret_cast<const void*>(&grad_kernel<MT>), smem);
    if (rc != ZIPML_OK) return rc;
    int ranks = 1;
    // (as many CTAs as the GPU holds at a time: two an SM for up to 16 ranks, one for more)
    const int busy = a.adapters < a.requests ? a.adapters : a.requests;
    while (ranks < 8 && (int64_t)blocks * busy * passes * ranks < (MT == 1 ? 2 : 1) * ctx->sm_count && (int64_t)ranks * kGradWarps * kGradChunk < a.tokens) ranks *= 2;
    if (a.adapters > 65535 || (int64_t)blocks * ranks > 0x7fffffffLL) return ZIPML_ERR_WORKSPACE;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(blocks * ranks), (unsigned)a.adapters, (unsigned)passes);
    cfg.blockDim = dim3(kGradThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, &grad_kernel<MT>, a, codes_map, dy_map);
    ctx->launches += 1;
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError());
}

int launch_project_grad(zipml_ctx* ctx, const GradArgs& in) {
    GradArgs a = in;
    a.down_blocks = a.grad_down ? (a.inputs + 127) / 128 : 0;
    a.up_blocks = a.grad_up ? (a.outputs + 63) / 64 : 0;
    if (a.down_blocks + a.up_blocks == 0 || a.adapters == 0) return ZIPML_OK;
    if (a.tokens > 0x7fffffffLL) return ZIPML_ERR_WORKSPACE;
    CUtensorMap codes_map{}, dy_map{};
    if (a.grad_down && a.tokens > 0) {
        const int rc = encode_map(ctx, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.codes, a.code_stride, a.tokens, a.code_stride, 128, kGradChunk, CU_TENSOR_MAP_SWIZZLE_128B,
                                  &codes_map);
        if (rc != ZIPML_OK) return rc;
    }
    a.dy_copied = (reinterpret_cast<uintptr_t>(a.dy) & 15) == 0 && a.lddy % 8 == 0;
    if (a.grad_up && a.tokens > 0 && a.dy_copied) {
        const int rc = encode_map(ctx, CU_TENSOR_MAP_DATA_TYPE_UINT16, a.dy, a.outputs, a.tokens, a.lddy * 2, 64, kGradChunk, CU_TENSOR_MAP_SWIZZLE_128B, &dy_map);
        if (rc != ZIPML_OK) return rc;
    }
    return a.rank <= 16 ? launch_grad_as<1>(ctx, a, codes_map, dy_map) : launch_grad_as<2>(ctx, a, codes_map, dy_map);
}

}  // namespace zipml
