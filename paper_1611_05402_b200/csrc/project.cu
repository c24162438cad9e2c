// Second stage of a projection with low-rank adapters: tokens times packed codes on the tensor cores, the adapters' products beside it
// in the same launch, the codes' grids in the epilogue.
#include <type_traits>

#include <cooperative_groups.h>

#include "project.cuh"
#include "tensor_core.cuh"

namespace zipml {

namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------------------------
// A CTA makes 128 features x NT tokens.  The features stand on the product's 128 rows and the tokens on its columns, so one
// kernel serves from a token (16 columns, the codes' bytes are what counts) to thousands.  Per 64 of the depth:
//   codes     a tensor copy brings the packed codes; eight warps turn them into 16-bit whole numbers code - 2^(cb-1), which are exact, and
//             lay them out as the product's left operand.  Forward: a code row is one depth and holds the features (MN-major
//             operand); backward: a code row is a feature (K-major).
//   tokens    a tensor copy lays the right operand out itself.
//   product   one thread issues 128 x NT x 16 four times, sums in tensor memory.
// The adapters then take further stages of the same ring: up_i's rows are the left operand as they lie, hidden the right one, in two
// 16-bit parts (high and low: 16 or more bits), zero for tokens of other adapters, over the 16-token window that holds i's tokens.  Their
// sums have columns of their own, since the grids' steps do not apply to them.
// The epilogue takes steps, sums and scales together in fp32 and rounds once.  With few tokens a cluster's CTAs divide the depth and
// add their results through each other's shared memory in a fixed order.
// ---------------------------------------------------------------------------------------------
constexpr int kProjRows = 128;                // features of a CTA
constexpr int kProjDepth = 64;                // depth of a stage: 128 bytes of 16-bit operand
constexpr int kUnpackWarps = 8;
constexpr int kProjThreads = 32 * (4 + kUnpackWarps);
constexpr int kRankChunk = 32;                // ranks of an adapter stage: high parts in the first half of the depth, low ones in the second
constexpr uint32_t kABytes = kProjRows * kProjDepth * 2;

template <int NT>
struct ProjShape {
    static constexpr int kStages = NT == 16 ? 6 : NT == 64 ? 5 : 4;
    static constexpr int kCodeStages = NT == 256 ? 3 : NT == 128 ? 6 : 8;
    static constexpr uint32_t kBBytes = NT * kProjDepth * 2;
    static constexpr uint32_t kCodeBytes = kProjRows * kProjDepth;      // 8-bit codes; narrower ones fill a part
    static constexpr uint32_t kRing = kStages * (kABytes + kBBytes) + kCodeStages * kCodeBytes;
    static constexpr uint32_t kColumns = NT == 16 ? 32 : 2 * NT;        // tensor memory: codes' sums, then adapters'
};

template <int NT>
struct ProjShared {
    uint64_t tokens_full[8], codes_full[8], operand_full[8], empty[8], codes_empty[8], done, plan;
    uint32_t tmem;
    int gave_up;
    int entries;                              // adapters of this tile that fall to this CTA
    int entry_id[NT], entry_lo[NT], entry_n[NT];
    int ids[NT];
    float sum[NT], row_scale[NT], hidden_scale[NT];
};

// Sixteen packed codes as bytes.
template <int CB>
__device__ __forceinline__ void codes_to_bytes(const uint8_t* p, uint32_t (&w)[4]) {
    if constexpr (CB == 8) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (CB == 4) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        const uint32_t u[2] = {v.x, v.y};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t even = u[i] & 0x0F0F0F0Fu, odd = (u[i] >> 4) & 0x0F0F0F0Fu;
            w[2 * i] = __byte_perm(even, odd, 0x5140);
            w[2 * i + 1] = __byte_perm(even, odd, 0x7362);
        }
    } else {
        const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
        uint32_t t[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = (v >> (2 * k)) & 0x03030303u;
        const uint32_t a0 = __byte_perm(t[0], t[1], 0x5140), a1 = __byte_perm(t[2], t[3], 0x5140);
        const uint32_t b0 = __byte_perm(t[0], t[1], 0x7362), b1 = __byte_perm(t[2], t[3], 0x7362);
        w[0] = __byte_perm(a0, a1, 0x5410); w[1] = __byte_perm(a0, a1, 0x7632);
        w[2] = __byte_perm(b0, b1, 0x5410); w[3] = __byte_perm(b0, b1, 0x7632);
    }
}

// Two codes, in the low bytes of p's halves under the byte of 128 (bf16) or 1024 (fp16), as code - 2^(CB-1): the code is the mantissa's
// lowest bits, and one exact subtraction takes the offset away.  (bf16's mantissa has 7 bits: an 8-bit code's top bit would count as
// exponent, so it chooses between 128 and 256 on the other side.)
template <bool BF16, int CB>
__device__ __forceinline__ uint32_t centred_pair(uint32_t p) {
    if constexpr (BF16) {
        uint32_t a = p, b = CB == 4 ? 0x43084308u : 0x43024302u;
        if constexpr (CB == 8) {
            a = p & 0xff7fff7fu;
            b = (p & 0x00800080u) ^ 0x43804380u;
        }
        const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const uint32_t b = CB == 8 ? 0x64806480u : CB == 4 ? 0x64086408u : 0x64026402u;
        const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&p), *reinterpret_cast<const __half2*>(&b));
        return *reinterpret_cast<const uint32_t*>(&v);
    }
}
template <bool BF16, int CB>
__device__ __forceinline__ uint4 centred_chunk(uint32_t w0, uint32_t w1) {      // 8 codes
    constexpr uint32_t kTop = BF16 ? 0x43434343u : 0x64646464u;
    return make_uint4(centred_pair<BF16, CB>(__byte_perm(w0, kTop, 0x4140)), centred_pair<BF16, CB>(__byte_perm(w0, kTop, 0x4342)),
                      centred_pair<BF16, CB>(__byte_perm(w1, kTop, 0x4140)), centred_pair<BF16, CB>(__byte_perm(w1, kTop, 0x4342)));
}

// One stage's codes into the left operand, two units of 16 codes a thread.  Bank conflicts: eight lanes store 16 bytes each at a time;
// forward they hold one depth's 8 units, whose first halves would meet in pairs 8 KB apart, so the upper 64 features store their second
// half first.
template <bool BF16, int CB, bool BACK>
__device__ __forceinline__ void unpack_stage(const uint8_t* codes, uint8_t* operand, int uid) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int u = uid + i * 32 * kUnpackWarps;
        uint32_t w[4];
        codes_to_bytes<CB>(codes + u * 2 * CB, w);
        const uint4 first = centred_chunk<BF16, CB>(w[0], w[1]), second = centred_chunk<BF16, CB>(w[2], w[3]);
        if constexpr (BACK) {
            const int row = u >> 2, chunk = 2 * (u & 3);                        // 16 of the depth of one feature
            uint8_t* p = operand + row * 128;
            *reinterpret_cast<uint4*>(p + ((chunk ^ (row & 7)) << 4)) = first;
            *reinterpret_cast<uint4*>(p + (((chunk + 1) ^ (row & 7)) << 4)) = second;
        } else {
            const int k = u >> 3, f16 = u & 7, chunk = 2 * (f16 & 3);           // 16 features of one depth
            uint8_t* p = operand + (f16 >> 2) * (kABytes / 2) + k * 128;
            const bool swap = f16 >= 4;
            *reinterpret_cast<uint4*>(p + (((chunk + swap) ^ (k & 7)) << 4)) = swap ? second : first;
            *reinterpret_cast<uint4*>(p + (((chunk + !swap) ^ (k & 7)) << 4)) = swap ? first : second;
        }
    }
}

// A 16-bit pair with what is not finite replaced by zero.
__device__ __forceinline__ uint32_t finite_pair(uint32_t w, uint32_t exponent, bool& bad) {
    if ((w & exponent) == exponent) { w &= 0xffff0000u; bad = true; }
    if ((w & (exponent << 16)) == (exponent << 16)) { w &= 0x0000ffffu; bad = true; }
    return w;
}

template <int NT, bool BACK, bool BF16>
__global__ void __launch_bounds__(kProjThreads, 1) project_kernel(ProjectArgs a, const __grid_constant__ CUtensorMap tokens_map,
                                                                  const __grid_constant__ CUtensorMap codes_map) {
    using Shape = ProjShape<NT>;
    constexpr int S = Shape::kStages, CS = Shape::kCodeStages;
    extern __shared__ uint8_t raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    ProjShared<NT>& sh = *reinterpret_cast<ProjShared<NT>*>(ring + Shape::kRing);
    uint8_t* const left = ring;                                       // S x 16 KB
    uint8_t* const right = ring + S * kABytes;
    uint8_t* const packed = right + S * Shape::kBBytes;
    cg::cluster_group cluster = cg::this_cluster();
    const int crank = (int)cluster.block_rank(), cranks = (int)cluster.num_blocks();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int feature_tiles = (a.features + kProjRows - 1) / kProjRows;
    const int tile = blockIdx.x / cranks;
    const int f0 = (tile % feature_tiles) * kProjRows;
    const int64_t t0 = (int64_t)(tile / feature_tiles) * NT;
    const int all_steps = (a.depth + kProjDepth - 1) / kProjDepth, per = (all_steps + cranks - 1) / cranks;
    const int step0 = min(crank * per, all_steps), steps = min(per, all_steps - step0);
    const int cb = a.bits;
    volatile int* gave_up = &sh.gave_up;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 8; ++i) {
            mbar_init(&sh.tokens_full[i], 1);
            mbar_init(&sh.codes_full[i], 1);
            mbar_init(&sh.operand_full[i], kUnpackWarps);
            mbar_init(&sh.empty[i], 1);
            mbar_init(&sh.codes_empty[i], kUnpackWarps);
        }
        mbar_init(&sh.done, 1);
        mbar_init(&sh.plan, 32);
        sh.gave_up = 0;
        mbar_fence_init();
    }
    if (warp == 3) {
        tc_alloc(&sh.tmem, Shape::kColumns);
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    const int chunks = a.up ? (a.rank + kRankChunk - 1) / kRankChunk : 0;

    if (warp == 0) {
        // the tokens' operand
        if (lane == 0) {
            if (a.early & 2) asm volatile("griddepcontrol.wait;" ::: "memory");
            int s = 0;
            for (; s < steps; ++s) {
                const int st = s % S;
                if (s >= S && !tc_wait(&sh.empty[st], (s / S - 1) & 1, gave_up, a.status, 93)) break;
                mbar_arrive_expect_tx(&sh.tokens_full[st], Shape::kBBytes);
                tc_copy_2d(smem_u32(right + st * Shape::kBBytes), &tokens_map, (step0 + s) * kProjDepth, (int)t0, &sh.tokens_full[st]);
            }
            if (s < steps)
                for (int i = max(0, s - S); i < s; ++i) tc_drain(&sh.tokens_full[i % S], (i / S) & 1);
        }
    } else if (warp == 2) {
        // the packed codes
        if (lane == 0) {
            const uint32_t bytes = (uint32_t)(kProjRows * kProjDepth * cb / 8);
            int s = 0;
            for (; s < steps; ++s) {
                const int st = s % CS;
                if (s >= CS && !tc_wait(&sh.codes_empty[st], (s / CS - 1) & 1, gave_up, a.status, 94)) break;
                mbar_arrive_expect_tx(&sh.codes_full[st], bytes);
                const int depth = (step0 + s) * kProjDepth;
                if (BACK) tc_copy_2d(smem_u32(packed + st * Shape::kCodeBytes), &codes_map, depth * cb / 8, f0, &sh.codes_full[st]);
                else tc_copy_2d(smem_u32(packed + st * Shape::kCodeBytes), &codes_map, f0 / 8 * cb, depth, &sh.codes_full[st]);
            }
            if (s < steps)
                for (int i = max(0, s - CS); i < s; ++i) tc_drain(&sh.codes_full[i % CS], (i / CS) & 1);
        }
    } else if (warp == 3) {
        // what the first stage has found out about the tokens, and the adapters they need: each with the window of its tokens
        if (a.early) asm volatile("griddepcontrol.wait;" ::: "memory");
        constexpr int PER = (NT + 31) / 32;
        int mine[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int t = lane + 32 * i;
            int id = kNoRequest;
            if (t < NT && t0 + t < a.tokens) {
                id = a.ids[t0 + t];
                sh.sum[t] = a.sum[t0 + t];
                sh.row_scale[t] = a.row_scale ? a.row_scale[t0 + t] : 1.0f;
                sh.hidden_scale[t] = a.up && id >= 0 ? a.hidden_scale[t0 + t] : 0.0f;
            }
            if (t < NT) sh.ids[t] = id;
            mine[i] = chunks > 0 ? id : -1;
        }
        int found = 0, entries = 0;
        for (;;) {
            int first = NT;
#pragma unroll
            for (int i = PER - 1; i >= 0; --i)
                if (mine[i] >= 0) first = lane + 32 * i;
            first = __reduce_min_sync(0xffffffffu, first);
            if (first >= NT) break;
            int id = -1;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (lane + 32 * i == first) id = mine[i];
            id = __shfl_sync(0xffffffffu, id, first & 31);
            int last = first;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (mine[i] == id) {
                    last = max(last, lane + 32 * i);
                    mine[i] = -1;
                }
            last = __reduce_max_sync(0xffffffffu, last);
            if (found++ % cranks == crank) {
                if (lane == 0) {
                    // (the first one takes every column, so that the others' sums start from zero)
                    const int lo = entries == 0 ? 0 : first & ~15;
                    sh.entry_id[entries] = id;
                    sh.entry_lo[entries] = lo;
                    sh.entry_n[entries] = entries == 0 ? NT : (last + 16 - lo) & ~15;
                }
                ++entries;
            }
        }
        if (lane == 0) sh.entries = entries;
        __syncwarp();
        mbar_arrive(&sh.plan);
    } else if (warp == 1) {
        // the products
        if (lane == 0) {
            bool ok = true;
            int s = 0;
            const uint32_t kind = tc_kind(BF16, !BACK, NT);
            for (; s < steps; ++s) {
                const int st = s % S;
                ok = tc_wait(&sh.tokens_full[st], (s / S) & 1, gave_up, a.status, 95) && tc_wait(&sh.operand_full[st], (s / S) & 1, gave_up, a.status, 96);
                if (!ok) break;
                tc_fence_after();
                const uint32_t la = smem_u32(left + st * kABytes), ra = smem_u32(right + st * Shape::kBBytes);
#pragma unroll
                for (int k = 0; k < kProjDepth / 16; ++k) {
                    const uint64_t da = BACK ? tc_operand(la + k * 32, 16, 1024) : tc_operand(la + k * 2048, kABytes / 2, 1024);
                    tc_mma(tmem, da, tc_operand(ra + k * 32, 16, 1024), kind, s > 0 || k > 0);
                }
                tc_commit(&sh.empty[st]);
            }
            if (ok && chunks > 0 && tc_wait(&sh.plan, 0, gave_up, a.status, 97)) {
                const int entries = sh.entries;
                for (int e = 0; ok && e < entries; ++e)
                    for (int c = 0; c < chunks; ++c, ++s) {
                        const int st = s % S;
                        ok = tc_wait(&sh.operand_full[st], (s / S) & 1, gave_up, a.status, 98);
                        if (!ok) break;
                        tc_fence_after();
                        const int lo = sh.entry_lo[e];
                        const uint32_t la = smem_u32(left + st * kABytes), ra = smem_u32(right + st * Shape::kBBytes) + lo * 128;
                        const uint32_t up_kind = tc_kind(BACK ? a.out_bf16 != 0 : BF16, true, sh.entry_n[e]);
                        const int ks = (min(kRankChunk, a.rank - c * kRankChunk) + 15) / 16;
                        for (int part = 0; part < 2; ++part)
                            for (int k = 0; k < ks; ++k)
                                tc_mma(tmem + Shape::kColumns / 2 + lo, tc_operand(la + k * 2048, kABytes / 2, 1024),
                                       tc_operand(ra + part * 64 + k * 32, 16, 1024), up_kind, e > 0 || c > 0 || part > 0 || k > 0);
                        tc_commit(&sh.empty[st]);
                    }
            }
            tc_commit(&sh.done);
            if (!ok) tc_drain(&sh.done, 0);
        }
    } else {
        const int uid = threadIdx.x - 128;
        int s = 0;
        bool ok = true;
        for (; s < steps; ++s) {
            const int st = s % S, cs = s % CS;
            ok = tc_wait(&sh.codes_full[cs], (s / CS) & 1, gave_up, a.status, 99);
            if (ok && s >= S) ok = tc_wait(&sh.empty[st], (s / S - 1) & 1, gave_up, a.status, 100);
            ok = __all_sync(0xffffffffu, ok);                          // (a warp gives up as a whole)
            if (!ok) break;
            const uint8_t* src = packed + cs * Shape::kCodeBytes;
            uint8_t* dst = left + st * kABytes;
            if (cb == 8) unpack_stage<BF16, 8, BACK>(src, dst, uid);
            else if (cb == 4) unpack_stage<BF16, 4, BACK>(src, dst, uid);
            else unpack_stage<BF16, 2, BACK>(src, dst, uid);
            tc_publish();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&sh.operand_full[st]);
                mbar_arrive(&sh.codes_empty[cs]);
            }
        }
        if (ok) ok = __all_sync(0xffffffffu, tc_wait(&sh.plan, 0, gave_up, a.status, 101));
        if (ok && chunks > 0) {
            if (a.early) asm volatile("griddepcontrol.wait;" ::: "memory");
            const bool bf16 = BACK ? a.out_bf16 != 0 : BF16;
            const uint32_t exponent = bf16 ? 0x7f80u : 0x7c00u;
            const uint16_t* up = reinterpret_cast<const uint16_t*>(a.up);
            const bool wide = ((reinterpret_cast<uintptr_t>(up) | (uintptr_t)((int64_t)a.features * 2)) & 15) == 0;
            const int entries = sh.entries;
            bool bad = false;
            for (int e = 0; ok && e < entries; ++e)
                for (int c = 0; c < chunks; ++c, ++s) {
                    const int st = s % S, id = sh.entry_id[e];
                    if (s >= S) ok = __all_sync(0xffffffffu, tc_wait(&sh.empty[st], (s / S - 1) & 1, gave_up, a.status, 102));
                    if (!ok) break;
                    uint8_t* dst = left + st * kABytes;
                    const int rows = min(kRankChunk, a.rank - c * kRankChunk), padded = (rows + 15) & ~15;
                    for (int u = uid; u < padded * 16; u += 32 * kUnpackWarps) {
                        const int k = u >> 4, chunk = u & 15, f = f0 + chunk * 8;
                        uint4 w = make_uint4(0, 0, 0, 0);
                        if (k < rows) w = load8_16(up + ((int64_t)id * a.rank + c * kRankChunk + k) * a.features + f, min(max(a.features - f, 0), 8), wide);
                        w.x = finite_pair(w.x, exponent, bad); w.y = finite_pair(w.y, exponent, bad);
                        w.z = finite_pair(w.z, exponent, bad); w.w = finite_pair(w.w, exponent, bad);
                        *reinterpret_cast<uint4*>(dst + (chunk >> 3) * (kABytes / 2) + k * 128 + (((chunk & 7) ^ (k & 7)) << 4)) = w;
                    }
                    uint8_t* tok = right + st * Shape::kBBytes;
                    const int lo = sh.entry_lo[e], n = sh.entry_n[e], per_row = padded >> 3;
                    for (int u = uid; u < n * per_row; u += 32 * kUnpackWarps) {
                        const int t = lo + u / per_row, chunk = u % per_row;
                        float v[8] = {};
                        if (sh.ids[t] == id) {
                            const float inv = 1.0f / sh.hidden_scale[t];               // (a power of two)
                            const float* h = a.hidden + (t0 + t) * a.rank + c * kRankChunk + chunk * 8;
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (chunk * 8 + i < rows) v[i] = h[i] * inv;
                        }
                        uint32_t high[4], low[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (bf16) {
                                high[i] = pack_pair<__nv_bfloat16>(v[2 * i], v[2 * i + 1]);
                                const float2 f = unpack_pair<__nv_bfloat16>(high[i]);
                                low[i] = pack_pair<__nv_bfloat16>(v[2 * i] - f.x, v[2 * i + 1] - f.y);
                            } else {
                                high[i] = pack_pair<__half>(v[2 * i], v[2 * i + 1]);
                                const float2 f = unpack_pair<__half>(high[i]);
                                low[i] = pack_pair<__half>(v[2 * i] - f.x, v[2 * i + 1] - f.y);
                            }
                        }
                        uint8_t* p = tok + t * 128;
                        *reinterpret_cast<uint4*>(p + ((chunk ^ (t & 7)) << 4)) = make_uint4(high[0], high[1], high[2], high[3]);
                        *reinterpret_cast<uint4*>(p + (((chunk + 4) ^ (t & 7)) << 4)) = make_uint4(low[0], low[1], low[2], low[3]);
                    }
                    tc_publish();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.operand_full[st]);
                }
            if (bad) set_status(a.status, ZIPML_ERR_NONFINITE, 103);
        }
        if (ok) ok = __all_sync(0xffffffffu, tc_wait(&sh.done, 0, gave_up, a.status, 104));
        if (ok) {
            tc_fence_after();
            // two warps on each 32 rows of tensor memory, every other 16 tokens each
            const int quarter = warp & 3, half = (warp - 4) >> 2;
            const int row = quarter * 32 + lane, f = f0 + row;
            const bool in = f < a.features;
            float alpha = 1.0f, beta = 1.0f;
            if (a.step && in) {
                alpha = a.step[f];
                beta = fmaf(a.center, alpha, a.lo[f]);
            }
            if (crank != 0) beta = 0.0f;
            const bool have_up = chunks > 0 && sh.entries > 0;
            float* join = reinterpret_cast<float*>(ring);
            for (int c = half; c < NT / 16; c += 2) {
                uint32_t v[16], w[16];
                if (steps > 0) tc_load16(tmem + ((uint32_t)(quarter * 32) << 16) + c * 16, v);
                if (have_up) tc_load16(tmem + ((uint32_t)(quarter * 32) << 16) + Shape::kColumns / 2 + c * 16, w);
                tc_load_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int t = c * 16 + i, id = sh.ids[t];
                    if (id == kNoRequest) continue;
                    float y = beta != 0.0f ? beta * sh.sum[t] : 0.0f;
                    if (steps > 0) y = fmaf(alpha * sh.row_scale[t], __uint_as_float(v[i]), y);
                    if (have_up && id >= 0) y = fmaf(sh.hidden_scale[t], __uint_as_float(w[i]), y);
                    if (cranks > 1) join[t * kProjRows + row] = y;
                    else if (in) {
                        if (a.out_bf16) reinterpret_cast<__nv_bfloat16*>(a.out)[(t0 + t) * a.ldo + f] = __float2bfloat16_rn(y);
                        else reinterpret_cast<__half*>(a.out)[(t0 + t) * a.ldo + f] = __float2half_rn(y);
                    }
                }
            }
            tc_fence_before();
        }
    }
    __syncthreads();
    if (warp == 3) {
        tc_fence_after();
        tc_free(tmem, Shape::kColumns);
    }
    if (cranks > 1) {
        cluster.sync();
        const float* join = reinterpret_cast<const float*>(ring);
        for (int t = crank + cranks * warp; t < NT; t += cranks * (kProjThreads / 32)) {
            if (sh.ids[t] == kNoRequest) continue;
            float y[4] = {};
            for (int c = 0; c < cranks; ++c) {
                const float* p = cluster.map_shared_rank(join, c) + t * kProjRows;
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] += p[i * 32 + lane];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int f = f0 + i * 32 + lane;
                if (f >= a.features) continue;
                if (a.out_bf16) reinterpret_cast<__nv_bfloat16*>(a.out)[(t0 + t) * a.ldo + f] = __float2bfloat16_rn(y[i]);
                else reinterpret_cast<__half*>(a.out)[(t0 + t) * a.ldo + f] = __float2half_rn(y[i]);
            }
        }
        cluster.sync();
    }
}

static int encode_map(zipml_ctx* ctx, CUtensorMapDataType type, const void* base, int64_t inner, int64_t rows, int64_t stride_bytes, int box_inner, int box_rows,
                      CUtensorMapSwizzle swizzle, CUtensorMap* out) {
    typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    if (!ctx->tmap_encode) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess || !fn) {
            (void)cudaGetLastError();
            return ZIPML_ERR_CUDA;
        }
        ctx->tmap_encode = fn;
    }
    const cuuint64_t dim[2] = {(cuuint64_t)inner, (cuuint64_t)rows};
    const cuuint64_t stride[1] = {(cuuint64_t)stride_bytes};
    const cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows}, each[2] = {1, 1};
    const CUresult r = reinterpret_cast<EncodeFn>(ctx->tmap_encode)(out, type, 2, const_cast<void*>(base), dim, stride, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                                                    swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? ZIPML_OK : ZIPML_ERR_CUDA;
}

template <int NT, bool BACK, bool BF16>
static int launch_project_as(zipml_ctx* ctx, const ProjectArgs& a, const CUtensorMap& tokens_map, const CUtensorMap& codes_map, int ranks) {
    auto kernel = &project_kernel<NT, BACK, BF16>;
    const size_t smem = 1024 + ProjShape<NT>::kRing + sizeof(ProjShared<NT>);
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return cuda_status(e);
    const int64_t tiles = (a.tokens + NT - 1) / NT * ((a.features + kProjRows - 1) / kProjRows);
    if (tiles * ranks > 0x7fffffffLL) return ZIPML_ERR_WORKSPACE;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles * ranks));
    cfg.blockDim = dim3(kProjThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.early ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, kernel, a, tokens_map, codes_map);
    ctx->launches += 1;
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError());
}

// Tokens of a tile and CTAs that divide the depth, by the cycles that a wave of tiles should take: a stage is bound by shared memory
// (both operands are read by the tensor core and the left one written by the unpacking warps, 128 bytes a cycle: NT + 256), a tile also pays for
// its start, its epilogue and, where the depth is divided, the exchange.
static void project_shape(const zipml_ctx* ctx, const ProjectArgs& a, int* tokens, int* ranks) {
    const int64_t feature_tiles = (a.features + kProjRows - 1) / kProjRows, steps = (a.depth + kProjDepth - 1) / kProjDepth;
    double best = 0.0;
    for (const int nt : {16, 64, 128, 256})
        for (int r = 1; r <= (nt == 256 ? 1 : 8); r *= 2) {
            if (r > 1 && steps / r < 4) break;
            const int64_t ctas = (a.tokens + nt - 1) / nt * feature_tiles * r;
            const int64_t waves = (ctas + ctx->sm_count - 1) / ctx->sm_count;
            const double cycles = (double)waves * ((double)((steps + r - 1) / r) * (nt + 256) + 3000 + nt * 16 + (r > 1 ? 1500 : 0));
            if (best == 0.0 || cycles < best) { best = cycles; *tokens = nt; *ranks = r; }
        }
}

template <bool BACK, bool BF16>
static int launch_project_typed(zipml_ctx* ctx, const ProjectArgs& a, const CUtensorMap& tm, const CUtensorMap& cm, int nt, int ranks) {
    if (nt == 16) return launch_project_as<16, BACK, BF16>(ctx, a, tm, cm, ranks);
    if (nt == 64) return launch_project_as<64, BACK, BF16>(ctx, a, tm, cm, ranks);
    if (nt == 128) return launch_project_as<128, BACK, BF16>(ctx, a, tm, cm, ranks);
    return launch_project_as<256, BACK, BF16>(ctx, a, tm, cm, ranks);
}

int launch_project(zipml_ctx* ctx, const ProjectArgs& a, const void* tokens_operand, int64_t ld_operand, bool operand_bf16, const zipml_dataset* w, bool backward) {
    int nt = 16, ranks = 1;
    project_shape(ctx, a, &nt, &ranks);
    CUtensorMap tokens_map, codes_map;
    int rc = encode_map(ctx, operand_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, tokens_operand, a.depth, a.tokens, ld_operand * 2,
                        kProjDepth, nt, CU_TENSOR_MAP_SWIZZLE_128B, &tokens_map);
    if (rc != ZIPML_OK) return rc;
    rc = encode_map(ctx, CU_TENSOR_MAP_DATA_TYPE_UINT8, w->plane1, w->row_bytes, w->m, w->row_bytes, (backward ? kProjDepth : kProjRows) * a.bits / 8,
                    backward ? kProjRows : kProjDepth, CU_TENSOR_MAP_SWIZZLE_NONE, &codes_map);
    if (rc != ZIPML_OK) return rc;
    if (backward) return launch_project_typed<true, false>(ctx, a, tokens_map, codes_map, nt, ranks);
    return operand_bf16 ? launch_project_typed<false, true>(ctx, a, tokens_map, codes_map, nt, ranks)
                        : launch_project_typed<false, false>(ctx, a, tokens_map, codes_map, nt, ranks);
}

}  // namespace zipml
