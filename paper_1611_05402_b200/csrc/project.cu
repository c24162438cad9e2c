// Second stage of a projection with low-rank adapters: tokens times packed codes on the tensor cores, the adapters' products beside it
// in the same launch, the codes' grids in the epilogue.
#include <type_traits>

#include <cooperative_groups.h>

#include "project.cuh"
#include "tensor_core.cuh"

namespace zipml {

namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------------------------
// A CTA makes 128 features x NT tokens, a pair of CTAs 256 x 256.  The features stand on the product's rows and the tokens on its columns, so
// one kernel serves from a token (16 columns, the codes' bytes are what counts) to thousands.  Per 64 of the depth, a stage:
//   codes     A tensor copy brings the packed codes.  Groups of four warps, each with a stage of its own, turn them into 16-bit whole numbers
//             code - 2^(bits-1), which are exact, and lay them out as the product's left operand; a fifth warp makes a group's stores
//             visible to the tensor cores.  Forward: a code row is one depth and holds the features (MN-major operand);
//             backward: a code row is a feature (K-major).
//   tokens    A tensor copy lays the right operand out itself.  Of a pair each CTA brings half of it, and the tensor cores share it.
//   product   One lane issues 128 (256) x NT x 16 four times, sums in tensor memory.  Backward: eight times, since dy step is not a 16-bit
//             number: in one part it would be off by 2^-12, as much as the rounding of an fp16 result, and more wherever the codes'
//             products and the lower ends' share cancel.  Its two parts (see split_scaled) have sums of their own.  The tensor cores cut what they
//             add to a sum instead of rounding it, so one sum of 1,024 products over a depth of 8192 was 1.6e-5 of the result off; the
//             high parts' sums are exact, and what the low ones' lose is that much of a part a few hundred times smaller.
// The adapters then take further stages: the ranks of the tile's adapters, each padded to a multiple of 8, follow one another as a depth of
// their own, 32 a stage.  up_i's rows are the left operand as they lie, hidden the right one, in two 16-bit parts (high and low: 16 or more
// bits), zero for tokens of other adapters, over the 16-token windows that hold the stage's tokens.  Their sums have columns of their own,
// since the grids' steps do not apply to them.
// The epilogue takes steps, sums and scales together in fp32 and rounds once.  With few tokens a cluster's CTAs divide the depth and
// add their results through each other's shared memory in a fixed order.
//
// What bounds it: shared memory.  A stage of a pair's CTA writes 16 KB of tokens and 4 or 8 KB of codes, reads those, writes 16 KB of left
// operand, and the tensor cores read 32 KB: some 600 cycles at 128 bytes each, and it takes 560 to 590, where the product alone takes 512.  A
// tile then waits for its start (2,000 cycles), the adapters (4,500) and the epilogue (7,500).  8192 x 8192 x 8192, 4 bits, rank 32: 776 us,
// 1.43 PFLOP/s; 4096 tokens x 4096 x 16384, 8 bits, rank 16: 460 us; backward 8192 x 8192 x 8192, 8 bits: 1,359 us, whose
// two parts' products run at 1.62 PFLOP/s (840 us with one part of 11 bits).  With single CTAs of 128 x 256, which read every token twice as often
// from L2, the first took 990 us.  Few tokens: some 500 cycles a stage against the 130 that the
// codes' bytes would take; without the unpacking 285.  Backward, with two parts: 650 for 16 tokens, 750 for 64, 1,020 for 128, 1,060 for a pair.
// ---------------------------------------------------------------------------------------------
constexpr int kProjRows = 128;                // features of a CTA
constexpr int kProjDepth = 64;                // depth of a stage: 128 bytes of 16-bit operand
constexpr int kGroups = 3;                    // groups of unpacking warps, each with every third stage
constexpr int kGroupWarps = 4;
constexpr int kGroupThreads = 32 * kGroupWarps;
constexpr int kFirstPublisher = 4 + kGroups * kGroupWarps;     // a warp for each group
constexpr int kSecondIssuer = kFirstPublisher + kGroups;
constexpr int kProjThreads = 32 * (kSecondIssuer + 1);
constexpr int kMostSlots = 12;
constexpr int kRankChunk = 32;                // ranks of an adapter stage: high parts in the first half of the depth, low ones in the second
constexpr uint32_t kLeftBytes = kProjRows * kProjDepth * 2;
constexpr float kCodeScale = 256.0f;          // of codes beside bf16 tokens (see centred_pair)

// Slots of the rings.  The left operand's is the deepest: unpacking a stage takes some 1,000 cycles from its codes' arrival to its last
// store, two products' worth, where a tensor copy of tokens only has L2's latency to cover.  A stage has one barrier that tells that both of
// its operands are there and one that tells that its product is done (the issuing warp waits and commits once a stage: each took it over 100
// cycles), in the left ring's order.  The groups' rings have a multiple of kGroups slots, so that a slot is always the same group's: a
// barrier tells a phase from the one before it only, and a group that came to a slot whose last phase belonged to another could be a phase
// early.
template <int NT, bool PAIR, bool BACK>
struct ProjShape {
    static constexpr int kLeft = 2 * kGroups;
    static constexpr int kParts = BACK ? 2 : 1;                         // of the tokens' operand
    static constexpr int kRight = BACK ? (NT >= 128 ? 3 : NT == 64 ? 4 : 6) : NT >= 128 ? 4 : 6;
    static constexpr int kRightRows = PAIR ? NT / 2 : NT;               // tokens of the operand that lie in this CTA
    static constexpr uint32_t kPartBytes = kRightRows * kProjDepth * 2, kRightBytes = kParts * kPartBytes;
    static constexpr uint32_t kCodeRing = (NT >= 128 ? (BACK ? 3 : 6) : NT == 64 ? (BACK ? 6 : 9) : 12) * kProjRows * kProjDepth;     // bytes for packed codes
    static_assert(kRight >= kGroups && kRight <= kLeft && kLeft % kGroups == 0 && kMostSlots % kGroups == 0, "slots by group");
    static constexpr uint32_t kRing = kLeft * kLeftBytes + kRight * kRightBytes + kCodeRing;
    // Tensor memory: the codes' sums of each issuing warp, for each part, then the adapters'.  Two warps issue where products are small: a turn's own
    // instructions, one after the other, take some 400 cycles, the products of 64 tokens 130 for each part.  Backward, the sums of 128
    // tokens and of a pair fill tensor memory: the first issuer's low sums are added to its high ones before the adapters' take their place.
    static constexpr int kIssuers = PAIR ? 1 : 2;
    static constexpr uint32_t kLowAt = kIssuers * NT;
    static constexpr bool kMerge = BACK && NT >= 128;
    static constexpr uint32_t kUpAt = kMerge ? kLowAt : kIssuers * kParts * NT;
    static constexpr uint32_t kColumns = PAIR || NT == 128 ? 512 : BACK ? (NT == 64 ? 512 : 128) : NT == 64 ? 256 : 64;
    static_assert(kUpAt + NT <= kColumns, "what was asked for");
    static constexpr int kWindows = PAIR ? 1 : 4 * NT;                   // stages of adapters at most, for their windows
};

struct ProjToken {                            // what the epilogue needs of a token
    float row_scale, sum, hidden_scale;
    int id;
};

template <int NT, bool PAIR, bool BACK>
struct ProjShared {
    using Shape = ProjShape<NT, PAIR, BACK>;
    ProjToken token[NT];
    uint64_t codes_full[kMostSlots], codes_empty[kMostSlots], written[2 * kGroups], full[2 * kGroups], empty[2 * kGroups];
    uint64_t up_full[kGroups], up_empty[kGroups], codes_done, merged, done, plan;
    uint32_t tmem;
    int gave_up;
    int entries;                              // adapters of this tile that fall to this CTA
    int entry_id[NT], entry_lo[PAIR ? 1 : NT], entry_end[PAIR ? 1 : NT];
    int entry[NT];                            // of a token, -1: none
    uint16_t window_lo[Shape::kWindows], window_n[Shape::kWindows];
};

// A slot of a ring and the parity of its current turn.
struct RingAt {
    int slot = 0;
    uint32_t turn = 0;
    __device__ __forceinline__ void next(int by, int slots) {
        slot += by;
        if (slot >= slots) { slot -= slots; turn ^= 1u; }
    }
};

// Sixteen packed codes, and as bytes.
template <int CB>
__device__ __forceinline__ void load_codes(const uint8_t* p, uint32_t (&w)[4]) {
    if constexpr (CB == 8) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (CB == 4) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}
template <int CB>
__device__ __forceinline__ void codes_to_bytes(uint32_t (&w)[4]) {
    if constexpr (CB == 4) {
        const uint32_t u[2] = {w[0], w[1]};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t even = u[i] & 0x0F0F0F0Fu, odd = (u[i] >> 4) & 0x0F0F0F0Fu;
            w[2 * i] = __byte_perm(even, odd, 0x5140);
            w[2 * i + 1] = __byte_perm(even, odd, 0x7362);
        }
    } else if constexpr (CB == 2) {
        uint32_t t[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = (w[0] >> (2 * k)) & 0x03030303u;
        const uint32_t a0 = __byte_perm(t[0], t[1], 0x5140), a1 = __byte_perm(t[2], t[3], 0x5140);
        const uint32_t b0 = __byte_perm(t[0], t[1], 0x7362), b1 = __byte_perm(t[2], t[3], 0x7362);
        w[0] = __byte_perm(a0, a1, 0x5410); w[1] = __byte_perm(a0, a1, 0x7632);
        w[2] = __byte_perm(b0, b1, 0x5410); w[3] = __byte_perm(b0, b1, 0x7632);
    }
}

// Two codes, in the low bytes of p's halves under the byte of 1/2 (bf16) or 1024 (fp16), as code - center, bf16's times 2^-8: the code is the mantissa's
// lowest bits, and one exact subtraction of `base` = that and the center takes the offset away.  (2^-8: a product with a bf16 token is then no
// larger than the token, which may be anything that fp32 holds; kCodeScale in the epilogue takes it back.)  EIGHT: 8-bit codes in bf16, whose mantissa
// has 7 bits: a code's top bit counts as exponent there, and the value is 128 + code below 128, 256 + 2 (code - 128) from there on, times 2^-8;
// less 256 it is what it should be, or twice that.  (Byte and logic instructions run at half the rate of the 16-bit arithmetic's and bound the
// unpacking: two of each a pair.)
template <bool BF16, bool EIGHT>
__device__ __forceinline__ uint32_t centred_pair(uint32_t p, uint32_t base) {
    if constexpr (BF16) {
        __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&p), *reinterpret_cast<const __nv_bfloat162*>(&base));
        if constexpr (EIGHT) {
            const uint32_t half = (p & 0x00800080u) ^ 0x3F803F80u;           // a half where the top bit is set, else one
            v = __hmul2(v, *reinterpret_cast<const __nv_bfloat162*>(&half));
        }
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&p), *reinterpret_cast<const __half2*>(&base));
        return *reinterpret_cast<const uint32_t*>(&v);
    }
}
template <bool BF16, bool EIGHT>
__device__ __forceinline__ uint4 centred_chunk(uint32_t w0, uint32_t w1, uint32_t base) {      // 8 codes
    constexpr uint32_t kTop = BF16 ? 0x3F3F3F3Fu : 0x64646464u;
    return make_uint4(centred_pair<BF16, EIGHT>(__byte_perm(w0, kTop, 0x4140), base), centred_pair<BF16, EIGHT>(__byte_perm(w0, kTop, 0x4342), base),
                      centred_pair<BF16, EIGHT>(__byte_perm(w1, kTop, 0x4140), base), centred_pair<BF16, EIGHT>(__byte_perm(w1, kTop, 0x4342), base));
}
// The base for codes of so many bits, in both halves: 128 (256 for EIGHT), times 2^-8, or 1024, and the center 2^(bits - 1).
template <bool BF16>
__device__ __forceinline__ uint32_t centre_base(int bits) {
    const uint32_t center = 1u << (bits - 1), h = BF16 ? 0x3F00u + center : 0x6400u + center;      // (8 bits in bf16: 0x3F80, which is 256 times 2^-8)
    return h | h << 16;
}

// A thread's place in a stage: kUnits units of 16 codes, from one to the next the same distance on in the packed codes and in the left
// operand.  Bank conflicts: eight lanes store 16 bytes each at a time, so four take one 128-byte row of the operand and four the next,
// whose swizzles differ in the lowest bit.  Forward: a unit is 16 features of one depth (MN-major, 64 features a row); backward 16 of
// the depth of one feature.
constexpr int kUnits = kProjRows * kProjDepth / 16 / kGroupThreads;
template <bool BACK>
struct UnitPlace {
    uint32_t from, to;                        // unit of the packed codes, byte of the operand
    static constexpr uint32_t kFromStep = kGroupThreads, kToStep = BACK ? 32 * 128 : 16 * 128;
    __device__ __forceinline__ explicit UnitPlace(int gid) {
        if constexpr (BACK) {
            const uint32_t row = gid >> 2, chunk = 2 * (gid & 3);
            from = gid;
            to = row * 128 + ((chunk ^ (row & 7)) << 4);
        } else {
            const uint32_t k = (gid >> 4) * 2 + (gid >> 2 & 1), f16 = (gid & 3) + (gid >> 3 & 1) * 4, chunk = 2 * (f16 & 3);
            from = k * 8 + f16;
            to = (f16 >> 2) * (kLeftBytes / 2) + k * 128 + ((chunk ^ (k & 7)) << 4);
        }
    }
};
static_assert(kGroupThreads == 128, "a turn of units is 16 depths of 128 features, or 32 features of 64 depths");

template <bool BF16, int CB, bool EIGHT, bool BACK>
__device__ __forceinline__ void unpack_stage(uint32_t (&w)[kUnits][4], uint8_t* to, uint32_t base) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        codes_to_bytes<CB>(w[i]);
        uint8_t* p = to + i * UnitPlace<BACK>::kToStep;
        *reinterpret_cast<uint4*>(p) = centred_chunk<BF16, EIGHT>(w[i][0], w[i][1], base);
        *reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(p) ^ 16) = centred_chunk<BF16, EIGHT>(w[i][2], w[i][3], base);
    }
}

// Marks (the sign's place) of what is not finite among 16-bit values, and the values with zero in its place.  `lowest`: the exponent's lowest bit in
// both halves of a word; added to a value without its sign it carries into the sign's place exactly where the exponent is all ones.
__device__ __forceinline__ uint32_t not_finite(uint32_t w, uint32_t lowest) { return ((w & 0x7fff7fffu) + lowest) & 0x80008000u; }
__device__ __forceinline__ uint32_t not_finite(const uint4& w, uint32_t lowest) {
    return not_finite(w.x, lowest) | not_finite(w.y, lowest) | not_finite(w.z, lowest) | not_finite(w.w, lowest);
}
__device__ __forceinline__ uint32_t keep_finite(uint32_t w, uint32_t lowest) {
    const uint32_t n = not_finite(w, lowest);
    return w & ~((n >> 15) * 0xffffu);                    // (a half's mark becomes all of its bits)
}

template <int NT, bool BACK, bool BF16, bool PAIR>
__global__ void __launch_bounds__(kProjThreads, 1) project_kernel(ProjectArgs a, const __grid_constant__ CUtensorMap tokens_map,
                                                                  const __grid_constant__ CUtensorMap codes_map) {
    using Shape = ProjShape<NT, PAIR, BACK>;
    constexpr int L = Shape::kLeft, R = Shape::kRight;
    extern __shared__ uint8_t raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    ProjShared<NT, PAIR, BACK>& sh = *reinterpret_cast<ProjShared<NT, PAIR, BACK>*>(ring + Shape::kRing);
    uint8_t* const left = ring;
    uint8_t* const right = ring + L * kLeftBytes;
    uint8_t* const packed = right + R * Shape::kRightBytes;
    cg::cluster_group cluster = cg::this_cluster();
    // CTAs that divide the depth; a pair's two divide the features instead
    const int side = PAIR ? (int)cluster.block_rank() : 0;
    const int crank = PAIR ? 0 : (int)cluster.block_rank(), cranks = PAIR ? 1 : (int)cluster.num_blocks();
    constexpr int kTileRows = PAIR ? 2 * kProjRows : kProjRows;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int feature_tiles = (a.features + kTileRows - 1) / kTileRows;
    const int tile = PAIR ? blockIdx.x / 2 : blockIdx.x / cranks;
    const int f0 = (tile % feature_tiles) * kTileRows + side * kProjRows;
    const int64_t t0 = (int64_t)(tile / feature_tiles) * NT;
    const int all_steps = (a.depth + kProjDepth - 1) / kProjDepth, per = (all_steps + cranks - 1) / cranks;
    const int step0 = min(crank * per, all_steps), steps = min(per, all_steps - step0);
    const int cb = container_bits(a.bits);
    const uint32_t code_bytes = (uint32_t)(kProjRows * kProjDepth / 8 * cb);
    const int code_slots = min(kMostSlots, (int)(Shape::kCodeRing / code_bytes) / kGroups * kGroups);
    volatile int* gave_up = &sh.gave_up;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kMostSlots; ++i) {
            mbar_init(&sh.codes_full[i], 1);
            mbar_init(&sh.codes_empty[i], kGroupWarps);
        }
        for (int i = 0; i < L; ++i) {
            mbar_init(&sh.written[i], kGroupWarps);
            mbar_init(&sh.full[i], 1 + (PAIR ? 2 : 1));                    // the tokens' copies and the publishing warps
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < kGroups; ++i) {
            mbar_init(&sh.up_full[i], (PAIR ? 2 : 1) * kGroupWarps);
            mbar_init(&sh.up_empty[i], 1);
        }
        mbar_init(&sh.codes_done, Shape::kIssuers);
        mbar_init(&sh.merged, (PAIR ? 2 : 1) * kGroups * kGroupWarps);
        mbar_init(&sh.done, 1);
        mbar_init(&sh.plan, 32);
        sh.gave_up = 0;
        mbar_fence_init();
    }
    if (warp == 3) {
        tc_alloc<PAIR>(&sh.tmem, Shape::kColumns);
        tc_fence_before();
    }
    __syncthreads();
    if constexpr (PAIR) cluster.sync();                               // (the other CTA's barriers and its tensor memory are there too)
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    const int rank8 = a.up ? (a.rank + 7) & ~7 : 0;
    const uint32_t per_rank8 = rank8 > 0 ? 0xffffffffu / (uint32_t)rank8 + 1u : 0u;   // (place / rank8 as a high product: exact below 2^16)
    const auto up_stages = [&] { return (sh.entries * rank8 + kRankChunk - 1) / kRankChunk; };      // of the adapters' ranks

    if (warp == 0) {
        // The tokens' operand.  (Here and below a warp comes to its waits as a whole and one lane, elected, issues: see tc_elect.)
        if (a.early & 2) asm volatile("griddepcontrol.wait;" ::: "memory");
        int s = 0;
        RingAt at, stage, ahead;                                           // stage s, and s - R, whose place it takes
        for (; s < steps; ++s, at.next(1, R), stage.next(1, L)) {
            if (s >= R) {
                if (!__all_sync(0xffffffffu, tc_wait(&sh.empty[ahead.slot], ahead.turn, gave_up, a.status, 93))) break;
                ahead.next(1, L);
            }
            const uint32_t dst = smem_u32(right) + at.slot * Shape::kRightBytes;
            if (tc_elect()) {
                if constexpr (PAIR) {
                    // (both halves count on the first CTA's barrier; the other's bytes may come before they are expected)
                    if (side == 0) mbar_arrive_expect_tx(&sh.full[stage.slot], 2 * Shape::kRightBytes);
                    for (int p = 0; p < Shape::kParts; ++p)
                        tc_copy_2d_pair(dst + p * Shape::kPartBytes, &tokens_map, (step0 + s) * kProjDepth, (int)(p * a.tokens + t0) + side * Shape::kRightRows,
                                        tc_peer(&sh.full[stage.slot], 0));
                } else {
                    mbar_arrive_expect_tx(&sh.full[stage.slot], Shape::kRightBytes);
                    for (int p = 0; p < Shape::kParts; ++p)
                        tc_copy_2d(dst + p * Shape::kPartBytes, &tokens_map, (step0 + s) * kProjDepth, (int)(p * a.tokens + t0), &sh.full[stage.slot]);
                }
            }
            __syncwarp();
        }
    } else if (warp == 2) {
        // the packed codes
        int s = 0;
        RingAt at;
        for (; s < steps; ++s, at.next(1, code_slots)) {
            if (s >= code_slots && !__all_sync(0xffffffffu, tc_wait(&sh.codes_empty[at.slot], at.turn ^ 1u, gave_up, a.status, 94))) break;
            const int depth = (step0 + s) * kProjDepth;
            const uint32_t dst = smem_u32(packed) + at.slot * code_bytes;
            if (tc_elect()) {
                mbar_arrive_expect_tx(&sh.codes_full[at.slot], code_bytes);
                if (BACK) tc_copy_2d(dst, &codes_map, depth / 8 * cb, f0, &sh.codes_full[at.slot]);
                else tc_copy_2d(dst, &codes_map, f0 / 8 * cb, depth, &sh.codes_full[at.slot]);
            }
            __syncwarp();
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
            ProjToken tok{1.0f, 0.0f, 1.0f, kNoRequest};
            if (t < NT && t0 + t < a.tokens) {
                tok.id = id = a.ids[t0 + t];
                tok.sum = a.sum[t0 + t];
                if (a.row_scale) tok.row_scale = a.row_scale[t0 + t];
                if (a.up && id >= 0) tok.hidden_scale = a.hidden_scale[t0 + t];
            }
            if (t < NT) sh.token[t] = tok;
            if (t < NT) sh.entry[t] = -1;
            mine[i] = rank8 > 0 ? id : -1;
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
            const bool here = found++ % cranks == crank;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (mine[i] == id) {
                    last = max(last, lane + 32 * i);
                    mine[i] = -1;
                    if (here) sh.entry[lane + 32 * i] = entries;
                }
            last = __reduce_max_sync(0xffffffffu, last);
            if (here) {
                if (lane == 0) {
                    sh.entry_id[entries] = id;
                    if constexpr (!PAIR) {
                        sh.entry_lo[entries] = first & ~15;
                        sh.entry_end[entries] = (last + 16) & ~15;
                    }
                }
                ++entries;
            }
        }
        __syncwarp();
        // The columns that a stage's tokens lie in.  The first stage takes all, so that the others' sums start from zero (and so does every one
        // of a pair's, which holds the operand's tokens in two places).
        if constexpr (!PAIR)
            for (int j = lane; j * kRankChunk < entries * rank8; j += 32) {
                int lo = j == 0 ? 0 : NT, end = j == 0 ? NT : 0;
                for (int e = j * kRankChunk / rank8; j > 0 && e < entries && e * rank8 < (j + 1) * kRankChunk; ++e) {
                    lo = min(lo, sh.entry_lo[e]);
                    end = max(end, sh.entry_end[e]);
                }
                sh.window_lo[j] = (uint16_t)lo;
                sh.window_n[j] = (uint16_t)(end - lo);
            }
        if (lane == 0) sh.entries = entries;
        __syncwarp();
        mbar_arrive(&sh.plan);
    } else if (warp == 1 || warp == kSecondIssuer) {
        // The products: a warp waits as a whole, one lane issues.  Two warps take every other stage, each into sums of its own; the first takes
        // the adapters' stages too.  Of a pair, the first CTA's first warp.
        const int issuer = warp == 1 ? 0 : 1;
        if (side == 0 && issuer < Shape::kIssuers) {
            bool ok = true;
            RingAt la, ra;
            la.next(issuer, L);
            ra.next(issuer, R);
            const uint32_t kind = tc_kind(BF16, !BACK, kTileRows, NT), sums = tmem + issuer * NT;
            // (operands by their first slot: an address in steps of 16 bytes is the description's lowest field)
            const uint64_t left_at = BACK ? tc_operand(smem_u32(left), 16, 1024) : tc_operand(smem_u32(left), kLeftBytes / 2, 1024);
            const uint64_t right_at = tc_operand(smem_u32(right), 16, 1024);
            for (int s = issuer; s < steps; s += Shape::kIssuers, la.next(Shape::kIssuers, L), ra.next(Shape::kIssuers, R)) {
                ok = __all_sync(0xffffffffu, tc_wait(&sh.full[la.slot], la.turn, gave_up, a.status, 95));
                if (!ok) break;
                tc_fence_after();
                const uint64_t lp = left_at + (uint32_t)la.slot * (kLeftBytes / 16), rp = right_at + (uint32_t)ra.slot * (Shape::kRightBytes / 16);
                if (tc_elect()) {
#pragma unroll
                    for (int p = 0; p < Shape::kParts; ++p)
#pragma unroll
                        for (int k = 0; k < kProjDepth / 16; ++k)
                            tc_mma<PAIR>(sums + p * Shape::kLowAt, lp + k * (BACK ? 2 : 128), rp + p * (Shape::kPartBytes / 16) + k * 2, kind, s > issuer || k > 0);
                    tc_commit<PAIR>(&sh.empty[la.slot]);
                }
                __syncwarp();
            }
            if (tc_elect()) tc_commit<PAIR>(&sh.codes_done);
            __syncwarp();
            if (issuer == 0) {
                if (ok && rank8 > 0) ok = __all_sync(0xffffffffu, tc_wait(&sh.plan, 0, gave_up, a.status, 97));
                if (ok && rank8 > 0) {
                    const int count = up_stages(), total = sh.entries * rank8;
                    const uint64_t up_at = tc_operand(smem_u32(left), kLeftBytes / 2, 1024);
                    if (Shape::kMerge && count > 0) ok = __all_sync(0xffffffffu, tc_wait(&sh.merged, 0, gave_up, a.status, 113));
                    for (int j = 0, slot = 0, turn = 0; ok && j < count; ++j) {
                        ok = __all_sync(0xffffffffu, tc_wait(&sh.up_full[slot], turn, gave_up, a.status, 98));
                        if (!ok) break;
                        tc_fence_after();
                        const int lo = PAIR ? 0 : sh.window_lo[j], n = PAIR ? NT : sh.window_n[j];
                        const uint64_t lp = up_at + (uint32_t)slot * (kLeftBytes / 16), rp = right_at + (uint32_t)slot * (Shape::kRightBytes / 16) + (uint32_t)lo * 8;
                        const uint32_t up_kind = tc_kind(BACK ? a.out_bf16 != 0 : BF16, true, kTileRows, n);
                        const int ks = (min(kRankChunk, total - j * kRankChunk) + 15) / 16;
                        if (tc_elect()) {
                            for (int part = 0; part < 2; ++part)
                                for (int k = 0; k < ks; ++k)
                                    tc_mma<PAIR>(tmem + Shape::kUpAt + lo, lp + k * 128, rp + part * 4 + k * 2, up_kind, j > 0 || part > 0 || k > 0);
                            tc_commit<PAIR>(&sh.up_empty[slot]);
                        }
                        __syncwarp();
                        if (++slot == kGroups) { slot = 0; turn ^= 1; }
                    }
                }
                if (tc_elect()) tc_commit<PAIR>(&sh.done);
                __syncwarp();
            }
        }
    } else if (warp >= kFirstPublisher && warp < kSecondIssuer) {
        // A group's stores, made visible to the tensor cores by a warp that has nothing else to do: the fence waits for what is on its way to
        // shared memory, 500 to 1,400 cycles beside running products, which the unpacking warps spent idle.
        RingAt la;
        la.next(warp - kFirstPublisher, L);
        for (int s = warp - kFirstPublisher; s < steps; s += kGroups, la.next(kGroups, L)) {
            if (!__all_sync(0xffffffffu, tc_wait(&sh.written[la.slot], la.turn, gave_up, a.status, 106))) break;
            tc_publish();
            __syncwarp();
            if (lane == 0) {
                if (PAIR && side != 0) tc_arrive_at(tc_peer(&sh.full[la.slot], 0));
                else mbar_arrive(&sh.full[la.slot]);
            }
        }
    } else {
        const int group = (warp - 4) / kGroupWarps, gid = (threadIdx.x - 128) % kGroupThreads;
        // the epilogue's feature of this lane (a group's warps take 32 rows of tensor memory each) and its grid
        const int row = (warp & 3) * 32 + lane, feature = f0 + row;
        float alpha = 1.0f, beta = 1.0f;
        if (a.step && feature < a.features) {
            alpha = a.step[feature];
            beta = fmaf(a.center, alpha, a.lo[feature]);
            if constexpr (BF16) alpha *= kCodeScale;
        }
        // (a warp gives up as a whole; the next stage's codes are on their way into registers while this one's are unpacked)
        const auto unpack = [&](auto container, auto eight) {
            constexpr int CB = decltype(container)::value;
            constexpr bool EIGHT = decltype(eight)::value;
            const uint32_t base = centre_base<BF16>(a.bits);
            const UnitPlace<BACK> place(gid);
            RingAt ca, la;
            ca.next(group, code_slots);
            la.next(group, L);
            uint32_t w[kUnits][4], next[kUnits][4];
            const auto fetch = [&](uint32_t (&v)[kUnits][4]) {
                if (!__all_sync(0xffffffffu, tc_wait(&sh.codes_full[ca.slot], ca.turn, gave_up, a.status, 99))) return false;
                const uint8_t* p = packed + ca.slot * code_bytes + place.from * (2 * CB);
#pragma unroll
                for (int i = 0; i < kUnits; ++i) load_codes<CB>(p + i * UnitPlace<BACK>::kFromStep * (2 * CB), v[i]);
                return true;
            };
            const auto give_back = [&] {
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.codes_empty[ca.slot]);
                ca.next(kGroups, code_slots);
            };
            if (group >= steps) return true;
            if (!fetch(w)) return false;
            give_back();
            for (int s = group; s < steps; s += kGroups, la.next(kGroups, L)) {
                const bool more = s + kGroups < steps;
                if (more && !fetch(next)) return false;
                if (s >= L && !__all_sync(0xffffffffu, tc_wait(&sh.empty[la.slot], la.turn ^ 1u, gave_up, a.status, 100))) return false;
                unpack_stage<BF16, CB, EIGHT, BACK>(w, left + la.slot * kLeftBytes + place.to, base);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.written[la.slot]);
                if (more) {
                    give_back();
#pragma unroll
                    for (int i = 0; i < kUnits; ++i)
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[i][k] = next[i][k];
                }
            }
            return true;
        };
        using std::integral_constant;
        bool ok = cb == 4   ? unpack(integral_constant<int, 4>(), std::false_type())
                  : cb == 2 ? unpack(integral_constant<int, 2>(), std::false_type())
                  : BF16 && a.bits == 8 ? unpack(integral_constant<int, 8>(), integral_constant<bool, BF16>())
                                        : unpack(integral_constant<int, 8>(), std::false_type());
        if (ok) ok = __all_sync(0xffffffffu, tc_wait(&sh.plan, 0, gave_up, a.status, 101));
        if (ok && rank8 > 0) {
            if (a.early) asm volatile("griddepcontrol.wait;" ::: "memory");
            const bool bf16 = BACK ? a.out_bf16 != 0 : BF16;
            const uint32_t lowest = bf16 ? 0x00800080u : 0x04000400u;
            const uint16_t* up = reinterpret_cast<const uint16_t*>(a.up);
            const bool wide = ((reinterpret_cast<uintptr_t>(up) | (uintptr_t)((int64_t)a.features * 2)) & 15) == 0;
            const bool wide_h = ((reinterpret_cast<uintptr_t>(a.hidden) | (uintptr_t)(a.rank * 4)) & 15) == 0;
            const int entries = sh.entries, count = up_stages(), total = entries * rank8;
            bool bad = false;
            // Stages again, each group with a slot of its own.  What a stage needs from global memory is on its way before its slot is free.
            constexpr int U = kRankChunk * 16 / kGroupThreads, V = 2;      // units of 8 features of a rank, of 8 ranks of a token
            uint4 w[U];
            float v[V][8];
            int lo = 0, units = 0, row_shift = 0;
            const auto load_hidden = [&](int j, int from) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int u = from + gid + i * kGroupThreads, t = lo + (u >> row_shift), at = j * kRankChunk + (u & ((1 << row_shift) - 1)) * 8;
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[i][k] = 0.0f;
                    if (u >= units) continue;
                    const int e = (int)__umulhi((uint32_t)at, per_rank8), r = at - e * rank8;
                    if (sh.entry[t] == e) {
                        const float* h = a.hidden + (t0 + t) * a.rank + r;
                        if (wide_h && r + 8 <= a.rank) {
                            const float4 x = *reinterpret_cast<const float4*>(h), y = *reinterpret_cast<const float4*>(h + 4);
                            v[i][0] = x.x; v[i][1] = x.y; v[i][2] = x.z; v[i][3] = x.w;
                            v[i][4] = y.x; v[i][5] = y.y; v[i][6] = y.z; v[i][7] = y.w;
                        } else {
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                if (r + k < a.rank) v[i][k] = h[k];
                        }
                    }
                }
            };
            const auto load_stage = [&](int j) {
                // (a thread takes 8 features of every eighth rank: eight neighbouring ranks of the depth are one adapter's)
                static_assert(kGroupThreads == 8 * 16, "a unit of ranks a turn");
                const int f = f0 + (gid & 15) * 8, there = min(max(a.features - f, 0), 8);
                const uint16_t* column = up + f;
                const uint16_t* from[U];
                bool held[U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int at = j * kRankChunk + i * 8, e = (int)__umulhi((uint32_t)at, per_rank8), r = at - e * rank8 + (gid >> 4);
                    held[i] = e < entries && r < a.rank;
                    from[i] = column + ((int64_t)sh.entry_id[held[i] ? e : 0] * a.rank + r) * a.features;
                }
                if (wide && there == 8) {
#pragma unroll
                    for (int i = 0; i < U; ++i) w[i] = held[i] ? *reinterpret_cast<const uint4*>(from[i]) : make_uint4(0, 0, 0, 0);
                } else {
#pragma unroll
                    for (int i = 0; i < U; ++i) w[i] = load8_16(from[i], held[i] ? there : 0, false);
                }
                lo = PAIR ? side * Shape::kRightRows : sh.window_lo[j];
                const int n = PAIR ? Shape::kRightRows : sh.window_n[j];
                row_shift = total - j * kRankChunk > 16 ? 2 : 1;           // (a stage's depth counts as 16 or 32)
                units = n << row_shift;
                load_hidden(j, 0);
            };
            if (group < count) load_stage(group);
            if constexpr (Shape::kMerge) {
                if (count > 0) ok = __all_sync(0xffffffffu, tc_wait(&sh.codes_done, 0, gave_up, a.status, 114));
                if (count > 0 && ok) {
                    tc_fence_after();
                    const uint32_t lanes_at = tmem + ((uint32_t)((warp & 3) * 32) << 16);
                    for (int c = group; c < NT / 16; c += kGroups) {
                        uint32_t high[16], low[16];
                        tc_load16(lanes_at + c * 16, high);
                        tc_load16(lanes_at + Shape::kLowAt + c * 16, low);
                        tc_load_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) high[i] = __float_as_uint(__uint_as_float(high[i]) + __uint_as_float(low[i]));
                        tc_store16(lanes_at + c * 16, high);
                    }
                    tc_store_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if (PAIR && side != 0) tc_arrive_at(tc_peer(&sh.merged, 0));
                        else mbar_arrive(&sh.merged);
                    }
                }
            }
            for (int j = group; ok && j < count; j += kGroups) {
                const int padded = 8 << row_shift;
                ok = j < kGroups ? tc_wait(&sh.codes_done, 0, gave_up, a.status, 102)
                                 : tc_wait(&sh.up_empty[group], (j / kGroups - 1) & 1, gave_up, a.status, 105);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                uint8_t* dst = left + group * kLeftBytes;
                uint32_t marks = 0;
#pragma unroll
                for (int i = 0; i < U; ++i) marks |= not_finite(w[i], lowest);
                if (marks != 0) {
                    bad = true;
#pragma unroll
                    for (int i = 0; i < U; ++i)
                        w[i] = make_uint4(keep_finite(w[i].x, lowest), keep_finite(w[i].y, lowest), keep_finite(w[i].z, lowest), keep_finite(w[i].w, lowest));
                }
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int u = gid + i * kGroupThreads, k = u >> 4, chunk = u & 15;
                    if (k >= padded) continue;
                    *reinterpret_cast<uint4*>(dst + (chunk >> 3) * (kLeftBytes / 2) + k * 128 + (((chunk & 7) ^ (k & 7)) << 4)) = w[i];
                }
                uint8_t* tok = right + group * Shape::kRightBytes;
                const auto store_hidden = [&](auto type, int from) {
                    using T = decltype(type);
                    float inv[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int u = from + gid + i * kGroupThreads;
                        inv[i] = u < units ? 1.0f / sh.token[lo + (u >> row_shift)].hidden_scale : 0.0f;       // (a power of two)
                    }
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int u = from + gid + i * kGroupThreads, t = lo + (u >> row_shift), chunk = u & ((1 << row_shift) - 1);
                        if (u >= units) continue;
                        uint32_t high[4], low[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) split_pair<T>(v[i][2 * k] * inv[i], v[i][2 * k + 1] * inv[i], high[k], low[k]);
                        uint8_t* p = tok + (PAIR ? t - lo : t) * 128;
                        *reinterpret_cast<uint4*>(p + ((chunk ^ (t & 7)) << 4)) = make_uint4(high[0], high[1], high[2], high[3]);
                        *reinterpret_cast<uint4*>(p + (((chunk + 4) ^ (t & 7)) << 4)) = make_uint4(low[0], low[1], low[2], low[3]);
                    }
                };
                for (int from = 0; from < units; from += V * kGroupThreads) {
                    if (from > 0) load_hidden(j, from);
                    if (bf16) store_hidden(__nv_bfloat16(), from);
                    else store_hidden(__half(), from);
                }
                tc_publish();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR && side != 0) tc_arrive_at(tc_peer(&sh.up_full[group], 0));
                    else mbar_arrive(&sh.up_full[group]);
                }
                if (j + kGroups < count) load_stage(j + kGroups);
            }
            if (bad) set_status(a.status, ZIPML_ERR_NONFINITE, 103);
        }
        if (ok) ok = __all_sync(0xffffffffu, tc_wait(&sh.codes_done, 0, gave_up, a.status, 109) && tc_wait(&sh.done, 0, gave_up, a.status, 104));
        // (a group's warps meet at barriers of their own from here on: all of them or none)
        if (tc_agree(ok, 1 + group, kGroupThreads)) {
            tc_fence_after();
            // The groups take every third 16 tokens.  A whole tile's rows pass through shared memory on their way out, so that a thread stores 16
            // bytes of a token's row; rows that are not aligned for that go out as they lie, 32 features a warp.
            const bool have_up = sh.entries > 0, wide_out = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ldo * 2)) & 15) == 0;
            if (crank != 0) beta = 0.0f;
            const uint32_t lanes_at = tmem + ((uint32_t)((warp & 3) * 32) << 16);
            const bool merged = Shape::kMerge && have_up;
            uint32_t v[16] = {}, v2[Shape::kIssuers == 2 ? 16 : 1] = {}, w[16] = {};
            const auto load = [&](int c) {
                if (steps > 0) tc_load16(lanes_at + c * 16, v);
                if constexpr (Shape::kIssuers == 2)
                    if (steps > 1) tc_load16(lanes_at + NT + c * 16, v2);
                if (have_up) tc_load16(lanes_at + Shape::kUpAt + c * 16, w);
            };
            // MODE 0: into the cluster's exchange, 1: staged, 2: straight out
            const auto finish = [&](auto type, auto mode) {
                using T = decltype(type);
                constexpr int MODE = decltype(mode)::value;
                float* join = reinterpret_cast<float*>(ring) + row;
                T* stages = reinterpret_cast<T*>(ring) + group * 2 * 16 * kProjRows;
                int turn = 0;
                if (group < NT / 16) load(group);
                for (int c = group; c < NT / 16; c += kGroups, turn ^= 1) {
                    T* stage = stages + turn * 16 * kProjRows;            // (two buffers in turn: the next barrier tells that this one has been read)
                    if constexpr (Shape::kParts == 2) {
                        uint32_t low[16];
                        if (steps > 0 && !merged) {
                            tc_load16(lanes_at + Shape::kLowAt + c * 16, low);
                            tc_load_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(low[i]));
                        }
                        if constexpr (Shape::kIssuers == 2)
                            if (steps > 1) {
                                tc_load16(lanes_at + Shape::kLowAt + NT + c * 16, low);
                                tc_load_wait();
#pragma unroll
                                for (int i = 0; i < 16; ++i) v2[i] = __float_as_uint(__uint_as_float(v2[i]) + __uint_as_float(low[i]));
                            }
                    }
                    tc_load_wait();
                    // (four tokens' values before the first is stored: a store to shared memory holds back every load behind it)
#pragma unroll
                    for (int i0 = 0; i0 < 16; i0 += 4) {
                        ProjToken tok[4];
                        float y[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) tok[i] = sh.token[c * 16 + i0 + i];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float sum = __uint_as_float(v[i0 + i]);
                            if constexpr (Shape::kIssuers == 2) sum += __uint_as_float(v2[i0 + i]);
                            y[i] = fmaf(alpha * tok[i].row_scale, sum, fmaf(tok[i].hidden_scale, __uint_as_float(w[i0 + i]), beta * tok[i].sum));
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int t = i0 + i;
                            if constexpr (MODE == 0) join[(c * 16 + t) * kProjRows] = y[i];
                            else if constexpr (MODE == 1) stage[t * kProjRows + row] = from_float<T>(y[i]);
                            else if (tok[i].id != kNoRequest && feature < a.features) reinterpret_cast<T*>(a.out)[(t0 + c * 16 + t) * a.ldo + feature] = from_float<T>(y[i]);
                        }
                    }
                    if (c + kGroups < NT / 16) load(c + kGroups);         // (on its way while these rows go out)
                    if constexpr (MODE == 1) {
                        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(kGroupThreads) : "memory");
                        const int at = f0 + (gid & 15) * 8;
                        uint4 y[2];
                        bool there[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int t = (gid >> 4) + i * 8;
                            y[i] = *reinterpret_cast<const uint4*>(stage + t * kProjRows + (gid & 15) * 8);
                            there[i] = sh.token[c * 16 + t].id != kNoRequest && at < a.features;
                        }
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            if (!there[i]) continue;
                            uint16_t* p = reinterpret_cast<uint16_t*>(a.out) + (t0 + c * 16 + (gid >> 4) + i * 8) * a.ldo + at;
                            if (at + 8 <= a.features) *reinterpret_cast<uint4*>(p) = y[i];
                            else {
                                const uint32_t e[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
#pragma unroll
                                for (int k = 0; k < 8; ++k)
                                    if (at + k < a.features) p[k] = (uint16_t)(e[k >> 1] >> (16 * (k & 1)));
                            }
                        }
                    }
                }
            };
            const auto finish_as = [&](auto type) {
                if (cranks > 1) finish(type, std::integral_constant<int, 0>());
                else if (wide_out) finish(type, std::integral_constant<int, 1>());
                else finish(type, std::integral_constant<int, 2>());
            };
            if (BACK ? a.out_bf16 != 0 : BF16) finish_as(__nv_bfloat16());
            else finish_as(__half());
            tc_fence_before();
        }
    }
    __syncthreads();
    if (*gave_up) tc_settle();
    if constexpr (PAIR) cluster.sync();                               // (neither's memory goes while the other may still be at it)
    if (warp == 3) {
        tc_fence_after();
        tc_free<PAIR>(tmem, Shape::kColumns);
    }
    if (cranks > 1) {
        cluster.sync();
        const float* join = reinterpret_cast<const float*>(ring);
        for (int t = crank + cranks * warp; t < NT; t += cranks * (kProjThreads / 32)) {
            if (sh.token[t].id == kNoRequest) continue;
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

// How a group of project_kernel ends when one of its warps waits for what does not come: 128 threads, a barrier that nothing arrives at and
// one that all has arrived at.  See zipml_wait_probe.
__global__ void __launch_bounds__(kGroupThreads) group_probe_kernel(unsigned long long limit, DeviceStatus* status) {
    __shared__ uint64_t never, there;
    __shared__ int given_up;
    volatile int* gave_up = &given_up;
    if (threadIdx.x == 0) {
        mbar_init(&never, 1);
        mbar_init(&there, 1);
        given_up = 0;
        mbar_fence_init();
        mbar_arrive(&there);
    }
    __syncthreads();
    const bool ok = __all_sync(0xffffffffu, tc_wait(threadIdx.x < 32 ? &never : &there, 0, gave_up, status, 115, limit));
    if (tc_agree(ok, 1, kGroupThreads)) asm volatile("bar.sync 1, %0;" ::"n"(kGroupThreads) : "memory");
    __syncthreads();
    if (*gave_up) tc_settle();
}

int launch_group_probe(zipml_ctx* ctx, int64_t limit_ns) {
    group_probe_kernel<<<1, kGroupThreads, 0, ctx->stream>>>((unsigned long long)limit_ns, ctx->d_status);
    ctx->launches += 1;
    return cuda_status(cudaGetLastError());
}

int encode_map(zipml_ctx* ctx, CUtensorMapDataType type, const void* base, int64_t inner, int64_t rows, int64_t stride_bytes, int box_inner, int box_rows,
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

template <int NT, bool BACK, bool BF16, bool PAIR = false>
static int launch_project_as(zipml_ctx* ctx, const ProjectArgs& a, const CUtensorMap& tokens_map, const CUtensorMap& codes_map, int ranks) {
    auto kernel = &project_kernel<NT, BACK, BF16, PAIR>;
    constexpr size_t smem = 1024 + ProjShape<NT, PAIR, BACK>::kRing + sizeof(ProjShared<NT, PAIR, BACK>);
    static_assert(smem <= kMostShared, "what a block may have");
    const int rc = allow_shared(ctx, reinterpret_cast<const void*>(kernel), smem);
    if (rc != ZIPML_OK) return rc;
    constexpr int kTileRows = PAIR ? 2 * kProjRows : kProjRows;
    if (PAIR) ranks = 2;
    const int64_t tiles = (a.tokens + NT - 1) / NT * ((a.features + kTileRows - 1) / kTileRows);
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
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, tokens_map, codes_map);
    ctx->launches += 1;
    return cuda_status(e != cudaSuccess ? e : cudaGetLastError());
}

// Tokens of a tile and CTAs that divide the depth, by the cycles that the waves of tiles should take, as measured: 480 a stage and 1 for every
// token of a single CTA's tile, 580 for a pair's (backward, with two parts: 540 and 3, 1,060), and for a tile's start, adapters and
// epilogue 4,500 and 42 for every token, where the depth is divided 1,500 more.  (Whole calls, one
// after the other, rank 16: 64 tokens x 4096 x 14336 38 us with tiles of 64, 40 with 128, 92 with 16; 200 x 4096 x 4096 29 us with the depth
// divided, 33 without; 1000 x 4096 x 4096 43 us by pairs, 64 with tiles of 128, 96 with 64.  Backward 64 x 4096 x 4096 37 us with the depth of tiles of
// 64 divided by four, 45 with tiles of 16; 1000 x 4096 x 4096 84 us by pairs, 94 with 128; 2048 x 1000 x 1000 52 us with 128, 56 by pairs.)
static void project_shape(const zipml_ctx* ctx, const ProjectArgs& a, bool backward, int* tokens, int* ranks, bool* pair) {
    const int64_t feature_tiles = (a.features + kProjRows - 1) / kProjRows, steps = (a.depth + kProjDepth - 1) / kProjDepth;
    double best = 0.0;
    for (const int nt : {16, 64, 128, 256})
        for (int r = 1; r <= (nt == 256 ? 1 : 8); r *= 2) {
            if (r > 1 && steps / r < 4) break;
            if (nt == 256 && a.up && a.tokens < (int64_t)a.requests * 32) break;      // (a pair takes all of a tile's columns for each adapter)
            const int64_t ctas = (a.tokens + nt - 1) / nt * feature_tiles * r;
            const int64_t waves = (ctas + ctx->sm_count - 1) / ctx->sm_count;
            const int stage = backward ? (nt == 256 ? 1060 : 540 + 3 * nt) : nt == 256 ? 580 : 480 + nt;
            const double cycles = (double)waves * ((double)((steps + r - 1) / r) * stage + 4500 + nt * 42 + (r > 1 ? 1500 : 0));
            if (best == 0.0 || cycles < best) { best = cycles; *tokens = nt; *ranks = r; }
        }
    *pair = *tokens == 256;
}

template <bool BACK, bool BF16>
static int launch_project_typed(zipml_ctx* ctx, const ProjectArgs& a, const CUtensorMap& tm, const CUtensorMap& cm, int nt, int ranks, bool pair) {
    if (pair) return launch_project_as<256, BACK, BF16, true>(ctx, a, tm, cm, ranks);
    if (nt == 16) return launch_project_as<16, BACK, BF16>(ctx, a, tm, cm, ranks);
    if (nt == 64) return launch_project_as<64, BACK, BF16>(ctx, a, tm, cm, ranks);
    return launch_project_as<128, BACK, BF16>(ctx, a, tm, cm, ranks);
}

int launch_project(zipml_ctx* ctx, const ProjectArgs& a, const void* tokens_operand, int64_t ld_operand, bool operand_bf16, const zipml_dataset* w, bool backward) {
    int nt = 16, ranks = 1;
    bool pair = false;
    project_shape(ctx, a, backward, &nt, &ranks, &pair);
    CUtensorMap tokens_map, codes_map;
    int rc = encode_map(ctx, operand_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, tokens_operand, a.depth,
                        (backward ? 2 : 1) * a.tokens, ld_operand * 2,
                        kProjDepth, pair ? nt / 2 : nt, CU_TENSOR_MAP_SWIZZLE_128B, &tokens_map);
    if (rc != ZIPML_OK) return rc;
    rc = encode_map(ctx, CU_TENSOR_MAP_DATA_TYPE_UINT8, w->plane1, w->row_bytes, w->m, w->row_bytes, (backward ? kProjDepth : kProjRows) * container_bits(a.bits) / 8,
                    backward ? kProjRows : kProjDepth, CU_TENSOR_MAP_SWIZZLE_NONE, &codes_map);
    if (rc != ZIPML_OK) return rc;
    if (backward) return launch_project_typed<true, false>(ctx, a, tokens_map, codes_map, nt, ranks, pair);
    return operand_bf16 ? launch_project_typed<false, true>(ctx, a, tokens_map, codes_map, nt, ranks, pair)
                        : launch_project_typed<false, false>(ctx, a, tokens_map, codes_map, nt, ranks, pair);
}

}  // namespace zipml
