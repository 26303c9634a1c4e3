// Device code that the attention kernels of both kinds of cache share: arguments and plan, queues of work items, the way out of a
// wave tile and of a chunk tile, the pipelined step of a chunk tile, the kernels around the two paths and their launches.
// A cache kind is a class template `Paths<D>` with the LDS its paths need, the blocks of its wave tiles a compute unit is to hold, and
//   static int wave<STREAM>(params, tile, split, kv head, LDS, claim)      one 16-column wave tile, a block's work
//   static void chunk(params, tile, split, kv head, LDS)                   one 128-column chunk tile
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <cstring>
#include <type_traits>

#include "internal.h"

namespace sarathi {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

struct AttnParams {
    const uint16_t *q;
    const uint16_t *k_cache;
    const uint16_t *v_cache;
    uint16_t *out;
    const int32_t *block_table;
    const TileDesc *tiles;
    const uint32_t *units;
    float *part_ml;
    float *part_o;
    int64_t num_pages;
    int32_t max_blocks;
    int32_t num_q_heads;
    int32_t num_kv_heads;
    int32_t group;
    int32_t num_tile_units;  // units [0, num_tile_units) are 128-column chunk tiles (one block each)
    int32_t num_units;       // the rest are 16-column wave tiles (one block each as well)
    float scale_log2;        // sm_scale * log2(e): the softmax runs in base 2
    int32_t *sched;          // scheduling words (see internal.h)
    int32_t window;          // sliding window: a query at position p sees keys p-window+1 .. p; 0 = all keys up to p
};

// Arguments of a launch that carries its plan along and reads it where the arguments are: what the allocation-free call does with a
// small plan, instead of a launch of its own that puts it into memory (64 tokens next to three decodes, 4 heads and one, 14.2 -> 11.0 us a
// pass, the host's time for two launches).  Instantiations of their own, and two sizes: 4 KiB of arguments keep the host 0.5 us longer.
constexpr size_t kSmallPlanArgBytes = 960;
template <size_t BYTES>
struct AttnArgs {
    AttnParams base;
    uint32_t units_off;  // bytes from the plan's start to its work units
    uint32_t plan[BYTES / 4];
};
static_assert(sizeof(AttnArgs<kPlanArgBytes>) <= 4096, "kernel arguments are limited to 4 KiB");
__device__ __forceinline__ AttnParams attn_params(const AttnParams &p) { return p; }
template <size_t BYTES>
__device__ __forceinline__ AttnParams attn_params(const AttnArgs<BYTES> &a) {
    AttnParams p = a.base;
    const uintptr_t plan = (uintptr_t)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(AttnArgs<BYTES>, plan);
    p.tiles = reinterpret_cast<const TileDesc *>(plan);
    p.units = reinterpret_cast<const uint32_t *>(plan + a.units_off);
    return p;
}

// What one work unit (tile, split) covers.
struct UnitRange {
    int32_t key_begin;
    int32_t key_end;   // exclusive
    int32_t part_row;  // first partial row of this split, or -1: write `out` directly
};
__device__ __forceinline__ UnitRange unit_range(const TileDesc &t, int split) {
    UnitRange r;
    r.key_begin = t.key_lo + split * t.keys_per_split;
    r.key_end = min(t.n_keys, r.key_begin + t.keys_per_split);
    r.part_row = t.n_splits > 1 ? t.part_row0 + split * t.n_cols : -1;
    return r;
}

// Read-only int32 data fetched with scalar loads (wave-uniform indices): the block table and the plan.
typedef const int32_t __attribute__((address_space(4))) *const_i32_ptr;

__device__ __forceinline__ uint32_t load_unit(const AttnParams &p, int i) {
    return (uint32_t)((const_i32_ptr)p.units)[__builtin_amdgcn_readfirstlane(i)];
}
__device__ __forceinline__ TileDesc load_tile_desc(const AttnParams &p, uint32_t unit) {
    const const_i32_ptr t = (const_i32_ptr)(p.tiles + (unit & ((1u << kUnitTileBits) - 1)));
    return TileDesc{t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7], t[8], t[9], t[10], t[11]};
}

// Queues of work items.  An item is a unit for one KV head, number unit * Hkv + head; list x of a queue holds the items that
// are x modulo 8, in order, behind one counter.  A block's home list is its index modulo 8 and thereby its XCD: items whose
// K/V meet in one L2 stay together.  Whoever finds a list empty goes on with the next, so that no XCD waits for another:
// with every compute unit streaming, the XCDs differ by up to 10 % in speed, and with the items dealt out evenly the slowest
// decides (1024 decodes and two chunks: XCDs ended between 1459 and 1632 us).  The counters are relaxed atomics: they hand out
// indices into the read-only plan.  They start at zero; the first `taken` items are the blocks' first ones.
constexpr int kNoItem = 0x7FFFFFFF;
constexpr int kOneEach = 0, kQueued = 1, kRoles = 2;  // how a launch of both kinds of tile hands them out
struct Queue {
    int32_t *counters;
    int n_items, taken, list;
    __device__ __forceinline__ int bump() const {
        return __hip_atomic_fetch_add(counters + list * kSchedStride, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // the item at count `got` of the list, or kNoItem
    __device__ __forceinline__ int item(int got) const {
        const int i = queue_item(taken, list, got);
        return i < n_items ? i : kNoItem;
    }
    // Moves to the list that has most left; false if all are empty.  All counters are read at once: going round by
    // fetch-and-add would cost a block eight round trips to memory at its end.
    __device__ __forceinline__ bool move_on() {
        int counts[kSchedLists], most = 0;
#pragma unroll
        for (int x = 0; x < kSchedLists; ++x)
            counts[x] = __hip_atomic_load(counters + x * kSchedStride, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int x = 0; x < kSchedLists; ++x) {
            const int left = n_items - queue_item(taken, x, counts[x]);
            if (left > most) most = left, list = x;
        }
        return most > 0;
    }
    // the item at count `got`, or where the list is at its end one of another list, or kNoItem
    __device__ __forceinline__ int take(int got) {
        int i = item(got);
        while (i == kNoItem && move_on()) i = item(bump());
        return i;
    }
};

// The thread's index, as a value the compiler cannot follow: the per-lane offsets made from it are then formed anew for every item
// a block takes instead of being kept in registers across items (28 more registers, and 15 spilled).
__device__ __forceinline__ int thread_of_item() {
    int t = (int)threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

constexpr float kNegSentinel = -1.0e30f;  // finite "no key seen yet" running maximum
constexpr float kRescaleSlack = 8.0f;     // raise the softmax reference only when exceeded by 2^8
typedef __attribute__((ext_vector_type(16))) float f32x16;

__device__ __forceinline__ bf16x8 load_bf16x8(const uint16_t *p) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p));
}

typedef void __attribute__((address_space(3))) *lds_ptr;
__device__ __forceinline__ uint32_t lds_address(const uint16_t *p) {
    return (uint32_t)(uintptr_t)(lds_ptr)(p);
}
__device__ __forceinline__ bf16x8 lds_bf16x8(const uint16_t *p) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p));
}

// s_waitcnt with only the vector-memory counter constrained (gfx9 encoding: vmcnt in bits
// 3:0 and 15:14, expcnt 6:4 and lgkmcnt 11:8 left at their maxima).
#define SARATHI_WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | (((n) >> 4) << 14) | 0x0F70)
// the same for the LDS (and scalar-load) counter at zero
#define SARATHI_WAIT_LDS() __builtin_amdgcn_s_waitcnt(0xC07F)

// K rows sit unpadded in LDS (a direct global->LDS load writes 1 KiB of consecutive bytes per
// wavefront); the 16-byte chunks of row r are XOR-swizzled with this key so that the 16 lanes
// of a b128 read, which walk 16 different rows at the same logical chunk, hit distinct banks.
template <int D>
__device__ __forceinline__ int k_swizzle(int r) {
    return D == 128 ? (r & 15) : ((r >> 1) & 7);
}
// LDS element offset of the 8-slot half `hh` of V^T row `d` of page `u`: the two halves of a
// row are swapped on every other group of eight channels (conflict-free reads).
template <int D>
__device__ __forceinline__ int v_lds_off(int u, int d, int hh) {
    return ((u * D + d) * 2 + (hh ^ ((d >> 3) & 1))) * 8;
}

template <int D>
struct SoftmaxState {
    f32x4 o[D / 16];  // O^T accumulators: channel 16t + 4g + i, column n
    float m;          // running maximum (base-2 scaled scores), identical in the 4 lanes of a column
    float l;          // this lane's share of the running sum (summed over g at the end)
};

// The way out of a wave tile: the four wavefronts' results are merged in wavefront order through LDS (each publishes its own at
// WS::kWaveElems times its number), and the block writes the final rows, or one set of partial rows if the tile is split across blocks.
// col0: the first of the tile's columns that `st` holds sixteen of.
template <int D, typename WS>
__device__ __forceinline__ void wave_finish(const AttnParams &p, const TileDesc &it, int split, int kvh, int tid, uint16_t *smem,
                                            const SoftmaxState<D> &st, int col0 = 0) {
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15;
    const int g = lane >> 4;
    const int q_start = it.q_start;
    const int G = p.group;
    uint16_t *const ring = smem + wave * WS::kWaveElems;
    float l = st.l + __shfl_xor(st.l, 16);
    l += __shfl_xor(l, 32);

    // Publish this wavefront's piece where its ring was: lane (n, g) holds channels 16c + 4g + i of column n.
    {
        float *o_w = reinterpret_cast<float *>(ring) + n * WS::kColStride + g * 4;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) *reinterpret_cast<f32x4 *>(o_w + c * 16) = st.o[c];
        if (g == 0) {
            float *ml = reinterpret_cast<float *>(ring) + WS::kOutFloats + n * 2;
            ml[0] = st.m;
            ml[1] = l;
        }
    }
    __syncthreads();
    // Merge: thread t owns column t / 16 and D / 16 consecutive channels of it.
    constexpr int CH = D / 16;
    const int at = tid >> 4, mc = col0 + at;  // among these sixteen, and in the tile
    const int ch0 = (tid & 15) * CH;
    if (mc >= it.n_cols) return;
    float m_w[4], m_max = kNegSentinel;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        m_w[w] = reinterpret_cast<const float *>(smem + w * WS::kWaveElems)[WS::kOutFloats + at * 2];
        m_max = fmaxf(m_max, m_w[w]);
    }
    float acc[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) acc[j] = 0.f;
    float l_tot = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float wt = __builtin_amdgcn_exp2f(m_w[w] - m_max);
        const float *merge = reinterpret_cast<const float *>(smem + w * WS::kWaveElems);
        l_tot += wt * merge[WS::kOutFloats + at * 2 + 1];
        const float *o_w = merge + at * WS::kColStride + ch0;
#pragma unroll
        for (int j = 0; j < CH; j += 4) {
            const f32x4 o4 = *reinterpret_cast<const f32x4 *>(o_w + j);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j + i] += wt * o4[i];
        }
    }
    const int mcol = it.col_begin + mc;
    const int mrow = mcol / G;
    const int mhead = kvh * G + (mcol - mrow * G);
    const UnitRange whole = unit_range(it, split);
    if (whole.part_row < 0) {
        const float inv = 1.0f / l_tot;
        uint16_t *op = p.out + ((int64_t)(q_start + mrow) * p.num_q_heads + mhead) * D + ch0;
#pragma unroll
        for (int j = 0; j < CH; j += 4) {
            const f32x4 o = {acc[j] * inv, acc[j + 1] * inv, acc[j + 2] * inv, acc[j + 3] * inv};
            *reinterpret_cast<u32x2 *>(op + j) = __builtin_bit_cast(u32x2, __builtin_convertvector(o, bf16x4));
        }
        return;
    }
    // Tile split across blocks: this block's (reference maximum, sum, unnormalised output).
    const int64_t prow = ((int64_t)(whole.part_row + mc) * p.num_kv_heads + kvh);
    float *po = p.part_o + prow * D + ch0;
#pragma unroll
    for (int j = 0; j < CH; j += 4) *reinterpret_cast<f32x4 *>(po + j) = f32x4{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]};
    if ((tid & 15) == 0) {
        p.part_ml[prow * 2 + 0] = m_max;
        p.part_ml[prow * 2 + 1] = l_tot;
    }
}

// ---------------------------------------------------------------------------------------
// Chunk-tile path: 4 waves x 32 columns, K/V tiles of 32 keys staged in LDS.
// ---------------------------------------------------------------------------------------
// LDS of the chunk-tile path: a ring of 4 K tiles and a ring of 4 V tiles (32 keys each).
// In the step that handles tile t the wave reads K(t+1) and V(t-1) while K(t+2), K(t+3), V(t+1)
// and V(t+2) are in flight from global memory straight into LDS (no staging registers).  Tile
// with index rel (relative to the unit's first tile) lives in slot rel % 4 of its ring.
constexpr int kRing = 4;

template <int D>
struct ChunkSmem {
    static constexpr int kTileElems = kTileKeys * D;  // one K tile or one V tile: 32 keys x D channels
    static constexpr int kVBase = kRing * kTileElems;
    static constexpr int kTotalElems = 2 * kRing * kTileElems;
};

constexpr int kCarry = 3;  // output-MFMA operands read one step ahead

// State a wave carries from one tile to the next in the software-pipelined chunk loop.
template <int D>
struct ChunkState {
    f32x16 oacc[D / 32];  // O^T accumulators: channel 32c + 8*(r/4) + 4h + r%4, column n
    // Two register sets used in turn by consecutive steps of the unrolled loop (a step reads one
    // and fills the other); steps outside that loop keep everything in set 0.
    f32x16 s[2];          // raw scores of the tile whose softmax is due (already masked)
    bf16x8 p[2][2];       // bf16 softmax weights of the previous tile (B operands of its output MFMAs)
    bf16x8 carry[kCarry]; // V operands of the next step's first output MFMAs, read at the end of this step
    float tmax;           // scaled maximum of the due scores over the column
    float m_ref;          // softmax reference, scaled base-2 units
    float l_run;          // this lane's share of the running sum
};

// One pipelined step.  Independent work of three tiles shares one basic block so that the
// matrix pipe and the vector ALU run side by side inside a single wavefront:
//   MFMA:  S^T(t+1) = K(t+1) Q^T    (HAS_NEXT)        O^T += V^T(t-1) P^T(t-1)      (HAS_PREV)
//   VALU:  P(t) = 2^(S(t)*scale - m_ref), row sums, bf16 packing; mask and maximum of S(t+1)
// k_chunk: this lane's (swizzled) K chunk offsets; K_OFF / V_OFF: element offsets of the ring
// slots read in this step (wave-uniform).
// Order of the MFMAs of a step: which kind slot i issues and its index within that kind.  A step
// with both kinds opens with three output MFMAs (their V operands were read at the end of the
// previous step, so the matrix pipe has work right after the barrier, before any read of this step
// returns), then all score MFMAs (one accumulator; the scores are complete a few slots before the
// end of the step, so that masking and the maximum of the next tile also run under MFMAs), then the
// remaining output MFMAs.
struct ChunkSlot {
    bool is_score;
    int sub;
};
constexpr ChunkSlot chunk_slot(int i, int n_s, int n_o) {
    const int lead = n_o < kCarry ? n_o : kCarry;
    if (i < lead) return ChunkSlot{false, i};
    if (i < lead + n_s) return ChunkSlot{true, i - lead};
    return ChunkSlot{false, i - n_s};
}
constexpr int chunk_last_score_slot(int n_s, int n_o) {
    return n_s == 0 ? -1 : (n_o < kCarry ? n_o : kCarry) + n_s - 1;
}

// PHASE >= 0: the tile's index inside the unit is PHASE modulo 4, which fixes the ring slots at
// compile time (K_OFF_RT / V_OFF_RT are ignored and the operand reads need no address
// arithmetic); PHASE < 0: slots given at run time.  The step reads register set PP and fills set
// PP ^ 1 (SWAP) or set PP again (the results are copied back).
// CARRY_IN: the operands of the first kCarry output MFMAs are in st.carry (read by the previous step);
// CARRY_OUT: this step reads them for the next step (whose previous tile, this step's current one,
// has been in LDS and visible since this step's barrier).
template <int D, bool HAS_PREV, bool HAS_NEXT, bool MASK_NEXT, bool CARRY_IN, bool CARRY_OUT, int PHASE = -1, int PP = 0,
          bool SWAP = false>
__device__ __forceinline__ void chunk_step(ChunkState<D> &st, const bf16x8 (&qreg)[D / 16], const uint16_t *smem,
                                           const int (&k_chunk)[D / 16], int v_rd, int K_OFF_RT, int V_OFF_RT, float scale,
                                           int next_key0, int pos_eff, int lo) {
    constexpr int TE_ = kTileKeys * D;
    static_assert(!CARRY_IN || HAS_PREV, "carried operands belong to output MFMAs");
    const int K_OFF = PHASE >= 0 ? ((PHASE + 1) & (kRing - 1)) * TE_ : K_OFF_RT;
    const int V_OFF = PHASE >= 0 ? ((PHASE + 3) & (kRing - 1)) * TE_ : V_OFF_RT;
    const int V_OFF_NEXT = (V_OFF + TE_) & (kRing * TE_ - 1);  // ring slot of the current tile
    constexpr int OUT = SWAP ? (PP ^ 1) : PP;
    constexpr int NS = D / 16;
    constexpr int NB = D / 32;
    constexpr int N_S = HAS_NEXT ? NS : 0;              // score MFMAs (one dependent chain through s_next)
    constexpr int N_O = HAS_PREV ? 2 * NB : 0;          // output MFMAs (NB accumulators, two pages each)
    constexpr int NM = N_S + N_O;
    constexpr int AHEAD = 3;                             // operand reads run this many MFMAs ahead
    auto is_score = [&](int i) { return chunk_slot(i, N_S, N_O).is_score; };
    auto sub_index = [&](int i) { return chunk_slot(i, N_S, N_O).sub; };

    // The step is laid out as NM slots fenced by scheduling barriers.  Slot i issues the LDS
    // read for MFMA i+AHEAD, then MFMA i, then its share of the vector-ALU work, which
    // executes while the matrix pipe is busy with MFMA i.
    auto operand = [&](int i) -> const uint16_t * {
        const int j = sub_index(i);
        if (is_score(i)) return smem + K_OFF + k_chunk[j < NS ? j : 0];
        // output MFMA j: page j / NB, channel block j % NB
        return smem + v_rd + (V_OFF + ((j / NB) * D + (j % NB) * 32) * 16);
    };
    static_assert(AHEAD == kCarry, "the operands carried between steps fill the read-ahead window");
    bf16x8 frag[AHEAD + 1];
    bf16x8 nxt[kCarry];
#pragma unroll
    for (int i = 0; i < AHEAD && i < NM; ++i) frag[i] = CARRY_IN ? st.carry[i] : lds_bf16x8(operand(i));

    f32x16 s_tmp;
    f32x16 &s_next = SWAP ? st.s[OUT] : s_tmp;
    const f32x16 &s_cur = st.s[PP];
    const bf16x8 p_old0 = st.p[PP][0], p_old1 = st.p[PP][1];

    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    uint32_t p_new[8];  // bf16 pairs of the current tile's weights: registers (2k, 2k+1)
    float e_even = 0.f;
    float psum = 0.f;
    float smax = -INFINITY;
    float neg_m = -st.m_ref;
    auto weight = [&](int r) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s_cur[r], scale, neg_m));
        psum += e;
        if (r & 1) {
            const bf16x2 pk = __builtin_convertvector(f32x2{e_even, e}, bf16x2);
            p_new[r >> 1] = __builtin_bit_cast(uint32_t, pk);
        } else {
            e_even = e;
        }
    };
    // mask + running maximum of register r of the next tile (key next_key0 + 16*(r/8) + r%8)
    auto next_max = [&](int r) {
        if (MASK_NEXT) {  // causal bound and, under a sliding window, the column's first visible key
            const int key = next_key0 + (r >> 3) * 16 + (r & 7);
            s_next[r] = (key <= pos_eff && key >= lo) ? s_next[r] : -INFINITY;
        }
        smax = fmaxf(smax, s_next[r]);
    };
    constexpr int LAST_SCORE = chunk_last_score_slot(N_S, N_O);  // slot of the last score MFMA
    constexpr int MAX_FROM = LAST_SCORE + 2;  // first slot in which the finished scores may be touched
    int w_done = 0, m_done = 0;         // compile-time after unrolling
    // Slot boundaries.  The arithmetic below has no side effects, so nothing but data flow
    // would keep it inside its slot; an empty asm that "touches" the values a slot produced and
    // one input of the next slot's arithmetic (the negated reference) pins both, and the
    // scheduling barrier keeps the machine scheduler from undoing the layout.  Neither emits
    // an instruction.
    asm volatile("" : "+v"(neg_m), "+v"(psum));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NM; ++i) {
        bf16x8 &ahead = frag[(i + AHEAD) % (AHEAD + 1)];
        if (i + AHEAD < NM) ahead = lds_bf16x8(operand(i + AHEAD));
        else if (CARRY_OUT)  // operand j = i + AHEAD - NM of the next step: page j / NB, channel block j % NB of the current tile
            nxt[i + AHEAD - NM] = lds_bf16x8(smem + v_rd + (V_OFF_NEXT + (((i + AHEAD - NM) / NB) * D + ((i + AHEAD - NM) % NB) * 32) * 16));
        const bf16x8 a = frag[i % (AHEAD + 1)];
        const int j = sub_index(i);
        if (is_score(i)) {
            if (j == 0) {
                f32x16 zero;
#pragma unroll
                for (int r = 0; r < 16; ++r) zero[r] = 0.f;
                s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qreg[0], zero, 0, 0, 0);
            } else {
                s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qreg[j < NS ? j : 0], s_next, 0, 0, 0);
            }
        } else {
            st.oacc[j % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, (j / NB) ? p_old1 : p_old0, st.oacc[j % NB], 0, 0, 0);
        }
        // vector-ALU share of this slot
        const int w_from = w_done;
        const int w_target = 16 * (i + 1) / (NM > 0 ? NM : 1);
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (r >= w_from && r < w_target) weight(r);
        w_done = w_target;
        if (HAS_NEXT && i >= MAX_FROM) {
            const int m_target = 16 * (i + 1 - MAX_FROM) / (NM > MAX_FROM ? NM - MAX_FROM : 1);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (r >= m_done && r < m_target) next_max(r);
            m_done = m_target;
        }
        // pin: this slot's MFMA result and the weights made here.  The operand fetched ahead in
        // this slot is NOT pinned (that would make the slot wait for it); the scheduling barrier
        // alone keeps the read where it was issued.
        bf16x8 &older = frag[i % (AHEAD + 1)];
        if (is_score(i))
            asm volatile("" : "+v"(s_next), "+v"(older), "+v"(neg_m), "+v"(psum), "+v"(e_even));
        else if (i > LAST_SCORE)
            asm volatile("" : "+v"(st.oacc[j % NB]), "+v"(older), "+v"(neg_m), "+v"(psum), "+v"(e_even), "+v"(s_next), "+v"(smax));
        else
            asm volatile("" : "+v"(st.oacc[j % NB]), "+v"(older), "+v"(neg_m), "+v"(psum), "+v"(e_even));
#pragma unroll
        for (int r = 1; r < 16; r += 2)
            if (r >= w_from && r < w_target) asm volatile("" : "+v"(p_new[r >> 1]));
        __builtin_amdgcn_sched_barrier(0);
    }
    // whatever did not fit into the slots (steps without MFMAs, or too few of them)
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (r >= w_done) weight(r);
    if (HAS_NEXT) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (r >= m_done) next_max(r);
        // the other half-wave holds the other 16 keys of the column: one VALU half-swap, no LDS trip
        const auto halves = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, smax),
                                                             __builtin_bit_cast(uint32_t, smax), false, false);
        smax = fmaxf(__builtin_bit_cast(float, (uint32_t)halves[0]), __builtin_bit_cast(float, (uint32_t)halves[1]));
        st.tmax = smax * scale;  // scale > 0
        if (!SWAP) st.s[OUT] = s_tmp;
    }
    st.l_run += psum;
    if (CARRY_OUT) {
        static_assert(!CARRY_OUT || NM >= kCarry, "a step that reads ahead for the next one has at least kCarry slots");
#pragma unroll
        for (int j = 0; j < kCarry; ++j) st.carry[j] = nxt[j];
    }
    typedef __attribute__((ext_vector_type(4))) uint32_t pk4;
    st.p[OUT][0] = __builtin_bit_cast(bf16x8, pk4{p_new[0], p_new[1], p_new[2], p_new[3]});
    st.p[OUT][1] = __builtin_bit_cast(bf16x8, pk4{p_new[4], p_new[5], p_new[6], p_new[7]});
}

// The way out of a chunk tile: this wavefront's 32 columns, final or as a piece's partial rows.
template <int D>
__device__ __forceinline__ void chunk_finish(const AttnParams &p, const UnitRange &ur, const ChunkState<D> &st, int q_start, int row, int head, int kvh,
                                             int wcol, bool col_valid, int h) {
    constexpr int NB = D / 32;
    const f32x16 (&oacc)[NB] = st.oacc;
    const float l_run = st.l_run;
    const float m_ref = st.m_ref;
    const float l = l_run + __shfl_xor(l_run, 32);
    // accumulator register r of block c: channel 32c + 8*(r/4) + 4h + r%4
    uint16_t *op = p.out + ((int64_t)(q_start + row) * p.num_q_heads + head) * D + h * 4;
    if (ur.part_row < 0) {
        if (!col_valid) return;
        const float inv = 1.0f / l;
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                f32x4 o = {oacc[c][q4 * 4 + 0], oacc[c][q4 * 4 + 1], oacc[c][q4 * 4 + 2], oacc[c][q4 * 4 + 3]};
                const bf16x4 o4 = __builtin_convertvector(o * inv, bf16x4);
                *reinterpret_cast<u32x2 *>(op + c * 32 + q4 * 8) = __builtin_bit_cast(u32x2, o4);
            }
        return;
    }
    // Split tile: publish this piece's (reference maximum, sum, unnormalised output).
    if (col_valid) {
        const int64_t prow = ((int64_t)(ur.part_row + wcol) * p.num_kv_heads + kvh);
        float *po = p.part_o + prow * D + h * 4;
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                f32x4 o = {oacc[c][q4 * 4 + 0], oacc[c][q4 * 4 + 1], oacc[c][q4 * 4 + 2], oacc[c][q4 * 4 + 3]};
                *reinterpret_cast<f32x4 *>(po + c * 32 + q4 * 8) = o;
            }
        if (h == 0) {
            p.part_ml[prow * 2 + 0] = m_ref;
            p.part_ml[prow * 2 + 1] = l;
        }
    }
}

// Item `item` of the wave tiles.  An item's KV head is rotated by its sequence: with 8 heads item % 8 is also the XCD, the
// pages of one head lie 8 x 4 KiB apart, and an XCD that runs the same head of every sequence reads addresses of one residue
// only.  (1024 decodes + 2 chunks 1677 -> 1662 us, the long-context hybrid batch 978 -> 974, 256 decodes 224.7 -> 224.3.)  The
// column tiles of one sequence keep sharing an XCD, and chunk tiles, whose tiles share K/V in its L2, are not rotated.
template <typename Paths, bool STREAM, typename Claim>
__device__ __forceinline__ int wave_item(const AttnParams &p, int item, uint16_t *smem, Claim claim) {
    const int blk = item / p.num_kv_heads, kvh = item - blk * p.num_kv_heads;
    const uint32_t u = load_unit(p, p.num_tile_units + blk);
    const TileDesc it = load_tile_desc(p, u);
    return Paths::template wave<STREAM>(p, it, (int)(u >> kUnitTileBits), (kvh + it.seq) % p.num_kv_heads, smem, claim);
}
template <typename Paths>
__device__ __forceinline__ void chunk_item(const AttnParams &p, int item, uint16_t *smem) {
    const int blk = item / p.num_kv_heads, kvh = item - blk * p.num_kv_heads;  // consecutive items = the KV heads of one unit
    const uint32_t u = load_unit(p, blk);
    Paths::chunk(p, load_tile_desc(p, u), (int)(u >> kUnitTileBits), kvh, smem);
}

// Chunk tiles: one block per (unit, KV head); one wavefront per SIMD so that the pipelined
// loop has the registers it needs, the matrix pipe / vector ALU overlap comes from inside the wave.
template <typename Paths, typename Args>
__global__ __launch_bounds__(256, 2) void attn_chunk_kernel(Args args) {
    const AttnParams p = attn_params(args);
    __shared__ __attribute__((aligned(16))) uint16_t smem[Paths::kChunkElems];
    chunk_item<Paths>(p, (int)blockIdx.x, smem);
}

// Wave tiles (decodes, tiny chunks): one item per block or, QUEUED, the first gridDim.x items by the blocks in order and the
// others from the queue.
template <typename Paths, bool STREAM, bool QUEUED, typename Args>
__global__ __launch_bounds__(256, Paths::kWaveBlocksPerUnit) void attn_wave_kernel(Args args) {
    const AttnParams p = attn_params(args);
    __shared__ __attribute__((aligned(16))) uint16_t smem[Paths::kWaveElems];
    const int block = (int)blockIdx.x;
    if constexpr (!QUEUED) {
        wave_item<Paths, STREAM>(p, block, smem, [] { return 0; });
    } else {
        __shared__ int32_t next_item;
        Queue q{p.sched, (p.num_units - p.num_tile_units) * p.num_kv_heads, (int)gridDim.x, block % kSchedLists};
        for (int item = block; item != kNoItem;) {
            const int got = wave_item<Paths, STREAM>(p, item, smem, [&] { return q.bump(); });
            if (threadIdx.x == 0) next_item = q.take(got);
            __syncthreads();  // (and everyone is done with the ring's bytes; the next write is behind the next item's barrier)
            item = __builtin_amdgcn_readfirstlane(next_item);
        }
    }
}

// Both kinds of unit in ONE launch (saves the second stream's fork and join).
//
// kOneEach: a block per item, the chunk tiles in front.
// kQueued: the first blocks run a chunk tile each and the others begin with a wave tile; then all take wave tiles from the queue.
// kRoles: chunk blocks are compute-bound and wave blocks memory-bound, and they overlap only when they share a compute
// unit; two chunk blocks on one unit leave it without a memory stream.  So one block per compute unit (the first
// half of the grid, which the hardware spreads over the units before it gives any of them a second block) works off the chunk
// tiles and the other the wave tiles, each kind longest first, and a block whose queue is empty takes from the other one.
template <typename Paths, int MODE, bool STREAM, typename Args>
__global__ __launch_bounds__(256, 2) void attn_hybrid_kernel(Args args) {
    const AttnParams p = attn_params(args);
    constexpr int kSmemElems = Paths::kChunkElems > Paths::kWaveElems ? Paths::kChunkElems : Paths::kWaveElems;
    __shared__ __attribute__((aligned(16))) uint16_t smem[kSmemElems];
    const int n_chunk = p.num_tile_units * p.num_kv_heads;
    const int block = (int)blockIdx.x;
    if constexpr (MODE == kOneEach) {
        if (block < n_chunk) chunk_item<Paths>(p, block, smem);
        else wave_item<Paths, STREAM>(p, block - n_chunk, smem, [] { return 0; });
    } else {
        __shared__ int32_t next_item;  // of the wave tiles; chunk tiles are numbered behind them
        const int n_wave = (p.num_units - p.num_tile_units) * p.num_kv_heads, blocks = (int)gridDim.x;
        const int chunk_blocks = MODE == kRoles ? blocks / 2 : n_chunk;
        Queue waves{p.sched, n_wave, min(n_wave, blocks - chunk_blocks), block % kSchedLists};
        Queue chunks{p.sched + kSchedLists * kSchedStride, n_chunk, min(n_chunk, chunk_blocks), block % kSchedLists};
        // the first thread's choice of the next item, after a wave tile whose claim returned `got` or after a chunk tile
        auto next = [&](bool after_wave, int got) -> int {
            if (MODE == kQueued) return waves.take(after_wave ? got : waves.bump());
            if (after_wave) {
                const int w = waves.item(got);
                if (w != kNoItem) return w;
            } else {
                const int c = chunks.item(chunks.bump());
                if (c != kNoItem) return n_wave + c;
            }
            for (;;) {  // the own list is at its end
                const bool more_waves = waves.move_on(), more_chunks = chunks.move_on();
                if (!more_waves && !more_chunks) return kNoItem;
                if (more_waves && (after_wave || !more_chunks)) {
                    const int w = waves.item(waves.bump());
                    if (w != kNoItem) return w;
                } else {
                    const int c = chunks.item(chunks.bump());
                    if (c != kNoItem) return n_wave + c;
                }
            }
        };
        int item;
        if (block < chunk_blocks && block < n_chunk) item = n_wave + block;
        else if (block >= chunk_blocks && block - chunk_blocks < n_wave) item = block - chunk_blocks;
        else {  // fewer items of the preferred kind than blocks that prefer it
            if (threadIdx.x == 0) next_item = next(block >= chunk_blocks, n_wave / kSchedLists + 1);
            __syncthreads();
            item = __builtin_amdgcn_readfirstlane(next_item);
            __syncthreads();
        }
        while (item != kNoItem) {
            const bool wave = item < n_wave;
            int got = 0;
            if (wave) got = wave_item<Paths, STREAM>(p, item, smem, [&] { return waves.bump(); });
            else chunk_item<Paths>(p, item - n_wave, smem);
            if (threadIdx.x == 0) next_item = next(wave, got);
            __syncthreads();  // (and everyone is done with the rings)
            item = __builtin_amdgcn_readfirstlane(next_item);
            __syncthreads();
        }
    }
}

// Arguments of the launches that move rows of a batch to or from the pages of a cache: a block handles the slots of one page record for one
// KV head.
struct AppendParams {
    const uint16_t *k_new;
    const uint16_t *v_new;
    uint16_t *k_cache;
    uint16_t *v_cache;
    const int32_t *block_table;
    const AppendUnit *units;
    int64_t num_pages;
    int32_t max_blocks;
    int32_t num_kv_heads;
    // The first copy_blocks blocks move copy_n16 16-byte words from copy_src to copy_dst instead (the attention
    // metadata of the same iteration, pinned host memory -> workspace, riding in this launch).
    // The next zero_blocks clear zero_n16 words at zero_dst (scheduling words of the attention launch that follows).
    u32x4 *copy_dst;
    const u32x4 *copy_src;
    uint32_t copy_n16;
    uint32_t copy_blocks;
    u32x4 *zero_dst;
    uint32_t zero_n16;
    uint32_t zero_blocks;
};

// Small batches carry their records in the kernel's arguments, of two sizes, since the host copies them at each launch (64 tokens and 3 decodes
// in 384 bytes of records instead of 3584: 11.1 -> 10.6 us a pass; the argument block is on the device when the
// blocks start; a record in pinned host memory is a read across the host link at the head of every block's
// chain of dependent loads: record -> block-table entry -> stores).
constexpr int kInlineAppendUnits = 224, kFewAppendUnits = 24;
template <int UNITS>
struct AppendParamsInline {
    AppendParams base;
    AppendUnit units[UNITS];
};
static_assert(sizeof(AppendParamsInline<kInlineAppendUnits>) <= 4096, "kernel arguments are limited to 4 KiB");

// The launches of sarathi::launch_attention for one kind of cache.
template <template <int> class Paths>
int launch_attention_paths(const sarathi_config &cfg, const AttnMeta &m, const void *q, const void *k_cache, const void *v_cache, int64_t num_pages,
                           float sm_scale, void *out, int which, void *stream) {
    if (m.num_units == 0) return (int)hipSuccess;
    AttnParams p;
    p.q = static_cast<const uint16_t *>(q);
    p.k_cache = static_cast<const uint16_t *>(k_cache);
    p.v_cache = static_cast<const uint16_t *>(v_cache);
    p.out = static_cast<uint16_t *>(out);
    p.block_table = m.block_table;
    p.tiles = m.tiles;
    p.units = m.units;
    p.part_ml = m.part_ml;
    p.part_o = m.part_o;
    p.num_pages = num_pages;
    p.max_blocks = m.max_blocks;
    p.num_q_heads = cfg.num_q_heads;
    p.num_kv_heads = cfg.num_kv_heads;
    p.group = cfg.num_q_heads / cfg.num_kv_heads;
    p.num_tile_units = m.num_tile_units;
    p.num_units = m.num_units;
    p.scale_log2 = sm_scale * 1.4426950408889634f;
    p.sched = m.sched;
    p.window = m.window;
    if (m.plan_bytes > 0 && (m.plan_bytes > kPlanArgBytes || m.queue_blocks > 0)) return (int)hipErrorInvalidConfiguration;
    // launch(arguments) of a launch of a block per item
    auto with_plan = [&](auto launch) {
        if (m.plan_bytes == 0) return launch(p);
        auto carry = [&](auto args) {
            args.base = p;
            args.units_off = (uint32_t)(reinterpret_cast<const char *>(m.units) - reinterpret_cast<const char *>(m.tiles));
            std::memcpy(args.plan, m.tiles, m.plan_bytes);
            launch(args);
        };
        if (m.plan_bytes <= kSmallPlanArgBytes) carry(AttnArgs<kSmallPlanArgBytes>{}); else carry(AttnArgs<kPlanArgBytes>{});
    };
    const bool stream_kv = m.stream_kv != 0;
    // unused LDS that lowers the blocks per compute unit; all it can take next to the blocks' own 64 KiB already leaves one
    const unsigned dyn_lds = (unsigned)std::min<int32_t>(m.lds_pad_bytes, 95 * 1024);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned chunk_blocks = (unsigned)m.num_tile_units * (unsigned)cfg.num_kv_heads;
    const unsigned wave_blocks = (unsigned)(m.num_units - m.num_tile_units) * (unsigned)cfg.num_kv_heads;
    const unsigned in_flight = m.queue_blocks > 0 ? (unsigned)m.queue_blocks : 0xFFFFFFFFu;
    auto with_stream = [&](auto launch) {
        if (stream_kv) launch(std::true_type{}); else launch(std::false_type{});
    };
    if (which == 4 || which == 5) {
        const dim3 grid(std::min(chunk_blocks + wave_blocks, in_flight));
        auto launch = [&](auto d, auto mode) {
            with_stream([&](auto hint) {
                auto go = [&](const auto &args) {
                    hipLaunchKernelGGL((attn_hybrid_kernel<Paths<decltype(d)::value>, decltype(mode)::value, decltype(hint)::value, std::decay_t<decltype(args)>>), grid,
                                       dim3(256), dyn_lds, st, args);
                };
                if constexpr (decltype(mode)::value == kOneEach) with_plan(go); else go(p);
            });
        };
        auto pick_mode = [&](auto d) {
            if (which == 5) launch(d, std::integral_constant<int, kRoles>{});
            else if (m.queue_blocks > 0) launch(d, std::integral_constant<int, kQueued>{});
            else launch(d, std::integral_constant<int, kOneEach>{});
        };
        if (cfg.head_dim == 128) pick_mode(std::integral_constant<int, 128>{});
        else pick_mode(std::integral_constant<int, 64>{});
        return (int)hipGetLastError();
    }
    if (chunk_blocks && (which & 1)) {
        with_plan([&](const auto &args) {
            using Args = std::decay_t<decltype(args)>;
            if (cfg.head_dim == 128)
                hipLaunchKernelGGL((attn_chunk_kernel<Paths<128>, Args>), dim3(chunk_blocks), dim3(256), dyn_lds, st, args);
            else
                hipLaunchKernelGGL((attn_chunk_kernel<Paths<64>, Args>), dim3(chunk_blocks), dim3(256), dyn_lds, st, args);
        });
    }
    if (wave_blocks && (which & 2)) {
        const dim3 grid(std::min(wave_blocks, in_flight));
        auto launch = [&](auto d, auto queued) {
            with_stream([&](auto hint) {
                auto go = [&](const auto &args) {
                    hipLaunchKernelGGL((attn_wave_kernel<Paths<decltype(d)::value>, decltype(hint)::value, decltype(queued)::value, std::decay_t<decltype(args)>>), grid,
                                       dim3(256), dyn_lds, st, args);
                };
                if constexpr (!decltype(queued)::value) with_plan(go); else go(p);
            });
        };
        auto pick_queued = [&](auto d) {
            if (m.queue_blocks > 0) launch(d, std::true_type{}); else launch(d, std::false_type{});
        };
        if (cfg.head_dim == 128) pick_queued(std::integral_constant<int, 128>{});
        else pick_queued(std::integral_constant<int, 64>{});
    }
    return (int)hipGetLastError();
}
}  // namespace sarathi
