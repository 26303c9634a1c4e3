// gfx950 kernels of libsarathi: KV append, hybrid-batch attention over the paged cache,
// and the split-KV merge.
//
// Attention kernel (16-column wave tile).  A work item is 16 query COLUMNS (col = row*G +
// head_in_group, all sharing one KV head) against a key range; a workgroup of four wavefronts owns
// it, each wavefront walks a quarter of the keys in tiles of 32 (two pages), and the four results
// are merged in LDS (a decode has four memory streams from its first cycle and ends four times
// sooner than on one wavefront).  Both contractions run on v_mfma_f32_16x16x32_bf16 in the
// TRANSPOSED form so that the score accumulators already are the operand of the second one:
//
//   S^T[key, col] = sum_c K[key, c] * Q[col, c]      A = K tile (16 keys x 32 ch), B = Q^T
//   O^T[c,  col] += sum_key V^T[c, key] * P^T[key, col]   A = V^T tile (16 ch x 32 keys), B = P^T
//
// Operand layout of the instruction (64 lanes; g = lane/16, n = lane%16): A lane holds row n,
// contraction indices 8g..8g+7; B lane holds column n, contraction indices 8g..8g+7; the
// accumulator lane holds column n, rows 4g..4g+3.  With the K rows of the two score MFMAs of a
// tile assigned as  row 4g'+i of MFMA b  <->  key 8g'+4b+i,  lane (g, n) ends up with the eight
// scores of column n for keys 8g..8g+7 of the tile: exactly the B operand (P^T) of the second
// contraction, and V^T for those eight keys is one 16-byte run of the channel-major V page.
// The softmax is per-lane work plus two cross-lane steps (lanes n, n+16, n+32, n+48); there are no barriers in the key loop.
// K and V reach the operands through LDS: direct global -> LDS loads of whole pages into a ring that each wavefront has for
// itself.  Loaded straight into operands, sixteen neighbouring lanes touch sixteen K rows (or 32-byte V^T rows) at once, and
// the vector-memory path of a compute unit handles such a load at half the rate of one that reads 1 KiB front to back: 57
// against 90 to 106 GB/s for one compute unit out of its caches, 36 against 52 from memory while 64 of them stream.  That path
// is what decodes share with the chunk tiles of the same launch.  Straight into operands, and through LDS: 512 tokens behind
// 1871 next to 64 decodes, 32 and 8 heads, 124.1 and 107.6 us a call; 256 decodes 224.0 and 216.7; 512 decodes of 64 channels, 58
// and 2 heads, 173 and 123.  (The first two with the streaming hint, the last one without.  Next to chunk
// tiles neither gains alone: 124.6 us with neither, 121.7 with the hint, 124.9 through LDS, 110.8 with both on another part.)
//
// Chunk-tile path (prefill chunks).  A workgroup of four wavefronts owns 128 columns of one
// sequence (32 per wave) and walks the key range in 32-key tiles staged once per workgroup in
// LDS (rings of four K tiles and four V tiles filled by direct global -> LDS loads, K three tiles
// ahead of the step and V two; one barrier per tile), so K/V are fetched from L2/HBM once per 128
// columns instead of once per 16.  The contractions use v_mfma_f32_32x32x16_bf16, again in
// transposed form with the K rows of a tile permuted (MFMA row 16u+8a+4h+b <-> key 16u+8h+4a+b)
// so that accumulator lane (h, n) holds, for column n, keys 8h..8h+7 of page u in registers
// 8u..8u+7: the B operand of the second contraction without any data movement.  K rows are
// XOR-swizzled in LDS and the two 16-byte halves of a V^T row are swapped on every other group
// of eight channels, which makes both the staging writes and the operand reads bank-conflict free.
//
// Both paths share one launch: a block runs chunk tiles or wave tiles, one of them or, in long launches, many from a queue, so the
// memory-bound decodes fill the machine next to the MFMA-bound chunk tiles (the paper's reason
// for hybrid batches, section 4.1).
//
// The running maximum is only raised when a tile exceeds it by more than 2^8 (the softmax is
// invariant to the reference point as long as sum and output use the same one), which removes
// the accumulator rescale from almost every tile.
//
// Split-KV.  A tile whose key range was cut into pieces has every piece write its partial
// (reference maximum, sum, unnormalised output) triple; a second, small kernel merges the
// pieces of each tile in index order, so the result is bitwise reproducible.  (Merging inside
// the attention kernel by the last piece to finish was built twice and dropped on its timings.
// With device-scope release/acquire fences every block writes back and invalidates a whole L2 of
// this multi-die part: several times slower.  Without fences, the partial rows themselves written and
// read with device-scope accesses, whole 512-byte rows at a time, and a piece that finds the others
// done merging without publishing: correct, and still slower than the second kernel in every case
// measured (a 512-token chunk alone 57 us against 40 + 13, chunks of 256 tokens 1,866 us per prompt
// against 1,717), because such accesses bypass the L2 that serves the second kernel's reads, and
// ONE block per tile reads what 16 blocks of the merge kernel read in parallel.)
//
// Masking is by select: keys beyond a column's position (causal mask inside a chunk, section
// 4.1 of the paper) or beyond the item's key range get score -inf; V of slots at or beyond
// ctx_len is zeroed so that stale cache contents (possibly NaN) cannot reach an accumulator.
#include "attn_device.h"

#include <mutex>

namespace sarathi {

// One direct global -> LDS load moves 16 bytes per lane (1 KiB per wavefront): lane l fetches base + byte_off(l) and the
// wavefront's data lands at LDS byte address lds_addr + 16 l.
// Written as inline assembly on purpose: the compiler's wait-count bookkeeping treats the builtin form as a flat access
// that may return out of order with LDS reads, and from then on turns every wait for an LDS operand into a full drain of
// the LDS queue (in the chunk loop one pipeline bubble per four MFMAs).  The loads issued here are waited for by hand
// (SARATHI_WAIT_VMCNT), they are the only vector-memory accesses of the key loops.
// A whole page of one KV head (N loads of 1 KiB) behind ONE write of the LDS base register: the instruction's immediate
// offset is added to the global address and to the LDS address alike, so load j uses offset 1024 j and a lane offset that
// has 1024 j taken off (rel_off[j] = byte offset inside the page minus 1024 j, which is never negative: load j fetches the
// page's j-th KiB).  STREAM: with the non-temporal hint (K/V read once, far more than the caches hold).
template <int N, bool STREAM = false>
__device__ __forceinline__ void dma_load_page(const uint16_t *base, const int (&rel_off)[N], uint32_t lds_addr) {
    static_assert(N == 2 || N == 4, "pages of 2 KiB (d = 64) or 4 KiB (d = 128) per KV head");
    if constexpr (N == 4 && !STREAM) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %1, %5\n\t"
                     "global_load_lds_dwordx4 %2, %5 offset:1024\n\t"
                     "global_load_lds_dwordx4 %3, %5 offset:2048\n\t"
                     "global_load_lds_dwordx4 %4, %5 offset:3072"
                     :
                     : "s"(lds_addr), "v"(rel_off[0]), "v"(rel_off[1]), "v"(rel_off[2]), "v"(rel_off[3]), "s"(base)
                     : "memory");
    } else if constexpr (N == 4) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %1, %5 nt\n\t"
                     "global_load_lds_dwordx4 %2, %5 offset:1024 nt\n\t"
                     "global_load_lds_dwordx4 %3, %5 offset:2048 nt\n\t"
                     "global_load_lds_dwordx4 %4, %5 offset:3072 nt"
                     :
                     : "s"(lds_addr), "v"(rel_off[0]), "v"(rel_off[1]), "v"(rel_off[2]), "v"(rel_off[3]), "s"(base)
                     : "memory");
    } else if constexpr (!STREAM) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %1, %3\n\t"
                     "global_load_lds_dwordx4 %2, %3 offset:1024"
                     :
                     : "s"(lds_addr), "v"(rel_off[0]), "v"(rel_off[1]), "s"(base)
                     : "memory");
    } else {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %1, %3 nt\n\t"
                     "global_load_lds_dwordx4 %2, %3 offset:1024 nt"
                     :
                     : "s"(lds_addr), "v"(rel_off[0]), "v"(rel_off[1]), "s"(base)
                     : "memory");
    }
}

// LDS of a wave-tile block: every wavefront has a ring of kRingTiles tiles of 32 keys of its own (K pages 0 and 1, V pages
// 0 and 1); at the end the same bytes hold its 16 columns x (D + 4) floats of unnormalised output (the pad spreads the
// columns over the banks) and 16 x (maximum, sum) for the merge.
template <int D>
struct WaveSmem {
    static constexpr int kPageElems = kPageSize * D;
    static constexpr int kTileElems = 4 * kPageElems;
    static constexpr int kRingTiles = D == 128 ? 1 : 2;
    static constexpr int kWaveElems = kRingTiles * kTileElems;
    static constexpr int kTotalElems = 4 * kWaveElems;
    static constexpr int kColStride = D + 4;
    static constexpr int kOutFloats = kWaveCols * kColStride;
    static_assert((kOutFloats + 2 * kWaveCols) * 4 <= kWaveElems * 2, "the merge data fits the wavefront's ring");
};

// What a wavefront needs to move its K/V pages from global memory to its ring.
template <int D>
struct WaveLoads {
    static constexpr int kLoads = kPageSize * D / 512;  // 1 KiB loads per page of one KV head
    const uint16_t *k_head;  // page 0 of this KV head
    const uint16_t *v_head;
    const_i32_ptr bt;      // this sequence's block-table row (scalar loads)
    int64_t page_stride;   // elements per page (all KV heads)
    int64_t last_page_id;  // num_pages - 1 (page ids are clamped: a corrupt table cannot fault)
    int32_t n_pages_seq;   // pages that hold positions < ctx_len
    uint32_t lds_addr;     // of this wavefront's ring
    int k_off[2][kLoads];  // this lane's byte offsets (see dma_load_page) for a tile's K pages 0 and 1
    int v_off[kLoads];
};

// The two block-table entries of a 32-key tile: wave-uniform, by scalar loads, which the vector-memory counter does not see.
struct TilePages {
    int32_t e0, e1;
};
template <int D>
__device__ __forceinline__ TilePages tile_pages(const WaveLoads<D> &ge, int tile) {
    // Pages at or beyond ceil(ctx_len/16) are never dereferenced: the index is clamped to the
    // sequence's last page and whatever is loaded for such keys is masked.
    return TilePages{ge.bt[min(tile * 2, ge.n_pages_seq - 1)], ge.bt[min(tile * 2 + 1, ge.n_pages_seq - 1)]};
}
template <int D>
__device__ __forceinline__ int64_t page_offset(const WaveLoads<D> &ge, int32_t entry) {
    return (entry < 0 ? 0 : (entry > ge.last_page_id ? ge.last_page_id : (int64_t)entry)) * ge.page_stride;
}
template <int D, bool STREAM>
__device__ __forceinline__ void issue_k(const WaveLoads<D> &ge, const TilePages &pages, int slot) {
    const uint32_t dst = ge.lds_addr + (uint32_t)(slot * WaveSmem<D>::kTileElems * 2);
    dma_load_page<WaveLoads<D>::kLoads, STREAM>(ge.k_head + page_offset(ge, pages.e0), ge.k_off[0], dst);
    dma_load_page<WaveLoads<D>::kLoads, STREAM>(ge.k_head + page_offset(ge, pages.e1), ge.k_off[1], dst + WaveSmem<D>::kPageElems * 2);
}
template <int D, bool STREAM>
__device__ __forceinline__ void issue_v(const WaveLoads<D> &ge, const TilePages &pages, int slot) {
    const uint32_t dst = ge.lds_addr + (uint32_t)((slot * WaveSmem<D>::kTileElems + 2 * WaveSmem<D>::kPageElems) * 2);
    dma_load_page<WaveLoads<D>::kLoads, STREAM>(ge.v_head + page_offset(ge, pages.e0), ge.v_off, dst);
    dma_load_page<WaveLoads<D>::kLoads, STREAM>(ge.v_head + page_offset(ge, pages.e1), ge.v_off, dst + WaveSmem<D>::kPageElems * 2);
}

// Scores of a tile from its K operands, masked, and their softmax weights as the B operand of the second contraction.
template <int D>
__device__ __forceinline__ bf16x8 tile_weights(const bf16x8 (&k)[2][D / 32], const bf16x8 (&qreg)[D / 32], SoftmaxState<D> &st,
                                               int tile, int g, int pos_eff, int min_pos_eff, int lo, int max_lo, float scale_log2) {
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[0][s], qreg[s], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[1][s], qreg[s], s1, 0, 0, 0);
    }
    const int key0 = tile * kTileKeys + g * 8;  // this lane's eight keys: key0 .. key0+7
    float t[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        t[j] = s0[j] * scale_log2;
        t[4 + j] = s1[j] * scale_log2;
    }
    if (tile * kTileKeys + (kTileKeys - 1) > min_pos_eff) {  // wave-uniform: some lane must mask
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = (key0 + j <= pos_eff) ? t[j] : -INFINITY;
    }
    if (tile * kTileKeys < max_lo) {  // wave-uniform: some lane's sliding window starts inside or after this tile
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = (key0 + j >= lo) ? t[j] : -INFINITY;
    }
    float tmax = fmaxf(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])), fmaxf(fmaxf(t[4], t[5]), fmaxf(t[6], t[7])));
    tmax = fmaxf(tmax, __shfl_xor(tmax, 16));
    tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
    if (__any(tmax > st.m + kRescaleSlack)) {  // wave-uniform; rare after the first tiles
        const float m_new = fmaxf(st.m, tmax);
        const float alpha = __builtin_amdgcn_exp2f(st.m - m_new);
        st.l *= alpha;
        st.m = m_new;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) st.o[c] *= alpha;
    }
    f32x8 p;
    float psum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        p[j] = __builtin_amdgcn_exp2f(t[j] - st.m);
        psum += p[j];
    }
    st.l += psum;
    return __builtin_convertvector(p, bf16x8);
}

// One wave-tile unit = one block.  The unit's key range is quartered (in multiples of 32 keys) among
// the block's four wavefronts, which run the same loop as independent split-KV pieces and then merge
// their (maximum, sum, unnormalised output) through LDS in wavefront order: the block writes the final
// rows, or one set of partial rows if the tile is split further across blocks.
//
// A wavefront's ring holds 16 KiB (one tile of 128 channels, two of 64): a tile's K operands are read into registers, its K
// pages' slots filled with those of the tile kRingTiles on, then the same with V, so 8 to 16 KiB of a wavefront are always
// on their way.  Two blocks to a compute unit reach the chip's rate so (6.7 TB/s; rings twice as deep are no faster: a unit
// needs 64 KiB in flight at 26 GB/s).  With 64 channels one tile instead of two is 1 to 6 % slower.
//
// claim() is called by the block's first thread while its last tiles are on their way: the next item's counter is read
// under the last loads, and not so early that a block sits on an item that another could have begun.  Returns what it returned.
template <int D, bool STREAM, typename Claim>
__device__ __forceinline__ int wave16_path(const AttnParams &p, const TileDesc &it, int split, int kvh, uint16_t *smem, Claim claim) {
    const int tid = thread_of_item();
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15;
    const int g = lane >> 4;
    const int seq = it.seq;
    const int ctx = it.ctx_len;
    const int q_start = it.q_start;
    const int prefix = ctx - it.q_len;
    const int G = p.group;
    UnitRange ur = unit_range(it, split);
    {   // this wavefront's quarter of the unit (possibly empty: then it contributes weight zero)
        const int quarter = ((ur.key_end - ur.key_begin + 3) / 4 + kTileKeys - 1) / kTileKeys * kTileKeys;
        const int b = ur.key_begin + wave * quarter;   // a multiple of 32, as every piece start
        ur.key_end = min(ur.key_end, b + quarter);
        ur.key_begin = min(b, ur.key_end);
    }
    const bool piece_empty = ur.key_begin >= ur.key_end;

    // Lanes beyond the tile's valid columns shadow column 0 of the tile and store nothing.
    const bool col_valid = n < it.n_cols;
    const int col = it.col_begin + (col_valid ? n : 0);
    const int row = col / G;
    const int head = kvh * G + (col - row * G);
    const int pos_eff = min(prefix + row, ur.key_end - 1);                 // last key this column may see here
    const int min_pos_eff = min(prefix + it.col_begin / G, ur.key_end - 1);  // the same for the tile's first column
    // first key inside this column's sliding window, and the largest such key over the tile's columns
    const int lo = p.window > 0 ? max(0, prefix + row - p.window + 1) : 0;
    const int max_lo = p.window > 0 ? max(0, prefix + (it.col_begin + it.n_cols - 1) / G - p.window + 1) : 0;

    bf16x8 qreg[D / 32];
    {
        const uint16_t *qp = p.q + ((int64_t)(q_start + row) * p.num_q_heads + head) * D + g * 8;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) qreg[s] = load_bf16x8(qp + s * 32);
    }

    using WS = WaveSmem<D>;
    using WL = WaveLoads<D>;
    constexpr int kRing = WS::kRingTiles;
    constexpr int kPair = 2 * WL::kLoads;  // loads of a tile's K pages, and of its V pages
    uint16_t *const ring = smem + wave * WS::kWaveElems;
    WL ge;
    ge.k_head = p.k_cache + (int64_t)kvh * WS::kPageElems;
    ge.v_head = p.v_cache + (int64_t)kvh * WS::kPageElems;
    ge.bt = (const_i32_ptr)(p.block_table + (int64_t)seq * p.max_blocks);
    ge.page_stride = (int64_t)p.num_kv_heads * WS::kPageElems;
    ge.last_page_id = p.num_pages - 1;
    ge.n_pages_seq = (ctx + kPageSize - 1) / kPageSize;
    ge.lds_addr = lds_address(ring);
    // Page 1's K rows take part in the same reads as page 0's rows of the same slots: its swizzle key is moved by as many
    // chunks as four rows move it, which those reads leave out.
    constexpr int kPageKey = D == 128 ? 4 : 2;
    constexpr int kChunks = D / 8;  // 16-byte chunks of a K row
#pragma unroll
    for (int j = 0; j < WL::kLoads; ++j) {
        const int q = j * 64 + lane, slot = q / kChunks, d = q >> 1;
#pragma unroll
        for (int u = 0; u < 2; ++u)
            ge.k_off[u][j] = slot * D * 2 + ((q % kChunks) ^ k_swizzle<D>(slot) ^ (u * kPageKey)) * 16 - j * 1024;
        ge.v_off[j] = (d * 2 + ((q & 1) ^ ((d >> 3) & 1))) * 16 - j * 1024;
    }
    // K operand: A-row n of MFMA b is page n/8, slot ((n/4)&1)*8 + 4b + n%4; contraction step s: chunk 4s + g of that row
    int k_rd[2][D / 32];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const int slot = ((n >> 2) & 1) * 8 + 4 * b + (n & 3);
            k_rd[b][s] = (n >> 3) * WS::kPageElems + slot * D + ((4 * s + g) ^ k_swizzle<D>(slot) ^ ((n >> 3) * kPageKey)) * 8;
        }
    // V operand of output tile c: A-row n is channel 16c + n, contraction indices 8g .. are slots 8*(g&1) .. of page g/2
    const int v_rd = 2 * WS::kPageElems + v_lds_off<D>(g >> 1, n, g & 1);

    SoftmaxState<D> st;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) st.o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    st.m = kNegSentinel;
    st.l = 0.f;

    const int tile_begin = ur.key_begin / kTileKeys;
    const int tile_end = piece_empty ? tile_begin : (ur.key_end + kTileKeys - 1) / kTileKeys;

    TilePages pages = tile_pages(ge, tile_begin);
    SARATHI_WAIT_VMCNT(0);  // the queries, so that from here on the counter counts the direct loads only
#pragma unroll
    for (int i = 0; i < kRing; ++i)
        if (tile_begin + i < tile_end) {
            issue_k<D, STREAM>(ge, pages, i);
            issue_v<D, STREAM>(ge, pages, i);
            pages = tile_pages(ge, tile_begin + i + 1);
        }
    // One tile.  `left`: tiles still in the ring or, if `more`, all of it: how many loads are younger than the tile's.
    auto step = [&](int tile, int slot, auto left, auto more) {
        constexpr int kYounger = 2 * decltype(left)::value - 1;
        constexpr bool kMore = decltype(more)::value;
        const uint16_t *t_lds = ring + slot * WS::kTileElems;
        SARATHI_WAIT_VMCNT(kYounger * kPair);
        asm volatile("" ::: "memory");
        bf16x8 k[2][D / 32];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int s = 0; s < D / 32; ++s) k[b][s] = lds_bf16x8(t_lds + k_rd[b][s]);
        SARATHI_WAIT_LDS();  // the operands are in registers: their slots may be filled again
        asm volatile("" ::: "memory");
        if (kMore) issue_k<D, STREAM>(ge, pages, slot);
        const bf16x8 pT = tile_weights<D>(k, qreg, st, tile, g, pos_eff, min_pos_eff, lo, max_lo, p.scale_log2);
        SARATHI_WAIT_VMCNT((kMore ? kYounger : kYounger - 1) * kPair);
        asm volatile("" ::: "memory");
        bf16x8 v[D / 16];
#pragma unroll
        for (int c = 0; c < D / 16; ++c) v[c] = lds_bf16x8(t_lds + v_rd + c * 16 * kPageSize);
        SARATHI_WAIT_LDS();
        asm volatile("" ::: "memory");
        if (kMore) {
            issue_v<D, STREAM>(ge, pages, slot);
            pages = tile_pages(ge, tile + kRing + 1);
        }
        if (tile * kTileKeys + kTileKeys > ctx) {  // wave-uniform: tile holds slots at or beyond ctx_len
            u32x4 keep;
            const int key0 = tile * kTileKeys + g * 8;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                keep[w] = ((key0 + 2 * w < ctx) ? 0x0000FFFFu : 0u) | ((key0 + 2 * w + 1 < ctx) ? 0xFFFF0000u : 0u);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) v[c] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, v[c]) & keep);
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) st.o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[c], pT, st.o[c], 0, 0, 0);
    };
    int tile = tile_begin, slot = 0;
    for (; tile + kRing + 1 < tile_end; ++tile) {
        step(tile, slot, std::integral_constant<int, kRing>{}, std::true_type{});
        slot = slot + 1 == kRing ? 0 : slot + 1;
    }
    int claimed = 0;
    if (tid == 0) claimed = claim();  // in front of the last tile's loads: results come back in order
    if (tile + kRing < tile_end) {
        step(tile, slot, std::integral_constant<int, kRing>{}, std::true_type{});
        ++tile;
        slot = slot + 1 == kRing ? 0 : slot + 1;
    }
    if (kRing == 2 && tile + 1 < tile_end) {
        step(tile, slot, std::integral_constant<int, 2>{}, std::false_type{});
        ++tile;
        slot ^= 1;
    }
    if (tile < tile_end) step(tile, slot, std::integral_constant<int, 1>{}, std::false_type{});

    wave_finish<D, WS>(p, it, split, kvh, tid, smem, st);
    return claimed;
}

template <int D>
__device__ __forceinline__ void chunk_tile_path(const AttnParams &p, const TileDesc &it, int split, int kvh,
                                                uint16_t *smem) {
    constexpr int NS = D / 16;            // contraction steps of the score MFMAs
    constexpr int NB = D / 32;            // 32-channel blocks of the output
    constexpr int CPR = D / 8;            // 16-byte chunks per K row
    constexpr int PAGE_ELEMS = kPageSize * D;
    constexpr int LOADS_PER_PAGE = PAGE_ELEMS / 512;  // 1 KiB wavefront loads per page of one KV head
    using SM = ChunkSmem<D>;
    constexpr int TE = SM::kTileElems;
    const int tid = thread_of_item();
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // wave-uniform by construction; tell the compiler
    const int n = lane & 31;
    const int h = lane >> 5;
    const int seq = it.seq;
    const int ctx = it.ctx_len;
    const int q_start = it.q_start;
    const int prefix = ctx - it.q_len;
    const int G = p.group;
    const UnitRange ur = unit_range(it, split);

    // Columns of this wave; lanes (and whole waves) without a valid column shadow the tile's first column.
    const int wcol = wave * 32 + n;
    const bool col_valid = wcol < it.n_cols;
    const int col = it.col_begin + (col_valid ? wcol : 0);
    const int row = col / G;
    const int head = kvh * G + (col - row * G);
    const int pos_eff = min(prefix + row, ur.key_end - 1);
    const int wave_first_col = it.col_begin + ((wave * 32 < it.n_cols) ? wave * 32 : 0);
    const int min_pos_eff = min(prefix + wave_first_col / G, ur.key_end - 1);  // wave-uniform
    // Sliding window: first key this column sees, and the largest such key over the wave's valid
    // columns (wave-uniform; a wave without valid columns shadows the tile's first column).
    const int wave_last_col = it.col_begin + ((wave * 32 < it.n_cols) ? min(wave * 32 + 31, it.n_cols - 1) : 0);
    const int lo = p.window > 0 ? max(0, prefix + row - p.window + 1) : 0;
    const int max_lo = p.window > 0 ? max(0, prefix + wave_last_col / G - p.window + 1) : 0;

    bf16x8 qreg[NS];  // B operand of the score MFMAs: column n, channels 16s + 8h ..
    {
        const uint16_t *qp = p.q + ((int64_t)(q_start + row) * p.num_q_heads + head) * D + h * 8;
#pragma unroll
        for (int s = 0; s < NS; ++s) qreg[s] = load_bf16x8(qp + s * 16);
    }

    // Global -> LDS traffic of a tile: wave 0/1 move K page 0/1, wave 2/3 move V page 0/1, each
    // as LOADS_PER_PAGE direct loads of 1 KiB.  Lane l of load j fills physical 16-byte chunk
    // q = 64j + l of the page's LDS image and therefore fetches the logical chunk that lives there.
    // K pages run three tiles ahead of the step, V pages two (V is consumed two steps later than K).
    const bool moves_v = wave >= 2;
    const int my_page = wave & 1;
    int g_off[LOADS_PER_PAGE];  // this lane's byte offset inside the page of one KV head, per load, minus 1024 j
#pragma unroll
    for (int j = 0; j < LOADS_PER_PAGE; ++j) {
        const int q = j * 64 + lane;
        const int k_slot = q / CPR;
        const int k_elem = k_slot * D + ((q % CPR) ^ k_swizzle<D>(k_slot)) * 8;
        const int v_d = q >> 1;
        const int v_elem = (v_d * 2 + ((q & 1) ^ ((v_d >> 3) & 1))) * 8;
        g_off[j] = (moves_v ? v_elem : k_elem) * 2 - j * 1024;  // relative to the load's own KiB (see dma_load_page)
    }
    const const_i32_ptr bt = (const_i32_ptr)(p.block_table + (int64_t)seq * p.max_blocks);  // read-only: scalar loads
    const int n_pages_seq = (ctx + kPageSize - 1) / kPageSize;
    const int64_t page_stride = (int64_t)p.num_kv_heads * kPageSize * D;
    const uint16_t *cache_head = (moves_v ? p.v_cache : p.k_cache) + (int64_t)kvh * PAGE_ELEMS;
    const int64_t last_page_id = p.num_pages - 1;
    const int tile_begin = ur.key_begin / kTileKeys;
    const int tile_end = (ur.key_end + kTileKeys - 1) / kTileKeys;
    const int n_tiles = tile_end - tile_begin;
    const int my_lds_base = (moves_v ? SM::kVBase : 0) + my_page * PAGE_ELEMS;
    const uint32_t smem_addr = lds_address(smem);
    // page id of this wave's page of tile `tile` (a scalar load: issue it a step before it is needed)
    // The raw table entry and its clamp are separate so that the entry can be fetched a step
    // before it is needed and only then looked at (the clamp would otherwise wait for the load).
    auto page_raw = [&](int tile) -> int32_t { return bt[min(tile * 2 + my_page, n_pages_seq - 1)]; };
    auto page_clamp = [&](int32_t raw) -> int64_t {
        const int64_t pg = raw;
        return pg < 0 ? 0 : (pg > last_page_id ? last_page_id : pg);
    };
    auto page_of = [&](int tile) -> int64_t { return page_clamp(page_raw(tile)); };
    // this wave's page `pg` of tile `tile` -> ring slot (tile - tile_begin) % 4
    auto issue_page = [&](int tile, int64_t pg) {
        const uint16_t *src = cache_head + pg * page_stride;
        const uint32_t dst = smem_addr + (uint32_t)(my_lds_base + ((tile - tile_begin) & (kRing - 1)) * TE) * 2;
        dma_load_page<LOADS_PER_PAGE>(src, g_off, dst);
    };
    auto issue_tile = [&](int tile) { issue_page(tile, page_of(tile)); };
    const int my_ahead = moves_v ? 2 : 3;  // tiles this wave's loads run ahead of the step

    ChunkState<D> st;
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.oacc[c][r] = 0.f;
    st.m_ref = kNegSentinel;
    st.l_run = 0.f;
    st.tmax = kNegSentinel;

    // MFMA row n of the score tile is key  16u + 8h' + 4a + b  for n = 16u + 8a + 4h' + b.
    const int k_row = (n & 16) | ((n & 4) << 1) | ((n & 8) >> 1) | (n & 3);
    int k_chunk[NS];  // element offset of contraction step s inside this lane's K row (swizzled)
#pragma unroll
    for (int s = 0; s < NS; ++s) k_chunk[s] = k_row * D + ((s * 2 + h) ^ k_swizzle<D>(k_row)) * 8;
    const int v_rd = SM::kVBase + v_lds_off<D>(0, n, h);  // + slot*TE + (u*D + 32c)*16 elements
    const float scale = p.scale_log2;
    // first tile of the range in which some column of this wave needs masking (wave-uniform)
    const int mask_from = max(tile_begin, min(tile_end, (min_pos_eff + 1) / kTileKeys));
    // tiles below this index hold keys in front of some column's sliding window (wave-uniform; = tile_begin without one)
    const int mask_until = max(tile_begin, min(tile_end, (max_lo + kTileKeys - 1) / kTileKeys));

    // Prologue: the first tiles start loading; when they have landed the scores of tile 0 are
    // formed (as the "next" tile of an otherwise empty step).
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < my_ahead && i < n_tiles) issue_tile(tile_begin + i);
    SARATHI_WAIT_VMCNT(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    {
#pragma unroll
        for (int r = 0; r < 16; ++r) st.s[0][r] = -INFINITY;  // "current" tile of the empty step: weights 0
        st.p[0][0] = st.p[0][1] = bf16x8{};
        const int key0 = tile_begin * kTileKeys + h * 8;
        if (tile_begin >= mask_from || tile_begin < mask_until)
            chunk_step<D, false, true, true, false, false>(st, qreg, smem, k_chunk, v_rd, 0, 0, scale, key0, pos_eff, lo);
        else
            chunk_step<D, false, true, false, false, false>(st, qreg, smem, k_chunk, v_rd, 0, 0, scale, key0, pos_eff, lo);
        st.l_run = 0.f;  // the empty step contributed exp2(-inf) = 0 terms only
    }

    int32_t pg_next = page_raw(tile_begin + my_ahead);  // table entry of the page the first step will fetch
    // Common head of a step for tile t, then the step proper.  Every loop below instantiates one
    // variant only, so its body stays a single basic block (plus the rare reference raise).
    // Every step but a unit's last fetches this wave's page of tile t + my_ahead; beyond the
    // unit's end that is a clamped, unused page landing in a free ring slot, which keeps the loop
    // body and the load counter the same for all steps.
    // pg_this: table entry of the page this step fetches; fetch_next: the step itself fetches the
    // entry of the step after it (single steps), or the caller brings entries in batches (the unrolled
    // group: while a scalar load is in flight every wait for an LDS read must wait for all of them,
    // so one batch per four steps costs a quarter of what one load per step did).
    auto step = [&](int tile, auto has_prev, auto has_next, auto mask_next, auto with_dma, auto phase, auto pp,
                    int32_t pg_this, auto fetch_next) {
        // Tile t+1 must have landed (only this wave's loads of one later tile may still be in
        // flight), and every wave must be done with the slots about to be overwritten (K of
        // tile t-1, V of tile t-2).
        if (decltype(with_dma)::value) SARATHI_WAIT_VMCNT(LOADS_PER_PAGE); else SARATHI_WAIT_VMCNT(0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int rel = tile - tile_begin;
        if (decltype(with_dma)::value) {
            issue_page(tile + my_ahead, page_clamp(pg_this));
            if (decltype(fetch_next)::value) pg_next = page_raw(tile + my_ahead + 1);  // looked at in the next step only
        }
        // Raise the softmax reference of the columns whose due tile exceeds it by more than the slack
        // (rare).  Three things carry the old reference: the output accumulators (tiles up to t-2), the
        // running sum (up to t-1) and the bf16 weights of tile t-1, which still wait for their output
        // MFMAs in this step; all three are brought to the new one.  Columns that keep their
        // reference get alpha = 1 (both half-waves of a column see the same tmax and m_ref).
        if (__any(st.tmax > st.m_ref + kRescaleSlack)) {
            const float m_new = (st.tmax > st.m_ref + kRescaleSlack) ? st.tmax : st.m_ref;
            const float alpha = __builtin_amdgcn_exp2f(st.m_ref - m_new);
            st.l_run *= alpha;
            st.m_ref = m_new;
#pragma unroll
            for (int c = 0; c < NB; ++c) st.oacc[c] *= alpha;
            constexpr int kSet = decltype(pp)::value;
#pragma unroll
            for (int u = 0; u < 2; ++u)
                st.p[kSet][u] = __builtin_convertvector(__builtin_convertvector(st.p[kSet][u], f32x8) * alpha, bf16x8);
        }
        const int next_key0 = (tile + 1) * kTileKeys + h * 8;
        constexpr int kPhase = decltype(phase)::value;
        // every step with a predecessor finds its first V operands carried over; every step with a successor reads them
        chunk_step<D, decltype(has_prev)::value, decltype(has_next)::value, decltype(mask_next)::value,
                   decltype(has_prev)::value, decltype(has_next)::value, kPhase, decltype(pp)::value, (kPhase >= 0)>(
            st, qreg, smem, k_chunk, v_rd, ((rel + 1) & (kRing - 1)) * TE, ((rel + 3) & (kRing - 1)) * TE, scale, next_key0,
            pos_eff, lo);
    };
    using T = std::true_type;
    using F = std::false_type;
    using DYN = std::integral_constant<int, -1>;  // ring slots taken from the tile index at run time
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    using P2 = std::integral_constant<int, 2>;
    using P3 = std::integral_constant<int, 3>;
    if (n_tiles == 1) {
        step(tile_begin, F{}, F{}, F{}, F{}, DYN{}, P0{}, pg_next, F{});
    } else {
        // first tile: nothing to accumulate yet
        if (tile_begin + 1 >= mask_from || tile_begin + 1 < mask_until) step(tile_begin, F{}, T{}, T{}, T{}, DYN{}, P0{}, pg_next, T{});
        else step(tile_begin, F{}, T{}, F{}, T{}, DYN{}, P0{}, pg_next, T{});
        // steady state, unmasked tiles: groups of four steps with the ring slots and the register
        // sets compiled in (the group starts at tile index 1 modulo 4 and leaves the state in set 0),
        // then single steps up to the causal diagonal
        int tile = tile_begin + 1;
        // tiles in front of a sliding window's start (none without a window), then single steps up to the
        // tile index the unrolled group expects
        for (; tile + 1 < tile_end && tile + 1 < mask_until; ++tile) step(tile, T{}, T{}, T{}, T{}, DYN{}, P0{}, pg_next, T{});
        for (; tile + 1 < tile_end && tile + 1 < mask_from && ((tile - tile_begin) & 3) != 1; ++tile)
            step(tile, T{}, T{}, F{}, T{}, DYN{}, P0{}, pg_next, T{});
        if (tile + 4 < tile_end && tile + 4 < mask_from) {
            // table entries of the pages the group's steps fetch; the next group's come in one batch
            int32_t e0 = pg_next, e1 = page_raw(tile + my_ahead + 1), e2 = page_raw(tile + my_ahead + 2),
                    e3 = page_raw(tile + my_ahead + 3);
            for (; tile + 4 < tile_end && tile + 4 < mask_from; tile += 4) {
                const int32_t n0 = page_raw(tile + my_ahead + 4), n1 = page_raw(tile + my_ahead + 5),
                              n2 = page_raw(tile + my_ahead + 6), n3 = page_raw(tile + my_ahead + 7);
                step(tile, T{}, T{}, F{}, T{}, P1{}, P0{}, e0, F{});
                step(tile + 1, T{}, T{}, F{}, T{}, P2{}, P1{}, e1, F{});
                step(tile + 2, T{}, T{}, F{}, T{}, P3{}, P0{}, e2, F{});
                step(tile + 3, T{}, T{}, F{}, T{}, P0{}, P1{}, e3, F{});
                e0 = n0, e1 = n1, e2 = n2, e3 = n3;
            }
            pg_next = e0;
        }
        for (; tile + 1 < tile_end && tile + 1 < mask_from; ++tile) step(tile, T{}, T{}, F{}, T{}, DYN{}, P0{}, pg_next, T{});
        // the tiles on the causal diagonal
        for (; tile + 1 < tile_end; ++tile) step(tile, T{}, T{}, T{}, T{}, DYN{}, P0{}, pg_next, T{});
        // last tile: no further scores to form, nothing more to fetch (and no load left in flight after it)
        step(tile_end - 1, T{}, F{}, F{}, F{}, DYN{}, P0{}, pg_next, F{});
    }
    // Epilogue: the output MFMAs of the last tile.  Only here can a tile hold slots at or beyond
    // ctx_len (a unit never extends past the sequence), whose V bits must be zeroed: stale cache
    // contents times a zero weight would still poison the accumulator if they were NaN or Inf.
    {
        const int last = tile_end - 1;
        const uint16_t *v_last = smem + v_rd + ((last - tile_begin) & (kRing - 1)) * TE;
        const bool tail = last * kTileKeys + kTileKeys > ctx;
#pragma unroll
        for (int c = 0; c < NB; ++c) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4 v = *reinterpret_cast<const u32x4 *>(v_last + (u * D + c * 32) * 16);
                if (tail) {
                    const int key0 = last * kTileKeys + u * kPageSize + h * 8;
#pragma unroll
                    for (int w = 0; w < 4; ++w)
                        v[w] &= ((key0 + 2 * w < ctx) ? 0x0000FFFFu : 0u) | ((key0 + 2 * w + 1 < ctx) ? 0xFFFF0000u : 0u);
                }
                st.oacc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), st.p[0][u],
                                                                      st.oacc[c], 0, 0, 0);
            }
        }
    }
    chunk_finish<D>(p, ur, st, q_start, row, head, kvh, wcol, col_valid, h);
}

// Per-call metadata, host -> device: a kernel that reads the pinned host buffer itself.  The runtime's copy
// goes through a copy kernel for a few kilobytes and through the DMA engine beyond that, and the DMA path
// leaves the stream idle for 10 us before and 13-23 us after the copy (kernel and copy trace of the
// decode-only batch, 13 KiB of metadata); a kernel of ours is followed by the next one at once.
__global__ __launch_bounds__(256) void upload_kernel(u32x4 *dst, const u32x4 *src, size_t n) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) dst[i] = src[i];
}

// The same for callers that own no pinned buffer: the bytes travel in the kernel's arguments (the runtime copies
// the argument block when the launch is enqueued, so the source is free at once).  3,840 bytes per launch.
constexpr uint32_t kArgPieceWords = kUploadArgBytes / 4;
struct ArgPiece {
    uint32_t w[kArgPieceWords];
};
__global__ __launch_bounds__(256) void upload_args_kernel(u32x4 *dst, ArgPiece piece, uint32_t n16) {
    const uint32_t i = threadIdx.x;
    if (i < n16) dst[i] = u32x4{piece.w[4 * i], piece.w[4 * i + 1], piece.w[4 * i + 2], piece.w[4 * i + 3]};
}

__global__ void zero_words_kernel(uint32_t *p, size_t n) {
    const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) p[i] = 0;
}

// ---------------------------------------------------------------------------------------
// Split-KV merge: out = sum_i w_i O_i / sum_i w_i l_i with w_i = 2^(m_i - max_i m_i), pieces
// taken in index order.  A block merges 8 columns of one split tile for one KV head: D/4
// threads per column, each owning four channels, so a piece's row is read as one coalesced
// run and the loop over pieces is unrolled to keep several loads in flight.
// ---------------------------------------------------------------------------------------
constexpr int kMergeCols = 8;  // columns per block of the merge kernel (must match the planner)

struct ReduceParams {
    const TileDesc *tiles;
    const uint32_t *reduce_units;  // (8-column group << kUnitTileBits) | tile index
    const float *part_ml;
    const float *part_o;
    uint16_t *out;
    int32_t num_q_heads;
    int32_t num_kv_heads;
    int32_t group;
};

// BATCH: pieces fetched at once.  Chunk tiles are cut into a few pieces of many rows and bound by their bytes: four (with
// eight, a batch of 56 tiles in two pieces took 25 us instead of 20).  Decodes that are cut to fill the chip have up to 32
// pieces of a few rows and are bound by latency: eight (32 pieces: 11.2 -> 6.8 us, 16 pieces 8.0 -> 6.5).  A launch has one
// size, by its finest cut: where both kinds are merged together eights and fours take the same time (14.2 and 14.5 us, 9.2
// and 8.1, 11.1 and 11.4, 8.3 and 8.5), and a launch per kind 2.5 to 3 us more.
template <int D, int BATCH>
__global__ __launch_bounds__(kMergeCols * D / 4) void splitkv_reduce_kernel(ReduceParams p) {
    constexpr int TPC = D / 4;  // threads per column
    const int kvh = blockIdx.x % p.num_kv_heads;
    const uint32_t u = p.reduce_units[blockIdx.x / p.num_kv_heads];
    const TileDesc it = p.tiles[u & ((1u << kUnitTileBits) - 1)];
    const int c = (int)(u >> kUnitTileBits) * kMergeCols + threadIdx.x / TPC;  // column inside the tile
    const int d4 = (threadIdx.x % TPC) * 4;
    if (c >= it.n_cols) return;
    const int col = it.col_begin + c;
    const int row = col / p.group;
    const int head = kvh * p.group + (col - row * p.group);
    const int64_t prow0 = ((int64_t)(it.part_row0 + c) * p.num_kv_heads + kvh);
    const int64_t split_stride = (int64_t)it.n_cols * p.num_kv_heads;
    const float *__restrict__ ml = p.part_ml;
    const float *__restrict__ po = p.part_o;
    // Loads first, arithmetic after: the pieces' rows were written by the attention launch and come from memory,
    // so a loop that loads, waits and accumulates piece by piece costs one memory latency per piece (and one more
    // per piece for the maxima).  BATCH pieces are fetched at once (indices beyond the last piece are clamped
    // to it: a valid, unused read), and the maxima of the later pieces as well; the sums still run in index order.
    const int n = it.n_splits;
    float m[BATCH], l[BATCH];
    f32x4 o[BATCH];
    auto fetch = [&](int base) {
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            const int64_t prow = prow0 + (int64_t)min(base + j, n - 1) * split_stride;
            const f32x2 v = *reinterpret_cast<const f32x2 *>(ml + prow * 2);
            m[j] = v[0];
            l[j] = v[1];
            o[j] = *reinterpret_cast<const f32x4 *>(po + prow * D + d4);
        }
    };
    fetch(0);
    float m_max = kNegSentinel;
#pragma unroll
    for (int j = 0; j < BATCH; ++j) m_max = fmaxf(m_max, m[j]);  // clamped entries repeat a valid piece
    for (int i = BATCH; i < n; i += BATCH) {
        float later[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) later[j] = ml[(prow0 + min(i + j, n - 1) * split_stride) * 2];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) m_max = fmaxf(m_max, later[j]);
    }
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float lsum = 0.f;
    for (int base = 0;;) {
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            if (base + j < n) {
                const float w = __builtin_amdgcn_exp2f(m[j] - m_max);
                lsum += w * l[j];
                acc += o[j] * w;
            }
        }
        base += BATCH;
        if (base >= n) break;
        fetch(base);
    }
    const bf16x4 o4 = __builtin_convertvector(acc * (1.0f / lsum), bf16x4);
    uint16_t *op = p.out + ((int64_t)(it.q_start + row) * p.num_q_heads + head) * D + d4;
    *reinterpret_cast<u32x2 *>(op) = __builtin_bit_cast(u32x2, o4);
}

// ---------------------------------------------------------------------------------------
// KV append: byte copies into the paged pools.  A block fills the slots [lo, hi) of one cache
// page for one KV head (a page unit, built by the host: a decode has one, a chunk one per page
// it touches), one thread per channel.  K rows go over as 16-byte pieces (a page holds them
// slot-major, so the hi - lo rows are one contiguous run).  V pages are channel-major: thread c
// owns the 32-byte row of channel c, gathers the tokens' values of that channel (a wavefront
// reads 128 contiguous bytes per token) and, when the whole page is new, writes the row with
// two 16-byte stores (the block writes the 4 KiB page front to back); a partly filled page
// gets 2-byte stores into its new slots only, the others keep their bytes.
// ---------------------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void kv_append_block(const AppendParams &p, const AppendUnit *units) {
    constexpr int kPieces = D / 8;  // 16-byte pieces of one K row
    if (blockIdx.x < p.copy_blocks) {
        const uint32_t i = blockIdx.x * D + threadIdx.x;
        if (i < p.copy_n16) p.copy_dst[i] = p.copy_src[i];
        return;
    }
    if (blockIdx.x < p.copy_blocks + p.zero_blocks) {
        const uint32_t i = (blockIdx.x - p.copy_blocks) * D + threadIdx.x;
        if (i < p.zero_n16) p.zero_dst[i] = u32x4{0, 0, 0, 0};
        return;
    }
    const unsigned blk = blockIdx.x - p.copy_blocks - p.zero_blocks;
    const int unit = (int)(blk / (unsigned)p.num_kv_heads);
    const int h = (int)(blk % (unsigned)p.num_kv_heads);
    const u32x4 rec = *reinterpret_cast<const u32x4 *>(units + unit);
    const int lo = (int)(rec[3] & 0xFFu), hi = (int)(rec[3] >> 8);
    const int n = hi - lo;
    const int64_t row_stride = (int64_t)p.num_kv_heads * D;
    const int64_t src = ((int64_t)(int)rec[2] * p.num_kv_heads + h) * D;
    const int tid = (int)threadIdx.x;
    // The block-table entry and the rows to move depend on the record only: all of these loads are issued
    // before the first is waited for (the table entry decides where the rows go, and whether they go at all).
    const int32_t *entry = p.block_table + (int64_t)(int)rec[0] * p.max_blocks + (int)rec[1];
    const int64_t page = *entry;

    // V: gather first (all loads in flight before any store)
    const uint16_t *vsrc = p.v_new + src + tid;
    uint16_t x[kPageSize];
#pragma unroll
    for (int i = 0; i < kPageSize; ++i) x[i] = (i < n) ? vsrc[i * row_stride] : (uint16_t)0;

    // K: n rows of D channels, destination contiguous
    constexpr int kRounds = (kPageSize * kPieces) / D;
    const uint16_t *ksrc = p.k_new + src;
    u32x4 krow[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int j = tid + r * D;
        const int i = j / kPieces, piece = j % kPieces;
        krow[r] = (i < n) ? *reinterpret_cast<const u32x4 *>(ksrc + i * row_stride + piece * 8) : u32x4{0, 0, 0, 0};
    }

    if (page < 0 || page >= p.num_pages) return;  // a corrupt table entry must not become a wild store
    const int64_t head_base = (page * p.num_kv_heads + h) * (int64_t)(kPageSize * D);
    uint16_t *kdst = p.k_cache + head_base + (int64_t)lo * D;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int j = tid + r * D;
        const int i = j / kPieces, piece = j % kPieces;
        if (i < n) *reinterpret_cast<u32x4 *>(kdst + i * D + piece * 8) = krow[r];
    }

    uint16_t *vdst = p.v_cache + head_base + (int64_t)tid * kPageSize;
    if (n == kPageSize) {
        u32x4 w0, w1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w0[e] = (uint32_t)x[2 * e] | ((uint32_t)x[2 * e + 1] << 16);
            w1[e] = (uint32_t)x[8 + 2 * e] | ((uint32_t)x[9 + 2 * e] << 16);
        }
        *reinterpret_cast<u32x4 *>(vdst) = w0;
        *reinterpret_cast<u32x4 *>(vdst + 8) = w1;
    } else {
#pragma unroll
        for (int i = 0; i < kPageSize; ++i)
            if (i < n) vdst[lo + i] = x[i];
    }
}

template <int D>
__global__ __launch_bounds__(D) void kv_append_kernel(AppendParams p) {
    kv_append_block<D>(p, p.units);
}
template <int D, int UNITS>
__global__ __launch_bounds__(D) void kv_append_inline_kernel(AppendParamsInline<UNITS> p) {
    kv_append_block<D>(p.base, p.units);
}

// ---------------------------------------------------------------------------------------
// Launchers
// ---------------------------------------------------------------------------------------
int launch_kv_append(const sarathi_config &cfg, const AppendMeta &m, const void *k_new, const void *v_new,
                     void *k_cache, void *v_cache, int64_t num_pages, void *stream) {
    if (m.num_units == 0) return (int)hipSuccess;
    AppendParams p;
    p.k_new = static_cast<const uint16_t *>(k_new);
    p.v_new = static_cast<const uint16_t *>(v_new);
    p.k_cache = static_cast<uint16_t *>(k_cache);
    p.v_cache = static_cast<uint16_t *>(v_cache);
    p.block_table = m.block_table;
    p.units = m.units;
    p.num_pages = num_pages;
    p.max_blocks = m.max_blocks;
    p.num_kv_heads = cfg.num_kv_heads;
    p.copy_dst = static_cast<u32x4 *>(m.copy_dst);
    p.copy_src = static_cast<const u32x4 *>(m.copy_src);
    p.copy_n16 = (uint32_t)((m.copy_bytes + 15) / 16);
    p.copy_blocks = (p.copy_n16 + (uint32_t)cfg.head_dim - 1) / (uint32_t)cfg.head_dim;
    p.zero_dst = static_cast<u32x4 *>(m.zero_dst);
    p.zero_n16 = (uint32_t)((m.zero_bytes + 15) / 16);
    p.zero_blocks = (p.zero_n16 + (uint32_t)cfg.head_dim - 1) / (uint32_t)cfg.head_dim;
    const unsigned blocks = p.copy_blocks + p.zero_blocks + (unsigned)m.num_units * (unsigned)cfg.num_kv_heads;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (m.units_host && m.num_units <= kInlineAppendUnits) {
        auto launch = [&](auto units) {
            constexpr int U = decltype(units)::value;
            AppendParamsInline<U> pi;
            pi.base = p;
            std::memcpy(pi.units, m.units_host, sizeof(AppendUnit) * (size_t)m.num_units);
            if (cfg.head_dim == 128)
                hipLaunchKernelGGL((kv_append_inline_kernel<128, U>), dim3(blocks), dim3(128), 0, st, pi);
            else
                hipLaunchKernelGGL((kv_append_inline_kernel<64, U>), dim3(blocks), dim3(64), 0, st, pi);
        };
        if (m.num_units <= kFewAppendUnits) launch(std::integral_constant<int, kFewAppendUnits>{});
        else launch(std::integral_constant<int, kInlineAppendUnits>{});
        return (int)hipGetLastError();
    }
    if (cfg.head_dim == 128)
        hipLaunchKernelGGL(kv_append_kernel<128>, dim3(blocks), dim3(128), 0, st, p);
    else
        hipLaunchKernelGGL(kv_append_kernel<64>, dim3(blocks), dim3(64), 0, st, p);
    return (int)hipGetLastError();
}

int launch_upload(void *dst, const void *pinned_src, size_t bytes, void *stream) {
    const size_t n = (bytes + 15) / 16;
    if (n == 0) return (int)hipSuccess;
    hipLaunchKernelGGL(upload_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream),
                       static_cast<u32x4 *>(dst), static_cast<const u32x4 *>(pinned_src), n);
    return (int)hipGetLastError();
}

int launch_upload_args(void *dst, const void *host_src, size_t bytes, void *stream) {
    static_assert(sizeof(ArgPiece) + 16 <= 4096, "kernel arguments are limited to 4 KiB");
    const char *src = static_cast<const char *>(host_src);
    char *d = static_cast<char *>(dst);
    for (size_t off = 0; off < bytes; off += sizeof(ArgPiece)) {
        const size_t n = bytes - off < sizeof(ArgPiece) ? bytes - off : sizeof(ArgPiece);
        ArgPiece piece;
        std::memcpy(piece.w, src + off, n);
        hipLaunchKernelGGL(upload_args_kernel, dim3(1), dim3(256), 0, static_cast<hipStream_t>(stream),
                           reinterpret_cast<u32x4 *>(d + off), piece, (uint32_t)((n + 15) / 16));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    return (int)hipSuccess;
}

// ---------------------------------------------------------------------------------------
// Scratch of the allocation-free entry point: one array in the device image of this library, so every GPU the
// library runs on holds its own copy until the process ends.  Host code never uses the array's name as an
// address: the device address is looked up once per device and used from then on.
// ---------------------------------------------------------------------------------------
constexpr size_t kStaticSchedBytes = (kSchedBytes + 255) / 256 * 256;
constexpr size_t kStaticScratchBytes = kStaticMetaBytes + kStaticSchedBytes + kStaticPartMlBytes + kStaticPartOBytes;
static __device__ __align__(256) unsigned char scratch[kStaticScratchBytes];

int static_scratch(StaticScratch *out) {
    constexpr int kMaxDevices = 64;
    static std::mutex lock;
    static char *base_of_device[kMaxDevices] = {};
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return (int)e;
    if (dev < 0 || dev >= kMaxDevices) return (int)hipErrorInvalidDevice;
    char *base;
    {
        std::lock_guard<std::mutex> guard(lock);
        if (!base_of_device[dev]) {
            void *ptr = nullptr;
            e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
            if (e != hipSuccess) return (int)e;
            if (!ptr) return (int)hipErrorInvalidSymbol;
            base_of_device[dev] = static_cast<char *>(ptr);
        }
        base = base_of_device[dev];
    }
    out->meta = base;
    out->sched = reinterpret_cast<int32_t *>(base + kStaticMetaBytes);
    out->part_ml = reinterpret_cast<float *>(base + kStaticMetaBytes + kStaticSchedBytes);
    out->part_o = reinterpret_cast<float *>(base + kStaticMetaBytes + kStaticSchedBytes + kStaticPartMlBytes);
    return (int)hipSuccess;
}

int launch_zero(void *ptr, size_t bytes, void *stream) {
    const size_t n = bytes / 4;
    if (n == 0) return (int)hipSuccess;
    hipLaunchKernelGGL(zero_words_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream),
                       static_cast<uint32_t *>(ptr), n);
    return (int)hipGetLastError();
}

int launch_reduce(const sarathi_config &cfg, const AttnMeta &m, void *out, int32_t first, int32_t count, void *stream) {
    if (count <= 0) return (int)hipSuccess;
    static_assert(kMergeCols == kReduceCols, "planner and merge kernel must agree on columns per block");
    ReduceParams p;
    p.tiles = m.tiles;
    p.reduce_units = m.reduce_units + first;
    p.part_ml = m.part_ml;
    p.part_o = m.part_o;
    p.out = static_cast<uint16_t *>(out);
    p.num_q_heads = cfg.num_q_heads;
    p.num_kv_heads = cfg.num_kv_heads;
    p.group = cfg.num_q_heads / cfg.num_kv_heads;
    const unsigned blocks = (unsigned)count * (unsigned)cfg.num_kv_heads;
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto launch = [&](auto d, auto batch) {
        constexpr int D = decltype(d)::value;
        hipLaunchKernelGGL((splitkv_reduce_kernel<D, decltype(batch)::value>), dim3(blocks), dim3(kMergeCols * D / 4), 0, st, p);
    };
    auto pick_batch = [&](auto d) {
        if (m.most_pieces <= 4) launch(d, std::integral_constant<int, 4>{});
        else launch(d, std::integral_constant<int, 8>{});
    };
    if (cfg.head_dim == 128) pick_batch(std::integral_constant<int, 128>{});
    else pick_batch(std::integral_constant<int, 64>{});
    return (int)hipGetLastError();
}

template <int D>
struct Bf16Paths {
    static constexpr int kWaveElems = WaveSmem<D>::kTotalElems, kChunkElems = ChunkSmem<D>::kTotalElems;
    static constexpr int kWaveBlocksPerUnit = 2;
    template <bool STREAM, typename Claim>
    static __device__ __forceinline__ int wave(const AttnParams &p, const TileDesc &it, int split, int kvh, uint16_t *smem, Claim claim) {
        return wave16_path<D, STREAM>(p, it, split, kvh, smem, claim);
    }
    static __device__ __forceinline__ void chunk(const AttnParams &p, const TileDesc &it, int split, int kvh, uint16_t *smem) {
        chunk_tile_path<D>(p, it, split, kvh, smem);
    }
};

int launch_attention(const sarathi_config &cfg, const AttnMeta &m, const void *q, const void *k_cache,
                     const void *v_cache, int64_t num_pages, float sm_scale, void *out, int which, void *stream) {
    return launch_attention_paths<Bf16Paths>(cfg, m, q, k_cache, v_cache, num_pages, sm_scale, out, which, stream);
}

}  // namespace sarathi
