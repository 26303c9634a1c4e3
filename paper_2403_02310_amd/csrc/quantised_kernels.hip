// gfx950 kernels of the 4-bit key/value cache: rows quantised into it, rows read back, and hybrid-batch attention over it.
//
// What it holds.  Magnitudes 0, 0.5, 1, 1.5, 2, 3, 4 and 6 with a sign in 4 bits, which this part converts two at a time to bf16 with a
// power of two multiplied in (v_cvt_scalef32_pk_bf16_fp4: the exponent of a float, 255 makes NaN), and back, rounding to the nearest and
// ties to the even code.  Each scale lies along the contraction that its numbers meet:
//   keys    32 neighbouring channels share 2^e, one byte: the score contracts over channels, and the conversion multiplies it in for nothing
//   values  the channels of a (position, head) share a float of four significant bits: the output contracts over positions, so it is
//           one factor of the position's softmax weight, in 32 bits, and the values enter the matrix instruction as they are held
// Code times scale has six significant bits at most: all of it is exact in bf16, in the operands and when read back.  A key's
// scale follows from its largest magnitude by integer arithmetic, a value's from one division whose rounding cannot matter (a quotient
// that needs more than four bits is further than a rounding from one that does not), and the quotient of a value and
// its scale meets a border between two codes exactly or misses it by far more than a rounding.
//
// Layout: lanes read what their operands need, front to back.  The record of a page and KV head (16 slots, D channels):
//   keys    [D/32 blocks][16 slots][16 bytes]                 channels in order, the lower in the low half of a byte
//   values  [4 quads][16][D/16][2 bytes]                      channel 16 c + n of slots 4 quad .. + 3 at [quad][n][c], the lower slot in the low half
//   scales  of the keys [D/32][16 slots] bytes, of the values [16 slots] floats
// With D = 128 a record is 2176 bytes, 17 lines of 128.
#include "attn_device.h"

namespace sarathi {

template <int D>
struct Record {
    static constexpr int kValues = 8 * D, kKeyScales = 16 * D, kValueScales = 16 * D + D / 2, kBytes = 16 * D + D / 2 + 64;
    static_assert(kBytes == (int)quantised_record_bytes(D), "the host allocates and checks with the same size");
};

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// Values 2 PAIR and 2 PAIR + 1 of the eight in a word, times the power of two in `scale`.
template <int PAIR>
__device__ __forceinline__ uint32_t unpack_pair(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, PAIR));
}
__device__ __forceinline__ u32x4 unpack_word(uint32_t codes, float scale) {
    return u32x4{unpack_pair<0>(codes, scale), unpack_pair<1>(codes, scale), unpack_pair<2>(codes, scale), unpack_pair<3>(codes, scale)};
}
// `codes` with two bf16 numbers, in units of the power of two `scale`, as values 2 PAIR and 2 PAIR + 1.
template <int PAIR>
__device__ __forceinline__ uint32_t pack_pair(uint32_t codes, uint32_t pair, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, pair), scale, PAIR);
}
__device__ __forceinline__ float key_scale(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// ---------------------------------------------------------------------------------------
// Wave tiles (decodes, tiny chunks): 16 query columns against a key range, a quarter of it to each wavefront, as in the bf16 cache's
// path.  With the layout above a lane's share of an operand is one load of 16 bytes (8 with 64 channels), 1 KiB front to
// back over the wavefront, straight into registers:
//   S^T[key, col]: A-row n of matrix instruction b is slot n of page b of the tile; contraction step s of lane group g is channels
//                  (D/4) g + 8 s .. + 7, in the queries alike, so a lane's channels lie in one block and have one scale
//   O^T[ch, col]:  accumulator lane (g, n) has the scores of slots 4 g .. + 3 of both pages, and the values of those eight are
//                  the contraction indices of its lane group
// ---------------------------------------------------------------------------------------
template <int D>
struct QuantisedWaveSmem {
    static constexpr int kColStride = D + 4;
    static constexpr int kOutFloats = kWaveCols * kColStride;
    static constexpr int kWaveElems = (kOutFloats + 2 * kWaveCols) * 2;
    static constexpr int kTotalElems = 4 * kWaveElems;
};

// A lane's share of a tile of 32 keys: codes, the bytes of its keys' scales, the scales of its values.
template <int D>
struct QuantisedTile {
    typedef __attribute__((ext_vector_type(D / 32))) uint32_t codes;
    codes k[2], v[2];
    uint32_t k_scale[2];
    f32x4 v_scale[2];
};

template <int D>
struct QuantisedLoads {
    const uint8_t *head;   // page 0 of this KV head
    const_i32_ptr bt;      // this sequence's block-table row
    int64_t page_stride;   // bytes per page (all KV heads)
    int64_t last_page_id;  // page ids are clamped: a corrupt table cannot fault
    int32_t n_pages_seq;   // pages that hold positions < ctx_len; those behind are never dereferenced
    uint32_t k_off, v_off, k_scale_off, v_scale_off;
};

template <typename T, bool STREAM>
__device__ __forceinline__ T load_as(const uint8_t *base, uint32_t off) {
    const T *at = reinterpret_cast<const T *>(base + off);
    if constexpr (STREAM) return __builtin_nontemporal_load(at);
    else return *at;
}

template <int D, bool STREAM>
__device__ __forceinline__ void load_tile(const QuantisedLoads<D> &ge, int tile, QuantisedTile<D> &t) {
    using codes = typename QuantisedTile<D>::codes;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int64_t entry = ge.bt[min(tile * 2 + b, ge.n_pages_seq - 1)];
        const uint8_t *rec = ge.head + (entry < 0 ? 0 : (entry > ge.last_page_id ? ge.last_page_id : entry)) * ge.page_stride;
        t.k[b] = load_as<codes, STREAM>(rec, ge.k_off);
        t.v[b] = load_as<codes, STREAM>(rec, ge.v_off);
        t.k_scale[b] = load_as<uint8_t, STREAM>(rec, ge.k_scale_off);
        t.v_scale[b] = load_as<f32x4, STREAM>(rec, ge.v_scale_off);
    }
}

template <int D, bool STREAM, typename Claim>
__device__ __forceinline__ int quantised_wave_path(const AttnParams &p, const TileDesc &it, int split, int kvh, uint16_t *smem, Claim claim) {
    const int tid = thread_of_item();
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15;
    const int g = lane >> 4;
    const int ctx = it.ctx_len;
    const int prefix = ctx - it.q_len;
    const int G = p.group;
    UnitRange ur = unit_range(it, split);
    {   // this wavefront's quarter of the unit (possibly empty: then it contributes weight zero)
        const int quarter = ((ur.key_end - ur.key_begin + 3) / 4 + kTileKeys - 1) / kTileKeys * kTileKeys;
        const int b = ur.key_begin + wave * quarter;   // a multiple of 32, as every piece start
        ur.key_end = min(ur.key_end, b + quarter);
        ur.key_begin = min(b, ur.key_end);
    }
    // Lanes beyond the tile's valid columns shadow column 0 of the tile and store nothing.
    const int col = it.col_begin + (n < it.n_cols ? n : 0);
    const int row = col / G;
    const int head = kvh * G + (col - row * G);
    const int pos_eff = min(prefix + row, ur.key_end - 1);                   // last key this column may see here
    const int min_pos_eff = min(prefix + it.col_begin / G, ur.key_end - 1);  // the same for the tile's first column
    // first key inside this column's sliding window, and the largest such key over the tile's columns
    const int lo = p.window > 0 ? max(0, prefix + row - p.window + 1) : 0;
    const int max_lo = p.window > 0 ? max(0, prefix + (it.col_begin + it.n_cols - 1) / G - p.window + 1) : 0;

    bf16x8 qreg[D / 32];
    {
        const uint16_t *qp = p.q + ((int64_t)(it.q_start + row) * p.num_q_heads + head) * D + g * (D / 4);
#pragma unroll
        for (int s = 0; s < D / 32; ++s) qreg[s] = load_bf16x8(qp + s * 8);
    }
    using R = Record<D>;
    QuantisedLoads<D> ge;
    ge.head = reinterpret_cast<const uint8_t *>(p.k_cache) + (int64_t)kvh * R::kBytes;
    ge.bt = (const_i32_ptr)(p.block_table + (int64_t)it.seq * p.max_blocks);
    ge.page_stride = (int64_t)p.num_kv_heads * R::kBytes;
    ge.last_page_id = p.num_pages - 1;
    ge.n_pages_seq = (ctx + kPageSize - 1) / kPageSize;
    const int block = g * D / 128;  // of 32 channels: lane groups share one with 64
    ge.k_off = (uint32_t)(block * 256 + n * 16 + (D == 64 ? (g & 1) * 8 : 0));
    ge.v_off = (uint32_t)(R::kValues + lane * (D / 8));
    ge.k_scale_off = (uint32_t)(R::kKeyScales + block * 16 + n);
    ge.v_scale_off = (uint32_t)(R::kValueScales + g * 16);

    SoftmaxState<D> st;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) st.o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    st.m = kNegSentinel;
    st.l = 0.f;
    const float scale = p.scale_log2;

    auto process = [&](const QuantisedTile<D> &t, int tile) {
        f32x4 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            s[b] = f32x4{0.f, 0.f, 0.f, 0.f};
            const float ks = key_scale(t.k_scale[b]);
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, unpack_word(t.k[b][i], ks)), qreg[i], s[b], 0, 0, 0);
        }
        f32x4 vs[2] = {t.v_scale[0], t.v_scale[1]};
        // Hidden keys: score -inf, and value scale 0, so that what a hidden slot holds (NaN among it) multiplies nothing.
        if (tile * kTileKeys + (kTileKeys - 1) > min_pos_eff || tile * kTileKeys < max_lo) {  // wave-uniform: some lane must mask
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = tile * kTileKeys + b * kPageSize + g * 4 + i;
                    const bool seen = key <= pos_eff && key >= lo;
                    s[b][i] = seen ? s[b][i] : -INFINITY;
                    vs[b][i] = seen ? vs[b][i] : 0.f;
                }
        }
        // The reference maximum is raised when a score exceeds it by more than the slack; only then is the column's maximum
        // looked for across its four lanes.
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) * scale;
        if (__any(top > st.m + kRescaleSlack)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(st.m, top);
            const float alpha = __builtin_amdgcn_exp2f(st.m - m_new);
            st.l *= alpha;
            st.m = m_new;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) st.o[c] *= alpha;
        }
        f32x8 w;
        float psum = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], scale, -st.m));
                psum += e;
                w[4 * b + i] = e * vs[b][i];
            }
        st.l += psum;
        // rounded to bf16 for the matrix instruction: each weight is off by at most 2^-8 of itself, averaged down over the keys
        const bf16x8 pT = __builtin_convertvector(w, bf16x8);
#pragma unroll
        for (int c = 0; c < D / 16; c += 2) {
            const uint32_t a = t.v[0][c / 2], b = t.v[1][c / 2];
            const u32x4 even = {unpack_pair<0>(a, 1.f), unpack_pair<1>(a, 1.f), unpack_pair<0>(b, 1.f), unpack_pair<1>(b, 1.f)};
            const u32x4 odd = {unpack_pair<2>(a, 1.f), unpack_pair<3>(a, 1.f), unpack_pair<2>(b, 1.f), unpack_pair<3>(b, 1.f)};
            st.o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), pT, st.o[c], 0, 0, 0);
            st.o[c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), pT, st.o[c + 1], 0, 0, 0);
        }
    };

    const int tile_begin = ur.key_begin / kTileKeys;
    const int tile_end = ur.key_begin >= ur.key_end ? tile_begin : (ur.key_end + kTileKeys - 1) / kTileKeys;
    int claimed = 0;
    if (tid == 0) claimed = claim();
    for (int tile = tile_begin; tile < tile_end; ++tile) {
        QuantisedTile<D> t;
        load_tile<D, STREAM>(ge, tile, t);
        process(t, tile);
    }
    wave_finish<D, QuantisedWaveSmem<D>>(p, it, split, kvh, tid, smem, st);
    return claimed;
}

template <int D>
struct QuantisedPaths {
    static constexpr int kWaveElems = QuantisedWaveSmem<D>::kTotalElems, kChunkElems = 8;
    static constexpr int kWaveBlocksPerUnit = 2;
    template <bool STREAM, typename Claim>
    static __device__ __forceinline__ int wave(const AttnParams &p, const TileDesc &it, int split, int kvh, uint16_t *smem, Claim claim) {
        return quantised_wave_path<D, STREAM>(p, it, split, kvh, smem, claim);
    }
    static __device__ __forceinline__ void chunk(const AttnParams &, const TileDesc &, int, int, uint16_t *) {}
};

// ---------------------------------------------------------------------------------------
// Rows into the cache.  A block fills the slots [lo, hi) of one page record: thread (slot, eight channels) quantises its keys and
// values, the largest magnitudes of a block of 32 channels and of a position are found across the lanes that hold
// them, and the values' codes, of which two slots share a byte, are turned in LDS and merged into what the page holds of its
// other slots.
// ---------------------------------------------------------------------------------------
template <int D>
struct RowsThread {
    static constexpr int kThreads = 2 * D, kPieces = D / 8;  // eight channels of a row each
    int slot, piece;
    __device__ __forceinline__ RowsThread() : slot((int)threadIdx.x / kPieces), piece((int)threadIdx.x % kPieces) {}
    // of the eight channels' codes in a record's keys, and of the byte of their scale
    __device__ __forceinline__ int key_word() const { return (piece >> 2) * 256 + slot * 16 + (piece & 3) * 4; }
    __device__ __forceinline__ int key_scale() const { return Record<D>::kKeyScales + (piece >> 2) * 16 + slot; }
};

// The largest of the magnitudes of eight bf16 numbers, as the bits of a bf16 (infinity and NaN are the largest).
__device__ __forceinline__ uint32_t largest_bits(const u32x4 &x) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7FFFu, (x[i] >> 16) & 0x7FFFu));
    return top;
}
constexpr uint32_t kInfBits = 0x7F80u;

template <int D>
__device__ __forceinline__ void kv_append_quantised_block(const AppendParams &p, const AppendUnit *units) {
    using R = Record<D>;
    constexpr int kThreads = RowsThread<D>::kThreads, kPieces = RowsThread<D>::kPieces;
    if (blockIdx.x < p.copy_blocks) {
        const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
        if (i < p.copy_n16) p.copy_dst[i] = p.copy_src[i];
        return;
    }
    if (blockIdx.x < p.copy_blocks + p.zero_blocks) {
        const uint32_t i = (blockIdx.x - p.copy_blocks) * kThreads + threadIdx.x;
        if (i < p.zero_n16) p.zero_dst[i] = u32x4{0, 0, 0, 0};
        return;
    }
    __shared__ uint32_t turned[kPageSize * kPieces];  // the values' codes by slot
    const unsigned blk = blockIdx.x - p.copy_blocks - p.zero_blocks;
    const int unit = (int)(blk / (unsigned)p.num_kv_heads);
    const int h = (int)(blk % (unsigned)p.num_kv_heads);
    const u32x4 about = *reinterpret_cast<const u32x4 *>(units + unit);
    const int lo = (int)(about[3] & 0xFFu), hi = (int)(about[3] >> 8);
    const RowsThread<D> t;
    const bool mine = t.slot >= lo && t.slot < hi;
    const int64_t page = p.block_table[(int64_t)(int)about[0] * p.max_blocks + (int)about[1]];
    const int64_t src = ((int64_t)((int)about[2] + t.slot - lo) * p.num_kv_heads + h) * D + t.piece * 8;
    u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    if (mine) {
        k = *reinterpret_cast<const u32x4 *>(p.k_new + src);
        v = *reinterpret_cast<const u32x4 *>(p.v_new + src);
    }
    if (page < 0 || page >= p.num_pages) return;  // a corrupt table entry must not become a wild store
    uint8_t *rec = reinterpret_cast<uint8_t *>(p.k_cache) + (page * p.num_kv_heads + h) * (int64_t)R::kBytes;

    // This thread's word of the values' codes: channels 16 c + n and 16 (c + 1) + n of a quad's slots.
    const int word = (int)threadIdx.x, n = word / (D / 32) % 16, c = word % (D / 32) * 2, slot0 = word / (D / 2) * 4;
    uint32_t filled = 0;  // the bits of slots that this call writes
#pragma unroll
    for (int i = 0; i < 4; ++i) filled |= (slot0 + i >= lo && slot0 + i < hi) ? 0x000F000Fu << (4 * i) : 0u;
    uint32_t *v_word = reinterpret_cast<uint32_t *>(rec + R::kValues) + word;
    const uint32_t held = (filled != 0 && filled != ~0u) ? *v_word : 0;

    // Keys: 2^e of 32 channels, which four lanes hold.  The largest is 1.f * 2^E; the smallest e with 1.f * 2^E <= 1.5 * 2^(e + 2).
    uint32_t top = largest_bits(k);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const int e = min(max((int)(top >> 7) - 129 + ((top & 127u) > 64u ? 1 : 0), -100), 124);
    const float k_unit = key_scale((uint32_t)(e + 127));
    uint32_t codes = pack_pair<0>(0, k[0], k_unit);
    codes = pack_pair<1>(codes, k[1], k_unit);
    codes = pack_pair<2>(codes, k[2], k_unit);
    codes = pack_pair<3>(codes, k[3], k_unit);
    if (mine) {
        const bool finite = top < kInfBits;
        *reinterpret_cast<uint32_t *>(rec + t.key_word()) = finite ? codes : 0u;
        if ((t.piece & 3) == 0) rec[t.key_scale()] = finite ? (uint8_t)(e + 127) : (uint8_t)255;
    }

    // Values: four bits of a sixth of the position's largest, rounded up.
    top = largest_bits(v);
#pragma unroll
    for (int step = 1; step < kPieces; step *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, step));
    const bool finite = top < kInfBits;
    const float sixth = fminf(fmaxf(__builtin_bit_cast(float, top << 16) / 6.0f, 0x1p-100f), 0x1p124f);
    const float unit_v = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, sixth) + 0xFFFFFu) & ~0xFFFFFu);
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[2 * i] = __builtin_bit_cast(float, v[i] << 16) / unit_v;
        y[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xFFFF0000u) / unit_v;
    }
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.0f, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[2], y[3], 1.0f, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[4], y[5], 1.0f, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[6], y[7], 1.0f, 3);
    turned[t.slot * kPieces + t.piece] = finite ? codes : 0u;
    if (mine && t.piece == 0) reinterpret_cast<float *>(rec + R::kValueScales)[t.slot] = finite ? unit_v : __builtin_nanf("");
    __syncthreads();
    if (filled == 0) return;
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int ch = (c + j) * 16 + n;
            out |= ((turned[(slot0 + i) * kPieces + ch / 8] >> (4 * (ch % 8))) & 15u) << (16 * j + 4 * i);
        }
    *v_word = (out & filled) | (held & ~filled);
}

template <int D>
__global__ __launch_bounds__(2 * D) void kv_append_quantised_kernel(AppendParams p) {
    kv_append_quantised_block<D>(p, p.units);
}
template <int D, int UNITS>
__global__ __launch_bounds__(2 * D) void kv_append_quantised_inline_kernel(AppendParamsInline<UNITS> p) {
    kv_append_quantised_block<D>(p.base, p.units);
}

// Rows out of the cache, the way back: k_new is the pool, k_cache and v_cache the rows.
template <int D>
__device__ __forceinline__ void kv_read_quantised_block(const AppendParams &p, const AppendUnit *units) {
    using R = Record<D>;
    __shared__ uint32_t words[2 * D];  // the values' codes as the page holds them
    const int unit = (int)(blockIdx.x / (unsigned)p.num_kv_heads);
    const int h = (int)(blockIdx.x % (unsigned)p.num_kv_heads);
    const u32x4 about = *reinterpret_cast<const u32x4 *>(units + unit);
    const int lo = (int)(about[3] & 0xFFu), hi = (int)(about[3] >> 8);
    const RowsThread<D> t;
    const int64_t page = p.block_table[(int64_t)(int)about[0] * p.max_blocks + (int)about[1]];
    if (page < 0 || page >= p.num_pages) return;  // the rows of a corrupt table entry stay as they are
    const uint8_t *rec = reinterpret_cast<const uint8_t *>(p.k_new) + (page * p.num_kv_heads + h) * (int64_t)R::kBytes;
    words[threadIdx.x] = reinterpret_cast<const uint32_t *>(rec + R::kValues)[threadIdx.x];
    const uint32_t k = *reinterpret_cast<const uint32_t *>(rec + t.key_word());
    const float k_unit = key_scale(rec[t.key_scale()]);
    const float v_unit = reinterpret_cast<const float *>(rec + R::kValueScales)[t.slot];
    __syncthreads();
    if (t.slot < lo || t.slot >= hi) return;
    uint32_t v = 0;
    const int c = t.piece >> 1;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t w = words[((t.slot >> 2) * 16 + (t.piece & 1) * 8 + j) * (D / 32) + c / 2];
        v |= ((w >> (16 * (c & 1) + 4 * (t.slot & 3))) & 15u) << (4 * j);
    }
    f32x8 y;
    const f32x2 y0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 0), y1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 1);
    const f32x2 y2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 2), y3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 3);
    y[0] = y0[0] * v_unit, y[1] = y0[1] * v_unit, y[2] = y1[0] * v_unit, y[3] = y1[1] * v_unit;
    y[4] = y2[0] * v_unit, y[5] = y2[1] * v_unit, y[6] = y3[0] * v_unit, y[7] = y3[1] * v_unit;
    const int64_t dst = ((int64_t)((int)about[2] + t.slot - lo) * p.num_kv_heads + h) * D + t.piece * 8;
    *reinterpret_cast<u32x4 *>(p.k_cache + dst) = unpack_word(k, k_unit);
    *reinterpret_cast<u32x4 *>(p.v_cache + dst) = __builtin_bit_cast(u32x4, __builtin_convertvector(y, bf16x8));
}

template <int D>
__global__ __launch_bounds__(2 * D) void kv_read_quantised_kernel(AppendParams p) {
    kv_read_quantised_block<D>(p, p.units);
}
template <int D, int UNITS>
__global__ __launch_bounds__(2 * D) void kv_read_quantised_inline_kernel(AppendParamsInline<UNITS> p) {
    kv_read_quantised_block<D>(p.base, p.units);
}

// ---------------------------------------------------------------------------------------
// Launchers
// ---------------------------------------------------------------------------------------
namespace {

AppendParams rows_params(const sarathi_config &cfg, const AppendMeta &m, int64_t num_pages) {
    AppendParams p{};
    p.block_table = m.block_table;
    p.units = m.units;
    p.num_pages = num_pages;
    p.max_blocks = m.max_blocks;
    p.num_kv_heads = cfg.num_kv_heads;
    return p;
}

// launch(head_dim, arguments): records in the arguments where few enough, as for the bf16 cache
template <typename Launch>
void with_records(const sarathi_config &cfg, const AppendMeta &m, const AppendParams &p, Launch launch) {
    auto pick = [&](const auto &args) {
        if (cfg.head_dim == 128) launch(std::integral_constant<int, 128>{}, args);
        else launch(std::integral_constant<int, 64>{}, args);
    };
    auto carry = [&](auto args) {
        args.base = p;
        std::memcpy(args.units, m.units_host, sizeof(AppendUnit) * (size_t)m.num_units);
        pick(args);
    };
    if (!m.units_host || m.num_units > kInlineAppendUnits) pick(p);
    else if (m.num_units <= kFewAppendUnits) carry(AppendParamsInline<kFewAppendUnits>{});
    else carry(AppendParamsInline<kInlineAppendUnits>{});
}
template <typename Args>
struct RecordsCarried : std::false_type {};
template <int UNITS>
struct RecordsCarried<AppendParamsInline<UNITS>> : std::true_type {
    static constexpr int kUnits = UNITS;
};

}  // namespace

int launch_kv_append_quantised(const sarathi_config &cfg, const AppendMeta &m, const void *k_new, const void *v_new, void *kv_cache, int64_t num_pages,
                               void *stream) {
    if (m.num_units == 0) return (int)hipSuccess;
    AppendParams p = rows_params(cfg, m, num_pages);
    p.k_new = static_cast<const uint16_t *>(k_new);
    p.v_new = static_cast<const uint16_t *>(v_new);
    p.k_cache = static_cast<uint16_t *>(kv_cache);
    const uint32_t threads = 2 * (uint32_t)cfg.head_dim;
    p.copy_dst = static_cast<u32x4 *>(m.copy_dst);
    p.copy_src = static_cast<const u32x4 *>(m.copy_src);
    p.copy_n16 = (uint32_t)((m.copy_bytes + 15) / 16);
    p.copy_blocks = (p.copy_n16 + threads - 1) / threads;
    p.zero_dst = static_cast<u32x4 *>(m.zero_dst);
    p.zero_n16 = (uint32_t)((m.zero_bytes + 15) / 16);
    p.zero_blocks = (p.zero_n16 + threads - 1) / threads;
    const dim3 grid(p.copy_blocks + p.zero_blocks + (unsigned)m.num_units * (unsigned)cfg.num_kv_heads);
    with_records(cfg, m, p, [&](auto d, const auto &args) {
        using Args = std::decay_t<decltype(args)>;
        constexpr int D = decltype(d)::value;
        hipStream_t st = static_cast<hipStream_t>(stream);
        if constexpr (RecordsCarried<Args>::value)
            hipLaunchKernelGGL((kv_append_quantised_inline_kernel<D, RecordsCarried<Args>::kUnits>), grid, dim3(2 * D), 0, st, args);
        else
            hipLaunchKernelGGL((kv_append_quantised_kernel<D>), grid, dim3(2 * D), 0, st, args);
    });
    return (int)hipGetLastError();
}

int launch_kv_read_quantised(const sarathi_config &cfg, const AppendMeta &m, const void *kv_cache, int64_t num_pages, void *k_rows, void *v_rows,
                             void *stream) {
    if (m.num_units == 0) return (int)hipSuccess;
    AppendParams p = rows_params(cfg, m, num_pages);
    p.k_new = static_cast<const uint16_t *>(kv_cache);
    p.k_cache = static_cast<uint16_t *>(k_rows);
    p.v_cache = static_cast<uint16_t *>(v_rows);
    const dim3 grid((unsigned)m.num_units * (unsigned)cfg.num_kv_heads);
    with_records(cfg, m, p, [&](auto d, const auto &args) {
        using Args = std::decay_t<decltype(args)>;
        constexpr int D = decltype(d)::value;
        hipStream_t st = static_cast<hipStream_t>(stream);
        if constexpr (RecordsCarried<Args>::value)
            hipLaunchKernelGGL((kv_read_quantised_inline_kernel<D, RecordsCarried<Args>::kUnits>), grid, dim3(2 * D), 0, st, args);
        else
            hipLaunchKernelGGL((kv_read_quantised_kernel<D>), grid, dim3(2 * D), 0, st, args);
    });
    return (int)hipGetLastError();
}

int launch_attention_quantised(const sarathi_config &cfg, const AttnMeta &m, const void *q, const void *kv_cache, int64_t num_pages, float sm_scale,
                               void *out, int which, void *stream) {
    return launch_attention_paths<QuantisedPaths>(cfg, m, q, kv_cache, nullptr, num_pages, sm_scale, out, which, stream);
}

}  // namespace sarathi
