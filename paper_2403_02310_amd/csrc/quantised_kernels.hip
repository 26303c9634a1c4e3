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

// The largest of the magnitudes of eight bf16 numbers, as the bits of a bf16 (infinity and NaN are the largest).
__device__ __forceinline__ uint32_t largest_bits(const u32x4 &x) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7FFFu, (x[i] >> 16) & 0x7FFFu));
    return top;
}
constexpr uint32_t kInfBits = 0x7F80u;

// ---------------------------------------------------------------------------------------
// Attention.  A wavefront holds 16 or 32 query columns and goes over its keys 32 at a time.  Wave tiles (decodes, tiny chunks): 32 columns
// against a key range, a quarter of it to each wavefront, as in the bf16 cache's path; a tile of up to 16 columns has code of
// its own.  Chunk tiles: 128 columns, 32 to each wavefront.  With the layout above a lane's share of an operand is one load
// of 16 bytes (of values with 64 channels 8), front to back over the wavefront, straight into registers:
//   S^T[key, col]: A-row n of matrix instruction b is slot n of page b of the tile, lane group g the channels of block g and its scale
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

// A lane's share of a tile of 32 keys: the codes of its keys and the bytes of their scales, the codes and the scales of its values.
template <int D>
struct QuantisedTile {
    typedef __attribute__((ext_vector_type(D / 32))) uint32_t words;
    u32x4 keys[2];
    uint32_t key_scales[2];
    words values[2];
    f32x4 value_scales[2];
};

// The two block-table entries of a tile, and the records they name: wave-uniform, by scalar loads and arithmetic.
struct QuantisedPages {
    int32_t entry[2];
};
typedef const __attribute__((address_space(1))) uint8_t *record_ptr;
struct QuantisedRecords {
    record_ptr of[2];
};

struct QuantisedLoads {
    record_ptr head;       // page 0 of this KV head
    const_i32_ptr bt;      // this sequence's block-table row
    uint32_t page_stride;  // bytes per page (all KV heads)
    int32_t last_page_id;  // page ids are clamped: a corrupt table cannot fault
    int32_t n_pages_seq;   // pages that hold positions < ctx_len; those behind are never dereferenced
    uint32_t k_off, v_off, k_scale_off, v_scale_off;  // this lane's, inside a record

    template <int D>
    __device__ __forceinline__ void init(const AttnParams &p, const TileDesc &it, int kvh) {
        head = (record_ptr)p.k_cache + (int64_t)kvh * Record<D>::kBytes;
        bt = (const_i32_ptr)(p.block_table + (int64_t)it.seq * p.max_blocks);
        page_stride = (uint32_t)p.num_kv_heads * Record<D>::kBytes;
        last_page_id = (int32_t)min(p.num_pages - 1, (int64_t)INT32_MAX);
        n_pages_seq = (it.ctx_len + kPageSize - 1) / kPageSize;
    }
    __device__ __forceinline__ QuantisedPages pages_of(int tile) const {
        return QuantisedPages{{bt[min(tile * 2, n_pages_seq - 1)], bt[min(tile * 2 + 1, n_pages_seq - 1)]}};
    }
    __device__ __forceinline__ QuantisedRecords records(const QuantisedPages &pages) const {
        QuantisedRecords r;
#pragma unroll
        for (int b = 0; b < 2; ++b) r.of[b] = head + (uint64_t)(uint32_t)min(max(pages.entry[b], 0), last_page_id) * page_stride;
        return r;
    }
    // Called once a tile: the lanes' offsets, seen as new, are added to the records by the loads themselves instead of being widened and
    // added to `head` ahead of the loop, which takes a 64-bit addition per lane and load.
    __device__ __forceinline__ void renew() { asm volatile("" : "+v"(k_off), "+v"(v_off), "+v"(k_scale_off), "+v"(v_scale_off)); }
    template <typename T, bool STREAM>
    static __device__ __forceinline__ T load_as(record_ptr base, uint32_t off) {
        const auto *at = reinterpret_cast<const __attribute__((address_space(1))) T *>(base + off);
        if constexpr (STREAM) return __builtin_nontemporal_load(at);
        else return *at;
    }
    // Loads of one tile stay together: results come back in order, and are waited for so.
    template <bool STREAM, int D>
    __device__ __forceinline__ void load(const QuantisedPages &pages, QuantisedTile<D> &t) {
        const QuantisedRecords r = records(pages);
        renew();
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            t.key_scales[b] = load_as<uint8_t, STREAM>(r.of[b], k_scale_off);
            t.keys[b] = load_as<u32x4, STREAM>(r.of[b], k_off);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            t.value_scales[b] = load_as<f32x4, STREAM>(r.of[b], v_scale_off);
            t.values[b] = load_as<typename QuantisedTile<D>::words, STREAM>(r.of[b], v_off);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
};

// Queries of 16 columns as the second operand of the score instructions, v_mfma_scale_f32_16x16x128_f8f6f4: the first takes 4-bit keys with their
// scales as they are held, nothing to unpack (against keys unpacked to bf16, four instructions and 32 conversions for two: 512 tokens
// next to 64 decodes of 32 and 8 heads 56.6 us and 52.9, 200 decodes of 58 and 2 heads of 64 channels 44.4 and 41.2).  The second takes 8-bit numbers of four
// significant bits, so a query is two of them, q = 2^e (h + l / 32) with 2^e 128 at most the column's largest: h is q rounded, l the rest.  That is q
// itself where it is more than 2^-15 of the column's largest, and off by at most 2^-23 of that elsewhere, as a sum in 32 bits that holds the
// largest is.  Lane group g holds channels 16 g .. + 15 (and 64 + 16 g ..), where the instruction has contraction indices 16 g .. and 64 + 16 g ..;
// with 64 channels the second half of the contraction takes the same keys again, and l.
template <int D>
struct PackedQueries {
    typedef __attribute__((ext_vector_type(8))) int words;
    static constexpr int kTerms = D / 64;  // instructions a page
    words w[kTerms];
    int scale[kTerms];

    __device__ __forceinline__ void load(const uint16_t *row, int g) {
        u32x4 x[D / 32];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            x[i] = *reinterpret_cast<const u32x4 *>(row + 16 * g + (i / 2) * 64 + (i % 2) * 8);
            top = max(top, largest_bits(x[i]));
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const int e = max((int)(top >> 7) - 7, 5);  // the byte of 2^e: the largest is 128 to 256 units
        const float unit = key_scale((uint32_t)(254 - e));
        int h[2 * (D / 32)], l[2 * (D / 32)];
#pragma unroll
        for (int i = 0; i < 2 * (D / 32); ++i) {
            h[i] = l[i] = 0;
            pair<false>(x[i / 2][i % 2 * 2], unit, h[i], l[i]);
            pair<true>(x[i / 2][i % 2 * 2 + 1], unit, h[i], l[i]);
        }
        const int byte = top < kInfBits ? e : 255;  // an infinite or NaN query: NaN scores
        if constexpr (D == 128) {
            w[0] = words{h[0], h[1], h[2], h[3], h[4], h[5], h[6], h[7]};
            w[1] = words{l[0], l[1], l[2], l[3], l[4], l[5], l[6], l[7]};
            scale[0] = byte;
            scale[1] = byte == 255 ? 255 : byte - 5;
        } else {
            w[0] = words{h[0], h[1], h[2], h[3], l[0], l[1], l[2], l[3]};
            scale[0] = byte == 255 || g < 2 ? byte : byte - 5;  // lane group g gives the scale of indices 32 g .. + 31
        }
    }
    template <bool HIGH>
    static __device__ __forceinline__ void pair(uint32_t bf16_pair, float unit, int &h, int &l) {
        const float a = __builtin_bit_cast(float, bf16_pair << 16) * unit, b = __builtin_bit_cast(float, bf16_pair & 0xFFFF0000u) * unit;
        h = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, h, HIGH);
        const f32x2 back = __builtin_amdgcn_cvt_pk_f32_fp8(h, HIGH);
        l = __builtin_amdgcn_cvt_pk_fp8_f32((a - back[0]) * 32.0f, (b - back[1]) * 32.0f, l, HIGH);
    }
    // Instruction TERM of a page's scores; 4: 4-bit keys, 0: 8-bit queries.
    template <int TERM>
    __device__ __forceinline__ f32x4 scores(const u32x4 &k, uint32_t k_scale, f32x4 s) const {
        const words key = {(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, w[TERM], s, 4, 0, 0, (int)k_scale, 0, scale[TERM]);
    }
};

// f(std::integral_constant<int, i>) for i = 0 .. N - 1
template <int N, typename F>
__device__ __forceinline__ void static_for(F f) {
    if constexpr (N > 0) {
        static_for<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// The largest of two score accumulators' numbers, NaN aside, without the instructions that fmaxf quietens its operands with.  The compiler
// does not see that the assembly reads what matrix instructions write, and they need a distance: the median, which it does see and which
// the others wait for, has it kept for both accumulators.
__device__ __forceinline__ float largest_of(const f32x4 &a, const f32x4 &b) {
    float top = __builtin_amdgcn_fmed3f(a[0], b[0], INFINITY);
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(top) : "v"(top), "v"(a[1]), "v"(a[2]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(top) : "v"(top), "v"(a[3]), "v"(b[1]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(top) : "v"(top), "v"(b[2]), "v"(b[3]));
    return top;
}

// 16 NC columns of one wavefront against keys [key_begin, key_end): what a block's wavefronts share out, columns or keys.
//
// kAhead tiles wait in registers.  Where the records come from memory (wave tiles) that is four, or two with 32 columns (us a call with one: 200 decodes
// of 58 and 2 heads of 64 channels 41 and 54; with two instead of four: 64 decodes of 32 and 8 heads next to 512 tokens 52.6 and 55.3), and the memory is the
// bound: 256 decodes of 32 and 8 heads read 418 MB in 71 us, 5.9 TB/s, 512 of 64 and 8 heads 1334 MB in 214, 6.2 TB/s.  Where they come out of a cache
// (chunk tiles) it is one, and issue is the bound, of vector and matrix instructions, which the two wavefronts of a SIMD run under each other: 2048
// tokens of 64 and 8 heads take 142 us, 0.99 Pflop/s (with two tiles 145; three wavefronts do not fit the registers).
template <int D, int NC>
struct QuantisedColumns {
    static constexpr int kOperands = D / 16;  // of output instructions: 16 channels each
    using Tile = QuantisedTile<D>;
    SoftmaxState<D> st[NC];
    PackedQueries<D> packed[NC];
    float scale;
    int pos_eff[NC], lo[NC];  // last key a column may see here, first key inside its sliding window
    // of the wavefront's first column, and of its last one: tiles in between hide no key from any column (wave-uniform; a wavefront
    // without columns of its own shadows the tile's first)
    int min_pos_eff, max_lo;
    f32x4 s[NC][2];  // a tile's scores, hidden keys at -inf
    QuantisedLoads ge;

    // col0: the first column, of the tile's first n_cols; lanes beyond them shadow the tile's first column and store nothing.
    __device__ __forceinline__ void init(const AttnParams &p, const TileDesc &it, int kvh, int col0, int key_end, int lane) {
        const int n = lane & 15, g = lane >> 4;
        const int prefix = it.ctx_len - it.q_len;
        const int G = p.group;
        scale = p.scale_log2;
#pragma unroll
        for (int cg = 0; cg < NC; ++cg) {
            const int mine = col0 + 16 * cg + n;
            const int col = it.col_begin + (mine < it.n_cols ? mine : 0);
            const int row = col / G;
            const int head = kvh * G + (col - row * G);
            pos_eff[cg] = min(prefix + row, key_end - 1);
            lo[cg] = p.window > 0 ? max(0, prefix + row - p.window + 1) : 0;
            packed[cg].load(p.q + ((int64_t)(it.q_start + row) * p.num_q_heads + head) * D, g);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) st[cg].o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
            st[cg].m = kNegSentinel;
            st[cg].l = 0.f;
        }
        const int first = col0 < it.n_cols ? col0 : 0, last = col0 < it.n_cols ? min(col0 + 16 * NC, it.n_cols) - 1 : 0;
        min_pos_eff = min(prefix + (it.col_begin + first) / G, key_end - 1);
        max_lo = p.window > 0 ? max(0, prefix + (it.col_begin + last) / G - p.window + 1) : 0;
        ge.template init<D>(p, it, kvh);
        const int block = D == 128 ? g : (g & 1);  // of 32 channels; with 64 channels the upper two lane groups take the same keys as the lower two
        ge.k_off = (uint32_t)(block * 256 + n * 16);
        ge.k_scale_off = (uint32_t)(Record<D>::kKeyScales + block * 16 + n);
        ge.v_off = (uint32_t)(Record<D>::kValues + lane * (D / 8));
        ge.v_scale_off = (uint32_t)(Record<D>::kValueScales + g * 16);
    }

    // Hides what a column may not see.  of: the scales of the tile's values.
    __device__ __forceinline__ void mask(f32x4 (&of)[2], int tile, int g) {
        if (tile * kTileKeys + (kTileKeys - 1) > min_pos_eff || tile * kTileKeys < max_lo) {  // wave-uniform: some lane must mask
            // A hidden key's weight is 0, which a scale that is not finite (a NaN among the values, or what a slot behind the context
            // holds) would turn into NaN.  Such a scale becomes 0, and the scores of those that see it NaN.
            bool finite = true;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) finite &= __builtin_isfinite(of[b][i]);
            if (!__all(finite)) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool bad = !__builtin_isfinite(of[b][i]);
#pragma unroll
                        for (int cg = 0; cg < NC; ++cg) s[cg][b][i] = bad ? __builtin_nanf("") : s[cg][b][i];
                        of[b][i] = bad ? 0.f : of[b][i];
                    }
            }
#pragma unroll
            for (int cg = 0; cg < NC; ++cg)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = tile * kTileKeys + b * kPageSize + g * 4 + i;
                        s[cg][b][i] = (key <= pos_eff[cg] && key >= lo[cg]) ? s[cg][b][i] : -INFINITY;
                    }
        }
    }
    // A column's reference maximum becomes at least its largest score.  top: this lane's.
    __device__ __forceinline__ void raise(int cg, float top) {
        SoftmaxState<D> &x = st[cg];
        float most = fmaxf(top, __shfl_xor(top, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float m_new = fmaxf(x.m, most * scale);
        const float alpha = __builtin_amdgcn_exp2f(x.m - m_new);
        x.l *= alpha;
        x.m = m_new;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) x.o[c] *= alpha;
    }
    // The first operand of output instructions C: channels 16 C .. + 15, the values of the eight slots that the lane's weights are of.
    template <int C>
    static __device__ __forceinline__ bf16x8 value_operand(const Tile &t) {
        const uint32_t a = t.values[0][C / 2], b = t.values[1][C / 2];
        constexpr int first = C % 2 * 2;
        return __builtin_bit_cast(bf16x8, u32x4{unpack_pair<first>(a, 1.f), unpack_pair<first + 1>(a, 1.f), unpack_pair<first>(b, 1.f),
                                                unpack_pair<first + 1>(b, 1.f)});
    }

    template <bool STREAM, int kAhead, typename Claim>
    __device__ __forceinline__ int run(const AttnParams &p, const TileDesc &it, int kvh, int col0, int key_begin, int key_end, int lane, Claim claim) {
        const int g = lane >> 4;
        init(p, it, kvh, col0, key_end, lane);

        auto process = [&](const Tile &t, int tile) {
#pragma unroll
            for (int cg = 0; cg < NC; ++cg) s[cg][0] = s[cg][1] = f32x4{0.f, 0.f, 0.f, 0.f};
            static_for<PackedQueries<D>::kTerms>([&](auto term) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int cg = 0; cg < NC; ++cg)
                        s[cg][b] = packed[cg].template scores<decltype(term)::value>(t.keys[b], t.key_scales[b], s[cg][b]);
            });
            f32x4 of[2] = {t.value_scales[0], t.value_scales[1]};
            mask(of, tile, g);
            bf16x8 w[NC];
            float top[NC];
            bool higher = false;
#pragma unroll
            for (int cg = 0; cg < NC; ++cg) {
                top[cg] = largest_of(s[cg][0], s[cg][1]);
                higher |= top[cg] * scale > st[cg].m + kRescaleSlack;
            }
            // Only where a score exceeds the reference maximum by more than the slack is the column's maximum looked for across its lanes.
            if (__any(higher)) {
#pragma unroll
                for (int cg = 0; cg < NC; ++cg) raise(cg, top[cg]);
            }
#pragma unroll
            for (int cg = 0; cg < NC; ++cg) {
                f32x8 x;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[cg][i / 4][i % 4], scale, -st[cg].m));
                    st[cg].l += e;
                    x[i] = e * of[i / 4][i % 4];
                }
                // rounded to bf16 for the matrix instruction: each weight is off by at most 2^-8 of itself, averaged down over the keys
                w[cg] = __builtin_convertvector(x, bf16x8);
            }
            static_for<kOperands>([&](auto at) {
                constexpr int c = decltype(at)::value;
                const bf16x8 v = value_operand<c>(t);
#pragma unroll
                for (int cg = 0; cg < NC; ++cg) st[cg].o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, w[cg], st[cg].o[c], 0, 0, 0);
            });
        };

        // The table entries of as many more tiles wait as well: a tile's loads never wait for a scalar one.  The loop proper has no
        // branch around a load, so that each wait is for as many loads as are younger than the tile's own.
        int tile = key_begin / kTileKeys;
        const int tile_end = key_begin >= key_end ? tile : (key_end + kTileKeys - 1) / kTileKeys;
        if (tile >= tile_end) return claim();
        Tile t[kAhead];
        QuantisedPages pages[kAhead];
        auto fetch = [&](QuantisedPages &to, int of_tile) {  // (beyond the range: the sequence's last page again, at most)
            to = ge.pages_of(of_tile);
            __builtin_amdgcn_sched_barrier(0);
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(pages[i], tile + i);
        if (tile + 2 * kAhead <= tile_end) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                ge.template load<STREAM>(pages[i], t[i]);
                fetch(pages[i], tile + kAhead + i);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (tile + i < tile_end) {
                    ge.template load<STREAM>(pages[i], t[i]);
                    fetch(pages[i], tile + kAhead + i);
                }
        }
        for (; tile + 2 * kAhead <= tile_end; tile += kAhead)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                process(t[i], tile + i);
                ge.template load<STREAM>(pages[i], t[i]);
                fetch(pages[i], tile + 2 * kAhead + i);
            }
        const int claimed = claim();  // the next item's counter is read under the last loads
        for (; tile < tile_end; tile += kAhead)
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (tile + i < tile_end) {
                    process(t[i], tile + i);
                    if (tile + kAhead + i < tile_end) ge.template load<STREAM>(pages[i], t[i]);
                }
        return claimed;
    }
};

// A wave tile: 16 or 32 columns, a quarter of the keys to each wavefront.
template <int D, int NC, bool STREAM, typename Claim>
__device__ __forceinline__ int quantised_wave_path(const AttnParams &p, const TileDesc &it, int split, int kvh, uint16_t *smem, Claim claim) {
    const int tid = thread_of_item();
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const UnitRange ur = unit_range(it, split);
    // this wavefront's quarter of the unit (possibly empty: then it contributes weight zero), which begins at a multiple of 32 as every piece does
    const int quarter = ((ur.key_end - ur.key_begin + 3) / 4 + kTileKeys - 1) / kTileKeys * kTileKeys;
    const int begin = min(ur.key_begin + wave * quarter, ur.key_end), end = min(begin + quarter, ur.key_end);
    QuantisedColumns<D, NC> columns;
    const int claimed = columns.template run<STREAM, NC == 1 ? 4 : 2>(p, it, kvh, 0, begin, end, tid & 63, [&] { return tid == 0 ? claim() : 0; });
    wave_finish<D, QuantisedWaveSmem<D>>(p, it, split, kvh, tid, smem, columns.st[0]);
    if constexpr (NC == 2) {
        __syncthreads();
        wave_finish<D, QuantisedWaveSmem<D>>(p, it, split, kvh, tid, smem, columns.st[1], 16);
    }
    return claimed;
}

// A chunk tile: 128 columns, 32 to each wavefront, all of the unit's keys.  The four wavefronts read the same records at about the same
// time, out of the compute unit's own cache but for the first; nothing is shared through LDS and no wavefront waits for another.
template <int D>
__device__ __forceinline__ void quantised_chunk_path(const AttnParams &p, const TileDesc &it, int split, int kvh) {
    const int tid = thread_of_item();
    const int lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int col0 = __builtin_amdgcn_readfirstlane(tid >> 6) * 32;
    if (col0 >= it.n_cols) return;
    const UnitRange ur = unit_range(it, split);
    QuantisedColumns<D, 2> columns;
    // the wavefront's last column sees no key behind its own, its first one none in front of its window
    const int prefix = it.ctx_len - it.q_len, first_row = (it.col_begin + col0) / p.group, last_row = (it.col_begin + min(col0 + 32, it.n_cols) - 1) / p.group;
    const int key_end = min(ur.key_end, prefix + last_row + 1);
    const int key_begin = p.window > 0 ? max(ur.key_begin, (prefix + first_row - p.window + 1) / kTileKeys * kTileKeys) : ur.key_begin;
    columns.template run<false, 1>(p, it, kvh, col0, key_begin, key_end, lane, [] { return 0; });
#pragma unroll
    for (int cg = 0; cg < 2; ++cg) {
        const SoftmaxState<D> &x = columns.st[cg];
        const int mine = col0 + 16 * cg + n;
        float l = x.l + __shfl_xor(x.l, 16);
        l += __shfl_xor(l, 32);
        if (mine >= it.n_cols) continue;
        if (ur.part_row < 0) {
            const int col = it.col_begin + mine, row = col / p.group, head = kvh * p.group + (col - row * p.group);
            uint16_t *op = p.out + ((int64_t)(it.q_start + row) * p.num_q_heads + head) * D + g * 4;
            const float inv = 1.0f / l;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) *reinterpret_cast<u32x2 *>(op + c * 16) = __builtin_bit_cast(u32x2, __builtin_convertvector(x.o[c] * inv, bf16x4));
        } else {  // a piece's (reference maximum, sum, unnormalised output)
            const int64_t prow = ((int64_t)(ur.part_row + mine) * p.num_kv_heads + kvh);
            float *po = p.part_o + prow * D + g * 4;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) *reinterpret_cast<f32x4 *>(po + c * 16) = x.o[c];
            if (g == 0) {
                p.part_ml[prow * 2 + 0] = x.m;
                p.part_ml[prow * 2 + 1] = l;
            }
        }
    }
}

template <int D>
struct QuantisedPaths {
    static constexpr int kWaveElems = QuantisedWaveSmem<D>::kTotalElems, kChunkElems = 8;
    static constexpr int kWaveBlocksPerUnit = 2;
    template <bool STREAM, typename Claim>
    static __device__ __forceinline__ int wave(const AttnParams &p, const TileDesc &it, int split, int kvh, uint16_t *smem, Claim claim) {
        if (it.n_cols > 16) return quantised_wave_path<D, 2, STREAM>(p, it, split, kvh, smem, claim);
        return quantised_wave_path<D, 1, STREAM>(p, it, split, kvh, smem, claim);
    }
    static __device__ __forceinline__ void chunk(const AttnParams &p, const TileDesc &it, int split, int kvh, uint16_t *) {
        quantised_chunk_path<D>(p, it, split, kvh);
    }
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

// Rows out of the cache, the way back: k_new is the pool, k_cache and v_cache the rows.  A block reads the records of HEADS KV heads of one page, all
// of them at once: what it waits for is the chain from its unit over the table to the records.  Bound by memory: 118,000 positions of 8 heads of
// 128 channels, 610 MB, take 109 us or 5.6 TB/s with two heads and rows that bypass the caches, 122 with one head (four 114), 117 with
// two and rows that do not.  STREAM: so many rows, which nothing finds in a cache later.
template <int D, int HEADS, bool STREAM>
__device__ __forceinline__ void kv_read_quantised_block(const AppendParams &p, const AppendUnit *units) {
    using R = Record<D>;
    __shared__ uint32_t words[HEADS][2 * D];  // the values' codes as the page holds them
    const unsigned groups = ((unsigned)p.num_kv_heads + HEADS - 1) / HEADS;
    const int unit = (int)(blockIdx.x / groups);
    const int h0 = (int)(blockIdx.x % groups) * HEADS;
    const u32x4 about = *reinterpret_cast<const u32x4 *>(units + unit);
    const int lo = (int)(about[3] & 0xFFu), hi = (int)(about[3] >> 8);
    const RowsThread<D> t;
    const int64_t page = p.block_table[(int64_t)(int)about[0] * p.max_blocks + (int)about[1]];
    if (page < 0 || page >= p.num_pages) return;  // the rows of a corrupt table entry stay as they are
    uint32_t k[HEADS], k_byte[HEADS];
    float v_unit[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {  // (a last group's missing heads: the last head again)
        const uint8_t *rec = reinterpret_cast<const uint8_t *>(p.k_new) + (page * p.num_kv_heads + min(h0 + i, p.num_kv_heads - 1)) * (int64_t)R::kBytes;
        words[i][threadIdx.x] = reinterpret_cast<const uint32_t *>(rec + R::kValues)[threadIdx.x];
        k[i] = *reinterpret_cast<const uint32_t *>(rec + t.key_word());
        k_byte[i] = rec[t.key_scale()];
        v_unit[i] = reinterpret_cast<const float *>(rec + R::kValueScales)[t.slot];
    }
    __syncthreads();
    if (t.slot < lo || t.slot >= hi) return;
    const int c = t.piece >> 1;
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        if (h0 + i >= p.num_kv_heads) return;
        uint32_t v = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t w = words[i][((t.slot >> 2) * 16 + (t.piece & 1) * 8 + j) * (D / 32) + c / 2];
            v |= ((w >> (16 * (c & 1) + 4 * (t.slot & 3))) & 15u) << (4 * j);
        }
        f32x8 y;
        const f32x2 y0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 0), y1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 1);
        const f32x2 y2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 2), y3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 3);
        y[0] = y0[0] * v_unit[i], y[1] = y0[1] * v_unit[i], y[2] = y1[0] * v_unit[i], y[3] = y1[1] * v_unit[i];
        y[4] = y2[0] * v_unit[i], y[5] = y2[1] * v_unit[i], y[6] = y3[0] * v_unit[i], y[7] = y3[1] * v_unit[i];
        const int64_t dst = ((int64_t)((int)about[2] + t.slot - lo) * p.num_kv_heads + h0 + i) * D + t.piece * 8;
        const u32x4 keys = unpack_word(k[i], key_scale(k_byte[i])), values = __builtin_bit_cast(u32x4, __builtin_convertvector(y, bf16x8));
        if constexpr (STREAM) {
            __builtin_nontemporal_store(keys, reinterpret_cast<u32x4 *>(p.k_cache + dst));
            __builtin_nontemporal_store(values, reinterpret_cast<u32x4 *>(p.v_cache + dst));
        } else {
            *reinterpret_cast<u32x4 *>(p.k_cache + dst) = keys;
            *reinterpret_cast<u32x4 *>(p.v_cache + dst) = values;
        }
    }
}

template <int D, int HEADS>
__global__ __launch_bounds__(2 * D) void kv_read_quantised_kernel(AppendParams p) {
    kv_read_quantised_block<D, HEADS, true>(p, p.units);
}
template <int D, int UNITS>
__global__ __launch_bounds__(2 * D) void kv_read_quantised_inline_kernel(AppendParamsInline<UNITS> p) {
    kv_read_quantised_block<D, 1, false>(p.base, p.units);
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
    with_records(cfg, m, p, [&](auto d, const auto &args) {
        using Args = std::decay_t<decltype(args)>;
        constexpr int D = decltype(d)::value;
        hipStream_t st = static_cast<hipStream_t>(stream);
        if constexpr (RecordsCarried<Args>::value) {
            const dim3 grid((unsigned)m.num_units * (unsigned)cfg.num_kv_heads);
            hipLaunchKernelGGL((kv_read_quantised_inline_kernel<D, RecordsCarried<Args>::kUnits>), grid, dim3(2 * D), 0, st, args);
        } else {
            const dim3 grid((unsigned)m.num_units * (unsigned)((cfg.num_kv_heads + 1) / 2));
            if (cfg.num_kv_heads > 1) hipLaunchKernelGGL((kv_read_quantised_kernel<D, 2>), grid, dim3(2 * D), 0, st, args);
            else hipLaunchKernelGGL((kv_read_quantised_kernel<D, 1>), grid, dim3(2 * D), 0, st, args);
        }
    });
    return (int)hipGetLastError();
}

int launch_attention_quantised(const sarathi_config &cfg, const AttnMeta &m, const void *q, const void *kv_cache, int64_t num_pages, float sm_scale,
                               void *out, int which, void *stream) {
    return launch_attention_paths<QuantisedPaths>(cfg, m, q, kv_cache, nullptr, num_pages, sm_scale, out, which, stream);
}

}  // namespace sarathi
