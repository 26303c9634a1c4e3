// The entry points of the 4-bit cache under AddressSanitizer / UndefinedBehaviorSanitizer, on the stand-ins of host_paths.cpp: the launchers
// below walk the records and the plan as the kernels do, on heap blocks of exactly the documented sizes.
#include "internal.h"
#define main host_paths_main
#define kWaveCols kQuantisedWaveCols
#include "host_paths.cpp"
#undef kWaveCols
#undef main

namespace sarathi {

static void walk_units(const sarathi_config &cfg, const AppendMeta &m, int64_t num_pages, bool write, uint8_t *pool, uint16_t *k, uint16_t *v) {
    const size_t record = quantised_record_bytes(cfg.head_dim);
    const size_t D = (size_t)cfg.head_dim, H = (size_t)cfg.num_kv_heads;
    if (m.copy_bytes) std::memcpy(m.copy_dst, m.copy_src, (m.copy_bytes + 15) / 16 * 16);
    if (m.zero_bytes) std::memset(m.zero_dst, 0, m.zero_bytes);
    for (int u = 0; u < m.num_units; ++u) {
        const AppendUnit &r = m.units[u];
        const int lo = r.lo_hi & 0xFF, hi = r.lo_hi >> 8;
        CHECK(r.seq >= 0 && r.seq < g_num_seqs && r.page_idx >= 0 && r.page_idx < m.max_blocks);
        CHECK(0 <= lo && lo < hi && hi <= kPageSize && r.row0 >= 0 && r.row0 + (hi - lo) <= g_num_tokens);
        const int64_t page = m.block_table[(int64_t)r.seq * m.max_blocks + r.page_idx];
        CHECK(page >= 0 && page < num_pages);
        for (size_t h = 0; h < H; ++h) {
            uint8_t *rec = pool + ((size_t)page * H + h) * record;
            for (int i = lo; i < hi; ++i) {
                const size_t row = ((size_t)(r.row0 + i - lo) * H + h) * D;
                if (write) rec[record - 64 + 4 * (size_t)i + 3] = (uint8_t)(k[row] + v[row + D - 1]);
                else k[row] = v[row + D - 1] = rec[record - 64 + 4 * (size_t)i + 3];
            }
        }
    }
}
int launch_kv_append_quantised(const sarathi_config &cfg, const AppendMeta &m, const void *k, const void *v, void *pool, int64_t num_pages, void *) {
    walk_units(cfg, m, num_pages, true, static_cast<uint8_t *>(pool), static_cast<uint16_t *>(const_cast<void *>(k)), static_cast<uint16_t *>(const_cast<void *>(v)));
    return 0;
}
int launch_kv_read_quantised(const sarathi_config &cfg, const AppendMeta &m, const void *pool, int64_t num_pages, void *k, void *v, void *) {
    CHECK(m.copy_bytes == 0 && m.zero_bytes == 0);
    walk_units(cfg, m, num_pages, false, static_cast<uint8_t *>(const_cast<void *>(pool)), static_cast<uint16_t *>(k), static_cast<uint16_t *>(v));
    return 0;
}
int launch_attention_quantised(const sarathi_config &cfg, const AttnMeta &m, const void *q, const void *pool, int64_t num_pages, float scale, void *out,
                               int which, void *stream) {
    return launch_attention(cfg, m, q, pool, nullptr, num_pages, scale, out, which, stream);
}

}  // namespace sarathi

int main() {
    std::mt19937_64 rng(11);
    auto rnd = [&](int lo, int hi) { return (int)(lo + rng() % (uint64_t)(hi - lo + 1)); };
    const int shapes[][3] = {{8, 2, 128}, {4, 1, 64}, {14, 2, 128}, {58, 2, 64}, {32, 8, 128}};
    for (int it = 0; it < 75; ++it) {
        const int *sh = shapes[it % 5];
        sarathi_config cfg{sh[0], sh[1], sh[2], 16, 0, 4096, 320, 0};
        const int S = it % 7 == 6 ? rnd(200, 300) : rnd(1, 24);
        std::vector<int32_t> qs(S), ql(S), cl(S);
        int64_t T = 0, pages_needed = 0;
        for (int s = 0; s < S; ++s) {
            ql[s] = rnd(0, 3) == 0 && S < 100 ? rnd(2, 300) : 1;
            cl[s] = ql[s] + rnd(0, it % 5 == 0 ? 9000 : 700);
            qs[s] = (int32_t)T;
            T += ql[s];
            pages_needed += (cl[s] + 15) / 16;
            cfg.max_blocks_per_seq = std::max(cfg.max_blocks_per_seq, (cl[s] + 15) / 16);
        }
        if (T > cfg.max_tokens) continue;
        sarathi_handle *h = nullptr;
        CHECK(sarathi_create(&cfg, &h) == SARATHI_OK);
        if (it % 3 == 1) CHECK(sarathi_set_option(h, "split_keys", 64) == SARATHI_OK && sarathi_set_option(h, "tile_split_keys", 64) == SARATHI_OK);
        if (it % 3 == 2) CHECK(sarathi_set_option(h, "window", rnd(1, 500)) == SARATHI_OK);
        if (it % 4 == 3) CHECK(sarathi_set_option(h, "resident_chunks", 1) == SARATHI_OK);
        if (it % 4 == 2) CHECK(sarathi_set_option(h, "item_queue", 1) == SARATHI_OK);
        const size_t page = sarathi_quantised_page_bytes(h);
        CHECK(page == (size_t)sh[1] * (16 * (size_t)sh[2] + (size_t)sh[2] / 2 + 64));
        std::vector<int32_t> bt((size_t)S * cfg.max_blocks_per_seq, -1);
        int64_t next = 0;
        for (int s = 0; s < S; ++s)
            for (int b = 0; b < (cl[s] + 15) / 16; ++b) bt[(size_t)s * cfg.max_blocks_per_seq + b] = (int32_t)next++;
        const size_t row = (size_t)cfg.num_kv_heads * cfg.head_dim;
        std::vector<uint16_t> k((size_t)T * row, 1), v((size_t)T * row, 2), q((size_t)T * cfg.num_q_heads * cfg.head_dim), out(q.size());
        std::vector<uint16_t> k_rows(k.size()), v_rows(v.size());
        std::vector<uint8_t> pool((size_t)pages_needed * page);
        const size_t ws_bytes = sarathi_workspace_bytes(h);
        void *ws = nullptr;
        CHECK(posix_memalign(&ws, 256, ws_bytes) == 0);
        std::memset(ws, 0xFF, ws_bytes);
        sarathi::g_num_seqs = S;
        sarathi::g_num_tokens = T;
        auto append = [&](void *to, void *scratch) {
            return sarathi_kv_append_quantised(h, k.data(), v.data(), to, bt.data(), qs.data(), ql.data(), cl.data(), S, (int32_t)T, pages_needed, scratch, nullptr);
        };
        auto attend = [&](const void *from, float scale, void *scratch) {
            return sarathi_hybrid_attention_quantised(h, q.data(), from, bt.data(), qs.data(), ql.data(), cl.data(), S, (int32_t)T, pages_needed, scale,
                                                      out.data(), scratch, nullptr);
        };
        auto read = [&](const void *from, void *to) {
            return sarathi_kv_read_quantised(h, from, bt.data(), qs.data(), ql.data(), cl.data(), S, (int32_t)T, pages_needed, to, v_rows.data(), nullptr);
        };
        CHECK(append(pool.data(), ws) == SARATHI_OK);
        for (int rep = 0; rep < 2; ++rep) CHECK(attend(pool.data(), 0.1f, ws) == SARATHI_OK);
        const sarathi_status st = sarathi_hybrid_attention_quantised_noalloc(h, q.data(), pool.data(), bt.data(), qs.data(), ql.data(), cl.data(), S, (int32_t)T,
                                                                             pages_needed, 0.1f, out.data(), nullptr);
        CHECK(st == SARATHI_OK);
        CHECK(read(pool.data(), k_rows.data()) == SARATHI_OK);
        for (int64_t t = 0; t < T; ++t) CHECK(k_rows[(size_t)t * row] == 3 && v_rows[(size_t)(t + 1) * row - 1] == 3);
        // refusals: nothing may be touched
        CHECK(append(nullptr, ws) == SARATHI_EINVAL && append(pool.data(), nullptr) == SARATHI_EWORKSPACE);
        CHECK(append(pool.data() + 8, ws) == SARATHI_EINVAL && append(pool.data(), static_cast<char *>(ws) + 16) == SARATHI_EWORKSPACE);
        CHECK(attend(nullptr, 0.1f, ws) == SARATHI_EINVAL && attend(pool.data() + 4, 0.1f, ws) == SARATHI_EINVAL);
        CHECK(attend(pool.data(), 0.f, ws) == SARATHI_EINVAL && attend(pool.data(), 0.1f, nullptr) == SARATHI_EWORKSPACE);
        CHECK(read(pool.data(), nullptr) == SARATHI_EINVAL && read(pool.data(), k_rows.data() + 1) == SARATHI_EINVAL && read(pool.data() + 1, k_rows.data()) == SARATHI_EINVAL);
        ql[0] += 1;
        CHECK(append(pool.data(), ws) != SARATHI_OK && attend(pool.data(), 0.1f, ws) != SARATHI_OK && read(pool.data(), k_rows.data()) != SARATHI_OK);
        free(ws);
        CHECK(sarathi_destroy(h) == SARATHI_OK);
    }
    CHECK(sarathi_quantised_page_bytes(nullptr) == 0);
    CHECK(sarathi_kv_read_quantised(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0, 0, nullptr, nullptr, nullptr) == SARATHI_EINVAL);
    std::printf("quantised paths clean\n");
    return 0;
}
