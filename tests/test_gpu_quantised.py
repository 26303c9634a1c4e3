"""GPU parity of the 4-bit cache: records and rows bit for bit against the reference, attention against the fp64 checker on what the
records stand for (exact in bf16, so the checker sees the very operands): a row within 1e-2 in the 2-norm, as on the bf16 path, since
the kernels round the softmax weights (times the values' scales) to bf16, each off by at most 2^-8 of itself, and the output once, which
both average down over keys or channels.  An element's bound stands at ``compare``."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle
from oracle import quantised_cache_reference as qref
from paper_2403_02310_amd import workloads as wl
from tests import parity

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hx():
    from paper_2403_02310_amd import harness
    return harness


SHAPES = {
    "mqa4_d64": wl.AttnShape(4, 1, 64),
    "gqa4_d128": wl.AttnShape(8, 2, 128),
    "gqa7_d128": wl.AttnShape(14, 2, 128),
    "mha_d64": wl.AttnShape(3, 3, 64),
    "mqa20_d128": wl.AttnShape(20, 1, 128),
    "gqa29_d64": wl.AttnShape(58, 2, 64),
}


def compare(got, ref, what, most):
    """``most``: the largest magnitude among the values.  An output is sum(w v) / sum(w).  Rounded weights are off by at most 2^-8 of
    themselves, which moves it by at most 2^-8 sum(w |v|) / sum(w) <= 2^-8 most; its own rounding by at most 2^-8 |out| <= 2^-8 most; the
    scores' fp32 sums of at most 128 products by well under a hundredth of that.  So 2^-7 * 1.02 * most bounds an element's error by
    arithmetic, and where that is more than the bf16 path's bound (values beyond 2.5 that one key decides) it takes its place."""
    assert got.shape == ref.shape and np.isfinite(got).all(), what
    err, norm = np.abs(got - ref), np.linalg.norm(ref, axis=-1)
    rel = np.linalg.norm(got - ref, axis=-1) / np.where(norm > 0, norm, 1.0)
    msg = "%s: max abs %.3e, max row rel %.3e" % (what, err.max(), rel.max())
    assert err.max() <= max(parity.ABS_TOL, 1.02 * 2.0 ** -7 * most) and rel.max() <= parity.ROW_REL_TOL, msg


def _held(kv):
    """What the cache holds of the rows of each sequence, bf16 bits."""
    return {i: qref.stands_for(*rows) for i, rows in kv.items()}


def _reference(b, kv, q_bits=None, window=0):
    held = _held(kv)
    k, v = (np.concatenate([held[i][j] for i in range(b.num_seqs)]) for j in range(2))
    ref = oracle.hybrid_attention(b.q_bits(0) if q_bits is None else q_bits, k, v, b.kv_start, b.q_start, b.q_len, b.ctx_len, b.sm_scale, window=window)
    return ref, np.abs(qref._f64(v)).max()


def _check(hx, b, opts=None, fill=0xFF, what=""):
    print("case", b.name, what, "seed", b.seed, "q_len", b.q_len[:8], "ctx", b.ctx_len[:8], opts, flush=True)
    h = hx.make_handle(b)
    for k, v in (opts or {}).items():
        h.set_option(k, v)
    st = hx.setup_and_run_quantised(b, fill, handle=h)
    ref = _reference(b, st["kv_host"], window=(opts or {}).get("window", 0))
    compare(hx.bf16_tensor_to_f64(st["out"]), ref[0], "%s %s" % (b.name, opts), ref[1])
    return st, ref


def _expected_pool(b, shape, fill):
    pool = np.full(shape, fill, np.uint8)
    for i in range(b.num_seqs):
        k, v = b.kv_bits(i)
        qref.append(pool, k, v, b.block_table[i:i + 1], [0], [int(b.ctx_len[i])], [int(b.ctx_len[i])])
    return pool


@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("fill", [0xFF, 0x00, 0x5A])
def test_records_after_appends_in_pieces(hx, shape, fill):
    """Prefixes, then chunks and decodes that begin and end at every slot: all bytes of the pool, untouched ones among them."""
    lens = [1, 2, 15, 16, 17, 31, 33, 40, 5, 9]
    q = [1, 1, 7, 16, 2, 1, 33, 13, 4, 8]
    b = wl._make("records_" + shape, SHAPES[shape], q, lens, 41)
    print("case", shape, fill, flush=True)
    h = hx.make_handle(b)
    st = hx.setup_and_run_quantised(b, fill, handle=h)
    np.testing.assert_array_equal(st["pool"].cpu().numpy(), _expected_pool(b, tuple(st["pool"].shape), fill))


@pytest.mark.parametrize("records", [1, 24, 25, 224, 225, 700])
@pytest.mark.parametrize("inline", [0, 1])
def test_append_and_read_with_records_in_arguments_or_in_memory(hx, records, inline):
    s = SHAPES["gqa4_d128"]
    b = wl._make("records", s, [1] * records, [1 + 7 * i % 90 for i in range(records)], 42)
    h = hx.make_handle(b)
    h.set_option("inline_append", inline)
    st = hx.setup_and_run_quantised(b, 0x11, handle=h)
    np.testing.assert_array_equal(st["pool"].cpu().numpy(), _expected_pool(b, tuple(st["pool"].shape), 0x11))
    k, v = (torch.empty(records, s.num_kv_heads, s.head_dim, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    h.kv_read_quantised(st["pool"], st["bt"], b.q_start, b.q_len, b.ctx_len, k, v)
    want = qref.read(_expected_pool(b, tuple(st["pool"].shape), 0x11), b.block_table, b.q_len, b.ctx_len, s.head_dim)
    for got, ref in zip((k, v), want):
        np.testing.assert_array_equal(hx.device_to_bits(got), ref)


@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("q_len,ctx", [([1], [1]), ([67], [197]), ([16, 16], [16, 48]), ([1, 300, 33, 1], [16, 300, 50, 777]), ([15, 17], [31, 17])])
def test_read_back_of_arbitrary_records(hx, shape, q_len, ctx):
    """Every byte pattern of codes, ordinary scales: rows equal the reference bit for bit; rows behind the last stay."""
    s = SHAPES[shape]
    b = wl._make("read", s, q_len, ctx, 43)
    h = hx.make_handle(b)
    rng = np.random.default_rng(44)
    pool = rng.integers(0, 256, h.quantised_cache_shape(b.num_pages), dtype=np.uint8)
    d = s.head_dim
    pool[..., 16 * d:16 * d + d // 2] = rng.integers(120, 135, pool[..., 16 * d:16 * d + d // 2].shape)
    scales = rng.choice(qref.VALUE_SCALES[(qref.VALUE_SCALES > 2.0 ** -6) & (qref.VALUE_SCALES < 64)], pool.shape[:2] + (16,)).astype(np.float32)
    pool[..., 16 * d + d // 2:] = scales.view(np.uint8)
    n = b.num_tokens
    k, v = (torch.full((n + 3, s.num_kv_heads, d), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    h.kv_read_quantised(torch.from_numpy(pool).cuda(), torch.from_numpy(b.block_table).cuda(), b.q_start, b.q_len, b.ctx_len, k, v)
    for got, ref in zip((k, v), qref.read(pool, b.block_table, b.q_len, b.ctx_len, d)):
        got = hx.device_to_bits(got)
        np.testing.assert_array_equal(qref._f64(got[:n]), qref._f64(ref))
        np.testing.assert_array_equal(qref._f64(got[n:]), 7.0)


@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_read_back_of_many_pages(hx, shape):
    """More pages than a launch's arguments hold, one, two and an odd number of KV heads, ragged ends: rows bit for bit."""
    s = SHAPES[shape]
    b = wl._make("read_many", s, [1500, 1, 1777, 33, 250], [1507, 40, 1777, 35, 999], 46)
    h = hx.make_handle(b)
    pool = np.full(h.quantised_cache_shape(b.num_pages), 0x21, np.uint8)
    d, rng = s.head_dim, np.random.default_rng(47)
    pool[..., :16 * d] = rng.integers(0, 256, pool[..., :16 * d].shape)
    pool[..., 16 * d:16 * d + d // 2] = rng.integers(120, 135, pool[..., 16 * d:16 * d + d // 2].shape)
    pool[..., 16 * d + d // 2:] = np.full(pool.shape[:2] + (16,), 0.6875, np.float32).view(np.uint8)
    k, v = (torch.full((b.num_tokens + 3, s.num_kv_heads, d), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    h.kv_read_quantised(torch.from_numpy(pool).cuda(), torch.from_numpy(b.block_table).cuda(), b.q_start, b.q_len, b.ctx_len, k, v)
    for got, ref in zip((k, v), qref.read(pool, b.block_table, b.q_len, b.ctx_len, d)):
        got = hx.device_to_bits(got)
        np.testing.assert_array_equal(qref._f64(got[:b.num_tokens]), qref._f64(ref))
        np.testing.assert_array_equal(qref._f64(got[b.num_tokens:]), 7.0)


def _rows_bits(values):
    return wl.f32_to_bf16_bits(np.asarray(values, np.float32))


def test_special_rows(hx):
    """Ties, zeros of both signs, subnormals, the largest numbers, infinities and NaN: codes and scales bit for bit."""
    s = wl.AttnShape(2, 1, 64)
    rows = [np.zeros(64), -np.zeros(64)]
    rows.append(np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0], 4))
    for top in (3.0, 2.25, 1.5 * 2.0 ** -20, 1.03125, 5.96875):           # a sixth of it on and off four bits
        rows.append(np.tile(np.array([1, -5, 7, 2, -3, 11, 12, -12, 10, 6, 4.5, -1.5, 8, 9, 0.5, 0]) * top / 12, 4))
    rows.append(np.full(64, 2.0 ** -130))
    rows.append(np.linspace(-1, 1, 64) * 2.0 ** -101)
    rows.append(np.linspace(-3.3e38, 3.3e38, 64))
    rows.append(np.full(64, 1.27e38))
    k = _rows_bits(np.stack(rows))[:, None, :]
    for bad in (0x7F80, 0xFF80, 0x7FC1):
        x = k[2:3].copy()
        x[0, 0, 37] = bad
        k = np.concatenate([k, x])
    n = len(k)
    b = wl._make("special", s, [n], [n], 45)
    h = hx.make_handle(b)
    pool = hx.make_quantised_pool(h, b.num_pages, 0x33)
    bt = torch.from_numpy(b.block_table).cuda()
    dev = hx.bits_to_device(k)
    h.kv_append_quantised(dev, dev, pool, bt, b.q_start, b.q_len, b.ctx_len)
    want = np.full(tuple(pool.shape), 0x33, np.uint8)
    qref.append(want, k, k, b.block_table, b.q_start, b.q_len, b.ctx_len)
    got = pool.cpu().numpy()
    at = 16 * 64 + 32
    np.testing.assert_array_equal(got[..., :at], want[..., :at])
    np.testing.assert_array_equal(np.ascontiguousarray(got[..., at:]).view(np.float32), np.ascontiguousarray(want[..., at:]).view(np.float32))  # NaN payloads aside
    out = [torch.empty_like(dev) for _ in range(2)]
    h.kv_read_quantised(pool, bt, b.q_start, b.q_len, b.ctx_len, *out)
    for x, ref in zip(out, qref.read(want, b.block_table, b.q_len, b.ctx_len, 64)):
        np.testing.assert_array_equal(qref._f64(hx.device_to_bits(x)), qref._f64(ref))


@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("seed", [101, 102])
def test_random_ragged_hybrid(hx, shape, seed):
    """Odd chunk sizes, mid-page prefixes, 1-token contexts, shuffled sequence order."""
    _check(hx, wl.random_hybrid(seed, SHAPES[shape], n_chunks=3, n_decodes=6, max_chunk=90, max_ctx=420))


def test_edge_lengths(hx):
    """Contexts of 1, 15, 16, 17, 31, 32, 33 as decodes and as whole prefills (prefix 0)."""
    for shape in ("gqa4_d128", "mqa4_d64"):
        lens = [1, 15, 16, 17, 31, 32, 33, 64, 65]
        _check(hx, wl._make("edges", SHAPES[shape], [1] * len(lens) + lens, lens + lens, 77))


@pytest.mark.parametrize("shape", ["gqa4_d128", "mqa4_d64", "gqa29_d64"])
@pytest.mark.parametrize("hint", [0, 1])
def test_decodes_of_every_number_of_tiles(hx, shape, hint):
    """Decodes whose wavefronts get no tile, one, two and so on, with ragged last tiles; uncut and in blocks of 128 keys."""
    ctx = list(range(1, 34, 8)) + [64, 96, 97, 128, 129, 160, 255, 256, 257, 290, 383, 384, 385, 512, 513, 640, 769, 897, 1025, 1153, 1601, 2049]
    b = wl._make("tiles_" + shape, SHAPES[shape], [1] * len(ctx), ctx, 91)
    for opts in ({}, {"split_keys": 32}, {"split_keys": 1 << 20}):
        _check(hx, b, {"stream_kv": hint, **opts})


OPTIONS = [{}, {"tile_split_keys": 64, "split_keys": 32}, {"tile_min_cols": 1}, {"tile_min_cols": 1 << 20}, {"interleave": 0}, {"interleave": 1},
           {"interleave": 2, "resident_chunks": 1}, {"item_queue": 1}, {"item_queue": 1, "resident_chunks": 0, "split_keys": 32}, {"decode_blocks_per_cu": 1},
           {"decode_blocks_per_cu": 2}, {"plan_at_append": 0}, {"resident_chunks": 1, "tile_split_keys": 96, "window": 333}]


@pytest.mark.parametrize("shape", ["gqa7_d128", "gqa4_d128", "mqa4_d64", "gqa29_d64"])
@pytest.mark.parametrize("opts", OPTIONS, ids=str)
def test_every_kind_of_launch_and_both_entry_points(hx, shape, opts):
    b = wl._make("launch_" + shape, SHAPES[shape], [300, 1, 37, 1, 129], [1300, 555, 37, 1, 2222], 79)
    st, ref = _check(hx, b, opts)
    first = st["out"].clone()
    h = st["handle"]
    st["out"].zero_()
    h.hybrid_attention_quantised(st["q"], st["pool"], st["bt"], b.q_start, b.q_len, b.ctx_len, b.sm_scale, st["out"])    # planned by itself
    assert torch.equal(first.view(torch.int16), st["out"].view(torch.int16)), opts
    st["out"].zero_()
    h.hybrid_attention_quantised_noalloc(st["q"], st["pool"], st["bt"], b.q_start, b.q_len, b.ctx_len, b.sm_scale, st["out"])
    compare(hx.bf16_tensor_to_f64(st["out"]), ref[0], "allocation-free %s" % opts, ref[1])


@pytest.mark.parametrize("shape", ["gqa4_d128", "gqa7_d128", "mqa4_d64"])
@pytest.mark.parametrize("window", [1, 17, 64, 300])
def test_sliding_window(hx, shape, window):
    b = wl._make("window_" + shape, SHAPES[shape], [300, 1, 37, 1, 1, 70], [1300, 555, 37, 1, 2000, 70], 84)
    for opts in ({}, {"tile_split_keys": 64, "split_keys": 32}, {"tile_min_cols": 1}, {"tile_min_cols": 1 << 20}):
        _check(hx, b, {"window": window, **opts})


@pytest.mark.parametrize("shape", ["gqa4_d128", "mqa4_d64"])
def test_peaky_scores_raise_the_softmax_reference_mid_sequence(hx, shape):
    b = wl._make("peaky_" + shape, SHAPES[shape], [260, 1, 1, 40], [1500, 900, 33, 40], 86, sm_scale=1.0)
    for opts in ({}, {"tile_split_keys": 96, "split_keys": 64}, {"tile_min_cols": 1}, {"tile_min_cols": 1 << 20}):
        _check(hx, b, opts)


def test_long_contexts_and_pools_beyond_32_bits(hx):
    """A decode over 131,072 keys, a 96-row chunk behind 100,000, and a pool whose last pages lie beyond 4 GiB."""
    s = SHAPES["gqa4_d128"]
    b = wl._make("very_long", s, [1, 96, 1], [131072, 100096, 77], 81, slack=1.0)
    far = 1_100_000                                                    # pages of 4352 bytes: 4.79 GB
    table = np.where(b.block_table >= 0, far - 1 - b.block_table, -1).astype(np.int32)
    b = wl.HybridBatch(b.name, b.shape, b.q_len, b.ctx_len, table, far, b.seed, b.sm_scale)
    _check(hx, b)


@pytest.mark.parametrize("bad", [0x7F80, 0xFF80, 0x7FC1])
@pytest.mark.parametrize("shape", ["gqa4_d128", "mqa4_d64"])
def test_what_hidden_positions_hold_reaches_no_row(hx, bad, shape):
    """Keys and values that are infinite or NaN behind a row's own position, in front of its window and beyond the context:
    rows that do not see them keep every bit, rows that do are NaN."""
    s = SHAPES[shape]
    q_len, ctx, window = [150, 1, 40, 1], [400, 700, 40, 45], 100
    b = wl._make("hidden_" + shape, s, q_len, ctx, 88)
    kv = {i: tuple(x.copy() for x in b.kv_bits(i)) for i in range(b.num_seqs)}
    clean = {i: tuple(x.copy() for x in rows) for i, rows in kv.items()}
    places = {0: [5, 390], 1: [0, 599], 2: [33]}
    for i, at in places.items():
        for j, x in enumerate(kv[i]):
            for p in at:
                x[p, :, 3 + 40 * j % 64] = bad
    for opts in ({}, {"tile_min_cols": 1}, {"tile_min_cols": 1 << 20}, {"tile_split_keys": 96, "split_keys": 32}):
        outs = []
        for rows in (clean, kv):
            h = hx.make_handle(b)
            h.set_option("window", window)
            for k, v in opts.items():
                h.set_option(k, v)
            outs.append(hx.bf16_tensor_to_f64(hx.setup_and_run_quantised(b, 0xFF, handle=h, kv_host=dict(rows))["out"]))
        t = 0
        for i in range(b.num_seqs):
            for r in range(q_len[i]):
                p = ctx[i] - q_len[i] + r
                sees = any(max(0, p - window + 1) <= x <= p for x in places.get(i, []))
                if sees:
                    assert np.isnan(outs[1][t]).all(axis=-1).any(), (opts, i, r)
                else:
                    np.testing.assert_array_equal(outs[0][t], outs[1][t], err_msg="%s %d %d" % (opts, i, r))
                t += 1


def test_page_placement_and_reruns_are_bitwise_stable(hx):
    b = wl.random_hybrid(5, SHAPES["gqa4_d128"], n_chunks=2, n_decodes=4, max_chunk=70, max_ctx=900)
    a = hx.device_to_bits(hx.setup_and_run_quantised(b)["out"])
    np.testing.assert_array_equal(a, hx.device_to_bits(hx.setup_and_run_quantised(b, 0x00)["out"]))
    perm = np.random.default_rng(9).permutation(b.num_pages).astype(np.int32)
    bt2 = np.where(b.block_table >= 0, perm[np.maximum(b.block_table, 0)], -1).astype(np.int32)
    b2 = wl.HybridBatch(b.name + "_perm", b.shape, b.q_len, b.ctx_len, bt2, b.num_pages, b.seed, b.sm_scale)
    np.testing.assert_array_equal(a, hx.device_to_bits(hx.setup_and_run_quantised(b2)["out"]))


def test_one_handle_serves_both_kinds_of_cache(hx):
    """Appends and attention of the two kinds in every order on one workspace: a plan of one kind is not used for the other."""
    b = wl._make("both", SHAPES["gqa4_d128"], [200, 1, 1, 37], [900, 700, 33, 37], 90)
    h = hx.make_handle(b)
    plain, quant = hx.setup_and_run(b, 0x7FC1, handle=h), hx.setup_and_run_quantised(b, 0xFF, handle=h)
    firsts = plain["out"].clone(), quant["out"].clone()
    parity.compare(hx.bf16_tensor_to_f64(firsts[0]), oracle.attention_for_batch(b), "bf16")
    ref, most = _reference(b, quant["kv_host"])
    compare(hx.bf16_tensor_to_f64(firsts[1]), ref, "4 bits", most)
    lengths = b.q_start, b.q_len, b.ctx_len
    for order in ("pq", "qp", "pp", "qq", "qpp", "pqq"):
        if order[0] == "p":
            h.kv_append(quant["k_new"], quant["v_new"], plain["k_cache"], plain["v_cache"], plain["bt"], *lengths)
        else:
            h.kv_append_quantised(quant["k_new"], quant["v_new"], quant["pool"], quant["bt"], *lengths)
        for kind in order[1:]:
            out = torch.zeros_like(firsts[0])
            if kind == "p":
                h.hybrid_attention(plain["q"], plain["k_cache"], plain["v_cache"], plain["bt"], *lengths, b.sm_scale, out)
            else:
                h.hybrid_attention_quantised(quant["q"], quant["pool"], quant["bt"], *lengths, b.sm_scale, out)
            assert torch.equal(out.view(torch.int16), firsts["pq".index(kind)].view(torch.int16)), order


def test_iterations_back_to_back_and_on_two_streams(hx):
    """Forty iterations without a host wait, reads among them, then on two streams in turn: every output equal to its first."""
    s = SHAPES["gqa4_d128"]
    batches = [wl._make("ring%d" % i, s, [70 + 9 * i, 1, 1, 5], [300 + 40 * i, 500 - 30 * i, 64 + i, 90], 300 + i, max_blocks=40) for i in range(3)]
    from paper_2403_02310_amd import binding
    h = binding.Handle(s.num_q_heads, s.num_kv_heads, s.head_dim, max_tokens=2048, max_seqs=128, max_blocks_per_seq=40)
    states = [hx.setup_and_run_quantised(b, 0xFF, handle=h) for b in batches]
    firsts = []
    for b, st in zip(batches, states):
        ref, most = _reference(b, st["kv_host"])
        compare(hx.bf16_tensor_to_f64(st["out"]), ref, b.name, most)
        rows = [torch.empty_like(st["k_new"]) for _ in range(2)]
        h.kv_read_quantised(st["pool"], st["bt"], b.q_start, b.q_len, b.ctx_len, *rows)
        firsts.append([hx.device_to_bits(x) for x in [st["out"]] + rows])

    def iteration(b, st, stream=None):
        out, rows = torch.empty_like(st["q"]), [torch.empty_like(st["k_new"]) for _ in range(2)]
        h.kv_append_quantised(st["k_new"], st["v_new"], st["pool"], st["bt"], b.q_start, b.q_len, b.ctx_len, stream=stream)
        h.hybrid_attention_quantised(st["q"], st["pool"], st["bt"], b.q_start, b.q_len, b.ctx_len, b.sm_scale, out, stream=stream)
        h.kv_read_quantised(st["pool"], st["bt"], b.q_start, b.q_len, b.ctx_len, *rows, stream=stream)
        return [out] + rows
    outs = [iteration(batches[i % 3], states[i % 3]) for i in range(40)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(24):
        on = streams[(i // 3) % 2]
        on.wait_stream(streams[1 - (i // 3) % 2])
        with torch.cuda.stream(on):
            outs.append(iteration(batches[(40 + i) % 3], states[(40 + i) % 3], on))
    torch.cuda.synchronize()
    for i, got in enumerate(outs):
        for x, ref in zip(got, firsts[i % 3]):
            np.testing.assert_array_equal(hx.device_to_bits(x), ref)


def test_captured_call_replays(hx):
    """The allocation-free call in a graph, replayed between the program's own work, against the eager result each time."""
    b = wl._make("graph", SHAPES["gqa4_d128"], [64, 1, 1], [192, 700, 300], 92)
    st, ref = _check(hx, b)
    h, out = st["handle"], torch.zeros_like(st["out"])
    call = lambda o: h.hybrid_attention_quantised_noalloc(st["q"], st["pool"], st["bt"], b.q_start, b.q_len, b.ctx_len, b.sm_scale, o)  # noqa: E731
    eager = torch.zeros_like(out)
    call(eager)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(out)
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16))
        again = torch.zeros_like(out)
        call(again)
        torch.cuda.synchronize()
        assert torch.equal(again.view(torch.int16), eager.view(torch.int16))
    compare(hx.bf16_tensor_to_f64(eager), ref[0], "eager", ref[1])


def test_pages_out_of_range_are_not_followed(hx):
    """Table entries beyond the pool: an append leaves the pool as it was there, a read the rows, attention stays inside the pool."""
    s = SHAPES["gqa4_d128"]
    b = wl._make("range", s, [20, 1], [40, 70], 93)
    st = hx.setup_and_run_quantised(b, 0x00)
    h, bad = st["handle"], b.block_table.copy()
    bad[0, 1], bad[1, 4] = b.num_pages + 5, -7
    bt, before = torch.from_numpy(bad).cuda(), st["pool"].clone()
    h.kv_append_quantised(st["k_new"], st["v_new"], st["pool"], bt, b.q_start, b.q_len, b.ctx_len)
    torch.cuda.synchronize()
    assert torch.equal(before, st["pool"])                              # the valid pages got the rows they had
    rows = [torch.full_like(st["k_new"], 7.0) for _ in range(2)]
    h.kv_read_quantised(st["pool"], bt, b.q_start, b.q_len, b.ctx_len, *rows)
    for x in rows:
        kept = (x == 7.0).flatten(1).all(1).cpu().numpy()
        np.testing.assert_array_equal(kept, [i < 12 or i == 20 for i in range(21)])   # positions 20..31 of page 1; the decode's page
    h.hybrid_attention_quantised(st["q"], st["pool"], bt, b.q_start, b.q_len, b.ctx_len, b.sm_scale, torch.empty_like(st["out"]))
    torch.cuda.synchronize()


def test_chunking_invariance(hx):
    """A 192-token prompt as 1 x 192, 3 x 64 and 192 x 1: the same records, outputs within the tolerance of the one result."""
    s = SHAPES["mqa4_d64"]
    q_all, pools = wl.normal_bf16((1, 0x51, 99), (192, 4, 64)), []
    for chunk in (192, 64, 1):
        iters = wl.config1_prompt(chunk)
        last = iters[-1]
        k_all, v_all = last.kv_bits(0)
        held = qref.stands_for(k_all, v_all)
        ref = oracle.hybrid_attention(q_all, *held, [0], [0], [192], [192], last.sm_scale)
        h = hx.make_handle(last)
        pool, bt, rows = hx.make_quantised_pool(h, last.num_pages), torch.from_numpy(last.block_table).cuda(), []
        for it in iters:
            n, ctx = int(it.q_len[0]), int(it.ctx_len[0])
            new = [hx.bits_to_device(x[ctx - n:ctx]) for x in (q_all, k_all, v_all)]
            rows.append(hx.bf16_tensor_to_f64(hx.run_iteration_quantised(h, it, pool, bt, *new)))
        compare(np.concatenate(rows), ref, "chunks of %d, %s" % (chunk, s), np.abs(qref._f64(held[1])).max())
        pools.append(pool.cpu().numpy())
    for p in pools[1:]:
        np.testing.assert_array_equal(p, pools[0])


def test_randomized_batches_shapes_and_options(hx):
    shapes = list(SHAPES.values()) + [wl.AttnShape(32, 8, 128), wl.AttnShape(8, 8, 64), wl.AttnShape(12, 4, 64)]
    rng = np.random.default_rng(20240312)
    for case in range(40):
        shape, opts = shapes[int(rng.integers(len(shapes)))], OPTIONS[int(rng.integers(len(OPTIONS)))]
        n_chunks = int(rng.integers(0, 4))
        n_dec = int(rng.integers(0 if n_chunks else 1, 40))
        max_ctx = int(rng.choice([60, 400, 1500, 4000]))
        b = wl.random_hybrid(9000 + case, shape, n_chunks, n_dec, max_chunk=min(int(rng.choice([8, 130, 400])), max_ctx), max_ctx=max_ctx)
        _check(hx, b, opts, what="case %d %s" % (case, shape))


@pytest.mark.parametrize("shape", ["gqa4_d128", "gqa29_d64"])
def test_queries_with_an_outlying_channel(hx, shape):
    """A query channel 2^13 times the others, against keys that are zero there: the other channels decide.  A query number is off by at most
    2^-23 of its head's largest, 2^-10 here; over the channels, whose signs are random, a score is off by about 2^-10 of a key's norm
    over sqrt(D), a thousandth, and a weight by as much of itself: a quarter of its rounding to bf16."""
    s = SHAPES[shape]
    q_len, ctx = [1, 64, 1], [700, 333, 65]
    b = wl._make("outlier", s, q_len, ctx, 48)
    h = hx.make_handle(b)
    pool = hx.make_quantised_pool(h, b.num_pages, 0xFF)
    bt = torch.from_numpy(b.block_table).cuda()
    zero, ks, vs = np.zeros(1, np.int32), [], []
    for i in range(b.num_seqs):
        k, v = (x.copy() for x in b.kv_bits(i))
        k[..., 5] = 0
        n = np.array([ctx[i]], np.int32)
        h.kv_append_quantised(hx.bits_to_device(k), hx.bits_to_device(v), pool, bt[i:i + 1], zero, n, n)
        held = qref.stands_for(k, v)
        ks.append(held[0]), vs.append(held[1])
    q_bits = b.q_bits(0).copy()
    q_bits[..., 5] = wl.f32_to_bf16_bits(np.float32([8192.0]))[0]
    q = hx.bits_to_device(q_bits)
    out = torch.empty_like(q)
    h.hybrid_attention_quantised(q, pool, bt, b.q_start, b.q_len, b.ctx_len, b.sm_scale, out)
    v = np.concatenate(vs)
    ref = oracle.hybrid_attention(q_bits, np.concatenate(ks), v, b.kv_start, b.q_start, b.q_len, b.ctx_len, b.sm_scale)
    compare(hx.bf16_tensor_to_f64(out), ref, b.name, np.abs(qref._f64(v)).max())
