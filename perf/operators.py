"""The 4-bit key/value cache: rows quantised as they are written, read back, and attended over in one scheduling iteration.

Three kinds of case.  ``write`` is ``Handle.kv_append_quantised`` of a batch's new keys and values and
``Handle.kv_read_quantised`` of the same positions; ``read`` is the latter over whole contexts, as for a request that moves
elsewhere; ``attention`` is ``Handle.hybrid_attention_quantised`` (or its allocation-free form) of one layer over prefill
chunks and decodes.

What the cache holds.  Both are 4-bit numbers of magnitudes 0, 0.5, 1, 1.5, 2, 3, 4 and 6 with a sign, rounded to the nearest,
ties to the even code, larger ones to 6.

  keys    32 neighbouring channels of a position share a scale 2^e: the smallest with max |k| <= 6 * 2^e, e in -100 .. 124,
          held as the byte e + 127; the byte 255 and a NaN for each value where one of the 32 is infinite or NaN
  values  the channels of a position and head share a scale m * 2^e, m in 8 .. 15: the smallest with max |v| <= 6 * m * 2^e,
          not below 2^-100 and not above 2^124, held as a 32-bit float; a NaN where one of them is infinite or NaN

A page of 16 positions of one KV head of D channels is one record of 16.5 D + 64 bytes:

  keys    [D/32 blocks][16 slots][16 bytes]: channels 2j and 2j+1 of the block in the low and the high half of byte j
  values  [4 slot quads][16][D/16][2 bytes]: channel 16 i + n of the quad's slots at [n][i], two slots to a byte, the lower in the low half
  scales  of the keys, [D/32][16 slots] bytes, then of the values, [16 slots] floats
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16

# query heads, key/value heads, head_dim
HEADS = {
    "tiny": (4, 1, 64),
    "mistral-7b": (32, 8, 128),
    "yi-34b": (56, 8, 128),
    "llama2-70b": (64, 8, 128),
    "llama2-70b/tp4": (16, 2, 128),
    "falcon-180b/tp4": (58, 2, 64),
}


def _case(name, kind, heads, chunks="", decodes=0, low=0, high=0, spread="uniform", lengths=0, window=0, entry="workspace"):
    """``chunks``: positions @ cached prefix, comma separated.  ``decodes`` sequences of ``low`` to ``high`` positions, the last of
    which is the iteration's (``read``: all of which are read)."""
    return {"name": name, "kind": kind, "heads": heads, "chunks": chunks, "decodes": decodes, "low": low, "high": high,
            "spread": spread, "lengths": lengths, "window": window, "entry": entry}


def listed():
    return [
        # A decode batch's new rows: one slot of a page each, launches and host time.
        _case("write_64_decodes", "write", "mistral-7b", "", 64, 256, 4096, lengths=1),
        # A large prefill budget: two chunks that begin and end inside pages, next to decodes.
        _case("write_2048_tokens", "write", "llama2-70b", "1299@0,680@4211", 69, 512, 4096, lengths=2),
        # The end of one short request, odd in length and place.
        _case("read_67_tokens", "read", "tiny", "67@130", lengths=3),
        # Long requests that move to another server.
        _case("read_long_contexts", "read", "mistral-7b", "", 11, 5000, 16384, lengths=4),
        # The smallest attention: a short prompt's chunk next to three decodes, one KV head of 64 channels, without a workspace.
        _case("tiny_hybrid", "attention", "tiny", "64@128", 3, 100, 300, lengths=5, entry="noalloc"),
        # A lightly loaded server: eight requests generate, nothing is prefilled.
        _case("mistral_8_decodes", "attention", "mistral-7b", "", 8, 256, 4096, lengths=6),
        # A decode-only iteration of a busy server, skewed context lengths.
        _case("mistral_256_decodes", "attention", "mistral-7b", "", 256, 64, 8192, "lognormal", lengths=7),
        # Stall-free batching's usual iteration: one 512-token chunk on top of what is cached and the running decodes.
        _case("mistral_hybrid", "attention", "mistral-7b", "512@1871", 64, 256, 4096, lengths=8),
        # The model's sliding window, ragged chunk, contexts beyond the window.
        _case("mistral_window", "attention", "mistral-7b", "435@6001", 77, 1024, 12288, lengths=9, window=4096),
        # Many query heads to a KV head of 64 channels: two column tiles read the same keys.
        _case("falcon_200_decodes", "attention", "falcon-180b/tp4", "", 200, 1024, 8192, lengths=10),
        # The largest decode batch that a 4-bit cache is for.
        _case("llama70b_512_decodes", "attention", "llama2-70b", "", 512, 512, 4096, lengths=11),
        # Prefill alone, a 2048-token budget: a prompt's first tokens and the ragged rest of another's.
        _case("llama70b_prefill", "attention", "llama2-70b", "1299@0,749@4211"),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of the same ranges: batch sizes, contexts, chunk lengths and token counts over their logarithms."""
    heads = rng.choice(sorted(HEADS))
    kind = rng.choice(["write", "read", "attention", "attention", "attention"])
    mode = rng.choice(["decodes", "hybrid", "hybrid", "chunks"])
    high = _log_uniform(rng, 512, 16384)
    most = 100_000 if kind == "read" else 1_100_000
    decodes = 0 if mode == "chunks" else max(1, min(_log_uniform(rng, 1, 512), most // high))
    chunks = []
    if mode != "decodes":
        for _ in range(rng.choice([1, 1, 2, 3])):
            chunks.append("%d@%d" % (_log_uniform(rng, 1, 682), rng.choice([0, _log_uniform(rng, 1, 8192)])))
    window = rng.choice([0, 0, 0, 4096]) if kind == "attention" else 0
    entry = rng.choice(["workspace", "workspace", "workspace", "noalloc"]) if kind == "attention" else "workspace"
    c = _case("", kind, heads, ",".join(chunks), decodes, _log_uniform(rng, 1, 256) if decodes else 0, high if decodes else 0,
              rng.choice(["uniform", "lognormal"]), rng.randrange(1 << 20), window, entry)
    del c["name"]
    return c


def _lengths(case):
    """(q_len, ctx_len) of the batch: chunks first, then the decodes."""
    q_len, ctx = [], []
    for text in filter(None, case["chunks"].split(",")):
        new, prefix = (int(t) for t in text.split("@"))
        q_len.append(new)
        ctx.append(prefix + new)
    n, low, high = case["decodes"], case["low"], case["high"]
    rng = np.random.default_rng([case["lengths"], 0xCA5E])
    if case["spread"] == "lognormal":
        got = np.clip(np.rint(np.exp(math.log(max(1.0, high / 8)) + 0.8 * rng.standard_normal(n))), low, high)
    else:
        got = rng.integers(low, high + 1, size=n)
    last = [int(c) for c in got]
    return np.array(q_len + (last if case["kind"] == "read" else [1] * n), np.int32), np.array(ctx + last, np.int32)


def _record(d):
    return 16 * d + d // 2 + 64


# ---- the plain form: elementary operations on whole tensors, in 32 bits ----

def _codes(y):
    """4-bit codes of ``y``, which is in units of the scale: of the seven borders between magnitudes, those behind an odd one are
    passed at the border itself, the others beyond it."""
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    for border, at in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= border) if at else (a > border)
    return code + 8 * (y < 0).to(torch.uint8)


def _quantise(k, v):
    """Codes and scales of rows [..., D]: keys' codes and bytes [..., D/32], values' codes and floats [...]."""
    k, v = k.float().unflatten(-1, (-1, 32)), v.float()
    bad = ~k.isfinite().all(-1)
    k = k.masked_fill(bad[..., None], 0.0)
    bits = k.abs().amax(-1).view(torch.int32)              # 1.f * 2^E: the smallest e with 1.f * 2^E <= 1.5 * 2^(e + 2)
    e = ((bits >> 23) - 129 + ((bits & 0x7FFFFF) > 0x400000).to(torch.int32)).clamp(-100, 124)
    k_codes = _codes(k * (((127 - e) << 23).view(torch.float32))[..., None]).flatten(-2)
    k_scale = torch.where(bad, 255, e + 127).to(torch.uint8)
    bad = ~v.isfinite().all(-1)
    v = v.masked_fill(bad[..., None], 0.0)
    top = (v.abs().amax(-1).double() / 6.0).float().clamp(2.0 ** -100, 2.0 ** 124)
    scale = ((top.view(torch.int32) + 0xFFFFF) & ~0xFFFFF).view(torch.float32)     # up to four significant bits
    v_codes = _codes((v.double() / scale.double()[..., None]).float())             # a border of the magnitudes is met exactly
    return k_codes, k_scale, v_codes, torch.where(bad, math.nan, scale)


def _pack(k_codes, k_scale, v_codes, v_scale):
    """Records of pages: codes [..., 16, D], keys' scales [..., 16, D/32], values' scales [..., 16] -> [..., record]."""
    k = k_codes.unflatten(-1, (-1, 16, 2)).transpose(-4, -3)                        # [block, slot, byte, half]
    v = v_codes.unflatten(-1, (-1, 16)).unflatten(-3, (4, 2, 2))                    # [quad, byte, half, i, n]
    n = v.dim()
    v = v.permute(*range(n - 5), n - 5, n - 1, n - 2, n - 4, n - 3)
    join = lambda c: (c[..., 0] | (c[..., 1] << 4)).flatten(-3) if c.dim() < n else (c[..., 0] | (c[..., 1] << 4)).flatten(-4)  # noqa: E731
    return torch.cat([join(k), join(v), k_scale.transpose(-1, -2).flatten(-2), v_scale.contiguous().view(torch.uint8)], -1)


def _unpack(records, d):
    """The inverse of ``_pack``."""
    halves = lambda b: torch.stack([b & 15, b >> 4], -1)                            # noqa: E731
    k = halves(records[..., :8 * d]).unflatten(-2, (d // 32, 16, 16)).transpose(-4, -3).flatten(-3)
    v = halves(records[..., 8 * d:16 * d]).unflatten(-2, (4, 16, d // 16, 2))       # [quad, n, i, byte, half]
    n = v.dim()
    v = v.permute(*range(n - 5), n - 5, n - 2, n - 1, n - 3, n - 4).flatten(-2).flatten(-4, -2)
    k_scale = records[..., 16 * d:16 * d + d // 2].unflatten(-1, (d // 32, 16)).transpose(-1, -2)
    return k, k_scale, v, records[..., 16 * d + d // 2:].contiguous().view(torch.float32)


def _magnitudes(code):
    """What the codes stand for, in units of the scale."""
    e, m = ((code >> 1) & 3).to(torch.int32), (code & 1).float()
    a = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * (((e + 126) << 23).view(torch.float32)))
    return torch.where(code > 7, -a, a)


def _values(records, d):
    """Keys and values [..., 16, D] that records stand for, 32 bits."""
    k, k_scale, v, v_scale = _unpack(records, d)
    scale = torch.where(k_scale == 255, math.nan, (k_scale.to(torch.int32) << 23).view(torch.float32))
    return (_magnitudes(k).unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2), _magnitudes(v) * v_scale[..., None]


def _places(s):
    """The pages of a batch's tokens, and each token's place among them and its slot there."""
    seq = np.repeat(np.arange(len(s["q_len"])), s["q_len"])
    at = np.arange(len(seq)) - s["q_start"][seq] + (s["ctx_len"] - s["q_len"])[seq]
    pages, back = np.unique(seq * s["table"].shape[1] + at // PAGE, return_inverse=True)
    return s["table"].flatten()[torch.from_numpy(pages).cuda()].long(), torch.from_numpy(back).cuda(), torch.from_numpy(at % PAGE).cuda()


def _plain_append(s):
    pages, back, slot = _places(s)
    held = _unpack(s["cache"][pages], s["d"])
    for old, new in zip(held, _quantise(s["k_new"], s["v_new"])):
        old.transpose(1, 2)[back, slot] = new
    s["cache"][pages] = _pack(*held)


def _plain_read(s):
    pages, back, slot = _places(s)
    return [x.transpose(1, 2)[back, slot].to(torch.bfloat16) for x in _values(s["cache"][pages], s["d"])]


def _plain_rows(s, seqs, rows, q_len, ctx_len):
    """Attention of sequences of at most ``q_len`` rows and ``ctx_len`` positions; ``rows``: their rows' places in the batch [S, q_len],
    the last ones of a shorter sequence repeated."""
    hq, hkv, d = HEADS[s["case"]["heads"]]
    k, v = _values(s["cache"][s["table"][seqs, : -(-ctx_len // PAGE)].clamp(min=0).long()], d)  # [S, pages, Hkv, 16, D]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))                                   # [S, Hkv, L, D]
    q = s["q"][rows].float().unflatten(2, (hkv, hq // hkv)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [S, Hkv, rows * group, D]
    at = s["ctx_dev"][seqs][:, None] - s["q_dev"][seqs][:, None] + (rows - s["start_dev"][seqs][:, None])   # a row's position
    key = torch.arange(k.shape[2], device="cuda")
    seen = key <= at[..., None]
    if s["case"]["window"]:
        seen &= key > at[..., None] - s["case"]["window"]
    score = torch.matmul(q, k.transpose(2, 3)).unflatten(2, (q_len, -1)) * s["scale"]
    score = score.masked_fill(~seen[:, None, :, None, :], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (q_len, -1)) / p.sum(-1, keepdim=True)
    return o.permute(0, 2, 1, 3, 4).flatten(2, 3).to(torch.bfloat16)


def _plain_attention(s):
    n = len(s["q_len"]) - s["case"]["decodes"]
    for i in range(n):                                     # chunks one by one, the decodes together
        t0, c = int(s["q_start"][i]), int(s["q_len"][i])
        rows = torch.arange(t0, t0 + c, device="cuda")[None]
        s["out"][t0:t0 + c] = _plain_rows(s, torch.tensor([i], device="cuda"), rows, c, int(s["ctx_len"][i]))[0]
    if s["case"]["decodes"]:
        seqs = torch.arange(n, len(s["q_len"]), device="cuda")
        rows = s["start_dev"][seqs][:, None]
        s["out"][int(s["q_start"][n]):] = _plain_rows(s, seqs, rows, 1, int(s["ctx_len"][n:].max()))[:, 0]
    return s["out"]


def prepare(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    q_len, ctx_len = _lengths(case)
    tokens = int(q_len.sum())
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)          # noqa: E731
    channel = torch.exp(0.5 * normal(hkv, 1, d))           # keys have channels that are larger throughout
    need = -(-ctx_len.astype(np.int64) // PAGE)
    pages = int(need.sum()) * 5 // 4 + 1                   # a pool that is not full, pages of a sequence scattered over it
    cache = torch.empty(pages, hkv, _record(d), device="cuda", dtype=torch.uint8)
    for at in range(0, pages, 8192):
        n = min(8192, pages - at)
        k, v = (normal(n, hkv, PAGE, d) * channel).to(torch.bfloat16), normal(n, hkv, PAGE, d).to(torch.bfloat16)
        cache[at:at + n] = _pack(*_quantise(k, v))
    order = torch.randperm(pages, device="cuda", generator=g, dtype=torch.int64).to(torch.int32)
    table = torch.full((len(q_len), int(need.max())), -1, device="cuda", dtype=torch.int32)
    at = 0
    for s, n in enumerate(need.tolist()):
        table[s, :n] = order[at:at + n]
        at += n
    q_start = np.concatenate([[0], np.cumsum(q_len)[:-1]]).astype(np.int32)
    state = {"case": case, "d": d, "q_start": q_start, "q_len": q_len, "ctx_len": ctx_len, "table": table, "cache": cache}
    if case["kind"] == "attention":
        state.update(q=normal(tokens, hq, d).to(torch.bfloat16), out=torch.empty(tokens, hq, d, device="cuda", dtype=torch.bfloat16),
                     scale=1.0 / math.sqrt(d))
        state.update({name: torch.from_numpy(a.astype(np.int64)).cuda() for name, a in (("start_dev", q_start), ("q_dev", q_len), ("ctx_dev", ctx_len))})
    else:
        state["rows"] = [torch.empty(tokens, hkv, d, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    if case["kind"] == "write":
        state.update(k_new=(normal(tokens, hkv, d) * channel[:, 0]).to(torch.bfloat16), v_new=normal(tokens, hkv, d).to(torch.bfloat16))
    if own:
        from paper_2403_02310_amd import binding
        handle = binding.Handle(hq, hkv, d, max_tokens=max(tokens, 4096), max_seqs=max(len(q_len), 64), max_blocks_per_seq=table.shape[1])
        if case["window"]:
            handle.set_option("window", case["window"])
        if case["kind"] == "write":
            handle.set_option("plan_at_append", 0)         # no attention call follows
        if case["kind"] != "read":
            handle.ensure_workspace()
        state["handle"] = handle
    return state


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        if kind == "attention":
            return _plain_attention(s)
        if kind == "write":
            _plain_append(s)
        return _plain_read(s)
    h, batch = s["handle"], (s["table"], s["q_start"], s["q_len"], s["ctx_len"])
    if kind == "attention":
        attend = h.hybrid_attention_quantised_noalloc if s["case"]["entry"] == "noalloc" else h.hybrid_attention_quantised
        return attend(s["q"], s["cache"], *batch, s["scale"], s["out"])
    if kind == "write":
        h.kv_append_quantised(s["k_new"], s["v_new"], s["cache"], *batch)
    return list(h.kv_read_quantised(s["cache"], *batch, *s["rows"]))


def work(case):
    hq, hkv, d = HEADS[case["heads"]]
    held, row = hkv * (d + d // 32 + 4), 2 * hkv * d * 2   # a position's bytes in the cache and as rows, all heads
    q_len, ctx_len = (a.tolist() for a in _lengths(case))
    tokens = sum(q_len)
    if case["kind"] != "attention":
        return {"bytes": tokens * (held + row * (2 if case["kind"] == "write" else 1)), "flops": 2 * tokens * hkv * d}
    cached = pairs = 0
    for q, c in zip(q_len, ctx_len):
        w = case["window"] or c
        cached += min(c, w + q - 1)                        # positions that some row sees
        pairs += sum(min(p + 1, w) for p in range(c - q, c)) if case["window"] else q * (c - q) + q * (q + 1) // 2
    return {"bytes": cached * held + tokens * 2 * hq * d * 2, "flops": 4 * d * hq * pairs}


# ---- in 64 bits, from the definition at the top, sequence by sequence ----

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest(y):
    """The number of the grid nearest to each of ``y``, an even place of the grid where two are as near."""
    places = [0, 2, 4, 6, 1, 3, 5, 7]
    grid = torch.tensor([_GRID[i] for i in places], device="cuda", dtype=torch.float64)
    out = torch.empty_like(y)
    for at in range(0, y.shape[0], 256):
        part = y[at:at + 256]
        out[at:at + 256] = grid[(part.abs()[..., None] - grid).abs().argmin(-1)] * torch.sign(part)
    return out


def _exact_held(k, v):
    """What the cache holds of finite rows [T, Hkv, D]."""
    k, v = k.double().unflatten(-1, (-1, 32)), v.double()
    e = torch.ceil(torch.log2((k.abs().amax(-1, keepdim=True) / 6).clamp(min=2.0 ** -100))).clamp(max=124.0)
    unit = torch.exp2(e)
    least = (v.abs().amax(-1, keepdim=True) / 6).clamp(2.0 ** -100, 2.0 ** 124)
    eighth = torch.exp2(torch.floor(torch.log2(least)) - 3)
    scale = torch.ceil(least / eighth) * eighth
    return (_nearest(k / unit) * unit).flatten(-2), _nearest(v / scale) * scale


def _exact_cached(s, i):
    """Keys and values [ctx, Hkv, D] of sequence i, byte by byte."""
    _, hkv, d = HEADS[s["case"]["heads"]]
    ctx = int(s["ctx_len"][i])
    rec = s["cache"][s["table"][i, : -(-ctx // PAGE)].long()]
    grid = torch.tensor(_GRID + tuple(-x for x in _GRID), device="cuda", dtype=torch.float64)
    slot, c = torch.arange(PAGE, device="cuda")[:, None], torch.arange(d, device="cuda")[None, :]
    k = rec[..., ((c // 32) * 16 + slot) * 16 + (c % 32) // 2] >> (4 * (c % 2)).to(torch.uint8)
    v = rec[..., 8 * d + ((slot // 4 * 16 + c % 16) * (d // 16) + c // 16) * 2 + slot % 4 // 2] >> (4 * (slot % 2)).to(torch.uint8)
    k_unit = torch.exp2(rec[..., 16 * d + (c // 32) * 16 + slot].double() - 127)
    v_unit = rec[..., 16 * d + d // 2:].contiguous().view(torch.float32).double()[..., None]
    return [(grid[(code & 15).int()] * unit).transpose(1, 2).reshape(-1, hkv, d)[:ctx] for code, unit in ((k, k_unit), (v, v_unit))]


def exact(case, seed):
    s = prepare(case, seed)
    hq, hkv, d = HEADS[case["heads"]]
    if case["kind"] == "write":
        return list(_exact_held(s["k_new"], s["v_new"]))
    seqs = list(zip(s["q_start"].tolist(), s["q_len"].tolist(), s["ctx_len"].tolist()))
    if case["kind"] == "read":
        rows = [[x[ctx - n:] for x in _exact_cached(s, i)] for i, (_, n, ctx) in enumerate(seqs)]
        return [torch.cat([r[j] for r in rows]) for j in range(2)]
    out = torch.empty(s["out"].shape, device="cuda", dtype=torch.float64)
    for i, (t0, n, ctx) in enumerate(seqs):
        k, v = _exact_cached(s, i)
        k, v = k.permute(1, 2, 0).contiguous(), v.permute(1, 0, 2).contiguous()     # [Hkv, D, ctx], [Hkv, ctx, D]
        keys = torch.arange(ctx, device="cuda")
        for r0 in range(0, n, 256):
            r1 = min(n, r0 + 256)
            at = torch.arange(ctx - n + r0, ctx - n + r1, device="cuda")
            q = s["q"][t0 + r0:t0 + r1].double().reshape(r1 - r0, hkv, hq // hkv, d).permute(1, 0, 2, 3).reshape(hkv, -1, d).contiguous()
            score = torch.bmm(q, k).reshape(hkv, r1 - r0, hq // hkv, ctx) * s["scale"]
            hidden = keys[None, :] > at[:, None]
            if case["window"]:
                hidden |= keys[None, :] <= at[:, None] - case["window"]
            p = torch.softmax(score.masked_fill_(hidden[None, :, None, :], -math.inf), dim=-1)
            o = torch.bmm(p.reshape(hkv, -1, ctx), v).reshape(hkv, r1 - r0, hq // hkv, d)
            out[t0 + r0:t0 + r1] = o.permute(1, 0, 2, 3).reshape(r1 - r0, hq, d)
    return out
