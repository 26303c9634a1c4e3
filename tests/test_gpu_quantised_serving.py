"""The 4-bit cache where the framework's own paths use it: the serving loop (appends, hybrid attention, rows read back of running requests)
and the token-budget profile."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle
from oracle import quantised_cache_reference as qref
from paper_2403_02310_amd import serving
from paper_2403_02310_amd import token_budget as tb
from paper_2403_02310_amd import workloads as wl

from tests.test_gpu_quantised import compare

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


@pytest.mark.parametrize("policy", ["stall_free", "prefill_first"])
@pytest.mark.parametrize("shape", [wl.AttnShape(8, 2, 128), wl.AttnShape(29, 1, 64)], ids=["gqa4_d128", "mqa29_d64"])
def test_requests_match_one_shot_attention(policy, shape):
    """A request's attention rows, gathered over all the batches it travelled in, against one computation over what the cache holds
    of its rows; the rows that running requests read back, bit for bit."""
    reqs = serving.synthetic_trace(21, 10, 50000.0, prompt_median=150, prompt_p90=420, output_median=8, output_p90=14,
                                   max_prompt=600, max_output=16)
    backend = serving.GpuBackend(seed=5, cache="4bit")
    loop = serving.ServingLoop(shape, reqs, backend, num_pages=600, token_budget=128, chunk_size=96, max_batch_size=16,
                               policy=policy, seed=2)
    print("policy", policy, "prompts", [r.prompt_len for r in reqs], "outputs", [r.output_len for r in reqs], flush=True)
    read = 0
    while loop.step() is not None:
        for r in loop.prefilling + loop.decoding:
            n = r.num_prefilled + r.num_decoded
            if n == 0 or len(loop.iterations) % 3:
                continue
            want = qref.stands_for(_bits(backend.k_all[r.token_base:r.token_base + n]), _bits(backend.v_all[r.token_base:r.token_base + n]))
            for got, ref in zip(backend.cached_rows(r), want):
                np.testing.assert_array_equal(qref._f64(_bits(got)), qref._f64(ref))
            read += 1
    assert read > 5 and len(loop.done) == len(reqs) and loop.pool.free == loop.pool.num_pages
    scale = 1.0 / np.sqrt(shape.head_dim)
    for r in loop.done:
        a, b = r.token_base, r.token_base + r.total_rows
        k, v = qref.stands_for(_bits(backend.k_all[a:b]), _bits(backend.v_all[a:b]))
        ref = oracle.hybrid_attention(_bits(backend.q_all[a:b]), k, v, [0], [0], [r.total_rows], [r.total_rows], scale)
        compare(backend.out_all[a:b].to(torch.float64).cpu().numpy(), ref, "request %d" % r.id, np.abs(qref._f64(v)).max())
    with pytest.raises(ValueError):
        backend.cached_rows(loop.done[0])


def test_token_budget_profile():
    shape, checked = wl.AttnShape(8, 2, 128), []

    def check(batch, dev):
        pool, bt = dev["kv_cache"].cpu().numpy(), dev["block_table"].cpu().numpy()
        k, v = qref.read(pool, bt, batch.ctx_len, batch.ctx_len, shape.head_dim)
        ref = oracle.hybrid_attention(_bits(dev["q"]), k, v, batch.kv_start, batch.q_start, batch.q_len, batch.ctx_len, batch.sm_scale)
        compare(dev["out"].to(torch.float64).cpu().numpy(), ref, batch.name, np.abs(qref._f64(v)).max())
        checked.append(batch.num_tokens)

    rows = tb.profile(tb.gpu_timer(reps=5, warmup=2, on_batch=check, cache="4bit"), shape, [4, 64, 512], [700] * 8, chunk_prefix=1500, seed=3)
    print(rows, flush=True)
    assert checked == [8, 64, 512] and all(r["seconds"] > 0 for r in rows)
