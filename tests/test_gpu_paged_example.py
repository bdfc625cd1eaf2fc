"""The example's whole path against the same prompts evicted without pages or supplied normalisers."""
import importlib.util
import os

import pytest
import torch

from tests import paged_ref as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_2606_15157_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("paged_prefill", os.path.join(ROOT, "examples", "paged_prefill.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("prompts,chunk,page", [((2900, 1337, 700), 512, 16), ((513, 64, 300), 100, 64)])
def test_chunked_prefill_then_eviction(example, prompts, chunk, page):
    steps = 4
    r = example.run(prompts=prompts, chunk=chunk, steps=steps, page=page)
    L, B, H_kv, S = len(r["route"]), len(prompts), r["H_kv"], r["S_cap"]
    H_q = r["out"].shape[1]
    for l in range(L):  # the gathered caches are the rows that were written
        if r["K"][l] is None:
            continue
        for s, n in enumerate(prompts):
            rows = r["qkv"][l][s][:n]
            assert torch.equal(r["K"][l][s, :, :n], rows[:, H_q:H_q + H_kv].transpose(0, 1))
            assert torch.equal(r["V"][l][s, :, :n], rows[:, H_q + H_kv:].transpose(0, 1))
    # the same eviction with the library's own normalisers: the scores agree, so the kept sets do, near-ties aside
    plan, lens = r["plan"], torch.tensor(prompts, dtype=torch.int32, device="cuda")
    bufs = plan.buffers(B, S)
    plan.evict_prefill(r["K"], r["V"], r["Q"], lens, B, S, bufs)
    own = {l: plan.scores(bufs, B, S, l).clone() for l in range(L) if r["Q"][l] is not None}
    for l, want in own.items():
        got = plan.scores(r["bufs"], B, S, l)
        for s, n in enumerate(prompts):
            if r["route"][l] == example.SNAPKV and n <= plan.budget[l]:
                continue  # every position is kept: nothing is scored
            a, b = got[s, :, :n], want[s, :, :n]
            assert ((a - b).abs() <= 2e-3 * b.abs() + 1e-9).all()
    assert torch.equal(bufs["out_count"], r["bufs"]["out_count"])
    same = (bufs["out_idx"] == r["bufs"]["out_idx"]).float().mean()
    assert same > 0.98
    # the FULL layer's last generated token against its whole history
    l = r["route"].index(example.FULL)
    for s, n in enumerate(prompts):
        rows = r["qkv"][l][s][:n + steps]
        m = n + steps
        K, V = rows[:, H_q:H_q + H_kv][None], rows[:, H_q + H_kv:][None]  # one page of m tokens
        q = rows[-1:, :H_q]
        want = ref.attention(K, V, [[0]], q, [0, 1], [m])
        ref.check_attention(r["out"][s:s + 1], None, want, torch.bfloat16)
    assert r["lens"].tolist() == [n + steps for n in prompts]
