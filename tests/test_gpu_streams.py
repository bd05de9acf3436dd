"""Calls on streams that the default stream does not wait for and that do not wait for it (torch.cuda.Stream): what a create call leaves
behind is finished when it returns, what a call allocates for itself or for its result belongs to the stream that it runs on."""
import numpy as np
import pytest
import torch

from helpers import dev_i32, ensure_built, weights_to
from paper_2408_05676_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    ensure_built()
    from paper_2408_05676_b200 import binding
    return binding


@pytest.mark.parametrize("int4", [False, True])
def test_a_new_cache_is_empty_before_the_call_returns(L, int4):
    """Some gigabytes to be zeroed; rows are imported at once, into the last pages, and are still there."""
    cfg = synth.model_cfg("tiny", n_layers=1, d_model=64, d_ffn=64, vocab=64, n_heads=8, n_kv_heads=8, head_dim=128)
    m = L.model_create(cfg, weights_to(synth.make_weights(cfg, seed=0), "cuda"), max_batch=1)
    pages = 1000000 if int4 else 160000
    x = torch.randn(160, 1024, device="cuda").to(torch.bfloat16)
    stream = torch.cuda.Stream(priority=-1)
    torch.cuda.synchronize()
    kv = (L.kv_create_int4 if int4 else L.kv_create)(m, 1, pages)
    done = torch.cuda.default_stream().query()
    L.kv_import(kv, 0, 0, (pages - 10) * 16, x, x, stream=stream)
    torch.cuda.synchronize()
    assert done
    k, v = L.kv_export(kv, 0, 0, (pages - 10) * 16, 160)
    assert torch.equal(k, v) and (k.float() - x.float()).abs().max() <= (0.5 if int4 else 0)


def test_a_new_model_is_ready_before_the_call_returns(L):
    """A workspace of gigabytes to be zeroed; a step runs at once."""
    cfg = synth.model_cfg("tiny", n_layers=2, d_model=512, d_ffn=65536, vocab=64, max_draft=63)
    W = weights_to(synth.make_weights(cfg, seed=3), "cuda")
    ids, n = dev_i32([0]), dev_i32([64])
    tokens = dev_i32([synth.make_prompt(64, cfg["vocab"], 1)])
    stream = torch.cuda.Stream(priority=-1)
    first = L.model_create(cfg, W, max_batch=512)
    kv = L.kv_create(first, 1, 8)
    torch.cuda.synchronize()
    want = L.verify_step(first, kv, ids, tokens, n)
    logits = torch.zeros_like(want)
    torch.cuda.synchronize()
    m = L.model_create(cfg, W, max_batch=512)
    assert torch.cuda.default_stream().query()
    L.verify_step(m, kv, ids, tokens, n, logits=logits, stream=stream)
    torch.cuda.synchronize()
    L.check(m)
    assert torch.equal(logits, want)


def test_a_model_that_first_meets_a_4bit_cache_in_a_step(L):
    """Its rows for projections are made in the step: nothing that is still to come touches them."""
    cfg = synth.model_cfg("tiny", n_layers=12, d_model=256, n_heads=32, n_kv_heads=8, head_dim=128, d_ffn=256, vocab=64, max_draft=8)
    W = weights_to(synth.make_weights(cfg, seed=3), "cuda")
    maker = L.model_create(cfg, W, max_batch=8)
    ids, n = dev_i32(range(8)), dev_i32([9] * 8)
    tokens = dev_i32([synth.make_prompt(9, cfg["vocab"], s) for s in range(8)])
    kv = L.kv_create_int4(maker, 8, 8)
    want = L.verify_step(maker, kv, ids, tokens, n)
    stream = torch.cuda.Stream(priority=-1)
    for busy in (2_000_000, 6_000_000, 10_000_000):        # clocks for which the default stream has work that it began before
        other = L.model_create(cfg, W, max_batch=2048)      # (18432 rows of 6144 numbers)
        logits = [torch.empty_like(want) for _ in range(60)]
        torch.cuda.synchronize()
        torch.cuda._sleep(busy)
        for x in logits:
            L.verify_step(other, kv, ids, tokens, n, logits=x, stream=stream)
        torch.cuda.synchronize()
        L.check(other)
        assert all(torch.equal(x, want) for x in logits)
