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
