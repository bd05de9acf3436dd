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


def test_two_models_step_over_one_4bit_cache_at_once(L):
    """On streams of their own, over sequences of their own: neither sees the other's partial results."""
    cfg = synth.model_cfg("tiny", n_layers=4, d_model=512, n_heads=8, n_kv_heads=2, head_dim=64, max_draft=8)
    models = [L.model_create(cfg, weights_to(synth.make_weights(cfg, seed=s), "cuda"), max_batch=2) for s in (1, 2)]
    kv = L.kv_create_int4(models[0], 4, 4 * 100)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    lens = [1400, 700, 1590, 30]
    for l in range(4):
        for b in range(4):
            L.kv_import(kv, b, l, 0, *(torch.randn(lens[b], 128, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)))
    L.kv_set_len(kv, range(4), lens)
    ids, n = [dev_i32([0, 1]), dev_i32([2, 3])], dev_i32([9, 9])
    tokens = [dev_i32([synth.make_prompt(9, cfg["vocab"], 10 * i + j) for j in range(2)]) for i in range(2)]
    want = [L.verify_step(m, kv, ids[i], tokens[i], n) for i, m in enumerate(models)]
    streams = [torch.cuda.Stream() for _ in models]
    out = [[torch.zeros_like(w) for _ in range(40)] for w in want]
    torch.cuda.synchronize()
    for r in range(40):
        for i, m in enumerate(models):
            L.verify_step(m, kv, ids[i], tokens[i], n, logits=out[i][r], stream=streams[i])
    torch.cuda.synchronize()
    for i, m in enumerate(models):
        L.check(m)
        assert all(torch.equal(x, want[i]) for x in out[i])


def _calls_with_results(L):
    """Calls whose result the binding allocates: a call on a stream, by name."""
    cfg = synth.model_cfg("tiny", n_layers=1, d_model=64, d_ffn=64, vocab=64, n_heads=4, n_kv_heads=4, head_dim=64, max_draft=3)
    m = L.model_create(cfg, weights_to(synth.make_weights(cfg, seed=0), "cuda"), max_batch=4)
    caches = [L.kv_create(m, 4, 16), L.kv_create_int4(m, 4, 16)]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(4, 4, 256, device="cuda", generator=g).to(torch.bfloat16)
    ids, n = dev_i32(range(4)), dev_i32([4] * 4)
    for kv in caches:
        L.kv_append(kv, 0, ids, n, x, x)
    tokens = dev_i32(np.arange(16).reshape(4, 4))
    chain = dev_i32([[-1, 0, 1, 2]] * 4)
    logits = torch.randn(4, 4, 64, device="cuda", generator=g)
    docs = [[list(range(60)) * 3] for _ in range(4)]
    pool_tokens, offs = synth.pool_from_documents(docs)
    pool = L.pool_build(pool_tokens, offs, 1, 3)
    prm = L.make_params(K=3, n_min=1, n_max=3, max_occ=64)
    tails, tail_len = dev_i32([[3, 4, 5]] * 4), dev_i32([3] * 4)
    hist, hist_len = dev_i32(np.tile(np.arange(20), (4, 1))), dev_i32([20] * 4)
    draft, draft_len = dev_i32([[6, 7, 8]] * 4), dev_i32([3] * 4)
    last = dev_i32([5] * 4)
    return dict(
        draft=lambda s: L.draft(pool, tails, tail_len, ids, prm, stream=s),
        draft_temp=lambda s: L.draft_temp(pool, tails, tail_len, ids, hist, hist_len, prm, stream=s),
        draft_tree=lambda s: L.draft_tree(pool, tails, tail_len, ids, prm, stream=s),
        make_rows=lambda s: L.make_rows(last, draft, draft_len, 3, stream=s),
        make_rows_tree=lambda s: L.make_rows_tree(last, draft, dev_i32([[0, 1, 2]] * 4), draft_len, 3, stream=s),
        kv_append=lambda s: L.kv_append(caches[1], 0, ids, n, x, x, q=x, stream=s),
        attend_int4=lambda s: L.attend_int4(caches[1], 0, ids, n, x, stream=s),
        kv_export=lambda s: L.kv_export(caches[0], 1, 0, 0, 4, stream=s),
        verify_step=lambda s: L.verify_step(m, caches[1], ids, tokens, n, stream=s),
        verify_step_tree=lambda s: L.verify_step_tree(m, caches[0], ids, tokens, chain, n, stream=s),
        adjust_logits=lambda s: L.adjust_logits(logits, tokens, n, stream=s),
        accept_commit=lambda s: L.accept_commit(None, None, logits, tokens, n, prm, stream=s),
        accept_tree=lambda s: L.accept_tree(None, None, logits, tokens, chain, n, prm, stream=s),
        verify_accept=lambda s: L.verify_accept(m, caches[1], ids, tokens, n, prm, commit=False, stream=s),
    )


def test_results_belong_to_the_stream_of_the_call(L):
    """The current stream still has work to do on memory that was given back: a call on another stream must not get that memory for
    its result."""
    stream = torch.cuda.Stream(priority=-1)
    flat = lambda r: [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]
    for name, call in _calls_with_results(L).items():
        want = [t.clone() for t in flat(call(None))]
        for s in (stream, stream.cuda_stream):               # (a handle will do as well)
            torch.cuda.synchronize()
            torch.cuda.empty_cache()
            stale = [torch.empty_like(t) for t in want]
            torch.cuda._sleep(40_000_000)                    # (some 20 ms)
            for t in stale:
                t.fill_(7)
            del stale, t
            got = flat(call(s))
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), name
