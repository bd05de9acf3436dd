"""A row's result over a 4-bit cache does not depend on its place in the call (csrc/attn_int4.cu): the same bits with drafts behind it and
alone, whatever the other sequences hold and how many rows they have, in whichever order they come.  Strict decoding equals plain greedy
decoding by this, also where two logits nearly tie, and a code that a last bit would turn."""
import numpy as np
import pytest
import torch

from helpers import dev_i32, ensure_built, weights_to
from paper_2408_05676_b200 import synth
from test_gpu_int4_cache import bf, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    ensure_built()
    from paper_2408_05676_b200 import binding
    return binding


# heads, kv heads, head_dim, sequences, rows, longest text: several CTAs a text, one, tiles of 8 to 40 rows, more than one tile; CTAs of two sizes
SHAPES = [(4, 4, 64, 1, 1, 4000), (8, 2, 128, 3, 9, 3000), (32, 32, 128, 2, 9, 600), (32, 32, 128, 16, 9, 300), (40, 40, 128, 12, 17, 500), (8, 1, 64, 2, 5, 2000),
          (4, 1, 128, 5, 33, 700), (2, 2, 64, 3, 64, 900), (4, 4, 64, 2, 41, 100), (8, 8, 64, 70, 3, 200), (32, 32, 64, 16, 1, 3000),
          (16, 16, 64, 24, 9, 2100)]


@pytest.mark.parametrize("heads,kv_heads,dim,B,rows,most", SHAPES)
def test_attention_of_a_row_anywhere(L, heads, kv_heads, dim, B, rows, most):
    rng = np.random.default_rng(heads * 100 + rows)
    kv = make(L, heads, kv_heads, dim, B, -(-(most + rows) // 16) + 3)
    lens = rng.integers(0, most, B)
    lens[0] = most
    w = kv_heads * dim
    for s in range(B):
        # (scores that rise here and there: references change on the way)
        k = rng.standard_normal((lens[s] + rows, w)) * np.linspace(0.5, 6, lens[s] + rows)[:, None]
        L.kv_import(kv, s, 0, 0, bf(k), bf(rng.standard_normal((lens[s] + rows, w))))
    q = bf(rng.standard_normal((B, rows, heads, dim)) * 2)
    ids = dev_i32(range(B))

    def call(lens, n, q, order=None):
        L.kv_set_len(kv, range(B), lens)
        o = np.arange(B) if order is None else order
        out = L.attend_int4(kv, 0, dev_i32(o), dev_i32(np.asarray(n)[o]), q[torch.as_tensor(o, device="cuda")].contiguous())
        back = torch.empty_like(out)
        back[torch.as_tensor(o, device="cuda")] = out
        return back

    full = call(lens, [rows] * B, q)
    assert torch.isfinite(full).all()
    assert torch.equal(call(lens, [rows] * B, q, rng.permutation(B)), full)                 # in another order
    for i in sorted(set(rng.integers(0, rows, 6).tolist()) | {0, rows - 1}):
        some = rng.integers(0, rows + 1, B)                                                 # among fewer rows
        some[0] = i + 1
        part = call(lens, some, q)
        for b in range(B):
            assert torch.equal(part[b, :some[b]], full[b, :some[b]])
        alone = torch.zeros_like(q)                                                         # alone, behind the tokens before it
        alone[:, 0] = q[:, i]
        assert torch.equal(call(lens + i, [1] * B, alone)[:, 0], full[:, i]), i
        gone = rng.random(B) < 0.5                                                          # where other texts have ended
        gone[0] = False
        left = call(np.where(gone, 0, lens), np.where(gone, 0, rows), q)
        for b in np.nonzero(~gone)[0]:
            assert torch.equal(left[b], full[b])


def test_a_trees_rows_beside_other_trees(L):
    """The rows of a token tree, where the other sequences have other trees, fewer rows, other lengths or none."""
    rng = np.random.default_rng(8)
    B, rows = 20, 17
    kv = make(L, 8, 8, 128, B, 80)
    lens = rng.integers(0, 1200, B)
    for s in range(B):
        L.kv_import(kv, s, 0, 0, bf(rng.standard_normal((lens[s] + rows, 1024)) * 2), bf(rng.standard_normal((lens[s] + rows, 1024))))
    q = bf(rng.standard_normal((B, rows, 8, 128)) * 2)
    par = lambda: np.array([[-1] + [rng.integers(0, i) for i in range(1, rows)] for _ in range(B)], np.int32)
    first, ids = par(), dev_i32(range(B))
    L.kv_set_len(kv, range(B), lens)
    full = L.attend_int4(kv, 0, ids, dev_i32([rows] * B), q, parents=dev_i32(first))
    for _ in range(4):
        keep = rng.random(B) < 0.4
        keep[0] = True
        n = np.where(keep, rows, rng.integers(0, rows + 1, B))
        L.kv_set_len(kv, range(B), np.where(keep, lens, rng.integers(0, 1200, B)))
        got = L.attend_int4(kv, 0, ids, dev_i32(n), q, parents=dev_i32(np.where(keep[:, None], first, par())))
        for b in np.nonzero(keep)[0]:
            assert torch.equal(got[b], full[b])


@pytest.mark.parametrize("over,B,K,ctx", [(dict(), 4, 8, 150), (dict(n_heads=4, n_kv_heads=2, head_dim=128, d_model=512), 3, 15, 700), (dict(), 40, 4, 61)])
def test_a_step_of_all_rows_and_of_one_after_the_other(L, over, B, K, ctx):
    """Logits of all K + 1 rows at once, and of each alone: the same bits; what the cache then holds as well."""
    cfg = synth.model_cfg("tiny", max_draft=K, **over)
    m = L.model_create(cfg, weights_to(synth.make_weights(cfg, seed=0, gain_jitter=0.1), "cuda"), max_batch=B)
    kv = L.kv_create_int4(m, B, B * ((ctx + K + 16) // 16))
    w = cfg["n_kv_heads"] * cfg["head_dim"]
    rng = np.random.default_rng(3)
    lens = ctx - rng.integers(0, 60, B)
    for l in range(cfg["n_layers"]):
        for b in range(B):
            L.kv_import(kv, b, l, 0, bf(rng.standard_normal((lens[b], w))), bf(rng.standard_normal((lens[b], w))))
    ids, text = dev_i32(range(B)), rng.integers(0, cfg["vocab"], (B, K + 1))
    held = lambda: [t for l in range(cfg["n_layers"]) for b in range(B) for t in L.kv_export(kv, b, l, int(lens[b]), K + 1)]
    L.kv_set_len(kv, range(B), lens)
    full = L.verify_step(m, kv, ids, dev_i32(text), dev_i32([K + 1] * B))
    cached = held()
    rows = np.full((B, K + 1), -1, np.int32)
    for i in range(K + 1):
        rows[:, 0] = text[:, i]
        L.kv_set_len(kv, range(B), lens + i)
        alone = L.verify_step(m, kv, ids, dev_i32(rows), dev_i32([1] * B))
        assert torch.equal(alone[:, 0], full[:, i]), i
    L.check(m)
    assert all(torch.equal(x, y) for x, y in zip(held(), cached))


@pytest.mark.parametrize("seed", range(6))
def test_strict_decoding_is_greedy_decoding(L, seed):
    cfg = synth.model_cfg("tiny")
    W = synth.make_weights(cfg, seed=seed)
    m = L.model_create(cfg, weights_to(W, "cuda"), max_batch=5)
    kv = L.kv_create_int4(m, 5, 5 * 40)
    prompts = [synth.make_prompt(n, cfg["vocab"], 100 * seed + n) for n in (64, 5, 130, 33, 300)]
    plain = L.generate(m, kv, None, prompts, [0] * 5, L.make_params(K=8, max_new=200))["out"]
    rng, docs = np.random.default_rng(seed), []
    for p, o in zip(prompts, plain):
        o = np.array(o)
        o[rng.random(len(o)) < 0.15] = 7
        docs.append([list(map(int, p)) + o.tolist()])
    pool, offs = synth.pool_from_documents(docs)
    h = L.pool_build(pool, offs, 1, 3)
    for fused in (0, 1):
        prm = L.make_params(K=8, n_min=1, n_max=3, max_occ=64, max_new=200, fused_accept=fused)
        spec = L.generate(m, kv, h, prompts, range(5), prm)
        assert spec["out"] == plain and spec["accepted"] > 200
