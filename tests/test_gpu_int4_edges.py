"""The 4-bit cache where it can go wrong once more: sums that two roundings would move, scores beyond all others, passes of a prompt with
more chunks than a launch takes, arrays that lie anywhere, what the profile counts.  Against the oracle in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from helpers import dev_i32, ensure_built, weights_to
from oracle import int4 as Q
from paper_2408_05676_b200 import synth
from test_gpu_int4_cache import bf, f64, held_rows, make

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def L():
    ensure_built()
    from paper_2408_05676_b200 import binding
    return binding


def test_prompts_of_more_chunks_than_a_launch_takes(L):
    """A workspace that would take all chunks of the prompts in one pass; the text and the cache are those of a small workspace."""
    cfg = synth.model_cfg("tiny", n_layers=2, max_draft=63)
    W = weights_to(synth.make_weights(cfg, seed=0), "cuda")
    prompts = [synth.make_prompt(4000 + b, cfg["vocab"], b) for b in range(9)]
    w = cfg["n_kv_heads"] * cfg["head_dim"]
    got = []
    for max_batch in (9, 1024):
        m = L.model_create(cfg, W, max_batch=max_batch)
        kv = L.kv_create_int4(m, 9, 9 * 260)
        out = L.generate(m, kv, None, prompts, [0] * 9, L.make_params(K=63, max_new=2))["out"]
        assert all(len(o) == 2 for o in out)
        got.append([np.stack([f64(x) for b in range(9) for x in L.kv_export(kv, b, l, 0, 3999)]).reshape(9, 2, 3999, w) for l in range(2)])
    for l in range(2):
        a, b = got[0][l], got[1][l]
        # (equal projections of equal rows, but for sums in another order: at most a code here and there)
        assert np.isfinite(b).all() and (np.abs(a - b) > 0.5 * a.std()).mean() < 1e-3, l


def test_generation_of_more_sequences_than_a_step_takes_is_refused_at_once(L):
    cfg = synth.model_cfg("tiny", n_layers=1, max_draft=1)
    m = L.model_create(cfg, weights_to(synth.make_weights(cfg, seed=0), "cuda"), max_batch=1025)
    kv = L.kv_create_int4(m, 1025, 1025)
    L.kv_set_len(kv, range(1025), [5] * 1025)
    with pytest.raises(L.LaserError) as e:
        L.generate(m, kv, None, [np.array([1], np.int32)] * 1025, [0] * 1025, L.make_params(K=1, max_new=2))
    assert e.value.status == -4
    assert list(L.kv_get_len(kv, range(1025))) == [5] * 1025
