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


def test_values_are_rounded_once(L):
    """Where s (16 + c) is halfway between two bf16 numbers and the zero, far smaller, decides: what the call hands back, what an export
    gives and what attention reads are one number, the oracle's."""
    dim, rng = 128, np.random.default_rng(3)
    rows = []
    for e in range(-20, 21):
        for sign in (1, -1):
            x = np.full(dim, 32.625, np.float64)
            x += 1.125 * rng.integers(-11, 2, dim)
            x[::32], x[1::32] = 18 + sign * 2.0 ** -19, 34.875
            rows.append(x * 2.0 ** e)
    x = np.array(rows, np.float32)
    n = len(rows)
    want = Q.held(x)
    _, s, z = Q.quantise(x)
    assert ((np.abs(z) < s * 2.0 ** -15) & (z != 0)).any()
    kv = make(L, 1, 1, dim, n, 1)
    t = torch.as_tensor(x, device="cuda").view(n, 1, dim)
    ko, vo = (torch.empty(n, 1, 1, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids, one = dev_i32(range(n)), dev_i32([1] * n)
    L.kv_append(kv, 0, ids, one, t, t, k_out=ko, v_out=vo)
    L.kv_check(kv)
    assert (f64(vo)[:, 0, 0] == want).all() and (f64(ko)[:, 0, 0] == want).all()      # (position 0: no rotation)
    for i in range(n):
        assert all((a[0, 0] == want[i]).all() for a in held_rows(L, kv, i, 0, 1)), i
    q = torch.zeros(n, 1, 1, dim, dtype=torch.bfloat16, device="cuda")
    assert (f64(L.attend_int4(kv, 0, ids, one, q))[:, 0, 0] == want).all()            # (one token: its value)


@pytest.mark.parametrize("rows", [1, 9, 33])
@pytest.mark.parametrize("dim", [64, 128])
def test_scores_of_any_size(L, rows, dim):
    """All scores far below zero, up to the largest numbers that 32 bits hold; texts whose scores jump there and back.  Equal scores weigh
    the same, and what is far below a row's highest weighs nothing."""
    n = 75
    sizes = [-1e10, -1e22, -1e33, 1e10, 1e33, -3.0e37 / 2 ** 4, "low then normal", "normal then low", "high once"]
    kv = make(L, 2, 1, dim, len(sizes), 8)
    rng = np.random.default_rng(2)
    q = np.zeros((len(sizes), rows, 2, dim), np.float32)
    q[..., 0], q[..., 1] = 1, -1
    k, v = np.zeros((len(sizes), n, dim)), rng.standard_normal((len(sizes), n, dim))
    for s, size in enumerate(sizes):
        big = np.zeros(n)
        if isinstance(size, float):
            big[:] = size
        elif size == "high once":
            big[41] = 1e30
        else:
            big[(slice(0, 40) if size == "low then normal" else slice(40, n))] = -1e33
        k[s, :, 0] = big
        L.kv_import(kv, s, 0, 0, bf(k[s]), bf(v[s]))
    L.kv_set_len(kv, range(len(sizes)), [n - rows] * len(sizes))
    out = f64(L.attend_int4(kv, 0, dev_i32(range(len(sizes))), dev_i32([rows] * len(sizes)), torch.as_tensor(q, device="cuda").to(torch.bfloat16)))
    L.kv_check(kv)
    for s in range(len(sizes)):
        held_k, held_v = held_rows(L, kv, s, 0, n)
        want, spread = Q.attend(q[s].astype(np.float64), held_k, held_v, n - rows, Q.paths(rows))
        tol = HALF * (1 + 2.0 ** -7) * spread + 2.0 ** -16 * (spread + np.abs(want)) + HALF * np.abs(want) + 2.0 ** -24
        assert (np.abs(out[s] - want) <= tol).all(), sizes[s]


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


@pytest.mark.parametrize("int4", [False, True])
@pytest.mark.parametrize("ko,vo", [(1, 0), (0, 2), (3, 1)])
def test_copies_to_arrays_that_lie_anywhere(L, int4, ko, vo):
    """laser_kv_import and _export take arrays of any alignment that their type allows, on either form of the cache."""
    kv = make(L, 2, 2, 64, 1, 4, int4=int4)
    rng = np.random.default_rng(4)
    x = [bf(rng.standard_normal((40, 128))) for _ in range(2)]
    flat = [torch.zeros(40 * 128 + 8, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    at = [t[o:o + 40 * 128].view(40, 128) for t, o in zip(flat, (ko, vo, ko, vo))]
    L.kv_import(kv, 0, 0, 3, *x)
    want = L.kv_export(kv, 0, 0, 3, 40)
    for t, y in zip(at, x):
        t.copy_(y)
    L.kv_import(kv, 0, 0, 20, *at[:2])
    st = L.lib.laser_kv_export(kv.handle, 0, 0, 20, 40, C.c_void_p(at[2].data_ptr()), C.c_void_p(at[3].data_ptr()), C.c_void_p(0))
    assert st == 0, L.lib.laser_last_error()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(at[2:], want))
    for t, o in zip(flat[2:], (ko, vo)):
        assert (t[:o] == 0).all() and (t[o + 40 * 128:] == 0).all()


def test_the_profile_counts_every_launch_around_the_cache(L):
    """Class 1 of laser_profile_read: a layer's attention, and on a 4-bit cache the storing of the step's rows, which is a launch of its
    own there."""
    cfg = synth.model_cfg("tiny", n_layers=3)
    m = L.model_create(cfg, weights_to(synth.make_weights(cfg, seed=0), "cuda"), max_batch=2)
    ids, n = dev_i32([0, 1]), dev_i32([9, 9])
    tokens = dev_i32(np.zeros((2, 9)))
    for create, launches in ((L.kv_create, 3), (L.kv_create_int4, 6)):
        kv = create(m, 2, 4)
        L.profile_enable(m, True)
        L.profile_read(m, 0), L.profile_read(m, 1)
        L.verify_step(m, kv, ids, tokens, n)
        gemms, other = L.profile_read(m, 0), L.profile_read(m, 1)
        L.profile_enable(m, False)
        assert gemms[1] == 3 * 4 + 1 and other[1] == launches and gemms[0] > 0 and other[0] > 0
