"""The 4-bit cache: rows appended to it (laser_kv_append), attention over it (laser_attend_int4), copies in and out, and the verify
forward and the generation loop on it, against the oracle in 64 bits.

Tolerances.  A bf16 result is off by at most half a step, 2^-8 relative (HALF).  Held keys and values are exact but where a code lies at
a border: rotation in fp32 is off by a few 2^-24 of the pair's length, so a code may be the neighbour (one step s) where the quotient is
that close to a half; such places are counted, at most 1 in 10^4.  Attention: probabilities enter the second product as bf16, in the
numerator and in the sum, so a row is off by at most 2^-8 of the mean distance of the values from the result (times 1 + 2^-7), plus the
result's own rounding; products of bf16 numbers are exact in fp32, their sums over head_dim features and the exponent are good to 2^-16
of that distance for scores below 100."""
import numpy as np
import pytest
import torch

from helpers import dev_i32, ensure_built, weights_to
from oracle import forward as O
from oracle import int4 as Q
from paper_2408_05676_b200 import synth
from test_gpu_tree import random_tree

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def L():
    ensure_built()
    from paper_2408_05676_b200 import binding
    return binding


def make(L, heads, kv_heads, dim, slots, pages, layers=1, seed=0, int4=True):
    cfg = synth.model_cfg("tiny", n_layers=layers, d_model=64, d_ffn=64, vocab=64, n_heads=heads, n_kv_heads=kv_heads, head_dim=dim)
    m = L.model_create(cfg, weights_to(synth.make_weights(cfg, seed=0), "cuda"), max_batch=1)
    kv = (L.kv_create_int4 if int4 else L.kv_create)(m, slots, slots * pages)
    L.kv_set_page_table(kv, np.random.default_rng(seed).permutation(slots * pages).astype(np.int32))
    return kv


def bf(x):
    return torch.as_tensor(np.asarray(x, np.float32), device="cuda").to(torch.bfloat16)


def f64(t):
    return t.double().cpu().numpy()


def held_rows(L, kv, slot, pos0, n, layer=0):
    cfg = kv.model.cfg
    k, v = L.kv_export(kv, slot, layer, pos0, n)
    return [f64(t).reshape(n, cfg["n_kv_heads"], cfg["head_dim"]) for t in (k, v)]


# ---- the format --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dim,kv_heads", [(128, 3), (64, 5)])
def test_import_then_export_is_the_format(L, dim, kv_heads):
    kv = make(L, kv_heads, kv_heads, dim, 2, 4, layers=2)
    rng = np.random.default_rng(1)
    n = 50
    x = rng.standard_normal((2, n, kv_heads, dim)) * 10.0 ** rng.integers(-3, 4, (2, n, kv_heads, 1))
    x[:, :8] += 100
    x[:, 8:16, :, 5] *= 50
    x[:, 16] = 0
    x[:, 17] = 7
    x[:, 18, :, ::2] = 1e-35
    x[:, 19] *= 1e30
    x[0, 20, 0, 3], x[1, 21, 0, 40], x[0, 22, 1, 41] = np.nan, np.inf, -np.inf
    t = bf(x)
    for layer, pos0 in ((0, 0), (1, 13)):
        L.kv_import(kv, 1, layer, pos0, t[0].reshape(n, -1), t[1].reshape(n, -1))
        got = held_rows(L, kv, 1, pos0, n, layer)
        for y in range(2):
            want = Q.held(t[y].float().cpu().numpy())
            assert np.isfinite(got[y]).all() and (got[y] == want).all()
    # one token over another, and its neighbours stay
    L.kv_import(kv, 1, 0, 9, t[0, 30:31].reshape(1, -1), t[1, 30:31].reshape(1, -1))
    again = held_rows(L, kv, 1, 0, n)
    for y in range(2):
        want = Q.held(t[y].float().cpu().numpy())
        want[9] = want[30]
        assert (again[y] == want).all()


# ---- append ------------------------------------------------------------------------------------------------------

APPEND = [  # heads, kv heads, head_dim, lens, n_rows, rows, tree, dtype, int4
    (4, 4, 64, [0], [1], 1, False, "bf16", True),
    (4, 1, 64, [5, 30, 0], [3, 0, 2], 3, False, "f32", True),
    (5, 5, 64, [15, 16, 17], [4, 4, 1], 4, False, "bf16", True),          # (a warp holds two heads of 64: an odd number of them)
    (32, 8, 128, [100, 7], [9, 5], 9, False, "bf16", True),
    (6, 2, 128, [20, 0, 3], [17, 12, 1], 17, True, "f32", True),
    (4, 2, 64, [1, 2], [64, 40], 64, True, "bf16", True),
    (8, 2, 128, [0, 3], [150, 33], 150, False, "f32", True),              # a prompt
    (4, 2, 128, [9, 40], [9, 4], 9, True, "bf16", False),                 # bf16 caches take rows as well
    (4, 4, 64, [0, 33], [5, 2], 5, False, "f32", False),
]


@pytest.mark.parametrize("heads,kv_heads,dim,lens,n_rows,rows,tree,dtype,int4", APPEND)
def test_append_matches_the_oracle(L, heads, kv_heads, dim, lens, n_rows, rows, tree, dtype, int4):
    rng = np.random.default_rng(3)
    B, pages = len(lens), 16
    kv = make(L, heads, kv_heads, dim, B + 1, pages, int4=int4)
    slots = rng.permutation(B + 1)[:B]
    L.kv_set_len(kv, slots, lens)
    width = (heads + 2 * kv_heads) * dim
    x = torch.as_tensor(rng.standard_normal((B, rows, width + 8)), device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    for b in range(B):
        x[b, n_rows[b]:] = float("nan")                   # rows that are not active are not read
    q, k, v = x[..., 4:4 + heads * dim], x[..., 4 + heads * dim:4 + (heads + kv_heads) * dim], x[..., 4 + (heads + kv_heads) * dim:4 + width]
    par = None
    if tree:
        par = np.full((B, rows), -1, np.int32)
        for b in range(B):
            par[b, 1:n_rows[b]] = random_tree(rng, n_rows[b] - 1) if n_rows[b] else []
    fill = lambda h: torch.full((B, rows, h, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    qo, ko, vo = fill(heads), fill(kv_heads), fill(kv_heads)
    before = [held_rows(L, kv, s, 0, pages * 16) for s in range(B + 1)]
    got = L.kv_append(kv, 0, dev_i32(slots), dev_i32(n_rows), k, v, q=q, parents=None if par is None else dev_i32(par), q_out=qo, k_out=ko, v_out=vo)
    L.kv_check(kv)
    assert got is qo and (L.kv_get_len(kv, slots) == lens).all()
    flips = total = 0
    x64 = f64(x)[..., 4:4 + width].reshape(B, rows, heads + 2 * kv_heads, dim)
    for b in range(B):
        n = n_rows[b]
        assert (f64(qo)[b, n:] == 7).all() and (f64(ko)[b, n:] == 7).all() and (f64(vo)[b, n:] == 7).all()
        depth = [len(p) - 1 for p in Q.paths(n, None if par is None else par[b])]
        rows_k, rows_v = held_rows(L, kv, slots[b], lens[b], n) if n else (np.zeros((0, kv_heads, dim)),) * 2
        assert (rows_k == f64(ko)[b, :n]).all() and (rows_v == f64(vo)[b, :n]).all()
        for i in range(n):
            y = np.concatenate([Q.rotate(x64[b, i, :heads + kv_heads], lens[b] + depth[i], 10000.0), x64[b, i, heads + kv_heads:]])
            pair = np.hypot(x64[b, i, :, :dim // 2], x64[b, i, :, dim // 2:])
            room = 2.0 ** -21 * np.concatenate([pair, pair], -1)                 # of the rotation in fp32
            assert (np.abs(f64(qo)[b, i] - y[:heads]) <= HALF * np.abs(y[:heads]) + room[:heads]).all()
            for out, want, r in ((rows_k[i], y[heads:heads + kv_heads], room[heads:heads + kv_heads]), (rows_v[i], y[heads + kv_heads:], 0)):
                if int4:
                    off = np.abs(out - Q.held(want.astype(np.float32)))
                    _, s, _ = Q.quantise(want.astype(np.float32))
                    assert (off <= 1.01 * np.repeat(s, 32, -1) + 2 * HALF * np.abs(want).max()).all()
                    flips += int((off > 0).sum())
                    total += off.size
                else:
                    assert (np.abs(out - want) <= HALF * np.abs(want) + r).all()
        # nothing else of the cache changed
        after = held_rows(L, kv, slots[b], 0, pages * 16)
        for y in range(2):
            keep = np.ones(pages * 16, bool)
            keep[lens[b]:lens[b] + n] = False
            assert (after[y][keep] == before[slots[b]][y][keep]).all()
    assert flips <= max(1, total // 10000), (flips, total)


def test_codes_of_values_at_borders_and_a_few_ulps_apart(L):
    """fp32 values are stored to the bit as the oracle has it: halfway between two codes and next to that, ranges of a few of the values'
    last places (the zero is then far from them, in steps), tiny steps, the largest magnitudes."""
    rng = np.random.default_rng(17)
    n, dim = 240, 128
    kv = make(L, 1, 1, dim, 1, 16)
    x = np.zeros((n, dim), np.float32)
    for i in range(n):
        kind, g = i % 6, rng.integers(0, 16, dim).astype(np.float64)
        g[::32], g[1::32] = 0, 15
        step = 2.0 ** int(rng.integers(-90, 100))
        if kind < 2:                                         # c + 1/2, and a last place beside it
            v = ((g + 0.5 * (g % 15 != 0)) * step).astype(np.float32)
            x[i] = v if kind == 0 else np.nextafter(v, np.float32(rng.choice([-1, 1]) * np.inf), dtype=np.float32)
        elif kind == 2:                                      # a few last places of a large number
            x[i] = (np.float32(step) * np.float32(rng.uniform(1, 2))).view(np.uint32).__add__(rng.integers(0, rng.choice([2, 3, 40, 5000]), dim)).astype(np.uint32).view(np.float32)
        elif kind == 3:                                      # steps near the least one
            x[i] = (rng.uniform(-8, 8, dim) * 2.0 ** -100 * 2.0 ** rng.integers(-3, 3)).astype(np.float32)
        elif kind == 4:
            x[i] = np.clip(rng.standard_normal(dim) * 2.0 ** 125, -3.4e38, 3.4e38).astype(np.float32)
        else:
            x[i] = (rng.standard_normal(dim) * 1e-3 + rng.choice([-1, 1]) * 10.0 ** rng.integers(0, 6)).astype(np.float32)
    t = torch.as_tensor(x, device="cuda").view(1, n, dim)
    vo = torch.empty(1, n, 1, dim, dtype=torch.bfloat16, device="cuda")
    L.kv_append(kv, 0, dev_i32([0]), dev_i32([n]), t, t, v_out=vo)
    L.kv_check(kv)
    want = Q.held(x)
    assert (f64(vo)[0, :, 0] == want).all()
    assert (held_rows(L, kv, 0, 0, n)[1][:, 0] == want).all()


def test_append_far_positions_and_unaligned_rows(L):
    """Angles of positions beyond 10^5 in 64 bits; rows whose alignment allows no wide loads give the same."""
    kv = make(L, 2, 1, 64, 1, 16384)
    L.kv_set_len(kv, [0], [200003])
    rng = np.random.default_rng(5)
    x = torch.as_tensor(rng.standard_normal((1, 4, 2 * 64 + 2 * 64)), device="cuda", dtype=torch.float32)
    odd = torch.zeros(4 * 259 + 1, dtype=torch.float32, device="cuda")[1:].view(1, 4, 259)
    odd[..., 1:257] = x
    outs = []
    for t, a in ((x, 0), (odd, 1)):
        q, k, v = (t[..., a + i:a + i + w] for i, w in ((0, 128), (128, 64), (192, 64)))
        ko = torch.empty(1, 4, 1, 64, dtype=torch.bfloat16, device="cuda")
        outs.append((L.kv_append(kv, 0, dev_i32([0]), dev_i32([4]), k, v, q=q, k_out=ko), ko))
    L.kv_check(kv)
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    got, x64 = f64(outs[0][0])[0], f64(x)[0, :, :128].reshape(4, 2, 64)
    for i in range(4):
        y = Q.rotate(x64[i], 200003 + i, 10000.0)
        assert (np.abs(got[i] - y) <= HALF * np.abs(y) + 2.0 ** -20 * 4).all()


def test_bad_rows_are_left_out_and_reported(L):
    kv = make(L, 4, 2, 64, 3, 2)
    L.kv_set_len(kv, [0, 1, 2], [30, 5, 32])
    x = torch.ones(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    q = torch.ones(3, 4, 4, 64, dtype=torch.bfloat16, device="cuda")
    before = [held_rows(L, kv, s, 0, 32) for s in range(3)]

    def calls(ids, n, status, parents=None, written=()):
        args = (dev_i32(ids), dev_i32(n))
        for attend in (False, True):
            if attend:
                out = torch.full_like(q, 5.0)
                L.attend_int4(kv, 0, *args, q, parents=parents, out=out)
                for b in range(3):
                    assert (f64(out)[b] == 5).all() == (b not in written or n[b] <= 0), b
            else:
                L.kv_append(kv, 0, *args, x, x, parents=parents)
            if status is None or (attend and parents is not None):
                L.kv_check(kv)
            else:
                with pytest.raises(L.LaserError) as e:
                    L.kv_check(kv)
                assert e.value.status == status
                L.kv_check(kv)                     # (reported once)
        after = [held_rows(L, kv, s, 0, 32) for s in range(3)]
        for s in range(3):
            n_s = n[ids.index(s)] if s in ids else 0
            if s in ids and ids.index(s) in written and n_s:
                continue
            assert all((a == b).all() for a, b in zip(after[s], before[s])), s

    calls([0, 1, 2], [4, 0, 0], -4)                # 30 + 4 > 32: nothing cached, no row of the result
    calls([2, 1, 0], [1, 0, 0], -4)
    calls([7, 1, 0], [2, 0, 0], -1)
    calls([-1, 0, 2], [1, 0, 0], -1)
    calls([1, 0, 2], [4, 5, 0], -4, written=(0,))  # (5 rows of 4: taken as 4, which do not fit)
    calls([1, 0, 2], [4, -3, 0], None, written=(0,))
    calls([1, 0, 2], [4, 0, 0], -1, parents=dev_i32([[-1, 0, 3, 1], [-1] * 4, [-1] * 4]), written=(0,))


# ---- attention ---------------------------------------------------------------------------------------------------

def fill(L, kv, slots, totals, rng, scale=1.0):
    """Random keys and values in the cache; returns what it holds."""
    cfg = kv.model.cfg
    w = cfg["n_kv_heads"] * cfg["head_dim"]
    out = []
    for s, n in zip(slots, totals):
        if n:
            L.kv_import(kv, int(s), 0, 0, bf(rng.standard_normal((n, w)) * scale), bf(rng.standard_normal((n, w)) + 0.5))
            out.append(held_rows(L, kv, int(s), 0, n))
        else:
            out.append([np.zeros((0, cfg["n_kv_heads"], cfg["head_dim"]))] * 2)
    return out


def check_rows(got, q, held, lens, n_rows, par, scores=100.0):
    for b in range(len(lens)):
        n = n_rows[b]
        if n == 0:
            continue
        want, spread = Q.attend(q[b, :n], *held[b], lens[b], Q.paths(n, None if par is None else par[b]))
        tol = HALF * (1 + 2.0 ** -7) * spread + 2.0 ** -16 * (spread + np.abs(want)) * scores / 100 + HALF * np.abs(want) + 2.0 ** -24
        assert (np.abs(got[b, :n] - want) <= tol).all(), (b, float((np.abs(got[b, :n] - want) / tol).max()))


ATTEND = [  # heads, kv heads, head_dim, lens, n_rows, rows, tree
    (4, 4, 64, [0], [1], 1, False),
    (4, 4, 128, [0, 1, 15, 16, 17], [1, 1, 1, 1, 1], 1, False),
    (8, 1, 128, [3, 200, 0, 31], [1, 1, 1, 0], 1, False),              # 8 rows of a tile that has 8
    (32, 8, 128, [700, 1, 64], [2, 1, 2], 2, False),
    (4, 4, 64, [100, 0, 37, 16, 5], [9, 4, 0, 1, 9], 9, False),
    (4, 4, 128, [513, 12], [9, 5], 9, False),
    (12, 4, 64, [47, 300], [7, 3], 7, False),                          # three heads a kv head: rows of 21
    (40, 40, 128, [33, 900], [17, 11], 17, True),
    (8, 2, 128, [20, 5, 130], [33, 64, 1], 64, True),
    (4, 1, 64, [0, 40], [64, 2], 64, True),
    (2, 2, 64, [0, 10], [300, 129], 300, False),                       # a prompt's rows
    (16, 1, 128, [5, 50], [3, 3], 3, False),                           # 16 heads a kv head
]


@pytest.mark.parametrize("heads,kv_heads,dim,lens,n_rows,rows,tree", ATTEND)
def test_attention_matches_the_oracle(L, heads, kv_heads, dim, lens, n_rows, rows, tree):
    rng = np.random.default_rng(7)
    B = len(lens)
    kv = make(L, heads, kv_heads, dim, B + 1, -(-(max(lens) + rows) // 16) + 1)
    slots = rng.permutation(B + 1)[:B]
    # what lies behind a sequence's rows is of any size, and is not seen
    fill(L, kv, slots, [l + n + 3 for l, n in zip(lens, n_rows)], rng, 1e30)
    held = fill(L, kv, slots, [l + n for l, n in zip(lens, n_rows)], rng)
    L.kv_set_len(kv, slots, lens)
    par = None
    if tree:
        par = np.full((B, rows), -1, np.int32)
        for b in range(B):
            par[b, 1:n_rows[b]] = random_tree(rng, n_rows[b] - 1)
    wide = torch.full((B, rows, heads * dim + 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    q = wide[..., 8:8 + heads * dim]
    for b in range(B):
        q[b, :n_rows[b]] = bf(rng.standard_normal((n_rows[b], heads * dim)))
    out = torch.full((B, rows, heads * dim + 6), 3.0, dtype=torch.bfloat16, device="cuda")
    L.attend_int4(kv, 0, dev_i32(slots), dev_i32(n_rows), q, parents=None if par is None else dev_i32(par), out=out[..., 2:2 + heads * dim])
    L.kv_check(kv)
    got = f64(out)
    assert (got[..., :2] == 3).all() and (got[..., 2 + heads * dim:] == 3).all()
    for b in range(B):
        assert (got[b, n_rows[b]:] == 3).all()
    shape = (B, rows, heads, dim)
    check_rows(got[..., 2:2 + heads * dim].reshape(shape), f64(q).reshape(shape), held, lens, n_rows, par)


@pytest.mark.parametrize("heads,kv_heads,dim,rows,lens", [(4, 1, 64, 1, [9000]), (8, 8, 128, 3, [4000, 17, 2500]), (2, 1, 128, 9, [5000, 5000]), (1, 1, 128, 1, [20000])])
def test_long_texts_are_shared_out_and_joined(L, heads, kv_heads, dim, rows, lens):
    rng = np.random.default_rng(8)
    B = len(lens)
    kv = make(L, heads, kv_heads, dim, B, -(-(max(lens) + rows) // 16))
    held = fill(L, kv, range(B), [l + rows for l in lens], rng, 2.0)
    L.kv_set_len(kv, range(B), lens)
    q = bf(rng.standard_normal((B, rows, heads, dim)))
    ids, n = dev_i32(range(B)), dev_i32([rows] * B)
    out = L.attend_int4(kv, 0, ids, n, q)
    L.kv_check(kv)
    check_rows(f64(out), f64(q), held, lens, [rows] * B, None)
    for _ in range(3):                                   # the same bits every time
        assert torch.equal(out, L.attend_int4(kv, 0, ids, n, q))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows", [8, 10, 16, 17, 24, 25, 32, 33, 40, 41])
def test_every_size_of_a_tile(L, dim, rows):
    """Tiles of 8 to 40 rows over texts of odd and even numbers of pages: some in many pieces, some of a page or two that share a warp's run."""
    rng = np.random.default_rng(100 + rows)
    lens = [3001, 3, 640, 17, 0, 1200, 31]
    B = len(lens)
    kv = make(L, 2, 2, dim, B, -(-(max(lens) + rows) // 16))
    held = fill(L, kv, range(B), [l + rows for l in lens], rng, 2.0)
    L.kv_set_len(kv, range(B), lens)
    n_rows = [rows, 1, rows, rows - 1, rows, 0, 2]
    q = bf(rng.standard_normal((B, rows, 2, dim)))
    out = torch.full_like(q, 7.0)
    L.attend_int4(kv, 0, dev_i32(range(B)), dev_i32(n_rows), q, out=out)
    L.kv_check(kv)
    check_rows(f64(out), f64(q), held, lens, n_rows, None)
    for b in range(B):
        assert (out[b, n_rows[b]:] == 7).all()


@pytest.mark.parametrize("rows,heads", [(9, 2), (1, 8), (9, 4)])
def test_the_most_sequences_with_heads_of_128(L, rows, heads):
    rng = np.random.default_rng(21)
    B = 1024
    kv = make(L, heads, 1, 128, B, 2)
    lens = np.where(np.arange(B) < 40, rng.integers(0, 33 - rows, B), 0)
    x = bf(rng.standard_normal((40 * 32, 128)))
    for i in range(40):
        L.kv_import(kv, i, 0, 0, x[32 * i:32 * i + 32], x[32 * i:32 * i + 32])
    L.kv_set_len_dev(kv, dev_i32(lens))
    q = bf(rng.standard_normal((B, rows, heads, 128)))
    out = torch.full_like(q, 2.0)
    L.attend_int4(kv, 0, dev_i32(range(B)), dev_i32([rows] * B), q, out=out)
    L.kv_check(kv)
    got = f64(out)
    held = [held_rows(L, kv, i, 0, int(lens[i]) + rows) for i in range(40)]
    check_rows(got[:40], f64(q)[:40], held, lens[:40].tolist(), [rows] * 40, None)
    assert (got[40:] == 0).all()      # (fresh pages hold zeros)


def test_a_text_does_not_depend_on_its_neighbours(L):
    """Alone, among others, in another order, with drafts behind it: results differ by no more than a bf16 step, and hardly ever."""
    rng = np.random.default_rng(9)
    lens = [700, 33, 1500, 5, 250, 64]
    kv = make(L, 8, 2, 128, 6, 100)
    fill(L, kv, range(6), [l + 9 for l in lens], rng)
    L.kv_set_len(kv, range(6), lens)
    q = bf(rng.standard_normal((6, 9, 8, 128)))
    full = f64(L.attend_int4(kv, 0, dev_i32(range(6)), dev_i32([9] * 6), q))
    order = [3, 5, 0, 1, 4, 2]
    other = f64(L.attend_int4(kv, 0, dev_i32(order), dev_i32([9] * 6), q[order].contiguous()))
    differ = 0
    for j, b in enumerate(order):
        alone = f64(L.attend_int4(kv, 0, dev_i32([b]), dev_i32([9]), q[b:b + 1].contiguous()))[0]
        first = f64(L.attend_int4(kv, 0, dev_i32([b]), dev_i32([1]), q[b:b + 1, :1].contiguous()))[0]
        for x, y in ((other[j], full[b]), (alone, full[b]), (first[0], full[b, 0])):
            assert (np.abs(x - y) <= 2 * HALF * np.abs(y) + 1e-6).all()
            differ += int((x != y).sum())
    assert differ <= 0.01 * 3 * full.size


def test_extreme_scores_and_values(L):
    """Scores of thousands, one key far above the others late in the text, equal keys, values at the format's ends."""
    rng = np.random.default_rng(10)
    kv = make(L, 2, 2, 128, 4, 20)
    n = 300
    k, v = rng.standard_normal((4, n, 256)), rng.standard_normal((4, n, 256))
    k[0] *= 300
    k[1, 250] *= 40
    k[2] = k[2, 0]
    k[3] = np.linspace(-30, 30, n)[:, None] * np.sign(rng.standard_normal(256))       # scores that rise all the way
    v[1] *= 1e30
    for s in range(4):
        L.kv_import(kv, s, 0, 0, bf(k[s]), bf(v[s]))
    held = [held_rows(L, kv, s, 0, n) for s in range(4)]
    L.kv_set_len(kv, range(4), [n - 2] * 4)
    q = bf(rng.standard_normal((4, 2, 2, 128)))
    out = f64(L.attend_int4(kv, 0, dev_i32(range(4)), dev_i32([2] * 4), q))
    assert np.isfinite(out).all()
    # (scores of up to 2^14 are good to 2^-24 of that in fp32, a thousandth; their weights to as much)
    top = max(float(np.abs(np.einsum("rhd,thd->rht", f64(q)[s], held[s][0])).max()) for s in range(4)) / np.sqrt(128)
    check_rows(out, f64(q), held, [n - 2] * 4, [2] * 4, None, scores=max(100.0, top))


def test_nan_in_one_sequence_stays_there(L):
    rng = np.random.default_rng(11)
    kv = make(L, 4, 2, 64, 2, 4)
    fill(L, kv, range(2), [40, 40], rng)
    L.kv_set_len(kv, range(2), [38, 38])
    q = bf(rng.standard_normal((2, 2, 4, 64)))
    good = L.attend_int4(kv, 0, dev_i32([0, 1]), dev_i32([2, 2]), q)
    bad = q.clone()
    bad[0, 1] = float("nan")
    out = L.attend_int4(kv, 0, dev_i32([0, 1]), dev_i32([2, 2]), bad)
    assert torch.equal(out[1], good[1]) and torch.equal(out[0, 0], good[0, 0]) and torch.isnan(out[0, 1]).all()


def test_offsets_beyond_32_bits(L):
    """A cache of more than 4 GB whose last pages are used."""
    kv = make(L, 64, 64, 128, 1, 30000)                   # 64 x 2560 bytes a page: 4.9 GB
    table = np.arange(30000)[::-1].astype(np.int32)
    L.kv_set_page_table(kv, table)
    rng = np.random.default_rng(12)
    held = fill(L, kv, [0], [70], rng)
    L.kv_set_len(kv, [0], [65])
    x = bf(rng.standard_normal((1, 5, 64 * 128)))
    vo = torch.empty(1, 5, 64, 128, dtype=torch.bfloat16, device="cuda")
    q = L.kv_append(kv, 0, dev_i32([0]), dev_i32([5]), x, x, q=x, v_out=vo)
    held = [held_rows(L, kv, 0, 0, 70)]
    assert (held[0][1][65:] == f64(vo)[0]).all()
    out = L.attend_int4(kv, 0, dev_i32([0]), dev_i32([5]), q)
    L.kv_check(kv)
    check_rows(f64(out), f64(q), held, [65], [5], None)


def test_many_sequences_in_a_call(L):
    rng = np.random.default_rng(13)
    kv = make(L, 1, 1, 64, 1024, 2)
    B = 1024
    lens = rng.integers(0, 31, B)
    n = rng.integers(0, 2, B)
    x = bf(rng.standard_normal((B * 32, 64)))
    for i in range(0, 64):
        L.kv_import(kv, i, 0, 0, x[32 * i:32 * i + 32], x[32 * i:32 * i + 32])
    L.kv_set_len_dev(kv, dev_i32(lens))
    q = bf(rng.standard_normal((B, 1, 1, 64)))
    out = torch.full_like(q, 2.0)
    L.attend_int4(kv, 0, dev_i32(range(B)), dev_i32(n), q, out=out)
    L.kv_check(kv)
    got = f64(out)
    held = [held_rows(L, kv, i, 0, int(lens[i]) + 1) for i in range(64)]
    check_rows(got[:64], f64(q)[:64], held, lens[:64].tolist(), n[:64].tolist(), None)
    assert (got[n == 0] == 2).all() and (got[64:][n[64:] == 1] == 0).all()      # (fresh pages hold zeros)
    with pytest.raises(L.LaserError) as e:
        L.attend_int4(kv, 0, dev_i32([0] * 1025), dev_i32([0] * 1025), torch.zeros(1025, 1, 1, 64, dtype=torch.bfloat16, device="cuda"))
    assert e.value.status == -4


def test_refusals(L):
    kv = make(L, 4, 2, 64, 1, 2)
    plain = make(L, 4, 2, 64, 1, 2, int4=False)
    q = torch.zeros(1, 65, 4, 64, dtype=torch.bfloat16, device="cuda")
    ids, n, par = dev_i32([0]), dev_i32([1]), torch.zeros(1, 65, dtype=torch.int32, device="cuda")

    def refused(status, f):
        with pytest.raises(L.LaserError) as e:
            f()
        assert e.value.status == status

    refused(-1, lambda: L.attend_int4(plain, 0, ids, n, q))
    refused(-1, lambda: L.attend_int4(kv, 1, ids, n, q))
    refused(-1, lambda: L.attend_int4(kv, -1, ids, n, q))
    refused(-1, lambda: L.attend_int4(kv, 0, ids, n, q, parents=par))                    # a tree of 65 rows
    shifted = torch.zeros(1, 2, 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    refused(-1, lambda: L.attend_int4(kv, 0, ids, n, shifted[..., 4:260]))               # rows not 16-byte aligned
    k = torch.zeros(1, 65, 128, dtype=torch.bfloat16, device="cuda")
    refused(-1, lambda: L.kv_append(kv, 0, ids, n, k, k, parents=par))
    refused(-1, lambda: L.kv_append(kv, 2, ids, n, k, k))
    refused(-1, lambda: L._chk(L.lib.laser_kv_append(kv.handle, 0, ids.data_ptr(), None, n.data_ptr(), 1, 1, 2, None, 0, k.data_ptr(), 128, k.data_ptr(), 128,
                                                     None, None, None, None)))
    refused(-1, lambda: L._chk(L.lib.laser_kv_append(kv.handle, 0, ids.data_ptr(), None, n.data_ptr(), 1, 1, 0, None, 0, k.data_ptr(), 127, k.data_ptr(), 128,
                                                     None, None, None, None)))
    cfg = synth.model_cfg("tiny", n_layers=1, d_model=64, d_ffn=64, vocab=64, n_heads=4, n_kv_heads=4, head_dim=32)
    W = weights_to(synth.make_weights(cfg, seed=0), "cuda")
    small = L.model_create(cfg, W, max_batch=1)
    refused(-6, lambda: L.kv_create_int4(small, 1, 1))
    refused(-6, lambda: L.kv_append(L.kv_create(small, 1, 1), 0, ids, n, k[:, :1], k[:, :1]))
    cfg = synth.model_cfg("tiny", precise=1)
    W = weights_to(synth.make_weights(cfg, seed=0), "cuda")
    precise = L.model_create(cfg, W, max_batch=1)
    refused(-6, lambda: L.kv_create_int4(precise, 1, 4))
    usual = L.model_create(dict(cfg, precise=0), W, max_batch=1)
    kv = L.kv_create_int4(usual, 1, 4)
    R = cfg["max_draft"] + 1
    refused(-6, lambda: L.verify_step(precise, kv, ids, torch.zeros(1, R, dtype=torch.int32, device="cuda"), n))
    for slots, pages in ((0, 4), (4, 3)):
        refused(-1, lambda: L.kv_create_int4(usual, slots, pages))


def test_more_work_than_32_bits_count_is_refused(L):
    kv = make(L, 1, 1, 64, 1, 16384)
    ids, n, x = dev_i32([0] * 160), dev_i32([0] * 160), torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    call = lambda B, rows: L.lib.laser_attend_int4(kv.handle, 0, ids.data_ptr(), None, n.data_ptr(), B, rows, x.data_ptr(), 64, x.data_ptr(), 64, None)
    assert call(160, 40 * 131071) == -4             # 160 x 131071 tiles x 16384 pages: 2.3e9 an SM
    assert call(1, 40 * 131073) == -4
    assert call(160, 1000) == 0                     # (no row is active)
    L.kv_check(kv)


# ---- together ----------------------------------------------------------------------------------------------------

def test_append_and_attend_on_another_stream_and_in_a_graph(L):
    rng = np.random.default_rng(14)
    kv = make(L, 8, 2, 128, 3, 20, layers=2)
    lens = [250, 3, 64]
    for layer in range(2):
        for s in range(3):
            L.kv_import(kv, s, layer, 0, bf(rng.standard_normal((lens[s], 256))), bf(rng.standard_normal((lens[s], 256))))
    L.kv_set_len(kv, range(3), lens)
    ids, n = dev_i32([2, 0, 1]), dev_i32([5, 9, 2])
    x = bf(rng.standard_normal((3, 9, 12 * 128)))
    y = bf(rng.standard_normal((3, 9, 12 * 128)))
    out = [torch.zeros(3, 9, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    qo = torch.zeros(3, 9, 8, 128, dtype=torch.bfloat16, device="cuda")
    inp = x.clone()

    def step():
        for layer in range(2):
            L.kv_append(kv, layer, ids, n, inp[..., 1024:1280], inp[..., 1280:], q=inp[..., :1024], q_out=qo)
            L.attend_int4(kv, layer, ids, n, qo, out=out[layer])

    want = []
    for src in (x, y):
        inp.copy_(src)
        step()
        want.append([t.clone() for t in out])
    assert not torch.equal(want[0][0], want[1][0])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        inp.copy_(x)
        for t in out:
            t.zero_()
        step()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for src, w in ((y, want[1]), (x, want[0]), (y, want[1])):
        inp.copy_(src)
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, w))
    L.kv_check(kv)


def forward64(W, cfg, held, lens, tokens, parents=None):
    """The decoder in fp64 whose attention takes the given keys and values (per layer and sequence: cached tokens, then the rows)."""
    H, dh, eps = cfg["n_heads"], cfg["head_dim"], cfg["rms_eps"]
    out, keys = [], []
    for b, toks in enumerate(tokens):
        paths = Q.paths(len(toks), None if parents is None else parents[b])
        x = W["tok_emb"][torch.as_tensor(toks, dtype=torch.int64)].double()
        pos = torch.tensor([lens[b] + len(p) - 1 for p in paths])
        for l, lw in enumerate(W["layers"]):
            h = O.rmsnorm(x, lw["attn_norm"].double(), eps)
            q = O.rope((h @ lw["wq"].double().T).view(-1, H, dh), pos, cfg["rope_theta"]).numpy()
            k = O.rope((h @ lw["wk"].double().T).view(-1, cfg["n_kv_heads"], dh), pos, cfg["rope_theta"]).numpy()
            keys.append((k, (h @ lw["wv"].double().T).view(-1, cfg["n_kv_heads"], dh).numpy()))
            a, _ = Q.attend(q, *held[l][b], lens[b], paths)
            x = x + torch.from_numpy(a.reshape(len(toks), -1)) @ lw["wo"].double().T
            h = O.rmsnorm(x, lw["ffn_norm"].double(), eps)
            g = h @ lw["w_gate"].double().T
            x = x + (g * torch.sigmoid(g) * (h @ lw["w_up"].double().T)) @ lw["w_down"].double().T
        out.append((O.rmsnorm(x, W["final_norm"].double(), eps) @ W["lm_head"].double().T).numpy())
    return out, keys


@pytest.mark.parametrize("over,tree", [(dict(), False), (dict(), True), (dict(n_heads=4, n_kv_heads=2, head_dim=128, d_model=512), False)])
def test_verify_step_on_a_4bit_cache(L, over, tree):
    """Logits against an exact forward that attends to what the cache holds, within the 2e-2 that bf16 operands take on this model;
    and what is held of the step's rows against their exact keys and values: a step of the format (two halves: their rounding, and
    the border that bf16 operands, 2^-6 of a row's largest, may push them over)."""
    cfg = synth.model_cfg("tiny", **over)
    W = synth.make_weights(cfg, seed=0, gain_jitter=0.1)
    B, R = 4, cfg["max_draft"] + 1
    m = L.model_create(cfg, weights_to(W, "cuda"), max_batch=B)
    kv = L.kv_create_int4(m, B, B * 12)
    rng = np.random.default_rng(4)
    L.kv_set_page_table(kv, rng.permutation(B * 12).astype(np.int32))
    lens, w = [150, 0, 37, 16], cfg["n_kv_heads"] * cfg["head_dim"]
    for b in range(B):
        for l in range(cfg["n_layers"]):
            if lens[b]:
                L.kv_import(kv, b, l, 0, bf(rng.standard_normal((lens[b], w))), bf(rng.standard_normal((lens[b], w))))
    L.kv_set_len(kv, range(B), lens)
    n = [R, 5, 1, 7]
    tokens, par = np.full((B, R), -1, np.int32), np.full((B, R), -1, np.int32)
    for b in range(B):
        tokens[b, :n[b]] = rng.integers(0, cfg["vocab"], n[b])
        par[b, 1:n[b]] = random_tree(rng, n[b] - 1) if tree else range(n[b] - 1)
    ids = dev_i32(range(B))
    if tree:
        logits = L.verify_step_tree(m, kv, ids, dev_i32(tokens), dev_i32(par), dev_i32(n))
    else:
        logits = L.verify_step(m, kv, ids, dev_i32(tokens), dev_i32(n))
    L.check(m)
    held = [[held_rows(L, kv, b, 0, lens[b] + n[b], l) for b in range(B)] for l in range(cfg["n_layers"])]
    want, keys = forward64(W, cfg, held, lens, [tokens[b, :n[b]] for b in range(B)], par)
    for b in range(B):
        assert np.abs(f64(logits)[b, :n[b]] - want[b]).max() <= 2e-2
        for l in range(cfg["n_layers"]):
            for y in range(2):
                x = keys[b * cfg["n_layers"] + l][y]
                _, s, _ = Q.quantise(x.astype(np.float32))
                room = 1.2 * np.repeat(s, 32, -1) + 2.0 ** -6 * np.abs(x).max()
                assert (np.abs(held[l][b][y][lens[b]:] - x) <= room).all()


def test_a_cache_serves_models_with_other_query_heads(L):
    """A cache is shaped by keys and values: whichever model made it, a step takes its heads from the model that runs."""
    cfgs = [synth.model_cfg("tiny", d_model=256, n_heads=h, n_kv_heads=2, head_dim=64) for h in (4, 10)]
    models = [L.model_create(c, weights_to(synth.make_weights(c, seed=7), "cuda"), max_batch=2) for c in cfgs]
    R = cfgs[0]["max_draft"] + 1
    rng = np.random.default_rng(23)
    tokens, n, ids = dev_i32(rng.integers(0, cfgs[0]["vocab"], (2, R))), dev_i32([R, 4]), dev_i32([0, 1])
    x = [bf(rng.standard_normal((40, 128))) for _ in range(2)]
    for m in models:
        got = []
        for maker in models:
            kv = L.kv_create_int4(maker, 2, 8)
            for l in range(cfgs[0]["n_layers"]):
                for b in range(2):
                    L.kv_import(kv, b, l, 0, x[0], x[1])
            L.kv_set_len(kv, [0, 1], [40, 23])
            logits = L.verify_step(m, kv, ids, tokens, n)
            L.check(m)
            got.append((logits[0], logits[1, :4], *held_rows(L, kv, 0, 0, 40 + R)))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert all((p == q).all() for p, q in zip(got[0][2:], got[1][2:])) and torch.isfinite(got[0][0]).all()


def test_tree_commit_moves_codes(L):
    """laser_kv_compact_path on a 4-bit cache: accepted rows move as they are, across pages, in every layer."""
    kv = make(L, 4, 2, 128, 3, 6, layers=2)
    rng = np.random.default_rng(6)
    for l in range(2):
        for s in range(3):
            L.kv_import(kv, s, l, 0, bf(rng.standard_normal((90, 256))), bf(rng.standard_normal((90, 256))))
    lens = [27, 0, 60]
    L.kv_set_len(kv, range(3), lens)
    before = [[held_rows(L, kv, s, 0, 90, l) for s in range(3)] for l in range(2)]
    path = np.full((3, 20), -1, np.int32)
    path[0, :4], path[2, :3] = [2, 5, 6, 19], [1, 2, 18]
    L.kv_compact_path(kv, dev_i32([0, 1, 2]), dev_i32(path), dev_i32([4, 0, 3]))
    for l in range(2):
        for s in range(3):
            want = [x.copy() for x in before[l][s]]
            for j, r in enumerate(path[s][path[s] >= 0]):
                for y in range(2):
                    want[y][lens[s] + j + 1] = before[l][s][y][lens[s] + r]
            after = held_rows(L, kv, s, 0, 90, l)
            for y in range(2):
                assert (after[y] == want[y]).all()


@pytest.mark.parametrize("form", ["chain", "tree", "fused"])
def test_generation_on_a_4bit_cache(L, form):
    """Drafts change nothing: the text is plain greedy decoding's on such a cache, prompts over several chunks."""
    cfg = synth.model_cfg("tiny")
    W = synth.make_weights(cfg, seed=0)
    m = L.model_create(cfg, weights_to(W, "cuda"), max_batch=4)
    kv = L.kv_create_int4(m, 4, 4 * 20)
    prompts = [synth.make_prompt(n, cfg["vocab"], 2000 + n) for n in (64, 5, 130, 33)]
    plain = L.generate(m, kv, None, prompts, [0] * 4, L.make_params(K=8, max_new=60))["out"]
    docs = []
    for p, o in zip(prompts, plain):
        o = list(o)
        o[10::11] = [7] * len(o[10::11])
        docs.append([list(map(int, p)) + o])
    pool, offs = synth.pool_from_documents(docs)
    h = L.pool_build(pool, offs, 1, 3)
    prm = L.make_params(K=8, n_min=1, n_max=3, max_occ=64, max_new=60, tree=int(form == "tree"), fused_accept=int(form == "fused"))
    spec = L.generate(m, kv, h, prompts, range(4), prm)
    assert spec["out"] == plain and spec["accepted"] > 60
