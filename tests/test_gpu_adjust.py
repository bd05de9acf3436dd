"""laser_adjust_logits against the oracle in 64 bits.

A logit passes through at most five fp32 operations, each off by 2^-24 of its result; none of them is larger than
the sum of the magnitudes that enter, so the result is off by at most 5 x 2^-24 of that sum (times the penalty's factor)."""
import numpy as np
import pytest
import torch

from helpers import dev_i32, ensure_built, weights_to
from oracle import accept as A
from oracle import adjust as J
from paper_2408_05676_b200 import synth
from test_gpu_tree import random_tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    ensure_built()
    from paper_2408_05676_b200 import binding
    return binding


def f32(x):
    return torch.as_tensor(np.asarray(x, np.float32), device="cuda")


def pack(bits, pad=0):
    """[.., V] truth values -> int32 words of 32 tokens, `pad` words more a row."""
    V = bits.shape[-1]
    words = np.zeros(bits.shape[:-1] + (-(-V // 32) + pad,), np.uint32)
    for v in range(V):
        words[..., v // 32] |= bits[..., v].astype(np.uint32) << np.uint32(v % 32)
    return torch.as_tensor(words.view(np.int32), device="cuda")


CASES = [  # B, rows, V, history, biases, mask, tree
    (1, 1, 1, 3, 0, None, False),
    (1, 1, 31, 0, 2, "seq", False),
    (2, 3, 33, 40, 5, "row", False),
    (3, 9, 4096, 200, 64, "row", False),
    (2, 64, 2049, 700, 300, "row", False),
    (2, 64, 513, 90, 3, "seq", True),
    (5, 17, 1000, 1500, 700, None, True),
    (70, 4, 5003, 300, 20, "row", True),              # (enough rows for the wider runs)
    (80, 2, 4096, 10, 300, "seq", False),
    (70, 4, 5004, 300, 20, "row", True),              # (rows that begin on 16 bytes, and end inside a run)
    (52, 17, 6148, 900, 100, "row", False),
    (148, 5, 4, 20, 3, "row", False),
]


@pytest.mark.parametrize("B,R,V,hist,nb,mask,tree", CASES)
def test_matches_the_oracle(L, B, R, V, hist, nb, mask, tree):
    rng = np.random.default_rng(B * 1000 + V)
    x = rng.standard_normal((B, R, V)).astype(np.float32) * 3
    n = rng.integers(0, R + 1, B)
    n[0] = R
    text = (rng.zipf(1.3, (B, max(hist, 1))) - 1) % (V + V // 8 + 1) - 1          # some ids are -1, or behind the vocabulary
    hl = rng.integers(0, hist + 1, B)
    hl[0] = hist
    pl = np.array([rng.integers(0, h + 2) for h in hl])
    tokens = (rng.zipf(1.3, (B, R)) - 1) % (V + 2)
    rep, freq, pres = 1 + rng.random(B), rng.random(B) - 0.3, rng.random(B) - 0.3
    counts = rng.integers(0, nb + 1, B) if nb else np.zeros(B, int)
    off = np.concatenate([[0], np.cumsum(counts)])
    ids = rng.integers(-1, V + 1, off[-1] + 1)
    ids[1::3] = ids[0]                                                           # the same token several times
    val = rng.standard_normal(off[-1] + 1).astype(np.float32)
    allowed = rng.random((B, R if mask == "row" else 1, V)) < 0.6 if mask else None
    if mask:
        allowed[0, 0] = False                                                    # a row of which nothing is left
        x[0, 0, 0] = np.nan
    par = None
    if tree:
        par = np.full((B, R), -1, np.int32)
        for b in range(B):
            par[b, 1:n[b]] = random_tree(rng, n[b] - 1) if n[b] else []
    out = torch.full((B, R, V), 11.0, device="cuda")
    f = lambda a: f32(a)
    d = dict(hist=dev_i32(text), hist_len=dev_i32(hl), prompt_len=dev_i32(pl), penalties=(f(rep), f(freq), f(pres)),
             bias=(dev_i32(off), dev_i32(ids), f(val)) if nb else None, allowed=pack(allowed, pad=2) if mask else None,
             parents=dev_i32(par) if tree else None)
    t = f32(x)
    assert L.adjust_logits(t, dev_i32(tokens), dev_i32(n), out=out, **d) is out
    got = out.double().cpu().numpy()
    same = t.clone()
    L.adjust_logits(same, dev_i32(tokens), dev_i32(n), out=same, **d)            # in place
    for b in range(B):
        assert (got[b, n[b]:] == 11).all()
        if n[b] == 0:
            continue
        on = None if allowed is None else np.broadcast_to(allowed[b], (R, V))[:n[b]]
        bias = [(int(ids[j]), float(val[j])) for j in range(off[b], off[b + 1])] if nb else []
        r32, f_32, p32 = float(np.float32(rep[b])), float(np.float32(freq[b])), float(np.float32(pres[b]))
        txt = text[b, :hl[b]] if hist else []
        want = J.adjust_sequence(x[b], tokens[b], n[b], txt, pl[b], r32, f_32, p32, bias, on, None if par is None else par[b])
        fin = np.isfinite(want)
        assert (np.isneginf(got[b, :n[b]]) == ~fin).all()
        most = np.bincount(np.clip(np.concatenate([np.asarray(txt, int), tokens[b]]), 0, V)).max()
        room = 5 * 2.0 ** -24 * (r32 * np.abs(np.nan_to_num(x[b, :n[b]])) + abs(f_32) * most + abs(p32) + sum(abs(v) for _, v in bias))
        assert (np.abs(got[b, :n[b]][fin] - want[fin]) <= room[fin]).all()
        assert torch.equal(same[b, :n[b]], out[b, :n[b]]) and torch.equal(same[b, n[b]:].isnan(), t[b, n[b]:].isnan())


def test_alignment_does_not_change_a_bit(L):
    """Rows on 16 bytes take another kernel than rows that are not: logits, result or both shifted by one to three numbers."""
    rng = np.random.default_rng(5)
    B, R, V = 50, 6, 6004
    x = f32(rng.standard_normal((B, R, V)))
    tok, n = dev_i32(rng.integers(0, V, (B, R))), dev_i32(rng.integers(0, R + 1, B))
    args = dict(hist=dev_i32(rng.integers(0, V, (B, 300))), hist_len=dev_i32([300] * B), prompt_len=dev_i32([100] * B),
                penalties=tuple(f32(rng.random(B) + 0.5) for _ in range(3)), allowed=pack(rng.random((B, R, V)) < 0.5))
    want = L.adjust_logits(x, tok, n, out=torch.zeros_like(x), **args)

    def shifted(by, values):
        t = torch.zeros(B * R * V + 4, device="cuda")[by:by + B * R * V].view(B, R, V)
        return t.copy_(values)

    for i, o in ((1, 0), (0, 1), (2, 2), (3, 1), (0, 0)):
        out = shifted(o, torch.zeros_like(x))
        assert torch.equal(L.adjust_logits(shifted(i, x), tok, n, out=out, **args), want), (i, o)


def test_infinities_nan_and_nothing_asked_for(L):
    x = f32([[[np.inf, -np.inf, np.nan, 0.0, -0.0, 3.4e38, -3.4e38, 1.0]]])
    tok, n = dev_i32([[0]]), dev_i32([1])
    assert torch.equal(L.adjust_logits(x, tok, n).nan_to_num(nan=7), x.nan_to_num(nan=7))
    # masked places keep nothing of what was there
    y = L.adjust_logits(x, tok, n, allowed=dev_i32([[[0b11000000]]]), bias=(dev_i32([0, 3]), dev_i32([0, 1, 2]), f32([np.inf, np.inf, np.nan])))
    assert torch.isneginf(y[0, 0, :6]).all() and torch.equal(y[0, 0, 6:], x[0, 0, 6:])
    z = L.adjust_logits(x, tok, n, hist=dev_i32([range(8)]), hist_len=dev_i32([8]), prompt_len=dev_i32([8]), penalties=(f32([2.0]), None, None))
    assert z[0, 0, 0] == np.inf and z[0, 0, 1] == -np.inf and z[0, 0, 2].isnan() and z[0, 0, 5] == f32(3.4e38) / 2 and z[0, 0, 6] == -np.inf and z[0, 0, 7] == 0.5


def test_rows_beyond_32_bits_of_bytes(L):
    B, R, V = 18, 64, 1000000                                   # 4.6 GB
    x = torch.zeros(B, R, V, device="cuda")
    n = np.zeros(B, int)
    n[B - 1] = R
    tok = np.full((B, R), 5, np.int32)
    L.adjust_logits(x, dev_i32(tok), dev_i32(n), penalties=(None, torch.ones(B, device="cuda"), None), out=x)
    got = x[B - 1, :, 5].cpu().numpy()
    assert (got == -np.arange(R)).all() and float(x.abs().sum()) == R * (R - 1) / 2


def test_the_order_of_a_tokens_biases_is_the_lists(L):
    """1e8 + 1 - 1e8: in fp32 the order decides; every run gives the list's."""
    V, x = 3000, torch.zeros(2, 1, 3000, device="cuda")
    vals, want = [], []
    rng = np.random.default_rng(0)
    ids = []
    for b in range(2):
        i = rng.integers(0, 4, 600) * 700
        v = rng.choice([1e8, -1e8, 1.0, 3.0], 600).astype(np.float32)
        acc = np.zeros(V, np.float32)
        for a, c in zip(i, v):
            acc[a] += c
        ids.append(i), vals.append(v), want.append(acc)
    args = dict(bias=(dev_i32([0, 600, 1200]), dev_i32(np.concatenate(ids)), f32(np.concatenate(vals))))
    for _ in range(5):
        got = L.adjust_logits(x, dev_i32([[0], [0]]), dev_i32([1, 1]), **args)
        assert (got[:, 0].cpu().numpy() == np.stack(want)).all()


def test_in_a_graph_and_on_another_stream(L):
    rng = np.random.default_rng(1)
    x = f32(rng.standard_normal((2, 3, 900)))
    tok, n, hist, hl = dev_i32(rng.integers(0, 900, (2, 3))), dev_i32([3, 2]), dev_i32(rng.integers(0, 900, (2, 50))), dev_i32([50, 20])
    pen = tuple(f32(rng.random(2) + 0.5) for _ in range(3))
    out = torch.zeros_like(x)
    call = lambda: L.adjust_logits(x, tok, n, hist=hist, hist_len=hl, penalties=pen, out=out)
    want = call().clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out.zero_()
        call()
    s.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    hl.copy_(dev_i32([0, 50]))
    g.replay()
    got = out.clone()
    assert torch.equal(got, call()) and not torch.equal(got, want)


def test_a_constrained_generation(L):
    """Verify over a 4-bit cache, adjust, accept, commit: only what the grammar allows is emitted, and nothing twice in a row under
    a strong penalty; every verdict is the oracle's on the adjusted logits."""
    cfg = synth.model_cfg("tiny")
    K, V, B = cfg["max_draft"], cfg["vocab"], 3
    m = L.model_create(cfg, weights_to(synth.make_weights(cfg, seed=0), "cuda"), max_batch=B)
    kv = L.kv_create_int4(m, B, B * 8)
    rng = np.random.default_rng(2)
    ids, prm = dev_i32(range(B)), L.make_params(K=K)
    grammar = rng.random((B, 1, V)) < 0.05
    words = pack(grammar)
    text = torch.zeros(B, 100, dtype=torch.int32, device="cuda")
    text[:, 0] = dev_i32(rng.integers(0, V, B))
    n_text = np.ones(B, int)
    emitted = [[] for _ in range(B)]
    for step in range(6):
        last = text[torch.arange(B), torch.as_tensor(n_text - 1)]
        # drafts: tokens that the grammar allows, and one that it does not
        d = np.stack([rng.choice(np.flatnonzero(grammar[b, 0]), K) for b in range(B)])
        d[:, 3] = [int(np.flatnonzero(~grammar[b, 0])[0]) for b in range(B)]
        tokens, n = L.make_rows(last.contiguous(), dev_i32(d), dev_i32([K, 2, 0]), K)
        logits = L.verify_step(m, kv, ids, tokens, n)
        L.adjust_logits(logits, tokens, n, hist=text, hist_len=dev_i32(n_text), prompt_len=dev_i32([1] * B),
                        penalties=(None, None, torch.full((B,), 50.0, device="cuda")), allowed=words, out=logits)
        got = L.accept_commit(kv, ids, logits, tokens, n, prm)
        want = A.accept_batch(logits.cpu().numpy(), tokens.cpu().numpy(), n.cpu().numpy(), A.STRICT)
        for g, w in zip(got, want):
            assert (g.cpu().numpy() == w).all()
        for b in range(B):
            for t in want[1][b][:want[2][b]]:
                text[b, n_text[b]] = int(t)
                n_text[b] += 1
                emitted[b].append(int(t))
    L.check(m)
    for b in range(B):
        assert len(emitted[b]) >= 6 and all(grammar[b, 0, t] for t in emitted[b]) and len(set(emitted[b])) == len(emitted[b])
    assert (L.kv_get_len(kv, range(B)) == n_text - 1).all()
