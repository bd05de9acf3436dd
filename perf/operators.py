"""What the operators around a verify step are measured on: the calls that a decoding program makes of them, and
their plain forms.

Three kinds of case:

    append    keys and values of a step's rows go to the 4-bit cache, queries and keys rotated on the way
    attend    attention of a step's rows over the 4-bit cache
    adjust    penalties, biases and grammar masks on the logits of a step, each row after the drafts on its path

The 4-bit cache holds, per token, head and group of 32 features, codes c of 0 .. 15 with a scale s and a zero z in
bf16; a code stands for the bf16 number nearest to s (16 + c) + z.
"""
import math

import torch

own = False
DEV = "cuda"
GROUP = 32
TOP = 2.0 ** 124       # what the cache stores lies within +-TOP
LEAST = 2.0 ** -100    # scales below it are zero


def listed():
    return [
        # one text of the smallest model, one token at a time: launch and latency
        dict(name="append-tiny-b1-decode", kind="append", heads=4, kv_heads=4, dim=64, batch=1, rows=1, ctx_lo=100, ctx_hi=100,
             tree=False, ragged=False, dtype="bf16"),
        # a layer of the headline step: 16 sequences of the 7B shape, a pending token and up to 8 drafts each
        dict(name="append-7b-b16-draft8", kind="append", heads=32, kv_heads=32, dim=128, batch=16, rows=9, ctx_lo=256, ctx_hi=768,
             tree=False, ragged=True, dtype="bf16"),
        # token trees of the scale-up shape, from the projections' fp32 sums
        dict(name="append-13b-b64-tree16", kind="append", heads=40, kv_heads=40, dim=128, batch=64, rows=17, ctx_lo=256, ctx_hi=1024,
             tree=True, ragged=True, dtype="fp32"),
        # prompts of up to 1024 tokens, grouped heads
        dict(name="append-gqa-b16-prompts", kind="append", heads=32, kv_heads=8, dim=128, batch=16, rows=1024, ctx_lo=0, ctx_hi=0,
             tree=False, ragged=True, dtype="bf16"),
        # one user waiting for one text: 9 rows against 512 tokens
        dict(name="attend-7b-b1-ctx512", kind="attend", heads=32, kv_heads=32, dim=128, batch=1, rows=9, ctx_lo=512, ctx_hi=512,
             tree=False, ragged=False),
        # a layer of the headline step over ragged contexts and draft lengths
        dict(name="attend-7b-b16-draft8", kind="attend", heads=32, kv_heads=32, dim=128, batch=16, rows=9, ctx_lo=256, ctx_hi=768,
             tree=False, ragged=True),
        # tree attention of the scale-up shape
        dict(name="attend-13b-b64-tree16", kind="attend", heads=40, kv_heads=40, dim=128, batch=64, rows=17, ctx_lo=256, ctx_hi=1024,
             tree=True, ragged=True),
        # single tokens of many long texts, grouped heads: the cache is all there is to read
        dict(name="attend-gqa-b64-ctx8k", kind="attend", heads=32, kv_heads=8, dim=128, batch=64, rows=1, ctx_lo=4096, ctx_hi=8192,
             tree=False, ragged=False),
        # drafts behind one very long text, grouped heads
        dict(name="attend-gqa-b1-ctx64k", kind="attend", heads=32, kv_heads=8, dim=128, batch=1, rows=9, ctx_lo=65536, ctx_hi=65536,
             tree=False, ragged=False),
        # one text, one row of logits
        dict(name="adjust-b1-decode", kind="adjust", batch=1, rows=1, vocab=32000, hist_lo=200, hist_hi=200, bias=16, mask="seq",
             tree=False, ragged=False),
        # the acceptance case's step: 64 sequences, up to 9 rows each, a grammar state per row
        dict(name="adjust-b64-draft8", kind="adjust", batch=64, rows=9, vocab=32000, hist_lo=256, hist_hi=768, bias=64, mask="row",
             tree=False, ragged=True),
        # token trees over a vocabulary whose rows are not aligned, long histories
        dict(name="adjust-b64-tree16-odd", kind="adjust", batch=64, rows=17, vocab=50257, hist_lo=512, hist_hi=2048, bias=300, mask="row",
             tree=True, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "adjust"])
    tree = rng.random() < 0.3
    ragged = rng.random() < 0.5
    if kind == "adjust":
        lo = _log_int(rng, 1, 1500)
        return dict(kind=kind, batch=_log_int(rng, 1, 64), rows=rng.randint(1, 17), vocab=rng.choice([4096, 32000, 32003, 50257, rng.randint(1000, 50000)]),
                    hist_lo=lo, hist_hi=lo + _log_int(rng, 1, 500), bias=_log_int(rng, 1, 300), mask=rng.choice(["none", "seq", "row"]),
                    tree=tree, ragged=ragged)
    heads, kv_heads, dim = rng.choice([(4, 4, 64), (4, 1, 64), (32, 32, 128), (32, 8, 128), (32, 4, 128), (40, 40, 128)])
    if kind == "append":
        prompts = rng.random() < 0.3
        lo = _log_int(rng, 1, 20000) - 1
        return dict(kind=kind, heads=heads, kv_heads=kv_heads, dim=dim, batch=_log_int(rng, 1, 12) if prompts else _log_int(rng, 1, 64),
                    rows=_log_int(rng, 65, 800) if prompts else rng.randint(1, 17), ctx_lo=lo, ctx_hi=lo + _log_int(rng, 1, 400),
                    tree=tree and not prompts, ragged=ragged, dtype=rng.choice(["bf16", "fp32"]))
    batch = _log_int(rng, 1, 64)
    rows = rng.choice([1, rng.randint(2, 17), rng.randint(2, 17)])
    most = max(2, min(65536, (64 * 8 * 128 * 6000) // (batch * kv_heads * dim * max(1, rows // 2))))   # the largest listed case's work
    hi = _log_int(rng, 2, most)
    return dict(kind=kind, heads=heads, kv_heads=kv_heads, dim=dim, batch=batch, rows=rows, ctx_lo=rng.randint(0, hi), ctx_hi=hi,
                tree=tree and rows > 2, ragged=ragged)


# ---- inputs -----------------------------------------------------------------------------------------------

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1009 + salt) & 0x7fffffff)
    return g


def _randint(g, lo, hi, shape):
    """int32 in lo .. hi."""
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV).to(torch.int32)


def _normal(g, *shape):
    return torch.empty(*shape, dtype=torch.float32, device=DEV).normal_(generator=g)


def _rows(case, g):
    """Rows of each sequence, and the parents of a token tree in depth-first order (or None)."""
    B, R = case["batch"], case["rows"]
    n = _randint(g, 1, R, (B,)) if case["ragged"] else torch.full((B,), R, dtype=torch.int32, device=DEV)
    if not case["tree"]:
        return n, None
    # a node continues the row before it, or the row before that one's parent was ..: up to three levels back
    par = torch.full((B, R), -1, dtype=torch.int64, device="cpu")
    up = torch.randint(0, 3, (B, R), generator=g, device=DEV).clamp_(min=0).cpu()
    for i in range(1, R):
        p = torch.full((B,), i - 1, dtype=torch.int64)
        for level in range(2):
            q = par.gather(1, p[:, None])[:, 0]
            p = torch.where((up[:, i] > level) & (q >= 0), q, p)
        par[:, i] = p
    return n, par.to(torch.int32).to(DEV)


def _keys_values(g, tokens, kv_heads, dim):
    """Keys and values of `tokens` tokens, bf16: a few features of the keys are larger than the others, as in trained models."""
    kv = torch.empty(2, tokens, kv_heads, dim, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    gain = 1 + 3 * (torch.rand(kv_heads, dim, generator=g, device=DEV) < 0.05)
    kv[0] *= gain.to(torch.bfloat16)
    return kv[0], kv[1]


def _cache(case, g, lens, slots, seed):
    """The library's 4-bit cache, one layer, its pages in no order."""
    from paper_2408_05676_b200 import binding as L
    B, R, H, Hkv, dh = (case[k] for k in ("batch", "rows", "heads", "kv_heads", "dim"))
    cfg = dict(n_layers=1, d_model=64, n_heads=H, n_kv_heads=Hkv, head_dim=dh, d_ffn=64, vocab=64, rms_eps=1e-5, rope_theta=10000.0,
               page_size=16, max_draft=min(R - 1, 63))
    w = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)
    layer = dict(wq=w(H * dh, 64), wk=w(Hkv * dh, 64), wv=w(Hkv * dh, 64), wo=w(64, H * dh), w_gate=w(64, 64), w_up=w(64, 64),
                 w_down=w(64, 64), attn_norm=w(64), ffn_norm=w(64))
    model = L.model_create(cfg, dict(tok_emb=w(64, 64), lm_head=w(64, 64), final_norm=w(64), layers=[layer]), max_batch=1)
    pages = -(-(case["ctx_hi"] + R) // 16)
    kv = L.kv_create_int4(model, B, B * pages)
    order = torch.randperm(B * pages, generator=torch.Generator().manual_seed(int(seed) & 0x7fffffff))
    L.kv_set_page_table(kv, order.to(torch.int32).numpy())
    by_slot = torch.zeros(B, dtype=torch.int32, device=DEV)
    by_slot[slots.long()] = lens
    L.kv_set_len_dev(kv, by_slot)
    return kv


def _prepare_append(case, seed):
    g = _gen(seed, 1)
    B, R, H, Hkv, dh = (case[k] for k in ("batch", "rows", "heads", "kv_heads", "dim"))
    n, par = _rows(case, g)
    lens = _randint(g, case["ctx_lo"], case["ctx_hi"], (B,))
    slots = torch.randperm(B, generator=g, device=DEV).to(torch.int32)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    qkv = _normal(g, B, R, (H + 2 * Hkv) * dh).to(dtype)        # one projection's result: q, k and v side by side in a row
    zeros = lambda heads: torch.zeros(B, R, heads, dh, dtype=torch.bfloat16, device=DEV)
    st = dict(case=case, n_rows=n, parents=par, lens=lens, slots=slots, qkv=qkv, q_out=zeros(H), k_out=zeros(Hkv), v_out=zeros(Hkv))
    if own:
        st["kv"] = _cache(case, g, lens, slots, seed)
    return st


def _prepare_attend(case, seed):
    g = _gen(seed, 2)
    B, R, H, Hkv, dh = (case[k] for k in ("batch", "rows", "heads", "kv_heads", "dim"))
    n, par = _rows(case, g)
    lens = _randint(g, case["ctx_lo"], case["ctx_hi"], (B,))
    slots = torch.randperm(B, generator=g, device=DEV).to(torch.int32)
    q = _normal(g, B, R, H, dh).to(torch.bfloat16)
    T = case["ctx_hi"] + R
    total = (lens + n).tolist()
    st = dict(case=case, n_rows=n, parents=par, lens=lens, slots=slots, q=q,
              out=torch.zeros(B, R, H, dh, dtype=torch.bfloat16, device=DEV))
    if own:
        from paper_2408_05676_b200 import binding as L
        kv = st["kv"] = _cache(case, g, lens, slots, seed)
    else:
        packed = lambda *s: torch.zeros(2, B, T, Hkv, *s, dtype=torch.uint8, device=DEV)
        codes = packed(dh // 2)
        scale, zero = (packed(dh // GROUP).to(torch.bfloat16) for _ in range(2))
        st.update(codes=codes, scale=scale, zero=zero)
    at = slots.tolist()
    for b in range(B):
        gb = _gen(seed, 1000 + b)
        k, v = _keys_values(gb, total[b], Hkv, dh)
        if own:
            L.kv_import(kv, at[b], 0, 0, k.reshape(total[b], -1), v.reshape(total[b], -1))
        else:
            for x, y in ((k, 0), (v, 1)):
                c, s, z = _quantise(x.float())
                c = c.reshape(*c.shape[:-1], dh // 2, 2).to(torch.uint8)
                codes[y, b, :total[b]] = c[..., 0] | (c[..., 1] << 4)
                scale[y, b, :total[b]], zero[y, b, :total[b]] = s.to(torch.bfloat16), z.to(torch.bfloat16)
    return st


def _prepare_adjust(case, seed):
    g = _gen(seed, 3)
    B, R, V = case["batch"], case["rows"], case["vocab"]
    n, par = _rows(case, g)
    logits = _normal(g, B, R, V) * 3
    hist_len = _randint(g, case["hist_lo"], case["hist_hi"], (B,))
    # texts repeat themselves: tokens by a power law, drafts among them
    perm = torch.randperm(V, generator=g, device=DEV)
    zipf = lambda *s: perm[(V ** torch.rand(*s, generator=g, device=DEV) - 1).long().clamp_(0, V - 1)].to(torch.int32)
    hist = zipf(B, case["hist_hi"])
    tokens = zipf(B, R)
    tokens[:, 0] = hist.gather(1, (hist_len - 1).long()[:, None])[:, 0]          # the pending token is the text's last
    prompt_len = (hist_len * torch.rand(B, generator=g, device=DEV)).to(torch.int32)
    rep = 1 + 0.3 * torch.rand(B, generator=g, device=DEV)
    freq, pres = (torch.rand(B, generator=g, device=DEV) for _ in range(2))
    nb = case["bias"]
    bias_off = torch.arange(B + 1, device=DEV).to(torch.int32) * nb
    bias_ids = (torch.randint(0, V, (B, 1), generator=g, device=DEV) + torch.arange(nb, device=DEV) * max(1, V // (nb + 1))) % V
    st = dict(case=case, n_rows=n, parents=par, logits=logits, hist=hist, hist_len=hist_len, tokens=tokens, prompt_len=prompt_len,
              penalties=(rep, freq, pres), bias=(bias_off, bias_ids.reshape(-1).to(torch.int32), 5 * _normal(g, B * nb)),
              allowed=None, out=torch.zeros_like(logits))
    if case["mask"] != "none":
        words = torch.randint(-2 ** 31, 2 ** 31, (B, R if case["mask"] == "row" else 1, -(-V // 32)), generator=g, device=DEV)
        st["allowed"] = words.to(torch.int32)
    return st


# ---- plain forms ------------------------------------------------------------------------------------------

def _quantise(x):
    """Codes [.., dh], scales and zeros [.., dh / GROUP] of fp32 values [.., dh]."""
    x = torch.nan_to_num(x, nan=0.0, posinf=TOP, neginf=-TOP).clamp(-TOP, TOP)
    x = x.reshape(*x.shape[:-1], -1, GROUP)
    lo, hi = x.amin(-1), x.amax(-1)
    s = ((hi - lo) / 15).to(torch.bfloat16).float()
    s = torch.where(s < LEAST, torch.zeros_like(s), s)
    z = (lo - 16 * s).to(torch.bfloat16).float()
    c = torch.round((x - z[..., None]) / s[..., None]) - 16
    c = torch.where(s[..., None] > 0, c.clamp(0, 15), torch.zeros_like(c))
    return c.flatten(-2), s, z


def _value(c, s, z):
    """What codes stand for, fp32 that bf16 can hold."""
    c = c.reshape(*c.shape[:-1], -1, GROUP)
    return (s[..., None] * (16 + c) + z[..., None]).to(torch.bfloat16).float().flatten(-2)


def _seen_rows(parents, B, R):
    """[B, R, R]: whether row j is row i or an ancestor of it."""
    if parents is None:
        return torch.ones(R, R, dtype=torch.bool, device=DEV).tril().expand(B, R, R)
    i = torch.arange(R, device=DEV)
    up = (parents[:, :, None] == i) | (i[:, None] == i)
    return torch.linalg.matrix_power(up.double(), R) > 0


def _active(s):
    return torch.arange(s["case"]["rows"], device=DEV) < s["n_rows"][:, None]


def _plain_append(s):
    B, R, H, Hkv, dh = (s["case"][k] for k in ("batch", "rows", "heads", "kv_heads", "dim"))
    x = s["qkv"].float().reshape(B, R, H + 2 * Hkv, dh)
    depth = torch.arange(R, device=DEV).expand(B, R) if s["parents"] is None else _seen_rows(s["parents"], B, R).sum(-1) - 1
    pos = (s["lens"][:, None] + depth).double()
    ang = pos[..., None] * 10000.0 ** (torch.arange(dh // 2, device=DEV, dtype=torch.float64) * (-2.0 / dh))
    c, sn = ang.cos().float()[:, :, None], ang.sin().float()[:, :, None]
    x1, x2 = x[:, :, :H + Hkv, :dh // 2], x[:, :, :H + Hkv, dh // 2:]
    y = torch.cat([x1 * c - x2 * sn, x2 * c + x1 * sn], -1)
    on = _active(s)[:, :, None, None]
    zero = torch.zeros((), device=DEV)
    q = torch.where(on, y[:, :, :H], zero).to(torch.bfloat16)
    k = torch.where(on, _value(*_quantise(y[:, :, H:])), zero).to(torch.bfloat16)
    v = torch.where(on, _value(*_quantise(x[:, :, H + Hkv:])), zero).to(torch.bfloat16)
    return dict(q=q, k=k, v=v)


def _plain_attend(s):
    B, R, H, Hkv, dh = (s["case"][k] for k in ("batch", "rows", "heads", "kv_heads", "dim"))
    T = s["codes"].shape[2]
    c = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).flatten(-2)
    k, v = _value(c.float(), s["scale"].float(), s["zero"].float()).unbind(0)          # [B, T, Hkv, dh]
    q = s["q"].float().reshape(B, R, Hkv, H // Hkv, dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, dh)
    x = (q @ k.permute(0, 2, 3, 1)) * (1 / math.sqrt(dh))                              # [B, Hkv, rows x heads, T]
    t = torch.arange(T, device=DEV)
    rel = t - s["lens"][:, None]                                                       # which of the step's rows a token is
    own_row = _seen_rows(s["parents"], B, R).gather(2, rel.clamp(0, R - 1)[:, None].expand(B, R, T))
    see = (rel < 0)[:, None] | ((rel < s["n_rows"][:, None])[:, None] & own_row)
    x = x.reshape(B, Hkv, R, H // Hkv, T).masked_fill(~see[:, None, :, None], -math.inf)
    p = (x - x.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    o = (p.reshape(B, Hkv, -1, T) @ v.permute(0, 2, 1, 3)).reshape(B, Hkv, R, H // Hkv, dh)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, R, H, dh)
    return torch.where(_active(s)[:, :, None, None], o, torch.zeros((), device=DEV)).to(torch.bfloat16)


def _plain_adjust(s):
    B, R, V = s["logits"].shape
    at = torch.arange(s["hist"].shape[1], device=DEV)
    live = at < s["hist_len"][:, None]
    made = live & (at >= s["prompt_len"][:, None])
    zeros = torch.zeros(B, V, device=DEV)
    text = zeros.scatter_add(1, s["hist"].long(), live.float())
    gen = zeros.scatter_add(1, s["hist"].long(), made.float())
    path = _seen_rows(s["parents"], B, R).float()
    path[:, :, 0] = 0                                                  # the pending token is in the text
    drafts = torch.zeros(B, R, V, device=DEV).scatter_add(2, s["tokens"].long()[:, None].expand(B, R, R), path)
    n = gen[:, None] + drafts
    rep, freq, pres = (p[:, None, None] for p in s["penalties"])
    x = s["logits"]
    x = torch.where(text[:, None] + drafts > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * n - pres * (n > 0)
    off, ids, val = s["bias"]
    owner = torch.searchsorted(off[1:].contiguous(), torch.arange(len(ids), device=DEV).to(torch.int32), right=True)
    x = x + torch.zeros(B * V, device=DEV).scatter_add(0, owner * V + ids.long(), val).reshape(B, 1, V)
    if s["allowed"] is not None:
        bit = torch.arange(32, device=DEV, dtype=torch.int32)
        on = ((s["allowed"][..., None] >> bit) & 1).flatten(-2)[..., :V] != 0
        x = x.masked_fill(~on, -math.inf)
    return torch.where(_active(s)[..., None], x, torch.zeros((), device=DEV))


# ---- the library's calls ------------------------------------------------------------------------------------

def _own_append(s):
    from paper_2408_05676_b200 import binding as L
    B, R, H, Hkv, dh = (s["case"][k] for k in ("batch", "rows", "heads", "kv_heads", "dim"))
    q, k, v = s["qkv"].split([H * dh, Hkv * dh, Hkv * dh], -1)
    L.kv_append(s["kv"], 0, s["slots"], s["n_rows"], k, v, q=q, parents=s["parents"], q_out=s["q_out"], k_out=s["k_out"], v_out=s["v_out"])
    return dict(q=s["q_out"], k=s["k_out"], v=s["v_out"])


def _own_attend(s):
    from paper_2408_05676_b200 import binding as L
    return L.attend_int4(s["kv"], 0, s["slots"], s["n_rows"], s["q"], parents=s["parents"], out=s["out"])


def _own_adjust(s):
    from paper_2408_05676_b200 import binding as L
    return L.adjust_logits(s["logits"], s["tokens"], s["n_rows"], s["hist"], s["hist_len"], s["prompt_len"], penalties=s["penalties"],
                           bias=s["bias"], allowed=s["allowed"], parents=s["parents"], out=s["out"])


_PREPARE = dict(append=_prepare_append, attend=_prepare_attend, adjust=_prepare_adjust)
_PLAIN = dict(append=_plain_append, attend=_plain_attend, adjust=_plain_adjust)
_OWN = dict(append=_own_append, attend=_own_attend, adjust=_own_adjust)


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, seed)


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------

def work(case):
    B, R = case["batch"], case["rows"]
    rows = B * ((R + 1) / 2 if case["ragged"] else R)
    if case["kind"] == "adjust":
        V = case["vocab"]
        words = -(-V // 32) * (0 if case["mask"] == "none" else rows if case["mask"] == "row" else B)
        hist = B * (case["hist_lo"] + case["hist_hi"]) / 2
        return dict(bytes=8 * rows * V + 4 * words + 4 * hist + 8 * B * case["bias"], flops=4 * rows * V)
    H, Hkv, dh = case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "append":
        read = (2 if case["dtype"] == "bf16" else 4) * rows * (H + 2 * Hkv) * dh
        return dict(bytes=read + 2 * rows * (H + 2 * Hkv) * dh + 0.625 * rows * 2 * Hkv * dh, flops=rows * (6 * H + 16 * Hkv) * dh)
    tokens = B * (case["ctx_lo"] + case["ctx_hi"]) / 2
    return dict(bytes=0.625 * 2 * Hkv * dh * (tokens + rows) + 4 * rows * H * dh, flops=4 * H * dh * (rows / B) * (tokens + rows))


# ---- the definitions in 64 bits -------------------------------------------------------------------------------

def _round_bf16(x):
    """The bf16 number nearest to x (ties to even), fp64 in and out: eight significant bits."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 256), e - 8)


def _held(x):
    """What the cache holds for fp64 features [.., 32 k], by the format's definition."""
    out = torch.empty_like(x)
    for a in range(0, x.shape[-1], GROUP):
        y = x[..., a:a + GROUP]
        low, high = y.min(-1, keepdim=True).values, y.max(-1, keepdim=True).values
        s = _round_bf16((high - low) / 15)
        z = _round_bf16(low - 16 * s)
        code = ((y - z) / s).round().sub(16).clamp(0, 15)
        out[..., a:a + GROUP] = torch.where(s >= LEAST, _round_bf16(z + s * (code + 16)), _round_bf16(low))
    return out


def _path(parents, i):
    """Row i's path from the root: itself and its ancestors, the chain's if there are no parents."""
    if parents is None:
        return list(range(i + 1))
    found = [i]
    while found[-1] > 0:
        found.append(parents[found[-1]])
    return found[::-1]


def _exact_append(s):
    B, R, H, Hkv, dh = (s["case"][k] for k in ("batch", "rows", "heads", "kv_heads", "dim"))
    n, lens = s["n_rows"].tolist(), s["lens"].tolist()
    par = None if s["parents"] is None else s["parents"].tolist()
    out = {k: torch.zeros(B, R, h, dh, dtype=torch.float64, device=DEV) for k, h in (("q", H), ("k", Hkv), ("v", Hkv))}
    turn = torch.exp(torch.arange(dh // 2, device=DEV, dtype=torch.float64) * (-2 * math.log(10000.0) / dh))
    for b in range(B):
        pos = torch.tensor([lens[b] + (i if par is None else len(_path(par[b], i)) - 1) for i in range(n[b])], dtype=torch.float64, device=DEV)
        x = s["qkv"][b, :n[b]].double().view(n[b], H + 2 * Hkv, 2, dh // 2)
        z = torch.complex(x[:, :, 0], x[:, :, 1])[:, :H + Hkv] * torch.polar(torch.ones_like(turn), pos[:, None] * turn)[:, None]
        z = torch.cat([z.real, z.imag], -1)
        out["q"][b, :n[b]] = z[:, :H]
        out["k"][b, :n[b]] = _held(z[:, H:])
        out["v"][b, :n[b]] = _held(x[:, H + Hkv:].reshape(n[b], Hkv, dh))
    return out


def _exact_attend(s):
    B, R, H, Hkv, dh = (s["case"][k] for k in ("batch", "rows", "heads", "kv_heads", "dim"))
    n, lens = s["n_rows"].tolist(), s["lens"].tolist()
    par = None if s["parents"] is None else s["parents"].tolist()
    out = torch.zeros(B, R, H, dh, dtype=torch.float64, device=DEV)
    for b in range(B):
        total = lens[b] + n[b]
        held = []
        for y in range(2):
            c = s["codes"][y, b, :total]
            u = torch.empty(total, Hkv, dh, dtype=torch.float64, device=DEV)
            u[..., 0::2], u[..., 1::2] = c % 16, c // 16
            sz = [p[y, b, :total].double().repeat_interleave(GROUP, -1) for p in (s["scale"], s["zero"])]
            held.append(_round_bf16(sz[0] * (u + 16) + sz[1]))
        hide = torch.zeros(n[b], total, dtype=torch.float64, device=DEV)
        hide[:, lens[b]:] = -math.inf
        for i in range(n[b]):
            hide[i, [lens[b] + j for j in _path(None if par is None else par[b], i)]] = 0
        for h in range(H):
            k, v = (x[:, h // (H // Hkv)] for x in held)
            out[b, :n[b], h] = torch.softmax(s["q"][b, :n[b], h].double() @ k.T / dh ** 0.5 + hide, -1) @ v
    return out


def _exact_adjust(s):
    B, R, V = s["logits"].shape
    n, hl, pl = (s[k].tolist() for k in ("n_rows", "hist_len", "prompt_len"))
    par = None if s["parents"] is None else s["parents"].tolist()
    off = s["bias"][0].tolist()
    out = torch.zeros(B, R, V, dtype=torch.float64, device=DEV)
    for b in range(B):
        rep, freq, pres = (float(p[b]) for p in s["penalties"])
        text, toks = s["hist"][b, :hl[b]].long(), s["tokens"][b].long()
        for i in range(n[b]):
            way = toks[[j for j in _path(None if par is None else par[b], i) if j > 0]]
            count = torch.bincount(torch.cat([text[pl[b]:], way]), minlength=V).double()
            known = torch.bincount(torch.cat([text, way]), minlength=V) > 0
            x = s["logits"][b, i].double()
            x = torch.where(known & (x > 0), x / rep, torch.where(known, x * rep, x))
            x = x - freq * count - pres * (count > 0).double()
            x = x.index_add(0, s["bias"][1][off[b]:off[b + 1]].long(), s["bias"][2][off[b]:off[b + 1]].double())
            if s["allowed"] is not None:
                m = s["allowed"][b, i if s["allowed"].shape[1] > 1 else 0].long() & 0xffffffff
                v = torch.arange(V, device=DEV)
                x = torch.where((m[v // 32] // 2 ** (v % 32)) % 2 == 1, x, torch.full_like(x, -math.inf))
            out[b, i] = x
    return out


_EXACT = dict(append=_exact_append, attend=_exact_attend, adjust=_exact_adjust)


def exact(case, seed):
    return _EXACT[case["kind"]](prepare(case, seed))
