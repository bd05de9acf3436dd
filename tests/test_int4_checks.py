"""Refusals of the calls on a 4-bit cache and of laser_adjust_logits, and what the binding hands over.  No GPU: the library returns
before any launch, or is a stand-in whose "GPU tensors" are host tensors that say they are on the GPU."""
import ctypes as C

import pytest
import torch

from helpers import ensure_built
from test_binding_checks import _gpu, _Recorder


@pytest.fixture(scope="module")
def L():
    ensure_built()
    from paper_2408_05676_b200 import binding
    return binding


def _kv(heads=4, kv_heads=2, dim=64):
    model = type("M", (), dict(cfg=dict(n_heads=heads, n_kv_heads=kv_heads, head_dim=dim)))()
    return type("K", (), dict(handle=1, model=model))()


def test_null_handles_are_refused(L):
    a = 0x1000
    assert L.lib.laser_kv_create_int4(None, 1, C.c_int64(1), C.byref(C.c_void_p())) == -1
    assert L.lib.laser_kv_append(None, 0, a, None, a, 1, 1, 0, None, 0, a, 64, a, 64, None, None, None, None) == -1
    assert L.lib.laser_attend_int4(None, 0, a, None, a, 1, 1, a, 64, a, 64, None) == -1
    assert L.lib.laser_kv_check(None, None) == -1
    assert b"null" in L.lib.laser_last_error()


BASE = dict(logits=0x10000, tokens=0x1000, parents=None, n_rows=0x1000, hist=None, hist_len=None, hist_stride=0, prompt_len=None,
            repetition=None, frequency=None, presence=None, bias_offsets=None, bias_ids=None, bias_values=None, allowed=None,
            mask_seq_stride=0, mask_row_stride=0, B=0, rows=4, V=100, out=0x90000, stream=None)


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(out=None), dict(tokens=None), dict(n_rows=None), dict(rows=0), dict(rows=65), dict(V=0), dict(B=-1), dict(B=65536),
    dict(hist=0x1000), dict(hist=0x1000, hist_len=0x1000, hist_stride=-1), dict(bias_ids=0x1000), dict(bias_offsets=0x1000, bias_ids=0x1000),
    dict(allowed=0x1000, mask_seq_stride=3), dict(allowed=0x1000, mask_seq_stride=4, mask_row_stride=3), dict(logits=0x10002),
    dict(B=2, out=0x10000 + 16), dict(B=2, out=0x10000 - 16), dict(B=2, out=0x10000 + 4 * 2 * 4 * 100 - 4)])
def test_adjust_logits_refuses(L, change):
    call = lambda d: L.lib.laser_adjust_logits(*d.values())
    assert call(BASE) == 0                                      # no sequence: nothing to do
    assert call(dict(BASE, out=BASE["logits"])) == 0
    assert call(dict(BASE, **change)) == -1 and len(L.lib.laser_last_error()) > 0


B, R = 2, 3


def _calls(L):
    i32 = lambda *s: _gpu(s)
    bf = lambda *s: _gpu(s, torch.bfloat16)
    rows = dict(seq_ids=i32(B), n_rows=i32(B), parents=i32(B, R))
    logits = dict(logits=_gpu((B, R, 40), torch.float32), tokens=i32(B, R), n_rows=i32(B), hist=i32(B, 9), hist_len=i32(B), prompt_len=i32(B),
                  rep=_gpu((B,), torch.float32), off=i32(B + 1), ids=i32(5), val=_gpu((5,), torch.float32), allowed=i32(B, R, 2), parents=i32(B, R))
    return {
        "kv_append": (dict(rows, k=bf(B, R, 128), v=bf(B, R, 128), q=bf(B, R, 256)),
                      lambda a: L.kv_append(_kv(), 0, a["seq_ids"], a["n_rows"], a["k"], a["v"], q=a["q"], parents=a["parents"], q_out=bf(B, R, 4, 64), stream=0)),
        "attend_int4": (dict(rows, q=bf(B, R, 4, 64)),
                        lambda a: L.attend_int4(_kv(), 0, a["seq_ids"], a["n_rows"], a["q"], parents=a["parents"], out=bf(B, R, 256), stream=0)),
        "adjust_logits": (logits, lambda a: L.adjust_logits(a["logits"], a["tokens"], a["n_rows"], a["hist"], a["hist_len"], a["prompt_len"],
                                                            (a["rep"], None, None), (a["off"], a["ids"], a["val"]), a["allowed"], a["parents"],
                                                            out=_gpu((B, R, 40), torch.float32), stream=0)),
    }


@pytest.mark.parametrize("name", ["kv_append", "attend_int4", "adjust_logits"])
def test_only_gpu_tensors_of_the_type_and_shape_reach_the_library(L, monkeypatch, name):
    rec = _Recorder()
    monkeypatch.setattr(L, "lib", rec)
    args, call = _calls(L)[name]
    call(args)
    assert [n for n, _ in rec.calls] == ["laser_" + name]
    for arg, t in args.items():
        host = t.as_subclass(torch.Tensor)
        for other in (host.numpy() if t.dtype != torch.bfloat16 else host.float().numpy(), host, t.to(torch.int64), t[:1]):
            with pytest.raises((AssertionError, AttributeError, TypeError)):
                call(dict(args, **{arg: other}))
    assert len(rec.calls) == 1


def test_rows_of_a_fused_projection_are_handed_over_where_they_lie(L, monkeypatch):
    rec = _Recorder()
    monkeypatch.setattr(L, "lib", rec)
    qkv = _gpu((B, R, 512), torch.bfloat16)
    q, k, v = qkv[..., :256], qkv[..., 256:384], qkv[..., 384:]
    L.kv_append(_kv(), 0, _gpu((B,)), _gpu((B,)), k, v, q=q, q_out=_gpu((B, R, 4, 64), torch.bfloat16), stream=0)
    a = rec.calls[0][1]
    assert a[8:14] == (qkv.data_ptr(), 512, qkv.data_ptr() + 512, 512, qkv.data_ptr() + 768, 512)
    for bad in (qkv.transpose(0, 1)[..., 256:384], k[:, :, ::2], qkv[:, ::2, 256:384]):
        with pytest.raises(AssertionError):
            L.kv_append(_kv(), 0, _gpu((B,)), _gpu((B,)), bad, v, stream=0)
