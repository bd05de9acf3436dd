"""Pins of the oracles of the 4-bit cache and of the adjusted logits: values checkable by eye, closed forms, library routines."""
import numpy as np
import torch

from oracle import adjust as J
from oracle import int4 as Q


def test_bf16_rounding_is_torchs():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(20000) * 10.0 ** rng.integers(-20, 20, 20000), [0.0, 1 + 2 ** -8, 1 + 3 * 2 ** -8, -1 - 2 ** -8]])
    x = x.astype(np.float32)
    assert (Q.bf16(x) == torch.from_numpy(x).to(torch.bfloat16).double().numpy()).all()


def test_codes_by_eye():
    x = np.zeros(32, np.float32)
    x[:16] = np.arange(16)                 # 0 .. 15: s = 1, z = -16, held exactly
    c, s, z = Q.quantise(x)
    assert s == 1 and z == -16 and (c[:16] == np.arange(16)).all() and (Q.value(c, s, z) == x).all()
    x[:16] += 0.5                          # group 0 .. 15.5: s = bf16(31/30) = 1.03125
    c, s, z = Q.quantise(x)
    assert s == 1.03125 and z == -16.5 and c[15] == 15 and c[0] == 0
    assert Q.value(c, s, z)[15] == Q.bf16(31 * 1.03125 - 16.5)


def test_constant_tiny_and_non_finite_groups():
    for v in (0.0, 3.0, -1.5, 1e-35, 2.0 ** -120):
        assert (Q.held(np.full(32, v, np.float32)) == Q.bf16(np.float32(v))).all()
    x = np.full(64, 1.0, np.float32)
    x[3], x[40], x[41] = np.nan, np.inf, -np.inf
    h = Q.held(x)
    assert np.isfinite(h).all() and h[3] == 0 and (h[:3] == 1).all()
    assert h[40] > 2.0 ** 123 and h[41] < -2.0 ** 123


def test_error_of_a_held_value():
    """A code is off by half a step, or at the ends by what the roundings of s (15 steps x 2^-8 relative) and z (|z| <= (16 + |lo / s|) s)
    take from the range; the held number is rounded once more."""
    rng = np.random.default_rng(1)
    for scale, off in ((1, 0), (1e-3, 0), (50, 3), (1, -20)):
        x = (rng.standard_normal((500, 32)) * scale + off).astype(np.float32)
        _, s, z = Q.quantise(x)
        bound = (0.5 + 31 * 2.0 ** -8) * s + 2.0 ** -8 * np.abs(z) + 2.0 ** -8 * np.abs(x).max(-1, keepdims=True)
        assert (np.abs(Q.held(x) - x) <= bound).all()


def test_attention_is_the_librarys_and_sees_paths():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((4, 4, 64)), rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64))
    out, _ = Q.attend(q, k, v, 5, Q.paths(4))
    t = lambda a: torch.from_numpy(a).transpose(0, 1)
    mask = torch.ones(4, 9, dtype=torch.bool).tril(5)
    want = torch.nn.functional.scaled_dot_product_attention(t(q), t(k).repeat_interleave(2, 0), t(v).repeat_interleave(2, 0), attn_mask=mask)
    assert np.abs(out - want.transpose(0, 1).numpy()).max() < 1e-12
    assert Q.paths(5, [-1, 0, 1, 0, 3]) == [[0], [0, 1], [0, 1, 2], [0, 3], [0, 3, 4]]
    x = Q.rotate(np.array([[1.0, 0.0]]), np.pi / 2, 10000.0)
    assert np.abs(x - [[0.0, 1.0]]).max() < 1e-12


def test_adjusted_logits_by_eye():
    x = np.array([[2.0, -2.0, 1.0, 0.5], [2.0, -2.0, 1.0, 0.5]], np.float32)
    # text 0 | 1 1, pending token 1, draft 2
    out = J.adjust_sequence(x, [1, 2], 2, [0, 1, 1], 1, repetition=2.0, frequency=0.25, presence=0.5, bias=[(3, 1.0), (3, 0.5), (9, 7.0)],
                            allowed=np.array([[1, 1, 1, 1], [1, 0, 1, 1]], bool))
    assert out[0].tolist() == [1.0, -4.0 - 0.5 - 0.5, 1.0, 2.0]
    assert out[1].tolist() == [1.0, -np.inf, 0.5 - 0.25 - 0.5, 2.0]
    tree = J.adjust_sequence(np.zeros((3, 4), np.float32), [1, 2, 3], 3, [1], 1, frequency=1.0, parents=[-1, 0, 0])
    assert tree.tolist() == [[0, 0, 0, 0], [0, 0, -1, 0], [0, 0, 0, -1]]
