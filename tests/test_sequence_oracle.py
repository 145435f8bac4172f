"""The fp64 statement of the sequence path (oracle/sequence_oracle.py) against torch and closed forms, and the host side of its calls."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so
from paper_2510_18239_b200 import binding


def test_attention_is_torchs():
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(n, h, 16, generator=g, dtype=torch.float64) for n, h in ((5, 4), (9, 2), (9, 2)))
    out, mag, _ = so.attend(q, k, v, so.causal(5, 9), 0.25)
    mask = torch.tensor(so.causal(5, 9))
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), k.repeat_interleave(2, 1).transpose(0, 1), v.repeat_interleave(2, 1).transpose(0, 1),
                                                            attn_mask=mask, scale=0.25).transpose(0, 1)
    assert np.allclose(out, want.numpy(), atol=1e-12) and (mag >= np.abs(out) - 1e-12).all()
    empty, _, _ = so.attend(q, k[:3], v[:3], so.causal(5, 3), 0.25)
    assert (empty[:2] == 0).all() and np.allclose(empty[2], v[0].repeat_interleave(2, 0).numpy())


def test_a_chain_is_causal_and_roots_see_themselves():
    assert (so.ancestors([-1, 0, 1, 2]) == so.causal(4, 4)).all()
    assert (so.ancestors([-1, -1, 5, 3, -9]) == np.eye(5, dtype=bool)).all()
    assert so.ancestors([-1, 0, 0, 2])[3].tolist() == [True, False, True, True]


def test_rotation_keeps_lengths_and_turns_by_differences():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((6, 2, 12))
    pos = np.array([0, 3, -4, 100, 7, 1 << 20])
    for inter in (False, True):
        y, z = so.norm_rotate(x, None, pos, 8, inter, 100.0, 1e-6), so.norm_rotate(x, None, pos * 0, 8, inter, 100.0, 1e-6)
        assert np.allclose((y ** 2).sum(-1), (z ** 2).sum(-1)) and np.allclose(y[..., 8:], z[..., 8:]) and np.allclose(y[0], z[0])
        a, b = (so.norm_rotate(np.tile(x[:1], (6, 1, 1)), None, pos + s, 12, inter, 100.0, 1e-6) for s in (0, 11))
        assert np.allclose(np.einsum("ihd,jhd->hij", a, a), np.einsum("ihd,jhd->hij", b, b), atol=1e-8)


def test_cached_rows():
    pages = np.arange(3 * 4 * 1 * 2, dtype=np.float64).reshape(3, 4, 1, 2)
    assert (so.cached_rows(pages, [2, 0, 7], 6) == np.concatenate((pages[2], pages[0, :2]))).all()
    assert (so.cached_rows(pages, [2, 3, -1], 12)[4:] == 0).all()


def test_entry_points_refuse_no_context():
    lib = binding.load_library()
    assert ctypes.sizeof(binding.lime_sequence) == 40
    assert lib.lime_set_sequence(None, ctypes.byref(binding.lime_sequence(4, 2, 32))) == 1
    assert lib.lime_sequence_workspace_bytes(None, 1, 1) == 0
    assert lib.lime_norm_rotate(None, None, 0, None, 0, None, 0, None, None, None, 1, None, 0, None, 0, None, None, 0, None, None, None) == 1
    assert lib.lime_attend_history(None, None, 0, None, None, 0, None, 0, None, 1, 1, 1, None, 0, None, 0, None) == 1
    assert lib.lime_attend_tree(None, None, 0, None, None, None, 0, None, 0, 1, 1, None, None, 0, 16, None, 0, None, None, None, 0, None, 0, None) == 1


@pytest.mark.parametrize("which", ["native", "python"])
def test_marshalling_refuses_what_is_no_cuda_tensor(which):
    calls = binding._native() if which == "native" else binding._PlainCalls
    q = torch.zeros(2, 4, 8)
    for f in (lambda: calls.attend_history(None, False, 4, 4, 8, q, q, q, q, None, None),
              lambda: calls.norm_rotate(None, False, 4, 4, 8, q, q, None, None, None, None, None, None, None, None, None, None, False),
              lambda: calls.attend_tree(None, False, 4, 4, 8, q, q, None, None, None, q, q, q, q, None, None)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        calls.attend_history(None, False, 4, 4, 8, [1], q, q, q, None, None)
    with pytest.raises(TypeError):
        calls.attend_tree(None, False)
