"""Refusals of the layer entry points and workspace sizes (no GPU): every case
fails on the host, before any device work."""
import ctypes

import numpy as np
import pytest

import paper_2606_11081_amd as g

BAD = g.gasloc.GASLOC_EINVAL


def test_null_context():
    lib = g.library()
    size = ctypes.c_size_t()
    ptr = np.zeros(2, np.int64).ctypes.data
    assert lib.gasloc_embedding(None, 0, 1, 1, 1.0, ptr, None, 0, None, 1) == BAD
    assert lib.gasloc_embedding_grad(None, 0, 1, 1, 1.0, ptr, None, 0, None, 1, None, 4, 0, None, 0) == BAD
    assert lib.gasloc_layer_norm(None, 0, 0, 1, 1e-5, ptr, None, 1, 0, None, 1, None) == BAD
    assert lib.gasloc_layer_norm_grad(None, 0, 0, 1, ptr, None, 1, None, None, 1, 0, None, 1, None, 4, 0, None, 0) == BAD
    assert lib.gasloc_linear(None, 0, 1, 1, ptr, None, 1, 0, None, 1, None, 0) == BAD
    assert lib.gasloc_linear_grad_input(None, 0, 1, 1, ptr, None, 1, 0, None, 1, None, 0) == BAD
    assert lib.gasloc_linear_grad_weight(None, 0, 1, 1, ptr, None, 1, None, 1, 0, None, 4, 0, None, 0) == BAD
    assert lib.gasloc_embedding_grad_workspace(None, 1, ptr, ctypes.byref(size)) == BAD
    assert lib.gasloc_layer_norm_grad_workspace(None, 1, ptr, ctypes.byref(size)) == BAD
    assert lib.gasloc_linear_workspace(None, 1, 1, ptr, 0, ctypes.byref(size)) == BAD
    assert "NULL" in g.gasloc.gasloc_last_error(None)


def test_activation_types():
    import torch

    assert g.gasloc._act("bf16") == g.gasloc._act(torch.bfloat16) == g.gasloc.GASLOC_BF16
    assert g.gasloc._act("f32") == g.gasloc._act(torch.float32) == g.gasloc.GASLOC_F32
    with pytest.raises(ValueError):
        g.gasloc._act(torch.float16)
