"""Arguments of the 4-bit calls that the binding refuses before anything is launched (no GPU)."""

import pytest
import torch

from paper_2609_07536_b200 import binding as B


def quantize(monkeypatch, inv_perm, copies, T=4, K=64):
    """The code that a call on host tensors is refused with; without a handle the library itself refuses what the binding lets through."""
    monkeypatch.setattr(B, "_device", lambda: -1)
    monkeypatch.setattr(B, "_current_raw_stream", lambda device: 0)
    monkeypatch.setattr(B, "_i32", torch.int32)
    monkeypatch.setattr(B, "_u8", torch.uint8)
    monkeypatch.setitem(B._types, torch.bfloat16, B.MOE_BF16)
    src, codes = torch.zeros((T, K), dtype=torch.bfloat16), torch.zeros((8, K // 2), dtype=torch.uint8)
    scales = torch.zeros(B.moe_mxfp4_scale_bytes(8, K, 1), dtype=torch.uint8)
    with pytest.raises(B.MoeError) as e:
        B.moe_mxfp4_quantize(None, src, codes, scales, 1, torch.zeros(4, dtype=torch.int32), inv_perm=inv_perm, copies=copies)
    return e.value.code


def test_a_flat_inv_perm_does_not_say_how_many_rows_a_token_has(monkeypatch):
    inv = torch.arange(8, dtype=torch.int32)
    assert quantize(monkeypatch, inv.reshape(4, 2), None) == B.MOE_ERR_NULL          # (as far as the library)
    assert quantize(monkeypatch, inv.reshape(4, 2), 2) == B.MOE_ERR_NULL
    assert quantize(monkeypatch, inv, 2) == B.MOE_ERR_NULL                            # flat, with the number of copies
    assert quantize(monkeypatch, inv, None) == B.MOE_ERR_SHAPE                        # one token with eight copies?
    assert quantize(monkeypatch, inv, 3) == B.MOE_ERR_SHAPE
    assert quantize(monkeypatch, inv.reshape(4, 2), 4) == B.MOE_ERR_SHAPE
    assert quantize(monkeypatch, inv.reshape(2, 2, 2), None) == B.MOE_ERR_SHAPE
    assert quantize(monkeypatch, inv[:6].reshape(3, 2), None) == B.MOE_ERR_SHAPE
    assert quantize(monkeypatch, inv.reshape(2, 4), None, T=1) == B.MOE_ERR_SHAPE     # two tokens, one row of them


def test_tiles_are_not_selected_without_a_handle():
    with pytest.raises(B.MoeError) as e:
        B.moe_mxfp4_select_tile(None, 4, 2, 16)
    assert e.value.code == B.MOE_ERR_NULL
