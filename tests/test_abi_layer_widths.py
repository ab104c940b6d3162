"""Widths that the library's 32-bit arguments cannot hold never reach it (no GPU:
tensors without memory)."""
import pytest
import torch


@pytest.fixture(scope="module")
def ace():
    from paper_2609_06072_amd import ace as mod
    return mod


@pytest.fixture
def calls(ace, monkeypatch):
    """Tensors without memory count as the current GPU's; what the library is
    called with, which is nothing here."""
    got = []
    monkeypatch.setattr(ace, "_on_device", lambda t: t.get_device())
    for name in ("ace_moe_dx", "ace_moe_combine_fwd", "ace_moe_combine_bwd", "ace_act_pack", "ace_act_unpack",
                 "ace_swiglu_fwd", "ace_swiglu_bwd"):
        monkeypatch.setattr(ace._lib, name, lambda *a, name=name: got.append(name) or 0)
    monkeypatch.setattr(ace, "_stream_on", lambda index, stream: None)
    monkeypatch.setattr(ace, "ace_workspace_bytes", lambda *a: 256)
    monkeypatch.setattr(ace, "_check_routing", lambda *a: None)
    return got


def meta(*shape):
    return torch.empty(*shape, dtype=torch.bfloat16, device="meta")


@pytest.mark.parametrize("d", [(1 << 32) + 8, 1 << 31])
def test_widths_past_32_bits(ace, calls, d):
    rt = ace.Routing(1, 1, 1, device="cpu")
    x, small = meta(1, d), meta(1, 8)
    packed = ace.PackedAct.__new__(ace.PackedAct)
    packed.rows, packed.d, packed.c = 1, d, ace.AcePackedAct()
    packed.codes = torch.empty(1, d, dtype=torch.int8, device="meta")
    for call in (lambda: ace.ace_act_pack(x, packed), lambda: ace.ace_act_unpack(packed, x),
                 lambda: ace.ace_swiglu_fwd(x, x, x), lambda: ace.ace_swiglu_fwd(packed, packed, x),
                 lambda: ace.ace_swiglu_bwd(x, x, x, x, x), lambda: ace.ace_moe_combine_fwd(x, rt, x),
                 lambda: ace.ace_moe_combine_bwd(x, rt, x),
                 lambda: ace.ace_moe_dx(small, meta(1, 8, d), rt, x), lambda: ace.ace_moe_dx(x, meta(1, d, 8), rt, small)):
        with pytest.raises(ValueError, match="2\\^31"):
            call()
    assert not calls
