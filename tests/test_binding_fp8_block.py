"""What the binding of the block-scaled expert weights refuses before the library is called (CPU only)."""
import pytest
import torch

import paper_2504_14960_amd as moe

E, H, F = 2, 256, 128


def _outputs():
    out = {}
    for name, shape in (("gate", (E, F, H)), ("up", (E, F, H)), ("down", (E, H, F)), ("wgu_t", (E, H, 2 * F)), ("wd_t", (E, F, H))):
        out[name] = torch.empty(shape, dtype=torch.uint8)
        out[name + "_scales"] = torch.empty((E, shape[1] // 128, moe.fp8_block_scale_stride(shape[2])), dtype=torch.uint8)
    return out


@pytest.fixture
def anywhere(monkeypatch):
    """Pointers of tensors in host memory, and a library that is not called: what is refused is refused by the checks in between."""
    from paper_2504_14960_amd import binding
    calls, stride = [], moe.lib().moe_fp8_block_scale_stride

    class Library:
        def moe_expert_weights_fp8_block(self, *args):
            calls.append(args)
            return 0
        moe_fp8_block_scale_stride = staticmethod(stride)
    library = Library()
    monkeypatch.setattr(binding, "lib", lambda: library)
    monkeypatch.setattr(binding, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(binding, "_stream", lambda: None)
    return calls


def _call(w, out):
    moe.expert_weights_fp8_block(*w, *out.values())


def _weights():
    return [torch.zeros(s) for s in ((E, F, H), (E, F, H), (E, H, F))]


@pytest.mark.parametrize("missing", list(_outputs()))
def test_codes_without_scales_and_scales_without_codes_are_refused(anywhere, missing):
    out = _outputs()
    out[missing] = None
    with pytest.raises(ValueError, match=missing.replace("_scales", "")):
        _call(_weights(), out)
    assert not anywhere


def test_a_whole_set_may_be_left_out(anywhere):
    out = _outputs()
    for name in ("wgu_t", "wgu_t_scales", "wd_t", "wd_t_scales"):
        out[name] = None
    _call(_weights(), out)
    assert len(anywhere) == 1 and anywhere[0][13:17] == (None,) * 4 and None not in anywhere[0][7:13]


@pytest.mark.parametrize("which", [0, 1, 2])
def test_weights_of_another_shape_are_refused(anywhere, which):
    w = _weights()
    w[which] = w[which].transpose(1, 2).contiguous()
    with pytest.raises(ValueError):
        _call(w, _outputs())
    assert not anywhere
