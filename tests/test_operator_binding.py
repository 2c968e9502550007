"""What the operators' Python layer refuses or hands on, and their host code's last refusals, without a GPU: numbers that the C types do not hold."""
import ctypes as C

import pytest

from paper_2211_13939_amd import binding
from tests.test_operators_host import INVAL, Made, lib  # noqa: F401  (a fixture)


def _bare(cls, **attributes):
    """An object without a library behind it: tensors of the meta device pass for its device's."""
    import torch
    o = cls.__new__(cls)
    o._torch, o._index, o.device, o._handle, o.calls = torch, -1, torch.device("meta"), None, []
    o._run = lambda *a: o.calls.append(a) or 0
    for k, v in attributes.items():
        setattr(o, k, v)
    return o


@pytest.mark.parametrize("field", range(3))
@pytest.mark.parametrize("number", [(1 << 64) + 1, -(1 << 64), 1 << 63])
def test_lengths_that_their_types_do_not_hold(field, number):
    lengths = [[1, 1], [0, 3], [2, 2]]
    assert binding.CrossBatch(*lengths).queries == 2
    lengths[field][1] = number
    with pytest.raises(ValueError):
        binding.CrossBatch(*lengths)
    if field != 1:
        lengths[field][1] = (1 << 32) + 2
        with pytest.raises(ValueError):
            binding.CrossBatch(*lengths)


def test_more_rows_than_an_int_holds():
    import torch
    op = _bare(binding.Norm, _dim=1, _types=[torch.bfloat16] * 3)
    y = torch.empty(5, 1, dtype=torch.bfloat16, device="meta")
    op.run_device(y, y=y)
    assert op.calls[0][1].rows == 5
    for rows in ((1 << 32) + 5, 1 << 32, (1 << 24) + 1):
        x = torch.empty(rows, 1, dtype=torch.bfloat16, device="meta")
        with pytest.raises(ValueError):
            op.run_device(x, y=x)
    assert len(op.calls) == 1


def test_no_memory_at_all():
    """k and v are not needed where no request has any, and not to be left out otherwise or one without the other."""
    import torch
    op = _bare(binding.CrossAttention, _dtype=torch.float32, _widths=(2, 128, 64))
    q, kv = (torch.empty(3, h, 64, device="meta") for h in (2, 1))
    op.run_device(binding.CrossBatch([1, 2], [0, 5], [0, 0]), q, None, None, q)
    t = op.calls[0][2]
    assert t.k is None and t.v is None and t.k_stride == t.v_stride == 0
    op.run_device(binding.CrossBatch([1, 2], [0, 1], [1, 2]), q, kv, kv, q)
    for k, v in ((None, None), (None, kv), (kv, None)):
        with pytest.raises(ValueError):
            op.run_device(binding.CrossBatch([1, 2], [0, 1], [1, 2]), q, k, v, q)
    with pytest.raises(ValueError):
        op.run_device(binding.CrossBatch([1, 2], [0, 0], [0, 0]), q, None, kv, q)
    assert len(op.calls) == 2


@pytest.mark.parametrize("make", [lambda **k: binding.Norm(binding.make_norm_config(64), [1.0] * 64, **k), lambda **k: binding.Linear8(binding.make_linear8_config(64, 32), [[1.0] * 64] * 32, **k),
                                  lambda **k: binding.CrossAttention(binding.make_cross_config(2, 1, 64), **k)])
def test_a_stream_of_another_device(make, monkeypatch):
    """An object's stream takes launches of its own device: one of another is refused before anything is laid down."""
    import torch
    from types import SimpleNamespace
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: pytest.fail("an arena was asked for"))
    with pytest.raises(ValueError, match="cuda:1"):
        make(stream=SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=16), device="cuda:0")


def test_scales_at_the_ends_of_fp32(lib):      # noqa: F811
    """Kernels take the scale times log2(e), which has to be a number too; one that fp32 rounds to 0 would be the default in the place of next to nothing."""
    import torch
    lib.fake_reset()
    m = Made(lib, "cross", binding.make_cross_config(2, 1, 64))
    b = binding.CrossBatch([1], [0], [1])
    for scale, rc in ((2.0 ** 127, 0), (2.3e38, 0), (2.4e38, INVAL), (3.4e38, INVAL), (1e-44, 0)):
        t = binding.TtsCrossTensors(q=1 << 20, k=2 << 20, v=3 << 20, out=4 << 20, scale=scale)
        assert lib.tts_cross_run(m.h, C.byref(b.c), C.byref(t)) == rc, scale
    m.close()
    op = _bare(binding.CrossAttention, _dtype=torch.float32, _widths=(2, 128, 64))
    q, kv = (torch.empty(1, h, 64, device="meta") for h in (2, 1))
    op.run_device(b, q, kv, kv, q, scale=1e-44)
    op.run_device(b, q, kv, kv, q)
    assert op.calls[0][2].scale > 0 and op.calls[1][2].scale == 0
    with pytest.raises(ValueError):
        op.run_device(b, q, kv, kv, q, scale=1e-46)
