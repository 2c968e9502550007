"""tts_rotary against its definition in 64 bits: layouts, parts of heads, scalings, positions to the ends of 32 bits, types, strides, in place, the gradient, graphs."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import past_ref as ref
from tests.helpers import say

pytestmark = pytest.mark.gpu


def _rows(torch, rng, rows, heads, d, bf16, pad=0):
    t = torch.from_numpy(rng.standard_normal((rows, heads * d + pad)).astype(np.float32)).to("cuda:0")
    return (t.bfloat16() if bf16 else t)[:, : heads * d].unflatten(1, (heads, d))


def _np(t):
    return t.double().cpu().numpy()


def _op(heads, d, rot, pairs, x_bf16, y_bf16, stream=None, **angles):
    import torch
    return binding.Rotary(binding.make_rotary_config(heads, d, binding.make_rotary_angles(rot, pairs, **angles), x_bf16, y_bf16), stream=stream or torch.cuda.current_stream())


def _run(torch, rows, heads, d, rot, pairs, x_bf16, y_bf16, positions=None, first=0, back=False, pad=0, y_pad=0, seed=0, in_place=False, **angles):
    rng = np.random.default_rng(seed)
    x = _rows(torch, rng, rows, heads, d, x_bf16, pad)
    y = x if in_place else _rows(torch, rng, rows, heads, d, y_bf16, y_pad)
    p = np.arange(first, first + rows) if positions is None else positions
    want, size = ref.rotary(_np(x), p, rot, pairs, back=back, **angles)
    kept = None if in_place or y_pad == 0 else y._base[:, heads * d:].clone()
    op = _op(heads, d, rot, pairs, x_bf16, y_bf16, **angles)
    op.run_device(x, y, positions=None if positions is None else torch.from_numpy(np.asarray(positions, np.int32)).to("cuda:0"), first=first, back=back)
    torch.cuda.synchronize()
    got = _np(y)
    tol = ref.rotary_tolerance(want, size, y_bf16)
    if x_bf16 == y_bf16:
        still = size == 0
        assert (got[still] == want[still]).all()       # columns that do not turn: bit for bit
    assert (np.abs(got - want) <= tol).all(), float(np.max(np.abs(got - want) - tol))
    if kept is not None:
        assert torch.equal(kept, y._base[:, heads * d:])
    op.close()
    return y


@pytest.mark.parametrize("x_bf16,y_bf16", [(True, True), (False, False), (True, False), (False, True)])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (96, 48), (40, 40), (128, 2), (72, 6), (8, 8), (256, 256), (256, 34), (24, 20), (136, 68)])
def test_shapes(d, rot, pairs, x_bf16, y_bf16):
    import torch
    say(f"case rotary {rot} of {d} {'pairs' if pairs else 'halves'} {x_bf16} {y_bf16}")
    for rows, heads in ((1, 1), (3, 5), (70, 17)):
        _run(torch, rows, heads, d, rot, pairs, x_bf16, y_bf16, first=1000, seed=d + rot + rows)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("angles", [dict(), dict(scaling=1, factor=8.0), dict(scaling=2, factor=4.0), dict(scaling=3, factor=8.0, trained_len=4096, low=1.0, high=32.0, magnitude=1.2),
                                    dict(scaling=3, factor=40.0, trained_len=100, low=0.0, high=0.5), dict(base=500000.0), dict(base=1.0), dict(magnitude=0.125)])
def test_scalings_and_positions_to_the_ends_of_32_bits(pairs, angles):
    """Every position is as exact as the first: none of an angle's turns is lost."""
    import torch
    p = [0, 1, -1, 2, 4095, 4096, 100000, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, -(1 << 31), -(1 << 30) - 7, 123456789]
    _run(torch, len(p), 3, 64, 64, pairs, False, False, positions=p, seed=3, **angles)
    _run(torch, len(p), 3, 64, 36, pairs, False, False, positions=p, seed=4, back=True, **angles)


@pytest.mark.parametrize("bf16", [False, True])
def test_strides_in_place_and_what_lies_between(bf16):
    """Heads of a joint projection (rows apart), the same rows turned where they are, results into rows that lie apart: nothing between them is touched."""
    import torch
    for pairs in (False, True):
        a = _run(torch, 50, 6, 64, 40, pairs, bf16, bf16, first=7, pad=24, y_pad=8, seed=9)
        b = _run(torch, 50, 6, 64, 40, pairs, bf16, bf16, first=7, pad=24, seed=9, in_place=True)
        assert torch.equal(a, b)


@pytest.mark.parametrize("rows,heads", [(9000, 24), (300, 200), (20000, 1)])
def test_many_rows(rows, heads):
    import torch
    rng = np.random.default_rng(rows)
    _run(torch, rows, heads, 64, 64, False, True, True, positions=rng.integers(-5, 30000, rows), seed=1)


@pytest.mark.parametrize("pairs", [False, True])
def test_the_gradient(pairs):
    """`back` of a gradient is what differences of the turned rows say, and takes positions from rows again."""
    import torch
    rng = np.random.default_rng(2)
    angles = dict(scaling=3, factor=8.0, trained_len=64, magnitude=1.25)
    x, grad = rng.standard_normal((5, 2, 24)), torch.from_numpy(rng.standard_normal((5, 2, 24)).astype(np.float32)).to("cuda:0")
    p = np.array([0, 3, 77, 1000, 99999])
    got = torch.empty_like(grad)
    op = _op(2, 24, 20, pairs, False, False, **angles)
    at = torch.from_numpy(p.astype(np.int32)).to("cuda:0")
    op.run_device(grad, got, positions=at, back=True)
    torch.cuda.synchronize()
    g = _np(grad)
    for index in np.ndindex(x.shape):
        e = np.zeros(x.shape)
        e[index] = 2.0 ** -10
        slope = (g * (ref.rotary(x + e, p, 20, pairs, **angles)[0] - ref.rotary(x - e, p, 20, pairs, **angles)[0])).sum() * 2.0 ** 9
        # (linear: differences are exact but for 64 bits' rounding; the kernel's tolerance as for a turned row)
        assert abs(float(got[index]) - slope) <= 1.25 * 2 * np.abs(g[index[0], index[1]]).max() * 4 * ref.EPS32 + 1e-9
    op.close()
    op = _op(2, 24, 20, pairs, False, False)
    y, z = torch.empty_like(grad), torch.empty_like(grad)
    op.run_device(grad, y, positions=at)
    op.run_device(y, z, positions=at, back=True)
    torch.cuda.synchronize()
    assert float((z - grad).abs().max()) <= 16 * ref.EPS32 * float(grad.abs().max())
    op.close()


@pytest.mark.parametrize("pairs", [False, True])
def test_columns_that_do_not_turn_hold_anything(pairs):
    """Infinities and NaN where nothing turns stay and touch nothing else."""
    import torch
    rng = np.random.default_rng(4)
    for rot in (20, 32, 6):
        x = _rows(torch, rng, 9, 3, 64, True)
        x[:, :, rot:] = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda:0").bfloat16().repeat(22)[: 64 - rot]
        y = torch.empty_like(x)
        op = _op(3, 64, rot, pairs, True, True)
        op.run_device(x, y, first=5)
        torch.cuda.synchronize()
        assert torch.isfinite(y[:, :, :rot]).all()
        a, b = x[:, :, rot:], y[:, :, rot:]
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[~torch.isnan(a)], b[~torch.isnan(b)])
        op.close()


def test_a_graph_reads_its_positions_anew():
    import torch
    rng = np.random.default_rng(5)
    op = binding.Rotary(binding.make_rotary_config(4, 64, binding.make_rotary_angles(64), True, True))
    x, p = _rows(torch, rng, 33, 4, 64, True), torch.zeros(33, dtype=torch.int32, device="cuda:0")
    y, z = torch.empty_like(x), torch.empty_like(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=op.stream):
        op.run_device(x, y, positions=p)
        op.run_device(y, y, first=3)
    for i in range(4):
        p.copy_(torch.from_numpy(rng.integers(0, 5000, 33).astype(np.int32)))
        x.copy_(_rows(torch, rng, 33, 4, 64, True))
        torch.cuda.synchronize()
        with torch.cuda.stream(op.stream):
            g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        op.run_device(x, z, positions=p)
        op.run_device(z, z, first=3)
        torch.cuda.synchronize()
        assert torch.equal(got, z), i
    op.close()


def test_no_rows():
    import torch
    op = _op(2, 64, 64, False, True, True)
    x = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda:0")
    op.run_device(x, x)
    torch.cuda.synchronize()
    op.close()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d,rot", [(96, 26), (64, 54), (64, 62), (40, 14), (256, 254), (256, 252), (256, 250), (256, 14), (248, 10), (256, 2)])
def test_halves_that_end_inside_a_chunk(d, rot, bf16):
    """Columns that two lanes have are turned once, in place too, and those that do not turn stay."""
    import torch
    say(f"case rotary {rot} of {d} in place {bf16}")
    for rows, heads in ((1, 1), (9, 3), (300, 6)):
        _run(torch, rows, heads, d, rot, False, bf16, bf16, first=77, in_place=True, seed=d + rot + rows)
        _run(torch, rows, heads, d, rot, False, not bf16, bf16, first=77, seed=d + rot + rows)
