"""tts_norm against its definition in 64 bits: widths, rows, types, strides, arrays in place, blocks of zeros, infinities, graphs."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import operator_ref as ref
from tests.helpers import say

pytestmark = pytest.mark.gpu


def _make(torch, rng, rows, dim, bf16, pad=0, scale=1.0):
    t = torch.from_numpy((scale * rng.standard_normal((rows, dim + pad))).astype(np.float32)).to("cuda:0")
    return (t.bfloat16() if bf16 else t)[:, pad // 2: pad // 2 + dim]


def _np(t):
    return t.double().cpu().numpy()


def _tolerance(dim):
    """Of y in fp32, relative: a lane adds at most 8 squares of each 64 * 8 columns of a row and then 12 partial sums, half of whose relative error the square
    root leaves; x + res, the mean, eps, square root, quotient and two products round once each."""
    return (0.5 * (dim / 64 + 8 + 12) + 8) * ref.EPS32


def _check_8(y8, scales, y, dim, slack):
    """8-bit rows against the unrounded y: the scale is the rule's (or the next where y's largest is at the border within `slack`), values are off by half a step."""
    b, s = y8.view(dtype=__import__("torch").uint8).cpu().numpy(), scales.view(dtype=__import__("torch").uint8).cpu().numpy()
    n = ref.blocks_of(dim)
    assert b.shape[1] == n * 128 and (b[:, dim:] == 0).all() and (s[:, n:] == 127).all()
    lo, hi = ref.scale_of(y * (1 - slack)) + 127, ref.scale_of(y * (1 + slack)) + 127
    assert ((s[:, :n] == lo) | (s[:, :n] == hi)).all()
    scale = np.repeat(2.0 ** (s[:, :n].astype(np.float64) - 127), 128, axis=1)[:, :dim]
    got = ref.TABLE[b[:, :dim]] * scale
    # half a step: 2^-4 of the value from 2^-6 up, 2^-10 below (in units of the scale)
    assert (np.abs(got - y) <= np.maximum(np.abs(y) * (2.0 ** -4 + slack), scale * 2.0 ** -10) + np.abs(y) * slack).all()


@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 8), (3, 127), (5, 128), (2, 129), (64, 512), (2100, 513), (2100, 1001), (7, 1024), (2049, 2040), (4, 2049), (9, 4096), (3, 8191), (2, 16384)])
@pytest.mark.parametrize("x_bf16,res_bf16,y_bf16", [(False, False, False), (True, False, True), (True, True, False), (False, True, True)])
def test_norm_against_64_bits(rows, dim, x_bf16, res_bf16, y_bf16):
    import torch
    say(f"case norm {rows} x {dim} {x_bf16} {res_bf16} {y_bf16}")
    rng = np.random.default_rng(rows * 1000 + dim)
    x, res = _make(torch, rng, rows, dim, x_bf16), _make(torch, rng, rows, dim, res_bf16, scale=3.0)
    gain = (1 + 0.2 * rng.standard_normal(dim)).astype(np.float32)
    op = binding.Norm(binding.make_norm_config(dim, x_bf16, res_bf16, y_bf16, eps=1e-5), gain, stream=torch.cuda.current_stream())
    t = lambda bf: torch.bfloat16 if bf else torch.float32   # noqa: E731
    total = torch.empty(rows, dim, dtype=t(res_bf16), device="cuda:0")
    y = torch.empty(rows, dim, dtype=t(y_bf16), device="cuda:0")
    y8 = torch.empty(rows, binding.width8(dim), dtype=torch.float8_e4m3fn, device="cuda:0")
    sc = torch.empty(rows, binding.scale_columns(dim), dtype=torch.float8_e8m0fnu, device="cuda:0")
    op.run_device(x, res=res, total=total, y=y, y8=y8, scales=sc)
    torch.cuda.synchronize()
    want_t, want_y = ref.norm(_np(x), _np(res), gain, np.float32(1e-5))
    tol = _tolerance(dim)
    assert (np.abs(_np(total) - want_t) <= (ref.EPS_BF16 if res_bf16 else ref.EPS32) * np.abs(want_t)).all()
    assert (np.abs(_np(y) - want_y) <= (tol + (ref.EPS_BF16 if y_bf16 else 0)) * np.abs(want_y)).all()
    _check_8(y8, sc, want_y, dim, tol)
    # without the residual and with each output alone: the same rows where they ask for the same
    y2 = torch.full_like(y, 7)
    op.run_device(total if res_bf16 == x_bf16 and not res_bf16 else x, y=y2)
    torch.cuda.synchronize()
    if res_bf16 == x_bf16 and not res_bf16:
        assert torch.equal(y2, y)                       # fp32: the sum itself was written down
    else:
        assert (np.abs(_np(y2) - ref.norm(_np(x), None, gain, np.float32(1e-5))[1]) <= (tol + (ref.EPS_BF16 if y_bf16 else 0)) * np.abs(ref.norm(_np(x), None, gain, np.float32(1e-5))[1])).all()
    op.close()


@pytest.mark.parametrize("rows,dim,pad", [(5, 300, 20), (2200, 130, 6), (3, 1001, 1)])
@pytest.mark.parametrize("bf16", [False, True])
def test_rows_apart_in_place_and_what_lies_between_is_left(rows, dim, pad, bf16):
    import torch
    rng = np.random.default_rng(dim)
    x = _make(torch, rng, rows, dim, bf16, pad)
    gain = np.ones(dim, np.float32)
    op = binding.Norm(binding.make_norm_config(dim, bf16, bf16, bf16), gain, stream=torch.cuda.current_stream())
    whole = torch.full((rows + 2, dim + pad), 5.0, dtype=x.dtype, device="cuda:0")
    res = whole[1:-1, :dim]
    res.copy_(_make(torch, rng, rows, dim, bf16))
    want_t, want_y = ref.norm(_np(x), _np(res), gain, np.float32(1e-5))
    op.run_device(x, res=res, total=res, y=x)           # the stream takes the sum, x the norm
    torch.cuda.synchronize()
    eps = ref.EPS_BF16 if bf16 else ref.EPS32
    assert (np.abs(_np(res) - want_t) <= eps * np.abs(want_t)).all()
    assert (np.abs(_np(x) - want_y) <= (_tolerance(dim) + eps) * np.abs(want_y)).all()
    whole[1:-1, :dim] = 5.0
    assert (whole == 5.0).all()
    op.close()


def test_rounding_alone_is_the_rules_bit_for_bit():
    """No norm: powers of two and ties in every place, blocks of zeros, the largest and least magnitudes, infinities and NaN."""
    import torch
    dim = 700
    rng = np.random.default_rng(4)
    v = rng.standard_normal((40, dim)) * 2.0 ** rng.integers(-140, 120, (40, 1))
    v[0] = 0
    v[1, 128:256] = 0
    v[2] = 448.0                                        # the largest at scale 1, and just above it
    v[3] = np.float32(448.0) * (1 + 2.0 ** -23)
    v[4, :] = (np.arange(dim) % 64 + 0.5) / 8           # ties
    v[5, :] = np.arange(dim) * 2.0 ** -11               # steps below the least normal number, and their ties
    v[5, 0::128] = 448
    v[6] = 2.0 ** -149
    v[7] = 3.4e38
    v = v.astype(np.float32)
    x = torch.from_numpy(v).to("cuda:0")
    op = binding.Norm(binding.make_norm_config(dim, kind=binding.NORM_NONE), stream=torch.cuda.current_stream())
    y8 = torch.empty(40, binding.width8(dim), dtype=torch.float8_e4m3fn, device="cuda:0")
    sc = torch.empty(40, binding.scale_columns(dim), dtype=torch.float8_e8m0fnu, device="cuda:0")
    op.run_device(x, y8=y8, scales=sc)
    torch.cuda.synchronize()
    want, want_s = ref.round8(v.astype(np.float64))
    np.testing.assert_array_equal(sc.view(torch.uint8).cpu().numpy(), want_s)
    np.testing.assert_array_equal(y8.view(torch.uint8).cpu().numpy(), want)
    # an infinity and a NaN: themselves alone
    w = rng.standard_normal((2, dim)).astype(np.float32)
    w[0, 5], w[0, 200], w[1, 699] = np.inf, -np.inf, np.nan
    x = torch.from_numpy(w).to("cuda:0")
    op.run_device(x, y8=y8[:2], scales=sc[:2])
    torch.cuda.synchronize()
    want, want_s = ref.round8(w.astype(np.float64))
    got = y8[:2].view(torch.uint8).cpu().numpy()
    np.testing.assert_array_equal(sc[:2].view(torch.uint8).cpu().numpy(), want_s)
    odd = ~np.isfinite(np.pad(w, ((0, 0), (0, binding.width8(dim) - dim))))
    assert ((got[odd] & 127) == 127).all()
    np.testing.assert_array_equal(got[~odd], want[~odd])
    op.close()


def test_no_rows_and_a_graph_of_another_streams_tensors():
    import torch
    rng = np.random.default_rng(9)
    op = binding.Norm(binding.make_norm_config(600, True, False, True), np.ones(600, np.float32))     # a stream of its own
    none = torch.empty(0, 600, dtype=torch.bfloat16, device="cuda:0")
    op.run_device(none, y=none)
    x, res = _make(torch, rng, 33, 600, True), _make(torch, rng, 33, 600, False)
    y, total = torch.empty_like(x), torch.empty_like(res)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=op.stream):
        op.run_device(x, res=res, total=total, y=y)
        op.run_device(y, res=total, total=total, y=y)   # the same objects again, on what the first call left
    for k in range(3):
        x.copy_(_make(torch, rng, 33, 600, True))
        torch.cuda.synchronize()
        with torch.cuda.stream(op.stream):
            g.replay()
        torch.cuda.synchronize()
        got, got_t = y.clone(), total.clone()
        op.run_device(x, res=res, total=total, y=y)
        op.run_device(y, res=total, total=total, y=y)
        torch.cuda.synchronize()
        assert torch.equal(got, y) and torch.equal(got_t, total), k
    op.close()


def test_as_many_rows_as_a_call_may_have():
    """2^24 rows of a workgroup each: more than one side of a grid takes."""
    import torch
    rows, dim = 1 << 24, 2049
    if torch.cuda.mem_get_info()[0] < 130 << 30:
        pytest.skip("110 GB")
    x = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda:0")
    at = [0, 1, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, rows - 1]
    some = _make(torch, np.random.default_rng(3), len(at), dim, True)
    x[at] = some
    op = binding.Norm(binding.make_norm_config(dim, True, kind=binding.NORM_NONE), stream=torch.cuda.current_stream())
    y8 = torch.empty(rows, binding.width8(dim), dtype=torch.float8_e4m3fn, device="cuda:0")
    sc = torch.empty(rows, binding.scale_columns(dim), dtype=torch.float8_e8m0fnu, device="cuda:0")
    y8.view(torch.uint8).fill_(1)
    op.run_device(x, y8=y8, scales=sc)
    torch.cuda.synchronize()
    want, want_s = ref.round8(_np(some))
    np.testing.assert_array_equal(y8.view(torch.uint8)[at].cpu().numpy(), want)
    np.testing.assert_array_equal(sc.view(torch.uint8)[at].cpu().numpy(), want_s)
    assert int(y8.view(torch.uint8).view(-1).view(torch.int64).ne(0).view(rows, -1).any(1).sum()) == len(at)
