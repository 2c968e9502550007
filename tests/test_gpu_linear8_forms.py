"""tts_linear8 in each of its forms: scales over all of their range and in more words than one, blocks of zeros, a NaN's row, rows around the array, replays of a graph."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import operator_ref as ref
from tests.helpers import say
from tests.test_gpu_linear8 import _rows8, _want

pytestmark = pytest.mark.gpu

# (rows, in_dim, out_dim) by the form that a device of 256 compute units takes for bf16 and for fp32 results (tests/test_operator_plans.py asks the rule)
SHAPES = {(5, 1300, 100): ("few", "few"), (50, 1300, 100): ("split", "split"), (2100, 200, 2050): ("64x128", "64x128"), (1100, 1300, 1000): ("64x64", "64x64"),
          (2900, 641, 1000): ("64x128", "64x64"), (5000, 641, 999): ("128x128", "64x128"), (8300, 641, 1000): ("256x128", "128x128"), (16500, 641, 1001): ("256x128", "256x128")}
LARGE = [s for s in SHAPES if s[0] > 1000]


def _wide(rng, rows, k, n, least, most):
    """Rows of any scales, as bytes, and fp32 weights whose own scales bring every block's products to size 1 or so."""
    blocks = ref.blocks_of(k)
    at = rng.integers(0, 16, (rows, blocks))
    steps = np.linspace(least, most, 16).round().astype(int)                  # the range's ends among them
    kx = np.where(np.arange(blocks) % 3 == 1, steps[at[:1]], steps[-1 - at[:1]]) + np.zeros((rows, 1), int)      # (a block's scales lie together: its weights' are their inverse)
    near = np.clip(kx + rng.integers(-1, 2, (rows, blocks)), least, most)
    codes = rng.integers(0, 127, (rows, blocks * 128)).astype(np.uint8) | (rng.integers(0, 2, (rows, blocks * 128)) * 128).astype(np.uint8)
    codes[:, k:] = 0
    sx = np.full((rows, -(-blocks // 4) * 4), 127, np.uint8)
    sx[:, :blocks] = near + 127
    wc = rng.integers(0, 127, (n, blocks * 128))
    wv = ref.TABLE[wc | (rng.integers(0, 2, wc.shape) * 128)]
    wv[:, ::128] = 448.0                                                       # the block's scale is the one meant
    kw = np.clip(-8 - kx[:1], -119, 119) - 8
    w = (wv.reshape(n, blocks, 128) * 2.0 ** np.clip(kw, -119, 119)[:, :, None]).reshape(n, -1)[:, :k]
    return codes, sx, w.astype(np.float32)


def _call(torch, codes, sx, w, bias, bf16):
    rows, n, k = codes.shape[0], w.shape[0], w.shape[1]
    op = binding.Linear8(binding.make_linear8_config(k, n, bf16), w, bias, stream=torch.cuda.current_stream())
    whole = torch.full((rows + 2, n + 3), 9.0, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    y = whole[1:-1, 1:n + 1]
    op.run_device(torch.from_numpy(codes).to("cuda:0").view(torch.float8_e4m3fn), torch.from_numpy(sx).to("cuda:0").view(torch.float8_e8m0fnu), y)
    torch.cuda.synchronize()
    got = y.double().cpu().numpy()
    whole[1:-1, 1:n + 1] = 9.0
    assert (whole == 9.0).all()                         # nothing around the rows was written
    op.close()
    return got


@pytest.mark.parametrize("rows,k,n", SHAPES)
@pytest.mark.parametrize("bf16", [False, True])
def test_scales_over_their_range(rows, k, n, bf16):
    """From the least to the largest: all of them with bf16 results, with fp32 ones those at which bf16 holds every e4m3 number (2^-124 .. 2^119)."""
    import torch
    say(f"case scales {rows} x {k} x {n} {'bf16' if bf16 else 'fp32'}")
    rng = np.random.default_rng(rows + n)
    codes, sx, w = _wide(rng, rows, k, n, *((-127, 120) if bf16 else (-124, 119)))
    bias = rng.standard_normal(n).astype(np.float32)
    want, tol = _want(codes, sx, w, bias, bf16)
    got = _call(torch, codes, sx, w, bias, bf16)
    assert np.isfinite(want).all() and (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("rows,n", [(8, 128), (64, 128), (16640, 128), (1040, 2048)])
@pytest.mark.parametrize("bf16", [False, True])
def test_every_number_at_the_ends_of_the_scales(rows, n, bf16):
    """Each e4m3 number by itself through weights that are a power of two on the diagonal.  bf16 results: exact at every scale.  fp32 results: exact from 2^-124 to 2^119; operands below are rounded
    to multiples of 2^-133, to even ones from between (what bf16 has there), and at 2^120 those up to 240 are exact."""
    import torch
    numbers = np.arange(256, dtype=np.uint8).reshape(2, 128).copy()
    numbers[(numbers & 127) == 127] = 0
    codes = np.tile(numbers, (rows // 2, 1))
    for byte in [0, 1, 2, 3, 4, 9, 10, 127, 245, 246, 247]:
        e = int(np.clip(127 - byte, -110, 110))
        w = np.zeros((n, 128), np.float32)
        w[np.arange(n), np.arange(n) % 128] = 2.0 ** e
        sx = np.full((rows, 4), 127, np.uint8)
        sx[:, 0] = byte
        c = np.where(ref.TABLE[codes & 127] > 240, 0, codes).astype(np.uint8) if byte == 247 and not bf16 else codes
        x = ref.TABLE[c] * 2.0 ** (byte - 127)
        if not bf16 and byte < 3:
            x = np.round(x * 2.0 ** 133) * 2.0 ** -133
        want = np.tile(x * 2.0 ** e, (1, n // 128))
        np.testing.assert_array_equal(_call(torch, c, sx, w, None, bf16), want, err_msg=str(byte))


@pytest.mark.parametrize("rows,k,n", LARGE)
@pytest.mark.parametrize("bf16", [False, True])
def test_zero_blocks_and_a_nan_in_large_calls(rows, k, n, bf16):
    import torch
    rng = np.random.default_rng(k)
    x = rng.standard_normal((rows, k)) * np.exp(rng.standard_normal((rows, 1)))
    x[:, 128:256] = 0
    x[7] = 0
    w = (rng.standard_normal((n, k)) / np.sqrt(k)).astype(np.float32)
    w[:, k // 128 * 128:] = 0
    w[5] = 0
    codes, sx = ref.round8(x)
    bad = [0, rows // 2, rows - 1]
    where = (codes[bad, 77].copy(), codes[bad, k - 1].copy())
    want, tol = _want(codes, sx, w, None, bf16)
    codes[bad[0], 77] = codes[bad[1], k - 1] = 0x7F
    codes[bad[2], 77] = 0xFF
    got = _call(torch, codes, sx, w, None, bf16)
    assert np.isnan(got[bad]).all()
    rest = np.setdiff1d(np.arange(rows), bad)
    assert (np.abs(got[rest] - want[rest]) <= tol[rest]).all() and (got[7] == 0).all() and (got[rest, 5] == 0).all()


@pytest.mark.parametrize("rows,k,n", [(2100, 200, 2050), (1100, 1300, 1000), (5000, 641, 999), (8300, 641, 1000)])
@pytest.mark.parametrize("bf16", [False, True])
def test_a_graph_of_a_large_call(rows, k, n, bf16):
    import torch
    rng = np.random.default_rng(3)
    w = rng.standard_normal((n, k)).astype(np.float32)
    op = binding.Linear8(binding.make_linear8_config(k, n, bf16), w)
    made = [_rows8(torch, rng.standard_normal((rows, k)))[2:] for _ in range(3)]
    x8, sx = (t.clone() for t in made[0])
    y = torch.empty(rows, n, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    op.run_device(x8, sx, y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=op.stream):
        op.run_device(x8, sx, y)
    for i, (a, b) in enumerate(made + made[:1]):
        x8.view(torch.uint8).copy_(a.view(torch.uint8))
        sx.view(torch.uint8).copy_(b.view(torch.uint8))
        y.fill_(5)
        torch.cuda.synchronize()
        with torch.cuda.stream(op.stream):
            g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        op.run_device(x8, sx, y)
        torch.cuda.synchronize()
        assert torch.equal(got, y), i
    op.close()


def test_more_tiles_than_a_row_of_the_grid_has():
    """2^20 of them and some, of as many rows as a call may have."""
    import torch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("22 GB")
    rows, k, n = 1 << 24, 128, 513
    rng = np.random.default_rng(5)
    w = (rng.standard_normal((n, k)) / np.sqrt(k)).astype(np.float32)
    at = [0, 1, 127, 128, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, 10000019, rows - 1]
    codes, sx = ref.round8(rng.standard_normal((len(at), k)))
    want, tol = _want(codes, sx, w, None, True)
    x8, scales = torch.zeros(rows, k, dtype=torch.uint8, device="cuda:0"), torch.full((rows, 4), 127, dtype=torch.uint8, device="cuda:0")
    x8[at], scales[at] = torch.from_numpy(codes).to("cuda:0"), torch.from_numpy(sx).to("cuda:0")
    y = torch.full((rows, n), 9.0, dtype=torch.bfloat16, device="cuda:0")
    op = binding.Linear8(binding.make_linear8_config(k, n, True), w, stream=torch.cuda.current_stream())
    op.run_device(x8.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), y)
    torch.cuda.synchronize()
    assert (np.abs(y[at].double().cpu().numpy() - want) <= tol).all()
    y[at] = 0
    assert not any(bool(part.any()) for part in y.split(1 << 20))
    op.close()
