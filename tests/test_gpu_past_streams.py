"""A block's own past on two streams, against the definition: attention on one waits for the rows that the other appends."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import past_ref as ref
from tests.helpers import say
from tests.test_gpu_cache import _np
from tests.test_gpu_paged import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
def test_what_streams_that_wait_for_each_other_give(bf16):
    """Pages, turned queries and results are NaN before each turn, and other inputs are in the turn before: what was read too early, or left over, would show."""
    import torch
    say(f"case past streams {'bf16' if bf16 else 'fp32'}")
    heads, kv, d, page, n = 4, 2, 64, 16, 400
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    cache = binding.Cache(binding.make_cache_config(kv, d, page, binding.make_rotary_angles(d), n_heads=heads, bf16=bf16, x_bf16=bf16), stream=one)
    attend = binding.PagedAttention(binding.make_paged_config(heads, kv, d, page, bf16), stream=two)
    type_ = torch.bfloat16 if bf16 else torch.float32
    table = torch.arange(-(-n // page), dtype=torch.int32, device="cuda:0").flip(0)[None].contiguous()
    kp, vp = (torch.empty(table.shape[1], kv, page, d, dtype=type_, device="cuda:0") for _ in range(2))
    q_out, out = (torch.empty(n, heads, d, dtype=type_, device="cuda:0") for _ in range(2))
    lse = torch.empty(n, heads, device="cuda:0")
    new, batch = cache.batch([n], [0], [0]), attend.batch([n], [n], [0])
    for seed in range(3):
        g = torch.Generator(device="cuda:0").manual_seed(seed)
        k, v, q = (torch.randn(n, h, d, generator=g, device="cuda:0").to(type_) for h in (kv, kv, heads))
        for t in (kp, vp, q_out, out, lse):
            t.fill_(float("nan"))
        one.wait_stream(torch.cuda.current_stream())
        two.wait_stream(torch.cuda.current_stream())
        cache.run_device(new, k, v, kp, vp, table, q=q, q_out=q_out)
        two.wait_stream(one)
        attend.run_device(batch, q_out, kp, vp, table, out, lse=lse)
        torch.cuda.current_stream().wait_stream(two)
        got, got_lse = out.clone(), lse.clone()
        torch.cuda.synchronize()
        for rows, pages in ((k, kp), (q, None)):
            y, size = ref.rotary(_np(rows), np.arange(n), d)
            turned = _np(q_out) if pages is None else _np(pages[table[0].long()].transpose(1, 2).reshape(-1, kv, d)[:n])
            assert (np.abs(turned - y) <= ref.rotary_tolerance(y, size, bf16)).all()
        # (of the rows as they were turned and rounded)
        _check(got, got_lse, ref.paged(_np(q_out), _np(kp), _np(vp), table.cpu().numpy(), page, [n], [n], [0]), d, n, bf16)
    cache.close()
    attend.close()
