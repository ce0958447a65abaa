"""Decoding calls whose grids have 2^32 threads and more along one dimension, which no launch takes."""
import pytest
import torch

from paper_2606_05875_amd import qcf
from test_gpu_decode import Batch, i32, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_with_bounds_of_many_rows(dtype):
    """A cut cache whose merge has a wave for each of 2^26 and more (row, head) pairs of the bounds."""
    say("attention with bounds of many rows", dtype)
    for kv, new, most in (([2500], [3], 2 ** 20), ([9, 1300], [1, 5], 2 ** 19 + 7)):
        x = Batch(kv, new, 64, 8, 64, dtype, 16, True, seed=41)
        assert len(kv) * most * 64 >= 2 ** 26
        x.check(*x.call(max_q=most))


def test_rope_store_of_many_rows():
    """2^24 and more rows, a block each: few source rows, turned and copied; every row is as a short call gives it."""
    say("rotary store of many rows")
    n, src, d = 2 ** 24 + 21, 64, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn((src, 1, d), generator=gen, device="cuda").bfloat16()
    freq = qcf.rope_frequencies(d, 1e4)
    idx = (torch.arange(n, device="cuda") % src).int()
    pos = torch.div(torch.arange(n, device="cuda"), src, rounding_mode="floor").remainder(8).int()
    out = torch.full((n, 1, d), 3.0, dtype=torch.bfloat16, device="cuda")
    qcf.qcf_rope_store(None, None, None, None, None, pos, freq, q_new=q, q_out=out, src_idx=idx)
    few = torch.empty((8 * src, 1, d), dtype=torch.bfloat16, device="cuda")
    qcf.qcf_rope_store(None, None, None, None, None, pos[:8 * src].clone(), freq, q_new=q, q_out=few, src_idx=idx[:8 * src].clone())
    whole = n // (8 * src) * (8 * src)
    assert (out[:whole].view(-1, 8 * src, d) == few.view(8 * src, d)).all()
    assert torch.equal(out[whole:], few[:n - whole])
