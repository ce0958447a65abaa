"""Pools and logits whose offsets pass 32 bits: the calls of include/qcf_turns.h give there what they give in small tensors,
bit for bit."""
import pytest
import torch

from paper_2606_05875_amd import qcf
from test_gpu_chunk import Chunk
from test_gpu_decode import DT, i32, say

pytestmark = pytest.mark.gpu
FAR = (1 << 32) + (1 << 28)   # bytes in front of what is used


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_far_into_a_pool(dtype, d):
    say("chunk attention far into a pool", dtype, d)
    for window in (0, 100):
        x = Chunk([300, 40, 900], [60, 9, 130], 16, 4, d, dtype, 16, window, seed=5)
        was = x.call()
        x.check(*was)
        n, row = x.k.shape[0], 4 * d * x.k.element_size()
        front = -(-FAR // (16 * row))                          # pages
        big = [torch.empty((front * 16 + n, 4, d), dtype=x.k.dtype, device="cuda") for _ in range(2)]
        for far, near in zip(big, (x.k, x.v)):
            far[front * 16:].copy_(near)
            far[:16].fill_(float("nan"))
        x.k, x.v = big
        now = x.call(table=torch.where(x.table >= 0, x.table + front, x.table))
        rows = int(x.cu[-1])
        for a, b in zip(was, now):
            assert torch.equal(a[:rows], b[:rows])
        del big, x, now
        torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_stores_and_copies_far_into_a_pool(dtype):
    say("norms, stores and copies far into a pool", dtype)
    hkv, d, rows = 4, 128, 40
    k, v = (torch.randn((rows, hkv, d), device="cuda").to(DT[dtype]) for _ in range(2))
    slots = torch.randperm(64, device="cuda")[:rows].to(torch.int32)
    near = [torch.zeros((64, hkv, d), dtype=k.dtype, device="cuda") for _ in range(2)]
    freq, pos = qcf.rope_frequencies(d, 1e4), torch.arange(rows, dtype=torch.int32, device="cuda")
    weight = torch.randn(d, device="cuda").to(DT[dtype])
    qcf.qcf_norm_rope_store(*near, k, v, slots, pos, freq, k_weight=weight)
    front = -(-FAR // (16 * hkv * d * k.element_size())) * 16   # rows, whole pages
    far = [torch.empty((front + 128, hkv, d), dtype=k.dtype, device="cuda") for _ in range(2)]
    for t in far:
        t[front:] = 0
    qcf.qcf_norm_rope_store(*far, k, v, slots + front, pos, freq, k_weight=weight)
    pages = torch.arange(4, dtype=torch.int32, device="cuda") + front // 16
    qcf.qcf_copy_pages(qcf.PoolSet(far), pages, pages + 4, 16)
    qcf.qcf_copy_pages(qcf.PoolSet(far), pages[:1], i32([0]), 16, rows=i32([9]))
    for t, s in zip(far, near):
        assert torch.equal(t[front:front + 64], s) and torch.equal(t[front + 64:], s) and torch.equal(t[:9], s[:9])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("probabilities", [True, False])
def test_logits_far_apart(dtype, probabilities):
    say("shaped logits, rows far apart", dtype, probabilities)
    vocab, rows, stride = 9001, 3, (1 << 30) + 3
    z = torch.randn((rows, vocab), device="cuda").to(DT[dtype])
    history = torch.randint(0, vocab, (2, 700), dtype=torch.int32, device="cuda")
    kw = dict(history=history[:, 3:503], hist_len=i32([500, 77]), prompt_len=i32([100, 0]), tokens=i32([4, 5, 6]),
              repetition=torch.tensor([1.5, 0.8], device="cuda"), presence=torch.tensor([0.5, 0.25], device="cuda"),
              probabilities=probabilities)
    cu = i32([0, 2, 3])
    near = torch.empty_like(z)
    qcf.qcf_shape_logits(near, z, cu, **kw)
    kw["history"] = history[:, 3:503].contiguous()
    dense = torch.empty_like(z)
    qcf.qcf_shape_logits(dense, z, cu, **kw)
    assert torch.equal(near, dense) and torch.isfinite(near).all()
    far, out = (torch.empty((rows - 1) * stride + vocab, dtype=z.dtype, device="cuda").as_strided((rows, vocab), (stride, 1))
                for _ in range(2))
    far.copy_(z)
    qcf.qcf_shape_logits(out, far, cu, **kw)
    assert torch.equal(out, near)
