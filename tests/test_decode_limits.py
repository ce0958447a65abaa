"""Sizes that no launch of the decoding calls takes are refused before anything is enqueued (no GPU)."""
import os

import pytest
import torch

from paper_2606_05875_amd import qcf

INVALID, UNSUPPORTED = 1, 2
A, B, C = 0x10000, 0x20000, 0x30000    # fake addresses: these calls never get to a kernel
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(qcf.lib_path()):
        from paper_2606_05875_amd.build import build
        build(verbose=False)
    return qcf.lib()


@pytest.mark.parametrize("dt", [F32, BF16])
def test_attention_of_whole_units(L, dt):
    """Units that are not cut are a block each, and a grid takes fewer than 2^32 threads; calls below the limit get
    to the next check, which refuses their mask."""
    def call(batch, max_q, max_kv, hkv=8):
        return L.qcf_tree_attn(A, None, B, 32, A, A + 4096, C, 1 << 20, hkv * 64, A, 200000, 200000, 16, A, A, 0, dt, batch,
                               max_q, max_kv, hkv, hkv, 64, 0.1, None, 0, None)
    for args in ((1 << 20, 1, 64), (1 << 20, 16, 512), (1 << 19, 17, 512)) if dt == F32 else ((1 << 20, 1, 512), (1 << 20, 1, 2048)):
        assert call(*args) == UNSUPPORTED, args
    for args in (((1 << 20) - 1, 1, 64), ((1 << 20) - 1, 16, 512), (1 << 18, 17, 512), (1 << 20, 1, 140000)):
        assert call(*args) == INVALID, args


def test_verification(L):
    def call(batch=4, vocab=1000):
        return L.qcf_verify_drafts(A, A, A, A, None, vocab, F32, 20, vocab, A, None, batch, A, 8, A, A, A, None, None, A, 0, None)
    assert call(batch=1 << 22) == UNSUPPORTED and call(vocab=(1 << 28) - 8191) == UNSUPPORTED
    assert call(batch=(1 << 22) - 1) == INVALID and call(vocab=(1 << 28) - 8192) == INVALID


def test_types_without_kernels():
    """The binding's own error, not that of a lookup."""
    for dt in (torch.float16, torch.float64, torch.int32):
        with pytest.raises(qcf.QcfError):
            qcf.qcf_tree_attn_workspace_size(1, 1, 100, 8, 2, 64, dt)
