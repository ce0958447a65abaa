"""A DraftStep's verifications over vocabularies of several sizes, beside a captured one."""
import numpy as np
import pytest
import torch

from oracle import decode as D
from paper_2606_05875_amd import qcf
from paper_2606_05875_amd.draft import DraftStep, PagedCache
from test_gpu_decode import host, i32, say

pytestmark = pytest.mark.gpu


def inputs(rng, rows, vocab):
    t = torch.softmax(2 * torch.from_numpy(rng.standard_normal((rows, vocab))), 1).float().cuda()
    u = torch.from_numpy(rng.random(rows).astype(np.float32) * np.float32(0.02)).cuda()
    return t, i32(rng.integers(0, vocab, rows)), u, torch.from_numpy(rng.random(2).astype(np.float32)).cuda()


def check(s, x, new):
    target, tokens, u, un = x
    cu = np.concatenate([[0], np.cumsum(new)])
    for b, (a, z) in enumerate(zip(cu[:-1], cu[1:])):
        path, toks = D.verify(host(target)[a:z], None, tokens.cpu().numpy()[a:z], None, u.cpu().numpy()[a:z], float(un[b]))
        assert s.path[b].cpu().tolist() == path + [-1] * (s.max_new - len(path))
        assert s.tokens_out[b].cpu().tolist() == toks + [-1] * (s.max_new - len(toks))


@pytest.mark.parametrize("vocab", [None, 300])
def test_vocabularies_of_several_sizes(vocab):
    """A larger vocabulary than the step was made for, or than its first one, takes a larger workspace; a pass that
    was captured with the smaller one keeps that, and replays give what they gave before."""
    say("vocabularies of several sizes", vocab)
    rng = np.random.default_rng(4)
    cache = PagedCache(1, 8, 16, 2, 64, 2, 4)
    s = DraftStep(cache, 8, 4, 4, qcf.rope_frequencies(64, 1e4), **({} if vocab is None else {"vocab": vocab}))
    assert (s.ws_verify is None) == (vocab is None)
    new = [3, 4]
    s.plan(i32(new))
    small = inputs(rng, 8, 300)
    s.verify(*small)
    check(s, small, new)
    first = s.ws_verify.data_ptr()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        s.verify(*small)
    for v in (20000, 5, 150000):
        x = inputs(rng, 8, v)
        s.verify(*x)
        check(s, x, new)
        fill = torch.full((1 << 16,), 0x7F, dtype=torch.uint8, device="cuda")  # takes up what has been freed
        for a, b in zip(small, inputs(rng, 8, 300)):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        check(s, small, new)
        assert (fill == 0x7F).all()
    assert s.ws_verify.data_ptr() != first
