"""What single rows of the attention over pages may rely on: how exact their weights are, that no other row's
values change their bits, and what they give where logits are not numbers.  Sizes reach every kernel: up to 16 and 32 query vectors per KV head, 64, 128 and 256 per
block, float32; short caches and ones that are cut over blocks."""
import math

import numpy as np
import pytest
import torch

from oracle import decode as D
from test_gpu_decode import HALF, Batch, host, say, within

pytestmark = pytest.mark.gpu

# kv, new, hq, hkv, d, page size, max_kv (None: the batch's own)
SIZES = [([70, 0], [3, 2], 8, 2, 64, 16, None), ([3000, 40], [1, 3], 16, 4, 128, 64, None), ([2500], [8], 8, 2, 128, 16, None),
         ([200, 31], [16, 9], 8, 2, 64, 128, None), ([2600, 5], [15, 4], 32, 8, 128, 32, None), ([90], [11], 8, 2, 128, 4, None)]
WIDE = [([900, 12], [30, 7], 16, 4, 128, 64, None), ([2300], [20], 16, 4, 64, 16, None), ([700, 64], [40, 9], 16, 4, 128, 16, 140000),
        ([400], [33], 16, 4, 64, 32, 140000), ([60, 9], [17, 20], 8, 2, 128, 8, None)]


@pytest.mark.parametrize("kv,new,hq,hkv,d,ps,most", SIZES)
def test_weights_keep_15_bits(kv, new, hq, hkv, d, ps, most):
    """Up to 64 query vectors per KV head a bf16 call's weights are two bf16 numbers: the first is cut short by
    less than 2^-7 of the weight, the second, 2^-23 of the weight more than that, rounded by 2^-8 of it.  The other terms are those of test_gpu_decode."""
    say("weights keep 15 bits", kv, new, hq, hkv, d, ps)
    x = Batch(kv, new, hq, hkv, d, "bf16", ps, True, seed=31, back=9)
    assert x.max_q * (hq // hkv) <= 64
    out, lse = x.call()
    x.check(out, lse)
    o = host(out)
    for b in range(len(kv)):
        a, z = x.cu[b], x.cu[b + 1]
        s = x.see[b]
        want, wl, absv, absx = D.tree_attention(host(x.q[a:z]), x.kh[b], x.vh[b], s, x.scale)
        off = d * 2.0 ** -24 * absx + 3 * 2.0 ** -23 * (np.abs(wl) + absx) + (s.shape[1] + 16) * 2.0 ** -24
        within(o[a:z], want, HALF["bf16"] * np.abs(want) + (2 * off + 2.0 ** -15 + 2.0 ** -22)[..., None] * absv, f"request {b}")


@pytest.mark.parametrize("kv,new,hq,hkv,d,ps,most", SIZES + WIDE)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits_leave_other_rows_bits(kv, new, hq, hkv, d, ps, most, dtype):
    """One row and head with logits beyond 2^28: the others' bits are those of a call without it."""
    say("large logits beside others", kv, new, hq, hkv, d, ps, most, dtype)
    x = Batch(kv, new, hq, hkv, d, dtype, ps, True, seed=32, back=9)
    most = x.max_kv if most is None else most
    was = x.call(max_kv=most)
    for row, head in ((0, 1), (new[0] - 1, hq - 1)):
        keep = x.q[row, head].clone()
        x.q[row, head] = 1e18
        now = x.call(max_kv=most)
        x.q[row, head] = keep
        rest = torch.ones(was[1].shape, dtype=torch.bool, device="cuda")
        rest[row, head] = False
        assert now[1][row, head].abs() > 1e15
        for a, b in zip(was, now):
            n = int(x.cu[-1])
            assert torch.equal(a[:n][rest[:n]], b[:n][rest[:n]])


@pytest.mark.parametrize("kv,new,hq,hkv,d,ps,most", SIZES + WIDE)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_that_are_not_finite(kv, new, hq, hkv, d, ps, most, dtype):
    """As the formula gives: a row whose logits are all NaN, or all -infinity, is NaN (its log-sum-exp too: -infinity
    stands for a row that sees no token); where some are -infinity these weigh nothing."""
    say("logits that are not finite", kv, new, hq, hkv, d, ps, most, dtype)
    x = Batch(kv, new, hq, hkv, d, dtype, ps, "random", seed=33)
    most = x.max_kv if most is None else most
    n = int(x.cu[-1])
    was, wl = (host(t)[:n] for t in x.call(max_kv=most))
    rest = np.ones(wl.shape, bool)
    row, head = new[0] - 1, hq - 1
    rest[row, head] = False
    keep = x.q[row, head].clone()
    x.q[row, head, 5] = math.nan
    o, e = (host(t)[:n] for t in x.call(max_kv=most))
    x.q[row, head] = keep
    if x.see[0][row].any():
        assert np.isnan(o[row, head]).all() and np.isnan(e[row, head])
    else:
        assert (o[row, head] == 0).all() and e[row, head] == -math.inf
    np.testing.assert_array_equal(o[rest], was[rest])
    np.testing.assert_array_equal(e[rest], wl[rest])

    x.q[:n, :, 7] = 1.0
    was, wl = (host(t)[:n] for t in x.call(max_kv=most))
    x.check(*x.call(max_kv=most))
    half = x.slot[0][::2]                                   # every other token of request 0, then all of them
    kbuf, kh = x.kbuf.clone(), x.kh[0].copy()
    x.k[torch.from_numpy(half).cuda(), :, 7] = -math.inf
    see = [s.copy() for s in x.see]
    see[0][:, ::2] = False
    o, e = (host(t)[:n] for t in x.call(max_kv=most))
    some, any_ = see[0].any(1), x.see[0].any(1)
    for i in range(new[0]):
        if some[i]:
            want, _, absv, _ = D.tree_attention(host(x.q[i:i + 1]), kh, x.vh[0], see[0][i:i + 1], x.scale)
            within(o[i:i + 1], want, HALF[dtype] * np.abs(want) + (2.0 ** -8 + 2.0 ** -10) * absv, f"row {i}")
        elif any_[i]:
            assert np.isnan(o[i]).all() and np.isnan(e[i]).all(), i
        else:
            assert (o[i] == 0).all() and (e[i] == -math.inf).all(), i
    x.k[torch.from_numpy(x.slot[0]).cuda(), :, 7] = -math.inf
    o, e = (host(t)[:n] for t in x.call(max_kv=most))
    x.kbuf.copy_(kbuf)
    for i in range(new[0]):
        if any_[i]:
            assert np.isnan(o[i]).all() and np.isnan(e[i]).all(), i
        else:
            assert (o[i] == 0).all() and (e[i] == -math.inf).all(), i
    np.testing.assert_array_equal(o[new[0]:], was[new[0]:])  # the other requests
    np.testing.assert_array_equal(e[new[0]:], wl[new[0]:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv,new,hq,hkv,d,ps", [([0], [1500], 2, 1, 128, 64), ([300, 0], [700, 1100], 4, 2, 64, 16)])
def test_prompts(kv, new, hq, hkv, d, ps, dtype):
    """Many new rows without a mask: every row sees the tokens up to its own."""
    say("prompts", kv, new, hq, hkv, d, ps, dtype)
    x = Batch(kv, new, hq, hkv, d, dtype, ps, False, seed=34)
    x.check(*x.call())


@pytest.mark.parametrize("kv,new,hq,hkv,d,ps,most", [s for s in SIZES + WIDE if s[0][0] >= 64])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_values_that_all_rows_see(kv, new, hq, hkv, d, ps, most, dtype):
    """An infinite value of a token before the new rows makes its column infinite, whatever its weight is (with a
    query of zeros every weight is 1), and no other."""
    say("infinite values", kv, new, hq, hkv, d, ps, most, dtype)
    x = Batch(kv, new, hq, hkv, d, dtype, ps, True, seed=35, back=9)
    most = x.max_kv if most is None else most
    for zeros in (False, True):
        if zeros:
            x.q[:int(x.cu[-1])] = 0
        was = host(x.call(max_kv=most)[0])[:new[0]]
        for value in (math.inf, -math.inf):
            for tokens in (x.slot[0][:1], x.slot[0][5:40:3]):
                at = torch.from_numpy(tokens).cuda()
                keep = x.v[at].clone()
                x.v[at, :, 3] = value
                o = host(x.call(max_kv=most)[0])[:new[0]]
                x.v[at] = keep
                assert (o[..., 3] == value).all()
                rest = [j for j in range(d) if j != 3]
                np.testing.assert_array_equal(o[..., rest], was[..., rest])
