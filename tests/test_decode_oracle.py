"""The decoding oracle against closed forms and counts that do not use it (CPU)."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from oracle import decode as D
from oracle import qcfuse as Q
from paper_2606_05875_amd import qcf


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(qcf.lib_path()):
        from paper_2606_05875_amd.build import build
        build(verbose=False)


def test_plan_gives_every_token_its_own_slot():
    rng = np.random.default_rng(0)
    kv, new, ps = rng.integers(0, 40, 9), rng.integers(0, 20, 9), 8
    held = [-(-k // ps) for k in kv]
    order = rng.permutation(200)
    table, at = np.full((9, 12), -1), 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    t, slots, pos, _, cu, end, have, head = D.page_plan(table, kv, new, order[at:], ps, 200, new.sum() + 3)
    assert head == sum(-(-(k + n) // ps) - h for k, n, h in zip(kv, new, held)) and cu[-1] == new.sum()
    used = []
    for b in range(9):
        slot = [t[b, j // ps] * ps + j % ps for j in range(end[b])]
        np.testing.assert_array_equal(slots[cu[b]:cu[b + 1]], slot[kv[b]:])
        np.testing.assert_array_equal(pos[cu[b]:cu[b + 1]], np.arange(kv[b], end[b]))
        used += slot
    assert len(set(used)) == len(used) and (slots[cu[-1]:] == -1).all()


def test_plan_tree():
    parents = np.array([-1, 0, 0, 1, 3, 2, 5, -1])
    _, _, pos, mask, *_ = D.page_plan(np.full((1, 4), -1), [10], [8], np.arange(9), 8, 9, 8, parents=parents, words=1)
    np.testing.assert_array_equal(pos, [10, 11, 11, 12, 13, 12, 13, 10])
    assert [set(np.nonzero(m)[0]) for m in mask] == [{0}, {0, 1}, {0, 2}, {0, 1, 3}, {0, 1, 3, 4}, {0, 2, 5},
                                                    {0, 2, 5, 6}, {7}]


@pytest.mark.parametrize("scaling", [dict(), dict(scaling="linear", factor=4.0),
                                     dict(scaling="by_parts", factor=8.0, low_turns=1.0, high_turns=4.0, trained_len=8192)])
def test_frequencies_of_the_library_and_the_oracle_agree(scaling):
    freq = torch.empty(64, dtype=torch.float64)
    qcf.qcf_rope_frequencies(freq, 5e5, **scaling)
    want = D.rope_frequencies(128, 5e5, **scaling)
    np.testing.assert_allclose(freq.numpy(), want, rtol=1e-14)
    plain = 5e5 ** (-np.arange(64) / 64)
    if scaling.get("scaling") == "by_parts":                    # fast pairs kept, slow ones stretched by 8
        np.testing.assert_allclose(want[:8], plain[:8], rtol=1e-14)
        np.testing.assert_allclose(want[-8:], plain[-8:] / 8, rtol=1e-14)
        assert (np.diff(want) < 0).all()


def test_rope_halves_match_the_cache_fusion_rotation():
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 2, 64)), np.array([0, 1, 77, 4000, 32000])
    y, _ = D.rope(x, pos, D.rope_frequencies(64, 1e4))
    np.testing.assert_allclose(y, Q.rope(x, pos, 1e4), atol=1e-12)
    # interleaved pairs are the halves' pairs in another order; norms are kept, times the magnitude
    perm = np.arange(64).reshape(2, 32).T.ravel()
    z, _ = D.rope(x[..., perm], pos, D.rope_frequencies(64, 1e4), interleaved=True, magnitude=1.5)
    np.testing.assert_allclose(z, 1.5 * y[..., perm], atol=1e-12)


def test_attention_against_torch():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((6, 4, 8)), rng.standard_normal((17, 2, 8)), rng.standard_normal((17, 2, 8))
    see = D.chain_see(6, 11)
    out, lse, _, _ = D.tree_attention(q, k, v, see, 0.3)
    t = lambda a: torch.from_numpy(a).permute(1, 0, 2)[None]
    want = torch.nn.functional.scaled_dot_product_attention(t(q), t(k), t(v), attn_mask=torch.from_numpy(see),
                                                            scale=0.3, enable_gqa=True)
    np.testing.assert_allclose(out, want[0].permute(1, 0, 2).numpy(), atol=1e-12)


@pytest.mark.parametrize("with_draft,parents", [(True, None), (True, [-1, 0, 0, 0]), (False, [-1, 0, 0, 0]),
                                                (True, [-1, 0, 1, 1])])
def test_verification_keeps_the_targets_distribution(with_draft, parents):
    """The first token that comes out follows the target's row 0, whatever is drafted: within four
    standard errors of a count over 20000 trials."""
    rng = np.random.default_rng(3)
    V, n, trials = 5, 4, 20000
    target, draft = rng.dirichlet(np.ones(V), n), rng.dirichlet(np.ones(V), n)
    up = parents or [-1, 0, 1, 2]
    count = np.zeros(V)
    for _ in range(trials):
        tok = [0] + [int(rng.choice(V, p=draft[up[j]])) if with_draft else (j + 1) % V for j in range(1, n)]
        _, out = D.verify(target, draft if with_draft else None, tok, parents, rng.random(n), rng.random())
        count[out[0]] += 1
    err = np.abs(count / trials - target[0])
    assert (err < 4 * np.sqrt(target[0] * (1 - target[0]) / trials)).all(), err
