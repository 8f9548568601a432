"""Pins of oracle/paged.py: properties and closed forms that do not repeat its code."""
import numpy as np
import pytest
import torch

from oracle import ops as O, paged as P


def test_page_table_by_hand():
    # three requests, pages of 4: 3 + 2 tokens (one page opened), nothing new, 0 + 5 tokens (two pages opened)
    table = [[7, -1, -1], [2, -1, -1], [-1, -1, -1]]
    t, starts, lens, pos, slots, need = P.page_table([3, 4, 0], [2, 0, 5], [9, 5, 1, 6], 4, table, 4, 10, 8)
    assert t.tolist() == [[7, 9, -1], [2, -1, -1], [5, 1, -1]]
    assert starts.tolist() == [0, 2, 2, 7] and lens.tolist() == [5, 4, 5] and need == 3
    assert pos.tolist() == [3, 4, 0, 1, 2, 3, 4, -1]
    assert slots.tolist() == [31, 36, 20, 21, 22, 23, 4, -1]
    # the free list ends after one page: the third request keeps nothing
    t, _, lens, _, slots, need = P.page_table([3, 4, 0], [2, 0, 5], [9, 5, 1, 6], 1, table, 4, 10, 8)
    assert lens.tolist() == [5, 4, 0] and need == 3 and slots.tolist() == [31, 36, -1, -1, -1, -1, -1, -1] and t[2].tolist() == [-1] * 3


def test_page_table_hands_out_every_page_once():
    rng = np.random.default_rng(0)
    for _ in range(20):
        R, page, cols = int(rng.integers(1, 9)), int(rng.integers(1, 6)), 7
        cached, fresh = rng.integers(0, 12, R), rng.integers(0, 10, R)
        ids = rng.permutation(200)
        held = [-(-c // page) for c in np.minimum(cached, cols * page)]
        table = np.full((R, cols), -1)
        for r in range(R):
            table[r, :held[r]] = ids[sum(held[:r]):sum(held[:r + 1])]
        t, starts, lens, pos, slots, need = P.page_table(cached, fresh, ids[sum(held):], 200 - sum(held), table, page, 200, int(fresh.sum()))
        used = slots[slots >= 0]
        assert len(set(used)) == len(used)
        assert need == sum(-(-int(n) // page) for n in lens) - sum(held)
        for r in range(R):
            assert lens[r] == min(cached[r] + fresh[r], cols * page) and len(set(t[r, :-(-int(lens[r]) // page)])) == -(-int(lens[r]) // page)


def test_rope_turns_pairs_and_depends_on_distance_only():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 8))
    a = [(P.rope(q, [p + 5], 8, 100.0) * P.rope(k, [p], 8, 100.0)).sum() for p in (0, 3, 1000000)]
    assert np.allclose(a, a[0], atol=1e-8)
    assert np.allclose(P.rope(np.array([[[1.0, 0, 0, 0]]]), [2], 2, 1.0)[0, 0], [np.cos(2), np.sin(2), 0, 0])


def test_head_norm_is_the_norm_of_a_head():
    rng = np.random.default_rng(2)
    x, g, b = rng.standard_normal((5, 3, 16)), rng.standard_normal(16), rng.standard_normal(16)
    assert np.allclose(P.head_norm(x, "layer", g, b, 1e-5), O.layer_norm(x, g, b))
    assert np.allclose(P.head_norm(x, "rms", g, None, 1e-5), O.rms_norm(x, g))


@pytest.mark.parametrize("hq,hkv", [(4, 4), (6, 2), (5, 1)])
def test_paged_attention_is_attention_over_the_gathered_cache(hq, hkv):
    g = torch.Generator().manual_seed(3)
    page, n, d = 4, 11, 8
    kp, vp = torch.randn(2, 9, page, hkv, d, generator=g, dtype=torch.float64)
    q = torch.randn(1, hq, d, generator=g, dtype=torch.float64)
    ids = [8, 0, 5]
    o, lse = P.paged_attention(q.numpy(), kp.numpy(), vp.numpy(), np.array([ids]), [n], 0.3)
    K = kp[ids].reshape(-1, hkv, d)[:n].repeat_interleave(hq // hkv, 1).transpose(0, 1)
    V = vp[ids].reshape(-1, hkv, d)[:n].repeat_interleave(hq // hkv, 1).transpose(0, 1)
    want = torch.nn.functional.scaled_dot_product_attention(q[0][:, None], K, V, scale=0.3)[:, 0]
    assert np.allclose(o[0], want.numpy())
    assert np.allclose(lse[0], torch.logsumexp((K @ q[0][:, :, None])[..., 0] * 0.3, 1).numpy())


def test_w4_unpacks_low_nibble_first():
    w = np.array([[0x2f, 0x80] + [0x88] * 14], np.uint8)
    W = P.unpack_w4(w, np.array([[0.5]]), None, 32)
    assert W[0, :4].tolist() == [3.5, -3.0, -4.0, 0.0] and not W[0, 4:].any()
    assert P.unpack_w4(w, np.array([[2.0]]), np.array([[15]], np.uint8), 32)[0, :2].tolist() == [0.0, -26.0]
