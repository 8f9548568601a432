"""The operators over a paged key / value cache against oracle/paged.py: page table and slots (equal), per-head norm + rotation +
store, attention of one new token, and a decode iteration that runs them together.

Tolerances, per element.  A store rounds by half a step: bf16 2^-8, fp32 2^-24 of the value.
Norm and rotation: the sums of d <= 256 squares are added as trees over the lanes (at most 8 + 6 additions deep), the square root, the
division and the products add a few roundings more, and mean and square root see x's own size: 40 * 2^-24 of the largest value that
occurs on the way.  The angle's rounding to fp32 (2^-25 of a revolution) and a sine of 2^-20 absolute in bf16 (the hardware's), 2^-22 in
fp32 (the library's), times the pair.
Attention: a logit's error is below (d + 4) 2^-24 of sum |q k| * |scale| (products exact in bf16, sums in fp32), and moves a weight by
that much, numerator and denominator; the weights themselves carry 2^-16 (bf16: two terms of 8 bits each) resp. 2^-22, and sums of up
to n keys in blocks (n / 16 + 64) 2^-24 of sum p |v|."""
import copy
import threading

import numpy as np
import pytest
import torch

from oracle import ops as O, paged as P
from paper_2404_13528_amd import binding as sm
from util import to_np

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
I32 = torch.int32


def ints(x, pad=None):
    return torch.tensor(x, dtype=I32).cuda()


def check(got, want, tol, what):
    got = to_np(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %s: %r for %r, tolerance %r" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], np.broadcast_to(tol, bad.shape)[bad][0])


# ------------------------------------------------------------------------------------------------ page table

def page_case(cached, fresh, page, cols, spare=5, short=0, pad=0, pitch=0, seed=0):
    """Runs sm_page_table and the oracle; the table's pitch may be larger than its row."""
    rng = np.random.default_rng(seed)
    R, row = len(cached), cols * page
    held = [-(-min(max(c, 0), row) // page) for c in cached]
    ends = [min(min(max(c, 0), row) + max(f, 0), row) for c, f in zip(cached, fresh)]
    new = sum(-(-e // page) - h for e, h in zip(ends, held))
    n_pages = sum(held) + new + spare
    ids = rng.permutation(n_pages)
    table = np.full((R, cols + pitch), -7)
    at = 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    free = ids[at:]
    n_free = max(0, new - short) if short else len(free)
    T = max(0, sum(max(f, 0) for f in fresh) + pad)
    want = P.page_table(cached, fresh, free, n_free, table[:, :cols], page, n_pages, T)
    td = ints(table)
    out = sm.page_table(ints(cached), ints(fresh), ints(free), ints([n_free]), td[:, :cols], page, n_pages, T)
    for _ in range(2):                                 # the same call again: the same result
        torch.cuda.synchronize()
        got = td.cpu().numpy()
        assert (got[:, :cols] == want[0]).all() and (got[:, cols:] == -7).all()
        for g, w, n in zip(out, want[1:5], out._fields):
            assert (g.cpu().numpy() == w).all(), (n, g.cpu().numpy(), w)
        assert out.need.item() == want[5]
        sm.page_table(ints(cached), ints(fresh), ints(free), ints([n_free]), td[:, :cols], page, n_pages, T, out=out)


@pytest.mark.parametrize("cached,fresh,page,cols", [
    ([0], [0], 1, 1), ([0], [1], 16, 1), ([15], [1], 16, 2), ([16], [1], 16, 2), ([17], [0], 16, 2), ([3, 4, 0], [2, 0, 5], 4, 3),
    ([0, 0, 0, 0], [0, 0, 0, 0], 8, 2), ([-5, 7, 3], [4, -9, 30], 8, 3),        # negative counts, a row that ends
    ([100, 0], [5, 40], 8, 4),                                                   # more cached than the row holds
    ([0, 31], [2500, 1], 32, 100), ([5], [5000], 1, 5005), ([7, 9], [1030, 2], 3, 400)])
def test_page_table_small(cached, fresh, page, cols):
    for pad, short, pitch in ((0, 0, 0), (3, 1, 2), (-1, 0, 1), (1500, 2, 0)):
        page_case(cached, fresh, page, cols, pad=pad, short=short, pitch=pitch)


@pytest.mark.parametrize("R", [1, 63, 64, 65, 255, 256, 257, 511, 768, 769, 1000, 1024, 1025, 2049, 5000])
def test_page_table_many_requests(R):
    rng = np.random.default_rng(R)
    cached = rng.integers(0, 50, R).tolist()
    page_case(cached, [1] * R, 16, 5, seed=R)
    page_case(cached, rng.integers(0, 40, R).tolist(), 8, 12, pad=100, short=R // 2, seed=R)
    page_case(cached, (rng.integers(0, 30, R) * (rng.random(R) < 0.1)).tolist(), 4, 20, pad=-int(R // 3), seed=R)


def test_page_table_without_tokens_or_free_pages():
    e = torch.empty(0, dtype=I32, device="cuda")
    t = ints([[3, -1]])
    out = sm.page_table(ints([5]), ints([4]), e, ints([9]), t, 8, 4, 0)        # no rows: the new tokens are not there
    assert out.lens.tolist() == [5] and out.starts.tolist() == [0, 0] and out.need.item() == 0
    out = sm.page_table(ints([5]), ints([4]), e, ints([9]), t, 8, 4, 4)        # no page to take, whatever n_free says
    assert out.lens.tolist() == [8] and out.slots.tolist() == [29, 30, 31, -1] and out.need.item() == 1 and t.tolist() == [[3, -1]]


def test_page_table_bad_pages_have_no_slot():
    out = sm.page_table(ints([1, 1, 0]), ints([1, 1, 2]), ints([99, 2]), ints([2]), ints([[-3], [64], [5]]), 16, 64, 4)
    assert out.slots.tolist() == [-1, -1, -1, -1] and out.lens.tolist() == [2, 2, 2]


def test_page_table_with_its_arrays_side_by_side_and_between_the_rows_of_the_table():
    """Everything in one buffer, adjacent or in the gap of the table's pitch: nothing overlaps, nothing is refused."""
    buf = torch.full((400,), -9, dtype=I32, device="cuda")
    table = buf[:90].view(3, 30)[:, :4]
    at = [90]

    def piece(n, values=None):
        t = buf[at[0]:at[0] + n]
        at[0] += n
        if values is not None:
            t.copy_(ints(values))
        return t
    cached, fresh = piece(3, [5, 0, 9]), piece(3, [2, 3, 9])
    free, n_free = buf[34:44], buf[74:75]                               # (rows 1 and 2 of the table begin at 30 and 60)
    free.copy_(torch.arange(50, 60, dtype=I32))
    n_free.fill_(10)
    table.copy_(ints([[7, -1, -1, -1], [-1] * 4, [3, 2, -1, -1]]))
    out = sm.PageTable(piece(4), piece(3), piece(15), piece(15), buf[89:90])
    want = P.page_table([5, 0, 9], [2, 3, 9], list(range(50, 60)), 10, table.cpu().numpy(), 8, 64, 15)
    sm.page_table(cached, fresh, free, n_free, table, 8, 64, 15, out=out)
    assert (table.cpu().numpy() == want[0]).all() and all((g.cpu().numpy() == w).all() for g, w in zip(out, want[1:]))
    assert (buf[at[0]:] == -9).all() and (buf[4:30] == -9).all()
    with pytest.raises(sm.SmError, match="overlap"):
        sm.page_table(out.lens, fresh, free, n_free, table, 8, 64, 15, out=out)      # (the next iteration needs other outputs)


def test_page_table_counts_at_the_limits():
    """Lengths and capacities at 2^30, where sums of two of them do not fit 31 bits."""
    big = 2 ** 30
    i = 2 ** 31 - 1
    out = sm.page_table(ints([i, 5]), ints([i, i]), ints([0]), ints([1]), ints([[0], [0]]), big, 1, 300)
    # the first request's row is full; all 300 rows are its tokens, without a slot; the second keeps its five
    assert out.starts.tolist() == [0, 300, 300] and out.lens.tolist() == [big, 5] and out.need.item() == 0
    assert (out.slots == -1).all() and out.positions[:2].tolist() == [big, big + 1] and out.positions[299].item() == big + 299
    out = sm.page_table(ints([0, big - 2]), ints([3, i]), ints([]), ints([i]), ints([[0], [0]]), big, 1, 8)
    assert out.starts.tolist() == [0, 3, 8] and out.lens.tolist() == [0, big] and out.need.item() == 1
    assert out.slots.tolist() == [-1, -1, -1, big - 2, big - 1, -1, -1, -1]


# ------------------------------------------------------------------------------------------------ norm + rotation + store

def head_norm_case(T, hq, hkv, d, rot, norm, dtype, paged=True, seed=0, page=16, base=10000.0, far=0, head_major=False, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn(T, hq + 2 * hkv + 1, d, generator=g) + mean).to(dtype)          # (one head more: rows with a gap)
    gam = {n: (1 + 0.2 * torch.randn(d, generator=g)).to(dtype) for n in ("q_gamma", "k_gamma")} if norm != "none" else {}
    bet = {n: (0.5 * torch.randn(d, generator=g)).to(dtype) for n in ("q_beta", "k_beta")} if norm == "layer" else {}
    pos = torch.randint(0, 3000, (T,), generator=g) + far
    n_pages = -(-T // page) + 2
    slots = torch.randperm(n_pages * page, generator=g)[:T]
    if T > 3:
        pos[2], slots[3] = -1, -1
        slots[1] = n_pages * page                                                     # just behind the pool
    fill = 77.0
    shape = (n_pages, hkv, page, d) if head_major else (n_pages, page, hkv, d)
    kp, vp = (torch.full(shape, fill, dtype=dtype, device="cuda") for _ in range(2))
    x = qkv.cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:hq + 2 * hkv]
    q_out = torch.full((T, hq, d), fill, dtype=dtype, device="cuda")
    kw = dict(norm=norm, rot=rot, rope_base=base, q_out=q_out, **{n: t.cuda() for n, t in {**gam, **bet}.items()})
    view = (lambda t: t.permute(0, 2, 1, 3)) if head_major else (lambda t: t)
    if paged:
        sm.head_norm_rope(q, k, v, pos.to(I32).cuda(), slots=slots.to(I32).cuda(), k_out=view(kp), v_out=view(vp), **kw)
        ko, vo = view(kp), view(vp)
    else:
        ko, vo = (torch.full((T, hkv, d), fill, dtype=dtype, device="cuda") for _ in range(2))
        sm.head_norm_rope(q, k, v, pos.to(I32).cuda(), k_out=ko, v_out=vo, **kw)
    torch.cuda.synchronize()
    xn = to_np(qkv)
    live = pos.numpy() >= 0
    for n, part, got in (("q", xn[:, :hq], q_out), ("k", xn[:, hq:hq + hkv], ko)):
        gamma, beta = (to_np(kw[n + s]) if n + s in kw else None for s in ("_gamma", "_beta"))
        normed = P.head_norm(part, norm, gamma, beta, 1e-5)
        want = P.rope(normed, pos.numpy(), rot, base)
        # the largest value on the way: x itself (before the mean is taken off) and the shift
        r = 1.0 if norm == "none" else np.abs(gamma).max() / np.sqrt(part.var(-1, keepdims=True) if norm == "layer" else (part ** 2).mean(-1, keepdims=True))
        big = np.abs(part).max(-1, keepdims=True) * r + (np.abs(beta).max() if beta is not None else 0)
        pair = np.abs(normed).max(-1, keepdims=True) * 2 * (2.0 ** -20 + 2 * np.pi * 2.0 ** -25 if dtype == BF16 else 2.0 ** -22 + 2 * np.pi * 2.0 ** -25)
        tol = HALF[dtype] * np.abs(want) + 40 * 2.0 ** -24 * big + (pair if rot else 0)
        if n == "q" or not paged:
            full, ft = np.full(got.shape, fill), np.zeros(got.shape)
            full[live], ft[live] = want[live], tol[live]
            check(got, full, ft, n)
        else:
            full, ft = np.full((n_pages * page, hkv, d), fill), np.zeros((n_pages * page, hkv, d))
            ok = live & (slots.numpy() >= 0) & (slots.numpy() < n_pages * page)
            full[slots.numpy()[ok]], ft[slots.numpy()[ok]] = want[ok], tol[ok]
            check(got, full.reshape(n_pages, page, hkv, d), ft.reshape(n_pages, page, hkv, d), n)
    vw = xn[:, hq + hkv:hq + 2 * hkv]
    if paged:
        full = np.full((n_pages * page, hkv, d), fill)
        full[slots.numpy()[ok]] = vw[ok]
        assert (to_np(vo).reshape(-1, hkv, d) == full).all()
    else:
        full = np.full((T, hkv, d), fill)
        full[live] = vw[live]
        assert (to_np(vo) == full).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("norm", ["rms", "layer", "none"])
@pytest.mark.parametrize("T,hq,hkv,d,rot", [(1, 1, 1, 64, 64), (5, 8, 2, 128, 128), (3, 3, 1, 96, 96), (7, 5, 5, 80, 32), (4, 2, 1, 256, 64),
                                            (6, 4, 4, 256, 256), (2, 7, 1, 16, 16), (33, 2, 2, 72, 16), (130, 12, 4, 64, 0)])
def test_head_norm_rope(T, hq, hkv, d, rot, norm, dtype):
    head_norm_case(T, hq, hkv, d, rot, norm, dtype, seed=T + d, head_major=T % 2 == 0, page=1 + T % 16)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_head_norm_rope_plain_rows_and_far_positions(dtype):
    head_norm_case(9, 6, 2, 128, 128, "rms", dtype, paged=False)
    head_norm_case(9, 6, 2, 64, 64, "none", dtype, paged=False, far=2 ** 31 - 3001)
    head_norm_case(700, 4, 1, 128, 64, "rms", dtype, far=1000000, base=5e5, page=64)
    head_norm_case(5, 4, 1, 64, 64, "layer", dtype, mean=30.0)                      # a mean that has to be taken off before squaring
    head_norm_case(1500, 2, 1, 128, 128, "rms", dtype, page=8)


@pytest.mark.parametrize("T", [767, 768, 900])
def test_head_norm_rope_around_the_change_of_form(T):
    """A token for four waves, or for one: the same results, in place and with parts left out as well."""
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, 7, 96, generator=g).to(BF16).cuda()
    gq, gk = (1 + 0.1 * torch.randn(2, 96, generator=g)).to(BF16).cuda()
    pos = torch.randint(0, 9999, (T,), generator=g).to(I32).cuda()
    pos[5] = -3
    kw = dict(q_gamma=gq, k_gamma=gk, rot=32)
    fill = [torch.zeros(T, n, 96, dtype=BF16, device="cuda") for n in (4, 1, 1)]
    q, k, v = sm.head_norm_rope(x[:, :4], x[:, 4:5], x[:, 5:6], pos, q_out=fill[0], k_out=fill[1], v_out=fill[2], **kw)
    for part in (slice(0, 300), slice(300, T)):                      # the few-token form, in two pieces
        f = [torch.zeros(pos[part].shape[0], n, 96, dtype=BF16, device="cuda") for n in (4, 1, 1)]
        got = sm.head_norm_rope(x[part, :4], x[part, 4:5], x[part, 5:6], pos[part], q_out=f[0], k_out=f[1], v_out=f[2], **kw)
        assert all(torch.equal(a, b[part]) for a, b in zip(got, (q, k, v)))
    k2 = sm.head_norm_rope(None, x[:, 4:5], None, pos, k_out=torch.zeros_like(k), **kw)[1]
    assert torch.equal(k2, k)
    y = x.clone()
    sm.head_norm_rope(y[:, :4], y[:, 4:5], y[:, 5:6], pos, q_out=y[:, :4], k_out=y[:, 4:5], v_out=y[:, 5:6], **kw)
    live = pos >= 0
    assert torch.equal(y[live][:, :4], q[live]) and torch.equal(y[live][:, 4:5], k[live]) and torch.equal(y[~live], x[~live]) and torch.equal(y[:, 6], x[:, 6])


def test_head_norm_rope_parts_in_place_and_empty():
    x = torch.randn(6, 4, 64, device="cuda")
    g = torch.ones(64, device="cuda")
    pos = torch.arange(6, dtype=I32, device="cuda")
    q, _, _ = sm.head_norm_rope(x, None, None, pos, q_gamma=g)
    _, k, _ = sm.head_norm_rope(None, x, None, pos, k_gamma=g)
    assert torch.equal(q, k)
    _, _, v = sm.head_norm_rope(None, None, x, pos)
    assert torch.equal(v, x)
    y = x.clone()
    sm.head_norm_rope(y, None, None, pos, q_gamma=g, q_out=y)
    assert torch.equal(y, q)
    out = sm.head_norm_rope(x[:0], x[:0], x[:0], pos[:0], q_gamma=g, k_gamma=g)
    assert [t.shape[0] for t in out] == [0, 0, 0]
    # zeros: the norm of a zero head is zero (eps), infinities and NaN stay in their head
    z = torch.zeros(2, 2, 64, device="cuda")
    z[0, 1, 3], z[1, 0, 5] = float("inf"), float("nan")
    o, _, _ = sm.head_norm_rope(z, None, None, pos[:2], q_gamma=g)
    assert not o[0, 0].any() and not o[1, 1].any() and not o[0, 1].isfinite().all() and o[1, 0].isnan().all()


@pytest.mark.parametrize("T", [6, 900])
def test_head_norm_rope_queries_alone_beside_slots(T):
    """Slots name places of keys and values; queries by themselves go to their rows whatever the slots say."""
    g = torch.Generator().manual_seed(T)
    q, gain, pos = torch.randn(T, 3, 64, generator=g).cuda(), torch.ones(64, device="cuda"), torch.arange(T, dtype=I32, device="cuda")
    slots = torch.arange(T, dtype=I32, device="cuda") - 2
    got = sm.head_norm_rope(q, None, None, pos, q_gamma=gain, slots=slots)
    assert torch.equal(got[0], sm.head_norm_rope(q, None, None, pos, q_gamma=gain)[0]) and got[1] is None and got[2] is None


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [5, 900])
@pytest.mark.parametrize("d, rot", [(64, 32), (128, 32), (128, 96), (256, 64), (96, 0)])
def test_head_norm_rope_features_behind_the_rotation_are_their_own(d, rot, T, dtype):
    """Without a norm they leave as they came, whatever they are; with one, an infinity gives NaN in its own place and 0 in the others."""
    g = torch.Generator().manual_seed(d + rot)
    x = torch.randn(T, 3, d, generator=g).to(dtype).cuda()
    x[1, 1, rot:] = float("inf")
    x[2, 0, rot + 3], x[2, 1, d - 1], x[2, 2, d - 9], x[3, 0, rot] = float("nan"), float("-inf"), float("inf"), -0.0
    pos = torch.arange(T, dtype=I32, device="cuda") + 7
    clean = x.clone()
    clean[:, :, rot:] = 0
    got, want = sm.head_norm_rope(x, None, None, pos, norm="none", rot=rot)[0], sm.head_norm_rope(clean, None, None, pos, norm="none", rot=rot)[0]
    as_int = torch.int16 if dtype == BF16 else I32
    assert torch.equal(got[:, :, rot:].contiguous().view(as_int), x[:, :, rot:].contiguous().view(as_int)) and torch.equal(got[:, :, :rot], want[:, :, :rot])
    o = sm.head_norm_rope(x, None, None, pos, rot=rot, q_gamma=torch.ones(d, dtype=dtype, device="cuda"))[0]
    assert o[2, 1, d - 1].isnan() and not o[2, 1, :d - 1].any() and o[2, 0].isnan().all()


# ------------------------------------------------------------------------------------------------ attention

def attn_case(lens, hq, hkv, d, page, dtype, seed=0, head_major=False, spare_cols=1, q_scale=1.0, scale=None, bad=(), poison=True, values=None):
    g = torch.Generator().manual_seed(seed)
    R = len(lens)
    cols = max(1, max(-(-max(n, 0) // page) for n in lens) + spare_cols)
    held = [min(cols, -(-max(n, 0) // page)) for n in lens]
    n_pages = sum(held) + 3
    ids = torch.randperm(n_pages, generator=g).tolist()
    table = np.full((R, cols + 1), 10 ** 9)                        # (entries behind a request's pages are no page at all)
    kp, vp = torch.randn(2, n_pages, page, hkv, d, generator=g)
    if poison:                                                     # places behind the last token, and pages of nobody
        kp[ids[-3]:ids[-3] + 1], vp[ids[-3]:ids[-3] + 1] = float("nan"), float("inf")
    at = 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
        n = min(max(lens[r], 0), cols * page)
        if poison and n % page:
            kp[table[r, held[r] - 1], n % page:], vp[table[r, held[r] - 1], n % page:] = float("nan"), float("-inf")
    for r, c, e in bad:
        table[r, c] = e
    kp, vp = kp.to(dtype), vp.to(dtype)
    q = (torch.randn(R, hq + 1, d, generator=g) * q_scale).to(dtype)
    s = d ** -0.5 if scale is None else scale
    o, lse, av, aw = P.paged_attention(to_np(q)[:, :hq], to_np(kp), to_np(vp), table[:, :cols], lens, s, want_bound=True)
    if head_major:
        kd, vd = (t.transpose(1, 2).contiguous().cuda().transpose(1, 2) for t in (kp, vp))
    else:
        kd, vd = kp.cuda(), vp.cuda()
    att = sm.PagedAttention(R, hq, hkv, d, page, cols, n_pages, dtype, scale=s)
    att.ws.fill_(0xff)                                             # nothing in the workspace is taken for granted (NaN everywhere)
    lse_d = torch.full((R, hq), 5.0, device="cuda")
    out = torch.full((R, hq + 2, d), 9.0, dtype=dtype, device="cuda")
    att(q.cuda()[:, :hq], kd, vd, ints(table)[:, :cols], ints(lens), out=out[:, 1:hq + 1], lse=lse_d)
    torch.cuda.synchronize()
    assert (out[:, 0] == 9).all() and (out[:, hq + 1] == 9).all()
    n = max(max(lens), 1)
    score = (d + 4) * 2.0 ** -24 * aw + (np.abs(np.where(np.isfinite(lse), lse, 0))[..., None] + 4) * 2.0 ** -23
    weight = (2.0 ** -16 if dtype == BF16 else 2.0 ** -22) + (n / 16 + 64) * 2.0 ** -24
    check(out[:, 1:hq + 1], o, HALF[dtype] * np.abs(o) + (2 * score + weight) * av, "o")
    fin = np.isfinite(lse)
    assert (to_np(lse_d)[~fin] == -np.inf).all() and (to_np(out[:, 1:hq + 1])[~fin] == 0).all()
    check(lse_d[torch.from_numpy(fin).cuda()], lse[fin], (2 * score[..., 0] + weight + 2.0 ** -22 * (1 + np.abs(np.where(fin, lse, 0))))[fin], "lse")


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 64), (4, 2, 128), (3, 1, 256), (16, 1, 64), (17, 1, 128), (10, 2, 96), (4, 4, 32), (8, 8, 8), (33, 1, 72), (5, 5, 248)])
def test_paged_attention_heads(hq, hkv, d, dtype):
    attn_case(LENS, hq, hkv, d, 16, dtype, seed=hq + d)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [1, 2, 3, 5, 8, 16, 24, 32, 48, 64, 100, 256])
def test_paged_attention_pages(page, dtype):
    attn_case(LENS + [4 * page, 4 * page + 1, 300], 4, 2, 64, page, dtype, seed=page, head_major=page % 2 == 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,hq,hkv,d,page", [([5000], 8, 2, 128, 16), ([4097], 2, 2, 256, 64), ([1, 3000, 0, 7, 2047], 4, 1, 64, 8),
                                                ([20000, 3], 2, 1, 64, 32), ([700] * 40, 4, 2, 64, 16), (list(range(300)), 2, 1, 32, 16)])
def test_paged_attention_long_and_many(lens, hq, hkv, d, page, dtype):
    attn_case(lens, hq, hkv, d, page, dtype, seed=len(lens))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_paged_attention_pages_that_are_not_there(dtype):
    """Entries outside the pool stand for no page: their keys are left out; a request without any page gets zero and -inf."""
    attn_case([100, 50, 16, 2000], 4, 2, 64, 16, dtype, bad=[(0, 0, -1), (0, 3, 10 ** 9), (1, 1, -2 ** 31), (2, 0, 2 ** 31 - 1), (3, 70, -5), (3, 0, 10 ** 6)])
    attn_case([40, 64], 4, 2, 64, 8, dtype, bad=[(0, c, -1) for c in range(5)] + [(1, c, 10 ** 7) for c in range(8)])


def test_paged_attention_lengths_outside_the_table():
    for dtype in (BF16, F32):
        attn_case([-3, 70, 2 ** 31 - 1, -2 ** 31][:2], 2, 1, 64, 16, dtype)
    # lengths past the row end at the row's end
    kp, vp = torch.randn(2, 8, 16, 1, 64, device="cuda")
    q, t = torch.randn(3, 2, 64, device="cuda"), ints([[0, 1], [2, 3], [4, 5]])
    att = sm.PagedAttention(3, 2, 1, 64, 16, 2, 8, F32)
    assert torch.equal(att(q, kp, vp, t, ints([32, 33, 2 ** 31 - 1])), att(q, kp, vp, t, ints([32, 32, 32])))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_paged_attention_scales(dtype):
    attn_case([300, 40], 4, 2, 64, 16, dtype, scale=0.0)
    attn_case([300, 40], 4, 2, 64, 16, dtype, scale=-0.2)
    attn_case([300, 700], 4, 2, 64, 16, dtype, q_scale=12.0)                # one key takes nearly all of the weight


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_paged_attention_infinite_and_nan_keys_stay_in_their_request(dtype):
    g = torch.Generator().manual_seed(5)
    kp, vp = torch.randn(2, 60, 16, 1, 64, generator=g).to(dtype).cuda()
    q = torch.randn(3, 2, 64, generator=g).to(dtype).cuda()
    table = ints(np.arange(60).reshape(3, 20).tolist())
    att = sm.PagedAttention(3, 2, 1, 64, 16, 20, 60, dtype)
    lens = ints([300, 300, 300])
    want = att(q, kp, vp, table, lens).clone()
    kp[21, 3] = float("nan")
    vp[45, 3] = float("inf")
    got = att(q, kp, vp, table, lens)
    assert torch.equal(got[0], want[0]) and got[1].isnan().all() and (got[2] == float("inf")).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("n", [1, 200, 300, 5000])
def test_paged_attention_nan_queries_and_keys_without_weight(n, d, dtype):
    """A request whose every logit is NaN gives NaN, not the zero of an empty one; keys whose logit is -inf weigh nothing, and where
    there are no others the request counts as empty."""
    g = torch.Generator().manual_seed(7)
    mp = (n + 15) // 16
    kp, vp = torch.randn(2, 4 * mp, 16, 1, d, generator=g).to(dtype).cuda()
    q = torch.randn(4, 2, d, generator=g).to(dtype).cuda()
    q[:, :, 3] = 1.0
    table = ints(np.arange(4 * mp).reshape(4, mp).tolist())
    att = sm.PagedAttention(4, 2, 1, d, 16, mp, 4 * mp, dtype)
    lens = ints([n] * 4)
    want = att(q, kp, vp, table, lens).clone()
    q[1, 1] = float("nan")
    kp[2 * mp:3 * mp, :, :, 3] = float("-inf")
    kp[3 * mp:].view(-1, d)[:n - 1, 3] = float("-inf")              # the last key alone has a weight
    lse = torch.empty(4, 2, device="cuda")
    got = att(q, kp, vp, table, lens, lse=lse)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1, 0], want[1, 0])
    assert got[1, 1].isnan().all() and lse[1, 1].isnan() and lse[1, 0].isfinite()
    assert not got[2].any() and (lse[2] == float("-inf")).all()
    last = vp[3 * mp:].view(-1, d)[n - 1]
    assert torch.equal(got[3], torch.stack([last, last])) and lse[3].isfinite().all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [2, 200, 1000])
def test_paged_attention_largest_values_of_keys_without_weight(n, d, dtype):
    """A key whose weight is zero (e^-256 of the first one's) adds nothing, however large its finite value is."""
    mp = (n + 15) // 16
    kp, vp = torch.zeros(2, mp, 16, 1, d, dtype=dtype, device="cuda")
    kp.view(-1, d)[1:, 0] = -256.0
    vp.view(-1, d)[1:] = torch.finfo(dtype).max
    vp.view(-1, d)[2::2] *= -1
    vp.view(-1, d)[0] = 1.5
    q = torch.zeros(1, 2, d, dtype=dtype, device="cuda")
    q[:, :, 0] = 1.0
    got = sm.PagedAttention(1, 2, 1, d, 16, mp, mp, dtype, scale=1.0)(q, kp, vp, torch.arange(mp, dtype=I32, device="cuda")[None], ints([n]))
    assert (got == 1.5).all(), got.unique().tolist()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [2, 200, 1000, 20000])
def test_paged_attention_values_whose_sum_is_no_float(n, d, dtype):
    """n equal weights on n values of half the type's largest: the mean is that value, which no rounding on the way leaves by more than
    (n / 16 + 64) 2^-24 (the blocks of the sums), though n times it is past the largest fp32 number."""
    mp = (n + 15) // 16
    kp, vp = torch.zeros(2, mp, 16, 1, d, dtype=dtype, device="cuda")
    vp.view(-1, d)[:n] = torch.finfo(dtype).max / 2
    q = torch.zeros(1, 2, d, dtype=dtype, device="cuda")
    got = sm.PagedAttention(1, 2, 1, d, 16, mp, mp, dtype)(q, kp, vp, torch.arange(mp, dtype=I32, device="cuda")[None], ints([n]))
    want = vp[0, 0, 0, 0].double()
    assert (got.double() / want - 1).abs().max() <= HALF[dtype] + (n / 16 + 64) * 2.0 ** -24


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("low", [-60, -100, -115, -126])
def test_paged_attention_smallest_values(low, dtype):
    """Values around 2^low: on top of the usual rounding a sum's steps are no finer than 2^-129, as are those of a bf16 result below 2^-126 (2^-133)."""
    g = torch.Generator().manual_seed(-low)
    n, d = 500, 64
    kp, vp = torch.randn(32, 16, 1, d, generator=g).to(dtype), (torch.randn(32, 16, 1, d, generator=g).double() * 2.0 ** low).to(dtype)
    q = torch.randn(1, 4, d, generator=g).to(dtype)
    ids = torch.randperm(32, generator=g)[None]
    o, lse, av, aw = P.paged_attention(to_np(q), to_np(kp), to_np(vp), ids.numpy(), [n], 0.125, want_bound=True)
    got = sm.PagedAttention(1, 4, 1, d, 16, 32, 32, dtype, scale=0.125)(q.cuda(), kp.cuda(), vp.cuda(), ids.to(I32).cuda(), ints([n]))
    score = (d + 4) * 2.0 ** -24 * aw + (np.abs(lse)[..., None] + 4) * 2.0 ** -23
    tol = HALF[dtype] * np.abs(o) + (2 * score + 2.0 ** -22 + (n / 16 + 64) * 2.0 ** -24) * av + (n / 16 + 64) * 2.0 ** -130 + 2.0 ** -134
    check(got, o, tol, "o")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_paged_attention_weights_carry_fp32(d, dtype):
    """Two keys with values 1 and -1 and logits 0 and -x: the result is tanh(x / 2), a difference of weights near 1 that shows what each of
    them has lost.  The smaller weight comes from its logit times log2 e and an exponential of one unit in the last place (2^-24 both, as
    x < 2^-10), and may lose 2^-23 when it is split; the larger is 1.  Half of that error is the result's: 2^-23, then the store."""
    x = (torch.arange(129, 257, 2).view(4, 16) * 2.0 ** -19).to(dtype).cuda()              # (eight bits: a bf16 each; bits down to 2^-19 in the weight)
    q = torch.zeros(4, 16, d, dtype=dtype, device="cuda")
    q[:, :, 0] = x
    kp, vp = torch.zeros(2, 1, 16, 1, d, dtype=dtype, device="cuda")
    kp[0, 1, 0, 0], vp[0, 0], vp[0, 1] = -1.0, 1.0, -1.0
    got = sm.PagedAttention(4, 16, 1, d, 16, 1, 1, dtype, scale=1.0)(q, kp, vp, ints([[0]] * 4), ints([2] * 4))
    want = torch.tanh(x.double() / 2)[..., None].expand(4, 16, d)
    check(got, to_np(want), HALF[dtype] * np.abs(to_np(want)) + 2.0 ** -23, "o")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R", [64, 65, 256, 257, 1500])
def test_paged_attention_many_requests(R, dtype):
    """Several requests per lane of the scan that cuts the work, empty ones among them."""
    rng = np.random.default_rng(R)
    lens = (rng.integers(0, 400, R) * (rng.random(R) < 0.7)).tolist()
    lens[R // 2], lens[-1] = 3000, 1
    attn_case(lens, 2, 1, 32, 16, dtype, seed=R)


def test_paged_attention_pools_of_different_layouts():
    """Keys head-major, values token-major with a gap between heads, one page as long as the whole request."""
    g = torch.Generator().manual_seed(12)
    for dtype, page, n in ((BF16, 16, 200), (F32, 700, 650)):
        cols = -(-n // page)
        ids = torch.randperm(cols + 2, generator=g)[:cols].tolist()
        kp = torch.randn(cols + 2, 3, page, 64, generator=g).to(dtype)
        vp = torch.randn(cols + 2, page, 3, 2, 64, generator=g).to(dtype)
        q = torch.randn(1, 6, 64, generator=g).to(dtype)
        o, _, av, aw = P.paged_attention(to_np(q), to_np(kp.transpose(1, 2)), to_np(vp[:, :, :, 1]), np.array([ids]), [n], 0.125, want_bound=True)
        got = sm.PagedAttention(1, 6, 3, 64, page, cols, cols + 2, dtype)(q.cuda(), kp.cuda().transpose(1, 2), vp.cuda()[:, :, :, 1], ints([ids]), ints([n]))
        check(got, o, HALF[dtype] * np.abs(o) + (2 * (68 * 2.0 ** -24 * aw + 2.0 ** -20) + 2.0 ** -16) * av, "o")


def test_paged_attention_captured_with_short_and_replayed_with_long_requests():
    g = torch.Generator().manual_seed(13)
    kp, vp = torch.randn(2, 300, 16, 2, 64, generator=g).to(BF16).cuda()
    q = torch.randn(3, 4, 64, generator=g).to(BF16).cuda()
    table = torch.randperm(300, generator=g).to(I32).cuda().reshape(3, 100)
    att, eager = (sm.PagedAttention(3, 4, 2, 64, 16, 100, 300, BF16) for _ in range(2))
    lens = ints([1, 0, 2])
    out, lse = att(q, kp, vp, table, lens).clone(), torch.empty(3, 4, device="cuda")
    torch.cuda.synchronize()
    cg = torch.cuda.CUDAGraph()
    with torch.cuda.graph(cg):
        att(q, kp, vp, table, lens, out=out, lse=lse)
    for now in ([1600, 0, 777], [0, 0, 0], [3, 1599, 128], [129, 128, 127], [1600, 1600, 1600]):
        lens.copy_(ints(now))
        cg.replay()
        torch.cuda.synchronize()
        want_lse = torch.empty_like(lse)
        want = eager(q, kp, vp, table, ints(now), lse=want_lse)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), now


def test_results_over_parts_of_a_cache_join_by_their_lse():
    """The even and the odd pages apart, joined by lse, are the whole."""
    g = torch.Generator().manual_seed(14)
    kp, vp = torch.randn(2, 40, 16, 1, 128, generator=g).cuda()
    q = torch.randn(1, 4, 128, generator=g).cuda()
    row = torch.randperm(40, generator=g).to(I32).cuda()[None]
    parts = [sm.PagedAttention(1, 4, 1, 128, 16, n, 40, F32) for n in (40, 20, 20)]
    lse = [torch.empty(1, 4, device="cuda") for _ in parts]
    o = [a(q, kp, vp, t.contiguous(), ints([16 * t.shape[1]]), lse=l).double() for a, t, l in zip(parts, (row, row[:, ::2], row[:, 1::2]), lse)]
    w = torch.softmax(torch.stack(lse[1:]).double(), 0)[..., None]
    assert (w[0] * o[1] + w[1] * o[2] - o[0]).abs().max() < 2e-5
    assert (torch.logsumexp(torch.stack(lse[1:]).double(), 0) - lse[0].double()).abs().max() < 1e-5


def test_paged_attention_without_requests():
    att = sm.PagedAttention(0, 4, 2, 64, 16, 4, 8, BF16)
    kp = torch.zeros(8, 16, 2, 64, dtype=BF16, device="cuda")
    e = torch.zeros(0, 4, 64, dtype=BF16, device="cuda")
    assert att(e, kp, kp, torch.zeros(0, 4, dtype=I32, device="cuda"), torch.zeros(0, dtype=I32, device="cuda")).shape == (0, 4, 64)


def test_paged_attention_offsets_past_32_bits():
    """A pool of more than 2^31 elements, only its last pages used."""
    n_pages, page, hkv, d = 70000, 16, 8, 256
    pool = torch.empty(n_pages, page, hkv, d, dtype=BF16, device="cuda")
    assert pool.numel() > 2 ** 31
    small = torch.randn(4, page, hkv, d, device="cuda").to(BF16)
    pool[-4:] = small
    q = torch.randn(2, 8, d, device="cuda").to(BF16)
    lens = ints([20, 32])
    big = sm.PagedAttention(2, 8, hkv, d, page, 2, n_pages, BF16)(q, pool, pool, ints([[69999, 69997], [69996, 69998]]), lens)
    want = sm.PagedAttention(2, 8, hkv, d, page, 2, 4, BF16)(q, small, small, ints([[3, 1], [0, 2]]), lens)
    assert torch.equal(big, want)
    # and the store into it
    x = torch.randn(3, hkv, d, device="cuda").to(BF16)
    slots = [69999 * 16 + 5, 69996 * 16, 0]
    sm.head_norm_rope(None, x, x, ints([0, 0, 0]), norm="none", rot=0, slots=ints(slots), k_out=pool, v_out=pool)
    assert torch.equal(pool.view(-1, hkv, d)[slots], x)


def test_paged_attention_is_deterministic_and_free_of_its_neighbours():
    """The same call gives the same bits; what other requests are in the batch, in the same number of tokens, changes rounding only."""
    g = torch.Generator().manual_seed(6)
    kp, vp = torch.randn(2, 400, 16, 2, 128, generator=g).to(BF16).cuda()
    q = torch.randn(4, 8, 128, generator=g).to(BF16).cuda()
    table = torch.randperm(400, generator=g).to(I32).cuda().reshape(4, 100)
    att = sm.PagedAttention(4, 8, 2, 128, 16, 100, 400, BF16)
    lens = ints([1600, 900, 3, 0])
    a = att(q, kp, vp, table, lens).clone()
    for _ in range(5):
        assert torch.equal(att(q, kp, vp, table, lens), a)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_paged_attention_of_a_request_beside_others(dtype):
    """The other lengths of a batch decide how long a chunk is: alone (one unit), among empty and short requests, beside one of 60000 keys (two units)
    and one of 400000 (the longest chunk).  The request's result stays the oracle's within the rounding of its sums."""
    g = torch.Generator().manual_seed(19)
    n, hq, hkv, d, page, n_pages = 1600, 4, 2, 64, 16, 150
    kp, vp = torch.randn(2, n_pages, page, hkv, d, generator=g).to(dtype)
    q1, row = torch.randn(1, hq, d, generator=g).to(dtype), torch.randperm(n_pages, generator=g)[:100]
    o, lse, av, aw = P.paged_attention(to_np(q1), to_np(kp), to_np(vp), row[None].numpy(), [n], d ** -0.5, want_bound=True)
    score = (d + 4) * 2.0 ** -24 * aw + (np.abs(lse)[..., None] + 4) * 2.0 ** -23
    weight = 2.0 ** -22 + (n / 16 + 64) * 2.0 ** -24
    kd, vd = kp.cuda(), vp.cuda()
    for others in ([], [0, 1, 17, 0, 300, 5] * 5, [60000], [3, 400000], [-2 ** 31, 2 ** 31 - 1, 200]):
        lens = others[:len(others) // 2] + [n] + others[len(others) // 2:]
        r, R = len(others) // 2, len(lens)
        cols = max(-(-min(max(x, 0), 10 ** 6) // page) for x in lens)              # (a length past the row ends at its end)
        table = torch.randint(0, n_pages, (R, cols), generator=g)
        table[r, :100] = row
        q = torch.randn(R, hq, d, generator=g).to(dtype)
        q[r] = q1[0]
        got_lse = torch.empty(R, hq, device="cuda")
        got = sm.PagedAttention(R, hq, hkv, d, page, cols, n_pages, dtype)(q.cuda(), kd, vd, table.to(I32).cuda(), ints(lens), lse=got_lse)
        check(got[r:r + 1], o, HALF[dtype] * np.abs(o) + (2 * score + weight) * av, "o beside %s" % others)
        check(got_lse[r:r + 1], lse, 2 * score[..., 0] + weight + 2.0 ** -22 * (1 + np.abs(lse)), "lse beside %s" % others)
        for i, x in enumerate(lens):
            assert (x > 0) == got_lse[i].isfinite().all().item() and (x > 0 or not got[i].any() and (got_lse[i] == -np.inf).all())


def test_objects_made_while_a_graph_is_captured():
    """Workspace and packed weights are the graph's; replays on other lengths, eager calls of other objects in between."""
    g = torch.Generator().manual_seed(20)
    kp, vp = torch.randn(2, 200, 16, 2, 64, generator=g).to(BF16).cuda()
    q, table = torch.randn(2, 4, 64, generator=g).to(BF16).cuda(), torch.randperm(200, generator=g).to(I32).cuda().reshape(2, 100)
    w, sc = torch.randint(0, 256, (48, 128), generator=g, dtype=torch.uint8).cuda(), torch.rand(48, 2, generator=g).to(BF16).cuda()
    lens = ints([0, 0])
    eager, lin = sm.PagedAttention(2, 4, 2, 64, 16, 100, 200, BF16), sm.LinearW4(w, sc)
    torch.cuda.synchronize()
    cg = torch.cuda.CUDAGraph()
    with torch.cuda.graph(cg):
        a, b = sm.PagedAttention(2, 4, 2, 64, 16, 100, 200, BF16), sm.LinearW4(w, sc)
        o = a(q, kp, vp, table, lens)
        y = b(o.view(2, 256))
    for now in ([1600, 3], [0, 700], [1600, 1600]):
        lens.copy_(ints(now))
        cg.replay()
        torch.cuda.synchronize()
        want = eager(q, kp, vp, table, lens)
        assert torch.equal(o, want) and torch.equal(y, lin(want.view(2, 256)))


# ------------------------------------------------------------------------------------------------ together

def serve(E, hq, hkv, d, page, dtype, prompts, steps, graph=False):
    """Prompts of ragged lengths, then decode iterations: pages, projection, norm + rotation + store, attention, output Linear; the
    attention's result compared with a full causal softmax over the whole sequence in float64."""
    g = torch.Generator().manual_seed(E + hq)
    R = len(prompts)
    w = {n: (torch.randn(o, i, generator=g) * i ** -0.5).to(dtype).cuda() for n, o, i in (("qkv", (hq + 2 * hkv) * d, E), ("out", E, hq * d))}
    qg, kg = ((1 + 0.1 * torch.randn(d, generator=g)).to(dtype).cuda() for _ in range(2))
    total = [p + steps for p in prompts]
    cols = max(-(-n // page) for n in total) + 1
    n_pages = sum(-(-n // page) for n in total) + 2
    free = torch.randperm(n_pages, generator=g).to(I32).cuda()
    kp, vp = (torch.full((n_pages, page, hkv, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    table = torch.full((R, cols), -1, dtype=I32, device="cuda")
    x_all = torch.randn(R, max(total), E, generator=g).to(dtype).cuda()
    att = sm.PagedAttention(R, hq, hkv, d, page, cols, n_pages, dtype)

    def project(x):
        return sm.linear(x, w["qkv"]).view(-1, hq + 2 * hkv, d)

    def rows(x, pt):
        y = project(x)
        return sm.head_norm_rope(y[:, :hq], y[:, hq:hq + hkv], y[:, hq + hkv:], pt.positions, q_gamma=qg, k_gamma=kg, slots=pt.slots, k_out=kp, v_out=vp)[0]

    cached, taken = torch.zeros(R, dtype=I32, device="cuda"), 0
    T = sum(prompts) + 3                                              # (padding rows)
    x = torch.zeros(T, E, dtype=dtype, device="cuda")
    x[:T - 3] = torch.cat([x_all[r, :p] for r, p in enumerate(prompts)])
    pt = sm.page_table(cached, ints(prompts), free, ints([n_pages]), table, page, n_pages, T)
    rows(x, pt)
    cached, taken = pt.lens, pt.need.item()
    qkv64 = to_np(torch.cat([project(x_all[r, :n].contiguous()) for r, n in enumerate(total)]))
    at = np.cumsum([0] + total)
    fresh = ints([1] * R)

    def step(x, cached, free, n_free):
        pt = sm.page_table(cached, fresh, free, n_free, table, page, n_pages, R)
        q = rows(x, pt)
        o = att(q, kp, vp, table, pt.lens)
        return pt, o, sm.linear(o.view(R, hq * d), w["out"])

    if graph:                                                         # static inputs, one captured iteration, replayed
        sx, sc, sf, sn = torch.zeros(R, E, dtype=dtype, device="cuda"), cached.clone(), torch.zeros_like(free), ints([0])
        torch.cuda.synchronize()
        cg = torch.cuda.CUDAGraph()
        with torch.cuda.graph(cg):
            spt, so, sy = step(sx, sc, sf, sn)
    for i in range(steps):
        xi = torch.stack([x_all[r, p + i] for r, p in enumerate(prompts)])
        if graph:
            sx.copy_(xi)
            sc.copy_(cached)
            sf[:n_pages - taken].copy_(free[taken:])
            sn.fill_(n_pages - taken)
            cg.replay()
            torch.cuda.synchronize()
            pt, o, y = spt, so.clone(), sy.clone()
            before = kp.clone(), vp.clone(), table.clone()
            pe, oe, ye = step(xi, cached, free[taken:].contiguous(), ints([n_pages - taken]))       # the same, eager
            assert torch.equal(o, oe) and torch.equal(y, ye) and all(torch.equal(a, b) for a, b in zip(pt, pe))
            assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(before, (kp, vp, table)))
        else:
            pt, o, y = step(xi, cached, free[taken:].contiguous(), ints([n_pages - taken]))
        assert pt.lens.tolist() == [p + i + 1 for p in prompts] and y.isfinite().all()
        taken += pt.need.item()
        cached = pt.lens.clone()
        for r, p in enumerate(prompts):
            n = p + i + 1
            z = qkv64[at[r]:at[r] + n]
            k = P.rope(P.head_norm(z[:, hq:hq + hkv], "rms", to_np(kg), None, 1e-5), np.arange(n), d, 10000.0)
            q = P.rope(P.head_norm(z[-1:, :hq], "rms", to_np(qg), None, 1e-5), [n - 1], d, 10000.0)[0]
            k, v = (np.repeat(t, hq // hkv, 1).transpose(1, 0, 2)[None] for t in (k, z[:, hq + hkv:]))
            want, prob = O.attention(q[None, :, None], k, v, d ** -0.5)
            want = want[0, :, 0]
            # keys and queries were rounded once more on the way to the pages: logits off by 2 * half a step of sum |q k|
            aw = (np.abs(q[:, None] * k[0]).sum(-1).max(-1) * d ** -0.5)[:, None]
            av = (np.abs(v[0]) * prob[0, :, 0][..., None]).sum(1)
            tol = HALF[dtype] * np.abs(want) + (2 * 2.2 * HALF[dtype] * aw + 1e-4 * (dtype == BF16) + 1e-5) * av
            check(o[r], want, tol, "step %d, request %d" % (i, r))


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("E,hq,hkv,d,page,dtype", [(256, 4, 2, 64, 16, BF16), (128, 6, 1, 128, 8, BF16), (64, 4, 4, 32, 4, F32)])
def test_serving_iterations(E, hq, hkv, d, page, dtype, graph):
    serve(E, hq, hkv, d, page, dtype, prompts=[37, 1, 130, 16], steps=5, graph=graph)


def test_two_objects_on_two_streams():
    """Two attentions with workspaces of their own at the same time, each on its stream."""
    g = torch.Generator().manual_seed(9)
    kp, vp = torch.randn(2, 512, 16, 2, 128, generator=g).to(BF16).cuda()
    q = torch.randn(2, 2, 8, 128, generator=g).to(BF16).cuda()
    table = torch.randperm(512, generator=g).to(I32).cuda().reshape(2, 256)
    lens = ints([4096, 4000])
    atts = [sm.PagedAttention(2, 8, 2, 128, 16, 256, 512, BF16) for _ in range(2)]
    want = [atts[0](q[i].contiguous(), kp, vp, table, lens).clone() for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(want[0]) for _ in range(2)]
    for _ in range(10):
        for i in range(2):
            atts[i](q[i], kp, vp, table, lens, out=outs[i], stream=streams[i])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_one_object_from_two_threads():
    """One stream, one workspace, split requests: each thread's queries and results with strides of their own."""
    g = torch.Generator().manual_seed(16)
    kp, vp = torch.randn(2, 512, 16, 2, 128, generator=g).to(BF16).cuda()
    table = torch.randperm(512, generator=g).to(I32).cuda().reshape(2, 256)
    att, lens = sm.PagedAttention(2, 8, 2, 128, 16, 256, 512, BF16), [ints([4096, 4000]), ints([300, 3000])]
    q = [torch.randn(2, 8, 128, generator=g).to(BF16).cuda(), torch.randn(2, 9, 256, generator=g).to(BF16).cuda()[:, 1:, :128]]
    out = [torch.empty(2, 8, 128, dtype=BF16, device="cuda"), torch.empty(2, 8, 136, dtype=BF16, device="cuda")[..., :128]]
    want = [att(q[i], kp, vp, table, lens[i]).clone() for i in range(2)]
    torch.cuda.synchronize()
    off = []

    def run(i):
        for _ in range(100):
            out[i].zero_()
            att(q[i], kp, vp, table, lens[i], out=out[i])
            off.append(not torch.equal(out[i], want[i]))
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(off) == 200 and not any(off)


def test_results_of_calls_on_a_side_stream():
    """Outputs that the calls make themselves, on a stream given by the caller: right, and their memory stays theirs while the stream runs."""
    g = torch.Generator().manual_seed(15)
    x = torch.randn(5000, 6, 64, generator=g).cuda()
    gain, pos = torch.ones(64, device="cuda"), torch.arange(5000, dtype=I32, device="cuda")
    want = sm.head_norm_rope(x, x, x, pos, q_gamma=gain, k_gamma=gain)
    w, sc = torch.randint(0, 256, (4096, 512), generator=g, dtype=torch.uint8).cuda(), torch.rand(4096, 8, generator=g).to(BF16).cuda()
    lin, xb = sm.LinearW4(w, sc, group=128), torch.randn(8, 1024, generator=g).to(BF16).cuda()
    y = lin(xb)
    one, none, n_free, t = ints([1] * 50), ints([0] * 50), ints([50]), torch.full((50, 3), -1, dtype=I32, device="cuda")
    free = torch.arange(50, dtype=I32, device="cuda")
    pt = sm.page_table(none, one, free, n_free, t, 16, 50, 50)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        got = sm.head_norm_rope(x, x, x, pos, q_gamma=gain, k_gamma=gain, stream=side) + (lin(xb, stream=side),) + \
            tuple(sm.page_table(none, one, free, n_free, t, 16, 50, 50, stream=side))
        lin(xb, stream=side)                                                        # (dropped at once: its memory is not the next tensor's yet)
        other = torch.zeros(8, 4096, dtype=BF16, device="cuda")
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want + (y,) + tuple(pt))) and not other.any()


def test_results_of_calls_on_a_side_stream_take_its_own_memory():
    """Memory that the current stream has just let go may still be in use there: what a call makes for another stream is not put into it."""
    x, pos, gain = torch.randn(5000, 6, 64, device="cuda"), torch.arange(5000, dtype=I32, device="cuda"), torch.ones(64, device="cuda")
    w, sc = torch.zeros(4096, 512, dtype=torch.uint8, device="cuda"), torch.ones(4096, 8, dtype=BF16, device="cuda")
    xb, side = torch.randn(1000, 1024, device="cuda").to(BF16), torch.cuda.Stream()
    lin, q = sm.LinearW4(w, sc), torch.randn(16, 256, 64, device="cuda").to(BF16)
    att, kp, t = sm.PagedAttention(16, 256, 1, 64, 16, 1, 4, BF16), torch.randn(4, 16, 1, 64, device="cuda").to(BF16), torch.zeros(16, 1, dtype=I32, device="cuda")
    one = torch.zeros(1, dtype=I32, device="cuda")
    calls = {"norm": lambda s: sm.head_norm_rope(x, None, None, pos, q_gamma=gain, stream=s)[0], "linear": lambda s: lin(xb, stream=s),
             "attention": lambda s: att(q, kp, kp, t, t[:, 0].contiguous(), stream=s), "pack": lambda s: sm.LinearW4(w, sc, stream=s).packed,
             "pages": lambda s: sm.page_table(one, one, one, one, t[:1], 16, 4, 500000, stream=s).starts}
    for name, call in calls.items():
        for _ in range(3):
            r = call(None)
            torch.cuda.synchronize()
            span = (r.untyped_storage().data_ptr(), r.untyped_storage().nbytes())
            del r                                                                   # (the next call of this size on this stream would get it)
            r = call(side).untyped_storage()
            side.synchronize()
            apart = r.data_ptr() >= span[0] + span[1] or span[0] >= r.data_ptr() + r.nbytes()
            assert apart, name


def busy(n):
    """Work of some milliseconds on the current stream that ends in n bytes of ones; their memory is let go at once."""
    a = torch.randn(4096, 4096, device="cuda")
    b = torch.empty(n, dtype=torch.uint8, device="cuda")
    for _ in range(10):
        a = a @ a * 0.01
    b.copy_((a.flatten()[:1] != 12345.0).to(torch.uint8).expand(n))
    return b.data_ptr()


def attention_and_linear():
    """name -> (make the object, call it, its memory), on inputs that are ready."""
    g = torch.Generator().manual_seed(17)
    kp, vp = torch.randn(2, 512, 16, 2, 128, generator=g).to(BF16).cuda()
    q, lens = torch.randn(2, 8, 128, generator=g).to(BF16).cuda(), ints([4096, 4000])
    table = torch.randperm(512, generator=g).to(I32).cuda().reshape(2, 256)
    w, sc = torch.randint(0, 256, (8192, 2048), generator=g, dtype=torch.uint8).cuda(), torch.rand(8192, 32, generator=g).to(BF16).cuda()
    x, bias = torch.randn(8, 4096, generator=g).to(BF16).cuda(), torch.randn(8192, generator=g).to(BF16).cuda()
    return {"attention": (lambda: sm.PagedAttention(2, 8, 2, 128, 16, 256, 512, BF16), lambda o, **kw: o(q, kp, vp, table, lens, **kw), lambda o: o.ws),
            "linear": (lambda: sm.LinearW4(w, sc, bias=bias), lambda o, **kw: o(x, **kw), lambda o: o.packed)}


@pytest.mark.parametrize("name", ["attention", "linear"])
@pytest.mark.parametrize("given", [True, False])
def test_objects_made_on_a_busy_stream_and_called_on_another(name, given):
    """The object's memory is that of a tensor which the current stream has still to fill; the first call goes to another stream at once."""
    make, call, memory = attention_and_linear()[name]
    side = torch.cuda.Stream()
    first = make()
    n = memory(first).numel()
    want = call(first).clone()
    torch.cuda.synchronize()
    held, same = [], 0
    for _ in range(3):
        at = busy(n)
        o = make()
        same += memory(o).data_ptr() == at
        if given:
            got = call(o, stream=side)
        else:
            with torch.cuda.stream(side):
                got = call(o)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        held.append(o)
    assert same > 0                                                   # (else nothing was tried)


@pytest.mark.parametrize("name", ["attention", "linear"])
def test_copies_of_objects(name):
    """A shallow copy shares the memory, a deep one has its own."""
    make, call, memory = attention_and_linear()[name]
    o = make()
    want = call(o).clone()
    shallow, deep = copy.copy(o), copy.deepcopy(o)
    assert memory(shallow).data_ptr() == memory(o).data_ptr() != memory(deep).data_ptr()
    memory(o).fill_(0xff) if name == "attention" else None
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for c in (shallow, deep):
        assert torch.equal(call(c), want)
        got = call(c, stream=side)
        side.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("name", ["attention", "linear"])
@pytest.mark.parametrize("given", [True, False])
def test_objects_that_go_while_another_stream_uses_them(name, given):
    """Their memory is not handed out before that stream is done."""
    make, call, memory = attention_and_linear()[name]
    side = torch.cuda.Stream()
    want = call(make()).clone()
    out = torch.empty_like(want)
    o = make()
    torch.cuda.synchronize()
    n, at = memory(o).numel(), memory(o).data_ptr()
    with torch.cuda.stream(side):
        busy(1 << 20)
        if not given:
            call(o, out=out)
    if given:
        call(o, out=out, stream=side)
    del o
    new = torch.zeros(n, dtype=torch.uint8, device="cuda")
    apart = new.data_ptr() >= at + n or at >= new.data_ptr() + n or side.query()      # (a stream that is done already has let go)
    torch.cuda.synchronize()
    assert apart and torch.equal(out, want)


def test_weights_dropped_while_another_stream_packs_them():
    """LinearW4 on a stream that is busy: the sources go at once, and tensors of their size are filled on the current stream."""
    g = torch.Generator().manual_seed(18)
    w, sc = torch.randint(0, 256, (4096, 1024), generator=g, dtype=torch.uint8).cuda(), torch.rand(4096, 16, generator=g).to(BF16).cuda()
    z = torch.randint(0, 16, (4096, 16), generator=g, dtype=torch.uint8).cuda()
    want = sm.LinearW4(w, sc, z).packed.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        a = [t.clone() for t in (w, sc, z)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            busy(1 << 20)
        lin = sm.LinearW4(*a, stream=side)
        at = {t.data_ptr() for t in a}
        del a
        new = [torch.zeros_like(t) for t in (w, sc, z)]
        apart = not at & {t.data_ptr() for t in new} or side.query()
        torch.cuda.synchronize()
        assert apart and torch.equal(lin.packed, want)


def test_copy_of_a_linear_that_another_stream_is_packing():
    g = torch.Generator().manual_seed(21)
    w, sc = torch.randint(0, 256, (4096, 1024), generator=g, dtype=torch.uint8).cuda(), torch.rand(4096, 16, generator=g).to(BF16).cuda()
    want = sm.LinearW4(w, sc).packed.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy(1 << 20)
    lin = sm.LinearW4(w, sc, stream=side)
    again = copy.deepcopy(lin)
    del lin
    torch.cuda.synchronize()
    assert torch.equal(again.packed, want)


def test_captured_with_the_stream_given():
    """Every call names the stream that is being captured, and makes or is given its results."""
    g = torch.Generator().manual_seed(22)
    x = torch.randn(20, 8, 64, generator=g).to(BF16).cuda()
    gain, pos = torch.ones(64, dtype=BF16, device="cuda"), torch.arange(20, dtype=I32, device="cuda")
    kp, vp = torch.randn(2, 20, 16, 2, 64, generator=g).to(BF16).cuda()
    table, lens = torch.arange(20, dtype=I32, device="cuda").view(10, 2).repeat(2, 1), torch.zeros(20, dtype=I32, device="cuda")
    lin = sm.LinearW4(torch.randint(0, 256, (40, 128), generator=g, dtype=torch.uint8).cuda(), torch.rand(40, 2, generator=g).to(BF16).cuda())
    att, eager = (sm.PagedAttention(20, 4, 2, 64, 16, 2, 20, BF16) for _ in range(2))
    one, free, n_free, pages = ints([1] * 20), ints(range(40)), ints([40]), torch.full((20, 3), -1, dtype=I32, device="cuda")
    y = torch.empty(20, 40, dtype=BF16, device="cuda")

    def calls(a, s, out):
        q = sm.head_norm_rope(x[:, :4], None, None, pos, q_gamma=gain, stream=s)[0]
        o = a(q, kp, vp, table, lens, stream=s)
        lin(o.view(20, 256), out=out, stream=s)
        return (q, o, out) + tuple(sm.page_table(lens, one, free, n_free, pages, 16, 40, 20, stream=s))
    calls(att, None, y)
    torch.cuda.synchronize()
    cg = torch.cuda.CUDAGraph()
    with torch.cuda.graph(cg):
        got = calls(att, torch.cuda.current_stream(), y)
    for i in range(3):
        x.copy_(torch.randn(20, 8, 64, generator=g).to(BF16))
        lens.copy_(torch.randint(0, 33, (20,), generator=g))
        cg.replay()
        torch.cuda.synchronize()
        want = calls(eager, None, torch.empty_like(y))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_binding_refuses_wrong_tensors():
    x = torch.randn(4, 2, 64, device="cuda")
    pos = torch.zeros(4, dtype=I32, device="cuda")
    with pytest.raises(TypeError):
        sm.head_norm_rope(x, None, None, pos.long(), norm="none")
    with pytest.raises(ValueError):
        sm.head_norm_rope(x, None, None, pos[:3], norm="none")
    with pytest.raises(ValueError):
        sm.head_norm_rope(x.transpose(1, 2), None, None, pos, norm="none")
    with pytest.raises(sm.SmError):
        sm.head_norm_rope(x, None, None, pos)                                       # the norm needs its gain
    att = sm.PagedAttention(4, 2, 1, 64, 16, 2, 8, F32)
    kp = torch.randn(8, 16, 1, 64, device="cuda")
    table = torch.zeros(4, 2, dtype=I32, device="cuda")
    with pytest.raises(ValueError):
        att(x, kp, kp[:7], table, pos)
    with pytest.raises(TypeError):
        att(x.to(BF16), kp, kp, table, pos)
    with pytest.raises(ValueError):
        att(x, kp, kp, table.t(), pos)
    with pytest.raises(sm.SmError):
        sm.PagedAttention(4, 3, 2, 64, 16, 2, 8, F32)
