"""Host side of the paged-cache operators and the 4-bit Linear without a GPU: what is refused, and that it is refused before any
pointer is looked at (the pointers here are made up)."""
import contextlib
import ctypes as C
import sys
import threading

import pytest
import torch

from paper_2404_13528_amd import binding as sm

A = C.c_void_p(1 << 20)          # 16-byte aligned, never dereferenced: every call here is refused on the host
ODD = C.c_void_p((1 << 20) + 2)


def page_cfg(n_req=4, page=16, max_pages=8, n_pages=64, free_cap=32, max_tokens=10, table_pitch=8):
    return sm.PageCfg(n_req, page, max_pages, n_pages, free_cap, max_tokens, table_pitch)


def page_call(cfg, *ptrs):
    return sm.lib().sm_page_table(C.byref(cfg) if cfg else None, *(ptrs or [A] * 10), None)


@pytest.mark.parametrize("change,code", [
    (dict(n_req=0), -2), (dict(n_req=65537), -2), (dict(page=0), -2), (dict(max_pages=0), -2), (dict(n_pages=0), -2), (dict(free_cap=-1), -2),
    (dict(max_tokens=-1), -2), (dict(table_pitch=7), -2), (dict(page=1 << 28), -2), (dict(max_tokens=(1 << 30) + 1), -2),
    (dict(n_req=65536, max_pages=1 << 15, table_pitch=1 << 15), -2), (dict(n_pages=(1 << 26) + 1), -2)])
def test_page_table_refuses_sizes(change, code):
    assert page_call(page_cfg(**change)) == code and len(sm.lib().sm_last_error()) > 0


def test_page_table_refuses_pointers():
    assert page_call(None) == -1
    for i in range(10):
        assert page_call(page_cfg(), *[None if j == i else A for j in range(10)]) == -1
        assert page_call(page_cfg(), *[ODD if j == i else A for j in range(10)]) == -1


def rope_desc(**change):
    d = sm.HeadNormRopeDesc()
    v = dict(dtype=sm.SM_BF16, tokens=4, heads_q=4, heads_kv=2, d=64, norm=2, eps=1e-5, rot=64, rope_base=10000.0, page=16, n_pages=4,
             q_gamma=A.value, k_gamma=A.value, q_beta=A.value, k_beta=A.value)
    v.update(change)
    for n, x in v.items():
        if n.endswith("stride"):
            for i, s in enumerate(x):
                getattr(d, n)[i] = s
        else:
            setattr(d, n, x)
    return d


def rope_call(d, q=A, k=A, v=A, positions=A, slots=A, q_out=A, k_out=A, v_out=A):
    return sm.lib().sm_head_norm_rope(C.byref(d) if d else None, q, k, v, positions, slots, q_out, k_out, v_out, None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), -1), (dict(tokens=-1), -2), (dict(tokens=(1 << 25) + 1), -2), (dict(heads_q=0), -2), (dict(heads_kv=0), -2), (dict(d=60), -2), (dict(d=264), -2), (dict(d=0), -2),
    (dict(rot=24), -2), (dict(rot=80), -2), (dict(rot=-16), -2), (dict(norm=3), -1), (dict(rope_base=0.5), -1), (dict(rope_base=float("nan")), -1),
    (dict(page=0), -2), (dict(n_pages=0), -2), (dict(n_pages=(1 << 26) + 1), -2), (dict(q_gamma=None), -1), (dict(k_gamma=None), -1),
    (dict(norm=1, q_beta=None), -1), (dict(norm=1, k_beta=None), -1), (dict(q_gamma=A.value + 8), -1), (dict(q_stride=(4, 64)), -2),
    (dict(q_out_stride=(64, 12)), -2), (dict(k_stride=(64, 4)), -2), (dict(k_out_stride=(4, 0, 0)), -2), (dict(v_out_stride=(0, 0, 4)), -2),
    (dict(dtype=sm.SM_F32, d=66), -2), (dict(dtype=sm.SM_F32, rot=12), -2)])
def test_head_norm_rope_refuses(change, code):
    assert rope_call(rope_desc(**change)) == code and len(sm.lib().sm_last_error()) > 0


def test_head_norm_rope_refuses_pointers():
    assert rope_call(None) == -1
    assert rope_call(rope_desc(), q=None, k=None, v=None) == -1
    for n in ("positions", "q_out", "k_out", "v_out"):
        assert rope_call(rope_desc(), **{n: None}) == -1
    for n in ("q", "k", "v", "positions", "slots", "q_out", "k_out", "v_out"):
        assert rope_call(rope_desc(), **{n: ODD}) == -1
    assert rope_call(rope_desc(tokens=0), positions=None) == 0          # nothing to do


def attn_desc(**change):
    d = sm.PagedAttentionDesc()
    v = dict(dtype=sm.SM_BF16, n_req=4, heads_q=8, heads_kv=2, d=128, page=16, max_pages=8, n_pages=64, scale=0.1, table_pitch=8)
    v.update(change)
    for n, x in v.items():
        if n.endswith("stride"):
            for i, s in enumerate(x):
                getattr(d, n)[i] = s
        else:
            setattr(d, n, x)
    return d


def attn_call(d, ptrs=None, ws_bytes=1 << 40):
    p = [A] * 8 if ptrs is None else ptrs
    return sm.lib().sm_paged_attention(C.byref(d) if d else None, *p, C.c_size_t(ws_bytes), None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=5), -1), (dict(n_req=-1), -2), (dict(n_req=65536), -2), (dict(heads_q=0), -2), (dict(heads_kv=0), -2), (dict(heads_kv=3), -2),
    (dict(d=4), -2), (dict(d=260), -2), (dict(d=264), -2), (dict(page=0), -2), (dict(max_pages=0), -2), (dict(n_pages=0), -2), (dict(table_pitch=7), -2),
    (dict(page=1 << 28), -2), (dict(n_pages=(1 << 26) + 1), -2), (dict(scale=float("inf")), -1), (dict(q_stride=(4, 0)), -2), (dict(o_stride=(0, 4)), -2),
    (dict(k_stride=(4, 0, 0)), -2), (dict(v_stride=(0, 0, 2)), -2), (dict(k_stride=(-8, 0, 0)), -2), (dict(v_stride=(0, -128, 0)), -2),
    (dict(k_stride=(1 << 35, 128, 128)), -2), (dict(v_stride=((1 << 35) // 63 + 8 - (1 << 35) // 63 % 8, 0, 0)), -2),
    (dict(n_req=65535, heads_q=65535, heads_kv=65535), -2)])
def test_paged_attention_refuses(change, code):
    assert attn_call(attn_desc(**change)) == code and len(sm.lib().sm_last_error()) > 0
    assert sm.lib().sm_paged_attention_workspace_bytes(C.byref(attn_desc(**change))) == 0


def test_paged_attention_refuses_pointers_and_small_workspaces():
    assert attn_call(None) == -1
    for i in (0, 1, 2, 3, 4, 5, 7):
        assert attn_call(attn_desc(), [None if j == i else A for j in range(8)]) == -1
    for i in range(8):
        assert attn_call(attn_desc(), [ODD if j == i else A for j in range(8)]) == -1
    need = sm.lib().sm_paged_attention_workspace_bytes(C.byref(attn_desc()))
    assert 0 < need and attn_call(attn_desc(), ws_bytes=need - 1) == -4
    assert attn_call(attn_desc(n_req=0), [None] * 8, 0) == 0


def test_paged_attention_workspace_is_bounded():
    """Partial results: some per workgroup, not some per page of the longest request."""
    for d in (attn_desc(n_req=256, max_pages=8192, table_pitch=8192, heads_q=64, heads_kv=8), attn_desc(n_req=1, max_pages=65536, table_pitch=65536, page=64)):
        assert sm.lib().sm_paged_attention_workspace_bytes(C.byref(d)) < 256 << 20


@pytest.mark.parametrize("N,K,group,taken", [(1, 32, 32, True), (7, 192, 64, True), (4096, 4096, 128, True), (0, 64, 32, False), (8, 96, 64, False), (8, 64, 16, False),
                                             (8, 64, 256, False), (8, 0, 32, False), ((1 << 24) + 1, 32, 32, False)])
def test_w4_sizes(N, K, group, taken):
    n = sm.lib().sm_linear_w4_packed_bytes(N, K, group)
    assert (n > 0) == taken
    if taken:                      # weights, scales and zero points, the rows rounded up to whole tiles
        assert n >= N * K // 2 + 3 * N * (K // group)
    else:
        d = sm.LinearW4Desc(1, N, K, group, 0)
        assert sm.lib().sm_linear_w4(C.byref(d), A, A, A, A, A, None) < 0 and len(sm.lib().sm_last_error()) > 0
        assert sm.lib().sm_linear_w4_pack(A, A, A, N, K, group, A, None) < 0


def test_w4_refuses_pointers():
    lib, d = sm.lib(), sm.LinearW4Desc(2, 64, 128, 128, 0)
    assert lib.sm_linear_w4(None, A, A, A, A, A, None) == -1
    for i in (0, 1, 4):
        assert lib.sm_linear_w4(C.byref(d), *[None if j == i else A for j in range(5)], None) == -1
    for i in range(5):
        assert lib.sm_linear_w4(C.byref(d), *[ODD if j == i else A for j in range(5)], None) == -1
    for i in (0, 1, 3):
        p = [A, A, A, A]
        p[i] = None
        assert lib.sm_linear_w4_pack(p[0], p[1], p[2], 64, 128, 128, p[3], None) == -1
    assert lib.sm_linear_w4(C.byref(sm.LinearW4Desc(2, 64, 128, 128, 2)), A, A, A, A, A, None) == -3
    assert lib.sm_linear_w4(C.byref(sm.LinearW4Desc(-1, 64, 128, 128, 0)), A, A, A, A, A, None) == -2
    assert lib.sm_linear_w4(C.byref(sm.LinearW4Desc(0, 64, 128, 128, 0)), None, None, None, None, None, None) == 0


def test_binding_refuses_host_tensors():
    i32 = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        sm.page_table(i32, i32, i32, i32[:1], i32.reshape(4, 1), 16, 4, 4)
    x = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):
        sm.head_norm_rope(x, None, None, i32)
    with pytest.raises(ValueError):
        sm.head_norm_rope(None, None, None, i32)
    with pytest.raises(ValueError):
        sm.LinearW4(torch.zeros(8, 16, dtype=torch.uint8), torch.zeros(8, 1, dtype=torch.bfloat16), group=32)


def test_binding_refuses_a_stream_of_another_device():
    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 5
    assert sm._raw_stream(torch.device("cuda", 1), Stream) == 5
    with pytest.raises(ValueError, match="stream is on cuda:1"):
        sm._raw_stream(torch.device("cuda", 0), Stream)


class Stream:
    """A stream by its number, with what is asked of it."""
    device = torch.device("cuda", 0)

    def __init__(self, number):
        self.cuda_stream, self.log = number, []

    def record_event(self):
        self.log.append("recorded")
        return "event of %d" % self.cuda_stream

    def wait_event(self, event):
        self.log.append(event)


def without_gpu(monkeypatch, **calls):
    """The binding with host tensors and Python functions in the library's place."""
    class Lib:
        sm_paged_attention_workspace_bytes = staticmethod(lambda desc: 256)
    for name, f in calls.items():
        setattr(Lib, name, staticmethod(f))
    monkeypatch.setattr(sm, "lib", lambda: Lib)
    monkeypatch.setattr(sm, "_device", lambda: torch.device("cpu"))
    monkeypatch.setattr(sm, "_raw_stream", lambda device, stream: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(0))
    monkeypatch.setattr(sm, "_capturing", lambda stream: False)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: empty(*a, **{**kw, "device": "cpu"}))


def in_threads(*calls, n):
    """Every call n times in a thread of its own, changing threads as often as Python can."""
    errors = []

    def run(call):
        try:
            for _ in range(n):
                call()
        except BaseException as e:
            errors.append(e)
    before = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        threads = [threading.Thread(target=run, args=(c,)) for c in calls]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(before)
    assert not errors, errors[:3]


def paged_attention_calls(att):
    """Two calls that differ in every stride."""
    q, wide = torch.zeros(4, 8, 64), torch.zeros(4, 16, 128)[:, ::2, :64]
    kp, vp = torch.zeros(6, 16, 2, 64), torch.zeros(6, 2, 16, 128)[..., :64].transpose(1, 2)
    table, lens = torch.zeros(4, 8, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    roomy = torch.zeros(4, 32, dtype=torch.int32)[:, :8]
    out, strided = torch.zeros(4, 8, 64), torch.zeros(4, 8, 96)[..., :64]
    return lambda: att(q, kp, kp, table, lens, out=out), lambda: att(wide, vp, vp, roomy, lens, out=strided)


def test_paged_attention_from_two_threads_has_the_strides_of_its_own_call(monkeypatch):
    seen, wrong = {}, []

    def call(desc, q, *rest):
        d = C.cast(desc, C.POINTER(sm.PagedAttentionDesc)).contents
        strides = (d.table_pitch, *d.q_stride, *d.o_stride, *d.k_stride, *d.v_stride)
        if seen.setdefault(q, strides) != strides:
            wrong.append(strides)
        return 0
    without_gpu(monkeypatch, sm_paged_attention=call)
    a, b = paged_attention_calls(sm.PagedAttention(4, 8, 2, 64, 16, 8, 6, torch.float32))
    a()
    b()
    assert sorted(seen.values()) == [(8, 512, 64, 512, 64, 2048, 128, 64, 2048, 128, 64), (32, 2048, 256, 768, 96, 4096, 128, 2048, 4096, 128, 2048)]
    in_threads(a, b, n=5000)
    assert not wrong, (len(wrong), wrong[0])


def test_packed_descriptors_are_the_structures():
    for packed, desc in ((sm._PAGE_CFG, sm.PageCfg), (sm._HEAD_NORM_ROPE, sm.HeadNormRopeDesc), (sm._PAGED_ATTENTION, sm.PagedAttentionDesc), (sm._LINEAR_W4, sm.LinearW4Desc)):
        assert packed.size == C.sizeof(desc)


def test_paged_attention_from_two_threads_one_call_at_a_time(monkeypatch):
    """The two kernels of a call share the object's workspace: no other call's may come between them in the stream."""
    inside, met = [0], []

    def call(*args):
        inside[0] += 1
        for _ in range(20):                                          # (time for the other thread, as the C call gives it)
            met.append(inside[0])
        inside[0] -= 1
        return 0
    without_gpu(monkeypatch, sm_paged_attention=call)
    in_threads(*paged_attention_calls(sm.PagedAttention(4, 8, 2, 64, 16, 8, 6, torch.float32)), n=1000)
    assert max(met) == 1


def test_memory_of_an_object_on_streams_other_than_its_own(monkeypatch):
    """The first call on each stream waits for what the memory was made from, and keeps it from being handed out early; a captured stream cannot wait
    for what is not in its graph, so its first call outside does."""
    class Memory:
        def __init__(self):
            self.streams = []

        def record_stream(self, s):
            self.streams.append(s.cuda_stream)

    dev, capturing = torch.device("cuda", 0), []
    made, side, third = Stream(5), Stream(6), Stream(7)
    monkeypatch.setattr(sm, "_capturing", lambda s: s.cuda_stream in capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: side)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: side.cuda_stream, raising=False)
    ws, bias = Memory(), Memory()
    kept = sm._Kept(dev, made, ws, bias)
    assert made.log == ["recorded"] and ws.streams == bias.streams == [5]
    assert kept.used_on(dev, made) == 5 and made.log == ["recorded"]
    for _ in range(3):                                               # the current stream, first
        assert kept.used_on(dev, None) == 6
        assert side.log == ["event of 5"] and ws.streams == bias.streams == [5, 6]
    capturing.append(7)
    assert kept.used_on(dev, third) == 7 and third.log == [] and ws.streams == [5, 6, 7]
    capturing.clear()
    assert kept.used_on(dev, third) == 7 and kept.used_on(dev, third) == 7 and third.log == ["event of 5"]
    capturing.append(6)                                              # made while a graph is captured: nothing to wait for outside it
    kept = sm._Kept(dev, None, ws)
    assert kept.used_on(dev, made) == 5 and made.log == ["recorded"]


def test_objects_use_their_memory_through_its_streams(monkeypatch):
    got = []
    without_gpu(monkeypatch, sm_paged_attention=lambda *a: got.append(a[-1]) or 0, sm_linear_w4=lambda *a: got.append(a[-1]) or 0, sm_linear_w4_pack=lambda *a: 0,
                sm_linear_w4_packed_bytes=lambda *a: 64)
    monkeypatch.setattr(sm._Kept, "used_on", lambda self, device, stream: tuple(t.data_ptr() for t in self.tensors))
    att = sm.PagedAttention(4, 8, 2, 64, 16, 8, 6, torch.float32)
    paged_attention_calls(att)[0]()
    bias = torch.zeros(8, dtype=torch.bfloat16)
    lin = sm.LinearW4(torch.zeros(8, 16, dtype=torch.uint8), torch.zeros(8, 1, dtype=torch.bfloat16), group=32, bias=bias)
    lin(torch.zeros(2, 32, dtype=torch.bfloat16))
    assert got == [(att.ws.data_ptr(),), (lin.packed.data_ptr(), bias.data_ptr())]


def recorded(monkeypatch):
    """What record_stream is told from now on: (address, stream)."""
    seen = set()
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: seen.add((t.data_ptr(), s.cuda_stream)))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    return seen


def test_weights_stay_allocated_until_they_are_packed(monkeypatch):
    without_gpu(monkeypatch, sm_linear_w4_pack=lambda *a: 0, sm_linear_w4_packed_bytes=lambda *a: 64)
    seen = recorded(monkeypatch)
    w, scales, zeros = torch.zeros(8, 16, dtype=torch.uint8), torch.zeros(8, 1, dtype=torch.bfloat16), torch.zeros(8, 1, dtype=torch.uint8)
    sm.LinearW4(w, scales, zeros, group=32, stream=Stream(9))
    assert {(t.data_ptr(), 9) for t in (w, scales, zeros)} <= seen
    seen.clear()
    sm.LinearW4(w, scales, group=32, stream=Stream(9))
    assert {(t.data_ptr(), 9) for t in (w, scales)} <= seen


def test_tensors_of_a_call_stay_allocated_until_its_stream_is_done(monkeypatch):
    without_gpu(monkeypatch, sm_paged_attention=lambda *a: 0, sm_linear_w4=lambda *a: 0, sm_linear_w4_pack=lambda *a: 0, sm_linear_w4_packed_bytes=lambda *a: 64,
                sm_page_table=lambda *a: 0, sm_head_norm_rope=lambda *a: 0)
    i32, bf16 = torch.int32, torch.bfloat16
    att = sm.PagedAttention(4, 8, 2, 64, 16, 8, 6, torch.float32)
    lin = sm.LinearW4(torch.zeros(8, 16, dtype=torch.uint8), torch.zeros(8, 1, dtype=bf16), group=32)
    q, kp, vp, out, lse = torch.zeros(4, 8, 64), torch.zeros(6, 16, 2, 64), torch.zeros(6, 16, 2, 64), torch.zeros(4, 8, 64), torch.zeros(4, 8)
    table, lens = torch.zeros(4, 8, dtype=i32), torch.zeros(4, dtype=i32)
    k, v, gains, pos, slots = torch.zeros(4, 2, 64), torch.zeros(4, 2, 64), torch.zeros(4, 64), torch.zeros(4, dtype=i32), torch.zeros(4, dtype=i32)
    x, res, y = torch.zeros(2, 32, dtype=bf16), torch.zeros(2, 8, dtype=bf16), torch.zeros(2, 8, dtype=bf16)
    cached, fresh, free, n_free = (torch.zeros(n, dtype=i32) for n in (4, 4, 6, 1))
    pt = sm.PageTable(*(torch.zeros(n, dtype=i32) for n in (5, 4, 3, 3, 1)))
    calls = [(lambda s: att(q, kp, vp, table, lens, out=out, lse=lse, stream=s), (q, kp, vp, table, lens, out, lse)),
             (lambda s: lin(x, residual=res, out=y, stream=s), (x, res, y)),
             (lambda s: sm.page_table(cached, fresh, free, n_free, table, 16, 6, 3, out=pt, stream=s), (cached, fresh, free, n_free, table, *pt)),
             (lambda s: sm.head_norm_rope(q, k, v, pos, "layer", q_gamma=gains[0], k_gamma=gains[1], q_beta=gains[2], k_beta=gains[3], slots=slots, q_out=out,
                                          k_out=kp, v_out=vp, stream=s), (q, k, v, pos, *gains, slots, out, kp, vp)),
             (lambda s: sm.head_norm_rope(None, None, v, pos, slots=slots, v_out=vp, stream=s), (v, pos, slots, vp))]
    seen = recorded(monkeypatch)
    for call, tensors in calls:
        seen.clear()
        call(Stream(9))
        assert {(t.data_ptr(), 9) for t in tensors} <= seen
    monkeypatch.setattr(torch.Tensor, "record_stream", None)         # the current stream: nothing to tell
    for call, _ in calls:
        call(None)


def test_page_table_refuses_outputs_over_inputs_or_each_other():
    """cached, fresh, free_pages (32), n_free, table (4 rows of 8, 24 apart), starts (5), lens, positions (10), slots (10), need."""
    sizes = [4, 4, 32, 1, 3 * 24 + 8, 5, 4, 10, 10, 1]
    base = [(1 << 20) + (1 << 12) * i for i in range(10)]
    cfg = page_cfg(table_pitch=24)
    for i in range(4, 10):
        for j in range(10):
            if i == j:
                continue
            for at in (base[j], base[j] + 4 * (sizes[j] - 1), base[j] - 4 * (sizes[i] - 1)):         # first, last and first place in common
                p = [C.c_void_p(at if k == i else base[k]) for k in range(10)]
                assert page_call(cfg, *p) == -1 and b"overlap" in sm.lib().sm_last_error(), (i, j, at)


def test_w4_refuses_results_over_operands():
    lib, d = sm.lib(), sm.LinearW4Desc(4, 64, 128, 128, 0)
    x, packed, bias, residual, y = ((1 << 20) + (1 << 16) * i for i in range(5))
    nbytes = {x: 4 * 128 * 2, packed: lib.sm_linear_w4_packed_bytes(64, 128, 128), bias: 128, residual: 512}
    for p, n in nbytes.items():
        for at in (p, p + n - 16, p - 512 + 16):
            if at != residual:
                assert lib.sm_linear_w4(C.byref(d), x, packed, bias, residual, at, None) == -1 and b"overlap" in lib.sm_last_error(), (p, at)
    for p, n in ((x, 64 * 64), (bias, 128), (residual, 64)):                                          # weights, scales, zero points
        for at in (p, p + n - 16, p - nbytes[packed] + 16):
            assert lib.sm_linear_w4_pack(x, bias, residual, 64, 128, 128, at, None) == -1 and b"overlap" in lib.sm_last_error()
