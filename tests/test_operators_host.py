"""Host-side checks of the operators around the cache that need no GPU: sizes, and refusals before anything is enqueued."""
import ctypes
import os

import pytest

from paper_2402_02750_amd import kivi

INVALID, UNSUPPORTED, WORKSPACE = kivi.KIVI_ERR_INVALID_ARG, kivi.KIVI_ERR_UNSUPPORTED, kivi.KIVI_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kivi.LIB_PATH):
        from paper_2402_02750_amd.build import build_library
        build_library(verbose=False)
    return kivi.load_library()


def _set(struct, changes):
    """changes: {"field" or "field.field": value}"""
    for name, value in changes.items():
        at = struct
        *path, last = name.split(".")
        for p in path:
            at = getattr(at, p)
        setattr(at, last, value)
    return struct


def _tensor():
    return kivi.kivi_tensor_t(0x1000, 4096, 128, 1024)


def _rotation(**kw):
    return _set(kivi.kivi_rotation_t(0x2000, 0x3000, 100, 128, 0), kw)


@pytest.mark.parametrize("job,call,rotation,status", [
    ({"src.data": None}, {}, None, INVALID),
    ({"src.data": 0x1008}, {}, None, INVALID),
    ({"dst.data": None}, {}, None, INVALID),
    ({"src.stride_h": 100}, {}, None, INVALID),
    ({"src.stride_t": -128}, {}, None, INVALID),
    ({"dst.stride_h": 0}, {}, None, INVALID),           # heads on top of each other
    ({"dst.stride_t": 64}, {}, None, INVALID),
    ({"weight": 0x4002}, {}, None, INVALID),
    ({"weight_offset": float("nan")}, {}, None, INVALID),
    ({"n_heads": 0}, {}, None, INVALID),
    ({"n_heads": 70000}, {}, None, INVALID),
    ({"src_type": 2}, {}, None, UNSUPPORTED),
    ({"dst_type": -1}, {}, None, UNSUPPORTED),
    ({}, {"n_jobs": 0}, None, INVALID),
    ({}, {"n_jobs": 3}, None, INVALID),
    ({}, {"n_rows": -1}, None, INVALID),
    ({}, {"eps": -1.0}, None, INVALID),
    ({}, {"eps": float("inf")}, None, INVALID),
    ({}, {}, {"table": None}, INVALID),
    ({}, {}, {"table": 0x2004}, INVALID),
    ({}, {}, {"positions": None}, INVALID),
    ({}, {}, {"positions": 0x3001}, INVALID),
    ({}, {}, {"n_positions": 0}, INVALID),
    ({}, {}, {"rotary_dim": 0}, INVALID),
    ({}, {}, {"rotary_dim": 144}, INVALID),
    ({}, {}, {"rotary_dim": 40}, UNSUPPORTED),
    ({}, {}, {"interleaved": 2}, INVALID),
    ({}, {"n_rows": 0}, {}, kivi.KIVI_OK),               # nothing to do: no launch
])
def test_norm_rotate_refusals(lib, job, call, rotation, status):
    jobs = (kivi.kivi_norm_rotate_job_t * 3)()
    for j in jobs:
        j.src, j.dst, j.n_heads = _tensor(), _tensor(), 8
    _set(jobs[0], job)
    r = ctypes.byref(_rotation(**rotation)) if rotation is not None else None
    args = dict(n_jobs=1, n_rows=5, eps=1e-6)
    args.update(call)
    assert lib.kivi_norm_rotate(jobs, args["n_jobs"], args["n_rows"], args["eps"], r, None) == status
    assert lib.kivi_norm_rotate(None, 1, 5, 1e-6, None, None) == INVALID


def _prompt(**kw):
    return _set(kivi.kivi_prompt_t(2, 8, 2, 128, 0, 64, 64, softmax_scale=0.1), kw)


@pytest.mark.parametrize("prompt,tensor,status", [
    ({"batch": 0}, {}, INVALID), ({"n_q_heads": 7}, {}, INVALID), ({"n_kv_heads": 0}, {}, INVALID),
    ({"head_dim": 64}, {}, UNSUPPORTED), ({"type": 3}, {}, UNSUPPORTED),
    ({"max_q": -1}, {}, INVALID), ({"max_k": -1}, {}, INVALID), ({"window": -1}, {}, INVALID), ({"sinks": -1}, {}, INVALID),
    ({"softmax_scale": float("nan")}, {}, INVALID), ({"softmax_scale": float("inf")}, {}, INVALID),
    ({"q_starts": 0x5002}, {}, INVALID), ({"k_starts": 0x5002}, {}, INVALID), ({"q_starts": 0x5000, "q_rows": -1}, {}, INVALID),
    ({}, {"q.data": None}, INVALID), ({}, {"k.data": None}, INVALID), ({}, {"v.data": 0x1004}, INVALID), ({}, {"out.data": None}, INVALID),
    ({}, {"k.stride_t": 12}, INVALID), ({}, {"q.stride_b": -8}, INVALID), ({}, {"out.stride_h": 64}, INVALID), ({}, {"out.stride_b": 0}, INVALID),
    ({"max_q": 0}, {"q.data": None}, kivi.KIVI_OK),
])
def test_prompt_refusals(lib, prompt, tensor, status):
    class Tensors(ctypes.Structure):
        _fields_ = [(n, kivi.kivi_tensor_t) for n in ("q", "k", "v", "out")]
    t = _set(Tensors(*(_tensor() for _ in range(4))), tensor)
    p = _prompt(**prompt)
    assert lib.kivi_prompt_attention(ctypes.byref(p), *(ctypes.byref(getattr(t, n)) for n in ("q", "k", "v", "out")), None, 0, None) == status
    if prompt and status not in (kivi.KIVI_OK,):
        n = ctypes.c_size_t(0)
        assert lib.kivi_prompt_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == status
    assert lib.kivi_prompt_attention(ctypes.byref(_prompt()), None, None, None, None, None, 0, None) == INVALID


def test_prompt_workspace(lib):
    """Few queries over many keys ask for a workspace, and one that is too small is refused."""
    p = _prompt(batch=1, n_q_heads=4, n_kv_heads=4, max_q=1, max_k=100000)
    n = ctypes.c_size_t(0)
    assert lib.kivi_prompt_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == 0
    assert lib.kivi_prompt_workspace_bytes(ctypes.byref(p), None) == INVALID
    t = _tensor()
    if n.value:
        assert lib.kivi_prompt_attention(ctypes.byref(p), *[ctypes.byref(t)] * 4, ctypes.c_void_p(0x6000), n.value - 1, None) == WORKSPACE
    assert lib.kivi_prompt_attention(ctypes.byref(p), *[ctypes.byref(t)] * 4, ctypes.c_void_p(0x6004), 1 << 30, None) == INVALID
    big = _prompt(batch=16, n_q_heads=32, n_kv_heads=32, max_q=4096, max_k=4096)
    assert lib.kivi_prompt_workspace_bytes(ctypes.byref(big), ctypes.byref(n)) == 0 and n.value == 0


@pytest.mark.parametrize("strides,sizes,status", [
    # b, h, t; batch, heads, rows.  (without a device a call that passes the checks ends with an error of the runtime)
    ((0, 128, 256), (1, 4, 3), INVALID),                # the second row over the third head of the first
    ((0, 128, 512), (1, 4, 3), None), ((0, 1024, 128), (1, 4, 8), None), ((0, 896, 128), (1, 4, 8), INVALID),
    ((1024, 128, 512), (2, 4, 3), INVALID), ((1536, 128, 512), (2, 4, 3), None), ((512, 128, 1024), (2, 4, 3), None),
    ((0, 128, 0), (1, 4, 1), None), ((1 << 62, 128, 512), (2, 4, 1), None),
])
def test_outputs_that_overlap(lib, strides, sizes, status):
    import torch
    if status is None and torch.cuda.is_available():
        pytest.skip("the buffers are made up")
    b, h, t = strides
    batch, heads, rows = sizes
    out = kivi.kivi_tensor_t(0x1000, b, h, t)
    p = _prompt(batch=batch, n_q_heads=heads, n_kv_heads=heads, max_q=rows, max_k=10)
    x = kivi.kivi_tensor_t(0x1000, 0, 128, 128 * heads)
    status_of = lib.kivi_prompt_attention(ctypes.byref(p), ctypes.byref(x), ctypes.byref(x), ctypes.byref(x), ctypes.byref(out), None, 0, None)
    assert status_of == (kivi.KIVI_ERR_HIP if status is None else status)


def test_rows_without_an_order(lib):
    """Sequences of one query each: their rows have to be apart all the same."""
    x, out = _tensor(), kivi.kivi_tensor_t(0x1000, 0, 128, 0)
    p = _prompt(batch=3, n_q_heads=1, n_kv_heads=1, max_q=1, max_k=4, q_starts=0x5000, q_rows=3)
    assert lib.kivi_prompt_attention(ctypes.byref(p), *[ctypes.byref(x)] * 3, ctypes.byref(out), None, 0, None) == INVALID


@pytest.mark.parametrize("max_q,max_k", [(0, 100), (0, 0), (5, 0), (0, 100000)])
def test_prompt_workspace_without_rows(lib, max_q, max_k):
    p = _prompt(batch=1, n_q_heads=4, n_kv_heads=4, max_q=max_q, max_k=max_k)
    n = ctypes.c_size_t(1)
    assert lib.kivi_prompt_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == 0 and n.value == 0


def _layout(**kw):
    return _set(kivi.make_paged_layout(4, 8, 2, 2, 64, 64, 10, 96), kw)


def test_paged_sizes(lib):
    s = kivi.kivi_paged_sizes(_layout())
    assert s.pages == 10 * 2 * 2 * (1024 + 2048)
    assert s.k_resid == s.v_resid == 4 * 2 * 96 * 256
    assert s.workspace > 0
    assert kivi.kivi_paged_sizes(_layout(bits=4)).pages == 10 * 2 * 2 * (1024 + 4096)
    assert lib.kivi_paged_sizes(ctypes.byref(_layout()), None) == INVALID
    huge = kivi.kivi_paged_sizes(_layout(n_pages=1 << 20, n_kv_heads=8, page_tokens=256))
    assert huge.pages == (1 << 20) * 8 * 8 * (1024 + 2048)


@pytest.mark.parametrize("kw,status", [
    (dict(max_sequences=0), INVALID), (dict(n_q_heads=7), INVALID), (dict(n_q_heads=258), UNSUPPORTED), (dict(head_dim=64), UNSUPPORTED), (dict(bits=8), UNSUPPORTED),
    (dict(group=64), UNSUPPORTED), (dict(residual=48), INVALID), (dict(residual=-32), INVALID), (dict(page_tokens=48), INVALID),
    (dict(page_tokens=16), INVALID), (dict(page_tokens=8192), INVALID), (dict(n_pages=0), INVALID), (dict(cap_r_tokens=64), INVALID),
    (dict(cap_r_tokens=100), INVALID), (dict(cap_r_tokens=(1 << 20) + 32), UNSUPPORTED),
])
def test_bad_paged_layouts(lib, kw, status):
    l = _layout(**kw)
    assert lib.kivi_paged_sizes(ctypes.byref(l), ctypes.byref(kivi.kivi_paged_sizes_t())) == status
    cache, batch, rows, query = _call()
    assert lib.kivi_paged_append(ctypes.byref(l), ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(rows), None) == status
    assert lib.kivi_paged_attention(ctypes.byref(l), ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(query), ctypes.c_void_p(0x6000), 1 << 30, None) == status


def _call():
    cache = kivi.kivi_paged_cache_t(0x1000, 0x2000, 0x3000)
    batch = kivi.kivi_paged_batch_t(3, 5, 5, 0x4000, 0x5000, None)
    rows = kivi.kivi_paged_rows_t(k=_tensor(), v=_tensor(), type=0, n_rows=12, max_new=4)
    query = kivi.kivi_paged_query_t(0x7000, 0x8000, 0, 0, 0, 0.1)
    return cache, batch, rows, query


@pytest.mark.parametrize("cache,batch", [
    ({"pages": None}, {}), ({"pages": 0x1008}, {}), ({"k_resid": None}, {}), ({"v_resid": 0x3004}, {}),
    ({}, {"batch": 0}), ({}, {"max_pages": -1}), ({}, {"page_table_stride": 4}), ({}, {"page_table": None}), ({}, {"page_table": 0x4002}),
    ({}, {"lengths": None}), ({}, {"lengths": 0x5001}), ({}, {"slots": 0x5003}), ({}, {"max_pages": 1 << 30, "page_table_stride": 1 << 30}),
])
def test_paged_caches_and_batches(lib, cache, batch):
    c, b, rows, query = _call()
    _set(c, cache), _set(b, batch)
    l = _layout()
    assert lib.kivi_paged_append(ctypes.byref(l), ctypes.byref(c), ctypes.byref(b), ctypes.byref(rows), None) == INVALID
    assert lib.kivi_paged_attention(ctypes.byref(l), ctypes.byref(c), ctypes.byref(b), ctypes.byref(query), ctypes.c_void_p(0x6000), 1 << 30, None) == INVALID


@pytest.mark.parametrize("rows,status", [
    ({"k.data": None}, INVALID), ({"v.data": 0x1008}, INVALID), ({"k.stride_h": 4}, INVALID), ({"type": 5}, UNSUPPORTED),
    ({"max_new": -1}, INVALID), ({"n_rows": -1}, INVALID), ({"n_rows": 11}, INVALID), ({"starts": 0x9001}, INVALID),
    ({"q.data": 0x1000}, INVALID), ({"q_out.data": 0x1000}, INVALID),
    ({"max_new": 0}, kivi.KIVI_OK),
])
def test_append_refusals(lib, rows, status):
    c, b, r, _ = _call()
    _set(r, rows)
    l = _layout()
    assert lib.kivi_paged_append(ctypes.byref(l), ctypes.byref(c), ctypes.byref(b), ctypes.byref(r), None) == status
    assert lib.kivi_paged_append(ctypes.byref(l), ctypes.byref(c), ctypes.byref(b), None, None) == INVALID


def test_append_refuses_a_bad_rotation(lib):
    c, b, r, _ = _call()
    rotation = _rotation(rotary_dim=100)
    r.rotation = ctypes.pointer(rotation)
    assert lib.kivi_paged_append(ctypes.byref(_layout()), ctypes.byref(c), ctypes.byref(b), ctypes.byref(r), None) == UNSUPPORTED
    rotation.rotary_dim, rotation.table = 64, None
    assert lib.kivi_paged_append(ctypes.byref(_layout()), ctypes.byref(c), ctypes.byref(b), ctypes.byref(r), None) == INVALID


@pytest.mark.parametrize("query,status", [
    ({"q": None}, INVALID), ({"out": None}, INVALID), ({"q": 0x7008}, INVALID), ({"out_type": 2}, UNSUPPORTED), ({"window": -1}, INVALID), ({"sinks": -4}, INVALID),
    ({"softmax_scale": float("nan")}, INVALID),
])
def test_attention_refusals(lib, query, status):
    c, b, _, q = _call()
    l = _layout()
    f = lib.kivi_paged_attention
    assert f(ctypes.byref(l), ctypes.byref(c), ctypes.byref(b), None, ctypes.c_void_p(0x6000), 1 << 30, None) == INVALID
    assert f(ctypes.byref(l), ctypes.byref(c), ctypes.byref(b), ctypes.byref(_set(q, query)), ctypes.c_void_p(0x6000), 1 << 30, None) == status


def test_attention_workspace(lib):
    c, b, _, q = _call()
    l = _layout()
    need = kivi.kivi_paged_sizes(l).workspace
    f = lib.kivi_paged_attention
    for ws, n in ((None, need), (0x6000, need - 1), (0x6008, need)):
        assert f(ctypes.byref(l), ctypes.byref(c), ctypes.byref(b), ctypes.byref(q), ctypes.c_void_p(ws), n, None) == WORKSPACE
    # an axis of steps that 31 bits do not hold
    wide = kivi.make_paged_layout(4, 2048, 256, 2, 64, 4096, 10, 96)
    _set(b, {"batch": 30000, "max_pages": 100000, "page_table_stride": 100000})
    assert f(ctypes.byref(wide), ctypes.byref(c), ctypes.byref(b), ctypes.byref(q), ctypes.c_void_p(0x6000), 1 << 30, None) == UNSUPPORTED


def test_binding_refuses_other_devices(lib):
    """Tensors that are not on the current GPU never reach the library."""
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        here = torch.zeros(1, 2, 128, dtype=torch.float16)
        with pytest.raises(kivi.KiviError):
            kivi.kivi_norm_rotate(here, here)
    else:
        assert kivi._type_of(torch.zeros(1, dtype=torch.bfloat16)) == kivi.KIVI_TYPE_BF16
        with pytest.raises(kivi.KiviError):
            kivi._type_of(torch.zeros(1))


def test_page_tables_whose_rows_overlap_are_refused(lib):
    torch = pytest.importorskip("torch")
    lengths = torch.ones(3, dtype=torch.int32)
    with pytest.raises(AssertionError):
        kivi.PagedBatch(torch.zeros(1, 4, dtype=torch.int32).expand(3, 4), lengths)
    with pytest.raises(AssertionError):
        kivi.PagedBatch(torch.zeros(4, 3, dtype=torch.int32).t(), lengths)
    with pytest.raises(AssertionError):
        kivi.PagedBatch(torch.zeros(2, 4, dtype=torch.int32), lengths)
    b = kivi.PagedBatch(torch.zeros(3, 8, dtype=torch.int32)[:, :4], lengths)
    assert (b.c.batch, b.c.max_pages, b.c.page_table_stride) == (3, 4, 8)
    assert kivi.PagedBatch(torch.zeros(1, 4, dtype=torch.int32).expand(1, 4), lengths[:1]).c.page_table_stride >= 4


def test_stream_of_another_device():
    class Stream:
        device_index, cuda_stream = 1, 0x1000
    assert kivi._stream_handle(Stream(), 1) == 0x1000
    with pytest.raises(kivi.KiviError) as e:
        kivi._stream_handle(Stream(), 0)
    assert e.value.status == INVALID


def test_products_of_counts(lib):
    """Counts whose product leaves the integers it is held in are refused, not wrapped."""
    n, most = ctypes.c_size_t(0), 2 ** 31 - 1
    for kw in (dict(batch=most, n_q_heads=most, n_kv_heads=most), dict(batch=65536, n_kv_heads=65536, n_q_heads=65536), dict(max_q=most, n_q_heads=8, n_kv_heads=1)):
        assert lib.kivi_prompt_workspace_bytes(ctypes.byref(_prompt(**kw)), ctypes.byref(n)) == UNSUPPORTED
    sizes = kivi.kivi_paged_sizes_t()
    for kw in (dict(n_pages=most, n_q_heads=most, n_kv_heads=most), dict(max_sequences=most, n_q_heads=1 << 30, n_kv_heads=1 << 30, cap_r_tokens=1 << 20)):
        assert lib.kivi_paged_sizes(ctypes.byref(_layout(**kw)), ctypes.byref(sizes)) == UNSUPPORTED
    cache = kivi.kivi_paged_cache_t(0x1000, 0x1000, 0x1000)
    batch = kivi.kivi_paged_batch_t(1 << 20, 4, 4, 0x1000, 0x1000, None)
    query = kivi.kivi_paged_query_t(0x1000, 0x1000, 0, 0, 0, 0.1)
    wide = _layout(n_q_heads=1 << 12, n_kv_heads=1 << 12)
    assert lib.kivi_paged_attention(ctypes.byref(wide), ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(query), ctypes.c_void_p(0x1000), 1 << 40, None) == UNSUPPORTED
    x = _tensor()
    for max_new, rows in ((most, most), (1 << 24, most)):
        batch = kivi.kivi_paged_batch_t(1 << 16, 4, 4, 0x1000, 0x1000, None)
        new = kivi.kivi_paged_rows_t(x, x, kivi.kivi_tensor_t(), kivi.kivi_tensor_t(), 0, rows, max_new, 0x1000, None)
        assert lib.kivi_paged_append(ctypes.byref(_layout(n_q_heads=1 << 14, n_kv_heads=1 << 14)), ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(new), None) == UNSUPPORTED
