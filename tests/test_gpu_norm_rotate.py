"""kivi_norm_rotate against a plain 64-bit form.

Tolerance: one rounding to the output's type, eps / 2 of the value (half the smallest step below the normal numbers), and fp32
arithmetic before it: the mean of squares (relative error of 128 additions at most 2^-17, half of that in the root), three products and the rotation's two
products and difference, 2^-22 of the pair's magnitude; 2^-16 of it covers both."""
import numpy as np
import pytest

import gpu_harness as gh
import operators_reference as ref
from paper_2402_02750_amd import kivi

pytestmark = pytest.mark.gpu

HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
SMALLEST = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -134}


def _types(torch):
    return {"fp16": torch.float16, "bf16": torch.bfloat16}


def _expected(x, weight, offset, eps, rows, interleaved):
    y = x
    if weight is not None:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (weight + offset)
    size = np.abs(y)
    if rows is not None:
        half = rows.shape[-1] // 2
        a, b = ref._pairs(2 * half, interleaved)
        size = size.copy()
        size[..., a] = size[..., b] = size[..., a] + size[..., b]
        y = ref.rotate(y, rows.astype(np.float64), interleaved)
    return y, size


def _check(got, want, size, dtype):
    got = got.double().cpu().numpy()
    err = np.abs(got - want) - (HALF_STEP[dtype] * np.abs(want) + 2.0 ** -16 * size + SMALLEST[dtype])
    assert err.max(initial=-1.0) <= 0, f"tolerance passed by {err.max():.3e}"


@pytest.mark.parametrize("rows,q_heads,kv_heads,dtype,rotary,interleaved,norm,offset", [
    (1, 4, 4, "fp16", 128, False, True, 0.0),
    (1, 32, 8, "bf16", 128, True, True, 1.0),
    (3, 71, 1, "fp16", 64, False, True, 0.0),
    (37, 28, 4, "fp16", 96, False, True, 0.0),
    (37, 5, 3, "bf16", 16, True, False, 0.0),
    (513, 40, 40, "fp16", 128, False, False, 0.0),
    (1001, 24, 8, "bf16", 128, False, True, 0.0),
    (4097, 32, 8, "fp16", 128, False, True, 0.0),
    (300, 1, 1, "fp16", 0, False, True, 0.0),
])
def test_against_plain_form(rows, q_heads, kv_heads, dtype, rotary, interleaved, norm, offset):
    torch = gh.require_gpu()
    print(f"case norm_rotate rows={rows} heads={q_heads}/{kv_heads} {dtype} rotary={rotary}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + q_heads)
    dt = _types(torch)[dtype]
    x = torch.randn(rows, q_heads + 2 * kv_heads, 128, device="cuda", generator=gen, dtype=dt) * 3
    w = [(torch.randn(128, device="cuda", generator=gen) * 0.3 + 1 - offset).to(dt) if norm else None for _ in range(2)]
    q, k = x[:, :q_heads], x[:, q_heads:q_heads + kv_heads]
    table = ref.table(700, rotary) if rotary else None
    pos = torch.randint(-3, 710, (rows,), device="cuda", generator=gen, dtype=torch.int32)      # (some outside the table)
    rotation = kivi.Rotation(torch.from_numpy(table).cuda(), interleaved) if rotary else None
    q_out, k_out = torch.full_like(q.contiguous(), float("nan")), torch.full_like(k.contiguous(), float("nan"))
    keep = x.clone()
    kivi.kivi_norm_rotate(q, q_out, k, k_out, w[0], w[1], 1e-5, offset, rotation, pos if rotary else None)
    torch.cuda.synchronize()
    assert torch.equal(x, keep)
    at = table[pos.cpu().numpy().clip(0, 699)] if rotary else None
    for got, src, weight in ((q_out, q, w[0]), (k_out, k, w[1])):
        want, size = _expected(src.double().cpu().numpy(), weight.double().cpu().numpy() if norm else None, offset, 1e-5, at, interleaved)
        _check(got, want, size, dtype)
    # one tensor alone, in place, with other strides (heads before rows)
    alone = q.transpose(0, 1).contiguous().transpose(0, 1)
    kivi.kivi_norm_rotate(alone, alone, q_weight=w[0], eps=1e-5, weight_offset=offset, rotation=rotation, positions=pos if rotary else None)
    assert torch.equal(alone, q_out)


def test_types_differ_and_rows_behind_stay():
    torch = gh.require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(9, 6, 128, device="cuda", generator=gen, dtype=torch.bfloat16)
    out = torch.full((20, 7, 128), 7.0, device="cuda", dtype=torch.float16)
    kivi.kivi_norm_rotate(x, out[:9, :6])
    torch.cuda.synchronize()
    assert torch.equal(out[:9, :6], x.half())
    assert (out[9:] == 7).all() and (out[:, 6] == 7).all()
    kivi.kivi_norm_rotate(x[:0], out[:0, :6])           # no rows
    # zeros stay zeros: eps keeps the norm finite
    zero = torch.zeros(2, 2, 128, device="cuda", dtype=torch.float16)
    kivi.kivi_norm_rotate(zero, zero, q_weight=torch.ones(128, device="cuda", dtype=torch.float16))
    assert (zero == 0).all()


def test_stream_and_graph():
    torch = gh.require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(50, 12, 128, device="cuda", generator=gen, dtype=torch.float16)
    pos = torch.arange(50, device="cuda", dtype=torch.int32)
    w = torch.ones(128, device="cuda", dtype=torch.float16)
    rotation = kivi.Rotation(torch.from_numpy(ref.table(100, 128)).cuda())
    want, out = torch.empty_like(x), torch.empty_like(x)
    kivi.kivi_norm_rotate(x, want, q_weight=w, rotation=rotation, positions=pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kivi.kivi_norm_rotate(x, out, q_weight=w, rotation=rotation, positions=pos, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kivi.kivi_norm_rotate(x, out, q_weight=w, rotation=rotation, positions=pos)
    for step in range(3):
        pos += 1
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        kivi.kivi_norm_rotate(x, want, q_weight=w, rotation=rotation, positions=pos)
        torch.cuda.synchronize()
        assert torch.equal(out, want), f"replay {step}"
