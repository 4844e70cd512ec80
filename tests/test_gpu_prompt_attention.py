"""kivi_prompt_attention against a plain 64-bit form.

Tolerance, element by element: the output's rounding, eps / 2 of the value; the probabilities' rounding, eps / 2 of each term, so eps / 2 of the
mean of |v| under the same weights (W); and fp32 sums before that: a logit of 128 products is off by at most 129 * 2^-24 of
the sum of their magnitudes (T), which moves a weight by that much relatively, and the mean by twice that times W; exponentials and the sums of
weights and outputs (chains of fewer than 2^10 additions between rescalings that are exact or rounded once) add less than 2^-13 of W.
The products of the second order are below a hundredth of these."""
import numpy as np
import pytest

import gpu_harness as gh
import operators_reference as ref
from paper_2402_02750_amd import kivi

pytestmark = pytest.mark.gpu

HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _tolerance(want, mean_abs, terms, dtype):
    eps = HALF_STEP[dtype]
    return 1.01 * eps * np.abs(want) + 1.01 * eps * mean_abs + (2 * 129 * 2.0 ** -24 * terms + 2.0 ** -13) * mean_abs + 2.0 ** -25


def _check(got, q, k, v, scale, window, sinks, dtype, what=""):
    """q [n_q, H_q, 128] and so on, CUDA tensors of one sequence."""
    if q.shape[0] == 0:
        return
    want, mean_abs, terms = ref.attention(*(x.double().cpu().numpy() for x in (q, k, v)), scale, ref.visible(q.shape[0], k.shape[0], window, sinks))
    got = got.double().cpu().numpy()
    over = np.abs(got - want) - _tolerance(want, mean_abs, terms, dtype)
    assert np.isfinite(got).all() and over.max() <= 0, f"{what}: tolerance passed by {over.max():.3e}"


def _dtype(torch, name):
    return {"fp16": torch.float16, "bf16": torch.bfloat16}[name]


@pytest.mark.parametrize("batch,q_heads,kv_heads,n_q,n_k,dtype,window,sinks", [
    (1, 4, 4, 1, 1, "fp16", 0, 0),
    (2, 4, 2, 1, 700, "fp16", 0, 0),            # one query: the single token's form
    (1, 8, 1, 3, 5000, "bf16", 0, 0),           # few queries, a long key range
    (1, 4, 4, 2, 4097, "fp16", 300, 4),
    (2, 4, 4, 63, 63, "fp16", 0, 0),
    (1, 4, 2, 64, 65, "bf16", 0, 0),
    (1, 2, 2, 129, 129, "fp16", 1, 0),          # every query sees itself alone
    (1, 2, 1, 300, 300, "fp16", 1, 5),
    (1, 7, 1, 333, 401, "bf16", 64, 64),
    (2, 4, 2, 257, 257, "fp16", 100, 130),      # sinks longer than the window
    (1, 2, 2, 500, 500, "fp16", 5000, 4),       # a window longer than the prompt
    (1, 4, 4, 1001, 1001, "fp16", 0, 0),
    (1, 2, 1, 1100, 1100, "bf16", 129, 3),
    (1, 2, 2, 200, 50, "fp16", 0, 0),           # more queries than keys: the first 150 see nothing
    (1, 2, 2, 40, 0, "fp16", 0, 0),             # no keys at all
    (3, 2, 2, 128, 128, "fp16", 0, 3),          # sinks without a window mean nothing
    (1, 71, 1, 70, 70, "fp16", 0, 0),
    (1, 2, 2, 300, 40, "fp16", 2 ** 31 - 1, 2 ** 31 - 1),
    (1, 4, 1, 90, 2300, "bf16", 700, 2 ** 31 - 1),      # sinks longer than everything
    (9, 16, 8, 140, 140, "fp16", 64, 32),       # 128-row tiles, pairs per die
])
def test_uniform_batches(batch, q_heads, kv_heads, n_q, n_k, dtype, window, sinks):
    torch = gh.require_gpu()
    print(f"case prompt b={batch} heads={q_heads}/{kv_heads} n={n_q}/{n_k} {dtype} window={window} sinks={sinks}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(n_q * 7 + n_k)
    dt = _dtype(torch, dtype)
    # [b, t, h, 128] in memory, as a projection leaves them
    q, k, v = (torch.randn(batch, n, h, 128, device="cuda", generator=gen, dtype=dt).transpose(1, 2) for n, h in ((n_q, q_heads), (n_k, kv_heads), (n_k, kv_heads)))
    out = torch.full((batch, q_heads, n_q, 128), float("nan"), device="cuda", dtype=dt)
    kivi.kivi_prompt_attention(q, k, v, out, 128 ** -0.5, window=window, sinks=sinks)
    torch.cuda.synchronize()
    for b in range(batch):
        _check(out[b].transpose(0, 1), *(x[b].transpose(0, 1) for x in (q, k, v)), 128 ** -0.5, window, sinks, dtype, f"sequence {b}")
    if n_q > n_k:
        assert (out[:, :, :n_q - n_k] == 0).all()


@pytest.mark.parametrize("dtype,window,sinks", [("fp16", 0, 0), ("bf16", 90, 7)])
def test_ragged_batches(dtype, window, sinks):
    """Sequences of different lengths with keys before their queries, empty ones, and rows that belong to nobody, which hold NaN."""
    torch = gh.require_gpu()
    print(f"case prompt ragged {dtype} window={window}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(17)
    dt = _dtype(torch, dtype)
    n_q, n_k = [5, 0, 130, 1, 64, 300], [5, 9, 400, 1, 64, 310]
    q_starts, k_starts = np.cumsum([3] + n_q), np.cumsum([2] + n_k)
    nan = float("nan")
    q, k, v = (torch.full((rows, h, 128), nan, device="cuda", dtype=dt) for rows, h in ((q_starts[-1] + 40, 6), (k_starts[-1] + 70, 2), (k_starts[-1] + 70, 2)))
    for x, s in ((q, q_starts), (k, k_starts), (v, k_starts)):
        x[s[0]:s[-1]] = torch.randn(int(s[-1] - s[0]), *x.shape[1:], device="cuda", generator=gen, dtype=dt)
    out = torch.full_like(q, 5.0)
    starts = [torch.tensor(s, dtype=torch.int32, device="cuda") for s in (q_starts, k_starts)]
    kivi.kivi_prompt_attention(q, k, v, out, 0.07, *starts, max_q=max(n_q), max_k=max(n_k), window=window, sinks=sinks)
    torch.cuda.synchronize()
    for b in range(len(n_q)):
        qs, ks = slice(q_starts[b], q_starts[b + 1]), slice(k_starts[b], k_starts[b + 1])
        _check(out[qs], q[qs], k[ks], v[ks], 0.07, window, sinks, dtype, f"sequence {b}")
    assert (out[:q_starts[0]] == 5).all() and (out[q_starts[-1]:] == 5).all()
    # starts that leave the rows, decrease or pass max_q: those sequences are left out, the others are what they were
    want = out.clone()
    bad_q = starts[0].clone()
    bad_q[-1] = q.shape[0] + 1
    out.fill_(5.0)
    kivi.kivi_prompt_attention(q, k, v, out, 0.07, bad_q, starts[1], max_q=max(n_q), max_k=max(n_k), window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert (out[q_starts[-2]:] == 5).all() and torch.equal(out[:q_starts[-2]], want[:q_starts[-2]])
    out.fill_(5.0)
    kivi.kivi_prompt_attention(q, k, v, out, 0.07, *starts, max_q=max(n_q) - 1, max_k=max(n_k), window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert (out[q_starts[-2]:q_starts[-1]] == 5).all() and torch.equal(out[:q_starts[-2]], want[:q_starts[-2]])


@pytest.mark.parametrize("batch,q_heads,kv_heads,n_q,n_k,dtype,window,sinks", [
    (9, 32, 32, 5, 75, "fp16", 0, 0),           # 288 tiles of rows
    (21, 32, 32, 3, 130, "bf16", 40, 3),        # 672
    (40, 32, 16, 16, 333, "fp16", 0, 0),        # 640, all 32 rows of each
    (22, 24, 24, 1, 1, "fp16", 0, 0),
    (24, 24, 12, 7, 0, "bf16", 0, 0),
])
def test_many_sequences_of_few_rows(batch, q_heads, kv_heads, n_q, n_k, dtype, window, sinks):
    test_uniform_batches(batch, q_heads, kv_heads, n_q, n_k, dtype, window, sinks)


@pytest.mark.parametrize("sequences,kv_heads", [(40, 8), (70, 8)])
def test_many_ragged_sequences_of_few_rows(sequences, kv_heads):
    torch = gh.require_gpu()
    print(f"case prompt ragged few rows {sequences} x {kv_heads}", flush=True)
    rng, gen = np.random.default_rng(sequences), torch.Generator(device="cuda").manual_seed(sequences)
    n_q = rng.integers(0, 9, sequences)
    n_k = n_q + rng.integers(0, 200, sequences) * rng.integers(0, 2, sequences)
    q_starts, k_starts = np.cumsum(np.r_[0, n_q]), np.cumsum(np.r_[0, n_k])
    heads = 4 * kv_heads
    q, k, v = (torch.randn(int(n), h, 128, device="cuda", generator=gen, dtype=torch.float16) for n, h in ((q_starts[-1], heads), (k_starts[-1], kv_heads), (k_starts[-1], kv_heads)))
    out = torch.full_like(q, 5.0)
    starts = [torch.tensor(s, dtype=torch.int32, device="cuda") for s in (q_starts, k_starts)]
    kivi.kivi_prompt_attention(q, k, v, out, 0.09, *starts, max_q=8, max_k=int(n_k.max()))
    torch.cuda.synchronize()
    for b in range(sequences):
        qs, ks = slice(q_starts[b], q_starts[b + 1]), slice(k_starts[b], k_starts[b + 1])
        _check(out[qs], q[qs], k[ks], v[ks], 0.09, 0, 0, "fp16", f"sequence {b}")


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
def test_scales(scale):
    torch = gh.require_gpu()
    print(f"case prompt scale={scale}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(1, 2, 200, 128, device="cuda", generator=gen, dtype=torch.float16) for _ in range(3))
    out = torch.empty_like(q)
    kivi.kivi_prompt_attention(q, k, v, out, scale, window=70, sinks=2)
    torch.cuda.synchronize()
    _check(out[0].transpose(0, 1), *(x[0].transpose(0, 1) for x in (q, k, v)), scale, 70, 2, "fp16")


def test_large_logits_and_masked_infinities():
    """Logits of some hundreds that rise along the keys (the running maximum moves often), and non-finite KEYS where the mask hides them."""
    torch = gh.require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(6)
    n = 400
    q, k, v = (torch.randn(1, 1, n, 128, device="cuda", generator=gen, dtype=torch.float16) for _ in range(3))
    k *= torch.linspace(0.1, 8, n, device="cuda", dtype=torch.float16)[:, None]
    out = torch.empty_like(q)
    kivi.kivi_prompt_attention(q, k, v, out, 0.5)
    torch.cuda.synchronize()
    _check(out[0].transpose(0, 1), *(x[0].transpose(0, 1) for x in (q, k, v)), 0.5, 0, 0, "fp16")
    want = out[:, :, :200].clone()
    k[:, :, 250:] = float("inf")
    k[:, :, 300:] = float("nan")
    kivi.kivi_prompt_attention(q, k, v, out, 0.5)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :, :200], want)


def test_graph_and_stream():
    torch = gh.require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(8)
    # few queries over many keys (parts that are joined), and a plain prompt
    for n_q, n_k in ((2, 6000), (300, 300)):
        print(f"case prompt graph {n_q}/{n_k}", flush=True)
        q, k, v = (torch.randn(1, 4, n, 128, device="cuda", generator=gen, dtype=torch.float16) for n in (n_q, n_k, n_k))
        want, out = torch.empty_like(q), torch.empty_like(q)
        kivi.kivi_prompt_attention(q, k, v, want, 0.1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        kivi.kivi_prompt_attention(q, k, v, out, 0.1, stream=side)
        side.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kivi.kivi_prompt_attention(q, k, v, out, 0.1)
        for step in range(3):
            q.normal_(generator=gen)
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            kivi.kivi_prompt_attention(q, k, v, want, 0.1)
            torch.cuda.synchronize()
            assert torch.equal(out, want), f"replay {step}"
