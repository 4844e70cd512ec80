"""The paged cache: kivi_paged_append bit for bit against the oracle, kivi_paged_attention against 64 bits.

Tolerance of the attention, element by element: the output's rounding, eps / 2 of the value.  Logits are sums of products of a code (exact) with s q
rounded to 21 bits (two fp16 parts) and of zero-points with q, in fp32: off by at most (2^-20 + 129 * 2^-24) of the sum T of the terms'
magnitudes, which moves the mean by twice that times W, the mean of the values' magnitudes (code times scale plus zero-point) under the same
weights.  Probabilities keep 20 bits, and their products with scales as many; sums and exponentials are fp32: 2^-13 of W, as for prompts."""
import numpy as np
import pytest

import gpu_harness as gh
import operators_reference as ref
from paper_2402_02750_amd import kivi

pytestmark = pytest.mark.gpu

HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


class Run:
    """Sequences in a paged cache on the GPU next to the oracle's."""

    def __init__(self, sequences, q_heads, kv_heads, bits, residual=64, page=64, most=600, cap_r=None, seed=1, slots=None):
        torch = gh.require_gpu()
        self.torch, self.rng = torch, np.random.default_rng(seed)
        self.q_heads, self.kv_heads, self.bits, self.residual, self.page = q_heads, kv_heads, bits, residual, page
        self.pages_each = -(-most // page)
        n_pages = sequences * self.pages_each + 2
        cap_r = residual + 32 if cap_r is None else cap_r
        self.slots = list(range(sequences)) if slots is None else slots
        self.layout = kivi.make_paged_layout(max(self.slots) + 1, q_heads, kv_heads, bits, residual, page, n_pages, cap_r)
        self.cache = kivi.PagedCache(self.layout)
        for buf in self.cache.buffers.values():
            buf.fill_(0xFF)                                             # NaN wherever nothing was stored
        order = self.rng.permutation(n_pages)[:sequences * self.pages_each].reshape(sequences, self.pages_each)
        wide = np.full((sequences, self.pages_each + 3), -7, np.int32)          # (rows of the table are strided)
        wide[:, :self.pages_each] = order
        self.table = torch.from_numpy(wide).cuda()[:, :self.pages_each]
        self.order = order
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.batch = kivi.PagedBatch(self.table, self.lengths, None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda"))
        self.oracle = [ref.Sequence(kv_heads, bits, residual) for _ in range(sequences)]
        self.gain = np.ones((kv_heads, 128))
        self.gain[:, self.rng.permutation(128)[:5]] = 10.0

    def new_rows(self, n):
        k = self.rng.standard_normal((n, self.kv_heads, 128)) * self.gain
        return k.astype(np.float16), self.rng.standard_normal((n, self.kv_heads, 128)).astype(np.float16)

    def append(self, counts, table=None, interleaved=False, bf16=False, uniform=False, positions=None):
        """counts[i] new tokens for sequence i."""
        torch = self.torch
        before = np.array([o.length for o in self.oracle])
        n = int(sum(counts))
        k, v = self.new_rows(n)
        q = self.rng.standard_normal((n, self.q_heads, 128)).astype(np.float16)
        kt, vt, qt = (torch.from_numpy(x).cuda() for x in (k, v, q))
        if bf16:
            kt, vt, qt = (x.bfloat16() for x in (kt, vt, qt))
            k, v, q = (x.float().cpu().numpy() for x in (kt, vt, qt))
            v = v.astype(np.float16)
        starts = np.cumsum([0] + list(counts)).astype(np.int32)
        self.lengths.copy_(torch.from_numpy((before + counts).astype(np.int32)))
        pos = np.concatenate([np.arange(b, b + c) for b, c in zip(before, counts)]) if n else np.zeros(0, int)
        if positions is not None:
            pos = positions
        rotation = kivi.Rotation(torch.from_numpy(table).cuda(), interleaved) if table is not None else None
        q_out = torch.full((n, self.q_heads, 128), float("nan"), dtype=torch.float16, device="cuda") if table is not None else None
        # the rows come out of a projection: [rows, q heads + 2 kv heads, 128]
        qkv = torch.cat([qt, kt, vt], 1)
        hq, h = self.q_heads, self.kv_heads
        kivi.kivi_paged_append(self.cache, self.batch, qkv[:, hq:hq + h], qkv[:, hq + h:], starts=None if uniform else torch.from_numpy(starts).cuda(),
                               max_new=max(max(counts), 1), rotation=rotation, q=qkv[:, :hq] if table is not None else None, q_out=q_out,
                               positions=torch.from_numpy(pos.astype(np.int32)).cuda() if positions is not None else None)
        torch.cuda.synchronize()
        if table is not None:
            at = table[pos.clip(0, len(table) - 1)]
            k = ref.rotate(k.astype(np.float32), at, interleaved).astype(np.float16)
            rq = ref.rotate(q.astype(np.float32), at, interleaved).astype(np.float16)
            assert np.array_equal(q_out.cpu().numpy().view(np.uint16), rq.view(np.uint16)), "rotated queries"
        k = k.astype(np.float16)
        for i, o in enumerate(self.oracle):
            if counts[i]:
                o.append(k[starts[i]:starts[i + 1]], v[starts[i]:starts[i + 1]])

    def check_cache(self):
        records, cap = self.cache.records().cpu().numpy().view(np.uint32), self.layout.cap_r_tokens
        rings = [self.cache.rows(n).cpu().numpy() for n in ("k_resid", "v_resid")]
        per_page = self.page // 32
        touched = np.zeros(records.shape[0], bool)
        for i, o in enumerate(self.oracle):
            want = o.records()
            for r in range(want.shape[0]):
                page = self.order[i, r // per_page]
                touched[page] = True
                got = records[page, :, r % per_page]
                assert np.array_equal(got, want[r]), f"sequence {i}, record {r}"
            slot = np.arange(want.shape[0] * 32, o.length) % cap
            for ring, rows in zip(rings, o.rows()):
                got = ring[self.slots[i]][:, slot].transpose(1, 0, 2)
                assert np.array_equal(got.view(np.uint16), rows.view(np.uint16)), f"sequence {i}, fp16 rows"
        assert (records[~touched] == 0xFFFFFFFF).all(), "a page that belongs to nobody was written"

    def attention(self, window=0, sinks=0, dtype="fp16", scale=128 ** -0.5, lost=None):
        """lost: per sequence, tokens whose pages are missing."""
        torch = self.torch
        n = len(self.oracle)
        q = torch.from_numpy(self.rng.standard_normal((n, self.q_heads, 128)).astype(np.float16)).cuda()
        out = torch.full(q.shape, 9.0, dtype=torch.float16 if dtype == "fp16" else torch.bfloat16, device="cuda")
        kivi.kivi_paged_attention(self.cache, self.batch, q, scale, out, window=window, sinks=sinks)
        torch.cuda.synchronize()
        got, qn = out.double().cpu().numpy(), q.cpu().numpy()
        for i, o in enumerate(self.oracle):
            if o.length == 0:
                assert (got[i] == 9).all(), f"sequence {i} is empty: its row stays"
                continue
            k, v, km, vm = o.values()
            see = ref.visible(1, o.length, window, sinks)
            if lost is not None:
                see[:, lost[i]] = False
            want, _, _ = ref.attention(qn[i][None], k, v, scale, see)
            # magnitudes: the logits' terms, and the values' under the same weights
            _, _, terms = ref.attention(np.abs(qn[i][None]), km, vm, scale, see)
            weights = _weighted(qn[i], k, vm, scale, see[0])
            tol = 1.01 * HALF_STEP[dtype] * np.abs(want[0]) + (2 * (2.0 ** -20 + 129 * 2.0 ** -24) * terms[0] + 2.0 ** -13) * weights + 2.0 ** -25
            over = np.abs(got[i] - want[0]) - tol
            assert np.isfinite(got[i]).all() and over.max() <= 0, f"sequence {i} of {o.length} tokens: tolerance passed by {over.max():.3e}"


def _weighted(q, k, vm, scale, see):
    """mean of vm under the attention's weights: [H_q, 128]"""
    rep = q.shape[0] // k.shape[1]
    out = np.zeros(q.shape)
    for h in range(q.shape[0]):
        x = np.where(see, scale * (k[:, h // rep] @ q[h].astype(np.float64)), -np.inf)
        p = np.where(see, np.exp(x - max(x.max(), -1e300)), 0.0)
        out[h] = p @ vm[:, h // rep] / max(p.sum(), 1e-300)
    return out


LENGTHS = [1, 2, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 160, 191, 224, 287, 355, 500]


@pytest.mark.parametrize("bits,q_heads,kv_heads,page,residual", [
    (2, 4, 4, 64, 64), (4, 3, 3, 128, 64), (4, 4, 2, 32, 64), (2, 12, 3, 128, 96), (4, 8, 1, 64, 32), (2, 16, 2, 32, 128), (4, 11, 1, 256, 64), (2, 3, 1, 64, 0),
])
def test_prompts_of_all_lengths(bits, q_heads, kv_heads, page, residual):
    print(f"case paged prompts bits={bits} heads={q_heads}/{kv_heads} page={page} R={residual}", flush=True)
    run = Run(len(LENGTHS), q_heads, kv_heads, bits, residual, page)
    run.append(LENGTHS)
    run.check_cache()
    run.attention()
    for window, sinks in ((1, 0), (40, 4), (100, 33), (300, 0), (90, 200), (10000, 4)):
        print(f"  window={window} sinks={sinks}", flush=True)
        run.attention(window, sinks)


@pytest.mark.parametrize("bits,q_heads,kv_heads,rotary,interleaved,bf16", [
    (2, 4, 4, 128, False, False), (4, 8, 2, 128, True, False), (2, 14, 2, 64, False, True), (4, 3, 3, 96, True, True), (2, 2, 1, 16, False, False),
])
def test_steps_with_rotation(bits, q_heads, kv_heads, rotary, interleaved, bf16):
    """Prompts, then single tokens, then chunks on top, all rotated on the way."""
    print(f"case paged steps bits={bits} heads={q_heads}/{kv_heads} rotary={rotary} bf16={bf16}", flush=True)
    table = ref.table(420, rotary)                     # (the longest sequence passes the table's end)
    run = Run(5, q_heads, kv_heads, bits, most=640)
    run.append([70, 1, 130, 95, 33], table, interleaved, bf16)
    run.check_cache()
    for _ in range(40):
        run.append([1] * 5, table, interleaved, bf16, uniform=True)
    run.check_cache()
    run.attention(dtype="bf16" if bf16 else "fp16")
    run.append([0, 200, 33, 1, 0], table, interleaved, bf16)
    run.check_cache()
    run.append([17, 2, 300, 64, 96], table, interleaved, bf16)
    run.check_cache()
    run.append([3] * 5, table, interleaved, bf16, uniform=True, positions=np.arange(15) * 9 - 4)
    run.check_cache()
    run.attention(window=77, sinks=5)


@pytest.mark.parametrize("bits,q_heads,kv_heads", [(2, 71, 1), (4, 128, 1), (2, 20, 2)])
def test_wide_groups(bits, q_heads, kv_heads):
    """More query heads per kv-head than a unit has: runs of them."""
    print(f"case paged wide groups {q_heads}/{kv_heads} bits={bits}", flush=True)
    run = Run(3, q_heads, kv_heads, bits)
    run.append([40, 500, 161])
    run.attention()
    run.attention(window=120, sinks=3)


@pytest.mark.parametrize("q_heads", [2, 6])
@pytest.mark.parametrize("scale", [0.0, -0.05])
def test_softmax_scales(scale, q_heads):
    run = Run(2, q_heads, 2, 2)
    run.append([400, 70])
    run.attention(scale=scale)
    run.attention(scale=scale, window=100, sinks=33)


def test_larger_rings_and_slots():
    """A ring with room to spare (a chunk is one launch then), rows of the batch in other slots, a batch smaller than the cache."""
    run = Run(3, 4, 2, 2, cap_r=256, slots=[6, 0, 3])
    for counts in ([200, 50, 7], [90, 100, 1], [1, 1, 1], [5, 64, 99]):
        run.append(counts)
        run.check_cache()
    run.attention()


def test_empty_and_invalid_sequences():
    """Empty sequences, slots and pages out of range, counts that do not fit: left out, the others unharmed."""
    torch = gh.require_gpu()
    run = Run(4, 4, 2, 2)
    run.append([300, 0, 200, 40])
    run.check_cache()
    run.attention()
    # a page outside [0, n_pages): its tokens count as masked
    per = run.page
    kept = run.table.clone()
    run.table[0, 1] = run.layout.n_pages
    run.table[2, 0] = -1
    lost = [np.arange(per, 2 * per), np.zeros(0, int), np.arange(0, per), np.zeros(0, int)]
    run.attention(lost=lost)
    run.attention(window=150, sinks=3, lost=lost)
    # a table narrower than the sequences
    narrow = kivi.PagedBatch(run.table[:, :0], run.lengths)
    q = torch.randn(4, 4, 128, device="cuda").half()
    out = torch.full((4, 4, 128), 9.0, dtype=torch.float16, device="cuda")
    kivi.kivi_paged_attention(run.cache, narrow, q, 0.1, out)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all() and (out[1] == 9).all()
    # slots outside the cache: nothing is read, the rows stay
    bad = kivi.PagedBatch(run.table, run.lengths, torch.tensor([-1, 1, 4, 3], dtype=torch.int32, device="cuda"))
    out.fill_(9.0)
    kivi.kivi_paged_attention(run.cache, bad, q, 0.1, out)
    torch.cuda.synchronize()
    assert (out[[0, 1, 2]] == 9).all() and torch.isfinite(out[3]).all() and not (out[3] == 9).all()
    # everything behind a missing page: a row that sees nothing but it is 0
    run.table.copy_(kept)
    before = [b.clone() for b in run.cache.buffers.values()]
    k, v = (torch.randn(8, 2, 128, device="cuda").half() for _ in range(2))
    starts = torch.tensor([0, 2, 1, 8, 9], dtype=torch.int32, device="cuda")        # fits | decreases | above max_new | outside the rows
    run.lengths += 2
    kivi.kivi_paged_append(run.cache, bad, k, v, starts=starts, max_new=4)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, run.cache.buffers.values()))      # (sequence 0's slot is -1)


def test_sequences_of_which_nothing_is_visible():
    """No fp16 rows (R = 0) and no pages: rows of 0, between sequences that have some."""
    torch = gh.require_gpu()
    run = Run(5, 4, 2, 2, residual=0, most=320)
    run.append([64, 33, 320, 32, 100])
    run.check_cache()
    run.attention()
    none = run.table.clone()
    none[[0, 2, 3]] = -1
    q = torch.randn(5, 4, 128, device="cuda").half()
    for table in (none, none[:, :0]):
        out = torch.full((5, 4, 128), 9.0, dtype=torch.float16, device="cuda")
        kivi.kivi_paged_attention(run.cache, kivi.PagedBatch(table, run.lengths), q, 0.1, out)
        torch.cuda.synchronize()
        assert (out[[0, 2, 3]] == 0).all() and torch.isfinite(out).all()
        assert not (out[[1, 4]] == 0).all(-1).any()


def test_two_rows_of_one_sequence_and_prefix_pages():
    """Attention may read one sequence twice, and pages that two sequences share."""
    torch = gh.require_gpu()
    run = Run(2, 4, 1, 2)
    run.append([400, 150])
    twice = kivi.PagedBatch(run.table[:1].repeat(3, 1), run.lengths[:1].repeat(3), torch.zeros(3, dtype=torch.int32, device="cuda"))
    q = torch.randn(1, 4, 128, device="cuda").half().repeat(3, 1, 1)
    out = torch.empty_like(q)
    kivi.kivi_paged_attention(run.cache, twice, q, 0.1, out)
    alone = torch.empty_like(q[:1])
    kivi.kivi_paged_attention(run.cache, kivi.PagedBatch(run.table[:1], run.lengths[:1]), q[:1], 0.1, alone)
    torch.cuda.synchronize()
    assert (out[0] - alone[0]).abs().max() <= 2 * 2.0 ** -11 * alone.abs().max()
    assert (out[1] - alone[0]).abs().max() <= 2 * 2.0 ** -11 * alone.abs().max()


@pytest.mark.parametrize("q_heads,kv_heads", [(4, 2), (2, 2), (7, 1)])
@pytest.mark.parametrize("bits,scale", [(2, 40.0), (4, 40.0), (2, 3000.0), (4, 3000.0), (2, 1e-3)])
def test_scales_out_of_the_ordinary(bits, scale, q_heads, kv_heads):
    """Keys and values whose group scales pass what the operands hold without a shift, next to small ones."""
    print(f"case paged scales bits={bits} heads={q_heads}/{kv_heads} values times {scale}", flush=True)
    run = Run(2, q_heads, kv_heads, bits, most=400)
    plain = run.new_rows

    def rows(n):
        k, v = plain(n)
        k, v = k.astype(np.float64), v.astype(np.float64)
        k[:, :, 7] *= scale / 4
        v[n // 2:, :, 32:64] *= scale                                  # from some token on, one group of channels
        return k.astype(np.float16), v.astype(np.float16)
    run.new_rows = rows
    run.append([330, 97])
    run.check_cache()
    run.attention(scale=0.01)


def test_long_sequences_are_divided():
    """One long sequence (many parts, joined), and a batch of many (several units per workgroup)."""
    run = Run(1, 9, 1, 2, most=20000, page=256, residual=128)
    run.append([19999])
    run.attention()
    run.attention(window=4000, sinks=70)
    run.attention()                                    # (the workspace is ready for the next call)
    for bits in (2, 4):
        one = Run(2, 1, 1, bits, most=9000, page=512, residual=128)
        one.append([8999, 5000])
        one.attention()
        one.attention(window=700, sinks=300)
    many = Run(150, 6, 3, 4, most=192)
    many.append([int(x) for x in np.random.default_rng(3).integers(1, 190, 150)])
    many.check_cache()
    many.attention()


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (8, 4)])
@pytest.mark.parametrize("batch", [65, 257, 300])
def test_batches_of_many_short_sequences(batch, q_heads, kv_heads):
    """More sequences than a workgroup looks at in one go, short ones with a few long ones between, whole and through a window."""
    print(f"case paged many batch={batch} heads={q_heads}/{kv_heads}", flush=True)
    run = Run(batch, q_heads, kv_heads, 2, most=704, page=64)
    lengths = np.random.default_rng(batch).integers(1, 41, batch)
    lengths[::19] = 700
    lengths[-1] = 333
    run.append([int(x) for x in lengths])
    run.attention()
    run.attention(window=50, sinks=3)


def test_graph_replays_follow_the_lengths():
    """A captured step (append with rotation, attention) replayed while lengths and pages move on, with eager calls between."""
    torch = gh.require_gpu()
    run = Run(3, 8, 2, 2, most=400)
    run.append([100, 60, 290])
    table = kivi.Rotation(torch.from_numpy(ref.table(500, 128)).cuda())
    gen = torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.randn(3, 12, 128, device="cuda", generator=gen).half()
    q_out, out = torch.empty(3, 8, 128, dtype=torch.float16, device="cuda"), torch.empty(3, 8, 128, dtype=torch.float16, device="cuda")
    eager = kivi.PagedCache(run.layout)
    for name in eager.buffers:
        eager.buffers[name].copy_(run.cache.buffers[name])

    def step(cache, to):
        kivi.kivi_paged_append(cache, run.batch, qkv[:, 8:10], qkv[:, 10:], rotation=table, q=qkv[:, :8], q_out=q_out)
        kivi.kivi_paged_attention(cache, run.batch, q_out, 0.1, to)
    run.lengths += 1
    step(run.cache, out)                               # (warm-up: the same step that the first replay repeats)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(run.cache, out)
    want = torch.empty_like(out)
    for i in range(70):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        step(eager, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), f"replay {i}"
        assert all(torch.equal(run.cache.buffers[n], eager.buffers[n]) for n in eager.buffers), f"replay {i}"
        run.lengths += 1
        qkv.normal_(generator=gen)
