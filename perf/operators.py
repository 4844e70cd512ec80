"""The serving operators around the packed cache, as cases that can be timed and checked.

A serving program runs, for each layer: per-head norms and the position rotation of queries and keys
(kivi_norm_rotate), the prompt's attention (kivi_prompt_attention), the append of keys and values to a paged
cache with packed records and an fp16 window (kivi_paged_append, which rotates on the way), and the attention of
one new token per sequence over that cache (kivi_paged_attention).  A case is one pass through one of them.

Where `own` is false, `run` computes the same in elementary torch operations in 32 bits; where it is true, it makes the
calls that a program makes.

The paged cache: page p holds for each kv-head page_tokens / 32 records; a record is 32 tokens' key codes, key scales,
key zero-points (one per channel), value scales, value zero-points (one per token and 32 channels) and value codes.  Of a
sequence of n tokens the first floor(max(n - R, 0) / 32) * 32 are packed, the others are fp16 rows in ring slot t % cap_r.
"""
import math
import random

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
GROUP = 32


# ---------------------------------------------------------------- cases

def _norm_rotate(name, rows, q_heads, kv_heads, dtype="fp16", rotary=128, interleaved=False, norm=True):
    return {"name": name, "op": "norm_rotate", "rows": rows, "q_heads": q_heads, "kv_heads": kv_heads, "dtype": dtype,
            "rotary": rotary, "interleaved": interleaved, "norm": norm}


def _prompt(name, batch, q_heads, kv_heads, tokens, dtype="fp16", window=0, sinks=0, before=0, spread=0):
    """`before`: keys of the sequence before its new tokens; `spread` > 0: sequences of different lengths, down to tokens / spread."""
    return {"name": name, "op": "prompt", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "tokens": tokens,
            "dtype": dtype, "window": window, "sinks": sinks, "before": before, "spread": spread}


def _append(name, batch, q_heads, kv_heads, before, new, bits=2, residual=128, page=64, dtype="fp16", rotate=True, spread=0):
    return {"name": name, "op": "append", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "before": before,
            "new": new, "bits": bits, "residual": residual, "page": page, "dtype": dtype, "rotate": rotate, "spread": spread}


def _decode(name, batch, q_heads, kv_heads, tokens, bits=2, residual=128, page=64, window=0, sinks=0, spread=0):
    return {"name": name, "op": "decode", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "tokens": tokens,
            "bits": bits, "residual": residual, "page": page, "window": window, "sinks": sinks, "spread": spread}


def listed():
    return [
        # one new token of one user, 32 / 8 heads, a model with per-head norms: launch latency
        _norm_rotate("norm_rotate_token", 1, 32, 8),
        # the benchmark's prompts (16 of 4096 tokens, 32 / 32 heads)
        _norm_rotate("norm_rotate_prompts", 16 * 4096, 32, 32, dtype="bf16"),
        # one short prompt, four heads
        _prompt("prompt_short", 1, 4, 4, 1001),
        # a batch of prompts, 32 / 8 heads, plain causal attention
        _prompt("prompt_batch", 4, 32, 8, 4096, dtype="bf16"),
        # one long prompt of odd length in a layer with a sliding window and four tokens that stay visible
        _prompt("prompt_window", 1, 32, 8, 8001, window=2048, sinks=4),
        # one user's next token, rotated on the way
        _append("append_token", 1, 32, 32, 3000, 1),
        # a serving batch: one token for each of 64 sequences of different lengths; some of them pack a group
        _append("append_batch", 64, 32, 8, 8000, 1, dtype="bf16", spread=16),
        # the benchmark's prompts into the cache (rotated already)
        _append("append_prompts", 16, 32, 32, 0, 4096, rotate=False),
        # one user in the middle of a chat
        _decode("decode_one_user", 1, 32, 32, 3001),
        # the serving batch of different lengths
        _decode("decode_batch", 64, 32, 8, 8000, spread=16),
        # long contexts at 4 bits, eight query heads per kv-head
        _decode("decode_long_4bit", 16, 64, 8, 32767, bits=4, page=128),
        # a layer with a sliding window over the same kind of cache
        _decode("decode_window", 32, 32, 32, 16001, window=4096, sinks=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(4, 4), (16, 8), (32, 32), (40, 40), (24, 8), (32, 8), (28, 4), (64, 8), (71, 1)]


def draw(rng):
    op = rng.choice(["norm_rotate", "prompt", "prompt", "append", "append", "decode", "decode", "decode"])
    q_heads, kv_heads = rng.choice(_HEADS)
    dtype = rng.choice(["fp16", "bf16"])
    window = rng.choice([0, 0, _log(rng, 1, 8192)])
    sinks = rng.choice([0, 4, rng.randrange(1, 100)]) if window else 0
    bits, page, residual = rng.choice([2, 2, 4]), rng.choice([32, 64, 64, 128, 256]), rng.choice([32, 64, 96, 128, 128, 192])
    spread = rng.choice([0, 0, 2, 16])
    if op == "norm_rotate":
        rows = _log(rng, 1, 16 * 4096 * 64 // (q_heads + kv_heads))
        return {"op": op, "rows": rows, "q_heads": q_heads, "kv_heads": kv_heads, "dtype": dtype,
                "rotary": rng.choice([128, 128, 64, 96]), "interleaved": rng.random() < 0.3, "norm": rng.random() < 0.7}
    if op == "prompt":
        tokens = _log(rng, 1, 8192)
        batch = _log(rng, 1, max(1, min(64, 4 * 32 * 4096 * 4096 // (q_heads * tokens * tokens))))
        if q_heads * tokens * tokens > 4 * 32 * 4096 * 4096:
            q_heads, kv_heads = 28, 4
        before = rng.choice([0, 0, _log(rng, 1, max(1, min(8000, 4 * 32 * 4096 * 4096 // (batch * q_heads * tokens) - tokens)))])
        return {"op": op, "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "tokens": tokens, "dtype": dtype,
                "window": window, "sinks": sinks, "before": before, "spread": spread}
    if op == "append":
        if rng.random() < 0.6:
            new, before = 1, _log(rng, 1, 16000)
            batch = _log(rng, 1, max(1, min(256, 64 * 8 * 16000 // (kv_heads * before))))
        else:
            new, before = _log(rng, 2, 16384), 0
            batch = _log(rng, 1, max(1, min(64, 16 * 32 * 4096 // (kv_heads * new))))
        return {"op": op, "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "before": before, "new": new, "bits": bits,
                "residual": residual, "page": page, "dtype": dtype, "rotate": rng.random() < 0.7, "spread": spread}
    tokens = _log(rng, 1, 32768)
    batch = _log(rng, 1, max(1, min(256, 16 * 8 * 32768 // (kv_heads * tokens))))
    return {"op": op, "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "tokens": tokens, "bits": bits, "residual": residual,
            "page": page, "window": window, "sinks": sinks, "spread": spread}


def _lengths(n, batch, spread):
    """Lengths of a batch: n, or between n / spread and n."""
    if not spread:
        return [n] * batch
    rng = random.Random(n * 1000 + batch)
    return [n if i == 0 else rng.randint(max(1, n // spread), max(1, n)) for i in range(batch)]


def _packed(n, residual):
    return max(n - residual, 0) // GROUP * GROUP


def _cap_r(residual):
    return residual + GROUP


def _pages_of(n, case):
    return -(-_packed(n, case["residual"]) // case["page"])


def _record_words(bits):
    return 256 + 2 * 128 * bits


# ---------------------------------------------------------------- inputs

_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _table(positions, rotary):
    """Cosines and sines of every position (angles in 64 bits), as a program makes them once."""
    freq = 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / rotary)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()


def _gain(heads, gen):
    """A few channels of large magnitude per kv-head: the pattern of keys that per-channel groups are made for."""
    gain = torch.ones(heads, D, device="cuda")
    at = torch.rand(heads, D, device="cuda", generator=gen).argsort(1)[:, :6]
    return gain.scatter_(1, at, 8 + 7 * torch.rand(heads, 6, device="cuda", generator=gen))


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(lens):
    return _ints([0] + lens).cumsum(0).int()


def _inputs_norm_rotate(case, seed):
    gen, dt = _generator(seed), _TYPES[case["dtype"]]
    heads = case["q_heads"] + 2 * case["kv_heads"]
    x = torch.randn(case["rows"], heads, D, device="cuda", generator=gen, dtype=dt)      # a projection's output: q, k, v of a row
    s = {"qkv": x, "q": x[:, :case["q_heads"]], "k": x[:, case["q_heads"]:case["q_heads"] + case["kv_heads"]]}
    s["positions"] = torch.randint(0, 8192, (case["rows"],), device="cuda", generator=gen, dtype=torch.int32)
    for n in ("q_weight", "k_weight"):
        s[n] = (1 + 0.2 * torch.randn(D, device="cuda", generator=gen)).to(dt) if case["norm"] else None
    s["table"] = _table(8192, case["rotary"])
    return s


def _inputs_prompt(case, seed):
    gen, dt = _generator(seed), _TYPES[case["dtype"]]
    new = _lengths(case["tokens"], case["batch"], case["spread"])
    keys = [n + case["before"] for n in new]
    s = {"new": new, "keys": keys, "q_starts": _starts(new), "k_starts": _starts(keys)}
    gain = (_gain(case["kv_heads"], gen) ** 0.5).to(dt)
    s["q"] = torch.randn(sum(new), case["q_heads"], D, device="cuda", generator=gen, dtype=dt)
    s["k"] = torch.randn(sum(keys), case["kv_heads"], D, device="cuda", generator=gen, dtype=dt) * gain
    s["v"] = torch.randn(sum(keys), case["kv_heads"], D, device="cuda", generator=gen, dtype=dt)
    return s


def _quantise(x, levels, dim):
    """Codes, scale and zero-point of fp16 groups along `dim`, by the quantiser's contract."""
    lo, hi = x.amin(dim, keepdim=True), x.amax(dim, keepdim=True)
    s = ((hi.float() - lo.float()) / levels).half()
    sf = s.float()
    code = ((x.float() - lo.float()) / torch.where(sf == 0, 1.0, sf)).round_().clamp_(0, levels)
    return torch.where(sf == 0, 0.0, code).int(), s, lo


def _code_words(codes, bits, keys):
    """[n, 32 tokens, 128 channels] codes -> [n, 128 * bits] words in the cache's order."""
    n = codes.shape[0]
    if keys:        # token = half 16 + row, channel = block 32 + kb 8 + (e4 e2 e1)
        x = codes.view(n, 2, 16, 4, 4, 2, 2, 2).permute(0, 4, 2, 3, 1, 5, 6, 7)            # n kb row block | half e4 e2 e1
    else:           # channel = block 32 + half 16 + row, token = kb 8 + (e4 e2 e1)
        x = codes.view(n, 4, 2, 2, 2, 4, 2, 16).permute(0, 1, 7, 5, 6, 2, 3, 4)            # n kb row block | half e4 e2 e1
    i = torch.arange(2, device=codes.device, dtype=torch.int32)
    half, e4, e2, e1 = i[:, None, None, None], i[:, None, None], i[:, None], i
    if bits == 2:
        w = (x << (e1 * 16 + 2 * (half * 4 + e4 * 2 + e2))).sum((4, 5, 6, 7), dtype=torch.int64)     # n kb row block
        w = w.reshape(n, 256)
    else:
        w = (x << (e1 * 16 + 4 * (half * 2 + e2))).sum((4, 6, 7), dtype=torch.int64)                # n kb row block e4
        w = w.view(n, 64, 2, 4).permute(0, 2, 1, 3).reshape(n, 512)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).int()


def _codes(words, bits, keys):
    """The inverse of _code_words, as integers [n, 32, 128]."""
    n = words.shape[0]
    i = torch.arange(2, device=words.device, dtype=torch.int32)
    half, e4, e2, e1 = i[:, None, None, None], i[:, None, None], i[:, None], i
    if bits == 2:
        x = words.view(n, 4, 16, 4, 1, 1, 1, 1) >> (e1 * 16 + 2 * (half * 4 + e4 * 2 + e2))
    else:
        w = words.view(n, 2, 64, 2, 2).permute(0, 2, 1, 3, 4).reshape(n, 4, 16, 4, 1, 2, 1, 1)
        x = w >> (e1 * 16 + 4 * (half * 2 + e2))
    x = x & (2 ** bits - 1)
    if keys:
        return x.permute(0, 4, 2, 3, 1, 5, 6, 7).reshape(n, 32, D)
    return x.permute(0, 1, 5, 6, 7, 3, 4, 2).reshape(n, 32, D)


def _records(k, v, bits):
    """[n, 32, 128] fp16 keys and values -> [n, words] records."""
    n, levels = k.shape[0], 2 ** bits - 1
    kc, ks, kz = _quantise(k, levels, 1)
    vc, vs, vz = _quantise(v.view(n, 32, 4, 32), levels, 3)
    parts = [t.reshape(n, 128).contiguous().view(torch.int32) for t in (ks, kz, vs, vz)]
    return torch.cat([_code_words(kc, bits, True)] + parts + [_code_words(vc.view(n, 32, D), bits, False)], 1)


def _unpack(rec, bits, dtype=torch.float32):
    """[n, words] records -> keys and values [n, 32, 128]."""
    n, w = rec.shape[0], 128 * bits
    ks, kz, vs, vz = rec[:, w:w + 256].contiguous().view(torch.float16).view(n, 4, 128).to(dtype).unbind(1)
    k = _codes(rec[:, :w].contiguous(), bits, True).to(dtype) * ks[:, None] + kz[:, None]
    v = _codes(rec[:, w + 256:].contiguous(), bits, False).to(dtype).view(n, 32, 4, 32)
    return k, (v * vs.view(n, 32, 4, 1) + vz.view(n, 32, 4, 1)).view(n, 32, D)


def _page_table(case, lens, gen):
    """Pages of all sequences in random order, and a few that belong to nobody."""
    used = [_pages_of(n, case) for n in lens]
    order = torch.randperm(sum(used) + 3, device="cuda", generator=gen).int()
    width = max(used) + 1
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(used) + 3


def _rows(case, lens, gen):
    """Keys (rotated) and values of all sequences as [tokens of the batch, kv-head, 128]."""
    h = case["kv_heads"]
    k = torch.randn(sum(lens), h, D, device="cuda", generator=gen, dtype=torch.float16) * _gain(h, gen).half()
    return k, torch.randn(sum(lens), h, D, device="cuda", generator=gen, dtype=torch.float16)


def _fill(case, lens, table, pool, rings, k, v):
    """What earlier calls left in the cache: records of the packed tokens, fp16 rows of the window."""
    h, tiles, at = case["kv_heads"], case["page"] // GROUP, 0
    for b, n in enumerate(lens):
        nq = _packed(n, case["residual"])
        for lo in range(0, nq, 8192):
            hi = min(nq, lo + 8192)
            kk, vv = (x[at + lo:at + hi].view(-1, 32, h, D).transpose(1, 2).reshape(-1, 32, D) for x in (k, v))
            t = torch.arange(lo // GROUP, hi // GROUP, device="cuda")
            pool[table[b, t // tiles].long(), :, t % tiles] = _records(kk, vv, case["bits"]).view(hi // GROUP - lo // GROUP, h, -1)
        slot = torch.arange(nq, n, device="cuda") % _cap_r(case["residual"])
        rings[0][b][:, slot] = k[at + nq:at + n].transpose(0, 1)
        rings[1][b][:, slot] = v[at + nq:at + n].transpose(0, 1)
        at += n


def _cache(case, lens_before, lens_after, gen):
    table, pages = _page_table(case, lens_after, gen)
    h = case["kv_heads"]
    pool = torch.zeros(pages, h, case["page"] // GROUP, _record_words(case["bits"]), dtype=torch.int32, device="cuda")
    rings = [torch.zeros(len(lens_after), h, _cap_r(case["residual"]), D, dtype=torch.float16, device="cuda") for _ in range(2)]
    k, v = _rows(case, lens_before, gen)
    _fill(case, lens_before, table, pool, rings, k, v)
    return {"table": table, "pool": pool, "k_ring": rings[0], "v_ring": rings[1], "lengths": _ints(lens_after)}


def _inputs_append(case, seed):
    gen, dt = _generator(seed), _TYPES[case["dtype"]]
    before = _lengths(case["before"], case["batch"], case["spread"]) if case["before"] else [0] * case["batch"]
    new = [1] * case["batch"] if case["new"] == 1 else _lengths(case["new"], case["batch"], case["spread"])
    after = [a + b for a, b in zip(before, new)]
    s = _cache(case, before, after, gen)
    x = torch.randn(sum(new), case["q_heads"] + 2 * case["kv_heads"], D, device="cuda", generator=gen, dtype=dt)
    hq, h = case["q_heads"], case["kv_heads"]
    x[:, hq:hq + h] *= _gain(h, gen).to(dt)
    s.update(qkv=x, q=x[:, :hq], k=x[:, hq:hq + h], v=x[:, hq + h:], new=new, before=before, starts=_starts(new),
             table_rot=_table(max(after), D) if case["rotate"] else None)
    return s


def _inputs_decode(case, seed):
    gen = _generator(seed)
    lens = _lengths(case["tokens"], case["batch"], case["spread"])
    s = _cache(case, lens, lens, gen)
    s.update(lens=lens, q=torch.randn(case["batch"], case["q_heads"], D, device="cuda", generator=gen, dtype=torch.float16))
    return s


def _handle(case, s):
    """The framework's handles of a paged cache that lies in the state's buffers."""
    from paper_2402_02750_amd import kivi
    layout = kivi.make_paged_layout(max_sequences=case["batch"], n_q_heads=case["q_heads"], n_kv_heads=case["kv_heads"], bits=case["bits"],
                                    residual=case["residual"], page_tokens=case["page"], n_pages=s["pool"].shape[0],
                                    cap_r_tokens=_cap_r(case["residual"]))
    s["cache"] = kivi.PagedCache(layout, pages=s["pool"], k_resid=s["k_ring"], v_resid=s["v_ring"])
    s["batch"] = kivi.PagedBatch(s["table"], s["lengths"])


def prepare(case, seed):
    s = {"norm_rotate": _inputs_norm_rotate, "prompt": _inputs_prompt, "append": _inputs_append, "decode": _inputs_decode}[case["op"]](case, seed)
    s["case"] = case
    if case["op"] == "norm_rotate":
        s["out"] = {"q": torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda"), "k": torch.empty(s["k"].shape, dtype=s["k"].dtype, device="cuda")}
    elif case["op"] == "prompt":
        s["out"] = torch.empty_like(s["q"])
    elif case["op"] == "append":
        s["q_out"] = torch.empty(s["q"].shape, dtype=torch.float16, device="cuda") if case["rotate"] else None
        s["out"] = _append_outputs(case, s)
    else:
        s["out"] = torch.empty_like(s["q"])
    if own:
        from paper_2402_02750_amd import kivi
        if case["op"] in ("append", "decode"):
            _handle(case, s)
        if case["op"] == "norm_rotate":
            s["rotation"] = kivi.Rotation(s["table"], interleaved=case["interleaved"])
        elif case["op"] == "append" and case["rotate"]:
            s["rotation"] = kivi.Rotation(s["table_rot"])
    return s


def _append_outputs(case, s):
    """The cache after the pass: code words (a bit contract), scales and zero-points, fp16 rows, and the rotated queries."""
    w = 128 * case["bits"]
    out = {"k_codes": s["pool"][..., :w], "v_codes": s["pool"][..., w + 256:], "scales": s["pool"].view(torch.float16)[..., 2 * w:2 * w + 512],
           "k_ring": s["k_ring"], "v_ring": s["v_ring"]}
    if s["q_out"] is not None:
        out["q"] = s["q_out"]
    return out


# ---------------------------------------------------------------- plain forms

def _rotate(x, cos, sin, interleaved):
    """x [..., 128], cos / sin [..., rotary / 2]; each product and the difference rounded on its own."""
    r = cos.shape[-1]
    if interleaved:
        a, b = x[..., 0:2 * r:2], x[..., 1:2 * r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r], x[..., r:2 * r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., 2 * r:]], -1)


def _plain_norm_rotate(s):
    case = s["case"]
    rows = s["table"][s["positions"].long()][:, None]
    cos, sin = rows.chunk(2, -1)
    got = {}
    for n in ("q", "k"):
        x = s[n].float()
        if case["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * s[n + "_weight"].float()
        got[n] = _rotate(x, cos, sin, case["interleaved"]).to(s[n].dtype)
    return got


def _padded(x, starts, most):
    """Rows of ragged sequences as [batch, most, ...]; the last row stands behind the end."""
    at = starts[:-1, None].long() + torch.arange(most, device=x.device)
    return x[at.clamp(max=x.shape[0] - 1)]


def _visible(n_q, n_k, most_q, most_k, window, sinks):
    """[batch, most_q, most_k]: whether query i of a sequence sees its key j."""
    i, j = torch.arange(most_q, device="cuda")[:, None], torch.arange(most_k, device="cuda")
    at = i + (n_k - n_q)[:, None, None]
    see = (j <= at) & (i < n_q[:, None, None])
    if window:
        see &= (at - j < window) | (j < sinks)
    return see


def _plain_prompt(s):
    case = s["case"]
    n_q, n_k = s["q_starts"].diff(), s["k_starts"].diff()
    most_q, most_k = max(s["new"]), max(s["keys"])
    h, rep = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    q = _padded(s["q"].float(), s["q_starts"], most_q).view(-1, most_q, h, rep, D).permute(0, 2, 3, 1, 4).contiguous()
    k = _padded(s["k"].float(), s["k_starts"], most_k).permute(0, 2, 3, 1).contiguous()[:, :, None]
    v = _padded(s["v"].float(), s["k_starts"], most_k).permute(0, 2, 1, 3).contiguous()[:, :, None]
    see = _visible(n_q, n_k, most_q, most_k, case["window"], case["sinks"])
    x = torch.matmul(q.view(-1, h, 1, rep * most_q, D), k).view(-1, h, rep, most_q, most_k)
    x.mul_(SCALE).masked_fill_(~see[:, None, None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.view(-1, h, 1, rep * most_q, most_k), v).view(-1, h, rep, most_q, D) / total.clamp(min=1e-30)
    out = out.permute(0, 3, 1, 2, 4).reshape(-1, most_q, case["q_heads"], D)
    keep = torch.arange(most_q, device="cuda") < n_q[:, None]
    return out[keep].to(s["q"].dtype)


def _plain_append(s):
    case = s["case"]
    h, r, cap, tiles = case["kv_heads"], case["residual"], _cap_r(case["residual"]), case["page"] // GROUP
    length = s["lengths"].long()
    n_new = s["starts"].diff().long()
    old = length - n_new
    seq = torch.repeat_interleave(torch.arange(case["batch"], device="cuda"), n_new, output_size=s["k"].shape[0])
    pos = torch.arange(s["k"].shape[0], device="cuda") - s["starts"][seq].long() + old[seq]
    k, v = s["k"].float(), s["v"].half()
    if case["rotate"]:
        cos, sin = s["table_rot"][pos][:, None].chunk(2, -1)
        k = _rotate(k, cos, sin, False)
        s["q_out"].copy_(_rotate(s["q"].float(), cos, sin, False))
    k = k.half()
    # groups that become packed: rows out of the ring (positions before the call) or of the new ones
    q0, q1 = ((n - r).clamp(min=0) // GROUP for n in (old, length))
    groups = sum(_packed(a + n, r) // GROUP - _packed(a, r) // GROUP for a, n in zip(s["before"], s["new"]))
    if groups:
        b = torch.repeat_interleave(torch.arange(case["batch"], device="cuda"), q1 - q0, output_size=groups)
        g = torch.arange(groups, device="cuda") - ((q1 - q0).cumsum(0) - (q1 - q0))[b] + q0[b]
        t = g[:, None] * GROUP + torch.arange(GROUP, device="cuda")
        fresh = t >= old[b][:, None]
        row = (s["starts"][b].long()[:, None] + t - old[b][:, None]).clamp(min=0)
        kk = torch.where(fresh[..., None, None], k[row], s["k_ring"][b[:, None], :, t % cap])
        vv = torch.where(fresh[..., None, None], v[row], s["v_ring"][b[:, None], :, t % cap])
        rec = _records(kk.transpose(1, 2).reshape(-1, 32, D), vv.transpose(1, 2).reshape(-1, 32, D), case["bits"])
        s["pool"][s["table"][b, g // tiles].long(), :, g % tiles] = rec.view(groups, h, -1)
    stay = pos >= q1[seq] * GROUP
    at = seq[stay], slice(None), pos[stay] % cap
    s["k_ring"][at] = k[stay]
    s["v_ring"][at] = v[stay]
    return s["out"]


def _plain_decode(s):
    case = s["case"]
    h, rep, cap, tiles = case["kv_heads"], case["q_heads"] // case["kv_heads"], _cap_r(case["residual"]), case["page"] // GROUP
    length = s["lengths"].long()
    packed = (length - case["residual"]).clamp(min=0) // GROUP * GROUP
    most = max(s["lens"])
    most_packed = _packed(most, case["residual"])
    t = torch.arange(most, device="cuda")
    rows = (packed[:, None] + torch.arange(case["residual"] + GROUP, device="cuda"))
    parts_k, parts_v, place = [], [], [rows]
    if most_packed:
        g = torch.arange(most_packed // GROUP, device="cuda")
        page = s["table"][:, g // tiles].long().clamp(min=0)
        k, v = _unpack(s["pool"][page, :, g % tiles].flatten(0, 2), case["bits"])
        k, v = (x.view(-1, g.numel(), h, GROUP, D).transpose(1, 2).reshape(-1, h, most_packed, D) for x in (k, v))
        parts_k, parts_v, place = [k], [v], [t[:most_packed].expand(case["batch"], -1), rows]
    ring = torch.arange(case["batch"], device="cuda")[:, None]
    k = torch.cat(parts_k + [s["k_ring"][ring, :, rows % cap].transpose(1, 2).float()], 2)
    v = torch.cat(parts_v + [s["v_ring"][ring, :, rows % cap].transpose(1, 2).float()], 2)
    place = torch.cat(place, 1)
    mine = torch.arange(place.shape[1], device="cuda") >= most_packed
    see = (place < length[:, None]) & (mine | (place < packed[:, None]))
    if case["window"]:
        see &= (place >= length[:, None] - case["window"]) | (place < case["sinks"])
    x = torch.matmul(s["q"].float().view(-1, h, rep, D), k.transpose(2, 3).contiguous()) * SCALE
    x.masked_fill_(~see[:, None, None], -math.inf)
    x = (x - x.amax(-1, keepdim=True)).exp_()
    out = torch.matmul(x, v) / x.sum(-1, keepdim=True)
    return out.view(-1, case["q_heads"], D).half()


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return {"norm_rotate": _plain_norm_rotate, "prompt": _plain_prompt, "append": _plain_append, "decode": _plain_decode}[op](state)
    from paper_2402_02750_amd import kivi
    s = state
    if op == "norm_rotate":
        kivi.kivi_norm_rotate(s["q"], s["out"]["q"], s["k"], s["out"]["k"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6,
                              rotation=s["rotation"], positions=s["positions"])
    elif op == "prompt":
        kivi.kivi_prompt_attention(s["q"], s["k"], s["v"], s["out"], SCALE, q_starts=s["q_starts"], k_starts=s["k_starts"], max_q=max(s["new"]),
                                   max_k=max(s["keys"]), window=case["window"], sinks=case["sinks"])
    elif op == "append":
        kivi.kivi_paged_append(s["cache"], s["batch"], s["k"], s["v"], starts=s["starts"] if case["new"] > 1 else None, max_new=max(s["new"]),
                               rotation=s.get("rotation"), q=s["q"] if case["rotate"] else None, q_out=s["q_out"])
    else:
        kivi.kivi_paged_attention(s["cache"], s["batch"], s["q"], SCALE, s["out"], window=case["window"], sinks=case["sinks"])
    return s["out"]


# ---------------------------------------------------------------- work

def _pairs(n_q, n_k, window, sinks):
    """Visible (query, key) pairs of a sequence."""
    total = 0
    first = n_k - n_q
    if not window:
        return sum(range(first + 1, n_k + 1)) if n_q < 64 else (first + 1 + n_k) * n_q // 2
    for p in range(first, n_k):
        lo = max(0, p - window + 1)
        total += p + 1 - lo + min(sinks, lo)
    return total


def work(case):
    op, hq, h = case["op"], case["q_heads"], case["kv_heads"]
    if op == "norm_rotate":
        rows = case["rows"]
        return {"bytes": rows * ((hq + h) * D * 2 * 2 + 4 + min(rows, 8192) / rows * case["rotary"] * 4), "flops": rows * (hq + h) * D * 8}
    if op == "prompt":
        new = _lengths(case["tokens"], case["batch"], case["spread"])
        pairs = sum(_pairs(n, n + case["before"], case["window"], case["sinks"]) for n in new)
        rows, keys = sum(new), sum(new) + case["before"] * len(new)
        return {"bytes": (rows * hq * 2 + keys * h * 2) * D * 2, "flops": 4 * D * hq * pairs}
    record = _record_words(case["bits"]) * 4
    if op == "append":
        before = _lengths(case["before"], case["batch"], case["spread"]) if case["before"] else [0] * case["batch"]
        new = [1] * case["batch"] if case["new"] == 1 else _lengths(case["new"], case["batch"], case["spread"])
        total = flops = 0
        for a, n in zip(before, new):
            q0, q1 = _packed(a, case["residual"]), _packed(a + n, case["residual"])
            old = max(0, min(q1, a) - q0)                       # rows that come out of the ring
            total += h * ((n + old) * 2 * 2 * D + (q1 - q0) // GROUP * record + (a + n - max(q1, a)) * 2 * 2 * D)
            total += n * (4 * D + hq * 2 * 2 * D) if case["rotate"] else 0
            flops += h * (q1 - q0) * D * 8 + (n * (hq + h) * D * 3 if case["rotate"] else 0)
        return {"bytes": total, "flops": flops}
    total = flops = 0
    for n in _lengths(case["tokens"], case["batch"], case["spread"]):
        nq = _packed(n, case["residual"])
        lo = max(0, n - case["window"]) if case["window"] else 0
        sinks = min(case["sinks"], lo)
        first = lo // GROUP                                     # the first record that the window reaches
        records = max(0, nq // GROUP - first) + min(-(-sinks // GROUP), first, nq // GROUP)
        total += h * (records * record + (n - max(nq, lo)) * 2 * 2 * D) + hq * D * 2 * 2
        flops += 4 * hq * D * (n - lo + sinks)
    return {"bytes": total, "flops": flops}


# ---------------------------------------------------------------- 64 bits

def _exact_rotate(x, angle_table, rotary, interleaved):
    c, s = angle_table[..., :rotary // 2].double(), angle_table[..., rotary // 2:].double()
    y = x.clone()
    pairs = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, rotary // 2), slice(rotary // 2, rotary))
    z = torch.complex(x[..., pairs[0]], x[..., pairs[1]]) * torch.complex(c, s)
    y[..., pairs[0]], y[..., pairs[1]] = z.real, z.imag
    return y


def _exact_attention(q, k, v, see):
    """q [rep, n, D], k / v [m, D], see [n, m] or None, all in 64 bits."""
    x = torch.matmul(q, k.t().contiguous()) * SCALE
    if see is not None:
        x.masked_fill_(~see, -math.inf)
    p = torch.softmax(x, -1)
    if see is not None:
        p = torch.nan_to_num(p)
    return torch.matmul(p, v)


def exact(case, seed):
    op, hq, h = case["op"], case["q_heads"], case["kv_heads"]
    rep = hq // h
    if op == "norm_rotate":
        s = _inputs_norm_rotate(case, seed)
        got = {}
        for n in ("q", "k"):
            got[n] = torch.empty(s[n].shape, dtype=torch.float64, device="cuda")
            for at in range(0, case["rows"], 8192):
                x = s[n][at:at + 8192].double()
                if case["norm"]:
                    x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * s[n + "_weight"].double()
                got[n][at:at + 8192] = _exact_rotate(x, s["table"][s["positions"][at:at + 8192].long()][:, None], case["rotary"], case["interleaved"])
        return got
    if op == "prompt":
        s = _inputs_prompt(case, seed)
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        a = c = 0
        for n, m in zip(s["new"], s["keys"]):
            for lo in range(0, n, 2048):
                hi = min(n, lo + 2048)
                p = torch.arange(m - n + lo, m - n + hi, device="cuda")[:, None]
                j = torch.arange(m, device="cuda")
                see = j <= p
                if case["window"]:
                    see &= (p - j < case["window"]) | (j < case["sinks"])
                for i in range(h):
                    q = s["q"][a + lo:a + hi, i * rep:(i + 1) * rep].double().transpose(0, 1).contiguous()
                    out[a + lo:a + hi, i * rep:(i + 1) * rep] = _exact_attention(q, s["k"][c:c + m, i].double(), s["v"][c:c + m, i].double(), see).transpose(0, 1)
            a, c = a + n, c + m
        return out
    if op == "append":
        s = _inputs_append(case, seed)
        pos = torch.cat([torch.arange(b, b + n, device="cuda") for b, n in zip(s["before"], s["new"])])
        k, got = s["k"].double(), {"k_codes": None, "v_codes": None, "scales": None}
        if case["rotate"]:
            at = s["table_rot"][pos][:, None]
            k = _exact_rotate(k, at, D, False)
            got["q"] = _exact_rotate(s["q"].double(), at, D, False)
        got["k_ring"], got["v_ring"] = s["k_ring"].double(), s["v_ring"].double()
        a = 0
        for b, (m, n) in enumerate(zip(s["before"], s["new"])):     # the new tokens that stay in the window
            lo = max(m, _packed(m + n, case["residual"]))
            slot = torch.arange(lo, m + n, device="cuda") % _cap_r(case["residual"])
            got["k_ring"][b][:, slot] = k[a + lo - m:a + n].transpose(0, 1)
            got["v_ring"][b][:, slot] = s["v"][a + lo - m:a + n].double().transpose(0, 1)
            a += n
        return got
    s = _inputs_decode(case, seed)
    out = torch.empty(case["batch"], hq, D, dtype=torch.float64, device="cuda")
    cap, tiles = _cap_r(case["residual"]), case["page"] // GROUP
    for b, n in enumerate(s["lens"]):
        nq = _packed(n, case["residual"])
        g = torch.arange(nq // GROUP, device="cuda")
        k, v = _unpack(s["pool"][s["table"][b, g // tiles].long(), :, g % tiles].flatten(0, 1), case["bits"], torch.float64)
        slot = torch.arange(nq, n, device="cuda") % cap
        t = torch.arange(n, device="cuda")
        see = None
        if case["window"]:
            see = ((n - 1 - t < case["window"]) | (t < case["sinks"]))[None]
        k, v = (x.view(-1, h, GROUP, D) for x in (k, v))
        for i in range(h):
            ki = torch.cat([k[:, i].reshape(-1, D), s["k_ring"][b, i, slot].double()])
            vi = torch.cat([v[:, i].reshape(-1, D), s["v_ring"][b, i, slot].double()])
            out[b, i * rep:(i + 1) * rep] = _exact_attention(s["q"][b, i * rep:(i + 1) * rep].double()[:, None], ki, vi, see)[:, 0]
    return out
