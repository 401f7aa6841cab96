"""The operators of a block step's attention over a paged cache, as they are measured.

`wino_rope_append` rotates the new rows' queries and keys and writes keys and values into the cache's pages;
`wino_attend` lets the new rows attend over the cache.  Each case is a dict of plain values:

    op       "append" or "attend"
    mask     "full", "causal" or "shadow" (which cached slots a new row sees)
    rows_min, rows_max        new rows of a sequence; shadow: twice the block's length
    context_min, context_max  slots held before the new rows (shadow: with the block's own); lengths are spread over
             their logarithm
    seqs, q_heads, kv_heads, dim, page, dtype, layout ("slots": [pages, slots, heads, dim] in memory, "heads":
             [pages, heads, slots, dim]); lens (the seed of the lengths)
    append only: rot (rotated dims), pairs ("half" or "interleaved"), scaling ("none", "linear" or "parts"), factor

With `own` false, `run` computes the operators in elementary torch operations; with `own` true it calls the library.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
BASE = 500000.0
TRAINED = 8192  # context length the unscaled frequencies were made for ("parts" scaling)
MASKS = {"full": 0, "causal": 1, "shadow": 2}


def _case(name, op, mask, seqs, rows, context, q_heads, kv_heads, dim, page, dtype, layout, lens, **more):
    c = dict(op=op, mask=mask, seqs=seqs, rows_min=rows[0], rows_max=rows[1],
             context_min=context[0], context_max=context[1], q_heads=q_heads, kv_heads=kv_heads,
             dim=dim, page=page, dtype=dtype, layout=layout, lens=lens, **more)
    if name:
        c["name"] = name
    return c


def listed():
    plain = dict(pairs="half", scaling="none", factor=1.0)
    return [
        # one token of one conversation: the latency of a call
        _case("token_b1", "attend", "causal", 1, (1, 1), (299, 299), 32, 8, 128, 16, "bf16", "slots", 1),
        # the smallest block step: 32 + 32 rows behind a prompt of 32 tokens in a canvas of 288
        _case("block_b1_l32", "attend", "shadow", 1, (64, 64), (256, 256), 32, 32, 128, 16, "bf16", "slots", 2),
        # a block of 128 (the paper's block length) behind a prompt of about 1000 tokens
        _case("block_b1_l128", "attend", "shadow", 1, (256, 256), (1025, 1025), 32, 32, 128, 64, "bf16", "heads", 3),
        # the batched loop's step: 16 sequences of different lengths, grouped heads
        _case("block_b16_l32", "attend", "shadow", 16, (64, 64), (32, 2048), 32, 8, 128, 16, "bf16", "slots", 4),
        # four blocks of 256 over long multimodal contexts
        _case("block_b4_l256", "attend", "shadow", 4, (512, 512), (512, 4096), 32, 32, 128, 32, "bf16", "heads", 5),
        # a server's decode step: 64 conversations of ragged lengths
        _case("tokens_b64", "attend", "causal", 64, (1, 1), (500, 32767), 32, 8, 128, 16, "fp16", "heads", 6),
        # one very long context, one token
        _case("token_b1_long", "attend", "causal", 1, (1, 1), (262143, 262143), 32, 8, 128, 64, "bf16", "slots", 7),
        # whole prompts of ragged lengths
        _case("prompt_b4", "attend", "causal", 4, (1000, 8192), (0, 0), 32, 8, 128, 64, "bf16", "heads", 8),
        # chunks of new tokens behind long contexts, 7 query heads to a key head, heads of 64
        _case("chunk_b3_d64", "attend", "causal", 3, (200, 1000), (8000, 30000), 14, 2, 64, 32, "fp16", "slots", 9),
        # the smallest block step's rows
        _case("append_b1_l32", "append", "shadow", 1, (64, 64), (256, 256), 32, 32, 128, 16, "bf16", "slots", 10,
              rot=128, **plain),
        # four blocks of 256
        _case("append_b4_l256", "append", "shadow", 4, (512, 512), (512, 4096), 32, 32, 128, 32, "bf16", "heads", 11,
              rot=128, **plain),
        # prompts, half of each head rotated in neighbouring pairs, scaled for contexts beyond the trained one
        _case("append_prompts", "append", "causal", 5, (1000, 16000), (0, 60000), 32, 8, 128, 64, "fp16", "slots", 12,
              rot=64, pairs="interleaved", scaling="parts", factor=8.0),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.7e12, w["flops"] / 1.9e15)


def draw(rng):
    most = max(_cost(c) for c in listed())
    most_bytes = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["attend", "attend", "append"])
        kind = rng.choice(["token", "block", "chunk", "prompt"])
        dim = rng.choice([64, 64, 80, 96, 128, 128, 128])
        kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16, 32])
        q_heads = kv_heads * rng.choice([1, 1, 2, 4, 5, 7, 8])
        if q_heads > 64:
            continue
        if kind == "token":
            mask, seqs, rows = "causal", 1 + _spread(rng, 0, 127), (1, 1)
            lo = _spread(rng, 0, 32767)
            context = (lo, lo + _spread(rng, 0, 65536))
        elif kind == "block":
            mask, seqs = rng.choice(["shadow", "shadow", "full"]), 1 + _spread(rng, 0, 31)
            length = 2 * (1 + _spread(rng, 0, 255))
            lo = _spread(rng, 0, 2048)
            rows, context = (length, length), (lo + length, lo + length + _spread(rng, 0, 4096))
        elif kind == "chunk":
            mask, seqs = "causal", 1 + _spread(rng, 0, 7)
            most_rows = 1 + _spread(rng, 15, 2000)
            lo = _spread(rng, 0, 30000)
            rows, context = (1 + most_rows // 4, 1 + most_rows), (lo, lo + _spread(rng, 0, 8000))
        else:
            mask, seqs = "causal", 1 + _spread(rng, 0, 7)
            most_rows = 1 + _spread(rng, 63, 8191)
            rows, context = (1 + most_rows // 8, 1 + most_rows), (0, 0)
        case = _case(None, op, mask, seqs, rows, context, q_heads, kv_heads, dim, rng.choice([16, 32, 64, 128, 256]),
                     rng.choice(["bf16", "fp16"]), rng.choice(["slots", "heads"]), rng.randrange(1 << 30))
        if op == "append":
            rot = rng.choice([dim, dim, dim // 2, dim // 2 + 8 if dim >= 80 else dim // 4])
            scaling = rng.choice(["none", "linear", "parts"])
            case.update(rot=rot, pairs=rng.choice(["half", "interleaved"]), scaling=scaling,
                        factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 32.0]))
        if _cost(case) <= most and work(case)["bytes"] <= most_bytes and _cache_bytes(case) < 8e9:
            return case


# ------------------------------------------------------------------ sizes


def _lengths(case):
    """Per sequence (new rows, slots every new row may see, first new slot, slots the cache holds in the end)."""
    rng = random.Random(case["lens"])
    out = []
    for _ in range(case["seqs"]):
        n = 1 + _spread(rng, case["rows_min"] - 1, case["rows_max"] - 1)
        ctx = _spread(rng, case["context_min"], case["context_max"])
        if case["mask"] == "shadow":
            # the block lies in the last part of the canvas, which holds `ctx` slots; its shadow is stored behind
            half = n // 2
            out.append((n, ctx, max(0, ctx - 2 * half), ctx + half))
        elif case["mask"] == "full":
            out.append((n, max(ctx, n), max(0, ctx - n), max(ctx, n)))
        else:
            out.append((n, ctx + n, ctx, ctx + n))
    return out


def _visible_pairs(case):
    total = 0
    for n, kv, new, held in _lengths(case):
        if case["mask"] == "causal":
            total += n * new + n * (n + 1) // 2
        elif case["mask"] == "full":
            total += n * kv
        else:
            half = n // 2
            total += half * kv + half * (kv + half - 1)
    return total


def _cache_bytes(case):
    P = case["page"]
    pages = sum(-(-held // P) + 1 for _, _, _, held in _lengths(case))
    return pages * P * case["kv_heads"] * case["dim"] * 4


def work(case):
    rows = sum(n for n, *_ in _lengths(case))
    held = sum(h for *_, h in _lengths(case))
    q, kv, D = case["q_heads"], case["kv_heads"], case["dim"]
    if case["op"] == "append":
        return {"bytes": rows * (2 * q + 4 * kv) * D * 2 + rows * 4, "flops": rows * (q + kv) * case["rot"] * 3}
    return {"bytes": 2 * rows * q * D * 2 + 2 * held * kv * D * 2, "flops": 4 * D * q * _visible_pairs(case)}


# ------------------------------------------------------------------ inputs


def _frequencies(case):
    """Rotary angles per position, float64 [rot / 2], and the factor on the rotated values."""
    rot, factor = case["rot"], case["factor"]
    f = BASE ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "parts":
        # turns over the trained context decide: many keep their frequency, few are interpolated
        turns = TRAINED * f / (2 * np.pi)
        keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _inputs(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    lens = _lengths(case)
    q, kv, D, P = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    rows = sum(n for n, *_ in lens)
    need = [-(-held // P) for *_, held in lens]
    n_pages, width = sum(need) + 1, max(need) + 1
    perm = np.random.default_rng(seed).permutation(n_pages)  # pages come in any order; one stays unused
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = perm[at:at + n]
        at += n

    def cache(scale):
        shape = (n_pages, P, kv, D) if case["layout"] == "slots" else (n_pages, kv, P, D)
        t = torch.empty(shape, dtype=dtype, device=dev).normal_(0.0, scale, generator=g)
        return t if case["layout"] == "slots" else t.transpose(1, 2)

    st = dict(case=case, lens=lens, dtype=dtype, rows=rows, k_cache=cache(1.25), v_cache=cache(1.0),
              table=torch.from_numpy(table).to(dev))
    starts = np.cumsum([0] + [n for n, *_ in lens])[:-1]
    ints = np.array([starts, [x[0] for x in lens], [x[1] for x in lens], [x[2] for x in lens]], dtype=np.int32)
    st["ints"] = torch.from_numpy(ints).to(dev)  # q_start, q_len, kv_len, new_slot
    if case["op"] == "attend":
        st["q"] = torch.empty((rows, q, D), dtype=dtype, device=dev).normal_(0.0, 1.25, generator=g)
        return st
    # the projections' output, one fused row per token
    qkv = torch.empty((rows, q + 2 * kv, D), dtype=dtype, device=dev).normal_(0.0, 1.0, generator=g)
    st["q"], st["k"], st["v"] = qkv[:, :q], qkv[:, q:q + kv], qkv[:, q + kv:]
    slots, positions = [], []
    for n, kvl, new, _ in lens:
        i = np.arange(n)
        if case["mask"] == "shadow":
            half = n // 2
            slots.append(np.where(i < half, new + i, kvl + i - half))
            positions.append(new + i % half)
        else:
            slots.append(new + i)
            positions.append(new + i)
    st["slot"] = torch.from_numpy(np.concatenate(slots).astype(np.int64)).to(dev)
    st["seq"] = torch.from_numpy(np.repeat(np.arange(len(lens)), [x[0] for x in lens])).to(dev)
    st["positions"] = torch.from_numpy(np.concatenate(positions).astype(np.int32)).to(dev)
    f, st["scale"] = _frequencies(case)
    st["freq"] = torch.from_numpy(f).to(dev)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["out"] = torch.empty((st["rows"], case["q_heads"], case["dim"]), dtype=st["dtype"], device="cuda")
    if own:
        import paper_2605_16941_gb300 as wino
        q_start, q_len, kv_len, new_slot = st["ints"]
        st["batch"] = wino.make_kv_batch(st["k_cache"], st["v_cache"], st["table"], q_start, q_len, kv_len, new_slot,
                                         n_rows=st["rows"], n_q_heads=case["q_heads"], mask=MASKS[case["mask"]])
        if case["op"] == "attend":
            st["ws"] = wino.attend_workspace(st["batch"])
        else:
            st["ws"] = wino.append_workspace()
            freq, factor = wino.wino_rope_frequencies(case["rot"], BASE, scaling=case["scaling"],
                                                      factor=case["factor"], trained_len=TRAINED)
            st["rope"] = wino.make_rope(freq.cuda(), rot_dim=case["rot"], factor=factor,
                                        interleaved=case["pairs"] == "interleaved", positions=st["positions"])
    return st


# ------------------------------------------------------------------ one pass


def run(st):
    append = st["case"]["op"] == "append"
    if own:
        import paper_2605_16941_gb300 as wino
        if append:
            wino.wino_rope_append(st["q"], st["k"], st["v"], st["batch"], st["rope"], st["ws"], q_out=st["out"])
            return st["out"], st["k_cache"], st["v_cache"]
        wino.wino_attend(st["q"], st["out"], st["batch"], st["ws"])
        return st["out"]
    return _plain_append(st) if append else _plain_attend(st)


def _pairs(case):
    j = torch.arange(case["rot"] // 2, device="cuda")
    return (j, j + case["rot"] // 2) if case["pairs"] == "half" else (2 * j, 2 * j + 1)


def _plain_append(st):
    case = st["case"]
    angle = st["positions"].double()[:, None] * st["freq"]
    cos, sin = (angle.cos() * st["scale"]).float()[:, None], (angle.sin() * st["scale"]).float()[:, None]
    a, b = _pairs(case)

    def rotate(x):
        y = x.float()
        xa, xb = y[..., a], y[..., b]
        y[..., a] = xa * cos - xb * sin
        y[..., b] = xb * cos + xa * sin
        return y.to(st["dtype"])

    page = st["table"][st["seq"], st["slot"] // case["page"]].long()
    at = st["slot"] % case["page"]
    st["out"].copy_(rotate(st["q"]))
    st["k_cache"][page, at] = rotate(st["k"])
    st["v_cache"][page, at] = st["v"]
    return st["out"], st["k_cache"], st["v_cache"]


def _seen(case, n, kv, new, held, i, dev):
    """Whether new rows i see the slots 0 .. held - 1."""
    j = torch.arange(held, device=dev)[None, :]
    if case["mask"] == "causal":
        return j <= new + i[:, None]
    if case["mask"] == "full":
        return (j < kv).expand(len(i), held)
    half = n // 2
    shadow = (i >= half)[:, None]
    return torch.where(shadow, j != new + (i - half)[:, None], j < kv)


def _plain_attend(st):
    case = st["case"]
    q, kvh, D = case["q_heads"], case["kv_heads"], case["dim"]
    out = st["out"]
    row = 0
    for s, (n, kv, new, held) in enumerate(st["lens"]):
        pages = st["table"][s, :-(-held // case["page"])].long()
        k = st["k_cache"][pages].flatten(0, 1)[:held].float().permute(1, 2, 0)  # [heads, D, slots]
        v = st["v_cache"][pages].flatten(0, 1)[:held].float().transpose(0, 1)  # [heads, slots, D]
        step = max(1, (1 << 28) // (q * held))
        for i0 in range(0, n, step):
            i = torch.arange(i0, min(n, i0 + step), device="cuda")
            x = st["q"][row + i0:row + i0 + len(i)].float().view(len(i), kvh, -1, D).transpose(0, 1)
            score = torch.matmul(x.flatten(1, 2), k).view(kvh, len(i), -1, held) * D ** -0.5
            score.masked_fill_(~_seen(case, n, kv, new, held, i, "cuda")[None, :, None], -math.inf)
            score -= score.amax(-1, keepdim=True)
            p = score.exp_()
            z = p.sum(-1, keepdim=True)
            o = torch.matmul(p.flatten(1, 2), v).view(kvh, len(i), -1, D) / z
            out[row + i0:row + i0 + len(i)] = o.transpose(0, 1).reshape(len(i), q, D).to(out.dtype)
        row += n
    return out


# ------------------------------------------------------------------ the definition in 64 bits


def exact(case, seed):
    st = _inputs(case, seed)
    return _exact_append(case, st) if case["op"] == "append" else _exact_attend(case, st)


def _exact_append(case, st):
    f, factor = _frequencies(case)
    t = torch.outer(st["positions"].double(), torch.from_numpy(f).cuda())
    turn = torch.polar(torch.full_like(t, factor), t)[:, None, :]

    def rotated(x):
        x = x.double()
        head, rest = x[..., :case["rot"]], x[..., case["rot"]:]
        if case["pairs"] == "interleaved":
            z = torch.view_as_complex(head.unflatten(-1, (-1, 2)).contiguous()) * turn
            head = torch.view_as_real(z).flatten(-2)
        else:
            re, im = head.chunk(2, -1)
            z = torch.complex(re.contiguous(), im.contiguous()) * turn
            head = torch.cat([z.real, z.imag], -1)
        return torch.cat([head, rest], -1)

    k, v = st["k_cache"].double(), st["v_cache"].double()
    rk, rv = rotated(st["k"]), st["v"].double()
    table, row = st["table"].cpu().numpy(), 0
    slots = st["slot"].cpu().numpy()
    for s, (n, *_) in enumerate(st["lens"]):
        here = slots[row:row + n]
        page = torch.from_numpy(table[s, here // case["page"]].astype(np.int64)).cuda()
        at = torch.from_numpy(here % case["page"]).cuda()
        k.index_put_((page, at), rk[row:row + n])
        v.index_put_((page, at), rv[row:row + n])
        row += n
    return rotated(st["q"]), k, v


def _exact_attend(case, st):
    D, group = case["dim"], case["q_heads"] // case["kv_heads"]
    out = torch.zeros((st["rows"], case["q_heads"], D), dtype=torch.float64, device="cuda")
    row = 0
    for s, (n, kv, new, held) in enumerate(st["lens"]):
        slot = torch.arange(held, device="cuda")
        page, at = st["table"][s].long()[slot // case["page"]], slot % case["page"]
        for h in range(case["kv_heads"]):
            k, v = st["k_cache"][page, at, h].double(), st["v_cache"][page, at, h].double()
            for g in range(h * group, (h + 1) * group):
                for i0 in range(0, n, 2048):
                    i = torch.arange(i0, min(n, i0 + 2048), device="cuda")
                    logits = st["q"][row + i0:row + i0 + len(i), g].double() @ k.T / math.sqrt(D)
                    if case["mask"] == "causal":
                        hidden = slot[None] > (new + i)[:, None]
                    elif case["mask"] == "full":
                        hidden = (slot >= kv)[None].expand(len(i), held)
                    else:
                        block = (i < n // 2)[:, None]
                        hidden = (block & (slot >= kv)[None]) | (~block & (slot[None] == (new + i - n // 2)[:, None]))
                    logits = logits.masked_fill(hidden, -math.inf)
                    out[row + i0:row + i0 + len(i), g] = torch.softmax(logits, -1) @ v
        row += n
    return out
