"""The operators of a layer whose positions are rotations and whose attention is a window, as cases that can be timed and
compared.

* ``append``   new rows of Q, K and V, Q and K turned by their positions, K and V into a paged cache
  (``ds_kv_append_rotary``): one row of every sequence of a decoding batch, the rows of a prompt, or a piece of one,
* ``prefill``  causal attention of packed prompts through a sliding window that leaves the first tokens visible
  (``ds_prefill_attention_window``),
* ``decode``   one query of every sequence over what its window and its first tokens leave of a paged cache
  (``ds_decode_attention_window``).

Rotation: of a head's first ``rot`` features, a pair (a, b) at position p becomes (a cos - b sin, b cos + a sin) with the p-th
row of a table, ``rot / 2`` cosines and ``rot / 2`` sines; pair i is features (i, i + rot / 2), or (2 i, 2 i + 1) where they are
adjacent.  Products and sums are rounded to 32 bits one by one.  The row is then held as bf16, and in 8 bits by rounding that:
a row is the ``s`` numbers of one token and key/value head, a = max |x_d|; e4m3: scale c = 2^e with the least e >= -100 for which
a <= 448 c, values RNE(x_d / c); int8: c = the least bf16 that is >= a / 127 and >= 2^-100, values RNE(x_d / c).  a = 0: c = 1.
K pages are [num_blocks, n_kv, 16, s], V pages the same in bf16 and [num_blocks, n_kv, s, 16] in 8 bits, scales
[num_blocks, n_kv, 16].

Window: the query of token i sees token j <= i if i - j < window or j < sinks.  Layer shapes are those of the framework's
configurations and of its benchmark (the tiny layer, OPT-13B / 175B, 64 query heads on 8 key/value heads) and 32 query heads on
one key/value head.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
MODELS = {  # query heads, key/value heads, head size, FFN size
    "tiny": (4, 4, 64, 1024),
    "opt13b": (40, 40, 128, 20480),
    "opt175b": (96, 96, 128, 49152),
    "gqa64x8": (64, 8, 128, 32768),
    "mqa32x1": (32, 1, 128, 16384),
}
KV_TYPES = {"bf16": 0, "e4m3": 1, "int8": 2}


def listed():
    return [
        # the tiny layer's two rows: a call is its launch
        dict(name="append_tiny_bf16_b2", kind="append", model="tiny", type="bf16", batch=2, rows="one", spread="uniform", lo=33,
             hi=40, rot=64, adjacent=False, shifted=False, pick=1),
        # a decoding batch, cache of 8 bits; half of a head turned, positions that are not the cache's
        dict(name="append_gqa_e4m3_b64", kind="append", model="gqa64x8", type="e4m3", batch=64, rows="one", spread="lognormal",
             lo=16, hi=2048, rot=64, adjacent=True, shifted=True, pick=2),
        # a ragged batch of chatbot prompts into the bf16 cache, K also as the prefill's attention takes it
        dict(name="append_opt13b_bf16_chat", kind="append", model="opt13b", type="bf16", batch=12, rows="prompt",
             spread="lognormal", lo=16, hi=2048, rot=128, adjacent=False, shifted=False, pick=3),
        # the largest: pieces of eight long documents, behind what their pages hold already, into a cache of 8 bits
        dict(name="append_gqa_int8_pieces", kind="append", model="gqa64x8", type="int8", batch=8, rows="piece", spread="uniform",
             lo=2000, hi=2900, rot=128, adjacent=False, shifted=False, pick=4),
        # two tiny prompts
        dict(name="prefill_tiny_b2", kind="prefill", model="tiny", batch=2, spread="uniform", lo=19, hi=32, window=16, sinks=4,
             pick=1),
        # a ragged batch of chatbot prompts, a window shorter than most of them
        dict(name="prefill_opt13b_chat_w256", kind="prefill", model="opt13b", batch=12, spread="lognormal", lo=16, hi=2048,
             window=256, sinks=4, pick=3),
        # two documents, grouped-query attention, no sinks
        dict(name="prefill_gqa_2x8192_w1024", kind="prefill", model="gqa64x8", batch=2, spread="uniform", lo=8192, hi=8192,
             window=1024, sinks=0, pick=1),
        # the largest: one long document
        dict(name="prefill_gqa_1x16383_w2048", kind="prefill", model="gqa64x8", batch=1, spread="uniform", lo=16383, hi=16383,
             window=2048, sinks=64, pick=1),
        # two short sequences of the tiny layer: latency
        dict(name="decode_tiny_int8_b2", kind="decode", model="tiny", type="int8", batch=2, spread="uniform", lo=33, hi=40,
             window=16, sinks=4, pick=1),
        # a decoding batch of conversations on bf16 pages, the hidden tokens' pages given back
        dict(name="decode_opt13b_bf16_b64_w1024", kind="decode", model="opt13b", type="bf16", batch=64, spread="uniform",
             lo=1500, hi=6000, window=1024, sinks=4, pick=5),
        # the chatbot's batch: many contexts shorter than the window, pages of 8 bits
        dict(name="decode_gqa_e4m3_b128_w512", kind="decode", model="gqa64x8", type="e4m3", batch=128, spread="lognormal",
             lo=1, hi=4096, window=512, sinks=4, pick=6),
        # one long document: few heads, the window is all there is to split
        dict(name="decode_gqa_bf16_b1_w8192", kind="decode", model="gqa64x8", type="bf16", batch=1, spread="uniform", lo=65537,
             hi=65537, window=8192, sinks=16, pick=1),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(("append", "append", "prefill", "prefill", "decode", "decode"))
    model = rng.choice(("tiny", "opt13b", "opt13b", "opt175b", "gqa64x8", "gqa64x8", "mqa32x1"))
    n, n_kv, s, _ = MODELS[model]
    case = dict(kind=kind, model=model, pick=rng.randrange(1 << 20))
    ragged = rng.random() < 0.4
    if kind == "append":
        case.update(type=rng.choice(("bf16", "e4m3", "int8")), rows=rng.choice(("one", "prompt", "piece")),
                    rot=rng.choice((16, 32, s // 2, s, s)), adjacent=rng.random() < 0.5, shifted=rng.random() < 0.3)
        if case["rows"] == "one":  # of sequences from the first token to long ones
            hi = _log(rng, 1, 4096)
            return dict(case, batch=_log(rng, 1, 256), spread="uniform", lo=0 if hi < 16 else hi // 4, hi=hi)
        batch = _log(rng, 1, 16)
        mean = max(1, _log(rng, 16, min(12000, 80000000 // ((n + n_kv) * s))) // batch)
        if ragged:
            return dict(case, batch=min(batch, 8), spread="lognormal", lo=1, hi=2 * mean)
        return dict(case, batch=batch, spread="uniform", lo=max(1, mean // 2), hi=mean)
    case["sinks"] = rng.choice((0, 1, 4, 4, 16, 33, _log(rng, 1, 128)))
    if kind == "prefill":  # from one token to long prompts; pairs, and what the plain form holds of them, as in the largest
        batch = _log(rng, 1, 16)
        hi = max(1, _log(rng, 1, 16383) // batch)
        window = _log(rng, 1, 4096)
        while window > 1 and batch * hi * min(window, hi) * n > 16383 * 2048 * 64:
            window //= 2
        if ragged:
            return dict(case, batch=batch, spread="lognormal", lo=1, hi=hi, window=window)
        return dict(case, batch=batch, spread="uniform", lo=max(1, hi // 2), hi=hi, window=window)
    case["type"] = rng.choice(("bf16", "e4m3", "int8"))
    batch = _log(rng, 1, 160)
    window = _log(rng, 1, 8192)
    while window > 1 and batch * (window + case["sinks"]) * n_kv * s > 64 * 1028 * 5120:
        window //= 2
    if ragged:
        return dict(case, batch=batch, spread="lognormal", lo=1, hi=4096, window=window)
    hi = _log(rng, 1, 60000)
    return dict(case, batch=batch, spread="uniform", lo=max(1, hi // 2), hi=hi, window=window)


def _lengths(case):
    """Prompt lengths (prefill), tokens in all (decode), new rows (append; of one row: tokens before it)."""
    rng = np.random.default_rng(case["pick"])
    if case["spread"] == "lognormal":
        v = np.exp(rng.normal(math.log(384), 0.8, case["batch"]))
        return np.clip(np.rint(v), case["lo"], case["hi"]).astype(np.int64)
    return rng.integers(case["lo"], case["hi"] + 1, case["batch"])


def _new_rows(case):
    """Of an append: tokens before, new rows, and what the positions are ahead of the cache's, for each sequence."""
    rng, lens = np.random.default_rng(case["pick"] + 7), _lengths(case)
    ahead = rng.integers(0, 3000, len(lens)) if case["shifted"] else np.zeros_like(lens)
    if case["rows"] == "one":
        return lens, np.ones_like(lens), ahead
    return (rng.integers(0, 2 * lens.max() + 2, len(lens)) if case["rows"] == "piece" else np.zeros_like(lens)), lens, ahead


def _positions(case):
    before, new, ahead = _new_rows(case)
    return np.concatenate([np.arange(b, b + r) + a for b, r, a in zip(before, new, ahead)])


def _tables(rng, first_pages, last_pages, pages):
    """Page ids, in no order and with a few that nobody has, for the pages [0, first) and [last, pages) of each sequence; -1
    for the others."""
    j = np.arange(max(1, int(pages.max())))
    held = (j < pages[:, None]) & ((j < first_pages[:, None]) | (j >= last_pages[:, None]))
    ids = rng.permutation(int(held.sum()) + 3).astype(np.int32)
    table = np.full(held.shape, -1, np.int32)
    table[held] = ids[:int(held.sum())]
    return table, len(ids)


class State:
    pass


def prepare(case, seed):
    n, n_kv, s, _ = MODELS[case["model"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    ids = np.random.default_rng(int(seed))

    def normal(*size):
        return torch.empty(size, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=gen)

    def i32(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    def rows(count, heads):
        # what a projection gives: features of unlike size, some of them far larger than the others, and a mean each
        spread = torch.exp(0.3 * normal(heads, s)) * torch.where(normal(heads, s) > 2.2, 4.0, 1.0)
        return (normal(count, heads, s) * spread + 0.5 * normal(heads, s)).bfloat16()

    st = State()
    st.case, st.b, st.handle = case, case["batch"], None
    if case["kind"] == "prefill":
        lens = _lengths(case)
        st.t, st.longest = int(lens.sum()), int(lens.max())
        st.cu_np = np.concatenate([[0], np.cumsum(lens)])
        st.cu = i32(st.cu_np)
        # Q and K as the rotation leaves them, V in the rows of the QKV product
        st.q, st.k = (1.5 * normal(st.t, n, s)).bfloat16(), rows(st.t, n_kv)
        st.v, st.stride = rows(st.t, n + 2 * n_kv)[:, n + n_kv:], (n + 2 * n_kv) * s
        st.o = torch.empty_like(st.q)
        return st
    if case["kind"] == "append":
        before, new, _ = _new_rows(case)
        st.t = int(new.sum())
        pages = -(-(before + new) // PAGE)
        table, st.nblk = _tables(ids, pages, pages, pages)
        st.ctx_lens, st.ctx_np = i32(before), before
        st.cu_np = np.concatenate([[0], np.cumsum(new)])
        st.cu = None if case["rows"] == "one" else i32(st.cu_np)
        place = _positions(case)
        st.positions = i32(place) if case["shifted"] else None
        # the table of a model's cosines and sines, angles in 64 bits
        angle = torch.arange(int(place.max()) + 1, dtype=torch.float64, device="cuda")[:, None] * torch.exp(
            -math.log(10000.0) * torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])
        st.table = torch.cat([torch.cos(angle), torch.sin(angle)], 1).float()
        # the rows of a QKV product
        qkv = torch.cat([rows(st.t, n), rows(st.t, n_kv), rows(st.t, n_kv)], 1)
        st.q, st.k, st.v = qkv.split([n, n_kv, n_kv], 1)
        st.stride = (n + 2 * n_kv) * s
        st.q_out = torch.empty(st.t, n, s, dtype=torch.bfloat16, device="cuda")
        st.k_out = torch.empty(st.t, n_kv, s, dtype=torch.bfloat16, device="cuda") if case["rows"] == "prompt" else None
    else:
        st.lens = _lengths(case)
        st.longest = int(st.lens.max())
        shown = np.maximum(st.lens - case["window"], 0)  # the window's first token
        table, st.nblk = _tables(ids, np.full(st.b, -(-case["sinks"] // PAGE)), shown // PAGE, -(-st.lens // PAGE))
        st.kv_lens = i32(st.lens)
        st.q = (1.5 * normal(st.b, n, s)).bfloat16()
        st.o = torch.empty_like(st.q)
    st.tables = i32(table)
    # the cache, filled to the last slot (those behind a sequence's end, or hidden, among them)
    st.kc, st.vc = (rows(st.nblk * PAGE, n_kv).view(st.nblk, PAGE, n_kv, s).transpose(1, 2).contiguous() for _ in range(2))
    st.ks = st.vs = None
    if case["type"] != "bf16":
        (st.kc, st.ks), (st.vc, st.vs) = _quantise(st.kc, case["type"]), _quantise(st.vc, case["type"])
        st.vc = st.vc.transpose(2, 3).contiguous()
    return st


def _quantise(x, kind):
    """Rows of bf16 numbers along the last axis -> (8-bit values, scales).  In 32 bits: a power of two divides exactly; a
    quotient of two numbers of 8 significant bits is 2^-10 away from every border that it does not lie on."""
    x = x.float()
    a = x.abs().amax(-1)
    if kind == "e4m3":
        m, e = torch.frexp(a)  # a = m 2^e, 1/2 <= m < 1; 448 = 7/8 2^9
        c = torch.ldexp(torch.ones_like(a), (e - 9 + (m > 0.875).int()).clamp(min=-100))
    else:
        near = (a / 127.0).bfloat16()
        up = (near.view(torch.int16) + 1).view(torch.bfloat16)
        c = torch.where(near.double() * 127.0 < a.double(), up, near).float().clamp(min=2.0 ** -100)
    c = torch.where(a == 0, torch.ones_like(c), c)
    v = x / c[..., None]
    return v.to(torch.float8_e4m3fn) if kind == "e4m3" else torch.round(v).to(torch.int8), c.bfloat16()


def _turn(x, turns, adjacent):
    """Rows [t, heads, s] and their rows of the table [t, rot], in 32 bits; bf16."""
    rot = turns.shape[1]
    x, cos, sin = x.float(), turns[:, None, :rot // 2], turns[:, None, rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if adjacent else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(2) if adjacent else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1).bfloat16()


def _plain_append(st):
    row = torch.arange(st.t, device="cuda")
    if st.cu is None:
        seq, pos = row, st.ctx_lens.long()
    else:
        cu = st.cu.long()
        seq = torch.searchsorted(cu, row, right=True) - 1
        pos = st.ctx_lens.long()[seq] + row - cu[seq]
    turns = st.table[pos if st.positions is None else st.positions.long()]
    q, k = _turn(st.q, turns, st.case["adjacent"]), _turn(st.k, turns, st.case["adjacent"])
    page, slot = st.tables.long()[seq, pos // PAGE], pos % PAGE
    if st.case["type"] == "bf16":
        st.kc[page, :, slot], st.vc[page, :, slot] = k, st.v
    else:
        k8, st.ks[page, :, slot] = _quantise(k, st.case["type"])
        v8, st.vs[page, :, slot] = _quantise(st.v, st.case["type"])
        # (assignment by index in bytes: torch does it for few of the 8-bit types)
        st.kc.view(torch.uint8)[page, :, slot] = k8.view(torch.uint8)
        st.vc.view(torch.uint8)[page, :, :, slot] = v8.view(torch.uint8)
    return {"q": q, "k": None if st.k_out is None else k, "k_cache": st.kc, "v_cache": st.vc, "k_scale": st.ks,
            "v_scale": st.vs}


def _attend(q, k, v, seen):
    """[.., queries, s] over [.., keys, s] where seen [.., queries, keys]; 0 where nothing is."""
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(q.shape[-1])
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)


def _plain_prefill(st):
    """Pieces of up to `window` queries, each over its first tokens and the band of keys that its windows reach."""
    n, n_kv, s, _ = MODELS[st.case["model"]]
    w, sinks = min(st.case["window"], st.longest), min(st.case["sinks"], st.longest)
    piece = max(w, min(16, st.longest))
    start, end = st.cu.long()[:-1, None, None], st.cu.long()[1:, None, None]
    first = piece * torch.arange(-(-st.longest // piece), device="cuda")[:, None]              # [pieces, 1]
    qi = first + torch.arange(piece, device="cuda")                                           # [pieces, queries]
    band = first - w + 1 + torch.arange(w + piece - 1, device="cuda")
    ki = torch.cat([torch.arange(sinks, device="cuda").expand(len(first), -1), band], 1)      # [pieces, keys]
    near = torch.arange(ki.shape[1], device="cuda") >= sinks
    # a first token that the band has too counts there
    there = torch.where(near, ki >= 0, ki < (first - w + 1).clamp(min=0))
    gap = qi[:, :, None] - ki[:, None, :]
    seen = there[:, None, :] & (gap >= 0) & (~near | (gap < w) | (ki < sinks)[:, None, :])
    at_q = (start + qi).clamp(max=st.t - 1)                                                   # [B, pieces, queries]
    at_k = (start + ki.clamp(min=0)).clamp(max=st.t - 1)
    q = st.q.float()[at_q].unflatten(3, (n_kv, n // n_kv)).permute(0, 1, 3, 4, 2, 5).flatten(3, 4)
    k, v = (x.float()[at_k].transpose(2, 3) for x in (st.k, st.v))                            # [B, pieces, n_kv, keys, s]
    o = _attend(q, k, v, seen.repeat(1, n // n_kv, 1)[None, :, None])
    o = o.unflatten(3, (n // n_kv, piece)).permute(0, 1, 4, 2, 3, 5).flatten(3, 4)            # [B, pieces, queries, n, s]
    out = torch.empty(st.t + 1, n, s, dtype=torch.float32, device="cuda")
    out[torch.where(start + qi < end, start + qi, torch.full_like(at_q, st.t))] = o           # (behind a prompt: the last row)
    return {"o": out[:st.t].bfloat16()}


def _plain_decode(st):
    case = st.case
    n, n_kv, s, _ = MODELS[case["model"]]
    lens = st.kv_lens.long()[:, None]
    w, sinks = min(case["window"], st.longest), min(case["sinks"], st.longest)
    shown = (lens - w).clamp(min=0)
    j = torch.arange(sinks, device="cuda").expand(st.b, -1)
    at = torch.cat([j, shown + torch.arange(w, device="cuda")], 1)
    seen = torch.cat([j < shown.clamp(max=sinks), shown + torch.arange(w, device="cuda") < lens], 1)
    at = torch.where(seen, at, lens - 1)
    page, slot = st.tables.long().gather(1, at // PAGE), at % PAGE
    if st.ks is None:
        k, v = st.kc[page, :, slot].float(), st.vc[page, :, slot].float()                     # [rows, keys, n_kv, s]
    else:
        kb, vb = st.kc.view(torch.uint8)[page, :, slot], st.vc.view(torch.uint8)[page, :, :, slot]
        k = kb.view(st.kc.dtype).float() * st.ks[page, :, slot].float()[..., None]
        v = vb.view(st.vc.dtype).float() * st.vs[page, :, slot].float()[..., None]
    o = _attend(st.q.float().view(st.b, n_kv, n // n_kv, s), k.transpose(1, 2), v.transpose(1, 2), seen[:, None, None])
    return {"o": o.reshape(st.q.shape).bfloat16()}


def _handle(st):
    """The layer's context and the workspace, as a program keeps them for all its calls."""
    if st.handle is None:
        from paper_2401_09670_amd import binding
        n, n_kv, s, ffn = MODELS[st.case["model"]]
        ctx, room = binding.Context(n * s, n, s, ffn, PAGE, n_kv_heads=n_kv), 0
        if st.case["kind"] == "decode":
            room = ctx.ds_decode_window_workspace_bytes(st.b, st.longest, st.case["window"], st.case["sinks"])
        st.handle = ctx, torch.empty(max(256, room), dtype=torch.uint8, device="cuda")
    return st.handle


def run(st):
    case = st.case
    if not own:
        return {"append": _plain_append, "prefill": _plain_prefill, "decode": _plain_decode}[case["kind"]](st)
    ctx, ws = _handle(st)
    if case["kind"] == "prefill":
        n, n_kv, s, _ = MODELS[case["model"]]
        ctx.ds_prefill_attention_window(st.q, n * s, st.k, n_kv * s, st.v, st.stride, st.cu, st.b, st.t, st.longest,
                                        case["window"], case["sinks"], st.o)
        return {"o": st.o}
    cache = (st.kc, st.vc, st.ks, st.vs, st.nblk, KV_TYPES[case["type"]])
    if case["kind"] == "append":
        ctx.ds_kv_append_rotary(st.q, st.stride, st.k, st.v, st.stride, st.cu, st.b, st.t, st.ctx_lens, st.positions, st.table,
                                st.table.shape[0], case["rot"], case["adjacent"], st.tables, st.tables.shape[1], *cache,
                                st.q_out, st.k_out)
        return {"q": st.q_out, "k": st.k_out, "k_cache": st.kc, "v_cache": st.vc, "k_scale": st.ks, "v_scale": st.vs}
    ctx.ds_decode_attention_window(st.q, st.kv_lens, st.tables, st.b, st.tables.shape[1], st.longest, case["window"],
                                   case["sinks"], *cache, st.o, ws)
    return {"o": st.o}


def _seen_pairs(lens, w, sinks):
    """Pairs of a query and a token that it sees, over prompts of these lengths."""
    i = np.arange(int(lens.max()), dtype=np.int64)
    upto = np.cumsum(np.minimum(i + 1, w) + np.minimum(np.maximum(i + 1 - w, 0), sinks))
    return float(upto[lens - 1].sum())


def work(case):
    """Rows, queries and results once, K and V of every token that is seen once, in the bytes they are kept in; a multiplication
    and an addition are two operations."""
    n, n_kv, s, _ = MODELS[case["model"]]
    lens, wide, narrow = _lengths(case), n * s, n_kv * s
    if case["kind"] == "prefill":
        t = float(lens.sum())
        return {"bytes": t * (4.0 * wide + 4.0 * narrow), "flops": 4.0 * wide * _seen_pairs(lens, case["window"], case["sinks"])}
    kept = 4.0 * narrow if case["type"] == "bf16" else 2.0 * narrow + 4.0 * n_kv  # bytes of a token's K and V in the cache
    if case["kind"] == "append":
        place = _positions(case)
        t = float(len(place))
        out = 2.0 * wide + kept + (2.0 * narrow if case["rows"] == "prompt" else 0.0)
        return {"bytes": t * (2.0 * wide + 4.0 * narrow + out) + 4.0 * case["rot"] * len(np.unique(place)),
                "flops": 3.0 * t * (n + n_kv) * case["rot"]}
    seen = np.minimum(lens, case["window"])
    tokens = float((seen + np.minimum(lens - seen, case["sinks"])).sum())
    return {"bytes": 4.0 * len(lens) * wide + kept * tokens, "flops": 4.0 * wide * tokens}


def _values(x, kind):
    """A row's 8-bit values and scale, in 64 bits from the definition: the least power of two / the least bf16 that holds it,
    and the values nearest to the quotient: e4m3 has steps of 2^(e - 3) in [2^e, 2^(e + 1)) for e >= -6."""
    a = x.abs().amax(-1, keepdim=True)
    top = 448.0 if kind == "e4m3" else 127.0
    c = torch.exp2(torch.ceil(torch.log2(a.clamp(min=2.0 ** -140) / top)).clamp(min=-100.0))
    c = torch.where(c * top < a, 2 * c, c)
    c = torch.where((c / 2 * top >= a) & (c > 2.0 ** -100), c / 2, c)
    if kind == "int8":  # c / 2 < the least <= c: of the 128 bf16 numbers there, the first that holds it
        c = c / 2 + c / 256 * torch.ceil((a / top - c / 2) / (c / 256)).clamp(min=0.0)
        c = c.clamp(min=2.0 ** -100)
    c = torch.where(a == 0, torch.ones_like(c), c)
    v = x / c
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3) if kind == "e4m3" else torch.ones_like(v)
    return torch.round(v / step) * step, c[..., 0]


def _softmax_of(q, k, v, seen):
    """[queries, s] over [keys, s] in 64 bits."""
    z = torch.where(seen, q @ k.t() / math.sqrt(q.shape[-1]), -math.inf)
    return torch.softmax(z, -1) @ v


def exact(case, seed):
    st = prepare(case, seed)
    n, n_kv, s, _ = MODELS[case["model"]]
    if case["kind"] == "append":
        rot, place = case["rot"], torch.from_numpy(_positions(case)).cuda()
        cos, sin = (x.double() for x in st.table[place].split(rot // 2, 1))

        def turned(x):
            y = x.double()
            for i in range(rot // 2):
                a, b = (2 * i, 2 * i + 1) if case["adjacent"] else (i, i + rot // 2)
                c, d = cos[:, i:i + 1], sin[:, i:i + 1]
                y[:, :, a], y[:, :, b] = x[:, :, a].double() * c - x[:, :, b].double() * d, x[:, :, b].double() * c + x[:, :, a].double() * d
            return y

        out = {"q": turned(st.q), "k": turned(st.k), "k_cache": st.kc.double(), "v_cache": st.vc.double(), "k_scale": None,
               "v_scale": None}
        k, v = out["k"], st.v.double()
        if case["type"] != "bf16":
            # a row is held as bf16 before it is held in 8 bits: 8 significant bits
            m, e = torch.frexp(k)
            (k, ck), (v, cv) = _values(torch.ldexp(torch.round(m * 256), e - 8), case["type"]), _values(v, case["type"])
            out["k_scale"], out["v_scale"] = st.ks.double(), st.vs.double()
        for i in range(st.b):
            r0, r1, before = int(st.cu_np[i]), int(st.cu_np[i + 1]), int(st.ctx_np[i])
            for page in range(before // PAGE, -(-(before + r1 - r0) // PAGE)):
                lo, hi = max(before, PAGE * page), min(before + r1 - r0, PAGE * page + PAGE)
                here, to, slots = slice(r0 + lo - before, r0 + hi - before), int(st.tables[i, page]), slice(lo % PAGE, lo % PAGE + hi - lo)
                out["k_cache"][to, :, slots] = k[here].transpose(0, 1)
                if case["type"] == "bf16":
                    out["v_cache"][to, :, slots] = v[here].transpose(0, 1)
                else:
                    out["v_cache"][to, :, :, slots] = v[here].permute(1, 2, 0)
                    out["k_scale"][to, :, slots], out["v_scale"][to, :, slots] = ck[here].t(), cv[here].t()
        if case["type"] == "int8":
            out["k_cache"] = out["v_cache"] = None
        if case["rows"] != "prompt":
            out["k"] = None
        return out
    w, sinks = case["window"], case["sinks"]
    o = torch.zeros(st.q.shape, dtype=torch.float64, device="cuda")
    if case["kind"] == "prefill":
        for i in range(st.b):
            here = slice(int(st.cu_np[i]), int(st.cu_np[i + 1]))
            at = torch.arange(here.stop - here.start, device="cuda")
            seen = (at[:, None] >= at) & ((at[:, None] - at < w) | (at < sinks))
            for head in range(n):
                kv = head // (n // n_kv)
                o[here, head] = _softmax_of(st.q[here, head].double(), st.k[here, kv].double(), st.v[here, kv].double(), seen)
        return {"o": o}
    for i, length in enumerate(int(x) for x in st.lens):
        at = [j for j in range(min(sinks, length - min(w, length)))] + list(range(length - min(w, length), length))
        at = torch.tensor(at, device="cuda")
        page, slot = st.tables[i].long()[at // PAGE], at % PAGE
        for kv in range(n_kv):
            k = st.kc[page, kv, slot].double()
            v = st.vc[page, kv, slot].double() if st.ks is None else st.vc.view(torch.uint8)[page, kv, :, slot].view(st.vc.dtype).double()
            if st.ks is not None:
                k = st.kc.view(torch.uint8)[page, kv, slot].view(st.kc.dtype).double() * st.ks[page, kv, slot].double()[:, None]
                v = v * st.vs[page, kv, slot].double()[:, None]
            heads = slice(kv * (n // n_kv), (kv + 1) * (n // n_kv))
            o[i, heads] = _softmax_of(st.q[i, heads].double(), k, v, torch.ones((), dtype=torch.bool, device="cuda"))
    return {"o": o}
