"""The operators around a paged key/value cache of 8 bits, and attention over a prefix that a batch shares, as cases that
can be timed and compared.

* ``handoff``  prompts' K and V rows quantised into pages (``ds_kv_migrate_quant``) and read back from them
  (``ds_kv_read_quant``),
* ``decode``   one token's rows of every sequence appended (``ds_kv_append_quant``), then its query's attention over the
  pages (``ds_decode_attention_quant``),
* ``shared``   one query of every sequence over a prefix that its group of sequences shares and over tokens of its own
  (``ds_decode_attention_shared``), on bf16 pages or on those of 8 bits.

A row is the ``s`` numbers of one token and key/value head; a = max |x_d| over it.  It is kept as 8-bit values and a scale c:
e4m3: c = 2^e with the least e >= -100 for which a <= 448 c, values RNE(x_d / c); int8: c = the least bf16 that is
>= a / 127 and >= 2^-100, values RNE(x_d / c).  a = 0: c = 1.  K pages are [num_blocks, n_kv, 16, s], V pages
[num_blocks, n_kv, s, 16], scales [num_blocks, n_kv, 16].  Layer shapes are those of the framework's configurations and of
its benchmark (the tiny layer, OPT-13B / 175B, 64 query heads on 8 key/value heads).
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
}
KV_TYPES = {"bf16": 0, "e4m3": 1, "int8": 2}


def listed():
    return [
        # the tiny layer's two prompts: a call is its launches
        dict(name="handoff_tiny_e4m3", kind="handoff", model="tiny", type="e4m3", batch=2, spread="uniform", lo=19, hi=32,
             pick=1),
        # a ragged batch of chatbot prompts, up to the prefill token cap
        dict(name="handoff_opt13b_int8_chat", kind="handoff", model="opt13b", type="int8", batch=12, spread="lognormal",
             lo=16, hi=2048, pick=3),
        # the largest: a pipeline stage's eight long prompts of OPT-175B
        dict(name="handoff_opt175b_e4m3_8x2048", kind="handoff", model="opt175b", type="e4m3", batch=8, spread="uniform",
             lo=2048, hi=2048, pick=1),
        # two short sequences of the tiny layer: latency
        dict(name="decode_tiny_int8_b2", kind="decode", model="tiny", type="int8", batch=2, spread="uniform", lo=33, hi=40,
             pick=1),
        # a single conversation
        dict(name="decode_opt13b_e4m3_b1", kind="decode", model="opt13b", type="e4m3", batch=1, spread="uniform", lo=700,
             hi=700, pick=1),
        # the benchmark's decode batch in the middle of its steps
        dict(name="decode_opt13b_e4m3_b64", kind="decode", model="opt13b", type="e4m3", batch=64, spread="uniform", lo=544,
             hi=544, pick=1),
        # the chatbot stack's decode batch: contexts as ragged as the requests
        dict(name="decode_opt13b_int8_b128_chat", kind="decode", model="opt13b", type="int8", batch=128,
             spread="lognormal", lo=16, hi=2048, pick=5),
        # grouped-query attention at long contexts
        dict(name="decode_gqa_e4m3_b48", kind="decode", model="gqa64x8", type="e4m3", batch=48, spread="uniform", lo=1024,
             hi=4096, pick=9),
        # one long document: few heads, the token axis is all there is to split
        dict(name="decode_gqa_int8_b1_long", kind="decode", model="gqa64x8", type="int8", batch=1, spread="uniform",
             lo=65537, hi=65537, pick=1),
        # five continuations of a tiny prompt whose last page is not full
        dict(name="shared_tiny_int8", kind="shared", model="tiny", type="int8", batch=5, groups=1, plo=45, phi=45,
             spread="uniform", lo=0, hi=20, pick=2),
        # a batch of conversations behind one system prompt, on the framework's bf16 pages
        dict(name="shared_opt13b_bf16_b64", kind="shared", model="opt13b", type="bf16", batch=64, groups=1, plo=2048,
             phi=2048, spread="uniform", lo=16, hi=256, pick=3),
        # questions about three long documents, grouped-query attention
        dict(name="shared_gqa_e4m3_b48", kind="shared", model="gqa64x8", type="e4m3", batch=48, groups=3, plo=4000,
             phi=9001, spread="uniform", lo=1, hi=300, pick=4),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(("handoff", "decode", "decode", "shared", "shared"))
    pick = rng.randrange(1 << 20)
    model = rng.choice(("tiny", "opt13b", "opt13b", "opt175b", "gqa64x8", "gqa64x8"))
    kv = rng.choice(("e4m3", "int8"))
    ragged = rng.random() < 0.4
    if kind == "handoff":  # from one short prompt to a full prefill batch
        batch = _log(rng, 1, 16)
        mean = max(1, _log(rng, 16, 4096) // batch)
        if ragged:
            return dict(kind=kind, model=model, type=kv, batch=batch, spread="lognormal", lo=1, hi=2048, pick=pick)
        return dict(kind=kind, model=model, type=kv, batch=batch, spread="uniform", lo=max(1, mean // 2),
                    hi=mean + mean // 2, pick=pick)
    if kind == "decode":  # from one sequence of one token to wide batches and long contexts
        batch = _log(rng, 1, 128)
        if ragged:
            return dict(kind=kind, model=model, type=kv, batch=batch, spread="lognormal", lo=1, hi=2048, pick=pick)
        hi = _log(rng, 1, max(64, 120000 // batch if model in ("tiny", "gqa64x8") else 40000 // batch))
        return dict(kind=kind, model=model, type=kv, batch=batch, spread="uniform", lo=max(1, hi // 2), hi=hi, pick=pick)
    batch = _log(rng, 2, 128)
    phi = _log(rng, 32, 12000 if model in ("tiny", "gqa64x8") else 4096)
    own_hi = _log(rng, 1, 300)
    return dict(kind=kind, model=model, type=rng.choice(("bf16", "e4m3", "int8")), batch=batch,
                groups=rng.randint(1, min(4, batch)), plo=max(1, phi // rng.choice((1, 2, 3))), phi=phi, spread="uniform",
                lo=own_hi // 4, hi=own_hi, pick=pick)


def _lengths(case):
    """Prompt lengths (handoff), tokens before the step (decode), tokens of a sequence's own (shared)."""
    rng = np.random.default_rng(case["pick"])
    if case["spread"] == "lognormal":
        v = np.exp(rng.normal(math.log(256 if case["kind"] == "handoff" else 384), 0.8, case["batch"]))
        return np.clip(np.rint(v), case["lo"], case["hi"]).astype(np.int64)
    return rng.integers(case["lo"], case["hi"] + 1, case["batch"])


def _groups(case):
    """First rows of the groups, batch behind them, and the groups' prefix lengths."""
    rng = np.random.default_rng(case["pick"] + 7)
    cuts = np.sort(rng.choice(np.arange(1, case["batch"]), case["groups"] - 1, replace=False))
    return np.concatenate([[0], cuts, [case["batch"]]]), rng.integers(case["plo"], case["phi"] + 1, case["groups"])


def _tables(rng, capacities):
    """Pages of sequences of these lengths, in no order and with a few ids that nobody has; -1 where none is needed."""
    need = -(-np.asarray(capacities) // PAGE)
    ids = rng.permutation(int(need.sum()) + 3).astype(np.int32)
    table = np.full((len(need), max(1, int(need.max()))), -1, np.int32)
    table[np.arange(table.shape[1]) < need[:, None]] = ids[:int(need.sum())]
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

    def rows(*size):
        # what a projection gives: features of unlike size, some of them far larger than the others, and a mean each
        spread = torch.exp(0.3 * normal(n_kv, s)) * torch.where(normal(n_kv, s) > 2.2, 4.0, 1.0)
        return normal(*size, n_kv, s) * spread + 0.5 * normal(n_kv, s)

    st = State()
    st.case, st.lens, st.handle = case, _lengths(case), None
    b = st.b = case["batch"]
    st.longest = int(st.lens.max())
    if case["kind"] == "handoff":
        st.t = int(st.lens.sum())
        table, st.nblk = _tables(ids, st.lens)
        st.cu = i32(np.concatenate([[0], np.cumsum(st.lens)]))
        st.k, st.v = rows(st.t).bfloat16(), rows(st.t).bfloat16()
        st.k_back, st.v_back = torch.empty_like(st.k), torch.empty_like(st.v)
    elif case["kind"] == "decode":
        table, st.nblk = _tables(ids, st.lens + 1)
        st.ctx_lens, st.kv_lens = i32(st.lens), i32(st.lens + 1)
        st.k_new, st.v_new = rows(b).bfloat16(), rows(b).bfloat16()
    else:
        st.cu_np, st.prefix_np = _groups(case)
        table, st.nblk = _tables(ids, np.concatenate([st.prefix_np, st.lens]))
        st.cu, st.prefix_lens, st.kv_lens = i32(st.cu_np), i32(st.prefix_np), i32(st.lens)
        st.prefix_tables, table = i32(table[:case["groups"]]), table[case["groups"]:]
        st.group_rows, st.longest_prefix = int(np.diff(st.cu_np).max()), int(st.prefix_np.max())
    st.tables = i32(table)
    if case["kind"] != "handoff":
        st.q = (1.5 * normal(b, n, s)).bfloat16()
        st.o = torch.empty_like(st.q)
    # the cache: zeros before the hand-off, else filled to the last slot (those behind a sequence's end among them)
    if case["type"] == "bf16":
        st.kc, st.vc = rows(st.nblk, PAGE).bfloat16(), rows(st.nblk, PAGE).bfloat16()
        st.kc, st.vc = st.kc.transpose(1, 2).contiguous(), st.vc.transpose(1, 2).contiguous()
        st.ks = st.vs = None
    elif case["kind"] == "handoff":
        kind = torch.float8_e4m3fn if case["type"] == "e4m3" else torch.int8
        st.kc = torch.zeros(st.nblk, n_kv, PAGE, s, dtype=torch.uint8, device="cuda").view(kind)
        st.vc = torch.zeros(st.nblk, n_kv, s, PAGE, dtype=torch.uint8, device="cuda").view(kind)
        st.ks = torch.zeros(st.nblk, n_kv, PAGE, dtype=torch.bfloat16, device="cuda")
        st.vs = torch.zeros_like(st.ks)
    else:
        st.kc, st.ks = _quantise(rows(st.nblk, PAGE).bfloat16().transpose(1, 2), case["type"])
        st.vc, st.vs = _quantise(rows(st.nblk, PAGE).bfloat16().transpose(1, 2), case["type"])
        st.kc = st.kc.contiguous()
        st.vc = st.vc.transpose(2, 3).contiguous()
    return st


def _quantise(x, kind):
    """Rows along the last axis -> (8-bit values, scales).  In 32 bits: a power of two divides exactly; a quotient of two
    numbers of 8 significant bits is 2^-10 away from every border that it does not lie on."""
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


def _softmax(scores, seen):
    """Along the last axis over what is seen; rows that see nothing are zero."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total)


def _pages(st, tables):
    """K and V of the pages that these tables name, [rows, n_kv, tokens, s] in 32 bits."""
    at = tables.long().clamp(min=0)
    k, v = st.kc[at].float(), st.vc[at].float()           # [rows, pages, n_kv, 16, s] and, of 8 bits, [.., s, 16]
    if st.ks is not None:
        k, v = k * st.ks[at].float()[..., None], v.transpose(3, 4) * st.vs[at].float()[..., None]
    return k.transpose(1, 2).flatten(2, 3), v.transpose(1, 2).flatten(2, 3)


def _scores(q, k):
    """[rows, n_kv, G, s] with [rows, n_kv, tokens, s]"""
    return torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(q.shape[-1])


def _plain_handoff(st):
    cu, pos = st.cu.long(), torch.arange(st.t, device="cuda")
    seq = torch.searchsorted(cu, pos, right=True) - 1
    pos = pos - cu[seq]
    page, slot = st.tables.long()[seq, pos // PAGE], pos % PAGE
    for_k, st.ks[page, :, slot] = _quantise(st.k, st.case["type"])
    for_v, st.vs[page, :, slot] = _quantise(st.v, st.case["type"])
    # (assignment by index, and what is read by it, in bytes: torch does either for few of the 8-bit types)
    kb, vb = st.kc.view(torch.uint8), st.vc.view(torch.uint8)
    kb[page, :, slot] = for_k.view(torch.uint8)
    vb[page, :, :, slot] = for_v.view(torch.uint8)
    k, v = kb[page, :, slot].view(st.kc.dtype), vb[page, :, :, slot].view(st.vc.dtype)
    return {"k": (k.float() * st.ks[page, :, slot].float()[..., None]).bfloat16(),
            "v": (v.float() * st.vs[page, :, slot].float()[..., None]).bfloat16(), "k_scale": st.ks, "v_scale": st.vs}


def _plain_decode(st):
    pos, row = st.ctx_lens.long(), torch.arange(st.b, device="cuda")
    page, slot = st.tables.long()[row, pos // PAGE], pos % PAGE
    k_new, st.ks[page, :, slot] = _quantise(st.k_new, st.case["type"])
    v_new, st.vs[page, :, slot] = _quantise(st.v_new, st.case["type"])
    st.kc.view(torch.uint8)[page, :, slot] = k_new.view(torch.uint8)
    st.vc.view(torch.uint8)[page, :, :, slot] = v_new.view(torch.uint8)
    k, v = _pages(st, st.tables)
    seen = torch.arange(k.shape[2], device="cuda") < st.kv_lens.long()[:, None]
    q = st.q.float().view(st.b, k.shape[1], -1, k.shape[3])
    o = torch.matmul(_softmax(_scores(q, k), seen[:, None, None]), v)
    return {"o": o.view_as(st.q).bfloat16(), "k_cache": st.kc, "v_cache": st.vc, "k_scale": st.ks, "v_scale": st.vs}


def _plain_shared(st):
    row = torch.arange(st.b, device="cuda")
    group = torch.searchsorted(st.cu.long(), row, right=True) - 1
    (kp, vp), (k, v) = _pages(st, st.prefix_tables), _pages(st, st.tables)
    groups, n_kv, far, s = kp.shape
    q = st.q.float().view(st.b, n_kv, -1, s)
    # every query against every group's prefix in one product, and of the result the row's own group
    every = _scores(q.transpose(0, 1).flatten(1, 2)[None], kp).view(groups, n_kv, st.b, -1, far)
    sp = every[group, :, row]                                                    # [rows, n_kv, G, far]
    seen_p = (torch.arange(far, device="cuda") < st.prefix_lens.long()[:, None])[group]
    seen = torch.arange(k.shape[2], device="cuda") < st.kv_lens.long()[:, None]
    p = _softmax(torch.cat([sp, _scores(q, k)], -1), torch.cat([seen_p, seen], -1)[:, None, None])
    mine = torch.nn.functional.one_hot(group, groups).float().t()[:, :, None, None, None]
    spread = (mine * p[None, ..., :far]).transpose(1, 2).flatten(2, 3)           # [groups, n_kv, rows G, far]
    o = torch.matmul(spread, vp).sum(0).view(n_kv, st.b, -1, s).transpose(0, 1) + torch.matmul(p[..., far:], v)
    return {"o": o.reshape(st.q.shape).bfloat16()}


def _handle(st):
    """The layer's context and the workspace, as a program keeps them for all its calls."""
    if st.handle is None:
        from paper_2401_09670_amd import binding
        n, n_kv, s, ffn = MODELS[st.case["model"]]
        ctx = binding.Context(n * s, n, s, ffn, PAGE, n_kv_heads=n_kv)
        room = 0
        if st.case["kind"] == "decode":
            room = ctx.ds_decode_quant_workspace_bytes(st.b, st.longest + 1)
        elif st.case["kind"] == "shared":
            room = ctx.ds_decode_shared_workspace_bytes(st.b, st.longest_prefix, max(1, st.longest))
        st.handle = ctx, torch.empty(max(256, room), dtype=torch.uint8, device="cuda")
    return st.handle


def run(st):
    case = st.case
    if not own:
        return {"handoff": _plain_handoff, "decode": _plain_decode, "shared": _plain_shared}[case["kind"]](st)
    ctx, ws = _handle(st)
    kind = KV_TYPES[case["type"]]
    cache = (st.kc, st.vc, st.ks, st.vs, st.nblk, kind)
    if case["kind"] == "handoff":
        ctx.ds_kv_migrate_quant(st.k, st.v, st.cu, st.b, st.t, st.longest, st.tables, st.tables.shape[1], *cache)
        ctx.ds_kv_read_quant(st.cu, st.b, st.t, st.longest, st.tables, st.tables.shape[1], *cache, st.k_back, st.v_back)
        return {"k": st.k_back, "v": st.v_back, "k_scale": st.ks, "v_scale": st.vs}
    if case["kind"] == "decode":
        ctx.ds_kv_append_quant(st.k_new, st.v_new, st.k_new[0].numel(), st.ctx_lens, st.tables, st.b, st.tables.shape[1],
                               *cache)
        ctx.ds_decode_attention_quant(st.q, st.kv_lens, st.tables, st.b, st.tables.shape[1], st.longest + 1, *cache, st.o,
                                      ws)
        return {"o": st.o, "k_cache": st.kc, "v_cache": st.vc, "k_scale": st.ks, "v_scale": st.vs}
    ctx.ds_decode_attention_shared(st.q, st.cu, case["groups"], st.group_rows, st.prefix_lens, st.prefix_tables,
                                   st.prefix_tables.shape[1], st.longest_prefix, st.kv_lens, st.tables, st.b,
                                   st.tables.shape[1], max(1, st.longest), *cache, st.o, ws)
    return {"o": st.o}


def work(case):
    """K and V of every token once, in the bytes they are kept in (a prefix once for its group), rows, queries and results
    once; a multiplication and an addition are two operations."""
    n, n_kv, s, _ = MODELS[case["model"]]
    lens, b, w = _lengths(case), case["batch"], n_kv * s
    kept = 4.0 * w if case["type"] == "bf16" else 2.0 * w + 4.0 * n_kv  # bytes of a token's K and V in the cache
    if case["kind"] == "handoff":
        t = float(lens.sum())
        return {"bytes": 2 * t * (4.0 * w + kept), "flops": 4.0 * t * w}
    ends = 4.0 * b * n * s  # queries and results
    if case["kind"] == "decode":
        tokens = float((lens + 1).sum())
        return {"bytes": ends + b * (4.0 * w + kept) + kept * tokens, "flops": 4.0 * n * s * tokens}
    cu, prefix = _groups(case)
    tokens = float(lens.sum())
    return {"bytes": ends + kept * (tokens + float(prefix.sum())),
            "flops": 4.0 * n * s * (tokens + float((np.diff(cu) * prefix).sum()))}


def _rounded(x, c, kind):
    """The 8-bit values nearest to x / c, in 64 bits: steps of 2^(e - 3) in [2^e, 2^(e + 1)) for e >= -6, or of 1."""
    v = x / c
    step = torch.ones_like(v)
    if kind == "e4m3":
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def _values(x, kind):
    """A row's 8-bit values and scale, from the definition: the least power of two / the least bf16 that holds it."""
    x = x.double()
    a = x.abs().amax(-1, keepdim=True)
    top = 448.0 if kind == "e4m3" else 127.0
    c = torch.exp2(torch.ceil(torch.log2(a.clamp(min=2.0 ** -140) / top)).clamp(min=-100.0))
    c = torch.where(c * top < a, 2 * c, c)
    c = torch.where((c / 2 * top >= a) & (c > 2.0 ** -100), c / 2, c)
    if kind == "int8":  # c / 2 < the least <= c: of the 128 bf16 numbers there, the first that holds it
        c = c / 2 + c / 256 * torch.ceil((a / top - c / 2) / (c / 256)).clamp(min=0.0)
        c = c.clamp(min=2.0 ** -100)
    c = torch.where(a == 0, torch.ones_like(c), c)
    return _rounded(x, c, kind), c[..., 0]


def _attend(q, k, v):
    """[n, s] over [tokens, n_kv, s] in 64 bits."""
    if k.shape[0] == 0:
        return torch.zeros_like(q)
    g = q.shape[0] // k.shape[1]
    q = q.view(k.shape[1], g, -1)
    s = torch.bmm(q, k.permute(1, 2, 0).contiguous()) / math.sqrt(q.shape[-1])
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.bmm(p, v.transpose(0, 1).contiguous()) / p.sum(-1, keepdim=True)
    return o.reshape(-1, q.shape[-1])


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "handoff":
        out = {}
        for name, x, scales in (("k", st.k, st.ks), ("v", st.v, st.vs)):
            values, c = _values(x, case["type"])
            out[name], out[name + "_scale"] = values * c[..., None], scales.double()
            first = 0
            for i, length in enumerate(st.lens):
                for j in range(0, int(length), PAGE):
                    here = c[first + j:first + min(int(length), j + PAGE)]
                    out[name + "_scale"][int(st.tables[i, j // PAGE]), :, :here.shape[0]] = here.t()
                first += int(length)
        return out

    def tokens(table, length):
        at = table[:-(-length // PAGE)].long()
        k, v = st.kc[at].double(), st.vc[at].double()
        if st.ks is not None:
            k, v = k * st.ks[at].double()[..., None], v.transpose(2, 3) * st.vs[at].double()[..., None]
        return [x.transpose(1, 2).flatten(0, 1)[:length] for x in (k, v)]

    o = torch.empty(st.q.shape, dtype=torch.float64, device="cuda")
    if case["kind"] == "decode":
        (kq, kc), (vq, vc) = _values(st.k_new, case["type"]), _values(st.v_new, case["type"])
        out = {"o": o, "k_scale": st.ks.double(), "v_scale": st.vs.double(), "k_cache": None, "v_cache": None}
        if case["type"] == "e4m3":
            out["k_cache"], out["v_cache"] = st.kc.double(), st.vc.double()
        for i, length in enumerate(st.lens):
            length = int(length)
            page, slot = int(st.tables[i, length // PAGE]), length % PAGE
            out["k_scale"][page, :, slot], out["v_scale"][page, :, slot] = kc[i], vc[i]
            if case["type"] == "e4m3":
                out["k_cache"][page, :, slot], out["v_cache"][page, :, :, slot] = kq[i], vq[i]
            k, v = tokens(st.tables[i], length)
            k = torch.cat([k, (kq[i] * kc[i][:, None])[None]])
            v = torch.cat([v, (vq[i] * vc[i][:, None])[None]])
            o[i] = _attend(st.q[i].double(), k, v)
        return out
    for g, length in enumerate(st.prefix_np):
        kp, vp = tokens(st.prefix_tables[g], int(length))
        for i in range(int(st.cu_np[g]), int(st.cu_np[g + 1])):
            k, v = tokens(st.tables[i], int(st.lens[i]))
            o[i] = _attend(st.q[i].double(), torch.cat([kp, k]), torch.cat([vp, v]))
    return {"o": o}
