"""Operator cases of a serving step over a cache of 8 bits: the language backbone's operators beside ``operators.py``.

The cache holds e4m3 codes with one power-of-two scale (fp32) for each block of tokens and head.  A step attends
over it, finds out which of its drafted tokens are right, and writes their keys and values:

- ``attention``: the new tokens of each request (16 bits) over its cached ones (8 bits) and over each other;
- ``verify``: drafted tokens, chains or trees, against the target's probabilities from given random numbers;
- ``quantise``: keys and values of all layers into their slots, blocks that gain tokens keeping what they had;
- ``dequantise``: cached tokens of all layers back as 16-bit rows.

Sizes: 256 or 1024 tokens a view and 27 layers as in ``synth.WORKLOADS``, heads of 64 and 72 as in its encoders, else
generic ones (64, 96, 128 and 256 wide, 1 to 16 query heads to a key head, vocabularies of 1000 to 131072).
"""
import math

import numpy as np
import torch

own = False

ATTN = dict(op="attention")
VIEW_HEADS = dict(heads=16, kv_heads=16, head_dim=72)


def listed():
    return [
        # the accepted token of eight robots: the smallest write
        dict(name="quantise_token", op="quantise", requests=8, new=1, length=700, layers=27, kv_heads=4, head_dim=64, page=16,
             block=16, type="bfloat16"),
        # the accepted drafts of a large batch, most into blocks that are partly filled
        dict(name="quantise_drafts", op="quantise", requests=256, new=6, length=2000, layers=32, kv_heads=8, head_dim=128,
             page=32, block=16, type="float16"),
        # prompts: eight views of 1024 tokens
        dict(name="quantise_views", op="quantise", requests=8, new=1024, length=1500, layers=27, kv_heads=16, head_dim=72,
             page=32, block=32, type="bfloat16"),
        # one robot's few tokens, back for a comparison with their 16-bit form
        dict(name="dequantise_few", op="dequantise", rows=37, layers=27, kv_heads=4, head_dim=64, page=16, block=16,
             type="bfloat16"),
        # a shared prompt goes back to a 16-bit cache
        dict(name="dequantise_many", op="dequantise", rows=4099, layers=32, kv_heads=8, head_dim=128, page=64, block=8,
             type="float16"),
        # one robot decoding after three views and an instruction: latency
        dict(name="attention_one", **ATTN, requests=1, new=1, length=1041, heads=16, kv_heads=4, head_dim=64, page=16, block=16,
             type="bfloat16", mask="causal", order="token"),
        # a serving batch decoding over long, ragged contexts: the cache's bytes
        dict(name="attention_decode", **ATTN, requests=32, new=1, length=16384, heads=32, kv_heads=8, head_dim=128, page=16,
             block=16, type="bfloat16", mask="causal", order="token"),
        # trees of up to 31 drafts being verified
        dict(name="attention_trees", **ATTN, requests=16, new=31, length=8192, heads=32, kv_heads=8, head_dim=128, page=64,
             block=32, type="float16", mask="tree", order="head"),
        # a new view's 256 tokens, each seeing all of them and the frames before
        dict(name="attention_views", **ATTN, requests=8, new=256, length=2048, **VIEW_HEADS, page=32, block=8, type="bfloat16",
             mask="all", order="token"),
        # one robot, a run of four drafts from a drafter without probabilities
        dict(name="verify_one", op="verify", requests=1, new=5, vocab=32768, tree=False, probs=False, greedy=False,
             type="bfloat16"),
        # a serving batch of trees whose drafts were drawn from the drafter's probabilities
        dict(name="verify_trees", op="verify", requests=64, new=16, vocab=131072, tree=True, probs=True, greedy=False,
             type="bfloat16"),
        # a large batch, the likeliest token of each row, an odd vocabulary in 32 bits
        dict(name="verify_greedy", op="verify", requests=500, new=4, vocab=50001, tree=False, probs=False, greedy=True,
             type="float32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantise", "quantise", "dequantise", "attention", "attention", "attention", "verify", "verify"])
    if op == "verify":
        while True:
            tree = rng.random() < 0.5
            case = dict(op=op, requests=_log(rng, 1, 512), new=_log(rng, 1, 32), vocab=_log(rng, 1000, 131072), tree=tree,
                        probs=rng.random() < 0.5, greedy=rng.random() < 0.3, type=rng.choice(["bfloat16", "float16", "float32"]))
            if case["greedy"]:
                case["probs"] = False
            if case["requests"] * case["new"] * case["vocab"] <= 64 * 16 * 131072:
                return case
    page = rng.choice([8, 16, 16, 32, 64, 128])
    block = rng.choice([b for b in (1, 2, 8, 16, 32, 64, 128) if b <= page])
    head_dim = rng.choice([64, 72, 80, 96, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 16])
    kind = rng.choice(["bfloat16", "bfloat16", "float16"])
    sizes = dict(kv_heads=kv_heads, head_dim=head_dim, page=page, block=block, type=kind)
    if op != "attention":
        layers = rng.randint(1, 32)
        rows = _log(rng, 1, min(8192, 120_000_000 // (layers * kv_heads * head_dim)))
        if op == "dequantise":
            return dict(op=op, rows=rows, layers=layers, **sizes)
        new = _log(rng, 1, min(1024, rows))
        return dict(op=op, requests=max(1, rows // new), new=new, length=_log(rng, 1, 2000), layers=layers, **sizes)
    heads = kv_heads * rng.choice([h for h in (1, 2, 4, 5, 7, 8, 16) if h * kv_heads <= 32])
    while True:
        new = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 2, 64), _log(rng, 64, 256)])
        mask = "causal" if new == 1 else rng.choice(["tree", "tree", "causal", "all"]) if new <= 64 else rng.choice(["causal", "all"])
        case = dict(op=op, requests=_log(rng, 1, 64), new=new, length=_log(rng, 16, 32768), heads=heads, **sizes, mask=mask,
                    order=rng.choice(["token", "token", "head"]))
        w, most = work(case), work(listed()[6])
        if w["bytes"] <= most["bytes"] and w["flops"] <= 4 * most["flops"]:
            return case


# ------------------------------------------------------------------------- inputs

def _ramp(n, most, least=1):
    """n ragged lengths up to `most`, the same ones for every seed (their order is the seed's)."""
    return np.maximum(least, np.round(most * (np.arange(n) + 1) / n)).astype(np.int64)


def _lengths(case):
    """(cached, new) tokens of each request."""
    n = case["requests"]
    return _ramp(n, case["length"]), _ramp(n, case["new"])


def _shuffle(r, *arrays):
    order = r.permutation(len(arrays[0]))
    return [a[order] for a in arrays]


def _int(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _dtype(case):
    return getattr(torch, case["type"])


def _cumulated(new):
    return np.concatenate([[0], np.cumsum(new)])


def _parents(r, new):
    """Parents of every request's drafts: the first row is the root, another hangs on one of the eight before it."""
    idx = np.concatenate([np.arange(n) for n in new])
    back = np.floor(r.random(len(idx)) ** 2 * np.minimum(idx, 8)).astype(np.int64)
    return np.where(idx == 0, -1, idx - 1 - back)


def _ancestors(parents, new):
    """Rows of 32-bit words: bit k of a draft's row is set for itself and its ancestors."""
    words = max(1, (int(new.max()) + 31) // 32)
    out = np.zeros((len(parents), words), np.uint32)
    first = 0
    for n in new:
        for i in range(first, first + int(n)):
            if parents[i] >= 0:
                out[i] = out[first + parents[i]]
            out[i, (i - first) // 32] |= np.uint32(1) << np.uint32((i - first) % 32)
        first += int(n)
    return out.view(np.int32)


def _filled(case, g, layers, pages, order="token"):
    """Caches of keys and values [layers, pages, page, heads, dim] (e4m3) and their scales [layers, pages, blocks, heads], as
    writing rows of ordinary size leaves them: the largest code of a block is near the format's end."""
    page, block, kv, dim = case["page"], case["block"], case["kv_heads"], case["head_dim"]
    out = []
    for _ in range(2):
        codes = torch.empty((layers, pages, page, kv, dim) if order == "token" else (layers, pages, kv, page, dim),
                            dtype=torch.float8_e4m3fn, device="cuda")
        for layer in range(layers):
            codes[layer] = (torch.randn(codes.shape[1:], generator=g, device="cuda") * 90).clamp(-448, 448).to(torch.float8_e4m3fn)
        scale = torch.tensor([2.0 ** -8, 2.0 ** -7, 2.0 ** -6], device="cuda")[
            torch.randint(0, 3, (layers, pages, page // block, kv), generator=g, device="cuda")]
        out.append((codes if order == "token" else codes.transpose(2, 3), scale))
    (k, ks), (v, vs) = out
    return dict(k_cache=k, v_cache=v, k_scale=ks, v_scale=vs)


def prepare(case, seed):
    r = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"quantise": _prepare_quantise, "dequantise": _prepare_dequantise, "attention": _prepare_attention,
            "verify": _prepare_verify}[case["op"]](case, r, g)


def _quantised_layout(s):
    import paper_2607_12287_gb300 as ivit
    c = s["k_cache"][0] if s["k_cache"].dim() == 5 else s["k_cache"]
    return ivit.make_quantised_layout(c, s["case"]["block"], s["case"]["type"])


def _prepare_quantise(case, r, g):
    page, layers, kv, dim = case["page"], case["layers"], case["kv_heads"], case["head_dim"]
    base, new = _shuffle(r, *_lengths(case))
    need = -(-(base + new) // page)
    first = base // page  # (pages in front of the new tokens' are of no use here)
    pages = int((need - first).sum()) + 3
    ids = r.permutation(pages)
    slots, at = [], 0
    for b, n, f, m in zip(base, new, first, need):
        mine = ids[at:at + m - f]
        t = np.arange(b, b + n)
        slots.append(mine[t // page - f] * page + t % page)
        at += m - f
    rows = int(new.sum())
    drafts = rows + rows // 2 + 3  # of the step's rows, those that were accepted
    kind = _dtype(case)
    source = torch.empty((2, layers, drafts, kv, dim), dtype=kind, device="cuda")
    for part in source.flatten(0, 1):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * 1.7)
    s = dict(case=case, k=source[0], v=source[1], row=_int(np.sort(r.permutation(drafts)[:rows])), slots=_int(np.concatenate(slots)),
             **_filled(case, g, layers, pages))
    if own:
        s["cache"] = _quantised_layout(s)
    return s


def _prepare_dequantise(case, r, g):
    rows, page = case["rows"], case["page"]
    pages = -(-rows // page) + 3
    at = np.arange(rows)
    slots = r.permutation(pages)[at // page] * page + at % page
    shape = (case["layers"], rows, case["kv_heads"], case["head_dim"])
    s = dict(case=case, slots=_int(slots), **_filled(case, g, case["layers"], pages),
             k=torch.zeros(shape, dtype=_dtype(case), device="cuda"), v=torch.zeros(shape, dtype=_dtype(case), device="cuda"))
    if own:
        s["cache"] = _quantised_layout(s)
    return s


def _prepare_attention(case, r, g):
    n, page, dt = case["requests"], case["page"], _dtype(case)
    heads, kv, dim = case["heads"], case["kv_heads"], case["head_dim"]
    length, new = _shuffle(r, *_lengths(case))
    rows = int(new.sum())
    need = -(-length // page)
    table_pages = int(need.max()) + 2
    pages = int(need.sum()) + 5
    table = np.full((n, table_pages), -1, np.int64)
    table[np.arange(table_pages)[None, :] < need[:, None]] = r.permutation(pages)[: int(need.sum())]
    caches = {k: c[0] for k, c in _filled(case, g, 1, pages, case["order"]).items()}
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dt)
    qkv = normal(rows, (heads + 2 * kv) * dim)
    part = lambda t, lo, m: t[:, lo * dim:(lo + m) * dim].unflatten(1, (m, dim))
    mask = _ancestors(_parents(r, new), new) if case["mask"] == "tree" else None
    s = dict(case=case, q=(1.5 * part(qkv, 0, heads)).contiguous(), k=part(qkv, heads, kv), v=part(qkv, heads + kv, kv), **caches,
             table=_int(table), length=_int(length), cu=_int(_cumulated(new)),
             mask=None if mask is None else torch.from_numpy(mask).cuda(), most_len=int(length.max()), most_new=int(new.max()),
             out=torch.empty(rows, heads, dim, dtype=dt, device="cuda"),
             lse=torch.empty(rows, heads, dtype=torch.float32, device="cuda"))
    if own:
        import paper_2607_12287_gb300 as ivit
        s["cache"] = _quantised_layout(s)
        s["cfg"] = ivit.make_attention_config(n, heads, table_pages, s["most_new"], case["mask"],
                                              0 if mask is None else mask.shape[1], 1 / math.sqrt(dim))
        s["workspace"] = torch.empty(ivit.ivit_tree_attention_quantised_workspace(s["cfg"], s["cache"]), dtype=torch.uint8,
                                     device="cuda")
    return s


def _prepare_verify(case, r, g):
    """Logits of a target that is sure of some tokens and less so of others, a drafter that is near it, and drafts: drawn from
    the drafter's probabilities, or its likeliest ones (of those the target's best in most rows)."""
    n, vocab, dt = case["requests"], case["vocab"], _dtype(case)
    (new,) = _shuffle(r, _ramp(n, case["new"]))
    rows = int(new.sum())
    cu = _cumulated(new)
    parent = _parents(r, new) if case["tree"] else np.concatenate([np.arange(m) - 1 for m in new])
    logits = torch.empty((rows, vocab), dtype=dt, device="cuda")
    probs = torch.empty((rows, vocab), dtype=torch.float32, device="cuda") if case["probs"] else None
    above = _int(np.maximum(parent, 0) + np.repeat(cu[:-1], new)).long()  # the row that a draft hangs on
    kids = [[] for _ in range(rows)]
    for i, (p, a) in enumerate(zip(parent, above.tolist())):
        if p >= 0:
            kids[a].append(i)
    tokens = torch.zeros(rows, dtype=torch.int64, device="cuda")
    most = max([1] + [len(k) for k in kids])
    pick = torch.zeros((rows, most), dtype=torch.int64, device="cuda")
    for lo in range(0, rows, 64):
        x = 3.0 * torch.randn((min(64, rows - lo), vocab), generator=g, device="cuda")
        logits[lo:lo + 64] = x.to(dt)
        y = x + 0.5 * torch.randn(x.shape, generator=g, device="cuda")
        if case["probs"]:
            p = torch.softmax(y, 1)
            probs[lo:lo + 64] = p
            for j in range(most):
                pick[lo:lo + 64, j] = (p / torch.empty_like(p).exponential_(generator=g)).argmax(1)
        elif case["greedy"]:
            pick[lo:lo + 64] = torch.topk(y, most, 1).indices
        else:  # the drafter's guess is now and then the token that sampling the target gives
            z = x - torch.empty_like(x).exponential_(generator=g).log()
            pick[lo:lo + 64] = torch.topk(torch.where(torch.rand((x.shape[0], 1), generator=g, device="cuda") < 0.3, y, z), most, 1).indices
    hung = [(i, a, j) for a, mine in enumerate(kids) for j, i in enumerate(mine)]
    if hung:
        i, a, j = (torch.tensor(c, device="cuda") for c in zip(*hung))
        tokens[i] = pick[a, j]
    empty = lambda m: torch.full((m,), -1, dtype=torch.int32, device="cuda")
    s = dict(case=case, logits=logits, probs=probs, tokens=tokens.int(), parent=_int(parent) if case["tree"] else None, cu=_int(cu),
             temperature=None, uniform=None, noise=None, most_new=int(new.max()), path=empty(rows), accepted=empty(n), next=empty(n))
    if not case["greedy"]:
        s["temperature"] = torch.from_numpy(r.uniform(0.6, 1.2, n).astype(np.float32)).cuda()
        s["uniform"] = torch.rand(rows, generator=g, device="cuda")
        s["noise"] = torch.empty((n, vocab), device="cuda").exponential_(generator=g)
    if own:
        import paper_2607_12287_gb300 as ivit
        s["cfg"] = ivit.make_verify_config(n, vocab, s["most_new"], case["type"])
    return s


# --------------------------------------------------------------------------- runs

def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["op"]](s)


def _own_quantise(s):
    import paper_2607_12287_gb300 as ivit
    ivit.ivit_kv_quantise(s["cache"], s["k"], s["v"], s["row"], s["slots"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    return [s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]]


def _e4m3(x):
    return x.to(torch.float8_e4m3fn)


def _plain_quantise(s):
    case, page, block = s["case"], s["case"]["page"], s["case"]["block"]
    slots, row = s["slots"].long(), s["row"].long()
    blocks, of = torch.unique(slots // block, return_inverse=True)
    page_of, block_of = blocks * block // page, blocks * block % page // block
    written = torch.zeros((len(blocks), block), dtype=torch.bool, device="cuda")
    written[of, slots % block] = True
    place = torch.arange(block, device="cuda")
    kept = ~written & (place < torch.where(written, place, -1).amax(1, keepdim=True))
    token = block_of[:, None] * block + place
    for x, cache, scale in ((s["k"], s["k_cache"], s["k_scale"]), (s["v"], s["v_cache"], s["v_scale"])):
        for layer in range(case["layers"]):
            rows = x[layer, row].float()
            size = torch.where(rows.isfinite(), rows.abs(), 0.0).amax(2)
            most = torch.zeros((len(blocks), size.shape[1]), device="cuda")
            most.index_reduce_(0, of, size, "amax")
            # the smallest power of two by which the largest value fits
            m, e = torch.frexp(most)
            e = torch.where(most == 0, -60, e - 9 + (m > 0.875).int())
            old = scale[layer, page_of, block_of]
            m, eo = torch.frexp(old)
            e = torch.where(kept.any(1, keepdim=True), torch.maximum(e, eo - (m == 0.5).int()), e).clamp(-60, 60)
            new = ((e + 127) << 23).view(torch.float32)
            codes = cache[layer].view(torch.uint8)
            before = codes[page_of[:, None], token].view(torch.float8_e4m3fn)
            again = _e4m3(before.float() * (old / new)[:, None, :, None]).view(torch.uint8)
            codes[page_of[:, None].expand_as(token)[kept], token[kept]] = again[kept]
            rows = torch.where(rows.isfinite(), rows, math.nan)
            codes[slots // page, slots % page] = _e4m3(rows / new[of][:, :, None]).view(torch.uint8)
            scale[layer, page_of, block_of] = new
    return [s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]]


def _own_dequantise(s):
    import paper_2607_12287_gb300 as ivit
    ivit.ivit_kv_dequantise(s["cache"], s["slots"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["k"], s["v"])
    return [s["k"], s["v"]]


def _plain_dequantise(s):
    page, block, slots = s["case"]["page"], s["case"]["block"], s["slots"].long()
    for out, cache, scale in ((s["k"], s["k_cache"], s["k_scale"]), (s["v"], s["v_cache"], s["v_scale"])):
        codes = cache.view(torch.uint8)[:, slots // page, slots % page].view(torch.float8_e4m3fn)
        out.copy_(codes.float() * scale[:, slots // page, slots % page // block][..., None])
    return [s["k"], s["v"]]


def _own_attention(s):
    import paper_2607_12287_gb300 as ivit
    ivit.ivit_tree_attention_quantised(s["cfg"], s["cache"], s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"],
                                       s["v_scale"], s["table"], s["length"], s["cu"], s["mask"], s["out"], s["lse"], s["workspace"])
    return [s["out"], s["lse"]]


def _plain_attention(s):
    case = s["case"]
    n, heads, kv, dim, page = case["requests"], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    group, new, rows = heads // kv, s["most_new"], s["q"].shape[0]
    cu, length = s["cu"].long(), s["length"].long()
    # the cached tokens of every request, padded to the longest: [request, head, token, dim]
    t = torch.arange(s["most_len"], device="cuda")
    pages = s["table"].long()[:, t // page].clamp(min=0)

    def cached(codes, scale):
        x = codes.view(torch.uint8)[pages, t % page].view(torch.float8_e4m3fn).float()
        return (x * scale[pages, t % page // case["block"]][..., None]).transpose(1, 2)

    # the new rows of every request, padded to the most
    j = torch.arange(new, device="cuda")
    here = j[None] < (cu[1:] - cu[:-1])[:, None]
    row = (cu[:-1, None] + j[None]).clamp(max=rows - 1)
    q = s["q"][row].float().view(n, new, kv, group, dim).permute(0, 2, 1, 3, 4).reshape(n, kv, new * group, dim)
    fresh = lambda x: x[row].permute(0, 2, 1, 3).float()
    sees = here[:, None, :].expand(n, new, new)
    if case["mask"] == "causal":
        sees = sees & (j[None, :] <= j[:, None])
    elif case["mask"] == "tree":
        word = s["mask"][row][:, :, j // 32]
        sees = sees & ((word >> (j % 32).int()) & 1).bool()
    sees = torch.cat([(t[None] < length[:, None])[:, None].expand(n, new, s["most_len"]), sees], 2)
    sees = sees[:, None, :, None].expand(n, kv, new, group, sees.shape[-1]).reshape(n, kv, new * group, -1)
    score = q @ torch.cat([cached(s["k_cache"], s["k_scale"]), fresh(s["k"])], 2).transpose(2, 3) * (1 / math.sqrt(dim))
    score = torch.where(sees, score, -math.inf)
    most = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(most == -math.inf, 0.0, most))
    total = p.sum(-1, keepdim=True)
    out = p @ torch.cat([cached(s["v_cache"], s["v_scale"]), fresh(s["v"])], 2) / torch.where(total == 0, 1.0, total)
    lse = (most + total.log())[..., 0]
    r = torch.arange(rows, device="cuda")
    req = torch.searchsorted(cu[1:], r, right=True)
    at = lambda x: x.view(n, kv, new, group, *x.shape[3:])[req, :, r - cu[req]].flatten(1, 2)
    return [at(out).to(s["q"].dtype), at(lse)]


def _own_verify(s):
    import paper_2607_12287_gb300 as ivit
    ivit.ivit_tree_verify(s["cfg"], s["logits"], s["probs"], s["tokens"], s["parent"], s["cu"], s["temperature"], s["uniform"],
                          s["noise"], s["path"], s["accepted"], s["next"])
    return [s["path"], s["accepted"], s["next"]]


def _plain_verify(s):
    """A request's rows in order: a row that hangs on the last accepted one is accepted or not; in 64 bits (a decision is next
    to a border now and then)."""
    cu, logits = s["cu"].long(), s["logits"]
    n, rows, greedy = len(cu) - 1, logits.shape[0], s["case"]["greedy"]
    count = cu[1:] - cu[:-1]
    at = torch.zeros(n, dtype=torch.long, device="cuda")  # the last accepted row
    path = torch.full((n, s["most_new"]), -1, dtype=torch.long, device="cuda")
    path[:, 0] = cu[:-1]
    accepted = torch.ones(n, dtype=torch.long, device="cuda")
    i = torch.arange(n, device="cuda")

    def weights(of):  # of the tokens after these requests' last accepted rows
        x = logits[cu[of] + at[of]].double()
        return torch.exp((x - x.amax(1, keepdim=True)) / s["temperature"][of, None].double())

    if greedy:
        best = logits[cu[:-1]].float().argmax(1)
    else:
        w = weights(i)
        total, taken = w.sum(1), torch.zeros(n, dtype=torch.float64, device="cuda")
        e = w.clone()
    for j in range(1, s["most_new"]):
        row = (cu[:-1] + j).clamp(max=rows - 1)
        above = s["parent"][row].long() if s["parent"] is not None else torch.full_like(row, j - 1)
        test = (j < count) & (above == at)
        x = s["tokens"][row].long()
        if greedy:
            ok = test & (x == best)
        else:
            u, mine = s["uniform"][row].double(), w[i, x]
            ok = test & (u * total * (s["probs"][cu[:-1] + at, x].double() if s["probs"] is not None else 1.0) < mine)
            no = (test & ~ok).nonzero()[:, 0]
            if s["probs"] is not None:
                taken[no] += total[no]
                w[no] = (e[no] - taken[no, None] * s["probs"][(cu[:-1] + at)[no]].double()).clamp(min=0)
            else:
                w[no, x[no]] = 0.0
            total[no] = w[no].sum(1)
        yes = ok.nonzero()[:, 0]
        at[yes] = j
        path[yes, accepted[yes]] = cu[yes] + j
        accepted[yes] += 1
        if greedy:
            best[yes] = logits[cu[yes] + j].float().argmax(1)
        else:
            e[yes] = weights(yes)
            w[yes], total[yes], taken[yes] = e[yes], e[yes].sum(1), 0.0
    final = best if greedy else (w / s["noise"].double()).argmax(1)
    r = torch.arange(rows, device="cuda")
    req = torch.searchsorted(cu[1:], r, right=True)
    return [path[req, r - cu[req]].int(), accepted.int(), final.int()]


_OWN = {"quantise": _own_quantise, "dequantise": _own_dequantise, "attention": _own_attention, "verify": _own_verify}
_PLAIN = {"quantise": _plain_quantise, "dequantise": _plain_dequantise, "attention": _plain_attention, "verify": _plain_verify}


# --------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "verify":
        n, vocab = case["requests"], case["vocab"]
        new = _ramp(n, case["new"])
        # rows that are looked at: the first, and of the others those behind a draft that was right (about two of three runs
        # of drafts go on; a tree is about as deep as the square root of its rows, twice)
        depth = np.minimum(new, 2 * np.sqrt(new)) if case["tree"] else new
        seen = float(((1 - (2 / 3) ** depth) * 3).sum())
        size = 4 if case["type"] == "float32" else 2
        # the drafter's probabilities are needed whole where a draft was not right, the noise for the last token
        return dict(bytes=int(vocab * (seen * size + (0 if case["greedy"] else 4 * n) + (4 * n * (case["new"] > 1) if case["probs"] else 0))
                              + int(new.sum()) * 16 + 8 * n), flops=int(4 * vocab * seen))
    kv, dim = case["kv_heads"], case["head_dim"]
    if case["op"] == "quantise":
        base, new = _lengths(case)
        rows, block = int(new.sum()), case["block"]
        kept = int((base % block).sum())  # tokens that stay in the blocks, read at least where the scale grows (about half)
        blocks = int((-(-(base + new) // block) - base // block).sum())
        return dict(bytes=case["layers"] * 2 * kv * (rows * dim * 3 + kept * dim // 2 + blocks * 4) + 8 * rows, flops=0)
    if case["op"] == "dequantise":
        return dict(bytes=case["rows"] * (case["layers"] * 2 * kv * (3 * dim) + 4), flops=0)
    heads = case["heads"]
    length, new = _lengths(case)
    rows = int(new.sum())
    keys = length + (new if case["mask"] == "all" else (new + 1) / 2)
    return dict(bytes=int((length * dim + -(-length // case["block"]) * 4).sum()) * 2 * kv + rows * ((2 * heads + 2 * kv) * dim * 2 + 4 * heads),
                flops=float(4 * dim * heads * (keys * new).sum()))


# --------------------------------------------------------------------------- exact

def exact(case, seed):
    """What run() returns, from the definitions in 64 bits, request by request and head by head."""
    if case["op"] == "verify":
        return None  # whole numbers
    s = prepare(case, seed)
    return {"quantise": _exact_quantise, "dequantise": _exact_dequantise, "attention": _exact_attention}[case["op"]](case, s)


def _nearest(x):
    """The nearest e4m3 value: 3 bits behind the first, steps of 2^-9 at least, ties to even."""
    powers = torch.tensor([2.0 ** k for k in range(-6, 9)], dtype=torch.float64, device="cuda")
    step = powers[(torch.bucketize(x.abs(), powers, right=True) - 1).clamp(min=0)] / 8
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_quantise(case, s):
    page, block = case["page"], case["block"]
    slots, row = s["slots"].tolist(), s["row"].tolist()
    groups = {}
    for i, slot in zip(row, slots):
        groups.setdefault(slot // block, {})[slot % block] = i
    done, scales = [], []
    powers = torch.tensor([2.0 ** k for k in range(-60, 61)], dtype=torch.float64, device="cuda")
    least = lambda size: torch.bucketize(size, powers[:-1])  # of the powers, the first that is not below `size`
    for x, cache, scale in ((s["k"], s["k_cache"], s["k_scale"]), (s["v"], s["v_cache"], s["v_scale"])):
        c, f = cache.double(), scale.double()
        ids = torch.tensor(list(groups), device="cuda")
        pages, blocks = ids * block // page, ids * block % page // block
        # [groups, block]: the row that is written, -1 where none is; whether a token stays there
        src = torch.full((len(groups), block), -1, dtype=torch.long)
        for gi, places in enumerate(groups.values()):
            for p, i in places.items():
                src[gi, p] = i
        src = src.cuda()
        last = (src >= 0).long().mul(torch.arange(1, block + 1, device="cuda")).amax(1, keepdim=True)
        stays = (src < 0) & (torch.arange(1, block + 1, device="cuda") < last)
        tokens = blocks[:, None] * block + torch.arange(block, device="cuda")
        for layer in range(case["layers"]):
            rows = x[layer].double()[src.clamp(min=0)]  # [groups, block, heads, dim]
            rows = torch.where((src >= 0)[:, :, None, None], rows, 0.0)
            most = rows.abs().amax((1, 3))
            old = f[layer, pages, blocks]
            new = powers[torch.where(stays.any(1)[:, None], torch.maximum(least(most / 448), least(old)), least(most / 448))]
            held = c[layer][pages[:, None], tokens]
            value = torch.where((src >= 0)[:, :, None, None], rows, held * old[:, None, :, None]) / new[:, None, :, None]
            value = torch.where(((src >= 0) | stays)[:, :, None, None], _nearest(value), held)
            c[layer][pages[:, None], tokens] = value
            f[layer, pages, blocks] = new
        done.append(c)
        scales.append(f)
    return done + scales


def _exact_dequantise(case, s):
    page, block, slots = case["page"], case["block"], s["slots"].long()
    done = []
    for cache, scale in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])):
        flat = cache.double() * scale.double().repeat_interleave(block, 2)[..., None]
        done.append(flat.flatten(1, 2)[:, slots])
    return done


def _exact_attention(case, s):
    page, kv = case["page"], case["kv_heads"]
    group, rows = case["heads"] // kv, s["q"].shape[0]
    out = torch.zeros(rows, case["heads"], case["head_dim"], dtype=torch.float64, device="cuda")
    lse = torch.full((rows, case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    cu, lengths = s["cu"].tolist(), s["length"].tolist()
    # the caches' values, block by block
    values = [c.float() * f.repeat_interleave(case["block"], 1)[..., None]
              for c, f in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"]))]  # (code x power of two: exact)
    for i, length in enumerate(lengths):
        lo, hi = cu[i], cu[i + 1]
        n = hi - lo
        at = torch.arange(length, device="cuda")
        pages = s["table"][i].long()[at // page]
        if case["mask"] == "tree":
            words = s["mask"][lo:hi].long().cpu().numpy() & 0xFFFFFFFF
            sees = torch.tensor([[bool(words[a, b // 32] >> (b % 32) & 1) for b in range(n)] for a in range(n)], device="cuda")
        else:
            sees = torch.ones(n, n, dtype=torch.bool, device="cuda")
            sees = sees.tril() if case["mask"] == "causal" else sees
        hidden = torch.cat([torch.zeros(n, length, dtype=torch.bool, device="cuda"), ~sees], 1)
        for h in range(kv):
            k = torch.cat([values[0][pages, at % page, h].double(), s["k"][lo:hi, h].double()])
            v = torch.cat([values[1][pages, at % page, h].double(), s["v"][lo:hi, h].double()])
            for q in range(h * group, (h + 1) * group):
                score = (s["q"][lo:hi, q].double() @ k.T / math.sqrt(case["head_dim"])).masked_fill(hidden, -math.inf)
                lse[lo:hi, q] = torch.logsumexp(score, 1)
                out[lo:hi, q] = torch.softmax(score, 1) @ v
    return [out, lse]
