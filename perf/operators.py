"""Operator cases of the language backbone's attention: the step that answers from the encoder's tokens.

Behind the encoder a policy has a language backbone.  It takes a view's tokens as a prompt, keeps
their keys and values in a cache of pages, and answers with tokens of its own, one at a time or as a
tree of drafted ones that is verified in one pass.  The operators are

- ``plan``: a step's pages, slots, positions and tree masks from the requests' lengths;
- ``rope``: the norm of every query and key head and the rotation by positions of one or three axes
  (time, height, width), keys and values going straight into the pages or the keys back to the caller;
- ``rope_backward``: its gradients, for fine-tuning the backbone on the encoder's tokens;
- ``attention``: the new tokens of each request over its cached ones and over each other (a tree of
  drafts, a causal run, or all of a view's tokens);
- ``write``: keys and values of the accepted drafts of every layer into their slots.

Sizes: 196, 256 or 1024 tokens a view and up to 32 views as in ``synth.WORKLOADS``, heads of 64 and 72 as in
its encoders, else generic ones (64, 96, 128 and 256 wide, 1 to 16 query heads to a key head).
"""
import math

import numpy as np
import torch

own = False

ATTN = dict(op="attention")
VIEW_HEADS = dict(heads=16, kv_heads=16, head_dim=72)


def listed():
    return [
        # eight robots, each about to decode one token: the lightest step
        dict(name="plan_decode", op="plan", requests=8, page=16, tree=False, new=1, length=700),
        # a serving batch: trees of up to 64 drafts after a verified step, some requests finished
        dict(name="plan_trees", op="plan", requests=512, page=32, tree=True, new=64, length=8192),
        # one token of eight requests into the cache: the smallest call of a layer
        dict(name="rope_decode", op="rope", rows=8, heads=32, kv_heads=8, head_dim=128, rot=128, axes=1, type="bfloat16",
             interleaved=False, norm=True, cached=True, page=16),
        # 32 views of 1024 tokens with (time, height, width) positions: the prompt of a serving batch
        dict(name="rope_views", op="rope", rows=32768, **VIEW_HEADS, rot=72, axes=3, type="bfloat16", interleaved=False,
             norm=True, cached=False, page=16),
        # a training batch of 32 views of 196 tokens
        dict(name="rope_backward_views", op="rope_backward", rows=6272, **VIEW_HEADS, rot=72, axes=3, type="bfloat16",
             interleaved=False, norm=True),
        # a training batch of text and view tokens, grouped heads, an odd number of rows
        dict(name="rope_backward_text", op="rope_backward", rows=16385, heads=32, kv_heads=8, head_dim=128, rot=128, axes=1,
             type="float16", interleaved=True, norm=True),
        # one robot decoding after three views and an instruction: latency
        dict(name="attention_one", **ATTN, requests=1, new=1, length=1041, heads=16, kv_heads=4, head_dim=64, page=16,
             type="bfloat16", mask="causal", order="token"),
        # a serving batch decoding over long, ragged contexts: the cache's bytes
        dict(name="attention_decode", **ATTN, requests=32, new=1, length=16384, heads=32, kv_heads=8, head_dim=128, page=16,
             type="bfloat16", mask="causal", order="token"),
        # trees of up to 31 drafts being verified
        dict(name="attention_trees", **ATTN, requests=16, new=31, length=8192, heads=32, kv_heads=8, head_dim=128, page=64,
             type="float16", mask="tree", order="head"),
        # a new view's 256 tokens, each seeing all of them and the frames before
        dict(name="attention_views", **ATTN, requests=8, new=256, length=2048, **VIEW_HEADS, page=32, type="bfloat16",
             mask="all", order="token"),
        # a few accepted drafts of one robot
        dict(name="write_few", op="write", rows=5, layers=27, kv_heads=4, head_dim=64, page=16, type="bfloat16"),
        # the accepted drafts of a large batch
        dict(name="write_many", op="write", rows=2048, layers=32, kv_heads=8, head_dim=128, page=32, type="float16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "rope", "rope", "rope_backward", "attention", "attention", "attention", "write"])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    if op == "plan":
        tree = rng.random() < 0.6
        return dict(op=op, requests=_log(rng, 1, 1000), page=page, tree=tree, new=_log(rng, 1, 64 if tree else 128),
                    length=_log(rng, 16, 8192))
    head_dim = rng.choice([64, 72, 80, 96, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 16])
    heads = kv_heads * rng.choice([h for h in (1, 2, 4, 5, 7, 8, 16) if h * kv_heads <= 32])
    kind = rng.choice(["bfloat16", "bfloat16", "float16"])
    sizes = dict(heads=heads, kv_heads=kv_heads, head_dim=head_dim)
    if op in ("rope", "rope_backward"):
        axes = rng.choice([1, 1, 3])
        rot = rng.choice([head_dim, head_dim, head_dim // 16 * 8])
        # (a pass has at most the largest listed one's bytes)
        rows = _log(rng, 1, min(32768, 75_000_000 // ((heads + 2 * kv_heads) * head_dim)))
        case = dict(op=op, rows=rows, **sizes, rot=rot, axes=axes, type=kind, interleaved=rng.random() < 0.3,
                    norm=rng.random() < 0.8)
        return dict(case, cached=rng.random() < 0.5, page=page) if op == "rope" else case
    if op == "write":
        layers = rng.randint(1, 32)
        return dict(op=op, rows=_log(rng, 1, min(2048, 60_000_000 // (layers * kv_heads * head_dim))), layers=layers,
                    kv_heads=kv_heads, head_dim=head_dim, page=page, type=kind)
    while True:
        new = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 2, 64), _log(rng, 64, 256)])
        mask = "causal" if new == 1 else rng.choice(["tree", "tree", "causal", "all"]) if new <= 64 else rng.choice(["causal", "all"])
        case = dict(op=op, requests=_log(rng, 1, 64), new=new, length=_log(rng, 16, 32768), **sizes, page=page, type=kind,
                    mask=mask, order=rng.choice(["token", "token", "head"]))
        w, most = work(case), work(listed()[7])
        if w["bytes"] <= most["bytes"] and w["flops"] <= 4 * most["flops"]:
            return case


# ------------------------------------------------------------------------- inputs

def _ramp(n, most, least=1):
    """n ragged lengths up to `most`, the same ones for every seed (their order is the seed's)."""
    return np.maximum(least, np.round(most * (np.arange(n) + 1) / n)).astype(np.int64)


def _plan_lengths(case):
    """(cached, new) tokens of each request; of sixteen one has finished and gives its pages back."""
    n = case["requests"]
    length, new = _ramp(n, case["length"]), _ramp(n, case["new"])
    done = np.arange(n) % 16 == 15
    return np.where(done, 0, length), np.where(done, 0, new)


def _shuffle(r, *arrays):
    order = r.permutation(len(arrays[0]))
    return [a[order] for a in arrays]


def _parents(r, new):
    """Parents of every request's drafts: the first is the root, another hangs on one of the eight before it."""
    idx = np.concatenate([np.arange(n) for n in new]) if len(new) else np.zeros(0, np.int64)
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


def _int(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _dtype(case):
    return getattr(torch, case["type"])


def _cumulated(new):
    return np.concatenate([[0], np.cumsum(new)])


def prepare(case, seed):
    r = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"plan": _prepare_plan, "rope": _prepare_rope, "rope_backward": _prepare_rope, "attention": _prepare_attention,
            "write": _prepare_write}[case["op"]](case, r, g)


def _prepare_plan(case, r, g):
    n, page = case["requests"], case["page"]
    base, new = _shuffle(r, *_plan_lengths(case))
    # the step before had reserved more than was accepted (drafts), or just what is there now (one token)
    held = np.where(base == 0, r.integers(1, case["length"] + 1, n), base + r.integers(0, case["new"], n))
    table_pages = -(-(case["length"] + 2 * case["new"]) // page) + 1
    held_pages = -(-held // page)
    most = np.where(base == 0, case["length"], base + case["new"])  # tokens that a request can hold before the step
    n_pages = int((-(-most // page) + -(-new // page) + 1).sum()) + 8
    ids = r.permutation(n_pages)
    table = np.full((n, table_pages), -1, np.int64)
    cols = np.arange(table_pages)[None, :] < held_pages[:, None]
    table[cols] = ids[: int(held_pages.sum())]
    free = ids[int(held_pages.sum()):]
    head = int(r.integers(0, n_pages))
    ring = np.zeros(n_pages, np.int64)
    ring[(head + np.arange(len(free))) % n_pages] = free
    rows = int(new.sum())
    words = (case["new"] + 31) // 32 if case["tree"] else 0
    s = dict(case=case, rows=rows, words=words, n_pages=n_pages, held=_int(held), base=_int(base), new=_int(new),
             parent=_int(_parents(r, new)) if case["tree"] else None, ring=_int(ring), ring_in=_int([head, len(free)]),
             table=_int(table))
    empty = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")
    s.update(cu=empty(n + 1), req=empty(rows), slots=empty(rows), pos=empty(rows),
             mask=empty(rows, words) if case["tree"] else None, ring_out=empty(2), status=empty(1))
    if own:
        import paper_2607_12287_gb300 as ivit
        s["cfg"] = ivit.make_plan_config(n, rows, table_pages, page, n_pages, words)
    return s


def _rotation(case, r):
    """(frequency, axis) of every pair: one ladder over all pairs, or one over each axis' share."""
    half = case["rot"] // 2
    if case["axes"] == 1:
        return 10000.0 ** (-np.arange(half) / half), np.zeros(half, np.int64)
    t = half // 4
    share = [t, (half - t) // 2, half - t - (half - t) // 2]
    freq = np.concatenate([100.0 ** (-np.arange(n) / max(1, n)) for n in share])
    return freq, np.repeat(np.arange(3), share)


def _prepare_rope(case, r, g):
    rows, heads, kv, dim, dt = case["rows"], case["heads"], case["kv_heads"], case["head_dim"], _dtype(case)
    i = np.arange(rows)
    if case["axes"] == 3:  # views of 1024 tokens on a 32 x 32 grid, one after another in time
        pos = np.stack([i // 1024 + r.integers(0, 8), i % 1024 // 32, i % 32])
    elif rows <= 64:  # decoding: a token of each request, anywhere in its context
        pos = r.integers(0, 1024, (1, rows))
    else:  # sequences of 1024 tokens
        pos = (i[None] + r.integers(0, 1024)) % 1024
    freq, axis = _rotation(case, r)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    qkv = (normal(rows, (heads + 2 * kv) * dim) * 1.7).to(dt)
    part = lambda t, lo, n: t[:, lo * dim:(lo + n) * dim].unflatten(1, (n, dim))
    s = dict(case=case, q=part(qkv, 0, heads), k=part(qkv, heads, kv), v=part(qkv, heads + kv, kv), pos=_int(pos),
             freq=torch.from_numpy(freq.astype(np.float32)).cuda(), axis=_int(axis),
             q_weight=(1 + 0.2 * normal(dim)).to(dt) if case["norm"] else None,
             k_weight=(1 + 0.2 * normal(dim)).to(dt) if case["norm"] else None)
    empty = lambda *shape: torch.zeros(shape, dtype=dt, device="cuda")
    if case["op"] == "rope":
        s["q_out"] = empty(rows, heads, dim)
        if case["cached"]:
            pages = -(-rows // case["page"]) + 3
            slot = r.permutation(pages)[i // case["page"]] * case["page"] + i % case["page"]
            s.update(slots=_int(slot), k_cache=empty(pages, case["page"], kv, dim), v_cache=empty(pages, case["page"], kv, dim))
        else:
            s["k_out"] = empty(rows, kv, dim)
    else:
        s["grad_q"], s["grad_k"] = normal(rows, heads, dim).to(dt), normal(rows, kv, dim).to(dt)
        dqkv = empty(rows, (heads + kv) * dim)
        s["dq"], s["dk"] = part(dqkv, 0, heads), part(dqkv, heads, kv)
        if case["norm"]:
            s["dq_weight"], s["dk_weight"] = (torch.empty(dim, dtype=torch.float32, device="cuda") for _ in range(2))
    if own:
        import paper_2607_12287_gb300 as ivit
        s["cfg"] = ivit.make_rope_config(heads, kv, dim, case["rot"], case["axes"], case["interleaved"], 1e-6, case["type"])
        if case["op"] == "rope_backward":
            s["workspace"] = torch.empty(ivit.ivit_qk_norm_rope_backward_workspace(s["cfg"]), dtype=torch.uint8, device="cuda")
        elif case["cached"]:
            s["cache"] = ivit.make_cache_layout(s["k_cache"])
    return s


def _attention_lengths(case):
    n = case["requests"]
    return _ramp(n, case["length"]), _ramp(n, case["new"])


def _prepare_attention(case, r, g):
    n, page, dt = case["requests"], case["page"], _dtype(case)
    heads, kv, dim = case["heads"], case["kv_heads"], case["head_dim"]
    length, new = _shuffle(r, *_attention_lengths(case))
    rows = int(new.sum())
    need = -(-length // page)
    table_pages = int(need.max()) + 2
    pages = int(need.sum()) + 5
    table = np.full((n, table_pages), -1, np.int64)
    table[np.arange(table_pages)[None, :] < need[:, None]] = r.permutation(pages)[: int(need.sum())]
    shape = (pages, page, kv, dim) if case["order"] == "token" else (pages, kv, page, dim)
    cache = lambda: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)
    kc, vc = cache(), cache()
    if case["order"] == "head":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dt)
    qkv = normal(rows, (heads + 2 * kv) * dim)
    part = lambda t, lo, m: t[:, lo * dim:(lo + m) * dim].unflatten(1, (m, dim))
    mask = _ancestors(_parents(r, new), new) if case["mask"] == "tree" else None
    s = dict(case=case, q=(1.5 * part(qkv, 0, heads)).contiguous(), k=part(qkv, heads, kv), v=part(qkv, heads + kv, kv),
             k_cache=kc, v_cache=vc, table=_int(table), length=_int(length), cu=_int(_cumulated(new)),
             mask=None if mask is None else torch.from_numpy(mask).cuda(), most_len=int(length.max()), most_new=int(new.max()),
             out=torch.empty(rows, heads, dim, dtype=dt, device="cuda"),
             lse=torch.empty(rows, heads, dtype=torch.float32, device="cuda"))
    if own:
        import paper_2607_12287_gb300 as ivit
        s["cache"] = ivit.make_cache_layout(kc)
        s["cfg"] = ivit.make_attention_config(n, heads, table_pages, s["most_new"], case["mask"],
                                              0 if mask is None else mask.shape[1], 1 / math.sqrt(dim))
        s["workspace"] = torch.empty(ivit.ivit_tree_attention_workspace(s["cfg"], s["cache"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_write(case, r, g):
    rows, layers, page, dt = case["rows"], case["layers"], case["page"], _dtype(case)
    kv, dim = case["kv_heads"], case["head_dim"]
    drafts = rows + rows // 2 + 3  # of the drafted rows, those that were accepted
    pages = -(-2 * rows // page) + 2
    source = torch.randn((2, layers, drafts, kv, dim), generator=g, device="cuda").to(dt)
    row = np.sort(r.permutation(drafts)[:rows])
    slot = r.permutation(pages * page)[:rows]
    caches = torch.zeros((2, layers, pages, page, kv, dim), dtype=dt, device="cuda")
    s = dict(case=case, k=source[0], v=source[1], row=_int(row), slots=_int(slot), k_cache=caches[0], v_cache=caches[1])
    if own:
        import paper_2607_12287_gb300 as ivit
        s["cache"] = ivit.make_cache_layout(s["k_cache"][0])
    return s


# --------------------------------------------------------------------------- runs

def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["op"]](s)


def _own_plan(s):
    import paper_2607_12287_gb300 as ivit
    ivit.ivit_step_plan(s["cfg"], s["held"], s["base"], s["new"], s["parent"], s["ring"], s["ring_in"], s["table"], s["cu"],
                        s["req"], s["slots"], s["pos"], s["mask"], s["ring_out"], s["status"])
    return [s[k] for k in ("cu", "req", "slots", "pos", "mask", "ring", "ring_out", "table", "status")]


def _plain_plan(s):
    case, page, n_pages, rows = s["case"], s["case"]["page"], s["n_pages"], s["rows"]
    held, base, new, table = (s[k].long() for k in ("held", "base", "new", "table"))
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    have, need = (held + page - 1) // page, (base + new + page - 1) // page
    grow, shrink = (need - have).clamp(min=0), (have - need).clamp(min=0)
    head, count = s["ring_in"].long()
    granted = grow.cumsum(0) - grow
    col = torch.arange(table.shape[1], device="cuda")[None]
    fresh = s["ring"].long()[(head + granted[:, None] + col - have[:, None]) % n_pages]
    table_out = torch.where((col >= have[:, None]) & (col < need[:, None]), fresh, table)
    # returned pages go behind the last free one (what is not returned lands in a spare place)
    returned = shrink.cumsum(0) - shrink
    back = (col >= need[:, None]) & (col < have[:, None])
    at = torch.where(back, (head + count + returned[:, None] + col - need[:, None]) % n_pages, n_pages)
    ring = torch.cat([s["ring"].long(), s["ring"].new_zeros(1).long()]).scatter(0, at.reshape(-1), table.reshape(-1))[:n_pages]
    ring_out = torch.stack([(head + grow.sum()) % n_pages, count - grow.sum() + shrink.sum()])
    r = torch.arange(rows, device="cuda")
    req = torch.searchsorted(cu[1:], r, right=True)
    j = r - cu[req]
    at = base[req] + j
    slots = table_out[req, at // page] * page + at % page
    mask, depth = None, j
    if case["tree"]:
        n = case["new"]
        # (I + A)^n has a positive entry wherever one node is an ancestor of the other, or itself
        step = torch.eye(n, device="cuda").repeat(len(new), 1, 1)
        parent = s["parent"].long()
        step[req, j, parent.clamp(min=0)] += (parent >= 0).float()
        above = (torch.linalg.matrix_power(step, n) > 0)[req, j]
        depth = above.sum(1) - 1
        bits = torch.nn.functional.pad(above.long(), (0, 32 * s["words"] - n)).view(rows, s["words"], 32)
        mask = (bits << torch.arange(32, device="cuda")).sum(2)
        mask = torch.where(mask >= 2 ** 31, mask - 2 ** 32, mask)
    status = torch.zeros(1, device="cuda")
    return [None if x is None else x.int() for x in (cu, req, slots, base[req] + depth, mask, ring, ring_out, table_out, status)]


def _own_rope(s):
    import paper_2607_12287_gb300 as ivit
    if s["case"]["cached"]:
        ivit.ivit_qk_norm_rope(s["cfg"], s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["pos"], s["freq"], s["axis"],
                               s["q_out"], None, s["cache"], s["k_cache"], s["v_cache"], s["slots"])
        return [s["q_out"], s["k_cache"], s["v_cache"]]
    ivit.ivit_qk_norm_rope(s["cfg"], s["q"], s["k"], None, s["q_weight"], s["k_weight"], s["pos"], s["freq"], s["axis"],
                           s["q_out"], s["k_out"])
    return [s["q_out"], s["k_out"]]


def _angles(s):
    a = s["pos"].float()[s["axis"].long()].T * s["freq"]
    return a.cos()[:, None], a.sin()[:, None]


def _pairs(x, rot, interleaved):
    x = x[..., :rot]
    return (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:])


def _joined(a, b, rest, interleaved):
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), rest], -1)


def _plain_rotated(x, weight, cos, sin, case):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * weight.float()
    a, b = _pairs(y, case["rot"], case["interleaved"])
    return _joined(a * cos - b * sin, b * cos + a * sin, y[..., case["rot"]:], case["interleaved"]).to(x.dtype)


def _plain_rope(s):
    case, (cos, sin) = s["case"], _angles(s)
    q = _plain_rotated(s["q"], s["q_weight"], cos, sin, case)
    k = _plain_rotated(s["k"], s["k_weight"], cos, sin, case)
    if not case["cached"]:
        return [q, k]
    slots = s["slots"].long()
    s["k_cache"][slots // case["page"], slots % case["page"]] = k
    s["v_cache"][slots // case["page"], slots % case["page"]] = s["v"]
    return [q, s["k_cache"], s["v_cache"]]


def _own_rope_backward(s):
    import paper_2607_12287_gb300 as ivit
    norm = s["case"]["norm"]
    dqw, dkw = (s["dq_weight"], s["dk_weight"]) if norm else (None, None)
    ivit.ivit_qk_norm_rope_backward(s["cfg"], s["grad_q"], s["grad_k"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["pos"],
                                    s["freq"], s["axis"], s["dq"], s["dk"], dqw, dkw, s["workspace"])
    return [s["dq"], s["dk"]] + ([dqw, dkw] if norm else [])


def _plain_gradient(g, x, weight, cos, sin, case):
    y = g.float()
    a, b = _pairs(y, case["rot"], case["interleaved"])
    y = _joined(a * cos + b * sin, b * cos - a * sin, y[..., case["rot"]:], case["interleaved"])
    if weight is None:
        return y.to(x.dtype), None
    x32 = x.float()
    r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + 1e-6)
    unit = x32 * r
    u = y * weight.float()
    return (r * (u - unit * (u * unit).mean(-1, keepdim=True))).to(x.dtype), (y * unit).sum((0, 1))


def _plain_rope_backward(s):
    cos, sin = _angles(s)
    dq, dqw = _plain_gradient(s["grad_q"], s["q"], s["q_weight"], cos, sin, s["case"])
    dk, dkw = _plain_gradient(s["grad_k"], s["k"], s["k_weight"], cos, sin, s["case"])
    return [dq, dk] + ([dqw, dkw] if s["case"]["norm"] else [])


def _own_attention(s):
    import paper_2607_12287_gb300 as ivit
    ivit.ivit_tree_attention(s["cfg"], s["cache"], s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["length"],
                             s["cu"], s["mask"], s["out"], s["lse"], s["workspace"])
    return [s["out"], s["lse"]]


def _plain_attention(s):
    case = s["case"]
    n, heads, kv, dim, page = case["requests"], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    group, new, rows = heads // kv, s["most_new"], s["q"].shape[0]
    cu, length = s["cu"].long(), s["length"].long()
    # the cached tokens of every request, padded to the longest: [request, head, token, dim]
    t = torch.arange(s["most_len"], device="cuda")
    pages = s["table"].long()[:, t // page].clamp(min=0)
    cached = lambda c: c[pages, t % page].transpose(1, 2).float()
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
    score = q @ torch.cat([cached(s["k_cache"]), fresh(s["k"])], 2).transpose(2, 3) * (1 / math.sqrt(dim))
    score = torch.where(sees, score, -math.inf)
    most = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(most == -math.inf, 0.0, most))
    total = p.sum(-1, keepdim=True)
    out = p @ torch.cat([cached(s["v_cache"]), fresh(s["v"])], 2) / torch.where(total == 0, 1.0, total)
    lse = (most + total.log())[..., 0]
    r = torch.arange(rows, device="cuda")
    req = torch.searchsorted(cu[1:], r, right=True)
    at = lambda x: x.view(n, kv, new, group, *x.shape[3:])[req, :, r - cu[req]].flatten(1, 2)
    return [at(out).to(s["q"].dtype), at(lse)]


def _own_write(s):
    import paper_2607_12287_gb300 as ivit
    ivit.ivit_kv_write(s["cache"], s["k"], s["v"], s["row"], s["slots"], s["k_cache"], s["v_cache"])
    return [s["k_cache"], s["v_cache"]]


def _plain_write(s):
    page, slots, row = s["case"]["page"], s["slots"].long(), s["row"].long()
    s["k_cache"][:, slots // page, slots % page] = s["k"][:, row]
    s["v_cache"][:, slots // page, slots % page] = s["v"][:, row]
    return [s["k_cache"], s["v_cache"]]


_OWN = {"plan": _own_plan, "rope": _own_rope, "rope_backward": _own_rope_backward, "attention": _own_attention, "write": _own_write}
_PLAIN = {"plan": _plain_plan, "rope": _plain_rope, "rope_backward": _plain_rope_backward, "attention": _plain_attention,
          "write": _plain_write}


# --------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "plan":
        base, new = _plan_lengths(case)
        words = (case["new"] + 31) // 32 if case["tree"] else 0
        n, rows = len(new), int(new.sum())
        return dict(bytes=4 * (4 * n + rows * (3 + words + bool(words)) + int((-(-new // case["page"])).sum()) + 6), flops=rows)
    kv, dim = case["kv_heads"], case["head_dim"]
    if case["op"] == "write":
        return dict(bytes=case["rows"] * (case["layers"] * 2 * kv * dim * 2 * 2 + 8), flops=0)
    heads = case["heads"]
    if case["op"] == "rope":
        vectors = heads + kv * (2 if case["cached"] else 1)
        return dict(bytes=case["rows"] * (2 * vectors * dim * 2 + 4 * case["axes"]), flops=case["rows"] * (heads + kv) * dim * 6)
    if case["op"] == "rope_backward":
        return dict(bytes=case["rows"] * (3 * (heads + kv) * dim * 2 + 4 * case["axes"]), flops=case["rows"] * (heads + kv) * dim * 12)
    length, new = _attention_lengths(case)
    rows = int(new.sum())
    keys = length + (new if case["mask"] == "all" else (new + 1) / 2)
    return dict(bytes=int(length.sum()) * 2 * kv * dim * 2 + rows * ((2 * heads + 2 * kv) * dim * 2 + 4 * heads),
                flops=float(4 * dim * heads * (keys * new).sum()))


# --------------------------------------------------------------------------- exact

def exact(case, seed):
    """What run() returns, from the definitions in 64 bits, request by request and head by head."""
    if case["op"] == "plan":
        return None  # whole numbers
    s = prepare(case, seed)
    return {"rope": _exact_rope, "rope_backward": _exact_rope_backward, "attention": _exact_attention,
            "write": _exact_write}[case["op"]](case, s)


def _turned(x, s, case, sign):
    """x[rows, heads, dim] in complex form: every pair times exp(i sign angle)."""
    rot, half = case["rot"], case["rot"] // 2
    angle = torch.stack([s["pos"][int(a)].double() * f for a, f in zip(s["axis"], s["freq"].double())], 1)
    turn = torch.polar(torch.ones_like(angle), sign * angle)
    first = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else half)
    out = x.clone()
    for h in range(x.shape[1]):
        z = torch.complex(x[:, h, first], x[:, h, second]) * turn
        out[:, h, first], out[:, h, second] = z.real, z.imag
    return out


def _exact_rope(case, s):
    done = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.double()
        if w is not None:
            y = y / (y.pow(2).sum(-1, keepdim=True) / case["head_dim"] + 1e-6).sqrt() * w.double()
        done.append(_turned(y, s, case, 1.0))
    if not case["cached"]:
        return done
    caches = []
    for c, x in ((s["k_cache"], done[1]), (s["v_cache"], s["v"].double())):
        flat = c.double().flatten(0, 1)
        flat[s["slots"].long()] = x
        caches.append(flat.view(c.shape))
    return [done[0]] + caches


def _exact_rope_backward(case, s):
    dx, dw = [], []
    for g, x, w in ((s["grad_q"], s["q"], s["q_weight"]), (s["grad_k"], s["k"], s["k_weight"])):
        y, x = _turned(g.double(), s, case, -1.0), x.double()
        if w is not None:
            # d/dx of w x / n(x), n = sqrt(mean x^2 + eps)
            n = (x.pow(2).sum(-1, keepdim=True) / case["head_dim"] + 1e-6).sqrt()
            dw.append((y * x / n).sum(1).sum(0))
            y = y * w.double()
            y = y / n - x * (y * x).sum(-1, keepdim=True) / (case["head_dim"] * n.pow(3))
        dx.append(y)
    return dx + dw


def _exact_attention(case, s):
    page, kv = case["page"], case["kv_heads"]
    group, rows = case["heads"] // kv, s["q"].shape[0]
    out = torch.zeros(rows, case["heads"], case["head_dim"], dtype=torch.float64, device="cuda")
    lse = torch.full((rows, case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    cu, lengths = s["cu"].tolist(), s["length"].tolist()
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
            k = torch.cat([s["k_cache"][pages, at % page, h], s["k"][lo:hi, h]]).double()
            v = torch.cat([s["v_cache"][pages, at % page, h], s["v"][lo:hi, h]]).double()
            for q in range(h * group, (h + 1) * group):
                score = (s["q"][lo:hi, q].double() @ k.T / math.sqrt(case["head_dim"])).masked_fill(hidden, -math.inf)
                lse[lo:hi, q] = torch.logsumexp(score, 1)
                out[lo:hi, q] = torch.softmax(score, 1) @ v
    return [out, lse]


def _exact_write(case, s):
    done = []
    for c, x in ((s["k_cache"], s["k"]), (s["v_cache"], s["v"])):
        d = torch.zeros(c.shape, dtype=torch.float64, device="cuda")
        for layer in range(case["layers"]):
            d[layer].flatten(0, 1)[s["slots"].long()] = x[layer, s["row"].long()].double()
        done.append(d)
    return done
