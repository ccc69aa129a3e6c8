"""GPU parity of the language backbone's operators against their 64-bit restatement.

Error bounds, per value, with u half a unit in the last place of the 16-bit type relative to a value
(2^-8 bf16, 2^-11 fp16):
- rotation: u |y| for the rounding, and 2^-18 of the head's largest input magnitude for the fp32
  arithmetic (a sum of up to 256 squares, one rsqrt, sine and cosine, four products: under 64 roundings);
- gradients: the same against the largest of |g|, |dx| of the head; weight gradients 2^-16 of the sum of
  the magnitudes of their terms;
- attention: u |o| for the rounding, u sum p |v| / sum p for probabilities of 16 bits, and 2^-14 of the
  same for fp32 scores (|s| < 2^6, each a sum of at most 256 products) in the exponent;
- lse: 2^-14 absolute (the error of a score).
Plans and copies are equal.
"""
import numpy as np
import pytest

from tests import backbone_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_12287_gb300 as p
    p.load()
    return p


def dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(getattr(torch, dtype))


def i32(a):
    return dev(np.asarray(a, np.int32))


def host(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------- plan

def plan_case(r, n, page, most_new, tree, cols=40, spare=6):
    new = r.integers(0, most_new + 1, n)
    base = r.integers(0, page * cols - most_new + 1, n)
    held = np.clip(base + r.integers(-2 * page, 2 * page + 1, n), 0, page * cols)
    done = r.random(n) < 0.2
    base, new = np.where(done, 0, base), np.where(done, 0, new)
    have = -(-held // page)
    need = -(-(base + new) // page)
    places = int(np.maximum(have, need).sum()) + spare
    ids = r.permutation(places)
    table = np.full((n, cols), -1, np.int64)
    used = 0
    for i in range(n):
        table[i, :have[i]] = ids[used:used + have[i]]
        used += have[i]
    head = int(r.integers(0, places))
    ring = np.full(places, -7, np.int64)
    ring[(head + np.arange(places - used)) % places] = ids[used:]
    rows = int(new.sum())
    parent = None
    if tree:
        parent = np.concatenate([[r.integers(-1, max(1, j)) for j in range(m)] for m in new] + [[]]).astype(np.int64)
    return dict(held=held, base=base, new=new, parent=parent, ring=ring, ring_in=[head, places - used], table=table,
                page=page, rows=rows)


def run_plan(pkg, c, max_rows, words, optional=True):
    import torch
    n, cols = c["table"].shape
    cfg = pkg.make_plan_config(n, max_rows, cols, c["page"], len(c["ring"]), words)
    out = lambda *shape: torch.full(shape, -77, dtype=torch.int32, device="cuda")
    ring, table = i32(c["ring"]), i32(c["table"])
    parent = c["parent"]
    if parent is not None:
        parent = i32(np.concatenate([parent, np.zeros(max_rows - len(parent) if max_rows > len(parent) else 0)]))
    res = dict(cu=out(n + 1), req=out(max_rows), slot=out(max_rows), pos=out(max_rows), mask=out(max_rows, words),
               ring=ring, ring_out=out(2), table=table, status=out(1))
    opt = lambda name: res[name] if optional else None
    pkg.ivit_step_plan(cfg, i32(c["held"]), i32(c["base"]), i32(c["new"]), parent, ring, i32(c["ring_in"]), table, res["cu"],
                       opt("req"), res["slot"], opt("pos"), opt("mask") if words else None, res["ring_out"], res["status"])
    want = ref.step_plan(c["held"], c["base"], c["new"], c["parent"], c["ring"], c["ring_in"], c["table"], c["page"],
                         max_rows, words)
    for name, w in zip(("cu", "req", "slot", "pos", "mask", "ring", "ring_out", "table"), want):
        if not optional and name in ("req", "pos", "mask"):
            continue
        w = w.view(np.int32) if w.dtype == np.uint32 else w
        np.testing.assert_array_equal(res[name].cpu().numpy(), w, err_msg=name)
    assert int(res["status"]) == want[-1]
    return want[-1]


@pytest.mark.parametrize("n,page,most_new,tree,words", [
    (1, 16, 1, False, 0), (1, 1, 5, True, 1), (7, 16, 9, True, 1), (33, 8, 70, True, 3), (5, 4, 70, True, 2),
    (600, 32, 12, True, 1), (1100, 16, 3, False, 1), (40, 64, 300, False, 10), (4096, 16, 2, False, 0),
])
def test_step_plan(pkg, n, page, most_new, tree, words):
    r = np.random.default_rng(n * 100 + page)
    c = plan_case(r, n, page, most_new, tree)
    assert run_plan(pkg, c, c["rows"], words) == 0
    assert run_plan(pkg, c, c["rows"] + 13, words) == 0      # rows past the step's
    assert run_plan(pkg, c, c["rows"], words, optional=False) == 0


def test_step_plan_of_long_prompts(pkg):
    # one request's pages and rows span many CTAs
    r = np.random.default_rng(3)
    c = plan_case(r, 3, 16, 1, False, cols=1000)
    places = 3000
    c.update(held=np.array([0, 16000, 5]), base=np.array([0, 0, 5]), new=np.array([15999, 0, 7001]),
             ring=r.permutation(places), ring_in=[2500, 2000], rows=23000)
    c["table"][1] = 10000 + np.arange(1000)
    c["table"][2, 0] = 17
    assert run_plan(pkg, c, 23000, 0) == 0


def test_step_plan_is_the_same_when_repeated(pkg):
    import torch
    c = plan_case(np.random.default_rng(9), 50, 16, 20, True)
    n, cols = c["table"].shape
    cfg = pkg.make_plan_config(n, c["rows"], cols, 16, len(c["ring"]), 1)
    out = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    ring, table, ins = i32(c["ring"]), i32(c["table"]), [i32(c[k]) for k in ("held", "base", "new", "parent")]
    res = [out(n + 1), out(c["rows"]), out(c["rows"]), out(c["rows"]), out(c["rows"], 1), out(2), out(1)]
    seen = []
    for _ in range(2):
        pkg.ivit_step_plan(cfg, *ins, ring, i32(c["ring_in"]), table, *res)
        seen.append([t.cpu().numpy().copy() for t in res + [ring, table]])
    for a, b in zip(*seen):
        np.testing.assert_array_equal(a, b)


def test_step_plan_refuses_what_it_cannot_grant(pkg):
    r = np.random.default_rng(5)
    c = plan_case(r, 20, 16, 9, True)
    few = dict(c, ring_in=[c["ring_in"][0], 0], held=np.minimum(c["held"], c["base"]))
    assert run_plan(pkg, few, c["rows"], 1) & 1
    assert run_plan(pkg, c, c["rows"] - 1, 1) == 4
    assert run_plan(pkg, dict(c, base=np.where(np.arange(20) == 3, 16 * 40, c["base"]), new=np.maximum(c["new"], 1)),
                    c["rows"] + 20, 1) & 2
    assert run_plan(pkg, dict(c, base=np.where(np.arange(20) == 3, -1, c["base"])), c["rows"], 1) == 8
    assert run_plan(pkg, dict(c, new=np.where(np.arange(20) == 3, 2 ** 31 - 1, c["new"])), c["rows"], 1) & 6
    assert run_plan(pkg, dict(c, ring_in=[len(c["ring"]), 1]), c["rows"], 1) == 8
    assert run_plan(pkg, dict(c, ring_in=[0, -1]), c["rows"], 1) == 8


# --------------------------------------------------------------------- rotation

def rope_case(r, rows, heads, kv, dim, rot, axes, dtype, weights, most_pos=2000):
    half = rot // 2
    freq = (10000.0 ** (-np.arange(half) / max(1, half))).astype(np.float32)
    axis = np.arange(half) % axes
    pos = r.integers(-5, most_pos, (axes, rows))
    qkv = dev(r.standard_normal((rows, (heads + 2 * kv) * dim)).astype(np.float32) * 1.5, dtype)
    part = lambda lo, m: qkv[:, lo * dim:(lo + m) * dim].unflatten(1, (m, dim))
    w = [dev((1 + 0.3 * r.standard_normal(dim)).astype(np.float32), dtype) if x in weights else None for x in "qk"]
    return dict(q=part(0, heads), k=part(heads, kv), v=part(heads + kv, kv), w=w, pos=pos, freq=freq, axis=axis)


def close_rotation(got, want, x, dtype, what):
    err = np.abs(host(got) - want)
    scale = np.maximum(np.abs(x).max(-1, keepdims=True), np.abs(want).max(-1, keepdims=True))
    bound = ref.UNIT[dtype] * np.abs(want) + 2.0 ** -18 * scale + 2.0 ** -25
    assert (err <= bound).all(), f"{what}: {np.max(err / bound)} of the bound"


ROPE = [  # rows, heads, kv, dim, rot, axes, interleaved, weights, type
    (1, 32, 8, 128, 128, 1, False, "qk", "bfloat16"), (7, 16, 16, 72, 72, 3, False, "qk", "bfloat16"),
    (5, 3, 1, 8, 8, 1, True, "qk", "float16"), (130, 6, 2, 64, 32, 2, True, "q", "float16"),
    (33, 5, 5, 80, 40, 3, False, "k", "bfloat16"), (9, 4, 2, 256, 256, 4, True, "", "bfloat16"),
    (2, 1, 1, 136, 0, 1, False, "qk", "float16"), (5000, 8, 2, 96, 96, 3, False, "qk", "bfloat16"),
    (1300, 7, 1, 248, 128, 1, False, "qk", "float16"),
]


@pytest.mark.parametrize("rows,heads,kv,dim,rot,axes,inter,weights,dtype", ROPE)
def test_qk_norm_rope(pkg, rows, heads, kv, dim, rot, axes, inter, weights, dtype):
    import torch
    r = np.random.default_rng(rows + dim)
    c = rope_case(r, rows, heads, kv, dim, rot, axes, dtype, weights)
    cfg = pkg.make_rope_config(heads, kv, dim, rot, axes, inter, 1e-5, dtype)
    page = 8
    pages = -(-rows // page) + 2
    # a cache with the heads outside the tokens, some rows without a slot
    kc, vc = (torch.full((pages, kv, page, dim), 3.0, dtype=c["q"].dtype, device="cuda").transpose(1, 2) for _ in range(2))
    slots = r.permutation(pages * page)[:rows].astype(np.int64)
    slots[::5] = -1
    if rows > 6:
        slots[6] = pages * page  # past the cache
    q_out = torch.empty((rows, heads, dim), dtype=c["q"].dtype, device="cuda")
    k_out = torch.empty((rows, kv, dim), dtype=c["q"].dtype, device="cuda")
    freq, axis = (dev(c["freq"]), i32(c["axis"])) if rot else (None, None)
    pkg.ivit_qk_norm_rope(cfg, c["q"], c["k"], c["v"], *c["w"], i32(c["pos"]), freq, axis, q_out, k_out,
                          pkg.make_cache_layout(kc), kc, vc, i32(slots))
    wants = []
    for x, w, out, name in ((c["q"], c["w"][0], q_out, "q"), (c["k"], c["w"][1], k_out, "k")):
        want = ref.rope(host(x), None if w is None else host(w), c["pos"], c["freq"], c["axis"], rot, inter, 1e-5)
        close_rotation(out, want, host(x), dtype, name)
        wants.append(want)
    # the caches hold the same keys and the values as they are, and nothing else has changed
    put = (slots >= 0) & (slots < pages * page)
    for cache, rows_of in ((kc, k_out), (vc, c["v"])):
        want = torch.full((pages * page, kv, dim), 3.0, dtype=cache.dtype, device="cuda")
        want[torch.from_numpy(slots[put]).cuda()] = rows_of[torch.from_numpy(put).cuda()]
        assert torch.equal(cache.reshape(pages * page, kv, dim), want)
    # in place, without a cache
    q2, k2 = c["q"], c["k"]
    pkg.ivit_qk_norm_rope(cfg, q2, k2, None, *c["w"], i32(c["pos"]), freq, axis, q2, k2)
    assert torch.equal(q2, q_out) and torch.equal(k2, k_out)


def test_rope_keeps_the_angle_of_large_positions(pkg):
    import torch
    dim, pos = 64, np.array([[0, 1, 2 ** 24, 2 ** 24 - 1, 10 ** 7 + 1, -2 ** 24, 1234567]])
    freq = (10000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    x = np.random.default_rng(1).standard_normal((7, 2, dim)).astype(np.float32)
    q, k = dev(x[:, :1], "float16"), dev(x[:, 1:], "float16")
    out, kout = torch.empty_like(q), torch.empty_like(k)
    pkg.ivit_qk_norm_rope(pkg.make_rope_config(1, 1, dim, dtype="float16"), q, k, None, None, None, i32(pos), dev(freq),
                          i32(np.zeros(32)), out, kout)
    want = ref.rope(host(q), None, pos, freq, np.zeros(32, int), dim, False, 0)
    close_rotation(out, want, host(q), "float16", "q")


@pytest.mark.parametrize("rows,heads,kv,dim,rot,axes,inter,weights,dtype", ROPE)
def test_qk_norm_rope_backward(pkg, rows, heads, kv, dim, rot, axes, inter, weights, dtype):
    import torch
    r = np.random.default_rng(rows + dim + 1)
    c = rope_case(r, rows, heads, kv, dim, rot, axes, dtype, weights)
    cfg = pkg.make_rope_config(heads, kv, dim, rot, axes, inter, 1e-5, dtype)
    g = [dev(r.standard_normal((rows, m, dim)).astype(np.float32), dtype) for m in (heads, kv)]
    dqk = torch.full((rows, (heads + kv) * dim), float("nan"), dtype=c["q"].dtype, device="cuda")
    d = [dqk[:, :heads * dim].unflatten(1, (heads, dim)), dqk[:, heads * dim:].unflatten(1, (kv, dim))]
    dw = [torch.full((dim,), float("nan"), device="cuda") if x in weights else None for x in "qk"]
    ws = torch.full((pkg.ivit_qk_norm_rope_backward_workspace(cfg),), 255, dtype=torch.uint8, device="cuda")
    freq, axis = (dev(c["freq"]), i32(c["axis"])) if rot else (None, None)
    call = lambda outs, dws: pkg.ivit_qk_norm_rope_backward(cfg, *g, c["q"], c["k"], *c["w"], i32(c["pos"]), freq, axis,
                                                            *outs, *dws, ws)
    call(d, dw)
    for x, w, gx, dx, dwx, name in zip((c["q"], c["k"]), c["w"], g, d, dw, "qk"):
        xs, gs = host(x), host(gx)
        want, want_w = ref.rope_backward(gs, xs, None if w is None else host(w), c["pos"], c["freq"], c["axis"], rot, inter, 1e-5)
        rms = np.sqrt((xs ** 2).mean(-1, keepdims=True) + 1e-5) if w is not None else 1.0
        close_rotation(dx, want, np.maximum(np.abs(gs), 2 * np.abs(gs) / rms), dtype, "d" + name)
        if w is not None:
            y = ref.rope(gs, None, -c["pos"], c["freq"], c["axis"], rot, inter, 0)
            size = np.abs(y * xs / rms).sum((0, 1))
            assert (np.abs(host(dwx) - want_w) <= 2.0 ** -16 * size + 1e-6).all(), name
    # the same sums again, and in place
    first = [t.clone() for t in dw if t is not None]
    kept = [t.clone() for t in d]
    call([g[0], g[1]], dw)
    assert all(torch.equal(a, b) for a, b in zip(first, [t for t in dw if t is not None]))
    assert torch.equal(g[0], kept[0]) and torch.equal(g[1], kept[1])


def test_rope_gradient_against_differences(pkg):
    # d(sum(g * y)) along a random direction, from differences of the 64-bit forward pass
    import torch
    r = np.random.default_rng(8)
    rows, heads, kv, dim, rot = 6, 3, 1, 64, 32
    c = rope_case(r, rows, heads, kv, dim, rot, 2, "float16", "qk")
    cfg = pkg.make_rope_config(heads, kv, dim, rot, 2, False, 1e-5, "float16")
    g = [dev(r.standard_normal((rows, m, dim)).astype(np.float32), "float16") for m in (heads, kv)]
    d = [torch.empty_like(t) for t in g]
    dw = [torch.empty(dim, device="cuda") for _ in range(2)]
    ws = torch.empty(pkg.ivit_qk_norm_rope_backward_workspace(cfg), dtype=torch.uint8, device="cuda")
    pkg.ivit_qk_norm_rope_backward(cfg, *g, c["q"], c["k"], *c["w"], i32(c["pos"]), dev(c["freq"]), i32(c["axis"]), *d, *dw, ws)
    for x, w, gx, dx, dwx in zip((c["q"], c["k"]), c["w"], g, d, dw):
        xs, wv, gs = host(x), host(w), host(gx)
        loss = lambda a, b: (gs * ref.rope(a, b, c["pos"], c["freq"], c["axis"], rot, False, 1e-5)).sum()
        tx, tw, h = r.standard_normal(xs.shape), r.standard_normal(dim), 1e-5
        for got, terms, diff in (
                ((host(dx) * tx).sum(), np.abs(host(dx) * tx).sum(), (loss(xs + h * tx, wv) - loss(xs - h * tx, wv)) / (2 * h)),
                ((host(dwx) * tw).sum(), np.abs(host(dwx) * tw).sum(), (loss(xs, wv + h * tw) - loss(xs, wv - h * tw)) / (2 * h))):
            # the rounding of dx to 16 bits, term by term, and the differences' own error (h^2 and 2^-52 / h)
            assert abs(got - diff) <= 2.0 ** -11 * terms + 1e-6 * terms + 1e-6


def test_rope_of_no_rows(pkg):
    import torch
    cfg = pkg.make_rope_config(4, 2, 64)
    e = lambda m: torch.empty((0, m, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    f, a, p = torch.ones(32, device="cuda"), i32(np.zeros(32)), i32(np.zeros(0))
    pkg.ivit_qk_norm_rope(cfg, e(4), e(2), None, w, w, p, f, a, e(4), e(2))
    dw = [torch.full((64,), float("nan"), device="cuda") for _ in range(2)]
    ws = torch.empty(pkg.ivit_qk_norm_rope_backward_workspace(cfg), dtype=torch.uint8, device="cuda")
    pkg.ivit_qk_norm_rope_backward(cfg, e(4), e(2), e(4), e(2), w, w, p, f, a, e(4), e(2), *dw, ws)
    assert all(bool((t == 0).all()) for t in dw)


# -------------------------------------------------------------------- attention

def attention_case(r, lengths, new, heads, kv, dim, page, dtype, order="token", spread=1.0):
    n, rows = len(lengths), int(np.sum(new))
    need = [-(-int(x) // page) for x in lengths]
    pages = sum(need) + 3
    ids, used = r.permutation(pages), 0
    table = np.full((n, max(need + [0]) + 2), -1, np.int64)
    for i, m in enumerate(need):
        table[i, :m] = ids[used:used + m]
        used += m
    shape = (pages, page, kv, dim) if order == "token" else (pages, kv, page, dim)
    cache = [dev(r.standard_normal(shape).astype(np.float32) * s, dtype) for s in (spread, 1.0)]
    if order == "head":
        cache = [c.transpose(1, 2) for c in cache]
    # (what lies in the pages past a request's tokens must not matter)
    for i, m in enumerate(lengths):
        if m % page:
            for c in cache:
                c[table[i, m // page], m % page:] = float("nan")
    qkv = dev(r.standard_normal((rows, (heads + 2 * kv) * dim)).astype(np.float32), dtype)
    part = lambda lo, m: qkv[:, lo * dim:(lo + m) * dim].unflatten(1, (m, dim))
    return dict(q=part(0, heads), k=part(heads, kv), v=part(heads + kv, kv), kc=cache[0], vc=cache[1], table=table,
                lengths=np.asarray(lengths), cu=np.concatenate([[0], np.cumsum(new)]).astype(np.int64), dtype=dtype)


def run_attention(pkg, c, mask, vis=None, lse=True, check=True, scale=None, max_new=None, mask_words=None):
    import torch
    rows, heads, dim = c["q"].shape
    new = np.diff(c["cu"])
    most = int(new.max()) if max_new is None else max_new
    words = (most + 31) // 32 if mask_words is None else mask_words
    scale = dim ** -0.5 if scale is None else scale
    packed = None
    if mask == "tree":
        packed = np.concatenate([ref.words(vis[i], words) for i in range(len(new))])
        packed = dev(packed)
    lay = pkg.make_cache_layout(c["kc"])
    cfg = pkg.make_attention_config(len(new), heads, c["table"].shape[1], most, mask, words if mask == "tree" else 0, scale)
    out = torch.full((rows, heads, dim), float("nan"), dtype=c["q"].dtype, device="cuda")
    got_lse = torch.full((rows, heads), float("nan"), device="cuda") if lse else None
    ws = torch.full((pkg.ivit_tree_attention_workspace(cfg, lay),), 255, dtype=torch.uint8, device="cuda")
    pkg.ivit_tree_attention(cfg, lay, c["q"], c["k"], c["v"], c["kc"], c["vc"], i32(c["table"]), i32(c["lengths"]), i32(c["cu"]),
                            packed, out, got_lse, ws)
    assert int(ws[:4].view(torch.int32)) == 0  # no wait of the kernel expired
    if not check:
        return out, got_lse
    sees = {"causal": lambda i, n: np.tril(np.ones((n, n), bool)), "all": lambda i, n: np.ones((n, n), bool),
            "tree": lambda i, n: vis[i]}[mask]
    want, want_lse, size = ref.attention(host(c["q"]), host(c["k"]), host(c["v"]), host(c["kc"]), host(c["vc"]), c["table"],
                                         c["lengths"], c["cu"], sees, scale)
    u = ref.UNIT[c["dtype"]]
    bound = u * np.abs(want) + (u + 2.0 ** -14) * size + 2.0 ** -25
    err = np.abs(host(out) - want)
    assert (err <= bound).all(), f"{np.nanmax(err / bound)} of the bound, {np.isnan(host(out)).sum()} NaN"
    if lse:
        got = host(got_lse)
        none = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got), none)
        assert (np.abs(got[~none] - want_lse[~none]) <= 2.0 ** -14).all()
    return out, got_lse


def trees(r, new):
    return [ref.ancestors([int(r.integers(-1 if j == 0 else max(0, j - 6), max(1, j))) if j else -1 for j in range(n)]) for n in new]


ATTENTION = [  # cached, new, heads, kv, dim, page, type, order
    ([0], [1], 4, 4, 64, 16, "bfloat16", "token"), ([1], [1], 8, 2, 64, 16, "float16", "token"),
    ([63], [1], 1, 1, 64, 8, "bfloat16", "token"), ([64], [1], 16, 4, 128, 16, "bfloat16", "head"),
    ([130, 0, 65, 700], [1, 3, 0, 9], 8, 2, 72, 16, "bfloat16", "token"),
    ([5, 64, 127, 128, 129], [2, 1, 64, 63, 65], 4, 2, 80, 1, "float16", "head"),
    ([1500], [31], 8, 1, 128, 64, "float16", "token"), ([40, 900, 33], [12, 1, 40], 14, 2, 96, 32, "bfloat16", "token"),
    ([100, 300], [17, 5], 5, 1, 256, 128, "float16", "head"), ([257], [3], 2, 2, 256, 16, "bfloat16", "token"),
    ([90, 10], [70, 130], 3, 3, 40, 16, "bfloat16", "token"), ([2000, 3, 777], [4, 4, 4], 8, 8, 8, 1024, "float16", "token"),
    ([33], [7], 32, 1, 200, 4, "bfloat16", "head"),
    # many rows per key head: tcgen05 tiles, last blocks of every kind, groups that do not divide 128
    ([300, 95, 96, 97, 0], [65, 96, 20, 1, 130], 8, 4, 72, 8, "bfloat16", "token"),
    ([191, 192, 500], [128, 33, 97], 5, 1, 80, 128, "float16", "head"), ([700], [256], 2, 2, 64, 64, "bfloat16", "token"),
    ([0, 0, 127, 128, 129], [140, 3, 128, 129, 70], 2, 2, 64, 16, "float16", "token"),
    ([0, 64, 200], [75, 64, 1], 7, 1, 128, 16, "bfloat16", "token"), ([500], [65], 6, 2, 112, 256, "bfloat16", "head"),
    ([300, 96], [50, 129], 2, 2, 88, 16, "bfloat16", "head"),
    # ... of heads above 128, whose last slices may be empty
    ([63, 64, 65, 500], [40, 1, 64, 20], 5, 1, 136, 16, "bfloat16", "token"), ([200, 0], [130, 17], 2, 2, 192, 32, "float16", "head"),
    ([300, 128, 1], [129, 256, 9], 4, 2, 256, 8, "bfloat16", "token"), ([900], [20], 32, 2, 256, 512, "bfloat16", "head"),
    # what tcgen05 does not take (small pages): tiles of 16, 32, 64 and 128 rows
    ([90, 65], [30, 2], 1, 1, 256, 4, "bfloat16", "token"), ([90, 65], [60, 2], 1, 1, 256, 2, "float16", "head"),
    ([129], [100], 1, 1, 200, 4, "bfloat16", "token"),
    ([64, 128], [16, 7], 1, 1, 80, 4, "bfloat16", "token"), ([70, 200], [20, 9], 2, 2, 64, 4, "bfloat16", "token"),
    ([70, 0, 130], [50, 3, 1], 1, 1, 128, 2, "float16", "token"), ([66], [12], 8, 4, 96, 4, "bfloat16", "token"),
    ([300, 40], [40, 17], 1, 1, 96, 1, "float16", "head"), ([90, 65], [30, 2], 1, 1, 256, 16, "bfloat16", "token"),
    ([90, 65], [60, 2], 1, 1, 256, 8, "float16", "head"), ([129], [100], 2, 1, 128, 4, "bfloat16", "token"),
]


@pytest.mark.parametrize("lengths,new,heads,kv,dim,page,dtype,order", ATTENTION)
@pytest.mark.parametrize("mask", ["causal", "all", "tree"])
def test_tree_attention(pkg, lengths, new, heads, kv, dim, page, dtype, order, mask):
    r = np.random.default_rng(sum(lengths) + sum(new) + dim)
    c = attention_case(r, lengths, new, heads, kv, dim, page, dtype, order)
    run_attention(pkg, c, mask, trees(r, new) if mask == "tree" else None)


@pytest.mark.parametrize("dim,most_new,n", [(64, 2, 700), (72, 2, 700), (40, 2, 700), (96, 2, 500), (256, 2, 300), (72, 20, 200),
                                            (96, 70, 40), (256, 20, 150)])
def test_many_short_requests(pkg, dim, most_new, n):
    # every CTA goes through several tiles of rows
    r = np.random.default_rng(2)
    lengths, new = r.integers(0, 90, n), r.integers(0, most_new + 1, n)
    c = attention_case(r, lengths, new, 6, 3, dim, 8, "bfloat16")
    run_attention(pkg, c, "causal", lse=False)


def test_rows_that_see_nothing(pkg):
    r = np.random.default_rng(4)
    new = [5, 40, 3]
    vis = [np.zeros((n, n), bool) for n in new]
    vis[1][7, 3] = vis[1][39, 0] = vis[1][39, 39] = True
    for lengths in ([0, 0, 0], [0, 0, 90]):
        c = attention_case(r, lengths, new, 4, 2, 64, 16, "bfloat16")
        out, lse = run_attention(pkg, c, "tree", vis)
        assert float(out[:5].abs().max()) == 0 and float(lse[:5].max()) == -np.inf


@pytest.mark.parametrize("new,page,dim", [(4, 16, 64), (20, 16, 64), (100, 16, 64), (4, 4, 64), (10, 4, 64), (20, 4, 64), (100, 4, 64),
                                          (4, 16, 256), (30, 16, 256), (60, 8, 128), (90, 8, 80), (30, 4, 256), (70, 8, 192), (50, 16, 96)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_does_not_see_does_not_reach_it(pkg, new, page, dim, bad):
    import torch
    r = np.random.default_rng(new)
    c = attention_case(r, [70], [new], 4, 2, dim, page, "float16")
    vis = [np.tril(np.ones((new, new), bool))]
    vis[0][:, 2] = False
    vis[0][new - 1, 2] = True          # only the last row sees draft 2
    clean, clean_lse = run_attention(pkg, c, "tree", vis)
    c["v"][2, 1, 5] = bad              # one value of one head
    c["k"][3] = c["k"][3]              # (its key is as it was)
    out, lse = run_attention(pkg, c, "tree", vis, check=False)
    assert torch.equal(lse, clean_lse)
    others = torch.ones(new, 4, dim, dtype=torch.bool)
    others[new - 1, 2:, 5] = False     # (query heads 2 and 3 read key head 1)
    assert torch.equal(out.cpu()[others], clean.cpu()[others])
    hit = out[new - 1, 2:, 5].float().cpu().numpy()
    assert np.isnan(hit).all() if np.isnan(bad) else np.array_equal(hit, [bad, bad])
    # a key that no other row sees
    c["v"][2, 1, 5] = 0.5
    c["k"][2] = bad
    out, lse = run_attention(pkg, c, "tree", vis, check=False)
    assert torch.equal(out[:new - 1], clean[:new - 1]) and torch.equal(lse[:new - 1], clean_lse[:new - 1])


def test_large_scores_and_growing_maximum(pkg):
    # scores up to a few hundred that grow along the keys: the running maximum moves in every tile
    r = np.random.default_rng(6)
    c = attention_case(r, [1000, 640], [2, 33], 4, 1, 64, 16, "float16", spread=1.0)
    grow = dev(np.linspace(0.01, 4.0, 1000).astype(np.float32), "float16")
    t = np.arange(1000)
    c["kc"][i32(c["table"][0][t // 16]).long(), i32(t % 16).long()] = c["q"][0, :1] * grow[:, None, None]
    run_attention(pkg, c, "causal", scale=0.125)


@pytest.mark.parametrize("group", [1, 8])
def test_offsets_past_32_bits(pkg, group):
    # pages at the far end of a cache of more than 2^32 elements
    import torch
    page, kv, dim = 16, 8, 128
    pages = (1 << 32) // (page * kv * dim) + 64
    r = np.random.default_rng(7)
    if torch.cuda.mem_get_info()[0] < 5 * pages * page * kv * dim:
        pytest.skip("needs 22 GB of device memory")
    c = attention_case(r, [300], [3], 8 * group, 8, dim, page, "bfloat16")
    small = [c["kc"], c["vc"]]
    far = (pages - 1 - np.arange(small[0].shape[0])).astype(np.int64)
    big = torch.empty((pages, page, kv, dim), dtype=torch.bfloat16, device="cuda")
    lay = pkg.make_cache_layout(big)
    # (one array holds both: keys in the last pages, values below them)
    near = far - 2 * len(far)
    fi, ni = torch.from_numpy(far).cuda(), torch.from_numpy(near).cuda()
    big[fi], big[ni] = small[0], small[1]
    want, _ = run_attention(pkg, c, "causal")
    used = c["table"] >= 0
    far_table = np.where(used, far[np.maximum(c["table"], 0)], -1)
    cfg = pkg.make_attention_config(1, 8 * group, far_table.shape[1], 3, "causal", 0, dim ** -0.5)
    ws = torch.empty(pkg.ivit_tree_attention_workspace(cfg, lay), dtype=torch.uint8, device="cuda")
    out = torch.empty((3, 8 * group, dim), dtype=torch.bfloat16, device="cuda")
    # values: the same table over a view that begins 2 * len(far) pages lower
    k_far = big[2 * len(far):]
    lay2 = pkg.make_cache_layout(k_far)
    table2 = np.where(used, far_table - 2 * len(far), -1)
    pkg.ivit_tree_attention(cfg, lay2, c["q"], c["k"], c["v"], k_far, big[:pages - 2 * len(far)], i32(table2), i32(c["lengths"]),
                            i32(c["cu"]), None, out, None, ws)
    assert torch.equal(out, want)
    # and the write that would have put them there
    src = torch.randn((1, 2, kv, dim), device="cuda").to(torch.bfloat16)
    slots = i32([pages * page - 1, pages * page - 5])
    pkg.ivit_kv_write(lay, src, src, i32([1, 0]), slots, big[None], big[None])
    assert torch.equal(big[-1, 15], src[0, 1]) and torch.equal(big[-1, 11], src[0, 0])


def test_on_another_stream_and_in_a_graph(pkg):
    import torch
    r = np.random.default_rng(10)
    c = attention_case(r, [500, 20], [1, 6], 8, 2, 64, 16, "bfloat16")
    want, want_lse = run_attention(pkg, c, "causal")
    lay = pkg.make_cache_layout(c["kc"])
    cfg = pkg.make_attention_config(2, 8, c["table"].shape[1], 6, "causal", 0, 64 ** -0.5)
    ws = torch.empty(pkg.ivit_tree_attention_workspace(cfg, lay), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(want), torch.empty_like(want_lse)
    args = [c["kc"], c["vc"], i32(c["table"]), i32(c["lengths"]), i32(c["cu"]), None, out, lse, ws]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pkg.ivit_tree_attention(cfg, lay, c["q"], c["k"], c["v"], *args)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.ivit_tree_attention(cfg, lay, c["q"], c["k"], c["v"], *args)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


# ------------------------------------------------------------------------ write

@pytest.mark.parametrize("layers,n,drafts,kv,dim,page,dtype,order", [
    (1, 1, 1, 1, 8, 1, "bfloat16", "token"), (27, 5, 9, 4, 64, 16, "bfloat16", "token"), (3, 70, 100, 2, 72, 8, "float16", "head"),
    (2, 33, 33, 8, 256, 64, "bfloat16", "head"),
])
def test_kv_write(pkg, layers, n, drafts, kv, dim, page, dtype, order):
    import torch
    r = np.random.default_rng(n + dim)
    # rows of a projection's output: keys and values beside each other
    src = dev(r.standard_normal((layers, drafts, 2 * kv * dim)).astype(np.float32), dtype)
    k, v = src[..., :kv * dim].unflatten(2, (kv, dim)), src[..., kv * dim:].unflatten(2, (kv, dim))
    pages = -(-n // page) + 2
    shape = (layers, pages, page, kv, dim) if order == "token" else (layers, pages, kv, page, dim)
    kc, vc = (torch.full(shape, 2.0, dtype=src.dtype, device="cuda") for _ in range(2))
    if order == "head":
        kc, vc = kc.transpose(2, 3), vc.transpose(2, 3)
    rows, slots = r.permutation(drafts)[:n], r.permutation(pages * page)[:n]
    if n > 4:
        rows[1], slots[2], slots[3], rows[4] = -1, -1, pages * page, drafts
    pkg.ivit_kv_write(pkg.make_cache_layout(kc[0]), k, v, i32(rows), i32(slots), kc, vc)
    ok = (rows >= 0) & (rows < drafts) & (slots >= 0) & (slots < pages * page)
    for cache, x in ((kc, k), (vc, v)):
        want = torch.full((layers, pages * page, kv, dim), 2.0, dtype=src.dtype, device="cuda")
        want[:, torch.from_numpy(slots[ok]).cuda()] = x[:, torch.from_numpy(rows[ok]).cuda()]
        assert torch.equal(cache.reshape(layers, pages * page, kv, dim), want)
