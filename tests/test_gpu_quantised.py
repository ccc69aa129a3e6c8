"""GPU parity of the 8-bit cache's operators and of the verification of drafts against their 64-bit restatement.

Writes are equal, code by code and scale by scale (powers of two make every step but the last rounding exact).  Reads: one
rounding, u |x| with u half a unit in the last place (2^-8 bf16, 2^-11 fp16; 2^-25 below fp16's normal range).  Attention,
per value: u |o| for the rounding, u sum p |v| / sum p for probabilities of 16 bits, and 2^-14 of the same for fp32 scores
(|s| < 2^6, each a sum of at most 256 products) in the exponent; lse 2^-14.  Verification: equal, where no decision is nearer than
2^-16 to its border (fp32 sums of up to 2^17 exponentials, in trees, and products of a few roundings; exponentials of
arguments up to 2^6).
"""
import numpy as np
import pytest

from tests import backbone_ref, quantised_ref as ref
from tests.test_gpu_backbone import dev, host, i32, trees

pytestmark = pytest.mark.gpu

UNIT = backbone_ref.UNIT


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_12287_gb300 as p
    p.load()
    return p


def codes_on_gpu(codes, order="token"):
    """uint8 codes [..., page, heads, dim] as a float8 tensor, whose heads lie in front of the tokens in memory if order is "head"."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(codes)).cuda()
    if order == "head":
        t = t.transpose(-3, -2).contiguous().transpose(-3, -2)
    return t.view(torch.float8_e4m3fn)


def codes_of(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def random_cache(r, lead, page, kv, dim, block, spread=(-9, -4)):
    """Codes and scales as writing leaves them."""
    codes = ref.encode(np.clip(r.standard_normal((*lead, page, kv, dim)) * 90, -448, 448))
    return codes, 2.0 ** r.integers(spread[0], spread[1], (*lead, page // block, kv)).astype(np.float32)


# ---------------------------------------------------------------- writing, reading

WRITES = [  # layers, requests' (cached, new) tokens, heads, dim, page, block, type, order
    (1, [(0, 1)], 1, 8, 1, 1, "bfloat16", "token"), (27, [(5, 1), (16, 1), (31, 1)], 4, 64, 16, 16, "bfloat16", "token"),
    (2, [(0, 70), (3, 13), (40, 25)], 2, 72, 8, 4, "float16", "head"), (3, [(7, 100)], 3, 256, 64, 32, "bfloat16", "token"),
    (2, [(1, 3), (2, 1), (3, 5), (15, 2)], 8, 128, 16, 8, "float16", "token"), (1, [(600, 1300)], 2, 40, 1024, 1024, "bfloat16", "token"),
    (2, [(0, 33)], 5, 104, 32, 1, "bfloat16", "head"), (1, [(9, 200), (100, 300)], 1, 16, 128, 128, "float16", "token"),
    (6, [(3 * i, 1 + i % 6) for i in range(60)], 8, 80, 32, 16, "bfloat16", "token"),
]


def write_case(r, layers, requests, kv, dim, page, block, dtype, order):
    slots, used, pages = [], 0, sum(-(-(b + n) // page) for b, n in requests) + 2
    ids = r.permutation(pages)
    for b, n in requests:
        t = np.arange(b, b + n)
        slots.append(ids[used + t // page] * page + t % page)
        used += -(-(b + n) // page)
    slots = np.concatenate(slots)
    n = len(slots)
    drafts = n + 4
    src = dev(r.standard_normal((layers, drafts, 2 * kv * dim)).astype(np.float32)
              * 2.0 ** r.integers(-6, 7, (layers, drafts, 1)).astype(np.float32), dtype)
    k, v = src[..., :kv * dim].unflatten(2, (kv, dim)), src[..., kv * dim:].unflatten(2, (kv, dim))
    rows = r.permutation(drafts)[:n]
    caches = [random_cache(r, (layers, pages), page, kv, dim, block) for _ in range(2)]
    return k, v, rows, slots, caches


def check_write(pkg, k, v, rows, slots, caches, block, dtype, order, repeat=2):
    import torch
    layers, pages, page = caches[0][0].shape[:3]
    kc, vc = (codes_on_gpu(c, order) for c, _ in caches)
    ks, vs = (dev(s) for _, s in caches)
    lay = pkg.make_quantised_layout(kc[0], block, dtype)
    ok = (rows >= 0) & (rows < k.shape[1])
    want = []
    for x, (c, s) in zip((k, v), caches):
        c, s, x = c.copy(), s.copy(), host(x)
        for layer in range(layers):
            ref.quantise(c[layer], s[layer], [x[layer, i] if o else None for i, o in zip(rows, ok)], slots, block)
        want.append((c, s))
    for _ in range(repeat):
        pkg.ivit_kv_quantise(lay, k, v, i32(rows), i32(slots), kc, vc, ks, vs)
        for (c, s), got_c, got_s in zip(want, (kc, vc), (ks, vs)):
            assert np.array_equal(host(got_s), s, equal_nan=True)  # (NaN: blocks that were not written)
            assert np.array_equal(codes_of(got_c), c)
    return kc, vc, ks, vs, lay


@pytest.mark.parametrize("layers,requests,kv,dim,page,block,dtype,order", WRITES)
def test_kv_quantise(pkg, layers, requests, kv, dim, page, block, dtype, order):
    r = np.random.default_rng(dim + len(requests))
    k, v, rows, slots, caches = write_case(r, layers, requests, kv, dim, page, block, dtype, order)
    if len(rows) > 6:  # entries that are skipped
        rows[1], slots[3], rows[4] = -1, -1, k.shape[1]
        slots[-1] = caches[0][0].shape[1] * page
    check_write(pkg, k, v, rows, slots, caches, block, dtype, order)


def test_skipped_entries_between_those_of_a_block(pkg):
    # runs of skipped entries inside a block's, some longer than what a block's CTA looks at together, and at both ends
    r = np.random.default_rng(41)
    for gap in (1, 30, 200, 700):
        requests = [(3, 9), (40, 20), (64, 33)]
        k, v, rows, slots, caches = write_case(r, 2, requests, 2, 72, 32, 16, "bfloat16", "token")
        at = np.sort(r.choice(len(rows) + 1, 6, replace=False))
        fill = lambda x, with_what: np.insert(x, np.repeat(at, gap), with_what)
        check_write(pkg, k, v, fill(rows, 0), fill(slots, -1), caches, 16, "bfloat16", "token")
        check_write(pkg, k, v, fill(rows, -1), fill(slots, -1), caches, 16, "bfloat16", "token", repeat=1)
    # a list of which nothing counts
    check_write(pkg, k, v, np.full(50, -1), np.arange(50), caches, 16, "bfloat16", "token", repeat=1)
    check_write(pkg, k, v, np.zeros(50, np.int64), np.full(50, -7), caches, 16, "bfloat16", "token", repeat=1)


@pytest.mark.parametrize("gap", [1, 31, 150, 400])
def test_skipped_entries_with_slots_of_other_blocks(pkg, gap):
    # entries without a row, whose slots are those of other blocks or are written by entries that count, inside a block's run: next to
    # each other, across the 32 entries that a CTA begins with, and past the 160 that it looks at together
    r = np.random.default_rng(43 + gap)
    for block, page in ((16, 32), (128, 128)):
        k, v, rows, slots, caches = write_case(r, 2, [(3, 9), (40, 20), (64, 73)], 2, 72, page, block, "bfloat16", "token")
        n, total = k.shape[1], caches[0][0].shape[1] * page
        at = np.sort(np.repeat(r.choice(len(rows) + 1, 12, replace=False), gap))
        none = r.choice([-1, n, n + 5, -(1 << 31), (1 << 31) - 1], len(at))
        check_write(pkg, k, v, np.insert(rows, at, none), np.insert(slots, at, r.integers(0, total, len(at))), caches, block, "bfloat16", "token")


def test_a_skipped_entry_of_another_block_between_two_of_one(pkg):
    # blocks of 16: entries 0 and 2 are of block 0, entry 1 has no row.  All places of the run are written by it, so the old scale does not
    # count; with a first place that stays it does.
    r = np.random.default_rng(44)
    for first in (0, 1):
        for lead in (0, 29, 30, 31):  # entries in front, each of a block of its own
            k, v, _, _, caches = write_case(r, 1, [(0, 16)] * 35, 2, 64, 16, 16, "bfloat16", "token")
            front = 16 * np.arange(3, 3 + lead)
            slots = np.concatenate([front, [first, 16, first + 1, 32]])
            rows = np.concatenate([np.arange(lead), [lead, -1, lead + 1, lead + 2]])
            for _, s in caches:
                s[:, 0] = 2.0 ** 20
            check_write(pkg, k, v, rows, slots, caches, 16, "bfloat16", "token")


def test_a_wait_that_expires_loses_nothing(pkg, tmp_path, monkeypatch):
    """Writes whose waits for their copies give up in some CTAs (quantise_probe.cu): the rows are read from where they lie."""
    import ctypes as C
    import subprocess
    from paper_2607_12287_gb300 import build as b
    so = str(tmp_path / "probe.so")
    subprocess.run([b.NVCC, *b.ARCH, *b.FLAGS, "-shared", f"{b.ROOT}/tests/quantise_probe.cu", b.LIB, "-Xlinker",
                    "-rpath=" + b.OUT_DIR, "-o", so], check=True)
    probe = C.CDLL(so)
    probe.ivit_kv_quantise.argtypes = pkg.load().ivit_kv_quantise.argtypes
    monkeypatch.setattr(pkg, "load", lambda *a: probe)
    counts = [0, 0, 0]
    for requests, layers, kv, dim, page, block, dtype in (
            ([(3 * i, 1 + i % 6) for i in range(60)], 6, 8, 80, 32, 16, "bfloat16"), ([(5, 700), (0, 333)], 27, 16, 72, 32, 32, "float16"),
            ([(9, 200), (100, 300)], 3, 2, 128, 128, 128, "bfloat16"), ([(1, 3), (2, 1)], 1, 3, 64, 16, 8, "float16")):
        for expire in (0, 1, 2):
            assert probe.probe_expire(expire) == 0
            r = np.random.default_rng(dim)
            k, v, rows, slots, caches = write_case(r, layers, requests, kv, dim, page, block, dtype, "token")
            rows[2], slots[3] = -1, -1
            check_write(pkg, k, v, rows, slots, caches, block, dtype, "token")
            counts[expire] += probe.probe_expired() - sum(counts)
    assert counts[0] == 0 and min(counts[1:]) > 100


def test_writes_and_reads_on_another_stream_and_in_a_graph(pkg):
    import torch
    r = np.random.default_rng(42)
    k, v, rows, slots, caches = write_case(r, 3, [(5, 40), (0, 3)], 4, 64, 16, 8, "float16", "token")
    kc, vc, ks, vs, lay = check_write(pkg, k, v, rows, slots, caches, 8, "float16", "token", repeat=1)
    want = [codes_of(kc), codes_of(vc), host(ks), host(vs)]
    back = [torch.zeros((3, len(slots), 4, 64), dtype=torch.float16, device="cuda") for _ in range(4)]
    rows, slots = i32(rows), i32(slots)
    pkg.ivit_kv_dequantise(lay, slots, kc, vc, ks, vs, back[0], back[1])
    fresh = lambda: [codes_on_gpu(caches[0][0]), codes_on_gpu(caches[1][0]), dev(caches[0][1]), dev(caches[1][1])]
    one, two, side = fresh(), fresh(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        pkg.ivit_kv_quantise(lay, k, v, rows, slots, *one)
        pkg.ivit_kv_dequantise(lay, slots, *one, back[2], back[3])
    side.synchronize()
    same = lambda c: all(np.array_equal(a, b, equal_nan=True) for a, b in zip([codes_of(c[0]), codes_of(c[1]), host(c[2]), host(c[3])], want))
    assert same(one) and torch.equal(back[0], back[2]) and torch.equal(back[1], back[3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.ivit_kv_quantise(lay, k, v, rows, slots, *two)
        pkg.ivit_kv_dequantise(lay, slots, *two, back[2], back[3])
    for _ in range(2):
        for x, y in zip(two, fresh()):
            x.view(torch.uint8).copy_(y.view(torch.uint8))
        back[2].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(two) and torch.equal(back[0], back[2])


def test_of_nothing(pkg):
    # no entries, no rows, no layers, requests without rows: nothing is touched
    import torch
    codes, scale = np.full((1, 2, 8, 2, 16), 0x33, np.uint8), np.full((1, 2, 2, 2), 0.5, np.float32)
    kc, vc, ks, vs = codes_on_gpu(codes), codes_on_gpu(codes), dev(scale), dev(scale)
    lay = pkg.make_quantised_layout(kc[0], 4)
    k = torch.ones((1, 3, 2, 16), dtype=torch.bfloat16, device="cuda")
    pkg.ivit_kv_quantise(lay, k, k, i32([]), i32([]), kc, vc, ks, vs)
    pkg.ivit_kv_quantise(lay, k[:, :0], k[:, :0], i32([0]), i32([0]), kc, vc, ks, vs)
    pkg.ivit_kv_quantise(lay, k[:0], k[:0], i32([0]), i32([0]), kc, vc, ks, vs)
    pkg.ivit_kv_dequantise(lay, i32([]), kc, vc, ks, vs, k[:, :0], k[:, :0])
    assert np.array_equal(codes_of(kc), codes) and np.array_equal(host(ks), scale) and (k == 1).all()
    cfg = pkg.make_verify_config(3, 10, 4, "float32")
    path, accepted, after = i32([5]), i32([7, 7, 7]), i32([7, 7, 7])
    pkg.ivit_tree_verify(cfg, torch.zeros((0, 10), device="cuda"), None, i32([]), None, i32([0, 0, 0, 0]), None, None, None, path, accepted, after)
    assert accepted.tolist() == [0, 0, 0] and after.tolist() == [-1, -1, -1] and path.tolist() == [5]
    c = attention_case(np.random.default_rng(1), [20, 30], [0, 2], 2, 2, 64, 8, 8, "bfloat16")
    c["cu"] = np.zeros(3, np.int64)
    args = call(pkg, c, "causal", max_new=50, fill=3.0)
    pkg.ivit_tree_attention_quantised(*args)
    assert (args[-3] == 3).all() and (args[-2] == 3).all()


def test_a_block_grows_token_by_token(pkg):
    # every call adds a token to the block: its scale follows the largest so far, the codes are rounded again
    import torch
    r = np.random.default_rng(1)
    page = block = 16
    codes, scale = (np.full((1, 3, page, 2, 64), 0x55, np.uint8), np.full((1, 3, 1, 2), 2.0 ** 30, np.float32))
    kc, vc, ks, vs = codes_on_gpu(codes), codes_on_gpu(codes), dev(scale), dev(scale)
    want = [(codes.copy(), scale.copy()), (codes.copy(), scale.copy())]
    lay = pkg.make_quantised_layout(kc[0], block)
    for t in range(2 * page):
        slot = (2 * page if t < page else 0) + t % page
        x = dev((r.standard_normal((2, 1, 1, 2, 64)) * 2.0 ** r.integers(-20, 20)).astype(np.float32), "bfloat16")
        pkg.ivit_kv_quantise(lay, x[0], x[1], i32([0]), i32([slot]), kc, vc, ks, vs)
        for part, (c, s) in zip(host(x), want):
            ref.quantise(c[0], s[0], [part[0, 0]], [slot], block)
        for (c, s), got_c, got_s in zip(want, (kc, vc), (ks, vs)):
            assert np.array_equal(host(got_s), s) and np.array_equal(codes_of(got_c), c), t


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_values_at_the_ends(pkg, dtype):
    # zeros, the smallest and largest values, values next to a scale's border, and such that are not finite
    import torch
    tiny, huge = (2.0 ** -133, 3.3e38) if dtype == "bfloat16" else (2.0 ** -24, 65504.0)
    rows = np.zeros((1, 9, 2, 16))
    rows[0, 1] = tiny
    rows[0, 2, 0, 3] = huge
    rows[0, 3, 1, :4] = [448, 449, -448, 2.0 ** -9]
    rows[0, 4, 0, :4] = [450, 1, 2.0 ** -5, -0.0]
    rows[0, 5, 0, :4] = [np.inf, 1, -np.inf, np.nan]
    rows[0, 6] = np.nan
    rows[0, 7, 1] = np.linspace(-448, 448, 16)
    rows[0, 8, 0] = 2.0 ** np.arange(-10, 6)
    k = dev(rows.astype(np.float32), dtype)
    caches = [(np.zeros((1, 4, 4, 2, 16), np.uint8), np.full((1, 4, 4, 2), np.nan, np.float32)) for _ in range(2)]
    check_write(pkg, k, k, np.arange(9), np.arange(9), caches, 1, dtype, "token")
    # blocks whose old scale is of no use
    for bad in (np.nan, 0.0, np.inf, -1.0):
        caches = [(np.full((1, 1, 4, 2, 16), 0x22, np.uint8), np.full((1, 1, 1, 2), bad, np.float32)) for _ in range(2)]
        check_write(pkg, k, k, np.array([8]), np.array([2]), caches, 4, dtype, "token")


def test_old_scales_that_are_no_powers_of_two(pkg):
    r = np.random.default_rng(3)
    caches = [(ref.encode(r.standard_normal((1, 2, 8, 2, 32)) * 90), (1.37 * 2.0 ** r.integers(-9, -5, (1, 2, 1, 2))).astype(np.float32))
              for _ in range(2)]
    k = dev((r.standard_normal((1, 2, 2, 32)) * 0.05).astype(np.float32), "float16")
    check_write(pkg, k, k, np.array([0, 1]), np.array([5, 14]), caches, 8, "float16", "token")


@pytest.mark.parametrize("layers,n,kv,dim,page,block,dtype,order", [
    (1, 1, 1, 8, 1, 1, "bfloat16", "token"), (27, 5, 4, 64, 16, 16, "bfloat16", "token"), (3, 70, 2, 72, 8, 2, "float16", "head"),
    (2, 333, 8, 256, 64, 32, "bfloat16", "head"), (1, 40, 3, 104, 128, 128, "float16", "token"),
])
def test_kv_dequantise(pkg, layers, n, kv, dim, page, block, dtype, order):
    import torch
    r = np.random.default_rng(n)
    pages = -(-n // page) + 2
    caches = [random_cache(r, (layers, pages), page, kv, dim, block, (-20, 7)) for _ in range(2)]
    caches[0][0][0, 0, 0, 0, 0] = 0x7f
    slots = r.permutation(pages * page)[:n]
    slots[0] = 0
    if n > 4:
        slots[1], slots[2] = -1, pages * page
    ok = (slots >= 0) & (slots < pages * page)
    kc, vc = (codes_on_gpu(c, order) for c, _ in caches)
    # rows of a wider array
    out = torch.full((layers, n, 2, kv, dim), 3.0, dtype=getattr(torch, dtype), device="cuda")
    k, v = out[:, :, 0], out[:, :, 1]
    pkg.ivit_kv_dequantise(pkg.make_quantised_layout(kc[0], block, dtype), i32(slots), kc, vc, *(dev(s) for _, s in caches), k, v)
    for got, (c, s) in zip((k, v), caches):
        got = host(got)
        assert (got[:, ~ok] == 3).all()
        for layer in range(layers):
            want = ref.decode(c[layer], s[layer], block).reshape(pages * page, kv, dim)[slots[ok]]
            nan = np.isnan(want)
            assert np.array_equal(np.isnan(got[layer, ok]), nan)
            assert (np.abs(got[layer, ok] - want)[~nan] <= UNIT[dtype] * np.abs(want)[~nan] + 2.0 ** -25 * (dtype == "float16")).all()


# ------------------------------------------------------------------------ attention

def attention_case(r, lengths, new, heads, kv, dim, page, block, dtype, order="token", spread=(-9, -5)):
    n, rows = len(lengths), int(np.sum(new))
    need = [-(-int(x) // page) for x in lengths]
    pages = sum(need) + 3
    ids, used = r.permutation(pages), 0
    table = np.full((n, max(need + [0]) + 2), -1, np.int64)
    for i, m in enumerate(need):
        table[i, :m] = ids[used:used + m]
        used += m
    caches = [random_cache(r, (pages,), page, kv, dim, block, spread) for _ in range(2)]
    # (what lies in the pages past a request's tokens must not matter, nor the scales of blocks that hold none)
    for i, m in enumerate(lengths):
        if m % page:
            for c, s in caches:
                c[table[i, m // page], m % page:] = 0x7f
                s[table[i, m // page], -(-(m % page) // block):] = np.nan
    qkv = dev(r.standard_normal((rows, (heads + 2 * kv) * dim)).astype(np.float32), dtype)
    part = lambda lo, m: qkv[:, lo * dim:(lo + m) * dim].unflatten(1, (m, dim))
    return dict(q=part(0, heads), k=part(heads, kv), v=part(heads + kv, kv), caches=caches, table=table, block=block, order=order,
                lengths=np.asarray(lengths), cu=np.concatenate([[0], np.cumsum(new)]).astype(np.int64), dtype=dtype)


def call(pkg, c, mask, packed=None, words=0, scale=None, max_new=None, fill=float("nan")):
    """The call's arguments on the GPU: configuration, layout, and what follows."""
    import torch
    rows, heads, dim = c["q"].shape
    most = int(np.diff(c["cu"]).max()) if max_new is None else max_new
    kc, vc = (codes_on_gpu(codes, c["order"]) for codes, _ in c["caches"])
    lay = pkg.make_quantised_layout(kc, c["block"], c["dtype"])
    cfg = pkg.make_attention_config(len(c["cu"]) - 1, heads, c["table"].shape[1], most, mask, words, dim ** -0.5 if scale is None else scale)
    out = torch.full((rows, heads, dim), fill, dtype=c["q"].dtype, device="cuda")
    lse = torch.full((rows, heads), fill, device="cuda")
    ws = torch.full((pkg.ivit_tree_attention_quantised_workspace(cfg, lay),), 255, dtype=torch.uint8, device="cuda")
    return [cfg, lay, c["q"], c["k"], c["v"], kc, vc, *(dev(s) for _, s in c["caches"]), i32(c["table"]), i32(c["lengths"]),
            i32(c["cu"]), packed, out, lse, ws]


def run_attention(pkg, c, mask, vis=None, check=True, scale=None, max_new=None, mask_words=None):
    import torch
    new = np.diff(c["cu"])
    words = (int(new.max()) + 31) // 32 if mask_words is None else mask_words
    packed = dev(np.concatenate([backbone_ref.words(vis[i], words) for i in range(len(new))])) if mask == "tree" else None
    args = call(pkg, c, mask, packed, words if mask == "tree" else 0, scale, max_new)
    pkg.ivit_tree_attention_quantised(*args)
    out, lse, ws = args[-3:]
    assert int(ws[:4].view(torch.int32)) == 0  # no wait of the kernel expired
    if check:
        check_attention(c, out, lse, mask, vis, args[0].scale)
    return out, lse


def check_attention(c, out, lse, mask, vis, scale):
    sees = {"causal": lambda i, n: np.tril(np.ones((n, n), bool)), "all": lambda i, n: np.ones((n, n), bool),
            "tree": lambda i, n: vis[i]}[mask]
    kc, vc = (ref.decode(codes, s, c["block"]) for codes, s in c["caches"])
    want, want_lse, size = backbone_ref.attention(host(c["q"]), host(c["k"]), host(c["v"]), kc, vc, c["table"], c["lengths"], c["cu"],
                                                  sees, scale)
    u = UNIT[c["dtype"]]
    bound = u * np.abs(want) + (u + 2.0 ** -14) * size + 2.0 ** -25
    err = np.abs(host(out) - want)
    assert (err <= bound).all(), f"{np.nanmax(err / bound)} of the bound, {np.isnan(host(out)).sum()} NaN"
    got, none = host(lse), np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(got), none)
    assert (np.abs(got[~none] - want_lse[~none]) <= 2.0 ** -14).all()


ATTENTION = [  # cached, new, heads, kv, dim, page, block, type, order
    ([0], [1], 4, 4, 64, 16, 16, "bfloat16", "token"), ([1], [1], 8, 2, 64, 16, 4, "float16", "token"),
    ([63], [1], 1, 1, 64, 8, 8, "bfloat16", "token"), ([64], [1], 16, 4, 128, 16, 16, "bfloat16", "head"),
    ([130, 0, 65, 700], [1, 3, 0, 9], 8, 2, 72, 16, 8, "bfloat16", "token"),
    ([5, 64, 127, 128, 129], [2, 1, 64, 63, 65], 4, 2, 80, 1, 1, "float16", "head"),
    ([1500], [31], 8, 1, 128, 64, 32, "float16", "token"), ([40, 900, 33], [12, 1, 40], 14, 2, 96, 32, 32, "bfloat16", "token"),
    ([100, 300], [17, 5], 5, 1, 256, 128, 64, "float16", "head"), ([257], [3], 2, 2, 256, 16, 2, "bfloat16", "token"),
    ([90, 10], [70, 130], 3, 3, 40, 16, 16, "bfloat16", "token"), ([2000, 3, 777], [4, 4, 4], 8, 8, 8, 1024, 1024, "float16", "token"),
    ([33], [7], 32, 1, 200, 4, 2, "bfloat16", "head"), ([31, 500], [1, 1], 6, 3, 104, 2, 1, "float16", "token"),
    # many rows per key head, groups that do not divide a tile
    ([300, 95, 96, 97, 0], [65, 96, 20, 1, 130], 8, 4, 72, 8, 8, "bfloat16", "token"),
    ([191, 192, 500], [128, 33, 97], 5, 1, 80, 128, 16, "float16", "head"), ([700], [256], 2, 2, 64, 64, 64, "bfloat16", "token"),
    ([0, 0, 127, 128, 129], [140, 3, 128, 129, 70], 2, 2, 64, 16, 1, "float16", "token"),
    ([0, 64, 200], [75, 64, 1], 7, 1, 128, 16, 16, "bfloat16", "token"), ([500], [65], 6, 2, 112, 256, 128, "bfloat16", "head"),
    ([300, 96], [50, 129], 2, 2, 88, 16, 8, "bfloat16", "head"), ([63, 64, 65, 500], [40, 1, 64, 20], 5, 1, 136, 16, 16, "bfloat16", "token"),
    ([200, 0], [130, 17], 2, 2, 192, 32, 16, "float16", "head"), ([300, 128, 1], [129, 256, 9], 4, 2, 256, 8, 4, "bfloat16", "token"),
    ([900], [20], 32, 2, 256, 512, 32, "bfloat16", "head"), ([129], [100], 1, 1, 200, 4, 4, "bfloat16", "token"),
    ([70, 0, 130], [50, 3, 1], 1, 1, 128, 2, 2, "float16", "token"), ([300, 40], [40, 17], 1, 1, 96, 1, 1, "float16", "head"),
    ([200, 10], [2, 1], 150, 1, 64, 16, 16, "bfloat16", "token"),
]


@pytest.mark.parametrize("lengths,new,heads,kv,dim,page,block,dtype,order", ATTENTION)
@pytest.mark.parametrize("mask", ["causal", "all", "tree"])
def test_tree_attention_quantised(pkg, lengths, new, heads, kv, dim, page, block, dtype, order, mask):
    r = np.random.default_rng(sum(lengths) + sum(new) + dim)
    c = attention_case(r, lengths, new, heads, kv, dim, page, block, dtype, order)
    run_attention(pkg, c, mask, trees(r, new) if mask == "tree" else None)


@pytest.mark.parametrize("dim,most_new,n", [(64, 2, 700), (72, 2, 700), (40, 2, 700), (96, 2, 500), (256, 2, 300), (72, 20, 200),
                                            (96, 70, 40), (256, 20, 150)])
def test_many_short_requests(pkg, dim, most_new, n):
    # every CTA goes through several tiles of rows
    r = np.random.default_rng(2)
    c = attention_case(r, r.integers(0, 90, n), r.integers(0, most_new + 1, n), 6, 3, dim, 8, 4, "bfloat16")
    run_attention(pkg, c, "causal")


@pytest.mark.parametrize("new", [2, 40])
def test_scales_far_apart(pkg, new):
    # blocks of values from 2^-50 to 2^20, in an order that makes the running maximum grow and others vanish; keys a little
    r = np.random.default_rng(5)
    c = attention_case(r, [600], [new], 4, 2, 64, 16, 4, "bfloat16")
    (kc, ks), (vc, vs) = c["caches"]
    vs[:] = 2.0 ** r.integers(-50, 21, vs.shape).astype(np.float32)
    run_attention(pkg, c, "causal")
    vs[:] = 2.0 ** -60                 # alone, and beside new rows of ordinary size
    run_attention(pkg, c, "causal")
    vs[:] = 1.7 * 2.0 ** r.integers(-9, -5, vs.shape).astype(np.float32)  # not ivit_kv_quantise's
    ks[:] = 1.3 * 2.0 ** r.integers(-9, -5, ks.shape).astype(np.float32)
    run_attention(pkg, c, "causal")


@pytest.mark.parametrize("new", [1, 30])
def test_queries_of_every_size(pkg, new):
    # bf16 queries beyond fp16's range, and tiny ones
    r = np.random.default_rng(8)
    for power in (-60, -30, 20, 60):
        c = attention_case(r, [300], [new], 4, 2, 72, 16, 16, "bfloat16")
        c["q"] = (c["q"].float() * 2.0 ** power).bfloat16()
        c["k"] = (c["k"].float() * 0).bfloat16()  # (the new rows' scores stay small)
        run_attention(pkg, c, "causal", scale=0.1 * 2.0 ** -power)
    c = attention_case(r, [100], [new], 4, 2, 64, 16, 16, "bfloat16")
    c["q"] = c["q"] * 0
    run_attention(pkg, c, "all")


def test_rows_that_see_nothing(pkg):
    r = np.random.default_rng(4)
    new = [5, 40, 3]
    vis = [np.zeros((n, n), bool) for n in new]
    vis[1][7, 3] = vis[1][39, 0] = vis[1][39, 39] = True
    for lengths in ([0, 0, 0], [0, 0, 90]):
        c = attention_case(r, lengths, new, 4, 2, 64, 16, 8, "bfloat16")
        out, lse = run_attention(pkg, c, "tree", vis)
        assert float(out[:5].abs().max()) == 0 and float(lse[:5].max()) == -np.inf


@pytest.mark.parametrize("new,page,dim", [(4, 16, 64), (20, 16, 64), (100, 16, 64), (4, 4, 64), (20, 4, 72), (100, 4, 64), (4, 16, 256),
                                          (30, 16, 256), (60, 8, 128), (90, 8, 80), (70, 8, 192), (50, 16, 96)])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_does_not_see_does_not_reach_it(pkg, new, page, dim, dtype, bad):
    import torch
    r = np.random.default_rng(new)
    c = attention_case(r, [70], [new], 4, 2, dim, page, page, dtype)
    vis = [np.tril(np.ones((new, new), bool))]
    vis[0][:, 2] = False
    vis[0][new - 1, 2] = True          # only the last row sees draft 2
    clean, clean_lse = run_attention(pkg, c, "tree", vis)
    c["v"][2, 1, 5] = bad              # one value of one head
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


def test_cached_codes_that_are_no_numbers(pkg):
    # a value that could not be kept (NaN) reaches its column of every row that sees it, and no other head or request
    r = np.random.default_rng(9)
    for new in (1, 33):
        c = attention_case(r, [80, 50], [new, new], 4, 2, 64, 16, 8, "bfloat16")
        c["caches"][1][0][c["table"][0, 2], 3, 1, 7] = 0x7f
        out, lse = run_attention(pkg, c, "causal", check=False)
        bad = np.isnan(host(out))
        assert bad[:new, 2:, 7].all() and bad.sum() == 2 * new and np.isfinite(host(lse)).all()


def test_tensors_of_another_device_than_the_current_one(pkg, monkeypatch):
    # refused before anything is launched, also by calls that give their stream
    import torch
    c = attention_case(np.random.default_rng(2), [20], [2], 4, 2, 64, 16, 16, "bfloat16")
    args = call(pkg, c, "causal")
    lay, k, kc, vc, ks, vs = args[1], args[3], *args[5:9]
    layers = [x[None] for x in (kc, vc, ks, vs)]
    stream = torch.cuda.current_stream()
    cfg = pkg.make_verify_config(1, 10, 4, "float32")
    rows, logits = i32([0, 1]), torch.zeros((2, 10), device="cuda")
    calls = [lambda: pkg.ivit_tree_attention_quantised(*args, stream=stream),
             lambda: pkg.ivit_kv_quantise(lay, k[None], k[None], rows, rows, *layers, stream=stream),
             lambda: pkg.ivit_kv_dequantise(lay, rows, *layers, k[None], k[None], stream=stream),
             lambda: pkg.ivit_tree_verify(cfg, logits, None, rows, None, i32([0, 2]), None, None, None, i32([0, 0]), i32([0]), i32([0]),
                                          stream=stream)]
    pkg._stream(None)
    monkeypatch.setattr(pkg, "_current", [pkg._current[0], lambda: 1])
    for f in calls:
        with pytest.raises(ValueError, match="the current device is cuda:1"):
            f()


@pytest.mark.parametrize("block", [4, 16])
@pytest.mark.parametrize("new", [1, 3, 30])
def test_scales_that_are_none(pkg, new, block):
    # scales that are not positive or not finite: such keys count as 0, such values as good as 0 (2^-80 of their codes, below the
    # bound's 2^-25), beside ordinary ones, and where no others are
    r = np.random.default_rng(14)
    for share in (0.3, 1.0):
        c = attention_case(r, [300, 9], [new, new], 4, 2, 64, 16, block, "bfloat16")
        none = np.array([0.0, -0.0, -1.0, -2.0 ** -8, 1e-40, np.nan, -np.inf, np.inf], np.float32)
        scales = [s for _, s in c["caches"]]
        at = [r.random(s.shape) < share for s in scales]
        for s, here in zip(scales, at):
            s[here] = r.choice(none, int(here.sum()))
        out, lse = run_attention(pkg, c, "causal", check=False)
        for s, here in zip(scales, at):
            s[here] = 0
        check_attention(c, out, lse, "causal", None, 64 ** -0.5)


@pytest.mark.parametrize("new", [1, 30])
def test_long_cache_of_scales_that_are_none(pkg, new):
    # (the sum of their probabilities, each over its scale, stays finite)
    r = np.random.default_rng(15)
    c = attention_case(r, [270000], [new], 2, 1, 64, 16, 16, "bfloat16")
    for _, s in c["caches"]:
        s[:] = 0
    run_attention(pkg, c, "causal")


def test_pages_outside_the_cache_read_as_zeros(pkg):
    r = np.random.default_rng(12)
    for new in (2, 50):
        for page in (4, 16):
            c = attention_case(r, [100], [new], 4, 2, 64, page, page, "bfloat16")
            c["table"][0, 1] = -1
            c["table"][0, 3] = 1 << 30
            out, lse = run_attention(pkg, c, "causal", check=False)
            zero = dict(c, caches=[(codes.copy(), s.copy()) for codes, s in c["caches"]])
            table = c["table"].copy()
            free = [p for p in range(zero["caches"][0][0].shape[0]) if p not in table][0]
            for codes, s in zero["caches"]:  # (a page of zeros, which no request has, in the place of both)
                codes[free], s[free] = 0, 1
            table[0, 1] = table[0, 3] = free
            zero["table"] = table
            # (each against the definition: two results may be twice its bound apart, for their probabilities are rounded
            # against other maxima)
            check_attention(zero, out, lse, "causal", None, 64 ** -0.5)
            run_attention(pkg, zero, "causal")


def test_large_scores_and_growing_maximum(pkg):
    # scores up to a few hundred that grow along the keys: the running maximum moves in every tile
    r = np.random.default_rng(6)
    c = attention_case(r, [1000, 640], [2, 33], 4, 1, 64, 16, 8, "float16", spread=(-7, -6))
    codes, scale = c["caches"][0]
    q = host(c["q"])[0, 0]
    t = np.arange(1000)
    codes[c["table"][0][t // 16], t % 16, 0] = ref.encode(q * np.linspace(0.3, 120.0, 1000)[:, None])
    run_attention(pkg, c, "causal", scale=0.125)


@pytest.mark.parametrize("group", [1, 8])
def test_offsets_past_32_bits(pkg, group):
    # pages at the far end of a cache of more than 2^32 codes
    import torch
    page, kv, dim, block = 16, 8, 128, 8
    pages = (1 << 32) // (page * kv * dim) + 64
    r = np.random.default_rng(7)
    if torch.cuda.mem_get_info()[0] < 3 * pages * page * kv * dim:
        pytest.skip("needs 13 GB of device memory")
    c = attention_case(r, [300], [3], 8 * group, 8, dim, page, block, "bfloat16")
    want, want_lse = run_attention(pkg, c, "causal")
    args = call(pkg, c, "causal")
    big = torch.empty((pages, page, kv, dim), dtype=torch.uint8, device="cuda")
    scales = [torch.empty((pages, page // block, kv), device="cuda") for _ in range(2)]
    n = c["caches"][0][0].shape[0]
    far = (pages - 1 - np.arange(n)).astype(np.int64)  # keys in the last pages, values of the same pages 2 n lower
    fi = torch.from_numpy(far).cuda()
    big[fi], big[fi - 2 * n] = args[5].view(torch.uint8), args[6].view(torch.uint8)
    # (the array of keys begins 2 n pages into the one of values; a table entry is a page of both)
    ids = np.where(c["table"] >= 0, far[np.maximum(c["table"], 0)] - 2 * n, -1)
    f8 = big.view(torch.float8_e4m3fn)
    keys, values = f8[2 * n:], f8[:pages - 2 * n]
    lay = pkg.make_quantised_layout(keys, block, "bfloat16")
    ks, vs = (s[:pages - 2 * n].contiguous() for s in scales)
    ks[fi - 2 * n], vs[fi - 2 * n] = args[7], args[8]
    args[1], args[5], args[6], args[7], args[8], args[9] = lay, keys, values, ks, vs, i32(ids)
    pkg.ivit_tree_attention_quantised(*args)
    assert torch.equal(args[-3], want) and torch.equal(args[-2], want_lse)
    # and a write and a read there
    src = torch.randn((1, 2, kv, dim), device="cuda").to(torch.bfloat16)
    lay = pkg.make_quantised_layout(f8, block, "bfloat16")
    slots = i32([pages * page - 1, pages * page - 16])
    for s in scales:
        s[-1] = 2.0 ** -9
    pkg.ivit_kv_quantise(lay, src, src, i32([1, 0]), slots, f8[None], f8[None], scales[0][None], scales[1][None])
    back = torch.zeros_like(src)
    pkg.ivit_kv_dequantise(lay, slots, f8[None], f8[None], scales[0][None], scales[1][None], back, back.clone())
    # (half a step of e4m3, and below 2^-6 of the scale 2^-10)
    assert ((back.float() - src[:, [1, 0]].float()).abs() <= 2.0 ** -4 * src[:, [1, 0]].float().abs() + 2.0 ** -16).all()


def test_rows_of_no_request_stay(pkg):
    import torch
    r = np.random.default_rng(13)
    for new in (2, 40):
        c = attention_case(r, [30, 70], [new, new + 1], 4, 2, 64, 16, 16, "bfloat16")
        want, want_lse = run_attention(pkg, c, "causal")
        pad = lambda t: torch.cat([t, t[:3] * float("nan")])
        padded = dict(c, q=pad(c["q"]), k=pad(c["k"]), v=pad(c["v"]))
        args = call(pkg, padded, "causal", fill=7.0)
        pkg.ivit_tree_attention_quantised(*args)
        n = want.shape[0]
        assert torch.equal(args[-3][:n], want) and torch.equal(args[-2][:n], want_lse)
        assert (args[-3][n:] == 7).all() and (args[-2][n:] == 7).all()


def test_on_another_stream_and_in_a_graph(pkg):
    import torch
    r = np.random.default_rng(10)
    for new in ([1, 6], [40, 3]):
        c = attention_case(r, [500, 20], new, 8, 2, 64, 16, 16, "bfloat16")
        want, want_lse = run_attention(pkg, c, "causal")
        args = call(pkg, c, "causal")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            pkg.ivit_tree_attention_quantised(*args)
        side.synchronize()
        assert torch.equal(args[-3], want) and torch.equal(args[-2], want_lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pkg.ivit_tree_attention_quantised(*args)
        for _ in range(3):
            args[-3].zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(args[-3], want) and torch.equal(args[-2], want_lse)


def test_bounds_that_are_not_reached_and_lengths_beyond_the_table(pkg):
    # max_new chooses the kernel: one row of many that were allowed; lengths longer than the table count as its tokens
    r = np.random.default_rng(14)
    for dim in (64, 72, 128, 256):
        c = attention_case(r, [100, 33], [1, 2], 4, 2, dim, 16, 16, "float16")
        want, want_lse = run_attention(pkg, c, "causal")
        run_attention(pkg, c, "causal", max_new=60000)
        c["table"] = c["table"][:, :7]
        c["lengths"] = np.array([112, 33])
        for codes, s in c["caches"]:
            codes[c["table"][0, 6]] = 0x11
            s[c["table"][0, 6]] = 0.25
        want, want_lse = run_attention(pkg, c, "causal")
        c["lengths"] = np.array([5000, 33])
        got, got_lse = run_attention(pkg, c, "causal", check=False)
        assert bool((got == want).all()) and bool((got_lse == want_lse).all())


def test_two_calls_at_once(pkg):
    # two streams, a workspace each
    import torch
    r = np.random.default_rng(15)
    cases = [attention_case(r, [900, 400, 10], new, 8, 2, 128, 16, 16, "bfloat16") for new in ([1, 1, 1], [30, 40, 2])]
    want = [run_attention(pkg, c, "causal") for c in cases]
    args = [call(pkg, c, "causal") for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for a, s in zip(args, streams):
            with torch.cuda.stream(s):
                pkg.ivit_tree_attention_quantised(*a)
    torch.cuda.synchronize()
    for a, (out, lse) in zip(args, want):
        assert torch.equal(a[-3], out) and torch.equal(a[-2], lse)


# --------------------------------------------------------------------- verification

def verify_case(r, new, vocab, tree, probs, dtype, temperature, peaked=3.0):
    n, rows = len(new), int(np.sum(new))
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    idx = np.concatenate([np.arange(m) for m in new] + [np.zeros(0, np.int64)]).astype(np.int64)
    parent = idx - 1 - (np.floor(r.random(rows) * np.minimum(idx, 4)).astype(np.int64) if tree else 0)
    parent[idx == 0] = -1
    logits = dev((peaked * r.standard_normal((rows, vocab))).astype(np.float32), dtype)
    z = host(logits) + 0.5 * r.standard_normal((rows, vocab))
    p = np.exp(z - z.max(1, keepdims=True)) if rows else z
    p = (p / p.sum(1, keepdims=True)).astype(np.float32) if rows else z.astype(np.float32)
    tokens = np.zeros(rows, np.int64)
    for i in range(rows):
        if parent[i] >= 0:
            a = i - idx[i] + parent[i]
            tokens[i] = (p[a] / r.exponential(size=vocab)).argmax() if probs or r.random() < 0.3 else z[a].argmax()
    t = None if temperature is None else np.broadcast_to(np.float32(temperature), (n,)).copy()
    return dict(logits=logits, probs=p if probs else None, tokens=tokens, parent=parent if tree else None, cu=cu, temperature=t,
                uniform=r.random(rows).astype(np.float32), noise=r.exponential(size=(n, vocab)).astype(np.float32), dtype=dtype)


def run_verify(pkg, c, max_new=None, fill=77, check=True, least=0.95):
    import torch
    n, vocab, rows = len(c["cu"]) - 1, c["logits"].shape[1], c["logits"].shape[0]
    most = max(1, int(np.diff(c["cu"]).max())) if max_new is None else max_new
    opt = lambda a: None if a is None else a if torch.is_tensor(a) else dev(a)
    path, accepted, after = (torch.full((m,), fill, dtype=torch.int32, device="cuda") for m in (rows, n, n))
    cfg = pkg.make_verify_config(n, vocab, most, c["dtype"])
    none = c["temperature"] is None
    pkg.ivit_tree_verify(cfg, c["logits"], opt(c["probs"]), i32(c["tokens"]), None if c["parent"] is None else i32(c["parent"]),
                         i32(c["cu"]), opt(c["temperature"]), None if none else opt(c["uniform"]), None if none else opt(c["noise"]),
                         path, accepted, after)
    got = [host(x).astype(np.int64) for x in (path, accepted, after)]
    if check:
        probs = None if c["probs"] is None else host(opt(c["probs"]))
        noise = None if c["noise"] is None else host(opt(c["noise"]))
        *want, margin = ref.verify(host(c["logits"]), probs, c["tokens"], c["parent"], c["cu"], c["temperature"], c["uniform"], noise, most)
        sure = margin > 2.0 ** -16
        assert sure.mean() >= least
        for i in np.nonzero(sure)[0]:
            lo, hi = c["cu"][i], c["cu"][i + 1]
            assert np.array_equal(got[0][lo:hi], want[0][lo:hi]) and got[1][i] == want[1][i] and got[2][i] == want[2][i], i
        assert (got[0][c["cu"][-1]:] == fill).all()
    return got


@pytest.mark.parametrize("new,vocab,tree,probs,dtype", [
    ([1], 1, False, False, "float32"), ([5], 1000, False, False, "bfloat16"), ([4, 0, 7, 1], 33, True, True, "float16"),
    ([16] * 20, 5001, True, True, "float32"), ([8] * 30, 777, True, False, "bfloat16"), ([40, 3, 100], 130, True, True, "bfloat16"),
    ([3] * 400, 300, False, True, "float16"), ([6, 6], 70001, False, True, "bfloat16"), ([5] * 8, 32768, True, False, "bfloat16"),
    ([12] * 40, 2048, True, True, "float32"), ([2] * 700, 64, False, True, "bfloat16"), ([6], 131072, True, True, "float16"),
    ([4] * 3, 262144, True, True, "float32"),
])
@pytest.mark.parametrize("temperature", [None, 0.7, 1.0, "mixed"])
def test_tree_verify(pkg, new, vocab, tree, probs, dtype, temperature):
    r = np.random.default_rng(vocab + len(new))
    t = np.where(r.random(len(new)) < 0.4, 0.0, r.uniform(0.3, 2.0, len(new))) if temperature == "mixed" else temperature
    c = verify_case(r, new, vocab, tree, probs, dtype, t)
    got = run_verify(pkg, c)
    if vocab > 1:
        # (drafts near the target: some are accepted)
        assert got[1].max() > 1 or len(new) < 4
    again = run_verify(pkg, c, check=False)
    assert all(np.array_equal(a, b) for a, b in zip(got, again))


def test_drafts_that_hang_on_one_row_in_many(pkg):
    # 200 candidates behind the first row, none likely, some of them twice, some outside the vocabulary
    r = np.random.default_rng(21)
    for probs in (False, True):
        c = verify_case(r, [201] * 6, 500, True, probs, "float32", 1.0, peaked=0.5)
        c["parent"] = np.tile(np.concatenate([[-1], np.zeros(200, np.int64)]), 6)
        c["tokens"] = r.integers(-2, 503, 6 * 201)
        run_verify(pkg, c, least=0.8)


@pytest.mark.parametrize("vocab,dtype", [(64, "bfloat16"), (5001, "float32"), (40000, "float16"), (131072, "float32")])
def test_what_is_left_after_likely_drafts(pkg, vocab, dtype):
    # without probabilities, logits 0, -2.25, -4.5, ...: each of the candidates behind the first row has 1 - e^-2.25 = 0.8946 of what the
    # ones before it leave, so what is left after k is e^(-2.25 k), 2^-52 after 16; one u on either side of the last one's share
    r = np.random.default_rng(29)
    share, counts = 1 - np.exp(-2.25), np.arange(1, 17)
    for near in (share - 0.02, share + 0.02):
        new, n = counts + 1, len(counts)
        c = verify_case(r, new, vocab, True, False, dtype, 1.0)
        order = r.permutation(vocab)[:40]
        logits = np.full((c["logits"].shape[0], vocab), -np.inf, np.float32)
        logits[:, order] = -2.25 * np.arange(40, dtype=np.float32)  # (up to -87.75: nine bits at most, eight of the first 17)
        c["logits"] = dev(logits, dtype)
        idx = np.concatenate([np.arange(m) for m in new])
        c["parent"], c["tokens"] = np.where(idx == 0, -1, 0), order[np.maximum(idx - 1, 0)]
        c["uniform"] = np.where(idx == np.repeat(new - 1, new), near, 0.95).astype(np.float32)
        _, accepted, _ = run_verify(pkg, c, least=1.0)
        assert (accepted == (2 if near < share else 1)).all()


def test_many_drafts_that_take_a_little_each(pkg):
    # 1000 candidates of 4096 equal tokens: what is left shrinks by one of them each time, and the last is accepted by its share
    r = np.random.default_rng(30)
    for off, want in ((-0.01, 2), (0.01, 1)):
        c = verify_case(r, [1002], 4096, True, False, "float32", 1.0)
        c["logits"][:] = 0.0
        c["parent"] = np.concatenate([[-1], np.zeros(1001, np.int64)])
        c["tokens"] = r.permutation(4096)[:1002]
        c["uniform"] = np.full(1002, 0.999, np.float32)
        c["uniform"][-1] = (1 + off) / (4096 - 1000)
        assert run_verify(pkg, c, least=1.0)[1][0] == want


def test_more_rows_than_are_looked_at(pkg):
    r = np.random.default_rng(22)
    c = verify_case(r, [9, 30, 2], 400, True, True, "bfloat16", 0.9)
    run_verify(pkg, c, max_new=6)


def test_logits_that_are_not_finite(pkg):
    import torch
    r = np.random.default_rng(23)
    for temperature in (None, 1.0):
        c = verify_case(r, [1, 3, 3, 2, 2], 300, False, False, "float32", temperature)
        c["logits"][0] = -np.inf                # no token has a probability
        c["logits"][1, :200] = -np.inf          # some have none
        c["logits"][4, ::2] = float("nan")
        c["logits"][7, 11] = c["logits"][7, 200] = np.inf  # two have it all
        c["tokens"][8] = 11
        got = run_verify(pkg, c)
        assert got[2][0] == -1


def test_ties_and_noise_that_takes_no_part(pkg):
    import torch
    r = np.random.default_rng(24)
    c = verify_case(r, [1, 1], 5000, False, False, "bfloat16", None)
    c["logits"][:] = 0.5
    c["logits"][0, 77] = c["logits"][0, 4000] = 2.0
    assert np.array_equal(run_verify(pkg, c)[2], [77, 0])
    c["temperature"] = np.ones(2, np.float32)
    c["noise"][:] = 1.0
    assert np.array_equal(run_verify(pkg, c, check=False)[2], [77, 0])
    c["noise"][0, :100] = 0.0
    c["noise"][1, :10] = -1.0
    c["noise"][1, 10] = np.nan
    assert np.array_equal(run_verify(pkg, c, check=False)[2], [4000, 11])


def test_nothing_left_to_draw(pkg):
    # probabilities of the drafter that leave nothing of the target's: the next token is the target's
    r = np.random.default_rng(25)
    c = verify_case(r, [2, 2], 50, False, True, "float32", 1.0)
    c["probs"][:] = 1.0
    c["uniform"][:] = 0.999
    got = run_verify(pkg, c)
    assert np.array_equal(got[1], [1, 1]) and (got[2] >= 0).all()


def test_rows_with_strides_and_any_alignment(pkg):
    import torch
    r = np.random.default_rng(26)
    c = verify_case(r, [5] * 10, 1000, True, True, "bfloat16", 0.8)
    want = run_verify(pkg, c)
    for pad, first in ((8, 0), (1, 0), (7, 3), (24, 8)):
        def wide(a):
            a = dev(a) if not torch.is_tensor(a) else a
            x = torch.full((a.shape[0], a.shape[1] + pad), float("nan"), dtype=a.dtype, device="cuda")
            x = torch.nn.functional.pad(x, (first, 0), value=float("nan"))[:, first:first + a.shape[1]]
            x.copy_(a)
            return x
        got = run_verify(pkg, dict(c, logits=wide(c["logits"]), probs=wide(c["probs"]), noise=wide(c["noise"])))
        assert all(np.array_equal(a, b) for a, b in zip(got, want))


def test_accepted_tokens_are_distributed_as_the_target(pkg):
    # 2^15 requests with a draft each, drawn from the drafter's probabilities: the first token after the known one follows p
    import torch
    r = np.random.default_rng(27)
    n, vocab = 1 << 15, 12
    logits = r.standard_normal((1, vocab)).astype(np.float32)
    z = r.standard_normal(vocab)
    q = (np.exp(z) / np.exp(z).sum()).astype(np.float32)
    p = np.exp(logits[0].astype(np.float64))
    p /= p.sum()
    for two in (False, True):
        m = 3 if two else 2
        drafts = r.choice(vocab, (n, m - 1), p=q / q.sum(dtype=np.float64))
        tokens = np.concatenate([np.zeros((n, 1), np.int64), drafts], 1).reshape(-1)
        parent = np.tile([-1] + [0] * (m - 1), n)
        c = dict(logits=dev(np.repeat(logits, n * m, 0)), probs=dev(np.repeat(q[None], n * m, 0)), tokens=tokens, parent=parent,
                 cu=np.arange(0, n * m + 1, m), temperature=np.ones(n, np.float32), uniform=r.random(n * m).astype(np.float32),
                 noise=r.exponential(size=(n, vocab)).astype(np.float32), dtype="float32")
        path, accepted, after = run_verify(pkg, c, check=False)
        first = np.where(accepted > 1, tokens[np.maximum(path.reshape(n, m)[:, 1], 0)], after)
        count = np.bincount(first, minlength=vocab)
        # a count is within 6 standard deviations of n p (chance of any outside: 12 * 2 * 1e-9)
        assert (np.abs(count - n * p) <= 6 * np.sqrt(n * p * (1 - p))).all()
        assert (accepted > 1).mean() > 0.3


# ---------------------------------------------------------------------- together

@pytest.mark.parametrize("dtype,block", [("bfloat16", 16), ("float16", 4)])
def test_a_decoding_loop(pkg, dtype, block):
    """Plan, attention over the 8-bit cache, verification, and the write of the accepted rows, step by step and in a captured
    graph on another stream: the cache holds what writing the accepted rows one after another would have left."""
    import torch
    r = np.random.default_rng(31)
    n, page, pages, cols, heads, kv, dim, layers, vocab, most = 5, 16, 64, 12, 4, 2, 64, 2, 200, 6
    kind = getattr(torch, dtype)
    empty = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    kc, vc = (torch.zeros((layers, pages, page, kv, dim), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((layers, pages, page // block, kv), device="cuda") for _ in range(2))
    lay = pkg.make_quantised_layout(kc[0], block, dtype)
    table, ring, ring_in = empty(n, cols) - 1, torch.randperm(pages).int().cuda(), i32([0, pages])
    held, base, new = empty(n), empty(n), i32([most] * n)
    rows = n * most
    parent = i32(np.tile([-1, 0, 0, 1, 1, 2], n))
    cu, slots, pos, mask, ring_out, status = empty(n + 1), empty(rows), empty(rows), empty(rows, 1), empty(2), empty(1)
    plan = pkg.make_plan_config(n, rows, cols, page, pages, 1)
    cfg = pkg.make_attention_config(n, heads, cols, most, "tree", 1, dim ** -0.5)
    vcfg = pkg.make_verify_config(n, vocab, most, dtype)
    ws = torch.empty(pkg.ivit_tree_attention_quantised_workspace(cfg, lay), dtype=torch.uint8, device="cuda")
    q, k, v = (torch.zeros((layers, rows, h, dim), dtype=kind, device="cuda") for h in (heads, kv, kv))
    out = torch.zeros((layers, rows, heads, dim), dtype=kind, device="cuda")
    logits, probs = torch.zeros((rows, vocab), dtype=kind, device="cuda"), torch.zeros((rows, vocab), device="cuda")
    tokens, path, accepted, after = empty(rows), empty(rows), empty(n), empty(n)
    temperature, uniform, noise = torch.full((n,), 0.9, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros((n, vocab), device="cuda")

    def step():
        pkg.ivit_step_plan(plan, held, base, new, parent, ring, ring_in, table, cu, None, slots, pos, mask, ring_out, status)
        for layer in range(layers):
            pkg.ivit_tree_attention_quantised(cfg, lay, q[layer], k[layer], v[layer], kc[layer], vc[layer], ks[layer], vs[layer], table,
                                              base, cu, mask, out[layer], None, ws)
        pkg.ivit_tree_verify(vcfg, logits, probs, tokens, parent, cu, temperature, uniform, noise, path, accepted, after)
        pkg.ivit_kv_quantise(lay, k, v, path, slots, kc, vc, ks, vs)

    want = {}  # (layer, request, which) -> codes and scales of its tokens in a cache of its own, page after page
    graph, side = None, torch.cuda.Stream()
    lengths = np.zeros(n, np.int64)
    for t in range(12):
        for x in (q, k, v):
            x.copy_(torch.from_numpy(r.standard_normal(tuple(x.shape)) * 2.0 ** r.integers(-3, 4)))
        c = verify_case(r, [most] * n, vocab, True, True, dtype, 0.9)
        c["parent"] = host(parent).astype(np.int64)
        for i in range(n):
            for j in range(1, most):
                a = i * most + c["parent"][i * most + j]
                c["tokens"][i * most + j] = (c["probs"][a] / r.exponential(size=vocab)).argmax()
        logits.copy_(c["logits"])
        for x, y in ((probs, c["probs"]), (uniform, c["uniform"]), (noise, c["noise"]), (tokens, c["tokens"])):
            x.copy_(torch.from_numpy(y))
        torch.cuda.synchronize()
        if t < 4:
            step()
        elif t < 8:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()
            torch.cuda.current_stream().wait_stream(side)
        else:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step()
            graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0 and int(ws[:4].view(torch.int32)) == 0
        # the attention over what the reference's caches hold
        *found, margin = ref.verify(host(logits), c["probs"], c["tokens"], c["parent"], c["cu"], np.full(n, 0.9, np.float32),
                                    c["uniform"], host(noise), most)
        assert margin.min() > 2.0 ** -16
        assert np.array_equal(host(path), found[0]) and np.array_equal(host(accepted), found[1]) and np.array_equal(host(after), found[2])
        vis = backbone_ref.ancestors([int(p) for p in c["parent"][:most]])
        for layer in range(layers):
            mine = []
            for which in range(2):
                pair = want.setdefault((layer, which), (np.zeros((n * cols, page, kv, dim), np.uint8),
                                                        np.zeros((n * cols, page // block, kv), np.float32)))
                mine.append(ref.decode(*pair, block))
            o, _, size = backbone_ref.attention(host(q[layer]), host(k[layer]), host(v[layer]), *mine, np.arange(n * cols).reshape(n, cols),
                                                lengths, c["cu"], lambda i, m: vis, dim ** -0.5)
            bound = UNIT[dtype] * np.abs(o) + (UNIT[dtype] + 2.0 ** -14) * size + 2.0 ** -25
            assert (np.abs(host(out[layer]) - o) <= bound).all()
        # the accepted rows into the reference's caches, request after request
        for layer in range(layers):
            for which, x in ((0, k), (1, v)):
                codes, scale = want[layer, which]
                for i in range(n):
                    rows_i = found[0][i * most:i * most + found[1][i]]
                    at = i * cols * page + lengths[i] + np.arange(len(rows_i))
                    ref.quantise(codes, scale, list(host(x[layer])[rows_i]), at, block)
        lengths += found[1]
        held.copy_(base + most)
        base.copy_(torch.from_numpy(lengths))
        ring_in.copy_(ring_out)
        pages_of = host(table).astype(np.int64)
        for layer in range(layers):
            for which, (codes, scale) in enumerate(((kc, ks), (vc, vs))):
                for i in range(n):
                    for j in range(-(-int(lengths[i]) // page)):
                        m = min(page, int(lengths[i]) - j * page)
                        wc, wscale = want[layer, which]
                        assert np.array_equal(codes_of(codes[layer, pages_of[i, j]])[:m], wc[i * cols + j, :m])
                        b = -(-m // block)
                        assert np.array_equal(host(scale[layer, pages_of[i, j]])[:b], wscale[i * cols + j, :b])
    assert lengths.min() > 12
