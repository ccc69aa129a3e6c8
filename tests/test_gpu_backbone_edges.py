"""The language backbone's operators at the edges of what their arguments may be.

Error bounds as in test_gpu_backbone.py."""
import numpy as np
import pytest

from tests import backbone_ref as ref
from tests.test_gpu_backbone import attention_case, close_rotation, dev, host, i32, rope_case, run_attention, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_12287_gb300 as p
    p.load()
    return p


# --------------------------------------------------------------------- rotation

@pytest.mark.parametrize("rows,heads,kv,dim,rot,inter,weights,dtype", [
    (1, 4, 2, 128, 128, False, "qk", "bfloat16"), (3, 8, 2, 128, 64, True, "qk", "float16"), (5, 6, 2, 64, 64, False, "qk", "bfloat16"),
    (5, 3, 3, 72, 72, False, "q", "bfloat16"), (7, 2, 1, 40, 40, True, "k", "float16"), (1, 2, 2, 8, 0, False, "qk", "float16"),
    (4, 2, 1, 256, 256, False, "qk", "bfloat16"), (4001, 8, 2, 96, 96, False, "qk", "bfloat16"),
])
def test_gradients_without_eps(pkg, rows, heads, kv, dim, rot, inter, weights, dtype):
    # eps = 0 and row counts that leave lanes of the last warp without a row
    import torch
    r = np.random.default_rng(rows + dim)
    c = rope_case(r, rows, heads, kv, dim, rot, 1, dtype, weights)
    cfg = pkg.make_rope_config(heads, kv, dim, rot, 1, inter, 0.0, dtype)
    g = [dev(r.standard_normal((rows, m, dim)).astype(np.float32), dtype) for m in (heads, kv)]
    d = [torch.full_like(t, float("nan")) for t in g]
    dw = [torch.full((dim,), float("nan"), device="cuda") if x in weights else None for x in "qk"]
    ws = torch.full((pkg.ivit_qk_norm_rope_backward_workspace(cfg),), 255, dtype=torch.uint8, device="cuda")
    freq, axis = (dev(c["freq"]), i32(c["axis"])) if rot else (None, None)
    pkg.ivit_qk_norm_rope_backward(cfg, *g, c["q"], c["k"], *c["w"], i32(c["pos"]), freq, axis, *d, *dw, ws)
    for x, w, gx, dx, dwx, name in zip((c["q"], c["k"]), c["w"], g, d, dw, "qk"):
        xs, gs = host(x), host(gx)
        want, want_w = ref.rope_backward(gs, xs, None if w is None else host(w), c["pos"], c["freq"], c["axis"], rot, inter, 0.0)
        rms = np.sqrt((xs ** 2).mean(-1, keepdims=True)) if w is not None else 1.0
        close_rotation(dx, want, np.maximum(np.abs(gs), 2 * np.abs(gs) / rms), dtype, "d" + name)
        if w is not None:
            y = ref.rope(gs, None, -c["pos"], c["freq"], c["axis"], rot, inter, 0)
            size = np.abs(y * xs / rms).sum((0, 1))
            assert (np.abs(host(dwx) - want_w) <= 2.0 ** -16 * size + 1e-6).all(), name


@pytest.mark.parametrize("axes", [1, 2, 3, 4])
def test_axes_that_are_none_count_as_the_first(pkg, axes):
    import torch
    r = np.random.default_rng(axes)
    rows, heads, kv, dim = 9, 4, 2, 64
    c = rope_case(r, rows, heads, kv, dim, dim, axes, "float16", "")
    cfg = pkg.make_rope_config(heads, kv, dim, dim, axes, False, 1e-6, "float16")
    odd = r.choice([-2 ** 31, -1, 0, 1, 2, 3, 4, 5, 100, 2 ** 31 - 1], dim // 2)
    odd[:4] = [2, 3, 1, -1]
    results = []
    for axis in (odd, np.where((odd >= 0) & (odd < axes), odd, 0)):
        args = (i32(c["pos"]), dev(c["freq"]), i32(axis))
        out, back = ([torch.empty((rows, m, dim), dtype=torch.float16, device="cuda") for m in (heads, kv)] for _ in range(2))
        pkg.ivit_qk_norm_rope(cfg, c["q"], c["k"], None, None, None, *args, *out)
        pkg.ivit_qk_norm_rope_backward(cfg, c["q"], c["k"], c["q"], c["k"], None, None, *args, *back)
        results.append(out + back)
    for a, b in zip(*results):
        assert torch.equal(a, b)


# -------------------------------------------------------------------- attention

@pytest.mark.parametrize("heads,kv,dim,most_new,n,dtype,mask", [
    (2, 2, 64, 90, 500, "bfloat16", "causal"), (4, 2, 80, 45, 400, "float16", "causal"), (2, 2, 128, 60, 400, "bfloat16", "causal"),
    (2, 1, 256, 30, 400, "float16", "causal"), (2, 2, 72, 250, 100, "bfloat16", "all"), (4, 4, 96, 40, 400, "float16", "causal"),
])
def test_values_that_are_not_finite_in_every_tile(pkg, heads, kv, dim, most_new, n, dtype, mask):
    # prompts over empty caches: a CTA goes through several tiles of rows, some with warps of padding rows alone, and
    # each tile's first keys hold infinities and NaN that some of its rows see
    r = np.random.default_rng(dim)
    new = r.integers(max(1, most_new // 2), most_new + 1, n)
    c = attention_case(r, [0] * n, new, heads, kv, dim, 8, dtype)
    first, last = i32(c["cu"][:-1]).long(), i32(c["cu"][1:] - 1).long()
    c["v"][first, :, 3] = float("inf")
    c["v"][(first + last) // 2, 0, dim - 1] = float("-inf")
    c["v"][last, kv - 1, 7] = float("nan")
    out, _ = run_attention(pkg, c, mask, lse=False, check=False, max_new=most_new)
    sees = {"causal": lambda i, m: np.tril(np.ones((m, m), bool)), "all": lambda i, m: np.ones((m, m), bool)}[mask]
    with np.errstate(invalid="ignore"):
        want, _, size = ref.attention(host(c["q"]), host(c["k"]), host(c["v"]), host(c["kc"]), host(c["vc"]), c["table"],
                                      c["lengths"], c["cu"], sees, dim ** -0.5)
    got, finite = host(out), np.isfinite(want)
    np.testing.assert_array_equal(got[~finite], want[~finite])
    u = ref.UNIT[dtype]
    bound = u * np.abs(want) + (u + 2.0 ** -14) * size + 2.0 ** -25
    assert (np.abs(got[finite] - want[finite]) <= bound[finite]).all()


@pytest.mark.parametrize("heads", [4, 16])  # (mma.sync, tcgen05)
def test_row_offsets_out_of_range(pkg, heads):
    # a request whose offsets are no range of rows has none; rows of no request are left as they are
    import torch
    c = attention_case(np.random.default_rng(heads), [40, 30], [5, 7], heads, 2, 64, 16, "bfloat16")
    want, want_lse = run_attention(pkg, dict(c, cu=np.array([0, 5, 5])), "causal", check=False, max_new=7)
    assert bool(torch.isfinite(want[:5]).all()) and bool(torch.isnan(want[5:]).all())
    far = 2 ** 31
    for cu in ([0, 5, -far], [0, 5, -1], [0, 5, 3], [-far, 5, -7], [-1, 5, -far]):
        out, lse = run_attention(pkg, dict(c, cu=np.array(cu)), "causal", check=False, max_new=7)
        for a, b in ((out, want), (lse, want_lse)):
            assert torch.equal(a[:5], b[:5]) and bool(torch.isnan(a[5:]).all()), cu
    # beyond the last row: up to it
    all_rows, _ = run_attention(pkg, c, "causal", max_new=7)
    out, _ = run_attention(pkg, dict(c, cu=np.array([0, 5, far - 1])), "causal", check=False, max_new=7)
    assert torch.equal(out, all_rows)


@pytest.mark.parametrize("heads,kv,dim,length,new,page,dtype", [
    (4, 1, 64, 160, 4, 16, "bfloat16"), (4, 1, 64, 160, 4, 16, "float16"), (16, 16, 128, 64, 2, 16, "bfloat16"),
    (8, 2, 72, 3000, 2, 16, "bfloat16"), (8, 2, 96, 3000, 4, 8, "float16"), (4, 2, 256, 700, 8, 32, "bfloat16"),
    (6, 1, 256, 700, 2, 4, "float16"), (8, 2, 64, 200, 8, 4, "bfloat16"), (8, 2, 80, 3000, 6, 4, "float16"),
    (16, 1, 128, 130, 2, 1, "bfloat16"), (4, 2, 256, 1000, 16, 2, "bfloat16"),  # (17 to 32 rows on small pages: tiles of 32)
])
def test_probabilities_keep_both_terms(pkg, heads, kv, dim, length, new, page, dtype):
    # Up to 16 rows per key head (32 on small pages) probabilities enter the product with V as two 16-bit terms.  Keys of
    # two kinds take turns, with scores q0 and q0 - q1 and values c and -c, all exact: the output nearly vanishes and with
    # it its own rounding, while an error of the second kind's probability adds up over all keys.  Bound, with w = sum p |v| /
    # sum p: u |o| for the output's rounding, u^2 w for the second term's, 2^-17 w for fp32 (the exponent, of at most
    # 16, to 2^-20; exp2 and the sums).
    import torch
    r = np.random.default_rng(dim + new)
    c = attention_case(r, [length], [new], heads, kv, dim, page, dtype)
    values = r.choice([-1.5, -1.0, -0.75, 0.75, 1.0, 1.5], (kv, dim))

    def fill(k, v, at, t):
        kind = (t % 2)[:, None]
        keys = np.zeros((len(t), kv, dim), np.float32)
        keys[..., 0], keys[..., 1] = 1, -kind
        k[at], v[at] = dev(keys, dtype), dev((values * (1 - 2 * kind[..., None])).astype(np.float32), dtype)

    t = np.arange(length)
    fill(c["kc"], c["vc"], (i32(c["table"][0][t // page]).long(), i32(t % page).long()), t)
    fill(c["k"], c["v"], slice(0, new), np.arange(new))
    q = np.zeros((new, heads, dim), np.float32)
    q[..., 0], q[..., 1] = r.uniform(-2, 2, (new, heads)), r.uniform(0.01, 0.06, (new, heads))
    c["q"] = dev(q, dtype)
    out, _ = run_attention(pkg, c, "all", scale=1.0, check=False)
    p = np.exp(-host(c["q"])[..., 1:2])
    v = np.repeat(values, heads // kv, 0)[None]
    u = ref.UNIT[dtype]
    want, size = v * (1 - p) / (1 + p), np.abs(v) + 0 * p
    bound = u * np.abs(want) + (u * u + 2.0 ** -17) * size
    # (one term would not do, for most rows)
    one = torch.from_numpy(p).to(c["q"].dtype).double().numpy()
    assert ((np.abs(v * (1 - one) / (1 + p) - want) > bound).any(-1)).mean() > 0.5
    assert (np.abs(host(out) - want) <= bound).all()


@pytest.mark.parametrize("heads,kv,dim,lengths,new,page,dtype", [
    (129, 1, 64, [70, 3], [1, 2], 16, "bfloat16"), (256, 1, 72, [100], [3], 16, "float16"), (200, 1, 128, [0, 65], [2, 1], 8, "bfloat16"),
    (130, 1, 256, [40], [1], 32, "float16"),
])
@pytest.mark.parametrize("mask", ["causal", "all", "tree"])
def test_groups_above_128_heads(pkg, heads, kv, dim, lengths, new, page, dtype, mask):
    r = np.random.default_rng(heads)
    c = attention_case(r, lengths, new, heads, kv, dim, page, dtype)
    run_attention(pkg, c, mask, trees(r, new) if mask == "tree" else None)


# ------------------------------------------------------------------------- plan

@pytest.mark.parametrize("free,status", [(2, 0), (3, 8), (4, 8)])
def test_plan_refuses_pages_that_are_free_and_held(pkg, free, status):
    # one request takes two pages, another returns two: with three free ones of four a page is on both sides, and the
    # returned ids would go where the taken ones are read
    import torch
    ring, table = torch.tensor([3, 0, 0, 2]), torch.tensor([[-1, -1, -1], [0, 1, -1]])
    cfg = pkg.make_plan_config(2, 32, 3, 16, 4)
    out = lambda n: torch.full((n,), -77, dtype=torch.int32, device="cuda")
    ring_dev, table_dev, cu, slots, ring_out, why = ring.int().cuda(), table.int().cuda(), out(3), out(32), out(2), out(1)
    pkg.ivit_step_plan(cfg, i32([0, 32]), i32([0, 0]), i32([32, 0]), None, ring_dev, i32([3, free]), table_dev, cu, None, slots,
                       None, None, ring_out, why)
    assert int(why) == status
    if status:
        assert torch.equal(ring_dev.cpu(), ring.int()) and torch.equal(table_dev.cpu(), table.int())
        assert ring_out.tolist() == [3, free] and cu.tolist() == [0, 0, 0] and slots.tolist() == [-1] * 32
    else:
        assert table_dev[0].tolist() == [2, 3, -1] and ring_dev.tolist() == [3, 0, 1, 2] and ring_out.tolist() == [1, 2]
        assert cu.tolist() == [0, 32, 32] and slots.tolist() == list(range(32, 48)) + list(range(48, 64))

def test_plans_of_many_requests_from_two_threads(pkg):
    # calls that need more shared memory than is allowed by default, of different sizes, at the same time
    import threading

    import torch
    failed = []

    def plans(n):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                cfg = pkg.make_plan_config(n, n, 1, 16, n)
                zeros = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
                ring, table, status = torch.arange(n, dtype=torch.int32, device="cuda"), zeros(n, 1), zeros(1)
                held, new, ring_in, cu, slots, ring_out = zeros(n), zeros(n) + 1, i32([0, n]), zeros(n + 1), zeros(n), zeros(2)
                stream.synchronize()
                for _ in range(3000):
                    pkg.ivit_step_plan(cfg, held, held, new, None, ring, ring_in, table, cu, None, slots, None, None, ring_out,
                                       status)
                stream.synchronize()
                assert int(status) == 0 and int(cu[n]) == n
        except Exception as e:  # noqa: BLE001 (a thread's exception is the test's)
            failed.append(repr(e))

    threads = [threading.Thread(target=plans, args=(n,)) for n in (4000, 4096)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
