"""The entry points of the 8-bit cache and of the verification refuse what they cannot do, before any device work, and the
restatement that the GPU tests use is what the format says.  CPU only."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2607_12287_gb300 as pkg
from tests import quantised_ref as ref
from tests.test_backbone_checks import ODD, ODD4, OK, Fake, attention_config, ints

ODD8 = 0x10008


@pytest.fixture(scope="module")
def lib():
    from paper_2607_12287_gb300 import build
    build.build()
    return pkg.load()


def layout(**change):
    lay = pkg.IvitQuantisedLayout(4, 16, 2, 64, pkg.IVIT_BF16, 8, 16 * 128, 128, 64)
    for k, v in change.items():
        setattr(lay, k, v)
    return lay


BAD_LAYOUTS = [("page_size", 0), ("page_size", 24), ("page_size", 2048), ("n_pages", 0), ("n_pages", 1 << 28), ("kv_heads", 0),
               ("kv_heads", 257), ("head_dim", 60), ("head_dim", 264), ("head_dim", 0), ("dtype", 2), ("page_stride", 12),
               ("token_stride", -128), ("head_stride", 4), ("block", 0), ("block", 3), ("block", 32), ("block", -8)]


def quantise(lib, lay, layers=2, n=3, n_src=5, **change):
    a = dict(k=OK, v=OK, rs=128, ls=640, row=OK, slot=OK, kc=OK, vc=OK, cs=8192, ks=OK, vs=OK, ss=16)
    a.update(change)
    return lib.ivit_kv_quantise(C.addressof(lay) if lay else None, layers, n, n_src, *a.values(), None)


def dequantise(lib, lay, layers=2, n=3, **change):
    a = dict(slot=OK, kc=OK, vc=OK, cs=8192, ks=OK, vs=OK, ss=16, k=OK, v=OK, rs=128, ls=640)
    a.update(change)
    return lib.ivit_kv_dequantise(C.addressof(lay) if lay else None, layers, n, *a.values(), None)


def workspace(lib, cfg, lay):
    return lib.ivit_tree_attention_quantised_workspace(C.addressof(cfg), C.addressof(lay))


def attention(lib, cfg, lay, n=9, **change):
    a = dict(q=OK, qs=512, k=OK, ks=128, v=OK, vs=128, kc=OK, vc=OK, kf=OK, vf=OK, table=OK, len=OK, cu=OK, mask=OK, out=OK, os=512,
             lse=OK, ws=OK, wb=1 << 40)
    a.update(change)
    return lib.ivit_tree_attention_quantised(C.addressof(cfg) if cfg else None, C.addressof(lay) if lay else None, n, *a.values(), None)


@pytest.mark.parametrize("field,value", BAD_LAYOUTS)
def test_layouts(lib, field, value):
    lay = layout(**{field: value})
    assert quantise(lib, lay) == dequantise(lib, lay) == attention(lib, attention_config(), lay) == pkg.IVIT_ERR_SHAPE
    assert workspace(lib, attention_config(), lay) == 0


def test_write_and_read_pointers_and_strides(lib):
    for f in (quantise, dequantise):
        assert f(lib, None) == f(lib, layout(), layers=-1) == f(lib, layout(), n=-1) == pkg.IVIT_ERR_ARG
        assert f(lib, layout(), n=(1 << 30) + 1) == pkg.IVIT_ERR_SHAPE
    assert quantise(lib, layout(), n=(1 << 20) + 1) == quantise(lib, layout(), layers=4097) == pkg.IVIT_ERR_SHAPE
    for f in (quantise, dequantise):
        for change in (dict(k=None), dict(v=None), dict(slot=None), dict(kc=None), dict(vc=None), dict(ks=None), dict(vs=None),
                       dict(k=ODD8), dict(v=ODD8), dict(kc=ODD4), dict(vc=ODD4), dict(ks=ODD), dict(vs=ODD), dict(slot=ODD), dict(rs=4),
                       dict(ls=-8), dict(cs=4), dict(ss=-1)):
            assert f(lib, layout(), **change) == pkg.IVIT_ERR_ARG, change
        assert f(lib, layout(), n=0, k=None) == f(lib, layout(), layers=0) == pkg.IVIT_OK
    assert quantise(lib, layout(), row=None) == quantise(lib, layout(), row=ODD) == pkg.IVIT_ERR_ARG
    assert quantise(lib, layout(), n_src=-1) == pkg.IVIT_ERR_ARG and quantise(lib, layout(), n_src=0, k=None) == pkg.IVIT_OK


@pytest.mark.parametrize("field,value", [("n_req", 0), ("n_req", 4097), ("heads", 0), ("heads", 7), ("heads", 258), ("max_pages", 0),
                                         ("max_pages", 1 << 27), ("max_new", 0), ("max_new", 65537), ("mask_mode", 3),
                                         ("mask_mode", -1), ("mask_words", 0), ("mask_words", 32769), ("scale", 0.0),
                                         ("scale", float("nan")), ("scale", float("inf"))])
def test_attention_configuration(lib, field, value):
    assert attention(lib, attention_config(**{field: value}), layout()) == pkg.IVIT_ERR_SHAPE
    assert workspace(lib, attention_config(**{field: value}), layout()) == 0


def test_attention_pointers_and_strides(lib):
    assert attention(lib, None, layout()) == attention(lib, attention_config(), None) == pkg.IVIT_ERR_ARG
    assert attention(lib, attention_config(), layout(), n=-1) == pkg.IVIT_ERR_ARG
    for change in (dict(q=None), dict(k=None), dict(vc=None), dict(kf=None), dict(vf=None), dict(table=None), dict(len=None), dict(cu=None),
                   dict(mask=None), dict(out=None), dict(ws=None), dict(q=ODD8), dict(kc=ODD4), dict(ws=ODD8), dict(mask=ODD), dict(lse=ODD),
                   dict(kf=ODD), dict(qs=4), dict(os=-8), dict(ks=0), dict(vs=0),
                   dict(wb=workspace(lib, attention_config(), layout()) - 1)):
        assert attention(lib, attention_config(), layout(), **change) == pkg.IVIT_ERR_ARG, change
    assert attention(lib, attention_config(), layout(), n=0, q=None) == pkg.IVIT_OK


def verify(lib, cfg, n=9, **change):
    a = dict(logits=OK, ls=1000, prob=OK, ps=1000, token=OK, parent=OK, cu=OK, temperature=OK, uniform=OK, noise=OK, ns=1000, path=OK,
             accepted=OK, next=OK)
    a.update(change)
    return lib.ivit_tree_verify(C.addressof(cfg) if cfg else None, n, *a.values(), None)


@pytest.mark.parametrize("field,value", [("n_req", 0), ("n_req", 65537), ("vocab", 0), ("vocab", (1 << 24) + 1), ("max_new", 0),
                                         ("max_new", 1025), ("dtype", 3), ("dtype", -1)])
def test_verify_configuration(lib, field, value):
    cfg = pkg.make_verify_config(3, 1000, 8)
    setattr(cfg, field, value)
    assert verify(lib, cfg) == pkg.IVIT_ERR_SHAPE
    assert "ivit_tree_verify" in pkg.ivit_last_error(None)


def test_verify_pointers_and_strides(lib):
    cfg = pkg.make_verify_config(3, 1000, 8)
    assert verify(lib, None) == verify(lib, cfg, n=-1) == pkg.IVIT_ERR_ARG
    assert verify(lib, cfg, n=(1 << 30) + 1) == pkg.IVIT_ERR_SHAPE
    for change in (dict(logits=None), dict(token=None), dict(cu=None), dict(path=None), dict(accepted=None), dict(next=None),
                   dict(uniform=None), dict(noise=None), dict(logits=ODD), dict(prob=ODD), dict(token=ODD), dict(noise=ODD), dict(path=ODD),
                   dict(ls=999), dict(ps=999), dict(ns=999)):
        assert verify(lib, cfg, **change) == pkg.IVIT_ERR_ARG, change
    assert verify(lib, pkg.make_verify_config(3, 1000, 8, "float32"), logits=0x10002) == pkg.IVIT_ERR_ARG
    assert verify(lib, cfg, n=0, cu=None) == pkg.IVIT_ERR_ARG


# ---------------------------------------------------------------------- binding

def f8(*shape, strides=None):
    return Fake(shape, torch.float8_e4m3fn, strides)


def f32(*shape, strides=None):
    return Fake(shape, torch.float32, strides)


def bf(*shape, strides=None):
    return Fake(shape, torch.bfloat16, strides)


def test_layout_of_a_tensor():
    lay = pkg.make_quantised_layout(f8(4, 16, 2, 64, strides=(2048, 64, 1024, 1)), 8, "float16")
    assert (lay.n_pages, lay.page_size, lay.kv_heads, lay.head_dim, lay.block) == (4, 16, 2, 64, 8)
    assert (lay.page_stride, lay.token_stride, lay.head_stride, lay.dtype) == (2048, 64, 1024, pkg.IVIT_FP16)
    for cache, exc in ((f8(4, 16, 128), ValueError), (f8(4, 16, 2, 64, strides=(2048, 128, 1, 2)), ValueError),
                       (bf(4, 16, 2, 64), TypeError), (Fake((4, 16, 2, 64), torch.uint8), TypeError)):
        with pytest.raises(exc):
            pkg.make_quantised_layout(cache, 8)
    with pytest.raises(TypeError):
        pkg.make_quantised_layout(f8(4, 16, 2, 64), 8, "float32")
    with pytest.raises(TypeError):
        pkg.make_verify_config(1, 10, 1, "float64")


def test_binding_rejects_tensors_it_would_misread(monkeypatch):
    monkeypatch.setattr(pkg, "load", lambda *a: pytest.fail("library reached"))
    monkeypatch.setattr(pkg, "_stream", lambda s: 0)
    one = f8(4, 16, 2, 64)
    lay = pkg.make_quantised_layout(one, 8)
    caches, scales = f8(3, 4, 16, 2, 64), f32(3, 4, 2, 2)
    good = dict(k=bf(3, 6, 2, 64), v=bf(3, 6, 2, 64), rows=ints(4), slots=ints(4), k_cache=caches, v_cache=caches, k_scale=scales,
                v_scale=scales)
    wrong = [(dict(k_cache=f8(2, 4, 16, 2, 64)), ValueError), (dict(v_cache=f8(3, 4, 16, 1, 64)), ValueError),
             (dict(k_cache=bf(3, 4, 16, 2, 64)), TypeError), (dict(v_cache=None), TypeError), (dict(k_scale=f32(3, 4, 1, 2)), ValueError),
             (dict(v_scale=f32(2, 4, 2, 2)), ValueError), (dict(k_scale=bf(3, 4, 2, 2)), TypeError), (dict(v_scale=None), TypeError),
             (dict(k_scale=f32(3, 4, 2, 2, strides=(32, 8, 4, 2))), ValueError),
             (dict(v_cache=f8(3, 4, 16, 2, 64, strides=(16384, 2048, 128, 64, 1))), ValueError),
             (dict(v=bf(3, 6, 2, 64, strides=(1536, 256, 64, 1))), ValueError), (dict(k=Fake((3, 6, 2, 64), torch.float16)), TypeError),
             (dict(k=torch.zeros(3, 6, 2, 64, dtype=torch.bfloat16)), ValueError)]
    for change, exc in wrong + [(dict(k=bf(6, 2, 64)), ValueError), (dict(v=bf(3, 5, 2, 64)), ValueError), (dict(slots=ints(3)), ValueError),
                                (dict(rows=None), TypeError)]:
        with pytest.raises(exc):
            pkg.ivit_kv_quantise(lay, **{**good, **change})
    del good["rows"]
    for change, exc in wrong + [(dict(slots=ints(5)), ValueError), (dict(slots=None), TypeError)]:
        with pytest.raises(exc):
            pkg.ivit_kv_dequantise(lay, **{**good, "slots": ints(6), **change})
    acfg = pkg.make_attention_config(2, 8, 3, 4, "tree", 1, 0.125)
    good = dict(q=bf(5, 8, 64), k_new=bf(5, 2, 64), v_new=bf(5, 2, 64), k_cache=one, v_cache=one, k_scale=f32(4, 2, 2), v_scale=f32(4, 2, 2),
                table=ints(2, 3), lengths=ints(2), cu_rows=ints(3), mask=ints(5, 1), out=bf(5, 8, 64), lse=f32(5, 8),
                workspace=Fake((1 << 28,), torch.uint8))
    for change, exc in ((dict(table=ints(2, 2)), ValueError), (dict(lengths=Fake((2,), torch.int64)), TypeError),
                        (dict(cu_rows=ints(2)), ValueError), (dict(mask=ints(4, 1)), ValueError), (dict(out=bf(4, 8, 64)), ValueError),
                        (dict(lse=Fake((5, 8), torch.float16)), TypeError), (dict(k_new=bf(5, 2, 32)), ValueError),
                        (dict(k_cache=f8(4, 8, 2, 64)), ValueError), (dict(v_cache=bf(4, 16, 2, 64)), TypeError),
                        (dict(k_scale=f32(4, 2, 1)), ValueError), (dict(v_scale=None), TypeError), (dict(k_cache=OK), TypeError)):
        with pytest.raises(exc):
            pkg.ivit_tree_attention_quantised(acfg, lay, **{**good, **change})
    vcfg = pkg.make_verify_config(2, 100, 4)
    good = dict(logits=bf(5, 100), draft_probs=f32(5, 100), tokens=ints(5), parent=ints(5), cu_rows=ints(3), temperature=f32(2),
                uniform=f32(5), noise=f32(2, 100), path=ints(5), accepted=ints(2), next_token=ints(2))
    for change, exc in ((dict(logits=bf(500)), ValueError), (dict(logits=None), ValueError), (dict(logits=bf(5, 99)), ValueError),
                        (dict(logits=f32(5, 100)), TypeError), (dict(logits=bf(5, 100, strides=(1, 5))), ValueError),
                        (dict(draft_probs=f32(4, 100)), ValueError), (dict(draft_probs=bf(5, 100)), TypeError), (dict(tokens=ints(4)), ValueError),
                        (dict(parent=ints(4)), ValueError), (dict(cu_rows=ints(2)), ValueError), (dict(temperature=f32(1)), ValueError),
                        (dict(uniform=f32(4)), ValueError), (dict(noise=f32(1, 100)), ValueError), (dict(noise=OK), TypeError),
                        (dict(path=ints(4)), ValueError), (dict(accepted=ints(1)), ValueError), (dict(next_token=ints(1)), ValueError),
                        (dict(logits=torch.zeros(5, 100, dtype=torch.bfloat16)), ValueError)):
        with pytest.raises(exc):
            pkg.ivit_tree_verify(vcfg, **{**good, **change})


class On(Fake):
    """A tensor of a given device."""
    is_cuda = True

    def __init__(self, t, device):
        super().__init__(t.shape, t.dtype, t.stride())
        self.device = torch.device("cuda", device)

    def get_device(self):
        return self.device.index


class Kind(On):
    """One of a type of its own, as parameters are."""


@pytest.mark.parametrize("given,kind", [(True, On), (False, On), (True, Kind)])
def test_binding_rejects_any_tensor_of_another_device(monkeypatch, given, kind):
    # each tensor of each call by itself, whether the call gives its stream or not
    reached = []
    pkg._tensor_type()
    monkeypatch.setattr(pkg, "load", lambda *a: reached.append(1) or pytest.fail("library reached"))
    monkeypatch.setattr(pkg, "_Tensor", On)
    monkeypatch.setitem(pkg._dtypes, "tensor", On)
    monkeypatch.setattr(pkg, "_current", [lambda device: 0, lambda: 1])
    stream = 0 if given else None
    lay, one = pkg.make_quantised_layout(f8(4, 16, 2, 64), 8), f8(4, 16, 2, 64)
    caches, scales = f8(3, 4, 16, 2, 64), f32(3, 4, 2, 2)
    layers = dict(k=bf(3, 6, 2, 64), v=bf(3, 6, 2, 64), slots=ints(6), k_cache=caches, v_cache=caches, k_scale=scales, v_scale=scales)
    acfg, vcfg = pkg.make_attention_config(2, 8, 3, 4, "tree", 1, 0.125), pkg.make_verify_config(2, 100, 4)
    calls = [(lambda **t: pkg.ivit_kv_quantise(lay, stream=stream, **t), dict(layers, rows=ints(6))),
             (lambda **t: pkg.ivit_kv_dequantise(lay, stream=stream, **t), layers),
             (lambda **t: pkg.ivit_tree_attention_quantised(acfg, lay, stream=stream, **t),
              dict(q=bf(5, 8, 64), k_new=bf(5, 2, 64), v_new=bf(5, 2, 64), k_cache=one, v_cache=one, k_scale=f32(4, 2, 2),
                   v_scale=f32(4, 2, 2), table=ints(2, 3), lengths=ints(2), cu_rows=ints(3), mask=ints(5, 1), out=bf(5, 8, 64),
                   lse=f32(5, 8), workspace=Fake((1 << 28,), torch.uint8))),
             (lambda **t: pkg.ivit_tree_verify(vcfg, stream=stream, **t),
              dict(logits=bf(5, 100), draft_probs=f32(5, 100), tokens=ints(5), parent=ints(5), cu_rows=ints(3), temperature=f32(2),
                   uniform=f32(5), noise=f32(2, 100), path=ints(5), accepted=ints(2), next_token=ints(2)))]
    for f, tensors in calls:
        for name in tensors:
            with pytest.raises(ValueError, match=f"^{name}: tensor on cuda:0, the current device is cuda:1"):
                f(**{k: kind(t, 0 if k == name else 1) for k, t in tensors.items()})
        with pytest.raises(pytest.fail.Exception):  # (all of the current one)
            f(**{k: kind(t, 1) for k, t in tensors.items()})
    assert len(reached) == len(calls)


def test_restated_codes_are_the_formats():
    codes = np.arange(256, dtype=np.uint8)
    assert np.array_equal(ref.VALUES, torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    r = np.random.default_rng(0)
    x = np.concatenate([r.standard_normal(20000) * 2.0 ** r.integers(-12, 8, 20000), ref.VALUES[:126], (ref.VALUES[:126] + ref.VALUES[1:127]) / 2])
    x = np.clip(np.concatenate([x, -x]), -448, 448).astype(np.float32)
    assert np.array_equal(ref.encode(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_restated_verification_accepts_as_the_target_would():
    # drafts drawn from the drafter's probabilities: the first token after the known one follows the target's, by counting
    r = np.random.default_rng(1)
    n, vocab = 4000, 5
    logits = r.standard_normal(vocab).astype(np.float32)
    p = np.exp(logits.astype(np.float64))
    p /= p.sum()
    q = np.array([0.5, 0.2, 0.1, 0.1, 0.1], np.float32)
    tokens = np.stack([np.zeros(n, np.int64), r.choice(vocab, n, p=q / q.sum(dtype=np.float64)), r.choice(vocab, n, p=q / q.sum(dtype=np.float64))], 1)
    path, accepted, after, _ = ref.verify(np.repeat(logits[None], 3 * n, 0), np.repeat(q[None], 3 * n, 0), tokens.reshape(-1),
                                          np.tile([-1, 0, 0], n), np.arange(0, 3 * n + 1, 3), np.ones(n, np.float32),
                                          r.random(3 * n).astype(np.float32), r.exponential(size=(n, vocab)).astype(np.float32), 3)
    first = np.where(accepted > 1, tokens.reshape(-1)[np.maximum(path.reshape(n, 3)[:, 1], 0)], after)
    count = np.bincount(first, minlength=vocab)
    assert (np.abs(count - n * p) <= 6 * np.sqrt(n * p * (1 - p))).all()
