"""The language backbone's entry points refuse what they cannot do, before any device work: bad
configurations, null and misaligned pointers (C ABI, raw addresses) and tensors that the kernels
would misread (Python binding).  CPU only."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2607_12287_gb300 as pkg
from tests.test_binding_checks import FakeCuda

OK, ODD4, ODD = 0x10000, 0x10004, 0x10001


@pytest.fixture(scope="module")
def lib():
    from paper_2607_12287_gb300 import build
    build.build()
    return pkg.load()


class Fake(FakeCuda):
    """A device tensor with strides."""

    def __init__(self, shape, dtype, strides=None):
        dense = [int(np.prod(shape[i + 1:])) for i in range(len(shape))]
        super().__init__(shape, dtype, strides is None or list(strides) == dense)
        self._strides = tuple(dense if strides is None else strides)

    def stride(self):
        return self._strides

    def data_ptr(self):
        return OK

    def __getitem__(self, i):
        assert i == 0
        return Fake(self.shape[1:], self.dtype, self._strides[1:])


def layout(**change):
    lay = pkg.IvitCacheLayout(4, 16, 2, 64, pkg.IVIT_BF16, 0, 16 * 128, 128, 64)
    for k, v in change.items():
        setattr(lay, k, v)
    return lay


BAD_LAYOUTS = [("page_size", 0), ("page_size", 24), ("page_size", 2048), ("n_pages", 0), ("n_pages", 1 << 28), ("kv_heads", 0),
               ("kv_heads", 257), ("head_dim", 60), ("head_dim", 264), ("head_dim", 0), ("dtype", 2), ("page_stride", 12),
               ("token_stride", -128), ("head_stride", 4)]


def plan(lib, cfg, **null_or_odd):
    names = ["held", "base", "new", "parent", "ring", "ring_in", "table", "cu", "req", "slot", "pos", "mask", "ring_out", "status"]
    ptr = {n: OK + 64 * i for i, n in enumerate(names)}
    ptr.update(null_or_odd)
    return lib.ivit_step_plan(C.addressof(cfg) if cfg else None, *[ptr[n] for n in names], None)


@pytest.mark.parametrize("field,value", [("n_req", 0), ("n_req", 4097), ("max_rows", -1), ("max_rows", 262145), ("max_pages", 0),
                                         ("max_pages", 262145), ("page_size", 3), ("page_size", 2048), ("n_pages", 0),
                                         ("n_pages", 1 << 27), ("mask_words", -1), ("mask_words", 32769)])
def test_plan_configuration(lib, field, value):
    cfg = pkg.make_plan_config(4, 10, 8, 16, 100, 1)
    setattr(cfg, field, value)
    assert plan(lib, cfg) == pkg.IVIT_ERR_SHAPE
    assert "ivit_step_plan" in pkg.ivit_last_error(None)


def test_plan_pointers(lib):
    cfg = pkg.make_plan_config(4, 10, 8, 16, 100, 1)
    assert plan(lib, None) == pkg.IVIT_ERR_ARG
    for n in ("held", "base", "new", "ring", "ring_in", "table", "cu", "slot", "ring_out", "status"):
        assert plan(lib, cfg, **{n: None}) == pkg.IVIT_ERR_ARG, n
    for n in ("held", "parent", "mask", "ring_out", "req", "pos"):
        assert plan(lib, cfg, **{n: ODD}) == pkg.IVIT_ERR_ARG, n
    assert plan(lib, cfg, ring_out=OK, ring_in=OK) == pkg.IVIT_ERR_ARG


def rope(lib, cfg, lay=None, n=3, **change):
    a = dict(q=OK, qs=512, k=OK, ks=512, v=OK if lay else None, vs=512, qw=OK, kw=OK, pos=OK, ps=3, freq=OK, axis=OK, qo=OK,
             qos=512, ko=OK, kos=512, lay=C.addressof(lay) if lay else None, kc=OK if lay else None, vc=OK if lay else None,
             slot=OK if lay else None)
    a.update(change)
    return lib.ivit_qk_norm_rope(C.addressof(cfg) if cfg else None, n, *a.values(), None)


def rope_backward(lib, cfg, n=3, **change):
    a = dict(gq=OK, gqs=512, gk=OK, gks=512, q=OK, qs=512, k=OK, ks=512, qw=OK, kw=OK, pos=OK, ps=3, freq=OK, axis=OK, dq=OK,
             dqs=512, dk=OK, dks=512, dqw=OK, dkw=OK, ws=OK, wb=1 << 40)
    a.update(change)
    return lib.ivit_qk_norm_rope_backward(C.addressof(cfg) if cfg else None, n, *a.values(), None)


@pytest.mark.parametrize("field,value", [("heads", 0), ("heads", 257), ("kv_heads", 0), ("head_dim", 12), ("head_dim", 264),
                                         ("rot_dim", -8), ("rot_dim", 72), ("rot_dim", 20), ("n_axes", 0), ("n_axes", 5),
                                         ("interleaved", 2), ("dtype", 2), ("eps", -1.0), ("eps", float("nan"))])
def test_rope_configuration(lib, field, value):
    cfg = pkg.make_rope_config(8, 2, 64)
    setattr(cfg, field, value)
    assert rope(lib, cfg) == pkg.IVIT_ERR_SHAPE
    assert rope_backward(lib, cfg) == pkg.IVIT_ERR_SHAPE
    assert lib.ivit_qk_norm_rope_backward_workspace(C.addressof(cfg)) == 0


def test_rope_pointers_and_strides(lib):
    cfg = pkg.make_rope_config(8, 2, 64)
    assert rope(lib, None) == rope(lib, cfg, n=-1) == pkg.IVIT_ERR_ARG
    assert rope_backward(lib, None) == rope_backward(lib, cfg, n=-1) == pkg.IVIT_ERR_ARG
    for change in (dict(q=None), dict(k=None), dict(pos=None), dict(freq=None), dict(axis=None), dict(qo=None), dict(ko=None),
                   dict(v=OK), dict(kc=OK), dict(slot=OK), dict(q=ODD4), dict(kw=ODD4), dict(freq=ODD), dict(qs=516), dict(kos=-8),
                   dict(ps=-1)):
        assert rope(lib, cfg, **change) == pkg.IVIT_ERR_ARG, change
    for change in (dict(v=None), dict(kc=None), dict(vc=None), dict(slot=None), dict(vs=4), dict(vc=ODD4), dict(slot=ODD)):
        assert rope(lib, cfg, layout(), **change) == pkg.IVIT_ERR_ARG, change
    for change in (dict(gq=None), dict(dk=None), dict(q=None), dict(ws=None), dict(dqw=OK, qw=None), dict(gq=ODD4), dict(ws=ODD4),
                   dict(dqs=12), dict(dkw=ODD), dict(gks=-8),
                   dict(wb=lib.ivit_qk_norm_rope_backward_workspace(C.addressof(cfg)) - 1)):
        assert rope_backward(lib, cfg, **change) == pkg.IVIT_ERR_ARG, change
    assert rope(lib, cfg, n=0, q=None) == pkg.IVIT_OK


@pytest.mark.parametrize("field,value", BAD_LAYOUTS)
def test_cache_layouts(lib, field, value):
    lay = layout(**{field: value})
    assert rope(lib, pkg.make_rope_config(8, 2, 64), lay) == pkg.IVIT_ERR_SHAPE
    assert attention(lib, attention_config(), lay) == pkg.IVIT_ERR_SHAPE
    assert workspace(lib, attention_config(), lay) == 0
    assert write(lib, lay) == pkg.IVIT_ERR_SHAPE


def test_cache_of_other_heads(lib):
    for change in (dict(kv_heads=4), dict(head_dim=128), dict(dtype=pkg.IVIT_FP16)):
        assert rope(lib, pkg.make_rope_config(8, 2, 64), layout(**change)) == pkg.IVIT_ERR_SHAPE


def attention_config(**change):
    cfg = pkg.make_attention_config(3, 8, 10, 5, "tree", 1, 0.125)
    for k, v in change.items():
        setattr(cfg, k, v)
    return cfg


def workspace(lib, cfg, lay):
    return lib.ivit_tree_attention_workspace(C.addressof(cfg), C.addressof(lay))


def attention(lib, cfg, lay, n=9, **change):
    a = dict(q=OK, qs=512, k=OK, ks=128, v=OK, vs=128, kc=OK, vc=OK, table=OK, len=OK, cu=OK, mask=OK, out=OK, os=512, lse=OK, ws=OK, wb=1 << 40)
    a.update(change)
    return lib.ivit_tree_attention(C.addressof(cfg) if cfg else None, C.addressof(lay) if lay else None, n, *a.values(), None)


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
    for change in (dict(q=None), dict(k=None), dict(vc=None), dict(table=None), dict(len=None), dict(cu=None), dict(mask=None),
                   dict(out=None), dict(ws=None), dict(q=ODD4), dict(kc=ODD4), dict(ws=ODD4), dict(mask=ODD), dict(lse=ODD),
                   dict(qs=4), dict(os=-8), dict(ks=0), dict(vs=0),
                   dict(wb=workspace(lib, attention_config(), layout()) - 1)):
        assert attention(lib, attention_config(), layout(), **change) == pkg.IVIT_ERR_ARG, change
    assert attention(lib, attention_config(), layout(), n=0, q=None) == pkg.IVIT_OK


def write(lib, lay, layers=2, n=3, n_src=5, **change):
    a = dict(k=OK, v=OK, rs=128, ls=640, row=OK, slot=OK, kc=OK, vc=OK, cs=8192)
    a.update(change)
    return lib.ivit_kv_write(C.addressof(lay) if lay else None, layers, n, n_src, *a.values(), None)


def test_write_pointers_and_strides(lib):
    assert write(lib, None) == write(lib, layout(), layers=-1) == write(lib, layout(), n=-1) == pkg.IVIT_ERR_ARG
    for change in (dict(k=None), dict(row=None), dict(slot=None), dict(vc=None), dict(k=ODD4), dict(kc=ODD4), dict(slot=ODD),
                   dict(rs=4), dict(ls=-8), dict(cs=4)):
        assert write(lib, layout(), **change) == pkg.IVIT_ERR_ARG, change
    assert write(lib, layout(), n=0, k=None) == write(lib, layout(), layers=0) == pkg.IVIT_OK


# ---------------------------------------------------------------------- binding

def bf(*shape, strides=None):
    return Fake(shape, torch.bfloat16, strides)


def ints(*shape):
    return Fake(shape, torch.int32)


def test_cache_layout_of_a_tensor():
    lay = pkg.make_cache_layout(bf(4, 16, 2, 64, strides=(2048, 64, 1024, 1)))
    assert (lay.n_pages, lay.page_size, lay.kv_heads, lay.head_dim) == (4, 16, 2, 64)
    assert (lay.page_stride, lay.token_stride, lay.head_stride, lay.dtype) == (2048, 64, 1024, pkg.IVIT_BF16)
    with pytest.raises(ValueError):
        pkg.make_cache_layout(bf(4, 16, 128))
    with pytest.raises(ValueError):
        pkg.make_cache_layout(bf(4, 16, 2, 64, strides=(2048, 128, 1, 2)))
    with pytest.raises(TypeError):
        pkg.make_cache_layout(Fake((4, 16, 2, 64), torch.float32))


def test_binding_rejects_tensors_it_would_misread(monkeypatch):
    monkeypatch.setattr(pkg, "load", lambda *a: pytest.fail("library reached"))
    cfg = pkg.make_rope_config(8, 2, 64, n_axes=3)
    cache = bf(4, 16, 2, 64)
    lay = pkg.make_cache_layout(cache)
    good = dict(q=bf(5, 8, 64, strides=(768, 64, 1)), k=bf(5, 2, 64), v=bf(5, 2, 64), q_weight=bf(64), k_weight=None,
                positions=ints(3, 5), freq=Fake((32,), torch.float32), axis=ints(32), q_out=bf(5, 8, 64), k_out=None, cache=lay,
                k_cache=cache, v_cache=cache, slots=ints(5))
    for change, exc in ((dict(q=bf(5, 8, 64, strides=(768, 96, 1))), ValueError), (dict(k=Fake((5, 2, 64), torch.float16)), TypeError),
                        (dict(k=bf(4, 2, 64)), ValueError), (dict(q=torch.zeros(5, 8, 64, dtype=torch.bfloat16)), ValueError),
                        (dict(v=None), TypeError), (dict(q_weight=bf(32)), ValueError), (dict(positions=ints(2, 5)), ValueError),
                        (dict(positions=ints(3, 4)), ValueError), (dict(freq=ints(32)), TypeError), (dict(slots=ints(4)), ValueError),
                        (dict(k_cache=bf(4, 8, 2, 64)), ValueError), (dict(v_cache=bf(4, 16, 2, 64, strides=(2048, 64, 1024, 1))), ValueError),
                        (dict(q=bf(40, 64)), ValueError), (dict(q_out=np.zeros((5, 8, 64))), TypeError)):
        with pytest.raises(exc):
            pkg.ivit_qk_norm_rope(cfg, **{**good, **change})
    acfg = pkg.make_attention_config(2, 8, 3, 4, "tree", 1, 0.125)
    good = dict(q=bf(5, 8, 64), k_new=bf(5, 2, 64), v_new=bf(5, 2, 64), k_cache=cache, v_cache=cache, table=ints(2, 3),
                lengths=ints(2), cu_rows=ints(3), mask=ints(5, 1), out=bf(5, 8, 64), lse=Fake((5, 8), torch.float32),
                workspace=Fake((1 << 28,), torch.uint8))
    for change, exc in ((dict(table=ints(2, 2)), ValueError), (dict(lengths=Fake((2,), torch.int64)), TypeError),
                        (dict(cu_rows=ints(2)), ValueError), (dict(mask=ints(4, 1)), ValueError), (dict(out=bf(4, 8, 64)), ValueError),
                        (dict(lse=Fake((5, 8), torch.float16)), TypeError), (dict(k_new=bf(5, 2, 32)), ValueError)):
        with pytest.raises(exc):
            pkg.ivit_tree_attention(acfg, lay, **{**good, **change})
    caches = bf(3, 4, 16, 2, 64)
    good = dict(k=bf(3, 6, 2, 64), v=bf(3, 6, 2, 64), rows=ints(4), slots=ints(4), k_cache=caches, v_cache=caches)
    for change, exc in ((dict(k=bf(6, 2, 64)), ValueError), (dict(v=bf(3, 5, 2, 64)), ValueError), (dict(slots=ints(3)), ValueError),
                        (dict(v=bf(3, 6, 2, 64, strides=(1536, 256, 64, 1))), ValueError), (dict(k_cache=bf(2, 4, 16, 2, 64)), ValueError),
                        (dict(v_cache=bf(3, 4, 16, 1, 64)), ValueError)):
        with pytest.raises(exc):
            pkg.ivit_kv_write(lay, **{**good, **change})
    pcfg = pkg.make_plan_config(2, 5, 3, 16, 20, 1)
    names = ["held", "base", "new", "parent", "ring", "ring_in", "table", "cu_rows", "req", "slots", "positions", "mask", "ring_out",
             "status"]
    sizes = [(2,), (2,), (2,), (5,), (20,), (2,), (2, 3), (3,), (5,), (5,), (5,), (5, 1), (2,), (1,)]
    for i, name in enumerate(names):
        args = [ints(*s) for s in sizes]
        args[i] = ints(*[*sizes[i][:-1], sizes[i][-1] - 1])
        with pytest.raises(ValueError, match=name):
            pkg.ivit_step_plan(pcfg, *args)
