"""Refusals of the router, the balance losses and the gradients: every check runs on the host, nothing is launched."""
import ctypes
import os

import pytest
import torch

import paper_2303_08999_amd as sr
from paper_2303_08999_amd import binding

BASE = 0x10000000


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2303_08999_amd import build
        build.build_library()
    return sr.load()


def T(slot, dtype, n, c, h, w, off=0):
    """A descriptor with a fake, aligned address, 16 MiB from its neighbours."""
    return sr.sr_tensor(BASE + (slot << 24) + off, dtype, n, c, h, w)


class Case:
    def __init__(self, **kw):
        self.L, self.scale, self.T, self.kind, self.layout = 72, 2, 8, sr.SR_ROUTE_SOFTMAX, sr.SR_COEFF_PLANAR
        self.n, self.H, self.W, self.cd, self.vd = 1, 16, 20, sr.SR_F16, sr.SR_F32
        self.__dict__.update(kw)
        pre = self.layout == sr.SR_COEFF_PRE_SHUFFLE
        s = self.scale if pre else 1
        self.coeff = T(0, self.cd, self.n, self.L * s * s, self.H // s, self.W // s)
        self.index = T(1, sr.SR_U8, self.n, self.T, self.H, self.W)
        self.value = T(2, self.vd, self.n, self.T, self.H, self.W)
        self.mask = T(3, sr.SR_U8, self.n, 1, self.H, self.W)
        self.dz = T(4, self.cd, self.n, self.L * s * s, self.H // s, self.W // s)
        self.counts, self.share, self.loss, self.ws = (BASE + (i << 24) for i in (5, 6, 7, 8))
        self.bytes = 1 << 40

    def args(self):
        return self.L, self.scale, self.T, self.kind, self.layout

    def route(self, lib):
        return lib.sr_list_route(self.coeff, *self.args(), self.mask, self.index, self.value, None)

    def balance(self, lib):
        return lib.sr_list_route_balance(self.coeff, *self.args(), self.mask, self.index, self.value, self.counts, self.share,
                                         self.loss, self.ws, self.bytes, None)

    def grad(self, lib):
        return lib.sr_list_route_grad(self.coeff, self.index, self.value, *self.args(), self.mask, self.counts, self.loss,
                                      self.dz, None)


def bad(**kw):
    """A case with one thing wrong, attributes of descriptors as tensor__field."""
    c = Case(**{k: v for k, v in kw.items() if "__" not in k and k in ("L", "T", "scale", "kind", "layout", "cd", "vd", "n")})
    for k, v in kw.items():
        if "__" in k:
            t, f = k.split("__")
            setattr(getattr(c, t), f, v)
        elif k not in ("L", "T", "scale", "kind", "layout", "cd", "vd", "n"):
            setattr(c, k, v)
    return c


COMMON = [
    (dict(L=257, T=1), -3), (dict(L=8, T=9), -3), (dict(T=0), -3), (dict(kind=3), -3), (dict(kind=-1), -3),
    (dict(layout=sr.SR_COEFF_BLOCKED), -3), (dict(layout=7), -3), (dict(cd=sr.SR_F8E4M3), -3), (dict(vd=sr.SR_BF16), -3),
    (dict(layout=sr.SR_COEFF_PRE_SHUFFLE, scale=5), -3), (dict(index__dtype=sr.SR_F16), -3), (dict(mask__dtype=sr.SR_F32), -3),
    (dict(index__c=7), -2), (dict(value__c=9), -2), (dict(mask__c=2), -2), (dict(index__w=21), -2), (dict(mask__h=15), -2),
    (dict(coeff__c=71), -2), (dict(value__n=2), -2), (dict(coeff__h=-1), -2),
    (dict(coeff=None), -1), (dict(index=None), -1), (dict(index__data=None), -1), (dict(mask__data=None), -1),
    (dict(coeff__data=BASE + 1), -7), (dict(value__data=BASE + (2 << 24) + 2), -7),
]


@pytest.mark.parametrize("what,status", COMMON, ids=lambda v: str(v))
@pytest.mark.parametrize("call", ["route", "balance", "grad"])
def test_refusals_of_all_three(lib, call, what, status):
    assert getattr(bad(**what), call)(lib) == status


def test_refusals_of_single_calls(lib):
    assert bad(value=None).route(lib) == -1
    assert bad(index__data=BASE).route(lib) == -4                        # the lists on top of the logits
    assert bad(value__data=BASE + (1 << 24) + 16).route(lib) == -4       # ... of one another
    assert bad(index__data=BASE + (3 << 24)).route(lib) == -4            # ... of the mask
    assert bad(kind=sr.SR_ROUTE_VALUES).balance(lib) == -3
    assert bad(counts=None).balance(lib) == -1
    assert bad(ws=None).balance(lib) == -2
    assert bad(bytes=sr.sr_list_route_workspace_bytes(72) - 1).balance(lib) == -2
    assert bad(ws=BASE + (8 << 24) + 8).balance(lib) == -7
    assert bad(counts=BASE + (5 << 24) + 4).balance(lib) == -7
    assert bad(share=BASE + (7 << 24)).balance(lib) == -4
    assert bad(ws=BASE).balance(lib) == -4
    assert bad(dz=None).grad(lib) == -1
    assert bad(counts=None).grad(lib) == -1                              # both or neither
    assert bad(loss=None).grad(lib) == -1
    assert bad(kind=sr.SR_ROUTE_VALUES).grad(lib) == -3                  # no losses there
    assert bad(dz__dtype=sr.SR_F32).grad(lib) == -3
    assert bad(dz__c=71).grad(lib) == -2
    assert bad(dz__data=BASE).grad(lib) == -4                            # not in place
    assert bad(dz__data=BASE + (4 << 24) + 1).grad(lib) == -7


def test_empty_calls(lib):
    for call in ("route", "grad"):
        c = Case(n=0)
        for t in (c.coeff, c.index, c.value, c.mask, c.dz):
            t.data = None
        assert getattr(c, call)(lib) == 0


def test_workspace_sizes(lib):
    assert sr.sr_list_route_workspace_bytes(0) == 0 and sr.sr_list_route_workspace_bytes(257) == 0
    assert 0 < sr.sr_list_route_workspace_bytes(1) < sr.sr_list_route_workspace_bytes(256) < 1 << 23
    assert sr.sr_dict_assemble_list_grad_workspace_bytes(72, 4) == 0 and sr.sr_dict_assemble_list_grad_workspace_bytes(257, 5) == 0
    assert 0 < sr.sr_dict_assemble_list_grad_workspace_bytes(1, 3) < sr.sr_dict_assemble_list_grad_workspace_bytes(256, 7) < 1 << 26


class Grad:
    def __init__(self, **kw):
        self.L, self.k, self.s, self.C, self.T, self.vd, self.io, self.n, self.h, self.w = 72, 5, 4, 3, 8, sr.SR_F16, sr.SR_F32, 1, 8, 12
        self.__dict__.update({k: v for k, v in kw.items() if "__" not in k})
        H, W = self.h * self.s, self.w * self.s
        self.lr = T(0, self.io, self.n, self.C, self.h, self.w)
        self.index, self.value = T(1, sr.SR_U8, self.n, self.T, H, W), T(2, self.vd, self.n, self.T, H, W)
        self.dict, self.mask = T(3, sr.SR_F32, 1, self.L, self.k, self.k), T(4, sr.SR_U8, self.n, 1, H, W)
        self.dout, self.dvalue = T(5, self.io, self.n, self.C, H, W), T(6, self.vd, self.n, self.T, H, W)
        self.ddict, self.ws, self.bytes = T(7, sr.SR_F32, 1, self.L, self.k, self.k), BASE + (8 << 24), 1 << 40
        for k, v in kw.items():
            if "__" in k:
                t, f = k.split("__")
                if f == "is":
                    setattr(self, t, v)
                else:
                    setattr(getattr(self, t), f, v)

    def call(self, lib):
        return lib.sr_dict_assemble_list_grad(self.lr, self.index, self.value, self.dict, self.L, self.k, self.s, self.C, self.T,
                                              self.mask, self.dout, self.dvalue, self.ddict, self.ws, self.bytes, None)


@pytest.mark.parametrize("what,status", [
    (dict(k=4), -3), (dict(s=5), -3), (dict(L=257), -3), (dict(C=17), -3), (dict(T=257), -3), (dict(vd=sr.SR_BF16), -3), (dict(io=sr.SR_BF16), -3),
    (dict(dout__dtype=sr.SR_F16), -3), (dict(dvalue__dtype=sr.SR_F32), -3), (dict(ddict__dtype=sr.SR_F16), -3), (dict(index__dtype=sr.SR_F32), -3),
    (dict(index__c=9), -2), (dict(dvalue__c=9), -2), (dict(dout__w=47), -2), (dict(mask__n=2), -2), (dict(ddict__c=71), -2), (dict(dict__h=3), -2),
    (dict(lr__is=None), -1), (dict(dout__is=None), -1), (dict(dvalue__is=None, ddict__is=None), -1), (dict(ddict__data=None), -1), (dict(dout__data=None), -1),
    (dict(ws__is=None), -2), (dict(bytes__is=100), -2), (dict(ws__is=BASE + (8 << 24) + 8), -7), (dict(dvalue__data=BASE + (6 << 24) + 1), -7),
    (dict(dvalue__data=BASE + (2 << 24)), -4), (dict(ddict__data=BASE + (3 << 24)), -4), (dict(ws__is=BASE + (7 << 24)), -4), (dict(ddict__data=BASE + (6 << 24)), -4),
], ids=lambda v: str(v))
def test_refusals_of_the_list_gradient(lib, what, status):
    assert Grad(**what).call(lib) == status


def test_the_binding_refuses_what_is_not_on_the_device(lib):
    z, idx, val = torch.zeros(1, 8, 2, 2), torch.zeros(1, 2, 2, 2, dtype=torch.uint8), torch.zeros(1, 2, 2, 2)
    with pytest.raises(ValueError, match="current device"):
        sr.sr_list_route(z, 8, 1, 2, 0, 0, None, idx, val)
    with pytest.raises(ValueError, match="current device"):
        sr.sr_list_route_balance(z, 8, 1, 2, 0, 0, None, idx, val, torch.zeros(9, dtype=torch.int64), torch.zeros(8), torch.zeros(2))
    with pytest.raises(ValueError, match="current device"):
        sr.sr_list_route_grad(z, idx, val, 8, 1, 2, 0, 0, None, None, None, z.clone())
    with pytest.raises(ValueError, match="current device"):
        sr.sr_dict_assemble_list_grad(torch.zeros(1, 1, 1, 1), idx, val, torch.zeros(8, 3, 3), 8, 3, 2, 1, 2, None,
                                      torch.zeros(1, 1, 2, 2), val.clone(), None)
