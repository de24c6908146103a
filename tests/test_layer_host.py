"""Refusals of the layers, their gradients and the clipping: every check runs on the host, nothing is launched."""
import ctypes
import os
import re

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
    def __init__(self, gated=False, dtype=sr.SR_F16, n=2, h=5, w=7, C=24, O=40):
        wide = 2 * O if gated else O
        self.gated, self.act = gated, sr.SR_ACT_SILU
        self.x, self.weight, self.bias = T(0, dtype, n, C, h, w), T(1, dtype, 1, 1, wide, C), T(2, dtype, 1, 1, 1, wide)
        self.y, self.residual = T(3, dtype, n, O, h, w), T(4, dtype, n, O, h, w)
        self.dx, self.dweight, self.dbias = T(5, dtype, n, C, h, w), T(6, dtype, 1, 1, wide, C), T(7, dtype, 1, 1, 1, wide)
        self.ws, self.bytes = BASE + (8 << 24), 1 << 40

    def forward(self, lib):
        x, weight, bias, y, residual = (t and ctypes.byref(t) for t in (self.x, self.weight, self.bias, self.y, self.residual))
        if self.gated:
            return lib.sr_layer_gated(x, weight, bias, self.act, y, self.ws, self.bytes, None)
        return lib.sr_layer_linear(x, weight, bias, self.act, residual, y, self.ws, self.bytes, None)

    def grad(self, lib):
        call = lib.sr_layer_gated_grad if self.gated else lib.sr_layer_linear_grad
        x, weight, bias, y, dx, dweight, dbias = (t and ctypes.byref(t) for t in (self.x, self.weight, self.bias, self.y, self.dx, self.dweight,
                                                                                   self.dbias))
        return call(x, weight, bias, self.act, y, dx, dweight, dbias, self.ws, self.bytes, None)


def bad(gated, what):
    """A case with things wrong: attributes, and descriptors' fields as tensor__field."""
    c = Case(gated)
    for k, v in what.items():
        if "__" in k:
            t, f = k.split("__")
            setattr(getattr(c, t), f, v)
        else:
            setattr(c, k, v)
    return c


COMMON = [
    (dict(x=None), -1), (dict(weight=None), -1), (dict(y=None), -1), (dict(x__data=None), -1), (dict(weight__data=None), -1),
    (dict(bias__data=None), -1), (dict(y__data=None), -1),
    (dict(act=5), -3), (dict(act=-1), -3), (dict(x__dtype=sr.SR_F8E4M3), -3), (dict(x__dtype=sr.SR_U8), -3), (dict(x__dtype=9), -3),
    (dict(weight__dtype=sr.SR_F32), -3), (dict(bias__dtype=sr.SR_BF16), -3), (dict(y__dtype=sr.SR_F32), -3),
    (dict(x__c=0), -3), (dict(x__c=65537), -3), (dict(y__c=0), -3), (dict(y__c=65537), -3), (dict(x__h=1 << 30, y__h=1 << 30), -3),
    (dict(x__h=65536, x__w=32768, x__n=1, y__h=65536, y__w=32768, y__n=1, residual=None), -3),
    (dict(x__n=-1), -2), (dict(y__w=8), -2), (dict(y__n=1), -2), (dict(x__c=23), -2), (dict(weight__h=41), -2), (dict(weight__w=25), -2),
    (dict(weight__n=2), -2), (dict(weight__c=2), -2), (dict(bias__w=41), -2), (dict(bias__h=2), -2), (dict(y__c=41, residual=None), -2),
    (dict(x__data=BASE + 1), -7), (dict(weight__data=BASE + (1 << 24) + 1), -7), (dict(bias__data=BASE + (2 << 24) + 1), -7),
    (dict(y__data=BASE + (3 << 24) + 1), -7),
]


@pytest.mark.parametrize("what,status", COMMON, ids=lambda v: str(v))
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
@pytest.mark.parametrize("call", ["forward", "grad"])
def test_refusals_of_all_four(lib, call, gated, what, status):
    assert getattr(bad(gated, what), call)(lib) == status


def test_refusals_of_single_calls(lib):
    assert bad(False, dict(residual__data=None)).forward(lib) == -1
    assert bad(False, dict(residual__dtype=sr.SR_F32)).forward(lib) == -3
    assert bad(False, dict(residual__c=41)).forward(lib) == -2
    assert bad(False, dict(residual__h=6)).forward(lib) == -2
    assert bad(False, dict(residual__data=BASE + (4 << 24) + 1)).forward(lib) == -7
    for gated in (False, True):
        for on in (0, 1, 2):                                            # y on an input
            assert bad(gated, dict(y__data=BASE + (on << 24))).forward(lib) == -4
        assert bad(gated, dict(dx=None, dweight=None, dbias=None)).grad(lib) == -1
        assert bad(gated, dict(dx__data=None)).grad(lib) == -1
        assert bad(gated, dict(dweight__data=None)).grad(lib) == -1
        assert bad(gated, dict(dbias__data=None)).grad(lib) == -1
        assert bad(gated, dict(dx__dtype=sr.SR_F32)).grad(lib) == -3
        assert bad(gated, dict(dweight__dtype=sr.SR_F32)).grad(lib) == -3
        assert bad(gated, dict(dbias__dtype=sr.SR_F32)).grad(lib) == -3
        assert bad(gated, dict(dx__c=25)).grad(lib) == -2
        assert bad(gated, dict(dx__w=8)).grad(lib) == -2
        assert bad(gated, dict(dweight__h=39)).grad(lib) == -2
        assert bad(gated, dict(dbias__w=39)).grad(lib) == -2
        assert bad(gated, dict(dx__data=BASE + (5 << 24) + 1)).grad(lib) == -7
        assert bad(gated, dict(dbias__data=BASE + (7 << 24) + 1)).grad(lib) == -7
        assert bad(gated, dict(ws=None)).grad(lib) == -2
        assert bad(gated, dict(bytes=16)).grad(lib) == -2
        assert bad(gated, dict(ws=BASE + (8 << 24) + 8)).grad(lib) == -7
        for out in ("dx", "dweight", "dbias"):
            for on in (0, 1, 2, 3):                                     # on an input or dy
                assert bad(gated, {out + "__data": BASE + (on << 24)}).grad(lib) == -4
        assert bad(gated, dict(dweight__data=BASE + (5 << 24) + 2)).grad(lib) == -4
        assert bad(gated, dict(dbias__data=BASE + (6 << 24))).grad(lib) == -4
        assert bad(gated, dict(ws=BASE + (3 << 24))).grad(lib) == -4
        assert bad(gated, dict(ws=BASE + (7 << 24))).grad(lib) == -4


@pytest.mark.parametrize("gated", [False, True])
def test_empty_calls(lib, gated):
    c = Case(gated, n=0)
    for t in (c.x, c.y, c.residual, c.dx):
        t.data = None
    assert c.forward(lib) == 0
    c.dweight = c.dbias = None                                          # nothing is left to write then
    assert c.grad(lib) == 0


def test_workspace_sizes(lib):
    for f, more in ((lib.sr_layer_linear_workspace_bytes, ()), (lib.sr_layer_gated_workspace_bytes, ()),
                    (lib.sr_layer_linear_grad_workspace_bytes, (sr.SR_ACT_GELU,)), (lib.sr_layer_gated_grad_workspace_bytes, ())):
        for args in ((-1, 64, 64, sr.SR_F16), (1 << 31, 64, 64, sr.SR_F16), (100, 0, 64, sr.SR_F16), (100, 65537, 64, sr.SR_F16),
                     (100, 64, 0, sr.SR_F16), (100, 64, 65537, sr.SR_F16), (100, 64, 64, sr.SR_U8), (100, 64, 64, sr.SR_F8E4M3)):
            assert f(*args, *more) == 0
    assert lib.sr_layer_linear_grad_workspace_bytes(100, 64, 64, sr.SR_F16, 7) == 0
    assert lib.sr_layer_linear_workspace_bytes(1, 2048, 2048, sr.SR_BF16) == 0
    for f, more in ((lib.sr_layer_linear_workspace_bytes, ()), (lib.sr_layer_gated_workspace_bytes, ()),
                    (lib.sr_layer_linear_grad_workspace_bytes, (sr.SR_ACT_GELU,)), (lib.sr_layer_gated_grad_workspace_bytes, ())):
        assert f(0, 64, 72, sr.SR_F16, *more) == 0                      # no rows
        f((1 << 31) - 257, 65536, 65536, sr.SR_F32, *more)              # the largest sizes there are
    # the gradient of z: rows of 16-byte pieces
    assert lib.sr_layer_gated_grad_workspace_bytes(100000, 64, 33, sr.SR_BF16) >= 100000 * 72 * 2
    assert lib.sr_layer_linear_grad_workspace_bytes(100000, 64, 33, sr.SR_BF16, sr.SR_ACT_RELU) >= 100000 * 40 * 2
    assert lib.sr_layer_linear_grad_workspace_bytes(100000, 64, 33, sr.SR_BF16, sr.SR_ACT_NONE) < 100000 * 33 * 2 + (64 << 20)


class Clip:
    def __init__(self, sizes=((1, 1, 8, 5), (1, 1, 1, 7), (1, 1, 1, 1)), dtypes=(sr.SR_F32, sr.SR_BF16, sr.SR_F16)):
        self.n = len(sizes)
        self.grads = (sr.sr_tensor * self.n)(*[T(i, d, *s) for i, (s, d) in enumerate(zip(sizes, dtypes))])
        self.outs = (sr.sr_tensor * self.n)(*[T(16 + i, d, *s) for i, (s, d) in enumerate(zip(sizes, dtypes))])
        self.most, self.norm, self.ws, self.bytes = 1.0, BASE + (32 << 24), BASE + (33 << 24), 1 << 40

    def call(self, lib):
        return lib.sr_grad_clip(self.grads, self.outs, self.n, self.most, self.norm, self.ws, self.bytes, None)


def test_refusals_of_clipping(lib):
    def refused(**kw):
        c = Clip()
        for k, v in kw.items():
            if "__" in k:
                t, f = k.split("__")
                setattr(getattr(c, t[:-1])[int(t[-1])], f, v)
            else:
                setattr(c, k, v)
        return c.call(lib)

    assert refused(grads=None) == -1
    assert refused(norm=None) == -1
    assert refused(grads1__data=None) == -1
    assert refused(outs2__data=None) == -1
    for n in (0, -1, sr.SR_MAX_GRADS + 1):
        assert refused(n=n) == -3
    for most in (-1.0, float("nan"), -float("inf")):
        assert refused(most=most) == -3
    assert refused(grads0__dtype=sr.SR_U8) == -3
    assert refused(grads0__dtype=sr.SR_F8E4M3) == -3
    assert refused(outs0__dtype=sr.SR_F16) == -3
    assert refused(grads0__n=1 << 30, outs0__n=1 << 30, grads0__c=1 << 30, outs0__c=1 << 30) == -3
    assert refused(grads0__w=-1) == -2
    assert refused(outs0__w=6) == -2
    assert refused(outs0__h=5, outs0__w=8) == -2
    assert refused(grads0__data=BASE + 2) == -7
    assert refused(grads1__data=BASE + (1 << 24) + 1) == -7
    assert refused(outs0__data=BASE + (16 << 24) + 2) == -7
    assert refused(norm=BASE + (32 << 24) + 2) == -7
    assert refused(ws=BASE + (33 << 24) + 8) == -7
    assert refused(ws=None) == -2
    assert refused(bytes=sr.sr_grad_clip_workspace_bytes(3) - 1) == -2
    assert refused(outs1__data=BASE) == -4                               # on another gradient
    assert refused(outs0__data=BASE + 4) == -4                           # on its own, but not in place
    assert refused(outs1__data=BASE + (16 << 24) + 158) == -4            # on another output's last element
    assert refused(norm=BASE) == -4
    assert refused(norm=BASE + (16 << 24)) == -4
    assert refused(ws=BASE + (2 << 24)) == -4
    assert refused(ws=BASE + (18 << 24) - 16) == -4


def test_the_same_tensor_twice_in_place_is_refused(lib):
    c = Clip()
    for i in (1, 2):
        c.grads[i] = c.grads[0]
        c.outs[i] = c.grads[0]
    c.outs[0] = c.grads[0]
    assert c.call(lib) == -4


def test_clip_workspace(lib):
    f = sr.sr_grad_clip_workspace_bytes
    assert f(0) == 0 and f(-1) == 0 and f(sr.SR_MAX_GRADS + 1) == 0
    assert 0 < f(1) <= f(129) <= f(sr.SR_MAX_GRADS) < 1 << 22


def test_the_binding_refuses_what_it_cannot_describe(lib):
    x, w, y = torch.zeros(4, 8), torch.zeros(3, 8), torch.zeros(4, 3)
    for call in (lambda: sr.sr_layer_linear(x, w, None, 0, None, y), lambda: sr.sr_layer_gated(x, torch.zeros(6, 8), None, 0, y),
                 lambda: sr.sr_layer_linear_grad(x, w, None, 0, y, x.clone(), None, None),
                 lambda: sr.sr_layer_gated_grad(x, torch.zeros(6, 8), None, 0, y, x.clone(), None, None)):
        with pytest.raises(ValueError, match="current device"):
            call()
    with pytest.raises(ValueError, match="one device"):
        sr.sr_grad_clip([x], None, 1.0, torch.zeros(2))
    with pytest.raises(ValueError, match="contiguous"):
        binding._rows(torch.zeros(8, 4).t(), -1)
    with pytest.raises(ValueError, match="contiguous"):
        binding._rows(torch.zeros(8), -1)
    with pytest.raises(ValueError, match="contiguous"):
        binding._matrix(torch.zeros(8, 4).t(), -1)
    with pytest.raises(ValueError, match="contiguous"):
        binding._matrix(torch.zeros(1, 8, 4), -1)
    with pytest.raises(TypeError):
        binding._rows(x.double(), -1)
    with pytest.raises(TypeError):
        binding._matrix(x.long(), -1)
    assert binding._rows(torch.zeros(2, 3, 5, 7), -1)[1:] == (sr.SR_F32, 2, 7, 3, 5)
    assert binding._rows(torch.zeros(3, 5, 7).half(), -1)[1:] == (sr.SR_F16, 1, 7, 3, 5)
    assert binding._rows(x, -1) == (x.data_ptr(), sr.SR_F32, 1, 8, 1, 4)
    assert binding._matrix(w.bfloat16(), -1)[1:] == (sr.SR_BF16, 1, 1, 3, 8) and binding._matrix(w[0], -1)[1:] == (sr.SR_F32, 1, 1, 1, 8)
    # what is packed is what the structure holds
    slots = binding._Slots()
    binding._fill5(slots, 0, *range(1, 31))
    for i in range(5):
        d = slots[i]
        assert [d.data, d.dtype, d.n, d.c, d.h, d.w] == list(range(6 * i + 1, 6 * i + 7))


def test_tensors_without_gaps():
    t = torch.zeros(4, 6, 8)
    assert binding._dense(t) and binding._dense(t.permute(2, 0, 1)) and binding._dense(t[:, :1][:2].permute(1, 0, 2)[:, :1])
    assert binding._dense(torch.zeros(2, 3, 4, 5).to(memory_format=torch.channels_last))
    assert not binding._dense(t[:, ::2]) and not binding._dense(t[..., :7]) and not binding._dense(torch.zeros(4, 1).expand(4, 3))


def test_lists_of_tensors_beyond_32_bits_are_described_whole():
    """No field of a description is cut to 32 bits: what is described has the tensor's elements, one piece behind the other."""
    def fields(t):
        packed = binding._elements(t)
        array = (sr.sr_tensor * (len(packed) // ctypes.sizeof(sr.sr_tensor))).from_buffer_copy(packed)
        return [(d.data, d.dtype, d.n, d.c, d.h, d.w) for d in array]

    for shape in ((1 << 31,), ((1 << 32) + 5,), (3 * 10 ** 9,), (1 << 32,), ((1 << 31) + 1, 1), (1 << 16, (1 << 16) + 1, 1, 1, 1), (1 << 11, 1 << 20, 1, 2, 1)):
        t = torch.empty(shape, dtype=torch.bfloat16)                     # memory that nothing touches
        at = t.data_ptr()
        for data, dtype, n, c, h, w in fields(t):
            assert data == at and dtype == sr.SR_BF16 and min(n, c, h, w) > 0
            at += 2 * n * c * h * w
        assert at == t.data_ptr() + 2 * t.numel(), shape
    t = torch.empty((1 << 16, (1 << 15) - 1, 1, 1, 1), dtype=torch.bfloat16)
    assert fields(t) == [(t.data_ptr(), sr.SR_BF16, (1 << 31) - (1 << 16), 1, 1, 1)]
    assert fields(torch.empty(2, 3, 4, 5, 6))[0][2:] == (6, 4, 5, 6)
    assert fields(torch.empty(7).half())[0][1:] == (sr.SR_F16, 1, 1, 1, 7) and fields(torch.tensor(1.0))[0][1:] == (sr.SR_F32, 1, 1, 1, 1)
    assert fields(torch.empty(3, 0)) == [(None, sr.SR_F32, 1, 1, 3, 0)]
    for data, dtype, n, c, h, w in fields(torch.empty((0, 1 << 32))):
        assert data is None and n * c * h * w == 0


def test_loads_to_lds_in_assembly_read_what_scalar_moves_have_just_written():
    """A load to LDS takes its base and m0 at once; a vector instruction that wrote one of them would have to be five wait states before it, which nothing counts
    for assembly.  So each of these loads moves both by itself, and the base last: m0 is one wait state away then."""
    csrc = os.path.join(os.path.dirname(binding.__file__), "csrc")
    found = 0
    for name in sorted(os.listdir(csrc)):
        with open(os.path.join(csrc, name)) as f:
            for text, outs in re.findall(r'asm volatile\s*\(\s*"([^"]*global_load_lds[^"]*)"\s*:([^:]*):', f.read()):
                assert re.fullmatch(r"s_mov_b32 %1, %4\\n\\ts_mov_b64 %0, %3\\n\\tglobal_load_lds_dword(x4)? %2, %0", text), (name, text)
                assert re.fullmatch(r'\s*"=&s"\(\w+\), "=&\{m0\}"\(\w+\)\s*', outs), (name, outs)
                found += 1
    assert found == 4
