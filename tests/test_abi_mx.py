"""Refusals of the entry points on block-scaled values, and of their binding: no GPU is touched."""
import ctypes as C

import pytest
import torch

import paper_2502_12224_amd.binding as B

P, ODD = 0x1000, 0x1004         # never dereferenced: validation fails first
OK, EINVAL, ESHAPE, EALIGN, EWORKSPACE = 0, 1, 2, 3, 4


def test_norm_refusals():
    f = B.lib().fate_add_rmsnorm
    good = dict(N=4, H=256, h=P, ht=0, ldh=256, d=P, dt=0, ldd=256, w=P, wt=0, eps=1e-6, ho=P, ldho=256, x=P, ldx=256,
                c=P, s=P)

    def call(**kw):
        return f(0, *{**good, **kw}.values())
    assert call(N=-1) == EINVAL and call(H=0) == ESHAPE and call(H=65537, ldh=70000, ldd=70000, ldho=70000, ldx=70000) == ESHAPE
    assert call(ht=2) == EINVAL and call(dt=7) == EINVAL and call(wt=-1) == EINVAL
    assert call(eps=-1.0) == EINVAL and call(eps=float("nan")) == EINVAL
    assert call(ho=0, x=0, c=0, s=0) == EINVAL and b"no output" in B.lib().fate_last_error()
    assert call(c=0) == EINVAL and call(s=0) == EINVAL
    assert call(ldh=255) == ESHAPE and call(ldd=255) == ESHAPE and call(ldho=1) == ESHAPE and call(ldx=255) == ESHAPE
    assert call(h=0) == EINVAL and call(h=ODD) == EALIGN and call(d=ODD) == EALIGN and call(w=ODD) == EALIGN
    assert call(ho=ODD) == EALIGN and call(x=ODD) == EALIGN and call(c=ODD) == EALIGN and call(s=ODD) == EALIGN
    assert call(ldho=264) == EINVAL                                       # in place, other distance
    assert call(N=0) == OK and call(N=0, h=0) == OK


def test_quantize_and_pack_refusals():
    L = B.lib()
    q = L.fate_mx_quantize
    assert q(0, P, 0, -1, 64, 64, P, P) == EINVAL and q(0, P, 0, 4, 0, 64, P, P) == ESHAPE
    assert q(0, P, 2, 4, 64, 64, P, P) == EINVAL and q(0, P, 0, 4, 64, 63, P, P) == ESHAPE
    assert q(0, 0, 0, 4, 64, 64, P, P) == EINVAL and q(0, P, 0, 4, 64, 64, ODD, P) == EALIGN
    assert q(0, P, 0, 4, 64, 64, P, 0) == EINVAL and q(0, 0, 0, 0, 64, 64, 0, 0) == OK
    p = L.fate_mx_pack_weight
    assert p(0, P, 0, 0, 64, 64, 4, P, P) == ESHAPE and p(0, P, 0, 4, 64, 64, 2, P, P) == EINVAL
    assert p(0, P, 0, 4, 64, 60, 4, P, P) == ESHAPE and p(0, P, 3, 4, 64, 64, 8, P, P) == EINVAL
    assert p(0, ODD, 0, 4, 64, 64, 4, P, P) == EALIGN
    assert B.fate_mx_weight_bytes(1408, 2048, 4) == (1408 * 1024, 1408 * 64)
    assert B.fate_mx_weight_bytes(33, 129, 8) == (64 * 256, 4 * 256)
    c = C.c_size_t(0)
    assert L.fate_mx_weight_bytes(4, 4, 4, C.byref(c), 0) == EINVAL and L.fate_mx_weight_bytes(4, 0, 4, C.byref(c), C.byref(c)) == ESHAPE


def test_linear_refusals():
    f = B.lib().fate_mx_linear
    good = dict(N=4, K=256, R=100, x=P, xt=0, ldx=256, xs=0, bits=4, wc=P, ws=P, bias=0, y=P, yt=0, ldy=100)

    def call(**kw):
        return f(0, *{**good, **kw}.values())
    assert call(N=(1 << 30) + 1, xt=2, xs=P) == ESHAPE
    assert call(N=-1) == EINVAL and call(K=0) == ESHAPE and call(R=0) == ESHAPE and call(bits=2) == EINVAL
    assert call(xt=1) == EINVAL and call(yt=2) == EINVAL and call(ldx=255) == ESHAPE and call(ldy=99) == ESHAPE
    assert call(xs=P) == EINVAL and call(K=65537, ldx=65537) == ESHAPE
    assert call(xt=2) == EINVAL                                            # 8-bit rows without scales
    assert call(x=0) == EINVAL and call(wc=ODD) == EALIGN and call(ws=0) == EINVAL and call(bias=ODD) == EALIGN
    assert call(y=ODD) == EALIGN and call(N=0, x=0, y=0) == OK


def _desc(N=4, H=256, E=8, k=2, I=512, bits=4, group=32, ns=1, Is=96, sb=8, sg=32, mode=0):
    return B.make_ffn_desc(N, H, E, k, I, bits, group, ns, Is, sb, sg, True, mode)


@pytest.mark.parametrize("kw,status", [
    (dict(N=-1), EINVAL), (dict(H=48), ESHAPE), (dict(H=0), ESHAPE), (dict(E=0), ESHAPE), (dict(E=257), ESHAPE),
    (dict(k=0), EINVAL), (dict(k=9), EINVAL), (dict(I=40), ESHAPE), (dict(bits=2), EINVAL), (dict(group=128), ESHAPE),
    (dict(ns=17), EINVAL), (dict(sb=3), EINVAL), (dict(sg=64), ESHAPE), (dict(Is=100), ESHAPE), (dict(mode=1), EINVAL),
    (dict(N=1 << 30), ESHAPE)])
def test_ffn_descriptor_refusals(kw, status):
    n = C.c_size_t(0)
    assert B.lib().fate_moe_ffn_mx_workspace(C.byref(_desc(**kw)), C.byref(n)) == status


def test_ffn_refusals():
    L = B.lib()
    d = _desc()
    need = B.fate_moe_ffn_mx_workspace(d)
    assert need >= 256 + 8 * 512 + 8 * 16 + 4 * 128 + 12 * 256 * 4
    assert B.fate_moe_ffn_mx_workspace(_desc(N=3)) <= need                 # enough for fewer tokens
    args = [0, C.addressof(d)] + [P] * 13 + [need]

    def call(i, v):
        return L.fate_moe_ffn_mx(*args[:i], v, *args[i + 1:])
    assert call(1, None) == EINVAL and call(2, 0) == EINVAL and call(3, ODD) == EALIGN
    for i in (4, 5, 6, 7, 8, 9, 10):
        assert call(i, 0) == EINVAL, i
    assert call(4, ODD) == EALIGN and call(11, ODD) == EALIGN
    assert call(11, 0) == EINVAL and call(12, ODD) == EALIGN and call(13, 0) == EINVAL
    assert call(14, 0) == EWORKSPACE and call(15, need - 1) == EWORKSPACE and call(14, ODD) == EALIGN
    d0 = _desc(N=0)
    assert L.fate_moe_ffn_mx(0, C.addressof(d0), *[0] * 13, 0) == OK


def test_other_calls_refuse_the_format():
    """A descriptor of block-scaled experts is no descriptor of the integer formats, and the other way round."""
    n = C.c_size_t(0)
    assert B.lib().fate_moe_ffn_q_workspace(C.byref(_desc()), C.byref(n)) == ESHAPE


def test_binding_refusals():
    x = torch.zeros(4, 100, dtype=torch.bfloat16)
    mx = B.mx_empty(4, 100, device="cpu")
    assert mx[0].shape == (4, 128) and mx[1].shape == (4, 4)
    bad = [lambda: B.fate_mx_quantize(x.half(), *mx), lambda: B.fate_mx_quantize(x, mx[0][:, :100], mx[1]),
           lambda: B.fate_mx_quantize(x, mx[0], mx[1][:2]), lambda: B.fate_mx_quantize(x.t(), *mx),
           lambda: B.fate_add_rmsnorm(x, delta=x[:2], h_out=x), lambda: B.fate_add_rmsnorm(x, h_out=x.float()),
           lambda: B.fate_add_rmsnorm(x, x=x), lambda: B.fate_add_rmsnorm(x, delta=x, h_out=x),
           lambda: B.fate_add_rmsnorm(x, weight=x[0, :50], h_out=x.clone()),
           lambda: B.fate_add_rmsnorm(x, x=x.float())]
    for f in bad:
        with pytest.raises(B.FateError):
            f()


def test_ffn_binding_refusals():
    N, H, E, k = 3, 128, 4, 2
    d = B.make_ffn_desc(N, H, E, k, 64, 4, 32, 0, 0, 4, 32, True)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    good = dict(x=B.mx_empty(N, H, device="cpu"), table=torch.zeros(E * 96, dtype=torch.uint8), counts=i32(E), offsets=i32(E + 1),
                perm=i32(N * k), inv=i32(N * k), order=i32(E), w=torch.zeros(N, k), gate=None, y=torch.zeros(N, H))

    def call(**kw):
        a = dict(good, **kw)
        B.fate_moe_ffn_mx(d, *a["x"], a["table"], a["counts"], a["offsets"], a["perm"], a["inv"], a["order"], a["w"], None, a["gate"],
                          a["y"], torch.zeros(1 << 20, dtype=torch.uint8))
    bad = [dict(w=torch.zeros(N, 2 * k)[:, ::2]), dict(w=torch.zeros(N, k + 1)[:, :k]), dict(perm=i32(2 * N * k)[::2]),
           dict(counts=i32(2 * E)[::2]), dict(perm=i32(N * k - 1)), dict(offsets=i32(E)), dict(w=torch.zeros(N, k).half()),
           dict(inv=i32(N * k).long()), dict(table=torch.zeros(E * 96 - 1, dtype=torch.uint8)), dict(y=torch.zeros(N, H).t()),
           dict(y=torch.zeros(N, H).bfloat16()), dict(x=B.mx_empty(N + 1, H, device="cpu")),
           dict(gate=torch.zeros(2 * H, dtype=torch.bfloat16)[::2]), dict(gate=torch.zeros(H))]
    for kw in bad:
        with pytest.raises(B.FateError):
            call(**kw)
