"""Operators on block-scaled values against the 64-bit oracle: quantiser, packed layout, norm, products, grouped FFN.

Tolerances count roundings.  bf16 outputs: half a step, 2^-8 of the value.  fp32 sums of n terms: n 2^-24 of the sum of
magnitudes.  The 8-bit matrix instruction adds eight products at a time, cut to 2^-15 of the largest: at most seven of
them lose, 7 2^-15 = 2.2e-4 of the sum of magnitudes.
"""
import ctypes as C
import dataclasses

import numpy as np
import pytest
import torch

from oracle import moe as O
from oracle import mx as X
import paper_2502_12224_amd.binding as B
from paper_2502_12224_amd.stack import MxBuffers, MxStack, mx_layer_forward
from workloads import SHAPES, gen_expert_unquantized
from helpers import DEV, check_routing, gpu_permute

pytestmark = pytest.mark.gpu
MFMA8 = 7 * 2.0 ** -15
EPS = 1e-6


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def special(x):
    """Blocks of zeros, of values far apart, of the smallest and the largest numbers, of NaN and infinities."""
    x = x.clone()
    n, K = x.shape
    x[0] = 0
    if n > 2:
        x[1, : min(K, 32)] *= 2.0 ** -120
        x[1, K // 2] = 3e38
        x[2, 0] = float("nan")
    if n > 4:
        x[3, K - 1] = float("inf")
        x[4, :] = 2.0 ** -133 * torch.sign(x[4])
    return x


# ---- quantiser and packed layout: whole numbers, equal to the oracle's ---------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 32), (3, 33), (5, 127), (7, 128), (37, 1000), (2, 5632), (130, 200), (5, 4104)])
def test_quantize(rows, K, dtype):
    x = special(torch.randn(rows, K, generator=gen(rows * 7 + K)) * 3).to(dtype)
    wide = torch.full((rows, K + 5), 7.0, dtype=dtype)             # rows with a distance, not 16-byte aligned
    wide[:, :K] = x
    ref = X.quantize(f64(x), 8)
    for src in (x.to(DEV), wide.to(DEV)[:, :K]):
        codes, scales = (t.fill_(99) for t in B.mx_empty(rows, K))
        B.fate_mx_quantize(src, codes, scales)
        assert np.array_equal(scales.cpu().numpy(), ref[1])
        got = codes.cpu().numpy()
        nan = np.repeat(ref[1] == 255, 32, axis=1)
        # (zeros keep their sign in the device's codes)
        assert np.array_equal(X.E4M3[got], X.E4M3[ref[0]], equal_nan=True) and (got[nan] == 0x7f).all()
    codes, scales = B.mx_empty(0, K)
    B.fate_mx_quantize(x[:0].to(DEV), codes, scales)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rows,K", [(1, 1), (16, 128), (33, 129), (31, 512), (64, 640), (5, 2000)])
def test_pack_weight(rows, K, bits):
    w = special(torch.randn(rows, K, generator=gen(rows + K)) * 0.02)
    for src in (w, w.to(torch.bfloat16)):
        codes, scales = X.quantize(f64(src), bits)
        want = X.pack_weight(codes, scales, bits)
        p = B.MxWeight(src.to(DEV), bits)
        got = p.codes.cpu().numpy(), p.scales.cpu().numpy()
        assert np.array_equal(got[1], want[1])
        if bits == 8:
            assert np.array_equal(X.E4M3[got[0]], X.E4M3[want[0]], equal_nan=True)
        else:
            lo, hi = (np.array_equal(X.E2M1[a], X.E2M1[b]) for a, b in ((got[0] & 15, want[0] & 15), (got[0] >> 4, want[0] >> 4)))
            assert lo and hi
    # numbers that are block-scaled already keep their values
    q = torch.from_numpy(X.requantized(f64(w[5:] if rows > 5 else torch.ones(1, K)), bits)).to(torch.float32)
    a, b = B.MxWeight(q.to(DEV), bits), B.MxWeight(q.to(torch.bfloat16).to(DEV), bits)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)


# ---- residual addition and norm ------------------------------------------------------------------------------------

def check_norm(h, delta, weight, eps=EPS, in_place=False, outputs="hxm", pad=0):
    N, H = h.shape

    def place(t):
        if t is None or not pad:
            return None if t is None else t.to(DEV)
        wide = torch.full((t.shape[0], H + pad), -5.0, dtype=t.dtype, device=DEV)
        wide[:, :H] = t.to(DEV)
        return wide[:, :H]
    hd, dd = place(h), place(delta)
    ho = None if "h" not in outputs else hd if in_place else place(torch.full_like(h, 3))
    x = place(torch.full((N, H), 3.0, dtype=torch.bfloat16)) if "x" in outputs else None
    mx = tuple(t.fill_(99) for t in B.mx_empty(N, H)) if "m" in outputs else None
    B.fate_add_rmsnorm(hd, dd, None if weight is None else weight.to(DEV), eps, h_out=ho, x=x, mx=mx)
    s, xr = X.add_rmsnorm(f64(h), None if delta is None else f64(delta), None if weight is None else f64(weight), eps)
    # s: one fp32 addition; x: the sum's error (n 2^-24 relative, halved by the root), and five roundings
    fine = np.isfinite(xr).all(axis=1)
    rel = (H / 2 + 8) * 2.0 ** -24
    s, xr = np.where(fine[:, None], s, 0), np.where(fine[:, None], xr, np.nan)
    if ho is not None:
        step = 2.0 ** -8 if h.dtype == torch.bfloat16 else 0
        assert (np.abs(f64(ho) - s)[fine] <= (np.abs(s) * (step + 2.0 ** -24) + 1e-44)[fine]).all()
    if x is not None:
        assert (np.abs(f64(x) - xr)[fine] <= (np.abs(xr) * (2.0 ** -8 + rel * 1.01) + 1e-40)[fine]).all()
        assert np.isnan(f64(x)[~fine]).any(axis=1).all()
    if mx is not None:
        codes, scales = (t.cpu().numpy() for t in mx)
        ref = X.quantize(xr, 8)
        got = X.dequantize(codes, scales, 8, H)
        # 2^-4 of the value or half of the smallest step, from a value that is `rel` off; the scale may be the next one
        # where the largest value sits on a border
        scale = np.repeat(2.0 ** (ref[1].astype(float) - 127), 32, axis=1)[:, :H]
        bound = np.abs(xr) * (2.0 ** -4 + 2 * rel) + scale * 2.0 ** -9
        assert (np.abs(got - xr)[fine] <= bound[fine]).all()
        assert (np.abs(got - xr)[fine] > np.abs(X.dequantize(*ref, 8, H) - xr)[fine] * (1 + 1e-6) + rel * np.abs(xr)[fine] * 2).mean() < 1e-3
        assert (codes[:, H:] == 0).all() and (scales[:, -(-H // 32):] == 0).all()
        assert np.isnan(got[~fine]).any(axis=1).all()
    if pad and ho is not None:
        assert (ho.as_strided((N, pad), (H + pad, 1), H) == -5).all() if not in_place else True
    return ho, x, mx


@pytest.mark.parametrize("N,H", [(1, 1), (1, 2048), (3, 31), (5, 64), (131, 1000), (7, 4097), (2, 8192), (2, 16640), (1, 65536),
                                 (2049, 512), (2050, 1000), (2048, 2048), (2051, 4096), (6, 513)])
@pytest.mark.parametrize("types", ["bbb", "fff", "bfb", "fbn"])
def test_add_rmsnorm(N, H, types):
    t = {"b": torch.bfloat16, "f": torch.float32}
    g = gen(N + H)
    h = (torch.randn(N, H, generator=g) * 4).to(t[types[0]])
    d = torch.randn(N, H, generator=g).to(t[types[1]])
    w = None if types[2] == "n" else (1 + 0.2 * torch.randn(H, generator=g)).to(t[types[2]])
    check_norm(h, d, w)


@pytest.mark.parametrize("outputs,in_place,pad,delta", [("h", True, 0, True), ("x", False, 3, False), ("m", False, 0, True),
                                                        ("hm", True, 8, True), ("hxm", False, 5, True), ("hx", False, 16, False)])
def test_add_rmsnorm_outputs_strides_and_in_place(outputs, in_place, pad, delta):
    g = gen(5)
    h = torch.randn(9, 328, generator=g)
    check_norm(h, torch.randn(9, 328, generator=g).to(torch.bfloat16) if delta else None, None, in_place=in_place,
               outputs=outputs, pad=pad)


@pytest.mark.parametrize("N", [6, 2050])
def test_add_rmsnorm_rows_of_zeros_nan_and_infinity(N):
    h = torch.randn(N, 256, generator=gen(1))
    h[0] = 0
    h[1, 7] = float("nan")
    h[2, 100] = float("inf")
    h[3] *= 1e-18
    check_norm(h, None, None, eps=1e-6)
    ho, x, mx = check_norm(h, torch.zeros(N, 256), None, eps=0.0)           # 0 / 0 in the first row
    assert torch.isnan(x[0]).all() and (mx[1][0] == 255).all() and (mx[1][3] != 255).all()
    B.fate_add_rmsnorm(h[:0].to(DEV), h_out=h[:0].to(DEV))


# ---- dense product -------------------------------------------------------------------------------------------------

def check_linear(N, K, R, bits, x_type, y_dtype, bias, seed, pad=0, x=None):
    g = gen(seed)
    w = torch.randn(R, K, generator=g) * 0.02
    x = torch.randn(N, K, generator=g) if x is None else x
    b = torch.randn(R, generator=g) if bias else None
    W = B.MxWeight(w.to(DEV), bits)
    Wn = X.requantized(f64(w), bits)
    if x_type == "mx":
        mx = B.mx_empty(N, K)
        B.fate_mx_quantize(x.to(DEV), *mx)
        src, xn = mx, X.requantized(f64(x))
    else:
        wide = torch.full((N, K + pad), 9.0, dtype=torch.bfloat16, device=DEV)
        wide[:, :K] = x.to(torch.bfloat16)
        src, xn = wide[:, :K], f64(x.to(torch.bfloat16))
    y = torch.full((N + 1, R + pad), -77.0, dtype=y_dtype, device=DEV)
    B.fate_mx_linear(src, W, y[:N, :R], None if b is None else b.to(DEV))
    assert (y[N] == -77).all() and (y[:, R:] == -77).all()                  # nothing behind the rows or the columns
    fine = np.isfinite(xn).all(axis=1)
    ref = xn[fine] @ Wn.T + (0 if b is None else f64(b))
    mag = np.abs(xn[fine]) @ np.abs(Wn).T + (0 if b is None else np.abs(f64(b)))
    bound = mag * ((K + 8) * 2.0 ** -24 + (MFMA8 if x_type == "mx" else 0)) + np.abs(ref) * (2.0 ** -8 if y_dtype == torch.bfloat16 else 0)
    got = f64(y[:N, :R])
    assert (np.abs(got[fine] - ref) <= bound * 1.001 + 1e-37).all(), (np.abs(got[fine] - ref) / bound).max()
    assert np.isnan(got[~fine]).all()
    return y


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("N,K,R", [(1, 1, 1), (1, 4096, 300), (2, 128, 33), (5, 1000, 4099), (13, 1403, 129), (16, 640, 257),
                                   (17, 256, 64), (33, 2100, 100), (3, 14336, 40), (1, 65536, 17), (1, 384, 8200)])
@pytest.mark.parametrize("y_dtype,bias", [(torch.float32, False), (torch.bfloat16, True)])
def test_linear_bf16_rows(N, K, R, bits, y_dtype, bias):
    check_linear(N, K, R, bits, "bf16", y_dtype, bias, N + K + R, pad=0 if K % 2 == 0 else 3)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("N,K,R", [(1, 1, 1), (1, 4096, 300), (4, 128, 4099), (16, 1403, 257), (16, 14336, 70), (17, 2048, 129),
                                   (31, 384, 512), (33, 512, 255), (64, 1408, 256), (65, 900, 260), (129, 2048, 300), (300, 640, 1030),
                                   (1000, 128, 64)])
@pytest.mark.parametrize("y_dtype,bias", [(torch.float32, True), (torch.bfloat16, False)])
def test_linear_8bit_rows(N, K, R, bits, y_dtype, bias):
    check_linear(N, K, R, bits, "mx", y_dtype, bias, N + K + R, pad=0 if R % 2 == 0 else 1)


@pytest.mark.parametrize("x_type", ["bf16", "mx"])
@pytest.mark.parametrize("N", [5, 40])
def test_linear_keeps_nan_and_infinity_to_their_token(N, x_type):
    x = torch.randn(N, 300, generator=gen(3))
    x[1, 5] = float("nan")
    x[N - 1, 299] = float("inf")
    # an infinity times weights that are not zero everywhere is infinite or, added up, NaN; the other tokens are fine
    if x_type == "bf16":
        x[N - 1, 0] = -float("inf")
        x[N - 1, 299] = float("nan")
    check_linear(N, 300, 90, 4, x_type, torch.float32, False, 3, x=x)


# ---- grouped FFN ---------------------------------------------------------------------------------------------------

class Ffn:
    """Experts of one layer as packed matrices and as the numbers they stand for."""

    def __init__(self, H, E, I, bits, n_shared=0, I_shared=0, shared_bits=4, seed=0, absent=(), sizes=None):
        g = gen(seed)
        self.H, self.E, self.I, self.bits, self.n_shared, self.I_shared, self.shared_bits = H, E, I, bits, n_shared, I_shared, shared_bits
        self.numbers, self.keep, structs = {}, [], []

        def make(I, b):
            mats = [torch.randn(*s, generator=g) * 0.05 for s in ((I, H), (I, H), (H, I))]
            ex = B.MxExpert(*(B.MxWeight(m.to(DEV), b) for m in mats))
            self.keep.append(ex)
            return tuple(X.requantized(f64(m), b) for m in mats), ex.struct()
        for e in range(E):
            n, st = make(I if sizes is None else sizes[e % len(sizes)], bits if isinstance(bits, int) else bits[e % len(bits)])
            if e in absent:
                st = B.fate_qexpert(0, 0, 0, 0, 0, 0, 4, 32, I, 0)
            else:
                self.numbers[e] = n
            structs.append(st)
        both = [make(I_shared, shared_bits) for _ in range(n_shared)]
        self.shared = [n for n, _ in both]
        self.structs = structs
        self.table = B.expert_table(structs)
        self.shared_table = B.expert_table([s for _, s in both]) if n_shared else None

    def desc(self, N, k, y_fp32=True):
        return B.make_ffn_desc(N, self.H, self.E, k, self.I, self.bits if isinstance(self.bits, int) else self.bits[0], 32,
                               self.n_shared, self.I_shared, self.shared_bits, 32, y_fp32)

    def run(self, mx, ids, w, gate=None, y_fp32=True, fill=0xff, stream=None):
        N, k = ids.shape
        d = self.desc(N, k, y_fp32)
        perm = gpu_permute(ids.to(DEV), self.E)
        ws = torch.full((B.fate_moe_ffn_mx_workspace(d),), fill, dtype=torch.uint8, device=DEV)
        ws[:256] = 0
        y = torch.full((N, self.H), float("nan"), dtype=torch.float32 if y_fp32 else torch.bfloat16, device=DEV)
        B.fate_moe_ffn_mx(d, *mx, self.table, *perm, w.to(DEV), self.shared_table, None if gate is None else gate.to(DEV), y, ws)
        torch.cuda.synchronize()
        return y, int(ws[:4].view(torch.int32)[0])


def routing(N, k, E, seed, skew=0.0):
    g = gen(seed)
    z = torch.randn(N, E, generator=g) - skew * torch.arange(E)
    p, ids = torch.topk(torch.softmax(z, dim=-1), k, dim=-1)
    return ids.to(torch.int32).contiguous(), p.contiguous()


def check_ffn(f, N, k, seed, y_fp32=True, gate=False, skew=0.0, ids=None, x=None, status=0):
    """Error of a row over its norm.  h is off by about 1e-4 of itself at most (MFMA8 with the signs of real data), a step
    of E4M3 is 2^-4 to 2^-3 of it, so a share of 1e-4 / 2^-4 = 1.6e-3 of the values at most rounds the other way and is off
    by 2^-3: sqrt(1.6e-3) / 8 = 5e-3 of the row, and more by sqrt(256 / I) where there are few of them to average.  That is
    an average over many values, but h has a long tail, and one of its largest values alone may round the other way: a row
    is allowed that flip beside (the value's step times its column of W2).  bf16: 2^-8 for y."""
    xf = torch.randn(N, f.H, generator=gen(seed)) if x is None else x
    mx = B.mx_empty(N, f.H)
    B.fate_mx_quantize(xf.to(DEV), *mx)
    r, w = routing(N, k, f.E, seed + 1, skew)
    ids = r if ids is None else ids
    sg = (torch.randn(f.H, generator=gen(seed + 2)) / f.H ** 0.5).to(torch.bfloat16) if gate else None
    y, st = f.run(mx, ids, w, sg, y_fp32)
    xn = X.requantized(f64(xf))
    ref = X.moe_ffn(xn, ids.numpy(), f64(w), f.numbers, f.shared, None if sg is None else f64(sg))
    got = f64(y)
    fine = np.isfinite(xn).all(axis=1)
    flip = np.nan_to_num(X.moe_ffn(xn, ids.numpy(), f64(w), f.numbers, f.shared, None if sg is None else f64(sg),
                                   lambda *m: np.tile(X.largest_flip(*m)[:, None], (1, f.H)))[:, 0])
    err = np.maximum(np.linalg.norm(got - ref, axis=1) - flip, 0)[fine] / np.maximum(np.linalg.norm(ref, axis=1)[fine], 1e-30)
    if N >= 10:     # the largest values do not flip in most rows
        assert np.median(np.linalg.norm(got - ref, axis=1)[fine] / np.maximum(np.linalg.norm(ref, axis=1)[fine], 1e-30)) <= \
            7.5e-3 * max(1.0, (256 / f.I) ** 0.5) + 2.0 ** -7
    tol = 5e-3 * max(1.0, (256 / f.I) ** 0.5) * 1.5 + (0 if y_fp32 else 2.0 ** -8)
    zero = np.linalg.norm(ref, axis=1)[fine] == 0
    assert (got[fine][zero] == 0).all() and (err[~zero] <= tol).all(), (err.max(), tol)
    assert np.isnan(got[~fine]).all()
    assert st == status
    return y


@pytest.mark.parametrize("N", [1, 2, 8, 13, 16, 17, 40, 150, 600])
@pytest.mark.parametrize("H,E,k,I,bits,ns,Is,sb", [(256, 8, 2, 512, 4, 0, 0, 4), (384, 10, 3, 288, 8, 2, 256, 4),
                                                   (2048, 12, 4, 352, 4, 1, 1440, 8), (32, 5, 1, 256, 4, 1, 160, 4)])
def test_ffn(N, H, E, k, I, bits, ns, Is, sb):
    f = Ffn(H, E, I, bits, ns, Is, sb, seed=H + I)
    check_ffn(f, N, k, N, y_fp32=N % 2 == 0, gate=ns == 1, skew=0.4 if N > 100 else 0.0)


@pytest.mark.parametrize("name,N", [("tiny", 5), ("qwen", 1), ("qwen", 13), ("deepseek", 8), ("mixtral", 1), ("deepseek", 48),
                                    ("qwen_prefill", 131), ("qwen_prefill", 512)])
def test_ffn_on_the_configured_shapes(name, N):
    """Widths of the configurations; as many experts as the oracle does in a few seconds."""
    c = SHAPES[name]
    E, I = min(c.E, 16), min(c.I, 2048)
    f = Ffn(c.H, E, I, c.bits, c.n_shared, c.I_shared, c.shared_bits, seed=3)
    check_ffn(f, N, c.k, N + 1, y_fp32=False, gate=c.shared_gate, skew=c.zipf_s / 4)


@pytest.mark.parametrize("N", [6, 90])
def test_ffn_mixed_widths_and_sizes(N):
    """4- and 8-bit copies in one layer, and entries of fewer neurons than I_max."""
    f = Ffn(256, 9, 416, (4, 8), sizes=(416, 32, 256), seed=4)
    check_ffn(f, N, 3, N)


def test_ffn_binding_refusals():
    f = Ffn(64, 4, 64, 4, 1, 64, seed=1)
    ids, w = routing(3, 2, 4, 1)
    d, tabs, mx = f.desc(3, 2), gpu_permute(ids.to(DEV), 4), B.mx_empty(3, 64)
    B.fate_mx_quantize(torch.zeros(3, 64, device=DEV), *mx)
    ws = torch.zeros(B.fate_moe_ffn_mx_workspace(d), dtype=torch.uint8, device=DEV)
    good = [d, *mx, f.table, *tabs, w.to(DEV), f.shared_table, None, torch.empty(3, 64, device=DEV), ws]
    B.fate_moe_ffn_mx(*good)
    for i, bad in [(1, mx[0][:2]), (2, mx[1].cpu()), (3, f.table[:100]), (4, tabs[0].long()), (5, tabs[1][:4]), (6, tabs[2].long()),
                   (7, tabs[3][:5]), (9, w.to(DEV).double()), (9, w.to(DEV)[:2]), (10, None), (10, f.shared_table[:50]),
                   (11, torch.zeros(64, device=DEV)), (12, torch.empty(3, 64, device=DEV, dtype=torch.bfloat16)), (13, ws[:-300])]:
        with pytest.raises(B.FateError):
            B.fate_moe_ffn_mx(*good[:i], bad, *good[i + 1:])


@pytest.mark.parametrize("E,k,ns,gate,y_fp32", [(1, 1, 0, False, True), (200, 8, 2, True, True), (256, 20, 3, True, False),
                                                (7, 3, 1, False, False), (70, 64, 1, True, True)])
def test_ffn_single_token(E, k, ns, gate, y_fp32):
    """One token: all its down products in one launch, many terms, experts named twice, absent ones, other widths."""
    f = Ffn(96, E, 64 if E > 100 else 288, (4, 8), ns, 480, 8, sizes=(64, 32) if E > 100 else (288, 96, 32), seed=E + k,
            absent=(E - 1,) if E > 1 else ())
    r, _ = routing(1, k, E, 5)
    status = 1 if E > 1 and E - 1 in r else 0
    check_ffn(f, 1, k, 4, y_fp32=y_fp32, gate=gate and ns > 0, status=status)
    ids = r.clone()
    ids[0, k // 2:] = ids[0, 0]
    if E > 1:
        ids[0, k - 1] = E - 1
    check_ffn(f, 1, k, 4, y_fp32=y_fp32, gate=gate and ns > 0, ids=ids, status=1 if E > 1 else 0)


@pytest.mark.parametrize("N,y_fp32", [(20, True), (40, False), (300, False)])
def test_ffn_long_reductions_in_parts(N, y_fp32):
    """A down product of few workgroups and a long reduction is cut into parts; entries shorter than a part's start."""
    f = Ffn(256, 4, 4608, 4, 1, 4608, 8, sizes=(4608, 32, 2336, 4608), seed=12)
    check_ffn(f, N, 2, N, y_fp32=y_fp32)


@pytest.mark.parametrize("N", [1, 2, 20, 70, 300])
def test_ffn_rounds_once_to_bf16(N):
    """The terms of a token's sum, parts of products among them, are fp32: a bf16 output is the fp32 one rounded."""
    f = Ffn(512, 4, 2304, 4, 1, 4608, 8, seed=21)
    ids, w = routing(N, 2, 4, N)
    mx = B.mx_empty(N, 512)
    B.fate_mx_quantize(torch.randn(N, 512, generator=gen(N)).to(DEV), *mx)
    gate = torch.randn(512, generator=gen(3)).to(torch.bfloat16)
    y, _ = f.run(mx, ids, w, gate, True)
    yb, _ = f.run(mx, ids, w, gate, False)
    assert torch.equal(yb, y.to(torch.bfloat16))


@pytest.mark.parametrize("N", [4, 70])
def test_ffn_absent_and_unreadable_experts(N):
    f = Ffn(256, 6, 256, 4, 1, 128, seed=5, absent=(1, 4))
    check_ffn(f, N, 3, N, status=1)
    st = f.structs[2]
    st.group = 128                              # an integer format's entry
    f.table = B.expert_table(f.structs)
    del f.numbers[2]
    check_ffn(f, N, 3, N, status=5)
    if N > 4:                                   # a table entry that is only partly there
        f.structs[0].w2 = None
        f.structs[3].s3 = None
        f.table = B.expert_table(f.structs)
        del f.numbers[0], f.numbers[3]
        check_ffn(f, N, 3, N, status=5)
    f.structs = [B.fate_qexpert(0, 0, 0, 0, 0, 0, 4, 32, 256, 0)] * 6
    f.table, f.numbers, f.shared_table, f.n_shared, f.shared = B.expert_table(f.structs), {}, None, 0, []
    y = check_ffn(f, N, 3, N, status=1)
    assert (y == 0).all()


@pytest.mark.parametrize("N", [3, 16, 50, 200])
def test_ffn_one_expert_takes_everything(N):
    """Every token names one expert, several times: groups of k N rows, the others empty."""
    f = Ffn(256, 7, 256, 4, seed=6)
    check_ffn(f, N, 4, N, ids=torch.full((N, 4), 3, dtype=torch.int32))


@pytest.mark.parametrize("N", [5, 60])
def test_ffn_nan_reaches_its_own_token_only(N):
    x = torch.randn(N, 256, generator=gen(8))
    x[2, 9] = float("nan")
    x[N - 1, 255] = -float("inf")
    check_ffn(Ffn(256, 4, 256, 4, 1, 256, seed=7), N, 2, N, x=x)


@pytest.mark.parametrize("N", [8, 120])
def test_ffn_reads_scales_of_all_sizes(N):
    """Rows of 2^-60 to 2^30: the up product scales with them, SwiGLU makes zero or the product of it."""
    x = torch.randn(N, 256, generator=gen(9)) * torch.exp2(torch.linspace(-60, 5, N)).unsqueeze(1)
    check_ffn(Ffn(256, 4, 256, 8, seed=8), N, 2, N, x=x)


def test_ffn_without_tokens_and_same_bits_every_time():
    f = Ffn(256, 8, 256, 4, 1, 128, seed=9)
    d = f.desc(0, 2)
    mx = B.mx_empty(0, 256)
    B.fate_moe_ffn_mx(d, *mx, f.table, *gpu_permute(torch.zeros(1, 2, dtype=torch.int32, device=DEV), 8),
                      torch.zeros(1, 2, device=DEV), f.shared_table, None, torch.empty(0, 256, device=DEV),
                      torch.zeros(B.fate_moe_ffn_mx_workspace(d), dtype=torch.uint8, device=DEV))
    for N in (3, 100):
        assert torch.equal(check_ffn(f, N, 2, N), check_ffn(f, N, 2, N))


# ---- together ------------------------------------------------------------------------------------------------------

def _small(name="mxtest"):
    return dataclasses.replace(SHAPES["tiny"], name=name, bits=4, group=128, layers=2, n_shared=1, I_shared=384, shared_bits=8,
                               shared_gate=True)


def _numbers(cfg, layer, e, shared=False):
    return tuple(X.requantized(f64(w), cfg.shared_bits if shared else cfg.bits)
                 for w in gen_expert_unquantized(cfg, layer, e, shared, DEV))


@pytest.mark.parametrize("N", [1, 5, 40])
def test_stack_of_layers_with_head(N):
    """Norm, routing, FFN and head as a program runs them; every stage against the oracle on the stage's own inputs."""
    cfg = _small()
    st = MxStack(cfg, layers=2, vocabulary=300)
    buf = MxBuffers(cfg, N, DEV)
    h = torch.randn(N, cfg.H, generator=gen(N)).to(DEV)
    y = None
    for l, lw in enumerate(st.layers):
        before, prev = f64(h), None if y is None else f64(y)
        y = mx_layer_forward(cfg, lw, st.layers[l + 1] if l == 0 else None, h, y, buf)
        s, x = X.add_rmsnorm(before, prev, None, EPS)
        assert np.abs(f64(h) - s).max() <= 2.0 ** -23 * np.abs(s).max()
        assert np.abs(f64(buf.x) - x).max() <= 2.0 ** -7 * np.abs(x).max()
        xb = buf.x.float().cpu().numpy()
        rid, rw, _, rz = O.gate_route(xb, lw.Wg.float().cpu().numpy(), None, cfg.k, cfg.renorm)
        check_routing(buf.ids, buf.w, rid, rw, rz, cfg.k)
        x8 = X.dequantize(*(t.cpu().numpy() for t in buf.mx), 8, cfg.H)
        ref = X.moe_ffn(x8, buf.ids.cpu().numpy(), f64(buf.w), {e: _numbers(cfg, l, e) for e in range(cfg.E)},
                        [_numbers(cfg, l, 0, True)], f64(lw.shared_gate))
        flip = X.moe_ffn(x8, buf.ids.cpu().numpy(), f64(buf.w), {e: _numbers(cfg, l, e) for e in range(cfg.E)},
                         [_numbers(cfg, l, 0, True)], f64(lw.shared_gate),
                         lambda *m: np.tile(X.largest_flip(*m)[:, None], (1, cfg.H)))[:, 0]
        err = (np.linalg.norm(f64(y) - ref, axis=1) - flip) / np.linalg.norm(ref, axis=1)
        assert (err <= 7.5e-3).all() and buf.status() == 0
    h2 = torch.randn(N, cfg.H, generator=gen(N)).to(DEV)
    logits = st.forward(h2, buf)
    assert logits.shape == (N, 300) and torch.isfinite(logits).all()
    assert torch.equal(logits, st.forward(torch.randn(N, cfg.H, generator=gen(N)).to(DEV), buf))


@pytest.mark.parametrize("N", [4, 64])
def test_captured_and_replayed(N):
    """A graph of the whole stack, replayed with other work between the replays, gives the eager results."""
    cfg = _small()
    st, buf = MxStack(cfg, layers=2, vocabulary=200), MxBuffers(cfg, N, DEV)
    h, logits = torch.empty(N, cfg.H, device=DEV), torch.empty(N, 200, device=DEV)
    start = torch.empty_like(h)

    def step():
        h.copy_(start)
        st.forward(h, buf, logits)
    start.copy_(torch.randn(N, cfg.H, generator=gen(0)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        start.copy_(torch.randn(N, cfg.H, generator=gen(i)))
        step()
        want = logits.clone()
        torch.cuda.synchronize()
        logits.fill_(0)
        torch.randn(1000, 1000, device=DEV).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(logits, want)


def test_two_streams_with_workspaces_of_their_own():
    f = Ffn(256, 8, 256, 4, seed=10)
    ids, w = routing(30, 2, 8, 1)
    xs = [torch.randn(30, 256, generator=gen(i)).to(DEV) for i in range(2)]
    d, tabs = f.desc(30, 2), gpu_permute(ids.to(DEV), 8)
    wd = w.to(DEV)
    want, got, state = [], [], []
    for x in xs:
        mx = B.mx_empty(30, 256)
        B.fate_mx_quantize(x, *mx)
        state.append((mx, torch.zeros(B.fate_moe_ffn_mx_workspace(d), dtype=torch.uint8, device=DEV)))
        y = torch.empty(30, 256, device=DEV)
        B.fate_moe_ffn_mx(d, *mx, f.table, *tabs, wd, None, None, y, state[-1][1])
        want.append(y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [torch.empty(30, 256, device=DEV) for _ in range(2)]
    for _ in range(5):
        for s, (mx, ws), y in zip(streams, state, got):
            B.fate_moe_ffn_mx(d, *mx, f.table, *tabs, wd, None, None, y, ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_copy_engine_brings_block_scaled_experts():
    """Experts of the format in a pinned pool: the cache step and its copy engine put them into slots and write entries
    that the FFN reads."""
    H, E, I, N = 256, 6, 256, 9
    f = Ffn(H, E, I, 4, seed=11)
    lib = B.lib()
    wc, ws = B.fate_mx_weight_bytes(I, H, 4)
    assert (wc, ws) == B.fate_mx_weight_bytes(H, I, 4)
    layout = B.fate_slot_layout(3 * (wc + ws), 0, wc, 2 * wc, 3 * wc, 3 * wc + ws, 3 * wc + 2 * ws, 4, 32, I)
    pool = torch.empty(E, layout.slot_bytes, dtype=torch.uint8, pin_memory=True)
    for e, ex in enumerate(f.keep):
        m = (ex.w1, ex.w3, ex.w2)
        pool[e].copy_(torch.cat([t.codes for t in m] + [t.scales for t in m]).cpu())
    total, staging = 2, 6
    slots_dev = torch.zeros(total + staging, layout.slot_bytes, dtype=torch.uint8, device=DEV)
    table = torch.zeros(E * C.sizeof(B.fate_qexpert), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    eng = lib.fate_hip_engine_create(1, E, total + staging, C.byref(layout), slots_dev.data_ptr(), pool.data_ptr(),
                                     table.data_ptr(), side.cuda_stream, torch.cuda.current_stream().cuda_stream)
    assert eng
    fn = B.COPY_FN(("fate_hip_engine_copy", lib))
    cache = lib.fate_cache_create(1, E, total, 0, 0, staging, fn, C.c_void_p(eng))
    try:
        for e in range(E):
            s = lib.fate_cache_slot_of(cache, 0, e)
            if s >= 0:
                B._check(lib.fate_hip_engine_preload(eng, 0, e, s))
        ids, w = routing(N, 2, E, 3)
        counts = torch.bincount(ids.reshape(-1).long(), minlength=E).to(torch.int32)
        order, slots, loads, n, st = (C.c_int32 * E)(), (C.c_int32 * E)(), (B.fate_cache_load * 16)(), C.c_int32(0), B.fate_cache_stats()
        B._check(lib.fate_hip_engine_begin_step(eng, None))
        B._check(lib.fate_expert_cache_step_dense(cache, 0, counts.data_ptr(), None, order, slots, C.byref(n), loads, 16, C.byref(st)))
        B._check(lib.fate_hip_engine_wait_ready(eng, slots, n.value))
        assert st.n_miss > 0
        mx = B.mx_empty(N, H)
        B.fate_mx_quantize(torch.randn(N, H, generator=gen(2)).to(DEV), *mx)
        want, _ = f.run(mx, ids, w)
        f.table = table
        got, status = f.run(mx, ids, w)
        assert status == 0 and torch.equal(got, want)
    finally:
        torch.cuda.synchronize()
        lib.fate_cache_destroy(cache)
        lib.fate_hip_engine_destroy(eng)
