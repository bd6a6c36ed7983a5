"""Performance cases of the operators on block-scaled 8- and 4-bit values.

Four operators, each called as a serving program calls it: the residual addition
with its root-mean-square norm and 8-bit output (`norm`), the quantisation of
rows (`quantize`), the product with one dense weight matrix (`linear`), and the
mixture-of-experts feed-forward over ragged groups of rows (`ffn`).

A value held in 8 bits is an E4M3 code (in 4 bits an E2M1 code) times a power of
two that 32 consecutive values of a row share.  With `own` false, `run` computes
the operators in elementary torch operations in 32 bits; with `own` true it calls
the library.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 32      # values that share a scale
STEP = 128      # rows of codes are padded with zeros to a multiple of this
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _case(name, kind, **options):
    case = {"name": name, "kind": kind}
    case.update(options)
    return case


def _norm(name, N, H, h_type="fp32", delta_type="fp32", weight="bf16"):
    return _case(name, "norm", N=N, H=H, h_type=h_type, delta_type=delta_type, weight=weight)


def _quantize(name, N, K, type="bf16"):
    return _case(name, "quantize", N=N, K=K, type=type)


def _linear(name, N, K, R, bits=4, x_type="bf16", y_type="bf16", bias=False):
    return _case(name, "linear", N=N, K=K, R=R, bits=bits, x_type=x_type, y_type=y_type, bias=bias)


def _ffn(name, N, H, E, k, I, bits=4, n_shared=0, I_shared=0, shared_bits=4, shared_gate=False, zipf=0.0):
    return _case(name, "ffn", N=N, H=H, E=E, k=k, I=I, bits=bits, n_shared=n_shared, I_shared=I_shared,
                 shared_bits=shared_bits, shared_gate=shared_gate, zipf=zipf)


def listed():
    return [
        # one user generating: the norm between two layers, nothing but latency
        _norm("norm_1", 1, 2048),
        # a short odd prompt on a model whose width is no multiple of the padding, everything kept in bf16
        _norm("norm_131_odd", 131, 1000, "bf16", "bf16", "fp32"),
        # a long packed prefill: memory bandwidth
        _norm("norm_16384", 16384, 4096, "bf16", "bf16"),
        # an odd batch of rows made elsewhere (the wide intermediate of a shared expert)
        _quantize("quantize_37", 37, 5632),
        # a long prefill's rows, kept in fp32 before
        _quantize("quantize_8192", 8192, 4096, "fp32"),
        # one user generating: logits over a vocabulary from bf16 activations, weight bytes and nothing else
        _linear("linear_1_vocabulary", 1, 4096, 32000, y_type="fp32"),
        # an odd decode batch through a small 8-bit projection with a bias, no size a multiple of anything
        _linear("linear_13_odd", 13, 1403, 4099, bits=8, bias=True),
        # a prompt through a projection on 8-bit activations: matrix cores
        _linear("linear_2048", 2048, 4096, 4096, x_type="mx"),
        # one user generating: 4 of 60 fine-grained experts and a gated shared one
        _ffn("ffn_qwen_1", 1, 2048, 60, 4, 1408, n_shared=1, I_shared=5632, shared_gate=True),
        # a small decode batch: most of the experts are read for one or two rows, 8-bit shared experts
        _ffn("ffn_deepseek_8", 8, 2048, 64, 6, 1408, n_shared=2, I_shared=1408, shared_bits=8),
        # a prompt with skewed routing: ragged groups from no row to hundreds
        _ffn("ffn_qwen_512", 512, 2048, 60, 4, 1408, n_shared=1, I_shared=5632, shared_gate=True, zipf=1.1),
        # a long prompt on few large experts: matrix cores
        _ffn("ffn_mixtral_2048", 2048, 4096, 8, 2, 14336),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    kind = rng.choice(["norm", "quantize", "linear", "linear", "ffn", "ffn"])
    if kind == "norm":
        case = _norm("", _log_int(rng, 1, 16384), _log_int(rng, 64, 4096), rng.choice(["bf16", "fp32"]),
                     rng.choice(["bf16", "fp32"]), rng.choice(["bf16", "fp32"]))
        if rng.random() < 0.5:
            case["H"] = -(-case["H"] // 128) * 128
    elif kind == "quantize":
        case = _quantize("", _log_int(rng, 1, 8192), _log_int(rng, 33, 6000), rng.choice(["bf16", "fp32"]))
    elif kind == "linear":
        case = _linear("", _log_int(rng, 1, 2048), _log_int(rng, 64, 4096), _log_int(rng, 64, 32000),
                       rng.choice([4, 4, 8]), rng.choice(["bf16", "mx"]), "bf16", rng.random() < 0.3)
        if case["x_type"] == "bf16" or rng.random() < 0.3:   # prompts come as 8-bit rows; bf16 rows are a decode batch
            case["N"] = _log_int(rng, 1, 64)
        if rng.random() < 0.5:
            case["K"] = -(-case["K"] // 128) * 128
        if case["x_type"] == "bf16" and rng.random() < 0.3:
            case["y_type"] = "fp32"
    else:
        n_shared = rng.randint(0, 2)
        case = _ffn("", _log_int(rng, 1, 1024), 256 * rng.randint(1, 16), rng.randint(4, 96), rng.randint(1, 4),
                    32 * rng.randint(4, 56), rng.choice([4, 4, 8]), n_shared, 32 * rng.randint(4, 100) if n_shared else 0,
                    rng.choice([4, 8]), n_shared > 0 and rng.random() < 0.5, rng.choice([0.0, 0.0, 1.1]))
        # as many experts as stay within about 1.2 G weights
        case["E"] = max(case["k"], min(case["E"], int(1.2e9 / (3.0 * case["H"] * case["I"]))))
    del case["name"]
    return case


# ---- the format ------------------------------------------------------------------------------------------------

def _pad(x, to=STEP):
    """Rows of x with zeros up to a multiple of `to`."""
    K = x.shape[-1]
    Kp = -(-K // to) * to
    return x if Kp == K else torch.nn.functional.pad(x, (0, Kp - K))


def _block_exponent(blocks, top):
    """Smallest power of two (its exponent) that leaves no value of a block above top = 1.75 * 2^8 or 1.5 * 2^2.
    frexp: amax = m * 2^e with m in [0.5, 1)."""
    m, e = torch.frexp(blocks.abs().amax(dim=-1, keepdim=True))
    limit, lead = (0.875, 9) if top == 448 else (0.75, 3)
    e = torch.clamp(e - lead + (m > limit).to(e.dtype), -127, 127)
    return torch.where(m == 0, torch.full_like(e, -127), e)


def _to_e4m3(x):
    """Rows [.., K] in 32 bits -> (E4M3 codes [.., Kp], scale bytes [.., Kp / 32])."""
    x = _pad(x)
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    e = _block_exponent(blocks, 448)
    codes = torch.ldexp(blocks, -e).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.reshape(x.shape), (e + 127).to(torch.uint8).squeeze(-1)


def _from_e4m3(codes, scales, dtype=torch.float32):
    v = codes.view(torch.float8_e4m3fn).to(dtype)
    v = v.reshape(*v.shape[:-1], -1, BLOCK) * _scale(scales, dtype).unsqueeze(-1)
    return v.reshape(codes.shape)


def _scale(scales, dtype):
    return torch.ldexp(torch.ones((), dtype=dtype, device=scales.device), scales.to(torch.int32) - 127)


def _to_e2m1(w):
    """Rows [.., K] in 32 bits -> (two E2M1 codes per byte, even column low [.., Kp / 2], scale bytes [.., Kp / 32])."""
    w = _pad(w)
    blocks = w.reshape(*w.shape[:-1], -1, BLOCK)
    e = _block_exponent(blocks, 6)
    v = torch.ldexp(blocks, -e)
    a = v.abs()
    # to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6; a tie goes to the even code
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + 8 * (v < 0)).reshape(w.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8).squeeze(-1)


def _from_weight(codes, scales, bits, dtype=torch.float32):
    """Stored weights [.., R, Kp] as numbers."""
    if bits == 8:
        return _from_e4m3(codes, scales, dtype)
    table = torch.tensor(_E2M1 + [-v for v in _E2M1], dtype=dtype, device=codes.device)
    byte = torch.arange(256, device=codes.device)
    pair = torch.stack([table[byte & 15], table[byte >> 4]], dim=-1)
    v = pair[codes.to(torch.int32)].reshape(*codes.shape[:-1], -1, BLOCK) * _scale(scales, dtype).unsqueeze(-1)
    return v.reshape(*codes.shape[:-1], -1)


# ---- inputs ----------------------------------------------------------------------------------------------------

def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _stored(g, count, R, K, bits):
    """`count` weight matrices [R, K], N(0, 0.02), stored in `bits`: (codes [count, R, ..], scales [count, R, Kp / 32])."""
    both = []
    for _ in range(count):
        w = _randn(g, R, K) * 0.02
        both.append(_to_e2m1(w) if bits == 4 else _to_e4m3(w))
    return torch.stack([c for c, _ in both]), torch.stack([s for _, s in both])


def _inputs(case, seed):
    """What both sides start from; weights as stored rows."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 17)
    kind = case["kind"]
    s = {"case": case}
    if kind == "norm":
        N, H = case["N"], case["H"]
        # a residual stream with a few wide channels, and a layer's output
        wide = 1 + 20 * (torch.rand(H, generator=g, device="cuda") < 0.01).to(torch.float32)
        s["h"] = (_randn(g, N, H) * wide).to(_TYPES[case["h_type"]])
        s["delta"] = (_randn(g, N, H) * 0.3).to(_TYPES[case["delta_type"]])
        s["weight"] = (1 + 0.1 * _randn(g, H)).to(_TYPES[case["weight"]])
    elif kind == "quantize":
        s["x"] = (_randn(g, case["N"], case["K"]) * torch.exp(0.5 * _randn(g, case["N"], 1))).to(_TYPES[case["type"]])
    elif kind == "linear":
        x = _randn(g, case["N"], case["K"])
        s["x"] = _to_e4m3(x) if case["x_type"] == "mx" else x.to(torch.bfloat16)
        s["w"] = _stored(g, 1, case["R"], case["K"], case["bits"])
        s["bias"] = _randn(g, case["R"]) if case["bias"] else None
    else:
        N, H, E, k, I = (case[n] for n in ("N", "H", "E", "k", "I"))
        logits = _randn(g, N, E)
        if case["zipf"]:
            rank = torch.randperm(E, generator=g, device="cuda").to(torch.float32) + 1
            logits = logits - case["zipf"] * torch.log(rank)
        top, ids = torch.topk(logits, k, dim=-1)
        p = torch.softmax(logits, dim=-1)
        s["w"] = torch.gather(p, 1, ids).contiguous()
        pairs = ids.reshape(-1)
        s["ids"] = ids.to(torch.int32).contiguous()
        s["counts"] = torch.bincount(pairs, minlength=E).to(torch.int32)
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.cumsum(s["counts"], 0)]).to(torch.int32)
        perm = torch.argsort(pairs, stable=True)
        s["perm"] = perm.to(torch.int32)
        s["inv_perm"] = torch.argsort(perm).to(torch.int32)
        s["order"] = torch.argsort(s["counts"], stable=True, descending=True).to(torch.int32)
        s["capacity"] = int(s["counts"].max())
        s["x"] = _to_e4m3(_randn(g, N, H))
        for name, R, K in (("w1", I, H), ("w3", I, H), ("w2", H, I)):
            s[name] = _stored(g, E, R, K, case["bits"])
        if case["n_shared"]:
            for name, R, K in (("v1", case["I_shared"], H), ("v3", case["I_shared"], H), ("v2", H, case["I_shared"])):
                s[name] = _stored(g, case["n_shared"], R, K, case["shared_bits"])
        s["gate"] = (_randn(g, H) / math.sqrt(H)).to(torch.bfloat16) if case["shared_gate"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _prepare_own(s)
    return s


def _pack(B, stored, bits, R, K):
    """The library's layout of every stored matrix; packing numbers that are block-scaled already keeps them as they are."""
    return [B.MxWeight(_from_weight(c, e, bits)[:, :K].to(torch.bfloat16).contiguous(), bits)
            for c, e in zip(*stored)]


def _prepare_own(s):
    """What a program keeps: weights in the library's layout, outputs and workspace."""
    import paper_2502_12224_amd.binding as B
    case = s["case"]
    dev = dict(device="cuda")
    if case["kind"] == "norm":
        N, H = case["N"], case["H"]
        s["out"] = {"h": torch.empty_like(s["h"]), "x": torch.empty(N, H, dtype=torch.bfloat16, **dev),
                    "mx": B.mx_empty(N, H)}
    elif case["kind"] == "quantize":
        s["out"] = B.mx_empty(case["N"], case["K"])
    elif case["kind"] == "linear":
        s["packed"] = _pack(B, s.pop("w"), case["bits"], case["R"], case["K"])[0]
        s["out"] = torch.empty(case["N"], case["R"], dtype=_TYPES[case["y_type"]], **dev)
    else:
        I, H, Is = case["I"], case["H"], case["I_shared"]
        mats = [_pack(B, s.pop(n), case["bits"], R, K) for n, R, K in (("w1", I, H), ("w3", I, H), ("w2", H, I))]
        s["experts"] = [B.MxExpert(*m) for m in zip(*mats)]
        s["table"] = B.expert_table([e.struct() for e in s["experts"]])
        s["shared_table"] = None
        if case["n_shared"]:
            mats = [_pack(B, s.pop(n), case["shared_bits"], R, K) for n, R, K in (("v1", Is, H), ("v3", Is, H), ("v2", H, Is))]
            s["shared"] = [B.MxExpert(*m) for m in zip(*mats)]
            s["shared_table"] = B.expert_table([e.struct() for e in s["shared"]])
        s["desc"] = B.make_ffn_desc(case["N"], H, case["E"], case["k"], I, case["bits"], 32, case["n_shared"], Is,
                                    case["shared_bits"], 32, y_is_fp32=False)
        s["workspace"] = torch.zeros(B.fate_moe_ffn_mx_workspace(s["desc"]), dtype=torch.uint8, **dev)
        s["out"] = torch.empty(case["N"], H, dtype=torch.bfloat16, **dev)


# ---- one pass --------------------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _values(codes, scales):
    """8-bit outputs as the numbers that codes and scales stand for."""
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}


EPS = 1e-6


def _run_own(s):
    import paper_2502_12224_amd.binding as B
    kind = s["case"]["kind"]
    if kind == "norm":
        out = s["out"]
        B.fate_add_rmsnorm(s["h"], s["delta"], s["weight"], EPS, h_out=out["h"], x=out["x"], mx=out["mx"])
        return {"h": out["h"], "x": out["x"], **_values(*out["mx"])}
    if kind == "quantize":
        B.fate_mx_quantize(s["x"], *s["out"])
        return _values(*s["out"])
    if kind == "linear":
        B.fate_mx_linear(s["x"], s["packed"], s["out"], bias=s["bias"])
        return s["out"]
    B.fate_moe_ffn_mx(s["desc"], *s["x"], s["table"], s["counts"], s["offsets"], s["perm"], s["inv_perm"], s["order"],
                      s["w"], s["shared_table"], s["gate"], s["out"], s["workspace"])
    return s["out"]


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        h = s["h"].to(torch.float32) + s["delta"].to(torch.float32)
        x = h * torch.rsqrt((h * h).mean(dim=-1, keepdim=True) + EPS) * s["weight"].to(torch.float32)
        return {"h": h.to(s["h"].dtype), "x": x.to(torch.bfloat16), **_values(*_to_e4m3(x))}
    if kind == "quantize":
        return _values(*_to_e4m3(s["x"].to(torch.float32)))
    if kind == "linear":
        w = _from_weight(s["w"][0][0], s["w"][1][0], case["bits"])
        x = _from_e4m3(*s["x"]) if case["x_type"] == "mx" else _pad(s["x"].to(torch.float32))
        y = x @ w.t()
        if s["bias"] is not None:
            y = y + s["bias"]
        return y.to(_TYPES[case["y_type"]])
    return _ffn_plain(s, case)


def _swiglu(x, w1, w3, w2):
    """Batched experts on batched rows [.., n, H]; h passes through 8 bits between the products."""
    a = x @ w1.transpose(-1, -2)
    h = a * torch.sigmoid(a) * (x @ w3.transpose(-1, -2))
    return _from_e4m3(*_to_e4m3(h)) @ w2.transpose(-1, -2)


def _ffn_plain(s, case):
    N, H, k, E = case["N"], case["H"], case["k"], case["E"]
    x = _from_e4m3(*s["x"])
    ids = s["ids"].to(torch.int64)
    mats = [s[n] for n in ("w1", "w3", "w2")]
    if N * k <= E:      # few rows: the experts that each of them names
        at = ids.reshape(-1)
        w = [_from_weight(c[at], e[at], case["bits"]) for c, e in mats]
        rows = _swiglu(x.repeat_interleave(k, dim=0).unsqueeze(1), *w)[:, 0, :H].reshape(N, k, H)
    else:               # every expert on its rows, padded to the largest group
        w = [_from_weight(c, e, case["bits"]) for c, e in mats]
        slot = s["offsets"][:E, None].to(torch.int64) + torch.arange(s["capacity"], device="cuda")
        token = s["perm"][slot.clamp(max=N * k - 1)].to(torch.int64) // k
        out = _swiglu(x[token], *w)
        at = s["inv_perm"].to(torch.int64).reshape(N, k) - s["offsets"].to(torch.int64)[ids]
        rows = out[ids, at][..., :H]
    y = (rows * s["w"].unsqueeze(-1)).sum(dim=1)
    if case["n_shared"]:
        v = [_from_weight(*s[n], case["shared_bits"]) for n in ("v1", "v3", "v2")]
        z = _swiglu(x.unsqueeze(0), *v)[..., :H].sum(dim=0)
        if s["gate"] is not None:
            z = z * torch.sigmoid(x[:, :H] @ s["gate"].to(torch.float32)).unsqueeze(-1)
        y = y + z
    return y.to(torch.bfloat16)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def _round_e4m3(x):
    """Rows in 64 bits -> (element values, scale values), from the definition: the smallest power of two 2^e with
    max |x| / 2^e <= 448, elements to the nearest of 8 steps per octave, 2^-9 apart below 2^-6, ties to even."""
    x = _pad(x).reshape(*x.shape[:-1], -1, BLOCK)
    most = x.abs().amax(dim=-1, keepdim=True)
    safe = torch.where(most > 0, most, torch.ones_like(most))
    e = torch.ceil(torch.log2(safe / 448))
    e = torch.where(safe > 448 * torch.exp2(e), e + 1, e)
    e = torch.where(safe <= 448 * torch.exp2(e - 1), e - 1, e)
    e = torch.where(most > 0, e.clamp(-127, 127), torch.full_like(e, -127))
    v = x / torch.exp2(e)
    octave = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    octave = torch.where(torch.exp2(octave) > v.abs().clamp(min=2.0 ** -6), octave - 1, octave)
    step = torch.exp2(octave - 3)
    return torch.round(v / step) * step, torch.exp2(e).squeeze(-1)


def _numbers(codes, scales, bits):
    """Stored rows as 64-bit numbers, by the fields of their codes."""
    if bits == 4:
        codes = torch.stack([codes & 15, codes >> 4], dim=-1).reshape(*codes.shape[:-1], -1)
        sign, e, m, man, bias = codes >> 3, (codes >> 1) & 3, codes & 1, 1, 1
    else:
        sign, e, m, man, bias = codes >> 7, (codes >> 3) & 15, codes & 7, 3, 7
    e, m = e.to(torch.float64), m.to(torch.float64) / 2 ** man
    v = torch.where(e > 0, (1 + m) * torch.exp2(e - bias), m * 2.0 ** (1 - bias)) * (1 - 2 * sign.to(torch.float64))
    return (v.reshape(*v.shape[:-1], -1, BLOCK) * torch.exp2(scales.to(torch.float64) - 127).unsqueeze(-1)).reshape(v.shape)


def _expert(x, w1, w3, w2):
    a, b = x @ w1.t(), x @ w3.t()
    h, scale = _round_e4m3(a / (1 + torch.exp(-a)) * b)
    return (h * scale.unsqueeze(-1)).reshape(x.shape[0], -1) @ w2.t()


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("norm", "quantize"):
        if kind == "norm":
            h = s["h"].double() + s["delta"].double()
            x = h / torch.sqrt((h ** 2).sum(dim=-1, keepdim=True) / case["H"] + EPS) * s["weight"].double()
            out = {"h": h, "x": x}
        else:
            out, x = {}, s["x"].double()
        codes, scales = _round_e4m3(x)
        return {**out, "codes": codes.reshape(x.shape[0], -1), "scales": scales}
    if kind == "linear":
        w = _numbers(s["w"][0][0], s["w"][1][0], case["bits"])[:, :case["K"]]
        x = _numbers(*s["x"], 8)[:, :case["K"]] if case["x_type"] == "mx" else s["x"].double()
        y = x @ w.t()
        return y if s["bias"] is None else y + s["bias"].double()
    N, H, k = case["N"], case["H"], case["k"]
    x = _numbers(*s["x"], 8)
    y = torch.zeros(N, H, dtype=torch.float64, device="cuda")
    for e in torch.nonzero(s["counts"]).reshape(-1).tolist():
        token, j = torch.nonzero(s["ids"] == e, as_tuple=True)
        out = _expert(x[token], *(_numbers(s[n][0][e], s[n][1][e], case["bits"]) for n in ("w1", "w3", "w2")))
        y.index_add_(0, token, out[:, :H] * s["w"][token, j].double().unsqueeze(-1))
    for v in range(case["n_shared"]):
        out = _expert(x, *(_numbers(s[n][0][v], s[n][1][v], case["shared_bits"]) for n in ("v1", "v3", "v2")))[:, :H]
        if s["gate"] is not None:
            out = out / (1 + torch.exp(-(x[:, :H] @ s["gate"].double()))).unsqueeze(-1)
        y += out
    return y


# ---- work ------------------------------------------------------------------------------------------------------

def _mx_bytes(rows, K, bits=8):
    return rows * K * (bits / 8 + 1 / BLOCK)


def _active(case):
    """Expected number of experts that N tokens select."""
    E, N = case["E"], case["N"]
    rng = np.random.default_rng(7)
    bias = -case["zipf"] * np.log(np.arange(1, E + 1))
    trials = 1 if N >= 256 else 8
    return sum(len(np.unique(np.argsort(-(rng.normal(size=(N, E)) + bias), axis=1)[:, :case["k"]])) for _ in range(trials)) / trials


def work(case):
    size = {"bf16": 2, "fp32": 4}
    kind, N = case["kind"], case["N"]
    if kind == "norm":
        H = case["H"]
        row = H * (2 * size[case["h_type"]] + size[case["delta_type"]] + 2) + _mx_bytes(1, H)
        return {"bytes": N * row + H * size[case["weight"]], "flops": 8.0 * N * H}
    if kind == "quantize":
        return {"bytes": N * case["K"] * size[case["type"]] + _mx_bytes(N, case["K"]), "flops": 3.0 * N * case["K"]}
    if kind == "linear":
        K, R = case["K"], case["R"]
        x = _mx_bytes(N, K) if case["x_type"] == "mx" else 2 * N * K
        return {"bytes": x + _mx_bytes(R, K, case["bits"]) + N * R * size[case["y_type"]] + (4 * R if case["bias"] else 0),
                "flops": 2.0 * N * K * R}
    H, k, I, ns, Is = (case[n] for n in ("H", "k", "I", "n_shared", "I_shared"))
    weights = 3 * _active(case) * _mx_bytes(I, H, case["bits"]) + 3 * ns * _mx_bytes(Is, H, case["shared_bits"])
    rows = _mx_bytes(N, H) + N * H * 2 + N * k * 12
    return {"bytes": weights + rows, "flops": 6.0 * H * N * (k * I + ns * Is)}
