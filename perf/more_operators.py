"""Experts in microscaled 4-bit floating point and the training side of the router in front of them, as cases with sizes: the
conversion of rows to blocks of 32 values with a common power of two and back, a matrix product and a layer's SwiGLU experts in
that format, the balance loss with its per-expert counts, and the gradient of the router's logits.

listed() names the cases; draw() gives further ones from the ranges they stand for; prepare() makes what a program holds
before the call (inputs from the seed, weights converted and laid out, output buffers); run() is one pass, in elementary
torch operations or, where `own` is set, by the package's entry points; exact() is the same result in 64 bits; work()
counts what the pass cannot do without.
"""
import math

import torch

own = False

WEIGHT_STD = 0.02
BLOCK = 32
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}


def _quantize(name, rows, K, dtype="bf16", tiled=False):
    return {"name": name, "kind": "quantize", "rows": rows, "K": K, "dtype": dtype, "tiled": tiled}


def _matmul(name, T, N, K, bias=False, dtype="bf16", out="bf16"):
    return {"name": name, "kind": "matmul", "T": T, "N": N, "K": K, "bias": bias, "dtype": dtype, "out": out}


def _ffn(name, T, H, F, E, k, zipf=0.0, dtype="bf16"):
    return {"name": name, "kind": "ffn", "T": T, "H": H, "F": F, "E": E, "k": k, "zipf": zipf, "dtype": dtype}


def _router(kind, name, T, E, k, score, dtype, keep=1.0, renorm=True):
    return {"name": name, "kind": kind, "T": T, "E": E, "k": k, "score": score, "dtype": dtype, "keep": keep, "renorm": renorm}


def listed():
    return [
        # activations of a decode batch, there and back
        _quantize("quantize_24", 24, 4096),
        # one expert-wide matrix's worth of rows, an odd number, laid out as weights are
        _quantize("quantize_8191", 8191, 14336, tiled=True),
        # a narrow matrix of the fine-grained layer's sizes for an odd decode batch, with a bias, fp32 output
        _matmul("matmul_61", 61, 1536, 2048, bias=True, out="f32"),
        # an expert-wide matrix over an odd prompt
        _matmul("matmul_2047", 2047, 14336, 4096),
        # one decode token on the Mixtral-8x7B-shaped layer
        _ffn("ffn_mixtral_1", 1, 4096, 14336, 8, 2),
        # the fine-grained layer (128 experts of 768, top-8) serving an odd batch
        _ffn("ffn_fine_61", 61, 2048, 768, 128, 8),
        # prefill of 512 tokens on the Mixtral-shaped layer
        _ffn("ffn_mixtral_512", 512, 4096, 14336, 8, 2),
        # the fine-grained layer's prefill with skewed expert load
        _ffn("ffn_fine_2047", 2047, 2048, 768, 128, 8, zipf=1.2),
        # a short micro-batch behind the fine-grained layer's router, logits as a bf16 product leaves them: nothing but latency
        _router("balance", "balance_24", 24, 128, 8, "softmax", "bf16"),
        # a long padded batch behind a router of 256 experts
        _router("balance", "balance_8191", 8191, 256, 8, "sigmoid", "f32", keep=0.8),
        # the same two, backwards
        _router("backward", "backward_24", 24, 128, 8, "softmax", "bf16"),
        _router("backward", "backward_8191", 8191, 256, 8, "sigmoid", "f32", keep=0.8),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        u = rng.random()
        if u < 0.2:
            case = _quantize("", _log_int(rng, 1, 8192), _log_int(rng, 32, 14336), rng.choice(["bf16", "bf16", "f16", "f32"]), rng.random() < 0.5)
        elif u < 0.45:
            case = _matmul("", _log_int(rng, 1, 4096), _log_int(rng, 64, 14336), _log_int(rng, 128, 14336), rng.random() < 0.3,
                           rng.choice(["bf16", "bf16", "f16"]), rng.choice(["bf16", "f32", "f16"]))
        elif u < 0.75:
            E = rng.choice([8, 8, 16, 60, 64, 128])
            case = _ffn("", _log_int(rng, 1, 2500), _log_int(rng, 256, 4096, 8), _log_int(rng, 256, 14336, 8), E,
                        min(E, rng.choice([1, 2, 2, 4, 6, 8])), rng.choice([0.0, 0.0, 1.2]) if E >= 60 else 0.0,
                        rng.choice(["bf16", "bf16", "f16"]))
            # the plain form's padded batch has a row for every token in every expert
            if case["H"] * case["F"] * E > 4096 * 14336 * 8 or E * case["T"] * max(case["H"], case["F"]) > 1 << 30:
                continue
        else:
            E = _log_int(rng, 8, 512)
            case = _router(rng.choice(["balance", "backward"]), "", _log_int(rng, 1, 16384), E, min(E, rng.choice([1, 2, 4, 6, 8, 10])),
                           rng.choice(["softmax", "sigmoid"]), rng.choice(["f32", "f32", "bf16", "f16"]), rng.choice([1.0, 1.0, 0.8, 0.1]),
                           rng.random() < 0.7)
        case.pop("name", None)
        if _cost(case) <= most:
            return case


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 4e15)


# ---------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(g, T, H, dtype):
    """Normals, about one row in twenty eight times as large, and one column in fifty."""
    x = torch.randn((T, H), generator=g, device="cuda")
    big = torch.rand((T, 1), generator=g, device="cuda") < 0.05
    wide = torch.rand((1, H), generator=g, device="cuda") < 0.02
    return (x * torch.where(big, 8.0, 1.0) * torch.where(wide, 8.0, 1.0)).to(DTYPES[dtype])


def _up(v, m):
    return (v + m - 1) // m * m


def _encode(w):
    """fp32 [N, K] -> (nibbles [N, Kp], exponent bytes [N, Kp / 32]) with Kp = K up to a multiple of 256; and the values they
    stand for, [N, K] bf16 (exact)."""
    N, K = w.shape
    Kp = _up(K, 256)
    b = torch.nn.functional.pad(w, (0, Kp - K)).view(N, Kp // BLOCK, BLOCK)
    a = b.abs().amax(-1, keepdim=True)
    e = torch.where(a > 0, torch.frexp(a).exponent - 3, -127).clamp_(-127, 127)      # floor(log2 a) - 2
    m = torch.ldexp(b.abs(), -e)
    v = torch.where(m < 2, torch.round(m * 2) / 2, torch.where(m < 4, torch.round(m), torch.round(m / 2) * 2)).clamp_(max=6.0)
    code = torch.where(v <= 2, v * 2, torch.where(v <= 4, v + 2, 7.0)).to(torch.uint8)
    nibble = torch.where(torch.signbit(b), code + 8, code).view(N, Kp)
    value = torch.ldexp(torch.copysign(v, b), e).view(N, Kp)[:, :K].to(torch.bfloat16)
    return nibble, (e[..., 0] + 127).to(torch.uint8), value


def _tiles(nibble, exponent):
    """Rows up to a multiple of 32, in tiles of 32 rows x 256 columns: lane 32 * kb + r of a tile holds row r, columns 128 * kb + 0
    .. 127, its chunk c (32 columns, 16 bytes, even columns in the low halves) at byte 1024 * c + 16 * lane; the four exponents of
    a lane lie together, lane after lane."""
    N, Kp = nibble.shape
    Np = _up(N, 32)
    q = torch.nn.functional.pad(nibble, (0, 0, 0, Np - N)).view(Np // 32, 32, Kp // 256, 2, 4, 16, 2)
    q = (q[..., 0] | (q[..., 1] << 4)).permute(0, 2, 4, 3, 1, 5).reshape(Np, Kp // 2)
    s = torch.nn.functional.pad(exponent, (0, 0, 0, Np - N)).view(Np // 32, 32, Kp // 256, 2, 4)
    return q, s.permute(0, 2, 3, 1, 4).reshape(Np, Kp // BLOCK)


def _weight(g, N, K):
    nibble, exponent, value = _encode(torch.randn((N, K), generator=g, device="cuda") * WEIGHT_STD)
    return _tiles(nibble, exponent), value


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["kind"] == "quantize":
        s["x"] = _activations(g, case["rows"], case["K"], case["dtype"])
        rows = _up(case["rows"], 32) if case["tiled"] else case["rows"]
        s["codes"] = torch.empty((rows, _up(case["K"], 256) // 2), dtype=torch.uint8, device="cuda")
        s["scale"] = torch.empty((rows, _up(case["K"], 256) // BLOCK), dtype=torch.uint8, device="cuda")
        s["y"] = torch.empty_like(s["x"])
    elif case["kind"] == "matmul":
        s["x"] = _activations(g, case["T"], case["K"], case["dtype"])
        s["wt"], s["wv"] = _weight(g, case["N"], case["K"])
        s["b"] = torch.randn((case["N"],), generator=g, device="cuda") if case["bias"] else None
        s["y"] = torch.empty((case["T"], case["N"]), dtype=DTYPES[case["out"]], device="cuda")
    elif case["kind"] == "ffn":
        T, H, F, E, k = (case[n] for n in "THFEk")
        s["x"] = _activations(g, T, H, case["dtype"])
        prior = -case["zipf"] * torch.log(torch.randperm(E, generator=g, device="cuda") + 1.0)
        top = (torch.randn((T, E), generator=g, device="cuda") + prior).softmax(-1).topk(k, dim=-1)
        s["idx"] = top.indices.to(torch.int32)
        s["gate"] = top.values / top.values.sum(-1, keepdim=True)
        s["v"], s["q"], s["s"] = [], [], []
        for n, m in ((F, H), (F, H), (H, F)):
            s["v"].append(torch.empty((E, n, m), dtype=torch.bfloat16, device="cuda"))
            s["q"].append(torch.empty((E, _up(n, 32), _up(m, 256) // 2), dtype=torch.uint8, device="cuda"))
            s["s"].append(torch.empty((E, _up(n, 32), _up(m, 256) // BLOCK), dtype=torch.uint8, device="cuda"))
            for e in range(E):
                (s["q"][-1][e], s["s"][-1][e]), s["v"][-1][e] = _weight(g, n, m)
        entries = [[t[e].data_ptr() for t in s["q"]] + [t[e].data_ptr() for t in s["s"]] for e in range(E)]
        s["table"] = torch.tensor(entries, dtype=torch.int64, device="cuda")
        s["y"] = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    else:
        T, E, k = (case[n] for n in "TEk")
        # a token's logits lean towards a few experts that are popular with all; a bias has moved some of the choices
        logits = 1.5 * torch.randn((T, E), generator=g, device="cuda") + torch.randn((E,), generator=g, device="cuda")
        s["logits"] = logits.to(DTYPES[case["dtype"]])
        s["idx"] = (logits + 0.3 * torch.randn((E,), generator=g, device="cuda")).topk(k, dim=-1).indices.to(torch.int32)
        # tokens of padding have no part in the loss
        s["kept"] = (torch.rand((T,), generator=g, device="cuda") < case["keep"]).to(torch.uint8) if case["keep"] < 1 else None
        s["coef"] = 0.01
        s["counts"] = torch.empty((E + 1,), dtype=torch.int32, device="cuda")
        if case["kind"] == "balance":
            s["mean"] = torch.empty((E,), dtype=torch.float32, device="cuda")
            s["loss"] = torch.empty((1,), dtype=torch.float32, device="cuda")
        else:
            s["dw"] = torch.randn((T, k), generator=g, device="cuda") * 0.1
            s["dloss"] = torch.rand((1,), generator=g, device="cuda") + 0.5
            s["grad"] = torch.empty_like(s["logits"])
            _counts(s, s["counts"])
    return s


def _counts(s, out):
    """How often each expert is chosen by the tokens that take part; behind them, how many tokens those are."""
    e = s["idx"].long()
    part = torch.ones_like(e) if s["kept"] is None else (s["kept"] != 0).long()[:, None].expand_as(e)
    out[:-1] = torch.zeros((s["E"],), dtype=torch.long, device=e.device).index_add_(0, e.reshape(-1), part.reshape(-1)).to(torch.int32)
    out[-1] = part[:, 0].sum().to(torch.int32)


# ---------------------------------------------------------------------------------------------------------- plain form

def _fake(x):
    """The values that the codes of rows x stand for, in x's type if that is 16 bits, else fp32: a block's power of two is that of
    its largest value's last two bits before the point; numbers of 4 bits to the nearest, ties to even, 6 at most."""
    T, K = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -K % BLOCK)).view(T, -1, BLOCK)
    a = b.abs().amax(-1, keepdim=True)
    e = torch.where(a > 0, torch.frexp(a).exponent - 3, -127)
    m = torch.ldexp(b, -e)
    n = m.abs()
    step = torch.where(n < 2, 0.5, torch.where(n < 4, 1.0, 2.0))
    v = (torch.round(m / step) * step).clamp(-6.0, 6.0)
    return torch.ldexp(v, e).view(T, -1)[:, :K]


def _matmul_plain(s):
    y = _fake(s["x"]) @ s["wv"].float().T
    if s["b"] is not None:
        y = y + s["b"]
    return y.to(DTYPES[s["out"]])


def _experts(x, w):
    """SwiGLU experts over rows x [n, m, H], already in the format's values, one expert of w for each of the n."""
    def times(r, i):
        return torch.bmm(r, w[i].float().transpose(1, 2).contiguous())

    a, u = times(x, 0), times(x, 1)
    h = a / (1.0 + torch.exp(-a)) * u
    return times(_fake(h.view(-1, h.shape[-1])).view(h.shape), 2)


def _ffn_plain(s):
    T, H, E, k = s["T"], s["H"], s["E"], s["k"]
    x = _fake(s["x"])
    e = s["idx"].reshape(-1).long()
    rows = torch.arange(T * k, device=e.device) // k
    if T * k <= E // 2:  # few pairs: each with its expert's weights
        o = _experts(x[rows][:, None], [v[e] for v in s["v"]])[:, 0]
    else:  # every expert over a batch with room for all tokens; a pair's row is its turn in its expert
        turn = torch.cumsum(torch.nn.functional.one_hot(e, E), 0).gather(1, e[:, None])[:, 0] - 1
        batch = torch.zeros((E, T, H), device=e.device)
        batch[e, turn] = x[rows]
        o = _experts(batch, s["v"])[e, turn]
    return (o.view(T, k, H) * s["gate"][..., None]).sum(1).to(torch.bfloat16)


def _shares(s, l):
    """A token's scores divided by their sum."""
    if s["score"] == "sigmoid":
        v = 1.0 / (1.0 + torch.exp(-l))
    else:
        v = torch.exp(l - l.amax(-1, keepdim=True))
    return v / v.sum(-1, keepdim=True)


def _balance_plain(s):
    counts = torch.empty_like(s["counts"])
    _counts(s, counts)
    p = _shares(s, s["logits"].double())
    if s["kept"] is not None:
        p = torch.where((s["kept"] != 0)[:, None], p, 0.0)
    tokens = counts[-1].double().clamp(min=1.0)
    mean = p.sum(0) / tokens
    loss = s["coef"] * s["E"] * (counts[:-1].double() / (tokens * s["k"]) * mean).sum()
    return counts, mean.float(), loss.float().view(1)


def _backward_plain(s):
    l = s["logits"].float()
    sigmoid = s["score"] == "sigmoid"
    rest = 1.0 / (1.0 + torch.exp(l)) if sigmoid else None                    # 1 - score
    # the gate weights
    e = s["idx"].long()
    if s["renorm"]:
        x = l.gather(1, e)
        x = torch.log(1.0 / (1.0 + torch.exp(-x))) if sigmoid else x
        q = torch.exp(x - x.amax(-1, keepdim=True))
        q = q / q.sum(-1, keepdim=True)
        part = q * (s["dw"] - (q * s["dw"]).sum(-1, keepdim=True))
        grad = torch.zeros_like(l).scatter_add(1, e, part)
        if sigmoid:
            grad = grad * rest
    elif sigmoid:
        grad = torch.zeros_like(l).scatter_add(1, e, s["dw"]) * rest * (1.0 / (1.0 + torch.exp(-l)))
    else:
        v = _shares(s, l)
        d = torch.zeros_like(l).scatter_add(1, e, s["dw"])
        grad = v * (d - (v * d).sum(-1, keepdim=True))
    # the loss
    p = _shares(s, l)
    tokens = s["counts"][-1].float().clamp(min=1.0)
    g = s["dloss"] * s["coef"] * s["E"] * s["counts"][:-1].float() / (tokens * tokens * s["k"])
    part = p * (g - (p * g).sum(-1, keepdim=True))
    if sigmoid:
        part = part * rest
    if s["kept"] is not None:
        part = torch.where((s["kept"] != 0)[:, None], part, 0.0)
    return (grad + part).to(s["logits"].dtype)


# ---------------------------------------------------------------------------------------------------------- one pass

_context = []


def _own(s):
    from paper_2603_19172_amd import binding as B
    if not _context:
        _context.append(B.Context(torch.cuda.current_device()))
    ctx = _context[0]
    if s["kind"] == "quantize":
        layout = B.LAYOUT_TILE if s["tiled"] else B.LAYOUT_ROWMAJOR
        m = ctx.quantize_mx4(s["x"], layout=layout, out=(s["codes"], s["scale"]))
        return ctx.dequantize_mx4(m, out=s["y"])
    if s["kind"] in ("balance", "backward"):
        score = B.SCORE_SIGMOID if s["score"] == "sigmoid" else B.SCORE_SOFTMAX
        if s["kind"] == "backward":
            return ctx.route_scored_backward(s["logits"], s["idx"], dw=s["dw"], score=score, renorm=s["renorm"], counts=s["counts"],
                                             coef=s["coef"], dloss=s["dloss"], keep=s["kept"], out=s["grad"])
        if "ws_buf" not in s:
            s["ws_buf"] = torch.empty((B.route_balance_workspace_bytes(s["T"], s["E"]),), dtype=torch.uint8, device="cuda")
        return ctx.route_balance(s["logits"], s["idx"], s["coef"], score=score, keep=s["kept"], counts=s["counts"], mean=s["mean"],
                                 loss=s["loss"], workspace=s["ws_buf"])
    if "ws_buf" not in s:  # a program's workspace, kept between its calls
        n = (B.matmul_mx4_workspace_bytes(s["T"], s["N"], s["K"]) if s["kind"] == "matmul"
             else B.moe_ffn_mx4_workspace_bytes(s["T"], s["H"], s["F"], s["E"], s["k"]))
        s["ws_buf"] = torch.empty((n,), dtype=torch.uint8, device="cuda")
    if s["kind"] == "matmul":
        w = B.Mx4Matrix(*s["wt"], s["N"], s["K"], B.LAYOUT_TILE)
        return ctx.matmul_mx4(s["x"], w, bias=s["b"], y=s["y"], workspace=s["ws_buf"])
    return ctx.moe_ffn_mx4(s["x"], s["idx"], s["gate"], s["table"], s["F"], y=s["y"], workspace=s["ws_buf"])


def run(state):
    s = state
    if own:
        return _own(s)
    if s["kind"] == "quantize":
        return _fake(s["x"]).to(s["x"].dtype)
    if s["kind"] == "matmul":
        return _matmul_plain(s)
    if s["kind"] == "ffn":
        return _ffn_plain(s)
    return _balance_plain(s) if s["kind"] == "balance" else _backward_plain(s)


# ---------------------------------------------------------------------------------------------------------- 64 bits

_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _values64(x):
    """What the codes of x's rows stand for: each number by its distance to the eight magnitudes."""
    x = x.double()
    n, K = x.shape
    out = torch.zeros_like(x)
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    middle = (grid[1:] + grid[:-1]) / 2
    even = torch.arange(8, device=x.device) % 2 == 0
    for c in range(0, K, 4096):
        part = x[:, c:c + 4096]
        w = _up(part.shape[1], BLOCK)
        b = torch.zeros((n, w), dtype=torch.float64, device=x.device)
        b[:, :part.shape[1]] = part
        b = b.view(n, w // BLOCK, BLOCK)
        peak = b.abs().max(-1, keepdim=True).values
        unit = torch.where(peak > 0, torch.exp2(torch.floor(torch.log2(torch.where(peak > 0, peak, 1.0))) - 2.0), 1.0)
        m = b.abs() / unit
        at = torch.searchsorted(middle, m)                       # the first middle that is not below m
        tie = (at < 7) & (middle[at.clamp(max=6)] == m)
        at = torch.where(tie & ~even[at], at + 1, at)
        out[:, c:c + 4096] = (grid[at] * unit * torch.sign(b)).view(n, w)[:, :part.shape[1]]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "quantize":
        return _values64(s["x"])
    if s["kind"] == "matmul":
        y = torch.matmul(_values64(s["x"]), s["wv"].double().T)
        return y if s["b"] is None else y + s["b"].double()
    if s["kind"] == "ffn":
        x = _values64(s["x"])
        y = torch.zeros((s["T"], s["H"]), dtype=torch.float64, device="cuda")
        for e in range(s["E"]):
            token, slot = (s["idx"] == e).nonzero(as_tuple=True)
            if not token.numel():
                continue
            w1, w3, w2 = (v[e].double() for v in s["v"])
            a = x[token] @ w1.T
            h = _values64(a * torch.sigmoid(a) * (x[token] @ w3.T))
            y.index_add_(0, token, h @ w2.T * s["gate"][token, slot].double()[:, None])
        return y
    l = s["logits"].double().requires_grad_(True)
    score = torch.sigmoid(l) if s["score"] == "sigmoid" else torch.softmax(l, -1)
    share = score / score.sum(-1, keepdim=True)
    part = torch.ones((s["T"],), dtype=torch.float64, device="cuda") if s["kept"] is None else s["kept"].double()
    tokens = max(1.0, float(part.sum()))
    mean = (share * part[:, None]).sum(0) / tokens
    often = (torch.nn.functional.one_hot(s["idx"].long(), s["E"]).sum(1) * part[:, None]).sum(0)
    loss = s["coef"] * s["E"] * (often / (tokens * s["k"]) * mean).sum()
    if s["kind"] == "balance":
        return None, mean.detach(), loss.detach().view(1)
    w = score.gather(1, s["idx"].long())
    if s["renorm"]:
        w = w / w.sum(-1, keepdim=True)
    return torch.autograd.grad((w * s["dw"].double()).sum() + s["dloss"].double()[0] * loss, l)[0]


# ---------------------------------------------------------------------------------------------------------- work

def work(case):
    c = case
    if c["kind"] == "quantize":
        n = c["rows"] * c["K"]
        return {"bytes": n * (2 * SIZES[c["dtype"]] + 2 * 17 / 32), "flops": 6 * n}
    if c["kind"] == "matmul":
        T, N, K = c["T"], c["N"], c["K"]
        return {"bytes": T * K * SIZES[c["dtype"]] + N * K * 17 / 32 + 4 * N * bool(c["bias"]) + T * N * SIZES[c["out"]], "flops": 2 * T * N * K}
    if c["kind"] == "ffn":
        T, H, F, E, k = (c[n] for n in "THFEk")
        met = E * (1.0 - (1.0 - k / E) ** T)  # experts that some token meets, where all are as likely
        return {"bytes": met * 3 * H * F * 17 / 32 + T * H * (SIZES[c["dtype"]] + 2) + 8 * T * k, "flops": 6 * T * k * H * F}
    T, E, k = (c[n] for n in "TEk")
    size = T * E * SIZES[c["dtype"]]
    if c["kind"] == "balance":
        return {"bytes": size + 4 * T * k + T * (c["keep"] < 1) + 12 * E, "flops": 8 * T * E}
    return {"bytes": 2 * size + 8 * T * k + T * (c["keep"] < 1) + 4 * E, "flops": 14 * T * E}
