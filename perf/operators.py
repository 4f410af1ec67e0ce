"""The routing of tokens by scores, groups and a balancing bias, and the products in 8-bit integers behind it, as cases with
sizes: the router's selection, the dynamic quantisation of rows, a matrix product with scales for each token and channel,
and a layer's SwiGLU experts in that arithmetic.

listed() names the cases; draw() gives further ones from the ranges they stand for; prepare() makes what a program holds
before the call (inputs from the seed, weights quantised and laid out, output buffers); run() is one pass, in elementary
torch operations or, where `own` is set, by the package's entry points; exact() is the same result in 64 bits; work()
counts what the pass cannot do without.
"""
import math

import torch

own = False

WEIGHT_STD = 0.02
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}


def _route(name, T, E, k, score, bias, groups, top_groups, best, dtype):
    return {"name": name, "kind": "route", "T": T, "E": E, "k": k, "score": score, "bias": bias, "groups": groups,
            "top_groups": top_groups, "best": best, "dtype": dtype}


def _ffn(name, T, H, F, E, k, zipf=0.0, dtype="bf16"):
    return {"name": name, "kind": "ffn", "T": T, "H": H, "F": F, "E": E, "k": k, "zipf": zipf, "dtype": dtype}


def listed():
    return [
        # one decode token: the router's selection among 256 experts in 8 groups, nothing but latency
        _route("route_sigmoid_1", 1, 256, 8, "sigmoid", True, 8, 4, 2, "f32"),
        # the same router over a long prompt
        _route("route_sigmoid_8192", 8192, 256, 8, "sigmoid", True, 8, 4, 2, "f32"),
        # the fine-grained layer's router with a balancing bias, an odd prompt, logits as a bf16 product leaves them
        _route("route_softmax_2047", 2047, 128, 8, "softmax", True, 1, 1, 1, "bf16"),
        # activations of a decode batch
        {"name": "quantize_24", "kind": "quantize", "rows": 24, "K": 4096, "dtype": "bf16"},
        # the intermediate of a long prefill: rows of the Mixtral layer's expert width, an odd number of them
        {"name": "quantize_8191", "kind": "quantize", "rows": 8191, "K": 14336, "dtype": "bf16"},
        # a projection of hidden size for one decode token
        {"name": "matmul_1", "kind": "matmul", "T": 1, "N": 4096, "K": 4096, "bias": False, "dtype": "bf16", "out": "bf16"},
        # a narrow matrix of the fine-grained layer's sizes for an odd decode batch, with a bias, fp32 output
        {"name": "matmul_61", "kind": "matmul", "T": 61, "N": 1536, "K": 2048, "bias": True, "dtype": "bf16", "out": "f32"},
        # an expert-wide matrix over a prompt
        {"name": "matmul_2048", "kind": "matmul", "T": 2048, "N": 14336, "K": 4096, "bias": False, "dtype": "bf16", "out": "bf16"},
        # one decode token on the Mixtral-8x7B-shaped layer
        _ffn("ffn_mixtral_1", 1, 4096, 14336, 8, 2),
        # the fine-grained layer (128 experts of 768, top-8) serving an odd batch
        _ffn("ffn_fine_61", 61, 2048, 768, 128, 8),
        # prefill of 512 tokens on the Mixtral-shaped layer
        _ffn("ffn_mixtral_512", 512, 4096, 14336, 8, 2),
        # the fine-grained layer's prefill with skewed expert load
        _ffn("ffn_fine_2048", 2048, 2048, 768, 128, 8, zipf=1.2),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        u = rng.random()
        if u < 0.25:
            groups = rng.choice([1, 1, 4, 8])
            per = _log_int(rng, 4, 64)
            E = groups * per if groups > 1 else _log_int(rng, 8, 512)
            top = rng.randint(1, groups)
            k = min(rng.choice([1, 2, 4, 6, 8, 10]), top * (E // groups))
            case = _route("", _log_int(rng, 1, 8192), E, k, rng.choice(["sigmoid", "softmax"]), rng.random() < 0.7, groups, top,
                          rng.choice([1, 2]) if groups > 1 else 1, rng.choice(["f32", "f32", "bf16", "f16"]))
        elif u < 0.4:
            case = {"kind": "quantize", "rows": _log_int(rng, 1, 8192), "K": _log_int(rng, 64, 14336), "dtype": rng.choice(["bf16", "bf16", "f16"])}
        elif u < 0.7:
            case = {"kind": "matmul", "T": _log_int(rng, 1, 4096), "N": _log_int(rng, 64, 14336), "K": _log_int(rng, 128, 14336),
                    "bias": rng.random() < 0.3, "dtype": rng.choice(["bf16", "bf16", "f16"]), "out": rng.choice(["bf16", "f32", "f16"])}
        else:
            E = rng.choice([8, 8, 16, 60, 64, 128])
            case = _ffn("", _log_int(rng, 1, 2500), _log_int(rng, 256, 4096, 8), _log_int(rng, 256, 14336, 8), E,
                        min(E, rng.choice([1, 2, 2, 4, 6, 8])), rng.choice([0.0, 0.0, 1.2]) if E >= 60 else 0.0,
                        rng.choice(["bf16", "bf16", "f16"]))
            # the plain form's padded batch has a row for every token in every expert
            if case["H"] * case["F"] * E > 4096 * 14336 * 8 or E * case["T"] * max(case["H"], case["F"]) > 1 << 30:
                continue
        case.pop("name", None)
        if _cost(case) <= most:
            return case


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 2e15)


# ---------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(g, T, H, dtype):
    """Normals, about one row in twenty eight times as large."""
    x = torch.randn((T, H), generator=g, device="cuda")
    big = torch.rand((T, 1), generator=g, device="cuda") < 0.05
    return (x * torch.where(big, 8.0, 1.0)).to(DTYPES[dtype])


def _weight(g, N, K):
    """int8 codes [N, K] and their scales [N] of normal weights."""
    w = torch.randn((N, K), generator=g, device="cuda") * WEIGHT_STD
    a = w.abs().amax(dim=1)
    return (w * (127.0 / a)[:, None]).round_().clamp_(-127, 127).to(torch.int8), a / 127.0


def _up(v, m):
    return (v + m - 1) // m * m


def _tiles(codes):
    """[N, K] -> [N up to a multiple of 32, K up to one of 128], zeros behind the ends, in tiles of 32 rows x 128 columns:
    16-byte chunk c of a tile's lane 32 * kb + r holds row r, columns 64 * kb + 16 * c and the 15 behind it."""
    N, K = codes.shape
    Np, Kp = _up(N, 32), _up(K, 128)
    if (Np, Kp) != (N, K):
        codes = torch.nn.functional.pad(codes, (0, Kp - K, 0, Np - N))
    return codes.reshape(Np // 32, 32, Kp // 128, 2, 4, 16).permute(0, 2, 4, 3, 1, 5).reshape(Np, Kp)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["kind"] == "route":
        T, E = case["T"], case["E"]
        # a token's logits lean towards a few experts that are popular with all
        logits = 1.5 * torch.randn((T, E), generator=g, device="cuda") + torch.randn((E,), generator=g, device="cuda")
        s["logits"] = logits.to(DTYPES[case["dtype"]])
        s["b"] = 0.1 * torch.randn((E,), generator=g, device="cuda") if case["bias"] else None
        s["idx"] = torch.empty((T, case["k"]), dtype=torch.int32, device="cuda")
        s["w"] = torch.empty((T, case["k"]), dtype=torch.float32, device="cuda")
    elif case["kind"] == "quantize":
        s["x"] = _activations(g, case["rows"], case["K"], case["dtype"])
        s["codes"] = torch.empty((case["rows"], _up(case["K"], 128)), dtype=torch.int8, device="cuda")
        s["scale"] = torch.empty((case["rows"],), dtype=torch.float32, device="cuda")
    elif case["kind"] == "matmul":
        s["x"] = _activations(g, case["T"], case["K"], case["dtype"])
        s["wq"], s["ws"] = _weight(g, case["N"], case["K"])
        s["wt"] = _tiles(s["wq"])
        s["b"] = torch.randn((case["N"],), generator=g, device="cuda") if case["bias"] else None
        s["y"] = torch.empty((case["T"], case["N"]), dtype=DTYPES[case["out"]], device="cuda")
    else:
        T, H, F, E, k = (case[n] for n in "THFEk")
        s["x"] = _activations(g, T, H, case["dtype"])
        prior = -case["zipf"] * torch.log(torch.randperm(E, generator=g, device="cuda") + 1.0)
        top = (torch.randn((T, E), generator=g, device="cuda") + prior).softmax(-1).topk(k, dim=-1)
        s["idx"] = top.indices.to(torch.int32)
        s["gate"] = top.values / top.values.sum(-1, keepdim=True)
        s["q"], s["s"], s["t"], entries = [], [], [], []
        for n, m in ((F, H), (F, H), (H, F)):
            s["q"].append(torch.empty((E, n, m), dtype=torch.int8, device="cuda"))
            s["t"].append(torch.empty((E, _up(n, 32), _up(m, 128)), dtype=torch.int8, device="cuda"))
            s["s"].append(torch.empty((E, n), dtype=torch.float32, device="cuda"))
            for e in range(E):
                s["q"][-1][e], s["s"][-1][e] = _weight(g, n, m)
                s["t"][-1][e] = _tiles(s["q"][-1][e])
        for e in range(E):
            entries.append([t[e].data_ptr() for t in s["t"]] + [t[e].data_ptr() for t in s["s"]])
        s["table"] = torch.tensor(entries, dtype=torch.int64, device="cuda")
        s["y"] = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------- plain form

def _order(v):
    """Indices of the last dimension by descending value, equal ones by index."""
    return torch.sort(v, dim=-1, descending=True, stable=True).indices


def _select(s):
    """The router's selection, with scores and what is compared in 64 bits."""
    l = s["logits"].double()
    T, E = l.shape
    G, k = s["groups"], s["k"]
    if s["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-l))
    else:
        z = torch.exp(l - l.amax(-1, keepdim=True))
        score = z / z.sum(-1, keepdim=True)
    c = score + s["b"].double() if s["b"] is not None else score
    if G > 1:
        per = c.view(T, G, E // G)
        value = torch.gather(per, 2, _order(per)[..., :s["best"]]).sum(-1)
        kept = torch.zeros((T, G), dtype=torch.bool, device=l.device)
        kept.scatter_(1, _order(value)[:, :s["top_groups"]], True)
        c = torch.where(kept.repeat_interleave(E // G, dim=1), c, -math.inf)
    idx = _order(c)[:, :k]
    w = torch.gather(score, 1, idx)
    return idx.to(torch.int32), (w / w.sum(-1, keepdim=True)).float()


def _quantize(x):
    """Codes and scales of rows; the quotient in 64 bits, so that what lies halfway between two codes is seen to."""
    a = x.float().abs().amax(-1, keepdim=True)
    some = torch.where(a > 0, a, 1.0)
    return torch.round(x.double() * 127.0 / some.double()).float(), a / 127.0


def _matmul(s):
    xq, xs = _quantize(s["x"])
    y = (xq @ s["wq"].float().T) * xs * s["ws"]
    if s["b"] is not None:
        y = y + s["b"]
    return y.to(DTYPES[s["out"]])


def _experts(xq, xs, q, sc):
    """SwiGLU experts over rows [n, m, H] of codes with scales [n, m, 1], one expert for each of the n."""
    def times(codes, scale, i):
        return torch.bmm(codes, q[i].transpose(1, 2).float()) * scale * sc[i][:, None, :]

    a, u = times(xq, xs, 0), times(xq, xs, 1)
    hq, hs = _quantize(a / (1.0 + torch.exp(-a)) * u)
    return times(hq, hs, 2)


def _ffn_plain(s):
    T, H, E, k = s["T"], s["H"], s["E"], s["k"]
    xq, xs = _quantize(s["x"])
    if T * k <= E // 2:  # few pairs: each with its expert's weights
        e = s["idx"].reshape(-1).long()
        rows = torch.arange(T * k, device=e.device) // k
        o = _experts(xq[rows][:, None], xs[rows][:, None], [q[e] for q in s["q"]], [c[e] for c in s["s"]])[:, 0]
    else:  # every expert over a batch with room for all tokens; a pair's row is its turn in its expert
        e = s["idx"].reshape(-1).long()
        rows = torch.arange(T * k, device=e.device) // k
        turn = torch.cumsum(torch.nn.functional.one_hot(e, E), 0).gather(1, e[:, None])[:, 0] - 1
        bx = torch.zeros((E, T, H), device=e.device)
        bs = torch.zeros((E, T, 1), device=e.device)
        bx[e, turn] = xq[rows]
        bs[e, turn] = xs[rows]
        o = _experts(bx, bs, s["q"], s["s"])[e, turn]
    return (o.view(T, k, H) * s["gate"][..., None]).sum(1).to(torch.bfloat16)


# ---------------------------------------------------------------------------------------------------------- one pass

_context = []


def _own(s):
    from paper_2603_19172_amd import binding as B
    if not _context:
        _context.append(B.Context(torch.cuda.current_device()))
    ctx = _context[0]
    if s["kind"] == "route":
        score = B.SCORE_SIGMOID if s["score"] == "sigmoid" else B.SCORE_SOFTMAX
        ctx.route_scored(s["logits"], s["k"], bias=s["b"], score=score, groups=s["groups"], top_groups=s["top_groups"],
                         group_best=s["best"], idx=s["idx"], w=s["w"])
        return s["idx"], s["w"]
    if s["kind"] == "quantize":
        ctx.quantize_rows(s["x"], out=(s["codes"], s["scale"]))
        return s["codes"], s["scale"]
    if "ws_buf" not in s:  # a program's workspace, kept between its calls
        n = (B.matmul_int8_workspace_bytes(s["T"], s["N"], s["K"]) if s["kind"] == "matmul"
             else B.moe_ffn_int8_workspace_bytes(s["T"], s["H"], s["F"], s["E"], s["k"]))
        s["ws_buf"] = torch.empty((n,), dtype=torch.uint8, device=s["x"].device)
    if s["kind"] == "matmul":
        return ctx.matmul_int8(s["x"], (s["wt"], s["ws"]), bias=s["b"], y=s["y"], workspace=s["ws_buf"])
    return ctx.moe_ffn_int8(s["x"], s["idx"], s["gate"], s["table"], s["F"], y=s["y"], workspace=s["ws_buf"])


def run(state):
    s = state
    if own:
        return _own(s)
    if s["kind"] == "route":
        return _select(s)
    if s["kind"] == "quantize":
        codes, scale = _quantize(s["x"])
        codes = torch.nn.functional.pad(codes, (0, s["codes"].shape[1] - codes.shape[1]))
        return codes.to(torch.int8), scale[:, 0]
    return _matmul(s) if s["kind"] == "matmul" else _ffn_plain(s)


# ---------------------------------------------------------------------------------------------------------- 64 bits

def _rows64(x):
    """(codes, scales) of the rows of x, all in 64 bits."""
    peak = x.double().abs().max(dim=-1, keepdim=True).values
    step = peak / 127.0
    return torch.where(peak > 0, torch.round(127.0 * x.double() / peak), 0.0), step


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "route":
        l = s["logits"].double()
        p = torch.sigmoid(l) if s["score"] == "sigmoid" else torch.softmax(l, -1)
        v = p + (0.0 if s["b"] is None else s["b"].double())
        n = s["E"] // s["groups"]
        if s["groups"] > 1:
            gv = v.unflatten(1, (s["groups"], n)).topk(min(s["best"], n), dim=-1).values.sum(-1)
            low = gv < gv.topk(s["top_groups"], dim=-1).values[:, -1:]
            v = v.masked_fill(low.repeat_interleave(n, dim=1), -math.inf)
        chosen = torch.argsort(v, dim=-1, descending=True, stable=True)[:, :s["k"]]
        w = p.gather(1, chosen)
        return None, w / w.sum(-1, keepdim=True)
    if s["kind"] == "quantize":
        return None, _rows64(s["x"])[1][:, 0]
    if s["kind"] == "matmul":
        codes, step = _rows64(s["x"])
        y = torch.matmul(codes, s["wq"].double().T) * (step * s["ws"].double())
        return y if s["b"] is None else y + s["b"].double()
    codes, step = _rows64(s["x"])
    y = torch.zeros((s["T"], s["H"]), dtype=torch.float64, device="cuda")
    for e in range(s["E"]):
        token, slot = (s["idx"] == e).nonzero(as_tuple=True)
        if not token.numel():
            continue
        w1, w3, w2 = (q[e].double() * c[e].double()[:, None] for q, c in zip(s["q"], s["s"]))
        x = codes[token] * step[token]
        a = x @ w1.T
        hc, hs = _rows64(a * torch.sigmoid(a) * (x @ w3.T))
        y.index_add_(0, token, (hc * hs) @ w2.T * s["gate"][token, slot].double()[:, None])
    return y


# ---------------------------------------------------------------------------------------------------------- work

def work(case):
    c = case
    if c["kind"] == "route":
        # an exponential, the group's comparisons and the selection: a few operations a logit
        return {"bytes": c["T"] * c["E"] * SIZES[c["dtype"]] + 8 * c["T"] * c["k"] + 4 * c["E"] * bool(c["bias"]), "flops": 8 * c["T"] * c["E"]}
    if c["kind"] == "quantize":
        n = c["rows"] * c["K"]
        return {"bytes": n * (SIZES[c["dtype"]] + 1) + 4 * c["rows"], "flops": 3 * n}
    if c["kind"] == "matmul":
        T, N, K = c["T"], c["N"], c["K"]
        return {"bytes": T * K * SIZES[c["dtype"]] + N * K + 4 * N * (1 + bool(c["bias"])) + T * N * SIZES[c["out"]], "flops": 2 * T * N * K}
    T, H, F, E, k = (c[n] for n in "THFEk")
    met = E * (1.0 - (1.0 - k / E) ** T)  # experts that some token meets, where all are as likely
    return {"bytes": met * (3 * H * F + 4 * (2 * F + H)) + T * H * (SIZES[c["dtype"]] + 2) + 8 * T * k, "flops": 6 * T * k * H * F}
