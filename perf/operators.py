"""The operators that carry one training step through the frozen experts of an
MoE layer, as timed cases: each with its plain form (elementary torch
operations in 32 bits) and with the calls that a program makes of the library.

Kinds:
  moe_dx    the input gradient of the expert projection y[p] = W_e x: per pair
            (the down projection) or summed over a token's slots (gate, up)
  pack      an 8-bit checkpoint of activation rows: written, and read back
  swiglu    a = g sigmoid(g) u forward (serving)
  swiglu_train
            the same forward writing 8-bit checkpoints of g and u, then the
            backward's part from them: a once more (the down projection's
            input, for its adapter's gradient), and dg and du
  swiglu_bwd
            the backward from g and u as they are
  combine   a token's expert outputs summed with the router weights
  combine_bwd
            its gradient: of the outputs and (``dw``) of the router weights

The checkpoint: blocks of 32 columns of a row share a byte s, the exponent
field (of a 32-bit float) of the block's largest |x|, one more where that one
would round to code 128 (but never 255); a value is held as the whole number
x * 2**(133 - s), rounded to nearest even and at most 127 in size, and read as
code * 2**(s - 133).  A block with a NaN or an infinity has s = 255 and reads
as NaN.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _moe(kind, dtype, T, d_in, d_out, E, k, zipf, shared, drop=0.0):
    return {"kind": kind, "dtype": dtype, "T": T, "d_in": d_in, "d_out": d_out, "E": E, "k": k,
            "zipf": zipf, "shared": shared, "drop": drop}


def _rows(kind, dtype, rows, d):
    return {"kind": kind, "dtype": dtype, "rows": rows, "d": d}


def _comb(kind, dtype, T, k, d, dw, drop=0.0):
    return {"kind": kind, "dtype": dtype, "T": T, "k": k, "d": d, "E": 64, "zipf": 0.8, "dw": dw,
            "drop": drop}


def listed():
    return [
        # a unit-test-sized full-precision step through the up projection
        dict(_moe("moe_dx", "f32", 256, 512, 1024, 8, 2, 0.0, True), name="dx_up_tiny_f32"),
        # a small batch through many small experts: their weights are the work
        dict(_moe("moe_dx", "bf16", 57, 1024, 2048, 64, 8, 0.8, False), name="dx_down_few_bf16"),
        # fine-tuning the OLMoE-like layer: gate (or up), summed over 8 slots
        dict(_moe("moe_dx", "bf16", 4096, 2048, 1024, 64, 8, 0.8, True), name="dx_gate_olmoe_bf16"),
        # the Qwen-like down projection: a gradient row per pair, odd token
        # count, some pairs dropped by the router's capacity
        dict(_moe("moe_dx", "bf16", 8191, 1408, 2048, 60, 4, 0.8, False, 0.03), name="dx_down_qwen_bf16"),
        # the Mixtral-like up projection: few, wide experts; the largest
        dict(_moe("moe_dx", "bf16", 16384, 4096, 14336, 8, 2, 0.0, True), name="dx_up_mixtral_bf16"),
        # the input rows of an OLMoE-like layer kept in 8 bits for its backward
        dict(_rows("pack", "bf16", 4096, 2048), name="pack_olmoe_bf16"),
        # pair rows in full precision, a width that ends inside a block
        dict(_rows("pack", "f32", 9999, 1420), name="pack_ragged_f32"),
        # a single decoded token with four routed experts: latency
        dict(_rows("swiglu", "bf16", 4, 1408), name="swiglu_token_bf16"),
        # a training step over the Qwen-like layer's pairs
        dict(_rows("swiglu_train", "bf16", 32768, 1408), name="swiglu_qwen_bf16"),
        # full precision without checkpoints
        dict(_rows("swiglu_bwd", "f32", 15992, 1024), name="swiglu_bwd_f32"),
        # the OLMoE-like layer's output
        dict(_comb("combine", "bf16", 4096, 8, 2048, False), name="combine_olmoe_bf16"),
        # the gradient of outputs and router weights, DeepSeek-like
        dict(_comb("combine_bwd", "bf16", 8192, 6, 2048, True), name="combine_bwd_deepseek_bf16"),
    ]


def _log_int(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return max(-(-lo // step) * step, min(hi // step * step, v))


def _cost_s(case):
    w = work(case)
    return max(w["bytes"] / 4e12, w["flops"] / (6e14 if case["dtype"] == "bf16" else 6e13))


def draw(rng):
    most = max(_cost_s(c) for c in listed())
    while True:
        kind = rng.choice(["moe_dx", "moe_dx", "moe_dx", "pack", "swiglu", "swiglu_train",
                           "swiglu_bwd", "combine", "combine_bwd"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        step = 8 if dtype == "bf16" else 4
        if kind == "moe_dx":
            E = rng.choice([4, 8, 8, 16, 32, 60, 64, 96, 128])
            c = _moe(kind, dtype, _log_int(rng, 1, 16384), _log_int(rng, 256, 4096, step),
                     _log_int(rng, 256, 14336, step), E, rng.choice([1, 2, 4, 6, 8]),
                     rng.choice([0.0, 0.8, 1.0]), rng.random() < 0.5, rng.choice([0.0, 0.0, 0.05]))
            if c["k"] > E or E * c["d_in"] * c["d_out"] > 8 * 4096 * 14336:
                continue
            if c["T"] * c["k"] * c["d_in"] > 1 << 28:
                continue
        elif kind in ("combine", "combine_bwd"):
            c = _comb(kind, dtype, _log_int(rng, 1, 16384), rng.choice([1, 2, 4, 6, 8, 16]),
                      _log_int(rng, 128, 8192, step), kind == "combine_bwd" and rng.random() < 0.6,
                      rng.choice([0.0, 0.05]))
        else:
            c = _rows(kind, dtype, _log_int(rng, 1, 65536), _log_int(rng, 64, 14336, step))
            if c["rows"] * c["d"] > 1 << 29:
                continue
        if _cost_s(c) <= most:
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, std, dtype):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _route(case, g):
    """Routed experts [T, k] (distinct in a row; -1 where dropped) and weights."""
    T, k, E = case["T"], case["k"], case["E"]
    u = torch.rand(T, E, generator=g, device="cuda").clamp_(1e-7, 1 - 1e-7)
    logits = -torch.log(-torch.log(u)) - case["zipf"] * torch.log(
        torch.arange(1, E + 1, device="cuda", dtype=torch.float32))
    ids = logits.topk(k, dim=1).indices
    w = torch.softmax(logits, dim=1).gather(1, ids).float().contiguous()
    ids = ids.to(torch.int32)
    if case["drop"]:
        lost = torch.rand(T, k, generator=g, device="cuda") < case["drop"]
        ids = torch.where(lost, torch.full_like(ids, -1), ids)
    return ids.contiguous(), w


def prepare(case, seed):
    g, dt, kind = _gen(seed), DTYPES[case["dtype"]], case["kind"]
    s = {"case": case, "own": own}
    if own:
        from paper_2609_06072_amd import ace
    if kind in ("moe_dx", "combine", "combine_bwd"):
        ids, w = _route(case, g)
        s["ids"] = ids
        if own:
            s["rt"] = ace.ace_group_permute(ids, case["E"], None, case["E"], ace.ACE_ROWS_EXPERT)
    if kind == "moe_dx":
        T, k, d_in, d_out, E = (case[n] for n in ("T", "k", "d_in", "d_out", "E"))
        s["dy"] = _normal(g, (T * k, d_out), 1.0, dt)
        s["W"] = _normal(g, (E, d_out, d_in), d_in ** -0.5, dt)
        if own:
            s["dx"] = torch.zeros(T if case["shared"] else T * k, d_in, dtype=dt, device="cuda")
            if case["shared"]:
                n = ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, T, k, d_in, d_out, E, 0)
                s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        else:
            # the pairs of each expert, as the library's routing keeps them
            key = ids.reshape(-1).long()
            key = torch.where(key < 0, torch.full_like(key, E), key)
            s["order"] = torch.argsort(key, stable=True)
            s["seg"] = [0] + torch.cumsum(torch.bincount(key, minlength=E + 1), 0).tolist()
    elif kind in ("combine", "combine_bwd"):
        T, k, d = case["T"], case["k"], case["d"]
        s["w"] = w
        if kind == "combine" or case["dw"]:
            s["y"] = _normal(g, (T * k, d), 1.0, dt)
        if kind == "combine_bwd":
            s["dout"] = _normal(g, (T, d), 1.0, dt)
            if own:
                s["dy"] = torch.zeros(T * k, d, dtype=dt, device="cuda")
                s["dw"] = torch.empty(T, k, device="cuda") if case["dw"] else None
        elif own:
            s["out"] = torch.empty(T, d, dtype=dt, device="cuda")
    else:
        n, d = case["rows"], case["d"]
        # features of unequal size, as hidden states have
        scale = torch.exp(0.7 * torch.randn(d, generator=g, device="cuda"))
        for name in (("x",) if kind == "pack" else ("g", "u")):
            s[name] = _normal(g, (n, d), 1.0, torch.float32).mul_(scale).to(dt)
        if kind in ("swiglu_train", "swiglu_bwd"):
            s["da"] = _normal(g, (n, d), 1.0, dt)
        if own:
            out = {"pack": ("x_out",), "swiglu": ("a",), "swiglu_train": ("a", "a_again", "dg", "du"),
                   "swiglu_bwd": ("dg", "du")}[kind]
            for name in out:
                s[name] = torch.empty(n, d, dtype=dt, device="cuda")
            if kind == "pack":
                s["packed"] = ace.PackedAct(n, d)
            if kind == "swiglu_train":
                s["g8"], s["u8"] = ace.PackedAct(n, d), ace.PackedAct(n, d)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _run_own(state) if state["own"] else _run_plain(state)


def _run_own(s):
    from paper_2609_06072_amd import ace
    case, kind = s["case"], s["case"]["kind"]
    if kind == "moe_dx":
        ace.ace_moe_dx(s["dy"], s["W"], s["rt"], s["dx"],
                       input_mode=ace.ACE_INPUT_SHARED if case["shared"] else ace.ACE_INPUT_PER_PAIR,
                       ws=s.get("ws"))
        return s["dx"]
    if kind == "pack":
        ace.ace_act_pack(s["x"], s["packed"])
        return ace.ace_act_unpack(s["packed"], s["x_out"])
    if kind == "swiglu":
        return ace.ace_swiglu_fwd(s["g"], s["u"], s["a"])
    if kind == "swiglu_train":
        ace.ace_swiglu_fwd(s["g"], s["u"], s["a"], g_packed=s["g8"], u_packed=s["u8"])
        ace.ace_swiglu_fwd(s["g8"], s["u8"], s["a_again"])
        ace.ace_swiglu_bwd(s["da"], s["g8"], s["u8"], s["dg"], s["du"])
        return {"a": s["a"], "a_again": s["a_again"], "dg": s["dg"], "du": s["du"]}
    if kind == "swiglu_bwd":
        ace.ace_swiglu_bwd(s["da"], s["g"], s["u"], s["dg"], s["du"])
        return {"dg": s["dg"], "du": s["du"]}
    if kind == "combine":
        return ace.ace_moe_combine_fwd(s["y"], s["rt"], s["out"], pair_w=s["w"])
    ace.ace_moe_combine_bwd(s["dout"], s["rt"], s["dy"], pair_w=s["w"], y=s.get("y"), dw=s["dw"])
    return {"dy": s["dy"], "dw": s["dw"]} if case["dw"] else {"dy": s["dy"]}


def _blocks(x, fill=0.0):
    """[n, d] -> [n, blocks, 32] (the last block filled up) in 32 bits."""
    n, d = x.shape
    pad = -d % 32
    x = x.float()
    if pad:
        x = torch.cat([x, x.new_full((n, pad), fill)], 1)
    return x.view(n, -1, 32)


def _pack(x):
    """(codes int8 [n, blocks, 32], s int32 [n, blocks, 1])"""
    v = _blocks(x)
    top = v.abs().amax(2, keepdim=True)     # NaN where the block holds one
    s = (top.view(torch.int32) & 0x7fffffff) >> 23
    bad = s == 255
    up = (torch.ldexp(top, 127 - s) * 64.0 >= 127.5) & (s < 254)
    s = torch.where(bad, s, s + up.int())
    code = torch.round(torch.ldexp(v, 127 - s) * 64.0).clamp_(-127.0, 127.0)
    return torch.where(bad, torch.zeros_like(code), code).to(torch.int8), s


def _unpack(codes, s, d):
    """The values (32 bits) that the codes stand for, [n, d]."""
    v = torch.ldexp(codes.float() * (1.0 / 64.0), s - 127)
    v = torch.where(s == 255, torch.full_like(v, math.nan), v)
    return v.reshape(codes.shape[0], -1)[:, :d]


def _swiglu_grads(da, g, u):
    sig = torch.sigmoid(g)
    return {"dg": da * u * sig * (1.0 + g * (1.0 - sig)), "du": da * g * sig}


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    dt = DTYPES[case["dtype"]]
    if kind == "moe_dx":
        T, k, d_in = case["T"], case["k"], case["d_in"]
        dx = torch.zeros(T * k, d_in, dtype=torch.float32 if case["shared"] else dt, device="cuda")
        for e in range(case["E"]):
            rows = s["order"][s["seg"][e]:s["seg"][e + 1]]
            if rows.numel():
                dx[rows] = (s["dy"][rows].float() @ s["W"][e].float()).to(dx.dtype)
        return dx.view(T, k, d_in).sum(1).to(dt) if case["shared"] else dx
    if kind == "pack":
        codes, e = _pack(s["x"])
        return _unpack(codes, e, case["d"]).to(dt)
    if kind == "swiglu":
        g = s["g"].float()
        return (g * torch.sigmoid(g) * s["u"].float()).to(dt)
    if kind == "swiglu_train":
        g, u, da = s["g"].float(), s["u"].float(), s["da"].float()
        out = {"a": (g * torch.sigmoid(g) * u).to(dt)}
        g8, u8 = _pack(s["g"]), _pack(s["u"])
        g, u = _unpack(*g8, case["d"]), _unpack(*u8, case["d"])
        out["a_again"] = (g * torch.sigmoid(g) * u).to(dt)
        out.update({n: v.to(dt) for n, v in _swiglu_grads(da, g, u).items()})
        return out
    if kind == "swiglu_bwd":
        grads = _swiglu_grads(s["da"].float(), s["g"].float(), s["u"].float())
        return {n: v.to(dt) for n, v in grads.items()}
    T, k, d = case["T"], case["k"], case["d"]
    routed = s["ids"] >= 0
    w = torch.where(routed, s["w"], torch.zeros_like(s["w"]))
    if kind == "combine":
        return (s["y"].view(T, k, d).float() * w[:, :, None]).sum(1).to(dt)
    dout = s["dout"].float()
    out = {"dy": (dout[:, None, :] * w[:, :, None]).to(dt).view(T * k, d)}
    if case["dw"]:
        dw = (s["y"].view(T, k, d).float() * dout[:, None, :]).sum(2)
        out["dw"] = torch.where(routed, dw, torch.zeros_like(dw))
    return out


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------

def _held(x):
    """What an 8-bit checkpoint of x [n, d] gives back, in 64 bits."""
    d = x.shape[1]
    parts = []
    for c in range(0, d, 32):
        v = x[:, c:c + 32].double()
        top = v.abs().max(1, keepdim=True).values
        # the smallest float with this exponent field: 2**(s - 127), the field 0 with 1
        _, e = torch.frexp(top)
        s = (e + 126).clamp(min=0).double()
        s = torch.where(top == 0, torch.zeros_like(s), s)
        s = s + ((top * 2.0 ** (133.0 - s) >= 127.5) & (s < 254))
        code = torch.round(v * 2.0 ** (133.0 - s)).clamp(-127.0, 127.0)
        parts.append(code * 2.0 ** (s - 133.0))
    return torch.cat(parts, 1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "moe_dx":
        if 2.0 * case["T"] * case["k"] * case["d_in"] * case["d_out"] > 2e13:
            return None
        T, k = case["T"], case["k"]
        ids = s["ids"].reshape(-1)
        out = torch.zeros(T if case["shared"] else T * k, case["d_in"], dtype=torch.float64, device="cuda")
        for e in range(case["E"]):
            p = torch.nonzero(ids == e).squeeze(1)
            if p.numel():
                # one pair of a token and expert at most: no index twice
                to = p // k if case["shared"] else p
                out[to] += torch.mm(s["dy"].index_select(0, p).double(), s["W"][e].double())
        return out
    if kind == "pack":
        return _held(s["x"])
    if kind == "swiglu":
        g, u = s["g"].double(), s["u"].double()
        return g / (1.0 + torch.exp(-g)) * u
    if kind in ("swiglu_train", "swiglu_bwd"):
        g, u, da = s["g"].double(), s["u"].double(), s["da"].double()
        out = {}
        if kind == "swiglu_train":
            out["a"] = g / (1.0 + torch.exp(-g)) * u
            g, u = _held(s["g"]), _held(s["u"])
            out["a_again"] = g / (1.0 + torch.exp(-g)) * u
        h = torch.exp(-g)
        out["dg"] = da * u * (1.0 + h + g * h) / (1.0 + h) ** 2
        out["du"] = da * g / (1.0 + h)
        return out
    T, k, d = case["T"], case["k"], case["d"]
    w = s["w"].double() * (s["ids"] >= 0)
    if kind == "combine":
        out = torch.zeros(T, d, dtype=torch.float64, device="cuda")
        for j in range(k):
            out += w[:, j, None] * s["y"][j::k].double()
        return out
    dout = s["dout"].double()
    dy = torch.empty(T * k, d, dtype=torch.float64, device="cuda")
    dw = torch.zeros(T, k, dtype=torch.float64, device="cuda")
    for j in range(k):
        dy[j::k] = w[:, j, None] * dout
        if case["dw"]:
            dw[:, j] = (s["y"][j::k].double() * dout).sum(1) * (s["ids"][:, j] >= 0)
    return {"dy": dy, "dw": dw} if case["dw"] else {"dy": dy}


# ---------------------------------------------------------------------------
# the work that a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    b, kind = 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind == "moe_dx":
        P, d_in, d_out = case["T"] * case["k"], case["d_in"], case["d_out"]
        rows = case["T"] if case["shared"] else P
        return {"bytes": b * (P * d_out + min(case["E"], P) * d_in * d_out + rows * d_in),
                "flops": 2 * P * d_in * d_out}
    if kind in ("combine", "combine_bwd"):
        T, k, d = case["T"], case["k"], case["d"]
        P = T * k
        if kind == "combine":
            return {"bytes": b * (P * d + T * d) + 4 * P, "flops": 2 * P * d}
        extra = P * d * b + 4 * P if case["dw"] else 0
        return {"bytes": b * (T * d + P * d) + 4 * P + extra, "flops": (3 if case["dw"] else 1) * P * d}
    n, d = case["rows"], case["d"]
    packed = n * (d + -(-d // 32))
    if kind == "pack":      # written, then read back
        return {"bytes": 2 * b * n * d + 2 * packed, "flops": 4 * n * d}
    if kind == "swiglu":
        return {"bytes": 3 * b * n * d, "flops": 5 * n * d}
    if kind == "swiglu_bwd":
        return {"bytes": 5 * b * n * d, "flops": 12 * n * d}
    # g, u -> a and two checkpoints; these -> a; these and da -> dg, du
    return {"bytes": 7 * b * n * d + 6 * packed, "flops": 30 * n * d}
