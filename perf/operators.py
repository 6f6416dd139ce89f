"""Low-rank adapters beside the shared 2:4 projections, and activations kept in 8 bits for the backward pass: their workloads.

A 2:4 layer that is fine-tuned or served for many fine-tunes keeps its packed weight; what differs from row to row is a low-rank
adapter.  Rows come in segments (requests, or sequences of a training batch); segment s holds the rows starts[s] .. starts[s + 1] - 1
and uses adapter adapters[s], or none (-1); rows of no segment have none either.  With s_n the scale of adapter n, A_n (R x I), B_n (R x O):

    forward           S = s_n X A_n^T          Z = base + S B_n        (base: the shared projection's output)
    input gradient    dS = s_n dZ B_n^T        dX = base + dS A_n      (base: the shared projection's input gradient)
    weight gradients  dA_n = sum dS^T X        dB_n = sum S^T dZ       (over the rows of adapter n)

Activation checkpoints hold e4m3 codes and one power of two for every 32 consecutive features (E8M0 bytes):

    pack              e = the least exponent >= -117 with max |x| <= 448 * 2^e, code = RNE_e4m3(x * 2^-e)
    backward          H = code * 2^e, A = act(H), dH = dA * act'(H)     (act: GELU in its tanh form, or none)
"""
import math

import torch

own = False

BLOCK = 32                     # features that share a scale
BITS8 = {"e4m3": (torch.float8_e4m3fn, 448.0), "e5m2": (torch.float8_e5m2, 57344.0)}


# ---- cases ------------------------------------------------------------------------------------------------------------
def _adapter(name, op, T, I, O, R, N, S, x, dz="bf16", decode=False, bare=0.0, tail=0, base=True):
    """x / dz: storage type of the activations and of the output gradient; decode: one row a segment; bare: share of segments without an adapter;
    tail: rows behind the last segment (a padded batch)."""
    return {"name": name, "op": op, "T": T, "I": I, "O": O, "R": R, "N": N, "S": S, "x": x, "dz": dz, "decode": decode, "bare": bare, "tail": tail, "base": base}


def _checkpoint(name, op, T, C, act="gelu", outputs="both"):
    return {"name": name, "op": op, "T": T, "C": C, "act": act, "outputs": outputs}


def listed():
    return [
        # one request's token through the attention input of the 774M block: latency alone
        _adapter("fwd one token", "fwd", 1, 1280, 3840, 16, 8, 1, "bf16", decode=True),
        # a decode batch of many requests, each with an adapter of its own choice, some without
        _adapter("fwd decode batch", "fwd", 96, 1280, 5120, 16, 64, 96, "bf16", decode=True, bare=0.1),
        # ragged prompts in one batch with padding behind them, second linear of the feed-forward block
        _adapter("fwd ragged prompts", "fwd", 2999, 5120, 1280, 64, 7, 23, "bf16", bare=0.1, tail=57),
        # training forward of the 8-bit recipe at the block's full batch
        _adapter("fwd training 8 bit", "fwd", 32768, 1280, 5120, 32, 1, 1, "e4m3"),
        # training backward of the 350M feed-forward block, four tasks in the batch
        _adapter("dgrad training", "dgrad", 16384, 1024, 4096, 16, 4, 8, "bf16"),
        # ragged batch in the 8-bit recipe: gradients in e5m2
        _adapter("dgrad 8 bit ragged", "dgrad", 5003, 1280, 3840, 128, 3, 11, "e4m3", dz="e5m2", tail=3),
        # weight gradients of the training batch, bf16
        _adapter("wgrad training", "wgrad", 16384, 1024, 4096, 16, 4, 8, "bf16"),
        # weight gradients straight from the 8-bit checkpoint of the layer input, ragged
        _adapter("wgrad checkpoint", "wgrad", 7777, 1280, 5120, 64, 3, 11, "checkpoint", bare=0.1),
        # checkpoint of a short batch's layer input, and of the pre-activations of a full one
        _checkpoint("pack short", "pack", 333, 1280),
        _checkpoint("pack training", "pack", 32768, 5120),
        # a short batch's layer input restored as it is
        _checkpoint("restore short", "backward", 333, 1296, act="none", outputs="A"),
        # the activation and its backward from the checkpoint of the pre-activations
        _checkpoint("backward training", "backward", 16384, 5120),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["fwd", "fwd", "dgrad", "wgrad", "pack", "backward"])
    if op in ("pack", "backward"):
        T, C = _log(rng, 1, 16384), 16 * _log(rng, 1, 320)
        act = rng.choice(["gelu", "none"])
        return {k: v for k, v in _checkpoint("", op, T, C, act, rng.choice(["both", "A", "dH"])).items() if k != "name"}
    T, I, O = _log(rng, 1, 16384), 16 * _log(rng, 4, 320), 16 * _log(rng, 4, 320)
    R = rng.choice([8, 16, 24, 32, 48, 64, 128])
    decode = op == "fwd" and T <= 256
    N = rng.randint(1, 64) if decode else rng.randint(1, 8)
    S = T if decode else rng.randint(1, min(T, 24))
    tail = rng.choice([0, 0, rng.randint(0, T // 4)]) if not decode else 0
    S = min(S, T - tail)
    x = rng.choice(["bf16", "bf16", "e4m3", "checkpoint"] if op == "wgrad" else ["bf16", "bf16", "e4m3"])
    dz = rng.choice(["bf16", "e4m3", "e5m2"])
    case = _adapter("", op, T, I, O, R, N, S, x, dz, decode, rng.choice([0.0, 0.2]), tail, rng.random() < 0.8)
    return {k: v for k, v in case.items() if k != "name"}


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _normal(gen, shape, std):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)


def _stored(t, kind):
    """A tensor as the framework stores it: (storage, its scale, block scales)."""
    if kind == "bf16":
        return t.to(torch.bfloat16), 1.0, None
    if kind == "checkpoint":
        codes, scales = _pack(t.to(torch.bfloat16))
        return codes, 1.0, scales
    dtype, top = BITS8[kind]
    scale = float(t.abs().max()) / top
    return (t / scale).clamp(-top, top).to(dtype), scale, None


def _layout(case, seed):
    """Segment bounds and their adapters (host lists): ragged lengths, an adapter more than once where there are more segments than adapters."""
    g = torch.Generator().manual_seed(seed)
    rows, S = case["T"] - case["tail"], case["S"]
    if case["decode"]:
        starts = list(range(S + 1))
    else:
        cuts = torch.randperm(max(rows - 1, 1), generator=g)[:S - 1] + 1 if S > 1 else torch.zeros(0)
        starts = [0] + sorted(int(c) for c in cuts) + [rows]
    ids = torch.randint(0, case["N"], (S,), generator=g)
    bare = torch.rand(S, generator=g) < case["bare"]
    return starts, torch.where(bare, -1, ids).tolist()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, op = case["T"], case["op"]
    if op == "pack":
        # pre-activations: a normal bulk, features of their own size, a few large values
        X = _normal(gen, (T, case["C"]), 1.0) * torch.exp(_normal(gen, (case["C"],), 0.7))
        return {"case": case, "X": X.to(torch.bfloat16)}
    if op == "backward":
        codes, scales = _pack(_normal(gen, (T, case["C"]), 1.5).to(torch.bfloat16))
        return {"case": case, "codes": codes, "scales": scales, "dA": _normal(gen, (T, case["C"]), 1e-3).to(torch.bfloat16)}
    I, O, R, N = case["I"], case["O"], case["R"], case["N"]
    starts, ids = _layout(case, seed)
    s = {"case": case,
         "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"),
         "adapters": torch.tensor(ids, dtype=torch.int32, device="cuda"),
         "A": _normal(gen, (N, R, I), 0.02).to(torch.bfloat16),
         "B": _normal(gen, (N, R, O), 0.02).to(torch.bfloat16),
         "scale": torch.rand(N, device="cuda", generator=gen) * 1.5 + 0.5}
    if op in ("fwd", "wgrad"):
        s["X"], s["x_scale"], s["x_blocks"] = _stored(_normal(gen, (T, I), 1.0), case["x"])
    if op in ("dgrad", "wgrad"):
        s["dZ"], s["dz_scale"], _ = _stored(_normal(gen, (T, O), 1e-3), case["dz"])
    if op == "wgrad":
        # what the forward pass and the input gradient left: zero for rows without an adapter, as those calls write them
        has = (_rows(s) >= 0)[:, None]
        s["S"], s["dS"] = _normal(gen, (T, R), 0.7) * has, _normal(gen, (T, R), 1e-3) * has
    elif case["base"]:
        s["base"] = _normal(gen, (T, O if op == "fwd" else I), 1.0 if op == "fwd" else 1e-3).to(torch.bfloat16)
    else:
        s["base"] = None
    return s


# ---- the plain form ---------------------------------------------------------------------------------------------------
def _rows(s):
    """The adapter of every row, -1 where it has none."""
    row = torch.arange(s["case"]["T"], dtype=torch.int32, device="cuda")
    at = torch.searchsorted(s["starts"], row, right=True) - 1            # the last segment that starts at the row or before it
    inside = (at >= 0) & (row < s["starts"][-1])
    return torch.where(inside, s["adapters"][at.clamp(0, s["case"]["S"] - 1)], -1)


def _values(codes, scale, blocks=None):
    v = codes.to(torch.float32)
    if blocks is not None:
        return v * torch.exp2(blocks.to(torch.float32) - 127.0).repeat_interleave(BLOCK, 1)[:, :v.shape[1]]
    return v if scale == 1.0 else v * scale


def _down_up(s, X, A, B):
    """(base + S B, S) with S = scale X A^T, each row with its own adapter."""
    ids, (N, R, _) = _rows(s), A.shape
    n, has = ids.clamp(min=0).long(), (ids >= 0)[:, None]
    A, B = A.to(torch.float32), B.to(torch.float32)
    if X.shape[0] <= N:                                                  # few rows: each row's own matrices
        S = (A[n] * X[:, None, :]).sum(2) * s["scale"][n][:, None] * has
        delta = (B[n] * S[:, :, None]).sum(1)
    else:                                                                # many rows: all adapters side by side, the others' parts masked
        mine = torch.arange(N, device="cuda") == ids[:, None]
        every = (X @ A.reshape(N * R, -1).t()).reshape(-1, N, R) * s["scale"][:, None] * mine[:, :, None]
        S = every.sum(1)
        delta = every.reshape(-1, N * R) @ B.reshape(N * R, -1)
    out = delta if s["base"] is None else s["base"].to(torch.float32) + delta
    return out.to(torch.bfloat16), S


def _pack(X):
    T, C = X.shape
    blocks = -(-C // BLOCK)
    x = torch.nn.functional.pad(X.to(torch.float32), (0, blocks * BLOCK - C)).reshape(T, blocks, BLOCK)
    m, e = torch.frexp(x.abs().amax(2))                                  # max = m * 2^e, m in [1/2, 1); 448 = 7/8 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-117)
    codes = torch.ldexp(x, -e[:, :, None]).to(torch.float8_e4m3fn).reshape(T, -1)[:, :C].contiguous()
    return codes, (e + 127).to(torch.uint8)


def _gelu(h):
    """The activation and its derivative."""
    t = torch.tanh(math.sqrt(2 / math.pi) * (h + 0.044715 * h * h * h))
    return 0.5 * h * (1 + t), 0.5 * (1 + t) + 0.5 * h * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * h * h)


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "pack":
        codes, scales = _pack(s["X"])
        return {"codes": codes, "scales": scales}
    if op == "backward":
        h = _values(s["codes"], 1.0, s["scales"])
        a, da = _gelu(h) if case["act"] == "gelu" else (h, None)
        out = {}
        if case["outputs"] != "dH":
            out["A"] = a.to(torch.bfloat16)
        if case["outputs"] != "A":
            out["dH"] = s["dA"].clone() if da is None else (s["dA"].to(torch.float32) * da).to(torch.bfloat16)
        return out
    if op == "fwd":
        Z, S = _down_up(s, _values(s["X"], s["x_scale"]), s["A"], s["B"])
        return {"Z": Z, "S": S}
    if op == "dgrad":
        dX, dS = _down_up(s, _values(s["dZ"], s["dz_scale"]), s["B"], s["A"])
        return {"dX": dX, "dS": dS}
    N, R = case["N"], case["R"]
    mine = (torch.arange(N, device="cuda") == _rows(s)[:, None])[:, :, None]
    spread = lambda v: (v[:, None, :] * mine).reshape(-1, N * R).t()     # noqa: E731
    dA = spread(s["dS"]) @ _values(s["X"], s["x_scale"], s["x_blocks"])
    dB = spread(s["S"]) @ _values(s["dZ"], s["dz_scale"])
    return {"dA": dA.reshape(N, R, -1), "dB": dB.reshape(N, R, -1)}


# ---- the framework's calls --------------------------------------------------------------------------------------------
def _own(s):
    import paper_2409_09099_amd as sste
    case = s["case"]
    op = case["op"]
    act = sste.ACT_GELU_TANH if case.get("act") == "gelu" else sste.ACT_NONE
    kinds = {"bf16": sste.BF16, "e4m3": sste.F8E4M3, "e5m2": sste.F8E5M2, "checkpoint": sste.F8BLOCK}
    if op == "pack":
        codes, scales = sste.checkpoint_pack(s["X"])
        return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales}
    if op == "backward":
        dA = s["dA"] if case["outputs"] != "A" else None
        A, dH = sste.checkpoint_backward(s["codes"], s["scales"], dA=dA, act=act, restore=case["outputs"] != "dH")
        return {k: v for k, v in (("A", A), ("dH", dH)) if v is not None}
    if op == "fwd":
        Z, S = sste.adapter_fwd(s["X"], s["starts"], s["adapters"], s["A"], s["B"], scale=s["scale"], base=s["base"], dtype=kinds[case["x"]], x_scale=s["x_scale"])
        return {"Z": Z, "S": S}
    if op == "dgrad":
        dX, dS = sste.adapter_dgrad(s["dZ"], s["starts"], s["adapters"], s["A"], s["B"], scale=s["scale"], base=s["base"], dtype=kinds[case["dz"]],
                                    dy_scale=s["dz_scale"])
        return {"dX": dX, "dS": dS}
    dA, dB = sste.adapter_wgrad(s["dZ"], s["X"], s["S"], s["dS"], s["starts"], s["adapters"], case["N"], dtype=kinds[case["dz"]], dy_scale=s["dz_scale"],
                                x_dtype=kinds[case["x"]], x_scale=s["x_scale"], x_blocks=s["x_blocks"])
    return {"dA": dA, "dB": dB}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    T = case["T"]
    if case["op"] in ("pack", "backward"):
        n, scales = T * case["C"], T * -(-case["C"] // BLOCK)
        if case["op"] == "pack":
            return {"bytes": 3 * n + scales, "flops": 4 * n}
        outputs = {"both": 6, "dH": 4, "A": 2}[case["outputs"]]
        return {"bytes": (1 + outputs) * n + scales, "flops": (20 if case["act"] == "gelu" else 1) * n}
    I, O, R = case["I"], case["O"], case["R"]
    size = {"bf16": 2, "e4m3": 1, "e5m2": 1, "checkpoint": 1 + 1 / BLOCK}
    used = min(case["N"], case["S"])
    flops = 2 * T * R * (I + O)
    if case["op"] == "wgrad":
        return {"bytes": T * (I * size[case["x"]] + O * size[case["dz"]] + 8 * R) + 4 * case["N"] * R * (I + O), "flops": flops}
    inner, outer, kind = (I, O, case["x"]) if case["op"] == "fwd" else (O, I, case["dz"])
    return {"bytes": T * (inner * size[kind] + outer * (4 if case["base"] else 2) + 4 * R) + 2 * used * R * (I + O), "flops": flops}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    f8 = torch.float64
    op, T = case["op"], case["T"]

    def decoded(codes, scale, blocks=None):
        v = codes.to(torch.float32).to(f8) * scale
        if blocks is not None:
            step = torch.pow(torch.tensor(2.0, dtype=f8, device="cuda"), blocks.to(f8) - 127)
            v = v * step[:, torch.arange(v.shape[1], device="cuda") // BLOCK]
        return v

    if op == "pack":
        out, bytes_ = torch.empty_like(s["X"], dtype=f8), []
        for c in range(0, case["C"], BLOCK):
            x = s["X"][:, c:c + BLOCK].to(f8)
            top = x.abs().amax(1)
            e = torch.full((T,), -117, dtype=torch.int64, device="cuda")
            guess = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)).to(torch.int64)
            for k in (guess + 1, guess, guess - 1):                      # the least of the three that holds the block
                e = torch.where(448 * torch.exp2(k.to(f8)) >= top, torch.maximum(k, torch.full_like(k, -117)), e)
            q = x / torch.exp2(e.to(f8))[:, None]
            step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
            out[:, c:c + BLOCK] = torch.round(q / step) * step           # to the nearest, ties to even
            bytes_.append(e + 127)
        return {"codes": out, "scales": torch.stack(bytes_, 1).to(torch.uint8)}
    if op == "backward":
        h = decoded(s["codes"], 1.0, s["scales"])
        out = {}
        k, c = math.sqrt(2 / math.pi), 0.044715
        sig = 1 / (1 + torch.exp(-2 * k * (h + c * h ** 3)))              # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
        if case["outputs"] != "dH":
            out["A"] = h * sig if case["act"] == "gelu" else h
        if case["outputs"] != "A":
            slope = sig + h * sig * (1 - sig) * 2 * k * (1 + 3 * c * h ** 2) if case["act"] == "gelu" else 1.0
            out["dH"] = s["dA"].to(f8) * slope
        return out
    starts, ids = s["starts"].tolist(), s["adapters"].tolist()
    I, O, R, N = case["I"], case["O"], case["R"], case["N"]
    if op == "wgrad":
        X, dZ = decoded(s["X"], s["x_scale"], s["x_blocks"]), decoded(s["dZ"], s["dz_scale"])
        dA, dB = torch.zeros(N, R, I, dtype=f8, device="cuda"), torch.zeros(N, R, O, dtype=f8, device="cuda")
        for a, b, n in zip(starts, starts[1:], ids):
            if n >= 0:
                dA[n] += s["dS"][a:b].to(f8).t().contiguous() @ X[a:b]
                dB[n] += s["S"][a:b].to(f8).t().contiguous() @ dZ[a:b]
        return {"dA": dA, "dB": dB}
    fwd = op == "fwd"
    V = decoded(s["X"], s["x_scale"]) if fwd else decoded(s["dZ"], s["dz_scale"])
    down, up = (s["A"], s["B"]) if fwd else (s["B"], s["A"])
    low = torch.zeros(T, R, dtype=f8, device="cuda")
    out = torch.zeros(T, O if fwd else I, dtype=f8, device="cuda") if s["base"] is None else s["base"].to(f8)
    for a, b, n in zip(starts, starts[1:], ids):
        if n >= 0:
            low[a:b] = s["scale"][n].to(f8) * (V[a:b] @ down[n].to(f8).t().contiguous())
            out[a:b] += low[a:b] @ up[n].to(f8)
    return {"Z": out, "S": low} if fwd else {"dX": out, "dS": low}
