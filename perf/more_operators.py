"""The operators on rows held in 8 bits, as cases to be timed.

``gcn_quantize`` and ``gcn_dequantize`` keep a matrix of activations as 8-bit
codes with a scale for each row and take it back; ``gcn_transform_q8`` is the
layer's product from such rows and weights with a scale for each column, in
8-bit integers; ``gcn_transform_bwd_q8`` is the backward pass of the layer's
product from a checkpoint in 8 bits.  Row counts and widths are those of
``inputs.SPECS`` (2048, 16384, 131072, 200000 and 2^21 vertices; 500, 256, 128,
64, 40, 16 and 7 columns) and of the model-size sweep (2048 columns).

``run`` computes the plain form in elementary torch operations, or, with
``own``, calls the library.  ``exact`` recomputes each case in float64.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
PREC = {"f32": 0, "f16": 1, "bf16": 2}     # gcn_precision
KIND = {"signed": 0, "relu": 1}            # gcn_q8_kind
LEVELS = {"signed": 127, "relu": 255}      # the largest code


def listed():
    return [
        # Hidden activations of the citation-network setup.  Bound by launches.
        {"name": "keep_er2k_f32", "op": "keep", "n": 2048, "f_in": 16, "kind": "relu", "prec": "f32"},
        # Features of the dense workload, of either sign; odd width.
        {"name": "keep_sbm16k_bf16", "op": "keep", "n": 16384, "f_in": 500, "kind": "signed", "prec": "bf16"},
        # Hidden activations of the largest training workload.
        {"name": "keep_rmat21_f16", "op": "keep", "n": 1 << 21, "f_in": 128, "kind": "relu", "prec": "f16"},
        # One vertex answered by a wide model: the weights are all there is to read.
        {"name": "product_one_row_f16", "op": "product", "n": 1, "f_in": 2048, "f_out": 2048, "kind": "relu",
         "prec": "f16"},
        # Output layer of the Barabasi-Albert workload, answered in fp32; odd width.
        {"name": "product_ba200k_f32", "op": "product", "n": 200000, "f_in": 128, "f_out": 40, "kind": "relu",
         "prec": "f32"},
        # First layer of the largest workload, its features kept in 8 bits.
        {"name": "product_rmat21_f16", "op": "product", "n": 1 << 21, "f_in": 128, "f_out": 128, "kind": "signed",
         "prec": "f16"},
        # A hidden layer of the widest model: bound by the matrix cores.
        {"name": "product_wide_bf16", "op": "product", "n": 32768, "f_in": 2048, "f_out": 2048, "kind": "relu",
         "prec": "bf16"},
        # Output layer of the citation-network setup.  Bound by launches.
        {"name": "backward_er2k_f32", "op": "backward", "n": 2048, "f_in": 16, "f_out": 7, "kind": "relu",
         "prec": "f32", "p": 0.5, "below": True},
        # First layer of the dense workload: features of either sign, nothing below.
        {"name": "backward_sbm16k_bf16", "op": "backward", "n": 16384, "f_in": 500, "f_out": 64, "kind": "signed",
         "prec": "bf16", "p": 0.0, "below": False},
        # Embedding layer of the link-prediction workload in fp32.
        {"name": "backward_rmat17_f32", "op": "backward", "n": 1 << 17, "f_in": 256, "f_out": 64, "kind": "relu",
         "prec": "f32", "p": 0.0, "below": True},
        # Output layer of the widest model.
        {"name": "backward_wide_f16", "op": "backward", "n": 32768, "f_in": 2048, "f_out": 16, "kind": "relu",
         "prec": "f16", "p": 0.5, "below": True},
        # Output layer of the largest training workload.
        {"name": "backward_rmat21_f16", "op": "backward", "n": 1 << 21, "f_in": 128, "f_out": 64, "kind": "relu",
         "prec": "f16", "p": 0.5, "below": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["keep", "product", "backward"])
    kind = rng.choice(["signed", "relu"])
    prec = rng.choice(["f32", "f16", "bf16"])
    b = BYTES[prec]
    case = {"op": op, "kind": kind, "prec": prec}
    case["f_in"] = _log_int(rng, 1, 4096 if op == "keep" else 2048)
    per_row, flops = case["f_in"] * (2 * b + 2), 1
    if op != "keep":
        case["f_out"] = _log_int(rng, 1, 2048 if op == "product" else 256)
        per_row = case["f_in"] + b * case["f_out"]
        flops = 2 * case["f_in"] * case["f_out"]
    if op == "backward":
        case["below"] = rng.random() < 0.75
        case["p"] = rng.choice([0.0, round(rng.uniform(0.05, 0.8), 3)]) if case["below"] and kind == "relu" else 0.0
        per_row += b * case["f_in"] if case["below"] else 0
        flops *= 2
    # at most 2^21 rows, and no more bytes and operations than the largest listed cases
    # (fp32 products of the backward pass count 16 times: their matrix instructions are that much slower)
    flops *= 16 if op == "backward" and prec == "f32" else 1
    most = max(1, min(1 << 21, (1 << 30) // per_row, (1 << 38) // flops))
    case["n"] = _log_int(rng, 1, most)
    return case


def _pad(f, m):
    return (f + m - 1) // m * m


# ------------------------------------------------------------ plain forms ----
# A row h is kept as codes and a scale s: with a the largest |h| (of either
# sign) or the largest h (relu), s is a / 127 or a / 255 cut off after 16
# significant bits, 2^-126 at the least, so that code times scale is exact in
# 32 bits.  The codes are h / s rounded to the nearest whole number, ties to
# even; relu: 0 where h <= 0 and at least 1 elsewhere, so that the codes hold
# the mask h > 0 exactly.

def _scale(a, levels):
    # a double keeps 52 bits behind its first: all but 15 of them cleared
    s = ((a.double() / levels).view(torch.int64) & ~((1 << 37) - 1)).view(torch.float64)
    return s.clamp(min=2.0 ** -126)


def _codes(h, kind):
    """Codes (float64, whole numbers) and scales (float64, a column)."""
    h = h.double()      # quotients next to a border
    a = (h.abs() if kind == "signed" else h.clamp(min=0.0)).amax(1, keepdim=True)
    s = _scale(a, LEVELS[kind])
    q = torch.round(h / s)
    if kind == "relu":
        q = torch.where(h > 0, q.clamp(min=1.0), 0.0)
    return q, s


def _row_blocks(n, per_row):
    step = max(1, (1 << 27) // max(1, per_row))
    return [(a, min(n, a + step)) for a in range(0, n, step)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, K, dt, kind = case["n"], case["f_in"], DTYPES[case["prec"]], case["kind"]
    st = dict(case, dt=dt, ld_q=_pad(K, 16), ld_in=_pad(K, 8))
    code_t = torch.int8 if kind == "signed" else torch.uint8

    def activations(a, b):
        """Features ~ N(0, 1), or hidden activations after ReLU and dropout;
        the rows' sizes differ."""
        h = torch.randn((b - a, K), generator=gen, device=DEV)
        h *= torch.exp(0.5 * torch.randn((b - a, 1), generator=gen, device=DEV))
        if kind == "relu":
            h = torch.where(torch.rand((b - a, K), generator=gen, device=DEV) < 0.5, 2.0 * h.clamp(min=0.0), 0.0)
        return h.to(dt)

    st["overflow"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if case["op"] == "keep":
        st["H"] = torch.zeros((n, st["ld_in"]), dtype=dt, device=DEV)
        for a, b in _row_blocks(n, K):
            st["H"][a:b, :K] = activations(a, b)
        # where the rows are kept, and where they come back to
        st["Hq"] = torch.zeros((n, st["ld_q"]), dtype=code_t, device=DEV)
        st["scale"] = torch.zeros(n, device=DEV)
        st["back"] = torch.zeros((n, st["ld_in"]), dtype=dt, device=DEV)
        return st
    N = case["f_out"]
    st["ld_out"] = _pad(N, 8)
    st["Hq"] = torch.zeros((n, st["ld_q"]), dtype=code_t, device=DEV)
    st["scale"] = torch.zeros(n, device=DEV)
    for a, b in _row_blocks(n, 2 * K):
        q, s = _codes(activations(a, b), kind)
        st["Hq"][a:b, :K] = q.to(code_t)
        st["scale"][a:b] = s[:, 0].float()
    W = (torch.rand((K, N), generator=gen, device=DEV) * 2 - 1) * math.sqrt(6.0 / (K + N))
    W = W.to(dt)
    if case["op"] == "product":
        # the weights as a program lays them out once: columns' codes contiguous
        st["ld_wq"] = _pad(K, 16)
        q, s = _codes(W.t(), "signed")
        st["Wq"] = torch.zeros((N, st["ld_wq"]), dtype=torch.int8, device=DEV)
        st["Wq"][:, :K] = q.to(torch.int8)
        st["w_scale"] = s[:, 0].float()
        st["w_sum"] = q.sum(1).to(torch.int32)
        st["S"] = torch.zeros((n, st["ld_out"]), dtype=dt, device=DEV)
        return st
    st["W"] = torch.zeros((K, st["ld_out"]), dtype=dt, device=DEV)
    st["W"][:, :N] = W
    st["G"] = torch.zeros((n, st["ld_out"]), dtype=dt, device=DEV)
    for a, b in _row_blocks(n, N):
        st["G"][a:b, :N] = (0.05 * torch.randn((b - a, N), generator=gen, device=DEV)).to(dt)
    st["dW"] = torch.zeros((K, st["ld_out"]), device=DEV)
    st["dZ"] = torch.zeros((n, st["ld_in"]), dtype=dt, device=DEV) if case["below"] else None
    st["db"] = torch.zeros(st["ld_in"], device=DEV) if case["below"] else None
    return st


def _plain_keep(st):
    q, s = _codes(st["H"][:, :st["f_in"]], st["kind"])
    s = s.float()
    return {"values": (q.float() * s).to(st["dt"]), "scale": s[:, 0]}


def _plain_product(st):
    K, N = st["f_in"], st["f_out"]
    q, w = st["Hq"][:, :K].float(), st["Wq"][:, :K].float().t().contiguous()
    acc = None
    for k in range(0, K, 256):      # sums of 256 products are exact in 32 bits, longer ones not
        part = q[:, k:k + 256] @ w[k:k + 256]
        acc = part if K <= 256 else (part.double() if acc is None else acc.add_(part))
    return {"S": (acc.float() * st["scale"][:, None] * st["w_scale"]).to(st["dt"])}


def _plain_backward(st):
    K, N, dt = st["f_in"], st["f_out"], st["dt"]
    q = st["Hq"][:, :K].float()
    h = (q * st["scale"][:, None]).to(dt).float()     # the rows as they are taken back
    g = st["G"][:, :N].float()
    out = {"dW": h.t() @ g}
    if st["below"]:
        dz = g @ st["W"][:, :N].float().t()
        if st["kind"] == "relu":
            dz = torch.where(q > 0, dz * (1.0 / (1.0 - st["p"])), 0.0)
        out["dZ"] = dz.to(dt)
        out["db"] = dz.sum(0, dtype=torch.float64).float()
    return out


# ---------------------------------------------------------- library calls ----

def _own(st):
    from paper_2010_12635_amd import gcn as G
    n, K, prec, kind = st["n"], st["f_in"], PREC[st["prec"]], KIND[st["kind"]]
    if st["op"] == "keep":
        G.gcn_quantize(n, K, prec, st["H"], st["ld_in"], kind, st["Hq"], st["ld_q"], st["scale"], st["overflow"])
        G.gcn_dequantize(n, K, kind, st["Hq"], st["ld_q"], st["scale"], prec, st["back"], st["ld_in"],
                         st["overflow"])
        return {"values": st["back"][:, :K], "scale": st["scale"]}
    N = st["f_out"]
    if st["op"] == "product":
        G.gcn_transform_q8(n, K, N, kind, st["Hq"], st["ld_q"], st["scale"], st["Wq"], st["ld_wq"], st["w_scale"],
                           st["w_sum"], prec, st["S"], st["ld_out"], st["overflow"])
        return {"S": st["S"][:, :N]}
    if "ws" not in st:      # the call's scratch, kept by the program between calls
        st["ws"] = torch.empty(G.gcn_transform_bwd_q8_workspace_size(n, K, N, prec), dtype=torch.uint8, device=DEV)
    act = G.GCN_ACT_RELU if st["kind"] == "relu" else G.GCN_ACT_NONE
    G.gcn_transform_bwd_q8(n, K, N, prec, kind, st["Hq"], st["ld_q"], st["scale"], st["W"], st["ld_out"], st["G"],
                           st["ld_out"], act, st["p"], st["dW"], st["dZ"], st["ld_in"], st["db"], st["overflow"],
                           st["ws"])
    out = {"dW": st["dW"][:, :N]}
    if st["below"]:
        out["dZ"], out["db"] = st["dZ"][:, :K], st["db"][:K]
    return out


def run(state):
    if own:
        return _own(state)
    return {"keep": _plain_keep, "product": _plain_product, "backward": _plain_backward}[state["op"]](state)


def work(case):
    n, K, b = case["n"], case["f_in"], BYTES[case["prec"]]
    if case["op"] == "keep":
        # rows in, codes and scales out; codes and scales in, rows out
        return {"bytes": n * K * (2 * b + 2) + 8 * n, "flops": 4 * n * K}
    N = case["f_out"]
    if case["op"] == "product":
        return {"bytes": n * (K + 4 + b * N) + N * (K + 8), "flops": 2 * n * K * N}
    total = n * (K + 4 + b * N) + 4 * K * N
    if case["below"]:
        total += b * (n * K + K * N) + 4 * K
    return {"bytes": total, "flops": 2 * n * K * N * (2 if case["below"] else 1)}


# ------------------------------------------------------------------ float64 ----

def exact(case, seed):
    st = prepare(case, seed)
    n, K, kind = case["n"], case["f_in"], case["kind"]
    if case["op"] == "keep":
        values = torch.empty((n, K), dtype=torch.float64, device=DEV)
        scale = torch.empty(n, dtype=torch.float64, device=DEV)
        for a, b in _row_blocks(n, K):
            h = st["H"][a:b, :K].double()
            top = torch.maximum(h.max(1).values, -h.min(1).values) if kind == "signed" else h.max(1).values
            # what is left over after whole units of the 16th bit is cut off
            x = torch.where(top > 0, top / LEVELS[kind], 2.0 ** -126)
            unit = x / torch.frexp(x).mantissa * 2.0 ** -16
            s = (x - torch.fmod(x, unit))[:, None]
            s = torch.where(s > 2.0 ** -126, s, 2.0 ** -126)
            # the nearest whole number: the lower one, or the next where more than half is left or half of an odd one
            low = torch.div(h, s, rounding_mode="floor")
            rest = h / s - low
            q = torch.where((rest > 0.5) | ((rest == 0.5) & (torch.remainder(low, 2) == 1)), low + 1, low)
            if kind == "relu":
                q[h <= 0] = 0
                q[(h > 0) & (q == 0)] = 1
            # rounded to the rows' type, as they are taken back
            values[a:b] = (q * s).to(st["dt"]).double()
            scale[a:b] = s[:, 0]
        return {"values": values, "scale": scale}
    N = case["f_out"]
    if case["op"] == "product":
        w = st["Wq"][:, :K].double().t().contiguous()
        out = torch.empty((n, N), dtype=torch.float64, device=DEV)
        for a, b in _row_blocks(n, K + N):
            out[a:b] = st["Hq"][a:b, :K].double() @ w
            out[a:b] *= st["scale"][a:b, None].double()
        return {"S": out * st["w_scale"].double()}
    dW = torch.zeros((K, N), dtype=torch.float64, device=DEV)
    dZ = torch.empty((n, K), dtype=torch.float64, device=DEV) if case["below"] else None
    wt = st["W"][:, :N].double().t().contiguous()
    for a, b in _row_blocks(n, 2 * K + N):
        q = st["Hq"][a:b, :K].double()
        h = (q * st["scale"][a:b, None].double()).to(st["dt"]).double()
        g = st["G"][a:b, :N].double()
        dW += h.t() @ g
        if case["below"]:
            d = g @ wt
            if kind == "relu":
                d *= (q != 0)
                d /= 1.0 - case["p"]
            dZ[a:b] = d
    out = {"dW": dW}
    if case["below"]:
        out["dZ"], out["db"] = dZ, dZ.sum(0)
    return out
