"""The operators on rows of class scores, as cases to be timed.

``gcn_top_logits`` keeps the largest logits of a teacher, ``gcn_distill``
trains a student on them (loss and gradient in one call) and
``gcn_sample_labels`` draws labels from a model's own distribution.  Row
counts and class counts are those of ``inputs.SPECS`` (7, 40 and 64 classes;
2048, 200000 and 2^21 vertices); the wide ones are generic, for scores over
an entity vocabulary.

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
LOSS_SCALE = 65536.0
NARROW = {"f32": 256, "f16": 512, "bf16": 512}   # widest rows with fused column sums (those of gcn_loss)


def listed():
    return [
        # Student on the citation-network setup: 7 classes, loss on the 140
        # labelled vertices only.  Bound by launches.
        {"name": "distill_er2k_f32", "kind": "distill", "n": 2048, "classes": 7, "k": 3, "n_mask": 140, "prec": "f32",
         "temperature": 2.0, "base": True, "colsum": True},
        # The largest training workload, every vertex distilled on top of the
        # cross-entropy's gradient, with the output layer's bias gradient.
        {"name": "distill_rmat21_f16", "kind": "distill", "n": 1 << 21, "classes": 64, "k": 8, "n_mask": 0,
         "prec": "f16", "temperature": 2.0, "base": True, "colsum": True},
        # Scores over an entity vocabulary, a batch of vertices; odd width.
        {"name": "distill_wide_bf16", "kind": "distill", "n": 2048, "classes": 50001, "k": 64, "n_mask": 0,
         "prec": "bf16", "temperature": 1.0, "base": False, "colsum": False},
        # A few very wide rows in full precision.
        {"name": "distill_few_rows_f32", "kind": "distill", "n": 12, "classes": 131072, "k": 32, "n_mask": 0,
         "prec": "f32", "temperature": 4.0, "base": False, "colsum": False},
        # What a teacher on the Barabasi-Albert workload hands on.
        {"name": "top_ba200k_f32", "kind": "top", "n": 200000, "classes": 40, "k": 5, "prec": "f32"},
        # The same for every vertex of the largest workload.
        {"name": "top_rmat21_f16", "kind": "top", "n": 1 << 21, "classes": 64, "k": 8, "prec": "f16"},
        # A teacher over an entity vocabulary.
        {"name": "top_wide_bf16", "kind": "top", "n": 2048, "classes": 50001, "k": 64, "prec": "bf16"},
        # One query vertex.
        {"name": "top_one_row_f32", "kind": "top", "n": 1, "classes": 131072, "k": 100, "prec": "f32"},
        # Labels drawn for the citation-network setup.  Bound by launches.
        {"name": "sample_er2k_f32", "kind": "sample", "n": 2048, "classes": 7, "prec": "f32", "temperature": 1.0,
         "top_k": 0, "top_p": 0.9, "min_p": 0.0, "unlabelled": 0.93},
        # Every filter at once, on nine tenths of the largest workload's
        # vertices (the others keep their labels).
        {"name": "sample_rmat21_f16", "kind": "sample", "n": 1 << 21, "classes": 64, "prec": "f16",
         "temperature": 0.8, "top_k": 16, "top_p": 0.95, "min_p": 0.02, "unlabelled": 0.9},
        # Nucleus of an entity vocabulary: hundreds of classes a row.
        {"name": "sample_wide_bf16", "kind": "sample", "n": 1024, "classes": 50001, "prec": "bf16",
         "temperature": 1.0, "top_k": 0, "top_p": 0.92, "min_p": 0.0, "unlabelled": 1.0},
        # One draw for one vertex.
        {"name": "sample_one_row_f32", "kind": "sample", "n": 1, "classes": 131072, "prec": "f32",
         "temperature": 0.7, "top_k": 50, "top_p": 0.95, "min_p": 0.0, "unlabelled": 1.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["distill", "top", "sample"])
    prec = rng.choice(["f32", "f16", "bf16"])
    classes = _log_int(rng, 2, 131072)
    # at most the largest listed case's bytes, and at most 2^21 rows
    most = max(1, min(1 << 21, (1 << 28) // (BYTES[prec] * classes)))
    n = _log_int(rng, 1, most)
    case = {"kind": kind, "n": n, "classes": classes, "prec": prec}
    if kind == "distill":
        case["k"] = _log_int(rng, 1, min(classes, 128))
        case["n_mask"] = 0 if rng.random() < 0.5 else rng.randint(1, n)
        case["temperature"] = round(rng.uniform(0.5, 5.0), 3)
        case["base"] = rng.random() < 0.5
        case["colsum"] = classes <= NARROW[prec] and rng.random() < 0.7
    elif kind == "top":
        case["k"] = _log_int(rng, 1, min(classes, 256))
    else:
        case["temperature"] = round(rng.uniform(0.4, 1.6), 3)
        case["top_k"] = rng.choice([0, _log_int(rng, 1, classes)])
        case["top_p"] = rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)])
        case["min_p"] = rng.choice([0.0, round(rng.uniform(0.001, 0.2), 4)])
        case["unlabelled"] = rng.choice([1.0, round(rng.uniform(0.2, 0.95), 3)])
    return case


def _ld(f):
    return (f + 7) // 8 * 8


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, C, dt = case["n"], case["classes"], DTYPES[case["prec"]]
    ld = _ld(C)
    st = dict(case, ld=ld, dt=dt)
    for key in ("temperature", "top_p", "min_p"):   # as the library receives them
        if key in st:
            st[key] = torch.tensor(st[key], dtype=torch.float32).item()
    # a trained network's scores: a normal background (wider for large
    # vocabularies, where most of the mass sits on few classes) and one
    # favoured class a row
    z = torch.randn((n, ld), generator=gen, device=DEV)
    z *= 1.0 + 0.25 * math.log(C)
    lead = torch.randint(0, C, (n, 1), generator=gen, device=DEV)
    z.scatter_add_(1, lead, torch.rand((n, 1), generator=gen, device=DEV) * 4.0)
    st["logits"] = z.to(dt)
    st["overflow"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if case["kind"] == "distill":
        K = case["k"]
        ldt = _ld(K)
        # K different classes a row, the favoured one first; values fall; one
        # row in 16 has fewer entries, one in 64 none (an unsure teacher)
        j = torch.arange(K, device=DEV)
        cls = (lead + j * max(1, C // K)) % C
        drop = torch.rand((n, K), generator=gen, device=DEV)
        val = 8.0 - torch.cumsum(drop * 2.0, 1)
        r = torch.rand((n, 1), generator=gen, device=DEV)
        here = torch.where(r < 1 / 64, 0, torch.where(r < 1 / 16, 1 + K // 2, K))
        cls = torch.where(j < here, cls, -1)
        st["top_values"] = torch.zeros((n, ldt), dtype=dt, device=DEV)
        st["top_values"][:, :K] = val.to(dt)
        st["top_classes"] = torch.full((n, ldt), -1, dtype=torch.int32, device=DEV)
        st["top_classes"][:, :K] = cls.to(torch.int32)
        st["mask"], st["rows"] = None, n
        if case["n_mask"]:
            st["mask"] = torch.zeros(n, dtype=torch.uint8, device=DEV)
            st["mask"][torch.randperm(n, generator=gen, device=DEV)[:case["n_mask"]]] = 1
            st["rows"] = case["n_mask"]
        st["scale"] = torch.full((1,), LOSS_SCALE if case["prec"] == "f16" else 1.0, device=DEV)
        # what gcn_loss left: the cross-entropy's gradient
        st["base"] = None
        if case["base"]:
            b = torch.randn((n, ld), generator=gen, device=DEV)
            st["base"] = (b * (st["scale"] * (0.3 / st["rows"]))).to(dt)
        st["loss"] = torch.zeros(1, device=DEV)
        st["dlogits"] = torch.zeros((n, ld), dtype=dt, device=DEV)
        st["dcol"] = torch.zeros(ld, device=DEV) if case["colsum"] else None
    elif case["kind"] == "top":
        st["values"] = torch.zeros((n, _ld(case["k"])), dtype=dt, device=DEV)
        st["ids"] = torch.zeros((n, _ld(case["k"])), dtype=torch.int32, device=DEV)
    else:
        st["mask"] = None
        if case["unlabelled"] < 1.0:
            st["mask"] = (torch.rand(n, generator=gen, device=DEV) < case["unlabelled"]).to(torch.uint8)
        st["u"] = torch.rand(n, generator=gen, device=DEV)
        st["labels"] = torch.randint(0, C, (n,), generator=gen, device=DEV, dtype=torch.int32)
        st["prob"] = torch.ones(n, device=DEV)
    return st


# ------------------------------------------------------------ plain forms ----

def _sorted(z):
    """Descending, the lower class first among equal values."""
    return torch.sort(z, dim=1, descending=True, stable=True)


def _plain_top(st):
    v, i = _sorted(st["logits"][:, :st["classes"]])
    return {"values": v[:, :st["k"]].clone(), "classes": i[:, :st["k"]].to(torch.int32)}


def _plain_distill(st):
    C, K, T = st["classes"], st["k"], st["temperature"]
    z = st["logits"][:, :C].float()
    x = (z - z.amax(1, keepdim=True)) / T
    e = torch.exp(x)
    s = e.sum(1, keepdim=True)
    cls = st["top_classes"][:, :K].long()
    here = cls >= 0
    t = torch.where(here, st["top_values"][:, :K].float(), -math.inf)
    some = here.any(1, keepdim=True)
    y = (t - torch.where(some, t.amax(1, keepdim=True), 0.0)) / T
    eq = torch.exp(y)
    sq = torch.where(some, eq.sum(1, keepdim=True), 1.0)
    q = eq / sq
    cls = cls.clamp(min=0)
    lnp = torch.gather(x, 1, cls) - torch.log(s)
    kl = torch.where(here, q * (y - torch.log(sq) - lnp), 0.0).sum(1)
    counts = some[:, 0]
    if st["mask"] is not None:
        counts = counts & (st["mask"] != 0)
    loss = (torch.where(counts, kl, 0.0).sum() * (T * T / st["rows"])).reshape(1)
    d = (e / s).scatter_add_(1, cls, -q)
    d = torch.where(counts[:, None], d * (st["scale"] * (T / st["rows"])), 0.0)
    if st["base"] is not None:
        d = d + st["base"][:, :C].float()
    out = {"loss": loss, "dlogits": d.to(st["dt"])}
    if st["colsum"]:
        out["colsum"] = d.sum(0)
    return out


def _plain_sample(st):
    C, T = st["classes"], st["temperature"]
    z = st["logits"][:, :C]
    v, i = _sorted(z)
    x = (v.double() - v[:, :1].double()) / T      # borders between classes need 64 bits
    w = torch.exp(x)
    keep = torch.ones_like(w, dtype=torch.bool)
    if 0 < st["top_k"] < C:
        keep[:, st["top_k"]:] = False
        w = torch.where(keep, w, 0.0)
    if st["top_p"] < 1.0:
        run = torch.cumsum(w, 1)
        keep &= run - w < st["top_p"] * run[:, -1:]
    if st["min_p"] > 0.0:
        keep &= x >= math.log(st["min_p"])
    kept = torch.zeros_like(keep).scatter_(1, i, keep)
    w = torch.where(kept, torch.exp((z.double() - v[:, :1].double()) / T), 0.0)
    run = torch.cumsum(w, 1)
    total = run[:, -1:]
    label = (run <= st["u"][:, None].double() * total).sum(1, keepdim=True)
    prob = (torch.gather(w, 1, label) / total)[:, 0].float()
    label = label[:, 0].to(torch.int32)
    if st["mask"] is not None:
        label = torch.where(st["mask"] != 0, label, st["labels"])
        prob = torch.where(st["mask"] != 0, prob, st["prob"])
    return {"labels": label, "prob": prob}


# ---------------------------------------------------------- library calls ----

def _workspace(st, size, *args):
    """The call's scratch, kept by the program between calls."""
    if "ws" not in st:
        st["ws"] = torch.empty(size(*args), dtype=torch.uint8, device=DEV)
    return st["ws"]


def _own(st):
    from paper_2010_12635_amd import gcn as G
    n, C, ld, prec = st["n"], st["classes"], st["ld"], PREC[st["prec"]]
    if st["kind"] == "top":
        K = st["k"]
        ws = _workspace(st, G.gcn_top_logits_workspace_size, n, C, K, prec)
        G.gcn_top_logits(n, C, ld, prec, st["logits"], K, st["values"].shape[1], st["values"], st["ids"],
                         st["overflow"], ws)
        return {"values": st["values"][:, :K], "classes": st["ids"][:, :K]}
    if st["kind"] == "distill":
        K = st["k"]
        ws = _workspace(st, G.gcn_distill_workspace_size, n, C, K, prec)
        G.gcn_distill(n, C, ld, prec, st["logits"], K, st["top_values"].shape[1], prec, st["top_values"],
                      st["top_classes"], st["mask"], st["rows"], st["temperature"], 1.0, st["scale"], st["base"],
                      st["loss"], st["dlogits"], st["overflow"], ws, dlogits_colsum=st["dcol"])
        out = {"loss": st["loss"], "dlogits": st["dlogits"][:, :C]}
        if st["colsum"]:
            out["colsum"] = st["dcol"][:C]
        return out
    ws = _workspace(st, G.gcn_sample_labels_workspace_size, n, C, prec)
    G.gcn_sample_labels(n, C, ld, prec, st["logits"], st["mask"], st["u"], st["temperature"], st["top_k"],
                        st["top_p"], st["min_p"], st["labels"], st["prob"], st["overflow"], ws)
    return {"labels": st["labels"], "prob": st["prob"]}


def run(state):
    if own:
        return _own(state)
    if state["kind"] == "top":
        return _plain_top(state)
    if state["kind"] == "distill":
        return _plain_distill(state)
    return _plain_sample(state)


def work(case):
    n, C, b = case["n"], case["classes"], BYTES[case["prec"]]
    rows = n * C * b
    if case["kind"] == "top":
        return {"bytes": rows + n * case["k"] * (b + 4), "flops": n * C}
    if case["kind"] == "distill":
        # rows outside the mask need no logits, but every row of the gradient is written
        read = (case["n_mask"] or n) / n
        total = rows * (1 + read + (1 if case["base"] else 0)) + read * n * case["k"] * (b + 4) + n
        return {"bytes": total, "flops": 10 * n * C * read}
    drawn = case["unlabelled"]
    return {"bytes": drawn * (rows + 12 * n) + n, "flops": 8 * n * C * drawn}


# ------------------------------------------------------------------ float64 ----

def _blocks(n, C, per_row):
    """Row ranges of at most about 2^26 numbers of work each."""
    step = max(1, (1 << 26) // max(1, per_row))
    return [(a, min(n, a + step)) for a in range(0, n, step)]


def _exact_distill(st):
    n, C, K, T = st["n"], st["classes"], st["k"], float(st["temperature"])
    logits, base = st["logits"], st["base"]
    grad = torch.empty((n, C), dtype=torch.float64, device=DEV)
    total = torch.zeros((), dtype=torch.float64, device=DEV)
    scale = float(st["scale"].item()) * T / st["rows"]
    for a, b in _blocks(n, C, C):
        lnp = logits[a:b, :C].double() / T
        lnp = lnp - torch.logsumexp(lnp, 1, keepdim=True)
        g = lnp.exp()
        on = torch.ones(b - a, dtype=torch.bool, device=DEV) if st["mask"] is None else st["mask"][a:b] != 0
        c = st["top_classes"][a:b, :K].long()
        t = st["top_values"][a:b, :K].double() / T
        t[c < 0] = -math.inf
        on = on & (c >= 0).any(1)
        t[~on] = 0.0
        lnq = t - torch.logsumexp(t, 1, keepdim=True)
        rows = torch.arange(b - a, device=DEV)
        for k in range(K):
            ok = on & (c[:, k] >= 0)
            r, ck, l = rows[ok], c[ok, k], lnq[ok, k]
            g[r, ck] -= l.exp()
            total += (l.exp() * (l - lnp[r, ck])).sum()
        g *= scale
        g[~on] = 0.0
        if base is not None:
            g += base[a:b, :C].double()
        grad[a:b] = g
    out = {"loss": (total * (T * T / st["rows"])).reshape(1), "dlogits": grad}
    if st["colsum"]:
        out["colsum"] = grad.sum(0)
    return out


def _exact_sample(st):
    """Prefix lengths by counting (narrow rows: every pair of classes
    compared) or by searching sorted sums (wide rows)."""
    n, C, T = st["n"], st["classes"], float(st["temperature"])
    k = st["top_k"] if 0 < st["top_k"] < C else C
    labels = st["labels"].clone()
    prob = st["prob"].double()
    for a, b in _blocks(n, C, C * C if C <= 512 else 4 * C):
        z = st["logits"][a:b, :C].double()
        w = ((z - z.max(1, keepdim=True).values) / T).exp()
        if C <= 512:
            i = torch.arange(C, device=DEV)
            ahead = (z[:, None, :] > z[:, :, None]) | ((z[:, None, :] == z[:, :, None]) & (i[None, :] < i[:, None]))
            rank = ahead.sum(2)
            inside = rank < k
            w_in = torch.where(inside, w, 0.0)
            before = (ahead * w_in[:, None, :]).sum(2)
            if st["top_p"] < 1.0:
                inside &= before < st["top_p"] * w_in.sum(1, keepdim=True)
        else:
            order = torch.argsort(-z, dim=1, stable=True)
            run = torch.gather(w, 1, order)[:, :k].cumsum(1)
            m = torch.full((b - a, 1), k, device=DEV)
            if st["top_p"] < 1.0:
                m = torch.minimum(m, torch.searchsorted(run, st["top_p"] * run[:, -1:].contiguous()) + 1)
            rank = torch.empty_like(order).scatter_(1, order, torch.arange(C, device=DEV).expand_as(order))
            inside = rank < m
        if st["min_p"] > 0.0:
            inside &= w >= st["min_p"]
        w = w * inside
        run = w.cumsum(1)
        at = torch.searchsorted(run, st["u"][a:b, None].double() * run[:, -1:], right=True)
        on = slice(None) if st["mask"] is None else st["mask"][a:b] != 0
        labels[a:b][on] = at[:, 0].to(torch.int32)[on]
        prob[a:b][on] = (torch.gather(w, 1, at) / run[:, -1:])[:, 0][on]
    return {"labels": labels, "prob": prob}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "distill":
        return _exact_distill(st)
    if case["kind"] == "sample":
        return _exact_sample(st)
    # the largest one after the other, each taken out of the row
    z = st["logits"][:, :case["classes"]].double().clone()
    vals, ids = [], []
    for _ in range(case["k"]):
        v = z.max(1, keepdim=True).values
        i = torch.where(z == v, torch.arange(z.shape[1], device=DEV), z.shape[1]).min(1, keepdim=True).values
        vals.append(v)
        ids.append(i)
        z.scatter_(1, i, -math.inf)
    return {"values": torch.cat(vals, 1), "classes": torch.cat(ids, 1).to(torch.int32)}
