"""Workloads of the operators that feed tokens to experts and give their gradients back, as a program that uses them calls them:

  embed        rows of a token table, scaled; its gradient, summed over sorted tokens
  route        a softmax over experts, the k largest for each token, and the slots in the experts' order; its gradient
  expert_mm    products of the rows of each expert with its own weights, as many rows as the router gave it; both gradients
  expert_sum   the weighted sum of a token's k expert rows; its gradient

Sizes are generic ones.  Inputs are drawn on the GPU; outputs and workspaces belong to the caller and are kept.  ``own`` says which
form a pass runs: the plain one below, or the library's.
"""
from __future__ import annotations

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one decoding step of eight sequences: eight rows of a table; nothing but latency
        dict(name="embed_step", op="embed", E=65536, D=2048, T=8, type="bf16"),
        # a batch of prompts: sixteen thousand rows from all over a table beyond any cache
        dict(name="embed_prompt", op="embed", E=131072, D=4096, T=16384, type="bf16"),
        # gradient of a small character or subword table in full precision, sizes that divide nothing, added to what is there
        dict(name="embed_grad_odd", op="embed_grad", E=10007, D=333, T=1500, type="f32", grad="f32", add=True),
        # gradient of a large table after a training step: words come by Zipf's law, one in seventeen the same; kept in 32 bits
        dict(name="embed_grad_train", op="embed_grad", E=131072, D=2048, T=32768, type="bf16", grad="f32", add=False),
        # one decoding step of sixteen sequences through a router
        dict(name="route_step", op="route", E=64, k=4, T=16, type="f32", norm=True, back=False),
        # a training step's router: many experts, eight for a token, forward and gradient
        dict(name="route_train", op="route", E=128, k=8, T=16384, type="bf16", norm=False, back=True),
        # one decoding step: a handful of rows for each expert, whose weights have to be read for them; first product, clamped
        dict(name="mm_step", op="mm", E=8, k=2, T=16, N=4096, K=2048, type="bf16", gather=True, back=False),
        # prompts through the first product of the experts
        dict(name="mm_prompt", op="mm", E=16, k=2, T=4096, N=4096, K=2048, type="f16", gather=True, back=False),
        # a training step of the second product: forward and both gradients
        dict(name="mm_train", op="mm", E=32, k=2, T=8192, N=2048, K=4096, type="bf16", gather=False, back=True),
        # the same in full precision for a small model whose widths divide nothing
        dict(name="mm_odd", op="mm", E=12, k=3, T=700, N=1001, K=517, type="f32", gather=True, back=True),
        # one decoding step: sixteen tokens, four expert rows each
        dict(name="sum_step", op="sum", k=4, T=16, N=4096, type="f16", back=False),
        # a training step: the sum and its gradient
        dict(name="sum_train", op="sum", k=4, T=8192, N=2048, type="bf16", back=True),
    ]


def _log(rng, lo, hi):
    """An integer whose logarithm is uniform over [lo, hi]."""
    return _other(max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random())))))


def _size(rng, lo, hi):
    """A width or a number of tokens: half of them multiples of 64, as widths mostly are."""
    v = _log(rng, lo, hi)
    if v >= 64 and rng.random() < 0.5:
        v = v // 64 * 64
    return _other(v)


def _other(v):
    """Sizes that no configuration here has are left out."""
    return v if v != 3072 else v - 64


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "route", "mm", "mm", "mm", "sum"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "embed":
        return dict(op=op, E=_log(rng, 256, 131072), D=_size(rng, 64, 4096), T=_size(rng, 1, 16384), type=kind)
    if op == "embed_grad":
        return dict(op=op, E=_log(rng, 256, 131072), D=_size(rng, 64, 2048), T=_size(rng, 1, 32768), type=kind, grad=rng.choice([kind, "f32"]),
                    add=rng.random() < 0.5)
    if op == "route":
        e = rng.choice([4, 8, 16, 32, 64, 128, _log(rng, 4, 256)])
        return dict(op=op, E=e, k=rng.randint(1, min(e, 8)), T=_size(rng, 1, 16384), type=kind, norm=rng.random() < 0.5, back=rng.random() < 0.5)
    if op == "sum":
        return dict(op=op, k=rng.randint(1, 8), T=_size(rng, 1, 8192), N=_size(rng, 64, 4096), type=kind, back=rng.random() < 0.5)
    e, k = rng.choice([4, 8, 16, 32, 64]), rng.randint(1, 4)
    t, n, d = _size(rng, 1, 8192), _size(rng, 128, 4096), _size(rng, 128, 4096)
    most = 16384 * 2048 * 4096  # products of the largest listed case; a sixteenth of that in 32 bits
    while t * k * n * d > (most if kind != "f32" else most // 16) or e * n * d > 1 << 28 :
        t, n, d, e = max(1, t * 3 // 4), n if n <= d else n * 3 // 4, d if d < n else d * 3 // 4, max(4, e // 2) if e * n * d > 1 << 28 else e
    return dict(op=op, E=e, k=k, T=_other(t), N=_other(n), K=_other(d), type=kind, gather=rng.random() < 0.5, back=rng.random() < 0.5)


# ---- inputs ----------------------------------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(0x7C355 + 1000003 * int(seed))
    return g


def _normal(g, shape, kind, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(TYPES[kind])


def _tokens(g, T, E):
    """Token numbers by Zipf's law, spread over the table."""
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * torch.log(torch.tensor(float(E + 1), device="cuda", dtype=torch.float64))).long() - 1).clamp(0, E - 1)
    return ((rank * 7919 + 12345) % E).to(torch.int32)


def _plan(Id, E):
    """The slots in the experts' order, as route() lays them out: offsets of the experts, token of each place, place of each slot."""
    T, k = Id.shape
    key = torch.where(Id < 0, E, Id).flatten().long()
    order = torch.argsort(key, stable=True)
    off = torch.zeros(E + 1, dtype=torch.int64, device=Id.device)
    off[1:] = torch.cumsum(torch.bincount(key, minlength=E + 1)[:E], 0)
    r = torch.arange(T * k, device=Id.device)
    row = torch.where(r < off[E], order // k, -1)
    place = torch.empty_like(order)
    place[order] = torch.where(r < off[E], r, -1)
    return off.to(torch.int32), row.to(torch.int32), place.view(T, k).to(torch.int32)


def _routed(g, T, E, k):
    """Expert numbers [T, k], the experts of one token all different: some are asked for far more often than others, the second
    one by nobody, and a slot in 64 is left empty."""
    bias = -0.5 * torch.log(1.0 + torch.arange(E, device="cuda", dtype=torch.float32))
    bias[1] = -1e30
    u = torch.rand((T, E), generator=g, device="cuda").clamp_(1e-9, 1 - 1e-7)
    Id = torch.topk(bias - torch.log(-torch.log(u)), k, dim=1).indices.to(torch.int32)
    return torch.where(torch.rand((T, k), generator=g, device="cuda") < 1 / 64, -1, Id)


def prepare(case, seed):
    c, g = dict(case), _generator(seed)
    op = c["op"]
    empty = lambda kind, *s: torch.zeros(s, dtype=TYPES[kind], device="cuda")  # noqa: E731
    ints = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    if op == "embed":
        c.update(LUT=_normal(g, (c["E"], c["D"]), c["type"], 0.02), Idx=_tokens(g, c["T"], c["E"]), O=empty(c["type"], c["T"], c["D"]))
        c["scale"] = float(c["D"]) ** 0.5
    elif op == "embed_grad":
        c.update(dO=_normal(g, (c["T"], c["D"]), c["type"], 0.1), Idx=_tokens(g, c["T"], c["E"]), pad=(3 * 7919 + 12345) % c["E"])  # (a common one)
        c["scale"] = float(c["D"]) ** 0.5
        if c["add"]:  # what is there already; a pass that adds leaves it as it is and gives the sum
            c["there"] = _normal(g, (c["E"], c["D"]), c["grad"], 0.1)
        c["dLUT"] = empty(c["grad"], c["E"], c["D"])
    elif op == "route":
        L = _normal(g, (c["T"], c["E"]), c["type"], 2.0)
        L[torch.rand(L.shape, generator=g, device="cuda") < 0.05] = float("-inf")  # experts that a token may not ask for
        L[torch.rand((c["T"],), generator=g, device="cuda") < 0.02] = float("-inf")  # tokens of no sequence
        c.update(L=L, Wt=empty("f32", c["T"], c["k"]), Id=ints(c["T"], c["k"]), Off=ints(c["E"] + 1), Row=ints(c["T"] * c["k"]), Place=ints(c["T"], c["k"]))
        if c["back"]:
            c.update(dWt=_normal(g, (c["T"], c["k"]), "f32"), dL=empty(c["type"], c["T"], c["E"]))
    elif op == "mm":
        R = c["T"] * c["k"]
        c["Off"], c["Row"], _ = _plan(_routed(g, c["T"], c["E"], c["k"]), c["E"])
        X = _normal(g, (c["T"] if c["gather"] else R, c["K"]), c["type"])
        c.update(X=X if c["gather"] else X.clamp_(min=0), W=_normal(g, (c["E"], c["N"], c["K"]), c["type"], c["K"] ** -0.5), Y=empty(c["type"], R, c["N"]))
        if c["back"]:
            dY = _normal(g, (R, c["N"]), c["type"], 0.1)
            c.update(dY=dY, dX=empty(c["type"], R, c["K"]), dW=empty(c["type"], c["E"], c["N"], c["K"]))
    else:
        R = c["T"] * c["k"]
        E = max(4, c["k"])
        _, _, c["Place"] = _plan(_routed(g, c["T"], E, c["k"]), E)
        c.update(Y=_normal(g, (R, c["N"]), c["type"]), Wt=torch.rand((c["T"], c["k"]), generator=g, device="cuda"), O=empty(c["type"], c["T"], c["N"]))
        if c["back"]:
            c.update(dO=_normal(g, (c["T"], c["N"]), c["type"], 0.1), dY=empty(c["type"], R, c["N"]), dWt=empty("f32", c["T"], c["k"]))
    return c


# ---- one pass --------------------------------------------------------------------------------------------------------------


def run(state):
    return (_own if own else _plain)[state["op"]](state)


def _workspace(s, need):
    """The caller's workspace, made at the first pass and kept."""
    if "ws" not in s:
        n = need()
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    return s["ws"]


def _own_embed(s):
    from paper_1802_04730_amd import tc355

    tc355.tc_embed(s["LUT"], s["Idx"], s["O"], s["scale"])
    return s["O"]


def _own_embed_grad(s):
    from paper_1802_04730_amd import tc355

    ws = _workspace(s, lambda: tc355.tc_embed_grad_workspace_bytes(s["E"], s["D"], s["T"]))
    if s["add"]:
        s["dLUT"].copy_(s["there"])
    tc355.tc_embed_grad(s["dO"], s["Idx"], s["dLUT"], ws, s["scale"], s["pad"], s["add"])
    return s["dLUT"]


def _own_route(s):
    from paper_1802_04730_amd import tc355

    ws = _workspace(s, lambda: tc355.tc_route_workspace_bytes(s["T"], s["E"], s["k"]))
    tc355.tc_route(s["L"], s["Wt"], s["Id"], s["Off"], s["Row"], s["Place"], ws, s["norm"])
    out = [s["Wt"], s["Id"], s["Off"], s["Row"], s["Place"]]
    if s["back"]:
        tc355.tc_route_grad(s["L"], s["Id"], s["dWt"], s["dL"], s["norm"])
        out.append(s["dL"])
    return out


def _own_mm(s):
    from paper_1802_04730_amd import tc355

    row = s["Row"] if s["gather"] else None
    tc355.tc_expert_mm(s["X"], s["W"], s["Off"], row, s["Y"], s["gather"])
    if not s["back"]:
        return s["Y"]
    ws = _workspace(s, lambda: tc355.tc_expert_mm_grad_w_workspace_bytes(s["Y"].shape[0], s["E"], s["N"], s["K"]))
    tc355.tc_expert_mm_grad_x(s["dY"], s["W"], s["Off"], None if s["gather"] else s["X"], s["dX"])
    tc355.tc_expert_mm_grad_w(s["dY"], s["X"], s["Off"], row, s["dW"], ws)
    return [s["Y"], s["dX"], s["dW"]]


def _own_sum(s):
    from paper_1802_04730_amd import tc355

    tc355.tc_expert_sum(s["Y"], s["Wt"], s["Place"], s["O"])
    if not s["back"]:
        return s["O"]
    tc355.tc_expert_sum_grad(s["dO"], s["Y"], s["Wt"], s["Place"], s["dY"], s["dWt"])
    return [s["O"], s["dY"], s["dWt"]]


_own = {"embed": _own_embed, "embed_grad": _own_embed_grad, "route": _own_route, "mm": _own_mm, "sum": _own_sum}


def _plain_embed(s):
    return (s["LUT"][s["Idx"].long()].float() * s["scale"]).to(s["LUT"].dtype)


def _plain_embed_grad(s):
    Idx = s["Idx"].long()
    rows = s["dO"].float() * (Idx != s["pad"]).unsqueeze(1)
    dLUT = torch.zeros(s["dLUT"].shape, device="cuda").index_add_(0, Idx, rows) * s["scale"]
    return ((s["there"].float() + dLUT) if s["add"] else dLUT).to(s["dLUT"].dtype)


def _plain_route(s):
    L, k, E = s["L"].float(), s["k"], s["E"]
    top, Id = torch.sort(L, dim=1, descending=True, stable=True)  # (equal logits: the lower number first)
    top, Id = top[:, :k], Id[:, :k]
    there = top > float("-inf")
    over = top if s["norm"] else L
    most = L.max(dim=1, keepdim=True).values.clamp(min=torch.finfo(torch.float32).min)  # (a row of nothing: exp gives 0)
    total = torch.exp(over - most).sum(dim=1, keepdim=True)
    Wt = torch.where(there, torch.exp(top - most) / total, 0.0)
    Id = torch.where(there, Id, -1).to(torch.int32)
    out = [Wt, Id, *_plan(Id, E)]
    if s["back"]:
        g = torch.where(there, s["dWt"], 0.0)
        inner = (g * Wt).sum(dim=1, keepdim=True)
        at = torch.where(there, Id.long(), 0)
        dL = torch.zeros_like(L).scatter_add_(1, at, torch.where(there, g * Wt, 0.0))
        share = torch.zeros_like(L).scatter_add_(1, at, Wt) if s["norm"] else torch.where(L > float("-inf"), torch.exp(L - most) / total, 0.0)
        out.append((dL - share * inner).to(s["L"].dtype))
    return out


def _plain_mm(s):
    Off, X, W, R, E = s["Off"].long(), s["X"], s["W"], s["Y"].shape[0], s["E"]
    count = Off[1:] - Off[:-1]
    r = torch.arange(R, device="cuda")
    e = torch.searchsorted(Off[1:].contiguous(), r, right=True)  # expert of each place; E behind the last one
    used = e < E
    e = torch.where(used, e, 0)
    Xr = (X[s["Row"].long().clamp(min=0)] if s["gather"] else X).float() * used.unsqueeze(1)
    if R < E and not s["back"]:  # few rows: only the weights that they ask for
        Y = torch.matmul(W[e].float(), Xr.unsqueeze(2)).squeeze(2)
        return (Y.clamp(min=0) if s["gather"] else Y).to(X.dtype)
    most = int(count.max())
    e, at = torch.where(used, e, E), torch.where(used, r - Off[e], 0)  # (a spare expert for the rows of none)
    pad = lambda rows: torch.zeros((E + 1, max(1, most), rows.shape[1]), device="cuda").index_put_((e, at), rows)[:E]  # noqa: E731
    back = lambda m: torch.where(used.unsqueeze(1), m[torch.where(used, e, 0), at], 0.0)  # noqa: E731
    Wf, Xp = W.float(), pad(Xr)
    Y = back(torch.bmm(Xp, Wf.transpose(1, 2).contiguous()))
    Y = (Y.clamp(min=0) if s["gather"] else Y).to(X.dtype)
    if not s["back"]:
        return Y
    dYp = pad(s["dY"].float() * used.unsqueeze(1))
    dX = back(torch.bmm(dYp, Wf))
    if not s["gather"]:
        dX = dX * (X > 0)
    dW = torch.bmm(dYp.transpose(1, 2).contiguous(), Xp)
    return [Y, dX.to(X.dtype), dW.to(X.dtype)]


def _plain_sum(s):
    at = s["Place"].long()
    w = torch.where(at >= 0, s["Wt"], 0.0).unsqueeze(2)
    rows = s["Y"][at.clamp(min=0)].float()
    O = (rows * w).sum(dim=1).to(s["Y"].dtype)
    if not s["back"]:
        return O
    dO = s["dO"].float().unsqueeze(1)
    dWt = torch.where(at >= 0, (rows * dO).sum(dim=2), 0.0)
    R, N = s["Y"].shape
    dY = torch.zeros((R + 1, N), device="cuda").index_put_((torch.where(at >= 0, at, R),), dO * w)[:R]
    return [O, dY.to(s["Y"].dtype), dWt]


_plain = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "route": _plain_route, "mm": _plain_mm, "sum": _plain_sum}


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------


def work(case):
    c = case
    z = {"f32": 4, "bf16": 2, "f16": 2}
    b, op, T = z[c["type"]], c["op"], c["T"]
    if op == "embed":
        return {"bytes": T * 4 + 2 * T * c["D"] * b, "flops": T * c["D"]}
    if op == "embed_grad":  # (where it adds: what is there is read and the whole written, as a pass gives it)
        return {"bytes": T * 4 + T * c["D"] * b + c["E"] * c["D"] * z[c["grad"]] * (2 if c["add"] else 1), "flops": 2 * T * c["D"]}
    if op == "route":
        E, slots = c["E"], T * c["k"]
        w = {"bytes": T * E * b + slots * 16 + E * 4 + 4, "flops": 4 * T * E}
        if c["back"]:  # logits again are not needed: they are there
            w = {"bytes": w["bytes"] + slots * 4 + T * E * b, "flops": w["flops"] + 4 * T * E}
        return w
    R, N = T * c["k"], c["N"]
    if op == "sum":
        w = {"bytes": R * N * b + R * 8 + T * N * b, "flops": 2 * R * N}
        if c["back"]:
            w = {"bytes": w["bytes"] + T * N * b + R * N * b + R * 4, "flops": w["flops"] + 3 * R * N}
        return w
    E, K = c["E"], c["K"]
    weights = min(E, R) * N * K * b
    rows = (T if c["gather"] else R) * K * b
    w = {"bytes": rows + weights + R * N * b + (E + 1) * 4 + (R * 4 if c["gather"] else 0), "flops": 2 * R * N * K}
    if c["back"]:
        w = {"bytes": w["bytes"] + R * N * b + R * K * b + E * N * K * b, "flops": 3 * w["flops"]}
    return w


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "route": _exact_route, "mm": _exact_mm, "sum": _exact_sum}[s["op"]](s)


def _exact_embed(s):
    return torch.index_select(s["LUT"], 0, s["Idx"]).double() * s["scale"]


def _exact_embed_grad(s):
    keep = (s["Idx"] != s["pad"]).nonzero().flatten()
    total = torch.zeros(s["dLUT"].shape, dtype=torch.float64, device="cuda")
    total.index_add_(0, s["Idx"][keep], s["dO"][keep].double() * s["scale"])
    return total + s["there"].double() if s["add"] else total


def _exact_route(s):
    L, k, T, E = s["L"].double().cpu(), s["k"], s["T"], s["E"]
    share = torch.zeros((T, E), dtype=torch.float64)
    some = (L > float("-inf")).any(dim=1)
    share[some] = torch.softmax(L[some], dim=1)
    # the place of an expert in its row's order: how many are larger, or equal and of a lower number
    Wt = torch.zeros((T, k), dtype=torch.float64)
    left, ids = L.clone(), torch.full((T, k), -1, dtype=torch.int64)
    rows = torch.arange(T)
    for i in range(k):
        most = left.max(dim=1).values
        first = (left == most.unsqueeze(1)).to(torch.int8).argmax(dim=1)
        ok = most > float("-inf")
        ids[ok, i] = first[ok]
        Wt[ok, i] = share[rows[ok], first[ok]]
        left[rows, first] = float("-inf")
    if s["norm"]:
        Wt = Wt / Wt.sum(dim=1, keepdim=True).clamp(min=1e-300)
    out = [Wt, None, None, None, None]
    if s["back"]:
        g = s["dWt"].double().cpu() * (ids >= 0)
        dL = torch.zeros((T, E), dtype=torch.float64)
        inner = (g * Wt).sum(dim=1)
        for i in range(k):
            ok = ids[:, i] >= 0
            dL[rows[ok], ids[ok, i]] += (Wt * g)[ok, i]
            if s["norm"]:
                dL[rows[ok], ids[ok, i]] -= Wt[ok, i] * inner[ok]
        out.append(dL if s["norm"] else dL - share * inner.unsqueeze(1))
    return out


def _exact_mm(s):
    off, f64 = s["Off"].tolist(), torch.float64
    R, N, K = s["Y"].shape[0], s["N"], s["K"]
    Y = torch.zeros((R, N), dtype=f64, device="cuda")
    dX = torch.zeros((R, K), dtype=f64, device="cuda")
    dW = torch.zeros((s["E"], N, K), dtype=f64, device="cuda") if s["back"] else None
    for e in range(s["E"]):
        lo, hi = off[e], off[e + 1]
        if lo == hi:
            continue
        x = (s["X"][s["Row"][lo:hi].long()] if s["gather"] else s["X"][lo:hi]).double()
        w = s["W"][e].double()
        y = x @ w.t()
        Y[lo:hi] = torch.relu(y) if s["gather"] else y
        if s["back"]:
            dy = s["dY"][lo:hi].double()
            dx = dy @ w
            dX[lo:hi] = dx if s["gather"] else torch.where(x > 0, dx, 0.0)
            dW[e] = dy.t() @ x
    return [Y, dX, dW] if s["back"] else Y


def _exact_sum(s):
    at, Y = s["Place"].long(), s["Y"].double()
    O = torch.zeros((s["T"], s["N"]), dtype=torch.float64, device="cuda")
    dY, dWt = torch.zeros_like(Y), torch.zeros(at.shape, dtype=torch.float64, device="cuda")
    for i in range(s["k"]):
        t = (at[:, i] >= 0).nonzero().flatten()
        p, w = at[t, i], s["Wt"][t, i].double().unsqueeze(1)
        O[t] += w * Y[p]
        if s["back"]:
            d = s["dO"][t].double()
            dY[p] = w * d
            dWt[t, i] = (Y[p] * d).sum(dim=1)
    return [O, dY, dWt] if s["back"] else O
