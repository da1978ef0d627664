"""Performance cases of the operators of a decoder layer whose MLP is a mixture of experts or has 4-bit weights.

Five operators, as such a layer uses them one after the other: the router's choice of experts for each token, with the order in
which the experts' products take the tokens; matrix products grouped by expert (with and without the gated activation); the
weighted sum of a token's experts; matrix products of few rows on 4-bit weights with a scale per group; and what joins one block
to the next: the norm behind a block, its gate, the scaled residual and the norm ahead of the next block.

Shapes are those of the layers that the tests and the benchmark use -- hidden 4096 with an MLP of 12288 or 14336 channels, leaf
256; hidden 5120, leaf 128 -- and generic experts of 768 to 14336 channels, 8 to 128 of them.  Batches go from one token to a
prefill and are ragged, as batches of requests are; experts are chosen unevenly, so some get many rows and some none.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6

# (experts, K, columns, leaf, k_first): first product of the experts (columns: channels of the activation), second product
EXPERTS_UP = [(64, 4096, 2048, 256, 1), (16, 4096, 2048, 256, 1), (32, 2048, 1024, 256, 1), (128, 2048, 768, 256, 1),
              (32, 5120, 1280, 128, 5), (8, 4096, 14336, 256, 1)]
EXPERTS_DOWN = [(64, 2048, 4096, 256, 1), (16, 2048, 4096, 256, 1), (32, 1024, 2048, 128, 1), (128, 768, 2048, 64, 3),
                (32, 1280, 5120, 64, 5), (8, 14336, 4096, 256, 7)]
# (K, N, leaf, k_first) of products on 4-bit weights
GEMMS_4 = [(4096, 4096, 256, 1), (12288, 4096, 256, 3), (14336, 4096, 256, 7), (4096, 6144, 256, 1), (4096, 12288, 256, 1),
           (5120, 5120, 128, 5), (5120, 7168, 128, 5)]


def listed():
    return [
        # The router of one decoded token: latency of the smallest call.
        dict(name="route_one_token", kind="route", dtype="fp32", T=1, E=128, k=8, renormalize=True),
        # The router of a long prefill, logits as a 16-bit product leaves them (with ties).
        dict(name="route_prefill", kind="route", dtype="bf16", T=8191, E=128, k=8, renormalize=True),
        # The experts' first product with its activation, a decode batch of four: most of 64 experts are not touched.
        dict(name="experts_up_decode", kind="grouped", form="swiglu", dtype="bf16", T=4, k=4, E=64, K=4096, N=2048, leaf=256, k_first=1),
        # The same product of a ragged prefill over 16 experts.
        dict(name="experts_up_prefill", kind="grouped", form="swiglu", dtype="bf16", T=1500, k=4, E=16, K=4096, N=2048, leaf=256, k_first=1),
        # The experts' second product of one token, narrow experts: latency.
        dict(name="experts_down_one_token", kind="grouped", form="same", dtype="fp16", T=1, k=8, E=128, K=768, N=2048, leaf=64, k_first=3),
        # The second product of a full prefill, 64 experts, about 500 rows each.
        dict(name="experts_down_prefill", kind="grouped", form="same", dtype="bf16", T=4096, k=8, E=64, K=2048, N=4096, leaf=256, k_first=1),
        # The weighted sum of the experts of a decode batch of odd size, onto the residual stream.
        dict(name="sum_decode", kind="sum", dtype="bf16", T=77, k=8, E=64, H=4096, P=0, residual=True),
        # The same for a prefill whose experts' second product is split over four shards: fp32 partial sums.
        dict(name="sum_prefill_tp4", kind="sum", dtype="bf16", T=1003, k=8, E=64, H=4096, P=4, residual=True),
        # One token through a gate/up-sized layer in 4 bits.
        dict(name="w4_one_token", kind="w4", dtype="bf16", M=1, K=4096, N=12288, leaf=256, k_first=1, group=128, zeros=False),
        # A decode batch of odd size through down_proj in 4 bits with zero points.
        dict(name="w4_batch", kind="w4", dtype="fp16", M=27, K=12288, N=4096, leaf=256, k_first=3, group=64, zeros=True),
        # Between the blocks of one decoded token: a gate per channel.
        dict(name="join_one_token", kind="join", dtype="bf16", M=1, H=4096, P=0, gate="channel", scale=1.0),
        # Between the blocks of a long prefill, 32B-class hidden size: a gate per token, the residual scaled.
        dict(name="join_prefill", kind="join", dtype="bf16", M=8191, H=5120, P=0, gate="row", scale=0.75),
    ]


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]; odd values as likely as even ones."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw_once(rng):
    kind = rng.choice(["route", "grouped", "grouped", "grouped", "sum", "w4", "w4", "join"])
    dt = rng.choice(["bf16", "bf16", "fp16"])
    if kind == "route":
        E = rng.choice([8, 16, 32, 64, 128, 256, _log_int(rng, 4, 512)])
        return dict(kind=kind, dtype=rng.choice(["fp32", "fp32", dt]), T=_log_int(rng, 1, 16384), E=E, k=rng.randint(1, min(10, E)),
                    renormalize=rng.random() < 0.7)
    if kind == "grouped":
        form = rng.choice(["swiglu", "swiglu", "same", "same", "fp32"])
        E, K, N, leaf, kf = rng.choice(EXPERTS_UP if form == "swiglu" else EXPERTS_DOWN)
        return dict(kind=kind, form=form, dtype=dt, T=_log_int(rng, 1, 4096), k=rng.choice([1, 2, 4, 6, 8]), E=E, K=K, N=N, leaf=leaf, k_first=kf)
    if kind == "sum":
        return dict(kind=kind, dtype=dt, T=_log_int(rng, 1, 4096), k=rng.choice([1, 2, 4, 6, 8]), E=64,
                    H=rng.choice([2048, 4096, 5120, 8 * _log_int(rng, 16, 1000)]), P=rng.choice([0, 0, 1, 2, 4, 8]), residual=rng.random() < 0.7)
    if kind == "w4":
        K, N, leaf, kf = rng.choice(GEMMS_4)
        return dict(kind=kind, dtype=dt, M=_log_int(rng, 1, 256), K=K, N=N, leaf=leaf, k_first=kf, group=rng.choice([32, 64, 128]),
                    zeros=rng.random() < 0.5)
    return dict(kind=kind, dtype=dt, M=_log_int(rng, 1, 8192), H=rng.choice([2048, 4096, 5120, 8 * _log_int(rng, 16, 2000)]),
                P=rng.choice([0, 0, 0, 1, 2, 4]), gate=rng.choice(["none", "channel", "row", "full"]), scale=rng.choice([1.0, 0.5, 0.75]))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw_once(rng)
        if _cost(case) <= most:
            return case


def work(case):
    """What a pass cannot do without: each input read once, each output written once; the products' operations."""
    k = case["kind"]
    size = 4 if case["dtype"] == "fp32" else 2
    if k == "route":
        return {"bytes": case["T"] * (case["E"] * size + 16 * case["k"]) + 4 * (case["E"] + 1), "flops": 0}
    if k == "grouped":
        T, E, K, N = case["T"], case["E"], case["K"], case["N"]
        R, columns = T * case["k"], N * (2 if case["form"] == "swiglu" else 1)
        touched = E * (1.0 - (1.0 - case["k"] / E) ** T)                # experts that an even choice touches
        return {"bytes": 2 * (T if case["form"] == "swiglu" else R) * K + 2 * touched * K * columns + R * N * (4 if case["form"] == "fp32" else 2) + 4 * R,
                "flops": 2 * R * K * columns}
    if k == "sum":
        T, H = case["T"], case["H"]
        rows = T * case["k"] * H * (4 * case["P"] if case["P"] else 2)
        return {"bytes": rows + T * H * (4 if case["residual"] else 2) + 8 * T * case["k"], "flops": 0}
    M = case["M"]
    if k == "w4":
        K, N, G = case["K"], case["N"], case["group"]
        return {"bytes": 2 * M * (K + N) + N * K / 2 + N * (K // G) * (3 if case["zeros"] else 2), "flops": 2 * M * N * K}
    H = case["H"]
    gate = {"none": 0, "channel": H, "row": M, "full": M * H}[case["gate"]]
    return {"bytes": M * H * ((4 * case["P"] if case["P"] else 2) + 6) + 4 * H + 2 * gate, "flops": 0}


# ---- inputs ----

def _rows(randn, M, n, dtype):
    """Rows of a residual stream: N(0, 1) with a few channels that are far larger, as trained models have them."""
    x = randn(M, n)
    x[:, :: max(1, n // 5)] *= 12.0
    return x.to(dtype)


def _order(experts, E):
    """Where the experts' products take their rows from: (token of each row in the order of the experts, first row of each
    expert, row of each choice).  A token's choices of an expert keep the order of the tokens."""
    T, k = experts.shape
    flat = experts.reshape(-1).long()
    order = torch.sort(flat, stable=True).indices
    ends = (flat[:, None] == torch.arange(E, device=flat.device)).sum(dim=0).cumsum(dim=0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    slots = torch.empty_like(order)
    slots[order] = torch.arange(T * k, device=flat.device)
    return (order // k).int(), offsets.int(), slots.reshape(T, k).int()


def _first_k(logits, k):
    """The k largest of each row in falling order, the lower index first among equals."""
    values, index = torch.sort(logits, dim=1, descending=True, stable=True)
    return values[:, :k], index[:, :k]


def _logits(randn, T, E):
    return 1.5 * randn(T, E) + randn(E)                                 # some experts are chosen far more often than others


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    k, dt = case["kind"], TYPES[case["dtype"]]
    s = dict(case=case)
    if k == "route":
        s["logits"] = _logits(randn, case["T"], case["E"]).to(dt)
        return s
    if k in ("grouped", "sum"):
        T, E = case["T"], case["E"]
        values, experts = _first_k(_logits(randn, T, E), case["k"])
        rows, s["offsets"], slots = _order(experts, E)
        R = T * case["k"]
        if k == "sum":
            H, P = case["H"], case["P"]
            s["slots"], s["weights"] = slots, torch.softmax(values, dim=1)
            s["y"] = (0.6 * randn(P, R, H)) if P else randn(R, H).to(dt)
            s["residual"] = _rows(randn, T, H, dt) if case["residual"] else None
            return s
        ends = s["offsets"].tolist()                                    # the plain form's loop; the framework's calls do not need it
        s["spans"] = [(e, ends[e], ends[e + 1]) for e in range(E) if ends[e + 1] > ends[e]]
        K, up = case["K"], case["form"] == "swiglu"
        s["rows"] = rows if up else None                                # the first product gathers tokens, the second has its rows in order
        s["X"] = randn(T if up else R, K).to(dt)
        s["W"] = torch.empty(E, K, case["N"] * (2 if up else 1), dtype=dt, device=DEV)
        for e in range(E):
            s["W"][e] = 0.02 * randn(*s["W"].shape[1:])
        return s
    if k == "w4":
        M, K, N, G = case["M"], case["K"], case["N"], case["group"]
        s["X"] = _rows(randn, M, K, dt)
        levels = (2.2 * randn(N, K) + 8).round().clamp(0, 15).to(torch.uint8)
        s["Wq"] = levels[:, 0::2] | (levels[:, 1::2] << 4)
        s["scales"] = (0.009 * torch.exp(0.3 * randn(N, K // G))).to(dt)
        s["zeros"] = (randn(N, K // G) + 8).round().clamp(0, 15).to(torch.uint8) if case["zeros"] else None
        return s
    M, H, P = case["M"], case["H"], case["P"]
    s["y"] = (0.6 * randn(P, M, H)) if P else _rows(randn, M, H, dt)
    s["residual"] = _rows(randn, M, H, dt)
    s["post_weight"], s["next_weight"] = (1 + 0.1 * randn(H)).to(dt), (1 + 0.1 * randn(H)).to(dt)
    shape = {"none": None, "channel": (H,), "row": (M, 1), "full": (M, H)}[case["gate"]]
    s["gate"] = None if shape is None else torch.sigmoid(randn(*shape)).to(dt)
    return s


# ---- the operators in plain form ----

def _plain_route(s, case):
    logits, k = s["logits"].float(), case["k"]
    values, experts = _first_k(logits, k)
    w = torch.exp(values - values[:, :1])
    over = w if case["renormalize"] else torch.exp(logits - values[:, :1])
    rows, offsets, slots = _order(experts, case["E"])
    return experts.int(), w / over.sum(dim=1, keepdim=True), offsets, rows, slots


def _plain_grouped(s, case):
    """A product for each expert that has rows.  With the activation: gate and up are 16-bit tensors by the operator's definition
    (it gives what two products and the activation between them give)."""
    dt, up = TYPES[case["dtype"]], case["form"] == "swiglu"
    X = s["X"] if s["rows"] is None else s["X"][s["rows"].long()]
    y = torch.cat([X[lo:hi].float() @ s["W"][e].float() for e, lo, hi in s["spans"]])
    if case["form"] == "fp32":
        return y
    if up:
        gate, up = y.to(dt).float().chunk(2, dim=1)
        y = gate / (1.0 + torch.exp(-gate)) * up
    return y.to(dt)


def _plain_sum(s, case):
    y = s["y"].sum(dim=0) if case["P"] else s["y"].float()
    y = (y[s["slots"].long()] * s["weights"][:, :, None]).sum(dim=1)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(TYPES[case["dtype"]])


def _levels(s):
    """The 4-bit elements [N, K]: the element with the even k in the low half of its byte."""
    q = s["Wq"]
    return torch.stack([q & 15, q >> 4], dim=2).reshape(q.shape[0], -1)


def _plain_w4(s, case):
    q = _levels(s).float().reshape(case["N"], -1, case["group"])
    zeros = 8.0 if s["zeros"] is None else s["zeros"].float()[:, :, None]
    W = ((q - zeros) * s["scales"].float()[:, :, None]).reshape(case["N"], case["K"])
    return (s["X"].float() @ W.t()).to(TYPES[case["dtype"]])


def _plain_norm(x, weight):
    return x * (1.0 / torch.sqrt(x.square().mean(dim=1, keepdim=True) + EPS)) * weight.float()


def _plain_join(s, case):
    dt = TYPES[case["dtype"]]
    y = s["y"].sum(dim=0).to(dt).float() if case["P"] else s["y"].float()        # the block's output is a 16-bit tensor
    n = _plain_norm(y, s["post_weight"])
    if s["gate"] is not None:
        n = n * s["gate"].float()
    hidden = (s["residual"].float() * case["scale"] + n).to(dt)
    return hidden, _plain_norm(hidden.float(), s["next_weight"]).to(dt)


# ---- the framework's calls ----

def _own(s, case):
    from paper_2511_17826_amd import binding as tb
    k = case["kind"]
    if k == "route":
        return tb.tbik_route_topk(s["logits"], case["k"], renormalize=case["renormalize"])
    if k == "grouped":
        if case["form"] == "swiglu":
            return tb.tbik_gemm_grouped_swiglu(s["X"], s["W"], s["offsets"], case["leaf"], case["k_first"], rows=s["rows"])
        return tb.tbik_gemm_grouped(s["X"], s["W"], s["offsets"], case["leaf"], case["k_first"], rows=s["rows"],
                                    out_dtype=torch.float32 if case["form"] == "fp32" else TYPES[case["dtype"]])
    if k == "sum":
        return tb.tbik_combine_experts(s["y"], s["slots"], s["weights"], residual=s["residual"], out_dtype=TYPES[case["dtype"]])
    if k == "w4":
        return tb.tbik_gemm_w4(s["X"], s["Wq"], s["scales"], case["leaf"], case["k_first"], zeros=s["zeros"])
    return tb.tbik_rmsnorm_residual_rmsnorm(s["y"], s["residual"], s["post_weight"], s["next_weight"], EPS,
                                            residual_scale=case["scale"], gate=s["gate"])


def run(state):
    s, case = state, state["case"]
    if own:
        return _own(s, case)
    return {"route": _plain_route, "grouped": _plain_grouped, "sum": _plain_sum, "w4": _plain_w4, "join": _plain_join}[case["kind"]](s, case)


# ---- the operators' definitions in 64 bits ----

def _on_grid(v, fraction_bits, lowest):
    """The nearest number with this many fraction bits and exponents from `lowest` on, ties to even."""
    step = torch.exp2(((torch.frexp(v).exponent - 1).clamp(min=lowest) - fraction_bits).double())
    return torch.round(v / step) * step


def _exact_16(v, dtype):
    return _on_grid(v, 7, -126) if dtype == "bf16" else _on_grid(v, 10, -14)


def _exact_norm(v, weight):
    return v * weight.double() / torch.sqrt((v * v).sum(dim=1, keepdim=True) / v.shape[1] + EPS)


def exact(case, seed):
    s = prepare(case, seed)
    k = case["kind"]
    if k == "route":
        p = torch.softmax(s["logits"].double(), dim=1)
        # The experts by counting how many of a row are ahead of one: larger, or equal with a lower index.
        l, E = s["logits"].double(), case["E"]
        index = torch.arange(E, device=DEV)
        place = torch.empty(l.shape, dtype=torch.int64, device=DEV)
        for lo in range(0, l.shape[0], 256):
            a = l[lo:lo + 256]
            ahead = (a[:, None, :] > a[:, :, None]) | ((a[:, None, :] == a[:, :, None]) & (index[None, :] < index[:, None]))
            place[lo:lo + 256] = ahead.sum(dim=2)
        experts = torch.argsort(place, dim=1)[:, :case["k"]]
        w = p.gather(1, experts)
        if case["renormalize"]:
            w = w / w.sum(dim=1, keepdim=True)
        chosen = torch.zeros(l.shape, dtype=torch.int64, device=DEV).scatter_(1, experts, 1)
        counts = chosen.sum(dim=0)
        first = counts.cumsum(dim=0) - counts
        slots = (first + chosen.cumsum(dim=0) - chosen).gather(1, experts)       # tokens of the expert ahead of this one
        rows = torch.empty(slots.numel(), dtype=torch.int64, device=DEV)
        rows[slots.reshape(-1)] = torch.arange(l.shape[0], device=DEV).repeat_interleave(case["k"])
        return experts, w, torch.cat([first, counts.sum()[None]]), rows, slots
    if k == "grouped":
        X = s["X"].double()
        owner = torch.searchsorted(s["offsets"][1:].contiguous(), torch.arange(case["T"] * case["k"], device=DEV, dtype=torch.int32), right=True)
        out = torch.empty(owner.shape[0], case["N"], dtype=torch.float64, device=DEV)
        for e in range(case["E"]):
            at = torch.nonzero(owner == e)[:, 0]
            if at.numel() == 0:
                continue
            y = torch.mm(X[at if s["rows"] is None else s["rows"][at].long()], s["W"][e].double())
            if case["form"] == "swiglu":
                y = _exact_16(y, case["dtype"])
                y = y[:, :case["N"]] * torch.special.expit(y[:, :case["N"]]) * y[:, case["N"]:]
            out[at] = y
        return out
    if k == "sum":
        y = s["y"].double().sum(dim=0) if case["P"] else s["y"].double()
        out = s["residual"].double() if s["residual"] is not None else torch.zeros(case["T"], case["H"], dtype=torch.float64, device=DEV)
        for j in range(case["k"]):
            out = out + s["weights"][:, j:j + 1].double() * y[s["slots"][:, j].long()]
        return out
    if k == "w4":
        group = torch.arange(case["K"], device=DEV) // case["group"]
        q = torch.empty(case["N"], case["K"], dtype=torch.float64, device=DEV)
        q[:, 0::2], q[:, 1::2] = (s["Wq"] % 16).double(), (s["Wq"] // 16).double()
        zero = 8 if s["zeros"] is None else s["zeros"].double()[:, group]
        return torch.mm(s["X"].double(), ((q - zero) * s["scales"].double()[:, group]).t().contiguous())
    y = _exact_16(s["y"].double().sum(dim=0), case["dtype"]) if case["P"] else s["y"].double()
    n = _exact_norm(y, s["post_weight"])
    hidden = case["scale"] * s["residual"].double() + (n if s["gate"] is None else s["gate"].double() * n)
    hidden = _exact_16(hidden, case["dtype"])
    return hidden, _exact_norm(hidden, s["next_weight"])
