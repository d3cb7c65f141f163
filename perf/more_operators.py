"""What the performance of the operators that train a routed network or a classifier is measured on: the
router's balance loss and gradient, and the softmax cross entropy of a product with many classes, with its
gradient.

With `own` false the operators are computed in their plain form (elementary torch operations in 32 bits, long
sums in 64, rounded once at the end), otherwise through the framework's entry points.  Plans are made once by
`prepare`, as a training program keeps them; activations, weights, labels and scores are handed over as they
lie in device memory.
"""
import math

import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}


def _router(op, name, tokens, experts, k, dtype, scoring, masked=0.0, parts="both"):
    """masked: share of the scores that are -inf; some rows are then closed altogether (padding).  parts: which
    gradients arrive (of the entries' weights, of the balance loss, or both)."""
    return {"name": name, "op": op, "tokens": tokens, "experts": experts, "k": k, "dtype": dtype,
            "scoring": scoring, "masked": masked, "parts": parts}


def _xent(op, name, rows, classes, width, dtype, unlabelled=0.0):
    """unlabelled: share of the rows that have no label (padding, nodes that are not trained on)."""
    return {"name": name, "op": op, "rows": rows, "classes": classes, "width": width, "dtype": dtype,
            "unlabelled": unlabelled}


def listed():
    return [
        # balance of a handful of decoded tokens: nothing but latency
        _router("balance", "balance_few", 8, 16, 2, "f32", "softmax_top"),
        # odd sizes, experts closed to some tokens, padded rows, sigmoid scores
        _router("balance", "balance_ragged", 5003, 129, 6, "f16", "sigmoid_top", masked=0.3),
        # the tokens of one training step of a network of many small experts
        _router("balance", "balance_step", 131072, 256, 8, "bf16", "softmax"),
        # gradient of a small batch, both losses
        _router("route_grad", "route_grad_few", 64, 8, 2, "f32", "softmax_top"),
        # the balance loss alone (a router whose weights are not trained by the task), padded rows
        _router("route_grad", "route_grad_balance", 4099, 60, 4, "bf16", "softmax", masked=0.2, parts="balance"),
        # the router's gradient of one training step
        _router("route_grad", "route_grad_step", 131072, 256, 8, "bf16", "sigmoid_top"),
        # one decoded token is scored against a vocabulary
        _xent("xent", "xent_one", 1, 65536, 4096, "bf16"),
        # a short text is scored; no size is a multiple of anything, some rows are padding
        _xent("xent", "xent_ragged", 203, 40009, 1037, "f16", unlabelled=0.3),
        # a batch of texts is scored
        _xent("xent", "xent_batch", 4096, 65536, 4096, "bf16"),
        # node classification on a graph: many rows, few classes, one node in ten has a label
        _xent("xent_train", "xent_train_nodes", 150000, 47, 128, "f32", unlabelled=0.9),
        # a small step of odd sizes, loss scaling, padded rows
        _xent("xent_train", "xent_train_ragged", 1021, 10007, 1000, "f16", unlabelled=0.2),
        # a training step over a large vocabulary
        _xent("xent_train", "xent_train_step", 8192, 131072, 4096, "bf16"),
    ]


def draw(rng):
    most = [max(work(c)[w] for c in listed()) for w in ("bytes", "flops")]

    def log_int(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    def size(lo, hi):       # every second one a multiple of 64, the others as they come
        n = log_int(lo, hi)
        return max(lo, n // 64 * 64) if rng.random() < 0.5 else n

    while True:
        op = rng.choice(["balance", "route_grad", "xent", "xent", "xent_train", "xent_train"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op in ("balance", "route_grad"):
            experts = log_int(4, 512)
            c = _router(op, "", log_int(1, 131072), experts, rng.randint(1, min(8, experts)), dtype,
                        rng.choice(["softmax", "softmax_top", "sigmoid", "sigmoid_top"]),
                        rng.choice([0.0, 0.0, 0.2, 0.5]), rng.choice(["both", "both", "weights", "balance"]))
        else:
            c = _xent(op, "", log_int(1, 16384), size(2, 131072), size(16, 8192), dtype,
                      rng.choice([0.0, 0.0, 0.1, 0.6]))
        w = work(c)
        if w["bytes"] <= most[0] and w["flops"] <= most[1]:
            del c["name"]
            return c


def work(case):
    es = _BYTES[case["dtype"]]
    if case["op"] in ("balance", "route_grad"):
        t, e, k = case["tokens"], case["experts"], case["k"]
        if case["op"] == "balance":
            return {"bytes": t * e * es + 4 * t * k + 8 * e + 8, "flops": 4 * t * e}
        extra = (4 * t * k if case["parts"] != "balance" else 0) + (4 * e + 8 if case["parts"] != "weights" else 0)
        return {"bytes": 2 * t * e * es + 4 * t * k + extra, "flops": 6 * t * e}
    t, v, d = case["rows"], case["classes"], case["width"]
    kept = t * (1.0 - case["unlabelled"])
    if case["op"] == "xent":
        return {"bytes": int((v * d + kept * d) * es + 12 * t), "flops": int(2 * kept * v * d)}
    return {"bytes": int((2 * v * d + kept * d + t * d) * es + 16 * t), "flops": int(6 * kept * v * d)}


# ------------------------------------------------------------------------------------------- inputs

def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    dtype = _DTYPE[case["dtype"]]
    if case["op"] in ("xent", "xent_train"):
        t, v, d = case["rows"], case["classes"], case["width"]
        w = torch.empty(v, d, device="cuda", dtype=dtype)
        w.normal_(0.0, 3.0 / math.sqrt(d), generator=gen)
        labels = torch.randint(0, v, (t,), device="cuda", generator=gen)
        # rows that know their label to a varying degree: their own logit is raised by 0 .. 12
        x = (normal(t, d) + w[labels].float() * (12.0 / 9.0 * uniform(t, 1))).to(dtype)
        labels[uniform(t) < case["unlabelled"]] = -1
        # gradient of the mean; where 16 bits would lose it (fp16) scaled up by the number of rows
        dloss = torch.full((t,), 1.0 if case["dtype"] == "f16" else 1.0 / t, device="cuda")
        return {"X": x, "W": w, "labels": labels.to(torch.int32), "dloss": dloss}
    t, e, k = case["tokens"], case["experts"], case["k"]
    scores = (normal(t, e) + 0.5 * normal(e)).to(dtype)
    if case["masked"]:
        closed = uniform(t, e) < case["masked"]
        closed[uniform(t) < 0.05] = True
        scores[closed] = -math.inf
    top = scores.float().topk(k, dim=1)
    colidx = torch.where(top.values > -math.inf, top.indices, -1).to(torch.int32)
    out = {"scores": scores, "colidx": colidx.reshape(-1),
           "rowptr": torch.arange(0, t * k + 1, k, device="cuda", dtype=torch.int32),
           "vals": torch.softmax(top.values, dim=1).nan_to_num(0.0).reshape(-1)}
    if case["op"] == "route_grad":
        # gradients of the sum over tokens, as a scaled loss gives them
        out["dvals"] = normal(t * k) if case["parts"] != "balance" else None
        out["counts"], out["dloss"] = None, None
        if case["parts"] != "weights":
            named = colidx.reshape(-1)[colidx.reshape(-1) >= 0].long()
            counts = torch.zeros(e + 1, device="cuda", dtype=torch.int32)
            counts[:e] = torch.bincount(named, minlength=e)
            counts[e] = (colidx >= 0).any(1).sum()
            out["counts"], out["dloss"] = counts, torch.full((1,), 0.01 * t, device="cuda")
    return out


def prepare(case, seed):
    state = {"case": case}
    state.update(_inputs(case, seed))
    if own:
        import paper_2407_00243_amd as tf
        if case["op"] == "balance":
            state["workspace"] = torch.empty(tf.tf_moe_balance_size(case["tokens"], case["experts"]),
                                             dtype=torch.uint8, device="cuda")
        elif case["op"] in ("xent", "xent_train"):
            state["plan"] = tf.XentPlan(case["classes"], case["width"], state["X"].dtype, max_rows=case["rows"])
    return state


# ---------------------------------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_2407_00243_amd as tf
    case, stream = state["case"], torch.cuda.current_stream().cuda_stream
    if case["op"] in ("xent", "xent_train"):
        X, W, labels, plan = state["X"], state["W"], state["labels"], state["plan"]
        loss = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
        lse = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
        plan.loss(X, W, labels, loss, lse, stream)
        if case["op"] == "xent":
            return loss, lse
        dX, dW = torch.empty_like(X), torch.empty_like(W)
        plan.grad(X, W, labels, lse, state["dloss"], dX, dW, stream)
        return loss, lse, dX, dW
    t, e = case["tokens"], case["experts"]
    scoring = {"softmax": tf.TF_ROUTE_SOFTMAX, "softmax_top": tf.TF_ROUTE_SOFTMAX_TOP,
               "sigmoid": tf.TF_ROUTE_SIGMOID, "sigmoid_top": tf.TF_ROUTE_SIGMOID_TOP}[case["scoring"]]
    A = tf.DeviceCsr(t, e, state["rowptr"], state["colidx"], state["vals"])
    if case["op"] == "balance":
        counts = torch.empty(e + 1, dtype=torch.int32, device="cuda")
        mass = torch.empty(e, dtype=torch.float32, device="cuda")
        loss = torch.empty(1, dtype=torch.float32, device="cuda")
        tf.tf_moe_balance(state["scores"], A, counts, mass, loss, state["workspace"], scoring, stream=stream)
        return counts, mass, loss
    dscores = torch.empty_like(state["scores"])
    tf.tf_moe_route_grad(state["scores"], A, dscores, scoring, scale=2.5, dvals=state["dvals"],
                         counts=state["counts"], dloss=state["dloss"], stream=stream)
    return dscores


def _run_plain(state):
    if state["case"]["op"] in ("xent", "xent_train"):
        return _xent_plain(state)
    return _router_plain(state)


def _xent_plain(state):
    case, labels = state["case"], state["labels"].long()
    kept = labels >= 0
    x, w = state["X"].float(), state["W"].float()
    row = torch.nonzero(kept).squeeze(1)
    x, y = x[row], labels[row]
    logits = x @ w.t()
    top = logits.amax(1, keepdim=True) if row.numel() else logits.new_zeros(0, 1)
    p = torch.exp(logits - top)
    total = p.sum(1, keepdim=True)
    lse_kept = (top + torch.log(total)).squeeze(1)
    loss = torch.zeros(case["rows"], device="cuda")
    lse = torch.zeros(case["rows"], device="cuda")
    lse[row] = lse_kept
    loss[row] = lse_kept - logits.gather(1, y[:, None]).squeeze(1)
    if case["op"] == "xent":
        return loss, lse
    del logits
    p /= total
    p[torch.arange(row.numel(), device="cuda"), y] -= 1.0
    p *= state["dloss"][row][:, None]
    dx = torch.zeros(case["rows"], case["width"], device="cuda")
    dx[row] = p @ w
    return loss, lse, dx.to(state["X"].dtype), (p.t() @ x).to(state["X"].dtype)


def _router_plain(state):
    case, l = state["case"], state["scores"].float()
    t, e, k = case["tokens"], case["experts"], case["k"]
    columns = state["colidx"].long().reshape(t, k)
    open_ = columns >= 0
    counted = open_.any(1, keepdim=True)
    sigmoid = case["scoring"].startswith("sigmoid")
    if sigmoid:
        share = torch.where(l > -math.inf, 1.0 / (1.0 + torch.exp(-l)), torch.zeros_like(l))
        slope = 1.0 - share
    else:
        top = l.amax(1, keepdim=True)
        share = torch.exp(l - torch.where(top > -math.inf, top, torch.zeros_like(top)))
        slope = torch.ones_like(l)
    total = share.sum(1, keepdim=True)
    p = torch.where(counted, share / total, torch.zeros_like(l))
    if case["op"] == "balance":
        counts = torch.zeros(e + 1, device="cuda", dtype=torch.int32)
        counts.index_add_(0, torch.where(open_, columns, e).reshape(-1),
                          torch.ones(t * k, device="cuda", dtype=torch.int32))
        counts[e] = counted.sum()
        named, rows = counts[:e].sum().clamp_min(1), counts[e].clamp_min(1)
        mass = p.double().sum(0) / rows
        return counts, mass.float(), (e * (mass * counts[:e] / named).sum()).float().reshape(1)
    d = torch.zeros_like(l)
    if case["parts"] != "weights":
        counts, n = state["counts"][:e].float(), state["counts"][e].float().clamp_min(1.0)
        f = counts / counts.sum().clamp_min(1.0)
        d += state["dloss"] * (e / n) * p * slope * (f - (p * f).sum(1, keepdim=True))
    if case["parts"] != "balance":
        # entries that are passed over point to a column behind the last one
        columns = torch.where(open_, columns, e)
        g = torch.zeros(t, e + 1, device="cuda")
        g.scatter_(1, columns, 2.5 * state["dvals"].reshape(t, k))
        chosen = torch.zeros(t, e + 1, device="cuda", dtype=torch.bool)
        chosen.scatter_(1, columns, True)
        g, chosen = g[:, :e], chosen[:, :e]
        if case["scoring"] == "sigmoid":
            d += share * slope * g * chosen
        else:
            q = p
            if case["scoring"] != "softmax":
                q = torch.where(chosen, share, torch.zeros_like(share))
                q = torch.where(counted, q / q.sum(1, keepdim=True), torch.zeros_like(q))
            d += q * slope * (g - (q * g).sum(1, keepdim=True))
    return d.to(state["scores"].dtype)


# ------------------------------------------------------------------------------- definition in 64 bits

def exact(case, seed):
    data = _inputs(case, seed)
    return _exact_xent(case, data) if case["op"] in ("xent", "xent_train") else _exact_router(case, data)


def _exact_xent(case, data):
    x, w, labels = data["X"].double(), data["W"].double(), data["labels"].long()
    t, v, d = case["rows"], case["classes"], case["width"]
    loss = torch.zeros(t, device="cuda", dtype=torch.float64)
    lse, dx, dw = torch.zeros_like(loss), torch.zeros_like(x), torch.zeros_like(w)
    for first in range(0, t, 2048):
        at = first + torch.nonzero(labels[first:first + 2048] >= 0).squeeze(1)
        if at.numel() == 0:
            continue
        logits = torch.matmul(x[at], w.transpose(0, 1).contiguous())
        lse[at] = torch.logsumexp(logits, dim=1)
        loss[at] = lse[at] - logits[torch.arange(at.numel(), device="cuda"), labels[at]]
        if case["op"] == "xent_train":
            g = torch.softmax(logits, dim=1)
            g[torch.arange(at.numel(), device="cuda"), labels[at]] -= 1.0
            g.mul_(data["dloss"].double()[at].unsqueeze(1))
            dx[at] = torch.matmul(g, w)
            dw += torch.matmul(g.transpose(0, 1).contiguous(), x[at])
    return (loss, lse) if case["op"] == "xent" else (loss, lse, dx, dw)


def _exact_router(case, data):
    t, e, k = case["tokens"], case["experts"], case["k"]
    l = data["scores"].double()
    one_hot = torch.zeros(t, e, device="cuda", dtype=torch.float64)
    columns = data["colidx"].long().reshape(t, k)
    for i in range(k):
        r = torch.nonzero(columns[:, i] >= 0).squeeze(1)
        one_hot[r, columns[r, i]] = 1.0
    active = one_hot.sum(1) > 0
    if case["scoring"].startswith("softmax"):
        log_share = l
        slope = torch.ones_like(l)
    else:
        log_share = torch.nn.functional.logsigmoid(l)
        slope = torch.sigmoid(-l)

    def shares(over):           # rows that add up to one over the places where `over` is
        z = log_share.masked_fill(over == 0, -math.inf)
        return torch.softmax(z, dim=1).nan_to_num(0.0) * active[:, None]

    p = shares(torch.ones_like(l))
    if case["op"] == "balance":
        counts = one_hot.sum(0)
        mass = p.sum(0) / max(1.0, active.sum().item())
        loss = e * torch.dot(mass, counts / max(1.0, counts.sum().item()))
        whole = torch.cat([counts, active.sum().reshape(1)]).to(torch.int32)
        return whole, mass, loss.reshape(1)
    d = torch.zeros_like(l)
    if case["parts"] != "weights":
        counts = data["counts"].double()
        f = counts[:e] / counts[:e].sum().clamp(min=1.0)
        inner = torch.mv(p, f)
        d += p * slope * (f[None, :] - inner[:, None]) * (data["dloss"].double() * e / counts[e].clamp(min=1.0))
    if case["parts"] != "balance":
        g = torch.zeros_like(l)
        dvals = data["dvals"].double().reshape(t, k)
        for i in range(k):
            r = torch.nonzero(columns[:, i] >= 0).squeeze(1)
            g[r, columns[r, i]] = 2.5 * dvals[r, i]
        if case["scoring"] == "sigmoid":
            d += torch.sigmoid(l) * slope * g
        else:
            q = p if case["scoring"] == "softmax" else shares(one_hot)
            d += q * slope * (g - (q * g).sum(1)[:, None])
    return d
