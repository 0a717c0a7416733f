"""Performance cases of the operators around the sparse FFN layer: what a program that uses it
as a routed residual block, for serving and for training, has them do.

norm      the RMS norm after a block, its gate and the scaled residual sum, and the norm before
          the next block: forward, or backward with the parameters' gradients
route     the router's softmax over a token's k best experts; training: with its gradient
experts   tokens into expert order and the experts' rows weighted back into tokens; training:
          with the gradients of both
clip      the norm of all gradients of a model part, and the gradients scaled to a largest norm

A case is a dict of plain values. `prepare` makes what the program holds before the call, `run`
makes one pass: in plain torch, or (`own`) through the library's entry points. `exact` is the
operator's definition in float64 and `work` what a pass cannot do without.
"""
from __future__ import annotations

import math

import torch

own = False

NORM_PRE, NORM_POST = 1, 2
EPS = 1e-6
RES_SCALE = 0.75  # the residual stream is damped a little at every block
MAX_NORM = 1.0


def _norm(**kw):
    """norms: which of the two norms the boundary has ("both", "pre", "post"); gate_c: a gate per
    channel; gate_t: a gate per token."""
    return dict(op="norm", **{**dict(way="forward", dtype="bf16", T=1, d=2048, norms="both", gate_c=True, gate_t=False),
                              **kw})


def _route(**kw):
    """normalise: the weights are a softmax over the chosen experts (else over all); masked: some
    experts are unavailable (logit -inf) to some tokens, all of them to a few."""
    return dict(op="route", **{**dict(way="forward", dtype="f32", T=1, E=8, k=2, normalise=True, scale=1.0,
                                      masked=False), **kw})


def _experts(**kw):
    """skew: how much more often the favourite experts are chosen (0: all alike); drop: the share
    of (token, choice) pairs that go to no expert."""
    return dict(op="experts", **{**dict(way="forward", dtype="bf16", T=1, d=2048, E=8, k=2, skew=0.0, drop=0.0), **kw})


def _clip(**kw):
    """n matrices of rows x cols in f32 (ragged: each of its own size below that), and as many
    vectors of cols; bf16: the share of the tensors that are bf16; large: the norm is above the
    largest one allowed, as in early training."""
    return dict(op="clip", **{**dict(n=2, rows=256, cols=1024, ragged=False, bf16=0.0, large=True), **kw})


def listed():
    return [
        # One token of one sequence being decoded at a 2048-wide block boundary: latency.
        _norm(name="norm_decode_1_token", T=1, d=2048),
        # The boundary between two blocks in a full prefill batch.
        _norm(name="norm_prefill_8192_tokens", T=8192, d=4096),
        # A training batch, backward, with both gates (a learned one per channel, one per token).
        _norm(name="norm_train_16384_tokens", way="backward", T=16384, d=4096, gate_t=True),
        # An odd width in exact precision, the gradient of a short ragged batch.
        _norm(name="norm_train_509_tokens_f32", way="backward", dtype="f32", T=509, d=1003),
        # A batch of 32 sequences being decoded through a layer of 64 experts.
        _route(name="route_decode_32_tokens", dtype="bf16", T=32, E=64, k=8),
        # A training batch over 64 experts, weights and their gradient, with masked experts.
        _route(name="route_train_16384_tokens", way="train", T=16384, E=64, k=8, masked=True),
        # 32 sequences being decoded, two of eight experts each.
        _experts(name="experts_decode_32_tokens", T=32, d=4096),
        # A full prefill batch over eight experts of uneven load.
        _experts(name="experts_prefill_8192_tokens", T=8192, d=4096, skew=1.0),
        # A training batch over eight experts: both directions and their gradients.
        _experts(name="experts_train_16384_tokens", way="train", T=16384, d=4096),
        # The gradients of the small layer (d = 256, f = 1024): launch bound.
        _clip(name="clip_small_layer", n=2, rows=256, cols=1024),
        # The two weight gradients of the layer at its benchmark size, and its vectors.
        _clip(name="clip_layer", n=2, rows=4096, cols=16384),
        # Eight gated experts and a few odd-sized parts: many tensors of many sizes and both types.
        _clip(name="clip_experts_ragged", n=96, rows=1024, cols=2816, ragged=True, bf16=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly multiples of 64, as models have, and odd ones."""
    d = _log_int(rng, lo, hi)
    return d if rng.random() < 0.3 else max(64, d // 64 * 64)


def draw(rng):
    op = rng.choice(["norm", "norm", "route", "experts", "experts", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        d = _width(rng, 64, 8192)
        return _norm(way=rng.choice(["forward", "backward"]), dtype=dtype, T=_log_int(rng, 1, min(16384, (1 << 26) // d)),
                     d=d, norms=rng.choice(["both", "both", "pre", "post"]), gate_c=rng.random() < 0.5,
                     gate_t=rng.random() < 0.5)
    if op == "route":
        E = rng.choice([8, 16, 32, 60, 64, 128, 160, 256])
        return _route(way=rng.choice(["forward", "train"]), dtype=dtype, T=_log_int(rng, 1, 16384), E=E,
                      k=rng.choice([1, 2, 4, 6, 8]), normalise=rng.random() < 0.5, scale=rng.choice([1.0, 2.5]),
                      masked=rng.random() < 0.5)
    if op == "experts":
        d, k = _width(rng, 64, 8192), rng.choice([1, 2, 4, 6, 8])
        es = 2 if dtype == "bf16" else 4
        return _experts(way=rng.choice(["forward", "train"]), dtype=dtype,
                        T=_log_int(rng, 1, min(16384, (1 << 28) // (d * k * es))), d=d,
                        E=rng.choice([8, 16, 60, 64, 160, 256]), k=k, skew=rng.choice([0.0, 0.5, 1.0]),
                        drop=rng.choice([0.0, 0.0, 0.1]))
    rows, cols = _log_int(rng, 64, 4096), _log_int(rng, 64, 16384)
    return _clip(n=_log_int(rng, 1, max(1, min(256, (1 << 27) // (rows * cols)))), rows=rows, cols=cols,
                 ragged=rng.random() < 0.5, bf16=rng.choice([0.0, 0.5, 1.0]), large=rng.random() < 0.7)


# ---- inputs ---------------------------------------------------------------------------------

def _act(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


class _Draw:
    """The case's random numbers on the GPU, from the seed alone."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 1000003 + 7)

    def normal(self, shape, std=1.0, dtype=torch.float32, mean=0.0):
        return torch.randn(shape, generator=self.g, device="cuda").mul_(std).add_(mean).to(dtype)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device="cuda")


def _clip_sizes(case):
    """[(elements, is bf16)] of the case's tensors, the same for every seed."""
    sizes, n = [], case["n"]
    for i in range(n):
        rows, cols = case["rows"], case["cols"]
        if case["ragged"]:  # spread evenly between a sixteenth of the rows and all of them, any width
            rows, cols = max(1, rows * (1 + (i * 7) % 16) // 16 - i % 3), max(1, cols - (i * 37) % 129)
        half = (i % 8) < 8 * case["bf16"]
        sizes += [(rows * cols, half), (cols, half)]
    return sizes


def _inputs(case, seed):
    r, op = _Draw(seed), case["op"]
    if op == "norm":
        T, d, act = case["T"], case["d"], _act(case)
        s = dict(Y=r.normal((T, d), 1.5, act) if case["norms"] != "pre" or case["gate_c"] or case["gate_t"] else None,
                 w_pre=r.normal((d,), 0.1, mean=1.0) if case["norms"] != "post" else None,
                 w_post=r.normal((d,), 0.1, mean=1.0) if case["norms"] != "pre" else None,
                 gate_c=r.normal((d,), 0.2, mean=0.5) if case["gate_c"] else None,
                 gate_t=r.uniform((T,)) if case["gate_t"] else None)
        if case["way"] == "forward":
            s["X"] = r.normal((T, d), 2.0, act)
        else:
            s["X_out"] = r.normal((T, d), 2.0, act)
            s["dX_out"] = r.normal((T, d), 1.0, act)
            s["dN"] = r.normal((T, d), 1.0, act) if case["norms"] != "post" else None
        return s
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        logits = r.normal((T, E), 1.5)
        if case["masked"]:
            off = r.uniform((T, E)) < 0.25
            off |= (r.uniform((T,)) < 0.01)[:, None]
            logits = logits.masked_fill(off, -math.inf)
        return dict(logits=logits.to(_act(case)), dweight=r.normal((T, k)) if case["way"] == "train" else None)
    if op == "experts":
        T, d, E, k, act = case["T"], case["d"], case["E"], case["k"], _act(case)
        favour = -case["skew"] * torch.arange(E, device="cuda", dtype=torch.float32) / max(1, E / 4)
        score = r.normal((T, E), 1.0) + favour
        expert = score.sort(dim=1, descending=True).indices[:, :k].to(torch.int32)
        expert = expert.contiguous()
        n = T * k - int(case["drop"] * T * k)  # the same for every seed
        if n < T * k:
            expert.view(-1)[torch.randperm(T * k, generator=r.g, device="cuda")[n:]] = -1
        s = dict(n=n, expert=expert, weight=r.uniform((T, k)) / k, X=r.normal((T, d), 1.0, act),
                 Ys=r.normal((n, d), 1.0, act))
        if case["way"] == "train":
            s.update(dY=r.normal((T, d), 1.0, act), dXs=r.normal((n, d), 1.0, act))
        return s
    sizes = _clip_sizes(case)
    total = sum(n for n, _ in sizes)
    std = (10.0 if case["large"] else 0.1) * MAX_NORM / math.sqrt(total)
    buckets = {}
    for name, half in (("f32", False), ("bf16", True)):  # gradients live in one bucket a type, end to end
        lens = [n for n, h in sizes if h == half]
        flat = r.normal((sum(lens),), std, torch.bfloat16 if half else torch.float32)
        buckets[name] = dict(flat=flat, grads=list(flat.split(lens)) if lens else [])
    return dict(buckets=buckets)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op, dev = case["op"], "cuda"
    new = torch.empty_like
    if op == "norm":
        if case["way"] == "forward":
            s.update(X_out=new(s["X"]), N=new(s["X"]) if s["w_pre"] is not None else None)
        else:
            s.update(dX=new(s["X_out"]), dY=None if s["Y"] is None else new(s["Y"]),
                     **{"d" + n: None if s[n] is None else new(s[n]) for n in ("w_pre", "w_post", "gate_c", "gate_t")})
    elif op == "route":
        s.update(expert=torch.empty((case["T"], case["k"]), dtype=torch.int32, device=dev),
                 weight=torch.empty((case["T"], case["k"]), device=dev), dlogits=new(s["logits"]))
    elif op == "experts":
        s.update(pos=new(s["expert"]), offsets=torch.empty((case["E"] + 1,), dtype=torch.int32, device=dev),
                 Xs=new(s["Ys"]), Y=new(s["X"]))
        if case["way"] == "train":
            s.update(dYs=new(s["Ys"]), dX=new(s["X"]), dweight=new(s["weight"]))
    else:
        for bkt in s["buckets"].values():
            bkt["out"] = new(bkt["flat"])
            bkt["outs"] = list(bkt["out"].split([g.numel() for g in bkt["grads"]])) if bkt["grads"] else []
        s.update(sumsq=torch.empty((1,), dtype=torch.float64, device=dev), norm=torch.empty((1,), device=dev))
    return s


# ---- the plain form: 32 bits, rounded once at the end ----------------------------------------

def _f(t):
    return None if t is None else t.float()


def _plain_norm(s, case):
    act, post, pre = _act(case), case["norms"] != "pre", case["norms"] != "post"
    gate = 1.0
    if s["gate_c"] is not None:
        gate = gate * s["gate_c"]
    if s["gate_t"] is not None:
        gate = gate * s["gate_t"][:, None]
    Y = _f(s["Y"])
    y_hat = None
    if Y is not None:
        r_y = torch.rsqrt(Y.square().mean(1, keepdim=True) + EPS) if post else 1.0
        y_hat = Y * r_y
    w_post = s["w_post"] if post else 1.0
    if case["way"] == "forward":
        X_out = RES_SCALE * _f(s["X"])
        if Y is not None:
            X_out = X_out + gate * (y_hat * w_post)
        N = X_out * torch.rsqrt(X_out.square().mean(1, keepdim=True) + EPS) * s["w_pre"] if pre else None
        return dict(X_out=X_out.to(act), N=None if N is None else N.to(act))
    D, out = _f(s["dX_out"]), {}
    if pre:
        X, dN = _f(s["X_out"]), _f(s["dN"])
        r_x = torch.rsqrt(X.square().mean(1, keepdim=True) + EPS)
        x_hat = X * r_x
        g = dN * s["w_pre"]
        D = D + r_x * (g - x_hat * (g * x_hat).mean(1, keepdim=True))
        out["dw_pre"] = (dN * x_hat).sum(0)
    out["dX"] = (RES_SCALE * D).to(act)
    if Y is not None:
        h = D * gate * w_post
        out["dY"] = (r_y * (h - y_hat * (h * y_hat).mean(1, keepdim=True)) if post else h).to(act)
        if post:
            out["dw_post"] = (D * gate * y_hat).sum(0)
        P = D * y_hat * w_post
        if s["gate_c"] is not None:
            out["dgate_c"] = (P if s["gate_t"] is None else P * s["gate_t"][:, None]).sum(0)
        if s["gate_t"] is not None:
            out["dgate_t"] = (P if s["gate_c"] is None else P * s["gate_c"]).sum(1)
    return out


def _plain_route(s, case):
    logits = _f(s["logits"])
    ok = logits > -math.inf  # false for NaN too
    best = torch.where(ok, logits, -math.inf).sort(dim=1, descending=True, stable=True)
    idx = best.indices[:, :case["k"]]
    taken = ok.gather(1, idx)
    top = torch.where(ok.any(1, keepdim=True), best.values[:, :1], 0.0)
    e_all = torch.where(ok, (logits - top).exp(), 0.0)
    e = e_all.gather(1, idx)
    den = (e if case["normalise"] else e_all).sum(1, keepdim=True)
    share = torch.where(taken, e / den, 0.0)
    out = dict(expert=torch.where(taken, idx, -1).to(torch.int32), weight=case["scale"] * share)
    if case["way"] == "train":
        G = case["scale"] * s["dweight"]
        mean = (share * G).sum(1, keepdim=True)
        if case["normalise"]:
            dl = torch.zeros_like(logits).scatter(1, idx, share * (G - mean))
        else:
            dl = torch.where(ok, -(e_all / den) * mean, 0.0).scatter_add(1, idx, share * G)
        out["dlogits"] = dl.to(s["logits"].dtype)
    return out


def _plain_experts(s, case):
    act, E, k, n = _act(case), case["E"], case["k"], s["n"]
    flat = s["expert"].reshape(-1)
    there = flat >= 0
    by_expert = torch.where(there, flat, E).sort(stable=True)
    slots = by_expert.indices
    pos = torch.empty_like(slots)
    pos[slots] = torch.arange(slots.numel(), device=slots.device)
    pos = pos.reshape(s["expert"].shape)
    there = there.reshape(s["expert"].shape)
    of = (by_expert.values[None, :] < torch.arange(E + 1, device=slots.device)[:, None]).sum(1)
    out = dict(pos=torch.where(there, pos, -1).to(torch.int32), offsets=of.to(torch.int32))
    tokens = slots[:n] // k
    out["Xs"] = s["X"][tokens]
    at = torch.where(there, pos, 0)
    w = torch.where(there, s["weight"], 0.0)[:, :, None]
    if n:
        rows = _f(s["Ys"][at])
        out["Y"] = torch.where(there[:, :, None], rows * w, 0.0).sum(1).to(act)
    else:
        out["Y"] = torch.zeros_like(s["X"])
    if case["way"] == "train":
        dY = _f(s["dY"])
        out["dYs"] = (dY[tokens] * s["weight"].reshape(-1)[slots[:n]][:, None]).to(act)
        if n:
            out["dweight"] = torch.where(there, (rows * dY[:, None, :]).sum(2), 0.0)
            out["dX"] = torch.where(there[:, :, None], _f(s["dXs"][at]), 0.0).sum(1).to(act)
        else:
            out["dweight"], out["dX"] = torch.zeros_like(s["weight"]), torch.zeros_like(s["X"])
    return out


def _plain_clip(s, case):
    a, b = s["buckets"]["f32"]["flat"], s["buckets"]["bf16"]["flat"]
    norm = (a.square().sum() + b.float().square().sum()).sqrt()
    by = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
    return dict(norm=norm.reshape(1), f32=a * by, bf16=(b.float() * by).to(torch.bfloat16))


# ---- the library -----------------------------------------------------------------------------

def _scratch(s, nbytes):
    """The workspace that a program keeps for its calls."""
    if s.get("workspace") is None or s["workspace"].numel() < nbytes:
        s["workspace"] = torch.empty(max(1, nbytes), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_norm(s, case):
    from paper_2603_23198_amd import binding as b
    norms = {"both": NORM_PRE | NORM_POST, "pre": NORM_PRE, "post": NORM_POST}[case["norms"]]
    kw = dict(norms=norms, w_pre=s["w_pre"], w_post=s["w_post"], gate_c=s["gate_c"], gate_t=s["gate_t"],
              res_scale=RES_SCALE, eps=EPS)
    if case["way"] == "forward":
        b.sfl_norm_forward(s["X"], s["Y"], X_out=s["X_out"], N=s["N"], **kw)
        return dict(X_out=s["X_out"], N=s["N"])
    ws = _scratch(s, b.sfl_norm_workspace_size(case["T"], case["d"], case["dtype"]))
    b.sfl_norm_backward(s["X_out"], s["Y"], s["dX_out"], s["dN"], dX=s["dX"], dY=s["dY"], dw_pre=s["dw_pre"],
                        dw_post=s["dw_post"], dgate_c=s["dgate_c"], dgate_t=s["dgate_t"], workspace=ws, **kw)
    return {n: s[n] for n in ("dX", "dY", "dw_pre", "dw_post", "dgate_c", "dgate_t")}


def _own_route(s, case):
    from paper_2603_23198_amd import binding as b
    kw = dict(normalise=case["normalise"], scale=case["scale"])
    b.sfl_route_forward(s["logits"], s["expert"], s["weight"], **kw)
    out = dict(expert=s["expert"], weight=s["weight"])
    if case["way"] == "train":
        b.sfl_route_backward(s["logits"], s["expert"], s["dweight"], s["dlogits"], **kw)
        out["dlogits"] = s["dlogits"]
    return out


def _own_experts(s, case):
    from paper_2603_23198_amd import binding as b
    ws = _scratch(s, b.sfl_expert_workspace_size(case["T"], case["k"], case["E"]))
    b.sfl_expert_dispatch(s["expert"], case["E"], s["pos"], s["offsets"], X=s["X"], Xs=s["Xs"], workspace=ws)
    b.sfl_expert_combine(s["Ys"], s["pos"], s["Y"], weight=s["weight"])
    out = {n: s[n] for n in ("pos", "offsets", "Xs", "Y")}
    if case["way"] == "train":
        b.sfl_expert_combine_backward(s["dY"], s["Ys"], s["pos"], s["weight"], dYs=s["dYs"], dweight=s["dweight"])
        b.sfl_expert_combine(s["dXs"], s["pos"], s["dX"])  # the gradient of the way there
        out.update({n: s[n] for n in ("dYs", "dweight", "dX")})
    return out


def _own_clip(s, case):
    from paper_2603_23198_amd import binding as b
    f32, bf16 = s["buckets"]["f32"], s["buckets"]["bf16"]
    grads = b.grad_list(f32["grads"] + bf16["grads"], f32["outs"] + bf16["outs"])
    ws = _scratch(s, b.sfl_grad_workspace_size(grads))
    b.sfl_grad_sumsq(grads, s["sumsq"], workspace=ws)
    b.sfl_grad_clip(grads, s["sumsq"], MAX_NORM, s["norm"])
    return dict(norm=s["norm"], f32=f32["out"], bf16=bf16["out"])


def run(s):
    case = s["case"]
    if own:
        out = dict(norm=_own_norm, route=_own_route, experts=_own_experts, clip=_own_clip)[case["op"]](s, case)
    else:
        out = dict(norm=_plain_norm, route=_plain_route, experts=_plain_experts, clip=_plain_clip)[case["op"]](s, case)
    return {n: t for n, t in out.items() if t is not None}


# ---- what a pass needs, and what it has to give ----------------------------------------------

def work(case):
    es = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "norm":
        T, d = case["T"], case["d"]
        block = case["norms"] != "pre" or case["gate_c"] or case["gate_t"]
        vectors = 4 * d * ((case["norms"] != "post") + (case["norms"] != "pre") + case["gate_c"]) + 4 * T * case["gate_t"]
        pre = case["norms"] != "post"
        if case["way"] == "forward":
            return {"bytes": T * d * es * (2 + block + pre) + vectors, "flops": T * d * 11}
        return {"bytes": T * d * es * (2 + 2 * block + 2 * pre) + 2 * vectors, "flops": T * d * 27}
    if case["op"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        back = T * E * es + T * k * 4 if case["way"] == "train" else 0
        return {"bytes": T * E * es + T * k * 8 + back, "flops": T * E * (k + 3)}
    if case["op"] == "experts":
        T, d, k = case["T"], case["d"], case["k"]
        n = T * k - int(case["drop"] * T * k)
        index = 8 * T * k + 4 * case["E"] + 4 * T * k
        there = (T + n) * d * es
        if case["way"] == "forward":
            return {"bytes": 2 * there + index, "flops": 2 * n * d}
        return {"bytes": 2 * there + index + (T + 2 * n) * d * es + there + 4 * T * k, "flops": 6 * n * d}
    sizes = _clip_sizes(case)
    nbytes = sum(n * (2 if half else 4) for n, half in sizes)
    # where nothing has to be scaled, the values still go to their place
    return {"bytes": 3 * nbytes, "flops": 3 * sum(n for n, _ in sizes)}


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "clip":
        g = [s["buckets"][n]["flat"].double() for n in ("f32", "bf16")]
        norm = math.sqrt(sum(float(v @ v) for v in g))
        by = min(1.0, MAX_NORM / norm)
        return dict(norm=torch.tensor([norm], dtype=torch.float64), f32=g[0] * by, bf16=g[1] * by)
    if op == "norm":
        return _exact_norm(s, case)
    if op == "route":
        return _exact_route(s, case)
    out = dict(pos=None, offsets=None)
    T, k, E = case["T"], case["k"], case["E"]
    expert = s["expert"].long()
    # the row of each (token, choice): those of lower experts, and those of its own before it
    onehot = torch.nn.functional.one_hot((expert + 1).reshape(-1), E + 1)[:, 1:]
    first = onehot.sum(0).cumsum(0) - onehot.sum(0)
    row = ((onehot.cumsum(0) - 1 + first) * onehot).sum(1).reshape(T, k)
    del onehot
    Y = torch.zeros_like(s["X"], dtype=torch.float64)
    out.update(Xs=torch.zeros_like(s["Ys"], dtype=torch.float64), Y=Y)
    if case["way"] == "train":
        out.update(dYs=torch.zeros_like(out["Xs"]), dX=torch.zeros_like(Y),
                   dweight=torch.zeros((T, k), dtype=torch.float64, device="cuda"))
    for j in range(k):
        t = (expert[:, j] >= 0).nonzero()[:, 0]
        p, w = row[t, j], s["weight"][t, j, None].double()
        out["Xs"][p] = s["X"][t].double()
        Y[t] += w * s["Ys"][p].double()
        if case["way"] == "train":
            dY = s["dY"][t].double()
            out["dYs"][p] = w * dY
            out["dweight"][t, j] = (dY * s["Ys"][p].double()).sum(1)
            out["dX"][t] += s["dXs"][p].double()
    return out


def _exact_norm(s, case):
    f = {n: t.double() if isinstance(t, torch.Tensor) else None for n, t in s.items()}
    T, d = case["T"], case["d"]
    one = torch.ones((1, 1), dtype=torch.float64, device="cuda")
    gc = one if f["gate_c"] is None else f["gate_c"][None, :]
    gt = one if f["gate_t"] is None else f["gate_t"][:, None]
    wp = one if f["w_post"] is None else f["w_post"][None, :]
    has_y, post, pre = f["Y"] is not None, case["norms"] != "pre", case["norms"] != "post"
    ry = 1 / (f["Y"].pow(2).sum(1, keepdim=True) / d + EPS).sqrt() if post else one
    if case["way"] == "forward":
        x = RES_SCALE * f["X"]
        if has_y:
            x += f["Y"] * ry * wp * gc * gt
        out = dict(X_out=x)
        if pre:
            out["N"] = x / (x.pow(2).sum(1, keepdim=True) / d + EPS).sqrt() * f["w_pre"]
        return out
    out, D = {}, f["dX_out"].clone()
    if pre:
        rx = 1 / (f["X_out"].pow(2).sum(1, keepdim=True) / d + EPS).sqrt()
        q = (f["dN"] * f["w_pre"] * f["X_out"]).sum(1, keepdim=True)
        D += rx * f["w_pre"] * f["dN"] - f["X_out"] * (rx.pow(3) * q / d)
        out["dw_pre"] = (f["dN"] * f["X_out"] * rx).sum(0)
    out["dX"] = RES_SCALE * D
    if has_y:
        q = (D * wp * gc * f["Y"]).sum(1, keepdim=True)  # sum of the incoming gradient times y
        dY = gt * D * (wp * gc) * ry
        if post:
            dY -= f["Y"] * (gt * ry.pow(3) * q / d)
            out["dw_post"] = (D * gt * f["Y"] * ry * gc).sum(0)
        out["dY"] = dY
        if f["gate_c"] is not None:
            out["dgate_c"] = (D * gt * f["Y"] * ry * wp).sum(0)
        if f["gate_t"] is not None:
            out["dgate_t"] = (q * ry)[:, 0]
    return out


def _exact_route(s, case):
    l, k = s["logits"].double(), case["k"]
    open_ = torch.isfinite(l)
    left, T = torch.where(open_, l, -math.inf), l.shape[0]
    mask = torch.zeros_like(open_)
    chosen = []
    for _ in range(k):  # the best of what is left, the lowest index of equal ones
        best = left.amax(1, keepdim=True)
        at = ((left == best) & open_ & ~mask).to(torch.int8).argmax(1)
        live = best[:, 0] > -math.inf
        chosen.append(torch.where(live, at, -1))
        rows = live.nonzero()[:, 0]
        mask[rows, at[rows]] = True
        left[rows, at[rows]] = -math.inf
    chosen = torch.stack(chosen, 1)
    live = chosen >= 0
    over = mask if case["normalise"] else open_
    p = torch.softmax(torch.where(over, l, -math.inf), 1).nan_to_num(0.0)  # rows without any expert: zeros
    share = torch.where(live, p.gather(1, chosen.clamp(min=0)), 0.0)
    out = dict(expert=None, weight=case["scale"] * share)
    if case["way"] == "train":
        up = torch.zeros_like(l)  # the gradient of the weights, at their experts
        t = torch.arange(T, device="cuda")[:, None].expand_as(chosen)[live]
        up[t, chosen[live]] = case["scale"] * s["dweight"].double()[live]
        out["dlogits"] = p * (up - (p * up).sum(1, keepdim=True))
    return out
