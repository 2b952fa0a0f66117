"""Low-rank adapters of many requests beside a shared projection, their gradients, and the norm and clipping of gradients.

A case is one call on data that a training or serving program has on the GPU: packed rows of many requests (`start`,
`adapter`), the shared matrix W [J][D], a pool of adapters as factor blocks U [n][R][J], V [n][R][D] with a rank and a scale
each; or a list of gradient tensors of many sizes.  Inputs are drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_ctx = None


def listed():
    return [
        # one token of one request: a serving step with nothing but latency
        dict(name="fwd_bf16_token", op="forward", dtype="bf16", T=1, J=1024, D=1024, n=4, R=16, S=1, pack="single", pad=0, save=False),
        # a decoding step: 64 requests, a token and mostly an adapter of its own each
        dict(name="fwd_bf16_decode", op="forward", dtype="bf16", T=64, J=4096, D=4096, n=32, R=16, S=64, pack="single", pad=0, save=False),
        # a batch of new prompts and running requests together, in a buffer with rows to spare
        dict(name="fwd_bf16_mixed", op="forward", dtype="bf16", T=640, J=8192, D=2048, n=16, R=32, S=40, pack="ragged", pad=64, save=False),
        # packed sequences of a training step, activations of the adapters kept for the backward pass
        dict(name="fwd_bf16_prompts", op="forward", dtype="bf16", T=8192, J=4096, D=4096, n=8, R=64, S=24, pack="ragged", pad=0, save=True),
        # fp32 rows at sizes as data sets have them
        dict(name="fwd_f32_ragged", op="forward", dtype="f32", T=777, J=1003, D=2047, n=6, R=12, S=9, pack="ragged", pad=0, save=True),
        # the training step's backward pass, with what the forward kept
        dict(name="bwd_bf16_train", op="backward", dtype="bf16", T=8192, J=4096, D=4096, n=8, R=16, S=24, pack="ragged", pad=0, save=True),
        # fine-tuning on a few short sequences, nothing kept
        dict(name="bwd_bf16_short", op="backward", dtype="bf16", T=200, J=1000, D=520, n=3, R=8, S=7, pack="ragged", pad=8, save=False),
        # fp32 at the size of the metric-learning workload
        dict(name="bwd_f32", op="backward", dtype="f32", T=512, J=1024, D=4096, n=4, R=16, S=8, pack="ragged", pad=0, save=True),
        # the gradients of adapters at seven projections of 32 layers
        dict(name="norm_adapters", op="norm", count=448, low=16 * 1024, high=16 * 8192, half=0.0, max_norm=1.0),
        # the gradients of a whole model of some large and many small tensors, fp32 and bf16
        dict(name="norm_model", op="norm", count=150, low=1000, high=40000000, half=0.5, max_norm=1.0),
        # a handful of small tensors: latency
        dict(name="clip_small", op="clip", count=6, low=64, high=20000, half=0.0, max_norm=1.0),
        # clipping of some hundred tensors of odd sizes
        dict(name="clip_mixed", op="clip", count=300, low=501, high=4000000, half=0.3, max_norm=1.0),
    ]


def draw(rng):
    def log(lo, hi, step=1):
        return max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step)

    op = rng.choice(["forward", "forward", "backward", "backward", "norm", "clip"])
    if op in ("norm", "clip"):
        low = log(1, 20000)
        high = low * log(1, 200)
        return dict(op=op, count=log(1, min(500, max(1, 300000000 // high))), low=low, high=high,
                    half=rng.choice([0.0, 0.3, 1.0]), max_norm=rng.choice([0.1, 1.0, 1e6]))
    dtype = rng.choice(["bf16", "bf16", "f32"])
    step = 8 if dtype == "bf16" else 1
    J, D = log(64, 8192, step), log(64, 8192, step)
    T = log(1, 8192)
    # no more work in all than the largest listed case of its type
    T = max(1, min(T, int((2.7e11 if dtype == "bf16" else 1e10) / (2 * J * D))))
    n = log(1, 64)
    pack = "single" if T <= 512 and rng.random() < 0.4 else "ragged"
    S = T if pack == "single" else log(1, min(T, 64))
    return dict(op=op, dtype=dtype, T=T, J=J, D=D, n=n, R=log(1, 128), S=S, pack=pack, pad=rng.choice([0, 0, 5]),
                save=rng.random() < 0.5)


def _sizes(case):
    """Elements of the tensors of a list, over the whole range on a logarithmic scale; their order of sizes is mixed."""
    n = case["count"]
    steps = [((k * 37) % n) / max(1, n - 1) for k in range(n)] if math.gcd(n, 37) == 1 else [k / max(1, n - 1) for k in range(n)]
    return [int(case["low"] * (case["high"] / case["low"]) ** s) for s in steps]


def _layout(case):
    """Where the tensors lie in the two buffers (fp32, bf16): [(bf16?, offset, elements)], and the buffers' lengths."""
    at, where = [0, 0], []
    for k, size in enumerate(_sizes(case)):
        b = 1 if (k * 0.6180339887) % 1.0 < case["half"] else 0
        where.append((b, at[b], size))
        at[b] += -(-size // 64) * 64
    return where, at


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, sigma=1.0):
        return torch.randn(shape, generator=g, device=DEV).mul_(sigma)

    s = {"case": case}
    if case["op"] in ("norm", "clip"):
        where, total = _layout(case)
        s["flat"] = [torch.zeros(total[0], device=DEV), torch.zeros(total[1], device=DEV, dtype=torch.bfloat16)]
        s["out"] = [torch.zeros_like(f) for f in s["flat"]]
        every = [torch.randn(t, generator=g, device=DEV).mul_(0.02) for t in total]
        s["src"], s["dst"] = [], []
        for b, o, size in where:
            s["src"].append(s["flat"][b][o:o + size])
            s["src"][-1].copy_(every[b][o:o + size])
            s["dst"].append(s["out"][b][o:o + size])
        s["norm"] = torch.zeros(1, device=DEV)
        return s
    T, J, D, n, R, S = (case[k] for k in ("T", "J", "D", "n", "R", "S"))
    dtype = DTYPES[case["dtype"]]
    rows = T + case["pad"]          # the buffers hold rows behind the last request
    if case["pack"] == "single":
        s["start"] = torch.arange(S + 1, device=DEV)
    else:                           # (a request may be empty)
        cuts = torch.randint(0, T + 1, (S + 1,), generator=g, device=DEV).sort().values
        cuts[0], cuts[S] = 0, T
        s["start"] = cuts
    s["adapter"] = torch.randint(0, n, (S,), generator=g, device=DEV, dtype=torch.int32)
    s["adapter"][torch.rand(S, generator=g, device=DEV) < 0.1] = -1         # some requests have none
    s["W"] = normal(J, D, sigma=D ** -0.5).to(dtype)
    s["X"] = normal(rows, D).to(dtype)
    s["U"] = normal(n, R, J, sigma=0.5 * R ** -0.5).to(dtype)
    s["V"] = normal(n, R, D, sigma=D ** -0.5).to(dtype)
    s["ranks"] = torch.randint((R + 1) // 2, R + 1, (n,), generator=g, device=DEV, dtype=torch.int32)
    s["ranks"][0] = R
    s["scale"] = torch.rand(n, generator=g, device=DEV) * 1.5 + 0.5
    if case["op"] == "forward":
        s["Y"] = torch.zeros(rows, J, device=DEV, dtype=dtype)
        s["H"] = torch.zeros(rows, R, device=DEV) if case["save"] else None
        return s
    s["dY"] = normal(rows, J, sigma=0.1).to(dtype)
    s["H"] = None
    if case["save"]:                # what the forward pass has left
        row, mask = _rows(s)
        at = row.clamp(min=0)[:, None] * R + torch.arange(R, device=DEV)
        H = (s["X"][:T].float() @ s["V"].reshape(n * R, D).float().T).gather(1, at) * s["scale"][row.clamp(min=0)][:, None]
        s["H"] = torch.zeros(rows, R, device=DEV)
        s["H"][:T] = torch.where(mask.gather(1, at), H, 0.0)
    s["dX"] = torch.zeros(rows, D, device=DEV, dtype=dtype)
    s["dU"] = torch.zeros(n, R, J, device=DEV)
    s["dV"] = torch.zeros(n, R, D, device=DEV)
    return s


def _rows(s):
    """The adapter of each packed row (-1: none), and which of all n R factor pairs the row uses."""
    c = s["case"]
    n, R = c["n"], c["R"]
    row = s["adapter"].long().repeat_interleave(s["start"].diff(), output_size=c["T"])
    slot = torch.arange(n, device=DEV).repeat_interleave(R)
    used = (torch.arange(R, device=DEV)[None, :] < s["ranks"][:, None]).reshape(-1)
    return row, (row[:, None] == slot[None, :]) & used[None, :]


def _list(s):
    import paper_1409_5705_amd as sfb

    if "list" not in s:             # made once for a set of tensors, as a program keeps it
        s["list"] = sfb.TensorList(s["src"], s["dst"] if s["case"]["op"] == "clip" else None)
    return s["list"]


def _context():
    global _ctx
    if _ctx is None:
        import paper_1409_5705_amd as sfb

        _ctx = sfb.Context(0)
    return _ctx


def run(s):
    c = s["case"]
    if own:
        ctx = _context()
        if c["op"] == "norm":
            ctx.sfb_grad_norm(_list(s), s["norm"])
            return s["norm"]
        if c["op"] == "clip":
            ctx.sfb_clip_grads(_list(s), c["max_norm"], s["norm"])
            return [s["norm"]] + s["out"]
        if c["op"] == "forward":
            ctx.sfb_adapter_forward(s["W"], s["X"], s["start"], s["adapter"], s["U"], s["V"], s["Y"], ranks=s["ranks"],
                                    scale=s["scale"], H=s["H"])
            return [s["Y"]] if s["H"] is None else [s["Y"], s["H"]]
        ctx.sfb_adapter_backward(s["W"], s["X"], s["dY"], s["start"], s["adapter"], s["U"], s["V"], s["dX"], s["dU"], s["dV"],
                                 ranks=s["ranks"], scale=s["scale"], H=s["H"])
        return [s["dX"], s["dU"], s["dV"]]
    if c["op"] in ("norm", "clip"):
        # (the gaps between the tensors hold zeros; squares in 64 bits: the sum is long)
        norm = sum(f.double().square().sum() for f in s["flat"]).sqrt()
        s["norm"].copy_(norm)
        if c["op"] == "norm":
            return s["norm"]
        coef = (c["max_norm"] / norm).clamp(max=1.0).float()
        for f, o in zip(s["flat"], s["out"]):
            o.copy_(f.float() * coef)
        return [s["norm"]] + s["out"]
    T, J, D, n, R = (c[k] for k in ("T", "J", "D", "n", "R"))
    row, mask = _rows(s)
    scale = s["scale"][row.clamp(min=0)][:, None]
    W, X = s["W"].float(), s["X"][:T].float()
    U, V = s["U"].reshape(n * R, J).float(), s["V"].reshape(n * R, D).float()
    at = row.clamp(min=0)[:, None] * R + torch.arange(R, device=DEV)
    if c["op"] == "forward":
        H = torch.where(mask, X @ V.T * scale, 0.0)
        s["Y"][:T] = (X @ W.T + H @ U).to(s["Y"].dtype)
        if s["H"] is None:
            return [s["Y"]]
        s["H"][:T] = torch.where(mask.gather(1, at), H.gather(1, at), 0.0)
        return [s["Y"], s["H"]]
    G = s["dY"][:T].float()
    if s["H"] is None:
        H = torch.where(mask, X @ V.T * scale, 0.0)
    else:
        H = torch.where(mask, s["H"][:T].repeat(1, n), 0.0)
    dH = torch.where(mask, G @ U.T * scale, 0.0)
    s["dX"][:T] = (G @ W + dH @ V).to(s["dX"].dtype)
    s["dU"].copy_((H.T @ G).view(n, R, J))
    s["dV"].copy_((dH.T @ X).view(n, R, D))
    return [s["dX"], s["dU"], s["dV"]]


def work(case):
    if case["op"] in ("norm", "clip"):
        where, _ = _layout(case)
        total = sum(size * (2 if b else 4) for b, _, size in where)
        return {"bytes": total * (2 if case["op"] == "clip" else 1) + 4, "flops": 2 * sum(w[2] for w in where)}
    T, J, D, n, R, S = (case[k] for k in ("T", "J", "D", "n", "R", "S"))
    e = 2 if case["dtype"] == "bf16" else 4
    factors = min(n, S) * R * (J + D)
    if case["op"] == "forward":
        return {"bytes": e * (T * D + J * D + factors + T * J) + (4 * T * R if case["save"] else 0),
                "flops": 2 * T * J * D + 2 * T * R * (J + D)}
    return {"bytes": e * (T * J + T * D + J * D + factors + T * D) + (4 * T * R if case["save"] else 0) + 4 * n * R * (J + D),
            "flops": 2 * T * J * D + 2 * T * R * (J + D) * 2 + (0 if case["save"] else 2 * T * R * D)}


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] in ("norm", "clip"):
        total = torch.zeros((), dtype=f64, device=DEV)
        for t in s["src"]:
            total += t.to(f64).pow(2).sum()
        norm = total.sqrt()
        if case["op"] == "norm":
            return norm.view(1)
        coef = min(1.0, case["max_norm"] / norm.item()) if norm.item() > 0 else 1.0
        return [norm.view(1)] + [f.to(f64) * coef for f in s["flat"]]
    T, J, D, n, R, S = (case[k] for k in ("T", "J", "D", "n", "R", "S"))
    rows = T + case["pad"]
    start, adapter, ranks = s["start"].tolist(), s["adapter"].tolist(), s["ranks"].tolist()
    X, W = s["X"].to(f64), s["W"].to(f64)
    of = {}                          # adapter: its rows, request by request
    for q in range(S):
        of.setdefault(adapter[q], []).extend(range(start[q], start[q + 1]))
    forward = case["op"] == "forward"
    src, other = (X, W.t().contiguous()) if forward else (s["dY"].to(f64), W)
    out = torch.zeros(rows, J if forward else D, dtype=f64, device=DEV)
    out[:T] = src[:T] @ other
    kept = torch.zeros(rows, R, dtype=f64, device=DEV)
    dU = torch.zeros(n, R, J, dtype=f64, device=DEV)
    dV = torch.zeros(n, R, D, dtype=f64, device=DEV)
    for a, at in of.items():
        if a < 0 or not at:
            continue
        at = torch.tensor(at, device=DEV)
        r = ranks[a]
        U, V, scale = s["U"][a, :r].to(f64), s["V"][a, :r].to(f64), s["scale"][a].to(f64)
        if forward or s["H"] is None:
            h = X[at] @ V.t().contiguous() * scale
        else:
            h = s["H"][at, :r].to(f64)
        if forward:
            out[at] += h @ U
            kept[at, :r] = h
            continue
        G = src[at]
        dh = G @ U.t().contiguous() * scale
        out[at] += dh @ V
        dU[a, :r] = h.t().contiguous() @ G
        dV[a, :r] = dh.t().contiguous() @ X[at]
    if not forward:
        return [out, dU, dV]
    return [out, kept] if case["save"] else [out]
