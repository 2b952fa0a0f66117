"""Factor blocks beside a shared matrix (sfb_adapter_forward, sfb_adapter_backward) against the formulas in 64 bits: lengths from
none to many tiles, odd sizes, ranks from 0 to 256, blocks shared by requests, rows of no request, and not-a-numbers in
every place that the calls must not look at."""
import numpy as np
import pytest
import torch

import adapter_ref as A

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
SENTINEL = 12345.0


@pytest.fixture(scope="module")
def sfb():
    import paper_1409_5705_amd as m
    m.lib()
    return m


@pytest.fixture(scope="module")
def ctx(sfb):
    c = sfb.Context(0)
    yield c
    c.close()


KEYS = ("W", "X", "dY", "U", "V", "start", "adapter", "ranks", "scale")


def to_dev(c):
    return {k: c[k].to("cuda:0") for k in KEYS}


def outputs(c):
    full = lambda *s, dt=F32: torch.full(s, SENTINEL, dtype=dt, device="cuda:0")  # noqa: E731
    return dict(Y=full(c["T"], c["J"], dt=c["dtype"]), H=full(c["T"], c["R"]), dX=full(c["T"], c["D"], dt=c["dtype"]),
                dU=full(c["n"], c["R"], c["J"]), dV=full(c["n"], c["R"], c["D"]))


def forward(ctx, d, o, W=None, H=True):
    ctx.sfb_adapter_forward(d["W"] if W is None else W, d["X"], d["start"], d["adapter"], d["U"], d["V"], o["Y"], ranks=d["ranks"],
                            scale=d["scale"], H=o["H"] if H else None)


def backward(ctx, d, o, W=None, H=None):
    ctx.sfb_adapter_backward(d["W"] if W is None else W, d["X"], d["dY"], d["start"], d["adapter"], d["U"], d["V"], o["dX"], o["dU"],
                             o["dV"], ranks=d["ranks"], scale=d["scale"], H=H)


def compare(c, o, names=("Y", "H", "dX", "dU", "dV")):
    ref, rows = A.reference(c)
    outside = torch.ones(c["T"], dtype=torch.bool)
    outside[rows] = False
    for k in names:
        per_row = k in ("Y", "H", "dX")
        A.check(k, o[k], ref, rows if per_row else None)
        if per_row and outside.any():           # as they were
            assert bool((o[k].cpu()[outside] == o[k].new_full((1,), SENTINEL).cpu()).all()), k


CASES = [
    # T, J, D, n, R, S, single, first, behind
    (1, 64, 64, 1, 1, 1, True, 0, 0),
    (1, 1000, 520, 4, 16, 1, True, 0, 0),
    (5, 72, 8, 3, 8, 5, True, 0, 0),
    (33, 8, 136, 2, 17, 3, False, 0, 0),
    (64, 1032, 264, 20, 16, 64, True, 0, 0),
    (70, 264, 1032, 20, 33, 60, True, 3, 7),
    (129, 136, 200, 5, 64, 9, False, 0, 0),
    (257, 520, 328, 3, 40, 2, False, 1, 0),
    (300, 256, 512, 2, 256, 6, False, 0, 20),
    (515, 392, 72, 7, 100, 130, False, 0, 3),
    (700, 128, 640, 40, 5, 200, False, 0, 0),
    (1100, 520, 264, 1, 12, 1, False, 0, 0),
    (2600, 264, 520, 2, 40, 7, False, 5, 9),
    (12, 1032, 1032, 40, 256, 7, False, 0, 0),
    (128, 2056, 1536, 9, 33, 100, False, 2, 1),
    (256, 2056, 1544, 9, 33, 12, False, 0, 1),
]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_forward_and_backward(ctx, case, dtype):
    T, J, D, n, R, S, single, first, behind = case
    print("adapter", case, dtype, flush=True)
    c = A.poison(A.make(T, J, D, n, R, S, dtype, seed=T + R, single=single, first=first, behind=behind))
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    backward(ctx, d, o)                       # projections computed again
    compare(c, o)
    p = outputs(c)
    p["H"] = o["H"]
    p["H"][torch.isnan(p["H"])] = 0
    backward(ctx, d, p, H=p["H"])             # and the forward call's taken
    compare(c, p, ("dX", "dU", "dV"))
    q = outputs(c)
    forward(ctx, d, q, H=False)
    assert torch.equal(q["Y"], o["Y"])
    assert bool((q["H"] == SENTINEL).all())


@pytest.mark.parametrize("J,D,n,R,S", [(4104, 72, 5, 24, 9), (72, 4104, 5, 24, 9), (4104, 136, 30, 70, 300), (200, 4360, 30, 70, 300), (264, 328, 5, 70, 9), (4360, 328, 5, 7, 20)])
def test_many_tiles(ctx, J, D, n, R, S):
    """Outputs of more tiles than the chip has compute units, rows of no request in the first and in the last ones."""
    c = A.poison(A.make(4200, J, D, n, R, S, BF16, seed=J + S, first=3, behind=260))
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    backward(ctx, d, o, H=o["H"])
    compare(c, o)


@pytest.mark.parametrize("T,J,D,n,R,S,dtype", [(8100, 4088, 264, 5, 20, 9, BF16), (8100, 264, 4088, 5, 20, 9, BF16), (520, 2056, 4096, 4, 12, 8, BF16),
                                               (9000, 136, 200, 3, 24, 40, BF16), (9000, 136, 200, 30, 40, 3000, BF16), (9000, 72, 131, 1, 5, 40, F32),
                                               (40000, 72, 64, 40, 8, 50, BF16), (385, 4104, 72, 5, 24, 40, BF16), (4601, 136, 200, 3, 24, 700, F32)])
def test_long_batches(ctx, T, J, D, n, R, S, dtype):
    """Large tiles in more than one round, parts of k, blocks whose rows lie far apart, one gradient of rows in several parts."""
    c = A.poison(A.make(T, J, D, n, R, S, dtype, seed=T + S, first=min(700, T // 8), behind=T // 30))
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    backward(ctx, d, o)
    compare(c, o)


@pytest.mark.parametrize("T,J,D,n,R", [(90, 1003, 2047, 2, 12), (90, 65, 63, 3, 5), (90, 2, 3, 2, 1), (90, 130, 1, 1, 7),
                                       (900, 1003, 1001, 2, 12), (1200, 1004, 601, 2, 3), (1200, 601, 1004, 2, 3), (1200, 1002, 603, 2, 3)])
def test_fp32_odd_sizes(ctx, T, J, D, n, R):
    c = A.poison(A.make(T, J, D, n, R, 4, F32, seed=J, behind=2))
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    backward(ctx, d, o)
    compare(c, o)


@pytest.mark.parametrize("T,J,D,n,R,S", [(0, 64, 64, 2, 4, 0), (9, 64, 64, 2, 4, 0), (9, 64, 64, 2, 7, 0), (9, 64, 72, 0, 4, 3), (40, 64, 64, 3, 4, 8), (300, 64, 64, 3, 5, 8)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_nothing_there(ctx, T, J, D, n, R, S, dtype):
    """No rows, no requests, no blocks, blocks of rank 0: outputs of rows that belong to requests are the shared matrix's alone,
    gradients zeros."""
    c = A.make(T, J, D, n, R, S, dtype, seed=1)
    if S == 8:
        c["ranks"][:] = 0
    if S == 0:
        c["start"] = torch.tensor([T])
    A.poison(c)
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    backward(ctx, d, o)
    compare(c, o)
    backward(ctx, d, o, H=torch.zeros_like(o["H"]))          # (nothing of H is in use either)
    compare(c, o)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_numbers_out_of_range(ctx, dtype):
    """Blocks outside the pool are none, ranks are clamped; no ranks and no scale: all pairs, 1."""
    c = A.make(60, 72, 136, 3, 9, 6, dtype, seed=4, none=0)
    c["adapter"] = torch.tensor([5, 0, -7, 3, 2, 1], dtype=torch.int32)
    c["ranks"] = torch.tensor([99, -4, 9], dtype=torch.int32)
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    backward(ctx, d, o)
    compare(c, o)
    c["ranks"][:], c["scale"][:] = 9, 1.0
    d, o = to_dev(c), outputs(c)
    d["ranks"] = d["scale"] = None
    forward(ctx, d, o)
    backward(ctx, d, o)
    compare(c, o)


@pytest.mark.parametrize("layout", ["copy", "planes"])
@pytest.mark.parametrize("T,J,D", [(3, 520, 200), (150, 264, 328), (400, 1000, 72), (520, 1000, 392), (600, 264, 2056), (8100, 4088, 264),
                                   (8100, 264, 4088)])
def test_attached_matrix(sfb, layout, T, J, D):
    """bf16 blocks beside the fp32 matrix that a context keeps a bf16 copy or two planes of."""
    c = A.make(T, J, D, 3, 16, 3, BF16, seed=8)
    W = torch.randn(J, D, generator=torch.Generator().manual_seed(2)) * D ** -0.5
    own = sfb.Context(0)
    Wd = W.to("cuda:0")
    (own.sfb_shadow_attach if layout == "copy" else own.sfb_split_attach)(Wd)
    # (the planes' high halves round ties away from zero)
    c["W"] = W.to(BF16) if layout == "copy" else ((W.view(torch.int32) + 0x8000) >> 16).to(torch.int16).view(BF16)
    d, o = to_dev(c), outputs(c)
    forward(own, d, o, W=Wd)
    backward(own, d, o, W=Wd)
    compare(c, o)
    own.close()


def test_block_is_what_apply_would_make(ctx, sfb):
    """W + scale U^T V by sfb_apply, and the projection with it, against the block beside W."""
    T, J, D, R = 65, 264, 520, 12
    c = A.make(T, J, D, 1, R, 1, F32, seed=5, none=0)
    c["adapter"][:] = 0
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    merged = d["W"].clone()
    s = float(c["scale"][0])
    ctx.sfb_apply(merged, d["U"][0].contiguous(), d["V"][0].contiguous(), -s)
    plain = outputs(c)
    ctx.sfb_adapter_forward(merged, d["X"], d["start"], torch.full_like(d["adapter"], -1), d["U"], d["V"], plain["Y"])
    ref, _ = A.reference(c)
    # both are within the fp32 bound of the exact value; the merged matrix is rounded once more (2^-24 of each element)
    extra = 2.0 ** -24 * (np.abs(c["X"].double().numpy()) @ np.abs(merged.cpu().double().numpy()).T)
    assert np.all(np.abs((plain["Y"] - o["Y"]).cpu().double().numpy()) <= 2 * ref["Y_tol"] + extra + 2.0 ** -22 * np.abs(ref["Y"]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,S,J,D", [(24, 24, 136, 200), (300, 12, 136, 200), (300, 12, 136, 40), (4200, 900, 4104, 40), (4200, 12, 40, 4104)])
def test_what_is_not_finite_stays_in_its_row(ctx, dtype, T, S, J, D):
    """Infinities and not-a-numbers in one request's rows or block do not reach the rows of others."""
    n, R = 4, 8
    c = A.make(T, J, D, n, R, S, dtype, seed=11, single=S == T, none=0)
    c["ranks"][:] = R
    c["adapter"] = (torch.arange(S) % n).to(torch.int32)
    ref, rows = A.reference(c)
    by, _ = A.rows_of(c)
    bad = by.get(1, [])
    good = sorted(set(rows) - set(bad))
    c["U"][1, 2, 5] = float("inf")
    c["V"][1, 3, 7] = float("nan")
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    backward(ctx, d, o)
    for k in ("Y", "dX"):
        A.check(k, o[k], ref, good)
    others = [0, 2, 3]
    for k in ("dU", "dV"):
        got = {k: torch.tensor(0)}
        A.check(k, o[k][others], {k: ref[k][others], k + "_tol": ref[k + "_tol"][others]})
    assert bool(torch.isnan(o["Y"][bad].float()).any())
    # an infinity in a factor is an infinity of the sum, not a not-a-number
    c = A.make(T, J, D, n, R, S, dtype, seed=12, single=S == T, none=0)
    c["ranks"][:] = R
    c["U"][:, 2, 5] = float("inf")
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    h = o["H"].cpu()
    assert bool((torch.isinf(o["Y"].cpu()[:, 5].float()) | (h[:, 2] == 0)).all())
    assert bool((torch.sign(o["Y"].cpu()[:, 5].float()) == torch.sign(h[:, 2])).all())


def test_gradients_against_differences(ctx):
    """d/ds of sum(Y * G) along random directions of X, U and V, by central differences of the forward call in fp32."""
    T, J, D, n, R, S = 40, 48, 56, 3, 6, 5
    c = A.make(T, J, D, n, R, S, F32, seed=21)
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    backward(ctx, d, o)
    g = torch.Generator(device="cuda:0").manual_seed(3)
    for name, grad in (("X", "dX"), ("U", "dU"), ("V", "dV")):
        step = torch.randn(d[name].shape, generator=g, device="cuda:0")
        loss = []
        for sign in (1, -1):
            e = dict(d)
            e[name] = d[name] + sign * 2.0 ** -4 * step
            p = outputs(c)
            forward(ctx, e, p)
            loss.append((p["Y"].double() * d["dY"].double()).sum().item())
        # Y is linear in each of them alone: the difference is exact but for the two sums' rounding
        got, want = (o[grad].double() * step.double()).sum().item(), (loss[0] - loss[1]) * 2.0 ** 3
        ref, _ = A.reference(c)
        room = 2.0 ** 5 * float((ref["Y_tol"] * 4 * np.abs(c["dY"].double().numpy())).sum())
        assert abs(got - want) <= room + 1e-4 * abs(want), (name, got, want, room)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,S,single", [(16, 16, True), (300, 6, False)])
def test_graph_replays_other_batches(sfb, dtype, T, S, single):
    """One captured forward and backward serves batches of other compositions; a second graph and eager calls in between."""
    J, D, n, R = 264, 328, 4, 16
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = sfb.Context(0)
        c = A.make(T, J, D, n, R, S, dtype, seed=31, single=single)
        d, o = to_dev(c), outputs(c)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            forward(ctx, d, o)
            backward(ctx, d, o, H=o["H"])
        big = A.make(4 * T, J, D, n, R, 3, dtype, seed=32)          # the workspace grows after the capture
        db, ob = to_dev(big), outputs(big)
        forward(ctx, db, ob)
        side.synchronize()
        for k in range(4):
            other = A.make(T, J, D, n, R, S, dtype, seed=40 + k, single=single, behind=0 if single else k)
            for key in KEYS:
                d[key].copy_(other[key].to("cuda:0"))
            for key in o:
                o[key].fill_(SENTINEL)
            graph.replay()
            side.synchronize()
            got = {key: v.clone() for key, v in o.items()}
            compare(other, got)
            e = outputs(other)
            forward(ctx, d, e)
            backward(ctx, d, e, H=e["H"])
            forward(ctx, db, ob)
            side.synchronize()
            for key in o:
                assert torch.equal(e[key], got[key]), key          # the same bits
    ctx.close()


def test_wrong_arguments(sfb, ctx):
    c = A.make(20, 64, 72, 2, 8, 3, BF16, seed=1)
    d, o = to_dev(c), outputs(c)
    for key, bad in (("X", d["X"][:, :64]), ("X", d["X"].float()), ("U", d["U"].float()), ("start", d["start"].int()),
                     ("start", d["start"][:-1]), ("adapter", d["adapter"].long()), ("ranks", d["ranks"][:1]),
                     ("scale", d["scale"].double()), ("W", d["W"].t())):
        e = dict(d)
        e[key] = bad
        with pytest.raises((TypeError, ValueError)):
            forward(ctx, e, o)
    with pytest.raises(sfb.SfbError) as err:          # an fp32 matrix that is not attached, beside bf16 blocks
        forward(ctx, d, o, W=d["W"].float())
    assert err.value.code == sfb.SFB_EINVAL
    with pytest.raises((TypeError, ValueError)):
        forward(ctx, d, dict(o, Y=o["Y"][:10]))
    with pytest.raises((TypeError, ValueError)):
        backward(ctx, d, dict(o, dU=o["dU"].to(BF16)))
    with pytest.raises(sfb.SfbError):                 # one of the two gradients
        ctx.sfb_adapter_backward(d["W"], d["X"], d["dY"], d["start"], d["adapter"], d["U"], d["V"], dU=o["dU"])
    torch.cuda.synchronize()
    assert bool((o["Y"] == o["Y"].new_full((1,), SENTINEL)).all())


def test_output_over_input(ctx):
    c = A.make(20, 64, 64, 2, 8, 3, BF16, seed=1)
    d, o = to_dev(c), outputs(c)
    with pytest.raises(ValueError):
        forward(ctx, d, dict(o, Y=d["X"]))
    for key in ("dY", "X"):
        with pytest.raises(ValueError):
            backward(ctx, d, dict(o, dX=d[key]))
    torch.cuda.synchronize()
    for key in ("X", "dY"):
        assert torch.equal(d[key].cpu(), c[key])


def test_large_offsets(ctx):
    """Buffers of more than 2^31 elements: the last rows of X and the last blocks of the pool."""
    T, J, D, n, R = 70000, 64, 32768, 1100, 64
    X = torch.zeros(T, D, dtype=BF16, device="cuda:0")
    V = torch.zeros(n, R, D, dtype=BF16, device="cuda:0")
    U = torch.zeros(n, R, J, dtype=BF16, device="cuda:0")
    W = torch.zeros(J, D, dtype=BF16, device="cuda:0")
    X[-1, -8:], V[-1, :, -4:], U[-1], W[:, -2:] = 1.0, 0.5, 0.25, 2.0
    start = torch.tensor([T - 40, T - 3, T], device="cuda:0")
    adapter = torch.tensor([0, n - 1], dtype=torch.int32, device="cuda:0")
    Y = torch.zeros(T, J, dtype=BF16, device="cuda:0")
    ctx.sfb_adapter_forward(W, X, start, adapter, U, V, Y)
    torch.cuda.synchronize()
    want = torch.zeros(3, J)
    want[-1] = 4.0 + 64 * 2.0 * 0.25
    assert torch.equal(Y[-3:].float().cpu(), want)
    assert float(Y[:-3].float().abs().max()) == 0.0
    del X, V, U, W, Y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,S,J,D,R", [(40, 5, 136, 200, 8), (700, 9, 136, 200, 20), (700, 9, 136, 200, 70)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinities_of_the_rows(ctx, dtype, T, S, J, D, R):
    """An infinity in a row of dY or X is one of the same sign in the gradients it enters, not a not-a-number, and reaches no
    other block's."""
    n = 3
    c = A.make(T, J, D, n, R, S, dtype, seed=T + R, none=0)
    c["ranks"][:] = R
    c["adapter"] = (torch.arange(S) % n).to(torch.int32)
    ref, rows = A.reference(c)
    by, _ = A.rows_of(c)
    t = by[1][len(by[1]) // 2]
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    h = o["H"][t].cpu()
    assert bool((h != 0).all())
    d["dY"][t, 17] = float("inf")
    ctx.sfb_adapter_backward(d["W"], d["X"], d["dY"], d["start"], d["adapter"], d["U"], d["V"], None, o["dU"], o["dV"], ranks=d["ranks"],
                             scale=d["scale"], H=o["H"])
    got = o["dU"][1].cpu()
    assert bool((got[:, 17] == torch.sign(h) * float("inf")).all())
    keep = torch.ones(J, dtype=torch.bool)
    keep[17] = False
    A.check("dU", got[:, keep], {"dU": ref["dU"][1][:, keep.numpy()], "dU_tol": ref["dU_tol"][1][:, keep.numpy()]})
    for k in ("dU", "dV"):
        A.check(k, o[k][[0, 2]], {k: ref[k][[0, 2]], k + "_tol": ref[k + "_tol"][[0, 2]]})
    d = to_dev(c)
    d["X"][t, 5] = float("-inf")
    ctx.sfb_adapter_backward(d["W"], d["X"], d["dY"], d["start"], d["adapter"], d["U"], d["V"], None, o["dU"], o["dV"], ranks=d["ranks"],
                             scale=d["scale"], H=o["H"])
    dh = float(c["scale"][1]) * (c["dY"][t].double() @ c["U"][1].double().T)
    assert bool((o["dV"][1][:, 5].cpu() == torch.sign(dh).float() * float("-inf")).all())
    A.check("dV", o["dV"][[0, 2]], {"dV": ref["dV"][[0, 2]], "dV_tol": ref["dV_tol"][[0, 2]]})


@pytest.mark.parametrize("T", [30, 400])
def test_two_contexts_on_two_streams(sfb, T):
    """Contexts of their own on side streams, at work at the same time; inputs made on the default stream."""
    c = A.make(T, 264, 328, 4, 16, 5, BF16, seed=6)
    ref, rows = A.reference(c)
    d = to_dev(c)
    torch.cuda.synchronize()
    runs = []
    for _ in range(2):
        stream = torch.cuda.Stream()
        own = sfb.Context(0, stream=stream)
        runs.append((stream, own, outputs(c)))
    torch.cuda.synchronize()
    for _ in range(5):
        for stream, own, o in runs:           # the current stream is the default one throughout
            forward(own, d, o)
            backward(own, d, o, H=o["H"])
    torch.cuda.synchronize()
    for stream, own, o in runs:
        compare(c, o)
        own.close()


@pytest.mark.parametrize("T", [20, 200, 900])
@pytest.mark.parametrize("start", [[5, 3, 10, 2], [-7, 4, 2000, 9], [3, 2 ** 40, -2 ** 40, 8], [900, 0, 900, 0]])
def test_starts_that_are_not_in_order(ctx, T, start):
    """What start may not hold: the results are unspecified, but nothing in front of and behind the outputs is touched."""
    c = A.make(T, 72, 136, 3, 20, 3, BF16, seed=9)
    c["start"] = torch.tensor(start)
    d = to_dev(c)
    wide = {}
    o = {}
    for k, v in outputs(c).items():
        wide[k] = torch.full((v.numel() + 1024,), SENTINEL, dtype=v.dtype, device="cuda:0")
        o[k] = wide[k][512:512 + v.numel()].view(v.shape)
    forward(ctx, d, o)
    backward(ctx, d, o, H=o["H"])
    backward(ctx, d, o)
    torch.cuda.synchronize()
    for k, w in wide.items():
        assert bool((w[:512] == w.new_full((1,), SENTINEL)).all()) and bool((w[-512:] == w.new_full((1,), SENTINEL)).all()), k


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [48, 900])
def test_training_steps(sfb, dtype, T):
    """Adapters trained beside a frozen matrix, as a program does it: forward, the gradient of a squared error, backward, the norm
    over the gradients of two projections and their clipping, the step; eagerly and from a graph, each step against 64 bits."""
    J, D, n, R, S, lr, bound = 72, 136, 3, 6, 4, 0.05, 0.5
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        own = sfb.Context(0)
        first = A.make(T, D, J, n, R, S, dtype, seed=50)          # J -> D, then D -> J
        second = A.make(T, J, D, n, R, S, dtype, seed=51)
        for k in ("start", "adapter", "ranks", "scale"):
            second[k] = first[k]
        a, b = to_dev(first), to_dev(second)
        target = torch.randn(T, J, generator=torch.Generator().manual_seed(3)).to("cuda:0")
        Ha, Hb = (torch.zeros(T, R, device="cuda:0") for _ in range(2))
        X1 = torch.zeros(T, D, device="cuda:0", dtype=dtype)
        Y = torch.zeros(T, J, device="cuda:0", dtype=dtype)
        dX1, G = torch.zeros_like(X1), torch.zeros_like(Y)
        grads = [torch.zeros(n, R, k, device="cuda:0") for k in (D, J, J, D)]
        lst, norm = sfb.TensorList(grads), torch.zeros(1, device="cuda:0")
        params = [a["U"], a["V"], b["U"], b["V"]]
        start = [p.clone() for p in params]
        common = dict(ranks=a["ranks"], scale=a["scale"])

        def step():
            own.sfb_adapter_forward(a["W"], a["X"], a["start"], a["adapter"], a["U"], a["V"], X1, H=Ha, **common)
            own.sfb_adapter_forward(b["W"], X1, a["start"], a["adapter"], b["U"], b["V"], Y, H=Hb, **common)
            G.copy_((Y.float() - target) / T)
            own.sfb_adapter_backward(b["W"], X1, G, a["start"], a["adapter"], b["U"], b["V"], dX1, grads[2], grads[3], H=Hb, **common)
            own.sfb_adapter_backward(a["W"], a["X"], dX1, a["start"], a["adapter"], a["U"], a["V"], None, grads[0], grads[1], H=Ha, **common)
            own.sfb_clip_grads(lst, bound, norm)
            for p, g in zip(params, grads):
                p.copy_(p.float() - lr * g)

        def check(before):
            """The step from `before` by the formulas, each part from the call's own inputs."""
            c2 = dict(second, X=X1.cpu(), dY=G.cpu(), U=before[2].cpu(), V=before[3].cpu())
            r2, rows = A.reference(c2)
            A.check("Y", Y, r2, rows)
            A.check("dX", dX1, r2, rows)
            c1 = dict(first, X=a["X"].cpu(), dY=dX1.cpu(), U=before[0].cpu(), V=before[1].cpu())
            r1, _ = A.reference(c1)
            A.check("Y", X1, r1, rows)
            raw = [r1["dU"], r1["dV"], r2["dU"], r2["dV"]]
            tol = [r1["dU_tol"], r1["dV_tol"], r2["dU_tol"], r2["dV_tol"]]
            want = np.sqrt(sum((x * x).sum() for x in raw))
            off = np.sqrt(sum((x * x).sum() for x in tol)) + 2.0 ** -23 * want
            assert abs(norm.item() - want) <= off and want > bound
            coef = bound / want
            for p, q, x, e in zip(params, before, raw, tol):
                new = q.double().cpu().numpy() - lr * coef * x
                room = lr * coef * (e + np.abs(x) * (off / want + 2.0 ** -21)) + 2.0 ** -22 * (np.abs(q.double().cpu().numpy()) + np.abs(new))
                half = 2.0 ** -8 if p.dtype == BF16 else 0.0
                assert np.all(np.abs(p.double().cpu().numpy() - new) <= room * (1 + half) + half * np.abs(new))

        eager = []
        for _ in range(3):
            before = [p.clone() for p in params]
            step()
            side.synchronize()
            check(before)
            eager.append([p.clone() for p in params])
        for p, s in zip(params, start):
            p.copy_(s)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for k in range(3):
            graph.replay()
            side.synchronize()
            for p, e in zip(params, eager[k]):
                assert torch.equal(p, e), k
            assert torch.isfinite(torch.randn(1 << 16, device="cuda:0").sum()).item()
    own.close()


def same_kind(got, want):
    """Not-a-numbers and infinities of either sign in the same places."""
    got, want = got.double().cpu().numpy(), np.asarray(want, dtype=np.float64)
    assert int((np.isnan(got) != np.isnan(want)).sum()) == 0
    for sign in (1, -1):
        assert int(((got == sign * np.inf) != (want == sign * np.inf)).sum()) == 0, sign


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,J,D,S", [(24, 136, 200, 5), (300, 136, 200, 9), (700, 136, 200, 9), (700, 40, 136, 700), (4200, 4104, 40, 60),
                                     (4200, 40, 4104, 60), (8100, 4088, 264, 9), (8100, 264, 4088, 9)])
def test_infinities_of_factors_and_of_projections(ctx, dtype, T, J, D, S):
    """A projection that overflows meets a factor that is infinite, zero or finite: what fp32 products and sums make of it, in
    this row alone, whichever kernel a batch of this size takes."""
    n, R, r = 3, 20, 17
    c = A.make(T, J, D, n, R, S, dtype, seed=T + J, single=S == T, none=0)
    c["ranks"][:] = R
    c["adapter"] = (torch.arange(S) % n).to(torch.int32)
    c["scale"][:] = 1.0
    by, every = A.rows_of(c)
    huge = [by[1][0], by[1][-1], by[2][len(by[2]) // 2]]
    for x, v in (("X", "V"), ("dY", "U")):                # row by row: projections of pair r are +-inf, the shared product stays finite
        c[v][:, :, 7] = 0
        c[v][:, r, 7] = 1e3
        c[x][:, 7] = 0
        c[x][huge, 7] = torch.tensor([2e38, -2e38, 2e38], dtype=dtype)
    c["W"][:, 7] *= 2.0 ** -20
    c["W"][7] *= 2.0 ** -20
    ref = {}
    for x, v, u, out in (("X", "V", "U", "Y"), ("dY", "U", "V", "dX")):
        e = dict(c, **{k: c[k].clone() for k in ("U", "V")})
        e[u][1, r, 3], e[u][1, r, 5], e[u][1, r, 11], e[u][1, r, 13], e[u][1, 2, 20] = float("inf"), float("-inf"), 0, float("nan"), float("inf")
        e[u][2, r, 3] = float("-inf")
        d, o = to_dev(e), outputs(e)
        h = torch.zeros(T, R, dtype=torch.float64)
        if out == "Y":
            forward(ctx, d, o)
            assert torch.equal(torch.isinf(o["H"]).nonzero().cpu(), torch.tensor([[t, r] for t in sorted(huge)]))
            W = c["W"].double().t()
        else:
            ctx.sfb_adapter_backward(d["W"], d["X"], d["dY"], d["start"], d["adapter"], d["U"], d["V"], o["dX"], ranks=d["ranks"], scale=d["scale"])
            W = c["W"].double()
        base = c[x].double() @ W
        for a in range(n):
            t = by[a]
            # (in fp32 the projection of a huge row overflows; everything else is far from that)
            h[t] = c[x][t].double() @ c[v][a].double().t()
            big = h[t].abs() > 1e39
            h[t] = torch.where(big, torch.sign(h[t]) * float("inf"), h[t])
        ref = base.clone()
        for a in range(n):
            t = torch.tensor(by[a])
            for k in range(R):
                ref[t] += h[t][:, k:k + 1] * e[u][a, k].double()[None, :]
        same_kind(o[out][every], ref[every].numpy())


# T, J, D, n, R, S, whether the pool's factors are further columns of the product
POOLS = [(512, 512, 512, 64, 16, 8, True), (512, 512, 512, 64, 128, 8, False), (256, 520, 1032, 64, 16, 30, True), (256, 520, 1032, 500, 16, 30, False),
         (512, 64, 64, 1500, 16, 512, False), (40, 264, 1000, 900, 16, 40, False), (1, 136, 1024, 1500, 16, 1, False)]


@pytest.mark.parametrize("case", POOLS)
def test_pools_on_both_sides(ctx, case):
    """Few rows beside pools small enough to be multiplied whole, and larger ones."""
    T, J, D, n, R, S, _ = case
    c = A.poison(A.make(T, J, D, n, R, S, BF16, seed=T + n, single=S == T))
    d, o = to_dev(c), outputs(c)
    forward(ctx, d, o)
    backward(ctx, d, o)
    compare(c, o)


def test_output_that_overlaps(sfb, ctx):
    """Views that share some rows with an input, and an output of another type at an input's place."""
    T, D, R = 20, 64, 64
    for dtype in (BF16, F32):
        c = A.make(T, 64, D, 2, R, 3, dtype, seed=1)
        d, o = to_dev(c), outputs(c)
        wide = torch.full((T + 8, D), SENTINEL, dtype=dtype, device="cuda:0")
        wide[:T] = d["X"]
        d["X"] = wide[:T]
        calls = [lambda: forward(ctx, d, dict(o, Y=wide[8:])), lambda: forward(ctx, d, dict(o, Y=d["W"][:T])),
                 lambda: backward(ctx, d, dict(o, dX=wide[8:])), lambda: backward(ctx, d, dict(o, dV=o["dU"]))]
        if dtype == F32:
            calls += [lambda: forward(ctx, d, dict(o, H=d["X"])), lambda: backward(ctx, d, o, H=o["dX"]), lambda: forward(ctx, d, dict(o, H=o["Y"]))]
        for call in calls:
            with pytest.raises((ValueError, sfb.SfbError)) as err:
                call()
            assert err.type is ValueError or err.value.code == sfb.SFB_EINVAL
        torch.cuda.synchronize()
        assert torch.equal(wide[:T].cpu(), c["X"]) and bool((wide[T:] == wide.new_full((1,), SENTINEL)).all())
        assert bool((o["dU"] == SENTINEL).all()) and torch.equal(d["W"].cpu(), c["W"])
