"""Norm and clipping of a list of tensors against 64-bit sums: empty and odd sizes, unaligned tensors, many of them, both
types, values whose squares leave fp32, not-finite ones; in place and into other tensors."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


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


def tensors(sizes, seed, bf16=lambda k: k % 3 == 1, offset=lambda k: 0):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    out = []
    for k, n in enumerate(sizes):
        dt = BF16 if bf16(k) else F32
        base = torch.randn(n + offset(k), generator=g, device="cuda:0").to(dt)
        out.append(base[offset(k):])
    return out


def norm64(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def check_clipped(src, dst, coef):
    for s, d in zip(src, dst):
        want = s.double() * coef
        half_step = 2.0 ** -8 if s.dtype == BF16 else 2.0 ** -24
        # the scale itself is rounded to fp32, and the product of fp32 values
        assert bool(((d.double() - want).abs() <= want.abs() * (half_step + 2.0 ** -23) + 1e-40).all())


LISTS = [
    ([1], lambda k: 0),
    ([0, 5, 0], lambda k: 0),
    ([7, 8, 9, 4095, 4096, 4097, 20001], lambda k: 0),
    ([13, 1000, 4099, 70001], lambda k: 1 + k % 3),
    ([3 + 17 * k for k in range(300)], lambda k: k % 2),
    ([5_000_003, 17, 1_234_567, 64], lambda k: 0),
    ([1] * 1500, lambda k: 0),
    ([4097] * 1100, lambda k: 0),
]


@pytest.mark.parametrize("which", range(len(LISTS)))
def test_norm_and_clip(sfb, ctx, which):
    sizes, offset = LISTS[which]
    print("clip", which, flush=True)
    src = tensors(sizes, which, offset=offset)
    before = [t.clone() for t in src]
    dst = [torch.full_like(t, 7.0) for t in src]
    norm = torch.full((1,), -1.0, device="cuda:0")
    want = norm64(src)
    ctx.sfb_grad_norm(sfb.TensorList(src), norm)
    assert abs(norm.item() - want) <= 2.0 ** -24 * want * 1.001
    for bound in (0.0, 0.25 * want, want * 2, float("inf")):
        norm.fill_(-1.0)
        ctx.sfb_clip_grads(sfb.TensorList(src, dst), bound, norm)
        assert abs(norm.item() - want) <= 2.0 ** -24 * want * 1.001
        check_clipped(before, dst, min(1.0, bound / want) if want > 0 else 1.0)
        assert all(torch.equal(a, b) for a, b in zip(src, before))
        if want < bound:
            assert all(torch.equal(a, b) for a, b in zip(dst, before))
    lst = sfb.TensorList(src)
    ctx.sfb_clip_grads(lst, want * 2, norm)                 # within the bound: left alone
    assert all(torch.equal(a, b) for a, b in zip(src, before))
    ctx.sfb_clip_grads(lst, 0.5 * want, norm)
    check_clipped(before, src, 0.5)
    again = norm.clone()
    for s, b in zip(src, before):
        s.copy_(b)
    ctx.sfb_clip_grads(lst, 0.5 * want, norm)
    assert torch.equal(again, norm)


@pytest.mark.parametrize("count", [700, 9000])
@pytest.mark.parametrize("table", [True, False])
def test_many_tensors(sfb, ctx, count, table):
    """More tensors than a launch takes as its arguments, described in device memory or in several launches; more pieces than
    the scaling pass adds up itself."""
    flat = torch.randn(count * 8, generator=torch.Generator(device="cuda:0").manual_seed(count), device="cuda:0")
    out = torch.full_like(flat, 7.0)
    src = [flat[8 * k:8 * k + 1 + k % 8] for k in range(count)]
    dst = [out[8 * k:8 * k + 1 + k % 8] for k in range(count)]
    inside = torch.arange(8, device="cuda:0")[None, :] <= (torch.arange(count, device="cuda:0") % 8)[:, None]
    want = math.sqrt(float((flat.view(count, 8).double() * inside).square().sum()))
    lst, norm = sfb.TensorList(src, dst), torch.zeros(1, device="cuda:0")
    assert lst.table is not None
    if not table:
        lst.table_ptr = None
    ctx.sfb_grad_norm(lst, norm)
    assert abs(norm.item() - want) <= 2.0 ** -24 * want * 1.001
    ctx.sfb_clip_grads(lst, 0.5 * want, norm.zero_())
    assert abs(norm.item() - want) <= 2.0 ** -24 * want * 1.001
    check_clipped([flat[inside.view(-1)]], [out[inside.view(-1)]], 0.5)
    assert bool((out.view(count, 8)[~inside] == 7.0).all())


def test_graph_replays(sfb):
    """Norm and clipping captured once, replayed on other values, against the eager calls."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        own = sfb.Context(0)
        src = tensors([7, 5000, 70001, 33] * 60, 5)
        dst = [torch.zeros_like(t) for t in src]
        lst, norm = sfb.TensorList(src, dst), torch.zeros(1, device="cuda:0")
        own.sfb_clip_grads(lst, 1.0, norm)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            own.sfb_clip_grads(lst, 1.0, norm)
        for k in range(3):
            for t, new in zip(src, tensors([7, 5000, 70001, 33] * 60, 6 + k)):
                t.copy_(new)
            for t in dst:
                t.zero_()
            graph.replay()
            side.synchronize()
            got = [norm.clone()] + [t.clone() for t in dst]
            own.sfb_clip_grads(lst, 1.0, norm)
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, [norm] + dst))
            assert abs(norm.item() - norm64(src)) <= 2.0 ** -23 * norm.item()
        own.close()


def test_empty_list(sfb, ctx):
    norm = torch.full((1,), -1.0, device="cuda:0")
    ctx.sfb_grad_norm(sfb.TensorList([]), norm)
    assert norm.item() == 0.0
    ctx.sfb_clip_grads(sfb.TensorList([torch.empty(0, device="cuda:0")]), 1.0, norm.fill_(-1.0))
    assert norm.item() == 0.0


@pytest.mark.parametrize("value", [3e38, 1e30, 1e-30, 1e-44])
def test_squares_outside_fp32(sfb, ctx, value):
    t = torch.full((1000,), value, device="cuda:0")
    want = norm64([t])
    norm = torch.zeros(1, device="cuda:0")
    out = torch.zeros_like(t)
    ctx.sfb_clip_grads(sfb.TensorList([t], [out]), 1.0, norm)
    if want < torch.finfo(F32).max:
        assert abs(norm.item() - want) <= 2.0 ** -24 * want + 1.5e-45
    else:
        assert math.isinf(norm.item())                      # beyond fp32, and still clipped to 1
    check_clipped([t], [out], min(1.0, 1.0 / want))
    if want > 1:
        assert abs(norm64([out]) - 1.0) < 1e-5


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 1, 4999])
def test_not_finite(sfb, ctx, bad, at):
    a, b = torch.ones(5000, device="cuda:0"), torch.ones(5000, device="cuda:0", dtype=BF16)
    (a if at != 1 else b)[at] = bad
    norm = torch.zeros(1, device="cuda:0")
    ctx.sfb_clip_grads(sfb.TensorList([a, b]), 1.0, norm)
    assert norm.item() == bad or (math.isnan(bad) and math.isnan(norm.item()))
    rest = torch.ones(5000, dtype=torch.bool, device="cuda:0")
    rest[at] = False
    for t in (a, b):
        assert bool((t[rest] == 0).all() if math.isinf(bad) else torch.isnan(t).all())


def test_more_than_2_31_elements(sfb, ctx):
    n = (1 << 31) + 5
    t = torch.zeros(n, device="cuda:0", dtype=BF16)
    t[-1], t[0] = 3.0, 4.0
    norm = torch.zeros(1, device="cuda:0")
    ctx.sfb_clip_grads(sfb.TensorList([t]), 1.0, norm)
    assert norm.item() == 5.0
    assert abs(t[-1].item() - 0.6) <= 0.6 * 2.0 ** -8 and abs(t[0].item() - 0.8) <= 0.8 * 2.0 ** -8
    del t
    torch.cuda.empty_cache()


def test_wrong_arguments(sfb, ctx):
    a = torch.ones(10, device="cuda:0")
    norm = torch.zeros(1, device="cuda:0")
    with pytest.raises(TypeError):
        sfb.TensorList([a.double()])
    with pytest.raises(TypeError):
        sfb.TensorList([torch.ones(3)])
    with pytest.raises(ValueError):
        sfb.TensorList([torch.ones(4, 4, device="cuda:0").t()])
    with pytest.raises(ValueError):
        sfb.TensorList([a], [a, a])
    with pytest.raises((TypeError, ValueError)):
        sfb.TensorList([a], [a.to(BF16)])
    for bound in (-1.0, float("nan")):
        with pytest.raises(sfb.SfbError) as e:
            ctx.sfb_clip_grads(sfb.TensorList([a]), bound, norm)
        assert e.value.code == sfb.SFB_EINVAL
    with pytest.raises((TypeError, ValueError)):
        ctx.sfb_grad_norm(sfb.TensorList([a]), norm.double())
    assert bool((a == 1).all())


def test_overlapping_tensors(sfb, ctx):
    """A tensor listed twice counts twice in the norm, and is not clipped: whose scaling is to come first?"""
    a, b = tensors([1000, 500], seed=8, bf16=lambda k: False)
    norm = torch.zeros(1, device="cuda:0")
    ctx.sfb_grad_norm(sfb.TensorList([a, b, a]), norm)
    assert abs(norm.item() - norm64([a, b, a])) <= 2.0 ** -23 * norm64([a, b, a])
    keep = [a.clone(), b.clone()]
    whole = torch.zeros(2000, device="cuda:0")
    for src, dst in (([a, b, a], None), ([a, a[10:20]], None), ([b, a], [a[:500], torch.empty_like(a)]),
                     ([a, a], [whole[:1000], whole[999:1999]])):
        with pytest.raises(ValueError):
            ctx.sfb_clip_grads(sfb.TensorList(src, dst), 1.0, norm)
    assert torch.equal(a, keep[0]) and torch.equal(b, keep[1]) and not bool(whole.any())
    ctx.sfb_clip_grads(sfb.TensorList([a, a], [whole[:1000], whole[1000:]]), 1.0, norm)          # read twice: two results
    assert torch.equal(whole[:1000], whole[1000:])
    check_clipped([a], [whole[:1000]], 1.0 / norm64([a, a]))


def test_lists_replaced_on_another_stream(sfb):
    """Lists of more tensors than a launch takes as its arguments, each made on the current stream for one call on a context of
    another one and gone before the call's kernels are: every call sees its own tensors."""
    side = torch.cuda.Stream()
    own = sfb.Context(0, stream=side)
    count, rounds = 200, 24
    flat = [torch.randn(count * 5000, generator=torch.Generator(device="cuda:0").manual_seed(k), device="cuda:0") for k in range(rounds)]
    before = [f.clone() for f in flat]
    busy = torch.randn(1 << 26, device="cuda:0")
    norms = [torch.zeros(1, device="cuda:0") for _ in range(2 * rounds)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):                   # work in front of the calls, so that the lists are gone first
            busy.mul_(0.5)
    for k, f in enumerate(flat):
        own.sfb_grad_norm(sfb.TensorList(f.split(5000)), norms[2 * k])
        own.sfb_clip_grads(sfb.TensorList(f.split(5000)), 1.0 + k, norms[2 * k + 1])
    torch.cuda.synchronize()
    for k, f in enumerate(flat):
        want = norm64([before[k]])
        for n in norms[2 * k:2 * k + 2]:
            assert abs(n.item() - want) <= 2.0 ** -24 * want * 1.001
        check_clipped([before[k]], [f], (1.0 + k) / want)
    own.close()


def test_captured_list_is_gone(sfb):
    """A graph of a call with a list that nobody else keeps, replayed after other lists have been made and used."""
    side = torch.cuda.Stream()
    own = sfb.Context(0, stream=side)
    flat = torch.zeros(200 * 300, device="cuda:0")
    other = torch.randn(200 * 300, device="cuda:0")
    norm, n2 = torch.zeros(1, device="cuda:0"), torch.zeros(1, device="cuda:0")
    own.sfb_clip_grads(sfb.TensorList(other.split(300)), 1e9, n2)
    torch.cuda.synchronize()
    lst = sfb.TensorList(flat.split(300))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        own.sfb_clip_grads(lst, 1.0, norm)
    del lst
    for k in range(3):
        for _ in range(4):
            own.sfb_clip_grads(sfb.TensorList(other.split(300)), 1e9, n2)
        src = torch.randn(200 * 300, generator=torch.Generator(device="cuda:0").manual_seed(k), device="cuda:0")
        flat.copy_(src)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = norm64([src])
        assert abs(norm.item() - want) <= 2.0 ** -24 * want * 1.001
        check_clipped([src], [flat], 1.0 / want)
    own.close()


@pytest.mark.parametrize("bound", [1.0, 0.3125, 2.0 ** -100, 2.0 ** -140])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 70, 2.0 ** -70])
def test_clipped_to_half_a_step(sfb, ctx, bound, size):
    """The scale is held in 64 bits and a result rounded once (bf16: to fp32 before): the error is half a step of its type, with a
    scale of 32 bits it would be twice that of an fp32 result."""
    src = [t.mul_(size) for t in tensors([100_000, 70_001, 33], seed=3)]
    want = norm64(src)
    norm = torch.zeros(1, device="cuda:0")
    dst = [torch.zeros_like(t) for t in src]
    ctx.sfb_clip_grads(sfb.TensorList(src, dst), bound, norm)          # (bound is an fp32 number)
    assert abs(norm.item() - want) <= (2.0 ** -24 + 2.0 ** -36) * want + 2.0 ** -150
    coef = bound / want
    assert coef < 1.0 or size < 1.0
    for s, d in zip(src, dst):
        exact = s.double() * min(1.0, coef)
        # 2^-36: the sum of 1.7e5 squares is off by 1.7e5 2^-53 at most, its root by half of that; the last term: half a denormal step
        room = exact.abs() * (2.0 ** -24 + 2.0 ** -36) + 2.0 ** -150
        if s.dtype == BF16:
            room += exact.abs() * 2.0 ** -8 * 1.001 + 2.0 ** -134
        assert bool(((d.double() - exact).abs() <= room).all())
