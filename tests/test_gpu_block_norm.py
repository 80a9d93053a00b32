"""Norms around a block and their gradients against the formulas in 64 bits.

Tolerances, with u = 2^-24 and half = eps / 2 of the stored type (a rounding is off by
half a step of its value at most): a row's sum adds 32 terms in a thread, then at most
5 shuffles and 16 warps, so it is off by 64 u at most and r by 40 u; a has 3 products
more, o two more: 48 u (|h| + |s g a|).  What that does to o r(o) grows with amp =
||h| + |s g a|| / |o|.  The gradients go through two such sums and a dozen products:
1024 u amp of the sums of magnitudes that they consist of.  Sums over the rows add at
most one rounding a row."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def make(seed, rows, d, dtype, after=True, gate="channel", before=True, ld=None):
    """Inputs of one call; with ld, rows lie that far apart in memory."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def draw(*shape, std=1.0, mean=0.0):
        t = (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)
        if ld is None or len(shape) == 1:
            return t
        wide = torch.full((shape[0], ld), 7.0, device="cuda", dtype=dtype)
        wide[:, :d] = t
        return wide[:, :d]
    h, y = draw(rows, d), draw(rows, d, std=0.5)
    opt = dict(w_after=draw(d, std=0.1, mean=1.0) if after else None,
               w_before=draw(d, std=0.1, mean=1.0) if before else None,
               gate={"none": None, "channel": draw(d, std=0.5),
                     "token": draw(rows, d, std=0.5)}[gate], scale=0.7, eps=1e-5)
    return h, y, opt, draw(rows, d), draw(rows, d) if before else None


def formula(h, y, opt):
    """(out, norm) in 64 bits, on doubles that may ask for gradients."""
    def r(v):
        return 1 / torch.sqrt((v * v).mean(1, keepdim=True) + opt["eps"])
    o = h
    if y is not None:
        a = y if opt["w_after"] is None else y * r(y) * opt["w_after"]
        if opt["gate"] is not None:
            a = a * opt["gate"]
        o = h + opt["scale"] * a
    return o, None if opt["w_before"] is None else o * r(o) * opt["w_before"]


def doubles(h, y, opt, grad=False):
    def f(t):
        return t.double().requires_grad_(grad) if isinstance(t, torch.Tensor) else t
    return f(h), f(y), {k: f(v) for k, v in opt.items()}


def close(got, ref, bound, what):
    half = torch.finfo(got.dtype).eps / 2
    worst = ((got.double() - ref).abs() - half * ref.abs() - bound).max().item() if got.numel() else 0
    assert worst <= 0, (what, worst)


def amp_of(h, y, opt):
    o = formula(h, y, opt)[0]
    s = h.abs() + (o - h).abs()
    return s, (s.norm(dim=1, keepdim=True) / o.norm(dim=1, keepdim=True).clamp(min=1e-300))


def check_forward(h, y, opt, out, norm):
    hd, yd, od = doubles(h, y, opt)
    ro, rn = formula(hd, yd, od)
    s, amp = amp_of(hd, yd, od)
    close(out, ro, 48 * U * s, "out")
    if rn is not None:
        r = 1 / torch.sqrt((ro * ro).mean(1, keepdim=True) + opt["eps"])
        w = od["w_before"].abs()
        close(norm, rn, w * r * (48 * U * s + ro.abs() * (44 + 48 * amp) * U), "norm")


def check_backward(h, y, opt, d_out, d_norm, got):
    hd, yd, od = doubles(h, y, opt, True)
    o, n = formula(hd, yd, od)
    total = 0.0
    if d_out is not None:
        total = total + (o * d_out.double()).sum()
    if n is not None:
        total = total + (n * d_norm.double()).sum()
    inputs = dict(h=hd, y=yd, **{k: od[k] for k in ("gate", "w_after", "w_before")})
    inputs = {k: v for k, v in inputs.items() if v is not None}
    ref = dict(zip(inputs, torch.autograd.grad(total, list(inputs.values()))))
    with torch.no_grad():
        rows = h.shape[0]
        amp = amp_of(hd, yd, od)[1]
        mag = d_out.double().abs() if d_out is not None else torch.zeros_like(hd)
        if n is not None:
            r = 1 / torch.sqrt((o * o).mean(1, keepdim=True) + opt["eps"])
            oh, v = (o * r).abs(), (d_norm.double() * od["w_before"]).abs()
            mag = mag + r * (v + oh * (v * oh).mean(1, keepdim=True))
            close(got["w_before"], ref["w_before"],
                  (U * (1024 * amp + rows) * d_norm.double().abs() * oh).sum(0), "w_before")
        tol = 1024 * U * amp
        close(got["h"], ref["h"], tol * mag, "h")
        if y is None:
            assert got["y"] is None
            return
        ry = 1 / torch.sqrt((yd * yd).mean(1, keepdim=True) + opt["eps"])
        yh = (yd * ry).abs()
        w = od["w_after"].abs() if od["w_after"] is not None else 1.0
        a = yh * w if od["w_after"] is not None else yd.abs()
        g = od["gate"].abs() if od["gate"] is not None else 1.0
        b = abs(opt["scale"]) * mag
        if od["gate"] is not None:
            bound = tol * b * a
            close(got["gate"], ref["gate"],
                  bound if opt["gate"].dim() == 2 else (bound + rows * U * b * a).sum(0), "gate")
        if od["w_after"] is not None:
            close(got["w_after"], ref["w_after"], ((tol + rows * U) * b * g * yh).sum(0), "w_after")
            u = b * g * w
            close(got["y"], ref["y"], tol * ry * (u + yh * (u * yh).mean(1, keepdim=True)), "y")
        else:
            close(got["y"], ref["y"], tol * b * g, "y")


SHAPES = [(1, 1), (3, 1), (700, 2), (1, 7), (5, 8), (65, 31), (33, 32), (130, 33), (40, 64),
          (9, 127), (257, 128), (50, 129), (300, 256), (31, 257), (6, 1000), (1999, 1001),
          (64, 2048), (7, 2049), (2500, 2048), (5, 4096), (3, 4100), (20, 8192), (2, 8193),
          (3, 16384), (2, 16383)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,d", SHAPES)
def test_shapes(rows, d, dtype):
    h, y, opt, d_out, d_norm = make(rows * 7 + d, rows, d, dtype)
    check_forward(h, y, opt, *api.block_norm(h, y, **opt))
    check_backward(h, y, opt, d_out, d_norm, api.block_norm_backward(h, y, d_out, d_norm, **opt))


@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("after,before", [(True, True), (True, False), (False, True),
                                          (False, False)])
@pytest.mark.parametrize("rows,d,dtype", [(37, 96, F32), (19, 515, BF16), (530, 4, BF16),
                                          (4, 4608, F32)])
def test_what_is_given(rows, d, dtype, after, before, gate):
    h, y, opt, d_out, d_norm = make(d, rows, d, dtype, after, gate, before)
    check_forward(h, y, opt, *api.block_norm(h, y, **opt))
    check_backward(h, y, opt, d_out, d_norm, api.block_norm_backward(h, y, d_out, d_norm, **opt))
    if before:  # the gradient of the norm alone
        check_backward(h, y, opt, None, d_norm, api.block_norm_backward(h, y, None, d_norm, **opt))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_norm_by_itself(dtype):
    h, _, opt, d_out, d_norm = make(3, 21, 300, dtype)
    opt.update(w_after=None, gate=None)
    out, norm = api.block_norm(h, **opt)
    assert torch.equal(out, h)
    check_forward(h, None, opt, out, norm)
    check_backward(h, None, opt, d_out, d_norm,
                   api.block_norm_backward(h, None, d_out, d_norm, **opt))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,ld,shift", [(64, 72, 0), (64, 71, 0), (64, 80, 1), (999, 1008, 0),
                                        (2048, 2056, 8)])
def test_strides_and_alignment(dtype, d, ld, shift):
    """The same bits as from packed rows, whatever the way they are read; what lies
    between the rows stays as it is."""
    h, y, opt, d_out, d_norm = make(5, 23, d, dtype, gate="token")

    def apart(t):
        wide = torch.full((23, ld + shift), 7.0, device="cuda", dtype=dtype)
        wide[:, shift:shift + d] = t
        return wide, wide[:, shift:shift + d]
    args = {n: apart(t) for n, t in dict(h=h, y=y, gate=opt["gate"], d_out=d_out, d_norm=d_norm,
                                         out=h, norm=h, d_h=h, d_y=h).items()}
    v = {n: a[1] for n, a in args.items()}
    strided = {**opt, "gate": v["gate"]}
    api.block_norm(v["h"], v["y"], out=v["out"], norm=v["norm"], **strided)
    check_forward(h, y, opt, v["out"].contiguous(), v["norm"].contiguous())
    got = api.block_norm_backward(v["h"], v["y"], v["d_out"], v["d_norm"], d_h=v["d_h"],
                                  d_y=v["d_y"], **strided)
    check_backward(h, y, opt, d_out, d_norm, got)
    for wide, inner in args.values():
        inner.fill_(7.0)
        assert bool((wide == 7.0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place(dtype):
    h, y, opt, d_out, d_norm = make(8, 3000, 72, dtype, gate="token")
    out, norm = api.block_norm(h, y, **opt)
    got = api.block_norm_backward(h, y, d_out, d_norm, **opt)
    g, do, dn = (t.clone() for t in (opt["gate"], d_out, d_norm))
    again = api.block_norm_backward(h, y, do, dn, d_h=do, d_y=dn, **{**opt, "gate": g})
    assert all(torch.equal(again[k], got[k]) for k in got)
    h2, y2 = h.clone(), y.clone()
    api.block_norm(h2, y2, out=h2, norm=y2, **opt)
    assert torch.equal(h2, out) and torch.equal(y2, norm)


def test_rows_do_not_depend_on_one_another():
    h, y, opt, d_out, d_norm = make(9, 4000, 2048, BF16, gate="token")
    out, norm = api.block_norm(h, y, **opt)
    got = api.block_norm_backward(h, y, d_out, d_norm, **opt)
    part = slice(1717, 1720)
    opt["gate"] = opt["gate"][part]
    o, n = api.block_norm(h[part], y[part], **opt)
    assert torch.equal(o, out[part]) and torch.equal(n, norm[part])
    few = api.block_norm_backward(h[part], y[part], d_out[part], d_norm[part], **opt)
    for k in ("h", "y", "gate"):
        assert torch.equal(few[k], got[k][part])


def test_a_row_of_nan_stays_by_itself():
    h, y, opt, d_out, d_norm = make(10, 600, 24, F32, gate="token")
    out, norm = api.block_norm(h, y, **opt)
    h[77, 3] = float("nan")
    y[78, 5] = float("inf")
    o, n = api.block_norm(h, y, **opt)
    keep = torch.ones(600, dtype=torch.bool, device="cuda")
    keep[77:79] = False
    assert torch.equal(o[keep], out[keep]) and torch.equal(n[keep], norm[keep])
    assert bool(n[77].isnan().all()) and bool(n[78].isnan().any())


def test_zero_rows_of_values():
    """A row of zeros: r is 1 / sqrt(eps), outputs and gradients are finite."""
    h, y, opt, d_out, d_norm = make(11, 4, 100, F32)
    h[1], y[1] = 0, 0
    out, norm = api.block_norm(h, y, **opt)
    assert torch.equal(out[1], torch.zeros_like(out[1])) and not norm[1].any()
    got = api.block_norm_backward(h, y, d_out, d_norm, **opt)
    assert all(bool(t.isfinite().all()) for t in got.values())


def test_no_rows():
    h, y, opt, d_out, d_norm = make(12, 0, 100, BF16)
    out, norm = api.block_norm(h, y, **opt)
    assert out.shape == norm.shape == (0, 100)
    got = api.block_norm_backward(h, y, d_out, d_norm, **opt)
    for k in ("gate", "w_after", "w_before"):
        assert got[k].shape == (100,) and not got[k].any()


def test_differences():
    """Gradients against central differences of the formula in 64 bits along a random
    direction (step 1e-4: what the difference leaves out is some 1e-8 of the terms)."""
    h, y, opt, d_out, d_norm = make(13, 6, 50, F32, gate="token")
    got = api.block_norm_backward(h, y, d_out, d_norm, **opt)
    hd, yd, od = doubles(h, y, opt)

    def total(a, b, o):
        out, norm = formula(a, b, o)
        return ((out * d_out.double()).sum() + (norm * d_norm.double()).sum()).item()
    g = torch.Generator(device="cuda").manual_seed(1)
    for name in ("h", "y", "gate", "w_after", "w_before"):
        at = {"h": hd, "y": yd}.get(name, od.get(name))
        v = torch.randn(at.shape, generator=g, device="cuda", dtype=torch.float64)
        ends = []
        for step in (1e-4, -1e-4):
            moved = at + step * v
            ends.append(total(moved if name == "h" else hd, moved if name == "y" else yd,
                              {**od, name: moved} if name in od else od))
        slope = (ends[0] - ends[1]) / 2e-4
        terms = (got[name].double() * v).abs().sum().item()
        assert abs((got[name].double() * v).sum().item() - slope) <= 1e-4 * terms, name


def test_streams_and_graphs():
    h, y, opt, d_out, d_norm = make(14, 500, 640, BF16)
    want = [*api.block_norm(h, y, **opt),
            *api.block_norm_backward(h, y, d_out, d_norm, **opt).values()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [*api.block_norm(h, y, stream=s, **opt),
           *api.block_norm_backward(h, y, d_out, d_norm, stream=s, **opt).values()]
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [*api.block_norm(h, y, **opt),
               *api.block_norm_backward(h, y, d_out, d_norm, **opt).values()]
    for t in got:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("change", [
    dict(y=None), dict(w_after=torch.ones(9)), dict(gate=torch.ones(3, 10)),
    dict(gate=torch.ones(10).double()), dict(norm=torch.ones(4, 10), w_before=None),
    dict(out=torch.ones(4, 9)), dict(h=torch.ones(4, 10).double()),
    dict(h=torch.ones(10, 4).T), dict(y=torch.ones(4, 10).bfloat16()), dict(h=torch.ones(4, 0))])
def test_refusals(change, monkeypatch):
    def enqueued(*args, **kw):
        raise AssertionError("the call went on")
    monkeypatch.setattr(B, "reflex_block_norm", enqueued)
    h, y, opt, _, _ = make(15, 4, 10, F32)
    args = {**dict(h=h, y=y, **opt), **{k: v.cuda() if v is not None else None
                                        for k, v in change.items()}}
    with pytest.raises(ValueError):
        api.block_norm(args.pop("h"), args.pop("y"), **args)


@pytest.mark.parametrize("change", [
    dict(d_norm=None), dict(d_out=None, d_norm=None, w_before=None), dict(y=None),
    dict(d_out=torch.ones(4, 9)), dict(d_h=torch.ones(3, 10)), dict(d_y=torch.ones(4, 9)),
    dict(y=None, w_after=None, gate=None, d_y=torch.ones(4, 10))])
def test_backward_refusals(change, monkeypatch):
    def enqueued(*args, **kw):
        raise AssertionError("the call went on")
    monkeypatch.setattr(B, "reflex_block_norm_backward", enqueued)
    h, y, opt, d_out, d_norm = make(16, 4, 10, F32)
    args = {**dict(h=h, y=y, d_out=d_out, d_norm=d_norm, **opt),
            **{k: v.cuda() if v is not None else None for k, v in change.items()}}
    first = [args.pop(n) for n in ("h", "y", "d_out", "d_norm")]
    with pytest.raises(ValueError):
        api.block_norm_backward(*first, **args)
