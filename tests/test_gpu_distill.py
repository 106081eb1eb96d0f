"""Distillation from a teacher's top logits: loss and gradient against plain softmaxes in 64 bits (GPU),
argument checks (CPU)."""
import ctypes as C
import math

import pytest
import torch

BF16, FP32 = torch.bfloat16, torch.float32
u = 2.0 ** -24
OUT = {FP32: u, BF16: 2.0 ** -8}  # an output's rounding, relative
INF = math.inf


@pytest.fixture(scope="module")
def cd():
    from paper_2512_13728_gb300 import build

    build.build()
    import paper_2512_13728_gb300 as pkg

    return pkg


def reference(z, ids, t, T, labels, hard, w):
    """loss, gradient, and for each the size that their errors are relative to."""
    z, w = z.double(), w.double()
    n, v = z.shape
    loss = torch.zeros(n, dtype=torch.float64, device=z.device)
    grad, size, loss_size = torch.zeros_like(z), torch.zeros_like(z), torch.zeros_like(loss)
    if hard < 1:
        there = (ids >= 0) & (ids < v) & (t.double() > -INF)
        some = there.any(1)
        lp = torch.where(there, t.double() / T, -INF)
        lp = torch.where(some[:, None], lp - torch.logsumexp(lp, 1, keepdim=True), 0.0)
        p = torch.where(there, lp.exp(), 0.0)
        lq = z / T - torch.logsumexp(z / T, 1, keepdim=True)
        at = ids.clamp(0, v - 1)
        lq_at = lq.gather(1, at)
        k = torch.where(p > 0, p * (lp - lq_at), 0.0).sum(1)
        loss = loss + (1 - hard) * T * T * torch.where(some, k, 0.0)
        loss_size = loss_size + (1 - hard) * T * T * torch.where(p > 0, p * (1 + lp.abs() + lq_at.abs()), 0.0).sum(1)
        c = (1 - hard) * T * some[:, None]
        target = torch.zeros_like(z).scatter_add_(1, at, p)
        grad = grad + torch.where(some[:, None], c * (lq.exp() - target), 0.0)
        size = size + torch.where(some[:, None], c * (lq.exp() + target), 0.0)
    if hard > 0:
        has = (labels >= 0) & (labels < v)
        y = labels.clamp(0, v - 1).long()[:, None]
        lq = z - torch.logsumexp(z, 1, keepdim=True)
        loss = loss + torch.where(has, -hard * lq.gather(1, y)[:, 0], 0.0)
        loss_size = loss_size + torch.where(has, hard * (1 + lq.gather(1, y)[:, 0].abs()), 0.0)
        one = torch.zeros_like(z).scatter_(1, y, 1.0)
        grad = grad + torch.where(has[:, None], hard * (lq.exp() - one), 0.0)
        size = size + torch.where(has[:, None], hard * (lq.exp() + one), 0.0)
    dead = w == 0
    return (torch.where(dead, 0.0, w * loss), torch.where(dead[:, None], 0.0, w[:, None] * grad),
            torch.where(dead, 0.0, w.abs() * loss_size), torch.where(dead[:, None], 0.0, w.abs()[:, None] * size))


def relative_error(z, t, T, top):
    """Bound of a probability's relative and a log-probability's absolute error: exponents (z - max) / T and
    (t - max) / T of three roundings each, ex2's 2^-22, sums over a thread's part of the row and trees."""
    def spread(x):  # below 200 T under its row's maximum a probability is 0 on both sides
        if not x.numel():
            return 0.0
        d = x.double().amax(1, keepdim=True) - x.double()
        return float(torch.where(d < 200 * T, d, 0.0).max())
    return u * (8 * (spread(z) + spread(t)) / min(T, 1.0) + z.shape[1] / 128 + top + 64)


def check(cd, z, ids, t, T, labels, hard, w, grad_out=None):
    loss, grad, loss_size, size = reference(z, ids, t, T, labels, hard, w)
    e = relative_error(z, t, T, ids.shape[1])
    got = cd.distill_loss(z, ids, t, T, labels if hard > 0 else None, hard, w)
    near = lambda x: (x.double() == loss) | ((x.double() - loss).abs() <= e * loss_size)  # noqa: E731  (infinities are equal)
    assert near(got).all()
    out = (torch.empty_like(got), grad_out if grad_out is not None else torch.full_like(z, float("nan")))
    l2, g2 = cd.distill_loss_grad(z, ids, t, T, labels if hard > 0 else None, hard, w, out=out)
    assert near(l2).all()
    assert ((g2.double() - grad).abs() <= 2 * e * size + OUT[z.dtype] * grad.abs()).all()
    return l2, g2


def make(n, v, k, dtype, seed=0, pad=0, offset=0, index=torch.int64, teacher_dtype=FP32):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + v + n)
    ld = v + pad
    buf = torch.full((n * ld + offset + 16,), float("nan"), dtype=dtype, device="cuda")
    z = buf[offset:offset + n * ld].view(n, ld)[:, :v]
    z.copy_(torch.randn(n, v, generator=g, device="cuda") * 3)
    ids = torch.rand(n, v, generator=g, device="cuda").topk(min(k, v), 1).indices if v <= 4096 else \
        (torch.randint(0, v, (n, 1), generator=g, device="cuda") + 1 + torch.arange(k, device="cuda") * (v // max(k, 1))) % v
    t = torch.randn(n, ids.shape[1], generator=g, device="cuda") * 4
    if ids.shape[1] > 1:
        ids[torch.rand(ids.shape, generator=g, device="cuda") < 0.1] = -1
    labels = torch.randint(0, v, (n,), generator=g, device="cuda")
    labels[torch.rand(n, generator=g, device="cuda") < 0.1] = -100
    w = torch.rand(n, generator=g, device="cuda") + 0.1
    w[torch.rand(n, generator=g, device="cuda") < 0.1] = 0
    return z, ids.to(index), t.to(teacher_dtype), labels.to(index), w, buf


CASES = [  # rows, vocab, top, pad of a row, offset of the first
    (1, 1, 1, 0, 0), (3, 2, 2, 0, 0), (2, 7, 3, 0, 1), (17, 33, 8, 0, 0), (5, 1000, 16, 24, 0), (64, 4097, 33, 0, 3),
    (300, 777, 1, 0, 0), (4, 50001, 64, 0, 0), (200, 50001, 20, 7, 5), (1, 131072, 256, 0, 0), (40, 100003, 100, 0, 0),
    (2, 300000, 1024, 0, 1), (3, 393216, 5, 0, 0), (7, 512, 512, 0, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("T,hard", [(1.0, 0.0), (2.0, 0.0), (0.5, 0.3), (3.5, 0.25), (2.0, 1.0)])
@pytest.mark.parametrize("n,v,k,pad,offset", CASES)
def test_loss_and_gradient(cd, n, v, k, pad, offset, T, hard, dtype):
    z, ids, t, labels, w, buf = make(n, v, k, dtype, pad=pad, offset=offset)
    l, g = check(cd, z, ids, t, T, labels, hard, w)
    l2, g2 = cd.distill_loss_grad(z, ids, t, T, labels, hard, w)
    assert torch.equal(l, l2) and torch.equal(g, g2)  # bit for bit
    before = buf.clone()
    cd.distill_loss_grad(z, ids, t, T, labels, hard, w, out=(l, z))  # in place
    assert torch.equal(z, g)
    z.zero_()  # around the rows nothing was written
    before[offset:offset + n * (v + pad)].view(n, v + pad)[:, :v].zero_()
    assert torch.equal(buf.nan_to_num(7.0), before.nan_to_num(7.0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gradient_rows_at_other_places(cd, dtype):
    """The gradient's rows begin elsewhere within 16 bytes than the logits'."""
    z, ids, t, labels, w, _ = make(9, 1003, 12, dtype, offset=1)
    for ld, off in ((1003, 0), (1008, 3), (1010, 1)):
        buf = torch.full((9 * ld + off + 8,), float("nan"), dtype=dtype, device="cuda")
        check(cd, z, ids, t, 1.5, labels, 0.5, w, grad_out=buf[off:off + 9 * ld].view(9, ld)[:, :1003])
        assert int(torch.isnan(buf).sum()) == buf.numel() - 9 * 1003


@pytest.mark.gpu
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("teacher_dtype", [BF16, FP32])
def test_types(cd, index, teacher_dtype):
    z, ids, t, labels, w, _ = make(20, 900, 10, BF16, index=index, teacher_dtype=teacher_dtype)
    check(cd, z, ids, t, 2.0, labels, 0.5, w)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("v", [600, 60000])
def test_masks(cd, dtype, v):
    """Masked vocabulary, absent entries in every way, repeated entries, label among the entries, rows left out."""
    z, ids, t, labels, w, _ = make(12, v, 8, dtype)
    ids = (torch.arange(8, device="cuda")[None] * 70 + torch.arange(12, device="cuda")[:, None]).long()
    w.fill_(0.5)
    labels.copy_(ids[:, 0])  # the label is an entry too
    z[0, 1::2] = -INF  # masked columns
    ids[0] = torch.arange(8, device="cuda") * 2
    z[1] = torch.finfo(dtype).min  # the lowest value everywhere but in one column
    z[1, ids[1, 0]] = 3.0
    t[1, 1:] = -INF
    ids[2] = -1  # no entries: by ids
    t[3] = -INF  # no entries: by logits
    labels[3] = v  # and no label: nothing left
    ids[4] = ids[4, 0]  # one entry eight times
    ids[5, 1], ids[5, 2] = v, 2 ** 40  # outside the vocabulary
    z[6] = float("nan")
    w[6] = 0  # left out, whatever it holds
    z[7] = INF
    w[7] = 0
    w[8] = -2.0
    t[9, 3:] = -INF
    labels[10] = -1
    z[11, 10:] = -INF  # few columns stay
    ids[11] = torch.arange(8, device="cuda")
    rows = [r for r in range(12) if r not in (6, 7)]
    for hard in (0.0, 0.4, 1.0):
        l, g = check(cd, z[rows], ids[rows], t[rows], 2.0, labels[rows], hard, w[rows])
        l, g = cd.distill_loss_grad(z, ids, t, 2.0, labels, hard, w)
        assert (g[6:8] == 0).all() and (l[6:8] == 0).all() and (g[3] == 0).all() and l[3] == 0
        if hard == 0:
            assert (g[2] == 0).all() and l[2] == 0
    # a teacher's entry in a masked column: an infinite loss, and a gradient that stays finite
    z[0, ids[0, 0]] = -INF
    l, g = cd.distill_loss_grad(z[:1], ids[:1], t[:1], 2.0)
    assert l[0] == INF and torch.isfinite(g).all()
    # a row without any finite logit has no softmax
    z[0] = -INF
    assert torch.isnan(cd.distill_loss(z[:1], ids[:1], t[:1], 2.0)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("v,k,pad,offset", [(600, 8, 0, 0), (2001, 200, 3, 1), (4100, 5, 0, 3), (8111, 40, 1, 0)])
def test_many_rows_of_few_logits(cd, v, k, pad, offset, dtype):
    """Every kind of row among many: masked, without entries, without label, left out, entries that come twice."""
    z, ids, t, labels, w, _ = make(801, v, k, dtype, pad=pad, offset=offset)
    kind = torch.arange(801, device="cuda") % 9
    ids[kind == 0] = torch.arange(k, device="cuda") * 2
    z[:, 1::2] = torch.where((kind == 0)[:, None], torch.full_like(z[:, 1::2], -INF), z[:, 1::2])
    ids[kind == 1] = -1
    t[kind == 2] = -INF
    labels[(kind == 2) | (kind == 3)] = -1
    ids[:, 0] = torch.where(kind == 4, ids[:, k - 1], ids[:, 0])
    labels[kind == 4] = ids[kind == 4, 0].to(labels.dtype)
    w[kind == 5] = 0
    for T, hard in ((2.0, 0.0), (1.5, 0.4), (1.0, 1.0)):
        rows = kind != 0 if hard > 0 else slice(None)  # a label in a masked column: an infinite loss
        l, g = cd.distill_loss_grad(z, ids, t, T, labels, hard, w)
        assert (g[kind == 5] == 0).all() and (l[kind == 5] == 0).all()
        check(cd, z[rows], ids[rows], t[rows], T, labels[rows], hard, w[rows])


@pytest.mark.gpu
def test_without_weights_entries_or_rows(cd):
    z, ids, t, labels, w, _ = make(6, 500, 4, FP32)
    w.fill_(1.0)
    l, g = cd.distill_loss_grad(z, ids, t, 2.0)
    l1, g1 = cd.distill_loss_grad(z, ids, t, 2.0, weights=w)
    assert torch.equal(l, l1) and torch.equal(g, g1)
    l, g = cd.distill_loss_grad(z, None, None, 2.0, labels=labels, hard=1.0)
    l1, g1 = cd.distill_loss_grad(z, ids, t, 5.0, labels=labels, hard=1.0, weights=w)
    assert torch.equal(l, l1) and torch.equal(g, g1)
    l, g = cd.distill_loss_grad(z, ids[:, :0], t[:, :0], 2.0)  # top = 0
    assert (l == 0).all() and (g == 0).all()
    l, g = cd.distill_loss_grad(z[:0], ids[:0], t[:0], 2.0)
    assert l.shape == (0,) and g.shape == (0, 500)


@pytest.mark.gpu
def test_gradient_against_differences(cd):
    z, ids, t, labels, w, _ = make(3, 40, 6, FP32, seed=3)
    w.copy_(torch.tensor([1.0, 0.5, 2.0]))
    T, hard, h = 1.5, 0.3, 2.0 ** -5
    _, g = cd.distill_loss_grad(z, ids, t, T, labels, hard, w)
    # |third derivative| <= w (1 - hard) / T + w hard; losses below 50 with errors of 1e-5 of them at most
    tol = h * h / 6 * 2 + 50 * 1e-5 * 2 / (2 * h) * 0.1
    for r in range(3):
        for j in (0, 7, 39, int(ids[r].max()), int(labels[r].clamp(min=0))):
            hi, lo = z.clone(), z.clone()
            hi[r, j] += h
            lo[r, j] -= h
            d = [float(cd.distill_loss(x, ids, t, T, labels, hard, w)[r].double()) for x in (hi, lo)]
            assert abs((d[0] - d[1]) / float(hi[r, j].double() - lo[r, j].double()) - float(g[r, j])) <= tol


@pytest.mark.gpu
def test_streams_and_refusals(cd):
    z, ids, t, labels, w, _ = make(30, 700, 5, BF16)
    want = cd.distill_loss_grad(z, ids, t, 2.0, weights=w)
    side = torch.cuda.Stream()
    out = tuple(torch.empty_like(x) for x in want)
    side.wait_stream(torch.cuda.current_stream())
    cd.distill_loss_grad(z, ids, t, 2.0, weights=w, out=out, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    f = cd.distill_loss_grad
    for bad in (lambda: f(z, ids, t, stream=side.cuda_stream), lambda: f(z.half(), ids, t), lambda: f(z.cpu(), ids, t),
                lambda: f(z.t().contiguous().t(), ids, t), lambda: f(z, ids[:29], t[:29]), lambda: f(z, ids, t[:, :4]),
                lambda: f(z, ids.float(), t), lambda: f(z, None, None), lambda: f(z, ids, t, labels=labels[:5], hard=0.5),
                lambda: f(z, ids, t, weights=w.double()), lambda: f(z, ids, t, out=(want[0], want[1].float()))):
        with pytest.raises(ValueError):
            bad()
    for kw in (dict(temperature=0.0), dict(temperature=float("inf")), dict(hard=-0.1), dict(hard=1.1), dict(hard=0.5)):
        with pytest.raises(cd.DionError) as e:
            f(z, ids, t, **kw)
        assert e.value.code == cd.native.DION_ERR_INVALID_ARG


def test_c_refusals(cd):
    """Refused on the host before any device call, so fake pointers are never read."""
    lib, n = cd.native.load(), cd.native

    def args(**kw):
        a = dict(rows=4, vocab=100, top=3, logits=0x1000, ld=100, ids=0x2000, ld_ids=3, teacher=0x3000, ld_teacher=3,
                 labels=0x4000, weights=None, dtype=0, id_dtype=1, teacher_dtype=0, label_dtype=1, temperature=1.0, hard=0.5)
        a.update(kw)
        return n.dion_distill(**a)

    p = C.c_void_p(0x9000)
    for kw, code in ((dict(rows=-1), 1), (dict(vocab=0), 1), (dict(top=-1), 1), (dict(ld=99), 1), (dict(dtype=5), 1),
                     (dict(logits=None), 1), (dict(ids=None), 1), (dict(teacher=None), 1), (dict(labels=None), 1),
                     (dict(ld_ids=2), 1), (dict(id_dtype=7), 1), (dict(label_dtype=7), 1), (dict(teacher_dtype=7), 1),
                     (dict(temperature=-1.0), 1), (dict(temperature=float("nan")), 1), (dict(hard=2.0), 1),
                     (dict(top=1025, ld_ids=1025, ld_teacher=1025), 2), (dict(vocab=393217, ld=400000), 2),
                     (dict(rows=1 << 31), 2), (dict(logits=0x1002), 3), (dict(ids=0x2004), 3), (dict(labels=0x4004), 3)):
        assert lib.dion_distill_loss(args(**kw), p, None) == code, kw
        assert lib.dion_distill_loss_grad(args(**kw), p, p, 100, None) == code, kw
    assert lib.dion_distill_loss(None, p, None) == 1
    assert lib.dion_distill_loss(args(), None, None) == 1
    assert lib.dion_distill_loss_grad(args(), p, None, 100, None) == 1
    assert lib.dion_distill_loss_grad(args(), p, p, 99, None) == 1
    assert lib.dion_distill_loss_grad(args(), p, C.c_void_p(0x9002), 100, None) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("v", [500, 70000])
def test_rows_of_the_lowest_value(cd, dtype, v):
    """A mask of the type's lowest value over a whole row leaves a uniform softmax, at every temperature."""
    z = torch.full((2, v), torch.finfo(dtype).min, dtype=dtype, device="cuda")
    z[1] = torch.finfo(dtype).max
    ids, t = torch.tensor([[3, 5]] * 2, device="cuda"), torch.zeros(2, 2, device="cuda")
    labels = torch.full((2,), 7, device="cuda")
    for T, hard in ((1.0, 0.0), (0.25, 0.5), (4.0, 0.5)):
        l, g = cd.distill_loss_grad(z, ids, t, T, labels, hard)
        want = (1 - hard) * T * T * math.log(v / 2) + hard * math.log(v)
        assert ((l.double() - want).abs() <= (v / 128 + 64) * u * want).all()
        rest = ((1 - hard) * T + hard) / v
        assert ((g[:, 8:].double() - rest).abs() <= rest * (OUT[dtype] + (v / 128 + 64) * u)).all()


def test_packed_structs_follow_the_header():
    from paper_2512_13728_gb300 import lm, native

    for packed, struct in ((lm._DISTILL, native.dion_distill), (lm._HEADS, native.dion_heads),
                           (lm._QK_SHAPE, native.dion_qk_shape)):
        assert packed.size == C.sizeof(struct)
        values = list(range(1, 1 + len(struct._fields_)))
        got = struct.from_buffer_copy(packed.pack(*values))
        assert [getattr(got, f[0]) for f in struct._fields_] == values


@pytest.mark.gpu
def test_offsets_beyond_32_bits(cd):
    n, v = 43_000, 50_001  # 2.15e9 logits, odd rows
    z = torch.zeros(n, v, dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    z[-5:] = (torch.randn(5, v, generator=g, device="cuda") * 3).to(BF16)
    tail = z[-5:].clone()
    ids = torch.randint(0, v, (n, 4), generator=g, device="cuda")
    t = torch.randn(n, 4, generator=g, device="cuda")
    w = torch.zeros(n, device="cuda")
    w[-5:] = 1.0
    loss, grad, loss_size, size = reference(tail, ids[-5:], t[-5:], 2.0, None, 0.0, w[-5:])
    e = relative_error(tail, t[-5:], 2.0, 4)
    l, gz = cd.distill_loss_grad(z, ids, t, 2.0, weights=w, out=(torch.empty(n, device="cuda"), z))  # in place
    assert ((l[-5:].double() - loss).abs() <= e * loss_size).all() and not l[:-5].any()
    assert ((gz[-5:].double() - grad).abs() <= 2 * e * size + OUT[BF16] * grad.abs()).all()
    assert not gz[n // 2].any()
