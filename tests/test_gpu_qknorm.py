"""Norm and rotation of queries and keys: forward and backward against plain formulas in 64 bits (GPU),
argument checks (CPU)."""
import ctypes as C

import pytest
import torch

BF16, FP32 = torch.bfloat16, torch.float32
u = 2.0 ** -24
OUT = {FP32: u, BF16: 2.0 ** -8}  # an output's rounding, relative
EPS = 1e-6


@pytest.fixture(scope="module")
def cd():
    from paper_2512_13728_gb300 import build

    build.build()
    import paper_2512_13728_gb300 as pkg

    return pkg


def turn(a, b, positions, freq, back=False):
    ang = positions.double()[..., None] * freq
    c, s = ang.cos()[:, :, None], ang.sin()[:, :, None]
    return (a * c + b * s, b * c - a * s) if back else (a * c - b * s, b * c + a * s)


def pairs(x, rot, inter):
    r = x[..., :rot]
    return (r[..., 0::2], r[..., 1::2], x[..., rot:]) if inter else (r[..., :rot // 2], r[..., rot // 2:], x[..., rot:])


def unpairs(a, b, rest, inter):
    r = torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1)
    return torch.cat([r, rest], -1)


def rotate(x, positions, freq, inter, back=False):
    a, b, rest = pairs(x, 2 * len(freq), inter)
    return unpairs(*turn(a, b, positions, freq, back), rest, inter)


def mix(x, freq, inter):
    """|a| + |b| for each element of a pair: what a rotation's errors are relative to."""
    a, b, rest = pairs(x.abs(), 2 * len(freq), inter)
    return unpairs(a + b, a + b, rest, inter)


def freq_of(rot, theta=10000.0):
    return theta ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1))


def forward_ref(x, w, positions, freq, inter):
    x = x.double()
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    v = n * w.double() if w is not None else n
    return rotate(v, positions, freq, inter), mix(v, freq, inter)


def backward_ref(g, x, w, positions, freq, inter):
    x, g = x.double(), g.double()
    w = torch.ones(x.shape[-1], dtype=torch.float64, device="cuda") if w is None else w.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    n, gu, size = x * r, rotate(g, positions, freq, inter, back=True), mix(g, freq, inter)
    dx = r * (w * gu - n * (w * gu * n).mean(-1, keepdim=True))
    dx_size = r * (w.abs() * size + n.abs() * (w.abs() * size * n.abs()).mean(-1, keepdim=True))
    terms = x[..., 0].numel()
    return dx, dx_size, (gu * n).sum((0, 1, 2)), (size * n.abs()).sum((0, 1, 2)) * (terms + 48) * u


def make(shape, dtype, layout, g):
    b, t, h, d = shape
    v = torch.randn(shape, generator=g, device="cuda")
    if layout == "packed":  # inside a wider row
        buf = torch.full((b, t, h + 3, d), float("nan"), dtype=dtype, device="cuda")
        out = buf[:, :, 1:h + 1]
    elif layout == "heads_first":
        out = torch.empty(b, h, t, d, dtype=dtype, device="cuda").transpose(1, 2)
    elif layout == "odd":  # rows that begin at any element
        out = torch.empty(b * t * h * (d + 1) + 1, dtype=dtype, device="cuda")[1:].view(b, t, h, d + 1)[..., :d]
    else:
        out = torch.empty(shape, dtype=dtype, device="cuda")
    return out.copy_(v)


CASES = [  # batch, tokens, heads, kv_heads, head_dim, rotary, interleaved, layout
    (1, 1, 1, 1, 2, 2, False, "plain"), (1, 1, 4, 0, 128, 128, False, "plain"), (5, 1, 16, 4, 128, 128, False, "packed"),
    (2, 33, 3, 3, 64, 64, False, "heads_first"), (3, 7, 5, 2, 80, 32, False, "packed"), (1, 300, 6, 1, 96, 0, False, "plain"),
    (2, 65, 4, 2, 256, 102, False, "plain"), (2, 17, 2, 2, 256, 256, False, "odd"), (1, 9, 8, 8, 128, 64, True, "packed"),
    (4, 50, 7, 1, 20, 12, True, "odd"), (2, 1025, 12, 12, 64, 64, True, "heads_first"), (1, 2, 40, 8, 250, 250, False, "plain"),
    (7, 129, 9, 3, 36, 24, False, "plain"), (1, 5, 1, 1, 6, 4, True, "plain"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("b,t,hq,hk,d,rot,inter,layout", CASES)
def test_forward_and_backward(cd, b, t, hq, hk, d, rot, inter, layout, weights, dtype):
    g = torch.Generator(device="cuda").manual_seed(d + t)
    q, k = make((b, t, hq, d), dtype, layout, g), make((b, t, hk, d), dtype, layout, g) if hk else None
    gq, gk = make(q.shape, dtype, "heads_first", g), make(k.shape, dtype, layout, g) if hk else None
    wq, wk = (torch.randn(d, generator=g, device="cuda") for _ in "qk") if weights else (None, None)
    pos = torch.randint(-1000, 1 << 20, (b, t), generator=g, device="cuda")
    freq = freq_of(rot)
    plan = cd.QKNormPlan(d, rot, interleaved=inter, eps=EPS)
    outs = plan.forward(q, k, wq, wk, pos)
    grads = plan.backward(gq, gk, q, k, wq, wk, pos)
    assert (outs[1] is None) == (k is None) and (grads[2] is None) == (not weights)
    for i, (x, gx, w) in enumerate(((q, gq, wq), (k, gk, wk))):
        if x is None:
            continue
        want, size = forward_ref(x, w, pos, freq, inter)
        # 2 d / lanes + 5 additions in the mean (half of that in r), the products, sine and cosine of an angle
        # whose fp32 fraction is 2^-25 half turns off, the rotation
        assert ((outs[i].double() - want).abs() <= 40 * u * size + OUT[dtype] * want.abs()).all()
        dx, dx_size, dw, dw_tol = backward_ref(gx, x, w, pos, freq, inter)
        assert ((grads[i].double() - dx).abs() <= 100 * u * dx_size + OUT[dtype] * dx.abs()).all()
        if w is not None:
            assert ((grads[2 + i].double() - dw).abs() <= dw_tol).all()
    again = plan.backward(gq, gk, q, k, wq, wk, pos)
    assert all(a is None or torch.equal(a, x) for a, x in zip(again, grads))  # bit for bit, dw among them
    # in place: the outputs take the inputs' memory, the rest of a packed buffer stays
    q2, k2 = (None if x is None else torch.empty_strided(x.shape, x.stride(), dtype=dtype, device="cuda").copy_(x) for x in (q, k))
    plan.forward(q2, k2, wq, wk, pos, out=(q2, k2))
    assert torch.equal(q2, outs[0]) and (k2 is None or torch.equal(k2, outs[1]))
    plan.backward(gq, gk, q, k, wq, wk, pos, out=(gq, gk, *(None if w is None else torch.empty_like(w) for w in (wq, wk))))
    assert torch.equal(gq, grads[0]) and (gk is None or torch.equal(gk, grads[1]))


MANY = [  # batch, tokens, heads, kv_heads, head_dim, rotary, interleaved, layout: many tokens with few heads
    (37, 811, 3, 3, 96, 96, False, "plain"), (40001, 1, 1, 1, 64, 64, False, "packed"), (3, 9999, 5, 1, 80, 32, False, "packed"),
    (1, 30011, 2, 0, 32, 16, True, "heads_first"), (9001, 7, 12, 3, 32, 32, False, "plain"), (5003, 3, 1, 2, 256, 102, False, "plain"),
    (101, 301, 3, 1, 20, 12, True, "odd"), (2, 15013, 1, 3, 128, 128, False, "odd"), (129, 257, 2, 1, 36, 0, False, "heads_first"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("b,t,hq,hk,d,rot,inter,layout", MANY)
def test_many_tokens_of_few_heads(cd, b, t, hq, hk, d, rot, inter, layout, dtype):
    """Sequences that end anywhere, default positions and one row of them; queries and keys with their own blocks."""
    g = torch.Generator(device="cuda").manual_seed(d + t)
    q, k = make((b, t, hq, d), dtype, layout, g), make((b, t, hk, d), dtype, layout, g) if hk else None
    gq, gk = make(q.shape, dtype, "plain", g), make(k.shape, dtype, layout, g) if hk else None
    wq, wk = (torch.randn(d, generator=g, device="cuda") for _ in "qk")
    row = torch.randint(-1000, 1 << 20, (t,), generator=g, device="cuda", dtype=torch.int32)
    each = torch.randint(-1000, 1 << 20, (b, t), generator=g, device="cuda")
    freq = freq_of(rot)
    plan = cd.QKNormPlan(d, rot, interleaved=inter, eps=EPS)
    for pos, given in ((torch.arange(t, device="cuda")[None], None), (row[None], row), (each, each)):
        outs = plan.forward(q, k, wq, wk, given)
        grads = plan.backward(gq, gk, q, k, wq, wk, given)
        for i, (x, gx, w) in enumerate(((q, gq, wq), (k, gk, wk))):
            if x is None:
                continue
            want, size = forward_ref(x, w, pos, freq, inter)  # bounds as above
            assert ((outs[i].double() - want).abs() <= 40 * u * size + OUT[dtype] * want.abs()).all()
            dx, dx_size, dw, dw_tol = backward_ref(gx, x, w, pos, freq, inter)
            assert ((grads[i].double() - dx).abs() <= 100 * u * dx_size + OUT[dtype] * dx.abs()).all()
            assert ((grads[2 + i].double() - dw).abs() <= dw_tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_positions(cd, index):
    """None, one row for all sequences, negative, and beyond any table: 2^31 - 1."""
    g = torch.Generator(device="cuda").manual_seed(4)
    q = make((2, 6, 3, 64), FP32, "plain", g)
    plan = cd.QKNormPlan(64, eps=EPS)
    default = plan.forward(q)[0]
    row = torch.arange(6, device="cuda", dtype=index)
    assert torch.equal(plan.forward(q, positions=row)[0], default)
    assert torch.equal(plan.forward(q, positions=row[None].expand(2, 6))[0], default)
    assert torch.equal(plan.forward(q[0], positions=row)[0], default[0])  # three dimensions
    far = torch.tensor([[2 ** 31 - 1, -2 ** 31, 123456789, -77, 2 ** 30, 1]] * 2, device="cuda", dtype=index)
    want, size = forward_ref(q, None, far, freq_of(64), False)
    # both angles come from inv_freq in 64 bits: off by 2^-52 of themselves at most, 2^31 2^-52 radians
    assert ((plan.forward(q, positions=far)[0].double() - want).abs() <= (40 * u + 2.0 ** -20) * size).all()


@pytest.mark.gpu
def test_own_frequencies(cd):
    g = torch.Generator(device="cuda").manual_seed(4)
    q = make((1, 50, 2, 32), FP32, "plain", g)
    f = [1.5, -0.25, 0.0, 7.0, 1e-4, 3.14159, 100.0, 0.5]
    plan = cd.QKNormPlan(32, 16, inv_freq=f, eps=EPS)
    pos = torch.arange(50, device="cuda")[None]
    want, size = forward_ref(q, None, pos, torch.tensor(f, dtype=torch.float64, device="cuda"), False)
    assert ((plan.forward(q)[0].double() - want).abs() <= 40 * u * size).all()
    with pytest.raises(ValueError):
        cd.QKNormPlan(32, 16, inv_freq=f[:7])


@pytest.mark.gpu
def test_zero_rows_large_values_and_empty(cd):
    plan = cd.QKNormPlan(64, eps=EPS)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = make((1, 4, 2, 64), FP32, "plain", g)
    x[0, 1] = 0
    x[0, 2] *= 1e12
    x[0, 3, 0, 5] = float("nan")
    y = plan.forward(x)[0]
    assert (y[0, 1] == 0).all() and torch.isfinite(y[0, :3]).all() and torch.isfinite(y[0, 3, 1]).all()
    assert torch.isnan(y[0, 3, 0]).all()
    w = torch.ones(64, device="cuda")
    for shape in ((0, 4, 2, 64), (3, 0, 2, 64)):
        e = torch.empty(shape, device="cuda")
        dq, dk, dwq, dwk = plan.backward(e, e, e, e, w, w)
        assert dq.shape == shape and (dwq == 0).all() and (dwk == 0).all()
        assert plan.forward(e, e, w, w)[0].shape == shape


@pytest.mark.gpu
def test_gradient_against_differences(cd):
    """d/dx and d/dw of sum(c * forward(x)), central differences in fp32 outputs summed in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(8)
    d, pos = 32, torch.tensor([[5, 900]], device="cuda")
    plan = cd.QKNormPlan(d, 24, eps=EPS)
    x, c = make((1, 2, 3, d), FP32, "plain", g), make((1, 2, 3, d), FP32, "plain", g)
    w = 1 + 0.3 * torch.randn(d, generator=g, device="cuda")
    dx, _, dw, _ = plan.backward(c, None, x, None, w, None, pos)

    def f(x, w):
        return float((plan.forward(x, None, w, None, pos)[0].double() * c.double()).sum())

    h = 2.0 ** -6
    # third derivatives stay below 20 |c|_1 here: h^2 / 6 of that, and outputs' errors of 40 u (|a| + |b|) over h
    tol = h * h / 6 * 20 * 32 + 40 * u * 2 * 192 * 4 / h
    for i in ((0, 0, 0, 0), (0, 1, 2, 13), (0, 0, 1, 31), (0, 1, 0, 24)):
        hi, lo = x.clone(), x.clone()
        hi[i] += h
        lo[i] -= h
        assert abs((f(hi, w) - f(lo, w)) / float(hi[i].double() - lo[i].double()) - float(dx[i])) <= tol
    for j in (0, 11, 12, 30):
        hi, lo = w.clone(), w.clone()
        hi[j] += h
        lo[j] -= h
        assert abs((f(x, hi) - f(x, lo)) / float(hi[j].double() - lo[j].double()) - float(dw[j])) <= tol


@pytest.mark.gpu
def test_streams_and_refusals(cd):
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k = make((2, 40, 4, 64), BF16, "plain", g), make((2, 40, 2, 64), BF16, "plain", g)
    plan = cd.QKNormPlan(64)
    want = plan.forward(q, k)
    side = torch.cuda.Stream()
    out = tuple(torch.empty_like(x) for x in want)
    side.wait_stream(torch.cuda.current_stream())
    plan.forward(q, k, out=out, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    w = torch.ones(64, device="cuda")
    for bad in (lambda: plan.forward(q, k, stream=side.cuda_stream), lambda: plan.forward(q.half(), k.half()),
                lambda: plan.forward(q, k.float()), lambda: plan.forward(q[..., :62], k), lambda: plan.forward(q, k[:, :39]),
                lambda: plan.forward(q.transpose(-1, -2).contiguous().transpose(-1, -2), k),
                lambda: plan.forward(q, k, w.double()), lambda: plan.forward(q, k, w[:63]),
                lambda: plan.forward(q, k, positions=torch.zeros(40, device="cuda")),
                lambda: plan.forward(q, k, positions=torch.zeros(3, 40, dtype=torch.long, device="cuda")),
                lambda: plan.forward(q, k, out=(q, None)), lambda: plan.backward(q, None, q, k),
                lambda: plan.backward(k, k, q, k)):
        with pytest.raises(ValueError):
            bad()


def test_c_refusals(cd):
    lib, n = cd.native.load(), cd.native
    for args, code in (((0, 0, 0, 1e4, None, 1e-6), 1), ((63, 0, 0, 1e4, None, 1e-6), 1), ((64, 65, 0, 1e4, None, 1e-6), 1),
                       ((64, 66, 0, 1e4, None, 1e-6), 1), ((64, -2, 0, 1e4, None, 1e-6), 1), ((64, 64, 0, 0.0, None, 1e-6), 1),
                       ((64, 64, 0, 1e4, None, -1.0), 1), ((64, 64, 0, 1e4, None, float("nan")), 1),
                       ((258, 64, 0, 1e4, None, 1e-6), 2), ((4, 4, 0, 1e4, (C.c_double * 2)(1.0, float("inf")), 0.0), 1)):
        out = C.c_void_p(1)
        assert lib.dion_qknorm_plan_create(*args, C.byref(out)) == code
        assert out.value is None
    assert lib.dion_qknorm_plan_create(64, 64, 0, 1e4, None, 1e-6, None) == n.DION_ERR_INVALID_ARG
    sh, h = n.dion_qk_shape(1, 1, 1, 0, 0), n.dion_heads(0x1000, 0, 0, 0)
    assert lib.dion_qknorm_forward(None, sh, h, None, None, None, h, None, None) == n.DION_ERR_INVALID_ARG
    assert lib.dion_qknorm_backward(None, sh, h, None, h, None, None, None, h, None, None, None, None) == n.DION_ERR_INVALID_ARG
    lib.dion_qknorm_plan_destroy(None)


@pytest.mark.gpu
def test_offsets_beyond_32_bits(cd):
    tokens, heads, d = 1_060_000, 16, 128  # 2.2e9 elements
    q = torch.zeros(1, tokens, heads, d, dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    tail = torch.randn(1, 3, heads, d, generator=g, device="cuda").to(BF16)
    q[:, -3:] = tail
    plan = cd.QKNormPlan(d, eps=EPS)
    y = plan.forward(q)[0]
    want, size = forward_ref(tail, None, torch.arange(tokens - 3, tokens, device="cuda")[None], freq_of(d), False)
    assert ((y[:, -3:].double() - want).abs() <= 40 * u * size + OUT[BF16] * want.abs()).all()
    assert not y[:, tokens // 2].any()
    dq = plan.backward(y, None, q, out=(y, None, None, None))[0]  # in place over the gradient
    pos = torch.arange(tokens - 3, tokens, device="cuda")[None]
    dx, dx_size, _, _ = backward_ref(plan.forward(tail, positions=pos)[0], tail, None, pos, freq_of(d), False)
    assert ((dq[:, -3:].double() - dx).abs() <= 100 * u * dx_size + OUT[BF16] * dx.abs()).all()
