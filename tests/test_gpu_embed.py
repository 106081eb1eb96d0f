"""Token embedding: lookup and gradient against plain sums in 64 bits (GPU), argument checks (CPU)."""
import ctypes as C
import math

import pytest
import torch

BF16, FP32 = torch.bfloat16, torch.float32
U = {FP32: 2.0 ** -24, BF16: 2.0 ** -8}  # an output's rounding (bf16 keeps 8 bits), relative


@pytest.fixture(scope="module")
def cd():
    from paper_2512_13728_gb300 import build

    build.build()
    import paper_2512_13728_gb300 as pkg

    return pkg


def tokens_of(kind, n, vocab, g):
    if kind == "uniform":
        return torch.randint(0, vocab, (n,), generator=g, device="cuda")
    if kind == "text":  # 1/rank law, some padding
        t = (torch.exp(torch.rand(n, generator=g, device="cuda") * math.log(vocab)).long() - 1).clamp(0, vocab - 1)
        t[torch.rand(n, generator=g, device="cuda") < 0.1] = -1
        return t
    if kind == "one":  # every token the same
        return torch.full((n,), vocab // 2, device="cuda")
    if kind == "ends":  # the first and the last row, and ids outside the table on both sides
        pick = torch.tensor([0, vocab - 1, -1, vocab, -100, 2 ** 31 + 5, vocab - 1], device="cuda")
        return pick[torch.randint(0, len(pick), (n,), generator=g, device="cuda")]
    assert kind == "padding"
    return torch.full((n,), -1, device="cuda")


def padded(rows, cols, ld, dtype, g, offset=0):
    """A rows x cols view with leading dimension ld whose first element sits `offset` elements into its buffer."""
    buf = torch.full((rows * ld + offset + ld,), float("nan"), dtype=dtype, device="cuda")
    v = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    v.copy_(torch.randn(rows, cols, generator=g, device="cuda"))
    return v, buf


SIZES = [  # tokens, vocab, dim, ld - dim, offset
    (1, 1, 1, 0, 0), (1, 1000, 256, 0, 0), (0, 17, 40, 0, 0), (7, 33, 771, 0, 0), (300, 50, 264, 8, 0),
    (2049, 513, 130, 2, 2), (5000, 70000, 64, 0, 1), (10000, 300, 1032, 4, 4), (33, 262145, 8, 0, 0), (4096, 4096, 2050, 0, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["text", "uniform", "ends"])
@pytest.mark.parametrize("table_dtype,out_dtype", [(FP32, FP32), (FP32, BF16), (BF16, BF16), (BF16, FP32)])
@pytest.mark.parametrize("n,vocab,dim,pad,offset", SIZES)
def test_lookup(cd, n, vocab, dim, pad, offset, table_dtype, out_dtype, kind):
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    tok = tokens_of(kind, n, vocab, g)
    table, _ = padded(vocab, dim, dim + pad, table_dtype, g, offset)
    out, buf = padded(n, dim, dim + pad, out_dtype, g, offset)
    before = buf.clone()
    plan = cd.EmbedPlan(vocab, dim, n)
    plan.lookup(tok, table, scale=0.7, out=out)
    real = (tok >= 0) & (tok < vocab)
    s = float(torch.tensor(0.7))  # the scale as fp32
    want = torch.where(real[:, None], table[tok.clamp(0, vocab - 1)].double() * s, 0.0)
    # one product rounded to fp32, then to the output's type
    assert ((out.double() - want).abs() <= want.abs() * (U[out_dtype] + 2 * U[FP32])).all()
    out.zero_()  # nothing outside the rows was written
    before_view = before[offset:offset + n * (dim + pad)].view(n, dim + pad)[:, :dim]
    before_view.zero_()
    assert torch.equal(buf.nan_to_num(7.0), before.nan_to_num(7.0))


def check_gradient(cd, tok, grad, vocab, out, accumulate, plan=None):
    n, dim = grad.shape
    real = (tok >= 0) & (tok < vocab)
    at, rows = tok[real], grad[real].double()
    s = 1.25
    base = out.double() if accumulate else torch.zeros(vocab, dim, dtype=torch.float64, device="cuda")
    want = base + s * torch.zeros_like(base).index_add_(0, at, rows)
    size = s * torch.zeros_like(base).index_add_(0, at, rows.abs())
    terms = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    # fp32 sums of `terms` addends (their bound holds for any order), the scale, the addition to out, and out's rounding
    tol = size * ((terms + 3) * U[FP32])[:, None] + want.abs() * (U[out.dtype] + 2 * U[FP32])
    plan = plan or cd.EmbedPlan(vocab, dim, n)
    plan.gradient(tok, grad, scale=s, out=out, accumulate=accumulate)
    assert ((out.double() - want).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["text", "uniform", "one", "ends", "padding"])
@pytest.mark.parametrize("grad_dtype,out_dtype", [(BF16, FP32), (FP32, FP32), (BF16, BF16), (FP32, BF16)])
@pytest.mark.parametrize("n,vocab,dim,pad,offset", SIZES)
def test_gradient(cd, n, vocab, dim, pad, offset, grad_dtype, out_dtype, kind):
    g = torch.Generator(device="cuda").manual_seed(3 * n + dim)
    tok = tokens_of(kind, n, vocab, g)
    grad, _ = padded(n, dim, dim + pad, grad_dtype, g, offset)
    for accumulate in (False, True):
        out, buf = padded(vocab, dim, dim + pad, out_dtype, g, offset)
        before = buf.clone()
        if not accumulate:
            out.fill_(float("inf"))  # every row is written
        check_gradient(cd, tok, grad, vocab, out, accumulate)
        out.zero_()
        before[offset:offset + vocab * (dim + pad)].view(vocab, dim + pad)[:, :dim].zero_()
        assert torch.equal(buf.nan_to_num(7.0), before.nan_to_num(7.0))


@pytest.mark.gpu
def test_gradient_many_tokens(cd):
    """More tokens than one cluster's sort takes, int32, a shape of three dimensions, one plan for calls of several sizes."""
    g = torch.Generator(device="cuda").manual_seed(5)
    vocab, dim = 5003, 72
    plan = cd.EmbedPlan(vocab, dim, 200_000)
    for shape in ((4, 50_000), (1, 1), (3, 1000), (2, 65_537)):
        tok = tokens_of("text", shape[0] * shape[1], vocab, g).int().view(shape)
        grad = torch.randn(*shape, dim, generator=g, device="cuda").to(BF16)
        out = plan.gradient(tok, grad, scale=1.25)
        check_gradient(cd, tok.view(-1).long(), grad.view(-1, dim), vocab, torch.empty_like(out), False, plan)
        again = plan.gradient(tok, grad, scale=1.25)
        assert torch.equal(out, again)  # the same from call to call


@pytest.mark.gpu
def test_gradient_is_the_derivative(cd):
    """d/dE of sum(c * lookup(E)): the lookup is linear, so differences are exact up to rounding."""
    g = torch.Generator(device="cuda").manual_seed(9)
    vocab, dim, n = 50, 24, 400
    tok = tokens_of("text", n, vocab, g)
    table = torch.randn(vocab, dim, generator=g, device="cuda")
    c = torch.randn(n, dim, generator=g, device="cuda")
    plan = cd.EmbedPlan(vocab, dim, n)
    grad = plan.gradient(tok, c, scale=0.5)
    for v, d in ((0, 0), (1, 5), (7, 23), (49, 3)):
        hi, lo = table.clone(), table.clone()
        hi[v, d] += 1.0
        lo[v, d] -= 1.0
        diff = ((plan.lookup(tok, hi, scale=0.5).double() - plan.lookup(tok, lo, scale=0.5).double()) * c.double()).sum()
        step = float(hi[v, d].double() - lo[v, d].double())
        # sums of up to n products of values below 5, each rounded to 2^-24
        assert abs(float(diff) / step - float(grad[v, d])) <= n * 5 * 5 * 2.0 ** -23


@pytest.mark.gpu
def test_nan_and_inf_stay_in_their_rows(cd):
    g = torch.Generator(device="cuda").manual_seed(1)
    tok = torch.tensor([3, -1, 5, 3, 9], device="cuda")
    grad = torch.randn(5, 16, generator=g, device="cuda")
    grad[1] = float("nan")  # padding's gradient is not read into any row
    grad[2, 4] = float("inf")
    out = cd.EmbedPlan(12, 16, 5).gradient(tok, grad)
    assert out[5, 4] == float("inf") and torch.isfinite(out).sum() == out.numel() - 1


@pytest.mark.gpu
def test_streams(cd):
    """On a side stream, with torch's current stream and with an explicit one."""
    g = torch.Generator(device="cuda").manual_seed(2)
    tok, table = tokens_of("text", 3000, 500, g), torch.randn(500, 320, generator=g, device="cuda")
    plan = cd.EmbedPlan(500, 320, 3000)
    want = plan.lookup(tok, table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = plan.lookup(tok, table)
    b = torch.empty_like(want)
    side.wait_stream(torch.cuda.current_stream())
    plan.lookup(tok, table, out=b, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)
    with pytest.raises(ValueError):
        plan.lookup(tok, table, stream=side.cuda_stream)


@pytest.mark.gpu
def test_refusals(cd):
    plan = cd.EmbedPlan(100, 32, 64)
    tok = torch.zeros(10, dtype=torch.long, device="cuda")
    table = torch.zeros(100, 32, device="cuda")
    for bad in (lambda: plan.lookup(tok.float(), table), lambda: plan.lookup(tok, table.half()),
                lambda: plan.lookup(tok, table[:, :31]), lambda: plan.lookup(tok, table[:99]),
                lambda: plan.lookup(tok, table.t().contiguous().t()), lambda: plan.lookup(tok.cpu(), table),
                lambda: plan.lookup(tok, table, out=torch.zeros(9, 32, device="cuda")),
                lambda: plan.gradient(tok, torch.zeros(9, 32, device="cuda")),
                lambda: plan.gradient(tok, torch.zeros(10, 32, device="cuda"), accumulate=True),
                lambda: plan.gradient(tok, torch.zeros(10, 32, device="cuda"), out=torch.zeros(99, 32, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(cd.DionError) as e:
        plan.gradient(torch.zeros(65, dtype=torch.long, device="cuda"), torch.zeros(65, 32, device="cuda"))
    assert e.value.code == cd.native.DION_ERR_INVALID_ARG
    with pytest.raises(cd.DionError):
        plan.lookup(tok, table, scale=float("nan"))


def test_c_refusals(cd):
    """Refused on the host before any device call, so fake pointers are never read."""
    lib, n = cd.native.load(), cd.native
    out = C.c_void_p(1)
    for args, code in (((0, 4, 4), 1), ((4, 0, 4), 1), ((4, 4, -1), 1), ((1 << 30, 4, 4), 2), ((4, 1 << 30, 4), 2),
                       ((4, 4, 1 << 30), 2)):
        assert lib.dion_embed_plan_create(*args, C.byref(out)) == code
        assert out.value is None
        out = C.c_void_p(1)
    assert lib.dion_embed_plan_create(4, 4, 4, None) == n.DION_ERR_INVALID_ARG
    p = C.c_void_p(0x10000)
    assert lib.dion_embed_lookup(None, p, 0, 1, p, 0, 4, 1.0, p, 0, 4, None) == n.DION_ERR_INVALID_ARG
    assert lib.dion_embed_gradient(None, p, 0, 1, p, 0, 4, 1.0, p, 0, 4, 0, None) == n.DION_ERR_INVALID_ARG
    lib.dion_embed_plan_destroy(None)


@pytest.mark.gpu
def test_offsets_beyond_32_bits(cd):
    """A table of more than 2^31 elements, and more than 2^31 elements of activations."""
    vocab, dim = 1_100_003, 2048
    g = torch.Generator(device="cuda").manual_seed(6)
    table = torch.empty(vocab, dim, dtype=BF16, device="cuda").normal_(generator=g)
    tok = torch.cat([torch.tensor([vocab - 1, 0, vocab - 2, vocab - 1], device="cuda"),
                     torch.randint(vocab // 2, vocab, (60,), generator=g, device="cuda")])
    plan = cd.EmbedPlan(vocab, dim, 1_100_000)
    assert torch.equal(plan.lookup(tok, table), table[tok])
    many = torch.randint(0, vocab, (1_100_000,), generator=g, device="cuda")  # beyond one cluster's sort as well
    out = plan.lookup(many, table)
    last = slice(1_099_900, 1_100_000)
    assert torch.equal(out[last], table[many[last]])
    d = plan.gradient(many, out, out=table)  # bf16 in and out
    for v in (int(many[-1]), int(many[0]), vocab - 1):
        at = (many == v).nonzero()[:, 0]
        want = out[at].double().sum(0)
        assert ((d[v].double() - want).abs() <= want.abs() * 2.0 ** -8 + len(at) ** 2 * 2.0 ** -20).all()
