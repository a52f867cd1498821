"""Single tokens of window attention with values that are not finite: the same results whether a cache is cut into ranges that a
second launch joins (one sequence) or not (1536 of them: as many workgroups as the cut aims at)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN, INF = float("nan"), float("inf")
ROWS, D = 600, 64   # three ranges of 208 rows in one sequence's cache


def caches(io, seed=0):
    gen = torch.Generator(DEV).manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(io)
    return dict(ck=rnd(1, 1, ROWS, D), cv=rnd(1, 1, ROWS, D), q=rnd(1, 3, D), k=rnd(1, 1, D), v=rnd(1, 1, D))


def ask(x, pos):
    """The token's result, of one sequence and of 1536 copies."""
    import paper_2605_09877_amd as kvm
    outs = []
    for n in (1, 1536):
        y = {m: t.repeat(n, *(1,) * (t.dim() - 1)) for m, t in x.items()}
        at = torch.full((n,), pos, dtype=torch.int32, device=DEV)
        out = kvm.window_decode(y["ck"], y["cv"], y["q"], y["k"], y["v"], at, window=ROWS)
        same = out.nan_to_num(nan=12345.0)
        assert torch.equal(same, same[:1].expand_as(same))
        outs.append(out[0])
    return outs


def definition(x, pos):
    """In 64 bits, q [H, d] against rows 0 .. pos with the token's own (pos < ROWS)."""
    k, v = x["ck"][0, 0].double().clone(), x["cv"][0, 0].double().clone()
    k[pos], v[pos] = x["k"][0, 0].double(), x["v"][0, 0].double()
    t = x["q"][0].double() @ k[:pos + 1].T.contiguous() / D ** 0.5
    p = torch.exp(t - t.amax(-1, keepdim=True))
    return (p @ v[:pos + 1]) / p.sum(-1, keepdim=True)


def check(x, pos):
    ref = definition(x, pos)
    nan = torch.isnan(ref)
    mag = x["cv"].double().nan_to_num(0, 0, 0).abs().max()
    for out in ask(x, pos):
        assert torch.equal(torch.isnan(out), nan)
        # one rounding to bf16, 2^-8; fp32 sums over at most 600 rows and 64 channels, logits up to 64 * 5 * 5 / 8
        tol = (2.0 ** -8 if out.dtype == torch.bfloat16 else 0) + (2 * ROWS + 4 * 80 * 200) * 2.0 ** -24
        good = torch.where(nan | torch.isinf(ref), 0, ref)
        assert torch.all((torch.where(nan | torch.isinf(ref), 0, out.double()) - good).abs() <= tol * mag)
        assert torch.equal(torch.where(torch.isinf(ref), ref, 0.0), torch.where(torch.isinf(ref), out.double(), 0.0))


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pos", [0, 150, 208, 599])
def test_a_query_that_is_not_a_number(io, pos):
    x = caches(io)
    x["q"][0, 1, 9] = NAN
    check(x, pos)


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pos,row", [(599, 0), (599, 207), (599, 300), (599, 599), (208, 208), (0, 0), (416, 416)])
def test_a_key_that_is_not_a_number(io, pos, row):
    """Also where it is the only row of its range (208, 416: the token's own)."""
    x = caches(io)
    where = x["k"][0, 0] if row == pos else x["ck"][0, 0, row]
    where[3] = NAN
    check(x, pos)


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [NAN, INF])
def test_a_value_in_a_range_whose_weight_is_0(io, value):
    """The first range's logits are 200 above the others', whose weights underflow: 0 times a value that is not finite is NaN."""
    x = caches(io)
    x["q"].fill_(1.0)
    x["ck"].mul_(0.01)
    x["ck"][0, 0, 5].fill_(200.0 * 8 / D)
    x["cv"][0, 0, 300, 2] = value
    outs = ask(x, 599)
    for out in outs:
        want = torch.zeros(3, D, dtype=torch.bool, device=DEV)
        want[:, 2] = True
        assert torch.equal(torch.isnan(out), want)
        tol = 2.0 ** -8 if io == torch.bfloat16 else 2.0 ** -16
        assert torch.all((out - x["cv"][0, 0, 5])[~want].abs() <= tol * x["cv"][0, 0, 5].abs().max())


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32])
def test_logits_of_minus_infinity_and_rows_without_a_token(io):
    """Nothing but logits of -infinity: zeros.  NaN in rows beyond the position: not looked at."""
    x = caches(io)
    x["q"].abs_().add_(0.5)
    x["ck"][..., 0] = -INF
    x["k"][..., 0] = -INF
    for out in ask(x, 599):
        assert torch.count_nonzero(out) == 0
    x = caches(io)
    x["ck"][0, 0, 101:] = NAN
    x["cv"][0, 0, 101:] = NAN
    for out in ask(x, 100):
        assert torch.isfinite(out).all()
    x["ck"][0, 0, 101:] = 0
    x["cv"][0, 0, 101:] = 0
    check(x, 100)
