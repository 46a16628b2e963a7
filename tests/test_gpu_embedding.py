"""GPU: embedding lookup and its gradient against float64.

Tolerances: a lookup is one product in float32, rounded to the type of the output: half a step each.  The sum of k terms in float32, in any
order, is off by at most (k - 1) 2^-24 of the sum of their absolute values (to first order; doubled here for the rest), the scale and an
addition to what was there by 2^-24 each of what they give, and the result is rounded once to its type."""
import numpy as np
import pytest
import torch

from paper_1806_04090_amd import binding
from gpu_common import ctx

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
U = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2 if t is not F32 else U


def tiny(t):
    """Half of the smallest step of a type (numbers below its smallest normal one)."""
    return torch.finfo(t).tiny * torch.finfo(t).eps / 2


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(shape, dtype, seed):
    return torch.randn(shape, generator=generator(seed), device="cuda").to(dtype)


def some_tokens(n, rows, seed, dtype=torch.int64, few=False):
    g = generator(seed)
    x = torch.randint(0, min(rows, 3) if few else rows, (n,), generator=g, device="cuda")
    if n > 8 and not few:
        x[torch.rand(n, generator=g, device="cuda") < 0.3] = int(x[0])           # one frequent token
    return x.to(dtype)


def check_lookup(table, tokens, scale, out, padding=-1):
    bad = (tokens == padding) | (tokens < 0) | (tokens >= table.shape[0])
    want = table.double()[tokens.long().clamp(0, table.shape[0] - 1)] * float(np.float32(scale))
    want[bad] = 0.0
    err = (out.double() - want).abs()
    assert (err <= want.abs() * (U + half_step(out.dtype)) * 1.001 + tiny(out.dtype)).all()


def check_grad(tokens, dy, grad, scale=1.0, before=None, padding=-1):
    rows, n = grad.shape[0], tokens.numel()
    live = (tokens != padding) & (tokens >= 0) & (tokens < rows)
    at = tokens.long()[live]
    terms = dy.double()[:n][live]
    zero = torch.zeros(grad.shape, device="cuda", dtype=torch.float64)
    sums, sizes = zero.index_add(0, at, terms), zero.index_add(0, at, terms.abs())
    count = torch.zeros(rows, device="cuda", dtype=torch.float64).index_add(0, at, torch.ones_like(at, dtype=torch.float64))
    s = float(np.float32(scale))
    want = sums * s
    bound = sizes * abs(s) * U * (2 * count[:, None] + 1)
    if before is not None:
        want = want + before.double()
        bound = bound + U * (before.double().abs() + sizes * abs(s))
    bound = bound + (want.abs() + bound) * half_step(grad.dtype) + tiny(grad.dtype)
    assert ((grad.double() - want).abs() <= bound).all()
    named = count > 0
    if before is None:
        assert (grad[~named] == 0).all()
    else:
        assert torch.equal(grad[~named], before[~named])


# tokens, rows, columns: one of each, odd columns, single lanes, columns over a group of lanes, one row, many tokens; three digits to sort by
SIZES = [(1, 1, 1), (1, 50, 8), (7, 5, 3), (64, 33, 64), (65, 1000, 257), (300, 70, 511), (513, 129, 1030), (1000, 1, 40), (4097, 300, 72),
         (16384, 5000, 33), (16385, 700, 16), (40_000, 200_003, 24), (100_001, 17, 130), (9000, 600_001, 5)]


@pytest.mark.parametrize("n, rows, cols", SIZES)
@pytest.mark.parametrize("dtype, out_type, token_type", [(F32, F32, torch.int64), (BF16, BF16, torch.int32), (F16, F32, torch.int64), (F32, F16, torch.int32)])
def test_lookup(n, rows, cols, dtype, out_type, token_type):
    table, tokens = normal((rows, cols), dtype, n + cols), some_tokens(n, rows, n, token_type)
    out = torch.full((n, cols), float("nan"), device="cuda", dtype=out_type)
    assert binding.atomo_embedding(ctx(), table, tokens, 1.7, out=out) is out
    check_lookup(table, tokens, 1.7, out)
    assert ctx().status()[0] == 0


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n, rows, cols", SIZES)
@pytest.mark.parametrize("dtype, grad_type, token_type", [(F32, F32, torch.int64), (BF16, F32, torch.int32), (BF16, BF16, torch.int64), (F16, F16, torch.int32)])
def test_grad(n, rows, cols, dtype, grad_type, token_type, accumulate):
    dy, tokens = normal((n, cols), dtype, n + 3 * cols), some_tokens(n, rows, n, token_type)
    grad = normal((rows, cols), grad_type, 5) if accumulate else torch.full((rows, cols), float("nan"), device="cuda", dtype=grad_type)
    before = grad.clone() if accumulate else None
    assert binding.atomo_embedding_grad(ctx(), tokens, dy, grad, 0.3, accumulate=accumulate) is grad
    check_grad(tokens, dy, grad, 0.3, before)
    assert ctx().status()[0] == 0


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 5000, 20_000])
def test_few_rows_take_long_sums(n):
    # runs of one token that begin and end at every place of what a wave adds up
    dy, tokens = normal((n, 70), BF16, n), some_tokens(n, 9, n, few=True)
    grad = torch.empty(9, 70, device="cuda")
    binding.atomo_embedding_grad(ctx(), tokens, dy, grad)
    check_grad(tokens, dy, grad)
    again = torch.empty_like(grad)
    binding.atomo_embedding_grad(ctx(), tokens, dy, again)
    assert torch.equal(grad, again)                              # the order of the sum is fixed


@pytest.mark.parametrize("accumulate", [False, True])
def test_more_than_a_million_tokens(accumulate):
    # more parts of the sort, and more keys in each, than of shorter lists; whole numbers, so that every sum is exact
    n, rows = 1_100_001, 5000
    g = generator(7)
    tokens = torch.randint(0, rows, (n,), generator=g, device="cuda")
    tokens[torch.rand(n, generator=g, device="cuda") < 0.3] = 77
    value = torch.randint(-2, 3, (n,), generator=g, device="cuda")
    grad = torch.ones(rows, 2, device="cuda")
    binding.atomo_embedding_grad(ctx(), tokens, torch.stack([value, -value], 1).to(BF16), grad, accumulate=accumulate)
    order = torch.argsort(tokens)
    ends = torch.bincount(tokens, minlength=rows).cumsum(0)
    total = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), value[order].cumsum(0)])
    want = total[ends] - total[torch.cat([ends.new_zeros(1), ends[:-1]])]
    assert torch.equal(grad, torch.stack([want, -want], 1).float() + (1.0 if accumulate else 0.0))


@pytest.mark.parametrize("n", [20, 3000, 30_000])
@pytest.mark.parametrize("padding", [-1, -100, 3, 10 ** 12])
def test_padding_and_tokens_outside_of_the_table(n, padding):
    rows, cols = 50, 36
    tokens = some_tokens(n, rows, 1)
    tokens[::5] = padding
    table, dy = normal((rows, cols), F32, 2), normal((n, cols), F32, 3)
    dy[tokens == padding] = float("nan")                         # nothing of a padded place is used
    table[3 if padding == 3 else 0] = float("inf")
    out = binding.atomo_embedding(ctx(), table, tokens, 2.0, padding=padding)
    assert (out[tokens == padding] == 0).all()
    table[3 if padding == 3 else 0] = 0.0
    check_lookup(table, tokens, 2.0, torch.nan_to_num(out, posinf=0.0, neginf=0.0), padding)
    grad = torch.full((rows, cols), float("nan"), device="cuda")
    binding.atomo_embedding_grad(ctx(), tokens, dy, grad, padding=padding)
    check_grad(tokens, dy, grad, padding=padding)
    assert ctx().status()[0] == 0
    # tokens that name nothing: left out as well, and reported, once
    for wrong in (-7, rows, 2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1, -2 ** 63):
        tokens[1] = wrong
        dy[1] = float("nan")
        out = binding.atomo_embedding(ctx(), table, tokens, 2.0, padding=padding)
        assert (out[1] == 0).all() and ctx().status()[0] == binding.ATOMO_EINVAL and ctx().status()[0] == 0
        binding.atomo_embedding_grad(ctx(), tokens, dy, grad, padding=padding)
        check_grad(tokens, dy, grad, padding=padding)
        assert ctx().status()[0] == binding.ATOMO_EINVAL and ctx().status()[0] == 0


@pytest.mark.parametrize("n", [1, 100, 20_000])
def test_nothing_but_padding_and_nothing_at_all(n):
    tokens = torch.full((n,), -1, device="cuda")
    grad = torch.full((300, 70), float("nan"), device="cuda")
    binding.atomo_embedding_grad(ctx(), tokens, normal((n, 70), F32, 0), grad)
    assert (grad == 0).all()
    none = tokens[:0]
    grad.fill_(float("nan"))
    binding.atomo_embedding_grad(ctx(), none, normal((0, 70), F32, 0), grad)
    assert (grad == 0).all()
    grad.fill_(3.0)
    for t in (none, tokens):
        binding.atomo_embedding_grad(ctx(), t, normal((t.numel(), 70), F32, 0), grad, accumulate=True)
    assert (grad == 3.0).all()
    assert binding.atomo_embedding(ctx(), grad, none).shape == (0, 70)


@pytest.mark.parametrize("dtype", TYPES)
def test_row_strides_and_odd_addresses(dtype):
    n, rows, cols = 700, 90, 61
    tokens = some_tokens(n, rows, 4)
    table = normal((rows, 80), dtype, 1)[:, 7:7 + cols]
    wide = torch.full((n + 5, 75), 9.0, device="cuda", dtype=dtype)
    out = wide[:, 3:3 + cols]
    binding.atomo_embedding(ctx(), table, tokens, 0.5, out=out)
    check_lookup(table, tokens, 0.5, out[:n])
    assert (wide[:, :3] == 9).all() and (wide[:, 3 + cols:] == 9).all() and (wide[n:] == 9).all()    # rows behind the last token, columns beside
    dy = normal((n, 97), dtype, 2)[:, 5:5 + cols]
    for accumulate in (False, True):
        wide = torch.full((rows, 75), 9.0, device="cuda", dtype=dtype)
        grad = wide[:, 3:3 + cols]
        binding.atomo_embedding_grad(ctx(), tokens, dy, grad, accumulate=accumulate)
        check_grad(tokens, dy, grad, before=torch.full((rows, cols), 9.0, device="cuda", dtype=dtype) if accumulate else None)
        assert (wide[:, :3] == 9).all() and (wide[:, 3 + cols:] == 9).all()
    one = normal((1, cols), dtype, 3)
    grad = torch.empty(rows, cols, device="cuda", dtype=F32)
    binding.atomo_embedding_grad(ctx(), tokens, one.expand(n, cols), grad)       # a broadcast gradient: row stride 0
    check_grad(tokens, one.expand(n, cols), grad)


def test_tokens_of_a_batch():
    table, tokens = normal((40, 12), BF16, 1), some_tokens(24, 40, 2).view(2, 3, 4)
    out = binding.atomo_embedding(ctx(), table, tokens, 3.0)
    assert out.shape == (2, 3, 4, 12) and out.dtype == BF16
    check_lookup(table, tokens.view(-1), 3.0, out.view(-1, 12))
    grad = torch.empty(40, 12, device="cuda")
    binding.atomo_embedding_grad(ctx(), tokens, out, grad)
    check_grad(tokens.view(-1), out.view(-1, 12), grad)


def test_offsets_beyond_32_bits():
    apart = 2 ** 31 + 24
    base = torch.zeros(2 * apart + 64, device="cuda", dtype=BF16)                # 8.6 GB: three rows of 64 far from each other
    far = base.as_strided((3, 64), (apart, 1))
    far.copy_(normal((3, 64), BF16, 1))
    tokens = torch.tensor([2, 0, 2, 1, 2], device="cuda")
    out = binding.atomo_embedding(ctx(), far, tokens)
    check_lookup(far, tokens, 1.0, out)
    dy = normal((5, 64), BF16, 2)
    binding.atomo_embedding_grad(ctx(), tokens, dy, far)
    check_grad(tokens, dy, far.clone())
    far.copy_(dy[:3])
    grad = torch.empty(3, 64, device="cuda")
    binding.atomo_embedding_grad(ctx(), tokens[:3], far, grad)
    check_grad(tokens[:3], far, grad)
    binding.atomo_embedding(ctx(), dy, tokens[:3], out=far)
    check_lookup(dy, tokens[:3], 1.0, far)


def test_gradient_against_differences():
    # the lookup is linear: <dy, lookup(W + E) - lookup(W)> = <grad, E>, exactly in whole numbers
    g = generator(3)
    tokens = some_tokens(500, 64, 5)
    w, e, dy = (torch.randint(-8, 9, s, generator=g, device="cuda").float() for s in ((64, 48), (64, 48), (500, 48)))
    change = binding.atomo_embedding(ctx(), w + e, tokens, 2.0) - binding.atomo_embedding(ctx(), w, tokens, 2.0)
    grad = torch.empty(64, 48, device="cuda")
    binding.atomo_embedding_grad(ctx(), tokens, dy, grad, 2.0)
    assert (dy.double() * change.double()).sum() == (grad.double() * e.double()).sum()


@pytest.mark.parametrize("n", [200, 9000, 50_000])
def test_captured_calls_replay(n):
    rows, cols = 300, 200
    c = binding.Context(0)
    c.reserve(binding.embedding_workspace_bytes(n, rows, cols))
    table, dy = normal((rows, cols), F32, 1), normal((n, cols), F32, 2)
    tokens, out, grad = some_tokens(n, rows, 3), torch.empty(n, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        binding.atomo_embedding(c, table, tokens, 2.0, out=out)
        binding.atomo_embedding_grad(c, tokens, dy, grad)
    # a call that makes the context take a larger workspace leaves the graph its own
    more = some_tokens(4 * n + 500_000, rows, 9)
    for k in range(4):
        tokens.copy_(some_tokens(n, rows, 10 + k))
        out.fill_(float("nan"))
        grad.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check_lookup(table, tokens, 2.0, out)
        check_grad(tokens, dy, grad)
        other = torch.empty(rows, 8, device="cuda")
        binding.atomo_embedding_grad(c, more, normal((more.numel(), 8), F32, k), other)
        torch.cuda.synchronize()
    assert c.status()[0] == 0


def test_a_captured_call_allocates_nothing():
    c = binding.Context(0)
    tokens, dy, grad = some_tokens(100_000, 50, 1), normal((100_000, 4), F32, 1), torch.empty(50, 4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        with pytest.raises(binding.AtomoError) as e:
            binding.atomo_embedding_grad(c, tokens, dy, grad)
        assert e.value.status == binding.ATOMO_ENOMEM
        grad.zero_()
    binding.atomo_embedding_grad(c, tokens, dy, grad)
    check_grad(tokens, dy, grad)


def test_on_another_stream():
    c, side = binding.Context(0), torch.cuda.Stream()
    table, dy, tokens = normal((500, 300), F32, 1), normal((3000, 300), F32, 2), some_tokens(3000, 500, 3)
    grad = torch.empty(500, 300, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    out = binding.atomo_embedding(c, table, tokens, stream=side)
    binding.atomo_embedding_grad(c, tokens, dy, grad, stream=side)
    side.synchronize()
    check_lookup(table, tokens, 1.0, out)
    check_grad(tokens, dy, grad)


def test_refusals():
    c, table, tokens = ctx(), torch.zeros(5, 4, device="cuda"), torch.zeros(3, device="cuda", dtype=torch.int64)
    out = torch.zeros(3, 4, device="cuda")
    for args in ((table.double(), tokens), (table, tokens.short()), (table, tokens.float()), (table, tokens, 1.0, out.double())):
        with pytest.raises(TypeError):
            binding.atomo_embedding(c, *args)
    for args in ((table.t(), tokens), (table[0], tokens), (table.cpu(), tokens), (table, tokens.cpu()), (table, torch.zeros(6, device="cuda").long()[::2]),
                 (table, tokens, 1.0, out.t()), (table, tokens.view(3, 1), 1.0, out.view(1, 3, 4))):
        with pytest.raises(ValueError):
            binding.atomo_embedding(c, *args)
    for args in ((table, tokens, 1.0, out[:2]), (table, tokens, 1.0, torch.zeros(3, 5, device="cuda")), (table, tokens, 1.0, out[:1].expand(3, 4))):
        with pytest.raises(binding.AtomoError):
            binding.atomo_embedding(c, *args)
    for dy, grad in ((out[:2], table), (out[:, :3], table), (out, table[:0])):
        with pytest.raises(binding.AtomoError):
            binding.atomo_embedding_grad(c, tokens, dy, grad)
    with pytest.raises(TypeError):
        binding.atomo_embedding_grad(c, tokens, out, table.int())
    assert c.status()[0] == 0
