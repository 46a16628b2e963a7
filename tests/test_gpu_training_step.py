"""GPU: the calls around the method together, as a training step makes them: lookup, the gradient of the table (sent as an
entry-wise message and decoded again), the norm of all gradients, the clipped AdamW step."""
import numpy as np
import pytest
import torch

from paper_1806_04090_amd import binding

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
VOCAB, DIM, OUT, TOKENS = 400, 96, 33, 1500
B1, B2, EPS, LR, DECAY, MAX_NORM = 0.9, 0.999, 1e-8, 1e-2, 0.1, 0.05


class Model:
    """logits = (scale * E[tokens]) W, loss = |logits - target|^2 / 2: its gradients are plain products."""

    def __init__(self, bits, through_message):
        self.c, self.through_message, self.t = binding.Context(0), through_message, 0
        g = torch.Generator(device="cuda")
        g.manual_seed(3)
        self.table = torch.randn(VOCAB, DIM, generator=g, device="cuda") * 0.02
        self.w = torch.randn(DIM, OUT, generator=g, device="cuda") * 0.1
        self.copy = torch.zeros(VOCAB, DIM, device="cuda", dtype=BF16)
        self.copy.copy_(self.table)
        self.tokens = torch.zeros(3, TOKENS // 3, dtype=torch.int64, device="cuda")
        self.target = torch.zeros(TOKENS, OUT, device="cuda")
        self.g_table, self.g_w = torch.zeros(VOCAB, DIM, device="cuda"), torch.zeros(DIM, OUT, device="cuda")
        self.states = [binding.alloc_adamw_state(n, bits, "cuda") for n in (VOCAB * DIM, DIM * OUT)]
        self.plan = binding.AdamwPlan(self.c, [self.table, self.w], [self.g_table, self.g_w], self.states, copies=[self.copy, None],
                                      weight_decay=[DECAY, 0.0], lr_mult=[0.5, 1.0])
        self.x = torch.empty(3, TOKENS // 3, DIM, device="cuda")
        self.norm = torch.empty(1, device="cuda")
        self.step_count = torch.zeros(1, dtype=torch.int64, device="cuda")

    def load(self, t):
        g = torch.Generator(device="cuda")
        g.manual_seed(100 + t)
        self.tokens.copy_(torch.randint(0, VOCAB // 2 if t % 2 else VOCAB, self.tokens.shape, generator=g, device="cuda"))
        self.tokens[:, -20:] = -1
        self.target.copy_(torch.randn(TOKENS, OUT, generator=g, device="cuda"))

    def step(self, count):
        scale = DIM ** 0.5
        binding.atomo_embedding(self.c, self.copy, self.tokens, scale, out=self.x)
        x = self.x.view(TOKENS, DIM)
        d_logits = (x @ self.w - self.target) * (self.tokens.view(-1, 1) >= 0) / TOKENS
        torch.mm(x.t(), d_logits, out=self.g_w)
        dx = (d_logits @ self.w.t()).view(3, TOKENS // 3, DIM)
        binding.atomo_embedding_grad(self.c, self.tokens, dx, self.g_table, scale)
        if self.through_message:                                 # a budget of all elements: every entry is kept as it is
            n = VOCAB * DIM
            msg = binding.alloc_entrywise_message(n, n, "cuda")
            binding.atomo_encode_entrywise(self.c, self.g_table.view(-1), float(n), 1, self.t, msg=msg)
            binding.atomo_decode(self.c, [msg], 1.0, out=self.g_table.view(-1))
        binding.atomo_adamw_grad_norm(self.c, self.plan, out=self.norm)
        binding.atomo_adamw_step(self.c, self.plan, LR, B1, B2, EPS, step=count, grad_norm=self.norm, max_norm=MAX_NORM, seed=11)

    def state(self, j):
        s = self.states[j]
        if s.m_scale is None:
            return s.m, s.v
        return tuple(binding.atomo_state8_unpack(self.c, k, q, e) for k, q, e in (("m", s.m, s.m_scale), ("v", s.v, s.v_scale)))


def reference_step(model, before, t):
    """Norm and parameters after the step, in float64, from the model's parameters and states before it."""
    (table, copy, w), states = before
    live = (model.tokens.view(-1) >= 0)
    at = model.tokens.view(-1).clamp(min=0)
    scale = DIM ** 0.5
    x = copy.double()[at] * scale * live[:, None]
    d_logits = (x @ w - model.target.double()) * live[:, None] / TOKENS
    g_w = x.t() @ d_logits
    g_table = torch.zeros(VOCAB, DIM, dtype=torch.float64, device="cuda").index_add(0, at, (d_logits @ w.t()) * live[:, None]) * scale
    norm = torch.sqrt(g_w.square().sum() + g_table.square().sum())
    out = []
    for p, g, (m, v), mult, decay in ((table, g_table, states[0], 0.5, DECAY), (w, g_w, states[1], 1.0, 0.0)):
        g = g * min(1.0, MAX_NORM / float(norm))
        m, v = B1 * m.view_as(p) + (1 - B1) * g, B2 * v.view_as(p) + (1 - B2) * g * g
        out.append((p - LR * mult * (m / (1 - B1 ** t) / ((v / (1 - B2 ** t)).sqrt() + EPS) + decay * p), g))
    return norm, out


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("through_message", [False, True])
def test_steps_against_float64(bits, through_message):
    model = Model(bits, through_message)
    for t in range(1, 5):
        model.load(t)
        model.t = t
        before = [x.double() for x in (model.table, model.copy, model.w)], [[y.double() for y in model.state(j)] for j in range(2)]
        model.step(t)
        norm, want = reference_step(model, before, t)
        # the norm: sums of at most TOKENS products of float32 numbers that were rounded a few times each
        assert abs(float(model.norm) - float(norm)) <= 1e-4 * float(norm)
        for got, old, (p, g) in zip((model.table, model.w), (before[0][0], before[0][2]), want):
            # a step is at most ten times the rate here (t <= 4); where |g| is not lost in the roundings of its sum, it is right to a thousandth of that
            sure = g.abs() > 1e-3 * g.abs().max()
            assert ((got.double() - p).abs()[sure] <= 1e-3 * 10 * LR).all()
            assert ((got.double() - old).abs() <= 10 * LR * 1.2).all()
        assert torch.equal(model.copy, model.table.to(BF16))
        # rows that no token has named so far have no gradient, and nothing but decay
        if t == 1:
            unnamed = torch.ones(VOCAB, dtype=torch.bool, device="cuda")
            unnamed[model.tokens[model.tokens >= 0]] = False
            assert unnamed.sum() >= VOCAB // 2 and (model.g_table[unnamed] == 0).all()
            change = model.table[unnamed].double() - before[0][0][unnamed] * (1 - LR * 0.5 * DECAY)
            assert change.abs().max() <= 3 * 2.0 ** -24 * float(before[0][0].abs().max())
    assert model.c.status()[0] == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_replays(bits):
    """Embedding, gradient, norm and update in one graph, its count of steps on the device, against the same steps made one by one."""
    a, b = Model(bits, False), Model(bits, False)
    a.c.reserve(binding.embedding_workspace_bytes(TOKENS, VOCAB, DIM))
    warm = torch.ones(8, 8, device="cuda") @ torch.ones(8, 8, device="cuda")     # (the library's own set-up is no part of the graph)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        a.step_count.add_(1)
        a.step(a.step_count)
    for t in range(1, 6):
        a.load(t)
        b.load(t)
        graph.replay()
        b.step(t)
        torch.cuda.synchronize()
        assert torch.equal(a.g_table, b.g_table) or (a.g_table - b.g_table).abs().max() <= 1e-5 * b.g_table.abs().max()
        assert abs(float(a.norm) - float(b.norm)) <= 1e-5 * float(b.norm)
        sure = b.g_table.abs() > 1e-3 * b.g_table.abs().max()
        assert ((a.table - b.table).abs()[sure] <= 1e-3 * 10 * LR * t).all()
    assert int(a.step_count) == 5 and float(warm[0, 0]) == 8.0


def test_two_graphs_of_one_context_take_turns():
    c = binding.Context(0)
    sizes = [(3000, 50, 64), (9000, 300, 20)]
    c.reserve(max(binding.embedding_workspace_bytes(*s) for s in sizes))
    tokens = [torch.zeros(n, dtype=torch.int64, device="cuda") for n, _, _ in sizes]
    dy = [torch.ones(n, cols, device="cuda") for n, _, cols in sizes]
    grads = [torch.empty(rows, cols, device="cuda") for _, rows, cols in sizes]
    graphs = []
    for x, d, g in zip(tokens, dy, grads):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], capture_error_mode="relaxed"):
            binding.atomo_embedding_grad(c, x, d, g)
    for turn in range(6):
        for k in (0, 1) if turn % 2 else (1, 0):
            tokens[k].copy_(torch.randint(0, sizes[k][1], (sizes[k][0],), device="cuda"))
            grads[k].fill_(float("nan"))
            graphs[k].replay()
        torch.cuda.synchronize()
        for k in range(2):                                       # sums of ones: exact
            counts = torch.bincount(tokens[k], minlength=sizes[k][1]).float()
            assert torch.equal(grads[k], counts[:, None].expand_as(grads[k]))
