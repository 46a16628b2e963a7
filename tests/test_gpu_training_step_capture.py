"""GPU: the training step's calls in a capture of torch's default mode."""
import pytest
import torch

from paper_1806_04090_amd import binding

pytestmark = pytest.mark.gpu


class Buffers:
    def __init__(self, n=9000, rows=300, cols=64):
        self.c = binding.Context(0)
        self.c.reserve(binding.embedding_workspace_bytes(n, rows, cols))
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        self.tokens = torch.randint(0, rows, (n,), generator=g, device="cuda")
        self.table = torch.randn(rows, cols, generator=g, device="cuda")
        self.out, self.grad = torch.empty(n, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
        self.p, self.s = torch.zeros(rows * cols, device="cuda"), binding.alloc_adamw_state(rows * cols, 8, "cuda")
        self.plan = binding.AdamwPlan(self.c, [self.p], [self.grad.view(-1)], [self.s])
        self.norm, self.values = torch.empty(1, device="cuda"), torch.empty(rows * cols, device="cuda")
        torch.cuda.synchronize()

    def calls(self):
        binding.atomo_embedding(self.c, self.table, self.tokens, 1.0, out=self.out)
        binding.atomo_embedding_grad(self.c, self.tokens, self.out, self.grad)
        binding.atomo_adamw_grad_norm(self.c, self.plan, out=self.norm)
        binding.atomo_adamw_step(self.c, self.plan, 1e-2, step=1, grad_norm=self.norm)
        binding.atomo_state8_unpack(self.c, "m", self.s.m, self.s.m_scale, out=self.values)

    def results(self):
        return self.out, self.grad, self.norm, self.p, self.s.m, self.s.v, self.values


def test_captured_in_the_default_mode():
    a, b = Buffers(), Buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.calls()
    for k in range(3):
        graph.replay()
        b.calls()
        torch.cuda.synchronize()
        for x, y in zip(a.results(), b.results()):
            assert torch.equal(x, y), k
    assert a.c.status()[0] == 0
