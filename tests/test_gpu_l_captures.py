"""A sequence of the full step's operators in one graph, each call on the results of the one before: calls whose launches overlap the end of
the previous kernel stand right behind ones that give memory back, and behind copies and clearings."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import block, chebboost
    return block, chebboost


class Sequence:
    """Off the grid -> norm -> few rows; off the grid -> on the grid -> parts of K -> int8 history -> prediction."""

    def __init__(self, lib):
        self.block, self.cb = lib
        block, cb = lib
        g = torch.Generator(device="cuda").manual_seed(4)
        r = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
        self.x, self.source = r(100, 333), r(100, 333)
        self.w = [r(640, 333) / 18, r(384, 640) / 25, r(4608, 640) / 25, r(72, 4608) / 68]
        self.layers = [block.cb_linear_create(w, *w.shape, cb.CB_BF16) for w in self.w]
        e = lambda *s: torch.empty(s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        self.a, self.b, self.c, self.d, self.e, self.f, self.p = (e(100, 640), e(100, 640), e(8, 384), e(100, 640), e(100, 4608), e(100, 72),
                                                                  e(100, 72))
        self.io, self.few = block.cb_linear_io(rows=100, out_dtype=cb.CB_BF16), block.cb_linear_io(rows=8, out_dtype=cb.CB_BF16)
        self.norm = block.cb_norm_desc(rows=100, hidden=640, x_dtype=cb.CB_BF16, out_dtype=cb.CB_BF16, eps=1e-6)
        self.plan = cb.cb_plan_create([9.0, 8.0], 1, [(0, 0, 7200, 0)], cb.CB_INT8, 0.0, 10.0)
        self.arena = torch.zeros(cb.cb_plan_cache_bytes(self.plan), dtype=torch.uint8, device="cuda")
        cb.cb_plan_bind_cache(self.plan, self.arena, self.arena.numel())

    def run(self, s):
        block, cb, L = self.block, self.cb, self.layers
        self.x.copy_(self.source)
        block.cb_linear_run(L[0], self.io, self.x, out=self.a, stream=s)
        block.cb_norm_residual(self.norm, self.a, out=self.b, stream=s)
        block.cb_linear_run(L[1], self.few, self.b, out=self.c, stream=s)
        block.cb_linear_run(L[0], self.io, self.x, out=self.d, stream=s)
        block.cb_linear_run(L[2], self.io, self.d, out=self.e, stream=s)
        block.cb_linear_run(L[3], self.io, self.e, out=self.f, stream=s)
        cb.cb_plan_reset(self.plan)
        cb.cb_cache_push(self.plan, [self.f], cb.CB_BF16, 9.0, s)
        cb.cb_extrapolate(self.plan, 9.0, [self.p], cb.CB_BF16, None, cb.CB_BF16, s)
        return [t.clone() for t in (self.a, self.b, self.c, self.d, self.e, self.f, self.p)]

    def close(self):
        self.cb.cb_plan_destroy(self.plan)
        for layer in self.layers:
            self.block.cb_linear_destroy(layer)


def test_a_full_step_in_one_graph(lib):
    q = Sequence(lib)
    s = torch.cuda.Stream()
    sources = [torch.randn(100, 333, device="cuda").bfloat16() for _ in range(4)]
    want = []
    with torch.cuda.stream(s):
        for x in sources:
            q.source.copy_(x)
            want.append(q.run(torch.cuda.current_stream()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
        got = q.run(torch.cuda.current_stream())
    for turn in range(3):
        for x, y in zip(sources, want):
            with torch.cuda.stream(s):
                q.source.copy_(x)
                graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, y)), turn
    assert lib[0].cb_linear_device_status() == 0 and lib[1].cb_plan_device_status(q.plan) == 0
    q.close()
