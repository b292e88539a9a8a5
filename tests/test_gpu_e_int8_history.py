"""The int8 history (cache type CB_INT8) on a GPU: what the cache write stores, bit by bit, and what
skipped steps read from it, against plain arithmetic in 64 bits.

Bounds (u = 2^-24), from the operations alone: a term w_j s_j q_j is off by the rounding of w_j, of
w_j s_j and of at most K additions, so a prediction by (K + 2) u sum_j |w_j s_j q_j| before its
one rounding to the output's type (half a step: 2^-9 of the next power of two in bf16, u in fp32).
A hidden state adds the roundings of its own sum, one per member and of everything it holds."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BLOCK = 64
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def cb():
    from paper_2608_23429_gb300 import build
    build.build()
    from paper_2608_23429_gb300 import chebboost
    return chebboost


def codes_of(x32):
    """Codes and scales (fp32) of a flat fp32 array, by the header's definition."""
    n = x32.size
    v = np.zeros(-(-n // BLOCK) * BLOCK, dtype=np.float32)
    v[:n] = x32
    v = v.reshape(-1, BLOCK)
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.abs(v).max(1) * np.float32(1.0 / 127.0)  # a NaN wins
        bits = ((s.view(np.uint32).astype(np.uint64) + 0xFFFF) & 0xFFFF0000).astype(np.uint32)
        s = np.where(np.isfinite(s), np.maximum(bits.view(np.float32), np.float32(2.0 ** -126)), np.float32(np.nan))
        q = np.rint(v * (np.float32(1.0) / s)[:, None])
    return q, s.astype(np.float32)


def slot_bytes(numels):
    return sum(-(-n // 256) * 256 + -(-2 * (-(-n // BLOCK)) // 256) * 256 for n in numels)


def slot_views(arena, slot, numels):
    """(codes, scale bits) of every tensor in a slot."""
    out, o = [], slot * slot_bytes(numels)
    for n in numels:
        blocks = -(-n // BLOCK)
        s0 = o + -(-n // 256) * 256
        out.append((arena[o:o + blocks * BLOCK].view(np.int8), arena[s0:s0 + 2 * blocks].view(np.uint16)))
        o = s0 + -(-2 * blocks // 256) * 256
    return out


def make_plan(cb, numels, groups, K, shapes=None):
    nodes = [999.0 - 40.0 * j for j in range(max(K, 2) + 3)]
    plan = cb.cb_plan_create(nodes, K, [(i, 0, n, g) for i, (n, g) in enumerate(zip(numels, groups))], cb.CB_INT8, 0.0, 999.0)
    if shapes:
        cb.cb_plan_set_shapes(plan, shapes)
    arena = torch.full((cb.cb_plan_cache_bytes(plan),), 0x5A, dtype=torch.uint8, device="cuda")
    cb.cb_plan_bind_cache(plan, arena, arena.numel())
    return plan, arena, nodes


def at_offset(t, off):
    """A copy of t that starts `off` elements behind a 256-byte boundary."""
    buf = torch.empty(t.numel() + off + 8, dtype=t.dtype, device="cuda")
    v = buf[off:off + t.numel()].view(t.shape)
    v.copy_(t)
    return v


SPECIAL = [0.0, -0.0, 1e-45, -3e-39, 2.0 ** -126, 1.0, -1.0, 127.0, 0.5, 1.5, 2.5, -2.5, 3.0e38, -3.3e38]


@pytest.mark.parametrize("feat", ["bf16", "fp32"])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("with_hidden", [False, True])
def test_write_is_bit_exact(cb, feat, off, with_hidden):
    numels = [1, 7, 63, 64, 65, 255, 256, 257, 2048, 4099, 3 * 333 * 577]
    g = torch.Generator().manual_seed(11 + off)
    feats = [torch.randn(n, generator=g) * torch.exp(3 * torch.randn(n, generator=g)) for n in numels]
    feats[4][:len(SPECIAL)] = torch.tensor(SPECIAL)
    feats[5][:] = 0.0
    feats[6][:] = 1e-42
    feats[7][:128] = torch.arange(128) - 64.0  # many ties
    feats = [at_offset(f.to(DT[feat]).cuda(), off) for f in feats]
    plan, arena, nodes = make_plan(cb, numels, list(range(len(numels))) if with_hidden else [-1] * len(numels), 2)
    code = cb.CB_BF16 if feat == "bf16" else cb.CB_FP32
    if with_hidden:
        x = [torch.zeros(n, device="cuda") for n in numels]
        cb.cb_cache_push_residual(plan, feats, code, nodes[0], x, cb.CB_FP32)
        for a, f in zip(x, feats):
            assert torch.equal(a, f.float() + 0.0)
    else:
        cb.cb_cache_push(plan, feats, code, nodes[0])
    torch.cuda.synchronize()
    host = arena.cpu().numpy()
    assert host[slot_bytes(numels):-cb.CB_STATUS_BYTES].min() == host[slot_bytes(numels):-cb.CB_STATUS_BYTES].max() == 0x5A
    for f, (q, s) in zip(feats, slot_views(host, 0, numels)):
        q0, s0 = codes_of(f.float().cpu().numpy())
        assert np.array_equal(s, (s0.view(np.uint32) >> 16).astype(np.uint16))
        assert np.array_equal(q.reshape(q0.shape), q0.astype(np.int8))
        held = q0.astype(np.float64) * s0[:, None]
        off_by = np.abs(held.ravel()[:f.numel()] - f.double().cpu().numpy())
        # half a step, and the roundings of 1/s and of x/s (each u of 127.5 steps at most)
        assert (off_by <= np.repeat(s0.astype(np.float64), BLOCK)[:f.numel()] * (0.5 + 256 * U)).all()
    cb.cb_plan_destroy(plan)


def test_blocks_with_values_that_are_not_finite(cb):
    numels = [64 * 6]
    f = torch.ones(64 * 6)
    f[3], f[64 + 9], f[128 + 1] = float("nan"), float("inf"), float("-inf")
    plan, arena, nodes = make_plan(cb, numels, [-1], 2)
    cb.cb_cache_push(plan, [f.cuda()], cb.CB_FP32, nodes[0])
    cb.cb_cache_push(plan, [torch.ones(384, device="cuda")], cb.CB_FP32, nodes[1])
    out = torch.zeros(384, device="cuda")
    cb.cb_extrapolate(plan, nodes[2], [out], cb.CB_FP32)
    got = out.cpu().numpy()
    assert np.isnan(got[:192]).all() and np.isfinite(got[192:]).all()
    cb.cb_plan_destroy(plan)


def lagrange(nodes, t):
    if t in nodes:
        return np.array([float(a == t) for a in nodes])
    return np.array([np.prod([(t - b) / (a - b) for b in nodes if b != a]) for a in nodes])


def near(got, want, slack, dtype):
    """got within `slack` of want before its rounding to dtype."""
    got = got.double().cpu().numpy().ravel()
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.maximum(np.abs(want) + slack, 2.0 ** -126)))
    half = np.exp2(e - 8) if dtype == "bf16" else np.exp2(e - 24)
    bad = ~(np.abs(got - want) <= slack + half)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], slack[bad][:4])


CASES = [
    # K, shapes of a group's members, members per group, io, gates, offset of outputs and hidden states
    (1, [(1, 1, 1)], 1, "bf16", None, 0),
    (2, [(1, 5, 13)], 2, "fp32", None, 0),
    (3, [(2, 77, 768)], 2, "bf16", "bf16", 0),
    (4, [(3, 33, 577)], 3, "bf16", "bf16", 1),
    (4, [(3, 33, 577)], 3, "fp32", "fp32", 3),
    (5, [(2, 64, 96), (1, 50, 72)], 1, "bf16", "fp32", 0),
    (5, [(2, 41, 1152)], 4, "fp32", "bf16", 0),
    (6, [(1, 256, 130), (4, 7, 24)], 2, "bf16", None, 8),
    (7, [(2, 19, 264)], 1, "bf16", "bf16", 4),
    (8, [(1, 300, 1152), (1, 1, 4097)], 2, "bf16", "bf16", 0),
    (8, [(2, 100, 513)], 2, "fp32", None, 1),
]


def filled(cb, K, shapes, nb, seed=0, steps=None, feat="bf16"):
    members = [s for s in shapes for _ in range(nb)]
    groups = [i // nb for i in range(len(members))]
    numels = [int(np.prod(s)) for s in members]
    plan, arena, nodes = make_plan(cb, numels, groups, K, members)
    g = torch.Generator().manual_seed(seed)
    held = []
    for j in range(K if steps is None else steps):
        fs = [torch.randn(s, generator=g).to(DT[feat]) for s in members]
        cb.cb_cache_push(plan, [f.cuda() for f in fs], cb.CB_BF16 if feat == "bf16" else cb.CB_FP32, nodes[j])
        held.append([np.concatenate([(q * s.astype(np.float64)[:, None]).ravel()]) [:f.numel()]
                     for f in fs for q, s in [codes_of(f.float().numpy().ravel())]])
    return plan, arena, nodes, members, groups, held


def expect(held, w, i):
    p = sum(wj * h[i] for wj, h in zip(w, held))
    size = sum(abs(wj) * np.abs(h[i]) for wj, h in zip(w, held))
    return p, (len(w) + 2) * U * size


@pytest.mark.parametrize("K,shapes,nb,io,gate,off", CASES)
@pytest.mark.parametrize("preds,hidden", [(True, False), (False, True), (True, True)])
def test_skipped_step(cb, K, shapes, nb, io, gate, off, preds, hidden):
    plan, arena, nodes, members, groups, held = filled(cb, K, shapes, nb, seed=K)
    t = nodes[K - 1] - 17.0
    w = lagrange(nodes[:K], t)
    g = torch.Generator().manual_seed(99)
    gates = [torch.randn(s[0], s[2], generator=g).to(DT[gate]).cuda() for s in members] if gate and hidden else None
    outs = [at_offset(torch.full(s, float("nan"), dtype=DT[io]).cuda(), off) for s in members] if preds else None
    x0 = [torch.randn(s, generator=g).to(DT[io]) for s in shapes]
    xs = [at_offset(x.cuda(), off) for x in x0] if hidden else None
    code = cb.CB_BF16 if io == "bf16" else cb.CB_FP32
    if gates:
        cb.cb_extrapolate_gated(plan, t, outs, code, xs, code, gates, cb.CB_BF16 if gate == "bf16" else cb.CB_FP32)
    else:
        cb.cb_extrapolate(plan, t, outs, code, xs, code)
    torch.cuda.synchronize()
    for grp, s in enumerate(shapes):
        total = x0[grp].double().numpy().ravel()
        size, slack = np.abs(total), 0.0
        for i in [i for i, gi in enumerate(groups) if gi == grp]:
            p, e = expect(held, w, i)
            if preds:
                near(outs[i], p, e, io)
            gv = gates[i].double().cpu().numpy()[:, None, :] if gates else np.ones((1, 1, 1))
            gv = np.broadcast_to(gv, s).ravel()
            total, size, slack = total + gv * p, size + np.abs(gv * p), slack + np.abs(gv) * e
        if hidden:
            near(xs[grp], total, slack + 1.01 * nb * U * size, io)
    cb.cb_plan_destroy(plan)


def test_every_entry_point_reads_the_same(cb):
    K, shapes, nb = 4, [(2, 40, 136)], 2
    plan, arena, nodes, members, groups, held = filled(cb, K, shapes, nb, seed=5, steps=6)  # the ring has turned
    live = nodes[2:6]
    t = nodes[5] - 9.0
    outs = lambda: [torch.zeros(s, device="cuda") for s in members]  # noqa: E731
    a, b, c, d = outs(), outs(), outs(), outs()
    cb.cb_extrapolate(plan, t, a, cb.CB_FP32)
    for i in range(len(members)):
        near(a[i], *expect(held[2:], lagrange(live, t), i), "fp32")
    slot_t, head, count = cb.cb_plan_history(plan, K)
    assert count == K
    cb.cb_extrapolate_ring(plan, slot_t, head, t, b, cb.CB_FP32)
    st = torch.full((1,), 7, dtype=torch.int32).pin_memory()
    cb.cb_extrapolate_noalloc(plan, arena, arena.numel() - cb.CB_STATUS_BYTES, slot_t, head, t, c, cb.CB_FP32, status=st)
    cb.cb_extrapolate_weights(plan, cb.cb_weights(plan, t), d, cb.CB_FP32)
    torch.cuda.synchronize()
    assert int(st[0]) == 0 and cb.cb_plan_device_status(plan) == 0
    for other in (b, c, d):
        assert all(torch.equal(u, v) for u, v in zip(a, other))
    # a target on a node returns what that entry holds
    cb.cb_extrapolate(plan, live[1], a, cb.CB_FP32)
    for i in range(len(members)):
        assert np.array_equal(a[i].double().cpu().numpy().ravel(), held[3][i])
    # no weight at all
    cb.cb_extrapolate_weights(plan, np.zeros(K), a, cb.CB_FP32)
    assert all(float(v.abs().max()) == 0.0 for v in a)
    cb.cb_plan_destroy(plan)


def test_partial_history_side_stream_and_empty_entries(cb):
    plan, arena, nodes, members, groups, held = filled(cb, 5, [(1, 30, 200), (1, 9, 64)], 2, seed=8, steps=2)
    with pytest.raises(cb.CbError) as e:
        cb.cb_extrapolate(plan, 700.0, [None] * 4, cb.CB_BF16)
    assert e.value.status == cb.CB_ERR_HISTORY_NOT_FULL
    cb.cb_plan_set_option(plan, cb.CB_OPT_PARTIAL_HISTORY, 1)
    t = nodes[1] - 11.0
    w = lagrange(nodes[:2], t)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = torch.zeros(members[1], device="cuda")
    x = torch.ones(members[3], device="cuda")
    torch.cuda.synchronize()
    cb.cb_extrapolate(plan, t, [None, out, None, None], cb.CB_FP32, [None, x], cb.CB_FP32, stream=s)
    s.synchronize()
    near(out, *expect(held, w, 1), "fp32")
    (p2, e2), (p3, e3) = expect(held, w, 2), expect(held, w, 3)
    near(x, 1.0 + p2 + p3, e2 + e3 + 2.02 * U * (1 + np.abs(p2) + np.abs(p3)), "fp32")
    cb.cb_plan_destroy(plan)


def test_step_in_a_graph_follows_the_history(cb):
    plan, arena, nodes, members, groups, held = filled(cb, 2, [(1, 16, 64)], 1, seed=3)
    out = torch.zeros(members[0], device="cuda")
    t = nodes[1] - 20.0
    cb.cb_extrapolate(plan, t, [out], cb.CB_FP32)
    torch.cuda.synchronize()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            cb.cb_extrapolate(plan, t, [out], cb.CB_FP32, stream=torch.cuda.current_stream())
    want = out.clone()
    arena[:slot_bytes([1024])].zero_()  # the graph reads what the arena holds when it runs
    graph.replay()
    torch.cuda.synchronize()
    near(out, *expect(held[1:], lagrange(nodes[:2], t)[1:], 0), "fp32")
    assert not torch.equal(out, want)
    cb.cb_plan_destroy(plan)


def test_offsets_beyond_2_31(cb):
    n = (1 << 31) + 4099
    plan, arena, nodes = make_plan(cb, [n], [0], 2)
    f = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, (1 << 31) - 1, 1 << 31, (1 << 31) + 1, n - 4096, n - 2, n - 1], device="cuda")
    for j, t in enumerate(nodes[:2]):
        f.fill_(0.25)
        f[at] = torch.arange(8, device="cuda").to(torch.bfloat16) * (j + 1) / 8
        cb.cb_cache_push(plan, [f], cb.CB_BF16, t)
    f.zero_()
    cb.cb_extrapolate(plan, nodes[2], None, cb.CB_BF16, [f], cb.CB_BF16)  # weights (-1, 2)
    got = f[at].double().cpu().numpy()
    # a value is held within half a step of its block's largest (7/4 at most), with weights 1 and 2
    assert (np.abs(got - (np.arange(8) * 3 / 8)) <= 3 * 0.5 * 1.01 * 1.75 / 127 + 2.0 ** -8 * 3).all()
    cb.cb_plan_destroy(plan)


def test_refusals(cb):
    plan, arena, nodes, members, groups, held = filled(cb, 2, [(1, 4, 64)], 1)
    out = torch.zeros(4, 64, device="cuda")

    def status(f, *a, **kw):
        with pytest.raises(cb.CbError) as e:
            f(*a, **kw)
        return e.value.status

    for bad in (cb.CB_INT8, cb.CB_E4M3, 9):
        assert status(cb.cb_cache_push, plan, [out], bad, nodes[2]) == cb.CB_ERR_ARG
        assert status(cb.cb_extrapolate, plan, nodes[2], [out], bad) == cb.CB_ERR_ARG
        assert status(cb.cb_extrapolate, plan, nodes[2], None, cb.CB_FP32, [out], bad) == cb.CB_ERR_ARG
        assert status(cb.cb_cache_push_residual, plan, [out], cb.CB_FP32, nodes[2], [out], bad) == cb.CB_ERR_ARG
    assert status(cb.cb_cache_push, plan, [out], cb.CB_FP32, nodes[1]) == cb.CB_ERR_ORDER
    assert status(cb.cb_cache_push, plan, [out.data_ptr() + 2], cb.CB_FP32, nodes[2]) == cb.CB_ERR_ALIGN
    assert status(cb.cb_extrapolate, plan, nodes[2], [out.data_ptr() + 1], cb.CB_BF16) == cb.CB_ERR_ALIGN
    assert cb.cb_plan_history(plan, 2)[2] == 2 and cb.cb_plan_history(plan, 2)[0][1] == nodes[1]
    cb.cb_plan_destroy(plan)
