"""The expert layers with a routing that is given, alone and behind the router, beside a shared expert of FP8 projections."""
import numpy as np
import pytest
import torch

from oracle import formats as F
from oracle import fp8 as P
from oracle import fp8_linear as L
from oracle import moe as M
from oracle import router as R

pytestmark = pytest.mark.gpu
H, I, E, K = 256, 128, 16, 4


@pytest.fixture(scope="module")
def B():
    from paper_2607_15810_b200 import binding
    return binding


def _bf(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(torch.bfloat16)


@pytest.fixture(scope="module")
def layer(B):
    g = torch.Generator().manual_seed(5)
    w13, w2 = _bf(g, E, 2 * I, H, scale=0.05), _bf(g, E, H, I, scale=0.05)
    packed = [B.fake_quant_weights(w.cuda(), want_fq=False, sf_layout=B.SF_TILED) for w in (w13, w2)]
    fp8 = [B.fp8_quantize_weights(w.cuda()) for w in (w13, w2)]
    return dict(w13=w13, w2=w2, packed=packed, fp8=fp8, a2=torch.tensor([0.01]).cuda())


def _calls(B, layer, n13=H // 2, n2=I // 2):
    """The two layers as functions of (x, logits, routing)."""
    return {
        "w4a4": lambda x, lg, rt, **kw: B.moe_w4a4_rac(x, lg, *layer["packed"], K, n13, n2, layer["a2"], routing=rt, **kw),
        "fp8": lambda x, lg, rt, **kw: B.moe_fp8_w8a8(x, lg, *layer["fp8"], K, routing=rt, **kw),
    }


def _x(T, seed=1):
    return _bf(torch.Generator().manual_seed(seed), T, H).cuda()


def _ids(T, seed=2):
    g = torch.Generator().manual_seed(seed)
    return torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(T)]).to(torch.int32).cuda()


# (the FP8 layer writes no weights out; those of the other one are the same bits where both take them from the same kernel: up to 128 and
# from 513 tokens on)
@pytest.mark.parametrize("kind,T", [("w4a4", T) for T in (1, 7, 60, 128, 129, 500, 513, 3000)] + [("fp8", T) for T in (1, 7, 60, 128, 513, 3000)])
@pytest.mark.parametrize("renorm", [True, False])
def test_the_layers_own_routing_given_back(B, layer, kind, T, renorm):
    call = _calls(B, layer)[kind]
    x, lg = _x(T), torch.randn(T, E, generator=torch.Generator().manual_seed(T)).cuda()
    own = call(x, lg, None, renormalize=renorm)
    exp = B.moe_w4a4_rac(x, lg, *layer["packed"], K, H // 2, I // 2, layer["a2"], renormalize=renorm, export=True)
    given = call(x, None, (exp["ids"], exp["weights"]))
    assert torch.equal(own["out"], given["out"])
    assert B.moe_async_status(given["workspace"]) == 0
    if kind == "w4a4":
        full = call(x, None, (exp["ids"], exp["weights"]), export=True)
        for k in ("ids", "weights", "offsets", "perm", "hq", "sel2", "out"):
            assert torch.equal(full[k], exp[k]), k


@pytest.mark.parametrize("kind", ["w4a4", "fp8"])
@pytest.mark.parametrize("T", [1, 60, 500, 700])
def test_empty_slots(B, layer, kind, T):
    """A slot without an expert is a slot of weight 0 (no residual compensation: its selection sees all rows)."""
    call = _calls(B, layer, 0, 0)[kind]
    x, ids = _x(T), _ids(T)
    w = torch.rand(T, K, generator=torch.Generator().manual_seed(3)).cuda()
    gone = torch.rand(T, K, generator=torch.Generator().manual_seed(4)).cuda() < 0.4
    gone[::3] = True                                       # tokens without any expert
    want = call(x, None, (ids, w.masked_fill(gone, 0.0)))["out"]
    for none in (-1, E, 2 ** 30, -2 ** 31):
        got = call(x, None, (ids.masked_fill(gone, none), w))
        assert torch.equal(got["out"], want) and B.moe_async_status(got["workspace"]) == 0
    assert (want[::3] == 0).all()


@pytest.mark.parametrize("kind", ["w4a4", "fp8"])
@pytest.mark.parametrize("T", [1, 60, 600])
def test_no_expert_at_all(B, layer, kind, T):
    for n in (0, 64):
        r = _calls(B, layer, n, n)[kind](_x(T), None, (torch.full((T, K), -1, dtype=torch.int32).cuda(), torch.ones(T, K).cuda()))
        assert (r["out"] == 0).all() and B.moe_async_status(r["workspace"]) == 0


@pytest.mark.parametrize("kind", ["w4a4", "fp8"])
@pytest.mark.parametrize("T", [1, 60, 500, 700])
def test_an_expert_named_twice(B, layer, kind, T):
    call = _calls(B, layer, 0, 0)[kind]
    x, e = _x(T), _ids(T)[:, :1]
    none = torch.full_like(e, -1)
    half = torch.full((T, 1), 0.5).cuda()
    for order in ([e, e, none, none], [none, e, none, e]):
        w = torch.cat([torch.zeros_like(half) if o is none else half for o in order], 1)
        got = call(x, None, (torch.cat(order, 1), w), **({"export": True} if kind == "w4a4" else {}))
        want = call(x, None, (torch.cat([e, none, none, none], 1), torch.cat([2 * half, half, half, half], 1)))
        assert torch.equal(got["out"], want["out"])            # y / 2 + y / 2, exactly
        if kind == "w4a4":
            assert int(got["offsets"][-1]) == T
    all_same = call(x, None, (e.expand(T, K).contiguous(), half.expand(T, K).contiguous() / 2))
    assert torch.equal(all_same["out"], want["out"]) and B.moe_async_status(all_same["workspace"]) == 0


def test_expert_shards_of_a_given_routing(B, layer):
    x, ids = _x(90), _ids(90)
    w = torch.rand(90, K).cuda()
    whole = torch.zeros(90, H).cuda()
    B.moe_w4a4_rac(x, None, *layer["packed"], K, 0, 0, layer["a2"], routing=(ids, w), out_f32=whole)
    total = torch.zeros(90, H).cuda()
    for lo, hi in ((0, 5), (5, 16)):
        part = torch.empty(90, H).cuda()
        shard = [{k: v[lo:hi].contiguous() for k, v in p.items() if v is not None} for p in layer["packed"]]
        B.moe_w4a4_rac(x, None, *shard, K, 0, 0, layer["a2"], routing=(ids, w), expert_range=(lo, hi), n_experts=E, out_f32=part)
        total += part
    # four float32 products each, added in two orders
    assert (total - whole).abs().max() <= 8 * 2.0 ** -24 * whole.abs().max() * 4


def _f32(t):
    return t.float().cpu().numpy()


def _fp8_layer(x, ids, w, w13, w2):
    """The FP8 layer from its definition, with this routing (token by token and slot by slot)."""
    xd = L.by_rows(x)
    out = np.zeros((len(x), H))
    dec13, dec2 = [L.weight(v)[2] for v in w13], [L.weight(v)[2] for v in w2]
    for t in range(len(x)):
        for e, wt in zip(ids[t], w[t]):
            if e < 0:
                continue
            g = dec13[e] @ xd[t]
            h = F.bf16_round(M.silu(g[:I]) * g[I:])
            hc, he = P.quantize_act(h[None])
            out[t] += wt * (dec2[e] @ P.dequantize_act(hc, he)[0])
    return out


def _block(B, layer, shared, x, logits, bias, workspaces=None):
    """Router, routed experts and a shared expert, as a model's layer runs them."""
    ids, w = B.route_experts(logits, K, score="sigmoid", bias=bias, n_group=4, topk_group=2, group_top=2, scale=2.5)
    routed = B.moe_fp8_w8a8(x, None, *layer["fp8"], K, routing=(ids, w))
    gu = B.fp8_linear(x, shared[0])["out"]
    h = torch.nn.functional.silu(gu[:, :I].float()) * gu[:, I:].float()
    y = B.fp8_linear(h.to(torch.bfloat16), shared[1])["out"]
    return ids, w, routed["out"], gu, h, y, routed["out"] + y


def _shared(B):
    g = torch.Generator().manual_seed(11)
    w = [_bf(g, 2 * I, H, scale=0.05), _bf(g, H, I, scale=0.05)]
    return w, [B.fp8_quantize_weights(v[None].cuda()) for v in w]


@pytest.mark.parametrize("T", [1, 50, 700])
def test_router_experts_and_shared_expert_together(B, layer, T):
    ws, shared = _shared(B)
    x = _x(T, 21)
    lg = torch.randn(T, E, generator=torch.Generator().manual_seed(22)).cuda()
    lg[::5, 3:9] = -float("inf")
    bias = (torch.randn(E, generator=torch.Generator().manual_seed(23)) * 0.1).cuda()
    ids, w, routed, gu, h, y, out = _block(B, layer, shared, x, lg, bias)
    some = range(0, T, max(1, T // 25))
    for t in some:
        assert ids[t].tolist() == R.choose(lg[t].double().cpu().numpy(), K, "sigmoid", bias.double().cpu().numpy(), 4, 2, 2)
    xs = _f32(x)[some]
    want = _fp8_layer(xs, ids.cpu().numpy()[some], w.double().cpu().numpy()[some], _f32(layer["w13"]), _f32(layer["w2"]))
    # h next to a rounding border may take the neighbouring code (a step of 2^-3 of one value in a hundred): 1e-2 of the norm, as for the
    # layer by itself
    assert np.linalg.norm(_f32(routed)[some] - want) <= 1e-2 * np.linalg.norm(want)
    # the shared expert stage by stage, each on what the stage before it left: every addition off by a step of float32 at most, one
    # rounding to bf16
    for got, inp, weight in ((gu, xs, ws[0]), (y, _f32(h.to(torch.bfloat16))[some], ws[1])):
        value, mags = L.forward(inp, _f32(weight))
        tol = inp.shape[1] * 2.0 ** -23 * mags
        assert (np.abs(_f32(got)[some] - value) <= tol + 2.0 ** -8 * (np.abs(value) + tol)).all()
    assert torch.equal(out, routed + y)


@pytest.mark.parametrize("T", [3, 600])
def test_the_block_captured_replayed_and_on_another_stream(B, layer, T):
    _, shared = _shared(B)
    x, lg = _x(T, 31), torch.randn(T, E, generator=torch.Generator().manual_seed(32)).cuda()
    bias = torch.zeros(E).cuda()
    want = [t.clone() for t in _block(B, layer, shared, x, lg, bias)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _block(B, layer, shared, x, lg, bias)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _block(B, layer, shared, x, lg, bias)
    x.copy_(_x(T, 41)), lg.copy_(torch.randn(T, E, generator=torch.Generator().manual_seed(42)))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    want = _block(B, layer, shared, x, lg, bias)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_training_step_of_the_shared_experts_projection_and_the_router(B):
    """Gradients of one loss through the projection and the router's weights, against the formulas of the oracles."""
    T, N = 130, 128
    g = torch.Generator().manual_seed(7)
    x, wt = _bf(g, T, H), _bf(g, N, H, scale=0.05)
    lg = torch.randn(T, E, generator=g)
    q = B.fp8_quantize_weights(wt[None].cuda())
    ids, w = B.route_experts(lg.cuda(), K, score="sigmoid", scale=2.5)
    out = B.fp8_linear(x.cuda(), q)["out"]
    # loss = sum_t sum_k w[t, k] * out[t, ids[t, k]]
    dw = torch.gather(out.float(), 1, ids.long())
    dl = B.route_experts_backward(lg.cuda(), ids, dw, score="sigmoid", scale=2.5).double().cpu().numpy()
    dout = torch.zeros(T, N).cuda().scatter_add_(1, ids.long(), w).to(torch.bfloat16)
    r = B.fp8_linear_backward(dout, x.cuda(), q)
    for t in range(0, T, 13):
        want = R.backward(lg[t].double().numpy(), ids[t].tolist(), dw[t].double().cpu().numpy(), "sigmoid", True, 2.5)
        assert (np.abs(dl[t] - want) <= 256 * 2.0 ** -24 * 2.5 * np.abs(dw[t].cpu().numpy()).max()).all()
    for got, (v, mags), depth, half in ((r["dx"], L.grad_input(_f32(dout), _f32(wt)), N, 2.0 ** -8), (r["dw"], L.grad_weight(_f32(dout), _f32(x)), T, 0.0)):
        tol = depth * 2.0 ** -23 * mags
        assert (np.abs(_f32(got) - v) <= tol + half * (np.abs(v) + tol) + 1e-38).all()


def test_refusals(B, layer):
    x, ids, w = _x(6), _ids(6), torch.rand(6, K).cuda()
    lg = torch.randn(6, E).cuda()
    for call in _calls(B, layer).values():
        for bad in ((ids.long(), w), (ids, w.double()), (ids[:5], w[:5]), (ids[:, :2], w[:, :2]), (ids.cpu(), w.cpu()), (ids, w.t().contiguous().t())):
            with pytest.raises(AssertionError):
                call(x, None, bad)
    with pytest.raises(AssertionError):                 # all experts' weights are here: how many there are is theirs to say
        B.moe_w4a4_rac(x, None, *layer["packed"], K, 0, 0, layer["a2"], routing=(ids, w), n_experts=2 * E)
    for call in _calls(B, layer).values():
        for both in ((lg, (ids, w)), (None, None)):
            with pytest.raises(AssertionError):
                call(x, *both)


def test_native_calls_and_their_python_twins_agree(B, layer, monkeypatch):
    """The binding's native functions and the ctypes path behind them: the same results, the caller's buffers back as they are."""
    if B._native is None:
        pytest.skip("built without the native functions")
    g = torch.Generator().manual_seed(77)
    x, ids = _x(40), _ids(40)
    w = torch.rand(40, K).cuda()
    lg, bias, dw = torch.randn(40, E).cuda(), torch.randn(E).cuda(), torch.randn(40, K).cuda()
    q = B.fp8_quantize_weights(_bf(g, 96, H)[None].cuda())
    dy = _bf(g, 40, 96).cuda()
    wide = _bf(g, 40, 2 * H).cuda()[:, :H]
    acc = torch.randn(96, H, generator=g).cuda()
    calls = [
        lambda: B.moe_w4a4_rac(x, None, *layer["packed"], K, 64, 64, layer["a2"], routing=(ids, w))["out"],
        lambda: B.moe_fp8_w8a8(x, None, *layer["fp8"], K, routing=(ids, w))["out"],
        lambda: B.route_experts(lg, K), lambda: B.route_experts(lg.bfloat16(), 3, score="sigmoid", bias=bias, n_group=4, topk_group=2, group_top=2, scale=2),
        lambda: B.route_experts_backward(lg, ids, dw, renormalize=False), lambda: B.route_experts_backward(lg[:, :16], ids, dw, score="sigmoid", scale=2.5),
        lambda: B.fp8_linear(x, q)["out"], lambda: B.fp8_linear(wide, q)["out"], lambda: B.fp8_linear(x[:1], {k: v[0] for k, v in q.items()})["out"],
        lambda: [B.fp8_linear_backward(dy, x, q)[k] for k in ("dx", "dw")],
        lambda: B.fp8_linear_backward(dy, x, q, dw=acc.clone(), accumulate=True)["dw"]]
    flat = lambda r: list(r) if isinstance(r, (tuple, list)) else [r]
    for i, call in enumerate(calls):
        a = flat(call())
        monkeypatch.setattr(B, "_native", None)
        b = flat(call())
        monkeypatch.undo()
        assert all(u.dtype == v.dtype and u.shape == v.shape and torch.equal(u, v) for u, v in zip(a, b)), i
    ws = torch.empty(B.fp8_linear_backward_workspace_bytes(40, 96, H), dtype=torch.uint8).cuda()
    out, dx, dwt = torch.empty(40, 96, dtype=torch.bfloat16).cuda(), torch.empty_like(x), torch.empty(96, H).cuda()
    r = B.fp8_linear(x, q, workspace=ws, out=out)
    assert r["out"] is out and r["workspace"] is ws
    r = B.fp8_linear_backward(dy, x, q, workspace=ws, dx=dx, dw=dwt)
    assert r["dx"] is dx and r["dw"] is dwt and r["workspace"] is ws


@pytest.mark.parametrize("T", [2, 60, 700])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), -float("nan")])
def test_as_many_channels_as_asked_for_whatever_x_holds(B, layer, T, value):
    """Scores that are infinite or no numbers, in every channel or in some: the selection has its size and its order."""
    x, ids = _x(T), _ids(T)
    w = torch.rand(T, K).cuda()
    for cols in (slice(0, H), slice(16, 100)):
        bad = x.clone()
        bad[::2, cols] = torch.tensor(value, dtype=torch.bfloat16)
        for gs in (None, torch.tensor([0.002]).cuda()):
            for n in (1, 100, H - 1):
                r = B.moe_w4a4_rac(bad, None, *layer["packed"], K, n, 0, layer["a2"], a13_gs=gs, routing=(ids, w), export=True)
                sel = r["sel13"].tolist()
                assert len(sel) == n and sel == sorted(set(sel)) and 0 <= sel[0] and sel[-1] < H
                assert B.moe_async_status(r["workspace"]) == 0


def _padded(T, seed):
    """x with the rows of tokens without any expert (every third) left open, and a routing that leaves them and single slots out."""
    x, ids, w = _x(T, seed), _ids(T, seed), torch.rand(T, K, generator=torch.Generator().manual_seed(seed)).cuda()
    empty = torch.arange(T).cuda() % 3 == 2
    ids[empty] = -1
    ids[::4, 1] = E
    w[(ids < 0) | (ids >= E)] = float("nan")               # (the weights of such slots are not read, or not used)
    return x, (ids, w), empty


@pytest.mark.parametrize("T", [3, 60, 600, 3000])
def test_rows_without_an_expert_count_in_the_scale_and_the_selection(B, layer, T):
    """The layer's x is its whole batch, tokens that no expert takes included: their rows are zeroed, and are then as if they were not there, or the scale is
    given and nothing selected."""
    x, rt, empty = _padded(T, 51)
    n = H // 2
    run = lambda x, n13, gs: B.moe_w4a4_rac(x, None, *layer["packed"], K, n13, I // 2, layer["a2"], a13_gs=gs, routing=rt, export=True)
    real = x[~empty].contiguous()
    zeroed = x.masked_fill(empty[:, None], 0.0)
    r = run(zeroed, n, None)
    assert r["a13_gs"].item() == np.float32(np.float32(real.abs().max().item()) / np.float32(2688.0))
    scores = B.rac_channel_scores(real)
    # float32 sums over some rows each, then float64: off by a step (2^-23) of the sum for each of the T rows at most
    chosen = torch.zeros(H, dtype=torch.bool).cuda()
    chosen[r["sel13"].long()] = True
    assert chosen.sum() == n and scores[chosen].min() * (1 + T * 2.0 ** -22) >= scores[~chosen].max()
    loud = x.clone()
    loud[empty] = 1e4
    assert run(loud, n, None)["a13_gs"].item() == np.float32(np.float32(torch.tensor(1e4, dtype=torch.bfloat16).item()) / np.float32(2688.0))
    gs = r["a13_gs"].clone()
    want = run(zeroed, 0, gs)["out"]
    assert (want[empty] == 0).all()
    for v in (1e30, float("nan"), float("inf")):
        got = run(x.masked_fill(empty[:, None], v), 0, gs)
        assert torch.equal(got["out"], want) and B.moe_async_status(got["workspace"]) == 0


@pytest.mark.parametrize("T", [3, 60, 600, 3000])
def test_rows_without_an_expert_are_of_no_account_in_the_fp8_layer(B, layer, T):
    x, rt, empty = _padded(T, 52)
    want = B.moe_fp8_w8a8(x, None, *layer["fp8"], K, routing=rt)["out"]
    assert (want[empty] == 0).all()
    for v in (0.0, 1e30, float("nan"), -float("inf")):
        got = B.moe_fp8_w8a8(x.masked_fill(empty[:, None], v), None, *layer["fp8"], K, routing=rt)
        assert torch.equal(got["out"], want) and B.moe_async_status(got["workspace"]) == 0


# the layer's three routing kernels (512 and 513 tokens apart), weights renormalised or not
@pytest.mark.parametrize("T", [1, 61, 500, 513, 3000])
@pytest.mark.parametrize("renorm", [True, False])
def test_the_softmax_routers_choice_given_to_the_layers_is_their_own(B, layer, T, renorm):
    lg = torch.randn(T, E, generator=torch.Generator().manual_seed(T + 7)).cuda()
    lg[::3, 4] = lg[::3, 9]                                # equal logits
    x, rt = _x(T, 61), B.route_experts(lg, K, renormalize=renorm)
    own = B.moe_w4a4_rac(x, lg, *layer["packed"], K, H // 2, I // 2, layer["a2"], renormalize=renorm, export=True)
    given = B.moe_w4a4_rac(x, None, *layer["packed"], K, H // 2, I // 2, layer["a2"], routing=rt, export=True)
    for k in ("ids", "offsets", "perm", "sel13", "sel2", "h", "hq"):
        assert torch.equal(given[k], own[k]), k
    # either weight: exp within 2 ulp in numerator and denominator (8 half steps), its argument (2 x 8 of them: |l - m| <= 8), sums of up to 16
    # terms (16), one or two divisions (4 each)
    assert ((given["weights"] - own["weights"]).abs() <= 2 * 48 * 2.0 ** -24 * own["weights"]).all()
    fp8 = [B.moe_fp8_w8a8(x, *a, *layer["fp8"], K, renormalize=renorm, routing=r)["out"] for a, r in (((lg,), None), ((None,), rt))]
    for a, b in ((own["out"], given["out"]), fp8):
        # K terms with weights that far apart (bounded by the terms' sum: 4 x the largest output of the row), one rounding to bf16 of either
        a, b = a.double(), b.double()
        assert ((a - b).abs() <= 2 * 2.0 ** -8 * a.abs() + 128 * 2.0 ** -24 * 4 * a.abs().amax(1, keepdim=True)).all()


def test_tensors_of_another_device_are_refused(B, layer, monkeypatch):
    """The launch goes to the current device's stream; here the tensors' device is the first and the second is called the current one."""
    x, lg, rt = _x(4), torch.randn(4, E).cuda(), (_ids(4), torch.rand(4, K).cuda())
    w = torch.zeros(1, 32, 64, dtype=torch.bfloat16).cuda()
    q = B.fp8_quantize_weights(w)
    monkeypatch.setattr(B, "_native", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in _calls(B, layer).values():
        for a in ((lg, None), (None, rt)):
            with pytest.raises(AssertionError):
                call(x, *a)
    for f in (lambda: B.fp8_quantize_weights(w), lambda: B.fp8_linear(w[0, :4], q), lambda: B.route_experts(lg, 2), lambda: B.route_experts_backward(lg, *rt)):
        with pytest.raises(AssertionError):
            f()
