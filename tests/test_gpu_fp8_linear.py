"""The dense FP8 projection and its gradients against the float64 product of the decoded operands."""
import numpy as np
import pytest
import torch

from oracle import fp8_linear as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2607_15810_b200 import binding
    return binding


def _f32(t):
    return t.float().cpu().numpy()


def _acts(T, K, seed, spread=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, K, generator=g)
    x[:, ::37] *= 12.0
    if spread:
        x *= torch.exp(2 * torch.randn(T, 1, generator=g)) * 1e-3
    return x.to(torch.bfloat16)


def _weight(N, K, seed):
    w = torch.randn(N, K, generator=torch.Generator().manual_seed(seed)) * 0.02
    w[: N // 2] *= 8.0
    return w.to(torch.bfloat16)


def _near(got, want, depth, bf16):
    """Each of `depth` additions is off by at most a step of float32 (2^-23) of a partial sum, which the sum of the magnitudes bounds; then one
    rounding to bf16 (half a step, 2^-8 of the value)."""
    value, mags = want
    err = np.abs(_f32(got).astype(np.float64) - value)
    tol = depth * 2.0 ** -23 * mags
    if bf16:
        tol = tol + 2.0 ** -8 * (np.abs(value) + tol)
    assert (err <= tol + 1e-38).all(), (err - tol).max()


# one element of each; sizes that end inside a block; tiles that a cluster shares; several tiles per CTA with few rows; CTA pairs
SHAPES = [(1, 16, 16), (1, 128, 128), (2, 4096, 128), (3, 144, 272), (16, 128, 4096), (33, 2064, 1040), (64, 256, 512), (65, 400, 384),
          (128, 512, 2048), (129, 256, 256), (200, 1536, 2048), (5, 19216, 144), (100, 19216, 144), (333, 2048, 768), (700, 4112, 256),
          (1501, 2000, 528), (2100, 1296, 400)]


@pytest.mark.parametrize("T,N,K", SHAPES)
def test_forward(B, T, N, K):
    x, w = _acts(T, K, T), _weight(N, K, N)
    q = B.fp8_quantize_weights(w[None].cuda())
    codes, exps, _ = L.weight(_f32(w))
    assert np.array_equal(q["q"][0].cpu().numpy(), codes)
    assert np.array_equal(q["exps"][0].cpu().numpy().astype(np.int32) - 127, exps)
    r = B.fp8_linear(x.cuda(), q)
    assert B.moe_async_status(r["workspace"]) == 0
    _near(r["out"], L.forward(_f32(x), _f32(w)), K, True)


# tiles of 192 columns, ending behind 16, 64, 96, 144 and 192 of them, in one round and several
@pytest.mark.parametrize("T,N,K", [(513, 4048, 1168), (640, 4096, 1296), (768, 4128, 1040), (700, 4176, 2000),
                                   (600, 4224, 2064), (1409, 4176, 1552)])
def test_forward_in_narrower_tiles(B, T, N, K):
    x, w = _acts(T, K, T), _weight(N, K, N)
    r = B.fp8_linear(x.cuda(), B.fp8_quantize_weights(w[None].cuda()))
    assert B.moe_async_status(r["workspace"]) == 0
    _near(r["out"], L.forward(_f32(x), _f32(w)), K, True)


# pairs with tiles of 256 columns, in one round and two; single CTAs with several tiles in turn
@pytest.mark.parametrize("T,N,K", [(1024, 4096, 1040), (1000, 4112, 2000), (2047, 4096, 1296), (700, 4112, 256), (2100, 1296, 528), (4099, 2064, 144)])
def test_one_product_of_many_tiles(B, T, N, K):
    x, w = _acts(T, K, T), _weight(N, K, N)
    q, wf = B.fp8_quantize_weights(w[None].cuda()), _f32(w)
    _near(B.fp8_linear(x.cuda(), q)["out"], L.forward(_f32(x), wf), K, True)
    dy, w = _acts(T, K, T + 1), _weight(K, N, N)       # the same sizes with the contraction along the output features, and along the tokens
    r = B.fp8_linear_backward(dy.cuda(), None, B.fp8_quantize_weights(w[None].cuda()), want_dw=False)
    _near(r["dx"], L.grad_input(_f32(dy), _f32(w)), K, True)
    dy, x = _acts(K, T // 16 * 16, T, spread=True), _acts(K, N, T + 1)
    r = B.fp8_linear_backward(dy.cuda(), x.cuda(), None, want_dx=False)
    _near(r["dw"], L.grad_weight(_f32(dy), _f32(x)), K, False)


@pytest.mark.parametrize("T,N,K", SHAPES)
def test_gradients(B, T, N, K):
    x, w, dy = _acts(T, K, T), _weight(N, K, N), _acts(T, N, T + 1, spread=True)
    q = B.fp8_quantize_weights(w[None].cuda())
    r = B.fp8_linear_backward(dy.cuda(), x.cuda(), q)
    assert B.moe_async_status(r["workspace"]) == 0
    _near(r["dx"], L.grad_input(_f32(dy), _f32(w)), N, True)
    _near(r["dw"], L.grad_weight(_f32(dy), _f32(x)), T, False)


# few tiles with a long contraction beside many with a short one: the long one split over clusters (192, 4100), the others' tiles in turn on the
# CTAs that are left (64, 333, 6000 and on), pairs with a long tile coming to the others' later (2048, 512)
@pytest.mark.parametrize("T,N,K", [(192, 8192, 256), (4100, 144, 272), (64, 1040, 4096), (64, 4096, 2064), (333, 2064, 2048), (640, 4112, 2048),
                                   (1, 6000, 1504), (40, 8192, 1040), (8192, 256, 1024), (2048, 2064, 2048), (512, 2048, 3024),
                                   (4300, 8192, 256)])
def test_gradients_of_uneven_products(B, T, N, K):
    x, dy, w = _acts(T, K, 1), _acts(T, N, 2, spread=True), _weight(N, K, 3)
    r = B.fp8_linear_backward(dy.cuda(), x.cuda(), B.fp8_quantize_weights(w[None].cuda()))
    assert B.moe_async_status(r["workspace"]) == 0
    _near(r["dx"], L.grad_input(_f32(dy), _f32(w)), N, True)
    _near(r["dw"], L.grad_weight(_f32(dy), _f32(x)), T, False)


@pytest.mark.parametrize("T,N,K", [(192, 8192, 256), (64, 4096, 2064), (512, 2048, 3024)])
def test_gradients_of_uneven_products_captured_and_beside_others(B, T, N, K):
    xs, dys = [_acts(T, K, s).cuda() for s in (1, 4)], [_acts(T, N, s).cuda() for s in (2, 5)]
    w = B.fp8_quantize_weights(_weight(N, K, 3)[None].cuda())
    want = [B.fp8_linear_backward(dy, x, w) for dy, x in zip(dys, xs)]
    x, dy = xs[0].clone(), dys[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = B.fp8_linear_backward(dy, x, w)
        again = B.fp8_linear_backward(dy, x, w, workspace=r["workspace"])         # right behind, on the same workspace
    for i in (0, 1, 0):
        x.copy_(xs[i]), dy.copy_(dys[i])
        graph.replay()
        torch.cuda.synchronize()
        for g in (r, again):
            assert torch.equal(g["dx"], want[i]["dx"]) and torch.equal(g["dw"], want[i]["dw"])
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(3):
        for s, dy, x in zip(streams, dys, xs):
            with torch.cuda.stream(s):
                got.append(B.fp8_linear_backward(dy, x, w))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert torch.equal(g["dx"], want[i % 2]["dx"]) and torch.equal(g["dw"], want[i % 2]["dw"])


def test_a_gradient_against_differences(B):
    """Values that E4M3 holds exactly, so that nothing is rounded on the way: the product is bilinear, its differences are exact."""
    rng = np.random.default_rng(0)
    x, w, dy = (torch.from_numpy(rng.integers(-7, 8, s).astype(np.float32)).to(torch.bfloat16) for s in ((40, 96), (64, 96), (40, 64)))
    q = B.fp8_quantize_weights(w[None].cuda())
    r = B.fp8_linear_backward(dy.cuda(), x.cuda(), q)

    def loss(xx, ww):
        out = B.fp8_linear(xx.cuda(), B.fp8_quantize_weights(ww[None].cuda()))["out"].double().cpu()
        return (out * dy.double()).sum().item()

    # outputs are sums of at most 96 products up to 49: integers of up to 13 bits, which bf16 rounds; keep one channel, whose are exact
    for c in (0, 50, 95):
        for t, n in ((0, 0), (13, 40), (39, 63)):
            only = torch.zeros_like(x)
            only[t, c] = 1.0
            assert loss(only, w) == r["dx"].double().cpu()[t, c].item() or \
                abs(loss(only, w) - r["dx"].double().cpu()[t, c].item()) <= 2.0 ** -8 * abs(loss(only, w))     # dx itself is bf16
            e = torch.zeros_like(w)
            e[n, c] = 1.0
            assert loss(x, e) == r["dw"].double().cpu()[n, c].item()


def test_zero_rows_and_values_at_the_ends_of_the_range(B):
    x = _acts(130, 256, 1)
    x[3] = 0
    x[5, :128] = 0
    x[7] *= 2.0 ** 100
    x[9] *= 2.0 ** -100
    x[11, 128:] *= 2.0 ** 60                            # blocks of one row 60 octaves apart
    x[13] = torch.finfo(torch.bfloat16).tiny
    x[13, 0] = 2.0 ** -133                              # below the normal numbers
    w = _weight(144, 256, 2)
    w[:128, :128] = 0
    q = B.fp8_quantize_weights(w[None].cuda())
    r = B.fp8_linear(x.cuda(), q)
    _near(r["out"], L.forward(_f32(x), _f32(w)), 256, True)
    assert (r["out"][3] == 0).all()


@pytest.mark.parametrize("T,N,K", [(9, 144, 400), (61, 272, 1040), (700, 1040, 528), (3300, 4096, 4112)])
def test_infinities_and_nans_stay_in_their_rows(B, T, N, K):
    """As a padded batch has them: the other rows of the product and of the input's gradient are what they were."""
    x, dy, w = _acts(T, K, 1).cuda(), _acts(T, N, 2).cuda(), B.fp8_quantize_weights(_weight(N, K, 3)[None].cuda())
    out, dx = B.fp8_linear(x, w)["out"], B.fp8_linear_backward(dy, None, w, want_dw=False)["dx"]
    bad = torch.zeros(T, dtype=torch.bool)
    bad[::3] = True
    bad = bad.cuda()
    for v in (float("nan"), float("inf"), float("-inf")):
        x2, dy2 = x.clone(), dy.clone()
        x2[bad], dy2[bad] = v, v
        assert torch.equal(B.fp8_linear(x2, w)["out"][~bad], out[~bad])
        assert torch.equal(B.fp8_linear_backward(dy2, None, w, want_dw=False)["dx"][~bad], dx[~bad])


def test_rows_apart_in_memory_and_given_outputs(B):
    T, N, K = 70, 272, 400
    w = B.fp8_quantize_weights(_weight(N, K, 1)[None].cuda())
    xs, ys = _acts(T, K + 64, 2).cuda(), _acts(T, N + 24, 3).cuda()
    x, dy = xs[:, 8:8 + K], ys[:, 16:16 + N]
    a, b = B.fp8_linear(x, w), B.fp8_linear(x.contiguous(), w)
    assert torch.equal(a["out"], b["out"])
    out = torch.full((T + 3, N), 5.0, dtype=torch.bfloat16, device="cuda")
    B.fp8_linear(x, w, out=out[:T])
    assert torch.equal(out[:T], b["out"]) and (out[T:] == 5.0).all()
    flat = torch.full((T * N + 16,), 5.0, dtype=torch.bfloat16, device="cuda")      # aligned to 16 bytes only
    B.fp8_linear(x, w, out=flat[8:8 + T * N].view(T, N))
    assert torch.equal(flat[8:8 + T * N].view(T, N), b["out"]) and (flat[:8] == 5.0).all() and (flat[-8:] == 5.0).all()
    g, h = B.fp8_linear_backward(dy, x, w), B.fp8_linear_backward(dy.contiguous(), x.contiguous(), w)
    assert torch.equal(g["dx"], h["dx"]) and torch.equal(g["dw"], h["dw"])
    one = B.fp8_linear(xs[5:6, 8:8 + K], w)["out"]
    assert torch.equal(one[0], b["out"][5])


@pytest.mark.parametrize("T,N,K", [(70, 272, 400), (300, 4112, 2064)])
def test_one_gradient_at_a_time_and_adding_up(B, T, N, K):
    x, dy, wt = _acts(T, K, 1).cuda(), _acts(T, N, 2).cuda(), _weight(N, K, 3)
    w = B.fp8_quantize_weights(wt[None].cuda())
    both = B.fp8_linear_backward(dy, x, w)
    dx = B.fp8_linear_backward(dy, None, w, want_dw=False)
    dw = B.fp8_linear_backward(dy, x, None, want_dx=False)
    assert dx["dw"] is None and dw["dx"] is None
    # alone, a product may split its contraction otherwise than beside the other one: the order of additions differs, the bound holds for any
    for r in (both, dx):
        _near(r["dx"], L.grad_input(_f32(dy), _f32(wt)), N, True)
    for r in (both, dw):
        _near(r["dw"], L.grad_weight(_f32(dy), _f32(x)), T, False)
    acc = torch.randn(N, K, generator=torch.Generator().manual_seed(4)).cuda()
    want = acc + both["dw"]                             # one float32 addition
    B.fp8_linear_backward(dy, x, w, dw=acc, accumulate=True)
    assert torch.equal(acc, want)


def test_no_tokens(B):
    w = B.fp8_quantize_weights(_weight(64, 96, 1)[None].cuda())
    x, dy = torch.empty(0, 96, dtype=torch.bfloat16).cuda(), torch.empty(0, 64, dtype=torch.bfloat16).cuda()
    assert B.fp8_linear(x, w)["out"].shape == (0, 64)
    r = B.fp8_linear_backward(dy, x, w)
    assert r["dx"].shape == (0, 96) and (r["dw"] == 0).all()
    acc = torch.ones(64, 96).cuda()
    B.fp8_linear_backward(dy, x, w, dw=acc, accumulate=True)
    assert (acc == 1).all()


@pytest.mark.parametrize("T,N,K", [(3, 512, 2048), (1500, 2064, 512)])
def test_captured_and_replayed(B, T, N, K):
    x, dy = _acts(T, K, 1).cuda(), _acts(T, N, 2).cuda()
    w = B.fp8_quantize_weights(_weight(N, K, 3)[None].cuda())
    B.fp8_linear(x, w), B.fp8_linear_backward(dy, x, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = B.fp8_linear(x, w)["out"]
        r = B.fp8_linear_backward(dy, x, w)
    x.copy_(_acts(T, K, 5))
    dy.copy_(_acts(T, N, 6))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    g = B.fp8_linear_backward(dy, x, w)
    assert torch.equal(out, B.fp8_linear(x, w)["out"]) and torch.equal(r["dx"], g["dx"]) and torch.equal(r["dw"], g["dw"])


def test_weights_and_inputs_written_right_before_the_call(B):
    """The weights are loaded before the kernel in front has ended: that has to be this call's own, not the one that writes them."""
    x, w = _acts(8, 2048, 1).cuda(), _weight(2048, 2048, 2).cuda()
    want = B.fp8_linear(x, B.fp8_quantize_weights(w[None]))["out"].clone()
    ws = torch.empty(B.fp8_linear_workspace_bytes(8, 2048, 2048), dtype=torch.uint8, device="cuda")
    for _ in range(20):
        zero = B.fp8_quantize_weights(torch.zeros_like(w)[None])
        r0 = B.fp8_linear(torch.zeros_like(x), zero, workspace=ws)["out"]
        q = B.fp8_quantize_weights(w[None])
        zero["q"].copy_(q["q"]), zero["atoms"].copy_(q["atoms"])
        r = B.fp8_linear(x.clone(), zero, workspace=ws)["out"]
        assert (r0 == 0).all() and torch.equal(r, want)


def test_two_calls_side_by_side(B):
    x, w = _acts(300, 1024, 1).cuda(), B.fp8_quantize_weights(_weight(1024, 1024, 2)[None].cuda())
    dy = _acts(300, 1024, 3).cuda()
    want = B.fp8_linear_backward(dy, x, w)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(B.fp8_linear_backward(dy, x, w))
    torch.cuda.synchronize()
    assert all(torch.equal(g["dx"], want["dx"]) and torch.equal(g["dw"], want["dw"]) for g in got)


def test_refusals(B):
    x, w = _acts(4, 64, 1).cuda(), B.fp8_quantize_weights(_weight(32, 64, 2)[None].cuda())
    with pytest.raises(B.QuadsError):                       # not a multiple of 16
        B.fp8_quantize_weights(torch.zeros(1, 24, 64, dtype=torch.bfloat16).cuda())
    with pytest.raises(B.QuadsError):
        B.fp8_quantize_weights(torch.zeros(1, 32, 40, dtype=torch.bfloat16).cuda())
    wide = _acts(4, 100, 1).cuda()
    with pytest.raises(B.QuadsError):                       # rows 100 elements apart
        B.fp8_linear(wide[:, :64], w)
    with pytest.raises(B.QuadsError):                       # 2-byte aligned
        B.fp8_linear(_acts(4, 128, 1).cuda()[:, 1:65], w)
    with pytest.raises(B.QuadsError) as e:
        B.fp8_linear(x, w, workspace=torch.empty(64, dtype=torch.uint8).cuda())
    assert e.value.status == -3
    for bad in (x.float(), x.cpu(), x[:, :32], x.t()):
        with pytest.raises(AssertionError):
            B.fp8_linear(bad, w)
    with pytest.raises(AssertionError):
        B.fp8_linear(x, B.fp8_quantize_weights(torch.zeros(2, 32, 64, dtype=torch.bfloat16).cuda()))
    dy = _acts(4, 32, 1).cuda()
    for kw in (dict(dw=torch.zeros(32, 64, dtype=torch.bfloat16).cuda()), dict(dw=torch.zeros(64, 32).cuda()), dict(accumulate=True),
               dict(dx=torch.zeros(4, 64).cuda())):
        with pytest.raises(AssertionError):
            B.fp8_linear_backward(dy, x, w, **kw)


# contractions of more than 4096 tokens, which leave the tensor core in pieces: in single CTAs, in clusters, in pairs, ending inside a block
@pytest.mark.parametrize("T,N,K", [(4300, 1296, 1296), (9001, 144, 272), (4227, 2064, 2064)])
def test_weight_gradients_of_long_batches(B, T, N, K):
    x, dy = _acts(T, K, T), _acts(T, N, T + 1, spread=True)
    want = L.grad_weight(_f32(dy), _f32(x))
    dw = B.fp8_linear_backward(dy.cuda(), x.cuda(), None, want_dx=False)["dw"]
    _near(dw, want, T, False)
    acc = torch.ones(N, K).cuda()
    B.fp8_linear_backward(dy.cuda(), x.cuda(), None, want_dx=False, dw=acc, accumulate=True)
    # the pieces are added to what was there one by one: each addition half a step of the partial sum
    tol = T * 2.0 ** -23 * want[1] + 4 * 2.0 ** -24 * (1 + want[1])
    assert (np.abs(_f32(acc).astype(np.float64) - 1 - want[0]) <= tol).all()


def test_more_elements_than_32_bits_count(B):
    T, K, N = 530000, 4096, 32
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(T, K, dtype=torch.bfloat16, device="cuda")
    for t in range(0, T, 53000):
        x[t:t + 53000] = torch.randn(53000, K, generator=g, device="cuda")
    w = B.fp8_quantize_weights(_weight(N, K, 1)[None].cuda())
    out = B.fp8_linear(x, w)["out"]
    for lo, hi in ((0, 70), (T // 2, T // 2 + 70), (T - 70, T)):
        _near(out[lo:hi], (L.by_rows(_f32(x[lo:hi])) @ L.weight(_f32(_weight(N, K, 1)))[2].T, np.abs(L.by_rows(_f32(x[lo:hi]))) @
                           np.abs(L.weight(_f32(_weight(N, K, 1)))[2]).T), K, True)


# many turns of a small ring: one CTA to a tile and all of the contraction, x quantized inside; several tiles to a CTA
@pytest.mark.parametrize("T,N,K", [(8, 16512, 4096), (16, 18944, 2880), (3, 19216, 1920), (1, 37904, 1040)])
def test_few_rows_through_the_whole_contraction_again_and_again(B, T, N, K):
    x, w = _acts(T, K, T), _weight(N, K, N)
    q = B.fp8_quantize_weights(w[None].cuda())
    xd = x.cuda()
    outs = [B.fp8_linear(xd, q) for _ in range(20)]
    assert all(B.moe_async_status(r["workspace"]) == 0 and torch.equal(r["out"], outs[0]["out"]) for r in outs)
    _near(outs[0]["out"], L.forward(_f32(x), _f32(w)), K, True)


def test_weights_quantized_where_the_call_in_front_reads_and_from_what_it_writes(B):
    """The weights' quantizer may be launched while the kernel in front still runs: it writes and reads behind that one's end."""
    T, N, K = 8192, 2048, 2048
    x, ws = _acts(T, K, 1).cuda(), [_weight(N, K, s)[None].cuda() for s in (2, 3)]
    qs = [B.fp8_quantize_weights(w) for w in ws]
    want = [B.fp8_linear(x, q)["out"] for q in qs]
    q = {k: v.clone() for k, v in qs[0].items()}
    got = []
    torch.cuda.synchronize()
    for i in range(1, 21):
        got.append(B.fp8_linear(x, q)["out"])
        B.check(B.lib.quads_fp8_quantize_weights(B._ptr(ws[i % 2]), 1, N, K, B._ptr(q["q"]), B._ptr(q["exps"]), B._ptr(q["atoms"]), B._stream()))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert torch.equal(out, want[i % 2]), i
    gs = torch.tensor([0.002]).cuda()
    fq = B.fake_quant_activations(ws[0][0], gs=gs)[0]
    torch.cuda.synchronize()
    want = B.fp8_quantize_weights(fq[None])
    for _ in range(20):
        got = B.fp8_quantize_weights(B.fake_quant_activations(ws[0][0], gs=gs)[0][None])
        assert all(torch.equal(got[k], want[k]) for k in want)
        del got


# up to 4096 tokens; longer, in clusters, in single CTAs and in pairs
@pytest.mark.parametrize("T,N,K", [(4096, 144, 272), (4096, 1296, 1296), (9000, 144, 272), (9000, 1296, 1296), (12289, 2064, 2064)])
def test_a_long_batch_is_added_in_pieces_of_4096_tokens(B, T, N, K):
    """Whole numbers, exact in every sum of products: what is rounded is the additions to what was there, one per piece or one for all."""
    g = torch.Generator(device="cuda").manual_seed(T + N)
    x, dy = (torch.randint(-7, 8, (T, c), generator=g, device="cuda").to(torch.bfloat16) for c in (K, N))
    start = torch.randn(N, K, generator=g, device="cuda") * 1e4
    pieces = [(dy[t:t + 4096].double().t() @ x[t:t + 4096].double()).float() for t in range(0, T, 4096)]
    dw = B.fp8_linear_backward(dy, x, None, want_dx=False)["dw"]
    assert torch.equal(dw, sum(pieces))
    for w in (None, B.fp8_quantize_weights(torch.ones(1, N, K, dtype=torch.bfloat16, device="cuda"))):
        acc = start.clone()
        B.fp8_linear_backward(dy, x, w, want_dx=w is not None, dw=acc, accumulate=True)
        one_by_one = start
        for p in pieces:
            one_by_one = one_by_one + p
        assert ((acc == one_by_one) | (acc == start + dw)).all()
        assert T > 4096 or torch.equal(acc, start + dw)


# in single CTAs, in clusters, in pairs
@pytest.mark.parametrize("T,N,K", [(16384, 1280, 1280), (16384, 144, 272), (16384, 1664, 1680), (9000, 1296, 1296)])
def test_weight_gradients_of_long_batches_keep_float32s_precision(B, T, N, K):
    """What leaving the tensor core every 4096 tokens is for: its additions cut off, and the relative error (2-norm) of terms of like magnitude grows
    with their number: 6.0e-8 at 1024 tokens, 2.2e-7 at 4096 and, in one piece, 4.8e-7 at 8192, 5.3e-7 at 9000, 1.16e-6 at 16384.  The sum of
    pieces of 4096 has their 2.2e-7, and the three additions of four of them are off by half a step each: 2.2e-7 + 3 x 2^-24."""
    g = torch.Generator().manual_seed(T + N)
    x, dy = (torch.randn(T, c, generator=g).to(torch.bfloat16) for c in (K, N))
    dw = B.fp8_linear_backward(dy.cuda(), x.cuda(), None, want_dx=False)["dw"]
    rows = torch.randperm(N, generator=g)[:64]
    want, _ = L.grad_weight(_f32(dy[:, rows]), _f32(x))
    assert np.linalg.norm(_f32(dw[rows.cuda()]) - want) <= (2.2e-7 + 3 * 2.0 ** -24) * np.linalg.norm(want)
