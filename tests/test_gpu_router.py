"""The router by itself and its gradient against the float64 oracle: chosen ids exactly, weights and gradients to float32 rounding."""
import io
import math

import numpy as np
import pytest
import torch

from oracle import router as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24                                         # half a step of float32
# exp within 2 ulp in numerator and denominator (8 U), its argument l - m rounded, |l - m| <= 16 (2 x 16 U), sums of up to 256 terms in a tree of
# depth 13 and the division (16 U)
W_RTOL = 56 * U


@pytest.fixture(scope="module")
def B():
    from paper_2607_15810_b200 import binding
    return binding


def _logits(T, E, seed, bf16=False, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(T, E, generator=g) * 1.5
    if masked:
        l[torch.rand(T, E, generator=g) < masked] = -math.inf
        l[::7] = -math.inf                             # rows with nothing to choose from
        l[3::11, : E // 2] = math.nan
    return l.to(torch.bfloat16) if bf16 else l


CASES = [
    # T, E, topk, score, renorm, bias, n_group, topk_group, group_top, scale, bf16, masked
    (1, 256, 8, "sigmoid", True, True, 8, 4, 2, 2.5, False, 0.0),
    (1, 1, 1, "softmax", True, False, 1, 1, 1, 1.0, False, 0.0),
    (7, 5, 5, "softmax", False, False, 1, 1, 1, 1.0, True, 0.0),
    (33, 128, 8, "softmax", True, False, 1, 1, 1, 1.0, False, 0.0),
    (61, 160, 6, "softmax", False, False, 8, 3, 1, 16.0, True, 0.1),
    (64, 256, 16, "softmax", True, True, 1, 1, 1, 1.0, True, 0.0),
    (100, 72, 4, "sigmoid", False, False, 4, 2, 2, 1.0, False, 0.3),
    (50, 255, 9, "sigmoid", True, True, 5, 1, 2, 2.5, False, 0.1),
    (50, 96, 16, "sigmoid", True, False, 32, 7, 2, 1.0, True, 0.5),
    (40, 33, 3, "softmax", True, True, 3, 2, 2, 1.0, False, 0.2),
    (200, 64, 1, "sigmoid", True, True, 1, 1, 1, 1.0, True, 0.0),
    (40, 8, 4, "softmax", True, False, 8, 5, 1, 1.0, True, 0.4),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c))
def test_choice_and_weights(B, case):
    T, E, k, score, renorm, with_bias, G, kept, top, scale, bf16, masked = case
    l = _logits(T, E, T + E, bf16, masked)
    bias = torch.randn(E, generator=torch.Generator().manual_seed(E)) * 0.2 if with_bias else None
    ids, w = B.route_experts(l.cuda(), k, score=score, bias=None if bias is None else bias.cuda(), n_group=G, topk_group=kept, group_top=top,
                             renormalize=renorm, scale=scale)
    ids, w, l64 = ids.cpu().numpy(), w.double().cpu().numpy(), l.double().numpy()
    for t in range(T):
        want = R.choose(l64[t], k, score, None if bias is None else bias.double().numpy(), G, kept, top)
        assert list(ids[t]) == want, t
        np.testing.assert_allclose(w[t], R.weights(l64[t], want, score, renorm, scale), rtol=W_RTOL, atol=0)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c))
def test_gradient(B, case):
    T, E, k, score, renorm, with_bias, G, kept, top, scale, bf16, masked = case
    l = _logits(T, E, T + E, bf16, masked)
    rng = np.random.default_rng(T)
    dw = rng.standard_normal((T, k)).astype(np.float32)
    ids = np.stack([R.choose(l[t].double().numpy(), k, score) for t in range(T)]).astype(np.int32)
    d = B.route_experts_backward(l.cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(dw).cuda(), score=score, renormalize=renorm, scale=scale)
    assert d.dtype == l.dtype
    d = d.double().cpu().numpy()
    for t in range(T):
        want = R.backward(l[t].double().numpy(), ids[t], dw[t].astype(np.float64), score, renorm, scale)
        # r (dw - sum r dw): r is off by 56 U of itself, the sum (k terms) by 72 U max |dw|, the rest by 8 U: together less than 256 U
        tol = 256 * U * scale * np.abs(dw[t]).max() + (2.0 ** -8 * np.abs(want) if bf16 else 0.0)
        assert (np.abs(d[t] - want) <= tol).all(), t


def test_ties_go_to_the_lower_id(B):
    l = torch.zeros(3, 256)
    l[1, 100:] = 1.0
    l[2, ::2] = -0.0
    for kw in (dict(), dict(n_group=8, topk_group=2), dict(score="sigmoid", bias=torch.zeros(256).cuda()),
               dict(score="sigmoid", n_group=8, topk_group=3, group_top=2)):
        ids, _ = B.route_experts(l.cuda(), 5, **kw)
        kw = {k: (v.cpu().numpy() if torch.is_tensor(v) else v) for k, v in kw.items()}
        score = kw.pop("score", "softmax")
        for t in range(3):
            assert ids[t].tolist() == R.choose(l[t].numpy(), 5, score, **kw)


def test_scores_that_differ_below_float32_are_told_apart(B):
    """Sigmoids of large logits round to the same float32 next to one another, and a bias added in float32 would hide what is left."""
    l = torch.tensor([[9.0, 9.0000010, 9.0000019, 8.9999990, 9.0, -1.0, -2.0, -3.0]] * 2)
    bias = torch.full((8,), 0.5)
    ids, _ = B.route_experts(l.cuda(), 5, score="sigmoid", bias=bias.cuda())
    assert ids[0].tolist() == [2, 1, 0, 4, 3] == R.choose(l[0].double().numpy(), 5, "sigmoid", bias.double().numpy())


def test_scores_that_round_to_one_are_in_the_logits_order(B):
    """Without a bias, whether the groups are told apart in float32 (the first two rows) or have equal sums in float64 as well."""
    l = torch.tensor([[40.0, 50.0, 45.0, 47.0, -9.0, -8.0, -7.0, -6.0, -9.0, -9.0, -9.0, -9.0],
                      [-9.0, -9.0, -9.0, -9.0, 1e-20, 3e-20, 2e-20, 0.0, -9.0, -9.0, -9.0, -9.0],
                      [40.0, 50.0, 45.0, 47.0, 60.0, 70.0, 65.0, 62.0, 41.0, 42.0, 43.0, 44.0]])
    kw = dict(score="sigmoid", n_group=3, topk_group=1, group_top=2)
    ids, _ = B.route_experts(l.cuda(), 3, **kw)
    assert ids.tolist() == [[1, 3, 2], [5, 6, 4], [1, 3, 2]]
    for t in range(3):
        assert ids[t].tolist() == R.choose(l[t].double().numpy(), 3, **kw)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_a_bias_of_minus_infinity_takes_an_expert_out(B, score):
    T, E = 40, 24
    l = _logits(T, E, 3)
    l[20:] = l[20:].clamp(-1e-7, 1e-7) - (40.0 if score == "sigmoid" else 0.0)       # (and where the choice is made in float64)
    bias = torch.zeros(E)
    bias[::2] = -math.inf
    bias[16:] = -math.inf                              # the last third: nobody
    for kw in (dict(), dict(n_group=3, topk_group=2, group_top=2), dict(n_group=3, topk_group=3, group_top=1)):
        ids, w = B.route_experts(l.cuda(), 10, score=score, bias=bias.cuda(), **kw)
        for t in range(T):
            want = R.choose(l[t].double().numpy(), 10, score, bias.double().numpy(), **kw)
            assert ids[t].tolist() == want and want[8:] == [-1, -1], t
            assert (w[t, 8:] == 0).all() and (w[t, :8] > 0).all()


def test_weights_of_scores_that_all_underflow(B):
    l = torch.tensor([[-200.0, -201.0, -300.0, -250.0], [60.0, -60.0, 0.0, 88.0]])
    for score in ("sigmoid", "softmax"):
        ids, w = B.route_experts(l.cuda(), 2, score=score)
        for t in range(2):
            want = R.weights(l[t].double().numpy(), ids[t].tolist(), score, True, 1.0)
            np.testing.assert_allclose(w[t].double().cpu().numpy(), want, rtol=(24 + 2 * 150) * U)


def test_an_id_that_stands_twice_and_ids_outside(B):
    l = _logits(4, 40, 1)
    ids = torch.tensor([[3, 3, 3, 7], [-1, 5, 40, 5], [-1, -1, -1, -1], [39, 0, -7, 2 ** 30]], dtype=torch.int32)
    dw = torch.randn(4, 4, generator=torch.Generator().manual_seed(2))
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            d = B.route_experts_backward(l.cuda(), ids.cuda(), dw.cuda(), score=score, renormalize=renorm).double().cpu().numpy()
            for t in range(4):
                want = R.backward(l[t].double().numpy(), ids[t].tolist(), dw[t].double().numpy(), score, renorm, 1.0)
                assert (np.abs(d[t] - want) <= 256 * U * dw[t].abs().max().item()).all()


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_one_expert_alone_has_the_whole_weight_and_no_gradient(B, score):
    l = _logits(300, 20, 4)
    m = l.clone()
    m[:, 3:] = -math.inf                               # three are left, and of them one
    m[:, 1:3] = math.nan
    for logits, k in ((l, 1), (l.to(torch.bfloat16), 1), (m, 5)):
        ids, w = B.route_experts(logits.cuda(), k, score=score, scale=2.5)
        assert (w[:, 0] == 2.5).all() and (w[:, 1:] == 0).all() and (ids[:, 1:] == -1).all()
        dw = torch.randn(300, k, generator=torch.Generator().manual_seed(5)).cuda()
        assert (B.route_experts_backward(logits.cuda(), ids, dw, score=score, scale=2.5) == 0).all()


@pytest.mark.parametrize("bf16", [False, True])
def test_strided_rows_and_given_outputs(B, bf16):
    big = _logits(20, 300, 5, bf16).cuda()
    view = big[:, 7:7 + 129]
    a = B.route_experts(view, 4, score="sigmoid")
    b = B.route_experts(view.contiguous(), 4, score="sigmoid")
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    dw = torch.randn(20, 4).cuda()
    out = torch.full((20, 200), 7.0, dtype=big.dtype, device="cuda")
    r = B.route_experts_backward(view, a[0], dw, score="sigmoid", out=out[:, 3:132])
    assert torch.equal(r, B.route_experts_backward(view.contiguous(), a[0], dw, score="sigmoid"))
    assert (out[:, :3] == 7.0).all() and (out[:, 132:] == 7.0).all()
    ids, w = torch.full((24, 4), 9, dtype=torch.int32).cuda(), torch.full((24, 4), 9.0).cuda()
    B.route_experts(view, 4, score="sigmoid", out=(ids[:20], w[:20]))
    assert torch.equal(ids[:20], a[0]) and torch.equal(w[:20], a[1]) and (ids[20:] == 9).all() and (w[20:] == 9.0).all()


def test_no_tokens(B):
    l = torch.empty(0, 16).cuda()
    ids, w = B.route_experts(l, 3)
    assert ids.shape == w.shape == (0, 3)
    assert B.route_experts_backward(l, ids, w).shape == (0, 16)


def test_captured_and_replayed_and_on_another_stream(B):
    l = _logits(70, 128, 9).cuda()
    bias = torch.randn(128).cuda() * 0.1
    dw = torch.randn(70, 8).cuda()

    def both():
        ids, w = B.route_experts(l, 8, score="sigmoid", bias=bias, n_group=4, topk_group=2, group_top=2)
        return ids, w, B.route_experts_backward(l, ids, dw, score="sigmoid")
    want = [t.clone() for t in both()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    l.copy_(_logits(70, 128, 10))
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(got[0], want[0])
    assert all(torch.equal(a, b) for a, b in zip(got, both()))


def test_refusals(B):
    l = _logits(4, 16, 0).cuda()
    for kw in (dict(topk=17), dict(topk=0), dict(topk=2, n_group=3), dict(topk=2, n_group=4, topk_group=5), dict(topk=9, n_group=4, topk_group=2),
               dict(topk=2, n_group=4, topk_group=2, group_top=3), dict(topk=2, n_group=16, topk_group=2, group_top=2), dict(topk=2, topk_group=2)):
        with pytest.raises(B.QuadsError):
            B.route_experts(l, **kw)
    with pytest.raises(B.QuadsError):
        B.route_experts(_logits(2, 257, 0).cuda(), 2)
    for bad in (l.cpu(), l.double(), l.t(), l[0]):
        with pytest.raises(AssertionError):
            B.route_experts(bad, 2)
    with pytest.raises(AssertionError):
        B.route_experts(l, 2, bias=torch.zeros(15).cuda())
    with pytest.raises(KeyError):
        B.route_experts(l, 2, score="tanh")
    ids, w = B.route_experts(l, 2)
    for i, d in ((ids.long(), w), (ids, w.double()), (ids[:3], w[:3]), (ids, w[:, :1])):
        with pytest.raises(AssertionError):
            B.route_experts_backward(l, i, d)


# many tokens, several to each warp in turn: every case again at such a size, odd, and sizes around the lanes' limits
MANY = [c[1:] for c in CASES] + [
    (256, 12, "sigmoid", True, True, 16, 16, 2, 1.0, False, 0.0), (240, 8, "softmax", False, True, 15, 4, 2, 1.0, False, 0.1),
    (256, 12, "softmax", True, False, 1, 1, 1, 1.0, True, 0.7), (24, 3, "sigmoid", True, True, 3, 1, 2, 1.0, True, 0.2),
    (17, 2, "softmax", True, False, 1, 1, 1, 1.0, False, 0.95), (256, 8, "sigmoid", True, False, 8, 4, 2, 2.5, True, 0.0)]


@pytest.mark.parametrize("case", MANY, ids=lambda c: "-".join(str(v) for v in c))
def test_many_tokens(B, case):
    E, k, score, renorm, with_bias, G, kept, top, scale, bf16, masked = case
    T = 4099
    l = _logits(T, E, E, bf16, masked)
    bias = torch.randn(E, generator=torch.Generator().manual_seed(E)) * 0.2 if with_bias else None
    kw = dict(score=score, bias=None if bias is None else bias.cuda(), n_group=G, topk_group=kept, group_top=top, renormalize=renorm, scale=scale)
    ld = l.cuda()
    ids, w = B.route_experts(ld, k, **kw)
    few = [B.route_experts(ld[a:a + 900], k, **kw) for a in range(0, T, 900)]
    assert torch.equal(ids, torch.cat([f[0] for f in few]))
    torch.testing.assert_close(w, torch.cat([f[1] for f in few]), rtol=2 * W_RTOL, atol=0)
    ids, w, l64 = ids.cpu().numpy(), w.double().cpu().numpy(), l.double().numpy()
    for t in list(range(0, T, 37)) + [T - 1]:
        want = R.choose(l64[t], k, score, None if bias is None else bias.double().numpy(), G, kept, top)
        assert list(ids[t]) == want, t
        np.testing.assert_allclose(w[t], R.weights(l64[t], want, score, renorm, scale), rtol=W_RTOL, atol=0)


@pytest.mark.parametrize("scale", [1.0, 1e-5, 30.0, -400.0])
def test_scores_that_crowd_together(B, scale):
    """Logits that hardly differ, or whose sigmoids reach 1 or 0: every token has neighbours that float32 cannot tell apart."""
    T, E = 2500, 96
    l = torch.randn(T, E, generator=torch.Generator().manual_seed(9)) * 1e-5
    l = l + scale if abs(scale) > 2 else l * scale
    bias = (torch.randint(0, 3, (E,), generator=torch.Generator().manual_seed(10)).float() * 0.25)
    for kw in (dict(bias=bias), dict(n_group=8, topk_group=3, group_top=2), dict(bias=bias, n_group=4, topk_group=2, group_top=2)):
        dev = {a: (v.cuda() if torch.is_tensor(v) else v) for a, v in kw.items()}
        for score in ("sigmoid", "softmax"):
            ids, _ = B.route_experts(l.cuda(), 6, score=score, **dev)
            few, _ = B.route_experts(l[:1000].cuda(), 6, score=score, **dev)
            assert torch.equal(ids[:1000], few)
            cpu = {a: (v.double().numpy() if torch.is_tensor(v) else v) for a, v in kw.items()}
            for t in range(0, T, 101):
                assert ids[t].tolist() == R.choose(l[t].double().numpy(), 6, score, **cpu), (score, t)


@pytest.mark.parametrize("native", [True, False])
def test_ids_and_weights_are_tensors_of_their_own(B, native, monkeypatch):
    """They can be saved together, as a rollout's routing is for the trainer, and either alone without the other's memory."""
    if not native:
        monkeypatch.setattr(B, "_native", None)
    for T in (1, 40, 3000):
        ids, w = B.route_experts(_logits(T, 64, T).cuda(), 5)
        assert ids.untyped_storage().data_ptr() != w.untyped_storage().data_ptr()
        assert ids.untyped_storage().nbytes() == w.untyped_storage().nbytes() == T * 5 * 4 and ids.storage_offset() == w.storage_offset() == 0
        f = io.BytesIO()
        torch.save((ids, w), f)
        f.seek(0)
        a, b = torch.load(f)
        assert a.dtype == torch.int32 and b.dtype == torch.float32 and torch.equal(a, ids) and torch.equal(b, w)


def test_sigmoids_below_what_the_exponential_of_the_negated_logit_reaches(B):
    """exp(-l) is infinite from l = -709.8 on, the sigmoid is above 0 down to -745: the choice is the float64 score's there, too."""
    l = torch.tensor([[-740.0, -715.0, -730.0, -712.0, -744.0, -720.0, -800.0, -760.0],
                      [-744.0, -744.0, -713.0, -713.0, -711.0, -760.0, -712.0, -760.0],
                      [-900.0, -800.0, -760.0, -750.0, -1000.0, -800.0, -760.0, -750.0],
                      [-1.0, -740.0, -715.0, -730.0, -712.0, -720.0, -699.0, -701.0]])            # (one that float32 tells from the others)
    for kw in (dict(bias=torch.zeros(8)), dict(n_group=4, topk_group=2, group_top=2), dict(bias=torch.zeros(8), n_group=2, topk_group=1, group_top=2)):
        ids, _ = B.route_experts(l.cuda(), 3, score="sigmoid", **{k: v.cuda() if torch.is_tensor(v) else v for k, v in kw.items()})
        for t in range(4):
            want = R.choose(l[t].double().numpy(), 3, "sigmoid", **{k: v.double().numpy() if torch.is_tensor(v) else v for k, v in kw.items()})
            assert ids[t].tolist() == want, (t, kw)


def test_weights_of_equal_logits_are_rounded_once(B):
    """Scores of 1 among k or E of them: numerator and sum are exact, and the quotient by an approximate reciprocal and a Newton step is off by some 2^-46 of itself
    before it is rounded; no 1 / n with n up to 256 is within 2^-32 of itself of the middle between two float32s."""
    for n in range(1, 257):
        want = torch.tensor(1.0 / n, dtype=torch.float64).float().item()
        l = torch.zeros(2, n).cuda()
        assert (B.route_experts(l, 1, renormalize=False)[1] == want).all(), n
        if n <= 16:
            assert (B.route_experts(torch.zeros(2, 40).cuda(), n)[1] == want).all(), n
            assert (B.route_experts(torch.zeros(2, 40).cuda(), n, score="sigmoid")[1] == want).all(), n
