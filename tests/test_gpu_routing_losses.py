"""The balance loss, its gradient, and the way from the mixture weights back to the node logits, against float64.

Tolerances (u = 2^-24, float32):
  mean          a float32 sum over the rows of one thread (at most n_rows), then at most 44 more float32 additions in a CTA, float64 above:
                (n_rows + 46) u relative to the mean itself (the weights are not negative), one rounding included;
  loss          a sum of such terms: the same relative bound and one rounding more;
  dmixture      one rounding: u relative;
  dlogits       at every node of d levels: sums M and S over 2^d leaves bottom-up, d + 1 roundings each, relative to sums of magnitudes; the
                quotients' reciprocal is good to 2 u, four products and a difference follow: 2 (d + 8) u (A_right (1 - c) + A_left c) with A
                the sum of mix_j |g_j|, and the slope of the balance loss itself is rounded once (u) and added (u).
                Weights under 2^-126 are lost: 2^-126 2^d |g| more.
"""
import numpy as np
import pytest
import torch

from oracle import fff_oracle as orc
from paper_2308_14711_b200 import binding, workloads as wl
from paper_2308_14711_b200.binding import FFFError, FFFLayer
from tests import util

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def tree(depth):
    nl = 1 << depth
    z = lambda *s: torch.zeros(s, device="cuda")
    return FFFLayer(1, 1, depth, 1, "relu", "f32", z(nl - 1, 1), None, z(nl, 1, 1), None, z(nl, 1, 1), None)


def mixture(B, depth, seed, spread):
    g = np.random.default_rng(seed)
    mix = np.ones((B, 1))
    for m in range(depth):
        c = 1 / (1 + np.exp(-g.standard_normal((B, 1 << m)) * spread))
        mix = np.stack([mix * (1 - c), mix * c], 2).reshape(B, -1)
    return mix.astype(np.float32)


def leaves(B, depth, seed, skew=False):
    g = np.random.default_rng(seed + 1)
    nl = 1 << depth
    return (np.minimum(g.zipf(1.3, B) - 1, nl - 1) if skew else g.integers(0, nl, B)).astype(np.int32)


def gpu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def node_gradients(mix, g, depth):
    """dlogits and the sum of magnitudes behind each, float64."""
    B, L = mix.shape
    out, mag = np.zeros((B, L - 1)), np.zeros((B, L - 1))
    for m in range(depth):
        w = mix.reshape(B, 1 << m, 2, L >> (m + 1))
        wg, wa = (w * g.reshape(w.shape)).sum(3), (w * np.abs(g).reshape(w.shape)).sum(3)
        w = w.sum(3)
        total = w.sum(2)
        # (1 - c as a quotient too: a difference would lose it where the node is nearly certain)
        left, c = (np.divide(w[:, :, k], total, out=np.zeros_like(total), where=total > 0) for k in (0, 1))
        at = slice((1 << m) - 1, (2 << m) - 1)
        out[:, at] = wg[:, :, 1] * left - wg[:, :, 0] * c
        mag[:, at] = wa[:, :, 1] * left + wa[:, :, 0] * c
    return out, mag


SIZES = [(0, 1), (0, 77), (1, 1), (1, 2), (1, 5), (1, 4097), (2, 3), (3, 1), (3, 2048), (4, 1001), (5, 7), (6, 130), (7, 65), (8, 1), (8, 3941),
         (9, 257), (11, 33), (11, 700), (12, 5), (13, 9), (15, 3)]


@pytest.mark.parametrize("kind", ["plain", "mask", "out_of_range", "nothing"])
@pytest.mark.parametrize("depth,B", SIZES)
def test_balance_loss(depth, B, kind):
    L = 1 << depth
    mix, leaf, mask = mixture(B, depth, B, 1.5), leaves(B, depth, depth, skew=depth > 6), None
    g = np.random.default_rng(5)
    if kind == "mask":
        mask = (g.random(B) < 0.7).astype(np.uint8) * 3
        mix[mask == 0] = np.nan                            # padding may hold anything
        mix[np.flatnonzero(mask == 0)[::2]] = np.inf
    if kind == "out_of_range":
        leaf[::3], leaf[1::5] = -1, L
        leaf[2::7] = np.iinfo(np.int32).min
    if kind == "nothing":
        mask = np.zeros(B, np.uint8)
        mix[:] = np.nan
    layer = tree(depth)
    counted = (leaf >= 0) & (leaf < L) & (np.ones(B, bool) if mask is None else mask != 0)
    n = int(counted.sum())
    counts = np.bincount(leaf[counted], minlength=L)
    mean = mix[counted].astype(np.float64).sum(0) / max(n, 1)
    loss = L * (counts / max(n, 1) * mean).sum()
    bound = (B + 46) * U
    first = None
    for _ in range(2):
        got, c, m = layer.balance_loss(gpu(mix), gpu(leaf), None if mask is None else gpu(mask))
        np.testing.assert_array_equal(c.cpu().numpy(), counts)
        assert got.shape == () and (np.abs(m.cpu().numpy() - mean) <= bound * mean + 1e-45).all()
        assert abs(float(got) - loss) <= (bound + U) * loss
        assert first is None or (float(got) == first[0] and torch.equal(m, first[1]))
        first = float(got), m.clone()
    if mask is not None:                                   # a bool mask is the same mask
        got, c2, m2 = layer.balance_loss(gpu(mix), gpu(leaf), gpu(mask).bool())
        assert torch.equal(c2, c) and torch.equal(m2, m) and float(got) == first[0]
    # its gradient
    dloss = torch.tensor([0.37], device="cuda")
    d = layer.balance_loss_backward(gpu(leaf), c, dloss, None if mask is None else gpu(mask)).cpu().numpy()
    ref = np.zeros((B, L))
    if n:
        ref[counted] = float(dloss) * L * counts / n / n
    assert d.shape == (B, L) and (np.abs(d - ref) <= 1.001 * U * ref).all()
    layer.close()


@pytest.mark.parametrize("depth,B,n_slices_more_than_one", [(3, 20000, True), (8, 50432, True), (11, 9000, True)])
def test_balance_loss_of_many_rows_on_one_handle_in_turn(depth, B, n_slices_more_than_one):
    """Batches of several slices, then a small one, then the first again: the scratch is clean in between."""
    layer = tree(depth)
    big, small = (mixture(B, depth, 1, 1.0), leaves(B, depth, 1)), (mixture(5, depth, 2, 1.0), leaves(5, depth, 2))
    results = []
    for mix, leaf in (big, small, big, small):
        loss, counts, mean = layer.balance_loss(gpu(mix), gpu(leaf))
        ref = mix.astype(np.float64).mean(0)
        np.testing.assert_array_equal(counts.cpu().numpy(), np.bincount(leaf, minlength=1 << depth))
        assert (np.abs(mean.cpu().numpy() - ref) <= (len(mix) + 46) * U * ref).all()
        results.append((float(loss), mean.clone()))
    assert results[0][0] == results[2][0] and torch.equal(results[0][1], results[2][1])
    assert results[1][0] == results[3][0] and torch.equal(results[1][1], results[3][1])
    layer.close()


@pytest.mark.parametrize("kind", ["upstream", "balance", "both", "both_masked", "both_out_of_range"])
@pytest.mark.parametrize("depth,B", SIZES)
def test_routing_backward(depth, B, kind):
    L = 1 << depth
    mix, leaf = mixture(B, depth, 3 * B, 6.0 if B % 2 else 1.0), leaves(B, depth, depth)
    g = np.random.default_rng(B)
    up = None if kind == "balance" else g.standard_normal((B, L)).astype(np.float32)
    mask = None
    if kind == "both_masked":
        mask = (g.random(B) < 0.6)
    if kind == "both_out_of_range":
        leaf[::2] = -5
    counted = (leaf >= 0) & (mask if mask is not None else True)
    counts = np.bincount(leaf[counted], minlength=L)
    n, layer, dloss = int(counted.sum()), tree(depth), 0.25
    if mask is not None:
        mix[~mask] = np.nan
        up[~mask] = np.inf
    args = {} if kind == "upstream" else dict(leaf_idx=gpu(leaf), counts=gpu(counts.astype(np.int32)), dloss=torch.tensor(dloss, device="cuda"))
    got = layer.routing_backward(gpu(mix), dmixture=gpu(up), token_mask=gpu(mask), **args)
    assert got.shape == (B, L - 1)
    grad = np.zeros((B, L)) if up is None else up.astype(np.float64)
    bal = np.zeros((B, L))
    if kind != "upstream" and n:
        bal[leaf >= 0] = dloss * (L * counts - n) / n / n          # (a constant over the leaves moves nothing: next test)
    keep = np.ones(B, bool) if mask is None else mask
    got = got.cpu().numpy()
    assert (got[~keep] == 0).all()
    ref, _ = node_gradients(mix[keep].astype(np.float64), (grad + bal)[keep], depth)
    _, mag = node_gradients(mix[keep].astype(np.float64), (np.abs(grad) + np.abs(bal))[keep], depth)
    bound = (2 * (depth + 8) + 2) * U * mag + 2.0 ** -126 * L * (np.abs(grad[keep]).max(initial=0) + np.abs(bal).max(initial=0))
    assert (np.abs(got[keep] - ref) <= bound).all()
    layer.close()


def test_gradients_are_those_of_the_loss():
    """Central differences in float64 of loss(node logits) = balance loss + <v, mixture>, and autograd of the same."""
    depth, B = 4, 13
    L = 1 << depth
    g = np.random.default_rng(0)
    z, v, leaf = g.standard_normal((B, L - 1)), g.standard_normal((B, L)), leaves(B, depth, 3)
    counts = np.bincount(leaf, minlength=L)
    alpha = 0.8

    def mix_of(z):
        mix = torch.ones((B, 1), dtype=torch.float64)
        for m in range(depth):
            c = torch.sigmoid(z[:, (1 << m) - 1:(2 << m) - 1])
            mix = torch.stack([mix * (1 - c), mix * c], 2).reshape(B, -1)
        return mix

    def f(z):
        mix = mix_of(z)
        return alpha * L * (torch.from_numpy(counts) / B * mix.mean(0)).sum() + (torch.from_numpy(v) * mix).sum()

    zt = torch.from_numpy(z).requires_grad_()
    f(zt).backward()
    layer = tree(depth)
    mix = mix_of(torch.from_numpy(z)).float().cuda().contiguous()
    got = layer.routing_backward(mix, dmixture=gpu(v.astype(np.float32)), leaf_idx=gpu(leaf), counts=gpu(counts.astype(np.int32)),
                                 dloss=torch.tensor([alpha], device="cuda")).cpu().double()
    # (mixture weights rounded to float32, 2^-24 relative each, and v; the magnitudes are below 4)
    assert (got - zt.grad).abs().max() <= 200 * U
    eps = 1e-5
    for b, k in ((0, 0), (3, 1), (7, 5), (12, L - 2)):
        hi, lo = z.copy(), z.copy()
        hi[b, k] += eps
        lo[b, k] -= eps
        slope = float(f(torch.from_numpy(hi)) - f(torch.from_numpy(lo))) / (2 * eps)
        assert abs(slope - float(got[b, k])) <= 200 * U + 1e-8
    # the same through the matrix of the balance loss's gradient
    d = layer.balance_loss_backward(gpu(leaf), gpu(counts.astype(np.int32)), torch.tensor([alpha], device="cuda"))
    two = layer.routing_backward(mix, dmixture=d + gpu(v.astype(np.float32)))
    assert (two.cpu().double() - zt.grad).abs().max() <= 400 * U
    layer.close()


def test_saturated_nodes():
    """Mixture weights of exactly 0 and 1, and subtrees whose weights all vanish: zeros, not NaN."""
    depth, B = 9, 64
    L = 1 << depth
    mix = np.zeros((B, L), np.float32)
    mix[np.arange(B), leaves(B, depth, 1)] = 1.0
    mix[5] = 1e-42                                        # below the smallest normal number throughout
    up = np.random.default_rng(1).standard_normal((B, L)).astype(np.float32)
    layer = tree(depth)
    got = layer.routing_backward(gpu(mix), dmixture=gpu(up)).cpu().numpy()
    assert (np.abs(got) <= 1e-39).all()                   # a node that is certain has no gradient
    layer.close()


def test_calls_are_captured_and_replayed_on_another_stream():
    depth, B = 8, 3000
    layer = tree(depth)
    mix, leaf = gpu(mixture(B, depth, 0, 1.0)), gpu(leaves(B, depth, 0))
    dloss = torch.ones(1, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def step():
        loss, counts, mean = layer.balance_loss(mix, leaf)
        return loss, counts, mean, layer.routing_backward(mix, leaf_idx=leaf, counts=counts, dloss=dloss)
    with torch.cuda.stream(side):
        eager = [t.clone() for t in step()]
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, eager))
    mix2, leaf2 = gpu(mixture(B, depth, 9, 2.0)), gpu(leaves(B, depth, 9))
    mix.copy_(mix2)
    leaf.copy_(leaf2)
    graph.replay()
    again = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    del graph
    layer.close()


def test_outputs_end_where_they_should():
    depth, B = 3, 1001
    L = 1 << depth
    layer = tree(depth)
    mix, leaf = gpu(mixture(B, depth, 0, 1.0)), gpu(leaves(B, depth, 0))
    counts = torch.full((L + 8,), -7, dtype=torch.int32, device="cuda")
    mean = torch.full((L + 8,), -7.0, device="cuda")
    dmix = torch.full((B * L + 8,), -7.0, device="cuda")
    dz = torch.full((B * (L - 1) + 8,), -7.0, device="cuda")
    loss = torch.full((4,), -7.0, device="cuda")
    one = torch.ones(1, device="cuda")
    lib, h = binding.lib(), layer.handle
    assert lib.fff_balance_loss(h, mix.data_ptr(), leaf.data_ptr(), None, loss.data_ptr(), counts.data_ptr(), mean.data_ptr(), B, None) == 0
    assert lib.fff_balance_loss_backward(h, leaf.data_ptr(), None, counts.data_ptr(), one.data_ptr(), dmix.data_ptr(), B, None) == 0
    assert lib.fff_routing_backward(h, mix.data_ptr(), dmix.data_ptr(), None, None, None, None, dz.data_ptr(), B, None) == 0
    torch.cuda.synchronize()
    assert (counts[L:] == -7).all() and (mean[L:] == -7).all() and (dmix[B * L:] == -7).all() and (dz[B * (L - 1):] == -7).all()
    assert (loss[1:] == -7).all() and (counts[:L] >= 0).all()
    # outputs one by one
    for k in range(3):
        only = [None, None, None]
        buf = [torch.full((1,), -7.0, device="cuda"), torch.full((L,), -7, dtype=torch.int32, device="cuda"), torch.full((L,), -7.0, device="cuda")]
        only[k] = buf[k].data_ptr()
        assert lib.fff_balance_loss(h, mix.data_ptr(), leaf.data_ptr(), None, *only, B, None) == 0
        torch.cuda.synchronize()
        assert torch.equal(buf[k], (loss[:1], counts[:L], mean[:L])[k])
    layer.close()


def test_an_empty_batch():
    layer = tree(3)
    e = lambda *s: torch.empty(s, device="cuda")
    loss, counts, mean = layer.balance_loss(e(0, 8), torch.empty(0, dtype=torch.int32, device="cuda"))
    assert float(loss) == 0 and (counts == 0).all() and (mean == 0).all()
    assert layer.balance_loss_backward(torch.empty(0, dtype=torch.int32, device="cuda"), counts, loss).shape == (0, 8)
    assert layer.routing_backward(e(0, 8), dmixture=e(0, 8)).shape == (0, 7)
    layer.close()


def test_a_step_of_training_the_routing_and_then_serving_in_4_bits():
    """FORWARD_T's weights and the leaves of the descent into the loss and back to the node weights; the loss falls along the gradient as the
    first order says; then the leaves are quantised, and the 4-bit layer routes as the trained one does."""
    cfg = wl.FFFConfig("run", 128, 64, 5, 16, "gelu", "bf16", 600, "clusters")
    case = util.make_case(cfg, seed=3)
    layer = util.make_layer(case)
    x = util.to_device(case.x, "bf16")
    y, mix, _ = layer.forward_train(x)
    leaf = layer.tree_descent(x)
    loss, counts, mean = layer.balance_loss(mix, leaf)
    dz = layer.routing_backward(mix, leaf_idx=leaf, counts=counts, dloss=torch.ones(1, device="cuda"))
    dw = dz.double().T @ x.double()
    node_w = util.to_device(case.weights["node_w"], "bf16").double()

    def loss_of(w):                                        # with the same f: counts carry no gradient
        z = x.double() @ w.T + util.to_device(case.weights["node_b"], "bf16").double()
        m = torch.ones((cfg.B, 1), dtype=torch.float64, device="cuda")
        for k in range(cfg.depth):
            c = torch.sigmoid(z[:, (1 << k) - 1:(2 << k) - 1])
            m = torch.stack([m * (1 - c), m * c], 2).reshape(cfg.B, -1)
        return float(cfg.n_leaves * (counts.double() / cfg.B * m.mean(0)).sum())
    # mixture weights are good to 2e-4 relative (bf16-exact products, float32 sigmoids), and so is the loss
    assert abs(loss_of(node_w) - float(loss)) <= 1e-3 * float(loss)
    step = 1e-4
    slope = (loss_of(node_w + step * dw) - loss_of(node_w - step * dw)) / (2 * step)
    assert abs(slope - float((dw * dw).sum())) <= 1e-2 * slope
    # serving
    dev = {k: util.to_device(v, "bf16") for k, v in case.weights.items()}
    c1, s1, v1 = binding.quantize_mx4(dev["w1"], want_values=True)
    c2, s2, v2 = binding.quantize_mx4(dev["w2"].transpose(1, 2).contiguous(), want_values=True)
    q = FFFLayer.from_mx4(cfg.D, cfg.O, cfg.depth, cfg.leaf_width, cfg.activation, dev["node_w"], dev["node_b"], c1, s1, dev["b1"], c2, s2, dev["b2"])
    plain = FFFLayer(cfg.D, cfg.O, cfg.depth, cfg.leaf_width, cfg.activation, "bf16", dev["node_w"], dev["node_b"], v1, dev["b1"],
                     v2.transpose(1, 2).contiguous(), dev["b2"])
    yq, leaf_q = q.forward_infer(x)
    yp, leaf_p = plain.forward_infer(x)
    assert torch.equal(leaf_q, leaf_p) and torch.equal(leaf_q, leaf)
    net = orc.Net(cfg.D, cfg.O, cfg.depth, cfg.leaf_width, cfg.activation, case.weights["node_w"], case.weights["node_b"], v1.float().cpu().numpy(),
                  case.weights["b1"], v2.float().transpose(1, 2).contiguous().cpu().numpy(), case.weights["b2"])
    y_ref, _ = orc.forward_i(net, case.x, threads=util.ORACLE_THREADS)
    util.check_outputs(yq, y_ref, "bf16")
    util.check_outputs(yp, y_ref, "bf16")
    loss_q, counts_q, _ = q.balance_loss(mix, leaf_q)
    assert torch.equal(counts_q, counts) and float(loss_q) == float(loss)
    for l in (layer, q, plain):
        l.close()


# ---- refusals

@pytest.fixture(params=["module", "ctypes"])
def call(request, monkeypatch):
    """The calls through the CPython module, and as they are made where that has not been built."""
    if request.param == "ctypes":
        monkeypatch.setattr(binding, "torch_call", lambda: None)
    else:
        assert binding.torch_call() is not None


def test_both_ways_of_calling_give_the_same(call):
    """Against the first way's results, on another stream too."""
    depth, B = 5, 301
    layer = tree(depth)
    mix, leaf, mask = gpu(mixture(B, depth, 2, 1.0)), gpu(leaves(B, depth, 2)), torch.arange(B, device="cuda") % 5 != 0
    up, one = torch.randn(B, 32, device="cuda", generator=torch.Generator("cuda").manual_seed(1)), torch.ones((), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    runs = []
    for stream in (None, side):
        loss, counts, mean = layer.balance_loss(mix.requires_grad_(), leaf, token_mask=mask, stream=stream)
        side.synchronize()
        d = layer.balance_loss_backward(leaf, counts, one, token_mask=mask.byte(), stream=stream)
        z = layer.routing_backward(mix, dmixture=up, leaf_idx=leaf, counts=counts, dloss=one, token_mask=mask, stream=stream)
        q = binding.quantize_mx4(up, want_values=True, stream=stream)
        torch.cuda.synchronize()
        assert not (loss.requires_grad or d.requires_grad or z.requires_grad)
        runs.append((loss, counts, mean, d, z) + q)
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    key = [t.detach().cpu() for t in runs[0]]
    global _first_way
    _first_way = globals().get("_first_way", key)
    assert all(torch.equal(a, b) for a, b in zip(_first_way, key))
    layer.close()


def test_calls_that_are_refused(call):
    layer = tree(3)
    mix, leaf = torch.rand(10, 8, device="cuda"), torch.zeros(10, dtype=torch.int32, device="cuda")
    counts, one = torch.ones(8, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    for bad in (dict(mixture=mix.double(), leaf_idx=leaf), dict(mixture=mix[:, :4], leaf_idx=leaf), dict(mixture=mix, leaf_idx=leaf.long()),
                dict(mixture=mix, leaf_idx=leaf[:9]), dict(mixture=mix, leaf_idx=leaf, token_mask=torch.ones(9, device="cuda").bool()),
                dict(mixture=mix, leaf_idx=leaf, token_mask=torch.ones(10, device="cuda")), dict(mixture=mix.cpu(), leaf_idx=leaf),
                dict(mixture=mix.T.contiguous().T, leaf_idx=leaf)):
        with pytest.raises(ValueError):
            layer.balance_loss(**bad)
    for bad in (dict(counts=counts[:4], dloss=one), dict(counts=counts, dloss=torch.ones(2, device="cuda")), dict(counts=counts.float(), dloss=one)):
        with pytest.raises(ValueError):
            layer.balance_loss_backward(leaf, **bad)
    for bad in (dict(), dict(counts=counts), dict(dloss=one), dict(dmixture=mix, counts=counts)):
        with pytest.raises(FFFError) as e:
            layer.routing_backward(mix, **bad)
        assert e.value.status == 1
    lib, h = binding.lib(), layer.handle
    p = lambda t: t.data_ptr()
    out = torch.zeros(200, device="cuda")
    assert lib.fff_balance_loss(h, None, p(leaf), None, p(out), None, None, 10, None) == 1
    assert lib.fff_balance_loss(h, p(mix), None, None, p(out), None, None, 10, None) == 1
    assert lib.fff_balance_loss(h, p(mix) + 4, p(leaf), None, p(out), None, None, 9, None) == 1
    assert lib.fff_balance_loss(h, p(mix), p(leaf), None, p(out) + 2, None, None, 10, None) == 1
    assert lib.fff_balance_loss(h, p(mix), p(leaf), None, p(out), None, None, -1, None) == 1
    assert lib.fff_balance_loss(h, p(mix), p(leaf), None, p(out), None, None, (1 << 31), None) == 2
    assert lib.fff_balance_loss_backward(h, p(leaf), None, None, p(one), p(out), 10, None) == 1
    assert lib.fff_balance_loss_backward(h, p(leaf), None, p(counts), p(one), p(out) + 4, 10, None) == 1
    assert lib.fff_routing_backward(h, p(mix), p(mix), None, None, None, None, None, 10, None) == 1
    assert lib.fff_routing_backward(h, p(mix), p(mix), None, None, None, None, p(out) + 8, 10, None) == 1
    assert lib.fff_balance_loss(h, p(mix), p(leaf), None, None, None, None, 10, None) == 0          # nothing asked for
    layer.close()


# sizes at which the kernels change their ways: a row per warp from 128 leaves on, rows by warps up to 512 and by CTAs (several at a time, the last
# group not full) above, slopes in shared memory up to 8192, more than 256 rows in a sum, several groups of slices
MORE_SIZES = [(0, 600), (2, 70001), (5, 3000), (6, 9001), (7, 127), (7, 40001), (8, 3), (9, 5000), (10, 64), (10, 1003), (11, 597), (12, 333),
              (13, 333), (14, 21), (16, 2)]


@pytest.mark.parametrize("kind", ["mask", "out_of_range"])
@pytest.mark.parametrize("depth,B", MORE_SIZES)
def test_balance_loss_where_its_ways_change(depth, B, kind):
    test_balance_loss(depth, B, kind)


@pytest.mark.parametrize("kind", ["upstream", "balance", "both_masked"])
@pytest.mark.parametrize("depth,B", MORE_SIZES)
def test_routing_backward_where_its_ways_change(depth, B, kind):
    test_routing_backward(depth, B, kind)


def test_rows_and_gradients_end_where_they_end():
    """Nothing behind the last row is written, and what lies behind the last row of the mixture weights is not used."""
    for depth, B in ((1, 77), (3, 61), (8, 5), (9, 3), (10, 1001), (11, 3), (13, 2)):
        L = 1 << depth
        mix, leaf, layer = mixture(B, depth, 7, 1.0), leaves(B, depth, 7), tree(depth)
        wide = torch.full((B * L + 4096,), float("nan"), device="cuda")
        wide[:B * L] = gpu(mix).flatten()
        x = wide[:B * L].view(B, L)
        loss, counts, mean = layer.balance_loss(x, gpu(leaf))
        want = layer.balance_loss(gpu(mix), gpu(leaf))
        assert float(loss) == float(want[0]) and torch.equal(mean, want[2])
        out, d = torch.full((B * (L - 1) + 64,), 7.0, device="cuda"), torch.full((B * L + 64,), 7.0, device="cuda")
        dloss, stream = torch.tensor([0.5], device="cuda"), torch.cuda.current_stream().cuda_stream
        lib, h, idx = binding.lib(), layer._h, gpu(leaf)
        assert lib.fff_routing_backward(h, x.data_ptr(), None, idx.data_ptr(), None, counts.data_ptr(), dloss.data_ptr(), out.data_ptr(), B, stream) == 0
        assert lib.fff_balance_loss_backward(h, idx.data_ptr(), None, counts.data_ptr(), dloss.data_ptr(), d.data_ptr(), B, stream) == 0
        torch.cuda.synchronize()
        assert (out[B * (L - 1):] == 7.0).all() and (d[B * L:] == 7.0).all()
        assert torch.equal(out[:B * (L - 1)].view(B, L - 1), layer.routing_backward(gpu(mix), leaf_idx=idx, counts=counts, dloss=dloss))
        layer.close()
