"""The work of the routing losses and of 4-bit leaf weights, as cases for timing: sizes, inputs, one pass, its cost.

Five operators of a fast feedforward layer of depth d (2^d leaves, 2^d - 1 nodes):

  balance     the balance loss of a batch, the tokens of every leaf and the mean mixture weights
  balance_d   its gradient with respect to the mixture weights
  routing_d   the gradient of the mixture weights (of any loss, of the balance loss, or of both) taken back to the node logits
  quantize    weights to microscaled 4-bit floats: e2m1 codes, one power-of-two scale per 32 of them
  forward     hard inference of a layer whose leaf weights are such codes

`run` computes them in elementary torch operations (own = False) or through the library (own = True).

Sizes come from paper_2308_14711_b200/workloads.py: 8, 256, 2048 and 32768 leaves, 768, 784 and 1024 columns, batches of whole
images of 197 tokens, 2048, 16384 and 65536 tokens.  Mixture weights are those of node logits that are normal with a spread that
grows as training hardens the nodes.  As in the parity tests, tokens with a routing logit close to zero are redrawn.
"""
from __future__ import annotations

import math

import torch

own = False

IMAGE = 197              # tokens of one image
MARGIN = 2e-3
MAX_PAIRS = 65536 * 2048                 # tokens times leaves of the largest mixture
MAX_WEIGHTS = 2048 * 32 * 2048           # leaf weights of the largest layer
MAX_PRODUCTS = 65536 * 32 * 2048         # tokens times the weights that one token meets
ACTS = ("relu", "gelu", "gelu_tanh", "silu")


def listed():
    return [
        # the routing of a small classifier: eight leaves, one batch; launches and latency count
        dict(name="balance_d3", op="balance", depth=3, B=2048, spread=1.0, valid=1.0),
        # the routing of a wide layer over a whole batch: one pass over half a gigabyte of mixture weights
        dict(name="balance_d11", op="balance", depth=11, B=65536, spread=2.0, valid=1.0),
        # sixteen images, the last of them padding
        dict(name="balance_d_d8", op="balance_d", depth=8, B=16 * IMAGE, spread=1.0, valid=0.95),
        # the wide layer, a quarter of its batch and a few tokens more
        dict(name="balance_d_d11", op="balance_d", depth=11, B=16411, spread=2.0, valid=0.9),
        # balance loss alone, small classifier
        dict(name="routing_d3", op="routing_d", depth=3, B=2048, spread=1.0, valid=1.0, upstream=False, balance=True),
        # a training step of the transformer layer: the gradient of the layer's output and the balance loss together, 256 images
        dict(name="routing_d8", op="routing_d", depth=8, B=256 * IMAGE, spread=2.0, valid=0.97, upstream=True, balance=True),
        # the leaf weights of the small classifier, float32
        dict(name="quantize_small", op="quantize", rows=256, cols=784, dtype="f32"),
        # the hidden weights of the wide layer, bf16
        dict(name="quantize_wide", op="quantize", rows=65536, cols=1024, dtype="bf16"),
        # one image through the transformer layer
        dict(name="forward_image", op="forward", D=768, O=768, depth=8, l=12, act="gelu", B=IMAGE, x="layernorm"),
        # the whole batch of 256 images
        dict(name="forward_images", op="forward", D=768, O=768, depth=8, l=12, act="gelu", B=256 * IMAGE, x="layernorm"),
        # the wide layer: its leaf weights outweigh everything else in bf16
        dict(name="forward_wide", op="forward", D=1024, O=1024, depth=11, l=32, act="gelu", B=65536, x="normal"),
        # the same layer while it serves a small batch, about one token in four leaves
        dict(name="forward_wide_few", op="forward", D=1024, O=1024, depth=11, l=32, act="gelu", B=500, x="normal"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["balance", "balance_d", "routing_d", "quantize", "forward", "forward"])
    if op == "quantize":
        cols = _log_int(rng, 1, 4096)
        return dict(op=op, rows=_log_int(rng, 1, min(131072, 65536 * 1024 // cols)), cols=cols, dtype=rng.choice(["f32", "bf16"]))
    if op != "forward":
        depth = rng.randint(0, 15)
        case = dict(op=op, depth=depth, B=_log_int(rng, 1, min(65536, MAX_PAIRS >> depth)), spread=rng.choice([0.5, 1.0, 2.0, 6.0]),
                    valid=rng.choice([1.0, 1.0, 0.9, 0.5]))
        if op == "routing_d":
            case["upstream"], case["balance"] = rng.choice([(True, True), (True, False), (False, True)])
            case["B"] = min(case["B"], 256 * IMAGE * 256 >> depth)
        return case
    D, O = (rng.choice([8 * _log_int(rng, 2, 192), _log_int(rng, 10, 1536)]) for _ in range(2))
    l = _log_int(rng, 1, 96)
    depth = rng.randint(0, 15)
    while depth > 0 and (l * (D + O) << depth) > MAX_WEIGHTS:
        depth -= 1
    return dict(op=op, D=D, O=O, depth=depth, l=l, act=rng.choice(ACTS), B=_log_int(rng, 1, min(65536, MAX_PRODUCTS // (l * (D + O)))),
                x=rng.choice(["normal", "layernorm", "clusters"]))


# ---- inputs ----------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 63) + 17)
    return g


def _normal(g, shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _mixture(g, B, depth, spread):
    """Products of sigmoids of normal node logits along the paths from the root."""
    mix = torch.ones((B, 1), device="cuda")
    for m in range(depth):
        z = torch.randn((B, 1 << m), generator=g, device="cuda") * spread
        mix = torch.stack((mix * torch.sigmoid(-z), mix * torch.sigmoid(z)), 2).reshape(B, 2 << m)
    return mix.contiguous()


def _routed(mix):
    """The leaf that the larger choice of every node leads to."""
    B, L = mix.shape
    leaf = torch.zeros(B, dtype=torch.int64, device="cuda")
    width = L
    while width > 1:
        width //= 2
        # weights of both halves of the range the token is in
        lo = torch.arange(width, device="cuda")[None, :] + (leaf * 2 * width)[:, None]
        left, right = mix.gather(1, lo).sum(1), mix.gather(1, lo + width).sum(1)
        leaf = 2 * leaf + (right >= left)
    return leaf.to(torch.int32)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _scale_codes(amax):
    """floor(log2(amax)) - 2 as a biased exponent, 0 at least; amax float32."""
    return ((amax.contiguous().view(torch.int32) >> 23) - 2).clamp_(min=0)


def _quantize(w):
    """Codes (one per byte) and biased scale exponents of the rows of w, by comparison with the midpoints (ties to the even code)."""
    rows, cols = w.shape
    nb = (cols + 31) // 32
    v = torch.nn.functional.pad(w.float(), (0, nb * 32 - cols)).reshape(rows, nb, 32)
    s = _scale_codes(v.abs().amax(2))
    v = v * torch.exp2((127 - s).float())[:, :, None]
    a = v.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for mid, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= mid) if up else (a > mid)
    code += (torch.signbit(v) & (code > 0)).to(torch.uint8) * 8
    return code.reshape(rows, nb * 32)[:, :cols], s.to(torch.uint8)


def _values(code, s, dtype=torch.float32):
    """The values that codes (one per byte) and scales stand for."""
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), dtype=dtype, device="cuda")
    scale = torch.exp2(s.to(dtype) - 127.0).repeat_interleave(32, dim=-1)[..., :code.shape[-1]]
    return table[code.long()] * scale


def _pack(code):
    cols = code.shape[-1]
    if cols % 2:
        code = torch.nn.functional.pad(code, (0, 1))
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous()


def _unpack(packed, cols):
    return torch.stack((packed & 15, packed >> 4), -1).flatten(-2)[..., :cols]


def _path_margin(x, node_w, depth):
    """Smallest |logit| on each token's path, in 64 bits."""
    B = x.shape[0]
    margin = torch.full((B,), math.inf, dtype=torch.float64, device="cuda")
    n = torch.zeros(B, dtype=torch.int64, device="cuda")
    xd = x.double()
    for m in range(depth):
        z = torch.empty(B, dtype=torch.float64, device="cuda")
        for b in range(0, B, 8192):
            z[b:b + 8192] = (node_w[(1 << m) - 1 + n[b:b + 8192]].double() * xd[b:b + 8192]).sum(1)
        margin = torch.minimum(margin, z.abs())
        n = 2 * n + (z >= 0)
    return margin


def _tokens(g, case, B):
    D = case["D"]
    x = torch.randn((B, D), generator=g, device="cuda")
    if case["x"] == "layernorm" and D > 8:
        x = (x - x.mean(1, keepdim=True)) / x.std(1, keepdim=True, unbiased=False)
    if case["x"] == "clusters":
        centres = torch.randn((16, D), generator=g, device="cuda")
        p = torch.arange(1, 17, device="cuda").float() ** -1.2
        x = centres[torch.multinomial(p, B, replacement=True, generator=g)] + 0.1 * x
    return x.bfloat16()


def _forward_inputs(case, seed):
    g = _generator(seed)
    D, O, d, l, B = case["D"], case["O"], case["depth"], case["l"], case["B"]
    nl, bf = 1 << d, torch.bfloat16
    s = dict(node_w=_normal(g, (nl - 1, D), D ** -0.5, bf), b1=_normal(g, (nl, l), 0.1, bf), b2=_normal(g, (nl, O), 0.1, bf))
    for key, rows, cols, std in (("w1", nl * l, D, D ** -0.5), ("w2", nl * l, O, l ** -0.5)):
        codes = torch.empty((rows, (cols + 1) // 2), dtype=torch.uint8, device="cuda")
        scales = torch.empty((rows, (cols + 31) // 32), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 26) // cols)
        for r in range(0, rows, step):
            c, s_ = _quantize(_normal(g, (min(step, rows - r), cols), std, bf))
            codes[r:r + step], scales[r:r + step] = _pack(c), s_
        s[key], s[key + "_scale"] = codes.reshape(nl, l, -1), scales.reshape(nl, l, -1)
    s["x"] = _tokens(g, case, B)
    for _ in range(8):
        bad = (_path_margin(s["x"], s["node_w"], d) < MARGIN).nonzero()[:, 0]
        if bad.numel() == 0:
            break
        s["x"][bad] = _tokens(g, case, bad.numel())
    return s


def _inputs(case, seed):
    op = case["op"]
    if op == "forward":
        return _forward_inputs(case, seed)
    g = _generator(seed)
    if op == "quantize":
        dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        w = torch.randn((case["rows"], case["cols"]), generator=g, device="cuda")
        # rows of different sizes, as trained neurons have them
        w *= torch.exp2(torch.randn((case["rows"], 1), generator=g, device="cuda") * 2.0 - 5.0)
        return dict(w=w.to(dtype))
    B, d = case["B"], case["depth"]
    s = dict(mixture=_mixture(g, B, d, case["spread"]))
    s["leaf"] = _routed(s["mixture"])
    valid = max(1, int(round(case["valid"] * B)))
    s["mask"] = None if valid == B else (torch.arange(B, device="cuda") < valid)
    counted = s["leaf"][:valid].long()
    s["counts"] = torch.zeros(1 << d, dtype=torch.int32, device="cuda").index_add_(0, counted, torch.ones_like(counted, dtype=torch.int32))
    s["dloss"] = torch.full((1,), 0.01, device="cuda") * (1.0 + torch.rand((1,), generator=g, device="cuda"))
    if case.get("upstream"):
        s["dmixture"] = torch.randn((B, 1 << d), generator=g, device="cuda") / B
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2308_14711_b200 import binding
        s["binding"] = binding
        if case["op"] == "forward":
            s["layer"] = binding.FFFLayer.from_mx4(case["D"], case["O"], case["depth"], case["l"], case["act"], s["node_w"], None,
                                                   s["w1"], s["w1_scale"], s["b1"], s["w2"], s["w2_scale"], s["b2"])
            s["layer"].reserve(case["B"])
        elif case["op"] != "quantize":
            # the layer whose routing it is (the smallest that has this tree)
            nl = 1 << case["depth"]
            z = lambda *shape: torch.zeros(shape, device="cuda")
            s["layer"] = binding.FFFLayer(1, 1, case["depth"], 1, "relu", "f32", z(nl - 1, 1), None, z(nl, 1, 1), None, z(nl, 1, 1), None)
    return s


# ---- one pass --------------------------------------------------------------------------------------

def _counted(s):
    B = s["mixture"].shape[0]
    return torch.ones(B, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]


def _plain_balance(s):
    mix, counted = s["mixture"], _counted(s)
    L = mix.shape[1]
    n = counted.sum()
    counts = torch.zeros(L, dtype=torch.int32, device="cuda")
    counts.index_add_(0, s["leaf"].long(), counted.to(torch.int32))
    mean = torch.where(counted[:, None], mix, 0.0).sum(0, dtype=torch.float64) / n
    loss = L * ((counts.double() / n) * mean).sum()
    return dict(loss=loss.float().reshape(()), counts=counts, mean=mean.float())


def _balance_slope(s, dtype):
    """d loss / d mixture[b, j] of a counted token b, for every j."""
    counts = s["counts"].to(dtype)
    n = counts.sum()
    return s["dloss"].to(dtype) * counts.shape[0] * (counts / n) / n


def _plain_balance_d(s):
    return dict(dmixture=torch.where(_counted(s)[:, None], _balance_slope(s, torch.float32)[None, :], 0.0))


def _plain_routing_d(s):
    case, mix = s["case"], s["mixture"]
    counted = _counted(s)[:, None]
    slope = torch.zeros((), device="cuda")
    if case["balance"]:
        # (a slope that is the same for every leaf moves nothing: weights sum to one)
        counts = s["counts"].double()
        n, L = counts.sum(), counts.shape[0]
        slope = (s["dloss"].double() * (L * counts - n) / (n * n)).float()[None, :]
    if case["upstream"]:
        slope = slope + s["dmixture"]
    m, t = mix, mix * slope
    levels = []
    while m.shape[1] > 1:
        ml, mr, tl, tr = m[:, 0::2], m[:, 1::2], t[:, 0::2], t[:, 1::2]
        total = ml + mr
        g = torch.where(total > 0, (tr * (ml / total) - tl * (mr / total)), 0.0)
        levels.append(torch.where(counted, g, 0.0))
        m, t = total, tl + tr
    out = torch.cat(levels[::-1], 1) if levels else torch.empty((mix.shape[0], 0), device="cuda")
    return dict(dlogits=out)


def _plain_quantize(s):
    code, scale = _quantize(s["w"])
    return dict(values=_values(code, scale).to(s["w"].dtype), scales=scale)


def _act(name, v):
    if name == "relu":
        return v.clamp(min=0)
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * 0.7071067811865476))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(0.7978845608028654 * (v + 0.044715 * v * v * v)))
    return v / (1 + torch.exp(-v))


def _plain_forward(s):
    case = s["case"]
    D, O, d, l, B = case["D"], case["O"], case["depth"], case["l"], case["B"]
    x = s["x"].float()
    n = torch.zeros(B, dtype=torch.int64, device="cuda")
    step = max(1, (1 << 26) // D)
    for m in range(d):
        z = torch.cat([(s["node_w"][(1 << m) - 1 + n[b:b + step]].float() * x[b:b + step]).sum(1) for b in range(0, B, step)])
        n = 2 * n + (z >= 0)
    y = torch.empty((B, O), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 27) // (l * (D + O)))
    for b in range(0, B, step):
        j = n[b:b + step]
        w1 = _values(_unpack(s["w1"][j], D), s["w1_scale"][j])
        w2 = _values(_unpack(s["w2"][j], O), s["w2_scale"][j])
        h = _act(case["act"], torch.bmm(w1, x[b:b + step, :, None])[:, :, 0] + s["b1"][j].float())
        y[b:b + step] = torch.bmm(h[:, None, :], w2)[:, 0] + s["b2"][j].float()
    return dict(y=y, leaf=n.to(torch.int32))


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"balance": _plain_balance, "balance_d": _plain_balance_d, "routing_d": _plain_routing_d,
                "quantize": _plain_quantize, "forward": _plain_forward}[op](s)
    if op == "balance":
        loss, counts, mean = s["layer"].balance_loss(s["mixture"], s["leaf"], token_mask=s["mask"])
        return dict(loss=loss, counts=counts, mean=mean)
    if op == "balance_d":
        return dict(dmixture=s["layer"].balance_loss_backward(s["leaf"], s["counts"], s["dloss"], token_mask=s["mask"]))
    if op == "routing_d":
        more = dict(leaf_idx=s["leaf"], counts=s["counts"], dloss=s["dloss"]) if s["case"]["balance"] else {}
        return dict(dlogits=s["layer"].routing_backward(s["mixture"], dmixture=s.get("dmixture"), token_mask=s["mask"], **more))
    if op == "quantize":
        _, scales, values = s["binding"].quantize_mx4(s["w"], want_values=True)
        return dict(values=values, scales=scales)
    y, leaf = s["layer"].forward_infer(s["x"])
    return dict(y=y, leaf=leaf)


# ---- cost and exact values -------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "quantize":
        n, e = case["rows"] * case["cols"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": n * (2 * e + 0.5) + case["rows"] * ((case["cols"] + 31) // 32), "flops": 3 * n}
    B, L = case["B"], 1 << case["depth"]
    if op == "forward":
        D, O, d, l = case["D"], case["O"], case["depth"], case["l"]
        seen = lambda n: n * -math.expm1(B * math.log1p(-1.0 / n)) if n > 1 else 1.0
        nodes = sum(seen(1 << m) for m in range(d))
        leaves = seen(L)
        weights = l * (0.5 * (D + O) + (D + 31) // 32 + (O + 31) // 32) + 2 * (l + O)
        return {"bytes": 2 * B * (D + O) + 4 * B + 2 * D * nodes + weights * leaves, "flops": 2.0 * B * (d * D + l * D + l * O)}
    mask = 0 if case["valid"] == 1.0 else B
    if op == "balance":
        return {"bytes": 4 * B * L * case["valid"] + 4 * B + mask + 8 * L, "flops": B * L}
    if op == "balance_d":
        return {"bytes": 4 * B * L + 4 * B + mask + 4 * L, "flops": B * L}
    return {"bytes": 4 * B * L * (case["valid"] * (1 + case["upstream"]) + 1) + mask + 4 * (L + B) * case["balance"], "flops": 8 * B * L}


def exact(case, seed):
    """The definitions in 64 bits."""
    op = case["op"]
    s = _inputs(case, seed)
    f64 = torch.float64
    if op == "quantize":
        # every element takes the nearest of the 15 values of its block's scale, the one with the even code at a tie
        w = s["w"].double()
        rows, cols = w.shape
        out = torch.zeros_like(w)
        scales = torch.zeros((rows, (cols + 31) // 32), dtype=torch.uint8, device="cuda")
        for b in range(0, cols, 32):
            block = w[:, b:b + 32]
            amax = block.abs().amax(1)
            e = torch.frexp(amax).exponent.to(f64) - 1 - 2          # amax = m 2^exponent, 1/2 <= m < 1
            e = torch.where(amax > 0, e, -127.0).clamp(min=-127.0)
            scales[:, b // 32] = (e + 127).to(torch.uint8)
            unit = torch.exp2(e)[:, None]
            q = block.abs() / unit
            step = torch.where(q < 2, 0.5, torch.where(q < 4, 1.0, 2.0))
            out[:, b:b + 32] = torch.copysign((torch.round(q / step) * step).clamp(max=6.0), block) * unit
        return dict(values=out, scales=scales)
    if op == "forward":
        D, O, d, l, B = case["D"], case["O"], case["depth"], case["l"], case["B"]
        if B * l * (D + O) > MAX_PRODUCTS:
            return None
        x = s["x"].double()
        n = torch.zeros(B, dtype=torch.int64, device="cuda")
        for m in range(d):
            for b in range(0, B, 8192):
                z = torch.linalg.vecdot(s["node_w"][(1 << m) - 1 + n[b:b + 8192]].double(), x[b:b + 8192])
                n[b:b + 8192] = 2 * n[b:b + 8192] + (z >= 0)
        order = torch.argsort(n, stable=True)
        leaves, counts = torch.unique_consecutive(n[order], return_counts=True)
        y = torch.empty((B, O), dtype=f64, device="cuda")
        start = 0
        for j, c in zip(leaves.tolist(), counts.tolist()):
            t = order[start:start + c]
            start += c
            w1 = _values(_unpack(s["w1"][j], D), s["w1_scale"][j], f64)
            w2 = _values(_unpack(s["w2"][j], O), s["w2_scale"][j], f64)
            h = _act(case["act"], x[t] @ w1.T + s["b1"][j].double())
            y[t] = h @ w2 + s["b2"][j].double()
        return dict(y=y, leaf=n.to(torch.int32))
    mix = s["mixture"].double()
    B, L = mix.shape
    rows = torch.arange(B, device="cuda") if s["mask"] is None else s["mask"].nonzero()[:, 0]
    f = torch.bincount(s["leaf"][rows].long(), minlength=L).double() / rows.numel()
    if op == "balance":
        mean = mix[rows].sum(0) / rows.numel()
        return dict(loss=(L * (f @ mean)).reshape(()), counts=(f * rows.numel()).round().to(torch.int32), mean=mean)
    slope = s["dloss"].double() * L * f / rows.numel()
    if op == "balance_d":
        out = torch.zeros((B, L), dtype=f64, device="cuda")
        out[rows] = slope
        return dict(dmixture=out)
    grad = torch.zeros((rows.numel(), L), dtype=f64, device="cuda")
    if case["balance"]:
        grad += slope
    if case["upstream"]:
        grad += s["dmixture"][rows].double()
    out = torch.zeros((B, L - 1), dtype=f64, device="cuda")
    mix = mix[rows]
    for m in range(case["depth"]):
        # level m: 2^m nodes, each over 2 * half leaves
        half = L >> (m + 1)
        w = mix.reshape(-1, 1 << m, 2, half)
        wg = (w * grad.reshape(w.shape)).sum(3)
        w = w.sum(3)
        total = w.sum(2)
        # d mix_j / d z = mix_j (1 - c) on the right of the node, -mix_j c on its left; c the right half's share, 1 - c the left half's
        left, right = (torch.where(total > 0, w[:, :, k] / total, 0.0) for k in (0, 1))
        out[rows, (1 << m) - 1:(2 << m) - 1] = wg[:, :, 1] * left - wg[:, :, 0] * right
    return dict(dlogits=out)
