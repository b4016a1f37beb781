"""Performance cases of the router with scores, groups and a balance bias, and of the 8-bit expert path.

A case names one operator and a model shape with its micro-batches:

* ``route``    - gating: softmax or sigmoid scores, a bias for the choice alone, groups of experts, top-k, weights; with the
  counts per expert and per virtual device;
* ``dispatch`` - token rows grouped by (virtual device, layer, expert) and quantised to e4m3 with a scale for each token and
  block of 128 elements;
* ``weights``  - bf16 weights to e4m3 with a scale for each 128 x 128 block;
* ``experts``  - the grouped SwiGLU expert pass on e4m3 rows and weights with those scales, bf16 out.

The plain forms are elementary torch operations in 32 bits (64 where a choice between near values is made); an e4m3 value
is v * 448 / max|v| over the block, rounded to nearest even, its scale max|v| / 448.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

E4M3 = torch.float8_e4m3fn
TOP = 448.0          # the largest e4m3 value
BLOCK = 128

# model shapes: layers, routed experts, top-k, shared experts, hidden, intermediate, virtual devices, routing skew
DECODE = dict(L=8, E=60, K=4, S=4, H=2048, I=1408, D=8, zipf=1.2)
FINE = dict(L=16, E=64, K=6, S=2, H=2048, I=1408, D=8, zipf=0.8)
LARGE = dict(L=4, E=8, K=2, S=0, H=4096, I=14336, D=8, zipf=1.0)
ODD = dict(L=5, E=31, K=3, S=1, H=1008, I=720, D=5, zipf=0.6)
# gating: score function, groups of experts, groups kept, members whose scores make a group's, bias, factor on the weights
SIGMOID = dict(score="sigmoid", groups=1, keep=1, best=1, bias=True, renorm=1, scale=2.5, half=False, masked=0.0)
GROUPED = dict(SIGMOID, groups=8, keep=4, best=2)
SOFTMAX = dict(score="softmax", groups=5, keep=2, best=1, bias=False, renorm=0, scale=1.0, half=True, masked=0.1)


def case(op, shape, N, T, **more):
    """N micro-batches of T tokens each (about T when `ragged`), staggered over the layers unless `same_layer`."""
    c = dict(shape, op=op, N=N, T=T, ragged=False, same_layer=False)
    c.update(more)
    return c


def listed():
    return [
        # gating of one token in each of four micro-batches: interactive decoding
        dict(case("route", FINE, 4, 1, **SIGMOID), name="route_one_token"),
        # requests of unequal length, bf16 logits cut out of a wider tensor, experts masked out, groups of twelve
        dict(case("route", DECODE, 7, 77, ragged=True, **SOFTMAX), name="route_softmax_ragged"),
        # prefill over many experts in eight groups: the largest gating
        dict(case("route", dict(FINE, E=256, K=8), 16, 4096, **GROUPED), name="route_wide"),
        # batched decoding of a model with shared experts
        dict(case("dispatch", DECODE, 8, 32), name="dispatch_decode"),
        # sizes that are multiples of 16 and of nothing larger, devices with unequal numbers of experts
        dict(case("dispatch", ODD, 5, 93, ragged=True), name="dispatch_odd"),
        # fine-grained experts, prefill: every row goes to eight places
        dict(case("dispatch", FINE, 16, 512), name="dispatch_fine"),
        # conversion of a few matrices whose sizes are no multiples of the block
        dict(case("weights", ODD, 1, 1, n_mat=7), name="weights_odd"),
        # conversion of one kind of matrix of two layers
        dict(case("weights", FINE, 1, 1, n_mat=132), name="weights_fine"),
        # interactive decoding: one token in each of four micro-batches, every matrix for a row or two
        dict(case("experts", DECODE, 4, 1), name="experts_one_token"),
        # batched decoding: weights are streamed for a handful of rows each
        dict(case("experts", DECODE, 8, 32), name="experts_decode"),
        # all micro-batches at one layer (prefill): several hundred rows per expert
        dict(case("experts", FINE, 16, 512, L=1, same_layer=True), name="experts_prefill"),
        # large experts, prompts of a thousand tokens: the largest case
        dict(case("experts", LARGE, 4, 1024), name="experts_large"),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "dispatch", "weights", "experts", "experts"])
    more = dict(ragged=rng.random() < 0.5, same_layer=rng.random() < 0.3, zipf=round(rng.uniform(0.0, 1.5), 2))
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8, 16])
        per = rng.randint(1, 256 // groups) if groups > 1 else rng.randint(8, 256)
        keep = rng.randint(1, groups)
        more.update(E=groups * per, K=min(rng.randint(1, 8), per * keep), groups=groups, keep=keep, best=rng.choice([1, 2]),
                    score=rng.choice(["sigmoid", "softmax"]), bias=rng.random() < 0.6, renorm=rng.choice([1, 1, 0]),
                    scale=rng.choice([1.0, 2.5]), half=rng.random() < 0.4, masked=rng.choice([0.0, 0.0, 0.2]))
        more["D"] = rng.randint(1, 8)
        return case(op, FINE, rng.randint(1, 16), log_int(rng, 1, 3000), **more)
    if op == "weights":
        more.update(H=8 * rng.randint(4, 500), I=8 * rng.randint(4, 250), n_mat=rng.randint(1, 60))
        return case(op, FINE, 1, 1, **more)
    shape = rng.choice([DECODE, FINE, ODD, ODD, LARGE] if op == "experts" else [DECODE, FINE, ODD, LARGE])
    if shape is LARGE:
        return case(op, shape, rng.randint(1, 4), log_int(rng, 1, 900), **more)
    if shape is ODD:
        more.update(E=rng.randint(9, 47), K=rng.randint(1, 6), S=rng.randint(0, 3), D=rng.randint(2, 8),
                    H=16 * rng.randint(8, 125), I=16 * rng.randint(8, 90))
    return case(op, shape, rng.randint(1, 8), log_int(rng, 1, 600), **more)


# ---- what a case stands for ---------------------------------------------------------------------
def tokens_of(c):
    """Tokens of every micro-batch: T each, or spread from about T/2 to 3T/2."""
    n, t = c["N"], c["T"]
    return [max(1, t // 2 + ((5 * j + 3) % n) * t // n) for j in range(n)] if c["ragged"] else [t] * n


def layers_of(c):
    return [0] * c["N"] if c["same_layer"] else [j * c["L"] // c["N"] for j in range(c["N"])]


def device_of_expert(c):
    return [e * c["D"] // c["E"] for e in range(c["E"])]


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def skewed_logits(c, gen):
    """N(0, 1) plus a popularity of the experts that is another one at every layer."""
    tokens, layers = tokens_of(c), layers_of(c)
    rank = torch.rand((c["L"], c["E"]), generator=gen, device="cuda").argsort(1).float()
    mb = torch.repeat_interleave(torch.arange(c["N"], device="cuda"), torch.tensor(tokens, device="cuda"))
    layer = torch.tensor(layers, device="cuda")[mb]
    z = torch.randn((sum(tokens), c["E"]), generator=gen, device="cuda") - c["zipf"] * torch.log1p(rank)[layer]
    return z, mb, layer


def group_plan(c, mb, layer):
    """Numbers of the groups of a step in which every micro-batch runs: device by device, there layer by layer, the device's
    routed experts and then the shared ones.  (group of every (token, expert), of every (token, shared expert), matrix of every
    group, groups before every device, active layers)"""
    E, S, D = c["E"], c["S"], c["D"]
    act = sorted(set(layers_of(c)))
    e2d = device_of_expert(c)
    number, matrix, first = {}, [], []
    for d in range(D):
        first.append(len(matrix))
        for l in act:
            for e in [e for e in range(E) if e2d[e] == d] + [E + s for s in range(S)]:
                number[d, l, e] = len(matrix)
                matrix.append(l * (E + S) + e)
    routed = torch.zeros((c["L"], E), dtype=torch.int64)
    shared = torch.zeros((c["L"], D, max(S, 1)), dtype=torch.int64)
    for (d, l, e), g in number.items():
        if e < E:
            routed[l, e] = g
        else:
            shared[l, d, e - E] = g
    tokens = torch.tensor(tokens_of(c), device="cuda")
    start = torch.cumsum(tokens, 0) - tokens
    at = torch.arange(len(mb), device="cuda") - start[mb]
    home = at * D // tokens[mb]
    return routed.cuda()[layer], shared.cuda()[layer, home, :S], torch.tensor(matrix, dtype=torch.int32, device="cuda"), first + [len(matrix)], len(act)


def make_step(c, B, **more):
    return B.MoEStep(c["L"], c["E"], c["K"], c["S"], c["H"], c["I"], c["D"], device_of_expert(c), sum(tokens_of(c)), **more)


def make_batch(c, B):
    return B.Batch([0] + np.cumsum(tokens_of(c)).tolist(), layers_of(c))


def prepare(c, seed):
    gen = generator(seed)
    s = dict(c=c)
    if c["op"] == "weights":
        s["w"] = torch.empty((c["n_mat"], c["I"], c["H"]), dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02, generator=gen)
        if own:
            from paper_2608_07964_b200 import binding as B
            s["step"] = B.MoEStep(1, 1, 1, 0, 64, 64, 1, [0], 1)
        return s
    logits, mb, layer = skewed_logits(c, gen)
    T = len(mb)
    if c["op"] == "route":
        if c["masked"]:
            logits = logits.masked_fill(torch.rand(logits.shape, generator=gen, device="cuda") < c["masked"], -math.inf)
            logits[T // 3] = -math.inf       # a token with nothing to choose from
        s["bias"] = 0.2 * torch.randn((c["L"], c["E"]), generator=gen, device="cuda") if c["bias"] else None
        if c["half"]:
            wide = torch.zeros((T, c["E"] + 4), dtype=torch.bfloat16, device="cuda")
            wide[:, :c["E"]] = logits
            logits = wide[:, :c["E"]]
        s.update(logits=logits, mb=mb, layer=layer, device=torch.tensor(device_of_expert(c), device="cuda"))
        if own:
            from paper_2608_07964_b200 import binding as B
            s["step"], s["batch"] = make_step(dict(c, H=64, I=64, S=0), B, renorm_topk=c["renorm"]), make_batch(c, B)
            s["router"] = B.Router(score=c["score"], bias=s["bias"], n_group=c["groups"], topk_group=c["keep"], group_top=c["best"], scale=c["scale"])
        return s
    idx = torch.topk(logits, c["K"], dim=1).indices
    routed, shared, matrix, first, n_layers = group_plan(c, mb, layer)
    if c["op"] == "dispatch":
        s.update(x=torch.randn((T, c["H"]), generator=gen, device="cuda").to(torch.bfloat16), idx=idx.to(torch.int32), routed=routed, shared=shared,
                 matrix=matrix, rows=T * (c["K"] + c["S"]))
        if own:
            from paper_2608_07964_b200 import binding as B
            s["step"], s["batch"] = make_step(dict(c, I=16), B, fp8=True), make_batch(c, B)
            s["step"].topk_idx.copy_(s["idx"])
            s["step"].eb_schedule(s["batch"], 1, B.POLICY_ALL)
        return s
    # experts: the rows and tables that a dispatch leaves
    group = torch.cat([routed.gather(1, idx), shared], 1).flatten()
    sizes = torch.bincount(group, minlength=len(matrix))
    off = torch.cat([sizes.new_zeros(1), torch.cumsum(sizes, 0)])
    R, kb, ib = len(group), -(-c["H"] // BLOCK), -(-c["I"] // BLOCK)
    e4m3 = lambda *shape: torch.randn(shape, generator=gen, device="cuda").mul_(104.0).clamp_(-TOP, TOP).to(E4M3)  # noqa: E731
    scale = lambda mean, *shape: torch.rand(shape, generator=gen, device="cuda").mul_(0.4).add_(0.8).mul_(mean)    # noqa: E731
    n, H, I = c["E"] + c["S"], c["H"], c["I"]
    s.update(x=e4m3(R, H), xs=scale(0.007, R, kb), matrix=matrix, off=off.to(torch.int32),
             gate=e4m3(c["L"] * n, I, H), up=e4m3(c["L"] * n, I, H), down=e4m3(c["L"] * n, H, I), gate_s=scale(2e-4, c["L"] * n, ib, kb),
             up_s=scale(2e-4, c["L"] * n, ib, kb), down_s=scale(2e-4, c["L"] * n, kb, ib), rows=R)
    # the plain form's plan: groups that have rows, their rows side by side up to the longest
    live = torch.nonzero(sizes).flatten()
    most = int(sizes.max())
    at = torch.arange(most, device="cuda")
    s["padded"] = torch.where(at < sizes[live, None], off[live, None] + at, R)      # row R is one of zeros
    s["live"] = matrix[live].long()
    s["place"] = torch.nonzero((at < sizes[live, None]).flatten()).flatten()
    if own:
        from paper_2608_07964_b200 import binding as B
        step = s["step"] = make_step(c, B, fp8=True)
        shape = lambda t: t.view(c["L"], n, *t.shape[1:])  # noqa: E731
        step.bind_weights_fp8(shape(s["gate"]), shape(s["gate_s"]), shape(s["up"]), shape(s["up_s"]), shape(s["down"]), shape(s["down_s"]))
        step.group_off[:len(off)].copy_(s["off"])
        step.group_w[:len(matrix)].copy_(matrix)
        step.step_meta[:3 + len(first)].copy_(torch.tensor([R, len(matrix), n_layers] + first))
        step.xq[:R].copy_(s["x"])
        step.xs[:R, :kb].copy_(s["xs"])
    return s


# ---- the plain forms ----------------------------------------------------------------------------
def route_plain(s):
    c, z = s["c"], s["logits"].double()
    T, E, K, G, D = len(z), c["E"], c["K"], c["groups"], c["D"]
    if c["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-z))
    else:
        top = z.amax(1, keepdim=True)
        p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
        score = p / p.sum(1, keepdim=True).clamp_min(1e-300)
    choice = score if s["bias"] is None else score + s["bias"].double()[s["layer"]]
    choice = torch.where(z == -math.inf, -math.inf, choice)
    if G > 1:
        best = choice.view(T, G, E // G).sort(dim=2, descending=True).values[:, :, :c["best"]]
        group = torch.where(best[:, :, 0] == -math.inf, -math.inf, torch.where(best == -math.inf, 0.0, best).sum(2))
        rank = group.sort(dim=1, descending=True, stable=True).indices.argsort(1)
        choice = torch.where((rank < c["keep"]).repeat_interleave(E // G, 1), choice, -math.inf)
    order = choice.sort(dim=1, descending=True, stable=True)
    idx = torch.where(order.values[:, :K] == -math.inf, -1, order.indices[:, :K])
    w = torch.where(idx < 0, 0.0, score.gather(1, idx.clamp_min(0)))
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    hit = torch.where(idx < 0, c["N"] * E, s["mb"][:, None] * E + idx).flatten()
    cnt = torch.bincount(hit, minlength=c["N"] * E + 1)[:-1].view(c["N"], E)
    load = torch.zeros((c["N"], D), dtype=cnt.dtype, device="cuda").index_add_(1, s["device"], cnt)
    return dict(idx=idx.to(torch.int32), w=(w * c["scale"]).float(), load=load.to(torch.int32), count=cnt.to(torch.int32))


def blocks_of(x):
    """The last axis in blocks of 128, the last of them filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % BLOCK)).unflatten(-1, (-1, BLOCK))


def quantise_rows(x):
    b = blocks_of(x)
    most = b.abs().amax(-1, keepdim=True)
    q = torch.where(most > 0, b * TOP / most, 0.0).to(E4M3)
    return q.flatten(-2)[..., :x.shape[-1]], (most / TOP).squeeze(-1)


def dispatch_plain(s):
    c = s["c"]
    group = torch.cat([s["routed"].gather(1, s["idx"].long()), s["shared"]], 1)
    slots = group.shape[1]
    order = group.flatten().argsort(stable=True)
    pos = torch.empty_like(order)
    pos[order] = torch.arange(len(order), device="cuda")
    off = torch.cumsum(torch.nn.functional.pad(torch.bincount(group.flatten(), minlength=len(s["matrix"])), (1, 0)), 0)
    src = order // slots
    q, scale = quantise_rows(s["x"].float())
    return dict(off=off.to(torch.int32), matrix=s["matrix"], src=src.to(torch.int32), pos=pos.view(-1, slots).to(torch.int32),
                q=q.view(torch.uint8)[src].view(E4M3), scale=scale[src])


def weights_plain(s):
    w = s["w"].float()
    n, N, K = w.shape
    b = torch.nn.functional.pad(w, (0, -K % BLOCK, 0, -N % BLOCK)).view(n, -(-N // BLOCK), BLOCK, -(-K // BLOCK), BLOCK)
    most = b.abs().amax((2, 4), keepdim=True)
    q = torch.where(most > 0, b * TOP / most, 0.0).to(E4M3).view(n, -(-N // BLOCK) * BLOCK, -1)[:, :N, :K]
    return dict(q=q, scale=(most / TOP).view(n, -(-N // BLOCK), -1))


def unscaled(q, scale):
    """Values of e4m3 matrices [n, rows, columns] with a scale for each 128 x 128 block."""
    s = scale.repeat_interleave(BLOCK, 1)[:, :q.shape[1]].repeat_interleave(BLOCK, 2)[:, :, :q.shape[2]]
    return q.float() * s


def experts_plain(s):
    live = s["live"]
    take = lambda q: q.view(torch.uint8)[live].view(E4M3)  # noqa: E731
    x = torch.nn.functional.pad((blocks_of(s["x"].float()) * s["xs"][..., None]).flatten(-2)[:, :s["x"].shape[1]], (0, 0, 0, 1))[s["padded"]]
    g = x @ unscaled(take(s["gate"]), s["gate_s"][live]).transpose(1, 2)
    u = x @ unscaled(take(s["up"]), s["up_s"][live]).transpose(1, 2)
    q, scale = quantise_rows(g / (1.0 + torch.exp(-g)) * u)
    h = (blocks_of(q.float()) * scale[..., None]).flatten(-2)[..., :q.shape[-1]]
    y = h @ unscaled(take(s["down"]), s["down_s"][live]).transpose(1, 2)
    return dict(y=y.flatten(0, 1)[s["place"]].to(torch.bfloat16))


def run(s):
    c = s["c"]
    if not own:
        return {"route": route_plain, "dispatch": dispatch_plain, "weights": weights_plain, "experts": experts_plain}[c["op"]](s)
    step = s["step"]
    if c["op"] == "route":
        step.eb_route_scored(s["batch"], s["router"], s["logits"])
        N = c["N"]
        return dict(idx=step.topk_idx, w=step.topk_w, load=step.mb_load[:N], count=step.mb_cnt[:N])
    if c["op"] == "dispatch":
        step.eb_permute_fp8(s["batch"], s["x"])
        R, G = s["rows"], len(s["matrix"])
        return dict(off=step.group_off[:G + 1], matrix=step.group_w[:G], src=step.row_src[:R], pos=step.pos, q=step.xq[:R],
                    scale=step.xs[:R, :-(-c["H"] // BLOCK)])
    if c["op"] == "weights":
        q, scale = step.quantize_weights(s["w"])
        return dict(q=q, scale=scale)
    step.eb_expert_ffn_grouped_fp8()
    return dict(y=step.yp[:s["rows"]])


# ---- the work, and the exact values -------------------------------------------------------------
def work(c):
    T, H, I = sum(tokens_of(c)), c["H"], c["I"]
    kb, ib = -(-H // BLOCK), -(-I // BLOCK)
    if c["op"] == "weights":
        return dict(bytes=c["n_mat"] * (3 * H * I + 4 * kb * ib), flops=2 * c["n_mat"] * H * I)
    if c["op"] == "route":
        # scores and choice: about ten operations a logit
        return dict(bytes=T * (c["E"] * (2 if c["half"] else 4) + 8 * c["K"]) + 4 * c["N"] * (c["E"] + c["D"]), flops=10 * T * c["E"])
    slots = c["K"] + c["S"]
    if c["op"] == "dispatch":
        return dict(bytes=2 * T * H + 4 * T * c["K"] + T * slots * (H + 4 * kb + 8), flops=3 * T * H)
    # matrices that have rows: those that T tokens of a layer choose, under the case's popularity, and the shared ones
    used = 0.0
    tokens, layers = tokens_of(c), layers_of(c)
    p = np.arange(1, c["E"] + 1, dtype=float) ** -c["zipf"]
    p /= p.sum()
    for l in set(layers):
        t = sum(n for n, k in zip(tokens, layers) if k == l)
        used += (1 - (1 - p) ** (t * c["K"])).sum() + c["S"]
    return dict(bytes=used * (3 * H * I + 12 * kb * ib) + T * slots * (3 * H + 4 * kb), flops=6.0 * T * slots * H * I)


def nearest_e4m3(v):
    """64-bit values to the nearest e4m3 value, ties to even: three bits behind the leading one, the smallest normal 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def exact(c, seed):
    s = prepare_inputs(c, seed)
    if c["op"] == "route":
        return exact_route(c, s)
    if c["op"] == "weights":
        w = s["w"].double()
        n, N, K = w.shape
        q, scale = torch.empty(w.shape, dtype=torch.float64, device="cuda"), torch.empty((n, -(-N // BLOCK), -(-K // BLOCK)), dtype=torch.float64, device="cuda")
        for i in range(0, N, BLOCK):
            for k in range(0, K, BLOCK):
                b = w[:, i:i + BLOCK, k:k + BLOCK]
                most = b.abs().amax((1, 2))
                q[:, i:i + BLOCK, k:k + BLOCK] = nearest_e4m3(b * TOP / most[:, None, None])
                scale[:, i // BLOCK, k // BLOCK] = most / TOP
        return dict(q=q, scale=scale)
    if c["op"] == "dispatch":
        src = dispatch_plain(s)["src"].long()
        x = s["x"].double()
        q, scale = torch.empty_like(x), []
        for k in range(0, c["H"], BLOCK):
            most = x[:, k:k + BLOCK].abs().amax(1)
            q[:, k:k + BLOCK] = nearest_e4m3(x[:, k:k + BLOCK] * TOP / most[:, None])
            scale.append(most / TOP)
        return dict(off=None, matrix=None, src=None, pos=None, q=q[src], scale=torch.stack(scale, 1)[src])
    return exact_experts(c, s)


def prepare_inputs(c, seed):
    global own
    kept, own = own, False
    try:
        return prepare(c, seed)
    finally:
        own = kept


def exact_route(c, s):
    z = s["logits"].double().cpu().numpy().astype(np.longdouble)
    T, E, K, G = len(z), c["E"], c["K"], c["groups"]
    dead = np.isneginf(z)
    if c["score"] == "sigmoid":
        score = 1 / (1 + np.exp(-z))
    else:
        p = np.exp(z - np.where(dead, -1e30, z).max(1, keepdims=True))
        score = np.where(dead, 0, p / np.maximum(p.sum(1, keepdims=True), 1e-300))
    choice = score if s["bias"] is None else score + s["bias"].double().cpu().numpy()[s["layer"].cpu().numpy()]
    choice = np.where(dead, -np.inf, choice)
    if G > 1:
        top = np.sort(choice.reshape(T, G, E // G), 2)[:, :, ::-1][:, :, :c["best"]]
        value = np.where(np.isneginf(top[:, :, 0]), -np.inf, np.where(np.isneginf(top), 0, top).sum(2))
        keep = np.argsort(-value, 1, kind="stable")[:, :c["keep"]]
        open_ = np.zeros((T, G), bool)
        np.put_along_axis(open_, keep, True, 1)
        choice = np.where(np.repeat(open_, E // G, 1), choice, -np.inf)
    idx = np.argsort(-choice, 1, kind="stable")[:, :K]
    ok = ~np.isneginf(np.take_along_axis(choice, idx, 1))
    w = np.where(ok, np.take_along_axis(score, idx, 1), 0)
    if c["renorm"]:
        w = w / np.maximum(w.sum(1, keepdims=True), 1e-300)
    return dict(idx=None, w=(w * c["scale"]).astype(np.float64), load=None, count=None)


def exact_experts(c, s):
    ones = torch.ones((BLOCK, BLOCK), dtype=torch.float64, device="cuda")

    def values(q, scale):
        return q.double() * torch.kron(scale.double(), ones)[:q.shape[0], :q.shape[1]]

    off, matrix = s["off"].tolist(), s["matrix"].tolist()
    y = torch.empty((s["rows"], c["H"]), dtype=torch.float64, device="cuda")
    for g, m in enumerate(matrix):
        a, b = off[g], off[g + 1]
        if a == b:
            continue
        x = s["x"][a:b].double()
        for k in range(0, c["H"], BLOCK):
            x[:, k:k + BLOCK] *= s["xs"][a:b, k // BLOCK, None].double()
        gate, up = x @ values(s["gate"][m], s["gate_s"][m]).T, x @ values(s["up"][m], s["up_s"][m]).T
        h = gate * torch.sigmoid(gate) * up
        for i in range(0, c["I"], BLOCK):
            most = h[:, i:i + BLOCK].abs().amax(1, keepdim=True)
            h[:, i:i + BLOCK] = nearest_e4m3(h[:, i:i + BLOCK] * (TOP / most)) * (most / TOP)
        y[a:b] = h @ values(s["down"][m], s["down_s"][m]).T
    return dict(y=y)
