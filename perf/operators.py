"""What is measured of block-sparse attention and of clipped updates: the calls that a program makes of them, over the sizes it makes them at.

A case is a dict of plain values:

    kind    "choose"  block means of the keys and the choice of key blocks for every tile of queries (once a layer)
            "attend"  softmax attention over chosen blocks (inference)
            "train"   the same with its row statistics, and the gradients of q, k and v
            "decode"  one serving step: the newest block's mean, the choice and the attention of a few new tokens over a long cache
            "clip"    global norm of many gradients and the clipped gradients
            "update"  global norm, then the clipped AdamW pass over all parameters
    B, H, Hkv, Nq, Nk, d, dtype     the problem: query head h reads key head h / (H / Hkv)
    qb, kb, sel                     queries that share a choice, keys of a block, blocks chosen per tile
    causal, first, near             the mask; leading blocks that every tile takes; tokens around a tile's own that it takes (-1: none)
    ragged                          batch entries hold different numbers of keys
    layout                          "bhnd" contiguous [B, H, N, d], or "bnhd": views of [B, N, H, d] memory, as a projection leaves them
    layers, hid, feat, mid, gtype   the optimiser's cases: layers of feature maps d -> hid [-> mid] -> feat, type of the gradients

Neighbouring tokens resemble each other (a clip's do): q and k are a drift over some tens of tokens plus noise, at unit scale.
"""
import math

import torch

own = False

ADAMW = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=0.5)
ADAMW_STEP = 100


def _case(name, kind, B=1, H=12, Hkv=0, Nq=32760, Nk=0, d=128, dtype="bf16", qb=128, kb=64, sel=64, causal=False, first=0, near=-1, ragged=False, layout="bhnd"):
    return dict(name=name, kind=kind, B=B, H=H, Hkv=Hkv or H, Nq=Nq, Nk=Nk or Nq, d=d, dtype=dtype, qb=qb, kb=kb, sel=sel, causal=causal, first=first,
                near=near, ragged=ragged, layout=layout)


def _params(name, kind, layers=1, H=12, d=128, hid=128, feat=128, mid=0, dtype="bf16", gtype="f32"):
    return dict(name=name, kind=kind, layers=layers, H=H, d=d, hid=hid, feat=feat, mid=mid, dtype=dtype, gtype=gtype)


def listed():
    return [
        # The smallest clip in use: two narrow fp32 heads of a 4 x 16 x 16 grid; launches and latency count.
        _case("choose_1k_f32_d64", "choose", H=2, Nq=1024, d=64, dtype="f32", qb=64, sel=4),
        # One layer at 81 x 480 x 832: an eighth of the keys for every tile.
        _case("choose_480p", "choose", first=1, near=64),
        # One layer at 81 x 720 x 1280 with classifier-free guidance.
        _case("choose_720p_cfg", "choose", B=2, Nq=75600, kb=128, sel=48),
        # One latent frame of 30 x 52 tokens: few tiles of queries.
        _case("attend_frame", "attend", Nq=1560, sel=8),
        # fp32 activations of an odd length in projection layout, two clips of different lengths: a user's debugging run.
        _case("attend_odd_f32_strided", "attend", B=2, Nq=5003, dtype="f32", qb=64, sel=16, near=0, ragged=True, layout="bnhd"),
        # One layer at 81 x 480 x 832, inference.
        _case("attend_480p", "attend", first=1, near=64),
        # The same layer in fine-tuning: forward and gradients.
        _case("train_480p", "train", first=1, near=64),
        # A causal layer with three query heads to a key head, in projection layout, a padded batch.
        _case("train_causal_grouped", "train", B=2, H=12, Hkv=4, Nq=4096, d=64, qb=64, sel=12, causal=True, first=1, near=0, ragged=True, layout="bnhd"),
        # One new token for each of four sequences over caches of up to 60 thousand keys.
        _case("decode_60k", "decode", B=4, H=12, Hkv=4, Nq=1, Nk=60000, sel=32, causal=True, first=1, near=64, ragged=True),
        # Gradients of one layer's maps of the default widths (2.4 M values in eight tensors), bf16 as a reduction leaves them.
        _params("clip_phi256_bf16", "clip", hid=256, feat=256, gtype="bf16"),
        # The smallest maps in use, updated with clipping.
        _params("update_d64_f32", "update", H=2, d=64, hid=64, feat=64, dtype="f32"),
        # The maps of all thirty layers (71 M values in 240 tensors), updated with clipping.
        _params("update_phi256_30layers", "update", layers=30, hid=256, feat=256),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no larger than the largest listed one."""
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(("choose", "attend", "attend", "train", "train", "decode", "clip", "update"))
        if kind in ("clip", "update"):
            d = rng.choice((64, 128, 128))
            hid = rng.choice((64, 128, 256, 384, 768)) if d == 128 else 64
            c = _params("", kind, layers=rng.choice((1, 1, 2, 3, 7, 15)), H=rng.choice((1, 2, 5, 12)), d=d, hid=hid, feat=rng.choice((64, 128, 256, 768)) if d == 128 else 64,
                        mid=rng.choice((0, 0, 0, 384)) if d == 128 else 0, dtype=rng.choice(("bf16", "f32")), gtype=rng.choice(("f32", "f32", "bf16")))
        else:
            Hkv = rng.choice((1, 2, 3, 4, 5, 12))
            c = _case("", kind, B=rng.choice((1, 1, 2, 3)), Hkv=Hkv, H=Hkv * rng.choice((1, 1, 1, 2, 3, 8)), d=rng.choice((64, 128, 128)), dtype=rng.choice(("bf16", "bf16", "bf16", "f32")),
                      qb=rng.choice((64, 128)), kb=rng.choice((64, 128)), causal=rng.random() < 0.4, first=rng.choice((0, 0, 1)), ragged=rng.random() < 0.4,
                      layout=rng.choice(("bhnd", "bnhd")))
            c["Nk"] = c["Nq"] = _log_uniform(rng, 200, 75600 if kind in ("choose", "decode") else 32760)
            if kind == "decode":
                c.update(Nq=rng.choice((1, 1, 1, 2, 5)), causal=True)
            blocks = -(-c["Nk"] // c["kb"])
            c["near"] = rng.choice((0, 0, 64)) if c["causal"] else rng.choice((-1, -1, 0, 64))
            span = min(c["qb"], c["Nq"]) + max(0, c["near"]) * (1 if c["causal"] else 2)
            least = c["first"] + (-(-(span - 1) // c["kb"]) + 1 if c["near"] >= 0 else 0)
            c["sel"] = min(blocks, max(least, 1, _log_uniform(rng, 2, 64)))
        c.pop("name")
        if _cost(c) <= most and (kind not in ("attend", "train") or _gathered(c) <= 4 << 30):
            return c


def _tiles(c):
    return -(-c["Nq"] // c["qb"])


def _blocks(c):
    return -(-c["Nk"] // c["kb"])


def _gathered(c):
    """Elements of the logits of all tiles, or of their keys, whichever are more."""
    keys = c["sel"] * c["kb"]
    return c["B"] * _tiles(c) * keys * max(c["H"] * c["qb"], c["Hkv"] * c["d"])


def _cost(c):
    return work(c)["flops"] + 300.0 * work(c)["bytes"]


def _param_shapes(c):
    H, last = c["H"], c["mid"] or c["hid"]
    one = [("w1", (H, c["hid"], c["d"])), ("b1", (H, c["hid"])), ("w2", (H, c["feat"], last)), ("b2", (H, c["feat"]))]
    if c["mid"]:
        one += [("w_mid", (H, c["mid"], c["hid"])), ("b_mid", (H, c["mid"]))]
    return [s for _ in range(c["layers"]) for _ in range(2) for s in one]


def work(case):
    """Bytes and operations that a pass cannot do without: inputs read once, outputs written once, the method's own products."""
    c = case
    if c["kind"] in ("clip", "update"):
        n = sum(math.prod(s) for _, s in _param_shapes(c))
        weights = sum(math.prod(s) for name, s in _param_shapes(c) if name.startswith("w"))
        g, io = 4 if c["gtype"] == "f32" else 2, 4 if c["dtype"] == "f32" else 2
        if c["kind"] == "clip":
            return {"bytes": 2.0 * g * n, "flops": 3.0 * n}
        return {"bytes": (24.0 + g) * n + io * weights, "flops": 18.0 * n}
    io, d = 2 if c["dtype"] == "bf16" else 4, c["d"]
    q, kv = c["B"] * c["H"] * c["Nq"] * d, c["B"] * c["Hkv"] * c["Nk"] * d
    means, chosen = 4.0 * c["B"] * c["Hkv"] * _blocks(c) * d, 4.0 * c["B"] * c["Hkv"] * _tiles(c) * c["sel"]
    scores = 2.0 * c["B"] * c["Hkv"] * _tiles(c) * _blocks(c) * d
    if c["kind"] == "choose":
        return {"bytes": io * (q + kv) + means + chosen, "flops": q + kv + scores}
    # keys that a query sees: all of its tile's blocks, and of a block on the diagonal about a half
    share = 1.0 if c["ragged"] is False else 0.75
    seen = min(c["sel"] * c["kb"], c["Nk"]) * share
    if c["causal"] and c["kind"] != "decode":
        seen = min(seen, c["Nk"] * share / 2)
    pairs = c["B"] * c["H"] * c["Nq"] * seen
    if c["kind"] == "decode":
        return {"bytes": io * (2.0 * q + 2.0 * c["B"] * c["Hkv"] * d * (seen + c["kb"])) + means + chosen, "flops": 4.0 * d * pairs + scores}
    if c["kind"] == "attend":
        return {"bytes": io * (2.0 * q + 2.0 * kv) + chosen, "flops": 4.0 * d * pairs}
    # q, k, v and the output's gradient in; the output, its statistics and three gradients out
    return {"bytes": io * (4.0 * q + 4.0 * kv) + 4.0 * q / d + chosen, "flops": 14.0 * d * pairs}


# ---- inputs ----------------------------------------------------------------------------------------------------------------------

def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _lengths(c, gen):
    """Keys held by each batch entry, on the GPU: all of them, or between half and all."""
    if not c["ragged"]:
        return None
    share = torch.rand(c["B"], generator=gen, device="cuda") * 0.5 + 0.5
    return torch.clamp((share * c["Nk"]).to(torch.int32), min=max(1, c["Nq"] if c["kind"] == "decode" else 1))


def _tokens(c, heads, n, gen, drift):
    shape = (c["B"], heads, n, c["d"]) if c["layout"] == "bhnd" else (c["B"], n, heads, c["d"])
    x = torch.empty(shape, dtype=_dtype(c["dtype"]), device="cuda")
    at = torch.arange(n, device="cuda") // 48
    for part in x:                              # a batch entry at a time
        noise = torch.randn(part.shape, generator=gen, device="cuda")
        if drift:
            slow = torch.randn((heads, n // 48 + 1, c["d"]), generator=gen, device="cuda")[:, at]
            noise = (noise + (slow if c["layout"] == "bhnd" else slow.transpose(0, 1))) * 0.5 ** 0.5
        part.copy_(noise)
    return x if c["layout"] == "bhnd" else x.transpose(1, 2)


def _inputs(c, seed):
    """q, k, v, the numbers of keys, the first query's positions and the output's gradient, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v = _tokens(c, c["H"], c["Nq"], gen, True), _tokens(c, c["Hkv"], c["Nk"], gen, True), _tokens(c, c["Hkv"], c["Nk"], gen, False)
    dout = _tokens(c, c["H"], c["Nq"], gen, False) if c["kind"] == "train" else None
    length = _lengths(c, gen)
    start = None
    if c["kind"] == "decode":                   # the new tokens are the last ones of their sequences
        start = (length if length is not None else torch.full((c["B"],), c["Nk"], dtype=torch.int32, device="cuda")) - c["Nq"]
    return q, k, v, length, start, dout


def _gradients(c, seed):
    """The layers' gradients, moments and weights in flat buffers, one view for each tensor, as they stand some steps into a run."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    shapes = _param_shapes(c)
    sizes = [math.prod(s) for _, s in shapes]
    n, weights = sum(sizes), sum(k for k, (name, _) in zip(sizes, shapes) if name.startswith("w"))

    def normal(std):
        return torch.randn(n, generator=gen, device="cuda") * std
    grad = (normal(1e-2) * torch.exp(normal(1.0))).to(_dtype(c["gtype"]))
    flat = dict(grad=grad)
    if c["kind"] == "update":
        flat.update(master=normal(0.1), m=grad.float() * 0.3 + normal(3e-3), v=(torch.rand(n, generator=gen, device="cuda") + 0.01) * 1e-4,
                    io=torch.zeros(weights, dtype=_dtype(c["dtype"]), device="cuda"))
    else:
        flat.update(out=torch.zeros_like(grad))
    views, at, at_io = [], 0, 0
    for (name, shape), k in zip(shapes, sizes):
        t = {f: flat[f][at:at + k].view(shape) for f in flat if f != "io"}
        if c["kind"] == "update":
            t["io"] = flat["io"][at_io:at_io + k].view(shape) if name.startswith("w") else None
            at_io += k if name.startswith("w") else 0
        views.append(t)
        at += k
    return flat, views


def _max_norm(c):
    """A limit that most steps exceed, as in a run's first part."""
    return 0.02 * math.sqrt(sum(math.prod(s) for _, s in _param_shapes(c)))


def prepare(case, seed):
    c = case
    if c["kind"] in ("clip", "update"):
        flat, views = _gradients(c, seed)
        state = dict(case=c, flat=flat, views=views, step=ADAMW_STEP, max_norm=_max_norm(c))
        if own:                                 # the lists of tensors that a program keeps over its steps
            from paper_2509_24899_amd import hybrid_attn as ha
            grads = [t["grad"] for t in views]
            state["grads"] = ha.TensorList(grads)
            if c["kind"] == "clip":
                state["outs"] = ha.TensorList([t["out"] for t in views])
            else:
                state["params"] = ha.ParamList([t["master"] for t in views], grads, [t["m"] for t in views], [t["v"] for t in views], [t["io"] for t in views])
        return state
    q, k, v, length, start, dout = _inputs(c, seed)
    state = dict(case=c, q=q, k=k, v=v, length=length, start=start)
    if c["kind"] in ("attend", "train"):
        state.update(blocks=_choice(c, q, _means(c, k, length), length, start), dout=dout)
    if c["kind"] == "decode":
        state.update(means=_means(c, k, length))
    return state


# ---- plain forms -----------------------------------------------------------------------------------------------------------------

def _held(c, length):
    """Keys held by each batch entry, [B, 1, 1]."""
    full = torch.full((c["B"],), c["Nk"], dtype=torch.int64, device="cuda") if length is None else length.long()
    return full[:, None, None]


def _first_position(c, start):
    return torch.full((c["B"],), c["Nk"] - c["Nq"], dtype=torch.int64, device="cuda") if start is None else start.long()


def _means(c, k, length):
    """Mean of the held keys of every block, [B, Hkv, blocks, d]; zero where a block holds none."""
    pos = torch.arange(_blocks(c) * c["kb"], device="cuda")
    there = pos < _held(c, length)[:, :, 0].view(-1, 1)
    kd = torch.nn.functional.pad(k.double(), (0, 0, 0, len(pos) - c["Nk"]))
    kd = torch.where(there[:, None, :, None], kd, 0.0).view(c["B"], c["Hkv"], _blocks(c), c["kb"], c["d"]).sum(3)
    return (kd / there.view(c["B"], 1, -1, c["kb"], 1).sum(3).clamp(min=1)).float()


def _last_means(c, k, length, means):
    """The mean of each batch entry's last block, written to its place in `means`."""
    held = _held(c, length).view(-1)
    block, entry = (held - 1) // c["kb"], torch.arange(c["B"], device="cuda")
    pos = block[:, None] * c["kb"] + torch.arange(c["kb"], device="cuda")
    there = pos < held[:, None]
    rows = k.transpose(1, 2)[entry[:, None], pos.clamp(max=c["Nk"] - 1)].double()
    mean = torch.where(there[..., None, None], rows, 0.0).sum(1) / there.sum(1)[:, None, None]
    means[entry, :, block] = mean.float()
    return means


def _choice(c, q, means, length, start):
    """The `sel` blocks with the highest scores of every tile in rising order, -1 behind the last."""
    B, Hkv, T, Tk, qb, kb = c["B"], c["Hkv"], _tiles(c), _blocks(c), c["qb"], c["kb"]
    rows = torch.nn.functional.pad(q.double(), (0, 0, 0, T * qb - c["Nq"])).view(B, Hkv, -1, T, qb, c["d"]).sum((2, 4))
    score = torch.matmul(rows, means.double().transpose(2, 3).contiguous())
    tile, block = torch.arange(T, device="cuda"), torch.arange(Tk, device="cuda")
    lo = _first_position(c, start)[:, None] + tile * qb                                             # positions of a tile's first and last query
    hi = (lo + qb - 1).minimum(_first_position(c, start)[:, None] + c["Nq"] - 1)
    seen = (block * kb < _held(c, length)).expand(B, T, Tk)
    if c["causal"]:
        seen = seen & (block * kb <= hi[..., None])
    forced = (block < c["first"]).expand(B, T, Tk)
    if c["near"] >= 0:
        forced = forced | ((block * kb + kb - 1 >= lo[..., None] - c["near"]) & (block * kb <= hi[..., None] + (0 if c["causal"] else c["near"])))
    score = torch.where(forced[:, None], math.inf, score)
    score = torch.where(seen[:, None], score, -math.inf)
    best, at = torch.sort(score, dim=3, descending=True, stable=True)
    at = torch.where(best[..., :c["sel"]] > -math.inf, at[..., :c["sel"]], Tk).sort(dim=3).values
    return torch.where(at < Tk, at, -1).to(torch.int32)


class _Chosen:
    """Every tile's keys and values side by side, the pairs that see each other, and the logits, in 32 bits."""

    def __init__(self, c, q, k, v, blocks, length, start):
        B, Hkv, T, qb, kb = c["B"], c["Hkv"], _tiles(c), c["qb"], c["kb"]
        self.c, self.shape = c, (B, Hkv, T, -1, c["d"])
        pos = (blocks.long()[..., None] * kb + torch.arange(kb, device="cuda")).flatten(3)           # [B, Hkv, T, keys]
        there = (blocks >= 0).repeat_interleave(kb, dim=3) & (pos < _held(c, length)[..., None])
        head = torch.arange(B * Hkv, device="cuda").view(B, Hkv, 1, 1)
        self.at = torch.where(there, pos, 0) + head * c["Nk"]
        seen = there[:, :, :, None, None]                                                            # [B, Hkv, T, group, qb, keys]
        if c["causal"]:
            row = (_first_position(c, start)[:, None] + torch.arange(T * qb, device="cuda")).view(B, 1, T, 1, qb, 1)
            seen = seen & (pos[:, :, :, None, None] <= row)
        self.k, self.v = (torch.where(there[..., None], x.float().reshape(-1, c["d"])[self.at], 0.0) for x in (k, v))
        self.q = self.tiles(q)
        self.scale = c["d"] ** -0.5
        s = torch.matmul(self.q, self.k.transpose(3, 4)) * self.scale
        self.s = torch.where(seen, s.view(B, Hkv, T, -1, qb, s.shape[-1]), -math.inf).view(s.shape)

    def tiles(self, x):
        """[B, H, Nq, d] as [B, Hkv, T, group * qb, d]."""
        c = self.c
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, _tiles(c) * c["qb"] - c["Nq"]))
        return x.view(c["B"], c["Hkv"], -1, _tiles(c), c["qb"], c["d"]).transpose(2, 3).reshape(self.shape)

    def rows(self, x):
        """The reverse of tiles(), for [B, Hkv, T, group * qb, ...]."""
        c = self.c
        x = x.view(c["B"], c["Hkv"], _tiles(c), -1, c["qb"], *x.shape[4:]).transpose(2, 3)
        return x.reshape(c["B"], c["H"], -1, *x.shape[5:])[:, :, :c["Nq"]]

    def forward(self):
        top = self.s.amax(4, keepdim=True)
        top = torch.where(top > -math.inf, top, 0.0)
        p = torch.exp(self.s - top)
        total = p.sum(4, keepdim=True)
        out = torch.matmul(p, self.v) / torch.where(total > 0, total, 1.0)
        return out, (top + torch.log(total))[..., 0]

    def gradients(self, out, lse, dout):
        c = self.c
        p = torch.exp(self.s - torch.where(lse > -math.inf, lse, 0.0)[..., None])
        do = self.tiles(dout)
        ds = p * (torch.matmul(do, self.v.transpose(3, 4)) - (do * out).sum(4, keepdim=True)) * self.scale
        into = torch.zeros((2, c["B"] * c["Hkv"] * c["Nk"], c["d"]), device="cuda")
        into[0].index_add_(0, self.at.flatten(), torch.matmul(ds.transpose(3, 4), self.q).view(-1, c["d"]))
        into[1].index_add_(0, self.at.flatten(), torch.matmul(p.transpose(3, 4), do).view(-1, c["d"]))
        return self.rows(torch.matmul(ds, self.k)), *into.view(2, c["B"], c["Hkv"], c["Nk"], c["d"])


def _norm(grads, max_norm):
    """(global norm, factor that brings it down to max_norm) in 64 bits."""
    norm = torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()
    return norm, (max_norm / norm).clamp(max=1.0)


def _adamw(t, factor, step):
    o = ADAMW
    g = t["grad"].float() * (o["grad_scale"] * factor)
    t["m"].mul_(o["beta1"]).add_(g, alpha=1 - o["beta1"])
    t["v"].mul_(o["beta2"]).add_((1 - o["beta2"]) * g * g)
    t["master"].mul_(1 - o["lr"] * o["weight_decay"])
    t["master"].sub_(o["lr"] / (1 - o["beta1"] ** step) * t["m"] / (t["v"].sqrt() / math.sqrt(1 - o["beta2"] ** step) + o["eps"]))
    if t["io"] is not None:
        t["io"].copy_(t["master"])


def _run_params(state):
    c = state["case"]
    if own:
        from paper_2509_24899_amd import hybrid_attn as ha
        result = ha.hybrid_attn_grad_norm(state["grads"], state["max_norm"])
        if c["kind"] == "clip":
            ha.hybrid_attn_grad_clip(state["grads"], result, out=state["outs"])
        else:
            ha.hybrid_attn_param_update_many(state["params"], kind=ha.HA_OPT_ADAMW, step=state["step"], clip=result, **ADAMW)
    else:
        norm, factor = _norm([t["grad"] for t in state["views"]], state["max_norm"])
        result = torch.stack([norm, factor]).float()
        if c["kind"] == "clip":
            [t["out"].copy_(t["grad"].float() * result[1]) for t in state["views"]]
        else:
            [_adamw(t, result[1], state["step"]) for t in state["views"]]
    state["step"] += 1
    return dict(result=result, **{f: x for f, x in state["flat"].items() if f != "grad"})


def run(state):
    c = state["case"]
    if c["kind"] in ("clip", "update"):
        return _run_params(state)
    q, k, v, length, start = (state[n] for n in ("q", "k", "v", "length", "start"))
    mask = dict(causal=c["causal"], q_start=start, key_len=length)
    near = dict(keep_first=c["first"], near=c["near"])
    if own:
        from paper_2509_24899_amd import hybrid_attn as ha
    if c["kind"] == "choose":
        if own:
            means = ha.hybrid_attn_key_means(k, c["kb"], key_len=length)
            return dict(means=means, blocks=ha.hybrid_attn_select_blocks(q, means, c["Nk"], c["sel"], c["qb"], c["kb"], **mask, **near))
        means = _means(c, k, length)
        return dict(means=means, blocks=_choice(c, q, means, length, start))
    if c["kind"] == "decode":
        if own:
            means = ha.hybrid_attn_key_means(k, c["kb"], key_len=length, only_last=1, out=state["means"])
            blocks = ha.hybrid_attn_select_blocks(q, means, c["Nk"], c["sel"], c["qb"], c["kb"], **mask, **near)
            return dict(means=means, blocks=blocks, out=ha.hybrid_attn_sparse_forward(q, k, v, blocks, c["qb"], c["kb"], **mask)[0])
        means = _last_means(c, k, length, state["means"])
        blocks = _choice(c, q, means, length, start)
        x = _Chosen(c, q, k, v, blocks, length, start)
        return dict(means=means, blocks=blocks, out=x.rows(x.forward()[0]).to(q.dtype))
    if own:
        out, lse = ha.hybrid_attn_sparse_forward(q, k, v, state["blocks"], c["qb"], c["kb"], **mask, with_lse=c["kind"] == "train")
        if c["kind"] == "attend":
            return out
        dq, dk, dv = ha.hybrid_attn_sparse_grad(q, k, v, state["blocks"], out, lse, state["dout"], c["qb"], c["kb"], **mask)
        return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)
    x = _Chosen(c, q, k, v, state["blocks"], length, start)
    out, lse = x.forward()
    if c["kind"] == "attend":
        return x.rows(out).to(q.dtype)
    dq, dk, dv = x.gradients(out, lse, state["dout"])
    return dict(out=x.rows(out).to(q.dtype), lse=x.rows(lse), dq=dq.to(q.dtype), dk=dk.to(q.dtype), dv=dv.to(q.dtype))


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------------------

def _exact_params(c, seed):
    flat, _ = _gradients(c, seed)
    g = flat["grad"].double()
    norm = g.norm()
    factor = min(1.0, _max_norm(c) / float(norm))
    result = torch.tensor([float(norm), factor], dtype=torch.float64, device="cuda")
    if c["kind"] == "clip":
        return dict(result=result, out=g * factor)
    o, g = ADAMW, g * (ADAMW["grad_scale"] * factor)
    m = o["beta1"] * flat["m"].double() + (1 - o["beta1"]) * g
    v = o["beta2"] * flat["v"].double() + (1 - o["beta2"]) * g ** 2
    step = m / (1 - o["beta1"] ** ADAMW_STEP) / ((v / (1 - o["beta2"] ** ADAMW_STEP)).sqrt() + o["eps"])
    master = flat["master"].double() * (1 - o["lr"] * o["weight_decay"]) - o["lr"] * step
    sizes = [(name, math.prod(s)) for name, s in _param_shapes(c)]
    parts = master.split([k for _, k in sizes])
    return dict(result=result, master=master, m=m, v=v, io=torch.cat([p for p, (name, _) in zip(parts, sizes) if name.startswith("w")]))


def exact(case, seed):
    c = case
    if c["kind"] in ("clip", "update"):
        return _exact_params(c, seed)
    q, k, v, length, start, dout = _inputs(c, seed)
    G, d, Nq, Nk, Tk = c["H"] // c["Hkv"], c["d"], c["Nq"], c["Nk"], _blocks(c)
    f64 = dict(dtype=torch.float64, device="cuda")
    out, lse = torch.zeros(q.shape, **f64), torch.zeros(q.shape[:3], **f64)
    grads = [torch.zeros(x.shape, **f64) for x in (q, k, v)] if c["kind"] == "train" else None
    means = torch.zeros((c["B"], c["Hkv"], Tk, d), **f64)
    blocks = torch.full((c["B"], c["Hkv"], _tiles(c), c["sel"]), -1, dtype=torch.int32, device="cuda")
    key, tile_of = torch.arange(Nk, device="cuda"), torch.arange(Nq, device="cuda") // c["qb"]
    for b in range(c["B"]):
        held = int(length[b]) if length is not None else Nk
        place = torch.arange(Nq, device="cuda") + (int(start[b]) if start is not None else Nk - Nq)
        for h in range(c["Hkv"]):
            kh, vh = k[b, h].double()[:held], v[b, h].double()[:held]
            sums = torch.zeros((Tk, d), **f64).index_add_(0, key[:held] // c["kb"], kh)
            means[b, h] = sums / torch.bincount(key[:held] // c["kb"], minlength=Tk).clamp(min=1)[:, None]
            # the choice, tile by tile from the scores of its queries
            each = sum(q[b, h * G + i].double() for i in range(G)) @ means[b, h].float().double().t()
            score = torch.zeros((_tiles(c), Tk), **f64).index_add_(0, tile_of, each)
            first = torch.full((_tiles(c),), 1 << 40, device="cuda").scatter_reduce(0, tile_of, place, "amin")
            last = torch.full((_tiles(c),), -1 << 40, device="cuda").scatter_reduce(0, tile_of, place, "amax")
            begins, ends = torch.arange(Tk, device="cuda") * c["kb"], torch.arange(1, Tk + 1, device="cuda") * c["kb"]
            taken = begins < c["first"] * c["kb"]
            if c["near"] >= 0:
                taken = taken | (ends > first[:, None] - c["near"]) & (begins <= last[:, None] + (0 if c["causal"] else c["near"]))
            score = score.masked_fill(taken, math.inf).masked_fill((begins >= held) | (c["causal"] & (begins > last[:, None])), -math.inf)
            rank = torch.argsort(torch.argsort(score, dim=1, descending=True, stable=True), dim=1, stable=True)
            chosen = (rank < c["sel"]) & (score > -math.inf)
            order = torch.where(chosen, torch.arange(Tk, device="cuda"), Tk).sort(dim=1).values[:, :c["sel"]]
            blocks[b, h, :, :order.shape[1]] = torch.where(order < Tk, order, -1).to(torch.int32)
            if c["kind"] == "choose":
                continue
            rows = max(1, (1 << 28) // max(1, held))
            for g in range(G):
                for r in range(0, Nq, rows):
                    at = slice(r, min(r + rows, Nq))
                    seen = chosen[tile_of[at]][:, key[:held] // c["kb"]]
                    if c["causal"]:
                        seen = seen & (key[:held] <= place[at, None])
                    qh = q[b, h * G + g, at].double()
                    s = ((qh @ kh.t()) * d ** -0.5).masked_fill_(~seen, -math.inf)
                    total = torch.logsumexp(s, 1)
                    p = torch.exp(s - torch.where(seen.any(1), total, 0.0)[:, None])
                    out[b, h * G + g, at], lse[b, h * G + g, at] = p @ vh, total
                    if grads:
                        do = dout[b, h * G + g, at].double()
                        dp = do @ vh.t()
                        ds = p * (dp - (p * dp).sum(1, keepdim=True)) * d ** -0.5
                        grads[0][b, h * G + g, at] = ds @ kh
                        grads[1][b, h, :held] += ds.t() @ qh
                        grads[2][b, h, :held] += p.t() @ do
    if c["kind"] == "choose":
        return dict(means=means, blocks=blocks)
    if c["kind"] == "attend":
        return out
    if c["kind"] == "decode":
        return dict(means=means, blocks=blocks, out=out)
    return dict(out=out, lse=lse, dq=grads[0], dk=grads[1], dv=grads[2])
