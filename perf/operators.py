"""The operators on a vocabulary table W [V, d] beside the decoding step: the LM head over 4-bit weights, the softmax
cross entropy of hidden rows over the allowed ids with its gradient, and the embedding of token ids with its gradient.

A case is a dict; kind says which operator it calls:
  head        B sequences x L window positions (x 2 with guidance lam) against n allowed ids of a 4-bit table with groups of
              `group` weights along d, with or without zero points
  loss        cross entropy of `rows` hidden rows over n allowed ids from v_lo on: loss and log normaliser
  train       the same and its gradients with respect to the rows and to W (bf16 or fp32)
  embed       `rows` ids of V, scaled rows of W
  embed_grad  gradient of the table for `rows` ids, bf16 or fp32
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one sequence decoded token by token over an image vocabulary: latency counts
        dict(name="head one token", kind="head", B=1, L=1, lam=0.0, V=16384, v_lo=0, n=16384, d=1280, group=64,
             zeros=False, tau=1.0),
        # a window of 32 positions with guidance over the whole vocabulary: the stream over the weights
        dict(name="head full vocabulary", kind="head", B=1, L=32, lam=3.0, V=65536, v_lo=0, n=65536, d=4096, group=128,
             zeros=False, tau=1.0),
        # sixteen sequences in one step, ragged: a matrix product over a short list of allowed ids
        dict(name="head batch", kind="head", B=16, L=30, lam=3.0, V=8200, v_lo=4, n=8191, d=4096, group=64, zeros=True,
             tau=0.9),
        # the score of a short text, or of one window
        dict(name="loss short", kind="loss", rows=77, V=16384, v_lo=0, n=16384, d=1280, tau=1.0),
        # the score of an image's tokens over the whole vocabulary
        dict(name="loss long", kind="loss", rows=2304, V=65536, v_lo=0, n=65536, d=4096, tau=1.0),
        # fine-tuning with few rows, odd sizes, gradient gathered in 32 bits
        dict(name="train ragged", kind="train", rows=515, V=16411, v_lo=5, n=16395, d=1288, tau=0.8, grad="f32"),
        # one image of 48 x 48 tokens, its codes alone allowed
        dict(name="train image", kind="train", rows=2304, V=8200, v_lo=4, n=8192, d=4096, tau=1.0, grad="bf16"),
        # a training batch over the whole vocabulary
        dict(name="train full vocabulary", kind="train", rows=4096, V=65536, v_lo=0, n=65536, d=4096, tau=1.0, grad="bf16"),
        # the drafts of a window, on their way into the model
        dict(name="embed window", kind="embed", rows=64, V=16384, d=1280, repeat=0.0),
        # a video's tokens, a training batch of them
        dict(name="embed sequence", kind="embed", rows=25600, V=64000, d=4096, repeat=0.2),
        # fine-tuning on one image of 24 x 24 tokens
        dict(name="embed_grad image", kind="embed_grad", rows=576, V=16384, d=1280, repeat=0.0, grad="f32"),
        # a training batch in which one id (padding, background) is a fifth of all
        dict(name="embed_grad sequence", kind="embed_grad", rows=25600, V=64000, d=4096, repeat=0.2, grad="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["head", "loss", "train", "embed", "embed_grad"])
    d = 8 * _log(rng, 8, 512)
    n = _log(rng, 500, 65536)
    v_lo = rng.choice([0, 0, rng.randint(1, 40)])
    V = n + v_lo + rng.choice([0, rng.randint(0, 60)])
    if kind == "head":
        L = rng.choice([1, 2, 5, 8, 16, 20, 30, 32, 64])
        B = _log(rng, 1, max(1, 512 // L))
        return dict(kind=kind, B=B, L=L, lam=rng.choice([0.0, 3.0]), V=V, v_lo=v_lo, n=n, d=d,
                    group=rng.choice([32, 64, 96, 128, 256]), zeros=rng.random() < 0.5, tau=rng.choice([1.0, 0.7]))
    if kind in ("loss", "train"):
        case = dict(kind=kind, rows=_log(rng, 1, 4096), V=V, v_lo=v_lo, n=n, d=d, tau=rng.choice([1.0, 0.7]))
        if kind == "train":
            case["grad"] = rng.choice(["bf16", "f32"])
        return case
    case = dict(kind=kind, rows=_log(rng, 1, 25600), V=n, d=d, repeat=rng.choice([0.0, 0.2, 0.6]))
    if kind == "embed_grad":
        case["grad"] = rng.choice(["bf16", "f32"])
    return case


# ---- inputs ----------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed & 0x7FFFFFFFFFFFFFFF)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _ids(c, g):
    """Token ids as texts and images have them: a few frequent, many rare, `repeat` of one id; one in 64 is left out (-1)."""
    u = torch.rand(c["rows"], generator=g, device="cuda")
    ids = (u ** 3 * c["V"]).long().clamp(max=c["V"] - 1)
    r = torch.rand(c["rows"], generator=g, device="cuda")
    ids = torch.where(r < c["repeat"], c["V"] // 2, ids)
    return torch.where(r > 1 - 1 / 64, -1, ids).to(torch.int32)


def _inputs(c, seed):
    g = _generator(seed)
    if c["kind"] == "head":
        C = 2 if c["lam"] else 1
        groups = -(-c["d"] // c["group"])
        x = dict(h=_randn(g, c["B"], C, c["L"], c["d"]).to(torch.bfloat16))
        # codes of both halves of a byte, even k in the low one
        x["codes"] = torch.randint(0, 256, (c["V"], c["d"] // 2), generator=g, device="cuda", dtype=torch.uint8)
        x["scales"] = (0.02 / 4.6 * torch.exp(0.3 * _randn(g, c["V"], groups))).to(torch.bfloat16)
        if c["zeros"]:
            x["zeros"] = torch.randint(4, 12, (c["V"], groups), generator=g, device="cuda", dtype=torch.uint8)
        return x
    if c["kind"] in ("loss", "train"):
        W = (_randn(g, c["V"], c["d"]) * 0.02).to(torch.bfloat16)
        t = torch.randint(0, c["n"], (c["rows"],), generator=g, device="cuda")
        # rows that know something of their target: its logit stands several deviations above the others
        h = _randn(g, c["rows"], c["d"])
        h += (6.0 / (0.02 * math.sqrt(c["d"]))) * W[c["v_lo"] + t].float()
        out = torch.rand(c["rows"], generator=g, device="cuda") < 1 / 16
        targets = torch.where(out, -1, t).to(torch.int32)
        w = torch.full((c["rows"],), 1.0 / c["rows"], device="cuda")
        return dict(h=h.to(torch.bfloat16), W=W, targets=targets, w=w)
    x = dict(ids=_ids(c, g))
    if c["kind"] == "embed":
        x["W"] = (_randn(g, c["V"], c["d"]) * 0.02).to(torch.bfloat16)
    else:
        x["dx"] = _randn(g, c["rows"], c["d"]).to(torch.bfloat16)
    return x


def _scale(c):
    return math.sqrt(c["d"])


def prepare(case, seed):
    c = dict(case)
    st = dict(case=c, x=_inputs(c, seed))
    if not own:
        return st
    from paper_2510_24211_amd import binding as B
    x, new = st["x"], lambda dtype, *shape: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if c["kind"] == "head":
        s = st["ctx"] = B.Scd(B.make_config(B=c["B"], L=c["L"], N=c["L"], V=c["V"], d=c["d"], v_lo=c["v_lo"],
                                            v_hi=c["v_lo"] + c["n"], temperature=c["tau"], cfg_lambda=c["lam"]))
        st["packed"] = s.pack_quantized(x["codes"], x["scales"], x.get("zeros"), c["group"])
        st["z"] = new(torch.float32, c["B"], c["L"], c["n"])
    elif c["kind"] in ("loss", "train"):
        s = st["ctx"] = B.Scd(B.make_config(B=1, L=1, N=1, V=c["V"], d=c["d"], v_lo=c["v_lo"], v_hi=c["v_lo"] + c["n"],
                                            temperature=c["tau"]))
        st["loss"], st["lse"] = new(torch.float32, c["rows"]), new(torch.float32, c["rows"])
        st["ws"] = s.cross_entropy_workspace(c["rows"])
        if c["kind"] == "train":
            st["dh"] = new(torch.bfloat16, c["rows"], c["d"])
            st["dW"] = torch.zeros(c["V"], c["d"], dtype=_TYPES[c["grad"]], device="cuda")
            st["ws_back"] = s.cross_entropy_backward_workspace(c["rows"], _TYPES[c["grad"]])
    else:
        s = st["ctx"] = B.Scd(B.make_config(B=1, L=1, N=1, V=c["V"], d=c["d"]))
        if c["kind"] == "embed":
            st["out"] = new(torch.bfloat16, c["rows"], c["d"])
        else:
            st["dW"] = new(_TYPES[c["grad"]], c["V"], c["d"])
            st["ws"] = s.embed_backward_workspace(c["rows"])
    return st


# ---- one pass --------------------------------------------------------------------------------
def _weights(c, x, dtype):
    """The allowed rows of the 4-bit table, dequantised."""
    lo, hi = c["v_lo"], c["v_lo"] + c["n"]
    codes = x["codes"][lo:hi]
    q = torch.stack([codes & 15, codes >> 4], dim=2).reshape(c["n"], c["d"]).to(dtype)
    o = x["zeros"][lo:hi].to(dtype) if c["zeros"] else torch.full_like(x["scales"][lo:hi], 8.0, dtype=dtype)
    s = x["scales"][lo:hi].to(dtype)
    spread = lambda t: t.repeat_interleave(c["group"], dim=1)[:, :c["d"]]  # noqa: E731
    return spread(s) * (q - spread(o))


def _plain_head(c, x):
    a = torch.matmul(x["h"].float().reshape(-1, c["d"]), _weights(c, x, torch.float32).t())
    a = a.reshape(c["B"], -1, c["L"], c["n"])
    z = (1.0 + c["lam"]) * a[:, 0] - c["lam"] * a[:, 1] if c["lam"] else a[:, 0]
    return z / c["tau"]


def _plain_loss(c, x):
    lo, n = c["v_lo"], c["n"]
    h, W = x["h"].float(), x["W"][lo:lo + n].float()
    z = torch.matmul(h, W.t()) / c["tau"]
    m = z.max(1, keepdim=True).values
    lse = m[:, 0] + torch.log(torch.exp(z - m).sum(1))
    t = x["targets"].long()
    valid = t >= 0
    zt = torch.gather(z, 1, t.clamp(min=0)[:, None])[:, 0]
    out = dict(loss=torch.where(valid, lse - zt, 0.0), lse=lse)
    if c["kind"] == "loss":
        return out
    dz = torch.exp(z - lse[:, None])
    dz[torch.arange(c["rows"], device="cuda"), t.clamp(min=0)] -= 1.0
    dz *= torch.where(valid, x["w"] / c["tau"], 0.0)[:, None]
    dW = torch.zeros(c["V"], c["d"], dtype=_TYPES[c["grad"]], device="cuda")
    dW[lo:lo + n] = torch.matmul(dz.t(), h).to(dW.dtype)
    out.update(dh=torch.matmul(dz, W).to(torch.bfloat16), dW=dW)
    return out


def _plain_embed(c, x):
    ids = x["ids"].long()
    rows = x["W"][ids.clamp(min=0)].float() * _scale(c)
    return torch.where((ids >= 0)[:, None], rows, 0.0).to(torch.bfloat16)


def _plain_embed_grad(c, x):
    keep = x["ids"] >= 0
    dW = torch.zeros(c["V"], c["d"], dtype=torch.float32, device="cuda")
    dW.index_add_(0, x["ids"][keep].long(), x["dx"][keep].float())
    return (dW * _scale(c)).to(_TYPES[c["grad"]])


def run(st):
    c, x = st["case"], st["x"]
    if not own:
        return {"head": _plain_head, "loss": _plain_loss, "train": _plain_loss, "embed": _plain_embed,
                "embed_grad": _plain_embed_grad}[c["kind"]](c, x)
    s = st["ctx"]
    if c["kind"] == "head":
        s.lm_head_quantized(x["h"], st["packed"], st["z"])
        return st["z"]
    if c["kind"] == "embed":
        s.embed(x["ids"], x["W"], _scale(c), st["out"])
        return st["out"]
    if c["kind"] == "embed_grad":
        s.embed_backward(x["ids"], x["dx"], _scale(c), st["dW"], st["ws"])
        return st["dW"]
    s.cross_entropy(x["h"], x["W"], x["targets"], st["loss"], st["lse"], st["ws"])
    if c["kind"] == "loss":
        return dict(loss=st["loss"], lse=st["lse"])
    s.cross_entropy_backward(x["h"], x["W"], x["targets"], st["lse"], x["w"], st["dh"], st["dW"], st["ws_back"])
    return dict(loss=st["loss"], lse=st["lse"], dh=st["dh"], dW=st["dW"])


def work(case):
    c, d = case, case["d"]
    if c["kind"] == "head":
        C = 2 if c["lam"] else 1
        rows, groups = c["B"] * c["L"], -(-d // c["group"])
        return {"bytes": c["n"] * (d // 2 + groups * (3 if c["zeros"] else 2)) + 2 * rows * C * d + 4 * rows * c["n"],
                "flops": 2 * rows * C * d * c["n"]}
    if c["kind"] == "embed":
        return {"bytes": c["rows"] * (4 + 4 * d), "flops": 0}
    size = 4 if c.get("grad") == "f32" else 2
    if c["kind"] == "embed_grad":
        return {"bytes": c["rows"] * (4 + 2 * d) + size * c["V"] * d, "flops": c["rows"] * d}
    given = 2 * d * (c["rows"] + c["n"]) + 12 * c["rows"]
    if c["kind"] == "loss":
        return {"bytes": given, "flops": 2 * c["rows"] * c["n"] * d}
    # the logits once, and the two products of the gradient
    return {"bytes": given + 2 * d * c["rows"] + size * d * c["n"] + 4 * c["rows"], "flops": 6 * c["rows"] * c["n"] * d}


# ---- the same in 64 bits ---------------------------------------------------------------------
def exact(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    d, f64 = c["d"], torch.float64
    if c["kind"] == "head":
        lo = c["v_lo"]
        k = torch.arange(d, device="cuda")
        # code of (v, k): byte k / 2, its half k mod 2; scale and origin of group k / group
        byte = x["codes"][lo:lo + c["n"], k // 2].to(torch.int32)
        q = (byte >> (4 * (k % 2)).to(torch.int32)) & 15
        at = k // c["group"]
        origin = x["zeros"][lo:lo + c["n"]][:, at].to(f64) if c["zeros"] else 8.0
        W = x["scales"][lo:lo + c["n"]].to(f64)[:, at] * (q.to(f64) - origin)
        z = torch.matmul(x["h"].to(f64), W.t())
        return ((1 + c["lam"]) * z[:, 0] - c["lam"] * z[:, -1]) / c["tau"]
    if c["kind"] == "embed":
        out = torch.zeros(c["rows"], d, dtype=f64, device="cuda")
        there = (x["ids"] >= 0).nonzero()[:, 0]
        out[there] = x["W"].to(f64)[x["ids"][there].long()] * math.sqrt(d)
        return out
    if c["kind"] == "embed_grad":
        # rows in the order of their ids, each stretch of one id summed up
        order = torch.argsort(x["ids"], stable=True)
        order = order[x["ids"][order] >= 0]
        out = torch.zeros(c["V"], d, dtype=f64, device="cuda")
        if len(order):
            ids, count = torch.unique_consecutive(x["ids"][order], return_counts=True)
            out[ids.long()] = torch.segment_reduce(x["dx"][order].to(f64), "sum", lengths=count, axis=0)
        return out * math.sqrt(d)
    lo = c["v_lo"]
    h, W = x["h"].to(f64), x["W"][lo:lo + c["n"]].to(f64)
    z = (h @ W.t()) / c["tau"]
    logp = torch.log_softmax(z, 1)
    there = x["targets"] >= 0
    onehot = torch.zeros_like(z)
    onehot[there.nonzero()[:, 0], x["targets"][there].long()] = 1.0
    out = dict(loss=-(onehot * logp).sum(1), lse=torch.logsumexp(z, 1))
    if c["kind"] == "loss":
        return out
    dz = there.to(f64)[:, None] * x["w"].to(f64)[:, None] * (torch.exp(logp) - onehot) / c["tau"]
    dW = torch.zeros(c["V"], d, dtype=f64, device="cuda")
    dW[lo:lo + c["n"]] = dz.t() @ h
    out.update(dh=dz @ W, dW=dW)
    return out
