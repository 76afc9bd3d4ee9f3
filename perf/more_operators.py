"""The operators at the end of a model, around its last norm: the root-mean-square norm with the residual's addition, in
bf16 or in 8 bits with scales, and its gradient; the LM head over 8-bit rows and weights with a scale per block of 128; the
global norm of gradients and their clipping.

A case is a dict; kind says which operator it calls:
  norm        `rows` hidden rows of d, added to a residual stream of type `res` (bf16, f32, or none): the stream and the normed rows
  norm8       the same with the normed rows as e4m3 codes and a scale per 128 of a row, for the LM head
  norm_grad   gradient of the norm with respect to its rows and its gains (of type `grad`)
  head        B sequences x L window positions (x 2 with guidance lam) against n allowed ids, rows and weights e4m3 with scales for each
              block of 128 (of a row; of 128 rows of the table)
  clip        the gradients (of type `grad`) of a table V x d and of `layers` layers: their norm, and what it leaves of them under
              max_norm, of type `out`
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_E4M3 = torch.float8_e4m3fn
_MOST = 448.0                     # the largest finite e4m3 number
_EPS = 1e-6


def listed():
    return [
        # the last hidden row of a decode token by token, on its way to the LM head: latency counts
        dict(name="norm8 one token", kind="norm8", rows=1, d=1280, res="bf16"),
        # an image of 48 x 48 tokens to be scored in 8 bits
        dict(name="norm8 image", kind="norm8", rows=2304, d=4096, res="bf16"),
        # a window of 32 positions with guidance, residual stream in 32 bits
        dict(name="norm window", kind="norm", rows=64, d=4096, res="f32"),
        # a training batch of video tokens
        dict(name="norm batch", kind="norm", rows=25600, d=4096, res="bf16"),
        # fine-tuning with few rows, odd sizes
        dict(name="norm_grad ragged", kind="norm_grad", rows=515, d=1288, res="f32", grad="f32"),
        # the training batch's way back
        dict(name="norm_grad batch", kind="norm_grad", rows=25600, d=4096, res="bf16", grad="bf16"),
        # one sequence decoded token by token over an image vocabulary
        dict(name="head one token", kind="head", B=1, L=1, lam=0.0, V=16384, v_lo=0, n=16384, d=1280, tau=1.0),
        # a window of 32 positions with guidance over the whole vocabulary: the stream over the weights
        dict(name="head full vocabulary", kind="head", B=1, L=32, lam=3.0, V=65536, v_lo=0, n=65536, d=4096, tau=1.0),
        # sixteen sequences in one step, ragged: a matrix product over a short list of allowed ids
        dict(name="head batch", kind="head", B=16, L=30, lam=3.0, V=8200, v_lo=4, n=8191, d=4096, tau=0.9),
        # eight videos in one step
        dict(name="head videos", kind="head", B=8, L=64, lam=3.0, V=64000, v_lo=0, n=64000, d=4096, tau=1.0),
        # a table and its norms, gradients gathered in 32 bits, clipped copies in 16
        dict(name="clip table", kind="clip", V=16411, d=1288, layers=2, grad="f32", out="bf16", max_norm=1.0),
        # a model's gradients
        dict(name="clip model", kind="clip", V=65536, d=4096, layers=8, grad="bf16", out="bf16", max_norm=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm8", "norm_grad", "head", "head", "clip"])
    if kind in ("norm", "norm8"):
        return dict(kind=kind, rows=_log(rng, 1, 25600), d=8 * _log(rng, 8, 512), res=rng.choice(["bf16", "f32", "none"]))
    if kind == "norm_grad":
        return dict(kind=kind, rows=_log(rng, 1, 25600), d=8 * _log(rng, 8, 512), res=rng.choice(["bf16", "f32"]),
                    grad=rng.choice(["bf16", "f32"]))
    if kind == "head":
        L = rng.choice([1, 2, 5, 8, 16, 20, 30, 32, 64])
        n = _log(rng, 500, 64000)
        v_lo = rng.choice([0, 0, rng.randint(1, 400)])
        return dict(kind=kind, B=_log(rng, 1, max(1, 512 // L)), L=L, lam=rng.choice([0.0, 3.0]), V=n + v_lo + rng.choice([0, rng.randint(0, 60)]),
                    v_lo=v_lo, n=n, d=16 * _log(rng, 4, 256), tau=rng.choice([1.0, 0.7]))
    grad = rng.choice(["bf16", "f32"])
    most = 65536 if grad == "bf16" else 32768
    return dict(kind=kind, V=_log(rng, 500, most), d=8 * _log(rng, 8, 512), layers=rng.randint(0, most // 8192), grad=grad,
                out=rng.choice(["bf16", grad]), max_norm=rng.choice([1.0, 0.5, 1e9]))


# ---- inputs ----------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed & 0x7FFFFFFFFFFFFFFF)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)


def _hidden(c, g):
    """Hidden rows as models have them: channels of different sizes, a few of them large; one row in 64 is padding (zeros)."""
    size = torch.exp(0.5 * _randn(g, c["d"])) * torch.where(_rand(g, c["d"]) < 0.01, 20.0, 1.0)
    there = (_rand(g, c["rows"], 1) >= 1 / 64).float()
    return _randn(g, c["rows"], c["d"]) * size * there


def _shapes(c):
    """A table and its norm; of each layer two norms and four square matrices."""
    d = c["d"]
    return [(c["V"], d), (d,)] + [(d,), (d,), (d, d), (d, d), (d, d), (d, d)] * c["layers"]


def _inputs(c, seed):
    g = _generator(seed)
    if c["kind"] in ("norm", "norm8"):
        x = dict(x=(0.3 * _hidden(c, g)).to(torch.bfloat16), gain=(1.0 + 0.3 * _randn(g, c["d"])).to(torch.bfloat16))
        if c["res"] != "none":
            x["residual"] = (_hidden(c, g) * (x["x"] != 0).any(1, keepdim=True)).to(_TYPES[c["res"]])
        return x
    if c["kind"] == "norm_grad":
        x = dict(sum=_hidden(c, g).to(_TYPES[c["res"]]), gain=(1.0 + 0.3 * _randn(g, c["d"])).to(torch.bfloat16))
        x["inv"] = torch.rsqrt(x["sum"].double().square().mean(1) + _EPS).float()
        # padding has no gradient
        there = (x["sum"] != 0).any(1, keepdim=True)
        x["dy"] = (_randn(g, c["rows"], c["d"]) * there).to(torch.bfloat16)
        x["dsum"] = (_randn(g, c["rows"], c["d"]) * there).to(torch.bfloat16)
        return x
    if c["kind"] == "head":
        C, G = 2 if c["lam"] else 1, -(-c["d"] // 128)
        code = lambda *shape: (100.0 * _randn(g, *shape)).clamp(-_MOST, _MOST).to(_E4M3)  # noqa: E731
        return dict(h=code(c["B"], C, c["L"], c["d"]), h_scales=torch.exp(0.3 * _randn(g, c["B"], C, c["L"], G)) / 100.0,
                    W=code(c["V"], c["d"]), W_scales=0.02 * torch.exp(0.3 * _randn(g, -(-c["V"] // 128), G)) / 100.0)
    return dict(grads=[(0.01 * _randn(g, *shape)).to(_TYPES[c["grad"]]) for shape in _shapes(c)])


def prepare(case, seed):
    c = dict(case)
    st = dict(case=c, x=_inputs(c, seed))
    if not own:
        return st
    from paper_2510_24211_amd import binding as B
    x, new = st["x"], lambda dtype, *shape: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if c["kind"] == "head":
        st["ctx"] = B.Scd(B.make_config(B=c["B"], L=c["L"], N=c["L"], V=c["V"], d=c["d"], v_lo=c["v_lo"], v_hi=c["v_lo"] + c["n"],
                                        temperature=c["tau"], cfg_lambda=c["lam"]))
        st["z"] = new(torch.float32, c["B"], c["L"], c["n"])
        return st
    s = st["ctx"] = B.Scd(B.make_config(B=1, L=1, N=1, V=c.get("V", 1), d=c["d"]))
    if c["kind"] == "clip":
        st["norm"] = new(torch.float32, 1)
        # the clipped gradients in one buffer, as an optimizer takes them
        st["flat"] = new(_TYPES[c["out"]], sum(t.numel() for t in x["grads"]))
        out = [t.view(like.shape) for t, like in zip(st["flat"].split([t.numel() for t in x["grads"]]), x["grads"])]
        st["grads"], st["out"] = B.TensorList(x["grads"]), B.TensorList(out)
        st["ws"] = s.gradient_norm_workspace(st["grads"])
        return st
    rows, d = c["rows"], c["d"]
    if c["kind"] == "norm_grad":
        st["dx"], st["dgain"] = new(torch.bfloat16, rows, d), new(_TYPES[c["grad"]], d)
        st["ws"] = s.norm_backward_workspace(rows)
        return st
    st["inv"] = new(torch.float32, rows)
    st["sum"] = new(_TYPES[c["res"]], rows, d) if c["res"] != "none" else None
    if c["kind"] == "norm":
        st["y"] = new(torch.bfloat16, rows, d)
    else:
        st["codes"], st["scales"] = new(_E4M3, rows, d), new(torch.float32, rows, -(-d // 128))
    return st


# ---- one pass --------------------------------------------------------------------------------
def _in_blocks(t):
    """The last dimension in blocks of 128, zeros behind its end."""
    return torch.nn.functional.pad(t, (0, -t.shape[-1] % 128)).reshape(*t.shape[:-1], -1, 128)


def _plain_norm(c, x):
    s = x["x"].float()
    if c["res"] != "none":
        s = s + x["residual"].float()
    inv = 1.0 / torch.sqrt((s * s).mean(1) + _EPS)
    y = s * inv[:, None] * x["gain"].float()
    out = dict(inv=inv)
    if c["res"] != "none":
        out["sum"] = s.to(_TYPES[c["res"]])
    if c["kind"] == "norm":
        out["y"] = y.to(torch.bfloat16)
        return out
    blocks = _in_blocks(y)
    out["scales"] = blocks.abs().amax(2) / _MOST
    codes = torch.where(out["scales"][..., None] > 0, blocks / out["scales"][..., None], 0.0)
    out["codes"] = codes.reshape(c["rows"], -1)[:, :c["d"]].to(_E4M3)
    return out


def _plain_norm_grad(c, x):
    s, dy = x["sum"].float(), x["dy"].float()
    inv = x["inv"][:, None]
    a = x["gain"].float() * dy
    dx = inv * (a - s * inv * inv * (a * s).mean(1, keepdim=True)) + x["dsum"].float()
    return dict(dx=dx.to(torch.bfloat16), dgain=(dy * s * inv).sum(0).to(_TYPES[c["grad"]]))


def _spread(codes, scales):
    return codes.float() * scales.repeat_interleave(128, dim=-1)[..., :codes.shape[-1]]


def _plain_head(c, x):
    lo, hi = c["v_lo"], c["v_lo"] + c["n"]
    W = _spread(x["W"][lo:hi], x["W_scales"].repeat_interleave(128, dim=0)[lo:hi])
    a = torch.matmul(_spread(x["h"], x["h_scales"]).reshape(-1, c["d"]), W.t()).reshape(c["B"], -1, c["L"], c["n"])
    z = (1.0 + c["lam"]) * a[:, 0] - c["lam"] * a[:, 1] if c["lam"] else a[:, 0]
    return z / c["tau"]


def _plain_clip(c, x):
    # (a sum of half a billion squares in 64 bits)
    norm = torch.stack([t.double().square().sum() for t in x["grads"]]).sum().sqrt().float()
    by = (c["max_norm"] / norm).clamp(max=1.0)
    return dict(norm=norm.reshape(1), flat=torch.cat([(t.float() * by).to(_TYPES[c["out"]]).reshape(-1) for t in x["grads"]]))


def run(st):
    c, x = st["case"], st["x"]
    if not own:
        return {"norm": _plain_norm, "norm8": _plain_norm, "norm_grad": _plain_norm_grad, "head": _plain_head, "clip": _plain_clip}[c["kind"]](c, x)
    s = st["ctx"]
    if c["kind"] == "head":
        s.lm_head_fp8(x["h"], x["h_scales"], x["W"], x["W_scales"], st["z"])
        return st["z"]
    if c["kind"] == "clip":
        s.gradient_norm(st["grads"], st["norm"], st["ws"])
        s.clip_gradients(st["grads"], st["out"], c["max_norm"], st["norm"])
        return dict(norm=st["norm"], flat=st["flat"])
    if c["kind"] == "norm_grad":
        s.norm_backward(x["sum"], x["gain"], x["inv"], x["dy"], st["dx"], st["dgain"], st["ws"], dsum=x["dsum"])
        return dict(dx=st["dx"], dgain=st["dgain"])
    out = dict(inv=st["inv"])
    if st["sum"] is not None:
        out["sum"] = st["sum"]
    if c["kind"] == "norm":
        s.norm(x["x"], x["gain"], st["y"], _EPS, residual=x.get("residual"), sum=st["sum"], inv=st["inv"])
        out["y"] = st["y"]
    else:
        s.norm_fp8(x["x"], x["gain"], st["codes"], st["scales"], _EPS, residual=x.get("residual"), sum=st["sum"], inv=st["inv"])
        out.update(codes=st["codes"], scales=st["scales"])
    return out


def work(case):
    c, d = case, case["d"]
    size = {"bf16": 2, "f32": 4, "none": 0}
    if c["kind"] == "head":
        C, G = 2 if c["lam"] else 1, -(-d // 128)
        rows = c["B"] * c["L"]
        return {"bytes": c["n"] * d + 4 * G * -(-c["n"] // 128) + rows * C * (d + 4 * G) + 4 * rows * c["n"], "flops": 2 * rows * C * d * c["n"]}
    if c["kind"] == "clip":
        count = sum(math.prod(shape) for shape in _shapes(c))
        return {"bytes": count * (size[c["grad"]] + size[c["out"]]) + 4, "flops": 3 * count}
    count = c["rows"] * d
    if c["kind"] == "norm_grad":
        return {"bytes": count * (size[c["res"]] + 6) + 4 * c["rows"] + d * (2 + size[c["grad"]]), "flops": 10 * count}
    y = 2 * count if c["kind"] == "norm" else count + 4 * c["rows"] * -(-d // 128)
    return {"bytes": count * (2 + 2 * size[c["res"]]) + y + 2 * d + 4 * c["rows"], "flops": 5 * count}


# ---- the same in 64 bits ---------------------------------------------------------------------
def exact(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    f64 = torch.float64
    if c["kind"] == "head":
        # code (m, k) stands for itself times the scale of block k / 128, code (v, k) of the table times that of block (v / 128, k / 128)
        k = torch.arange(c["d"], device="cuda") // 128
        v = torch.arange(c["v_lo"], c["v_lo"] + c["n"], device="cuda")
        W = x["W"].to(f64)[v] * x["W_scales"].to(f64)[v // 128][:, k]
        z = torch.matmul(x["h"].to(f64) * x["h_scales"].to(f64)[..., k], W.t())
        return ((1 + c["lam"]) * z[:, 0] - c["lam"] * z[:, -1]) / c["tau"]
    if c["kind"] == "clip":
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t.to(f64))) ** 2 for t in x["grads"]))
        by = min(1.0, c["max_norm"] / norm)
        return dict(norm=torch.tensor([norm], dtype=f64, device="cuda"), flat=torch.cat([t.to(f64).flatten() for t in x["grads"]]).mul_(by))
    gain = x["gain"].to(f64)
    if c["kind"] == "norm_grad":
        # by the chain rule through u = s inv: du = gain dy, ds = inv (du - u <u, du> / d)
        s, dy = x["sum"].to(f64), x["dy"].to(f64)
        inv = (s.pow(2).sum(1, keepdim=True) / c["d"] + _EPS).pow(-0.5)
        u, du = s * inv, gain * dy
        ds = inv * (du - u * ((u * du).sum(1, keepdim=True) / c["d"]))
        return dict(dx=ds + x["dsum"].to(f64), dgain=(u * dy).sum(0))
    s = x["x"].to(f64) + (x["residual"].to(f64) if "residual" in x else 0.0)
    inv = (s.pow(2).sum(1) / c["d"] + _EPS).pow(-0.5)
    y = torch.einsum("rd,r,d->rd", s, inv, gain)
    out = dict(inv=inv)
    if "residual" in x:
        out["sum"] = s
    if c["kind"] == "norm":
        out["y"] = y
        return out
    edges = range(0, c["d"], 128)
    out["scales"] = torch.stack([y[:, k:k + 128].abs().max(1).values for k in edges], 1) / _MOST
    out["codes"] = torch.cat([y[:, k:k + 128] / out["scales"][:, i:i + 1].clamp(min=1e-300) for i, k in enumerate(edges)], 1)
    return out
