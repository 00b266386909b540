"""The operators of a training iteration's weight update and of its blocks'
normalization, as cases that can be timed.

They are the kernels that three of the recipes predict (a fused optimizer, mixed
precision, fused element-wise kernels), each reached through `binding`:

  clip   the global norm of many gradient tensors, then the gradients unscaled
         and clipped into other tensors
  adam   an Adam step over many tensors, with the gradients as they are
  step   the norm, then an Adam step that takes the clipping factor from it
  rms    the residual's addition and the root-mean-square norm, plain or in 8 bits
  rmsg   its gradient

A list of tensors lies in one flat buffer for each of its parts (gradients,
weights, moments), as frameworks keep them for their collectives: the framework
gets the tensors, the plain form works on the flat buffers, so it needs no
loop over tensors.  Gaps between tensors hold zeros, which stay zeros.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
RMS_EPS = 1e-6
FIRST_STEP = 10                 # steps taken before the first pass
LOSS_SCALE = 1024.0             # carried by half-precision gradients
E4M3_MOST = 448.0
MOST = 1_300_000_000            # elements of the longest list
MOST_ROWS = 1 << 28             # elements of the largest norm


def listed():
    return [
        # a small model's gradients, odd sizes end to end: launches and latency
        dict(name="clip_small", op="clip", shape="ragged", tensors=61, longest=20_000, pick=1, grad="f32", align=1, max_norm=0.05),
        # the gradients of VGG-19 in f32
        dict(name="clip_vgg19", op="clip", shape="vgg19", grad="f32", align=1, max_norm=1.0),
        # 24 layers of hidden size 1,024 in bf16, clipped into f32 for an optimizer of the user's own
        dict(name="clip_transformer", op="clip", shape="transformer", hidden=1024, layers=24, grad="bf16", align=64, max_norm=1.0),
        # one small model's weight update in f32
        dict(name="adam_small", op="adam", shape="ragged", tensors=61, longest=20_000, pick=2, grad="f32", param="f32", align=1),
        # the weight update of VGG-19 in f32
        dict(name="adam_vgg19", op="adam", shape="vgg19", grad="f32", param="f32", align=64),
        # mixed precision: bf16 weights with f32 masters, norm and update together
        dict(name="step_transformer", op="step", shape="transformer", hidden=1024, layers=24, grad="bf16", param="bf16", align=64, max_norm=1.0),
        # the same of a model four times as large, half-precision gradients of a scaled loss
        dict(name="step_transformer_large", op="step", shape="transformer", hidden=2048, layers=24, grad="f16", param="f16", align=64, max_norm=1.0),
        # one token each of a few requests, answered in 8 bits for the next product
        dict(name="rms_tokens", op="rms", rows=4, cols=4096, kind="bf16", weight="bf16", residual=True, out="e4m3", group=0, keep=False, pad=0),
        # whole prompts, a scale for each 128 columns
        dict(name="rms_prompt", op="rms", rows=8192, cols=4096, kind="bf16", weight="bf16", residual=True, out="e4m3", group=128, keep=False, pad=0),
        # the forward pass of training at an odd width in f32, rows of a wider buffer, with what the gradient needs
        dict(name="rms_odd", op="rms", rows=4099, cols=1237, kind="f32", weight="f32", residual=True, out="same", group=0, keep=True, pad=19),
        # its gradient at the hidden size of the transformer workload
        dict(name="rmsg_train", op="rmsg", rows=16384, cols=1024, kind="bf16", weight="f32", dh=True, pad=0),
        # and at a large one
        dict(name="rmsg_wide", op="rmsg", rows=32768, cols=8192, kind="bf16", weight="bf16", dh=True, pad=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("clip", "adam", "step", "rms", "rmsg", "rms", "rmsg"))
    kind = rng.choice(("f32", "bf16", "f16"))
    weight = rng.choice(("f32", kind))
    if op in ("rms", "rmsg"):
        cols = _log_int(rng, 64, 16384)
        rows = _log_int(rng, 1, min(65536, MOST_ROWS // cols))
        pad = rng.choice((0, 0, 8, _log_int(rng, 1, 100)))
        c = dict(op=op, rows=rows, cols=cols, kind=kind, weight=weight, pad=pad)
        if op == "rmsg":
            return dict(c, dh=rng.random() < 0.7)
        out = rng.choice(("same", "e4m3"))
        return dict(c, residual=rng.random() < 0.8, out=out, group=rng.choice((0, 128)) if out == "e4m3" else 0,
                    keep=rng.random() < 0.5)
    shape = rng.choice(("ragged", "ragged", "transformer"))
    if shape == "ragged":
        tensors = _log_int(rng, 1, 1000)
        c = dict(op=op, shape=shape, tensors=tensors, longest=_log_int(rng, 1000, min(100_000_000, MOST // tensors)),
                 pick=rng.randrange(1 << 20))
    else:
        hidden = _log_int(rng, 64, 2048)
        c = dict(op=op, shape=shape, hidden=hidden, layers=_log_int(rng, 1, min(24, MOST // (12 * hidden * hidden + 13 * hidden))))
    c.update(grad=kind, align=rng.choice((1, 8, 64)))
    if op in ("adam", "step"):
        c["param"] = rng.choice(("f32", "bf16")) if kind == "f32" else kind
    if op != "adam":
        c["max_norm"] = rng.choice((0.01, 1.0))
    return c


# ---------------------------------------------------------------------------
# the tensors of a model
def _sizes(case):
    """(sizes of the tensors that weight decay applies to, sizes of the others)."""
    if case["shape"] == "transformer":      # 12 h^2 + 13 h a layer: the gradient bytes of the all-reduce workload
        h, n = case["hidden"], case["layers"]
        return [h * h, h * h, h * h, h * h, 4 * h * h, 4 * h * h] * n, [h, h, h, h, 4 * h, h, h, h, h, h] * n
    if case["shape"] == "vgg19":
        chans = [3, 64, 64, 128, 128, 256, 256, 256, 256, 512, 512, 512, 512, 512, 512, 512, 512]
        fc = [512 * 49, 4096, 4096, 1000]
        return ([9 * a * b for a, b in zip(chans, chans[1:])] + [a * b for a, b in zip(fc, fc[1:])], chans[1:] + fc[1:])
    r = random.Random(case["pick"])
    sizes = [_log_int(r, 1, case["longest"]) for _ in range(case["tensors"])]
    k = (3 * len(sizes) + 3) // 4
    return sizes[:k], sizes[k:]


def _layout(case):
    """(first element of each tensor, its size, whether it decays, elements
    that hold the decayed ones, elements in all)."""
    a, b = _sizes(case)
    size = np.array(a + b, np.int64)
    room = -(-size // case["align"]) * case["align"]
    first = np.concatenate([[0], np.cumsum(room)])
    return first[:-1], size, np.arange(len(size)) < len(a), int(first[len(a)]), int(first[-1])


def _flat(layout, kind, gen, std, square=False):
    """A flat buffer of normal values, zeros between the tensors."""
    first, size, _, _, total = layout
    x = torch.randn(total, generator=gen, device=DEV)
    x.mul_(std)
    if square:
        x.square_()
    ends = first + size
    gaps = [torch.arange(int(e), int(n), device=DEV) for e, n in zip(ends, np.append(first[1:], total)) if e < n]
    if gaps:
        x[torch.cat(gaps)] = 0.0
    return x.to(TYPES[kind])


class Tensors:
    """The handle a training program makes once for its tensors."""

    def __init__(self, layout, parts):
        from paper_2006_03318_amd import binding
        first, size, decay = layout[:3]
        self.free = binding.dd_tensors_free
        self.handle = binding.dd_tensors_load([
            dict({k: x[int(f):int(f) + int(n)] for k, x in parts.items()}, decay=bool(d)) for f, n, d in zip(first, size, decay)])

    def __del__(self):
        if hasattr(self, "handle"):
            self.free(self.handle)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case}
    if case["op"] in ("rms", "rmsg"):
        return _prepare_rows(case, gen, s)
    lay = _layout(case)
    kind = case["grad"]
    scaled = kind == "f16"
    s["grad"] = _flat(lay, kind, gen, 1e-3 * (LOSS_SCALE if scaled else 1.0))
    s["split"] = lay[3]
    s["stats"] = torch.zeros(3, device=DEV)                 # norm, factor, whether something is not finite
    s["inv_scale"] = torch.full((1,), 1.0 / LOSS_SCALE, device=DEV) if scaled else None
    parts = {"grad": s["grad"]}
    if case["op"] == "clip":
        s["clipped"] = torch.zeros_like(s["grad"], dtype=torch.float32)
    if case["op"] in ("adam", "step"):
        s["master"] = _flat(lay, "f32", gen, 0.02)
        s["m"] = _flat(lay, "f32", gen, 1e-3)
        s["v"] = _flat(lay, "f32", gen, 1e-3, square=True)
        s["step"] = torch.full((1,), FIRST_STEP, dtype=torch.int64, device=DEV)
        low = case["param"] != "f32"
        if low:
            s["param"] = s["master"].to(TYPES[case["param"]])
            parts.update(param=s["param"], master=s["master"], m=s["m"], v=s["v"])
        else:
            parts.update(param=s["master"], m=s["m"], v=s["v"])
    if own:     # a program makes its lists once: the handle is kept like the tensors are
        s["tensors"] = Tensors(lay, parts)
        if case["op"] == "clip":
            s["target"] = Tensors(lay, {"grad": s["clipped"]})
    return s


def _prepare_rows(case, gen, s):
    rows, cols, kind = case["rows"], case["cols"], TYPES[case["kind"]]

    def rand(std=1.0, pad=0):
        return (torch.randn(rows, cols + pad, generator=gen, device=DEV) * std).to(kind)[:, :cols]

    s["weight"] = (1.0 + 0.2 * torch.randn(cols, generator=gen, device=DEV)).to(TYPES[case["weight"]])
    if case["op"] == "rms":
        s["x"] = rand(pad=case["pad"])
        s["residual"] = rand(3.0) if case["residual"] else None
        groups = -(-cols // case["group"]) if case["group"] else 1
        s["out"] = torch.empty(rows, cols, device=DEV, dtype=torch.float8_e4m3fn if case["out"] == "e4m3" else kind)
        s["scales"] = torch.empty(rows, groups, device=DEV) if case["out"] == "e4m3" else None
        s["h"] = torch.empty(rows, cols, device=DEV, dtype=kind) if case["residual"] else None
        s["rstd"] = torch.empty(rows, device=DEV) if case["keep"] else None
        return s
    s["h"] = rand(3.0, pad=case["pad"])
    s["dy"] = rand(1e-2)
    s["dh"] = rand(1e-2) if case["dh"] else None
    s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + RMS_EPS)
    s["dx"] = torch.empty(rows, cols, device=DEV, dtype=kind)
    s["dw"] = torch.empty_like(s["weight"])
    return s


# ---------------------------------------------------------------------------
# one pass
def run(s):
    if own:
        return _run_own(s, s["case"])
    return {"clip": _plain_clip, "adam": _plain_adam, "step": _plain_step, "rms": _plain_rms,
            "rmsg": _plain_rmsg}[s["case"]["op"]](s, s["case"])


def _run_own(s, case):
    from paper_2006_03318_amd import binding as B
    op = case["op"]
    if op == "rms":
        B.dd_rms_norm(s["x"], s["residual"], s["weight"], RMS_EPS, s["out"], h=s["h"], rstd=s["rstd"], scales=s["scales"], group=case["group"])
        return {k: s[k] for k in ("out", "scales", "h", "rstd") if s[k] is not None}
    if op == "rmsg":
        B.dd_rms_norm_grad(s["dy"], s["h"], s["weight"], s["rstd"], s["dx"], s["dw"], dh=s["dh"])
        return {"dx": s["dx"], "dw": s["dw"]}
    t = s["tensors"].handle
    if op != "adam":
        B.dd_grad_norm(t, s["stats"], max_norm=case["max_norm"], d_inv_scale=s["inv_scale"])
    if op == "clip":
        B.dd_grad_clip(t, s["target"].handle, s["stats"])
        return {"stats": s["stats"], "clipped": s["clipped"]}
    B.dd_adam_step(t, s["step"], s["stats"] if op == "step" else None, lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY)
    return _state_of(s)


def _state_of(s):
    return {k: s[k] for k in ("param", "master", "m", "v", "step", "stats") if k in s and not (k == "stats" and s["case"]["op"] == "adam")}


def _plain_norm(s, case):
    g = s["grad"].float()
    u = s["inv_scale"] if s["inv_scale"] is not None else torch.ones(1, device=DEV)
    norm = (g * g).sum().sqrt() * u
    factor = u * torch.clamp(case["max_norm"] / norm, max=1.0)
    s["stats"] = torch.cat([norm, factor, (~torch.isfinite(norm)).float()])


def _plain_clip(s, case):
    _plain_norm(s, case)
    return {"stats": s["stats"], "clipped": s["grad"].float() * s["stats"][1]}


def _plain_step(s, case):
    _plain_norm(s, case)
    return _plain_update(s, s["grad"].float() * s["stats"][1])


def _plain_adam(s, case):
    return _plain_update(s, s["grad"].float())


def _plain_update(s, g):
    """The gradients of these cases are finite: no update is skipped."""
    t = s["step"].add_(1).double()
    by_m = (LR / (1.0 - BETA1 ** t)).float()
    by_v = (1.0 / torch.sqrt(1.0 - BETA2 ** t)).float()
    s["m"].mul_(BETA1).add_(g, alpha=1.0 - BETA1)
    s["v"].mul_(BETA2).addcmul_(g, g, value=1.0 - BETA2)
    s["master"][:s["split"]].mul_(1.0 - LR * DECAY)
    s["master"].sub_(s["v"].sqrt().mul_(by_v).add_(ADAM_EPS).reciprocal_().mul_(s["m"]).mul_(by_m))
    if "param" in s:
        s["param"].copy_(s["master"])
    return _state_of(s)


def _plain_rms(s, case):
    h = s["x"].float()
    if case["residual"]:
        h = h + s["residual"].float()
    rstd = torch.rsqrt((h * h).mean(1, keepdim=True) + RMS_EPS)
    y = h * rstd * s["weight"].float()
    got = {}
    if case["out"] == "e4m3":
        cols = case["cols"]
        group = case["group"] or cols
        wide = torch.nn.functional.pad(y, (0, -cols % group)).view(case["rows"], -1, group)
        scale = wide.abs().amax(2).clamp(min=2.0 ** -100) / E4M3_MOST
        q = (wide / scale[:, :, None]).view(case["rows"], -1)[:, :cols]
        got.update(out=q.to(torch.float8_e4m3fn), scales=scale)
    else:
        got["out"] = y.to(s["x"].dtype)
    if case["residual"]:
        got["h"] = h.to(s["x"].dtype)
    if case["keep"]:
        got["rstd"] = rstd[:, 0]
    return got


def _plain_rmsg(s, case):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = s["h"].float() * rstd
    dw = (dy * xh).sum(0)
    dy = dy * s["weight"].float()
    dx = (dy - xh * (dy * xh).mean(1, keepdim=True)) * rstd
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["dy"].dtype), "dw": dw.to(s["weight"].dtype)}


# ---------------------------------------------------------------------------
def work(case):
    if case["op"] in ("rms", "rmsg"):
        n, w = case["rows"] * case["cols"], case["cols"] * BYTES[case["weight"]]
        b = BYTES[case["kind"]]
        if case["op"] == "rmsg":
            return {"bytes": n * b * (4 if case["dh"] else 3) + 2 * w + 4 * case["rows"], "flops": 10 * n}
        groups = -(-case["cols"] // case["group"]) if case["group"] else 1
        out = n + 4 * case["rows"] * groups if case["out"] == "e4m3" else n * b
        return {"bytes": n * b * (3 if case["residual"] else 1) + out + w + (4 * case["rows"] if case["keep"] else 0),
                "flops": 6 * n}
    n = sum(map(sum, _sizes(case)))
    b = BYTES[case["grad"]]
    if case["op"] == "clip":
        return {"bytes": n * (b + 4), "flops": 3 * n}
    low = BYTES[case["param"]] if case["param"] != "f32" else 0
    return {"bytes": n * (b + 24 + low), "flops": (15 if case["op"] == "adam" else 18) * n}


def exact(case, seed):
    """The definitions, in 64 bits, on the same inputs."""
    s = prepare(case, seed)
    got = {}
    if case["op"] == "rms":
        rows, cols, w = case["rows"], case["cols"], s["weight"].double()
        h = s["x"].double()
        if case["residual"]:
            h = h + s["residual"].double()
            got["h"] = h
        rstd = 1.0 / (h.pow(2).sum(1) / cols + RMS_EPS).sqrt()
        if case["keep"]:
            got["rstd"] = rstd
        y = h * rstd[:, None] * w
        if case["out"] == "same":
            return dict(got, out=y)
        group = case["group"] or cols
        scale = torch.stack([c.abs().max(1).values for c in y.split(group, 1)], 1).clamp(min=2.0 ** -100) / E4M3_MOST
        return dict(got, out=y / scale.repeat_interleave(group, 1)[:, :cols], scales=scale)     # not rounded to 8 bits
    if case["op"] == "rmsg":
        rows, cols, w = case["rows"], case["cols"], s["weight"].double()
        got = {"dx": torch.empty(rows, cols, dtype=torch.float64, device=DEV), "dw": torch.zeros(cols, dtype=torch.float64, device=DEV)}
        for a in range(0, rows, 4096):
            z = slice(a, a + 4096)
            r, dy = s["rstd"][z].double()[:, None], s["dy"][z].double()
            n = s["h"][z].double() * r
            got["dw"] += (dy * n).sum(0)
            dot = (dy * w * n).sum(1, keepdim=True) / cols
            got["dx"][z] = r * (dy * w - n * dot)
            if s["dh"] is not None:
                got["dx"][z] += s["dh"][z].double()
        return got
    factor = 1.0
    if case["op"] != "adam":
        u = 1.0 / LOSS_SCALE if s["inv_scale"] is not None else 1.0
        norm = u * math.sqrt(sum(float(c.double().square().sum()) for c in s["grad"].split(1 << 26)))
        factor = u * min(1.0, case["max_norm"] / norm)
        got["stats"] = torch.tensor([norm, factor, 0.0], dtype=torch.float64, device=DEV)
    if case["op"] == "clip":
        return dict(got, clipped=s["grad"].double() * factor)
    t = FIRST_STEP + 1
    p, m, v = (torch.empty(s["grad"].numel(), dtype=torch.float64, device=DEV) for _ in range(3))
    for a in range(0, p.numel(), 1 << 26):
        z = slice(a, min(a + (1 << 26), p.numel()))
        g = s["grad"][z].double() * factor
        m[z] = BETA1 * s["m"][z].double() + (1 - BETA1) * g
        v[z] = BETA2 * s["v"][z].double() + (1 - BETA2) * g ** 2
        keep = 1.0 - LR * DECAY * (torch.arange(z.start, z.stop, device=DEV) < s["split"])
        p[z] = s["master"][z].double() * keep - LR * (m[z] / (1 - BETA1 ** t)) / ((v[z] / (1 - BETA2 ** t)) ** 0.5 + ADAM_EPS)
    got.update(master=p, m=m, v=v, step=None)
    if "param" in s:
        got["param"] = p
    return got
