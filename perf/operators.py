"""Performance cases of the stand-alone operators around a training step: the clipped policy loss and the preference loss with their
gradients, the norm of many gradients and clipping by it.

`own` false computes them in their plain form; `own` true makes the calls of the C ABI's Python binding.
"""
import math

import numpy as np
import torch

own = False

CLASSES = 200      # of the framework's image classifiers
MOST = 1 << 30     # logits of the largest case, rounded up


# ---------------------------------------------------------------------------------------------------- the cases
def _policy(name, rows, classes, dtype, kl, pad=0, weighted=False, masked=0.0, train=True):
    return dict(name=name, op="policy", rows=rows, classes=classes, pad=pad, dtype=dtype, kl=kl, weighted=weighted, masked=masked, train=train)


def _preference(name, pairs, longest, classes, dtype, pad=0, masked=0.3, smoothing=0.0, train=True):
    return dict(name=name, op="preference", pairs=pairs, longest=longest, classes=classes, pad=pad, dtype=dtype, masked=masked, smoothing=smoothing,
                train=train)


def _grads(name, op, tensors, dtype, total=0, clipped=True):
    return dict(name=name, op=op, tensors=tensors, dtype=dtype, total=total, clipped=clipped)


def listed():
    """`pad`: elements between the end of a row of logits and the next row; `masked`: share of the rows without a label; `longest`: of a
    preference case's sequences (0: each is one row); `tensors`: a model's name, or a number of ragged tensors of `total` elements in all."""
    return [
        # The step of the image classifiers: 64 rows of float32 logits, all latency.
        _policy("policy_b64_c200", 64, CLASSES, "f32", "sampled"),
        # Scoring a batch of tokens without a gradient: one read of the logits.
        _policy("policy_r2048_v32000_forward", 2048, 32000, "bf16", "sampled", masked=0.2, train=False),
        # The exact divergence from the reference model's distribution; odd classes in padded rows, padding tokens masked.
        _policy("policy_r4096_v50257_full_kl", 4096, 50257, "bf16", "full", pad=47, masked=0.1),
        # The largest: a micro-batch of 8192 tokens over a large vocabulary, each token weighted (a mean per answer).
        _policy("policy_r8192_v128000", 8192, 128000, "bf16", "sampled", weighted=True),
        # The step of the image classifiers on 32 pairs of images.
        _preference("preference_b64_c200", 32, 0, CLASSES, "f32", masked=0.0),
        # Four pairs of short answers of unequal lengths behind masked prompts.
        _preference("preference_p4_v32000", 4, 300, 32000, "bf16", smoothing=0.1),
        # The largest: eight pairs of answers up to 1000 tokens, an odd vocabulary without padding: rows start at any even address.
        _preference("preference_p8_v100003", 8, 1000, 100003, "bf16"),
        # The smallest model of the framework: four matrices of a perceptron.
        _grads("norm_mlp", "norm", "mlp", "f32"),
        # Ragged bf16 tensors that start anywhere.
        _grads("norm_37_ragged_bf16", "norm", "37", "bf16", total=60_000_000),
        # The framework's largest model: 296 tensors, 303 million gradients.
        _grads("norm_vit_l", "norm", "vit_l", "f32"),
        # Many small tensors: 158 of an inverted-residual network, 2.5 million gradients.
        _grads("clip_mobilenetv2", "clip", "mobilenetv2", "f32"),
        # The base transformer's 152 tensors, 86 million gradients.
        _grads("clip_vit_b", "clip", "vit_b", "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        u, dtype = rng.random(), rng.choice(("bf16", "bf16", "f32"))
        pad = rng.choice((0, 0, rng.randint(1, 63)))
        train = rng.random() < 0.8
        if u < 0.35:
            case = _policy("", _log_int(rng, 1, 16384), _log_int(rng, 2, 160000), dtype, rng.choice(("none", "sampled", "sampled", "full")), pad,
                           rng.random() < 0.4, rng.choice((0.0, rng.uniform(0.0, 0.6))), train)
            size = case["rows"] * case["classes"]
        elif u < 0.65:
            case = _preference("", _log_int(rng, 1, 128), rng.choice((0, _log_int(rng, 2, 2000))), _log_int(rng, 2, 160000), dtype, pad,
                               rng.choice((0.0, rng.uniform(0.0, 0.6))), rng.choice((0.0, rng.uniform(0.01, 0.2))), train)
            size = _offsets(case)[-1] * case["classes"]
        else:
            tensors = rng.choice(("mlp", "vit_b", "mobilenetv2", "vit_small") + (str(_log_int(rng, 1, 700)),) * 3)
            total = _log_int(rng, 1000, 300_000_000) if tensors.isdigit() else 0
            case = _grads("", rng.choice(("norm", "clip")), tensors, dtype, total, rng.random() < 0.75)
            size = sum(_sizes(case))
        case.pop("name")
        if 64 <= size <= MOST * (0.5 if dtype == "f32" or case.get("kl") == "full" else 0.97):
            return case


def _offsets(case):
    """Where a preference case's sequences begin: lengths spread over their logarithm, one in twelve empty."""
    n = 2 * case["pairs"]
    if case["longest"] == 0:
        return list(range(n + 1))
    rng = np.random.RandomState(case["pairs"] * 7919 + case["longest"])
    lengths = np.exp(rng.uniform(math.log(max(1.0, case["longest"] / 6)), math.log(case["longest"]), n)).round().astype(int)
    lengths[rng.rand(n) < 1 / 12] = 0
    lengths[0] = case["longest"]
    return np.concatenate([[0], np.cumsum(lengths)]).tolist()


def _vit(width, mlp, blocks, tokens, patch_dim, classes):
    block = [width, width, 3 * width * width, 3 * width, width * width, width, width, width, mlp * width, mlp, width * mlp, width]
    return [width * patch_dim, width, width, tokens * width] + block * blocks + [width, width, classes * width, classes]


def _mobilenet():
    out, cin = [32 * 27, 32, 32], 32
    for t, c, n, _ in ((1, 16, 1, 1), (6, 24, 2, 2), (6, 32, 3, 2), (6, 64, 4, 2), (6, 96, 3, 1), (6, 160, 3, 2), (6, 320, 1, 1)):
        for _ in range(n):
            hid = t * cin
            out += ([hid * cin, hid, hid] if t != 1 else []) + [hid * 9, hid, hid, c * hid, c, c]
            cin = c
    return out + [1280 * cin, 1280, 1280, CLASSES * 1280, CLASSES]


def _sizes(case):
    """Elements of each gradient."""
    name = case["tensors"]
    if name.isdigit():
        rng = np.random.RandomState(int(name) * 31 + case["total"] % 1009)
        share = np.exp(rng.uniform(0.0, 7.0, int(name)))
        return np.maximum(1, share / share.sum() * case["total"]).astype(np.int64).tolist()
    return {"mlp": lambda: [256 * 256] * 3 + [10 * 256], "vit_small": lambda: _vit(192, 320, 2, 197, 200, 56),
            "vit_b": lambda: _vit(768, 3072, 12, 197, 768, CLASSES), "vit_l": lambda: _vit(1024, 4096, 24, 197, 768, CLASSES),
            "mobilenetv2": _mobilenet}[name]()


def _places(case):
    """Where each gradient starts in its arena: at multiples of 64 elements for a model, right behind the last one otherwise."""
    sizes, align = _sizes(case), 1 if case["tensors"].isdigit() else 64
    ends = np.cumsum([(s + align - 1) // align * align for s in sizes])
    return [0] + ends[:-1].tolist(), sizes, int(ends[-1])


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---------------------------------------------------------------------------------------------------- inputs
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
BETA = 0.1


def _logits(case, rows, gen):
    """Logits as a trained model gives them: normal, and the label's among the larger ones; labels; the label's log probability."""
    C, ld = case["classes"], case["classes"] + case["pad"]
    label = torch.randint(0, C, (rows,), generator=gen, device="cuda")
    logits = torch.empty(rows, ld, dtype=_dtype(case), device="cuda")
    logp = torch.empty(rows, dtype=torch.float64, device="cuda")
    above = torch.rand(rows, generator=gen, device="cuda") * (2.0 + math.log(C))
    per = max(1, (1 << 27) // ld)
    for r in range(0, rows, per):
        x = torch.randn(min(per, rows - r), ld, generator=gen, device="cuda") * 2.0
        at = label[r:r + per, None]
        x.scatter_add_(1, at, above[r:r + per, None])
        logits[r:r + per] = x
        x = logits[r:r + per, :C].float()
        logp[r:r + per] = (x.gather(1, at).double() - torch.logsumexp(x, 1, keepdim=True).double())[:, 0]
    none = torch.rand(rows, generator=gen, device="cuda") < case["masked"]
    return logits, torch.where(none, -1, label).to(torch.int32), logp


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    normal = lambda n, std: torch.randn(n, generator=gen, device="cuda", dtype=torch.float64) * std  # noqa: E731
    if case["op"] in ("norm", "clip"):
        begin, sizes, total = _places(case)
        s["arena"] = torch.randn(total, generator=gen, device="cuda").mul_(1e-2).to(_dtype(case))
        s["grads"] = [s["arena"][b:b + n] for b, n in zip(begin, sizes)]
        # about a third of the norm, or beyond it
        s["max_norm"] = 1e-2 * math.sqrt(total) * (0.3 if case["clipped"] else 3.0)
        if case["op"] == "clip":
            s["out"] = torch.zeros_like(s["arena"])
            s["outs"] = [s["out"][b:b + n] for b, n in zip(begin, sizes)]
    else:
        rows = case["rows"] if case["op"] == "policy" else _offsets(case)[-1]
        s["rows"] = rows
        s["logits"], s["label"], logp = _logits(case, rows, gen)
        if case["train"]:
            s["grad"] = torch.zeros_like(s["logits"])
        if case["op"] == "policy":
            # the policy has moved a little since the tokens were drawn.  Within rounding of the borders of the clipping two right answers
            # differ by the whole gradient of a row, so no ratio lies there
            moved = normal(rows, 0.25)
            for border in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
                moved = torch.where((moved - border).abs() < 1e-3, moved + 3e-3, moved)
            s["old"] = (logp - moved).float()
            s["ref"] = (logp + normal(rows, 0.3)).float()
            s["advantage"] = normal(rows, 1.0).float()
            answer = torch.arange(rows, device="cuda") // 97
            s["weight"] = (1.0 / (torch.bincount(answer)[answer] * (answer[-1] + 1))).float() if case["weighted"] else None
            if case["kl"] == "full":
                s["ref_logits"] = s["logits"].clone()
                per = max(1, (1 << 27) // s["logits"].shape[1])
                for r in range(0, rows, per):
                    part = s["ref_logits"][r:r + per]
                    part += torch.randn(part.shape, generator=gen, device="cuda").to(part.dtype) * 0.3
        else:
            off = torch.tensor(_offsets(case), device="cuda")
            total = torch.cat([logp.new_zeros(1), torch.where(s["label"] >= 0, logp, 0.0).cumsum(0)])
            seq = total[off[1:]] - total[off[:-1]]
            ref = seq + normal(2 * case["pairs"], 5.0)
            # no margin lies within rounding of zero, where pairs are counted
            margin = (seq - ref).reshape(-1, 2)
            ref[0::2] += torch.where((margin[:, 0] - margin[:, 1]).abs() < 0.1, 0.5, 0.0)
            s["ref"], s["offsets"] = ref.float(), off.to(torch.int32)
    if own:
        s["call"] = _bound(s)   # what a program holds besides: the workspace, the outputs, its argument structs
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _rows_plain(x, label):
    """exp(x - max), its sum, and per row whether there is a label, where, its log probability and log sum exp (in 64 bits: sequences add
    hundreds of the former, whose difference counts)."""
    C = x.shape[1]
    there = (label >= 0) & (label < C)
    at = torch.where(there, label, 0).long()[:, None]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    lse = top.double() + torch.log(total.double())
    return e, total, there, at, (x.gather(1, at).double() - lse)[:, 0], lse


def _policy_plain(s):
    x = s["logits"][:, :s["classes"]].float()
    e, total, there, at, lp, lse = _rows_plain(x, s["label"])
    w = torch.where(there, s["weight"] if s["weight"] is not None else 1.0 / there.sum().clamp(min=1).float(), 0.0)
    rho, A = torch.exp(lp - s["old"]).float(), s["advantage"]
    over = ((A > 0) & (rho > 1 + CLIP_HIGH)) | ((A < 0) & (rho < 1 - CLIP_LOW))
    surrogate = torch.where(A > 0, rho.clamp(max=1 + CLIP_HIGH), rho.clamp(min=1 - CLIP_LOW)) * A
    g, kl = -torch.where(over, 0.0, rho * A), torch.zeros_like(A)
    if s["kl"] == "sampled":
        d = s["ref"] - lp
        kl, g = (torch.expm1(d) - d).float(), g - KL * torch.expm1(d).float()
    elif s["kl"] == "full":
        y = s["ref_logits"][:, :s["classes"]].float()
        y_top = y.amax(1, keepdim=True)
        y_lse = y_top.double() + torch.log(torch.exp(y - y_top).sum(1, keepdim=True).double())
        apart = x - y - (lse - y_lse).float()   # log p - log q
        kl = (e * apart).sum(1) / total[:, 0]
    mean = lambda v: (w * torch.where(there, v, 0.0)).double().sum().float()  # noqa: E731
    out = {"loss": mean(KL * kl - surrogate), "stats": torch.stack([mean(surrogate), mean(kl), mean(over.float())]), "logp": torch.where(there, lp, 0.0).float()}
    if s["train"]:
        g = torch.where(there, w * g, 0.0)[:, None]
        if s["kl"] == "full":
            apart -= kl[:, None]
            e *= (KL * w[:, None] * apart - g) / total
        else:
            e *= -g / total
        e.scatter_add_(1, at, g)
        out["grad"] = torch.where(there[:, None], e, 0.0).to(s["logits"].dtype)
    return out


def _preference_plain(s):
    x = s["logits"][:, :s["classes"]].float()
    e, total, there, at, lp, _ = _rows_plain(x, s["label"])
    off = s["offsets"].long()
    run = torch.cat([torch.zeros(1, dtype=torch.float64, device=x.device), torch.where(there, lp, 0.0).cumsum(0)])
    seq = run[off[1:]] - run[off[:-1]]
    gain = (seq - s["ref"]).reshape(-1, 2)
    z = BETA * (gain[:, 0] - gain[:, 1])
    eps = s["smoothing"]
    up, down = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
    loss = ((1 - eps) * torch.log1p(torch.exp(-z)) + eps * torch.log1p(torch.exp(z))).mean()
    out = {"loss": loss.float(), "stats": torch.stack([z.mean().float(), (z > 0).float().mean()]), "logp": seq.float()}
    if s["train"]:
        dz = (eps * up - (1 - eps) * down) * (BETA / s["pairs"])
        of = (torch.arange(x.shape[0], device=x.device)[:, None] >= off[None, 1:]).sum(1)
        g = torch.where(there, torch.stack([dz, -dz], 1).reshape(-1)[of], 0.0).float()[:, None]
        e *= -g / total
        e.scatter_add_(1, at, g)
        out["grad"] = e.to(s["logits"].dtype)
    return out


def _norm_plain(s):
    each = torch.stack([g.float().square().sum() for g in s["grads"]])
    return each.double().sum().sqrt(), {"norm": each.double().sum().sqrt().float(), "tensor_norm": each.sqrt()}


def _clip_plain(s):
    norm, out = _norm_plain(s)
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
    out["grads"] = (s["arena"].float() * scale).to(s["arena"].dtype)
    return out


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _bound(s):
    from paper_2312_14227_amd import binding as et
    stream = torch.cuda.current_stream().cuda_stream
    f32 = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    room = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
    at = lambda t: t.data_ptr() if t is not None else 0  # noqa: E731
    dtype = et.ET_BF16 if s["dtype"] == "bf16" else et.ET_F32
    if s["op"] in ("norm", "clip"):
        numel = et.sizes([g.numel() for g in s["grads"]])
        grads = et.pointers([g.data_ptr() for g in s["grads"]])
        ws = room(et.et_grad_norm_ws_bytes(numel))
        norm, each = f32(1), f32(len(s["grads"]))
        out = {"norm": norm[0], "tensor_norm": each}
        if s["op"] == "norm":
            return lambda: et.et_grad_norm(grads, numel, dtype, at(ws), ws.numel(), stream, at(norm), at(each)), out
        # the arena is scaled as one piece, with what lies between its tensors
        whole = et.pointers([at(s["arena"])]), et.pointers([at(s["out"])]), et.sizes([s["arena"].numel()])
        out["grads"] = s["out"]

        def clip():
            et.et_grad_norm(grads, numel, dtype, at(ws), ws.numel(), stream, at(norm), at(each))
            et.et_grad_scale(*whole, dtype, at(norm), s["max_norm"], stream)
        return clip, out
    rows, C, ld, grad, loss = s["rows"], s["classes"], s["logits"].shape[1], s.get("grad"), f32(1)
    out = {"loss": loss[0]} | ({"grad": grad[:, :C]} if grad is not None else {})
    if s["op"] == "policy":
        ws = room(et.et_policy_loss_ws_bytes(rows))
        out["stats"], out["logp"] = f32(3), f32(rows)
        kl = {"sampled": dict(ref_logp=at(s["ref"])), "full": dict(ref_logits=at(s.get("ref_logits")), ref_stride=ld), "none": {}}[s["kl"]]
        p = et.make_policy(at(s["old"]), at(s["advantage"]), weight=at(s["weight"]), clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL,
                           logp=at(out["logp"]), stats=at(out["stats"]), **kl)
        return lambda: et.et_policy_loss(rows, C, at(s["logits"]), dtype, ld, at(s["label"]), p, at(grad), dtype, ld, at(ws), ws.numel(), stream,
                                         at(loss)), out
    ws = room(et.et_preference_loss_ws_bytes(rows, s["pairs"]))
    out["stats"], out["logp"] = f32(2), f32(2 * s["pairs"])
    # (every row a sequence: the call takes that without offsets)
    p = et.make_preference(at(s["offsets"]) if s["longest"] else 0, ref_logp=at(s["ref"]), beta=BETA, label_smoothing=s["smoothing"], logp=at(out["logp"]), stats=at(out["stats"]))
    return lambda: et.et_preference_loss(rows, s["pairs"], C, at(s["logits"]), dtype, ld, at(s["label"]), p, at(grad), dtype, ld, at(ws), ws.numel(),
                                         stream, at(loss)), out


def run(state):
    if own:
        call, out = state["call"]
        call()
        return out
    return {"policy": _policy_plain, "preference": _preference_plain, "norm": lambda s: _norm_plain(s)[1], "clip": _clip_plain}[state["op"]](state)


# ---------------------------------------------------------------------------------------------------- work, and the answers in 64 bits
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("norm", "clip"):
        n = sum(_sizes(case))
        return {"bytes": n * size * (2 if case["op"] == "clip" else 1) + 4 * len(_sizes(case)), "flops": n * (3 if case["op"] == "clip" else 2)}
    rows = case["rows"] if case["op"] == "policy" else _offsets(case)[-1]
    there = rows * (1 - case["masked"])   # a row without a label has a gradient of zeros and needs no logits
    matrices = there * (2 if case.get("kl") == "full" else 1) + rows * case["train"]
    flops = there * case["classes"] * ((10 if case.get("kl") == "full" else 4) + (3 if case["train"] else 0))
    return {"bytes": matrices * case["classes"] * size + 20 * rows, "flops": flops}


def exact(case, seed):
    global own
    kept, own = own, False
    s = prepare(case, seed)
    own = kept
    if case["op"] in ("norm", "clip"):
        begin, sizes, _ = _places(case)
        each = torch.tensor([float(torch.linalg.vector_norm(s["arena"][b:b + n].double())) for b, n in zip(begin, sizes)], dtype=torch.float64)
        norm = math.sqrt(math.fsum(v * v for v in each.tolist()))
        out = {"norm": torch.tensor(norm, dtype=torch.float64), "tensor_norm": each}
        if case["op"] == "clip":
            out["grads"] = s["arena"].double() * min(1.0, s["max_norm"] / norm)
        return out
    rows, C = s["rows"], case["classes"]
    grad = torch.zeros(rows, C, dtype=torch.float64, device="cuda") if case["train"] else None
    per = max(1, (1 << 26) // C)
    label = s["label"].long()
    there = label >= 0
    lp = torch.zeros(rows, dtype=torch.float64, device="cuda")
    for r in range(0, rows, per):   # p in the gradient's place
        x = torch.log_softmax(s["logits"][r:r + per, :C].double(), 1)
        lp[r:r + per] = x.gather(1, label[r:r + per, None].clamp(min=0))[:, 0]
        if grad is not None:
            grad[r:r + per] = x.exp()
    lp[~there] = 0.0
    if case["op"] == "policy":
        n = int(there.sum())
        w = (s["weight"].double() if s["weight"] is not None else torch.full_like(lp, 1.0 / max(1, n))) * there
        A, rho = s["advantage"].double(), (lp - s["old"].double()).exp()
        # as float32 numbers, which is what the call takes
        low, high = 1 - float(np.float32(CLIP_LOW)), 1 + float(np.float32(CLIP_HIGH))
        coef = float(np.float32(KL))
        best = torch.minimum(rho * A, rho.clamp(low, high) * A)
        cut = best < rho * A
        kl, slope = torch.zeros_like(lp), -torch.where(cut, 0.0, rho * A)
        if case["kl"] == "sampled":
            d = s["ref"].double() - lp
            kl, slope = d.exp() - d - 1, slope + coef * (1 - d.exp())
        for r in range(0, rows if case["kl"] == "full" else 0, per):
            p = torch.log_softmax(s["logits"][r:r + per, :C].double(), 1)
            far = p - torch.log_softmax(s["ref_logits"][r:r + per, :C].double(), 1)
            p = p.exp()
            kl[r:r + per] = (p * far).sum(1)
            if grad is not None:
                grad[r:r + per] = p * (coef * (far - kl[r:r + per, None]) - slope[r:r + per, None])
        if grad is not None:
            if case["kl"] != "full":
                grad *= -slope[:, None]
            grad[torch.arange(rows, device="cuda")[there], label[there]] += slope[there]
            grad *= w[:, None]
        mean = lambda v: (w * torch.where(there, v, 0.0)).sum()  # noqa: E731
        out = {"loss": mean(coef * kl - best), "stats": torch.stack([mean(best), mean(kl), mean(cut.double())]), "logp": lp}
    else:
        off = _offsets(case)
        seq = torch.tensor([math.fsum(lp[a:b].tolist()) for a, b in zip(off, off[1:])], dtype=torch.float64, device="cuda")
        beta, eps = float(np.float32(BETA)), float(np.float32(case["smoothing"]))
        z = beta * ((seq[0::2] - s["ref"][0::2].double()) - (seq[1::2] - s["ref"][1::2].double()))
        log_up, log_down = torch.nn.functional.logsigmoid(z), torch.nn.functional.logsigmoid(-z)
        out = {"loss": -((1 - eps) * log_up + eps * log_down).mean(), "stats": torch.stack([z.mean(), (z > 0).double().mean()]), "logp": seq}
        if grad is not None:
            d = (eps * log_up.exp() - (1 - eps) * log_down.exp()) * beta / case["pairs"]
            for i, (a, b) in enumerate(zip(off, off[1:])):
                grad[a:b] *= (-d if i % 2 == 0 else d)[i // 2] * there[a:b, None]
                k = torch.arange(a, b, device="cuda")[there[a:b]]
                grad[k, label[k]] += (d if i % 2 == 0 else -d)[i // 2]
    if grad is not None:
        out["grad"] = grad
    return out
