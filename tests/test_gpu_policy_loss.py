"""et_policy_loss against the float64 definition: classes around every width a kernel may treat differently, both types, each divergence, strides and
alignments, masked rows that hold anything, logits of minus infinity and of the type's lowest value, and the calls a captured or concurrent program makes."""
import numpy as np
import pytest

from loss_util import Rows, close, dev, half_step, rel, round_to
from oracle import losses

pytestmark = pytest.mark.gpu

LOW, HIGH, KL = (float(np.float32(v)) for v in (0.2, 0.28, 0.07))


class Case:
    def __init__(self, rows, C, bf16, kl="sampled", gbf16=None, seed=0, stride=None, gstride=None, skip=0, gskip=0, weighted=False, train=True, in_place=False,
                 spread=2.0, masked=0.25, edit=None):
        rng = np.random.default_rng(seed + 1000 * C + rows)
        self.rows, self.C, self.bf16, self.gbf16, self.kl = rows, C, bf16, bf16 if gbf16 is None else gbf16, kl
        x = rng.normal(0, spread, (rows, C))
        self.label = rng.integers(0, C, rows)
        x[np.arange(rows), self.label] += rng.uniform(0, 2 + np.log(C), rows)
        y = x + rng.normal(0, 0.4, x.shape)
        x, y = round_to(x, bf16), round_to(y, bf16)
        self.x, self.y = x.double().numpy(), y.double().numpy()
        lp = np.array([losses.log_softmax(v)[a] for v, a in zip(self.x, self.label)])
        moved = rng.normal(0, 0.3, rows)
        for border in (np.log(1 - LOW), np.log(1 + HIGH)):       # (within rounding of a border both answers are right)
            moved[np.abs(moved - border) < 1e-3] += 3e-3
        f32 = lambda v: np.float32(v).astype(np.float64)  # noqa: E731
        self.old, self.adv, self.ref = f32(lp - moved), f32(rng.normal(0, 1, rows)), f32(lp + rng.normal(0, 0.3, rows))
        self.weight = f32(rng.uniform(0.1, 1, rows)) if weighted else None
        none = rng.random(rows) < masked
        self.label[none] = rng.choice([-1, -100, C, 2 ** 31 - 1, -2 ** 31], none.sum())
        if edit:
            edit(self)
        self.logits = Rows(rows, C, bf16, stride, skip).put(round_to(self.x, bf16))
        self.refs = Rows(rows, C, bf16, None if stride is None else stride + 1, 1 if skip else 0).put(round_to(self.y, bf16))
        self.grad = None
        if train:
            self.grad = self.logits if in_place else Rows(rows, C, self.gbf16, gstride, gskip)
        self.d = {k: dev(getattr(self, k)) if getattr(self, k) is not None else None for k in ("old", "adv", "ref", "weight")}
        self.d["label"] = dev(self.label, np.int32)

    def call(self, stream=None, ws=None):
        import torch
        from paper_2312_14227_amd import binding as et
        n = et.et_policy_loss_ws_bytes(self.rows)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if ws is None else ws
        self.loss, self.stats, self.logp = (torch.full((k,), 7.0, device="cuda") for k in (1, 3, self.rows))
        at = lambda t: t.data_ptr() if t is not None else 0  # noqa: E731
        kw = {"sampled": dict(ref_logp=at(self.d["ref"])), "full": dict(ref_logits=self.refs.ptr(), ref_stride=self.refs.stride), "none": {}}[self.kl]
        self.p = et.make_policy(at(self.d["old"]), at(self.d["adv"]), weight=at(self.d["weight"]), clip_low=LOW, clip_high=HIGH, kl_coef=KL, logp=at(self.logp),
                                stats=at(self.stats), **kw)
        ty = lambda b: et.ET_BF16 if b else et.ET_F32  # noqa: E731
        self.go = lambda s: et.et_policy_loss(self.rows, self.C, self.logits.ptr(), ty(self.bf16), self.logits.stride, at(self.d["label"]), self.p,
                                              self.grad.ptr() if self.grad else 0, ty(self.gbf16), self.grad.stride if self.grad else 0, at(self.ws), n, s, at(self.loss))
        torch.cuda.synchronize()
        self.go((stream or torch.cuda.current_stream()).cuda_stream)
        torch.cuda.synchronize()
        return self

    def want(self):
        return losses.policy_loss(self.x, self.label, self.old, self.adv, LOW, HIGH, KL, self.ref if self.kl == "sampled" else None,
                                  self.y if self.kl == "full" else None, self.weight)

    def check(self):
        w, R = self.want(), 4 * rel(self.C)
        there = (self.label >= 0) & (self.label < self.C) & np.isfinite(w["logp"])
        lp = w["logp"]
        close(self.logp.cpu().numpy(), lp, R * (1 + np.abs(lp)), "logp")
        # the size of a row's terms: what their sum is off by is relative to them
        n = max(1, ((self.label >= 0) & (self.label < self.C)).sum())
        weight = np.where(there, self.weight if self.weight is not None else 1.0 / n, 0.0)
        with np.errstate(all="ignore"):
            ratio = np.where(there, np.exp(lp - self.old), 0)
            d = np.where(there, self.ref - lp, 0) if self.kl == "sampled" else np.zeros(self.rows)
            size = np.where(there, (1 + np.abs(lp)) * (np.abs(self.adv) * (1 + ratio) + KL * np.exp(d) * (self.kl == "sampled")), 0)
            far, kl_size = np.zeros_like(self.x), np.zeros(self.rows)
            p = np.zeros_like(self.x)
            for r in np.flatnonzero(there):
                p[r] = np.exp(losses.log_softmax(self.x[r]))
                if self.kl == "full":
                    on = p[r] > 0
                    far[r, on] = 1 + 3 * (np.abs(self.x[r, on]) + np.abs(self.y[r, on])).max()
                    kl_size[r] = KL * far[r].max()
        total = (weight * (size + kl_size)).sum()
        close(self.loss.item(), w["loss"], R * total + 1e-30, "loss")
        scale = 1 if self.kl == "none" else 1 / KL
        close(self.stats.cpu().numpy(), w["stats"], [R * total + 1e-30, R * total * scale + 1e-30, 1e-6 * max(1, weight.sum())], "stats")
        if self.grad:
            g = np.where(there[:, None], w["grad"], 0)
            bound = half_step(self.gbf16) * np.abs(g) + R * weight[:, None] * (size[:, None] * p + KL * p * far)
            onehot = np.flatnonzero(there)
            bound[onehot, self.label[onehot]] += R * (weight * size)[onehot] * (1 - p[onehot, self.label[onehot]])
            close(self.grad.host(), w["grad"], bound + 1e-37, "grad")
            assert self.grad.untouched()
        assert self.logits is self.grad or (self.logits.untouched() and np.array_equal(self.logits.host(), self.x, equal_nan=True))
        return self


CLASSES = [1, 2, 3, 5, 8, 31, 63, 64, 65, 200, 255, 256, 257, 511, 513, 1000, 1023, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 8191, 8193, 16383, 16385, 24577, 32767,
           32768, 32769, 50257, 65535, 65537, 100003, 131071, 131073, 200001]


@pytest.mark.parametrize("kl", ["sampled", "full"])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C", CLASSES)
def test_classes(C, bf16, kl):
    Case(5 if C > 300 else 23, C, bf16, kl).call().check()


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 15, 16, 17, 63, 64, 65, 257, 1023, 2047, 2049, 4100, 33000])
@pytest.mark.parametrize("C,bf16", [(7, True), (40, False)])
def test_rows(rows, C, bf16):
    Case(rows, C, bf16, seed=1, weighted=rows % 2 == 0).call().check()


@pytest.mark.parametrize("rows,C", [(700, 1500), (300, 9000), (600, 33000)])
def test_more_rows_than_run_at_once(rows, C):
    Case(rows, C, True, "full" if C == 9000 else "sampled", seed=2, masked=0.1).call().check()


@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
@pytest.mark.parametrize("bf16,gbf16", [(False, True), (True, False)])
@pytest.mark.parametrize("C", [200, 3001, 40001, 150001])
def test_a_gradient_of_another_type(C, bf16, gbf16, kl):
    Case(6, C, bf16, kl, gbf16, weighted=True).call().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C", [13, 200, 4097, 40003, 140001])
@pytest.mark.parametrize("skip,gskip,pad,gpad", [(1, 0, 0, 0), (3, 5, 1, 0), (0, 1, 47, 3), (2, 2, 6, 6), (8, 8, 64, 8)])
def test_strides_and_alignments(C, bf16, skip, gskip, pad, gpad):
    Case(4, C, bf16, "full" if pad == 1 else "sampled", stride=C + pad, gstride=C + gpad, skip=skip, gskip=gskip, masked=0.3).call().check()


@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
@pytest.mark.parametrize("C,bf16", [(200, False), (5001, True), (50257, True), (140001, True), (70001, False)])
def test_in_place(C, bf16, kl):
    Case(7, C, bf16, kl, in_place=True, stride=C + 3, skip=1).call().check()


@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
@pytest.mark.parametrize("C", [200, 4001, 50257, 140001])
def test_without_a_gradient(C, kl):
    Case(9, C, True, kl, train=False).call().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C", [40, 200, 1500, 6000, 40001, 140001])
@pytest.mark.parametrize("kl", ["sampled", "full"])
def test_masked_logits_and_rows(C, bf16, kl):
    """Logits of minus infinity and of the lowest value of the type, rows of nothing but either, confident rows, huge logits, and masked rows full of NaN."""
    lowest = -3.3895313892515355e38 if bf16 else -3.4028234663852886e38

    def edit(c):
        rng = np.random.default_rng(5)
        c.label[:] = rng.integers(0, C, c.rows)
        keep = c.x[np.arange(c.rows), c.label].copy()
        off = rng.random(c.x.shape) < 0.5
        c.x[0][off[0]] = -np.inf
        c.y[0][off[0]] = -np.inf
        c.x[1][off[1]] = lowest
        c.y[1][off[1]] = lowest
        c.x[2] = -np.inf                                      # no distribution
        c.x[3] = lowest                                       # an even one
        c.y[3] = lowest
        c.x[4] = np.where(np.arange(C) == c.label[4], 0, -np.inf)   # one class is left
        c.y[4] = c.x[4]
        c.x[5] = np.where(np.arange(C) == c.label[5], 30, c.x[5])   # p of the label within 1e-8 of 1
        c.y[5] = c.x[5]
        c.x[6] *= 2.0 ** 12                                   # differences of thousands
        c.y[6] = c.x[6]
        c.x[:2][np.arange(2), c.label[:2]] = keep[:2]
        c.y[:2][np.arange(2), c.label[:2]] = keep[:2]
        c.label[7:] = [-1, C, -5]
        c.x[7:9], c.y[7:9] = np.nan, np.inf
        for name in ("old", "adv", "ref"):
            getattr(c, name)[7:9] = np.nan
        c.weight[7:9] = np.nan
        for r in (0, 1, 3, 4, 5, 6):
            c.x[r] = round_to(c.x[r], bf16).double().numpy()
            lp = losses.log_softmax(c.x[r])[c.label[r]]
            c.old[r], c.ref[r] = np.float32(lp - 0.05), np.float32(lp + 0.1)

    Case(10, C, bf16, kl, weighted=True, edit=edit).call().check()


@pytest.mark.parametrize("C", [200, 6000, 70001])
def test_not_a_number_stays_in_its_row(C):
    def edit(c):
        c.label[:] = 1
        c.x[1, 3], c.x[2, 0] = np.nan, np.inf
        c.adv[4] = np.nan

    c = Case(6, C, True, "none", edit=edit, masked=0).call()
    g = c.grad.host()
    assert np.isnan(g[1]).all() and np.isnan(g[4]).all() and np.isnan(g[2]).any() and np.isnan(c.loss.item())
    assert np.isfinite(g[[0, 3, 5]]).all() and np.isnan(c.logp.cpu().numpy()[1])


@pytest.mark.parametrize("weighted", [False, True])
def test_no_row_at_all(weighted):
    c = Case(70, 300, True, masked=1.0, weighted=weighted).call().check()
    assert c.loss.item() == 0 and not c.grad.host().any()


def test_no_divergence_where_its_coefficient_is_zero():
    global KL
    kept, KL = KL, 0.0
    try:
        c = Case(8, 300, False, "sampled", masked=0)
        c.d["ref"].fill_(80.0)                                # (its exponential is beyond float32)
        c.call()
        g, c.kl = c.grad.host(), "none"
        w = c.want()
        assert np.abs(g - w["grad"]).max() <= 1e-5 * np.abs(w["grad"]).max() and abs(c.loss.item() - w["loss"]) <= 1e-5
        assert c.stats[1].item() > 1e30
    finally:
        KL = kept


@pytest.mark.parametrize("C,kl", [(200, "sampled"), (5000, "full"), (140001, "sampled")])
def test_the_same_bits_again_and_on_another_stream(C, kl):
    import torch
    c = Case(90, C, True, kl).call()
    first = [t.clone() for t in (c.loss, c.stats, c.logp, c.grad.flat)]
    side = torch.cuda.Stream()
    c.call(stream=side)
    assert all(torch.equal(a, b) for a, b in zip(first, (c.loss, c.stats, c.logp, c.grad.flat)))


@pytest.mark.parametrize("C,kl", [(200, "sampled"), (9001, "full"), (70001, "none")])
def test_captured_and_replayed(C, kl):
    import torch
    c = Case(33, C, True, kl, weighted=kl == "none").call()
    other = Case(33, C, True, kl, seed=9, weighted=kl == "none").call()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        c.go(torch.cuda.current_stream().cuda_stream)
    want = {False: [t.clone() for t in (c.loss, c.stats, c.logp, c.grad.flat)], True: [t.clone() for t in (other.loss, other.stats, other.logp, other.grad.flat)]}
    mine = [c.logits.flat.clone(), c.refs.flat.clone()] + [t.clone() if t is not None else None for t in c.d.values()]
    theirs = [other.logits.flat, other.refs.flat] + list(other.d.values())
    for k in range(4):
        for t, a, b in zip([c.logits.flat, c.refs.flat] + list(c.d.values()), mine, theirs):
            if t is not None:
                t.copy_(b if k % 2 else a)
        for t in (c.loss, c.stats, c.logp, c.grad.flat):
            t.fill_(-3.0)
        c.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[bool(k % 2)], (c.loss, c.stats, c.logp, c.grad.flat))), k


def test_two_calls_at_once():
    import torch
    a, b = Case(400, 9001, True, "full", seed=1), Case(400, 9001, True, "sampled", seed=2)
    a.call(), b.call()
    want = [t.clone() for c in (a, b) for t in (c.loss, c.grad.flat)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in (a, b):
        c.loss.fill_(0), c.grad.flat.fill_(-3.0)
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip((a, b), streams):
            c.go(s.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, [t for c in (a, b) for t in (c.loss, c.grad.flat)]))


def test_offsets_beyond_32_bits():
    Case(3, 1000, True, stride=1_200_000_001, gstride=1_100_000_003, masked=0).call().check()


@pytest.mark.parametrize("rows,C,bf16,kl,train", [(300, 20000, True, "sampled", True), (260, 16001, False, "none", True), (300, 70001, True, "sampled", True),
                                                  (300, 20000, True, "sampled", False), (257, 9000, False, "full", False), (200, 40000, True, "full", False)])
def test_more_rows_than_compute_units_and_fewer(rows, C, bf16, kl, train):
    Case(rows, C, bf16, kl, seed=3, train=train, masked=0.1).call().check()


@pytest.mark.parametrize("train", [True, False])
@pytest.mark.parametrize("rows,C,bf16", [(8192, 7, True), (8193, 40, False), (20000, 7, False), (40001, 9, True)])
def test_many_rows_of_one_weight(rows, C, bf16, train):
    Case(rows, C, bf16, seed=4, train=train).call().check()


@pytest.mark.parametrize("kl", ["sampled", "full"])
@pytest.mark.parametrize("C,bf16", [(200, True), (3001, False), (40001, True)])
def test_captured_with_many_rows_of_one_weight(C, bf16, kl):
    """More rows than one workgroup counts, with labels that change between replays, so that the weight of a row does."""
    import torch
    rows = 8200 if C < 1000 else 300
    c = Case(rows, C, bf16, kl, seed=5).call()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        c.go(torch.cuda.current_stream().cuda_stream)
    kept = c.d["label"].clone()
    for k in range(3):
        c.d["label"].copy_(kept)
        c.d["label"][:rows // 3 * k] = -1
        c.call(ws=c.ws)
        want = [v.clone() for v in (c.grad.flat, c.logp)]
        loss, stats = c.loss.clone(), c.stats.clone()
        c.grad.flat.fill_(-3.0), c.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want[0], c.grad.flat), k
        assert torch.isfinite(loss).all() and torch.isfinite(stats).all()


@pytest.mark.parametrize("kl", ["sampled", "full"])
@pytest.mark.parametrize("rows,C,bf16,train", [(2100, 50257, True, True), (900, 128000, True, True), (4200, 24001, True, True), (1100, 50257, False, True),
                                               (2100, 50257, True, False)])
def test_more_logits_than_the_caches_hold(rows, C, bf16, train, kl):
    """The same bits as from parts of the rows, small enough to stay in the caches."""
    import torch
    from paper_2312_14227_amd import binding as et
    torch.manual_seed(rows)
    ty, dtype = (et.ET_BF16, torch.bfloat16) if bf16 else (et.ET_F32, torch.float32)
    x = torch.randn(rows, C, device="cuda", dtype=dtype) * 2
    y = x + torch.randn(1, C, device="cuda", dtype=dtype) / 4
    label = torch.randint(0, C, (rows,), device="cuda", dtype=torch.int32)
    label[::7] = -1
    old, adv, weight = -8 + torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda"), torch.rand(rows, device="cuda")

    def run(at, n, grad, logp):
        ws, loss = torch.full((et.et_policy_loss_ws_bytes(n),), 0xFF, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda")
        kw = dict(ref_logits=y[at:].data_ptr(), ref_stride=C) if kl == "full" else dict(ref_logp=old[at:].data_ptr())
        p = et.make_policy(old[at:].data_ptr(), adv[at:].data_ptr(), weight=weight[at:].data_ptr(), clip_low=LOW, clip_high=HIGH, kl_coef=KL,
                           logp=logp[at:].data_ptr(), **kw)
        et.et_policy_loss(n, C, x[at:].data_ptr(), ty, C, label[at:].data_ptr(), p, grad[at:].data_ptr() if train else 0, ty, C, ws.data_ptr(), ws.numel(),
                          torch.cuda.current_stream().cuda_stream, loss.data_ptr())
        torch.cuda.synchronize()
        return loss.item()

    outs = [(torch.full_like(x, 7.0), torch.full((rows,), 7.0, device="cuda")) for _ in range(2)]
    whole = run(0, rows, *outs[0])
    step = (rows + 2) // 3
    parts = [run(at, min(step, rows - at), *outs[1]) for at in range(0, rows, step)]
    assert torch.equal(outs[0][1], outs[1][1]) and torch.equal(outs[0][0], outs[1][0])
    assert abs(whole - sum(parts)) <= 1e-5 * sum(abs(v) for v in parts) + 1e-4


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C", [200, 6000, 140001])
def test_a_class_that_the_reference_gives_probability_zero(C, bf16):
    """1e30 stands for the infinite difference: the divergence is p of that class times that, and the other rows' stay as they are."""
    def edit(c):
        c.label[:] = 3
        c.x[1, 9], c.y[1, 9] = c.x[1].max(), -np.inf
        c.x[2, 9], c.y[2, 9] = -np.inf, -np.inf

    c = Case(4, C, bf16, "full", edit=edit, masked=0).call()
    p = np.exp(losses.log_softmax(c.x[1]))
    kl = c.stats[1].item()
    assert abs(kl - p[9] * 1e30 / 4) <= 1e-4 * p[9] * 1e30 / 4
    g = c.grad.host()
    assert np.isfinite(g).all() and abs(g[1, 9] - KL / 4 * p[9] * (1 - p[9]) * 1e30) <= (1e-4 + half_step(bf16)) * KL / 4 * p[9] * 1e30
    kept, c.y[1, 9] = c.y[1, 9], c.x[1, 9]
    w = c.want()["grad"]
    c.y[1, 9] = kept
    assert np.abs(g[[0, 2, 3]] - w[[0, 2, 3]]).max() <= 2 * half_step(bf16) * np.abs(w).max() + 1e-5 * np.abs(w).max()


@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
@pytest.mark.parametrize("rows,C,bf16,kw", [(4100, 1000, True, {}), (4097, 512, False, dict(weighted=True)), (5001, 1, True, {}), (4500, 130, True, dict(in_place=True, stride=133, skip=1)),
                                            (4300, 220, False, dict(gbf16=True, gstride=301, gskip=3)), (4300, 510, True, dict(gbf16=False, stride=1030, skip=5)),
                                            (9000, 77, False, dict(train=False)), (4099, 255, False, dict(masked=0.9)), (2100, 1000, True, {})])
def test_many_short_rows(rows, C, bf16, kw, kl):
    Case(rows, C, bf16, kl, seed=6, **kw).call().check()


@pytest.mark.parametrize("kl", ["sampled", "full"])
def test_many_short_rows_give_what_few_do(kl):
    """Rows with masks, nothing, NaN and huge values among many: every row's outputs as from a call of a few."""
    def edit(c):
        rng = np.random.default_rng(1)
        c.x[5::50] = -np.inf
        c.x[6::50][rng.random(c.x[6::50].shape) < 0.7] = -np.inf
        c.y[6::50] = c.x[6::50]
        c.x[7::50] *= 8.0
        c.x[8::50, 0] = np.nan

    c = Case(4500, 201, True, kl, seed=7, weighted=True, edit=edit).call()
    g, lp = c.grad.host(), c.logp.cpu().numpy()
    rows = 1000
    for at in range(0, 4500, rows):
        n = min(rows, 4500 - at)
        part = Case(n, 201, True, kl, seed=8, weighted=True, masked=0)
        for name in ("x", "y", "label", "old", "adv", "ref", "weight"):
            setattr(part, name, getattr(c, name)[at:at + n])
        part.logits.put(round_to(part.x, True)), part.refs.put(round_to(part.y, True))
        part.d = {k: dev(getattr(part, k)) for k in ("old", "adv", "ref", "weight")}
        part.d["label"] = dev(part.label, np.int32)
        part.call()
        # (two kernels may contract their products differently: a step of the type, and of float32 some)
        np.testing.assert_allclose(part.grad.host(), g[at:at + n], rtol=2.0 ** -7, atol=1e-12)
        np.testing.assert_allclose(part.logp.cpu().numpy(), lp[at:at + n], rtol=1e-5, atol=1e-6)
    assert np.isnan(g[8::50]).any() and not np.isnan(g[9::50]).any()
