"""et_preference_loss against the float64 definition: lengths from none to many rows, classes around every width a kernel may treat differently, masked tokens,
rows of no sequence, offsets that make no sense, and the calls a captured program makes."""
import numpy as np
import pytest

from loss_util import Rows, close, dev, half_step, rel, round_to
from oracle import losses

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, lengths, C, bf16, gbf16=None, seed=0, front=0, behind=0, beta=0.1, eps=0.0, ref=True, pad=0, gpad=0, skip=0, gskip=0, masked=0.3,
                 train=True, in_place=False, offsets=True, edit=None):
        self.pairs, self.C, self.bf16, self.gbf16 = len(lengths) // 2, C, bf16, bf16 if gbf16 is None else gbf16
        self.offsets = (front + np.concatenate([[0], np.cumsum(lengths)])).astype(int)
        self.given = offsets
        self.rows = max(1, int(self.offsets[-1]) + behind)
        self.beta, self.eps = float(np.float32(beta)), float(np.float32(eps))
        rng = np.random.default_rng(seed + C)
        x = rng.normal(0, 2, (self.rows, C))
        self.label = rng.integers(0, C, self.rows)
        x[np.arange(self.rows), self.label] += rng.uniform(0, 2 + np.log(C), self.rows)
        none = rng.random(self.rows) < masked
        self.label[none] = rng.choice([-1, C, -2 ** 31], none.sum())
        self.x = round_to(x, bf16).double().numpy()
        self.ref = None
        if ref:
            L = losses.preference_loss(self.x, self.label, self.offsets, 1.0)["logp"]
            self.ref = np.float32(L + rng.normal(0, 4, L.size)).astype(np.float64)
        if edit:
            edit(self)
        self.logits = Rows(self.rows, C, bf16, C + pad, skip).put(round_to(self.x, bf16))
        self.grad = (self.logits if in_place else Rows(self.rows, C, self.gbf16, C + gpad, gskip)) if train else None
        self.d = [dev(self.label, np.int32), dev(self.offsets, np.int32), dev(self.ref) if ref else None]

    def call(self, stream=None):
        import torch
        from paper_2312_14227_amd import binding as et
        n = et.et_preference_loss_ws_bytes(self.rows, self.pairs)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        self.loss, self.stats, self.logp = (torch.full((k,), 7.0, device="cuda") for k in (1, 2, 2 * self.pairs))
        at = lambda t: t.data_ptr() if t is not None else 0  # noqa: E731
        p = et.make_preference(at(self.d[1]) if self.given else 0, at(self.d[2]), self.beta, self.eps, at(self.logp), at(self.stats))
        ty = lambda b: et.ET_BF16 if b else et.ET_F32  # noqa: E731
        self.go = lambda s: et.et_preference_loss(self.rows, self.pairs, self.C, self.logits.ptr(), ty(self.bf16), self.logits.stride, at(self.d[0]), p,
                                                  self.grad.ptr() if self.grad else 0, ty(self.gbf16), self.grad.stride if self.grad else 0, at(self.ws), n, s,
                                                  at(self.loss))
        torch.cuda.synchronize()
        self.go((stream or torch.cuda.current_stream()).cuda_stream)
        torch.cuda.synchronize()
        return self

    def outputs(self):
        return [self.loss, self.stats, self.logp] + ([self.grad.flat] if self.grad else [])

    def check(self):
        w, R = losses.preference_loss(self.x, self.label, self.offsets, self.beta, self.eps, self.ref), 4 * rel(self.C)
        L, n = w["logp"], np.diff(self.offsets)
        size = np.zeros(L.size)                                # sums of |log p| + 1 per row
        for i in range(L.size):
            for r in range(self.offsets[i], self.offsets[i + 1]):
                if 0 <= self.label[r] < self.C:
                    lp = losses.log_softmax(self.x[r])[self.label[r]]
                    size[i] += 1 + (abs(lp) if np.isfinite(lp) else 0)
        close(self.logp.cpu().numpy(), L, R * size + 2.0 ** -24 * np.abs(L), "logp")
        off = R * self.beta * (size[0::2] + size[1::2]) + 2.0 ** -23 * np.abs(w["z"])
        close(self.loss.item(), w["loss"], off.mean() + R * abs(w["loss"]), "loss")
        near = np.mean(np.abs(w["z"]) <= off) if self.ref is not None else 0
        close(self.stats.cpu().numpy(), w["stats"], [off.mean(), near + 1e-6], "stats")
        if not self.grad:
            return self
        before = self.x if self.grad is self.logits else np.full((self.rows, self.C), self.grad.fill)
        g = np.where(np.isnan(w["grad"]), before, w["grad"])
        bound = np.zeros_like(g)
        for i in range(L.size):
            d = self.beta / self.pairs * min(1.0, off[i // 2] + R)   # what the pair's factor is off by: the sigmoid's slope is at most 1/4
            for r in range(self.offsets[i], self.offsets[i + 1]):
                unit = np.abs(w["grad"][r]) / max(1e-300, np.abs(w["grad"][r]).max())
                bound[r] = half_step(self.gbf16) * np.abs(w["grad"][r]) + R * np.abs(w["grad"][r]) + d * unit + 1e-37
        close(self.grad.host(), g, bound, "grad")
        assert self.grad.untouched()
        return self


CLASSES = [1, 2, 3, 9, 63, 65, 200, 256, 1000, 1025, 2049, 4096, 4099, 8191, 16385, 32768, 50257, 65537, 131073, 200001]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C", CLASSES)
def test_classes(C, bf16):
    Case([2, 3, 1, 0], C, bf16, front=1, behind=2).call().check()


LENGTHS = [[1, 1], [0, 0], [0, 1], [1, 0], [5, 0, 0, 7], [1] * 64, [300, 200], [1, 2000, 700, 3], list(range(40)), [0] * 20 + [3, 4], [257, 255, 256, 1]]


@pytest.mark.parametrize("lengths", range(len(LENGTHS)))
@pytest.mark.parametrize("C,bf16", [(11, False), (300, True)])
def test_lengths(lengths, C, bf16):
    Case(LENGTHS[lengths], C, bf16, behind=lengths % 3, eps=0.1 if lengths % 2 else 0.0, beta=0.02).call().check()


@pytest.mark.parametrize("pairs", [1, 2, 31, 32, 33, 500, 3000])
@pytest.mark.parametrize("C,bf16", [(200, False), (3000, True)])
def test_every_row_a_sequence(pairs, C, bf16):
    if pairs * C <= 200000:
        Case([1] * (2 * pairs), C, bf16, offsets=False, masked=0.1, beta=0.7).call().check()


@pytest.mark.parametrize("ref", [False, True])
@pytest.mark.parametrize("eps", [0.0, 0.2, 1.0])
@pytest.mark.parametrize("beta", [0.05, 3.0])
def test_coefficients(beta, eps, ref):
    Case([4, 6, 2, 2, 5, 1], 77, False, ref=ref, eps=eps, beta=beta).call().check()


@pytest.mark.parametrize("bf16,gbf16", [(False, True), (True, False)])
@pytest.mark.parametrize("C", [200, 3001, 40001, 150001])
def test_a_gradient_of_another_type(C, bf16, gbf16):
    Case([2, 3], C, bf16, gbf16, behind=1).call().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C", [13, 200, 4097, 40003])
@pytest.mark.parametrize("skip,gskip,pad,gpad", [(1, 0, 0, 0), (3, 5, 1, 0), (0, 1, 47, 3), (2, 2, 6, 6)])
def test_strides_and_alignments(C, bf16, skip, gskip, pad, gpad):
    Case([3, 2], C, bf16, skip=skip, gskip=gskip, pad=pad, gpad=gpad, front=1, behind=1).call().check()


@pytest.mark.parametrize("C,bf16", [(200, False), (5001, True), (50257, True), (140001, True)])
def test_in_place(C, bf16):
    Case([3, 2, 0, 1], C, bf16, in_place=True, pad=3, skip=1, front=1, behind=1).call().check()


@pytest.mark.parametrize("C", [200, 5001, 140001])
def test_without_a_gradient(C):
    Case([3, 2, 0, 1], C, True, train=False, behind=2).call().check()


def test_more_rows_than_run_at_once():
    Case([900, 1500, 40, 2000], 600, True, beta=0.01).call().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C", [40, 1500, 40001])
def test_masked_logits_and_rows(C, bf16):
    lowest = -3.3895313892515355e38 if bf16 else -3.4028234663852886e38

    def edit(c):
        rng = np.random.default_rng(3)
        c.label[:] = rng.integers(0, C, c.rows)
        own = np.arange(C) == c.label[:, None]
        off = (rng.random(c.x.shape) < 0.5) & ~own
        c.x[0][off[0]], c.x[1][off[1]] = -np.inf, lowest
        c.x[2], c.x[3] = -np.inf, lowest
        c.x[4] = np.where(own[4], 0, -np.inf)
        c.x[5][own[5]] = 30
        c.label[6:8] = -1
        c.x[6:8] = np.nan
        c.x[8:] = np.inf                                       # behind the last sequence
        c.ref[:] = np.float32(losses.preference_loss(c.x, c.label, c.offsets, 1.0)["logp"] - 1)

    Case([3, 2, 1, 2], C, bf16, behind=2, edit=edit).call().check()


def test_a_label_of_probability_zero():
    """Its sequence's sum is minus infinity: the loss is infinite or nothing, the sigmoid saturates, and no gradient becomes NaN."""
    def edit(c):
        c.label[:] = 2
        c.x[0, 2] = -np.inf

    c = Case([1, 1, 1, 1], 50, False, edit=edit, masked=0, ref=False).call()
    assert c.loss.item() == np.inf and c.logp[0].item() == -np.inf and np.isfinite(c.grad.host()).all()
    assert np.isclose(c.grad.host()[0, 2], -c.beta / 2, rtol=1e-5)


def test_offsets_that_make_no_sense():
    """Cut to the rows that exist: nothing is read or written out of range, and pairs with sensible offsets keep their values."""
    import torch
    c = Case([3, 2, 4, 1], 130, True, masked=0).call()
    want = c.logp.clone()
    c.d[1] = dev([0, 3, 5, 2 ** 31 - 1, 2 ** 31 - 1], np.int32)
    c.call()
    assert torch.equal(c.logp[:2], want[:2]) and torch.isfinite(c.loss).all() and c.grad.untouched()
    for bad in ([-2 ** 31, 3, 5, 9, 10], [5, 3, 9, -7, 100], [10, 10, 10, 10, 0], [2 ** 31 - 1] * 5, [-1] * 5):
        c.d[1] = dev(bad, np.int32)
        c.call()
        assert c.grad.untouched() and torch.isfinite(c.loss).all()


@pytest.mark.parametrize("lengths,C", [([1] * 40, 200), ([30, 20, 7, 9], 9001), ([2, 3], 140001)])
def test_captured_and_replayed(lengths, C):
    import torch
    c = Case(lengths, C, True, behind=1).call()
    other = Case(lengths, C, True, behind=1, seed=9).call()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        c.go(torch.cuda.current_stream().cuda_stream)
    want = {0: [t.clone() for t in c.outputs()], 1: [t.clone() for t in other.outputs()]}
    inputs = [c.logits.flat] + c.d
    mine, theirs = [t.clone() for t in inputs], [other.logits.flat] + other.d
    for k in range(4):
        for t, a, b in zip(inputs, mine, theirs):
            t.copy_(b if k % 2 else a)
        for t in c.outputs():
            t.fill_(-3.0)
        c.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[k % 2], c.outputs())), k


def test_the_same_bits_on_another_stream():
    import torch
    c = Case([40, 50, 3, 60], 3001, True).call()
    first = [t.clone() for t in c.outputs()]
    c.call(stream=torch.cuda.Stream())
    assert all(torch.equal(a, b) for a, b in zip(first, c.outputs()))


def test_offsets_beyond_32_bits():
    Case([1, 2], 1000, True, pad=1_200_000_001, gpad=1_100_000_003, masked=0).call().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C", [1, 2, 7, 40, 200, 511, 777, 1000, 1024, 1025, 2047, 2048, 2049])
def test_pairs_of_single_rows(C, bf16):
    Case([1] * 14, C, bf16, offsets=False, eps=0.1).call().check()


@pytest.mark.parametrize("bf16,gbf16", [(False, True), (True, False), (True, True)])
@pytest.mark.parametrize("C,skip,gskip,pad,gpad", [(200, 1, 0, 0, 0), (301, 3, 5, 1, 0), (1000, 0, 1, 47, 3), (13, 2, 2, 6, 6)])
def test_strides_of_single_rows(C, skip, gskip, pad, gpad, bf16, gbf16):
    Case([1] * 10, C, bf16, gbf16, offsets=False, skip=skip, gskip=gskip, pad=pad, gpad=gpad).call().check()


@pytest.mark.parametrize("train", [True, False])
@pytest.mark.parametrize("C", [200, 999])
def test_single_rows_in_place_and_without_a_gradient(C, train):
    Case([1] * 10, C, True, offsets=False, in_place=train, train=train, pad=5, skip=3).call().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C", [40, 200, 1000])
def test_masked_logits_and_single_rows(C, bf16):
    lowest = -3.3895313892515355e38 if bf16 else -3.4028234663852886e38

    def edit(c):
        rng = np.random.default_rng(4)
        c.label[:] = rng.integers(0, C, c.rows)
        own = np.arange(C) == c.label[:, None]
        off = (rng.random(c.x.shape) < 0.5) & ~own
        c.x[0][off[0]], c.x[1][off[1]] = -np.inf, lowest
        c.x[2], c.x[3] = -np.inf, lowest
        c.x[4] = np.where(own[4], 0, -np.inf)
        c.x[5][own[5]] = 30
        c.label[[6, 7, 8, 11]] = [-1, C, -2 ** 31, 2 ** 31 - 1]
        c.x[[6, 7]], c.x[[8, 11]] = np.nan, np.inf
        c.ref[:] = np.float32(losses.preference_loss(c.x, c.label, c.offsets, 1.0)["logp"] - 1)

    Case([1] * 12, C, bf16, offsets=False, edit=edit).call().check()


@pytest.mark.parametrize("offsets", [False, True])
def test_not_a_number_stays_in_its_pair(offsets):
    def edit(c):
        c.label[:] = 5
        c.x[2, 7] = np.nan

    c = Case([1] * 6, 300, True, offsets=offsets, edit=edit, masked=0, ref=False).call()
    g = c.grad.host()
    assert np.isnan(g[2:4]).all() and np.isfinite(g[[0, 1, 4, 5]]).all() and np.isnan(c.loss.item())


@pytest.mark.parametrize("bf16", [False, True])
def test_single_rows_captured_and_replayed(bf16):
    import torch
    c = Case([1] * 40, 200, bf16, offsets=False).call()
    other = Case([1] * 40, 200, bf16, offsets=False, seed=9).call()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        c.go(torch.cuda.current_stream().cuda_stream)
    want = [[t.clone() for t in v.outputs()] for v in (c, other)]
    inputs = [c.logits.flat, c.d[0], c.d[2]]
    values = [[t.clone() for t in inputs], [other.logits.flat, other.d[0], other.d[2]]]
    for k in range(4):
        for t, v in zip(inputs, values[k % 2]):
            t.copy_(v)
        for t in c.outputs():
            t.fill_(-3.0)
        c.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[k % 2], c.outputs())), k


@pytest.mark.parametrize("rows,C,bf16", [(4096, 24576, True), (2048, 50257, False)])
def test_more_logits_than_the_caches_hold(rows, C, bf16):
    """Sums of the same bits as from a half of the pairs, which stays in the caches, and gradients of half its size (a power of two: exactly)."""
    import torch
    from paper_2312_14227_amd import binding as et
    torch.manual_seed(rows)
    ty, dtype = (et.ET_BF16, torch.bfloat16) if bf16 else (et.ET_F32, torch.float32)
    x = torch.randn(rows, C, device="cuda", dtype=dtype)
    label = torch.randint(0, C, (rows,), device="cuda", dtype=torch.int32)
    label[::5] = -1
    grads = [torch.full_like(x, 7.0) for _ in range(2)]
    logp = [torch.zeros(8, device="cuda") for _ in range(2)]
    offsets = torch.arange(9, device="cuda", dtype=torch.int32) * (rows // 8)

    def run(k, at, n, pairs):
        ws, loss = torch.full((et.et_preference_loss_ws_bytes(n, pairs),), 0xFF, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda")
        p = et.make_preference(offsets.data_ptr(), 0, 0.001, 0.0, logp[k][at * 8 // rows:].data_ptr(), 0)
        et.et_preference_loss(n, pairs, C, x[at:].data_ptr(), ty, C, label[at:].data_ptr(), p, grads[k][at:].data_ptr(), ty, C, ws.data_ptr(), ws.numel(),
                              torch.cuda.current_stream().cuda_stream, loss.data_ptr())
        torch.cuda.synchronize()

    run(0, 0, rows, 4)
    for at in (0, rows // 2):
        run(1, at, rows // 2, 2)
    assert torch.equal(logp[0], logp[1]) and torch.equal(grads[0] * 2, grads[1])


@pytest.mark.parametrize("C,bf16,kw", [(600, True, {}), (77, False, dict(gbf16=True, pad=3, skip=1)), (512, False, dict(in_place=True)), (1024, True, dict(train=False))])
def test_many_short_rows(C, bf16, kw):
    Case([1700, 0, 1, 1900, 500, 400], C, bf16, front=1, behind=3, beta=0.01, **kw).call().check()
