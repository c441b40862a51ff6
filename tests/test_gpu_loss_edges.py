"""et_policy_loss and et_preference_loss where something is not finite: probabilities of zero, infinite logits, references without a distribution."""
import numpy as np
import pytest

from loss_util import close, half_step, rel
from oracle import losses
from test_gpu_policy_loss import KL, Case as Policy
from test_gpu_preference_loss import Case as Preference

pytestmark = pytest.mark.gpu

LOWEST = {True: -3.3895313892515355e38, False: -3.4028234663852886e38}


@pytest.mark.parametrize("eps", [0.0, 0.1, 1.0])
@pytest.mark.parametrize("row", [0, 1])
@pytest.mark.parametrize("C,offsets", [(50, False), (50, True), (3000, False)])
def test_an_infinite_margin(C, offsets, row, eps):
    """A token of probability zero in the preferred sequence (row 0) or the other: the pair's loss is 0 or infinite, its gradient finite, the other pair's as ever."""
    def edit(c):
        c.label[:] = 2
        c.x[row, 2] = -np.inf

    c = Preference([1, 1, 1, 1], C, False, edit=edit, masked=0, ref=False, eps=eps, offsets=offsets).call()
    w, R = losses.preference_loss(c.x, c.label, c.offsets, c.beta, c.eps), 4 * rel(C)
    z = w["z"][1]
    assert w["loss"] == np.inf if eps == 0.1 or (row == 0) == (eps == 0.0) else w["loss"] < 1 + abs(z)
    lp = np.array([losses.log_softmax(v)[2] for v in c.x])
    size = c.beta * sum(1 + abs(v) for v in lp[2:])             # (what the other margin is off by, and its loss and factor, whose slopes are at most 1)
    close(c.loss.item(), w["loss"], R * (size + 1), "loss")
    close(c.stats.cpu().numpy(), w["stats"], [0, 1e-6], "stats")
    assert c.logp[row].item() == -np.inf
    p = np.exp([losses.log_softmax(v) for v in c.x])
    close(c.grad.host(), w["grad"], half_step(False) * np.abs(w["grad"]) + R * c.beta / 2 * (1 + size) * np.maximum(p, np.arange(C) == 2) + 1e-37, "grad")


@pytest.mark.parametrize("rows,C,bf16,kw", [(9, 200, False, {}), (9, 6000, True, {}), (9, 140001, True, {}), (4500, 40, True, {}), (9, 200, True, dict(train=False)),
                                            (9, 5001, True, dict(in_place=True))])
def test_a_reference_that_gives_the_label_probability_zero(rows, C, bf16, kw):
    """exp(d) - d - 1 at d = -infinity is infinite, and its slope along d is -1."""
    def edit(c):
        c.label[1:3] = 0
        c.ref[1] = -np.inf

    c = Policy(rows, C, bf16, edit=edit, **kw).call().check()
    assert c.loss.item() == np.inf and (not c.grad or np.isfinite(c.grad.host()).all())


def _shifted(c, w):
    """Bounds of the gradient with the exact divergence: what a difference x - y is off by is relative to how far both lie below their row's maxima."""
    R, n = 4 * rel(c.C), ((c.label >= 0) & (c.label < c.C)).sum()
    bound, kl_size, size = np.zeros_like(c.x), np.zeros(c.rows), np.zeros(c.rows)
    for r in range(c.rows):
        if 0 <= c.label[r] < c.C and np.isfinite(w["grad"][r]).all():
            lp = losses.log_softmax(c.x[r])
            p = np.exp(lp)
            far = 1 + 3 * ((c.x[r].max() - c.x[r]) + (c.y[r].max() - c.y[r]))[p > 0].max()
            size[r] = (1 + abs(lp[c.label[r]])) * abs(c.adv[r]) * (1 + np.exp(lp[c.label[r]] - c.old[r]))
            kl_size[r] = KL * far
            bound[r] = half_step(c.gbf16) * np.abs(w["grad"][r]) + R / n * ((size[r] + kl_size[r]) * p + size[r] * (np.arange(c.C) == c.label[r])) + 1e-37
    return bound, R / n * (size + kl_size)


REFERENCES = [(6, 200, False, {}), (6, 200, True, dict(in_place=True)), (6, 6000, True, {}), (6, 70001, False, {}), (6, 140001, True, {}), (4500, 100, True, {}),
              (6, 200, True, dict(train=False)), (6, 40001, True, dict(train=False))]


@pytest.mark.parametrize("rows,C,bf16,kw", REFERENCES)
def test_a_reference_without_a_distribution(rows, C, bf16, kw):
    """A reference row with NaN or plus infinity in it, or nothing but minus infinity: the row's divergence and gradient are NaN, and with them the loss; the other rows' stay."""
    def edit(c):
        c.label[:5] = 3
        c.y[1, 7], c.y[2, 9], c.y[3], c.y[4, 3] = np.nan, np.inf, -np.inf, np.nan

    c = Policy(rows, C, bf16, "full", edit=edit, masked=0.1 if rows > 6 else 0, **kw).call()
    assert np.isnan(c.loss.item()) and np.isnan(c.stats[1].item()) and np.isfinite(c.stats[0].item())
    if c.grad:
        g = c.grad.host()
        assert np.isnan(g[1:5]).all()
        with np.errstate(all="ignore"):
            w = c.want()
        at = np.r_[0:1, 5:rows]
        close(g[at], w["grad"][at], _shifted(c, w)[0][at], "grad")


def test_a_reference_without_a_distribution_where_the_coefficient_is_zero(monkeypatch):
    """The divergence is reported; the loss and the gradient are those without one."""
    import test_gpu_policy_loss as t
    monkeypatch.setattr(t, "KL", 0.0)

    def edit(c):
        c.y[1, 7], c.y[2], c.y[3, 5] = np.nan, -np.inf, np.inf

    c = Policy(6, 300, False, "full", edit=edit, masked=0).call()
    assert np.isnan(c.stats[1].item())
    c.kl = "none"
    w, R = c.want(), 4 * rel(300)
    size = (1 + np.abs(w["logp"])) * np.abs(c.adv) * (1 + np.exp(w["logp"] - c.old)) / 6
    close(c.loss.item(), w["loss"], R * size.sum(), "loss")
    close(c.grad.host(), w["grad"], half_step(False) * np.abs(w["grad"]) + R * size[:, None] + 1e-37, "grad")


@pytest.mark.parametrize("rows,C,bf16,kw", REFERENCES)
def test_rows_of_the_lowest_value_on_one_side(rows, C, bf16, kw):
    """Nothing but the type's lowest value is an even distribution, also where the other side's logits are ordinary ones."""
    def edit(c):
        c.label[:5] = 3
        c.x[1], c.y[2] = LOWEST[bf16], LOWEST[bf16]
        c.y[3, 50:] = c.x[3, 50:] = LOWEST[bf16]
        c.x[4] = np.where(np.arange(C) % 2, c.x[4], LOWEST[bf16])
        c.old[:5] = -np.log(C)

    c = Policy(rows, C, bf16, "full", edit=edit, masked=0.1 if rows > 6 else 0, **kw).call()
    w = c.want()
    bound, each = _shifted(c, w)
    assert w["stats"][1] < 100
    close(c.loss.item(), w["loss"], each.sum(), "loss")
    close(c.stats.cpu().numpy()[:2], w["stats"][:2], each.sum() / KL, "stats")
    if c.grad:
        close(c.grad.host(), w["grad"], bound, "grad")


@pytest.mark.parametrize("by", [3e4, 1e7, -1e7, 1e30])
@pytest.mark.parametrize("rows,C,train", [(5, 200, True), (5, 6000, True), (5, 70001, True), (4500, 40, True), (5, 40001, False)])
def test_a_shift_between_policy_and_reference(rows, C, train, by):
    """Logits count up to a constant per row: what both rows have in common does not reach the divergence."""
    def edit(c):
        c.y = np.float32(c.y + by).astype(np.float64)

    c = Policy(rows, C, False, "full", edit=edit, train=train, masked=0).call()
    w = c.want()
    bound, each = _shifted(c, w)
    close(c.loss.item(), w["loss"], each.sum(), "loss")
    close(c.stats[1].item(), w["stats"][1], each.sum() / KL, "divergence")
    if train:
        close(c.grad.host(), w["grad"], bound, "grad")


@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
@pytest.mark.parametrize("rows,C,bf16,kw", [(6, 200, False, {}), (6, 6000, True, {}), (6, 140001, True, {}), (4500, 40, True, {}), (6, 5001, True, dict(in_place=True))])
def test_an_infinite_logit_of_the_label(rows, C, bf16, kw, kl):
    """Infinity less infinity, as with any other class of infinite logit: NaN, in its row alone."""
    def edit(c):
        c.label[:3] = 1
        c.x[1, 1] = np.inf

    c = Policy(rows, C, bf16, kl, edit=edit, masked=0, **kw).call()
    g = c.grad.host()
    assert np.isnan(c.loss.item()) and np.isnan(c.logp[1].item()) and np.isnan(g[1]).all() and np.isfinite(np.delete(g, 1, 0)).all()


@pytest.mark.parametrize("lengths,C,bf16,offsets", [([1, 1, 1, 1], 300, True, False), ([1, 1, 1, 1], 300, True, True), ([1, 1, 1, 1], 9000, False, False), ([3, 2, 1, 4], 60001, True, True),
                                                    ([1500, 1500, 900, 900], 100, True, True)])
def test_an_infinite_logit_of_the_label_of_a_pair(lengths, C, bf16, offsets):
    def edit(c):
        c.label[:] = 1
        c.x[0, 1] = np.inf

    c = Preference(lengths, C, bf16, edit=edit, masked=0, ref=False, offsets=offsets, beta=0.01).call()
    n = lengths[0] + lengths[1]
    g = c.grad.host()
    assert np.isnan(c.loss.item()) and np.isnan(c.logp[0].item()) and np.isnan(g[:n]).all() and np.isfinite(g[n:]).all()


@pytest.mark.parametrize("C,bf16", [(40, False), (130, True), (9001, True), (140001, True)])
@pytest.mark.parametrize("offsets", [[0, 5, 3, 8, 10], [5, 3, 9, -7, 100], [0, 10, 0, 10, 10], [10, 4, 6, 2, 0], [2, 9, 9, 1, 8], [-2 ** 31, 7, 2 ** 31 - 1, 3, 9], [3, 8, 2, 2, 2]])
def test_offsets_that_descend(offsets, C, bf16):
    """A row in several sequences counts in each, one that ends in front of its beginning is empty, and the gradient is zero: the same bits every time."""
    import torch
    from loss_util import dev
    c = Preference([3, 2, 4, 1], C, bf16, masked=0.1, ref=False, beta=0.5)
    c.d[1] = dev(offsets, np.int32)
    c.call()
    o, R = np.clip(offsets, 0, c.rows), 4 * rel(C)
    L, size = np.zeros(4), np.zeros(4)
    for i in range(4):
        for r in range(max(o[i], o[0]), min(o[i + 1], o[4])):
            if 0 <= c.label[r] < C:
                lp = losses.log_softmax(c.x[r])[c.label[r]]
                L[i], size[i] = L[i] + lp, size[i] + 1 + abs(lp)
    z = c.beta * (L[0::2] - L[1::2])
    off = R * c.beta * (size[0::2] + size[1::2]) + 2.0 ** -23 * np.abs(z)
    close(c.logp.cpu().numpy(), L, R * size + 2.0 ** -24 * np.abs(L), "logp")
    close(c.loss.item(), np.logaddexp(0, -z).mean(), off.mean() + R, "loss")
    close(c.stats[0].item(), z.mean(), off.mean(), "margin")
    g = c.grad.host()
    assert (g[o[0]:max(o[0], o[4])] == 0).all() and (np.delete(g, range(o[0], max(o[0], o[4])), 0) == c.grad.fill).all() and c.grad.untouched()
    first = [t.clone() for t in c.outputs()]
    c.call(stream=torch.cuda.Stream())
    assert all(torch.equal(a, b) for a, b in zip(first, c.outputs()))
    c.d[1] = dev(c.offsets, np.int32)                            # and nothing of it is left for the next call
    c.call().check()


def _together(bf16, rows, C, parts, pad):
    """`parts` matrices whose rows lie beside each other in one buffer."""
    import torch
    flat = torch.full((rows, parts * (C + pad)), -3.0, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    return flat, [flat[:, k * (C + pad):k * (C + pad) + C] for k in range(parts)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C,pad", [(200, 0), (1001, 3), (33001, 0)])
def test_matrices_whose_rows_lie_beside_each_other(C, pad, bf16):
    """Logits, the reference's and the gradient in one buffer, and the gradient in the logits' place beside the reference: within the bounds of the definition.  (Not the bits of
    buffers of their own: the vectors of a row begin at multiples of 16 bytes, so its address decides in which order its C terms are added, and two orders of them differ by up to
    2 (C / 64 + 20) roundings of 2^-24, of which the bound counts as many for each.)"""
    import torch
    from paper_2312_14227_amd import binding as et
    c = Policy(7, C, bf16, "full", masked=0.2).call().check()
    ty = et.ET_BF16 if bf16 else et.ET_F32
    for in_place in (False, True):
        flat, part = _together(bf16, 7, C, 3, pad)
        part[0].copy_(c.logits.view), part[1].copy_(c.refs.view)
        grad, stride = part[0 if in_place else 2], flat.shape[1]
        p = et.make_policy(c.d["old"].data_ptr(), c.d["adv"].data_ptr(), ref_logits=part[1].data_ptr(), ref_stride=stride, clip_low=c.p.clip_low, clip_high=c.p.clip_high,
                           kl_coef=KL, logp=c.logp.data_ptr(), stats=c.stats.data_ptr())
        for t in (c.loss, c.logp, c.stats, c.grad.view):
            t.fill_(7.0)
        et.et_policy_loss(7, C, part[0].data_ptr(), ty, stride, c.d["label"].data_ptr(), p, grad.data_ptr(), ty, stride, c.ws.data_ptr(), c.ws.numel(),
                          torch.cuda.current_stream().cuda_stream, c.loss.data_ptr())
        torch.cuda.synchronize()
        c.grad.put(grad)
        c.check()
        assert torch.equal(part[1], c.refs.view) and (in_place or torch.equal(part[0], c.logits.view))
        assert bool((flat[:, [k * (C + pad) + C + i for k in range(3) for i in range(pad)]] == -3.0).all())
