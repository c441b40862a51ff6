"""et_policy_loss and et_preference_loss: calls of sizes that take a launch of their own or another number of threads, captured ones whose every output is compared, and the mean error
of log probabilities."""
import numpy as np
import pytest


pytestmark = pytest.mark.gpu


def _at(t):
    return t.data_ptr() if t is not None else 0


class Calls:
    """Rows of normal logits; go() enqueues a call into `outputs`."""

    def __init__(self, rows, C, bf16, kl, train, seed=0):
        import torch
        from paper_2312_14227_amd import binding as et
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rows, self.C, self.train = rows, C, train
        self.type, self.dtype = (et.ET_BF16, torch.bfloat16) if bf16 else (et.ET_F32, torch.float32)
        normal = lambda *n: torch.randn(n, generator=gen, device="cuda", dtype=self.dtype if len(n) > 1 else torch.float32)  # noqa: E731
        self.x = normal(rows, C)
        self.y = self.x + normal(1, C) / 4 if kl == "full" else None
        self.old, self.adv = normal(rows) / 4 - float(np.log(C)), normal(rows)
        self.ref = normal(rows) / 4 - float(np.log(C)) if kl == "sampled" else None
        self.label = torch.randint(0, C, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        self.ws = torch.empty(et.et_policy_loss_ws_bytes(rows), dtype=torch.uint8, device="cuda")

    def outputs(self):
        import torch
        like = lambda n: torch.full((n,), -3.0, device="cuda")  # noqa: E731
        return [like(1), like(3), like(self.rows)] + ([torch.full_like(self.x, -3.0)] if self.train else [])

    def go(self, out):
        import torch
        from paper_2312_14227_amd import binding as et
        p = et.make_policy(_at(self.old), _at(self.adv), ref_logp=_at(self.ref), ref_logits=_at(self.y), ref_stride=self.C, kl_coef=0.05, logp=_at(out[2]), stats=_at(out[1]))
        et.et_policy_loss(self.rows, self.C, _at(self.x), self.type, self.C, _at(self.label), p, _at(out[3]) if self.train else 0, self.type, self.C, _at(self.ws),
                          self.ws.numel(), torch.cuda.current_stream().cuda_stream, _at(out[0]))


@pytest.mark.parametrize("kl", ["sampled", "full"])
@pytest.mark.parametrize("rows,C,bf16,train", [(8200, 200, True, True), (20000, 130, False, True), (8200, 3001, False, True), (8300, 24001, True, True), (8193, 70001, False, True),
                                               (8200, 200, True, False), (8200, 24001, True, False)])
def test_captured_with_rows_that_a_launch_counts(rows, C, bf16, train, kl):
    """Replays give the bits of calls one at a time in every output, with labels that change between them, and with them the weight of a row."""
    import torch
    c = Calls(rows, C, bf16, kl, train)
    eager, captured = c.outputs(), c.outputs()
    c.go(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        c.go(captured)
    label, seen = c.label.clone(), []
    for k in range(4):
        c.label.copy_(label)
        c.label[:rows // 5 * k] = -1 if k % 2 else C
        for t in eager + captured:
            t.fill_(-3.0)
        c.ws.fill_(0xFF)
        c.go(eager)
        torch.cuda.synchronize()
        c.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, captured)), k
        assert bool((captured[2][:rows // 5 * k] == 0).all()) and torch.isfinite(captured[0]).item()
        seen.append(captured[0].item())
    assert len(set(seen)) == 4


@pytest.mark.parametrize("train", [True, False])
@pytest.mark.parametrize("pairs,C,bf16,offsets", [(500, 3000, True, False), (3000, 200, False, False), (3000, 3000, True, False), (4096, 7, True, False), (4097, 7, False, False),
                                                  (8000, 40, True, False), (4097, 7, False, True), (9000, 12, True, True)])
def test_many_pairs(pairs, C, bf16, offsets, train):
    """Up to 4096 pairs are added by 256 threads, more by 1024; each pair's values against float64 on the device."""
    import torch
    from loss_util import half_step, rel
    from paper_2312_14227_amd import binding as et
    c = Calls(2 * pairs, C, bf16, "none", train, seed=pairs)
    rows, beta, R = 2 * pairs, 0.5, 4 * rel(C)
    c.label[::7] = -1
    out = [torch.full((n,), -3.0, device="cuda") for n in (1, 2, rows)] + ([torch.full_like(c.x, -3.0)] if train else [])
    ws = torch.full((et.et_preference_loss_ws_bytes(rows, pairs),), 0xFF, dtype=torch.uint8, device="cuda")
    off = torch.arange(rows + 1, device="cuda", dtype=torch.int32)
    p = et.make_preference(_at(off) if offsets else 0, 0, beta, 0.0, _at(out[2]), _at(out[1]))
    et.et_preference_loss(rows, pairs, C, _at(c.x), c.type, C, _at(c.label), p, _at(out[3]) if train else 0, c.type, C, _at(ws), ws.numel(),
                          torch.cuda.current_stream().cuda_stream, _at(out[0]))
    torch.cuda.synchronize()
    there, at = c.label >= 0, c.label.clamp(min=0).long()[:, None]
    logp = torch.log_softmax(c.x.double(), 1)
    L = torch.where(there, logp.gather(1, at)[:, 0], 0.0)
    z = beta * (L[0::2] - L[1::2])
    loss = torch.nn.functional.softplus(-z)
    assert bool(((out[2] - L).abs() <= R * (1 + L.abs())).all())
    off_z = R * beta * (2 + L[0::2].abs() + L[1::2].abs())      # (the slope of the loss in z is at most 1, of its derivative 1/4)
    assert abs(out[0].item() - loss.mean().item()) <= off_z.mean().item() + R * loss.mean().item()
    assert abs(out[1][0].item() - z.mean().item()) <= off_z.mean().item()
    # (a margin within its error of zero may fall on either side; one of two masked rows is zero, and counts on neither)
    near = ((z.abs() <= off_z) & (z != 0)).double().mean().item()
    assert abs(out[1][1].item() - (z > 0).double().mean().item()) <= near + 2.0 ** -23
    if train:
        d = -torch.sigmoid(-z) * beta / pairs
        g = torch.stack([d, -d], 1).reshape(-1, 1) * there[:, None]
        one = torch.zeros_like(logp).scatter_(1, at, 1.0)
        want = g * (one - logp.exp())
        bound = half_step(bf16) * want.abs() + (R + off_z.repeat_interleave(2)[:, None]) * beta / pairs * (one + logp.exp()) + 1e-37
        assert bool(((out[3].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("C,train", [(100003, True), (100003, False), (250007, True)])
def test_the_mean_error_of_log_probabilities(C, train, up, bf16):
    """Errors of one sign add up over a sequence.  float32's log2 e is 1.335e-8 of itself too small, which by itself puts the logarithm of a sum of exp(x - m) off by as much times the mean of
    x - m.  Here that is 8: above the reference m, which is among the first classes (of each thread's first vector: at most 8192, and 8 in front) and is not raised for what lies up to 11
    above, or below it, one class being 8 above the others, of which there are enough to hold most of the probability.  So 1.07e-7 are to be taken off, of one sign or the other.  What is
    left: the exponential's own systematic part, a small part of its 2^-23, and roundings (of log p to float32: 2^-22 / sqrt(12) up to 16), which average out over 2048 rows and more
    to 2e-9.  The bound, 4e-8, lies between."""
    import torch
    from paper_2312_14227_amd import binding as et
    rows = 4096 if C < 200000 else 2048
    gen = torch.Generator(device="cuda").manual_seed(C)
    ty, dtype = (et.ET_BF16, torch.bfloat16) if bf16 else (et.ET_F32, torch.float32)
    x = torch.empty(rows, C, dtype=dtype, device="cuda")
    exact = torch.empty(rows, dtype=torch.float64, device="cuda")
    label = torch.randint(0, C, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    for r in range(0, rows, 512):
        v = torch.rand(512, C, generator=gen, device="cuda")
        if up:
            v[:, :8200] -= 8.0
        else:
            v[:, 4] = 8.5
        x[r:r + 512] = v.to(dtype)
        exact[r:r + 512] = torch.log_softmax(x[r:r + 512].double(), 1).gather(1, label[r:r + 512, None].long())[:, 0]
    old, adv, logp, loss = exact.float(), torch.ones(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(et.et_policy_loss_ws_bytes(rows), dtype=torch.uint8, device="cuda")
    p = et.make_policy(_at(old), _at(adv), logp=_at(logp))
    et.et_policy_loss(rows, C, _at(x), ty, C, _at(label), p, _at(x) if train else 0, ty, C, _at(ws), ws.numel(), torch.cuda.current_stream().cuda_stream, _at(loss))
    torch.cuda.synchronize()
    mean = (logp.double() - exact).mean().item()
    assert abs(mean) <= 4e-8, mean
