"""et_grad_norm and et_grad_clip against the float64 definition: tensors of any number, size and alignment, values at the ends of the range, in place and
not, and the calls a captured program makes."""
import numpy as np
import pytest

from oracle import losses

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, sizes, bf16, seed=0, skip=0, gap=0, scale=1e-2, out=None, edit=None):
        """gap: elements between tensors; out: None: in place, else how far the outputs' addresses are off the inputs'."""
        import torch
        rng = np.random.default_rng(seed)
        self.sizes, self.dtype, self.bf16 = list(sizes), torch.bfloat16 if bf16 else torch.float32, bf16
        starts = skip + np.concatenate([[0], np.cumsum([s + gap for s in sizes])]).astype(int)
        total = int(starts[-1]) + 8
        host = torch.from_numpy(rng.standard_normal(total, np.float32) * np.float32(scale))
        if edit:
            edit(host, starts)
        self.arena = host.cuda().to(self.dtype)
        self.views = [self.arena[a:a + n] for a, n in zip(starts, sizes)]
        self.host = [v.double().cpu().numpy() for v in self.views]
        self.out_arena = self.arena if out is None else torch.full((total + out,), 5.0, dtype=self.dtype, device="cuda")
        self.outs = self.views if out is None else [self.out_arena[out + a:out + a + n] for a, n in zip(starts, sizes)]

    def bind(self, max_norm=None, tensor_norm=True):
        import torch
        from paper_2312_14227_amd import binding as et
        n = len(self.sizes)
        room = et.et_grad_norm_ws_bytes(self.sizes)
        self.ws = torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda")
        self.norm, self.each = torch.full((1,), -1.0, device="cuda"), torch.full((n + 1,), -1.0, device="cuda")
        ptr = lambda vs: [v.data_ptr() if v.numel() else 0 for v in vs]  # noqa: E731
        ty = et.ET_BF16 if self.bf16 else et.ET_F32
        each = self.each.data_ptr() if tensor_norm else 0
        if max_norm is None:
            self.go = lambda s: et.et_grad_norm(ptr(self.views), self.sizes, ty, self.ws.data_ptr(), room, s, self.norm.data_ptr(), each)
        else:
            outs = None if self.out_arena is self.arena else ptr(self.outs)
            self.go = lambda s: et.et_grad_clip(ptr(self.views), outs, self.sizes, ty, max_norm, self.ws.data_ptr(), room, s, self.norm.data_ptr(), each)
        return self

    def call(self, max_norm=None, **kw):
        import torch
        self.bind(max_norm, **kw)
        self.go(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return self

    def check_norm(self, tensor_norm=True):
        norm, each = losses.grad_norm(self.host)
        # a square root of sums in float64, rounded once to float32
        assert abs(self.norm.item() - norm) <= 2.0 ** -23 * norm + 2.0 ** -149, (self.norm.item(), norm)
        got = self.each.cpu().numpy()
        assert got[-1] == -1
        if tensor_norm:
            np.testing.assert_allclose(got[:-1], each, rtol=2.0 ** -23, atol=2.0 ** -149)
        else:
            assert (got == -1).all()
        return self

    def check_clip(self, max_norm):
        self.check_norm()
        m = float(np.float32(max_norm))
        _, _, want = losses.grad_clip(self.host, m)
        # the coefficient and the product are rounded to float32, and the product to the type
        bound = 2.0 ** -22 + (2.0 ** -8 if self.bf16 else 0)
        for v, w, h in zip(self.outs, want, self.host):
            got = v.double().cpu().numpy()
            assert (np.abs(got - w) <= bound * np.abs(w) + 1e-38).all()
            if losses.grad_norm(self.host)[0] <= m:
                assert np.array_equal(got, h)
        return self


SIZES = [[1], [2], [63], [4096], [16384], [16385], [65537], [300000], [3, 1, 2], [0, 5, 0], [0, 0], [1] * 700, [16384] * 3, [5000, 70000, 1, 33333], [17] * 121,
         [100] * 240 + [50000], [1_000_003], [262144, 262143, 262145]]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("k", range(len(SIZES)))
def test_norm(k, bf16):
    Case(SIZES[k], bf16, seed=k).call().check_norm()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("skip,gap", [(0, 1), (1, 0), (1, 3), (2, 7), (3, 2), (5, 64)])
def test_alignments(skip, gap, bf16):
    c = Case([40001, 7, 16385, 0, 99, 123456], bf16, skip=skip, gap=gap, out=1)
    c.call().check_norm()
    c.call(0.7).check_clip(0.7)


@pytest.mark.parametrize("out", [None, 0, 3])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("k", range(len(SIZES)))
@pytest.mark.parametrize("share", [0.37, 2.0])
def test_clip(k, bf16, out, share):
    c = Case(SIZES[k], bf16, seed=50 + k, out=out, gap=k % 3)
    around = c.arena.clone()
    max_norm = float(np.float32(share * losses.grad_norm(c.host)[0]))
    c.call(max_norm).check_clip(max_norm)
    # what lies between the tensors, and the inputs, are as they were
    at = 0 if out is None else out
    if out is None:
        for v in c.views:
            around_view = around[v.storage_offset():v.storage_offset() + v.numel()]
            around_view.copy_(v)
        assert bool((around == c.arena).all())
    else:
        assert bool((around == c.arena).all())
        for v in c.outs:
            c.out_arena[v.storage_offset():v.storage_offset() + v.numel()] = 5.0
        assert bool((c.out_arena == 5.0).all())


def test_no_tensor_and_no_tensor_norms():
    from paper_2312_14227_amd import binding as et
    c = Case([4], False)
    c.sizes, c.views, c.host, c.outs = [], [], [], []
    c.call().check_norm()
    assert c.norm.item() == 0
    c.call(1.0)
    assert c.norm.item() == 0
    Case([500, 70000], True).call(tensor_norm=False).check_norm(tensor_norm=False)
    assert et.et_grad_norm_ws_bytes([]) > 0


@pytest.mark.parametrize("k", [3, 8, 13])
def test_limits_of_clipping(k):
    c = Case(SIZES[k], False, out=0)
    c.call(0.0)
    assert all(not v.any() for v in c.outs)
    norm = np.float32(losses.grad_norm(c.host)[0])
    for m in (np.nextafter(norm, np.float32(9)), np.float32(np.inf)):   # at least the norm: nothing changes
        c.call(float(m))
        assert all(np.array_equal(v.double().cpu().numpy(), h) for v, h in zip(c.outs, c.host))


@pytest.mark.parametrize("scale", [1e-30, 1e-42, 1e18, 3e30])
def test_no_overflow_or_underflow_inside(scale):
    Case([5000, 70001], False, scale=scale).call().check_norm()


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("sizes", [[5000], [5000, 70001, 300000]])
@pytest.mark.parametrize("out", [None, 1])
def test_a_norm_that_is_not_finite_changes_nothing(sizes, bad, out):
    def edit(host, starts):
        host[starts[0] + 4321] = float(bad)

    c = Case(sizes, False, edit=edit, out=out)
    c.call(0.1)
    assert c.norm.item() == np.inf if not np.isnan(bad) else np.isnan(c.norm.item())
    assert np.isfinite(c.each.cpu().numpy()[1:]).all()
    assert all(np.array_equal(v.double().cpu().numpy(), h, equal_nan=True) for v, h in zip(c.outs, c.host))


def test_a_norm_beyond_float32_changes_nothing():
    c = Case([200000], False, scale=1.0, edit=lambda h, s: h.fill_(3e38), out=0)
    c.call(1.0)
    assert c.norm.item() == np.inf and all(np.array_equal(v.double().cpu().numpy(), h) for v, h in zip(c.outs, c.host))


@pytest.mark.parametrize("k", [3, 11, 13])
def test_captured_and_replayed(k):
    import torch
    c = Case(SIZES[k], True, out=0)
    max_norm = 0.5 * float(losses.grad_norm(c.host)[0])
    c.call(max_norm)
    first = [t.clone() for t in (c.norm, c.each, c.out_arena)]
    kept = c.arena.clone()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        c.go(torch.cuda.current_stream().cuda_stream)
    for r in range(4):
        c.arena.copy_(kept * (2 if r % 2 else 1))
        c.ws.fill_(0xFF)
        c.norm.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert c.norm.item() == first[0].item() * (2 if r % 2 else 1)
        assert torch.equal(c.out_arena, first[2])            # (twice the gradient, half the coefficient: exact)


def test_the_same_bits_again_and_on_another_stream():
    import torch
    c = Case([1_000_003, 5, 70000], False, out=0)
    c.call(0.3)
    first = [t.clone() for t in (c.norm, c.each, c.out_arena)]
    c.out_arena.fill_(5.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c.go(side.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (c.norm, c.each, c.out_arena)))


def test_offsets_beyond_32_bits():
    """4.4e9 elements in one tensor: values at both ends, zeros between."""
    import torch
    from paper_2312_14227_amd import binding as et
    n = 4_400_000_003
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[-1], g[n // 2] = 3.0, 4.0, 12.0
    room = et.et_grad_norm_ws_bytes([n])
    ws, norm = torch.empty(room, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda")
    et.et_grad_clip([g.data_ptr()], None, [n], et.ET_BF16, 6.5, ws.data_ptr(), room, torch.cuda.current_stream().cuda_stream, norm.data_ptr())
    torch.cuda.synchronize()
    assert norm.item() == 13.0 and [g[0].item(), g[-1].item(), g[n // 2].item()] == [1.5, 2.0, 6.0]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("out", [None, 0, 3])
@pytest.mark.parametrize("norm", [0.5, 2.0, float("inf"), float("nan")])
def test_scaling_by_a_norm_from_elsewhere(norm, out, bf16):
    import torch
    from paper_2312_14227_amd import binding as et
    c = Case([5000, 0, 70003, 1] + [9] * 130, bf16, out=out, gap=1)
    given = torch.tensor([norm], device="cuda")
    ptr = lambda vs: [v.data_ptr() if v.numel() else 0 for v in vs]  # noqa: E731
    et.et_grad_scale(ptr(c.views), None if out is None else ptr(c.outs), c.sizes, et.ET_BF16 if bf16 else et.ET_F32, given.data_ptr(), 0.75,
                     torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    f = 0.375 if norm == 2.0 else 1.0
    assert all((np.abs(v.double().cpu().numpy() - f * h) <= (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(h) * (f != 1)).all() for v, h in zip(c.outs, c.host))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("out", [None, 0, 1])
def test_more_than_the_caches_hold(out, bf16):
    """Past 128 MB, and past what a launch reads without keeping it, with tensors on both sides of each border."""
    n = 2 if bf16 else 1
    c = Case([30_000_001 * n, 7, 26_000_003 * n, 300, 4_000_000], bf16, out=out, gap=1)
    max_norm = float(np.float32(0.5 * losses.grad_norm(c.host)[0]))
    c.call().check_norm()
    c.call(max_norm).check_clip(max_norm)
