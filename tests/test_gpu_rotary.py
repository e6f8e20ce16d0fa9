"""Rotary positions of queries and keys (lite_attn_rotary_fwd / _bwd) against their definition in 64 bits."""
import pytest
import torch

import layer_reference as ref
from paper_2511_11062_amd import layer

pytestmark = pytest.mark.gpu

# What 32-bit arithmetic may add to the rounding of a result, as a share of |a| + |b| of a pair: the mean of squares is a sum
# of at most 8 products in a thread, 6 steps in a wave and 4 between waves (20 roundings of 2^-24 at most, halved by the root),
# the root, the two factors and the turn are another 8, cos and sin are off by 2^-22 (the angle is taken in 64 bits, as a part
# of a turn of at most 1/2 it is rounded once to 24 bits: pi * 2^-24, the functions add 2^-23): below 18 + 12 = 30 of 2^-24,
# 2^-19.
SLACK = 2.0 ** -19


class Case:
    def __init__(self, batch=1, heads=(3, 3), d=128, grid=(2, 3, 5), text=0, start=0, n=None, dtype="bf16", weights="f32",
                 norm="none", halves=False, pairs=None, far=None, source="bnhd", target="bhnd", seed=1, shift=0):
        self.__dict__.update(locals())
        self.n = grid[0] * grid[1] * grid[2] + text - start if n is None else n
        self.pairs = d // 2 if pairs is None else pairs
        g = ref.gen(seed)
        kind = ref.TYPES[dtype]
        n, (hq, hk) = self.n, heads

        def tensor(h, layout, data=None):
            """[B,H,N,d] view of memory in `layout`, `shift` elements off its allocation's start."""
            shape = {"bnhd": (batch, n, h, d), "bhnd": (batch, h, n, d), "packed": (batch, n, hq + 2 * hk, d)}[layout]
            count = shape[0] * shape[1] * shape[2] * shape[3]
            flat = torch.full((count + shift,), float("nan"), dtype=kind, device="cuda")
            t = flat[shift:].view(shape)
            t = t.transpose(1, 2) if layout != "bhnd" else t
            if data is not None:
                t.copy_(data)
            return t

        self.tensor = tensor
        scale = torch.exp(0.5 * ref.randn(g, d))
        if source == "packed":
            x = tensor(hq + 2 * hk, "packed", ref.randn(g, batch, hq + 2 * hk, n, d) * scale)
            self.q, self.k = x[:, :hq], x[:, hq:hq + hk]
        else:
            self.q = tensor(hq, source, ref.randn(g, batch, hq, n, d) * scale)
            self.k = tensor(hk, source, ref.randn(g, batch, hk, n, d) * scale)
        self.freqs = torch.zeros(3, self.pairs, dtype=torch.float64, device="cuda")
        side = self.pairs // 3
        split = (self.pairs - 2 * side, side, side)
        self.freqs.copy_(torch.from_numpy(layer.lite_attn_rotary_freqs(split, 10000.0).copy()))
        self.positions = None
        if far is not None:
            self.positions = torch.randint(-far, far + 1, (batch, 3, n), generator=g, device="cuda", dtype=torch.int32)
            self.where = self.positions.double().transpose(1, 2)
        else:
            self.where = ref.grid_positions(grid, start, n)[None]
        self.w = (None, None)
        if norm != "none" and weights:
            self.w = tuple((1.0 + 0.3 * ref.randn(g, *((h, d) if norm == "row" else (d,)))).to(ref.TYPES[weights])
                           for h in heads)
        self.g = g
        self.desc = layer.make_rotary_desc(batch, n, hq, hk, d, dtype=ref.KINDS[dtype],
                                           weight_dtype=ref.KINDS[weights or "f32"], norm=ref.NORMS[norm], halves=halves,
                                           pairs=self.pairs, grid=grid, eps=1e-6)

    def places(self):
        return dict(positions=ref.at(self.positions), positions_stride_b=3 * self.n if self.positions is not None else 0,
                    token_start=self.start, hip_stream=ref.stream())

    def forward(self, q_out=None, k_out=None):
        q_out = self.tensor(self.heads[0], self.target) if q_out is None else q_out
        k_out = self.tensor(self.heads[1], self.target) if k_out is None and self.heads[1] else k_out
        layer.lite_attn_rotary_fwd(self.desc, ref.heads_view(self.q), ref.heads_view(self.k) if self.heads[1] else None,
                                   ref.heads_view(q_out), ref.heads_view(k_out) if self.heads[1] else None,
                                   self.freqs.data_ptr(), q_weight=ref.at(self.w[0]), k_weight=ref.at(self.w[1]),
                                   **self.places())
        return q_out, k_out

    def expected(self, x, w):
        return ref.rotary(x.double(), None if w is None else w.double(), self.freqs, self.where, self.norm, self.halves, 1e-6)

    def check_forward(self):
        kept = self.q.clone(), self.k.clone()
        got = self.forward()
        for name, x, w, out, old in zip("qk", (self.q, self.k), self.w, got, kept):
            if out is None:
                continue
            want = self.expected(x, w)
            # the turn mixes a pair: its slack is a share of both entries before it, which are as large as after it
            ref.check(name, out, want, SLACK * ref.partner_sum(want, self.pairs, self.halves) * 1.5)
            assert torch.equal(x, old)

    def backward(self, grads, dq=None, dk=None, weights=True):
        new = lambda h: self.tensor(h, "bnhd")
        hq, hk = self.heads
        dq = new(hq) if dq is None else dq
        dk = new(hk) if dk is None and hk else dk
        dw = [torch.full(w.shape, float("nan"), device="cuda") if w is not None and weights else None for w in self.w]
        need = layer.lite_attn_rotary_bwd_workspace(self.desc)
        space = torch.full((max(16, need) // 4,), float("nan"), device="cuda")
        layer.lite_attn_rotary_bwd(self.desc, ref.heads_view(self.q), ref.heads_view(self.k) if hk else None,
                                   ref.heads_view(grads[0]), ref.heads_view(grads[1]) if hk else None, ref.heads_view(dq),
                                   ref.heads_view(dk) if hk else None, self.freqs.data_ptr(), q_weight=ref.at(self.w[0]),
                                   k_weight=ref.at(self.w[1]), dq_weight=ref.at(dw[0]), dk_weight=ref.at(dw[1]),
                                   workspace=space.data_ptr(), workspace_bytes=need, **self.places())
        return dq, dk, dw

    def gradients(self):
        return [self.tensor(h, self.target, ref.randn(self.g, self.batch, h, self.n, self.d)) for h in self.heads]

    def check_backward(self):
        grads = self.gradients()
        dq, dk, dw = self.backward(grads)
        for name, x, w, g, dx, dwx in zip("qk", (self.q, self.k), self.w, grads, (dq, dk), dw):
            if x.shape[1] == 0:
                continue
            x = x.double().requires_grad_()
            w = None if w is None else w.double().requires_grad_()
            out = self.expected(x, w)
            want = torch.autograd.grad(out, [x] if w is None else [x, w], g.double())
            # dx = rstd (dn - n mean(dn n)): both terms, of entries of size |dn| and |n| rms(dn), are off by a share of
            # themselves; 40 roundings of 2^-24 bound each (two sums like SLACK's, and the factors)
            back = ref.rotary(g.double(), None, self.freqs, -self.where, "none", self.halves, 0.0)
            size = ref.partner_sum(back, self.pairs, self.halves) * 1.5
            slack = 2 * SLACK * size
            if self.norm != "none":
                dims = (1, 3) if self.norm == "row" else (3,)
                xd = x.detach()
                rstd = 1.0 / torch.sqrt((xd * xd).mean(dim=dims, keepdim=True) + 1e-6)
                wd = torch.ones_like(xd) if w is None else (w.detach()[:, None] if self.norm == "row" else w.detach()).expand_as(xd)
                dn = size * wd.abs()
                n = (xd * rstd).abs()
                slack = 2 * SLACK * rstd * (dn + n * (dn * n).mean(dim=dims, keepdim=True))
            ref.check("d" + name, dx, want[0], slack)
            if w is not None:
                # terms dz x rstd are off by SLACK each, their sum in 32 bits by a rounding for each term at most
                terms = (size * (xd * rstd).abs())
                terms = terms.sum(dim=(0, 2)) if self.norm == "row" else terms.sum(dim=(0, 1, 2))
                count = self.batch * self.n * (1 if self.norm == "row" else x.shape[1])
                ref.check("d%s_weight" % name, dwx, want[1], terms * (2 * SLACK + 2.0 ** -24 * min(count + 8, 4096)))


@pytest.mark.parametrize("norm", ["none", "head", "row"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_forward_and_backward(dtype, halves, norm):
    c = Case(batch=2, heads=(5, 5), grid=(3, 5, 7), text=9, dtype=dtype, weights=dtype, norm=norm, halves=halves)
    c.check_forward()
    c.check_backward()


# heads of every width that a thread's eight entries divide and of some that they do not; more heads than a workgroup takes;
# shared key heads; no key heads
@pytest.mark.parametrize("norm", ["none", "head", "row"])
@pytest.mark.parametrize("heads,d,pairs,halves", [
    ((1, 1), 2, 1, False), ((3, 2), 6, 3, True), ((2, 2), 8, 4, False), ((9, 3), 16, 5, True), ((4, 1), 34, 17, True),
    ((7, 7), 64, 24, True), ((2, 2), 72, 36, False), ((5, 5), 72, 36, True), ((3, 3), 80, 40, True), ((6, 2), 96, 48, False),
    ((33, 3), 128, 64, True), ((40, 40), 128, 64, False), ((3, 3), 128, 30, True), ((2, 2), 128, 30, False),
    ((3, 1), 128, 0, False), ((2, 0), 128, 64, False), ((3, 3), 256, 128, True), ((2, 1), 510, 255, True),
    ((2, 2), 512, 256, False)])
def test_heads(heads, d, pairs, halves, norm):
    c = Case(batch=2, heads=heads, d=d, pairs=pairs, halves=halves, norm=norm, grid=(2, 3, 3), text=3, dtype="f16")
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("n", [1, 2, 3, 17, 255])
@pytest.mark.parametrize("batch", [1, 3])
def test_short_calls(batch, n):
    c = Case(batch=batch, heads=(4, 2), grid=(5, 6, 11), start=74, n=n, norm="head", halves=True)
    c.check_forward()
    c.check_backward()


def test_more_tokens_than_workgroups_and_than_angles_at_a_time():
    c = Case(heads=(2, 2), d=32, grid=(7, 33, 41), text=300, norm="head", dtype="f32")
    c.check_forward()
    c.check_backward()
    c = Case(heads=(8, 8), d=128, grid=(11, 60, 31), text=0, norm="row")
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("far", [3, 100000, 2 ** 31 - 1])
def test_given_positions(far):
    """Any 32-bit position, negative ones among them: the angle is exact to 2^-53 of the number of turns, 2^31 / 2 pi of them
    leave 4e-8 radians."""
    c = Case(batch=2, heads=(3, 1), grid=(1, 1, 1), n=19, far=far, dtype="f32", norm="head")
    c.check_forward()
    c.check_backward()


def test_text_and_parts_of_the_sequence():
    """Tokens behind the grid are not turned; a call of a part of the sequence gives what the whole gives, to the bit."""
    whole = Case(heads=(3, 3), grid=(2, 4, 5), text=7, norm="row")
    out = whole.forward()[0]
    text = whole.expected(whole.q, whole.w[0])[:, :, 40:]
    plain = whole.q.double() / torch.sqrt((whole.q.double() ** 2).mean(dim=(1, 3), keepdim=True) + 1e-6) * whole.w[0].double()[:, None]
    assert torch.equal(text, plain[:, :, 40:])
    for start, n in ((0, 1), (11, 20), (39, 2), (46, 1)):
        part = Case(heads=(3, 3), grid=(2, 4, 5), start=start, n=n, norm="row")
        part.q.copy_(whole.q[:, :, start:start + n])
        part.w = whole.w
        assert torch.equal(part.forward()[0], out[:, :, start:start + n])


@pytest.mark.parametrize("source,target", [("packed", "bhnd"), ("packed", "bnhd"), ("bhnd", "bnhd")])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_layouts_and_alignment(source, target, shift):
    for dtype in ("bf16", "f32"):
        c = Case(batch=2, heads=(4, 2), grid=(2, 3, 4), source=source, target=target, dtype=dtype, norm="head", shift=shift)
        c.check_forward()
        c.check_backward()
        c = Case(batch=2, heads=(4, 2), grid=(2, 3, 4), source=source, target=target, dtype=dtype, halves=True, shift=shift)
        c.check_forward()
        c.check_backward()


@pytest.mark.parametrize("heads,d,norm", [((30, 30), 72, "head"), ((37, 9), 72, "none"), ((24, 24), 128, "head"),
                                          ((9, 20), 80, "head"), ((33, 33), 64, "none"), ((17, 3), 512, "head"),
                                          ((12, 12), 90, "head"), ((70, 2), 6, "head")])
@pytest.mark.parametrize("target", ["bhnd", "bnhd"])
def test_heads_in_several_parts(heads, d, norm, target):
    """More heads than a workgroup takes, in parts that do not come out even, of one token and of several."""
    for dtype in ("bf16", "f32"):
        c = Case(batch=2, heads=heads, d=d, grid=(3, 7, 11), text=6, norm=norm, target=target, dtype=dtype)
        c.check_forward()
        c.check_backward()


def test_inputs_shared_by_batch_entries_and_heads():
    """Strides of 0: one key head for all, one batch entry for all."""
    c = Case(batch=3, heads=(4, 4), grid=(2, 3, 4), norm="row")
    c.q = c.q[:1].expand(3, -1, -1, -1)
    c.k = c.k[:, :1].expand(-1, 4, -1, -1)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("norm", ["none", "head", "row"])
def test_in_place(norm):
    c = Case(batch=2, heads=(5, 3), grid=(4, 5, 6), norm=norm, source="packed")
    want = c.forward()
    grads = c.gradients()
    wdq, wdk, wdw = c.backward(grads)
    dq, dk, dw = c.backward(grads, dq=grads[0], dk=grads[1])
    assert torch.equal(dq, wdq) and torch.equal(dk, wdk)
    assert all(a is None or torch.equal(a, b) for a, b in zip(dw, wdw))
    got = c.forward(q_out=c.q, k_out=c.k)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_only_what_is_asked_for():
    """Without weights, without gradients of theirs, without a workspace."""
    for norm in ("head", "row"):
        c = Case(heads=(3, 2), norm=norm, weights=None, grid=(3, 4, 5))
        c.check_forward()
        c.check_backward()
        c = Case(heads=(3, 2), norm=norm, grid=(3, 4, 5))
        grads = c.gradients()
        want = c.backward(grads)
        dq, dk = torch.empty_like(want[0]), torch.empty_like(want[1])
        layer.lite_attn_rotary_bwd(c.desc, ref.heads_view(c.q), ref.heads_view(c.k), *map(ref.heads_view, grads),
                                   ref.heads_view(dq), ref.heads_view(dk), c.freqs.data_ptr(), q_weight=ref.at(c.w[0]),
                                   k_weight=ref.at(c.w[1]), **c.places())
        assert torch.equal(dq, want[0]) and torch.equal(dk, want[1])
    c = Case(heads=(3, 2), grid=(3, 4, 5))
    grads = c.gradients()
    want = c.backward(grads)
    dq, dk = torch.empty_like(want[0]), torch.empty_like(want[1])
    layer.lite_attn_rotary_bwd(c.desc, None, None, *map(ref.heads_view, grads), ref.heads_view(dq), ref.heads_view(dk),
                               c.freqs.data_ptr(), **c.places())  # no norm: the inputs are not needed
    assert torch.equal(dq, want[0]) and torch.equal(dk, want[1])


def test_no_tokens():
    c = Case(batch=2, heads=(3, 3), n=0, norm="head")
    c.forward()
    assert all((dw == 0).all() for dw in c.backward(c.gradients())[2])


def test_infinities_stay_with_their_token():
    c = Case(batch=1, heads=(3, 3), grid=(2, 3, 4), norm="row", dtype="f32")
    clean = c.forward()[0].clone()
    c.q[0, 1, 5, 7] = float("inf")
    c.q[0, 2, 9, 0] = float("nan")
    got = c.forward()[0]
    others = [t for t in range(24) if t not in (5, 9)]
    assert torch.equal(got[:, :, others], clean[:, :, others])
    assert torch.isnan(got[0, 1, 5, 7]) and torch.isnan(got[0, :, 9]).all()


@pytest.mark.parametrize("d,pairs", [(128, 40), (72, 30), (64, 0), (20, 7)])
@pytest.mark.parametrize("halves", [False, True])
def test_entries_that_are_not_turned_stand_alone(d, pairs, halves):
    c = Case(heads=(3, 2), d=d, pairs=pairs, grid=(2, 3, 4), halves=halves)
    grads = c.gradients()
    want, wdq = c.forward()[0].clone(), c.backward(grads)[0].clone()
    for column in range(2 * pairs, d, 5):
        for bad in (float("inf"), float("nan")):
            kept = c.q[0, 1, 7, column].clone(), grads[0][0, 1, 7, column].clone()
            c.q[0, 1, 7, column] = grads[0][0, 1, 7, column] = bad
            got, dq = c.forward()[0], c.backward(grads)[0]
            for new, old in ((got, want), (dq, wdq)):
                assert torch.equal(torch.isfinite(new), torch.ones_like(new, dtype=torch.bool).index_put_(
                    tuple(torch.tensor([x], device="cuda") for x in (0, 1, 7, column)), torch.tensor(False, device="cuda")))
                new[0, 1, 7, column] = old[0, 1, 7, column]
                assert torch.equal(new, old)
            c.q[0, 1, 7, column], grads[0][0, 1, 7, column] = kept


def test_rows_beyond_4_gib():
    """A tensor whose tokens lie more than 2^32 bytes and 2^31 elements apart from its start."""
    c = Case(heads=(2, 2), d=64, grid=(1, 2, 2), norm="head")
    stride = (1 << 30) + 64
    big = torch.empty(3 * stride + 2 * 64, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((1, 2, 4, 64), (0, 64, stride, 1))
    far.copy_(c.q)
    want = c.forward()[0]
    c.q = far
    assert torch.equal(c.forward()[0], want)
    out = torch.empty(3 * stride + 2 * 64, dtype=torch.bfloat16, device="cuda").as_strided((1, 2, 4, 64), (0, 64, stride, 1))
    assert torch.equal(c.forward(q_out=out)[0], want)


def test_gradient_against_differences():
    """(f(x + h v) - f(x - h v)) / 2h, f the sum of the results times fixed factors, against the gradient times v.  In 32 bits f is
    off by 2^-20 of the sum of its terms' sizes at most; with h = 2^-6 the difference's own error, h^2 / 6 of a third derivative of
    a few units, is smaller yet."""
    c = Case(batch=2, heads=(3, 3), d=64, grid=(2, 3, 4), dtype="f32", norm="row", halves=True)
    grads = c.gradients()
    dq, dk, dw = c.backward(grads)
    x0 = c.q.clone()
    h = 2.0 ** -6

    def f():
        out = c.forward()[0].double() * grads[0].double()
        return out.sum().item(), out.abs().sum().item()

    for trial in range(4):
        v = ref.randn(c.g, *c.q.shape)
        c.q.copy_(x0 + h * v)
        up, size = f()
        c.q.copy_(x0 - h * v)
        down, _ = f()
        c.q.copy_(x0)
        want = (dq.double() * v.double()).sum().item()
        third = (v.norm() ** 3 / x0.norm() * 6).item() * h * h / 6 + 1e-3 * abs(want)
        assert abs((up - down) / (2 * h) - want) <= 2 * 2.0 ** -20 * size / (2 * h) + third


def test_same_bits_every_time_on_any_stream_and_from_a_graph():
    c = Case(batch=2, heads=(6, 3), grid=(5, 9, 13), norm="row", text=5)
    grads = c.gradients()
    want_f, want_b = c.forward(), c.backward(grads)

    def same(f, b):
        assert all(torch.equal(x, y) for x, y in zip(f, want_f))
        assert torch.equal(b[0], want_b[0]) and torch.equal(b[1], want_b[1])
        assert all(torch.equal(x, y) for x, y in zip(b[2], want_b[2]))

    same(c.forward(), c.backward(grads))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f, b = c.forward(), c.backward(grads)
    side.synchronize()
    same(f, b)
    graph = torch.cuda.CUDAGraph()
    q_out, k_out = torch.empty_like(want_f[0]), torch.empty_like(want_f[1])
    dq, dk = torch.empty_like(want_b[0]), torch.empty_like(want_b[1])
    dw = [torch.empty_like(x) for x in want_b[2]]
    need = layer.lite_attn_rotary_bwd_workspace(c.desc)
    space = torch.empty(need // 4, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.forward(q_out=q_out, k_out=k_out)
        layer.lite_attn_rotary_bwd(c.desc, ref.heads_view(c.q), ref.heads_view(c.k), *map(ref.heads_view, grads),
                                   ref.heads_view(dq), ref.heads_view(dk), c.freqs.data_ptr(), q_weight=ref.at(c.w[0]),
                                   k_weight=ref.at(c.w[1]), dq_weight=ref.at(dw[0]), dk_weight=ref.at(dw[1]),
                                   workspace=space.data_ptr(), workspace_bytes=need, **c.places())
    for _ in range(3):
        for t in (q_out, k_out, dq, dk, *dw):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        same((q_out, k_out), (dq, dk, dw))
        same(c.forward(), c.backward(grads))
