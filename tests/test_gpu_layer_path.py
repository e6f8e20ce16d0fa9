"""The operators around the attention call run together, as a block of a model uses them, each step against its definition in 64
bits on what the step before left."""
import math

import pytest
import torch

import layer_reference as ref
from paper_2511_11062_amd import inputs, layer, report
from paper_2511_11062_amd import lite_attn as la

pytestmark = pytest.mark.gpu

SLACK = 2.0 ** -18  # 32-bit arithmetic, as in the operators' own tests
GRID, TEXT, HEADS, BATCH = (3, 9, 11), 37, 3, 2
N, DIM = 3 * 9 * 11 + 37, 3 * 128


class Block:
    """x -> norm, scale, shift -> q, k, v -> norm over the token, positions -> attention -> projection -> gate, stream, norm."""

    def __init__(self):
        g = ref.gen(71)
        self.x = 2.0 * ref.randn(g, BATCH, N, DIM) + 0.5
        self.mod = 0.3 * ref.randn(g, BATCH, 6, DIM)
        self.w_qkv = (ref.randn(g, DIM, 3 * DIM) / math.sqrt(DIM)).bfloat16()
        self.w_out = (ref.randn(g, DIM, DIM) / math.sqrt(DIM)).bfloat16()
        self.wq, self.wk = (1.0 + 0.2 * ref.randn(g, HEADS, 128) for _ in range(2))
        self.freqs = torch.from_numpy(layer.lite_attn_rotary_freqs((22, 21, 21)).copy()).cuda()
        self.norm = layer.make_residual_desc(BATCH, N, DIM)
        self.rotary = layer.make_rotary_desc(BATCH, N, HEADS, HEADS, norm=layer.LITE_ATTN_NORM_ROW, grid=GRID)
        self.mask = la.lite_attn_init_mask(BATCH, HEADS, N, max_steps=4, protect=(N - TEXT, TEXT))
        empty = lambda *s: torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda")
        self.h, self.h2 = empty(BATCH, N, DIM), empty(BATCH, N, DIM)
        self.x2 = torch.full_like(self.x, float("nan"))
        self.q, self.k, self.v, self.o = (empty(BATCH, HEADS, N, 128) for _ in range(4))

    def row(self, i):
        t = self.mod[:, i:i + 1]
        return t.data_ptr(), t.stride(0), t.stride(1)

    def run(self, step):
        s = torch.cuda.current_stream().cuda_stream  # the mask's too
        layer.lite_attn_residual_norm_fwd(self.norm, ref.rows_view(self.x), None, None, ref.rows_view(self.h), scale=self.row(0),
                                          shift=self.row(1), hip_stream=s)
        self.qkv = (self.h @ self.w_qkv).view(BATCH, N, 3 * HEADS, 128)
        q, k, v = (self.qkv[:, :, i * HEADS:(i + 1) * HEADS].transpose(1, 2) for i in range(3))
        layer.lite_attn_rotary_fwd(self.rotary, ref.heads_view(q), ref.heads_view(k), ref.heads_view(self.q),
                                   ref.heads_view(self.k), self.freqs.data_ptr(), q_weight=self.wq.data_ptr(),
                                   k_weight=self.wk.data_ptr(), hip_stream=s)
        self.v.copy_(v)
        la.lite_attn_fwd(self.q.data_ptr(), self.k.data_ptr(), self.v.data_ptr(), self.o.data_ptr(), self.mask, -float("inf"), step)
        self.y = self.o.transpose(1, 2).reshape(BATCH, N, DIM) @ self.w_out
        layer.lite_attn_residual_norm_fwd(self.norm, ref.rows_view(self.x), ref.rows_view(self.y), ref.rows_view(self.x2),
                                          ref.rows_view(self.h2), gate=self.row(2), scale=self.row(3), shift=self.row(4),
                                          hip_stream=s)

    def check(self):
        m = self.mod.double()
        x = self.x.double()

        def modulated(t, scale, shift):
            n = ref.normed(t, "layer", 1e-6)
            r = 1.0 / torch.sqrt((t - t.mean(dim=-1, keepdim=True)).square().mean(dim=-1, keepdim=True) + 1e-6)
            size = r * (t.abs() + t.abs().mean(dim=-1, keepdim=True))
            return n * (1.0 + scale) + shift, 2 * SLACK * ((1.0 + scale).abs() * size + shift.abs())

        want, slack = modulated(x, m[:, 0:1], m[:, 1:2])
        ref.check("h", self.h, want, slack)
        pos = ref.grid_positions(GRID, 0, N)[None]
        for i, (got, w) in enumerate(((self.q, self.wq), (self.k, self.wk))):
            t = self.qkv[:, :, i * HEADS:(i + 1) * HEADS].transpose(1, 2).double()
            want = ref.rotary(t, w.double(), self.freqs, pos, "row", False, 1e-6)
            ref.check("qk"[i], got, want, 2.0 ** -19 * ref.partner_sum(want, 64, False) * 1.5)
        q, k, v = (t.double() for t in (self.q, self.k, self.v))
        want = torch.softmax(q @ k.transpose(2, 3).contiguous() / math.sqrt(128.0), dim=-1) @ v
        off = (self.o.double() - want).abs()
        assert off.max() <= 1e-2 * want.abs().max() and off.mean() <= 1e-3  # the attention call's own tolerances
        x2 = x + m[:, 2:3] * self.y.double()
        off = SLACK * (x.abs() + (m[:, 2:3] * self.y.double()).abs())
        ref.check("x2", self.x2, x2, off)
        want, slack = modulated(x2, m[:, 3:4], m[:, 4:5])
        ref.check("h2", self.h2, want, slack)


def test_a_block():
    b = Block()
    try:
        la.lite_attn_set_stream(b.mask, torch.cuda.current_stream().cuda_stream)
        b.run(0)
        torch.cuda.synchronize()
        b.check()
    finally:
        la.lite_attn_free_mask(b.mask)


def test_a_block_from_a_graph():
    """Captured with the attention call between them and replayed on new inputs, eager work in between."""
    b = Block()
    try:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            la.lite_attn_set_stream(b.mask, side.cuda_stream)
            b.run(0)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.run(0)
        g = ref.gen(72)
        for _ in range(3):
            b.x.copy_(2.0 * ref.randn(g, BATCH, N, DIM) - 0.5)
            b.x2.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            b.check()
    finally:
        la.lite_attn_free_mask(b.mask)


def test_report_turns_its_inputs():
    wl = inputs.Workload("path", 1, 2, (2, 12, 13), text_tokens=20, steps=2, seed=5)
    seq = inputs.DriftSequence(wl, "cuda:0")
    data = [next(seq) for _ in range(2)]
    freqs = torch.from_numpy(layer.lite_attn_rotary_freqs((22, 21, 21)).copy()).cuda()
    pos = ref.grid_positions(wl.grid, 0, wl.seqlen)[None]
    turned = [(*report.turn_by_position(wl, q, k), v) for q, k, v in data]
    for (q, k, _), (tq, tk, _) in zip(data, turned):
        for a, b in ((q, tq), (k, tk)):
            want = ref.rotary(a.double(), None, freqs, pos, "none", False, 0.0)
            ref.check("turned", b, want, 2.0 ** -19 * ref.partner_sum(want, 64, False) * 1.5)
        assert torch.equal(tq[:, :, wl.video_tokens:], q[:, :, wl.video_tokens:])
    dense, rows = report.run_sequence(wl, turned, [-float("inf")] * 2)
    assert len(dense) == 2 and all(torch.isfinite(o).all() for o in dense)
    _, rows = report.run_sequence(wl, turned, [-3.0] * 2, dense)
    assert all(0.0 <= r["eta"] < 1.0 for r in rows)
