"""The dense operators next to the sparse steps, as a decode with drafted tokens runs them: a dense gated layer, the draft's
distributions from the 4-bit copy of the classifier and a bare selection, the target's from the classifier step, and the
verification of the drafts; eagerly, on a stream of its own, and as a replayed graph."""
import numpy as np
import pytest
import torch

import hire_testlib as T
from paper_2402_09360_amd import inputs as I

pytestmark = pytest.mark.gpu

D, UNITS, VOCAB, B, N, K, KP = 256, 1024, 4096, 3, 4, 32, 256


@pytest.fixture(scope="module")
def hire():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2402_09360_amd import hire as H
    return H


class Decode:
    """What a program keeps: layers, outputs, one workspace per entry point."""

    def __init__(self, hire, seed):
        self.hire = hire
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        draw = lambda *shape, std=1.0: (torch.randn(shape, generator=gen, device="cuda") * std).to(torch.bfloat16)
        self.x = draw(B * (N + 1), D)
        self.layer = hire.GatedLayer(draw(UNITS, D, std=D ** -0.5), draw(UNITS, D, std=D ** -0.5), draw(UNITS, D, std=UNITS ** -0.5))
        w = draw(VOCAB, D, std=4 * D ** -0.5)
        self.classifier = hire.SoftmaxLayer.with_int4_scorer(w)
        self.copy = hire.hire_pack_mxfp4(w)
        rows = B * (N + 1)
        self.ffn = hire.GatedOutputs(self.layer, rows)
        self.ffn_ws = hire.alloc_workspace(hire.hire_gated_ffn_workspace_bytes(self.layer, rows))
        self.top = hire.SoftmaxOutputs(self.classifier, rows, K, KP)
        self.top_ws = hire.alloc_workspace(hire.hire_softmax_workspace_bytes(self.classifier, rows, K, KP))
        self.logits = torch.empty((B * N, VOCAB), device="cuda")
        self.mx_ws = hire.alloc_workspace(hire.hire_mxfp4_product_workspace_bytes(B * N, VOCAB, D))
        self.select_ws = hire.alloc_workspace(max(256, hire.hire_topk_workspace_bytes(B * N, VOCAB, K, hire.ORDER_RANK)))
        self.u, self.s = (torch.rand(shape, generator=gen, device="cuda") for shape in ((B, N), (B,)))
        self.draft_prob = torch.empty((B, N, K), device="cuda")
        self.draft_idx = torch.empty((B, N, K), dtype=torch.int32, device="cuda")
        self.tokens = torch.empty((B, N), dtype=torch.int32, device="cuda")
        self.drafts = hire.Drafts(self.tokens, VOCAB, self.top.top_prob.view(B, N + 1, K), self.u, self.s,
                                  target_idx=self.top.top_idx.view(B, N + 1, K), draft_prob=self.draft_prob,
                                  draft_idx=self.draft_idx)
        self.out = hire.DraftOutputs(self.drafts)
        self.ver_ws = hire.alloc_workspace(hire.hire_verify_draft_workspace_bytes(self.drafts))

    def step(self, stream=None):
        h = self.hire
        h.hire_gated_ffn_step(self.layer, self.x, self.ffn, self.ffn_ws, stream=stream)
        y = self.ffn.y.view(B, N + 1, D)
        drafted = y[:, :N].reshape(B * N, D)
        h.hire_mxfp4_product_bf16(drafted, self.copy, self.logits, self.mx_ws, stream=stream)
        idx, val = h.topk_select(self.logits, K, rank_order=True, workspace=self.select_ws, stream=stream)
        self.draft_idx.copy_(idx.view(B, N, K))
        self.draft_prob.copy_(torch.softmax(val, dim=1).view(B, N, K))
        self.tokens.copy_(self.draft_idx[:, :, 0])
        h.hire_softmax_step(self.classifier, self.ffn.y, K, KP, self.top, self.top_ws, stream=stream)
        h.hire_verify_draft(self.drafts, self.out, self.ver_ws, stream=stream)

    def result(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.ffn.y, self.logits, self.top.top_idx, self.top.top_prob, self.draft_idx, self.draft_prob,
                                    self.out.tokens, self.out.accepted)]


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_against_the_definitions(hire):
    for seed in (1, 2, 3):
        d = Decode(hire, seed)
        d.step()
        y, logits, top_idx, top_prob, draft_idx, draft_prob, tokens, accepted = d.result()
        x, wg, wu, w2 = (t.double() for t in (d.x, d.layer.wg, d.layer.wu, d.layer.w2u))
        g = x @ wg.t()
        want = (g * torch.sigmoid(g) * (x @ wu.t())) @ w2
        assert float((y.double() - want).abs().max()) <= 2.0 ** -7 * float(want.abs().max())
        drafted = y.view(B, N + 1, D)[:, :N].reshape(B * N, D).double()
        want = drafted @ hire.hire_unpack_mxfp4(d.copy).double().t()
        room = 2 * (D + 8) * 2.0 ** -24 * (drafted.abs() @ hire.hire_unpack_mxfp4(d.copy).double().abs().t())
        assert bool(((logits.double() - want).abs() <= room).all())
        # the verification of these very lists, token by token
        for b in range(B):
            a = 0
            while a < N:
                t = int(d.tokens[b, a])
                p = dict(zip(top_idx.view(B, N + 1, K)[b, a].tolist(), top_prob.view(B, N + 1, K)[b, a].tolist()))
                q = dict(zip(draft_idx[b, a].tolist(), draft_prob[b, a].tolist()))
                if not float(d.u[b, a]) * q[t] < p.get(t, 0.0):
                    break
                assert int(tokens[b, a]) == t
                a += 1
            assert int(accepted[b]) == a
            names, probs = top_idx.view(B, N + 1, K)[b, a].tolist(), top_prob.view(B, N + 1, K)[b, a].double().tolist()
            if a < N:
                q = dict(zip(draft_idx[b, a].tolist(), draft_prob[b, a].double().tolist()))
                probs = [max(p - q.get(v, 0.0), 0.0) for v, p in zip(names, probs)]
            run = np.cumsum(probs)
            assert int(tokens[b, a]) == names[int(np.argmax(run > float(d.s[b]) * run[-1]))]
            assert all(int(v) == -1 for v in tokens[b, a + 1:])


def test_stream_of_its_own_and_replays(hire):
    d = Decode(hire, 4)
    d.step()
    want = d.result()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        d.step()
    assert equal(d.result(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.step()
    for seed in (5, 6, 7):
        other = Decode(hire, seed)
        d.x.copy_(other.x)
        d.u.copy_(other.u)
        d.s.copy_(other.s)
        graph.replay()
        got = d.result()
        d.step()
        assert equal(got, d.result())


def test_two_streams_at_once(hire):
    """Workspaces of their own: the same results as one after the other."""
    pair = [Decode(hire, 8), Decode(hire, 9)]
    want = []
    for d in pair:
        d.step()
        want.append(d.result())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for d, s in zip(pair, streams):
            with torch.cuda.stream(s):
                d.step()
    for d, w in zip(pair, want):
        assert equal(d.result(), w)


def test_explicit_stream_argument(hire):
    d = Decode(hire, 10)
    d.step()
    want = d.result()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    hire.hire_gated_ffn_step(d.layer, d.x, d.ffn, d.ffn_ws, stream=side)
    hire.hire_softmax_step(d.classifier, d.ffn.y, K, KP, d.top, d.top_ws, stream=side)
    hire.hire_verify_draft(d.drafts, d.out, d.ver_ws, stream=side)
    assert equal(d.result(), want)


def test_training_steps_see_the_changed_weights(hire):
    """Two steps of gradient descent on a layer: the gradients that the second step sees are those of the changed weights."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    draw = lambda *shape, std=1.0: (torch.randn(shape, generator=gen, device="cuda") * std).to(torch.bfloat16)
    x, goal = draw(96, 64), draw(96, 64)
    layer = hire.GatedLayer(draw(128, 64, std=0.125), draw(128, 64, std=0.125), draw(128, 64, std=0.1), act="gelu")
    out, grads = hire.GatedOutputs(layer, 96, train=True), hire.GatedGradients(layer, 96)
    ws = hire.alloc_workspace(max(hire.hire_gated_ffn_workspace_bytes(layer, 96),
                                  hire.hire_gated_ffn_backward_workspace_bytes(layer, 96)))
    for _ in range(2):
        hire.hire_gated_ffn_step(layer, x, out, ws)
        dy = (out.y.float() - goal.float()).to(torch.bfloat16)
        hire.hire_gated_ffn_backward(layer, x, out, dy, grads, ws)
        leaves = [t.double().requires_grad_(True) for t in (x, layer.wg, layer.wu, layer.w2u)]
        xd, wg, wu, w2 = leaves
        y = (torch.nn.functional.gelu(xd @ wg.t(), approximate="tanh") * (xd @ wu.t())) @ w2
        y.backward(dy.double())
        for got, leaf in zip((grads.dx, grads.dwg, grads.dwu, grads.dw2u), leaves):
            # three roundings to bf16 (h; dg and du, or dh; the result), each off by at most 2^-8 of its value and by
            # 2^-8 / sqrt(3) in the root mean square: 2^-8 of the norm together, and twice that is allowed
            assert float((got.double() - leaf.grad).norm()) <= 2.0 ** -7 * float(leaf.grad.norm())
        for w, g in ((layer.wg, grads.dwg), (layer.wu, grads.dwu), (layer.w2u, grads.dw2u)):
            w.sub_((1e-3 * g.float()).to(torch.bfloat16))


def test_offsets_beyond_32_bits(hire):
    """Rows whose places lie beyond 2^32 bytes, checked against the same tokens alone."""
    rows, d, units = 140000, 64, 16384
    gen = torch.Generator(device="cuda")
    gen.manual_seed(12)
    draw = lambda *shape, std=1.0: (torch.randn(shape, generator=gen, device="cuda") * std).to(torch.bfloat16)
    layer = hire.GatedLayer(draw(units, d, std=0.125), draw(units, d, std=0.125), draw(units, d, std=units ** -0.5))
    x, dy = draw(rows, d), draw(rows, d)
    out, grads = hire.GatedOutputs(layer, rows, train=True), hire.GatedGradients(layer, rows)
    ws = hire.alloc_workspace(max(hire.hire_gated_ffn_workspace_bytes(layer, rows),
                                  hire.hire_gated_ffn_backward_workspace_bytes(layer, rows)))
    hire.hire_gated_ffn_step(layer, x, out, ws)
    hire.hire_gated_ffn_backward(layer, x, out, dy, grads, ws)
    torch.cuda.synchronize()
    tail = slice(rows - 100, rows)
    few, few_grads = hire.GatedOutputs(layer, 100, train=True), hire.GatedGradients(layer, 100)
    hire.hire_gated_ffn_step(layer, x[tail].contiguous(), few, ws)
    hire.hire_gated_ffn_backward(layer, x[tail].contiguous(), few, dy[tail].contiguous(), few_grads, ws)
    torch.cuda.synchronize()
    for a, b in ((out.y[tail], few.y), (grads.dx[tail], few_grads.dx)):   # other cuts of k: other orders of fp32 sums
        assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -7 * float(b.float().abs().max())
    del out, grads, ws, few, few_grads
    codes = torch.randint(0, 256, (600000, 8192), dtype=torch.uint8, device="cuda", generator=gen)
    w = hire.Mxfp4(codes, torch.randint(120, 126, (600000, 512), dtype=torch.uint8, device="cuda", generator=gen))
    last = hire.Mxfp4(codes[-64:].contiguous(), w.scales[-64:].contiguous())
    values = hire.hire_unpack_mxfp4(last).double()
    for tokens in (1, 5, 20):
        xt = draw(tokens, 16384)
        y = torch.empty((tokens, 600000), device="cuda")
        ws = hire.alloc_workspace(hire.hire_mxfp4_product_workspace_bytes(tokens, 600000, 16384))
        hire.hire_mxfp4_product_bf16(xt, w, y, ws)
        want = xt.double() @ values.t()
        room = 2 * (16384 + 8) * 2.0 ** -24 * (xt.double().abs() @ values.abs().t())
        assert bool(((y[:, -64:].double() - want).abs() <= room).all()), tokens
