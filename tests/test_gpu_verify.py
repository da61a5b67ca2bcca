"""Verification of drafted tokens against the rule itself, one sequence and one token at a time, in exact fractions (64 bits
for vocabularies of thousands): every output has to be equal."""
from fractions import Fraction

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hire():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2402_09360_amd import hire as H
    return H


def distribution(prob, idx, vocab, exact):
    """[(token, probability)] in the order in which sums run; of entries of one token the first."""
    num = Fraction if exact else float
    if idx is None:
        return [(v, num(float(x))) for v, x in enumerate(prob)]
    out, seen = [], set()
    for v, x in zip(idx.tolist(), prob.tolist()):
        if 0 <= v < vocab and v not in seen:
            seen.add(v)
            out.append((v, num(x)))
    return out


def expected(c, exact=True):
    B, n, vocab = c["B"], c["n"], c["vocab"]
    num = Fraction if exact else float
    at = lambda name, b, i: None if c.get(name) is None else c[name][b, i]
    tokens_out, accepted_out = np.full((B, n + 1), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        length = n if c.get("lengths") is None else min(max(int(c["lengths"][b]), 0), n)
        a, refused = 0, False
        while a < length:
            d = int(c["tokens"][b, a])
            p = dict(distribution(c["target"][b, a], at("target_idx", b, a), vocab, exact))
            if c.get("draft") is None:
                q = {d: num(1)}
            else:
                q = dict(distribution(c["draft"][b, a], at("draft_idx", b, a), vocab, exact))
            if not (0 <= d < vocab and num(float(c["accept_u"][b, a])) * q.get(d, num(0)) < p.get(d, num(0))):
                refused = True
                break
            tokens_out[b, a] = d
            a += 1
        p = distribution(c["target"][b, a], at("target_idx", b, a), vocab, exact)
        rest = [(v, max(x - (q.get(v, num(0)) if refused else num(0)), num(0))) for v, x in p]
        if not any(x > 0 for _, x in rest):
            rest = [(v, max(x, num(0))) for v, x in p]
        mark = num(float(c["sample_u"][b])) * sum(x for _, x in rest)
        run = num(0)
        for v, x in rest:
            run += x
            if run > mark:
                tokens_out[b, a] = v
                break
        accepted_out[b] = a
    return tokens_out, accepted_out


def call(hire, c, repeat=1):
    dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()
    drafts = hire.Drafts(dev(c["tokens"]), c["vocab"], dev(c["target"]), dev(c["accept_u"]), dev(c["sample_u"]),
                         target_idx=dev(c.get("target_idx")), draft_prob=dev(c.get("draft")), draft_idx=dev(c.get("draft_idx")),
                         lengths=dev(c.get("lengths")))
    nbytes = hire.hire_verify_draft_workspace_bytes(drafts)
    guard = torch.full((nbytes + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    ws = guard[256:256 + nbytes]
    ws.fill_(0xFF)
    out = hire.DraftOutputs(drafts)
    for _ in range(repeat):
        out.tokens.fill_(-7)
        out.accepted.fill_(-7)
        hire.hire_verify_draft(drafts, out, ws)
    torch.cuda.synchronize()
    assert bool((guard[:256] == 0x5A).all()) and bool((guard[256 + nbytes:] == 0x5A).all())
    return out.tokens.cpu().numpy(), out.accepted.cpu().numpy()


def same(hire, c, exact=True):
    got, want = call(hire, c), expected(c, exact)
    assert np.array_equal(got[1], want[1]), (got[1], want[1])
    assert np.array_equal(got[0], want[0]), (got[0], want[0])
    return got


def draw(seed, B, n, vocab, target, draft, k=8, ragged=True, kd=None):
    """Two alike distributions, tokens mostly from the draft's largest entries, garbage behind a sequence's length."""
    rng = np.random.default_rng(seed)
    kd = kd or k
    z = rng.standard_normal((B, n + 1, vocab)) * 2
    zq = z[:, :n] + 0.5 * rng.standard_normal((B, n, vocab))
    soft = lambda t: (np.exp(t - t.max(-1, keepdims=True)) / np.exp(t - t.max(-1, keepdims=True)).sum(-1, keepdims=True)).astype(np.float32)
    top = lambda t, m: np.argsort(-t, axis=-1, kind="stable")[..., :m].astype(np.int32)
    c = dict(B=B, n=n, vocab=vocab, accept_u=rng.random((B, n), np.float32), sample_u=rng.random(B, np.float32))
    if target == "dense":
        c["target"] = soft(z)
    else:
        c["target_idx"] = top(z, k)
        c["target"] = soft(np.take_along_axis(z, c["target_idx"], -1))
    if draft == "dense":
        c["draft"] = soft(zq)
    elif draft == "list":
        c["draft_idx"] = top(zq, kd)
        c["draft"] = soft(np.take_along_axis(zq, c["draft_idx"], -1))
    rank = np.minimum(rng.geometric(0.6, (B, n)) - 1, vocab - 1)
    c["tokens"] = np.take_along_axis(top(zq, vocab), rank[..., None], -1)[..., 0].astype(np.int32) if n else np.zeros((B, 0), np.int32)
    if ragged and n:
        c["lengths"] = rng.integers(0, n + 1, B).astype(np.int32)
        for b, length in enumerate(c["lengths"]):
            c["tokens"][b, length:] = 0x7FFFFFFF
            c["accept_u"][b, length:] = np.nan
            c["target"][b, length + 1:] = np.nan
            if "draft" in c:
                c["draft"][b, length:] = np.nan
            for name in ("target_idx", "draft_idx"):
                if name in c:
                    c[name][b, length + (name == "target_idx"):] = -(1 << 31)
    return c


@pytest.mark.parametrize("target", ["dense", "list"])
@pytest.mark.parametrize("draft", ["dense", "list", "certain"])
@pytest.mark.parametrize("B,n,vocab,k", [(1, 1, 1, 1), (3, 2, 2, 2), (5, 4, 37, 8), (70, 3, 130, 65), (2, 63, 40, 7), (4, 0, 50, 9)])
def test_small_vocabularies(hire, target, draft, B, n, vocab, k):
    if n == 0 and draft != "certain":
        draft = "certain"
    print(target, draft, B, n, vocab, k, flush=True)
    for seed in range(4):
        same(hire, draw(seed, B, n, vocab, target, draft, k, ragged=seed % 2 == 0, kd=max(1, k - 1)))


@pytest.mark.parametrize("target,draft", [("dense", "dense"), ("dense", "list"), ("dense", "certain"), ("list", "dense"),
                                          ("list", "list"), ("list", "certain")])
@pytest.mark.parametrize("B,n,vocab,k", [(1, 3, 50021, 700), (6, 2, 4099, 4096), (2, 5, 20000, 1025), (1, 1, 300000, 33)])
def test_long_rows(hire, target, draft, B, n, vocab, k):
    print(target, draft, B, n, vocab, k, flush=True)
    same(hire, draw(vocab + B, B, n, vocab, target, draft, k, ragged=False, kd=k // 2 + 1), exact=False)


def test_many_sequences_of_long_rows(hire):
    same(hire, draw(9, 80, 1, 33000, "dense", "dense"), exact=False)


def edge(vocab=8, n=3, **changes):
    """A sequence of which every token is accepted, uniform distributions; changes by name."""
    c = dict(B=1, n=n, vocab=vocab, tokens=np.arange(n, dtype=np.int32)[None] % vocab,
             target=np.full((1, n + 1, vocab), 1.0 / vocab, np.float32), draft=np.full((1, n, vocab), 1.0 / vocab, np.float32),
             accept_u=np.full((1, n), 0.5, np.float32), sample_u=np.full(1, 0.5, np.float32))
    c.update(changes)
    return c


def test_edges_of_the_rule(hire):
    below_one = np.float32(1.0 - 2.0 ** -24)
    assert same(hire, edge())[1][0] == 3
    assert same(hire, edge(sample_u=np.zeros(1, np.float32)))[0][0, 3] == 0
    assert same(hire, edge(sample_u=np.full(1, below_one)))[0][0, 3] == 7
    assert same(hire, edge(accept_u=np.full((1, 3), below_one)))[1][0] == 3
    # u q = p is refused, and then nothing is left of p - q: the target's distribution itself
    c = edge(accept_u=np.array([[0.5, 1.0, 0.5]], np.float32))
    assert same(hire, c)[1][0] == 1
    # a drafted token without probability in either distribution
    c = edge()
    c["target"][0, 1, 1] = 0.0
    assert same(hire, c)[1][0] == 1
    c = edge()
    c["draft"][0, 1, 1] = 0.0
    assert same(hire, c)[1][0] == 3
    # mass at one place only, the first and the last; none at all
    for place in (0, 7):
        c = edge()
        c["target"][0, 3] = 0.0
        c["target"][0, 3, place] = 1e-30
        for s in (0.0, 0.3, float(below_one)):
            c["sample_u"] = np.full(1, s, np.float32)
            assert same(hire, c)[0][0, 3] == place
    c = edge()
    c["target"][0, 3] = 0.0
    assert same(hire, c)[0][0, 3] == -1
    c["target"][0, 0] = 0.0
    assert same(hire, c)[0].tolist() == [[-1, -1, -1, -1]]
    # tokens outside the vocabulary are refused and taken off nothing
    for bad in (-1, 8, 1 << 30, -(1 << 31)):
        for draft in (np.full((1, 3, 8), 0.01, np.float32), None):
            c = edge(tokens=np.array([[0, bad, 2]], np.int32), draft=draft, accept_u=np.zeros((1, 3), np.float32))
            assert same(hire, c)[1][0] == 1
    # lengths beyond either end
    assert same(hire, edge(lengths=np.array([99], np.int32)))[1][0] == 3
    assert same(hire, edge(lengths=np.array([-5], np.int32)))[1][0] == 0


@pytest.mark.parametrize("dense_target", [False, True])
def test_lists_with_repeats_and_padding(hire, dense_target):
    """The first entry of a token counts; entries that name no token do not."""
    rng = np.random.default_rng(3)
    for seed in range(6):
        c = draw(100 + seed, 4, 3, 40, "dense" if dense_target else "list", "list", k=20, ragged=False)
        for name in ("target_idx", "draft_idx"):
            if name in c:
                idx = c[name]
                idx[...] = rng.integers(-3, 44, idx.shape)
        same(hire, c)


@pytest.mark.parametrize("target,draft", [("dense", "dense"), ("dense", "list"), ("list", "list"), ("list", "dense")])
def test_rows_that_start_anywhere(hire, target, draft):
    """Distributions at addresses that are multiples of four bytes and of nothing more."""
    c = draw(77, 5, 3, 2048, target, draft, 100, ragged=False)
    want = expected(c, exact=False)

    def moved(name):
        if c.get(name) is None:
            return None
        t = torch.from_numpy(np.ascontiguousarray(c[name]))
        buffer = torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda")
        buffer[1:1 + t.numel()] = t.cuda().flatten()
        return buffer[1:1 + t.numel()].view(t.shape)

    drafts = hire.Drafts(moved("tokens"), c["vocab"], moved("target"), moved("accept_u"), moved("sample_u"),
                         target_idx=moved("target_idx"), draft_prob=moved("draft"), draft_idx=moved("draft_idx"))
    out = hire.DraftOutputs(drafts)
    hire.hire_verify_draft(drafts, out, hire.alloc_workspace(hire.hire_verify_draft_workspace_bytes(drafts)))
    assert np.array_equal(out.tokens.cpu().numpy(), want[0]) and np.array_equal(out.accepted.cpu().numpy(), want[1])


def test_repeats_are_equal(hire):
    for target, draft in (("dense", "dense"), ("list", "list")):
        c = draw(5, 7, 4, 9000, target, draft, 300)
        first, again = call(hire, c), call(hire, c, repeat=3)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


@pytest.mark.parametrize("target,draft", [("dense", "list"), ("dense", "dense"), ("list", "list")])
def test_captured_and_replayed(hire, target, draft):
    cases = [draw(20 + s, 5, 3, 3001, target, draft, 64, ragged=False) for s in range(4)]
    names = [n for n in ("tokens", "target", "target_idx", "draft", "draft_idx", "accept_u", "sample_u") if n in cases[0]]
    t = {n: torch.from_numpy(cases[0][n]).cuda() for n in names}
    drafts = hire.Drafts(t["tokens"], 3001, t["target"], t["accept_u"], t["sample_u"], target_idx=t.get("target_idx"),
                         draft_prob=t["draft"], draft_idx=t.get("draft_idx"))
    out, ws = hire.DraftOutputs(drafts), hire.alloc_workspace(hire.hire_verify_draft_workspace_bytes(drafts))
    hire.hire_verify_draft(drafts, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hire.hire_verify_draft(drafts, out, ws)
    for c in cases[1:] + cases[:1]:
        for n in names:
            t[n].copy_(torch.from_numpy(c[n]))
        graph.replay()
        torch.cuda.synchronize()
        want = expected(c, exact=False)
        assert np.array_equal(out.tokens.cpu().numpy(), want[0]) and np.array_equal(out.accepted.cpu().numpy(), want[1])


def test_binding_refuses(hire):
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")
    tok, p, u, s = z(2, 3, dtype=torch.int32), z(2, 4, 10), z(2, 3), z(2)
    hire.Drafts(tok, 10, p, u, s)
    idx = z(2, 4, 10, dtype=torch.int32)
    for bad in (lambda: hire.Drafts(tok.long(), 10, p, u, s), lambda: hire.Drafts(tok, 11, p, u, s),
                lambda: hire.Drafts(tok, 10, p[:, :3], u, s), lambda: hire.Drafts(tok, 10, p, u[:, :2], s),
                lambda: hire.Drafts(tok, 10, p, u, s[:1]), lambda: hire.Drafts(tok, 10, p.double(), u, s),
                lambda: hire.Drafts(tok, 10, p, u, s, target_idx=idx[:, :, :5]),
                lambda: hire.Drafts(tok, 10, p, u, s, target_idx=idx.long()),
                lambda: hire.Drafts(tok, 10, p, u, s, draft_prob=p), lambda: hire.Drafts(tok, 10, p, u, s, draft_idx=idx),
                lambda: hire.Drafts(tok, 10, p, u, s, lengths=tok), lambda: hire.Drafts(tok.cpu(), 10, p, u, s)):
        with pytest.raises(hire.HireError):
            bad()
    drafts = hire.Drafts(tok, 10, p, u, s)
    with pytest.raises(hire.HireError):
        hire.hire_verify_draft(drafts, hire.DraftOutputs(drafts), torch.empty(0, dtype=torch.uint8, device="cuda"))
