"""The dense gated FFN, the microscaled 4-bit product and the verification of drafted tokens as a program uses them.

A case is one call pattern: a gated FFN layer for the tokens of a decode step or of a prompt, a training step of it
(forward and backward), a matrix in microscaled 4-bit floating point times tokens, the packing itself, or drafted tokens
checked against the target's probabilities.  `run` computes it with the framework's kernels where `own` is true and in
elementary torch operations otherwise; both take the same inputs, `exact` has the operators' definitions in 64 bits.

Sizes are those of the repository's configurations (d_model 256 / 2048, d_ff 1024 / 16384, 256000 classes, batches up to
64, lists of k = 64) and generic ones between and around them.
"""
import math

import torch

own = False

_C_GELU = 2.0 * math.sqrt(2.0 / math.pi)
_A_GELU = 0.044715


def listed():
    return [
        # a layer of config 1 for one token: the smallest call, launches and host time
        dict(name="gated_small_b1", op="gated", act="silu", T=1, d=256, ff=1024, train=False),
        # interactive decoding: one token through a dense layer of the ~1B decoder
        dict(name="gated_1b_b1", op="gated", act="silu", T=1, d=2048, ff=16384, train=False),
        # a batch of requests, or the drafted tokens of a few
        dict(name="gated_1b_b48", op="gated", act="gelu", T=48, d=2048, ff=16384, train=False),
        # a prompt of odd length
        dict(name="gated_1b_prompt1021", op="gated", act="silu", T=1021, d=2048, ff=16384, train=False),
        # a training step of a small odd layer: few tokens, sizes that fill no tile
        dict(name="gated_train_odd", op="gated", act="gelu", T=333, d=800, ff=2504, train=True),
        # continued training at the ~1B shape
        dict(name="gated_train_1b", op="gated", act="silu", T=4096, d=2048, ff=16384, train=True),
        # the classifier's logits of one token from its 4-bit copy
        dict(name="mx_classifier_b1", op="mx", form="bf16", T=1, rows=256000, cols=2048, y="f32"),
        # an FFN matrix for a ragged decode batch
        dict(name="mx_ffn_b33", op="mx", form="bf16", T=33, rows=16384, cols=2048, y="f32"),
        # a prompt: tokens quantised in the call, both operands microscaled
        dict(name="mx_prompt4096", op="mx", form="mx", T=4096, rows=16384, cols=2048, y="bf16"),
        # weights packed and read back, as a program converts a layer and checks it
        dict(name="mx_pack", op="pack", rows=16384, cols=2048),
        # sequences of four drafted tokens, both distributions the classifier step's lists
        dict(name="verify_lists_b8", op="verify", B=8, n=4, target="list", draft="list", V=256000, k=64),
        # a batch with dense distributions of both models
        dict(name="verify_dense_b48", op="verify", B=48, n=5, target="dense", draft="dense", V=256000, k=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gated"] * 5 + ["mx"] * 4 + ["pack"] + ["verify"] * 3)
    if op == "gated":
        train = rng.random() < 0.4
        d, ff = 8 * _log(rng, 32, 512), 8 * _log(rng, 64, 2048)
        most = min(8192, int(1.3e11 / (d * ff * (1 if train else 0.4))))
        T = rng.choice([1, _log(rng, 2, 64), _log(rng, 65, most), _log(rng, 65, most)])
        act = rng.choice(["silu", "gelu"] if train else ["silu", "gelu", "relu"])
        return dict(op=op, act=act, T=T, d=d, ff=ff, train=train)
    if op == "mx":
        form, cols = rng.choice(["bf16", "mx"]), 32 * _log(rng, 8, 256)
        rows = _log(rng, 100, min(256000, (1 << 29) // cols))
        T = rng.choice([1, _log(rng, 2, 64)])
        if form == "mx" and rng.random() < 0.6:
            T = _log(rng, 65, max(66, min(8192, int(1.3e11 / (rows * cols)))))
        return dict(op=op, form=form, T=T, rows=rows, cols=cols, y=rng.choice(["f32", "bf16"]))
    if op == "pack":
        cols = 32 * _log(rng, 1, 512)
        return dict(op=op, rows=_log(rng, 1, max(2, min(65536, (1 << 26) // cols))), cols=cols)
    target = rng.choice(["list", "dense"])
    draft = rng.choice(["list", "dense", "certain"])
    V = _log(rng, 1000, 256000)
    n = rng.randint(1, 12)
    return dict(op=op, B=_log(rng, 1, 64), n=n, target=target, draft=draft, V=V,
                k=_log(rng, 8, min(1024, V // 2)) if "list" in (target, draft) else 0)


# ---- inputs ----------------------------------------------------------------------------------------------------

class _Gen:
    """Seeded values on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 6007 + 29)

    def f32(self, shape, std=1.0):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32).mul_(std)

    def bf16(self, shape, std=1.0):
        return self.f32(shape, std).to(torch.bfloat16)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32)


def _pow2(e):
    """2^e in 64 bits from whole numbers e, by the exponent's bits: exp2 and ldexp may be off by a last place."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _mx_quantise(v):
    """Microscaled 4-bit floating point of an fp32 [rows, cols] matrix: codes 0..15 [rows, cols] and scale bytes
    [rows, cols / 32].  Half steps go to the even code, which by the codes' order is the even number."""
    rows, cols = v.shape
    b = v.view(rows, cols // 32, 32)
    amax = b.abs().amax(dim=2)
    bad = ~torch.isfinite(amax)
    safe = torch.where(bad | (amax == 0), torch.full_like(amax, 4.0), amax)
    e = (torch.frexp(safe)[1] - 3).clamp(min=-127)  # frexp: safe = f 2^e', 1/2 <= f < 1
    r = b.abs().double() * _pow2(-e).unsqueeze(2)
    code = torch.zeros(r.shape, dtype=torch.uint8, device=v.device)
    for c, (lo, closed) in enumerate([(0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)]):
        code += ((r >= lo) if closed else (r > lo)).to(torch.uint8)
    code += 8 * torch.signbit(b).to(torch.uint8)
    byte = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return code.view(rows, cols), byte


def _mx_pack(code):
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous()


_MX_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx_values(codes, scales, dtype):
    """The values that packed codes and scale bytes stand for."""
    rows = codes.shape[0]
    nib = torch.stack((codes & 15, codes >> 4), dim=2).view(rows, -1)
    table = torch.tensor(_MX_VALUES + tuple(-x for x in _MX_VALUES), dtype=dtype, device=codes.device)
    v = table[nib.long()].view(rows, -1, 32)
    return (v * _pow2(scales.int() - 127).to(dtype).unsqueeze(2)).view(rows, -1)


def _draft_inputs(c, gen):
    """Target and draft distributions that resemble each other, tokens drawn from the draft's, ragged lengths."""
    B, n, V, k = c["B"], c["n"], c["V"], c["k"]
    dev = "cuda"
    s = {}
    target = torch.empty((B, n + 1, V), device=dev) if c["target"] == "dense" else None
    draft = torch.empty((B, n, V), device=dev) if c["draft"] == "dense" else None
    if c["target"] == "list":
        s["target_idx"] = torch.empty((B, n + 1, k), dtype=torch.int32, device=dev)
        target = torch.empty((B, n + 1, k), device=dev)
    if c["draft"] == "list":
        s["draft_idx"] = torch.empty((B, n, k), dtype=torch.int32, device=dev)
        draft = torch.empty((B, n, k), device=dev)
    tokens = torch.zeros((B, n), dtype=torch.int32, device=dev)
    pick = gen.uniform((B, n))
    for b in range(B):
        z = gen.f32((n + 1, V), 2.5)
        zq = z[:n] + gen.f32((n, V), 0.4)
        if c["target"] == "dense":
            target[b] = torch.softmax(z, dim=1)
        else:
            top = torch.topk(z, k, dim=1)
            s["target_idx"][b], target[b] = top.indices.to(torch.int32), torch.softmax(top.values, dim=1)
        if c["draft"] == "dense":
            q = torch.softmax(zq, dim=1)
            draft[b] = q
            at = (q.double().cumsum(dim=1) > pick[b].double().unsqueeze(1)).to(torch.uint8).argmax(dim=1)
            tokens[b] = at.to(torch.int32)
        elif c["draft"] == "list":
            top = torch.topk(zq, k, dim=1)
            q = torch.softmax(top.values, dim=1)
            s["draft_idx"][b], draft[b] = top.indices.to(torch.int32), q
            at = (q.double().cumsum(dim=1) > pick[b].double().unsqueeze(1)).to(torch.uint8).argmax(dim=1)
            tokens[b] = top.indices.gather(1, at.unsqueeze(1)).squeeze(1).to(torch.int32)
        else:
            tokens[b] = zq.argmax(dim=1).to(torch.int32)
    lengths = n - (gen.uniform((B,)) * 1.3).to(torch.int32).mul_((gen.uniform((B,)) * (n + 1)).to(torch.int32))
    s.update(target=target, draft=draft, tokens=tokens, lengths=lengths.clamp_(0, n).to(torch.int32),
             accept_u=gen.uniform((B, n)), sample_u=gen.uniform((B,)))
    return s


def prepare(case, seed):
    c, gen = case, _Gen(seed)
    s = dict(case=c)
    if c["op"] == "gated":
        T, d, ff = c["T"], c["d"], c["ff"]
        s.update(x=gen.bf16((T, d)), wg=gen.bf16((ff, d), d ** -0.5), wu=gen.bf16((ff, d), d ** -0.5),
                 w2=gen.bf16((ff, d), ff ** -0.5))
        if c["train"]:
            s["dy"] = gen.bf16((T, d), d ** -0.5)
    elif c["op"] == "mx":
        T, rows, cols = c["T"], c["rows"], c["cols"]
        s["x"] = gen.bf16((T, cols))
        codes, scales = [], []
        for r in range(0, rows, 8192):  # a matrix of 256000 rows in parts: the 64-bit quotients would take 4 GB
            code, byte = _mx_quantise(gen.bf16((min(8192, rows - r), cols), cols ** -0.5).float())
            codes.append(_mx_pack(code))
            scales.append(byte)
        s["w_codes"], s["w_scales"] = torch.cat(codes), torch.cat(scales)
    elif c["op"] == "pack":
        w = gen.f32((c["rows"], c["cols"]), c["cols"] ** -0.5)
        s["w"] = (w * torch.exp(gen.f32((c["rows"], 1)))).to(torch.bfloat16)
    else:
        s.update(_draft_inputs(c, gen))
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """What a program of the framework keeps besides: descriptors, output buffers, workspaces."""
    from paper_2402_09360_amd import hire
    c = s["case"]
    if c["op"] == "gated":
        s["layer"] = hire.GatedLayer(s["wg"], s["wu"], s["w2"], act=c["act"])
        s["out"] = hire.GatedOutputs(s["layer"], c["T"], train=c["train"])
        nbytes = hire.hire_gated_ffn_workspace_bytes(s["layer"], c["T"])
        if c["train"]:
            s["grads"] = hire.GatedGradients(s["layer"], c["T"])
            nbytes = max(nbytes, hire.hire_gated_ffn_backward_workspace_bytes(s["layer"], c["T"]))
        s["ws"] = hire.alloc_workspace(max(nbytes, 256))
    elif c["op"] == "mx":
        s["wq"] = hire.Mxfp4(s["w_codes"], s["w_scales"])
        if c["form"] == "mx":
            s["xq"] = hire.Mxfp4.empty(c["T"], c["cols"])
        s["y"] = torch.empty((c["T"], c["rows"]), dtype=torch.float32 if c["y"] == "f32" else torch.bfloat16,
                             device="cuda")
        nbytes = hire.hire_mxfp4_product_workspace_bytes(c["T"], c["rows"], c["cols"])
        s["ws"] = hire.alloc_workspace(max(nbytes, 256))
    elif c["op"] == "pack":
        s["wq"] = hire.Mxfp4.empty(c["rows"], c["cols"])
        s["back"] = torch.empty((c["rows"], c["cols"]), dtype=torch.bfloat16, device="cuda")
    else:
        s["drafts"] = hire.Drafts(s["tokens"], c["V"], s["target"], s["accept_u"], s["sample_u"],
                                  target_idx=s.get("target_idx"), draft_prob=s["draft"],
                                  draft_idx=s.get("draft_idx"), lengths=s["lengths"])
        s["out"] = hire.DraftOutputs(s["drafts"])
        s["ws"] = hire.alloc_workspace(max(hire.hire_verify_draft_workspace_bytes(s["drafts"]), 256))


# ---- a pass ----------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2402_09360_amd import hire
    c = s["case"]
    if c["op"] == "gated":
        hire.hire_gated_ffn_step(s["layer"], s["x"], s["out"], s["ws"])
        if not c["train"]:
            return dict(y=s["out"].y)
        g = s["grads"]
        hire.hire_gated_ffn_backward(s["layer"], s["x"], s["out"], s["dy"], g, s["ws"])
        return dict(y=s["out"].y, dx=g.dx, dwg=g.dwg, dwu=g.dwu, dw2u=g.dw2u)
    if c["op"] == "mx":
        if c["form"] == "mx":
            hire.hire_pack_mxfp4(s["x"], out=s["xq"])
            hire.hire_mxfp4_product(s["xq"], s["wq"], s["y"], s["ws"])
        else:
            hire.hire_mxfp4_product_bf16(s["x"], s["wq"], s["y"], s["ws"])
        return dict(y=s["y"])
    if c["op"] == "pack":
        hire.hire_pack_mxfp4(s["w"], out=s["wq"])
        hire.hire_unpack_mxfp4(s["wq"], out=s["back"])
        return dict(w=s["back"])
    hire.hire_verify_draft(s["drafts"], s["out"], s["ws"])
    return dict(tokens=s["out"].tokens, accepted=s["out"].accepted)


def _activation(g, kind):
    """The activation and its derivative."""
    if kind == "relu":
        return torch.clamp(g, min=0), (g > 0).to(g.dtype)
    z = g if kind == "silu" else _C_GELU * (g + _A_GELU * g * g * g)
    dz = torch.ones_like(g) if kind == "silu" else _C_GELU * (1.0 + 3.0 * _A_GELU * g * g)
    sig = torch.sigmoid(z)
    return g * sig, sig + g * sig * (1.0 - sig) * dz


def _run_plain(s):
    c = s["case"]
    if c["op"] == "gated":
        x, wg, wu, w2 = (s[k].float() for k in ("x", "wg", "wu", "w2"))
        g, u = x @ wg.t(), x @ wu.t()
        a, da = _activation(g, c["act"])
        h = a * u
        out = dict(y=(h @ w2).to(torch.bfloat16))
        if c["train"]:
            dy = s["dy"].float()
            dh = dy @ w2.t()
            dg, du = dh * u * da, dh * a
            out["dx"] = (dg @ wg + du @ wu).to(torch.bfloat16)
            out["dwg"] = (dg.t() @ x).to(torch.bfloat16)
            out["dwu"] = (du.t() @ x).to(torch.bfloat16)
            out["dw2u"] = (h.t() @ dy).to(torch.bfloat16)
        return out
    if c["op"] == "mx":
        x = s["x"].float()
        if c["form"] == "mx":
            code, byte = _mx_quantise(x)
            x = _mx_values(_mx_pack(code), byte, torch.float32)
        y = x @ _mx_values(s["w_codes"], s["w_scales"], torch.float32).t()
        return dict(y=y if c["y"] == "f32" else y.to(torch.bfloat16))
    if c["op"] == "pack":
        code, byte = _mx_quantise(s["w"].float())
        return dict(w=_mx_values(_mx_pack(code), byte, torch.float32).to(torch.bfloat16))
    return _verify_plain(s, c)


def _at_tokens(prob, idx, tokens):
    """prob [B, n, V] (or lists with idx [B, n, k]) at tokens [B, n], in 64 bits; 1 for a missing prob."""
    if prob is None:
        return torch.ones(tokens.shape, dtype=torch.float64, device=tokens.device)
    if idx is None:
        return prob.gather(2, tokens.long().unsqueeze(2)).squeeze(2).double()
    return torch.where(idx == tokens.unsqueeze(2), prob.double(), torch.zeros((), dtype=torch.float64, device="cuda")).sum(2)


def _verify_plain(s, c):
    B, n, V = c["B"], c["n"], c["V"]
    tokens, lengths = s["tokens"], s["lengths"]
    rows = torch.arange(B, device="cuda")
    p_at = _at_tokens(s["target"][:, :n], None if s.get("target_idx") is None else s["target_idx"][:, :n], tokens)
    q_at = _at_tokens(s["draft"], s.get("draft_idx"), tokens)
    ok = (s["accept_u"].double() * q_at < p_at) & (torch.arange(n, device="cuda") < lengths.unsqueeze(1))
    accepted = ok.to(torch.int32).cumprod(dim=1).sum(dim=1)
    # the distribution behind the accepted tokens: the target's, less the draft's where a token was refused
    p = s["target"][rows, accepted].double()
    at = torch.clamp(accepted, max=n - 1)
    refused = accepted < lengths
    if s["draft"] is None:
        q = torch.zeros((B, V), dtype=torch.float64, device="cuda")
        q[rows, tokens[rows, at].long()] = 1.0
    elif s.get("draft_idx") is None:
        q = s["draft"][rows, at].double()
    else:
        q = torch.zeros((B, V), dtype=torch.float64, device="cuda")
        q.scatter_(1, s["draft_idx"][rows, at].long(), s["draft"][rows, at].double())
    if s.get("target_idx") is not None:
        q = q.gather(1, s["target_idx"][rows, accepted].long())
    rest = torch.where(refused.unsqueeze(1), torch.clamp(p - q, min=0.0), p)
    rest = torch.where((rest.sum(dim=1, keepdim=True) > 0), rest, p)
    cum = rest.cumsum(dim=1)
    pos = (cum > s["sample_u"].double().unsqueeze(1) * cum[:, -1:]).to(torch.uint8).argmax(dim=1)
    nxt = pos if s.get("target_idx") is None else s["target_idx"][rows, accepted, pos]
    place = torch.arange(n + 1, device="cuda").unsqueeze(0)
    out = torch.where(place < accepted.unsqueeze(1), torch.nn.functional.pad(tokens, (0, 1)), -1)
    out = torch.where(place == accepted.unsqueeze(1), nxt.to(torch.int32).unsqueeze(1), out)
    return dict(tokens=out.to(torch.int32), accepted=accepted.to(torch.int32))


# ---- what is moved and computed --------------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "gated":
        T, d, ff = c["T"], c["d"], c["ff"]
        nbytes, flops = 6 * d * ff + 4 * T * d, 6 * T * d * ff
        if c["train"]:  # x, dy and the weights read, y, dx and the gradients written
            nbytes, flops = nbytes + 6 * d * ff + 4 * T * d, 3 * flops
        return dict(bytes=nbytes, flops=flops)
    if c["op"] == "mx":
        T, rows, cols = c["T"], c["rows"], c["cols"]
        return dict(bytes=rows * cols * 17 // 32 + 2 * T * cols + T * rows * (4 if c["y"] == "f32" else 2),
                    flops=2 * T * rows * cols)
    if c["op"] == "pack":
        return dict(bytes=c["rows"] * c["cols"] * (2 * 2 + 17 / 16), flops=2 * c["rows"] * c["cols"])
    B, n = c["B"], c["n"]
    row = (4 * c["V"] if c["target"] == "dense" else 8 * c["k"])
    row += {"dense": 4 * (c["V"] if c["target"] == "dense" else c["k"]), "list": 8 * c["k"], "certain": 0}[c["draft"]]
    lists = (4 * c["k"] * n if c["target"] == "list" else 0) + (4 * c["k"] * n if c["draft"] == "list" else 0)
    return dict(bytes=B * (row + lists + 16 * n + 4 * (n + 3)), flops=3 * B * row // 4)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    c = case
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if c["op"] == "gated":
        return _gated_exact(s, c)
    if c["op"] == "mx":
        x = s["x"].double()
        if c["form"] == "mx":
            x = _mx_nearest(x)
        y = torch.empty((c["T"], c["rows"]), dtype=torch.float64, device="cuda")
        table = torch.tensor([(-1) ** (i >> 3) * _MX_VALUES[i & 7] for i in range(16)], dtype=torch.float64, device="cuda")
        for r in range(0, c["rows"], 16384):
            codes = s["w_codes"][r:r + 16384].int()
            w = torch.empty((codes.shape[0], c["cols"]), dtype=torch.float64, device="cuda")
            w[:, 0::2], w[:, 1::2] = table[codes % 16], table[codes // 16]
            w *= (s["w_scales"][r:r + 16384].long() + 896 << 52).view(torch.float64).repeat_interleave(32, dim=1)
            y[:, r:r + 16384] = x @ w.t()
        return dict(y=y)
    if c["op"] == "pack":
        return dict(w=_mx_nearest(s["w"].double()))
    return _verify_exact(s, c)


def _gated_exact(s, c):
    x, wg, wu, w2 = (s[k].double() for k in ("x", "wg", "wu", "w2"))
    g, u = x @ wg.t(), x @ wu.t()
    if c["act"] == "relu":
        a, da = torch.relu(g), (g > 0).double()
    elif c["act"] == "silu":
        e = torch.exp(-g)
        a, da = g / (1 + e), (1 + e + g * e) / (1 + e) ** 2
    else:
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (g + _A_GELU * g ** 3))
        a = 0.5 * g * (1 + t)
        da = 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * _A_GELU * g * g)
    h = a * u
    out = dict(y=h @ w2)
    if c["train"]:
        dy = s["dy"].double()
        dh = dy @ w2.t()
        out["dw2u"] = h.t() @ dy
        dg, du = dh * u * da, dh * a
        out["dwg"], out["dwu"] = dg.t() @ x, du.t() @ x
        out["dx"] = dg @ wg + du @ wu
        out = {k: out[k] for k in ("y", "dx", "dwg", "dwu", "dw2u")}
    return out


def _mx_nearest(v):
    """Every value of a 64-bit matrix rounded to the nearest of its block's grid, half steps to the even multiple."""
    b = v.view(v.shape[0], -1, 32)
    amax = b.abs().amax(dim=2, keepdim=True)
    power = (torch.where(amax == 0, torch.ones_like(amax), amax).view(torch.int64) >> 52 << 52).view(torch.float64)
    scale = torch.clamp(power / 4.0, min=2.0 ** -127)  # the exponent's bits alone are the power of two below amax
    r = torch.clamp(b.abs() / scale, max=6.0)
    step = torch.where(r < 2.0, 0.5, torch.where(r < 4.0, 1.0, 2.0)).double()
    return torch.copysign(torch.round(r / step) * step * scale, b).view(v.shape)


def _verify_exact(s, c):
    """One sequence after the other, one drafted token after the other, on the host."""
    B, n, V = c["B"], c["n"], c["V"]
    tokens, lengths = s["tokens"].cpu(), s["lengths"].cpu()
    accept_u, sample_u = s["accept_u"].cpu().double(), s["sample_u"].cpu().double()

    def row(prob, idx, b, i):
        full = torch.zeros(V, dtype=torch.float64)
        if idx is None:
            return full.copy_(prob[b, i].cpu())
        full[idx[b, i].cpu().long()] = prob[b, i].cpu().double()
        return full

    def draft_row(b, i):
        if s["draft"] is not None:
            return row(s["draft"], s.get("draft_idx"), b, i)
        full = torch.zeros(V, dtype=torch.float64)
        full[int(tokens[b, i])] = 1.0
        return full

    out = torch.full((B, n + 1), -1, dtype=torch.int32)
    accepted = torch.zeros(B, dtype=torch.int32)
    for b in range(B):
        i = 0
        while True:
            p = row(s["target"], s.get("target_idx"), b, i)
            if i == int(lengths[b]):
                rest = p
                break
            q, t = draft_row(b, i), int(tokens[b, i])
            if float(accept_u[b, i]) * float(q[t]) < float(p[t]):
                out[b, i] = t
                i += 1
                continue
            rest = (p - q).clamp_(min=0.0)
            if float(rest.sum()) == 0.0:
                rest = p
            break
        order = torch.arange(V) if s.get("target_idx") is None else s["target_idx"][b, i].cpu().long()
        cum = rest[order].cumsum(0)
        out[b, i] = int(order[int((cum > sample_u[b] * cum[-1]).nonzero()[0])])
        accepted[b] = i
    return dict(tokens=out.cuda(), accepted=accepted.cuda())
