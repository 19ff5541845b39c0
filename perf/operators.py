"""The operators around the layer, as measured cases: the gated linear recurrence, the norms of queries and keys with
the position rotation, and the short causal convolution that feeds both.

``run`` computes an operator in its plain form (elementary torch operations in 32 bits or more, rounded once at the end)
or, where ``own`` is true, by the library's calls.  A case:

  op      scan_step | scan_fwd | scan_train | norm_fwd | norm_train | conv_step | conv_fwd | conv_train
  B, T    sequences and tokens of each; with ``nseq``, T packed tokens in that many sequences (B = 1)
  io      dtype of the token tensors
  C       channels (scan, conv);  W: taps;  Hq, Hk, D: heads of queries and keys and their size (norm)
  carry   the sequences continue others: states come in, and gradients for the states that went out

Shapes are those of the benchmark configurations (8 heads of 128 and rows of 2048 tokens, 16 heads and rows of
4096, packed rows of 131072 tokens) and of the decode and fp32 cases; ``draw`` gives others of the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6


def _scan(op, B, T, C, io, complement, carry, **more):
    return dict(op="scan_" + op, B=B, T=T, C=C, io=io, complement=complement, carry=carry, **more)


def _norm(op, B, T, Hq, Hk, D, io, norm, weights, rot, **more):
    return dict(op="norm_" + op, B=B, T=T, Hq=Hq, Hk=Hk, D=D, io=io, norm=norm, weights=weights, rot=rot, **more)


def _conv(op, B, T, C, W, io, silu, bias, carry, **more):
    return dict(op="conv_" + op, B=B, T=T, C=C, W=W, io=io, silu=silu, bias=bias, carry=carry, **more)


def listed():
    return [
        # one user's generation, one token: the latency of a single call
        dict(name="scan_step_1", **_scan("step", 1, 1, 1024, "bf16", True, True)),
        # the prompt of one request, whose last state goes to the decode cache
        dict(name="scan_fwd_1x2048", **_scan("fwd", 1, 2048, 1024, "bf16", True, False)),
        # the 340M model's training batch
        dict(name="scan_train_8x2048", **_scan("train", 8, 2048, 1024, "bf16", True, False)),
        # packed training rows: eight documents, none a multiple of a tile but the longest
        dict(name="scan_train_packed_131k", **_scan("train", 1, 131072, 1024, "bf16", False, True, nseq=8, seed=4)),
        # fp32 training of a small model on ragged lengths (gradient checks)
        dict(name="scan_train_fp32", **_scan("train", 3, 1001, 384, "fp32", False, True)),
        # a serving batch of one token each, far positions, rotated grouped-query heads
        dict(name="norm_fwd_64_tokens", **_norm("fwd", 64, 1, 16, 4, 128, "bf16", "rms", True, "half")),
        # the unit queries and keys of the 340M layer, read out of the convolution's output rows
        dict(name="norm_train_8x2048", **_norm("train", 8, 2048, 8, 8, 128, "bf16", "l2", False, "none", fused=True)),
        # the 1.3B heads with learned weights and rotation
        dict(name="norm_train_rot_4x4096", **_norm("train", 4, 4096, 16, 16, 128, "bf16", "rms", True, "half")),
        # a serving batch of one token each
        dict(name="conv_step_512", **_conv("step", 512, 1, 2048, 4, "bf16", True, False, True)),
        # the 340M layer's queries and keys, training
        dict(name="conv_train_8x2048", **_conv("train", 8, 2048, 2048, 4, "bf16", True, False, False)),
        # packed training rows
        dict(name="conv_train_packed_131k", **_conv("train", 1, 131072, 1024, 4, "bf16", True, True, True, nseq=8, seed=4)),
        # fp32, three taps without activation, ragged length
        dict(name="conv_train_fp32", **_conv("train", 3, 1001, 384, 3, "fp32", False, True, True)),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], even over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["scan_step", "scan_fwd", "scan_train", "scan_train", "norm_fwd", "norm_train", "norm_train",
                     "conv_step", "conv_fwd", "conv_train", "conv_train"])
    kind, what = op.split("_")
    io = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    most = 1 << 26                  # elements of a drawn case
    if what == "step":              # one token each, or a few (speculative steps)
        B, T = _log_int(rng, 1, 512), rng.choice([1, 1, 1, 2, 5, 16])
        if kind == "scan":
            return _scan("step", B, T, 64 * _log_int(rng, 1, 64), io, rng.random() < 0.5, True)
        return _conv("step", B, T, 64 * _log_int(rng, 1, 64), rng.choice([4, 4, 3, 2]), io, rng.random() < 0.7,
                     rng.random() < 0.5, True)
    more = {}
    T = _log_int(rng, 1, 65536)
    if T > 64 and rng.random() < 0.4:
        more = dict(nseq=rng.randint(1, 24), seed=rng.randrange(1 << 20))
    if kind == "norm":
        D = rng.choice([128, 128, 64, 64, 96, 256, 80])
        Hq = rng.choice([1, 2, 4, 8, 16, 12])
        Hk = rng.choice([h for h in (1, 2, 4, 8, 16, 12) if Hq % h == 0])
        width = (Hq + Hk) * D
    else:
        # channels of whole heads, of a slice, or any
        C = rng.choice([64 * _log_int(rng, 1, 64), 64 * _log_int(rng, 1, 64), 8 * _log_int(rng, 1, 256), rng.randint(1, 700)])
        width = C
    T = max(1, min(T, most // width))
    B = 1 if more else _log_int(rng, 1, max(1, min(64, most // (T * width))))
    if kind == "scan":
        return _scan(what, B, T, C, io, rng.random() < 0.5, rng.random() < 0.5, **more)
    if kind == "conv":
        return _conv(what, B, T, C, rng.choice([4, 4, 3, 2]), io, rng.random() < 0.7, rng.random() < 0.5,
                     rng.random() < 0.5, **more)
    return _norm(what, B, T, Hq, Hk, D, io, rng.choice(["l2", "rms"]), rng.random() < 0.6,
                 rng.choice(["none", "half", "half", "pairs"]), fused=rng.random() < 0.3, **more)


# ---- inputs --------------------------------------------------------------------------------------------------

def _lengths(case):
    if not case.get("nseq"):
        return [case["T"]] * case["B"]
    rnd = torch.Generator().manual_seed(case["seed"])
    w = torch.exp(4.0 * torch.rand(case["nseq"], generator=rnd, dtype=torch.float64))
    ends = torch.round(torch.cumsum(w, 0) / w.sum() * case["T"]).long().tolist()
    ends[-1] = case["T"]
    return [b - a for a, b in zip([0] + ends[:-1], ends)]      # a short one may be empty


def prepare(case, seed):
    """Inputs, output buffers and what a program keeps between calls, on the GPU."""
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    io = torch.bfloat16 if case["io"] == "bf16" else torch.float32
    kind, what = case["op"].split("_")
    lens = _lengths(case)
    S, N = len(lens), case["B"] * case["T"]

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device=dev)

    def empty(*shape, dtype=io):
        return torch.empty(*shape, device=dev, dtype=dtype)

    s = dict(case=case, lens=lens, cu=None)
    if case.get("nseq"):
        s["cu"] = torch.tensor([0] + lens, dtype=torch.int32).cumsum(0, dtype=torch.int32).to(dev)
    if kind == "scan":
        C = case["C"]
        s["x"] = randn(N, C).to(io)
        # each channel has a memory of its own, from a token to a few thousand; the token moves it
        rate = torch.exp(math.log(3e-4) + (math.log(0.7) - math.log(3e-4)) * rand(C))
        s["gate"] = -rate * 2.0 * torch.sigmoid(randn(N, C))
        s["out"] = empty(N, C)
        if what == "step":
            s["state"] = randn(S, C)
            return s
        s["init_state"] = randn(S, C) if case["carry"] else None
        s["final_state"] = empty(S, C, dtype=torch.float32)
        if what == "train":
            s["dout"] = randn(N, C).to(io)
            s["dfinal_state"] = randn(S, C) if case["carry"] else None
            s["dx"], s["dgate"] = empty(N, C), empty(N, C, dtype=torch.float32)
            s["dinit_state"] = empty(S, C, dtype=torch.float32)
        return s
    if kind == "conv":
        C, W = case["C"], case["W"]
        s["x"] = randn(N, C).to(io)
        s["weight"] = randn(C, W) / math.sqrt(W)
        s["bias"] = 0.1 * randn(C) if case["bias"] else None
        s["out"] = empty(N, C)
        if what == "step":
            s["state"] = randn(S, W - 1, C).to(io)
            return s
        s["init_state"] = randn(S, W - 1, C).to(io) if case["carry"] else None
        s["final_state"] = empty(S, W - 1, C)
        if what == "train":
            s["dout"] = randn(N, C).to(io)
            s["dfinal_state"] = randn(S, W - 1, C).to(io) if case["carry"] else None
            s["dx"], s["dweight"] = empty(N, C), empty(C, W, dtype=torch.float32)
            s["dbias"] = empty(C, dtype=torch.float32) if case["bias"] else None
            s["dinit_state"] = empty(S, W - 1, C)
        return s
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if case.get("fused"):           # one row of queries, keys and as many values a token
        rows = randn(N, (Hq + 2 * Hk) * D).to(io)
        s["q"] = rows[:, :Hq * D].view(N, Hq, D)
        s["k"] = rows[:, Hq * D:(Hq + Hk) * D].view(N, Hk, D)
    else:
        s["q"], s["k"] = randn(N, Hq, D).to(io), randn(N, Hk, D).to(io)
    s["q_weight"] = 1.0 + 0.2 * randn(D) if case["weights"] else None
    s["k_weight"] = 1.0 + 0.2 * randn(D) if case["weights"] else None
    s["inv_freq"] = s["positions"] = None
    if case["rot"] != "none":
        R = D // 16 * 16
        s["inv_freq"] = 10000.0 ** (-torch.arange(0, R, 2, device=dev, dtype=torch.float64) / R)
        first = torch.randint(0, 131072 - 4096, (S,), generator=gen, device=dev)   # continued rows, far caches
        s["positions"] = torch.cat([torch.arange(n, device=dev) + f for n, f in zip(lens, first)]).to(torch.int32)
    s["q_out"], s["k_out"] = empty(N, Hq, D), empty(N, Hk, D)
    if what == "train":
        s["dq_out"], s["dk_out"] = randn(N, Hq, D).to(io), randn(N, Hk, D).to(io)
        s["dq"], s["dk"] = empty(N, Hq, D), empty(N, Hk, D)
        s["dq_weight"] = empty(D, dtype=torch.float32) if case["weights"] else None
        s["dk_weight"] = empty(D, dtype=torch.float32) if case["weights"] else None
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------

def _places(s):
    """Of each token: its sequence, its place there, and the tokens left behind it."""
    dev = s["x"].device
    lens = torch.tensor(s["lens"], device=dev)
    ends = torch.cumsum(lens, 0)
    t = torch.arange(int(s["x"].shape[0]), device=dev)
    seq = torch.searchsorted(ends, t, right=True)
    pos = t - (ends - lens)[seq]
    return seq, pos, lens[seq] - 1 - pos


def _affine_scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis, by doubling."""
    d = 1
    while d < a.shape[0]:
        b = torch.cat([b[:d], torch.addcmul(b[d:], a[d:], b[:-d])])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _rows(state, seq, where):
    """state[seq] where it holds, else zeros."""
    return torch.where(where[:, None], state[seq], 0.0) if state is not None else 0.0


def _scan_plain(s, train):
    # in 64 bits: a gate next to one has lost its distance from it in 32, and thousands of them are multiplied
    case = s["case"]
    N, C = s["x"].shape
    S = len(s["lens"])
    x, g, init = s["x"].double(), s["gate"].double(), s["init_state"]
    seq, pos, left = _places(s)
    first, last = pos == 0, left == 0
    a = torch.exp(g)
    keep = -torch.expm1(g) if case["complement"] else None
    b = x * keep if case["complement"] else x
    inside = torch.where(first[:, None], 0.0, a)
    h = _affine_scan(inside, b + a * _rows(init, seq, first))
    ends = torch.cumsum(torch.tensor(s["lens"], device=x.device), 0) - 1
    empty = (torch.tensor(s["lens"], device=x.device) == 0)[:, None]
    none = torch.zeros(S, C, device=x.device)
    final = torch.where(empty, none if init is None else init, h[ends.clamp_min(0)]).float()
    if not train:
        return [h.to(s["x"].dtype), final]
    before = torch.where(first[:, None], 0.0, torch.cat([h[:1], h[:-1]])) + _rows(init, seq, first)
    df = s["dfinal_state"]
    later = torch.where(last[:, None], 0.0, torch.cat([a[1:], a[:1]]))     # a_{t+1}, none behind a sequence's end
    dh = _affine_scan(later.flip(0), (s["dout"].double() + _rows(df, seq, last)).flip(0)).flip(0)
    dg = a * (before - x if case["complement"] else before) * dh
    dx = dh * keep if case["complement"] else dh
    starts = ends + 1 - torch.tensor(s["lens"], device=x.device)
    dinit = torch.where(empty, none if df is None else df, (a * dh)[starts.clamp_max(N - 1)]).float()
    io = s["x"].dtype
    return [h.to(io), final, dx.to(io), dg.float(), dinit]


def _scan_step_plain(s):
    case = s["case"]
    B, T, C = case["B"], case["T"], case["C"]
    x, g = s["x"].float().view(B, T, C), s["gate"].view(B, T, C)
    a = torch.exp(g)
    b = -torch.expm1(g) * x if case["complement"] else x
    h = s["state"]
    out = []
    for t in range(T):
        h = a[:, t] * h + b[:, t]
        out.append(h)
    s["state"].copy_(h)
    return [torch.stack(out, 1).view(B * T, C).to(s["x"].dtype), s["state"]]


def _conv_plain(s, train, init):
    case, io = s["case"], s["x"].dtype
    W = case["W"]
    seq, pos, left = _places(s)
    N, C = s["x"].shape
    S = len(s["lens"])
    x, w = s["x"].float(), s["weight"]
    init = torch.zeros(S, W - 1, C, device=x.device) if init is None else init.float()
    ext = torch.cat([init.reshape(S * (W - 1), C), x])      # the rows in front of each sequence, then the tokens
    t = torch.arange(N, device=x.device)

    def taken(j):                                           # row of the token j before each
        return torch.where(pos >= j, S * (W - 1) + t - j, seq * (W - 1) + W - 1 + pos - j)

    z = torch.zeros_like(x) if s["bias"] is None else s["bias"].expand_as(x)
    for j in range(W):
        z = z + w[:, W - 1 - j] * ext[taken(j)]
    sig = torch.sigmoid(z)
    y = z * sig if case["silu"] else z
    lens = torch.tensor(s["lens"], device=x.device)
    ends = torch.cumsum(lens, 0)
    back = torch.arange(W - 1, 0, -1, device=x.device)      # the cache: the last W - 1 rows, oldest first
    at = torch.where(lens[:, None] >= back, S * (W - 1) + ends[:, None] - back,
                     torch.arange(S, device=x.device)[:, None] * (W - 1) + (W - 1) + lens[:, None] - back)
    final = ext[at.reshape(-1)].view(S, W - 1, C).to(io)
    if not train:
        return [y.to(io), final]
    dz = s["dout"].float()
    if case["silu"]:
        dz = dz * sig * (1.0 + z * (1.0 - sig))
    df = torch.zeros(S, W - 1, C, device=x.device) if s["dfinal_state"] is None else s["dfinal_state"].float()
    dext = torch.zeros_like(ext)
    dw = []
    for j in range(W):
        rows = taken(j)
        dext[S * (W - 1):] += torch.where((left >= j)[:, None], w[:, W - 1 - j] * dz[(t + j).clamp_max(N - 1)], 0.0)
        early = (pos < j).nonzero()[:, 0]                   # taps that reach the rows in front: one token a row and tap
        dext[rows[early]] += w[:, W - 1 - j] * dz[early]
        dw.append((dz * ext[rows]).sum(0, dtype=torch.float64).float())
    for i in range(W - 1):
        dext[at[:, i]] += df[:, i]
    dinit = dext[:S * (W - 1)].view(S, W - 1, C).to(io)
    got = [y.to(io), final, dext[S * (W - 1):].to(io), torch.stack(dw[::-1], 1), dinit]
    return got if s["bias"] is None else got + [dz.sum(0, dtype=torch.float64).float()]


def _conv_step_plain(s):
    y, final = _conv_plain(s, False, s["state"])
    s["state"].copy_(final)
    return [y, s["state"]]


def _turn(x, cos, sin, layout):
    """Rotates pairs of the first 2 n features of x by the angles of [T, 1, n]."""
    n = cos.shape[-1]
    if layout == "half":
        p, q = x[..., :n], x[..., n:2 * n]
        return torch.cat([p * cos - q * sin, p * sin + q * cos, x[..., 2 * n:]], -1)
    p, q = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    return torch.cat([torch.stack([p * cos - q * sin, p * sin + q * cos], -1).flatten(-2), x[..., 2 * n:]], -1)


def _norm_plain(s, train):
    case = s["case"]
    D, io = case["D"], s["q"].dtype
    if case["rot"] != "none":
        angle = (s["positions"].double()[:, None] * s["inv_freq"])[:, None]
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    outs, grads, dws = [], [], []
    for n in ("q", "k"):
        x, w = s[n].float(), s[n + "_weight"]
        share = 1.0 / D if case["norm"] == "rms" else 1.0
        r = torch.rsqrt(x.square().sum(-1, keepdim=True) * share + EPS)
        u = x * r
        y = u if w is None else u * w
        if case["rot"] != "none":
            y = _turn(y, cos, sin, case["rot"])
        outs.append(y.to(io))
        if train:
            dy = s["d" + n + "_out"].float()
            if case["rot"] != "none":
                dy = _turn(dy, cos, -sin, case["rot"])
            if w is not None:
                dws.append((dy * u).sum((0, 1), dtype=torch.float64).float())
                dy = dy * w
            grads.append((r * (dy - u * (dy * u).sum(-1, keepdim=True) * share)).to(io))
    return outs + grads + dws


def _plain(s):
    kind, what = s["case"]["op"].split("_")
    if kind == "scan":
        return _scan_step_plain(s) if what == "step" else _scan_plain(s, what == "train")
    if kind == "conv":
        return _conv_step_plain(s) if what == "step" else _conv_plain(s, what == "train", s["init_state"])
    return _norm_plain(s, what == "train")


# ---- the library's calls -------------------------------------------------------------------------------------

def _keep(s):
    """Parameters and workspace, made on the first pass and kept."""
    import paper_2605_13473_b200 as osdn
    case = s["case"]
    kind, what = case["op"].split("_")
    shape = dict(B=case["B"], T=case["T"], io_dtype=case["io"], cu_seqlens=s["cu"])
    if kind == "scan":
        shape |= dict(C=case["C"], input_gate="complement" if case["complement"] else "plain")
        s["p"] = osdn.make_scan_params(**shape, flags=osdn.FLAG_SAVE_RESIDUALS if what == "train" else 0)
        s["p_bwd"] = osdn.make_scan_params(**shape, flags=osdn.FLAG_RESIDUALS_VALID)
        nbytes = osdn.osdn_scan_workspace_bytes(s["p"])
    elif kind == "conv":
        s["p"] = osdn.make_conv_params(**shape, C=case["C"], W=case["W"], activation="silu" if case["silu"] else "none")
        nbytes = osdn.osdn_short_conv_workspace_bytes(s["p"])
    else:
        s["p"] = osdn.make_qk_norm_params(**shape, Hq=case["Hq"], Hk=case["Hk"], D=case["D"], norm=case["norm"], eps=EPS,
                                          rot_dim=0 if s["inv_freq"] is None else 2 * s["inv_freq"].numel(),
                                          rot_layout="pairs" if case["rot"] == "pairs" else "half",
                                          q_row=s["q"].stride(0), k_row=s["k"].stride(0))
        nbytes = osdn.osdn_qk_norm_workspace_bytes(s["p"])
    s["workspace"] = torch.empty(nbytes, device="cuda:0", dtype=torch.uint8) if what == "train" else None
    s["lib"] = osdn
    return osdn


def _own(s):
    osdn = s.get("lib") or _keep(s)
    op, p = s["case"]["op"], s["p"]
    if op == "scan_step":
        osdn.osdn_scan_step(p, s["x"], s["gate"], s["state"], s["out"])
        return [s["out"], s["state"]]
    if op == "conv_step":
        osdn.osdn_short_conv_step(p, s["x"], s["weight"], s["bias"], s["state"], s["out"])
        return [s["out"], s["state"]]
    if op.startswith("scan"):
        osdn.osdn_scan_fwd(p, s["x"], s["gate"], s["init_state"], s["out"], s["final_state"], s["workspace"])
        if op == "scan_fwd":
            return [s["out"], s["final_state"]]
        osdn.osdn_scan_bwd(s["p_bwd"], s["x"], s["gate"], s["init_state"], s["dout"], s["dfinal_state"], s["dx"],
                           s["dgate"], s["dinit_state"], s["workspace"])
        return [s["out"], s["final_state"], s["dx"], s["dgate"], s["dinit_state"]]
    if op.startswith("conv"):
        osdn.osdn_short_conv_fwd(p, s["x"], s["weight"], s["bias"], s["init_state"], s["out"], s["final_state"])
        if op == "conv_fwd":
            return [s["out"], s["final_state"]]
        osdn.osdn_short_conv_bwd(p, s["x"], s["weight"], s["bias"], s["init_state"], s["dout"], s["dfinal_state"],
                                 s["dx"], s["dweight"], s["dbias"], s["dinit_state"], s["workspace"])
        got = [s["out"], s["final_state"], s["dx"], s["dweight"], s["dinit_state"]]
        return got if s["bias"] is None else got + [s["dbias"]]
    osdn.osdn_qk_norm_fwd(p, s["q"], s["k"], s["q_weight"], s["k_weight"], s["inv_freq"], s["positions"], s["q_out"],
                          s["k_out"])
    if op == "norm_fwd":
        return [s["q_out"], s["k_out"]]
    osdn.osdn_qk_norm_bwd(p, s["q"], s["k"], s["q_weight"], s["k_weight"], s["inv_freq"], s["positions"], s["dq_out"],
                          s["dk_out"], s["dq"], s["dk"], s["dq_weight"], s["dk_weight"], s["workspace"])
    got = [s["q_out"], s["k_out"], s["dq"], s["dk"]]
    return got if s["q_weight"] is None else got + [s["dq_weight"], s["dk_weight"]]


def run(s):
    return _own(s) if own else _plain(s)


# ---- the definition in 64 bits -------------------------------------------------------------------------------

def _blocks(a, b, size=256):
    """h_t = a_t h_{t-1} + b_t, token by token within blocks that run side by side, then block by block."""
    N, C = a.shape
    n = -(-N // size)
    pad = n * size - N
    a = torch.cat([a, a.new_ones(pad, C)]).view(n, size, C)
    b = torch.cat([b, b.new_zeros(pad, C)]).view(n, size, C)
    h, reach = torch.empty_like(b), torch.empty_like(a)
    h[:, 0], reach[:, 0] = b[:, 0], a[:, 0]
    for i in range(1, size):
        torch.addcmul(b[:, i], a[:, i], h[:, i - 1], out=h[:, i])
        torch.mul(a[:, i], reach[:, i - 1], out=reach[:, i])
    for j in range(1, n):
        h[j] += reach[j] * h[j - 1, -1]
    return h.view(n * size, C)[:N]


def _scan_exact(s, train):
    case = s["case"]
    x, g = s["x"].double(), s["gate"].double()
    C = case["C"]
    S = len(s["lens"])
    given = s["state"] if case["op"] == "scan_step" else s["init_state"]
    init = x.new_zeros(S, C) if given is None else given.double()
    a = g.exp()
    b = x * (-torch.expm1(g)) if case["complement"] else x
    cut, into = a.clone(), b.clone()
    begin = [sum(s["lens"][:i]) for i in range(S)]
    some = [i for i in range(S) if s["lens"][i]]
    t0 = torch.tensor([begin[i] for i in some], device=x.device)
    t1 = torch.tensor([begin[i] + s["lens"][i] - 1 for i in some], device=x.device)
    who = torch.tensor(some, device=x.device)
    into[t0] += a[t0] * init[who]
    cut[t0] = 0.0
    h = _blocks(cut, into)
    final = init.clone()
    final[who] = h[t1]
    if not train:
        return [h, final]
    before = torch.roll(h, 1, 0)
    before[t0] = init[who]
    df = torch.zeros_like(init) if s["dfinal_state"] is None else s["dfinal_state"].double()
    into = s["dout"].double()
    into[t1] += df[who]
    cut = torch.roll(a, -1, 0)
    cut[t1] = 0.0
    dh = _blocks(cut.flip(0), into.flip(0)).flip(0)
    dinit = df.clone()
    dinit[who] = a[t0] * dh[t0]
    if case["complement"]:
        return [h, final, dh * (-torch.expm1(g)), a * (before - x) * dh, dinit]
    return [h, final, dh, a * before * dh, dinit]


def _conv_exact(s, train):
    case = s["case"]
    W, C = case["W"], case["C"]
    S = len(s["lens"])
    given = s["state"] if case["op"] == "conv_step" else s["init_state"]
    x = s["x"].double().requires_grad_(train)
    w = s["weight"].double().requires_grad_(train)
    bias = None if s["bias"] is None else s["bias"].double().requires_grad_(train)
    init = (x.new_zeros(S, W - 1, C) if given is None else given.double()).detach().requires_grad_(train)
    outs, finals, at = [], [], 0
    for i, n in enumerate(s["lens"]):
        ext = torch.cat([init[i], x[at:at + n]])
        if n:
            z = (ext.unfold(0, W, 1) * w).sum(-1)
            z = z if bias is None else z + bias
            outs.append(z / (1.0 + torch.exp(-z)) if case["silu"] else z)
        finals.append(ext[n:])
        at += n
    out, final = torch.cat(outs), torch.stack(finals)
    if not train:
        return [out, final]
    loss = (out * s["dout"].double()).sum()
    if s["dfinal_state"] is not None:
        loss = loss + (final * s["dfinal_state"].double()).sum()
    wanted = [x, w, init] + ([] if bias is None else [bias])
    grads = torch.autograd.grad(loss, wanted)
    return [out.detach(), final.detach(), *grads]


def _norm_exact(s, train):
    case = s["case"]
    outs, loss, wanted, weights = [], 0.0, [], []
    for n in ("q", "k"):
        x = s[n].double().requires_grad_(train)
        y = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() if case["norm"] == "rms" else x / (x.pow(2).sum(-1, keepdim=True) + EPS).sqrt()
        if s[n + "_weight"] is not None:
            w = s[n + "_weight"].double().requires_grad_(train)
            weights.append(w)
            y = y * w
        if case["rot"] != "none":
            angle = s["positions"].double()[:, None, None] * s["inv_freq"]
            m = angle.shape[-1]
            pairs = torch.stack([y[..., :m], y[..., m:2 * m]], -1) if case["rot"] == "half" else y[..., :2 * m].unflatten(-1, (m, 2))
            turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), angle))
            turned = torch.cat([turned[..., 0], turned[..., 1]], -1) if case["rot"] == "half" else turned.flatten(-2)
            y = torch.cat([turned, y[..., 2 * m:]], -1)
        outs.append(y.detach())
        if train:
            wanted.append(x)
            loss = loss + (y * s["d" + n + "_out"].double()).sum()
    return outs + list(torch.autograd.grad(loss, wanted + weights)) if train else outs


def exact(case, seed):
    s = prepare(case, seed)
    kind, what = case["op"].split("_")
    return {"scan": _scan_exact, "conv": _conv_exact, "norm": _norm_exact}[kind](s, what == "train")


def work(case):
    """Every input read once and every output written once; a few operations an element."""
    kind, what = case["op"].split("_")
    e = 2 if case["io"] == "bf16" else 4
    N, S = case["B"] * case["T"], case.get("nseq") or case["B"]
    if kind == "scan":
        n, st = N * case["C"], 4 * S * case["C"]
        if what == "step":
            return dict(bytes=n * (2 * e + 4) + 2 * st, flops=4 * n)
        states = st * (2 if case["carry"] else 1)
        fwd = n * (2 * e + 4) + states
        if what == "fwd":
            return dict(bytes=fwd, flops=4 * n)
        return dict(bytes=fwd + n * (3 * e + 8) + states, flops=16 * n)
    if kind == "conv":
        n, W = N * case["C"], case["W"]
        st, par = e * S * (W - 1) * case["C"], 4 * case["C"] * (W + case["bias"])
        if what == "step":
            return dict(bytes=2 * e * n + 2 * st + par, flops=2 * W * n)
        states = st * (2 if case["carry"] else 1)
        if what == "fwd":
            return dict(bytes=2 * e * n + states + par, flops=2 * W * n)
        return dict(bytes=5 * e * n + 2 * states + 3 * par, flops=8 * W * n)
    n = N * (case["Hq"] + case["Hk"]) * case["D"]
    side = 0 if case["rot"] == "none" else 4 * N + 4 * case["D"]
    if what == "fwd":
        return dict(bytes=2 * e * n + side, flops=8 * n)
    return dict(bytes=5 * e * n + 2 * side, flops=24 * n)
