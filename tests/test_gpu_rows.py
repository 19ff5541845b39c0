"""The operators on rows of channels on the GPU: against the 64-bit reference with its derived bounds, at the sizes and
masks where they can go wrong, and as a user runs them together."""
import pytest
import torch

import paper_2605_13473_b200 as osdn
import rows_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
MARK = 77.0    # what rows that are to stay hold


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _cu(lens):
    return torch.tensor([0] + lens, dtype=torch.int32).cumsum(0, dtype=torch.int32).to(DEV)


# ---- the gated linear recurrence ---------------------------------------------------------------------------
def _scan_inputs(N, C, io, seed, gates="mixed"):
    g = _gen(seed)
    x = torch.randn(N, C, generator=g).to(DT[io])
    gate = -torch.exp(torch.rand(N, C, generator=g) * 9.0 - 8.5)          # 2e-4 .. 1.6
    if gates == "edges":
        pick = torch.rand(N, C, generator=g)
        for lo, v in ((0.0, 0.0), (0.1, float("-inf")), (0.15, -120.0), (0.2, -86.0), (0.25, -1e-9), (0.3, -0.34657359),
                      (0.35, -0.34657362)):
            gate = torch.where((pick >= lo) & (pick < lo + 0.05), torch.tensor(v), gate)
    return x, gate


def _run_scan(x, gate, lens, dense, C, io, comp, init, dout, dfin, pad=0, saved=True):
    N = x.shape[0]
    cu = None if dense else _cu(lens)
    shape = dict(B=len(lens) if dense else 1, T=lens[0] if dense else N, C=C, io_dtype=io,
                 input_gate="complement" if comp else "plain", cu_seqlens=cu)
    p = osdn.make_scan_params(**shape, flags=osdn.FLAG_SAVE_RESIDUALS if saved else 0)
    S = len(lens)
    d = {k: None if v is None else v.to(DEV) for k, v in dict(x=x, gate=gate, init=init, dout=dout, dfin=dfin).items()}
    out, dx = (torch.full((N, C), MARK, device=DEV, dtype=DT[io]) for _ in range(2))
    dg = torch.full((N, C), MARK, device=DEV)
    fin, dinit = (torch.full((S, C), MARK, device=DEV) for _ in range(2))
    ws = torch.full((osdn.osdn_scan_workspace_bytes(p),), 255, device=DEV, dtype=torch.uint8)
    osdn.osdn_scan_fwd(p, d["x"], d["gate"], d["init"], out, fin, ws if saved else None)
    pb = osdn.make_scan_params(**shape, flags=osdn.FLAG_RESIDUALS_VALID if saved else 0)
    osdn.osdn_scan_bwd(pb, d["x"], d["gate"], d["init"], d["dout"], d["dfin"], dx, dg, dinit, ws)
    torch.cuda.synchronize()
    return out, fin, dx, dg, dinit


SCAN_SHAPES = [
    # lens, dense, C
    ([1], True, 1), ([1], True, 64), ([2, 2, 2], True, 20), ([127], True, 64), ([128, 128], True, 3), ([129], True, 132),
    ([300, 300], True, 68), ([1000], True, 8), ([2500], True, 64), ([4200], True, 16), ([9000], True, 4), ([700] * 5, True, 200),
    ([5, 1, 0, 300, 1, 1, 0, 0, 129, 64], False, 72), ([0, 0, 1], False, 5), ([3000, 17, 1200], False, 64),
    ([1] * 300, False, 12), ([0, 777], False, 130), ([128, 128, 256, 512], False, 64), ([2, 3] * 200, False, 33),
]


@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("comp", [False, True])
@pytest.mark.parametrize("lens,dense,C", SCAN_SHAPES)
def test_scan_matches_reference(io, comp, lens, dense, C):
    N = sum(lens)
    x, gate = _scan_inputs(N, C, io, N + C)
    g = _gen(N * 7 + C)
    init, dfin = torch.randn(len(lens), C, generator=g), torch.randn(len(lens), C, generator=g)
    dout = torch.randn(N, C, generator=g).to(DT[io])
    got = _run_scan(x, gate, lens, dense, C, io, comp, init, dout, dfin)
    want = ref.scan(x, gate, lens, init, comp, dout, dfin)
    for name, a, b in zip(("out", "final_state", "dx", "dgate", "dinit_state"), got, want):
        ref.check(a, b, name)


@pytest.mark.parametrize("comp", [False, True])
@pytest.mark.parametrize("lens,dense,C", [([400, 400], True, 64), ([200, 0, 333], False, 36), ([50], True, 7)])
def test_scan_edge_gates_and_missing_states(comp, lens, dense, C):
    """Gates of 0, -inf, far below and around the series' border; no states in; the backward on its own forward."""
    N = sum(lens)
    x, gate = _scan_inputs(N, C, "fp32", 5, "edges")
    dout = torch.randn(N, C, generator=_gen(6))
    got = _run_scan(x, gate, lens, dense, C, "fp32", comp, None, dout, None, saved=False)
    for name, a, b in zip(("out", "final_state", "dx", "dgate", "dinit_state"), got, ref.scan(x, gate, lens, None, comp, dout, None)):
        ref.check(a, b, name)


@pytest.mark.parametrize("io", ["bf16", "fp32"])
def test_scan_keeps_long_memories(io):
    """Gates of -3e-4 over 6000 tokens: a factor rounded to fp32 would lose 1e-4 of its distance from one."""
    N, C = 6000, 64
    x = torch.randn(N, C, generator=_gen(1)).to(DT[io])
    gate = -3e-4 * (0.5 + torch.rand(N, C, generator=_gen(2)))
    got = _run_scan(x, gate, [N], True, C, io, True, None, x, None)
    want = ref.scan(x, gate, [N], None, True, x, None)
    for name, a, (v, _) in zip(("final", "dgate", "dinit"), (got[1], got[3], got[4]), (want[1], want[3], want[4])):
        rel = float((a.double().cpu() - v).norm() / v.norm())
        assert rel < 3e-6, (name, rel)      # 2^-24 times the square root of a memory of 3300 tokens


def test_scan_gradients_are_differences():
    """Against central differences of the 64-bit reference's own forward (the formula, not the kernel's path)."""
    lens, C = [7, 0, 4], 3
    N = sum(lens)
    x, gate = _scan_inputs(N, C, "fp32", 3)
    init = torch.randn(3, C, generator=_gen(4))
    dout, dfin = torch.randn(N, C, generator=_gen(5)), torch.randn(3, C, generator=_gen(6))
    for comp in (False, True):
        _, _, dx, dg, dinit = _run_scan(x, gate, lens, False, C, "fp32", comp, init, dout, dfin)

        def loss(x_, g_, i_):
            o, f = ref.scan(x_, g_, lens, i_, comp)
            return float((o[0] * dout).sum() + (f[0] * dfin).sum())

        base = [x.double(), gate.double(), init.double()]
        for k, grad in enumerate((dx, dg, dinit)):
            for at in [(0, 0), (1, 2), (2, 1)]:
                step = 1e-5
                up, dn = [t.clone() for t in base], [t.clone() for t in base]
                up[k][at] += step
                dn[k][at] -= step
                slope = (loss(*up) - loss(*dn)) / (2 * step)
                assert abs(slope - float(grad[at])) < 1e-5 * (1 + abs(slope)), (comp, k, at)


@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("B,T,C", [(1, 1, 1), (3, 1, 100), (2, 5, 7), (130, 1, 64), (4, 17, 36)])
def test_scan_step_matches_reference(io, B, T, C):
    x, gate = _scan_inputs(B * T, C, io, B + T + C)
    state = torch.randn(B, C, generator=_gen(9))
    for comp in (False, True):
        st = state.to(DEV)
        out = torch.empty(B * T, C, device=DEV, dtype=DT[io])
        p = osdn.make_scan_params(B=B, T=T, C=C, io_dtype=io, input_gate="complement" if comp else "plain")
        osdn.osdn_scan_step(p, x.to(DEV), gate.to(DEV), st, out)
        assert osdn.osdn_last_launch_count() == 1
        want = ref.scan(x, gate, [T] * B, state, comp)
        ref.check(out, want[0], "out")
        ref.check(st, want[1], "state")


# ---- the short convolution ---------------------------------------------------------------------------------
def _run_conv(x, w, bias, lens, dense, io, silu, init, dout, dfin):
    N, C = x.shape
    S, W = len(lens), w.shape[1]
    p = osdn.make_conv_params(B=S if dense else 1, T=lens[0] if dense else N, C=C, W=W, io_dtype=io,
                              activation="silu" if silu else "none", cu_seqlens=None if dense else _cu(lens))
    d = {k: None if v is None else v.to(DEV) for k, v in dict(x=x, w=w, bias=bias, init=init, dout=dout, dfin=dfin).items()}
    out, dx = (torch.full((N, C), MARK, device=DEV, dtype=DT[io]) for _ in range(2))
    fin, dinit = (torch.full((S, W - 1, C), MARK, device=DEV, dtype=DT[io]) for _ in range(2))
    dw, db = torch.full((C, W), MARK, device=DEV), torch.full((C,), MARK, device=DEV)
    osdn.osdn_short_conv_fwd(p, d["x"], d["w"], d["bias"], d["init"], out, fin)
    ws = torch.full((osdn.osdn_short_conv_workspace_bytes(p),), 255, device=DEV, dtype=torch.uint8)
    osdn.osdn_short_conv_bwd(p, d["x"], d["w"], d["bias"], d["init"], d["dout"], d["dfin"], dx, dw,
                             None if bias is None else db, dinit, ws)
    torch.cuda.synchronize()
    return out, fin, dx, dw, db, dinit


CONV_SHAPES = [
    ([1], True, 1, 4), ([1, 1], True, 64, 3), ([2, 2, 2], True, 24, 4), ([3], True, 8, 2), ([65], True, 9, 4), ([64, 64], True, 512, 4),
    ([200] * 3, True, 40, 3), ([1000], True, 264, 4), ([5, 1, 0, 30, 2, 1, 0, 3, 129, 64], False, 72, 4), ([0, 0, 1, 0], False, 5, 4),
    ([700, 17, 300], False, 64, 3), ([1] * 150 + [2] * 40, False, 16, 4), ([64, 64, 128], False, 36, 2), ([3, 2] * 60, False, 8, 3),
]


@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("lens,dense,C,W", CONV_SHAPES)
def test_conv_matches_reference(io, silu, lens, dense, C, W):
    N, S = sum(lens), len(lens)
    g = _gen(N + C + W)
    x, dout = (torch.randn(N, C, generator=g).to(DT[io]) for _ in range(2))
    w, bias = torch.randn(C, W, generator=g), torch.randn(C, generator=g)
    init, dfin = (torch.randn(S, W - 1, C, generator=g).to(DT[io]) for _ in range(2))
    got = _run_conv(x, w, bias, lens, dense, io, silu, init, dout, dfin)
    want = ref.conv(x, w, bias, lens, init, silu, io == "bf16", dout, dfin)
    for name, a, b in zip(("out", "final_state", "dx", "dweight", "dbias", "dinit_state"),
                          got, want):
        ref.check(a, b, name)


@pytest.mark.parametrize("lens,dense,C,W", [([70, 70], True, 16, 4), ([3, 0, 90], False, 12, 3)])
def test_conv_without_bias_and_states(lens, dense, C, W):
    N = sum(lens)
    g = _gen(1)
    x, dout, w = torch.randn(N, C, generator=g), torch.randn(N, C, generator=g), torch.randn(C, W, generator=g)
    out, fin, dx, dw, db, dinit = _run_conv(x, w, None, lens, dense, "fp32", True, None, dout, None)
    want = ref.conv(x, w, None, lens, None, True, False, dout, None)
    for name, a, b in zip(("out", "final", "dx", "dw", "dinit"), (out, fin, dx, dw, dinit),
                          (want[0], want[1], want[2], want[3], want[5])):
        ref.check(a, b, name)
    assert bool((db == MARK).all())


def test_conv_large_arguments_saturate():
    """Far positive and negative pre-activations: z and 0, slopes 1 and 0, nothing that is not a number."""
    x = torch.tensor([[1.0, -1.0, 30.0, -30.0, 1e4, -1e4, 1e30, -1e30]] * 6)
    w = torch.zeros(8, 4)
    w[:, 3] = 1.0
    for io in ("fp32", "bf16"):
        out, _, dx, dw, _, _ = _run_conv(x.to(DT[io]), w, None, [6], True, io, True, None, torch.ones(6, 8).to(DT[io]), None)
        want = ref.conv(x.to(DT[io]), w, None, [6], None, True, io == "bf16", torch.ones(6, 8), None)
        ref.check(out, want[0], "out")
        assert bool(torch.isfinite(dx).all()) and bool((dx[:, 4].float() == 1.0).all()) and bool((dx[:, 5].float() == 0.0).all())


@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("B,T,C,W", [(1, 1, 1, 4), (3, 1, 64, 4), (2, 5, 9, 3), (130, 1, 40, 2), (4, 2, 24, 4)])
def test_conv_step_matches_reference(io, B, T, C, W):
    g = _gen(B + T + C)
    x, state = torch.randn(B * T, C, generator=g).to(DT[io]), torch.randn(B, W - 1, C, generator=g).to(DT[io])
    w, bias = torch.randn(C, W, generator=g), torch.randn(C, generator=g)
    st, out = state.to(DEV), torch.empty(B * T, C, device=DEV, dtype=DT[io])
    osdn.osdn_short_conv_step(osdn.make_conv_params(B=B, T=T, C=C, W=W, io_dtype=io), x.to(DEV), w.to(DEV), bias.to(DEV), st, out)
    assert osdn.osdn_last_launch_count() == 1
    want = ref.conv(x, w, bias, [T] * B, state, True, io == "bf16")
    ref.check(out, want[0], "out")
    assert torch.equal(st.double().cpu(), want[1][0])


# ---- norms of queries and keys -----------------------------------------------------------------------------
def _run_norm(case, seed=0, rows=None):
    io, N, Hq, Hk, D, kind, weights, R, layout, pos = case
    g = _gen(seed + N + D)
    x = {n: torch.randn(N, h, D, generator=g).to(DT[io]) for n, h in (("q", Hq), ("k", Hk))}
    dy = {n: torch.randn(N, h, D, generator=g).to(DT[io]) for n, h in (("q", Hq), ("k", Hk))}
    w = {n: (1.0 + 0.3 * torch.randn(D, generator=g)) if weights else None for n in "qk"}
    inv = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R) if R else None
    positions = None
    if R and pos == "far":
        positions = torch.randint(0, 1 << 30, (N,), generator=g).to(torch.int32)
        positions[0] = 2 ** 31 - 1
    elif R and pos == "negative":
        positions = -torch.arange(N, dtype=torch.int32)
    p = osdn.make_qk_norm_params(B=1, T=N, Hq=Hq, Hk=Hk, D=D, io_dtype=io, norm=kind, eps=1e-5, rot_dim=R, rot_layout=layout)
    to = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    yq, dq = (torch.full((N, Hq, D), MARK, device=DEV, dtype=DT[io]) for _ in range(2))
    yk, dk = (torch.full((N, Hk, D), MARK, device=DEV, dtype=DT[io]) for _ in range(2))
    dwq, dwk = (torch.full((D,), MARK, device=DEV) if weights else None for _ in range(2))
    args = (to(x["q"]), to(x["k"]), to(w["q"]), to(w["k"]), to(inv), to(positions))
    osdn.osdn_qk_norm_fwd(p, *args, yq, yk)
    ws = torch.full((osdn.osdn_qk_norm_workspace_bytes(p),), 255, device=DEV, dtype=torch.uint8)
    osdn.osdn_qk_norm_bwd(p, *args, to(dy["q"]), to(dy["k"]), dq, dk, dwq, dwk, ws if weights else None)
    torch.cuda.synchronize()
    angle = None if not R else ref.angles(torch.arange(N) if positions is None else positions, inv)
    for n, y, dx, dw in (("q", yq, dq, dwq), ("k", yk, dk, dwk)):
        want = ref.norm(x[n], w[n], kind, 1e-5, angle, layout, dy[n])
        ref.check(y, want[0], n)
        ref.check(dx, want[1], "d" + n)
        if weights:
            ref.check(dw, want[2], "dw" + n)


NORM_CASES = [
    # io, tokens, Hq, Hk, D, norm, weights, rot_dim, layout, positions
    ("bf16", 1, 1, 1, 128, "l2", False, 0, "half", None), ("fp32", 1, 16, 4, 128, "rms", True, 128, "half", "far"),
    ("bf16", 37, 8, 8, 128, "l2", False, 0, "half", None), ("bf16", 64, 16, 4, 128, "rms", True, 128, "half", "far"),
    ("fp32", 65, 4, 2, 64, "rms", True, 64, "pairs", "far"), ("fp32", 33, 3, 1, 96, "l2", True, 96, "half", None),
    ("fp32", 33, 5, 5, 80, "rms", False, 80, "half", "far"), ("fp32", 20, 2, 2, 256, "rms", True, 64, "half", "negative"),
    ("bf16", 20, 1, 1, 8, "l2", True, 0, "half", None), ("fp32", 20, 7, 1, 24, "rms", True, 16, "half", "far"),
    ("fp32", 50, 12, 6, 128, "rms", True, 64, "pairs", "negative"), ("bf16", 5000, 3, 1, 64, "rms", True, 64, "half", "far"),
    ("fp32", 3000, 8, 8, 128, "l2", True, 128, "half", None), ("bf16", 700, 20, 20, 112, "rms", True, 112, "pairs", None),
    ("fp32", 9, 40, 2, 200, "l2", True, 192, "pairs", "far"),
]


@pytest.mark.parametrize("case", NORM_CASES, ids=lambda c: "-".join(map(str, c)))
def test_norm_matches_reference(case):
    _run_norm(case)


def test_norm_of_zero_rows_and_of_one_large_value():
    """A zero head has u = 0 and a finite gradient of du / sqrt(eps); large values stay finite as their squares do."""
    N, H, D = 3, 2, 64
    q = torch.zeros(N, H, D)
    q[1, 0, 5], q[2] = 1e18, 1e-20
    dy = torch.randn(N, H, D, generator=_gen(1))
    p = osdn.make_qk_norm_params(B=1, T=N, Hq=H, Hk=H, D=D, io_dtype="fp32", norm="l2", eps=1e-6)
    y, yk, dq, dk = (torch.empty(N, H, D, device=DEV) for _ in range(4))
    osdn.osdn_qk_norm_fwd(p, q.to(DEV), q.to(DEV), None, None, None, None, y, yk)
    osdn.osdn_qk_norm_bwd(p, q.to(DEV), q.to(DEV), None, None, None, None, dy.to(DEV), dy.to(DEV), dq, dk, None, None)
    want = ref.norm(q, None, "l2", 1e-6, None, "half", dy)
    ref.check(y, want[0], "y")
    ref.check(dq, want[1], "dq")
    assert torch.equal(y, yk) and torch.equal(dq, dk)


def test_norm_reads_and_writes_parts_of_wider_rows():
    N, Hq, Hk, D = 70, 4, 2, 64
    for io in ("bf16", "fp32"):
        wide = torch.randn(N, (Hq + 2 * Hk) * D, generator=_gen(2)).to(DT[io]).to(DEV)
        q, k = wide[:, :Hq * D].view(N, Hq, D), wide[:, Hq * D:(Hq + Hk) * D]
        grad = torch.full_like(wide, MARK)
        dq, dk = grad[:, :Hq * D].view(N, Hq, D), grad[:, Hq * D:(Hq + Hk) * D].view(N, Hk, D)
        row = wide.shape[1]
        p = osdn.make_qk_norm_params(B=2, T=N // 2, Hq=Hq, Hk=Hk, D=D, io_dtype=io, q_row=row, k_row=row, dq_row=row, dk_row=row)
        yq, yk = torch.empty(N, Hq, D, device=DEV, dtype=DT[io]), torch.empty(N, Hk, D, device=DEV, dtype=DT[io])
        dyq, dyk = torch.randn_like(yq), torch.randn_like(yk)
        osdn.osdn_qk_norm_fwd(p, q, k, None, None, None, None, yq, yk)
        osdn.osdn_qk_norm_bwd(p, q, k, None, None, None, None, dyq, dyk, dq, dk, None, None)
        for a, y, dy, d in ((q, yq, dyq, dq), (k.view(N, Hk, D), yk, dyk, dk)):
            want = ref.norm(a, None, "l2", 1e-6, None, "half", dy)
            ref.check(y, want[0], "y")
            ref.check(d, want[1], "dx")
        assert bool((grad[:, (Hq + Hk) * D:] == MARK).all())


def test_norm_in_place():
    N, H, D = 40, 8, 128
    q, k, dyq, dyk = (torch.randn(N, H, D, generator=_gen(i)).to(torch.bfloat16).to(DEV) for i in range(4))
    p = osdn.make_qk_norm_params(B=1, T=N, Hq=H, Hk=H, D=D, io_dtype="bf16")
    y = [torch.empty_like(q) for _ in range(4)]
    osdn.osdn_qk_norm_fwd(p, q, k, None, None, None, None, y[0], y[1])
    osdn.osdn_qk_norm_bwd(p, q, k, None, None, None, None, dyq, dyk, y[2], y[3], None, None)
    osdn.osdn_qk_norm_bwd(p, q, k, None, None, None, None, dyq, dyk, dyq, dyk, None, None)
    osdn.osdn_qk_norm_fwd(p, q, k, None, None, None, None, q, k)
    for a, b in zip((q, k, dyq, dyk), y):
        assert torch.equal(a, b)


def test_norm_counts_places_from_the_sequence_start():
    lens, D = [3, 0, 5, 1], 32
    N = sum(lens)
    q = torch.randn(N, 2, D, generator=_gen(3))
    inv = 100.0 ** (-torch.arange(0, 16, 2, dtype=torch.float64) / 16)
    y, yk = torch.empty(N, 2, D, device=DEV), torch.empty(N, 2, D, device=DEV)
    for cu, B, T, places in ((_cu(lens), 1, N, [0, 1, 2, 0, 1, 2, 3, 4, 0]), (None, 3, 3, [0, 1, 2] * 3)):
        p = osdn.make_qk_norm_params(B=B, T=T, Hq=2, Hk=2, D=D, io_dtype="fp32", rot_dim=16, cu_seqlens=cu)
        osdn.osdn_qk_norm_fwd(p, q.to(DEV), q.to(DEV), None, None, inv.to(DEV), None, y, yk)
        ref.check(y, ref.norm(q, None, "l2", 1e-6, ref.angles(torch.tensor(places), inv), "half")[0], "y")


# ---- what all three promise --------------------------------------------------------------------------------
@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,pad", [([100, 0, 60], 50), ([1], 300), ([0, 0], 5), ([128, 128], 1), ([300], 700)])
def test_rows_behind_the_last_sequence_stay(io, lens, pad):
    N, live, S = sum(lens) + pad, sum(lens), len(lens)
    C, W, H, D = 64, 4, 2, 32
    g = _gen(pad)
    x = torch.randn(N, C, generator=g)
    x[live:] = float("nan")                                   # must reach nothing
    x = x.to(DT[io])
    gate = -torch.rand(N, C, generator=g)
    gate[live:] = float("nan")
    init, dfin = torch.randn(S, C, generator=g), torch.randn(S, C, generator=g)
    out, fin, dx, dg, dinit = _run_scan(x, gate, lens, False, C, io, True, init, x, dfin)
    want = ref.scan(x[:live], gate[:live], lens, init, True, x[:live], dfin)
    for name, a, b in zip(("out", "fin", "dx", "dg", "dinit"), (out[:live], fin, dx[:live], dg[:live], dinit), want):
        ref.check(a, b, name)
    for a in (out, dx, dg):
        assert bool((a[live:] == MARK).all())
    w, bias = torch.randn(C, W, generator=g), torch.randn(C, generator=g)
    init, dfin = (torch.randn(S, W - 1, C, generator=g).to(DT[io]) for _ in range(2))
    got = _run_conv(x, w, bias, lens, False, io, True, init, x, dfin)
    want = ref.conv(x[:live], w, bias, lens, init, True, io == "bf16", x[:live], dfin)
    for k, (a, b) in enumerate(zip(got, want)):
        ref.check(a[:live] if k in (0, 2) else a, b, k)
    assert bool((got[0][live:] == MARK).all()) and bool((got[2][live:] == MARK).all())
    q, w = x.view(N, H, D).to(DEV), torch.ones(D, device=DEV)
    p = osdn.make_qk_norm_params(B=1, T=N, Hq=H, Hk=H, D=D, io_dtype=io, cu_seqlens=_cu(lens))
    y = [torch.full_like(q, MARK) for _ in range(4)]
    dw = [torch.empty(D, device=DEV) for _ in range(2)]
    osdn.osdn_qk_norm_fwd(p, q, q, w, w, None, None, y[0], y[1])
    osdn.osdn_qk_norm_bwd(p, q, q, w, w, None, None, q, q, y[2], y[3], *dw,
                          torch.empty(osdn.osdn_qk_norm_workspace_bytes(p), device=DEV, dtype=torch.uint8))
    for a in y:
        assert bool((a[live:] == MARK).all())
    want = ref.norm(x[:live].view(live, H, D), w, "l2", 1e-6, None, "half", x[:live].view(live, H, D))
    ref.check(y[0][:live], want[0], "y")
    ref.check(y[2][:live], want[1], "dq")
    for a in dw:
        ref.check(a, want[2], "dw")


def _bundle(io, B, T, C, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    d = dict(x=r(B * T, C).to(DT[io]), gate=-torch.rand(B * T, C, generator=g, device=DEV), dout=r(B * T, C).to(DT[io]),
             w=r(C, 4), inv=10000.0 ** (-torch.arange(0, 64, 2, device=DEV, dtype=torch.float64) / 64), qw=r(64))
    e = lambda *s, dt=DT[io]: torch.empty(*s, device=DEV, dtype=dt)  # noqa: E731
    f = torch.float32
    H = C // 64
    d |= dict(h=e(B * T, C), fin=e(B, C, dt=f), dx=e(B * T, C), dg=e(B * T, C, dt=f), di=e(B, C, dt=f), y=e(B * T, C),
              cdx=e(B * T, C), dw=e(C, 4, dt=f), q=e(B * T, H, 64), k=e(B * T, H, 64), dq=e(B * T, H, 64), dk=e(B * T, H, 64),
              dqw=e(64, dt=f), dkw=e(64, dt=f))
    ps = osdn.make_scan_params(B=B, T=T, C=C, io_dtype=io, flags=osdn.FLAG_SAVE_RESIDUALS)
    pb = osdn.make_scan_params(B=B, T=T, C=C, io_dtype=io, flags=osdn.FLAG_RESIDUALS_VALID)
    pc = osdn.make_conv_params(B=B, T=T, C=C, W=4, io_dtype=io)
    pn = osdn.make_qk_norm_params(B=B, T=T, Hq=H, Hk=H, D=64, io_dtype=io, rot_dim=64)
    ws = [torch.empty(n, device=DEV, dtype=torch.uint8) for n in (osdn.osdn_scan_workspace_bytes(ps),
          osdn.osdn_short_conv_workspace_bytes(pc), osdn.osdn_qk_norm_workspace_bytes(pn))]

    def run():
        osdn.osdn_short_conv_fwd(pc, d["x"], d["w"], None, None, d["y"], None)
        osdn.osdn_scan_fwd(ps, d["y"], d["gate"], None, d["h"], d["fin"], ws[0])
        osdn.osdn_scan_bwd(pb, d["y"], d["gate"], None, d["dout"], None, d["dx"], d["dg"], d["di"], ws[0])
        osdn.osdn_short_conv_bwd(pc, d["x"], d["w"], None, None, d["dx"], None, d["cdx"], d["dw"], None, None, ws[1])
        y, g_ = d["y"].view(B * T, H, 64), d["dx"].view(B * T, H, 64)
        osdn.osdn_qk_norm_fwd(pn, y, y, d["qw"], d["qw"], d["inv"], None, d["q"], d["k"])
        osdn.osdn_qk_norm_bwd(pn, y, y, d["qw"], d["qw"], d["inv"], None, g_, g_, d["dq"], d["dk"], d["dqw"], d["dkw"], ws[2])

    names = ("h", "fin", "dx", "dg", "di", "y", "cdx", "dw", "q", "k", "dq", "dk", "dqw", "dkw")
    return d, run, lambda: [d[n].clone() for n in names]


def test_calls_repeat_bit_by_bit_on_other_streams_at_once_and_in_graphs():
    one, run1, read1 = _bundle("bf16", 2, 1500, 320, 1)
    two, run2, read2 = _bundle("fp32", 3, 700, 192, 2)
    run1()
    run2()
    want1, want2 = read1(), read2()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):                                        # two callers at once
        with torch.cuda.stream(s1):
            run1()
        with torch.cuda.stream(s2):
            run2()
    torch.cuda.synchronize()
    assert all(map(torch.equal, read1(), want1)) and all(map(torch.equal, read2(), want2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run1()
    other = {n: torch.randn_like(one[n].float()).to(one[n].dtype) for n in ("x", "dout")}
    saved = {n: one[n].clone() for n in other}
    for n, t in other.items():
        one[n].copy_(t)
    graph.replay()
    got = read1()
    run1()
    torch.cuda.synchronize()
    assert all(map(torch.equal, got, read1())) and not torch.equal(got[0], want1[0])
    for n, t in saved.items():
        one[n].copy_(t)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(map(torch.equal, read1(), want1))


def test_offsets_past_32_bits():
    """More than 2^31 elements; the last rows against a call on those rows alone."""
    C, T = 1024, (1 << 21) + 300
    tail = 200
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(T, C, device=DEV, dtype=torch.bfloat16)
    x.normal_(generator=g)
    out, dx = torch.empty_like(x), torch.empty_like(x)
    w = torch.randn(C, 4, device=DEV)
    small = x[-tail - 3:].contiguous()
    sout, sdx = torch.empty_like(small), torch.empty_like(small)
    for xx, oo, dd in ((x, out, dx), (small, sout, sdx)):
        p = osdn.make_conv_params(B=1, T=xx.shape[0], C=C, W=4, io_dtype="bf16")
        osdn.osdn_short_conv_fwd(p, xx, w, None, None, oo, None)
        osdn.osdn_short_conv_bwd(p, xx, w, None, None, xx, None, dd, torch.empty_like(w), None, None,
                                 torch.empty(osdn.osdn_short_conv_workspace_bytes(p), device=DEV, dtype=torch.uint8))
    assert torch.equal(out[-tail:], sout[-tail:]) and torch.equal(dx[-tail:], sdx[-tail:])
    for xx, oo, dd in ((x, out, dx), (small, sout, sdx)):
        p = osdn.make_qk_norm_params(B=1, T=xx.shape[0], Hq=4, Hk=4, D=128, io_dtype="bf16", q_row=C, k_row=C, dq_row=C, dk_row=C)
        n = xx.shape[0]
        q, k = xx[:, :512].view(n, 4, 128), xx[:, 512:].view(n, 4, 128)
        yq = oo.view(-1)[:n * 512].view(n, 4, 128)
        yk = oo.view(-1)[n * 512:].view(n, 4, 128)
        osdn.osdn_qk_norm_fwd(p, q, k, None, None, None, None, yq, yk)
        osdn.osdn_qk_norm_bwd(p, q, k, None, None, None, None, yq, yk, dd[:, :512].view(n, 4, 128), dd[:, 512:].view(n, 4, 128), None, None)
    assert torch.equal(dx[-tail:], sdx[-tail:])
    assert torch.equal(out.view(-1)[-tail * 512:], sout.view(-1)[-tail * 512:])
    gate = torch.full((T, C), -0.5, device=DEV)
    gate[-tail] = float("-inf")                               # nothing from before reaches the last rows
    dg = torch.empty_like(gate)
    fins = []
    for xx, gg, oo, dd, ddg in ((x, gate, out, dx, dg), (small[3:], gate[-tail:].clone(), sout[3:], sdx[3:], torch.empty(tail, C, device=DEV))):
        p = osdn.make_scan_params(B=1, T=xx.shape[0], C=C, io_dtype="bf16")
        ws = torch.empty(osdn.osdn_scan_workspace_bytes(p), device=DEV, dtype=torch.uint8)
        fin = torch.empty(1, C, device=DEV)
        osdn.osdn_scan_fwd(p, xx, gg, None, oo, fin, None)
        osdn.osdn_scan_bwd(p, xx, gg, None, xx, None, dd, ddg, None, ws)
        fins.append((fin, ddg))
    ref_room = lambda a, b, r: bool(((a.float() - b.float()).abs() <= r * (b.float().abs() + 1)).all())  # noqa: E731
    assert ref_room(out[-tail:], sout[-tail:], 2.0 ** -8) and ref_room(dx[-tail:], sdx[-tail:], 2.0 ** -8)
    assert ref_room(fins[0][0], fins[1][0], 1e-5) and ref_room(fins[0][1][-tail + 1:], fins[1][1][1:], 1e-5)


def test_a_block_from_projection_to_layer_and_its_decode():
    """Convolution -> norms -> the layer over a prompt, then token by token from the caches, against the whole sequence
    at once; the recurrence on the convolution's values beside it."""
    B, T, extra, H, D = 2, 70, 5, 2, 64
    C, L = 3 * H * D, T + extra
    g = torch.Generator(device=DEV).manual_seed(3)
    proj = torch.randn(B, L, C, generator=g, device=DEV)
    w, bias = torch.randn(C, 4, generator=g, device=DEV) / 2, 0.1 * torch.randn(C, generator=g, device=DEV)
    beta = torch.sigmoid(torch.randn(B, L, H, generator=g, device=DEV))
    gate = -0.1 * torch.nn.functional.softplus(torch.randn(B, L, H, generator=g, device=DEV))
    rgate = -torch.rand(B, L, H * D, generator=g, device=DEV)
    inv = 10000.0 ** (-torch.arange(0, D, 2, device=DEV, dtype=torch.float64) / D)

    def mix(n, first, convd):
        rows = convd.view(B * n, C)
        q, k = torch.empty(B * n, H, D, device=DEV), torch.empty(B * n, H, D, device=DEV)
        pos = torch.arange(first, first + n, device=DEV, dtype=torch.int32).repeat(B)
        p = osdn.make_qk_norm_params(B=B, T=n, Hq=H, Hk=H, D=D, io_dtype="fp32", rot_dim=D, q_row=C, k_row=C)
        osdn.osdn_qk_norm_fwd(p, rows[:, :H * D].view(-1, H, D), rows[:, H * D:2 * H * D].view(-1, H, D), None, None, inv, pos, q, k)
        return q, k, rows[:, 2 * H * D:].contiguous()

    def prefill(n):
        x = proj[:, :n].contiguous()
        y, cache = torch.empty_like(x), torch.empty(B, 3, C, device=DEV)
        osdn.osdn_short_conv_fwd(osdn.make_conv_params(B=B, T=n, C=C, W=4, io_dtype="fp32"), x, w, bias, None, y, cache)
        q, k, v = mix(n, 0, y)
        p = osdn.make_params(B=B, T=n, H=H, K=D, V=D, io_dtype="fp32")
        out, S, d = torch.empty(B * n, H, D, device=DEV), torch.empty(B, H, D, D, device=DEV), torch.empty(B, H, D, device=DEV)
        ws = torch.empty(osdn.osdn_workspace_bytes(p, False), device=DEV, dtype=torch.uint8)
        osdn.osdn_fwd(p, q, k, v.view(-1, H, D), beta[:, :n].contiguous(), gate[:, :n].contiguous(), None, None, None, out, S, d, ws)
        h, r = torch.empty_like(v), torch.empty(B, H * D, device=DEV)
        osdn.osdn_scan_fwd(osdn.make_scan_params(B=B, T=n, C=H * D, io_dtype="fp32", input_gate="complement"), v,
                           rgate[:, :n].contiguous(), None, h, r)
        return out.view(B, n, H, D), h.view(B, n, -1), cache, S, d, r

    out, h, _, S_all, d_all, r_all = prefill(L)
    o, hh, cache, S, d, r = prefill(T)
    assert torch.allclose(o, out[:, :T], atol=1e-5, rtol=1e-4) and torch.allclose(hh, h[:, :T], atol=1e-5, rtol=1e-5)
    one = dict(B=B, T=1, io_dtype="fp32")
    for t in range(T, L):
        y = torch.empty(B, C, device=DEV)
        osdn.osdn_short_conv_step(osdn.make_conv_params(**one, C=C, W=4), proj[:, t].contiguous(), w, bias, cache, y)
        q, k, v = mix(1, t, y)
        ot, ht = torch.empty(B, H, D, device=DEV), torch.empty(B, H * D, device=DEV)
        osdn.osdn_decode_step(osdn.make_params(**one, H=H, K=D, V=D), q, k, v.view(B, H, D), beta[:, t].contiguous(),
                              gate[:, t].contiguous(), None, S, d, ot)
        osdn.osdn_scan_step(osdn.make_scan_params(**one, C=H * D, input_gate="complement"), v, rgate[:, t].contiguous(), r, ht)
        assert torch.allclose(ot, out[:, t], atol=1e-5, rtol=1e-4) and torch.allclose(ht, h[:, t], atol=1e-5, rtol=1e-5)
    assert torch.allclose(S, S_all, atol=1e-5, rtol=1e-4) and torch.allclose(r, r_all, atol=1e-5, rtol=1e-5)


@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("B,T", [(130, 523), (131, 70), (300, 200), (1300, 9)])
def test_scan_of_many_sequences(io, B, T):
    """More walks than SMs, with few and with many rows: copies of one sequence give copies of its result."""
    C = 64
    x, gate = _scan_inputs(T, C, io, B + T)
    g = _gen(B)
    init, dfin, dout = torch.randn(1, C, generator=g), torch.randn(1, C, generator=g), torch.randn(T, C, generator=g).to(DT[io])
    many = lambda t: t.repeat(B, 1)  # noqa: E731
    got = _run_scan(many(x), many(gate), [T] * B, True, C, io, True, many(init), many(dout), many(dfin))
    for name, a, b in zip(("out", "final", "dx", "dgate", "dinit"), got, ref.scan(x, gate, [T], init, True, dout, dfin)):
        ref.check(a.view(B, -1, C)[0].contiguous(), b, name)
        ref.check(a.view(B, -1, C)[B - 1].contiguous(), b, name)
        if T >= 64:    # short sequences share units, at places of their own
            assert bool((a.view(B, -1, C) == a.view(B, -1, C)[:1]).all()), name


@pytest.mark.parametrize("lens", [[40000], [25000, 1, 0, 6, 14993]])
def test_scan_of_one_long_row_split_over_a_cluster(lens):
    C, N = 64, sum(lens)
    x, gate = _scan_inputs(N, C, "bf16", 77)
    g = _gen(78)
    init, dfin = torch.randn(len(lens), C, generator=g), torch.randn(len(lens), C, generator=g)
    dout = torch.randn(N, C, generator=g).to(torch.bfloat16)
    got = _run_scan(x, gate, lens, len(lens) == 1, C, "bf16", False, init, dout, dfin)
    for name, a, b in zip(("out", "final", "dx", "dgate", "dinit"), got, ref.scan(x, gate, lens, init, False, dout, dfin)):
        ref.check(a, b, name)


@pytest.mark.parametrize("T,Hq,Hk,D", [(9500, 3, 2, 64), (5000, 1, 1, 128), (2500, 5, 1, 256)])
def test_norm_of_many_tokens_behind_a_padded_end(T, Hq, Hk, D):
    """Whole tokens to a lane group, heads of odd numbers, the last sequence's end inside the rows."""
    live = T - 333
    g = _gen(T)
    q, k = torch.randn(T, Hq, D, generator=g), torch.randn(T, Hk, D, generator=g)
    q[live:], k[live:] = float("nan"), float("nan")
    w = 1.0 + 0.2 * torch.randn(D, generator=g)
    inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    cu = _cu([1000, 0, live - 1000])
    places = torch.cat([torch.arange(1000), torch.arange(live - 1000)])
    d = lambda t: t.to(DEV)  # noqa: E731
    for layout in ("half", "pairs"):
        p = osdn.make_qk_norm_params(B=1, T=T, Hq=Hq, Hk=Hk, D=D, io_dtype="fp32", norm="rms", rot_dim=D, rot_layout=layout, cu_seqlens=cu)
        y = [torch.full_like(t, MARK, device=DEV) for t in (q, k, q, k)]
        dw = [torch.empty(D, device=DEV) for _ in range(2)]
        osdn.osdn_qk_norm_fwd(p, d(q), d(k), d(w), None, d(inv), None, y[0], y[1])
        osdn.osdn_qk_norm_bwd(p, d(q), d(k), d(w), None, d(inv), None, d(q), d(k), y[2], y[3], dw[0], None,
                              torch.empty(osdn.osdn_qk_norm_workspace_bytes(p), device=DEV, dtype=torch.uint8))
        angle = ref.angles(places, inv)
        for t, wt, a, b, s in ((q, w, y[0], y[2], dw[0]), (k, None, y[1], y[3], None)):
            want = ref.norm(t[:live], wt, "rms", 1e-6, angle, layout, t[:live])
            ref.check(a[:live], want[0], "y")
            ref.check(b[:live], want[1], "dx")
            if s is not None:
                ref.check(s, want[2], "dw")
        for a in y:
            assert bool((a[live:] == MARK).all())


@pytest.mark.parametrize("broken", [[0, 300, 100, 500], [0, 600, 600, 900], [-50, 100, 200, 400], [700, 20, 10, -3], [0, 0, 0, 0]])
def test_broken_boundaries_stay_inside_the_tensors(broken):
    """What comes out is undefined; what lies around the tensors is not touched and every call ends."""
    N, C, guard = 500, 64, 64
    cu = torch.tensor(broken, dtype=torch.int32, device=DEV)

    def inside(*shape, dt=torch.float32):
        n = 1
        for s in shape:
            n *= s
        whole = torch.full((n + 2 * guard,), MARK, device=DEV, dtype=dt)
        return whole, whole[guard:guard + n].view(*shape)

    bufs = {}

    def out(name, *shape, dt=torch.float32):
        bufs[name], view = inside(*shape, dt=dt)
        return view

    x = torch.randn(N, C, device=DEV)
    gate = -torch.rand(N, C, device=DEV)
    p = osdn.make_scan_params(B=1, T=N, C=C, io_dtype="fp32", cu_seqlens=cu)
    ws = torch.zeros(osdn.osdn_scan_workspace_bytes(p), device=DEV, dtype=torch.uint8)
    st = torch.randn(3, C, device=DEV)
    osdn.osdn_scan_fwd(p, x, gate, st, out("h", N, C), out("f", 3, C))
    osdn.osdn_scan_bwd(p, x, gate, st, x, st, out("dx", N, C), out("dg", N, C), out("di", 3, C), ws)
    p = osdn.make_conv_params(B=1, T=N, C=C, W=4, io_dtype="fp32", cu_seqlens=cu)
    w, st = torch.randn(C, 4, device=DEV), torch.randn(3, 3, C, device=DEV)
    ws = torch.zeros(osdn.osdn_short_conv_workspace_bytes(p), device=DEV, dtype=torch.uint8)
    osdn.osdn_short_conv_fwd(p, x, w, None, st, out("y", N, C), out("cf", 3, 3, C))
    osdn.osdn_short_conv_bwd(p, x, w, None, st, x, st, out("cdx", N, C), out("dw", C, 4), None, out("cdi", 3, 3, C), ws)
    p = osdn.make_qk_norm_params(B=1, T=N, Hq=1, Hk=1, D=C, io_dtype="fp32", rot_dim=16, cu_seqlens=cu)
    inv = torch.ones(8, device=DEV, dtype=torch.float64)
    q = x.view(N, 1, C)
    osdn.osdn_qk_norm_fwd(p, q, q, None, None, inv, None, out("q", N, 1, C), out("k", N, 1, C))
    osdn.osdn_qk_norm_bwd(p, q, q, None, None, inv, None, q, q, out("dq", N, 1, C), out("dk", N, 1, C), None, None)
    torch.cuda.synchronize()
    for name, b in bufs.items():
        assert bool((b[:guard] == MARK).all()) and bool((b[-guard:] == MARK).all()), name


@pytest.mark.parametrize("lens,bad", [([3, 2, 4, 1, 70], 1), ([100, 37, 300, 0, 5], 2), ([20000, 5, 12000, 3000], 1), ([9000, 16000, 7000], 1)])
def test_a_sequence_of_nan_and_infinities_stays_alone(lens, bad):
    """Neighbours in a packed batch get what they get beside finite values, forward and backward, across CTAs and clusters."""
    C, N = 64, sum(lens)
    lo = sum(lens[:bad])
    hi = lo + lens[bad]
    g = _gen(N)
    x, gate = _scan_inputs(N, C, "fp32", N)
    dout, init, dfin = torch.randn(N, C, generator=g), torch.randn(len(lens), C, generator=g), torch.randn(len(lens), C, generator=g)
    w = torch.randn(C, 4, generator=g)
    cinit, cdfin = (torch.randn(len(lens), 3, C, generator=g) for _ in range(2))
    keep = torch.ones(N, dtype=torch.bool)
    keep[lo:hi] = False
    others = [s for s in range(len(lens)) if s != bad]
    for poison in ("values", "gates"):
        px, pg, pd = x.clone(), gate.clone(), dout.clone()
        (px if poison == "values" else pg)[lo:hi] = float("nan")
        px[lo:hi, ::2] = float("inf")
        pd[lo:hi, 1::2] = float("-inf")
        a = _run_scan(x, gate, lens, False, C, "fp32", False, init, dout, dfin)
        b = _run_scan(px, pg, lens, False, C, "fp32", False, init, pd, dfin)
        for k, (u, v) in enumerate(zip(a, b)):
            m = keep if k in (0, 2, 3) else others
            assert torch.equal(u[m], v[m]), (poison, k)
        a = _run_conv(x, w, None, lens, False, "fp32", True, cinit, dout, cdfin)
        b = _run_conv(px, w, None, lens, False, "fp32", True, cinit, pd, cdfin)
        for k in (0, 1, 2, 5):
            m = keep if k in (0, 2) else others
            assert torch.equal(a[k][m], b[k][m]), (poison, k)


def test_conv_weight_sums_past_32_bits():
    """Channels times taps beyond 2^32: every channel's own gradient, exact for one token without activation."""
    C, W = 859_000_064, 4
    g = torch.Generator(device=DEV).manual_seed(1)
    x, dout = (torch.empty(1, C, device=DEV, dtype=torch.bfloat16).normal_(generator=g) for _ in range(2))
    w = torch.empty(C, W, device=DEV)
    w[:, :3], w[:, 3] = 1.0, dout[0]
    p = osdn.make_conv_params(B=1, T=1, C=C, W=W, io_dtype="bf16", activation="none")
    out, dx = torch.empty_like(x), torch.empty_like(x)
    dw, db = torch.full((C, W), MARK, device=DEV), torch.full((C,), MARK, device=DEV)
    ws = torch.empty(osdn.osdn_short_conv_workspace_bytes(p), device=DEV, dtype=torch.uint8)
    osdn.osdn_short_conv_fwd(p, x, w, None, None, out, None)
    osdn.osdn_short_conv_bwd(p, x, w, None, None, dout, None, dx, dw, db, None, ws)
    for at in range(0, C, 1 << 27):                           # products of two bf16 values are fp32 values
        part = slice(at, min(at + (1 << 27), C))
        prod = x[0, part].float() * dout[0, part].float()
        assert torch.equal(dw[part, 3], prod) and torch.equal(out[0, part], prod.bfloat16())
        assert not bool(dw[part, :3].any()) and torch.equal(db[part], dout[0, part].float())
        assert torch.equal(dx[0, part], dout[0, part].float().square().bfloat16())


@pytest.mark.parametrize("comp", [False, True])
@pytest.mark.parametrize("lens,dense,C", [([100], True, 64), ([20000], True, 64), ([300, 9000, 50], False, 64), ([2000], True, 5),
                                          ([40] * 3, True, 64), ([9, 0, 30], False, 5)])
def test_scan_state_that_is_not_finite_stays_so(comp, lens, dense, C):
    """However a walk hands its state on: rows behind an infinity or NaN are not finite to the sequence's end, gates of -inf and
    gates that add up to it in between or not; the rows in front, the other channels and the other sequences are as without."""
    N, s = sum(lens), len(lens) - 1 if len(lens) < 3 else (1 if lens[1] else 2)
    lo = sum(lens[:s])
    hi = lo + lens[s]
    x, gate = _scan_inputs(N, C, "fp32", 11, "edges")
    gate[torch.rand(N, C, generator=_gen(12)) < 0.05] = -3e38
    g = _gen(13)
    dout, init, dfin = torch.randn(N, C, generator=g), torch.randn(len(lens), C, generator=g), torch.randn(len(lens), C, generator=g)
    mid, ch = lo + lens[s] // 3, (torch.arange(C) % 2 == 0)
    gate[mid, ch] = -0.5                                      # there the input reaches the state
    gate[mid - 1, ch] = -0.5
    want = _run_scan(x, gate, lens, dense, C, "fp32", comp, init, dout, dfin)
    px, pd = x.clone(), dout.clone()
    px[mid, ch] = torch.where(torch.arange(int(ch.sum())) % 3 == 0, float("nan"), float("inf"))
    pd[mid, ch] = float("-inf")
    rows = torch.arange(N)
    behind, ahead = (rows >= mid) & (rows < hi), (rows <= mid) & (rows >= lo)
    out, fin, _, _, _ = _run_scan(px, gate, lens, dense, C, "fp32", comp, init, dout, dfin)
    hit = behind[:, None] & ch[None]
    assert not bool(torch.isfinite(out.cpu()[hit]).any()) and not bool(torch.isfinite(fin.cpu()[s, ch]).any())
    assert torch.equal(out.cpu()[~hit], want[0].cpu()[~hit])
    _, _, dx, dg, dinit = _run_scan(x, gate, lens, dense, C, "fp32", comp, init, pd, dfin)
    hit = ahead[:, None] & ch[None]
    assert not bool(torch.isfinite(dg.cpu()[hit]).any()) and not bool(torch.isfinite(dinit.cpu()[s, ch]).any())
    if not comp:
        assert not bool(torch.isfinite(dx.cpu()[hit]).any())
    assert torch.equal(dx.cpu()[~hit], want[2].cpu()[~hit]) and torch.equal(dg.cpu()[~hit], want[3].cpu()[~hit])
    if dense and len(lens) == 1:                              # token by token
        st, y = init.to(DEV), torch.empty(N, C, device=DEV)
        p = osdn.make_scan_params(B=1, T=N, C=C, io_dtype="fp32", input_gate="complement" if comp else "plain")
        osdn.osdn_scan_step(p, px.to(DEV), gate.to(DEV), st, y)
        assert torch.equal(torch.isfinite(y), torch.isfinite(out)) and torch.equal(torch.isfinite(st), torch.isfinite(fin))
