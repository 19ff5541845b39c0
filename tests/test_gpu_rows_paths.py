"""The operators on rows of channels at sizes whose kernels and branches only larger batches reach: chunks of more than eight rows
and several to a warp (convolution), whole tokens to a lane group (norms), sixteen warps (recurrence)."""
import math

import numpy as np
import pytest
import torch

import paper_2605_13473_b200 as osdn
import rows_reference as ref
from test_gpu_rows import DEV, DT, MARK, _gen, _run_conv, _run_scan, _scan_inputs

pytestmark = pytest.mark.gpu


# ---- the short convolution: chunks of 24 rows and more from 19000 rows on, several to a warp from 303104 (fp32: 454656) ---
LONG_ROWS = [
    # lens, dense, C, W
    ([700003], True, 8, 4), ([233000] * 3, True, 8, 3), ([400000, 0, 1, 2, 299000, 5, 1000], False, 8, 4), ([61, 40000, 0, 3, 30001], False, 136, 2),
    ([50001], True, 5, 4),
]


@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,dense,C,W", LONG_ROWS)
def test_conv_sums_over_long_rows_are_exact_for_whole_numbers(io, lens, dense, C, W):
    """Inputs of -1, 0 and 1: every result and every partial sum is a whole number below 2^24 (bf16: 256), so none is rounded
    and no row may be missing or counted twice."""
    N, S = sum(lens), len(lens)
    g = _gen(N + C)
    trits = lambda *s: torch.randint(-1, 2, s, generator=g, dtype=torch.int8)  # noqa: E731
    x, dout = trits(N, C).to(DT[io]), (trits(N, C) | 1).to(DT[io])            # -1 and 1
    w, bias = trits(C, W).float(), trits(C).float()
    init, dfin = trits(S, W - 1, C).to(DT[io]), trits(S, W - 1, C).to(DT[io])
    got = _run_conv(x, w, bias, lens, dense, io, False, init, dout, dfin)
    want = ref.conv(x, w, bias, lens, init, False, io == "bf16", dout, dfin)
    for name, a, (v, _) in zip(("out", "final_state", "dx", "dweight", "dbias", "dinit_state"), got, want):
        assert float(v.abs().max()) < (256 if a.dtype == torch.bfloat16 else 2 ** 24)
        bad = a.double().cpu().reshape(v.shape) != v
        assert not bool(bad.any()), (name, int(bad.sum()), bad.nonzero()[0].tolist())


@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,dense,C,W", [([70001], True, 8, 4), ([61, 20000, 0, 3, 15001], False, 136, 4), ([30001], True, 7, 3)])
def test_conv_with_activation_over_long_rows(io, lens, dense, C, W):
    """A term of a weight's sum goes through the rows of its warp's chunks (160 at most, one chunk to a warp here), the CTA's four warps,
    888 / 16 CTAs and their sixteen sums: fewer than 256 additions."""
    N, S = sum(lens), len(lens)
    g = _gen(N + C + W)
    x, dout = (torch.randn(N, C, generator=g).to(DT[io]) for _ in range(2))
    dout = dout.abs()                                                          # sums that grow with every row
    w, bias = torch.randn(C, W, generator=g), torch.randn(C, generator=g)
    init, dfin = (torch.randn(S, W - 1, C, generator=g).to(DT[io]) for _ in range(2))
    got = _run_conv(x, w, bias, lens, dense, io, True, init, dout, dfin)
    want = ref.conv(x, w, bias, lens, init, True, io == "bf16", dout, dfin, chain=256)
    for name, a, b in zip(("out", "final_state", "dx", "dweight", "dbias", "dinit_state"), got, want):
        ref.check(a, b, name)


# ---- norms: whole tokens to a lane group from 9472 (D <= 64), 4736 (D <= 128) and 2368 tokens on -----------------------------
WHOLE_TOKENS = [
    # io, tokens, Hq, Hk, D, norm, weights, rot_dim, layout, far positions, parts of wider rows
    ("bf16", 9500, 3, 1, 64, "rms", True, 64, "half", True, False), ("bf16", 4800, 8, 2, 128, "rms", True, 128, "half", True, True),
    ("bf16", 4737, 2, 2, 128, "l2", True, 128, "pairs", False, True), ("bf16", 5001, 5, 1, 96, "rms", True, 96, "half", True, False),
    ("bf16", 2400, 3, 2, 256, "rms", True, 64, "half", True, True), ("bf16", 4736, 6, 3, 128, "l2", False, 0, "half", False, True),
    ("bf16", 5000, 4, 4, 80, "l2", False, 80, "pairs", True, False), ("fp32", 4800, 5, 5, 80, "rms", True, 80, "half", True, True),
    ("fp32", 9501, 1, 1, 24, "l2", True, 16, "pairs", True, False), ("bf16", 40000, 2, 1, 64, "rms", True, 64, "half", False, True),
]


@pytest.mark.parametrize("case", WHOLE_TOKENS, ids=lambda c: "-".join(map(str, c)))
def test_norm_of_whole_tokens(case):
    """The gradients of the outputs are the inputs, so that the weights' sums grow with every token.  A term of them goes through
    the heads of its lane group's tokens (40000 tokens: five of them; the others two at most), the CTA's 32 groups, 296 / 16 CTAs and their
    sixteen sums: fewer than 128 additions."""
    io, N, Hq, Hk, D, kind, weights, R, layout, far, wide = case
    g = _gen(N + D)
    x = {n: torch.randn(N, h, D, generator=g).to(DT[io]) for n, h in (("q", Hq), ("k", Hk))}
    w = {n: (1.0 + 0.3 * torch.randn(D, generator=g)) if weights else None for n in "qk"}
    inv = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R) if R else None
    pos = torch.randint(0, 1 << 30, (N,), generator=g).to(torch.int32) if far else None
    row = (Hq + Hk) * D + 16
    rows = dict(q_row=row, k_row=row, dq_row=row, dk_row=row) if wide else {}
    p = osdn.make_qk_norm_params(B=1, T=N, Hq=Hq, Hk=Hk, D=D, io_dtype=io, norm=kind, eps=1e-5, rot_dim=R, rot_layout=layout, **rows)
    to = lambda t: None if t is None else t.to(DEV)  # noqa: E731

    def pair():
        if not wide:
            return None, torch.full((N, Hq, D), MARK, device=DEV, dtype=DT[io]), torch.full((N, Hk, D), MARK, device=DEV, dtype=DT[io])
        whole = torch.full((N, row), MARK, device=DEV, dtype=DT[io])
        return whole, whole[:, :Hq * D].view(N, Hq, D), whole[:, Hq * D:(Hq + Hk) * D].view(N, Hk, D)

    _, q, k = pair()
    q.copy_(x["q"]), k.copy_(x["k"])
    grads, dq, dk = pair()
    yq, yk = (torch.full((N, h, D), MARK, device=DEV, dtype=DT[io]) for h in (Hq, Hk))
    dw = {n: torch.full((D,), MARK, device=DEV) if weights else None for n in "qk"}
    args = (q, k, to(w["q"]), to(w["k"]), to(inv), to(pos))
    osdn.osdn_qk_norm_fwd(p, *args, yq, yk)
    ws = torch.full((osdn.osdn_qk_norm_workspace_bytes(p),), 255, device=DEV, dtype=torch.uint8)
    osdn.osdn_qk_norm_bwd(p, *args, to(x["q"]), to(x["k"]), dq, dk, dw["q"], dw["k"], ws if weights else None)
    angle = ref.angles(torch.arange(N) if pos is None else pos, inv) if R else None
    for n, y, dx in (("q", yq, dq), ("k", yk, dk)):
        want = ref.norm(x[n], w[n], kind, 1e-5, angle, layout, x[n], chain=128)
        ref.check(y, want[0], n)
        ref.check(dx, want[1], "d" + n)
        if weights:
            ref.check(dw[n], want[2], "dw" + n)
    if wide:
        assert bool((grads[:, (Hq + Hk) * D:] == MARK).all())


@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_norm_of_whole_tokens_in_place(io, layout):
    """The backward has the next heads' rows on their way while it writes over the gradients it has read."""
    N, Hq, Hk, D = 9000, 6, 3, 128
    q, dyq = (torch.randn(N, Hq, D, generator=_gen(i)).to(DT[io]).to(DEV) for i in range(2))
    k, dyk = (torch.randn(N, Hk, D, generator=_gen(i)).to(DT[io]).to(DEV) for i in (2, 3))
    w = 1.0 + 0.3 * torch.randn(D, generator=_gen(4)).to(DEV)
    inv = 10000.0 ** (-torch.arange(0, D, 2, device=DEV, dtype=torch.float64) / D)
    p = osdn.make_qk_norm_params(B=1, T=N, Hq=Hq, Hk=Hk, D=D, io_dtype=io, norm="rms", rot_dim=D, rot_layout=layout)
    ws = torch.empty(osdn.osdn_qk_norm_workspace_bytes(p), device=DEV, dtype=torch.uint8)
    y = [torch.empty_like(t) for t in (q, k, q, k)]
    dw = [torch.empty(D, device=DEV) for _ in range(4)]
    osdn.osdn_qk_norm_fwd(p, q, k, w, w, inv, None, y[0], y[1])
    osdn.osdn_qk_norm_bwd(p, q, k, w, w, inv, None, dyq, dyk, y[2], y[3], dw[0], dw[1], ws)
    osdn.osdn_qk_norm_bwd(p, q, k, w, w, inv, None, dyq, dyk, dyq, dyk, dw[2], dw[3], ws)
    osdn.osdn_qk_norm_fwd(p, q, k, w, w, inv, None, q, k)
    for a, b in zip((q, k, dyq, dyk, dw[2], dw[3]), y + dw[:2]):
        assert torch.equal(a, b)


# ---- the recurrence: sixteen warps ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("io", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,C,comp", [
    ([40000], 64, True), ([25000, 1, 0, 6, 14993], 64, True),                           # split
    ([300, 1, 0, 0, 217, 120], 7680, True), ([300, 1, 0, 0, 217, 120], 7680, False),    # packed, as many walks as take no split
    ([100, 0, 203], 7680, True), ([520], 7688, False),                                  # eight warps; a last block of eight channels
])
def test_scan_of_sixteen_warps(io, lens, C, comp):
    N = sum(lens)
    x, gate = _scan_inputs(N, C, io, 77)
    g = _gen(78)
    init, dfin = torch.randn(len(lens), C, generator=g), torch.randn(len(lens), C, generator=g)
    dout = torch.randn(N, C, generator=g).to(DT[io])
    got = _run_scan(x, gate, lens, len(lens) == 1, C, io, comp, init, dout, dfin)
    for name, a, b in zip(("out", "final", "dx", "dgate", "dinit"), got, ref.scan(x, gate, lens, init, comp, dout, dfin)):
        ref.check(a, b, name)


@pytest.mark.parametrize("lens,dense,B", [([9000], True, 1), ([300, 0, 8000, 777], False, 1), ([40] * 50, True, 50)])
def test_scan_backward_with_kept_and_recomputed_states_is_the_same(lens, dense, B):
    C, N = 64, sum(lens)
    x, gate = _scan_inputs(N, C, "bf16", 5)
    g = _gen(6)
    init, dfin, dout = torch.randn(len(lens), C, generator=g), torch.randn(len(lens), C, generator=g), torch.randn(N, C, generator=g).to(DT["bf16"])
    a = _run_scan(x, gate, lens, dense, C, "bf16", True, init, dout, dfin)
    b = _run_scan(x, gate, lens, dense, C, "bf16", True, init, dout, dfin, saved=False)
    assert all(map(torch.equal, a, b))


@pytest.mark.parametrize("T,B", [(131072, 1), (2048, 128)])
def test_scan_of_equal_gates_rounds_as_its_rows_do(T, B):
    """A gate of -1e-4 at every row.  A row's rounding, 2^-24 of the state at most and of either sign, is remembered for 10^4 rows:
    2^-24 (1 - a^2)^-1/2 = 2^-24 sqrt(5000) in all, however a walk is split; twice that for a product of two states."""
    C, rate = 8, 1e-4
    g = _gen(1)
    x, dout = 0.5 + torch.randn(T, C, generator=g), 0.5 + torch.randn(T, C, generator=g)
    gate = torch.full((T, C), -rate)
    many = lambda t: t.repeat(B, 1)  # noqa: E731
    got = _run_scan(many(x), many(gate), [T] * B, True, C, "fp32", False, None, many(dout), None)
    a = math.exp(float(gate[0, 0]))
    xs, ds = x.double().numpy(), dout.double().numpy()
    h, e, before, dh = np.zeros(C), np.zeros(C), np.empty((T, C)), np.empty((T, C))
    for t in range(T):
        before[t] = h
        h = a * h + xs[t]
    for t in range(T - 1, -1, -1):
        dh[t] = ds[t] + e
        e = a * dh[t]
    out = np.concatenate([before[1:], h[None]])
    room = 2.0 ** -24 * (2 * rate) ** -0.5
    for name, y, want, r in zip(("out", "final", "dx", "dgate", "dinit"), got, (out, h[None], dh, before * (a * dh), e[None]),
                                (room, room, room, 2 * room, room)):
        y = y.double().cpu().view(B, -1, C)[B - 1].numpy()
        off = np.linalg.norm(y - want) / np.linalg.norm(want)
        assert off <= r, (name, off, r)
