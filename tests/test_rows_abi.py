"""What the operators on rows of channels refuse, before anything is launched: the C ABI with pointers that are never
followed, and the checks of the marshalled calls."""
import ctypes

import pytest
import torch

import paper_2605_13473_b200 as osdn
from paper_2605_13473_b200.build import build

NULL, FAKE, ODD = ctypes.c_void_p(None), ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)
OK, INVALID, SHAPE, MISALIGNED, SMALL = 0, -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    build()
    return osdn.load_library()


def _size(n):
    return ctypes.c_size_t(n)


def scan_params(**more):
    return osdn.make_scan_params(**(dict(B=2, T=100, C=24, io_dtype="bf16") | more))


def conv_params(**more):
    return osdn.make_conv_params(**(dict(B=2, T=100, C=24, W=4, io_dtype="bf16") | more))


def norm_params(**more):
    return osdn.make_qk_norm_params(**(dict(B=2, T=100, Hq=4, Hk=2, D=64, io_dtype="bf16") | more))


def test_structures_are_those_of_the_header(lib):
    """Sizes as a C compiler lays them out (int32 fields, then pointers and int64 on eight bytes)."""
    assert ctypes.sizeof(osdn.ScanParams) == 40 and ctypes.sizeof(osdn.ConvParams) == 48
    assert ctypes.sizeof(osdn.QkNormParams) == 96


@pytest.mark.parametrize("change,code", [
    (dict(B=0), INVALID), (dict(T=0), SHAPE), (dict(C=0), SHAPE), (dict(T=-1), SHAPE), (dict(B=1 << 20, T=1 << 20), SHAPE),
    (dict(T=1 << 20, C=1 << 20), SHAPE),
])
def test_shapes_refused(lib, change, code):
    for make, ws, call, n in ((scan_params, lib.osdn_scan_workspace_bytes, lib.osdn_scan_step, 4),
                              (conv_params, lib.osdn_short_conv_workspace_bytes, lib.osdn_short_conv_step, 5)):
        p = make(**change)
        assert ws(ctypes.byref(p)) == 0
        assert call(ctypes.byref(p), *([FAKE] * n), NULL) == code
    if "C" not in change:
        p = norm_params(**change)
        assert lib.osdn_qk_norm_workspace_bytes(ctypes.byref(p)) == 0
        assert lib.osdn_qk_norm_fwd(ctypes.byref(p), *([FAKE] * 8), NULL) == code


def test_scan_refusals(lib):
    p = scan_params()
    r, need = ctypes.byref(p), lib.osdn_scan_workspace_bytes(ctypes.byref(p))
    assert need >= 2 * 24 * 4
    fwd = lambda *a: lib.osdn_scan_fwd(r, *a, NULL)  # noqa: E731
    assert fwd(NULL, FAKE, NULL, FAKE, NULL, NULL, _size(0)) == INVALID
    assert fwd(FAKE, NULL, NULL, FAKE, NULL, NULL, _size(0)) == INVALID
    assert fwd(FAKE, FAKE, NULL, NULL, NULL, NULL, _size(0)) == INVALID
    for k in range(5):
        a = [FAKE] * 5
        a[k] = ODD
        assert fwd(*a, NULL, _size(0)) == MISALIGNED
    p.flags = osdn.FLAG_SAVE_RESIDUALS
    assert fwd(FAKE, FAKE, NULL, FAKE, NULL, NULL, _size(need)) == INVALID
    assert fwd(FAKE, FAKE, NULL, FAKE, NULL, FAKE, _size(need - 1)) == SMALL
    bwd = lambda *a: lib.osdn_scan_bwd(r, *a, NULL)  # noqa: E731
    for k in (0, 1, 3, 5, 6, 8):
        a = [FAKE] * 9
        a[k] = NULL
        assert bwd(*a, _size(need)) == INVALID
    for k in range(9):
        a = [FAKE] * 9
        a[k] = ODD
        assert bwd(*a, _size(need)) == MISALIGNED
    assert bwd(*([FAKE] * 9), _size(need - 1)) == SMALL
    p.input_gate = 2
    assert bwd(*([FAKE] * 9), _size(need)) == INVALID
    p.input_gate, p.io_dtype = 0, 2
    assert bwd(*([FAKE] * 9), _size(need)) == INVALID
    q = scan_params()
    q.nseq = 3
    assert lib.osdn_scan_workspace_bytes(ctypes.byref(q)) == 0          # packed without cu_seqlens, and with B = 2
    q.cu_seqlens = 0x1000
    assert lib.osdn_scan_workspace_bytes(ctypes.byref(q)) == 0
    q.B = 1
    assert lib.osdn_scan_workspace_bytes(ctypes.byref(q)) > 0
    assert lib.osdn_scan_step(ctypes.byref(q), FAKE, FAKE, FAKE, FAKE, NULL) == INVALID   # dense only
    assert lib.osdn_scan_fwd(None, *([FAKE] * 6), _size(0), NULL) == INVALID


def test_conv_refusals(lib):
    for W in (0, 1, 5):
        p = conv_params(W=W)
        assert lib.osdn_short_conv_workspace_bytes(ctypes.byref(p)) == 0
        assert lib.osdn_short_conv_fwd(ctypes.byref(p), *([FAKE] * 6), NULL) == SHAPE
    p = conv_params()
    r, need = ctypes.byref(p), lib.osdn_short_conv_workspace_bytes(ctypes.byref(p))
    for k in (0, 1, 4):
        a = [FAKE] * 6
        a[k] = NULL
        assert lib.osdn_short_conv_fwd(r, *a, NULL) == INVALID
    for k in range(6):
        a = [FAKE] * 6
        a[k] = ODD
        assert lib.osdn_short_conv_fwd(r, *a, NULL) == MISALIGNED
    for k in (0, 1, 4, 6, 7, 10):
        a = [FAKE] * 11
        a[k] = NULL
        assert lib.osdn_short_conv_bwd(r, *a, _size(need), NULL) == INVALID
    for k in range(11):
        a = [FAKE] * 11
        a[k] = ODD
        assert lib.osdn_short_conv_bwd(r, *a, _size(need), NULL) == MISALIGNED
    assert lib.osdn_short_conv_bwd(r, *([FAKE] * 11), _size(need - 1), NULL) == SMALL
    p.activation = 2
    assert lib.osdn_short_conv_fwd(r, *([FAKE] * 6), NULL) == INVALID


@pytest.mark.parametrize("change,code", [
    (dict(D=4), SHAPE), (dict(D=68), SHAPE), (dict(D=264), SHAPE), (dict(rot_dim=8), SHAPE), (dict(rot_dim=80), SHAPE),
    (dict(Hq=0), INVALID), (dict(Hk=0), INVALID), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(q_row=248), INVALID), (dict(q_row=260), INVALID), (dict(k_row=127), INVALID), (dict(dq_row=1), INVALID),
    (dict(dk_row=-128), INVALID),
])
def test_norm_shapes_refused(lib, change, code):
    p = norm_params(**change)
    assert lib.osdn_qk_norm_workspace_bytes(ctypes.byref(p)) == 0
    assert lib.osdn_qk_norm_fwd(ctypes.byref(p), *([FAKE] * 8), NULL) == code
    assert lib.osdn_qk_norm_bwd(ctypes.byref(p), *([FAKE] * 13), _size(1 << 30), NULL) == code


def test_norm_refusals(lib):
    p = norm_params(rot_dim=64, q_row=512, k_row=512)
    r, need = ctypes.byref(p), lib.osdn_qk_norm_workspace_bytes(ctypes.byref(p))
    for k in (0, 1, 4, 6, 7):
        a = [FAKE] * 8
        a[k] = NULL
        assert lib.osdn_qk_norm_fwd(r, *a, NULL) == INVALID
    for k in range(8):
        a = [FAKE] * 8
        a[k] = ODD
        assert lib.osdn_qk_norm_fwd(r, *a, NULL) == MISALIGNED
    bwd = lambda a, n=need: lib.osdn_qk_norm_bwd(r, *a, _size(n), NULL)  # noqa: E731
    for k in (0, 1, 2, 3, 4, 6, 7, 8, 9, 12):       # 2, 3: a weight's gradient without the weight
        a = [FAKE] * 13
        a[k] = NULL
        assert bwd(a) == INVALID
    for k in range(13):
        a = [FAKE] * 13
        a[k] = ODD
        assert bwd(a) == MISALIGNED
    assert bwd([FAKE] * 13, need - 1) == SMALL
    p.norm = 2
    assert bwd([FAKE] * 13) == INVALID
    p.norm, p.rot_layout = 0, 2
    assert bwd([FAKE] * 13) == INVALID


def test_marshalled_calls_refuse_what_is_not_theirs(lib):
    x = torch.zeros(200, 24, dtype=torch.bfloat16)
    g, st = torch.zeros(200, 24), torch.zeros(2, 24)
    with pytest.raises(TypeError, match="not this call's params"):
        osdn.osdn_scan_step(conv_params(), x, g, st, x)
    with pytest.raises(TypeError, match="not this call's params"):
        osdn.osdn_short_conv_fwd(osdn.make_params(B=1, T=1, H=1, K=64, V=64, io_dtype="fp32"), x, g, None, None, x, None)
    with pytest.raises(TypeError):
        osdn.osdn_scan_step(None, x, g, st, x)
    with pytest.raises(RuntimeError, match="unsupported shape"):
        osdn.osdn_scan_step(scan_params(T=0), x, g, st, x)
    with pytest.raises(ValueError):
        osdn.make_scan_params(B=1, T=4, C=8, io_dtype="fp32", cu_seqlens=torch.zeros(2, dtype=torch.int32))
    if torch.cuda.is_available():
        with pytest.raises(ValueError, match="x: not on the current CUDA device"):
            osdn.osdn_scan_step(scan_params(), x, g, st, x)


@pytest.mark.gpu
def test_marshalled_calls_check_their_tensors():
    d = "cuda:0"
    x, g, st = torch.zeros(200, 24, dtype=torch.bfloat16, device=d), torch.zeros(200, 24, device=d), torch.zeros(2, 24, device=d)
    step = lambda *a: osdn.osdn_scan_step(scan_params(), *a)  # noqa: E731
    step(x, g, st, x.clone())
    for bad, says in (((x.float(), g, st, x), "x: wrong dtype"), ((x, g.double(), st, x), "gate: wrong dtype"),
                      ((x, g, st[:1], x), "state: 24 elements, 48 expected"), ((x, g.t().contiguous().t(), st, x), "gate: must be contiguous"),
                      ((x, g.cpu(), st, x), "gate: not on the current CUDA device"), ((x, g, st, x[:100]), "out: 2400 elements")):
        with pytest.raises(ValueError, match=says):
            step(*bad)
    with pytest.raises(TypeError, match="gate"):
        step(x, 5, st, x)
    with pytest.raises(RuntimeError, match="invalid argument"):
        step(x, g, None, x)
    with pytest.raises(RuntimeError, match="not sufficiently aligned"):
        step(x, torch.zeros(4801, device=d)[1:].view(200, 24), st, x)
    wide = torch.zeros(200, 512, dtype=torch.bfloat16, device=d)
    q, k = wide[:, :256].view(200, 4, 64), wide[:, 256:384].view(200, 2, 64)
    y, yk = torch.empty(200, 4, 64, dtype=torch.bfloat16, device=d), torch.empty(200, 2, 64, dtype=torch.bfloat16, device=d)
    osdn.osdn_qk_norm_fwd(norm_params(q_row=512, k_row=512), q, k, None, None, None, None, y, yk)
    with pytest.raises(ValueError, match="q: must be contiguous|q: rows"):
        osdn.osdn_qk_norm_fwd(norm_params(), q, k, None, None, None, None, y, yk)
    with pytest.raises(ValueError, match="k: rows"):
        osdn.osdn_qk_norm_fwd(norm_params(q_row=512, k_row=640), q, k, None, None, None, None, y, yk)
    with pytest.raises(ValueError, match="q: rows"):
        osdn.osdn_qk_norm_fwd(norm_params(q_row=512, k_row=512), q.transpose(0, 1), k, None, None, None, None, y, yk)


@pytest.mark.parametrize("name", ["q", "k", "dq", "dk"])
@pytest.mark.parametrize("io", ["bf16", "fp32"])
def test_views_of_as_many_elements_in_other_rows_are_refused(lib, name, io):
    """A view that steps by the params' row but has fewer (or other) rows ends before the kernels' last token.  Told from the
    shapes alone, before any device is asked for."""
    T, H, D, row = 8, 2, 16, 160
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[io]
    p = osdn.make_qk_norm_params(B=1, T=T, Hq=H, Hk=H, D=D, io_dtype=io, **{name + "_row": row})
    packed = {n: torch.zeros(T, H, D, dtype=dt) for n in ("q", "k", "q_out", "k_out", "dq", "dk")}
    wide = torch.zeros(T, row, dtype=dt)
    fits = [wide[:, :H * D].view(T, H, D), wide[:, 32:32 + H * D]]
    short = [wide[:T // 2, :2 * H * D].view(T // 2, 2 * H, D), torch.zeros(1, T * H, D, dtype=dt), wide[:T // 4, :4 * H * D].view(2, 8, D),
             wide[:T // 2, :2 * H * D], torch.zeros(1, T * H * D, dtype=dt), torch.zeros(T * H * D, dtype=dt)]
    other = [wide[:, :H * D].view(T, H, D).flip(0).transpose(1, 2), wide.view(2, T // 2, row)[:, :, :H * D],
             torch.zeros(T, H * row, dtype=dt).view(T, H, row)[:, :, :D]]

    def call(view):
        t = packed | {name: view}
        if name in "qk":
            osdn.osdn_qk_norm_fwd(p, t["q"], t["k"], None, None, None, None, t["q_out"], t["k_out"])
        else:
            osdn.osdn_qk_norm_bwd(p, t["q"], t["k"], None, None, None, None, t["q_out"], t["k_out"], t["dq"], t["dk"], None, None)

    for view in short + other:
        assert view.numel() == T * H * D
        with pytest.raises(ValueError, match=name + ": rows are not laid out as the params say"):
            call(view)
    for view in fits:                # only where the tensors are is left to complain about
        with pytest.raises((ValueError, RuntimeError)) as e:
            call(view)
        assert "rows" not in str(e.value) and "elements" not in str(e.value)
    one = osdn.make_qk_norm_params(B=1, T=1, Hq=H, Hk=H, D=D, io_dtype=io, **{name + "_row": row})
    p, packed = one, {n: v[:1] for n, v in packed.items()}
    with pytest.raises((ValueError, RuntimeError)) as e:      # one token: no step to compare
        call(torch.zeros(1, H, D, dtype=dt))
    assert "rows" not in str(e.value)


@pytest.mark.gpu
def test_boundaries_elsewhere_are_refused():
    """cu_seqlens of another device would be read by the kernels of this one.  (Here: params whose tensor is host memory; what
    they point at is never followed.)"""
    d = "cuda:0"
    cu = torch.tensor([0, 3, 8], dtype=torch.int32, device=d)
    x, g, w, q = torch.randn(8, 16, device=d), -torch.rand(8, 16, device=d), torch.randn(16, 4, device=d), torch.randn(8, 2, 8, device=d)
    y, yq, yk = torch.empty_like(x), torch.empty_like(q), torch.empty_like(q)
    calls = [(osdn.make_scan_params(B=1, T=8, C=16, io_dtype="fp32", cu_seqlens=cu), lambda p: osdn.osdn_scan_fwd(p, x, g, None, y, None)),
             (osdn.make_conv_params(B=1, T=8, C=16, W=4, io_dtype="fp32", cu_seqlens=cu),
              lambda p: osdn.osdn_short_conv_fwd(p, x, w, None, None, y, None)),
             (osdn.make_qk_norm_params(B=1, T=8, Hq=2, Hk=2, D=8, io_dtype="fp32", cu_seqlens=cu),
              lambda p: osdn.osdn_qk_norm_fwd(p, q, q, None, None, None, None, yq, yk))]
    for p, call in calls:
        call(p)
        p._cu_seqlens = cu.cpu()
        with pytest.raises(ValueError, match="cu_seqlens: not on the current CUDA device"):
            call(p)
        p._cu_seqlens = cu
        call(p)
        del p._cu_seqlens                 # a pointer set by hand
        call(p)
    torch.cuda.synchronize()


def test_channels_up_to_where_their_blocks_stay_in_32_bits(lib):
    most = 2 ** 31 - 1024
    for make, ws, call, n in ((scan_params, lib.osdn_scan_workspace_bytes, lib.osdn_scan_step, 4),
                              (conv_params, lib.osdn_short_conv_workspace_bytes, lib.osdn_short_conv_step, 5)):
        for C in (most + 1, 2 ** 31 - 1):
            p = make(B=1, T=1, C=C)
            assert ws(ctypes.byref(p)) == 0 and call(ctypes.byref(p), *([FAKE] * n), NULL) == SHAPE
        assert ws(ctypes.byref(make(B=1, T=1, C=most))) >= 4 * most
