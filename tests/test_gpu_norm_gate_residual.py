"""Norm after a block, gate, scaled residual and norm before the next block, against the definition in 64 bits.

Tolerances, relative to the larger of the value and the RMS of its row's tensor: fp32 arithmetic 1e-5, as for the
library's other row operators (a statistic is a tree sum of up to 32768 terms, off by a few 2^-24; each element takes
fewer than ten further roundings), and bf16 outputs one rounding more, 2^-8 of the value."""
import pytest
import torch

import decoder_reference as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def make(rows, cols, x_dtype, y_dtype, groups, seed=0, mean=0.25, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, y = (n(rows, cols) * 2).to(x_dtype), (n(rows, cols) * spread + mean).to(y_dtype)
    gate = None if groups is None else (n(groups, cols) * 0.5).to(y_dtype)
    vec = dict(post_gamma=n(cols) * 0.3 + 1, post_beta=n(cols) * 0.1, pre_gamma=n(cols) * 0.3 + 1, pre_beta=n(cols) * 0.1)
    return x, y, gate, vec


def close(got, want, extra=0.0):
    assert got is not None
    tau = want.pow(2).mean().sqrt()
    bound = (1e-5 + extra) * torch.maximum(want.abs(), tau) + (2 ** -8 * want.abs() if got.dtype == BF16 else 0)
    worst = ((got.double() - want).abs() / bound.clamp_min(1e-300)).max().item()
    assert worst <= 1.0, worst


def run(rows, cols, x_dtype=BF16, y_dtype=BF16, post="rms", pre="rms", groups=None, gate_rows=None, alpha=1.25, eps=1e-5,
        extra=0.0, drop=(), **kw):
    from paper_2511_03586_b200 import api
    x, y, gate, vec = make(rows, cols, x_dtype, y_dtype, groups, **kw)
    for name in drop:
        vec[name] = None
    h, n = api.pd_norm_gate_residual_norm(y, x, gate=gate, gate_rows=gate_rows, alpha=alpha, eps=eps, post_norm=post,
                                          pre_norm=pre, **vec)
    wh, wn = ref.norm_gate_residual_norm(y, x, gate, gate_rows or max(1, -(-rows // (groups or 1))), alpha, eps, post,
                                         vec["post_gamma"], vec["post_beta"], pre, vec["pre_gamma"], vec["pre_beta"])
    assert h.dtype == x_dtype and n.dtype == y_dtype
    close(h, wh, extra)
    close(n, wn, extra)


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16), (BF16, F32), (F32, F32)], ids=str)
@pytest.mark.parametrize("norms", [("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("layer", "none"), ("none", "none"),
                                   ("rms", "layer")], ids=str)
@pytest.mark.parametrize("cols", [64, 1000, 1001, 4096])
def test_types_and_norms(types, norms, cols):
    run(37, cols, *types, *norms, groups=1)


@pytest.mark.parametrize("cols", [1, 7, 8, 256, 264, 512, 520, 1024, 1032, 2048, 2056, 4104, 8192, 8200, 16384, 16392, 32768,
                                  32776, 40000])
@pytest.mark.parametrize("types", [(BF16, BF16), (F32, F32)], ids=str)
def test_every_row_length_path(cols, types):
    run(5, cols, *types, "layer", "rms", groups=5)


@pytest.mark.parametrize("rows,groups,gate_rows", [(1, 1, None), (1, None, None), (33, 33, 1), (33, 3, 11), (33, 4, 10),
                                                   (33, 1, 33), (33, 1, 1000), (1, 1, 7)])
def test_gates(rows, groups, gate_rows):
    for cols in (320, 1031):
        run(rows, cols, groups=groups, gate_rows=gate_rows)


def test_missing_vectors():
    run(9, 640, post="layer", pre="layer", drop=("post_gamma", "pre_beta"))
    run(9, 641, post="layer", pre="layer", drop=("post_beta", "pre_gamma", "pre_beta"))
    run(9, 640, drop=("post_gamma", "post_beta", "pre_gamma", "pre_beta"))


def test_many_rows():
    run(30000, 128, F32, BF16, groups=30000)
    run(70000, 9)


@pytest.mark.parametrize("cols", [1024, 1023])
def test_large_mean(cols):
    # |mean| = 1000 spreads: v - mean is exact to half a step of v, 2^-24 * 1000 of a spread
    run(16, cols, F32, F32, "layer", "layer", mean=1000.0, extra=4 * 1000 * 2.0 ** -24)


def test_rows_of_zeros_and_one_column():
    from paper_2511_03586_b200 import api
    for cols in (64, 65):
        z = torch.zeros(3, cols, device="cuda")
        h, n = api.pd_norm_gate_residual_norm(z, z, post_norm="layer", pre_norm="rms")
        assert (h == 0).all() and (n == 0).all()


@pytest.mark.parametrize("cols", [512, 2048, 777])
def test_in_place_and_partial_outputs(cols):
    from paper_2511_03586_b200 import api
    x, y, gate, vec = make(40, cols, BF16, BF16, 1)
    h, n = api.pd_norm_gate_residual_norm(y, x, gate=gate, **vec)
    x2, y2 = x.clone(), y.clone()
    api.pd_norm_gate_residual_norm(y2, x2, gate=gate, h=x2, n=y2, **vec)
    assert torch.equal(x2, h) and torch.equal(y2, n)
    # only one of the outputs
    import ctypes
    d = api.NormGateResidualDesc(40, cols, 40, api.PD_BF16, api.PD_BF16, 1, 1, 1.0, 1e-5)
    ptr = lambda t: t.data_ptr()  # noqa: E731
    args = [ptr(y), ptr(x), ptr(gate), ptr(vec["post_gamma"]), None, ptr(vec["pre_gamma"]), None]
    only = torch.zeros_like(x)
    stream = torch.cuda.current_stream().cuda_stream
    assert api._lib.pd_norm_gate_residual_norm(ctypes.byref(d), *args, ptr(only), None, stream) == 0
    assert torch.equal(only, h)
    assert api._lib.pd_norm_gate_residual_norm(ctypes.byref(d), *args, None, ptr(only), stream) == 0
    assert torch.equal(only, n)


def test_unaligned_tensors_and_streams():
    from paper_2511_03586_b200 import api
    x, y, gate, vec = make(21, 640, BF16, BF16, 21)
    want = api.pd_norm_gate_residual_norm(y, x, gate=gate, **vec)
    flat = torch.empty(21 * 640 + 1, dtype=BF16, device="cuda")
    shifted = flat[1:].view(21, 640)
    shifted.copy_(y)
    h, n = api.pd_norm_gate_residual_norm(shifted, x, gate=gate, **vec)   # two bytes off: the scalar path
    for got, w in zip((h, n), want):
        assert ((got.double() - w.double()).abs() <= 2 ** -7 * w.double().abs() + 1e-5).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        h, n = api.pd_norm_gate_residual_norm(y, x, gate=gate, **vec)
    s.synchronize()
    assert torch.equal(h, want[0]) and torch.equal(n, want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h, n = api.pd_norm_gate_residual_norm(y, x, gate=gate, **vec)
    h.zero_(), n.zero_()
    g.replay()
    assert torch.equal(h, want[0]) and torch.equal(n, want[1])


def test_binding_refusals():
    from paper_2511_03586_b200 import api
    x, y, gate, vec = make(4, 64, BF16, BF16, 4)
    with pytest.raises(ValueError):
        api.pd_norm_gate_residual_norm(y, x[:3])
    with pytest.raises(ValueError):
        api.pd_norm_gate_residual_norm(y, x, gate=gate[:1], gate_rows=2)
    with pytest.raises(TypeError):
        api.pd_norm_gate_residual_norm(y, x, gate=gate.float())
    with pytest.raises(ValueError):
        api.pd_norm_gate_residual_norm(y, x, post_gamma=vec["post_gamma"][:8].contiguous())
    with pytest.raises(TypeError):
        api.pd_norm_gate_residual_norm(y.half(), x)
    with pytest.raises(ValueError):
        api.pd_norm_gate_residual_norm(y.t(), x.t())
    with pytest.raises(api.PdError):
        api.pd_norm_gate_residual_norm(y, x, eps=-1.0)


@pytest.mark.parametrize("cols", [1032, 2048, 4096, 4104, 8192])
@pytest.mark.parametrize("norms", [("rms", "rms"), ("layer", "layer"), ("none", "layer"), ("rms", "none"), ("none", "none")], ids=str)
def test_prefetched_rows(cols, norms):
    """bf16 streams of many rows: more rows than the persistent groups take in three turns, and not a multiple of them."""
    run(3 * 8 * 148 + 5 if cols <= 2048 else 3 * 4 * 148 + 7, cols, BF16, BF16, *norms, groups=1)
    run(2000, cols, BF16, BF16, *norms, groups=7, drop=("post_beta", "pre_gamma"))


def test_prefetched_rows_in_place():
    from paper_2511_03586_b200 import api
    x, y, gate, vec = make(4000, 4096, BF16, BF16, 4000)
    h, n = api.pd_norm_gate_residual_norm(y, x, gate=gate, post_norm="layer", **vec)
    x2, y2 = x.clone(), y.clone()
    api.pd_norm_gate_residual_norm(y2, x2, gate=gate, post_norm="layer", h=x2, n=y2, **vec)
    assert torch.equal(x2, h) and torch.equal(y2, n)
    for _ in range(3):
        again = api.pd_norm_gate_residual_norm(y, x, gate=gate, post_norm="layer", **vec)
        assert torch.equal(again[0], h) and torch.equal(again[1], n)
    assert api.pd_get_device_status() == 0


@pytest.mark.parametrize("cols", [2048, 4096, 8192])
def test_in_place_with_rows_prefetched(cols):
    """Rows are copied to shared memory while the one before is written over its own inputs: none may come out twice normed."""
    from paper_2511_03586_b200 import api
    rows = 4000
    x, y, gate, vec = make(rows, cols, BF16, BF16, rows)
    h, n = api.pd_norm_gate_residual_norm(y, x, gate=gate, **vec)
    for _ in range(3):
        x2, y2 = x.clone(), y.clone()
        api.pd_norm_gate_residual_norm(y2, x2, gate=gate, h=x2, n=y2, **vec)
        assert torch.equal(x2, h) and torch.equal(y2, n)
    assert api.pd_get_device_status() == 0
