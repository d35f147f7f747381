"""Rows to 8 bits and 8-bit products on the device against plain implementations in 64 bits."""
import numpy as np
import pytest

from paper_2408_08146_amd import KoalaError, QuantizedLinear, quantize_rows, quantize_weight

pytestmark = pytest.mark.gpu


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def rounded(x, bf16):
    import torch
    t = torch.from_numpy(np.asarray(x, np.float32))
    return t.to(torch.bfloat16).float().numpy() if bf16 else t.numpy()


def agrees(got, want, tol, f32):
    """fp32: within tol of the 64-bit value; bfloat16: a rounding of some number within tol of it (rounding keeps order)."""
    got = got.double().cpu().numpy()
    lo, hi = (want - tol, want + tol) if f32 else (rounded(want - tol, True).astype(np.float64), rounded(want + tol, True).astype(np.float64))
    return ((lo <= got) & (got <= hi)).all()


def quantized(x, form="plain", gain=None, eps=1e-6, bf16=False, pad=0, extra=0):
    """x (float32 numpy) through the device: int8 rows, scales and the bytes behind the rows."""
    import torch
    rows, cols = x.shape[0], x.shape[1] // (2 if form == "swiglu" else 1)
    wide = torch.full((rows, (x.shape[1] + 7) // 8 * 8 + pad), float("nan"), device="cuda").to(torch.bfloat16 if bf16 else torch.float32)
    wide[:, :x.shape[1]] = dev(x).to(wide.dtype)
    q = torch.full((rows, (cols + 15) // 16 * 16 + extra), 99, dtype=torch.int8, device="cuda")
    s = torch.empty(rows, device="cuda")
    quantize_rows(wide[:, :x.shape[1]], q, s, form=form, gain=gain, eps=eps)
    return q.cpu().numpy()[:, :cols], s.cpu().numpy(), q.cpu().numpy()[:, cols:]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 15), (2, 16), (65, 17), (3, 100), (26, 4096), (2, 8200), (1, 17920), (2, 33001), (3, 70016), (3, 4099), (2, 20001)])
def test_plain_rows_are_rounded_as_defined(bf16, rows, cols):
    rng = np.random.default_rng(cols)
    x = rounded(rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, 1))), bf16)
    q, s, behind = quantized(x, bf16=bf16, pad=8 * (cols % 3), extra=16)
    want_s = (np.abs(x).max(1) / np.float32(127)).astype(np.float32)
    assert (s == want_s).all()
    assert (q == np.rint(x / want_s[:, None])).all()
    pad = (cols + 15) // 16 * 16 - cols
    assert not behind[:, :pad].any() and (behind[:, pad:] == 99).all()


def silu(x):
    return x / (1 + np.exp(-x))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("form", ["norm", "swiglu"])
@pytest.mark.parametrize("rows,cols", [(1, 7), (3, 64), (26, 4096), (2, 13824), (2, 40007), (3, 1001), (2, 20001)])
def test_normed_and_gated_rows(bf16, form, rows, cols):
    """A value rounds to within half a step of the scale; the value itself and the scale are fp32: the sum of squares of n terms is
    within (n / 1024 + 20) 2^-24 (n terms over at least 64 threads, joined in a tree), everything else a few roundings."""
    rng = np.random.default_rng(cols + rows)
    width = 2 * cols if form == "swiglu" else cols
    x = rounded(rng.standard_normal((rows, width)) * 3, bf16)
    gain = rounded(1 + 0.2 * rng.standard_normal(cols), cols % 2)
    x64 = x.astype(np.float64)
    if form == "norm":
        import torch
        v = x64 / np.sqrt((x64 ** 2).mean(1, keepdims=True) + 1e-5) * gain
        g = dev(gain, torch.bfloat16 if cols % 2 else torch.float32)
    else:
        v, g = silu(x64[:, 0::2]) * x64[:, 1::2], None
    q, s, _ = quantized(x, form=form, gain=g, eps=1e-5, bf16=bf16)
    rel = (cols / 64 + 20) * 2.0 ** -24
    top = np.abs(v).max(1)
    assert (np.abs(s - top / 127) <= rel * top / 127).all()
    assert (np.abs(q * s[:, None].astype(np.float64) - v) <= s[:, None] * 0.5 + 2 * rel * np.abs(v) + 1e-30).all()
    assert (np.abs(q).max(1) == 127).all()


def test_rows_of_zeros_tiny_values_and_values_that_are_not_finite():
    x = np.zeros((7, 40), np.float32)
    x[1, 3], x[2, 39], x[3, 0] = np.inf, np.nan, -np.inf
    x[4] = 1e-45
    x[5, 1], x[6, 2] = 1e-38, 3e38
    q, s, _ = quantized(x)
    assert s[0] == 1 and not q[0].any()
    assert np.isnan(s[1:4]).all() and not q[1:4].any()
    assert s[4] > 0 and np.abs(q[4].astype(np.int32)).max() <= 127
    assert s[5] > 0 and q[5, 1] in (126, 127, -127) and q[6, 2] == 127 and np.isfinite(s[6])


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 64, 65, 130, 300])
@pytest.mark.parametrize("out,cols", [(1, 16), (5, 48), (16, 64), (33, 80), (100, 1040), (257, 4096), (520, 128)])
def test_products(f32, rows, out, cols):
    """Sums are exact; the result rounds three times (sum to fp32, two scales), four with an addend, and once to bfloat16."""
    import torch
    rng = np.random.default_rng(rows * out + cols)
    q, w = (rng.integers(-128, 128, (n, cols), dtype=np.int8) for n in (rows, out))
    qs, ws = (np.exp(rng.standard_normal(n)).astype(np.float32) * 0.01 for n in (rows, out))
    dt = torch.float32 if f32 else torch.bfloat16
    y = torch.full((rows, out), 7.0, dtype=dt, device="cuda")
    lin = QuantizedLinear(dev(w), dev(ws))
    lin.forward(dev(q), dev(qs), y)
    want = (q.astype(np.float64) @ w.astype(np.float64).T) * qs.astype(np.float64)[:, None] * ws.astype(np.float64)
    assert agrees(y, want, 4 * 2.0 ** -24 * np.abs(want), f32)
    # a residual stream updated in place, rows inside wider ones on every side
    add = rounded(rng.standard_normal((rows, out)), not f32)
    wide = torch.full((rows, out + 13), 5.0, dtype=dt, device="cuda")
    wide[:, 3:3 + out] = dev(add).to(dt)
    qw = torch.full((rows, cols + 32), 77, dtype=torch.int8, device="cuda")
    qw[:, :cols] = dev(q)
    ww = torch.full((out, cols + 16), 77, dtype=torch.int8, device="cuda")
    ww[:, :cols] = dev(w)
    view = wide[:, 3:3 + out]
    QuantizedLinear(ww[:, :cols], dev(ws)).forward(qw, dev(qs), view, add=view)
    both = want + add
    assert agrees(view, both, 4 * 2.0 ** -24 * (np.abs(want) + np.abs(add)), f32)
    assert (wide[:, :3] == 5).all() and (wide[:, 3 + out:] == 5).all()


@pytest.mark.parametrize("rows", [1, 20, 40, 60])
@pytest.mark.parametrize("out", [6650, 11003, 16000, 22001, 32000])
def test_products_of_many_channels(rows, out):
    """Two to eight groups of 16 channels a workgroup, one to four tiles of rows, a last run that ends early, rows among wider ones."""
    import torch
    rng = np.random.default_rng(rows + out)
    q, w = (dev(rng.integers(-128, 128, (n, 2832 + 16), dtype=np.int8)) for n in (rows, out))
    q, w = q[:, :2832], w[:, :2832]
    qs, ws = (np.exp(rng.standard_normal(n)).astype(np.float32) * 0.01 for n in (rows, out))
    want = ((q.double() @ w.double().T) * dev(qs).double()[:, None] * dev(ws).double()).cpu().numpy()   # the sums are exact
    y = torch.full((rows, out), 7.0, device="cuda")
    QuantizedLinear(w, dev(ws)).forward(q, dev(qs), y)
    assert agrees(y, want, 4 * 2.0 ** -24 * np.abs(want), True)


@pytest.mark.parametrize("rows,out,cols", [(2047, 8001, 4144), (1999, 4095, 11056), (700, 6650, 12304), (1023, 3999, 9040), (2000, 8192, 1088),
                                           (160, 9001, 6672), (289, 6145, 11040), (1499, 6650, 6672), (217, 12289, 17936), (899, 5501, 4112)])
def test_products_of_many_rows(rows, out, cols):
    """Tiles of 128 to 256 rows, one to seven parts of the sums, an odd number of steps and ends inside of them; whatever stands behind a
    row's end takes no part."""
    import torch
    rng = np.random.default_rng(rows)
    q, w = (rng.integers(-128, 128, (n, cols + 16), dtype=np.int8) for n in (rows, out))
    q[:, :16] = w[:, :16] = -128
    qs, ws = (np.exp(rng.standard_normal(n)).astype(np.float32) * 0.01 for n in (rows, out))
    q, w = dev(q)[:, :cols], dev(w)[:, :cols]
    want = ((q.double() @ w.double().T) * dev(qs).double()[:, None] * dev(ws).double()).cpu().numpy()   # the sums are exact
    y = torch.full((rows, out), 7.0, device="cuda")
    lin = QuantizedLinear(w, dev(ws))
    lin.forward(q, dev(qs), y)
    assert agrees(y, want, 4 * 2.0 ** -24 * np.abs(want), True)
    z = torch.full((rows, out), 3.0, dtype=torch.bfloat16, device="cuda")
    lin.forward(q, dev(qs), z, add=z)
    assert agrees(z, want + 3.0, 4 * 2.0 ** -24 * (np.abs(want) + 3.0), False)


def test_the_longest_sum_of_the_largest_products_fits():
    import torch
    q = torch.full((3, 131056), -128, dtype=torch.int8, device="cuda")
    w = torch.full((18, 131056), -128, dtype=torch.int8, device="cuda")
    y = torch.empty(3, 18, device="cuda")
    one = lambda n: torch.ones(n, device="cuda")
    QuantizedLinear(w, one(18)).forward(q, one(3), y)
    assert (y == float(131056 * 16384)).all()


def test_weights_to_8_bits():
    import torch
    w = torch.randn(40, 64, device="cuda").bfloat16()
    w[3] = 0
    q, s = quantize_weight(w)
    assert q.dtype == torch.int8 and not q[3].any() and s[3] == 1
    assert ((q.float() * s[:, None] - w.float()).abs() <= s[:, None] * 0.50001).all() and (q[:3].abs().amax(1) == 127).all()


def test_a_layer_of_products_captured_in_a_graph_replays():
    import torch
    w = torch.randint(-127, 128, (700, 512), dtype=torch.int8, device="cuda")
    lin = QuantizedLinear(w, torch.rand(700, device="cuda"))
    x = torch.randn(40, 512, device="cuda")
    q, s = torch.empty(40, 512, dtype=torch.int8, device="cuda"), torch.empty(40, device="cuda")
    y, e = torch.empty(2, 40, 700, device="cuda")

    def step(out):
        quantize_rows(x, q, s)
        lin.forward(q, s, out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(y)
    for _ in range(4):
        x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        step(e)
        assert torch.equal(got, e)


def status(call):
    try:
        call()
    except KoalaError as e:
        return e.status
    return 0


def test_what_is_refused():
    import torch
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    i8 = torch.int8
    SHAPE, ALIGN, UNSUP = -2, -3, -5
    quant = lambda *a, **o: status(lambda: quantize_rows(*a, **o))
    assert quant(z(2, 32), z(2, 32, dt=i8), z(2)) == 0
    assert quant(z(2, 32, dt=torch.float16), z(2, 32, dt=i8), z(2)) == UNSUP and quant(z(2, 32), z(2, 32), z(2)) == UNSUP
    assert quant(z(2, 32), z(2, 32, dt=i8), z(3)) == SHAPE and quant(z(2, 32), z(3, 32, dt=i8), z(2)) == SHAPE
    assert quant(z(2, 24), z(2, 24, dt=i8), z(2)) == SHAPE                          # no room for the row's last bytes
    assert quant(z(2, 33, dt=torch.bfloat16)[:, :32], z(2, 32, dt=i8), z(2)) == ALIGN
    assert quant(z(2, 31), z(2, 32, dt=i8), z(2), form="swiglu") == SHAPE and quant(z(2, 32), z(2, 32, dt=i8), z(2), form="other") == UNSUP
    assert quant(z(2, 32), z(2, 32, dt=i8), z(2), form="norm") == -1
    assert quant(z(2, 32), z(2, 32, dt=i8), z(2), form="norm", gain=z(31)) == SHAPE
    assert quant(z(2, 32), z(2, 32, dt=i8), z(2), form="norm", gain=z(32), eps=-1.0) == SHAPE
    lin = QuantizedLinear(z(5, 32, dt=i8), z(5))
    fwd = lambda *a, **o: status(lambda: lin.forward(*a, **o))
    assert fwd(z(2, 32, dt=i8), z(2), z(2, 5)) == 0
    assert fwd(z(2, 16, dt=i8), z(2), z(2, 5)) == SHAPE and fwd(z(2, 32, dt=i8), z(2), z(2, 6)) == SHAPE
    assert fwd(z(2, 32, dt=i8), z(3), z(2, 5)) == SHAPE and fwd(z(2, 32, dt=i8), z(2), z(2, 5, dt=torch.float16)) == UNSUP
    assert fwd(z(2, 32), z(2), z(2, 5)) == UNSUP and fwd(z(2, 32, dt=i8), z(2), z(2, 5), add=z(2, 5, dt=torch.bfloat16)) == SHAPE
    assert fwd(z(2, 33, dt=i8)[:, 1:], z(2), z(2, 5)) == ALIGN
    assert fwd(z(2, 32, dt=i8), z(2), z(5, 2).t()) == SHAPE
    assert status(lambda: QuantizedLinear(z(5, 24, dt=i8), z(5)).forward(z(2, 32, dt=i8), z(2), z(2, 5))) == SHAPE
    assert status(lambda: QuantizedLinear(z(1, 131072, dt=i8), z(1)).forward(z(2, 131072, dt=i8), z(2), z(2, 1))) == SHAPE
    assert status(lambda: QuantizedLinear(z(5, 32), z(5))) == UNSUP and status(lambda: QuantizedLinear(z(5, 32, dt=i8), z(4))) == SHAPE
