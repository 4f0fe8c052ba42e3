"""Products with 4-bit weights against the definition in 64 bits."""
import pytest
import torch

from paper_2509_24257_b200 import binding as vb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _weights(n, k, group, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = (torch.randn(n, k, generator=g, device=DEV) * 0.02).to(torch.bfloat16)
    return w, vb.w4_quantise(w, group)


def _plain(w4):
    """What the weights stand for, in float64, from the stored form."""
    packed = w4.codes.to(torch.int64)
    w = torch.stack([packed & 15, packed >> 4], -1).reshape(w4.n, w4.k).double() - 8
    return w * w4.scales.double().repeat_interleave(w4.group, 0).T


def _bound(x, w, residual, y, dtype):
    """Every one of the k / 16 products of 16, of the k / group scaled sums and of at most 40 joins is rounded or cut to 24 bits of a
    running sum that is at most sum |x w|; the residual is added and the result rounded once more."""
    size = x.double().abs() @ w.abs().T
    steps = x.shape[1] / 16 + x.shape[1] / 32 + 40
    b = steps * 2.0 ** -23 * size + 2.0 ** -23 * (y.abs() + (residual.double().abs() if residual is not None else 0))
    return b * 1.01 + (2.0 ** -8 * y.abs() * 1.01 if dtype == torch.bfloat16 else 0) + 1e-37


def _check(x, w4, dtype=torch.float32, residual=None, **kw):
    got = vb.op_w4_matvec(x, w4, residual=residual, dtype=dtype, **kw)
    w = _plain(w4)
    want = x.double() @ w.T + (residual.double() if residual is not None else 0)
    assert got.dtype == dtype and got.shape == want.shape
    assert bool(((got.double() - want).abs() <= _bound(x, w, residual, want, dtype)).all())
    return got


def _x(rows, k, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(rows, k, generator=g, device=DEV).to(torch.bfloat16)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(8, 128), (16, 256), (24, 384), (40, 1024), (4096, 128), (1000, 2048), (136, 4096), (2056, 4224), (72, 8192), (264, 14336),
                                 (24, 28672), (16, 32768), (24, 33792), (136, 65664)])
def test_sizes(n, k, group):
    _, w4 = _weights(n, k, group)
    for rows in (1, 5, 8):
        _check(_x(rows, k), w4)


@pytest.mark.parametrize("n,k,group", [(8, 32, 32), (32, 96, 32), (64, 64, 64), (48, 192, 64), (64, 2080, 32), (64, 6464, 64), (5720, 32, 32)])
def test_inputs_that_fill_no_whole_chunk(n, k, group):
    _, w4 = _weights(n, k, group)
    _check(_x(3, k), w4)
    _check(_x(33, k), w4, torch.bfloat16)


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 130, 257])
def test_rows(rows):
    _, w4 = _weights(520, 1280, 128)
    _check(_x(rows, 1280), w4, torch.bfloat16)
    _check(_x(rows, 1280), w4, residual=torch.randn(rows, 520, device=DEV))
    _, w4 = _weights(136, 6400, 64)
    _check(_x(rows, 6400), w4)


@pytest.mark.parametrize("n,k,rows", [(28672, 4096, 1), (28672, 4096, 64), (4096, 14336, 5), (14336, 4096, 20)])
def test_large(n, k, rows):
    _, w4 = _weights(n, k, 128)
    _check(_x(rows, k), w4)


def test_strided_rows_and_outputs():
    _, w4 = _weights(520, 1280, 64)
    wide = _x(12, 1280 + 64)
    for rows in (3, 12):
        x = wide[:rows, 64:]
        out = torch.full((rows, 1000), 7.0, dtype=torch.bfloat16, device=DEV)
        vb.op_w4_matvec(x, w4, out=out[:, 3:523])
        assert torch.equal(out[:, 3:523], vb.op_w4_matvec(x.contiguous(), w4))
        assert bool((out[:, :3] == 7).all()) and bool((out[:, 523:] == 7).all())


@pytest.mark.parametrize("rows", [4, 40])
def test_residual_in_place_and_of_another_tensor(rows):
    _, w4 = _weights(264, 2048, 128)
    x, res = _x(rows, 2048), torch.randn(rows, 264, device=DEV)
    want = _check(x, w4, residual=res)
    inplace = res.clone()
    assert vb.op_w4_matvec(x, w4, residual=inplace, out=inplace) is inplace
    assert torch.equal(inplace, want)
    assert torch.equal(vb.op_w4_matvec(x, w4, residual=res, dtype=torch.bfloat16), want.to(torch.bfloat16))


@pytest.mark.parametrize("rows", [6, 24])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_row_that_is_not_finite_touches_no_other(rows, bad):
    _, w4 = _weights(136, 4352, 128)
    x = _x(rows, 4352)
    clean = vb.op_w4_matvec(x, w4, dtype=torch.float32)
    x[2, 77] = bad
    got = vb.op_w4_matvec(x, w4, dtype=torch.float32)
    keep = [r for r in range(rows) if r != 2]
    assert torch.equal(got[keep], clean[keep])
    assert not bool(torch.isfinite(got[2]).any())


def test_a_scale_that_is_nan_touches_its_output_only():
    w, w4 = _weights(136, 512, 128)
    clean = vb.op_w4_matvec(_x(3, 512), w4, dtype=torch.float32)
    w[5, 300] = float("inf")
    bad = vb.w4_quantise(w, 128)
    got = vb.op_w4_matvec(_x(3, 512), bad, dtype=torch.float32)
    keep = [i for i in range(136) if i != 5]
    assert torch.equal(got[:, keep], clean[:, keep]) and bool(torch.isnan(got[:, 5]).all())


@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantisation_is_the_definition(group):
    g = torch.Generator(device=DEV).manual_seed(3)
    w = (torch.randn(40, 512, generator=g, device=DEV) * torch.logspace(-30, 30, 40, device=DEV)[:, None]).to(torch.bfloat16)
    w[3] = 0
    w[4, :group] = 0
    w[5, 7] = float("nan")
    w[6, group] = -float("inf")
    w[7] = 3e-39  # scales below the normal range
    wide = torch.zeros(40, 1024, dtype=torch.bfloat16, device=DEV)
    wide[:, 512:] = w
    w4 = vb.w4_quantise(wide[:, 512:], group)
    a = w.float().reshape(40, -1, group)
    top = a.abs().amax(-1)
    scale = torch.where(torch.isfinite(top), top / 7, float("nan")).to(torch.bfloat16)
    assert torch.equal(torch.isnan(w4.scales.T), torch.isnan(scale))  # (a NaN has no bits of its own)
    assert torch.equal(w4.scales.T.nan_to_num(-1.0), scale.nan_to_num(-1.0))
    s = scale.double()
    codes = torch.where((s > 0).unsqueeze(-1), (a.double() / s.unsqueeze(-1)).round().clamp(-7, 7), 0.0)
    packed = w4.codes.long()
    got = torch.stack([packed & 15, packed >> 4], -1).reshape(40, -1, group) - 8
    assert torch.equal(got.double(), codes.nan_to_num(0.0))
    deq = vb.w4_dequantise(w4, torch.float32)
    ok = torch.isfinite(_plain(w4))
    assert torch.equal(deq[ok].double(), _plain(w4)[ok].float().double()) and bool(torch.isnan(deq[~ok]).all())
    assert torch.equal(vb.w4_dequantise(w4)[ok], _plain(w4)[ok].float().to(torch.bfloat16))
    out = torch.full((40, 520), 5.0, dtype=torch.bfloat16, device=DEV)
    vb.w4_dequantise(w4, out=out[:, :512])
    assert bool((out[:, 512:] == 5).all())


@pytest.mark.parametrize("rows", [3, 30])
def test_repeatable_captured_and_on_another_stream(rows):
    _, w4 = _weights(1032, 9216, 128)
    x = _x(rows, 9216)
    want = vb.op_w4_matvec(x, w4, dtype=torch.float32)
    for _ in range(20):
        assert torch.equal(vb.op_w4_matvec(x, w4, dtype=torch.float32), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = vb.op_w4_matvec(x, w4, dtype=torch.float32, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out, buf = torch.zeros_like(want), x.clone()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.op_w4_matvec(buf, w4, out=out, status=status)
    buf.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, vb.op_w4_matvec(x.flip(0).contiguous(), w4, dtype=torch.float32)) and int(status.item()) == 0


def test_two_calls_at_once():
    _, a = _weights(2056, 16384, 64)
    _, b = _weights(4096, 4096, 128)
    xa, xb = _x(8, 16384), _x(40, 4096)
    want = [vb.op_w4_matvec(xa, a), vb.op_w4_matvec(xb, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        outs[0].append(vb.op_w4_matvec(xa, a, stream=streams[0]))
        outs[1].append(vb.op_w4_matvec(xb, b, stream=streams[1]))
    torch.cuda.synchronize()
    for got, w in zip(outs, want):
        assert all(torch.equal(g, w) for g in got)


def test_no_rows_and_refusals():
    _, w4 = _weights(136, 512, 128)
    assert vb.op_w4_matvec(_x(1, 512)[:0], w4).shape == (0, 136)
    x = _x(2, 512)
    for bad in (x.float(), x[:, :256], x.T, x.cpu()):
        with pytest.raises(ValueError):
            vb.op_w4_matvec(bad, w4)
    with pytest.raises(ValueError):
        vb.op_w4_matvec(x, w4, residual=torch.zeros(2, 136, device=DEV, dtype=torch.bfloat16))
    with pytest.raises(vb.VerillmError):
        vb.op_w4_matvec(_x(2, 516)[:, 1:513], w4)  # rows not 16-byte aligned
    with pytest.raises(ValueError):
        vb.W4Weights(w4.codes, w4.scales, 64)
    with pytest.raises(ValueError):
        vb.w4_quantise(torch.zeros(8, 100, device=DEV, dtype=torch.bfloat16), 32)
    with pytest.raises(AttributeError):
        w4.codes = None
