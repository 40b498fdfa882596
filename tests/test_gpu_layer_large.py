"""Arrays of more than 2^31 elements: rows and tokens at the start, in the middle and at the end get what they get in a call of their own."""
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


@pytest.fixture(autouse=True)
def memory(t):
    if t.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of the device")
    yield
    t.cuda.empty_cache()


def parts(rows, some):
    return [(a, a + some) for a in (0, rows // 2, rows - some)]


@pytest.mark.parametrize("rows,width", [(70000, 32760), (70000, 32761), (600000, 4100)])
def test_norm(t, qnn, rows, width):
    assert rows * width > 1 << 31
    x = t.empty((rows, width), dtype=t.bfloat16, device=DEV).normal_(generator=t.Generator(device=DEV).manual_seed(width))
    r, gain = x.flip(0), t.ones(width, dtype=t.bfloat16, device=DEV)
    rows8, y, h, rstd = qnn.rms_norm_i8(x, gain, 1e-6, r, both=True)
    dx, _ = qnn.rms_norm_backward(x, h, gain, rstd, y)
    decoded, other = qnn.i8_decode(rows8), qnn.i8_quantize(x)
    for a, b in parts(rows, 5):
        one, y1, h1, rstd1 = qnn.rms_norm_i8(x[a:b].clone(), gain, 1e-6, r[a:b].clone(), both=True)
        assert t.equal(one.codes, rows8.codes[a:b]) and t.equal(one.scales, rows8.scales[a:b])
        assert t.equal(y1, y[a:b]) and t.equal(h1, h[a:b]) and t.equal(rstd1, rstd[a:b])
        assert t.equal(qnn.rms_norm_backward(x[a:b].clone(), h1, gain, rstd1, y1)[0], dx[a:b])
        assert t.equal(qnn.i8_decode(one), decoded[a:b])
        again = qnn.i8_quantize(x[a:b].clone())
        assert t.equal(again.codes, other.codes[a:b]) and t.equal(again.scales, other.scales[a:b])


@pytest.mark.parametrize("rows,n,k", [(300000, 8200, 8200), (300001, 8195, 200)])
def test_gemm(t, qnn, rows, n, k):
    assert rows * n > 1 << 31
    g = t.Generator(device=DEV).manual_seed(k)
    x, w = (qnn.i8_quantize(t.empty((m, k), dtype=t.bfloat16, device=DEV).normal_(generator=g)) for m in (rows, n))
    y = qnn.i8_gemm(x, w)
    for a, b in parts(rows, 40):
        assert t.equal(qnn.i8_gemm(qnn.I8Rows(x.codes[a:b], x.scales[a:b].clone()), w), y[a:b])
    assert qnn.tensor_path_status() == 0


def test_route(t, qnn):
    tokens, experts, top = 9000000, 256, 8
    g = t.Generator(device=DEV).manual_seed(3)
    l, bias = t.empty((tokens, experts), dtype=t.bfloat16, device=DEV).normal_(generator=g), t.randn(experts, device=DEV, generator=g) * 0.05
    r = qnn.route(l, top, "softmax", bias)
    d = qnn.route_backward(r.weights, l, r.experts, "softmax", False)
    for a, b in parts(tokens, 100):
        one = qnn.route(l[a:b].clone(), top, "softmax", bias)
        assert t.equal(one.experts, r.experts[a:b]) and t.equal(one.weights, r.weights[a:b])
        assert t.equal(qnn.route_backward(one.weights, l[a:b].clone(), one.experts, "softmax", False), d[a:b])
    flat = r.experts.reshape(-1).long()
    assert t.equal(r.offsets[1:].long(), t.bincount(flat, minlength=experts).cumsum(0)) and r.offsets[0].item() == 0
    assert t.equal(r.order[r.place.reshape(-1).long()], t.arange(flat.numel(), device=DEV, dtype=t.int32))
    expert = flat[r.order.long()]
    same = expert[1:] == expert[:-1]
    assert bool((expert[1:] >= expert[:-1]).all()) and bool((r.order[1:][same] > r.order[:-1][same]).all())
