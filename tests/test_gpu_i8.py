"""dropmatch_quantize_i8, dropmatch_matmul_i8 and dropmatch_linear_i8 against plain 64-bit statements (engine_ref.py)."""
import pytest
import torch

import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding
import engine_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    c = pk.Context(0)
    yield c
    assert c.device_error() == 0
    c.close()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def integers(rows, d, seed, more=0):
    """int8 [rows, d], every value allowed, in rows of a multiple of 16 bytes; the bytes between them would spoil a sum."""
    ld = (d + 15) // 16 * 16 + 16 * more
    store = torch.randint(-128, 128, (rows, ld), generator=gen(seed), device=DEV, dtype=torch.int8)
    return store[:, :d]


def product(q, q_scale, W, w_scale):
    """The definition in 64 bits."""
    return (q.double() @ W.double().T) * w_scale.double()[None] * q_scale.double()[:, None]


def close(got, want):
    """The conversion of the sum, two products, one rounding: (3 u + half a step) relative, 2^-126 for what underflows."""
    tol = want.abs() * (3 * ref.U + ref.half_step(got.dtype) * (1 + 2.0 ** -6)) + 2.0 ** -126
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 15), (5, 16), (9, 17), (2, 512), (70, 1000), (1, 1024), (4, 1025), (3, 4096), (1, 8191), (2, 40001), (700, 64)])
@pytest.mark.parametrize("more,offset", [(0, 0), (1, 1), (8, 8)])
def test_quantize(ctx, rows, n, dtype, more, offset):
    buf = torch.full((offset + rows * (n + more),), float("nan"), dtype=DT[dtype], device=DEV)
    x = buf[offset:].view(rows, n + more)[:, :n]
    x.copy_(torch.randn((rows, n), generator=gen(n), device=DEV) * 3)
    q, scale = ctx.quantize_i8(x)
    want, want_scale = ref.quantize(x)
    assert torch.equal(q.double(), want) and torch.equal(scale.double(), want_scale)
    assert q.stride(0) % 16 == 0 or rows == 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_special_rows(ctx, dtype):
    top = torch.finfo(DT[dtype]).max
    for n in (40, 2000):
        x = torch.randn((12, n), generator=gen(n), device=DEV).to(DT[dtype])
        x[0] = 0
        x[1] = torch.finfo(DT[dtype]).tiny                      # scale at its least value
        x[2, 0], x[2, 1] = top, -top
        x[3] *= 1e-38
        x[4, n - 1] = float("nan")
        x[5, 3] = float("inf")
        x[6, 0] = float("-inf")
        x[7] = torch.arange(n, device=DEV) % 255 - 127.0        # whole numbers
        x[8] = (torch.arange(n, device=DEV) % 254 - 127 + 0.5)  # halves
        x[8, 0] = 127.0
        q, scale = ctx.quantize_i8(x)
        want, want_scale = ref.quantize(x)
        assert torch.equal(q.double(), want)
        assert torch.equal(scale.double().nan_to_num(-1.0), want_scale.nan_to_num(-1.0))


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,d", [(1, 1, 1), (1, 128, 128), (2, 129, 16), (3, 5, 17), (31, 127, 200), (32, 256, 128), (33, 300, 4096), (64, 1000, 1000),
                                      (65, 257, 33), (127, 511, 640), (128, 128, 256), (129, 128, 256), (130, 129, 100), (256, 700, 512), (257, 1001, 384),
                                      (300, 40, 96), (513, 640, 1024), (1000, 333, 127)])
def test_matmul(ctx, rows, V, d, out):
    for more in (0, 3):
        q, W = integers(rows, d, 1, more), integers(V, d, 2, 2 * more)
        q_scale = torch.rand((rows,), generator=gen(3), device=DEV) + 0.01
        w_scale = torch.rand((V,), generator=gen(4), device=DEV) + 0.01
        close(ctx.matmul_i8(q, q_scale, W, w_scale, dtype=DT[out]), product(q, q_scale, W, w_scale))


@pytest.mark.parametrize("rows,V,d", [(1, 128256, 4096), (61, 32003, 4096), (129, 40000, 2048), (700, 20011, 1536)])
def test_matmul_over_many_tiles(ctx, rows, V, d):
    q, W = integers(rows, d, 5), integers(V, d, 6)
    one, w_scale = torch.ones((rows,), device=DEV), torch.ones((V,), device=DEV)
    close(ctx.matmul_i8(q, one, W, w_scale), product(q, one, W, w_scale))
    close(ctx.matmul_i8(q, one, W, w_scale, dtype=torch.bfloat16), product(q, one, W, w_scale))


def test_matmul_extreme_sums(ctx):
    """The longest sums of the largest products: past 2^30 and exact."""
    d = 131071
    q, W = torch.full((3, d + 1), -128, dtype=torch.int8, device=DEV)[:, :d], torch.full((130, d + 1), -128, dtype=torch.int8, device=DEV)[:, :d]
    W[::2] = 127
    one, w_scale = torch.ones((3,), device=DEV), torch.ones((130,), device=DEV)
    got = ctx.matmul_i8(q, one, W, w_scale)
    assert torch.equal(got, product(q, one, W, w_scale).float())


def test_scales_that_underflow_overflow_or_are_no_numbers(ctx):
    q, W = integers(4, 256, 7), integers(200, 256, 8)
    q_scale = torch.tensor([1e-30, 1e30, float("nan"), 0.0], device=DEV)
    w_scale = torch.full((200,), 1e-20, device=DEV)
    w_scale[::3] = 1e30
    got, want = ctx.matmul_i8(q, q_scale, W, w_scale), product(q, q_scale, W, w_scale)
    assert bool(torch.isnan(got[2]).all()) and bool((got[3] == 0).all())
    close(got[0], want[0])
    inf = want[1].abs() > torch.finfo(torch.float32).max
    assert torch.equal(torch.isinf(got[1]), inf)
    close(got[1][~inf], want[1][~inf])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,V,d", [((1,), 1000, 4096), ((2, 3), 517, 100), ((61,), 4096, 256), ((5, 40), 300, 8192), ((3, 1, 100), 2049, 777)])
def test_linear(ctx, shape, V, d, dtype):
    x = torch.randn((*shape, d), generator=gen(d), device=DEV).to(DT[dtype])
    W, w_scale = ctx.quantize_i8(torch.randn((V, d), generator=gen(V), device=DEV) * 0.02)
    q, q_scale = ref.quantize(x.reshape(-1, d))
    want = product(q, q_scale, W, w_scale).view(*shape, V)
    got = ctx.linear_i8(x, W, w_scale)
    assert got.dtype == x.dtype and got.shape == want.shape
    close(got, want)
    close(ctx.linear_i8(x, W, w_scale, dtype=torch.float32), want)
    assert torch.equal(ctx.matmul_i8(*ctx.quantize_i8(x), W, w_scale), ctx.linear_i8(x, W, w_scale, dtype=torch.float32))
    # against the unquantised product: each factor is off by half a step of its scale at most
    exact = x.double().reshape(-1, d) @ (W.double() * w_scale.double()[:, None]).T
    bound = 0.5 * q_scale[:, None] * (W.double().abs().sum(1) * w_scale.double())[None]
    assert bool(((want.reshape(-1, V) - exact).abs() <= bound * (1 + 1e-6)).all())


def test_rows_do_not_depend_on_the_others(ctx):
    x = torch.randn((400, 512), generator=gen(1), device=DEV)
    W, w_scale = ctx.quantize_i8(torch.randn((1000, 512), generator=gen(2), device=DEV))
    whole = ctx.linear_i8(x, W, w_scale)
    for a, b in ((0, 1), (5, 40), (100, 300), (399, 400)):
        assert torch.equal(ctx.linear_i8(x[a:b], W, w_scale), whole[a:b])


def test_a_row_that_is_no_number_stays_alone(ctx):
    x = torch.randn((5, 300), generator=gen(1), device=DEV)
    x[2, 7] = float("nan")
    W, w_scale = ctx.quantize_i8(torch.randn((600, 300), generator=gen(2), device=DEV))
    got = ctx.linear_i8(x, W, w_scale)
    assert bool(torch.isnan(got[2]).all()) and not bool(torch.isnan(got[[0, 1, 3, 4]]).any())


def test_strided_output_and_what_lies_between(ctx):
    """Through the C entry point: columns past V and rows behind the last stay as they are."""
    for rows, V, d in ((3, 100, 64), (140, 333, 200)):
        q, W = integers(rows, d, 1), integers(V, d, 2)
        one, w_scale = torch.ones((rows,), device=DEV), torch.ones((V,), device=DEV)
        for dtype, code in ((torch.float32, binding.F32), (torch.bfloat16, binding.BF16)):
            ld = V + 5
            buf = torch.full((3 + (rows + 2) * ld,), 9.0, dtype=dtype, device=DEV)
            out = buf[3:].view(rows + 2, ld)
            st = binding.lib().dropmatch_matmul_i8(ctx._h, q.data_ptr(), q.stride(0), one.data_ptr(), rows, W.data_ptr(), W.stride(0), w_scale.data_ptr(),
                                                   V, d, out.data_ptr(), code, ld, None)
            assert st == binding.OK
            torch.cuda.synchronize()
            close(out[:rows, :V], product(q, one, W, w_scale))
            out[:rows, :V] = 9.0
            assert bool((buf == 9.0).all())


def test_streams_graph_and_two_calls_at_once(ctx):
    x, y = torch.randn((50, 1024), generator=gen(1), device=DEV), torch.randn((200, 512), generator=gen(2), device=DEV).bfloat16()
    W, w_scale = ctx.quantize_i8(torch.randn((9000, 1024), generator=gen(3), device=DEV))
    U, u_scale = ctx.quantize_i8(torch.randn((5000, 512), generator=gen(4), device=DEV))
    want_x, want_y = ctx.linear_i8(x, W, w_scale), ctx.linear_i8(y, U, u_scale)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(s1):
            got_x = ctx.linear_i8(x, W, w_scale)
        with torch.cuda.stream(s2):
            got_y = ctx.linear_i8(y, U, u_scale)
    torch.cuda.synchronize()
    assert torch.equal(got_x, want_x) and torch.equal(got_y, want_y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        V, v_scale = ctx.quantize_i8(W.float() * w_scale[:, None])          # W written right ahead of the product
        captured = ctx.linear_i8(x, V, v_scale)
    x2 = torch.randn_like(x)
    x.copy_(x2)
    W.copy_(torch.randint(-127, 128, W.shape, device=DEV, dtype=torch.int8))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(captured, ctx.linear_i8(x2, *ctx.quantize_i8(W.float() * w_scale[:, None])))


def test_output_rows_far_apart(ctx):
    """Offsets past 2^31 entries of the output."""
    ld, V, d = 1 << 30, 200, 64
    q, W = integers(4, d, 1), integers(V, d, 2)
    one, w_scale = torch.ones((4,), device=DEV), torch.ones((V,), device=DEV)
    buf = torch.empty(3 * ld + V, dtype=torch.bfloat16, device=DEV)
    st = binding.lib().dropmatch_matmul_i8(ctx._h, q.data_ptr(), q.stride(0), one.data_ptr(), 4, W.data_ptr(), W.stride(0), w_scale.data_ptr(), V, d,
                                           buf.data_ptr(), binding.BF16, ld, None)
    assert st == binding.OK
    close(buf.as_strided((4, V), (ld, 1)), product(q, one, W, w_scale))


def test_nothing_to_do(ctx):
    W, w_scale = ctx.quantize_i8(torch.randn((10, 32), device=DEV))
    assert ctx.linear_i8(torch.empty((0, 32), device=DEV), W, w_scale).shape == (0, 10)
    q, scale = ctx.quantize_i8(torch.empty((0, 32), device=DEV))
    assert q.shape == (0, 32) and scale.shape == (0,)


def test_waits_that_run_out_leave_nan(ctx):
    """A limit of one cycle: whichever wait is not satisfied at once gives up; the call ends, says so, and what it did not
    compute is NaN."""
    c = pk.Context(0)
    W, w_scale = integers(40000, 2048, 1), torch.ones((40000,), device=DEV)
    for rows in (3, 200):
        q, one = integers(rows, 2048, 2), torch.ones((rows,), device=DEV)
        want = product(q, one, W, w_scale)
        c.debug_set_wait_limit(1)
        got = c.matmul_i8(q, one, W, w_scale)
        assert c.device_error() != 0
        wrong = torch.isnan(got)
        assert bool(wrong.any())
        close(got[~wrong], want[~wrong])
        c.debug_set_wait_limit(0)
        close(c.matmul_i8(q, one, W, w_scale), want)
        assert c.device_error() == 0
    c.close()


def test_refusals(ctx):
    L = binding.lib()
    x, q, scale = torch.zeros((4, 64), device=DEV), torch.zeros((4, 64), dtype=torch.int8, device=DEV), torch.zeros(4, device=DEV)

    def quantize(**kw):
        v = dict(h=ctx._h, x=x.data_ptr(), dtype=binding.F32, ld=64, rows=4, n=64, q=q.data_ptr(), ldq=64, scale=scale.data_ptr(), s=None)
        v.update(kw)
        return L.dropmatch_quantize_i8(*v.values())

    assert quantize() == binding.OK
    for bad in (dict(h=None), dict(x=None), dict(x=x.data_ptr() + 1), dict(dtype=2), dict(ld=63), dict(rows=-1), dict(n=0), dict(q=None),
                dict(q=q.data_ptr() + 8), dict(ldq=48), dict(ldq=72), dict(scale=None), dict(scale=scale.data_ptr() + 2), dict(q=x.data_ptr())):
        assert quantize(**bad) == binding.EINVAL, bad
    assert quantize(n=2 ** 30 + 1, ld=2 ** 31, ldq=2 ** 31) == binding.EUNSUPPORTED
    assert quantize(rows=0, x=None, q=None, scale=None) == binding.OK

    W, w_scale, out = torch.zeros((100, 64), dtype=torch.int8, device=DEV), torch.zeros(100, device=DEV), torch.zeros((4, 100), device=DEV)

    def matmul(**kw):
        v = dict(h=ctx._h, a=q.data_ptr(), lda=64, a_scale=scale.data_ptr(), rows=4, w=W.data_ptr(), ldw=64, w_scale=w_scale.data_ptr(), V=100, d=64,
                 out=out.data_ptr(), dtype=binding.F32, ldo=100, s=None)
        v.update(kw)
        return L.dropmatch_matmul_i8(*v.values())

    def linear(**kw):
        v = dict(h=ctx._h, x=x.data_ptr(), xdtype=binding.F32, ldx=64, rows=4, w=W.data_ptr(), ldw=64, w_scale=w_scale.data_ptr(), V=100, d=64,
                 q=q.data_ptr(), ldq=64, q_scale=scale.data_ptr(), out=out.data_ptr(), dtype=binding.F32, ldo=100, s=None)
        v.update(kw)
        return L.dropmatch_linear_i8(*v.values())

    both = [dict(h=None), dict(rows=-1), dict(w=None), dict(w=W.data_ptr() + 1), dict(ldw=63), dict(ldw=72), dict(w_scale=None), dict(V=0), dict(d=0),
            dict(out=None), dict(out=out.data_ptr() + 2), dict(dtype=5), dict(ldo=99), dict(out=W.data_ptr())]
    for fn, more in ((matmul, [dict(a=None), dict(a=q.data_ptr() + 4), dict(lda=48), dict(lda=65), dict(a_scale=None), dict(out=q.data_ptr())]),
                     (linear, [dict(x=None), dict(x=x.data_ptr() + 3), dict(xdtype=-1), dict(ldx=60), dict(q=None), dict(q=q.data_ptr() + 1), dict(ldq=32),
                               dict(q_scale=None), dict(q=out.data_ptr()), dict(q=W.data_ptr()), dict(q=x.data_ptr())])):
        assert fn() == binding.OK
        for bad in both + more:
            assert fn(**bad) == binding.EINVAL, bad
        assert fn(V=2 ** 30 + 1, ldo=2 ** 31) == binding.EUNSUPPORTED
        assert fn(d=131072, ldw=2 ** 20, **({"lda": 2 ** 20} if fn is matmul else {"ldq": 2 ** 20, "ldx": 2 ** 20})) == binding.EUNSUPPORTED
        assert fn(rows=0, out=None, w=None) == binding.OK
    torch.cuda.synchronize()
    odd = torch.zeros((100, 72), dtype=torch.int8, device=DEV)
    for args in ((x.half(), W, w_scale), (x.cpu(), W, w_scale), (x, W.float(), w_scale), (x, W[:, :32], w_scale), (x, odd, w_scale),
                 (x, W, w_scale[:50]), (x, W, w_scale.double()), (torch.zeros((4, 72), device=DEV), odd, w_scale), (x, W.t(), w_scale)):
        with pytest.raises(TypeError):
            ctx.linear_i8(*args)
    with pytest.raises(TypeError):
        ctx.linear_i8(x, W, w_scale, dtype=torch.float16)
    with pytest.raises(TypeError):
        ctx.matmul_i8(q, scale[:3], W, w_scale)
    with pytest.raises(TypeError):
        ctx.matmul_i8(q.float(), scale, W, w_scale)
    with pytest.raises(TypeError):
        ctx.quantize_i8(x.double())
