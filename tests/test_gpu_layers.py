"""GPU: layer norm, its gradient and dropout against their definitions in float64, at the sizes, types, pitches and values where
they can go wrong.  Bounds come with the definitions (fit_reference)."""
import numpy as np
import pytest
import torch

import fit_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    import paper_2303_13803_amd as mm
    c = mm.Context(1, 1)
    yield c
    c.close()


def matrix(rng, rows, width, kind, pad=0, shift=0, scale=1.0, offset=0.0):
    """A device matrix of the type, `pad` values between rows and `shift` before the first; everything else is a marker."""
    whole = torch.full((rows * (width + pad) + shift + 16,), -77.0, dtype=TYPES[kind], device="cuda")
    view = whole[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width]
    view.copy_(torch.from_numpy(rng.normal(offset, scale, (rows, width))).to("cuda"))
    return whole, view


def host(t):
    return t.double().cpu().numpy()


def untouched(whole, view):
    """The markers around a matrix are as they were."""
    mark = torch.ones_like(whole, dtype=torch.bool)
    torch.as_strided(mark, view.shape, view.stride(), view.storage_offset()).fill_(False)
    assert bool((whole[mark] == -77.0).all())


# every way a row is laid over lanes, its edges, and rows shorter than a vector
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 251, 256, 257, 500, 513, 1024, 1025, 2048, 2049, 4096, 4100, 8191, 8192]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_norm_and_gradient_by_width(ctx, kind, width):
    rng = np.random.default_rng(width)
    rows = 67 if width < 2000 else 9
    pad, shift = width % 5, width % 3
    whole_x, x = matrix(rng, rows, width, kind, pad, shift, 2.0, 0.5)
    whole_y, y = matrix(rng, rows, width, kind, (pad + 1) % 4, shift)
    whole_dy, dy = matrix(rng, rows, width, kind, 0, (shift + 1) % 3, 0.1)
    w, b = (torch.from_numpy(rng.normal(1, 0.3, width)).float().cuda() for _ in range(2))
    ctx.layer_norm(x, w, b, y, eps=1e-5)
    value, bound = ref.norm_rows(host(x), host(w), host(b), 1e-5)[:2]
    ref.within(host(y), value, bound, "y", HALF_STEP[kind])
    untouched(whole_y, y)
    dw, db = torch.full((width,), 5.0, device="cuda"), torch.full((width,), 5.0, device="cuda")
    ctx.layer_norm_grad(x, dy, w, y, dw, db, eps=1e-5)
    dx, e_dx, dw64, e_dw, db64, e_db = ref.norm_grad_rows(host(x), host(dy), host(w), 1e-5)
    ref.within(host(y), dx, e_dx, "dx", HALF_STEP[kind])
    ref.within(host(dw), dw64, e_dw, "dw")
    ref.within(host(db), db64, e_db, "db")
    untouched(whole_y, y)
    untouched(whole_x, x)
    untouched(whole_dy, dy)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 63, 4095, 4097, 40001])
def test_norm_and_gradient_by_rows(ctx, kind, rows):
    rng = np.random.default_rng(rows)
    width = 40
    x, dy = matrix(rng, rows, width, kind, 0, 0, 1.0, 3.0)[1], matrix(rng, rows, width, kind, 3)[1]
    w, b = (torch.from_numpy(rng.normal(1, 0.3, width)).float().cuda() for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dw, db = torch.empty(width, device="cuda"), torch.empty(width, device="cuda")
    work = torch.full((ctx.layer_norm_grad_work(rows, width),), 255, dtype=torch.uint8, device="cuda")     # NaN in every word
    ctx.layer_norm(x, w, b, y)
    ctx.layer_norm_grad(x, dy, w, dx, dw, db, work=work)
    value, bound = ref.norm_rows(host(x), host(w), host(b), 1e-5)[:2]
    ref.within(host(y), value, bound, "y", HALF_STEP[kind])
    dx64, e_dx, dw64, e_dw, db64, e_db = ref.norm_grad_rows(host(x), host(dy), host(w), 1e-5)
    ref.within(host(dx), dx64, e_dx, "dx", HALF_STEP[kind])
    ref.within(host(dw), dw64, e_dw, "dw")
    ref.within(host(db), db64, e_db, "db")
    again = torch.empty(width, device="cuda")
    ctx.layer_norm_grad(x, dy, w, dx, again, db)
    assert torch.equal(again, dw)                       # the same bits
    # in place, over either input
    into = x.clone()
    ctx.layer_norm(into, w, b, into)
    assert torch.equal(into, y)
    for k in range(2):
        args = [x.clone(), dy.clone()]
        ctx.layer_norm_grad(args[0], args[1], w, args[k], again, db)
        assert torch.equal(args[k], dx)


@pytest.mark.parametrize("width", [64, 250, 1024, 5000])
def test_norm_in_place_by_width(ctx, width):
    rng = np.random.default_rng(width)
    x = matrix(rng, 300, width, "f16")[1]
    w, b = (torch.from_numpy(rng.normal(1, 0.3, width)).float().cuda() for _ in range(2))
    y = torch.empty_like(x)
    ctx.layer_norm(x, w, b, y)
    ctx.layer_norm(x, w, b, x)
    assert torch.equal(x, y)


def test_norm_of_no_rows(ctx):
    x = torch.empty((0, 12), device="cuda")
    w = torch.ones(12, device="cuda")
    ctx.layer_norm(x, w, w, x)
    dw, db = torch.full((12,), 3.0, device="cuda"), torch.full((12,), 3.0, device="cuda")
    ctx.layer_norm_grad(x, x, w, x, dw, db)
    assert dw.tolist() == db.tolist() == [0.0] * 12
    ctx.dropout(x, x, 0.5, 1)


@pytest.mark.parametrize("kind", TYPES)
def test_norm_of_unusual_rows(ctx, kind):
    """Rows without variance, far from zero, of the type's extremes, and with infinities and NaN, which stay in their row."""
    width = 48
    x = torch.zeros((7, width), dtype=TYPES[kind], device="cuda")
    x[1] = 3.0
    x[2] = torch.arange(width, device="cuda") % 2 + 1000                # a mean a thousand deviations away
    x[3] = torch.finfo(TYPES[kind]).tiny
    x[4, 5], x[5, 7], x[6, 9] = float("inf"), float("nan"), 1.0
    w, b = torch.full((width,), 1.5, device="cuda"), torch.full((width,), 0.25, device="cuda")
    y = torch.empty_like(x)
    ctx.layer_norm(x, w, b, y, eps=1e-5)
    got = host(y)
    finite = [0, 1, 2, 3, 6]
    value, bound = ref.norm_rows(host(x)[finite], host(w), host(b), 1e-5)[:2]
    ref.within(got[finite], value, bound, "y", HALF_STEP[kind])
    assert np.isnan(got[4]).all() and np.isnan(got[5]).all()


def test_norm_beyond_32_bits(ctx):
    """Offsets past 2^32 values: the last rows of a matrix of 5.4 billion values, rows far apart."""
    rows, width, pitch = 1310, 100, 1 << 22
    whole = torch.empty(rows * pitch, dtype=torch.float16, device="cuda")
    x = whole.view(rows, pitch)[:, :width]
    x.normal_()
    w = torch.ones(width, device="cuda")
    b = torch.zeros(width, device="cuda")
    close = x.contiguous()
    y = torch.empty_like(close)
    ctx.layer_norm(close, w, b, y)
    z = torch.empty_like(close)
    ctx.layer_norm(x, w, b, z)
    assert torch.equal(y, z)
    ctx.dropout(close, y, 0.3, 5)
    ctx.dropout(x, x, 0.3, 5)
    assert torch.equal(x, y)
    del whole


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows, width, pad", [(1, 1, 0), (1, 7, 0), (1, 8, 0), (3, 8, 0), (5, 3, 2), (67, 13, 0), (67, 13, 5), (64, 64, 0), (64, 64, 8), (301, 250, 1), (2, 8192, 3), (4001, 33, 0)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999])
def test_dropout(ctx, kind, rows, width, pad, p):
    rng = np.random.default_rng(rows * 1000 + width)
    whole_x, x = matrix(rng, rows, width, kind, pad, pad % 2)
    whole_y, y = matrix(rng, rows, width, kind, pad, 1)
    seed, step, layer = (1 << 63) + 12345, (1 << 40) + 9, 65535
    ctx.dropout(x, y, p, seed, step=step, layer=layer)
    keep = ref.kept(rows, width, p, seed, step, layer)
    # a product of two values of float32 and its rounding to the type
    ref.within(host(y), host(x) * keep, 2.0 ** -24 * np.abs(host(x) * keep), "y", HALF_STEP[kind])
    assert ((host(y) == 0) == (keep == 0)).all() or kind == "f16"      # (a small fp16 value may round to 0)
    untouched(whole_y, y)
    on_device = torch.tensor([step], dtype=torch.int64, device="cuda")
    z = torch.empty_like(y)
    ctx.dropout(x, z, p, seed, step=on_device, layer=layer)
    assert torch.equal(z, y)
    ctx.dropout(x, x, p, seed, step=step, layer=layer)
    assert torch.equal(x, y)
    untouched(whole_x, x)


def test_dropout_drops_what_is_not_a_number(ctx):
    x = torch.full((64, 64), float("nan"), device="cuda")
    x[::2] = float("-inf")
    y = torch.empty_like(x)
    ctx.dropout(x, y, 0.5, 3)
    keep = torch.from_numpy(ref.kept(64, 64, 0.5, 3, 0, 0) > 0).cuda()
    assert bool((y[~keep] == 0).all()) and bool(torch.isnan(y[1::2][keep[1::2]]).all()) and bool((y[::2][keep[::2]] == float("-inf")).all())


def test_layers_refuse_tensors_that_do_not_fit(ctx):
    x = torch.zeros((8, 16), device="cuda")
    w = torch.ones(16, device="cuda")
    for bad in (x.t(), x[:, ::2], x.expand(2, 8, 16), x.double(), x.cpu(), x[0]):
        with pytest.raises((TypeError, ValueError)):
            ctx.layer_norm(bad, w, w, bad)
    with pytest.raises(ValueError):
        ctx.layer_norm(x, w, w, x[:4])
    with pytest.raises(ValueError):
        ctx.layer_norm(x, w[:8], w, x)
    with pytest.raises(ValueError):
        ctx.layer_norm(x[:1].expand(8, 16), w, w, x)          # rows that overlap
    with pytest.raises(TypeError):
        ctx.layer_norm_grad(x, x, w, x, w.double(), w)
    with pytest.raises(TypeError):
        ctx.dropout(x, x, 0.5, 1, step=torch.zeros(1, device="cuda"))
    from paper_2303_13803_amd import MuxmatchError
    for call in (lambda: ctx.dropout(x, x, 1.0, 1), lambda: ctx.layer_norm(x, w, w, x, eps=0.0), lambda: ctx.dropout(x, x, 0.5, 1, layer=70000),
                 lambda: ctx.layer_norm_grad(x, x, w, x, w, w, work=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(MuxmatchError):
            call()


def test_layers_on_a_stream_and_in_a_graph(ctx):
    """A hidden layer forward and backward, captured on a stream of its own with the step on the device, replayed with eager work
    of torch in between; every replay against eager calls with that step."""
    import paper_2303_13803_amd as mm
    stream = torch.cuda.Stream()
    mine = mm.Context(1, 1, stream=stream)
    rows, width = 500, 70
    x, dy = torch.randn((rows, width), device="cuda"), torch.randn((rows, width), device="cuda")
    w, b, step = torch.rand(width, device="cuda"), torch.rand(width, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    outs = [torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)]
    work = torch.empty(mine.layer_norm_grad_work(rows, width), dtype=torch.uint8, device="cuda")

    def layer(c, step, o, scratch):
        c.layer_norm(x, w, b, o[0])
        c.dropout(o[0], o[0], 0.25, 42, step=step, layer=3)
        c.dropout(dy, o[1], 0.25, 42, step=step, layer=3)
        c.layer_norm_grad(x, o[1], w, o[1], o[2], o[3], work=scratch)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        layer(mine, step, outs, work)
    for k in range(4):
        step.fill_(k * (1 << 33) + 5)
        x.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        fresh = [torch.empty_like(o) for o in outs]
        layer(ctx, k * (1 << 33) + 5, fresh, None)
        for a, e in zip(outs, fresh):
            assert torch.equal(a, e), k
    mine.close()
