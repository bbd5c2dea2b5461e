"""The operators that produce gradients (``include/lionmuon_grad.h``) on the GPU,
against float64 references.

Tolerances. A result in a 16-bit type is off by at most half a step, eps/2 of
its value, plus what fp32 arithmetic adds before it is rounded; that part is
bounded by a count of roundings (2^-24 each, 2^-23 where the matrix unit
truncates) times the sum of the magnitudes that enter.
"""
import numpy as np
import pytest
import torch

import grad_reference as ref
from paper_2605_19811_amd import gradients as gr
from paper_2605_19811_amd import lionmuon as lm

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def half_step(dt):
    return torch.finfo(dt).eps / 2


def make(shape, dt, seed, std=1.0, pad=0, off=0):
    """Random tensor on the GPU; `pad` extra columns lie between its rows, and it
    starts `off` elements into its buffer. The buffer around it holds NaN."""
    g = torch.Generator().manual_seed(seed)
    v = (torch.randn(*shape, generator=g) * std).to(dt)
    buf = torch.full((off + shape[0] * (shape[1] + pad),), float("nan"), dtype=dt, device="cuda")
    t = buf[off:].view(shape[0], shape[1] + pad)[:, :shape[1]]
    t.copy_(v)
    return t


def f64(t):
    return t.detach().cpu().double().numpy()


def close(got, want, bound, what=""):
    d = np.abs(f64(got) - want)
    bad = ~(d <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(d - bound)} over its bound"


def codes_of(k):
    return f64(k.codes.contiguous().view(torch.float8_e4m3fn).float())


# -- checkpoints -------------------------------------------------------------
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (3, 16), (2, 127), (5, 128), (4, 129), (33, 257),
                                   (7, 1003), (300, 640), (1, 20000), (5000, 3)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_checkpoint_codes_and_values(shape, dtype):
    x = make(shape, TYPES[dtype], 1, pad=3, off=1)
    k = gr.lionmuon_checkpoint(x)
    want, e = ref.checkpoint(f64(x))
    top = f64(x) != 0
    got_e = f64(k.scales).astype(int) - 127
    assert (got_e == e).all()
    vals = codes_of(k) * np.ldexp(1.0, np.repeat(got_e, 128, axis=1)[:, :shape[1]])
    assert (vals == want).all() and top.any()
    for t in (torch.float32, torch.bfloat16):            # both hold the values exactly
        assert (f64(gr.lionmuon_checkpoint_restore(k, t)) == want).all()
    half = gr.lionmuon_checkpoint_restore(k, torch.float16)
    assert torch.equal(half, torch.from_numpy(want).to(torch.float16).cuda())
    # the bytes between the columns and the next multiple of 16 are 0
    whole = torch.as_strided(k.codes, (shape[0], -(-shape[1] // 16) * 16), k.codes.stride())
    assert (whole[:, shape[1]:] == 0).all()


def test_checkpoint_borders_ties_and_special_values():
    """Maxima at and next to 448 2^e, ties of the rounding, subnormal codes, zero
    blocks, tiny blocks, NaN and infinities beside ordinary values."""
    rows = []
    for top in (448.0, 448.0 * (1 + 2.0 ** -20), 447.99997, 224.0, 224.00002, 1.75, 1.7500001, 1.0,
                3.0e38, 1e-30, 1e-38, 1e-45, 0.0):
        r = np.linspace(-1.0, 1.0, 128) * top
        r[5] = top
        rows.append(r)
    steps = np.arange(1, 129) / 2.0                       # halves of code steps
    rows += [steps * 2.0 ** -9 * 64, steps * 2.0 ** -10, np.r_[448.0, steps[:127] * 2.0 ** -10]]
    odd = np.linspace(-3, 3, 128)
    for v in (np.nan, np.inf, -np.inf):
        r = odd.copy()
        r[[0, 64, 127]] = v
        rows.append(r)
    rows.append(np.full(128, np.nan))
    x = torch.tensor(np.array(rows), dtype=torch.float32, device="cuda")
    k = gr.lionmuon_checkpoint(x)
    want, e = ref.checkpoint(f64(x))
    assert (f64(k.scales).astype(int) - 127 == e).all()
    got = f64(gr.lionmuon_checkpoint_restore(k, torch.float32))
    np.testing.assert_array_equal(got, want)


# -- activations -------------------------------------------------------------
def act_inputs(kind, rows, cols, dtype, pad=5, off=1):
    dt = TYPES[dtype]
    a = make((rows, cols * (2 if kind == "swiglu" else 1)), dt, 3, 3.0, pad, off)
    dh = make((rows, cols), dt, 4, 1.0, pad, off)
    return a, dh


def gate_error(x, kind):
    """Bound of the gate's relative error in fp32. Its argument t is off by four roundings,
    and by one more in base 2: 5 * 2^-24 |t|, which the exponential turns into that much
    of its result; exponential, sum, reciprocal and products: eight roundings. Beyond
    |t| = 90 the exponential is below every normal number."""
    t = np.abs(np.split(x, 2, axis=1)[0] if kind == "swiglu" else
               2 * ref.GELU_C * (x + ref.GELU_A * x ** 3))
    return 2.0 ** -24 * (5 * np.minimum(t, 90.0) + 8)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 9), (2, 64), (5, 127), (4, 128), (3, 129),
                                       (17, 256), (9, 771), (200, 384), (1, 5000)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("kind", ["gelu", "swiglu"])
def test_activation_and_gradient(kind, dtype, rows, cols):
    a, dh = act_inputs(kind, rows, cols, dtype)
    hs = half_step(a.dtype)
    h, kept = gr.lionmuon_activation(a, kind, checkpoint=True)
    x = f64(a)
    want = ref.activation(x, kind)
    close(h, want, (hs * 1.01 + gate_error(x, kind)) * np.abs(want) + tiny(a.dtype), "h")
    assert torch.equal(h, gr.lionmuon_activation(a, kind)[0])
    vals, e = ref.checkpoint(x)
    assert (f64(gr.lionmuon_checkpoint_restore(kept, torch.float32)) == vals).all()
    for src, v in ((a, x), (kept, vals)):
        da, again = gr.lionmuon_activation_grad(dh, src, kind, recompute=True)
        want = ref.activation_grad(f64(dh), v, kind)
        if kind == "swiglu":
            g, u = np.split(np.abs(v), 2, axis=1)
            d = np.abs(f64(dh))
            mag = np.concatenate([d * u * (1 + g), d * g], axis=1)
        else:
            mag = np.abs(f64(dh)) * (1 + np.abs(v) + np.abs(v) ** 3)
        fp = gate_error(v, kind)
        if kind == "swiglu":
            fp = np.concatenate([fp, fp], axis=1)
        close(da, want, hs * np.abs(want) * 1.01 + fp * mag + tiny(a.dtype), "da")
        want = ref.activation(v, kind)
        close(again, want, (hs * 1.01 + gate_error(v, kind)) * np.abs(want) + tiny(a.dtype), "h again")
        only, none = gr.lionmuon_activation_grad(dh, src, kind)
        assert none is None and torch.equal(only, da)


def tiny(dt):
    """Half the distance of a type's smallest numbers, where results are subnormal (fp32:
    where an exponential is)."""
    return {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -120, torch.float32: 2.0 ** -120}[dt]


@pytest.mark.parametrize("kind", ["gelu", "swiglu"])
def test_activation_gradient_against_differences(kind):
    rows, cols = 6, 40
    a, dh = act_inputs(kind, rows, cols, "fp32")
    da, _ = gr.lionmuon_activation_grad(dh, a, kind)
    x, d, step = f64(a), f64(dh), 1e-5
    want = np.empty_like(x)
    for c in range(x.shape[1]):
        up, down = x.copy(), x.copy()
        up[:, c] += step
        down[:, c] -= step
        want[:, c] = (d * (ref.activation(up, kind) - ref.activation(down, kind))).sum(1) / (2 * step)
    # differences: step^2 times third derivatives (below 10 |x u d|), 2^-53 / step
    np.testing.assert_allclose(f64(da), want, rtol=1e-5, atol=1e-5)


def test_activation_large_magnitudes():
    x = torch.tensor([[-1e4, -100.0, -30.0, 0.0, 30.0, 100.0, 1e4, float("nan")]], device="cuda")
    for dt in TYPES.values():
        h, _ = gr.lionmuon_activation(x.to(dt), "gelu")
        v = f64(h)[0]
        assert (v[:4] == 0).all() and (v[4:7] == f64(x.to(dt))[0, 4:7]).all() and np.isnan(v[7])
        da, _ = gr.lionmuon_activation_grad(torch.ones_like(x).to(dt), x.to(dt), "gelu")
        assert (f64(da)[0, :7] == [0, 0, 0, 0.5, 1, 1, 1]).all()


# -- norm --------------------------------------------------------------------
NORM_SHAPES = [(1, 1), (1, 5), (3, 8), (8, 1024), (5, 511), (6, 513), (4, 1100), (3, 2048), (7, 2049),
               (2, 4100), (3, 8192), (2, 8193), (2, 16384), (4100, 40), (2500, 2304)]


@pytest.mark.parametrize("shape", NORM_SHAPES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_norm_and_gradient(shape, dtype):
    rows, cols = shape
    dt = TYPES[dtype]
    eps = 1e-5
    x, r = make(shape, dt, 5, 1.0, 3, 1), make(shape, dt, 6, 2.0, 5, 3)
    dy, dres = make(shape, dt, 7, 1.0, 1, 1), make(shape, dt, 8, 1.0, 2, 1)
    w = make((1, cols), torch.float32, 9)[0].contiguous()
    y, s, rstd, kept = gr.lionmuon_rmsnorm(x, w, residual=r, eps=eps, checkpoint=True)
    total = (x.float() + r.float()).to(dt)
    assert torch.equal(s, total)
    want, wr = ref.rmsnorm(f64(s), f64(w), eps)
    # sum of squares: at most 32 serial additions a lane, ten tree levels; then
    # division, square root, reciprocal and two products
    fp = 2.0 ** -24 * 50
    close(rstd, wr, fp * wr, "rstd")
    close(y, want, (half_step(dt) * 1.01 + fp) * np.abs(want) + tiny(dt), "y")
    e = f64(kept.scales).astype(int) - 127
    near = ref.block_exponents(want * (1 + 2 * fp)), ref.block_exponents(want * (1 - 2 * fp))
    assert ((e == near[0]) | (e == near[1])).all()
    scale = np.ldexp(1.0, np.repeat(e, 128, axis=1)[:, :cols])
    y8 = gr.lionmuon_checkpoint_restore(kept, torch.float32)
    close(y8, want, (2.0 ** -4 * 1.001) * np.abs(want) + 2.0 ** -10 * scale, "y8")
    only8 = gr.lionmuon_rmsnorm(x, w, residual=r, eps=eps, out=False, checkpoint=True)
    assert only8[0] is None and torch.equal(only8[3].codes, kept.codes)
    # without a residual the stream is x itself
    y0, s0, rstd0, none = gr.lionmuon_rmsnorm(s, w, eps=eps)
    assert none is None and s0 is s and torch.equal(y0, y) and torch.equal(rstd0, rstd)
    # gradients, from the stream and from its checkpoint
    k = gr.lionmuon_checkpoint(s)
    rs = f64(rstd)
    for src, v in ((s, f64(s)), (k, ref.checkpoint(f64(s))[0])):
        dx, dw = gr.lionmuon_rmsnorm_grad(dy, src, w, rstd, residual_grad=dres)
        wdx, wdw = ref.rmsnorm_grad(f64(dy), v, f64(w), rs, f64(dres))
        xh, t = np.abs(v) * rs[:, None], np.abs(f64(dy) * f64(w))
        mag = rs[:, None] * (t + xh * (t * xh).mean(1, keepdims=True)) + np.abs(f64(dres))
        close(dx, wdx, half_step(dt) * 1.01 * np.abs(wdx) + fp * mag + tiny(dt), "dx")
        mag = (np.abs(f64(dy)) * xh).sum(0)
        close(dw, wdw, 2.0 ** -24 * (rows + 64) * mag, "dw")
        dx0, none = gr.lionmuon_rmsnorm_grad(dy, src, w, rstd, weight_grad=False)
        assert none is None
        w0, _ = ref.rmsnorm_grad(f64(dy), v, f64(w), rs)
        mag = rs[:, None] * (t + xh * (t * xh).mean(1, keepdims=True))
        close(dx0, w0, half_step(dt) * 1.01 * np.abs(w0) + fp * mag + tiny(dt), "dx alone")
        none, dw1 = gr.lionmuon_rmsnorm_grad(dy, src, w, rstd, out=False)
        assert none is None and torch.equal(dw1, dw)
        acc = torch.full_like(dw, 2.0)
        gr.lionmuon_rmsnorm_grad(dy, src, w, rstd, out=False, weight_grad=acc, accumulate=True)
        assert torch.equal(acc, dw + 2.0)


def test_norm_in_place_forms_and_zero_rows():
    x, r = make((9, 300), torch.bfloat16, 1), make((9, 300), torch.bfloat16, 2)
    w = torch.rand(300, device="cuda")
    y, s, rstd, _ = gr.lionmuon_rmsnorm(x, w, residual=r)
    r2 = r.contiguous().clone()
    y2, s2, _, _ = gr.lionmuon_rmsnorm(x, w, residual=r2, sum_out=r2)
    assert s2 is r2 and torch.equal(r2, s) and torch.equal(y2, y)
    dy, dres = make((9, 300), torch.bfloat16, 3), make((9, 300), torch.bfloat16, 4)
    dx, dw = gr.lionmuon_rmsnorm_grad(dy, s, w, rstd, residual_grad=dres)
    d2 = dres.contiguous().clone()
    assert gr.lionmuon_rmsnorm_grad(dy, s, w, rstd, residual_grad=d2, out=d2)[0] is d2
    assert torch.equal(d2, dx)
    # no rows: nothing to norm, a weight gradient of 0 (or what was there)
    e = x[:0]
    assert gr.lionmuon_rmsnorm(e, w)[0].shape == (0, 300)
    rs = torch.empty(0, device="cuda")
    dx, dw = gr.lionmuon_rmsnorm_grad(e, e, w, rs)
    assert dx.shape == (0, 300) and (dw == 0).all()
    dw.fill_(3.0)
    gr.lionmuon_rmsnorm_grad(e, e, w, rs, weight_grad=dw, accumulate=True)
    assert (dw == 3.0).all()
    # a row of zeros: rstd = 1 / sqrt(eps), y = 0; with eps = 0 not finite
    z = torch.zeros(2, 64, device="cuda")
    y, _, rstd, _ = gr.lionmuon_rmsnorm(z, torch.ones(64, device="cuda"), eps=1e-6)
    assert (y == 0).all() and torch.allclose(rstd, torch.full_like(rstd, 1e3))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("cols", [1, 5, 67, 131, 1003])
def test_bytes_behind_the_last_code_are_zero_in_rows_of_nan_too(cols, dtype):
    x = make((5, cols), TYPES[dtype], cols)
    x[1, 0], x[3, cols - 1] = float("nan"), float("inf")
    w = torch.ones(cols, device="cuda")
    ld = -(-cols // 16) * 16
    for write in (lambda k: gr.lionmuon_checkpoint(x, out=k),
                  lambda k: gr.lionmuon_rmsnorm(x, w, checkpoint=k),
                  lambda k: gr.lionmuon_activation(x, "gelu", checkpoint=k)):
        codes = torch.full((5, ld), 9, dtype=torch.uint8, device="cuda")
        write(gr.Checkpoint(codes[:, :cols], torch.zeros(5, -(-cols // 128), dtype=torch.uint8, device="cuda")))
        assert (codes[:, cols:] == 0).all()


def test_norm_gradient_against_differences():
    rows, cols, eps = 5, 24, 1e-5
    s, dy = make((rows, cols), torch.float32, 1), make((rows, cols), torch.float32, 2)
    w = make((1, cols), torch.float32, 3)[0].contiguous()
    rstd = gr.lionmuon_rmsnorm(s, w, eps=eps)[2]
    dx, dw = gr.lionmuon_rmsnorm_grad(dy, s, w, rstd)
    x, d, ww, step = f64(s), f64(dy), f64(w), 1e-5
    for c in range(cols):
        up, down = x.copy(), x.copy()
        up[:, c] += step
        down[:, c] -= step
        want = (d * (ref.rmsnorm(up, ww, eps)[0] - ref.rmsnorm(down, ww, eps)[0])).sum(1) / (2 * step)
        np.testing.assert_allclose(f64(dx)[:, c], want, rtol=1e-5, atol=1e-5)
        wu, wd = ww.copy(), ww.copy()
        wu[c] += step
        wd[c] -= step
        want = (d * (ref.rmsnorm(x, wu, eps)[0] - ref.rmsnorm(x, wd, eps)[0])).sum() / (2 * step)
        np.testing.assert_allclose(f64(dw)[c], want, rtol=1e-5, atol=1e-5)


# -- grouped products --------------------------------------------------------
def group_sizes(total, experts, seed):
    """Skewed sizes with empty experts, the first and the last among them."""
    r = np.random.RandomState(seed)
    p = np.exp(1.2 * r.randn(experts))
    if experts >= 4:
        p[[0, experts // 2, experts - 1]] = 0.0
    return r.multinomial(total, p / p.sum())


def group(total, experts, n, k, dt, seed, lead=0, tail=0, pad=0, off=0, sizes=None):
    sizes = group_sizes(total, experts, seed) if sizes is None else np.asarray(sizes)
    at = lead + np.concatenate([[0], np.cumsum(sizes)])
    rows = int(at[-1]) + tail
    x = make((rows, k), dt, seed, 1.0, pad, off)
    dy = make((rows, n), dt, seed + 1, 1.0, pad, off)
    w = make((experts * n, k), dt, seed + 2, 1.0, pad, off)
    w = torch.as_strided(w, (experts, n, k), (n * w.stride(0), w.stride(0), 1), w.storage_offset())
    return x, dy, w, torch.tensor(at, dtype=torch.int32, device="cuda"), at


GROUPS = [
    # rows, experts, n, k, sizes
    (1, 1, 1, 1, None), (1, 1, 64, 64, None), (5, 1, 33, 17, None), (7, 3, 8, 264, [0, 7, 0]),
    (2, 8, 256, 512, None), (16, 8, 320, 1024, None), (40, 6, 130, 72, None), (64, 1, 128, 128, None),
    (65, 2, 129, 127, [64, 1]), (200, 5, 136, 200, None), (255, 2, 257, 65, [128, 127]),
    (300, 70, 48, 56, None), (513, 4, 71, 1003, None), (1000, 3, 384, 320, None),
    (1500, 1, 640, 192, None), (2100, 2, 96, 264, [1, 2099]), (5000, 9, 192, 136, None),
    (700, 300, 40, 24, None),
]


def sum_bound(depth):
    """Roundings of a product's sum: the matrix unit adds at most four products
    exactly and truncates each addition (2^-23 of a partial sum)."""
    return (depth / 4 + 16) * 2.0 ** -23


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout", ["aligned", "odd"])
@pytest.mark.parametrize("rows,experts,n,k,sizes", GROUPS)
def test_grouped_products(rows, experts, n, k, sizes, layout, dtype):
    dt = TYPES[dtype]
    lead, tail = (0, 0) if layout == "aligned" else (3, 9)
    pad, off = (0, 0) if layout == "aligned" else (3, 1)
    x, dy, w, offsets, at = group(rows, experts, n, k, dt, rows + n, lead, tail, pad, off, sizes)
    inside = np.zeros(x.shape[0], dtype=bool)
    inside[at[0]:at[-1]] = True
    hs = half_step(dt) * 1.01
    # products: rows of no expert and the columns between rows stay as they were
    for call, a, width, depth, args in (
            (gr.lionmuon_grouped_product, x, n, k, (f64(x), f64(w))),
            (gr.lionmuon_grouped_input_grad, dy, k, n, (f64(dy), f64(w).transpose(0, 2, 1)))):
        buf = torch.full((x.shape[0], width + pad + 2), 7.0, dtype=dt, device="cuda")
        out = buf[:, 1:1 + width] if layout == "odd" else buf[:, :width].contiguous()
        got = call(a, w, offsets, out=out)
        assert got is out
        want, mag = ref.grouped(np.nan_to_num(args[0]), args[1], at)
        close(out[torch.from_numpy(inside).cuda()], want[inside],
              hs * np.abs(want[inside]) + sum_bound(depth) * mag[inside] + tiny(dt), call.__name__)
        assert (out[torch.from_numpy(~inside).cuda()] == 7.0).all()
        if layout == "odd":
            assert (buf[:, 0] == 7.0).all() and (buf[:, 1 + width:] == 7.0).all()
        assert torch.equal(call(a, w, offsets, out=torch.full_like(out, 7.0)), out)
    # weight gradient: new, accumulated, into strided buffers
    want, mag = ref.grouped_weight(f64(dy), f64(x), at)
    longest = max(np.diff(at))
    bound = sum_bound(longest) * mag + 1e-30
    dw = gr.lionmuon_grouped_weight_grad(dy, x, offsets)
    close(dw, want, bound, "dw")
    flat = torch.full((experts * (n + 1) * (k + pad) + 5,), 0.5, device="cuda")
    out = torch.as_strided(flat, (experts, n, k), ((n + 1) * (k + pad), k + pad, 1), 3)
    gr.lionmuon_grouped_weight_grad(dy, x, offsets, out=out, accumulate=True)
    assert torch.equal(out, 0.5 + dw)
    mask = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(mask, out.shape, out.stride(), 3).fill_(False)
    assert (flat[mask] == 0.5).all()
    if dtype == "bf16":
        kept = gr.lionmuon_checkpoint(x)
        vals = gr.lionmuon_checkpoint_restore(kept, torch.bfloat16)
        got = gr.lionmuon_grouped_weight_grad(dy, kept, offsets)
        want, mag = ref.grouped_weight(f64(dy), f64(vals), at)
        close(got, want, sum_bound(longest) * mag + 1e-30, "dw from a checkpoint")


def test_weight_gradient_in_splits():
    """Few tiles and many rows: the rows of an expert go to several workgroups."""
    rows, n, k = 9000, 136, 72
    assert gr.lionmuon_grouped_workspace_bytes(rows, 2, n, k) > 0
    for sizes in ([rows, 0], [1, rows - 1], [4000, 5000]):
        x, dy, _, offsets, at = group(rows, 2, n, k, torch.bfloat16, 11, sizes=sizes)
        want, mag = ref.grouped_weight(f64(dy), f64(x), at)
        dw = gr.lionmuon_grouped_weight_grad(dy, x, offsets)
        # chains of 256 rows in the matrix unit, added up in fp32
        close(dw, want, (256 / 4 + rows / 256 + 16) * 2.0 ** -23 * mag + 1e-30, "dw")
        err = np.linalg.norm(f64(dw) - want) / np.linalg.norm(want)
        assert err < 1.5e-6
        kept = gr.lionmuon_checkpoint(x)
        same = gr.lionmuon_checkpoint_restore(kept)
        a = gr.lionmuon_grouped_weight_grad(dy, kept, offsets)
        assert torch.equal(a, gr.lionmuon_grouped_weight_grad(dy, same, offsets))


def test_nan_and_inf_stay_in_their_rows():
    """A NaN in one row (also in a row of no expert, or of another expert in the
    same tile) reaches that row's outputs and that expert's gradient only."""
    x, dy, w, offsets, at = group(200, 3, 72, 88, torch.bfloat16, 5, tail=8, sizes=[70, 60, 70])
    y0 = gr.lionmuon_grouped_product(x, w, offsets)
    d0 = gr.lionmuon_grouped_weight_grad(dy, x, offsets)
    x2 = x.clone()
    x2[75, 3] = float("nan")
    x2[203:] = float("inf")
    dy2 = dy.clone()
    dy2[205:] = float("nan")
    y = gr.lionmuon_grouped_product(x2, w, offsets)
    keep = torch.ones(200, dtype=torch.bool, device="cuda")
    keep[75] = False
    assert torch.equal(y[:200][keep], y0[:200][keep]) and y[75].isnan().all()
    d = gr.lionmuon_grouped_weight_grad(dy2, x2, offsets)
    assert torch.equal(d[0], d0[0]) and torch.equal(d[2], d0[2])
    assert d[1][:, 3].isnan().all() and not d[1][:, 4].isnan().any()


def test_offsets_that_break_the_rule_stay_inside():
    x, dy, w, _, _ = group(300, 4, 72, 88, torch.bfloat16, 6, sizes=[75] * 4)
    for bad in ([0, 400, 100, 900, 300], [-5, 50, 20, 300, 2 ** 31 - 1], [-(2 ** 31)] * 5, [300, 200, 100, 50, 0]):
        offsets = torch.tensor(bad, dtype=torch.int64).to(torch.int32).cuda()
        buf = torch.full((302, 74), 7.0, dtype=torch.bfloat16, device="cuda")
        gr.lionmuon_grouped_product(x, w, offsets, out=buf[1:301, 1:73])
        assert (buf[0] == 7).all() and (buf[301] == 7).all() and (buf[:, 0] == 7).all()
        gr.lionmuon_grouped_weight_grad(dy, x, offsets)
        torch.cuda.synchronize()


# -- streams, graphs, one run of all of them --------------------------------
def layer(x, residual, wn, w1, w2, offsets, dout):
    """One training pass of an expert layer: norm, two grouped products around a
    gated activation, and every gradient; the kept tensors are checkpoints."""
    y, s, rstd, y8 = gr.lionmuon_rmsnorm(x, wn, residual=residual, checkpoint=True)
    a = gr.lionmuon_grouped_product(y, w1, offsets)
    h, a8 = gr.lionmuon_activation(a, "swiglu", checkpoint=True)
    out = gr.lionmuon_grouped_product(h, w2, offsets)
    dh = gr.lionmuon_grouped_input_grad(dout, w2, offsets)
    da, h2 = gr.lionmuon_activation_grad(dh, a8, "swiglu", recompute=True)
    g2 = gr.lionmuon_grouped_weight_grad(dout, h2, offsets)
    dy = gr.lionmuon_grouped_input_grad(da, w1, offsets)
    g1 = gr.lionmuon_grouped_weight_grad(da, y8, offsets)
    dx, gn = gr.lionmuon_rmsnorm_grad(dy, s, wn, rstd, residual_grad=dout)
    return out, dx, g1, g2, gn


def layer_inputs(seed=0, rows=600, d=192, f=256, experts=4):
    x, r = make((rows, d), torch.bfloat16, seed), make((rows, d), torch.bfloat16, seed + 1)
    wn = 1 + 0.1 * make((1, d), torch.float32, seed + 2)[0].contiguous()
    w1 = make((experts * 2 * f, d), torch.bfloat16, seed + 3, d ** -0.5).view(experts, 2 * f, d)
    w2 = make((experts * d, f), torch.bfloat16, seed + 4, f ** -0.5).view(experts, d, f)
    at = np.concatenate([[0], np.cumsum(np.random.RandomState(seed).multinomial(rows, [0.4, 0.3, 0.0, 0.3]))])
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    return x, r, wn, w1, w2, offsets, make((rows, d), torch.bfloat16, seed + 5, 0.1)


def test_gradients_of_a_layer_feed_the_step():
    """The whole pass against autograd in float64, then a Muon and a Lion step on the
    gradients, in place.

    What comes from checkpoints agrees as far as they do: a value m 2^k, 1 <= m < 2, is
    rounded to steps of 2^-3 2^k, root mean square 2^-3 / sqrt(12) = 0.0361 of 2^k,
    at most that of the value. dW1 has three such factors (the norm's output, g and
    u), g's through silu' and silu'', whose relative slopes are about 1.5 at most where
    the gradient is large: 0.0361 sqrt(1 + 1 + 1.5^2) = 0.074. The others have two."""
    args = layer_inputs()
    out, dx, g1, g2, gn = layer(*args)
    x, r, wn, w1, w2, offsets, dout = [t.cpu() for t in args]
    p = [t.double().requires_grad_() for t in (x, wn, w1, w2)]
    s = (x.float() + r.float()).bfloat16().double() + (p[0] - p[0].detach())
    y = s * torch.rsqrt((s * s).mean(1, keepdim=True) + 1e-5) * p[1]
    at = offsets.tolist()
    parts = []
    for e in range(4):
        g, u = (y[at[e]:at[e + 1]] @ p[2][e].T).chunk(2, 1)
        parts.append((torch.nn.functional.silu(g) * u) @ p[3][e].T)
    full = torch.cat(parts)
    full.backward(dout.double())
    for got, want, tol in ((out, full.detach(), 1e-2), (dx.cpu().double() - dout.double(), p[0].grad, 7.5e-2),
                           (gn, p[1].grad, 7.5e-2), (g1, p[2].grad, 7.5e-2),
                           (g2, p[3].grad, 7.5e-2)):
        got = got.cpu().double()
        assert float((got - want).norm() / want.norm()) < tol
    params, grads = [], []
    for w, g in ((args[3], g1), (args[4], g2)):
        for e in range(4):
            params.append(w[e].float())
            grads.append(g[e])
    params.append(args[2].clone())
    grads.append(gn)
    momentum = [torch.zeros_like(q) for q in params]
    before = [q.clone() for q in params]
    cfg = lm.config(lr_muon=0.02, lr_lion=0.01)
    for t in (0, 1):
        lm.lionmuon_step_ex(params, grads, momentum, t, 2, 0.9, 0.99, 0.0, cfg)
    torch.cuda.synchronize()
    for i, (q, b) in enumerate(zip(params, before)):
        assert torch.isfinite(q).all()
        assert torch.equal(q, b) == (i in (2, 6))          # the expert without rows has gradient 0


def test_streams_and_repeats_give_the_same_bits():
    args = layer_inputs(3)
    want = layer(*args)
    side = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for st in side:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for st in side:
            with torch.cuda.stream(st):
                got.append(layer(*args))
    torch.cuda.synchronize()
    for g in got:
        for a, b in zip(g, want):
            assert torch.equal(a, b)
    # the stream argument, as an object and as a handle
    x, w, offsets = args[0], args[3], args[5]
    y0 = gr.lionmuon_grouped_product(x, w, offsets)
    for st in (side[0], side[0].cuda_stream):
        side[0].wait_stream(torch.cuda.current_stream())
        y = gr.lionmuon_grouped_product(x, w, offsets, stream=st)
        side[0].synchronize()
        assert torch.equal(y, y0)


def test_captured_layer_replays_with_new_inputs():
    """Two graphs of the same pass, each with its own workspaces, replayed with
    eager work and new inputs (other expert sizes too) in between."""
    a, b = layer_inputs(7), layer_inputs(8)
    graphs = []
    for args in (a, b):
        static = [t.clone() for t in args]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            layer(*static)
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = layer(*static)
        graphs.append((g, static, out))
    for turn in range(4):
        new = layer_inputs(20 + turn)
        for g, static, out in graphs:
            for t, v in zip(static, new):
                t.copy_(v)
            g.replay()
        want = layer(*new)
        torch.cuda.synchronize()
        for g, static, out in graphs:
            for x, y in zip(out, want):
                assert torch.equal(x, y)


# -- large tiles -------------------------------------------------------------
def gpu_products(call, a, w, at, transpose):
    """float64 products on the GPU, rows of no expert 0."""
    y = torch.zeros(a.shape[0], w.shape[2] if transpose else w.shape[1], dtype=torch.float64, device="cuda")
    for e in range(w.shape[0]):
        r = slice(int(at[e]), int(at[e + 1]))
        y[r] = a[r].double() @ (w[e].double() if transpose else w[e].double().t())
    return y


# the largest tiles, a last round in quarters (4200 x 4100: 17 x 17 tiles of 256), and
# operands off 16 bytes at either side
@pytest.mark.parametrize("experts,rows,n,k,pad", [(1, 4200, 4100, 512, 0), (3, 4300, 4096, 264, 0), (2, 4000, 2051, 776, 0),
                                                  (2, 4000, 776, 2051, 0), (2, 3000, 1100, 1500, 1)])
def test_large_products(experts, rows, n, k, pad):
    dt = torch.bfloat16
    x, dy, w, offsets, at = group(rows, experts, n, k, dt, 31, tail=5, pad=pad, off=pad)
    inside = slice(0, int(at[-1]))
    for call, a, depth, transpose in ((gr.lionmuon_grouped_product, x, k, False),
                                      (gr.lionmuon_grouped_input_grad, dy, n, True)):
        want = gpu_products(call, a, w, at, transpose)
        out = torch.full(want.shape, 7.0, dtype=dt, device="cuda")
        call(a, w, offsets, out=out)
        # independent terms of mean square v: a sum of `depth` is off by at most depth v^0.5 times
        # the roundings of sum_bound, and by half a step of its own
        v = float(a[inside].double().square().mean() * w.double().square().mean()) ** 0.5
        err = (out[inside].double() - want[inside]).abs()
        assert (err <= half_step(dt) * 1.01 * want[inside].abs() + sum_bound(depth) * depth * v).all()
        assert (out[int(at[-1]):] == 7.0).all()


# several large tiles a workgroup, one after the other: contractions of less than a
# stage, of one, two and a part of one; more experts than lanes, empty ones among them
@pytest.mark.parametrize("experts,rows,n,k", [(1, 16400, 4104, 8), (1, 16400, 4104, 64), (3, 20000, 4096, 128),
                                              (70, 30000, 2048, 136), (9, 40000, 2304, 200)])
def test_products_of_several_rounds(experts, rows, n, k):
    dt = torch.bfloat16
    x, dy, w, offsets, at = group(rows, experts, n, k, dt, 53, lead=2, tail=3)
    inside = slice(int(at[0]), int(at[-1]))
    for call, a, b, depth, transpose in (
            (gr.lionmuon_grouped_product, x, w, k, False),
            (gr.lionmuon_grouped_input_grad, x, w.transpose(1, 2).contiguous(), k, True)):
        want = gpu_products(call, a, b, at, transpose)
        out = torch.full(want.shape, 7.0, dtype=dt, device="cuda")
        call(a, b, offsets, out=out)
        v = float(a[inside].double().square().mean() * b.double().square().mean()) ** 0.5
        err = (out[inside].double() - want[inside]).abs()
        assert (err <= half_step(dt) * 1.01 * want[inside].abs() + sum_bound(depth) * depth * v).all()
        assert (out[:int(at[0])] == 7.0).all() and (out[int(at[-1]):] == 7.0).all()
        assert torch.equal(call(a, b, offsets, out=torch.full_like(out, 7.0)), out)


@pytest.mark.parametrize("experts,rows,n,k", [(1, 5000, 512, 1280), (3, 9000, 700, 640), (2, 700, 2560, 1152),
                                              (1, 70, 256, 128), (1, 20000, 300, 1000)])
def test_weight_gradient_from_a_checkpoint_is_that_of_its_values(experts, rows, n, k):
    x, dy, _, offsets, at = group(rows, experts, n, k, torch.bfloat16, 41, tail=3)
    kept = gr.lionmuon_checkpoint(x)
    same = gr.lionmuon_checkpoint_restore(kept)
    got = gr.lionmuon_grouped_weight_grad(dy, kept, offsets)
    assert torch.equal(got, gr.lionmuon_grouped_weight_grad(dy, same, offsets))
    want = torch.stack([dy[at[e]:at[e + 1]].double().t() @ same[at[e]:at[e + 1]].double() for e in range(experts)])
    for e in range(experts):
        if at[e + 1] > at[e]:
            assert float((got[e].double() - want[e]).norm() / want[e].norm()) < 1e-6
    # scales that cannot be copied four at a time give the same
    wide = torch.zeros(kept.scales.shape[0], kept.scales.shape[1] + 5, dtype=torch.uint8, device="cuda")
    wide[:, 1:1 + kept.scales.shape[1]] = kept.scales
    odd = gr.Checkpoint(kept.codes, wide[:, 1:1 + kept.scales.shape[1]])
    assert float((gr.lionmuon_grouped_weight_grad(dy, odd, offsets) - got).norm() / got.norm()) < 1e-6


# -- rows 16-byte aligned, widths that are not --------------------------------
def aligned_rows(rows, cols, dt, seed):
    """Random (rows, cols) tensor whose rows start 16-byte aligned; what lies between
    them is NaN."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((rows, cols // 8 * 8 + 8), float("nan"), dtype=dt, device="cuda")
    buf[:, :cols] = torch.randn(rows, cols, generator=g).to(dt).cuda()
    return buf[:, :cols]


# every width modulo eight, by each of the tile sizes of the two gradients, rows of several stages
@pytest.mark.parametrize("rows,sizes,n,k", [(200, [200], 144, 64), (300, [100, 200], 296, 296),
                                            (4000, [1333, 2667], 1024, 768), (4200, [4200], 4096, 1024)])
@pytest.mark.parametrize("extra", range(1, 8))
def test_last_columns_of_widths_off_16_bytes_in_aligned_rows(rows, sizes, n, k, extra):
    dt, experts = torch.bfloat16, len(sizes)
    n, k = n + extra, k + extra
    x, dy, w = (aligned_rows(r, c, dt, s) for r, c, s in ((rows, k, 1), (rows, n, 2), (experts * n, k, 3)))
    w = torch.as_strided(w, (experts, n, k), (n * w.stride(0), w.stride(0), 1))
    at = np.concatenate([[0], np.cumsum(sizes)])
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    dx, dw = gr.lionmuon_grouped_input_grad(dy, w, offsets), gr.lionmuon_grouped_weight_grad(dy, x, offsets)
    y = gr.lionmuon_grouped_product(x, w, offsets)
    for e in range(experts):
        r = slice(int(at[e]), int(at[e + 1]))
        a, b, c = dy[r].double(), w[e].double(), x[r].double()
        for got, p, q, hs in ((dx[r], a, b, half_step(dt)), (y[r], c, b.t(), half_step(dt)), (dw[e], a.t(), c, 0.0)):
            want, mag = p @ q, p.abs() @ q.abs()
            err = (got.double() - want).abs()
            assert (err <= hs * 1.01 * want.abs() + sum_bound(p.shape[1]) * mag).all()


def test_gelu_gradient_of_numbers_of_any_size():
    """Where x^2 leaves the type's range the slope is 1 or 0, as from |x| = 16 on; up to
    there the border of the two forms is not seen."""
    for name, dt in TYPES.items():
        top = torch.finfo(dt).max
        v = [m for m in (15.9, 16.0, 16.1, 1e3, 6e4, 1e10, 1e19, 2e19, 1e20, 1e30, top) if m <= top]
        x = torch.tensor([v + [-m for m in v]], dtype=torch.float64).to(dt).cuda()
        da, h = gr.lionmuon_activation_grad(torch.ones_like(x), x, "gelu", recompute=True)
        assert (f64(da)[0, :len(v)] == 1).all() and (f64(da)[0, len(v):] == 0).all(), name
        assert (f64(h)[0, :len(v)] == f64(x)[0, :len(v)]).all() and (f64(h)[0, len(v):] == 0).all(), name
        # from a checkpoint, whose values these are (one in each block)
        kept = gr.lionmuon_checkpoint(torch.full((1, 128), 2.0 ** 15 if dt == torch.float16 else 2.0 ** 100, dtype=dt, device="cuda"))
        assert (gr.lionmuon_activation_grad(torch.ones(1, 128, dtype=dt, device="cuda"), kept, "gelu")[0] == 1).all()
        nan = torch.full((1, 3), float("nan"), dtype=dt, device="cuda")
        assert gr.lionmuon_activation_grad(torch.ones_like(nan), nan, "gelu")[0].isnan().all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_checkpoint_of_the_largest_numbers_is_finite(dtype):
    """Above 1.9375 * 2^127 the nearest code of a block with e = 120 would stand for 2^128."""
    dt = TYPES[dtype]
    top = torch.finfo(dt).max
    v = torch.tensor([top, -top, 1.9375 * 2.0 ** 127, -1.9453125 * 2.0 ** 127, 1.875 * 2.0 ** 127, 1.75 * 2.0 ** 127,
                      -1.7578125 * 2.0 ** 127, 2.0 ** 127, 3e37, -1.0, 0.0], dtype=torch.float64)
    x = torch.full((3, 200), 0.5, dtype=dt, device="cuda")
    x[0, 5:5 + len(v)] = v.to(dt).cuda()
    x[1, 140] = top
    x[2, 0], x[2, 1] = top, float("nan")
    for k in (gr.lionmuon_checkpoint(x), gr.lionmuon_activation(x, "gelu", checkpoint=True)[1]):
        e = f64(k.scales).astype(int) - 127
        assert (e == ref.block_exponents(f64(x))).all() and e.max() == 120
        for t in (torch.float32, torch.bfloat16):
            got, want = f64(gr.lionmuon_checkpoint_restore(k, t)), f64(x)
            assert np.isnan(got[2, 1])
            got[2, 1] = want[2, 1] = 0.0
            scale = np.ldexp(1.0, np.repeat(e, 128, axis=1)[:, :200])
            assert (np.abs(got - want) <= 2.0 ** -4 * np.abs(want) * (np.abs(want) >= 2.0 ** -6 * scale) + 2.0 ** -10 * scale).all()
            assert (np.abs(got) <= 240 * 2.0 ** 120).all() and got[0, 5] == -got[0, 6] == 240 * 2.0 ** 120


# -- tensors that are passed in and written -----------------------------------
def test_tensors_that_are_written_count_as_changed():
    """Every output that is passed in, so that autograd notices a saved tensor that a
    call has overwritten; inputs do not count."""
    dt = torch.bfloat16
    x, r, dy = (make((6, 256), dt, s) for s in (1, 2, 3))
    w = torch.rand(256, device="cuda")
    at = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")
    stack = torch.randn(2, 64, 256, device="cuda").to(dt)
    rstd = gr.lionmuon_rmsnorm(x, w)[2]

    def new(*shape, t=dt):
        return torch.zeros(*shape, dtype=t, device="cuda")

    def kept():
        return gr.Checkpoint(new(6, 256, t=torch.uint8), new(6, 2, t=torch.uint8))

    def versions(ts):
        return [t._version for t in ts]

    inputs = [x, r, dy, w, at, stack, rstd]
    k, dout = gr.lionmuon_checkpoint(x), new(6, 64)
    for call, outputs in (
            (lambda a: gr.lionmuon_checkpoint_restore(k, out=a), [new(6, 256)]),
            (lambda a: gr.lionmuon_activation(x, "gelu", out=a), [new(6, 256)]),
            (lambda a, b: gr.lionmuon_activation_grad(dy, k, "gelu", out=a, recompute=b), [new(6, 256), new(6, 256)]),
            (lambda a, b: gr.lionmuon_rmsnorm(x, w, residual=r, out=a, sum_out=b), [new(6, 256), new(6, 256)]),
            (lambda a, b: gr.lionmuon_rmsnorm_grad(dy, k, w, rstd, out=a, weight_grad=b), [new(6, 256), new(256, t=torch.float32)]),
            (lambda a: gr.lionmuon_grouped_product(x, stack, at, out=a), [new(6, 64)]),
            (lambda a: gr.lionmuon_grouped_input_grad(dout, stack, at, out=a), [new(6, 256)]),
            (lambda a: gr.lionmuon_grouped_weight_grad(dout, k, at, out=a), [new(2, 64, 256, t=torch.float32)])):
        before, held = versions(outputs), versions(inputs)
        call(*outputs)
        assert all(v > b for v, b in zip(versions(outputs), before))
        assert versions(inputs) == held
    for write in (lambda c: gr.lionmuon_checkpoint(x, out=c), lambda c: gr.lionmuon_activation(x, "gelu", checkpoint=c),
                  lambda c: gr.lionmuon_rmsnorm(x, w, checkpoint=c)):
        for c in (kept(), gr.Checkpoint.empty(6, 256)):
            codes, scales = c.codes, c.scales
            before = versions([codes, scales])
            write(c)
            assert all(v > b for v, b in zip(versions([codes, scales]), before))
    # a backward pass that needs the residual as it was
    p = torch.ones(6, 256, device="cuda", requires_grad=True)
    stream = r.float()
    loss = (p * stream).sum()
    gr.lionmuon_rmsnorm(x.float(), w, residual=stream, sum_out=stream)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        out = new(6, 256)
        assert gr.lionmuon_rmsnorm(x, w, out=out)[0] is out and (out != 0).any()


def test_offsets_of_no_expert_are_refused():
    x, dy = make((6, 64), torch.bfloat16, 1), make((6, 32), torch.bfloat16, 2)
    for n in (0, 1):
        offsets = torch.zeros(n, dtype=torch.int32, device="cuda")
        out = torch.zeros(max(n - 1, 0), 32, 64, device="cuda")
        for call in (lambda: gr.lionmuon_grouped_weight_grad(dy, x, offsets),
                     lambda: gr.lionmuon_grouped_weight_grad(dy, x, offsets, out=out),
                     lambda: gr.lionmuon_grouped_product(x, out.bfloat16(), offsets),
                     lambda: gr.lionmuon_grouped_input_grad(dy, out.bfloat16(), offsets)):
            with pytest.raises(lm.LionMuonError) as e:
                call()
            assert e.value.status == lm.LM_ERR_INVALID_ARGUMENT
