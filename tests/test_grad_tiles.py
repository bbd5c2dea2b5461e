"""The products grouped by expert by each of their tiles, in every layout of the
operands that has a kernel of its own.

CPU: the sizes below get the tile that they stand for (``grad_plan_driver.cpp``).
GPU: products against float64, operands 16-byte aligned (widths are multiples of
eight or not) and off it, both types, experts of several stages, of more than one
sum of 512 rows and without rows, NaN in rows of no expert and between rows.

Tolerances: a 16-bit result is off by at most half a step, eps/2 of its value. Sums
are fp32: at most one rounding of 2^-23 for each four products and 16 more, times
the sum of the products' magnitudes.
"""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2605_19811_amd import gradients as gr

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2605_19811_amd", "csrc")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}

# rows, experts, columns of the output, contraction, tile
ROW_PRODUCTS = [(2001, 3, 4104, 136, 0), (1500, 9, 4099, 72, 0), (3000, 70, 1037, 200, 0), (4100, 1, 4101, 8, 0),
                (700, 9, 2312, 72, 1), (2000, 1, 1033, 136, 1), (700, 70, 1149, 264, 1), (1999, 7, 1003, 776, 1),
                (200, 5, 300, 520, 2), (65, 1, 65, 72, 2), (300, 70, 77, 136, 2)]
# rows, experts, n, k, tile, whether long experts are cut into parts
WEIGHT_GRADIENTS = [(2003, 1, 1543, 2568, 0, False), (700, 9, 2051, 264, 0, False), (9000, 2, 2056, 520, 0, True),
                    (1301, 1, 1544, 2055, 1, False), (900, 20, 75, 2056, 1, False), (9001, 2, 517, 2056, 1, True),
                    (300, 3, 72, 136, 2, False), (1200, 20, 75, 130, 2, False), (3000, 3, 71, 131, 2, True)]
# which operands are off 16 bytes
LAYOUTS = [(False, False), (False, True), (True, False), (True, True)]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_sizes_get_the_tiles_that_they_stand_for(tmp_path):
    exe = str(tmp_path / "grad_plan")
    subprocess.run(["g++", "-O1", "-std=c++17", f"-I{CSRC}", os.path.join(HERE, "grad_plan_driver.cpp"), "-o", exe],
                   check=True)

    def plans(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, v.split())) for v in out.strip().split("\n")]

    for aligned in (0, 1):
        got = plans([f"row {r} {e} {w} {d} {aligned}" for r, e, w, d, _ in ROW_PRODUCTS])
        assert got == [(t,) for *_, t in ROW_PRODUCTS]
    got = plans([f"weight {r} {e} {n} {k}" for r, e, n, k, _, _ in WEIGHT_GRADIENTS])
    assert [(t, part > 0) for t, part in got] == [(t, cut) for *_, t, cut in WEIGHT_GRADIENTS]


def tensor(rows, cols, dt, seed, off):
    """Random (rows, cols) tensor with NaN between its rows, which start 16-byte
    aligned, or (`off`) an odd number of elements apart from an odd address."""
    ld, first = (cols | 1) + 2 if off else cols // 8 * 8 + 8, 1 if off else 0
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((first + rows * ld,), float("nan"), dtype=dt, device="cuda")
    t = buf[first:].view(rows, ld)[:, :cols]
    t.copy_(torch.randn(rows, cols, generator=g, device="cuda"))
    assert (t.data_ptr() % 16 == 0) != off and (t.stride(0) % 8 == 0) != off
    return t


def offsets_of(rows, experts, seed):
    """Three rows of no expert, experts of skewed sizes (some without rows), rest."""
    r = np.random.RandomState(seed)
    p = np.exp(0.8 * r.randn(experts))
    if experts >= 3:
        p[[experts // 2]] = 0.0
    sizes = r.multinomial(rows - 8, p / p.sum()) if rows > 100 else np.array([rows - 8])
    at = 3 + np.concatenate([[0], np.cumsum(sizes)])
    return at, torch.tensor(at, dtype=torch.int32, device="cuda")


def stack_of(experts, n, k, dt, seed, off):
    t = tensor(experts * n, k, dt, seed, off)
    return torch.as_strided(t, (experts, n, k), (n * t.stride(0), t.stride(0), 1), t.storage_offset())


def canvas(rows, cols, dt, off):
    """A view for a result and the buffer around it, of 7s."""
    ld = cols + 5 if off else cols // 8 * 8 + 8
    buf = torch.full((rows, ld), 7.0, dtype=dt, device="cuda")
    return buf[:, 1:1 + cols] if off else buf[:, :cols], buf


def right(got, a, b, half):
    want, mag = a @ b, a.abs() @ b.abs()
    bound = half * 1.01 * want.abs() + (a.shape[1] / 4 + 16) * 2.0 ** -23 * mag
    return bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("off", LAYOUTS)
@pytest.mark.parametrize("rows,experts,width,depth,tile", ROW_PRODUCTS)
def test_row_products_by_every_tile(rows, experts, width, depth, tile, off, dtype):
    dt = TYPES[dtype]
    half = torch.finfo(dt).eps / 2
    at, offsets = offsets_of(rows, experts, rows + width)
    x = tensor(rows, depth, dt, 1, off[0])
    x[:at[0]] = float("nan")
    x[at[-1]:] = float("inf")
    along, across = stack_of(experts, width, depth, dt, 2, off[1]), stack_of(experts, depth, width, dt, 3, off[1])
    for call, w, transpose in ((gr.lionmuon_grouped_product, along, True), (gr.lionmuon_grouped_input_grad, across, False)):
        out, buf = canvas(rows, width, dt, off[0])
        assert call(x, w, offsets, out=out) is out
        for e in range(experts):
            a, b = x[at[e]:at[e + 1]].double(), w[e].double()
            assert right(out[at[e]:at[e + 1]], a, b.t() if transpose else b, half), (call.__name__, e)
        assert (out[:at[0]] == 7).all() and (out[at[-1]:] == 7).all()
        first = 1 if off[0] else 0
        assert (buf[:, :first] == 7).all() and (buf[:, first + width:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("off", LAYOUTS)
@pytest.mark.parametrize("rows,experts,n,k,tile,cut", WEIGHT_GRADIENTS)
def test_weight_gradients_by_every_tile(rows, experts, n, k, tile, cut, off, dtype):
    dt = TYPES[dtype]
    at, offsets = offsets_of(rows, experts, rows + n)
    assert max(np.diff(at)) > (512 if experts <= 3 and rows > 300 else 60)
    dy, x = tensor(rows, n, dt, 4, off[0]), tensor(rows, k, dt, 5, off[1])
    values = x
    cases = [(x, False)]
    if dtype == "bf16":
        # from a checkpoint: scales copied four at a time (not `off`), or one by one
        kept = gr.lionmuon_checkpoint(x)
        blocks = kept.scales.shape[1]
        lds = blocks | 1 if off[1] else blocks // 4 * 4 + 4
        scales = torch.zeros(rows, lds, dtype=torch.uint8, device="cuda")[:, :blocks]
        scales.copy_(kept.scales)
        cases.append((gr.Checkpoint(kept.codes, scales), True))
        values = gr.lionmuon_checkpoint_restore(kept)
    for src, coded in cases:
        base = torch.full((experts * (n * (k + 3) + 2) + 1,), 0.5, device="cuda")
        out = torch.as_strided(base, (experts, n, k), (n * (k + 3) + 2, k + 3, 1), 1)
        dw = gr.lionmuon_grouped_weight_grad(dy, src, offsets)
        gr.lionmuon_grouped_weight_grad(dy, src, offsets, out=out, accumulate=True)
        assert torch.equal(out, 0.5 + dw)
        out.fill_(0.5)
        assert (base == 0.5).all()
        v = values if coded else x
        for e in range(experts):
            a, b = dy[at[e]:at[e + 1]].double(), v[at[e]:at[e + 1]].double()
            assert right(dw[e], a.t(), b, 0.0), (coded, e)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,depth", [(64, 64, 131072), (300, 1100, 32768), (2500, 2056, 16384)])
def test_long_contractions_of_one_sign(rows, width, depth, dtype):
    """The sums of a long contraction do not drift: the matrix unit adds 16 products at a
    time and rounds to nearest, so that depth / 16 independent errors of 2^-24 of a
    partial sum at most stay below eight times their root (the number of results is
    below 2^23). One-sided errors would reach depth / 32 * 2^-24, two to six times
    that, beside half a step of the result."""
    dt = TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(depth)
    x = (torch.rand(rows, depth, generator=g, device="cuda") * 0.5 + 0.5).to(dt)
    w = ((torch.rand(1, width, depth, generator=g, device="cuda") * 0.5 + 0.5) * 2.0 ** -6).to(dt)
    offsets = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    want = torch.zeros(rows, width, dtype=torch.float64, device="cuda")
    for c in range(0, depth, 8192):
        want += x[:, c:c + 8192].double() @ w[0, :, c:c + 8192].double().t()
    drift = 8 * 2.0 ** -24 * (depth / 16) ** 0.5
    across = w.transpose(1, 2).contiguous()
    for got in (gr.lionmuon_grouped_product(x, w, offsets), gr.lionmuon_grouped_input_grad(x, across, offsets)):
        assert ((got.double() - want).abs() <= (torch.finfo(dt).eps / 2 + drift) * want).all()
    # fp32 results are folded every 512: eight times the root of that, and as much for the folds
    dy, xt = w[0].t().contiguous(), x.t().contiguous()
    dw = gr.lionmuon_grouped_weight_grad(dy, xt, torch.tensor([0, depth], dtype=torch.int32, device="cuda"))[0]
    folds = 8 * 2.0 ** -24 * (32 ** 0.5 + (depth / 512) ** 0.5)
    assert ((dw.double() - want.t()).abs() <= folds * want.t()).all()
