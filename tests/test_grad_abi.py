"""Host-side tests of ``include/lionmuon_grad.h`` (no GPU needed): exported names,
workspace sizes, and every refusal, which comes before any device work."""
import ctypes
import os
import re

import pytest

from paper_2605_19811_amd import gradients as gr
from paper_2605_19811_amd import lionmuon as lm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "lionmuon_grad.h")
BAD, UNSUPPORTED, SMALL = (lm.LM_ERR_INVALID_ARGUMENT, lm.LM_ERR_UNSUPPORTED,
                           lm.LM_ERR_WORKSPACE_TOO_SMALL)
F32, BF16, F16 = 0, 1, 2
BASE = 1 << 40                        # addresses that nothing dereferences
GAP = 1 << 32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lm.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return gr._lib()


def at(i):
    return BASE + i * GAP


def mat(i, rows, cols, ld=None, dtype=BF16, reserved=0, data=None):
    return gr.lm_matrix(at(i) if data is None else data, rows, cols, cols if ld is None else ld,
                        dtype, reserved)


def stack(i, count, rows, cols, ld=None, stride=None, dtype=BF16, reserved=0, data=None):
    ld = cols if ld is None else ld
    return gr.lm_stack(at(i) if data is None else data, count, rows, cols, ld,
                       rows * ld if stride is None else stride, dtype, reserved)


def kept(i, rows, cols, ld=None, lds=None, codes=None, scales=None):
    return gr.lm_checkpoint(at(i) if codes is None else codes,
                            at(i) + GAP // 2 if scales is None else scales, rows, cols,
                            -(-cols // 16) * 16 if ld is None else ld,
                            -(-cols // 128) if lds is None else lds)


def refused(lib, status, want=BAD, text=""):
    assert status == want
    message = lib.lionmuon_last_error().decode()
    assert message and text in message, message


def test_header_declares_the_binding_names(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(lionmuon_\w+)\s*\(", text)))
    assert names == sorted(gr.GRAD_EXPORTED)
    for name in names:
        assert hasattr(lib, name)
    assert f"LM_CHECKPOINT_BLOCK {gr.CHECKPOINT_BLOCK}" in text
    assert f"LM_RMSNORM_MAX_COLS {gr.RMSNORM_MAX_COLS}" in text


def test_structs_have_the_sizes_of_the_header():
    assert [ctypes.sizeof(t) for t in (gr.lm_matrix, gr.lm_stack, gr.lm_checkpoint)] == [40, 56, 48]


@pytest.mark.parametrize("change,text", [
    (dict(dtype=3), "dtype"), (dict(reserved=1), "reserved"), (dict(ld=63), "ld"), (dict(rows=-1), "negative"),
    (dict(ld=1 << 22), "2^22"), (dict(rows=1 << 31), "rows"), (dict(data=0), "null"),
    (dict(data=BASE + 1), "misaligned")])
def test_matrix_descriptors(lib, change, text):
    args = dict(rows=8, cols=64)
    args.update({k: v for k, v in change.items() if k in args})
    m = mat(0, **args, **{k: v for k, v in change.items() if k not in args})
    refused(lib, lib.lionmuon_checkpoint(m, kept(1, args["rows"] if args["rows"] > 0 else 8, 64), None), text=text)


@pytest.mark.parametrize("change,text", [
    (dict(ld=72), "16"), (dict(ld=48), "ld_codes"), (dict(lds=0), "ld_scales"), (dict(codes=BASE + GAP + 8), "aligned"),
    (dict(codes=0), "null"), (dict(scales=0), "null")])
def test_checkpoint_descriptors(lib, change, text):
    refused(lib, lib.lionmuon_checkpoint(mat(0, 8, 64), kept(1, 8, 64, **change), None), text=text)
    refused(lib, lib.lionmuon_checkpoint_restore(kept(1, 8, 64, **change), mat(0, 8, 64), None), text=text)


def test_checkpoint_shapes_and_overlaps(lib):
    refused(lib, lib.lionmuon_checkpoint(mat(0, 8, 64), kept(1, 8, 65), None), text="shape")
    refused(lib, lib.lionmuon_checkpoint(None, kept(1, 8, 64), None), text="null")
    refused(lib, lib.lionmuon_checkpoint(mat(0, 8, 64), None, None), text="null")
    refused(lib, lib.lionmuon_checkpoint(mat(0, 8, 64), kept(0, 8, 64, codes=at(0) + 512), None), text="overlap")
    refused(lib, lib.lionmuon_checkpoint(mat(0, 8, 64), kept(1, 8, 64, scales=at(1) + 16), None), text="overlap")
    refused(lib, lib.lionmuon_checkpoint_restore(kept(1, 8, 64), mat(1, 8, 64), None), text="overlap")
    # nothing to do
    assert lib.lionmuon_checkpoint(mat(0, 0, 64, data=0), kept(1, 0, 64, codes=0, scales=0), None) == lm.LM_OK
    assert lib.lionmuon_checkpoint(mat(0, 5, 0), kept(1, 5, 0), None) == lm.LM_OK


def test_views_side_by_side_do_not_overlap(lib):
    """Columns of one buffer: refused where they overlap only (rows = 0 in the
    product ends a valid call before the device)."""
    two = mat(0, 4, 128, ld=192, dtype=F32)
    for shift, ok in ((128, True), (127, False), (64, False), (0, False)):
        out = mat(0, 4, 64, ld=192, dtype=F32, data=at(0) + shift * 4)
        status = lib.lionmuon_activation(two, 1, out, kept(9, 4, 127), None)     # wrong shape
        refused(lib, status, text="shape")
        status = lib.lionmuon_rmsnorm_grad(mat(1, 4, 64, dtype=F32), out, None, at(2), at(3), None,
                                           mat(0, 4, 64, ld=192, dtype=F32), None, 2, None, 0, None)
        refused(lib, status, text="accumulate")
        status = lib.lionmuon_activation_grad(out, None, kept(9, 4, 128), 1, two, mat(0, 4, 64, dtype=F32), None)
        refused(lib, status, text="overlap")


def test_activation_arguments(lib):
    f = lib.lionmuon_activation
    a, h = mat(0, 8, 128), mat(1, 8, 64)
    refused(lib, f(a, 2, h, None, None), text="kind")
    refused(lib, f(a, 0, h, None, None), text="shape")
    refused(lib, f(mat(0, 8, 64), 1, h, None, None), text="shape")
    refused(lib, f(mat(0, 8, 128, dtype=F16), 1, h, None, None), text="type")
    refused(lib, f(a, 1, h, kept(2, 8, 64), None), text="shape")
    refused(lib, f(a, 1, mat(0, 8, 64), None, None), text="overlap")
    refused(lib, f(a, 1, h, kept(1, 8, 128), None), text="overlap")
    g = lib.lionmuon_activation_grad
    dh, da = mat(2, 8, 64), mat(3, 8, 128)
    refused(lib, g(dh, None, None, 1, da, None, None), text="either")
    refused(lib, g(dh, a, kept(4, 8, 128), 1, da, None, None), text="either")
    refused(lib, g(dh, a, None, 1, mat(3, 8, 64), None, None), text="shape")
    refused(lib, g(dh, mat(0, 8, 64), None, 1, da, None, None), text="shape")
    refused(lib, g(dh, None, kept(4, 8, 64), 1, da, None, None), text="shape")
    refused(lib, g(dh, mat(0, 8, 128, dtype=F32), None, 1, da, None, None), text="type")
    refused(lib, g(dh, a, None, 1, mat(3, 8, 128, dtype=F32), None, None), text="type")
    refused(lib, g(dh, a, None, 1, da, mat(5, 8, 128), None), text="shape")
    refused(lib, g(dh, a, None, 1, da, mat(3, 8, 64), None), text="overlap")
    refused(lib, g(dh, a, None, 1, mat(0, 8, 128), None, None), text="overlap")
    assert g(mat(2, 0, 64), mat(0, 0, 128), None, 1, mat(3, 0, 128), None, None) == lm.LM_OK


def test_norm_arguments(lib):
    f = lib.lionmuon_rmsnorm
    x, y, w = mat(0, 8, 64), mat(1, 8, 64), at(2)
    refused(lib, f(x, None, None, 1e-5, y, None, None, None, None), text="weight")
    refused(lib, f(x, None, w + 2, 1e-5, y, None, None, None, None), text="weight")
    for eps in (-1e-5, float("nan"), float("inf")):
        refused(lib, f(x, None, w, eps, y, None, None, None, None), text="eps")
    refused(lib, f(x, None, w, 1e-5, y, mat(3, 8, 64), None, None, None), text="residual")
    refused(lib, f(x, mat(3, 8, 65), w, 1e-5, y, None, None, None, None), text="shape")
    refused(lib, f(x, mat(3, 8, 64, dtype=F16), w, 1e-5, y, None, None, None, None), text="type")
    refused(lib, f(x, None, w, 1e-5, mat(0, 8, 64), None, None, None, None), text="overlap")
    refused(lib, f(x, None, w, 1e-5, y, None, at(1) + 16, None, None), text="overlap")
    refused(lib, f(x, None, w, 1e-5, y, None, at(4) + 2, None, None), text="rstd")
    refused(lib, f(x, None, w, 1e-5, y, None, None, kept(4, 8, 63), None), text="shape")
    # the sum may be the residual itself, nothing else of it
    refused(lib, f(x, mat(3, 8, 64), w, 1e-5, y, mat(3, 8, 64, data=at(3) + 128), None, None, None), text="overlap")
    refused(lib, f(mat(0, 8, 0), None, w, 1e-5, None, None, None, None, None), text="element")
    refused(lib, f(mat(0, 2, 16385), None, w, 1e-5, None, None, None, None, None), UNSUPPORTED, "16384")
    assert f(mat(0, 0, 64), None, w, 1e-5, mat(1, 0, 64), None, None, None, None) == lm.LM_OK


def test_norm_gradient_arguments(lib):
    g = lib.lionmuon_rmsnorm_grad
    dy, s, w, r, dx, dw = mat(0, 8, 64), mat(1, 8, 64), at(2), at(3), mat(4, 8, 64), at(5)
    need = gr.lionmuon_rmsnorm_workspace_bytes(8, 64)
    assert need == 2 * 64 * 4                       # two workgroups of four rows
    ok = dict(dy=dy, s=s, kept=None, w=w, r=r, res=None, dx=dx, dw=dw, acc=0, ws=at(6), n=need)

    def call(**kw):
        a = {**ok, **kw}
        return g(a["dy"], a["s"], a["kept"], a["w"], a["r"], a["res"], a["dx"], a["dw"], a["acc"],
                 a["ws"], a["n"], None)

    refused(lib, call(s=None), text="either")
    refused(lib, call(kept=kept(7, 8, 64)), text="either")
    refused(lib, call(s=None, kept=kept(7, 8, 65)), text="shape")
    refused(lib, call(w=None), text="weight")
    refused(lib, call(r=None), text="rstd")
    refused(lib, call(acc=2), text="accumulate")
    refused(lib, call(dw=dw + 1), text="dweight")
    refused(lib, call(s=mat(1, 8, 64, dtype=F32)), text="type")
    refused(lib, call(dx=mat(4, 7, 64)), text="shape")
    refused(lib, call(n=need - 1), SMALL, str(need))
    refused(lib, call(ws=None, n=0), SMALL)
    refused(lib, call(ws=None), text="both")
    refused(lib, call(ws=at(6) + 64), text="256")
    refused(lib, call(dx=mat(0, 8, 64)), text="overlap")
    refused(lib, call(ws=at(1)), text="overlap")
    refused(lib, call(dw=at(4) + 64), text="overlap")
    refused(lib, call(res=mat(4, 8, 64, data=at(4) + 2)), text="overlap")
    refused(lib, call(dy=mat(0, 8, 16385), s=mat(1, 8, 16385)), UNSUPPORTED)
    assert call(dx=None, dw=None, ws=None, n=0) == lm.LM_OK
    with pytest.raises(lm.LionMuonError):
        gr.lionmuon_rmsnorm_workspace_bytes(8, 0)
    with pytest.raises(lm.LionMuonError):
        gr.lionmuon_rmsnorm_workspace_bytes(-1, 8)


def test_grouped_arguments(lib):
    p, d = lib.lionmuon_grouped_product, lib.lionmuon_grouped_input_grad
    x, w, off, y, dy = mat(0, 8, 64), stack(1, 3, 32, 64), at(2), mat(3, 8, 32), mat(4, 8, 32)
    refused(lib, p(x, w, None, y, None), text="offsets")
    refused(lib, p(x, w, off + 2, y, None), text="offsets")
    refused(lib, p(x, stack(1, 3, 32, 65), off, y, None), text="columns")
    refused(lib, p(x, w, off, mat(3, 8, 33), None), text="shape")
    refused(lib, p(x, w, off, mat(3, 7, 32), None), text="shape")
    refused(lib, p(x, stack(1, 0, 32, 64), off, y, None), text="expert")
    refused(lib, p(mat(0, 8, 0), stack(1, 3, 32, 0), off, y, None), text="at least 1")
    refused(lib, p(x, stack(1, 3, 32, 64, stride=32 * 64 - 1), off, y, None), text="stride")
    refused(lib, p(x, stack(1, 3, 32, 64, reserved=1), off, y, None), text="reserved")
    refused(lib, p(x, stack(1, 3, 32, 64, data=0), off, y, None), text="null")
    refused(lib, p(x, stack(1, 3, 32, 64, dtype=F16), off, y, None), text="type")
    refused(lib, p(mat(0, 8, 64, dtype=F32), stack(1, 3, 32, 64, dtype=F32), off, mat(3, 8, 32, dtype=F32), None), UNSUPPORTED)
    refused(lib, p(x, w, off, mat(3, 8, 32, data=at(0) + 64), None), text="overlap")
    refused(lib, p(x, w, off, mat(3, 8, 32, data=at(2)), None), text="overlap")
    refused(lib, p(mat(0, 1 << 30, 64), w, off, mat(3, 1 << 30, 32), None), text="rows")
    assert p(mat(0, 0, 64, data=0), w, off, mat(3, 0, 32, data=0), None) == lm.LM_OK
    refused(lib, d(mat(4, 8, 33), w, off, mat(5, 8, 64), None), text="columns")
    refused(lib, d(dy, w, off, mat(5, 8, 63), None), text="shape")
    refused(lib, d(dy, w, off, mat(5, 8, 64, dtype=F16), None), text="type")
    refused(lib, d(dy, w, off, mat(1, 8, 64), None), text="overlap")
    assert d(mat(4, 0, 32), w, off, mat(5, 0, 64), None) == lm.LM_OK


def test_weight_gradient_arguments(lib):
    g = lib.lionmuon_grouped_weight_grad
    dy, x, off = mat(0, 8, 32), mat(1, 8, 64), at(2)
    dw = stack(3, 3, 32, 64, dtype=F32)
    refused(lib, g(dy, None, None, off, dw, 0, None, 0, None), text="either")
    refused(lib, g(dy, x, kept(4, 8, 64), off, dw, 0, None, 0, None), text="either")
    refused(lib, g(dy, x, None, None, dw, 0, None, 0, None), text="offsets")
    refused(lib, g(dy, x, None, off, dw, 2, None, 0, None), text="accumulate")
    refused(lib, g(dy, x, None, off, stack(3, 3, 32, 64), 0, None, 0, None), text="fp32")
    refused(lib, g(dy, x, None, off, stack(3, 3, 33, 64, dtype=F32), 0, None, 0, None), text="columns")
    refused(lib, g(dy, mat(1, 8, 65), None, off, dw, 0, None, 0, None), text="shape")
    refused(lib, g(dy, mat(1, 8, 64, dtype=F16), None, off, dw, 0, None, 0, None), text="type")
    refused(lib, g(dy, None, kept(4, 9, 64), off, dw, 0, None, 0, None), text="shape")
    refused(lib, g(mat(0, 8, 32, dtype=F16), None, kept(4, 8, 64), off, dw, 0, None, 0, None), UNSUPPORTED, "bf16")
    refused(lib, g(mat(0, 8, 32, dtype=F32), mat(1, 8, 64, dtype=F32), None, off, dw, 0, None, 0, None), UNSUPPORTED)
    refused(lib, g(dy, x, None, off, stack(1, 3, 32, 64, dtype=F32), 0, None, 0, None), text="overlap")
    refused(lib, g(dy, x, None, off, dw, 0, at(5) + 1, 512, None), text="256")
    refused(lib, g(dy, x, None, off, dw, 0, None, 512, None), text="both")
    rows, n, k = 1 << 16, 64, 64
    need = gr.lionmuon_grouped_workspace_bytes(rows, 1, n, k)
    assert need % (n * k * 4) == 0 and need // (n * k * 4) >= 2       # whole partials
    big = mat(0, rows, n), mat(1, rows, k), None, off, stack(3, 1, n, k, dtype=F32), 0
    refused(lib, g(*big, None, 0, None), SMALL)
    refused(lib, g(*big, at(5), need - 4, None), SMALL, str(need))
    refused(lib, g(*big, at(3), need, None), text="overlap")
    for bad in ((-1, 1, 8, 8), (8, 0, 8, 8), (8, 1, 0, 8), (8, 1, 8, 0), (8, 1, 1 << 22, 8), (1 << 30, 1, 8, 8)):
        with pytest.raises(lm.LionMuonError):
            gr.lionmuon_grouped_workspace_bytes(*bad)
    assert gr.lionmuon_grouped_workspace_bytes(0, 5, 8, 8) == 0


def test_binding_refuses_host_tensors_and_wrong_kinds():
    import torch
    x = torch.zeros(4, 64)
    for call in (lambda: gr.lionmuon_checkpoint(x), lambda: gr.lionmuon_activation(x, "gelu"),
                 lambda: gr.lionmuon_rmsnorm(x, torch.ones(64)),
                 lambda: gr.lionmuon_rmsnorm_grad(x, x, torch.ones(64), torch.ones(4)),
                 lambda: gr.lionmuon_grouped_product(x, torch.zeros(1, 8, 64), torch.tensor([0, 4])),
                 lambda: gr.lionmuon_grouped_input_grad(x, torch.zeros(1, 64, 8), torch.tensor([0, 4])),
                 lambda: gr.lionmuon_grouped_weight_grad(x, x, torch.tensor([0, 4])),
                 lambda: gr.lionmuon_checkpoint_restore(gr.Checkpoint.empty(4, 64, "cpu"))):
        with pytest.raises(lm.LionMuonError) as e:
            call()
        assert e.value.status == BAD
    with pytest.raises(ValueError):
        gr.lionmuon_activation(x, "relu")
    with pytest.raises(TypeError):
        gr.lionmuon_checkpoint([1.0])
    with pytest.raises(TypeError):
        gr.lionmuon_checkpoint_restore(x)
    u8 = torch.uint8
    with pytest.raises(lm.LionMuonError):
        gr.Checkpoint(torch.zeros(4, 64), torch.zeros(4, 1, dtype=u8))
    with pytest.raises(lm.LionMuonError):
        gr.Checkpoint(torch.zeros(4, 129, dtype=u8), torch.zeros(4, 1, dtype=u8))
    k = gr.Checkpoint.empty(3, 129, "cpu")
    assert k.shape == (3, 129) and k.codes.stride(0) == 144 and k.scales.shape == (3, 2)


def test_products_too_large_for_a_launch_are_refused(lib):
    w = stack(1, 1 << 16, 16384, 64)
    refused(lib, lib.lionmuon_grouped_product(mat(0, 1 << 26, 64), w, at(2), mat(3, 1 << 26, 16384), None),
            UNSUPPORTED, "tiles")
    refused(lib, lib.lionmuon_grouped_weight_grad(mat(0, 8, 16384), mat(4, 8, 64), None, at(2),
                                                  stack(1, 1 << 16, 16384, 64, dtype=F32), 0, None, 0, None),
            UNSUPPORTED, "tiles")
    refused(lib, lib.lionmuon_grouped_product(mat(0, 8, 64), stack(1, (1 << 16) + 1, 8, 64), at(2),
                                              mat(3, 8, 8), None), UNSUPPORTED, "experts")
    refused(lib, lib.lionmuon_grouped_product(mat(0, 1 << 30, 64), stack(1, 1, 8, 64), at(2),
                                              mat(3, 1 << 30, 8), None), BAD, "rows")


def test_checkpoint_with_a_short_last_row_of_scales_is_refused():
    import torch
    u8 = torch.uint8
    scales = torch.as_strided(torch.zeros(7, dtype=u8), (2, 3), (4, 1))
    with pytest.raises(lm.LionMuonError):
        gr.Checkpoint(torch.zeros(2, 384, dtype=u8), scales)
    gr.Checkpoint(torch.zeros(2, 384, dtype=u8), torch.as_strided(torch.zeros(8, dtype=u8), (2, 3), (4, 1)))


def test_checkpoint_with_codes_that_end_inside_16_bytes_is_refused():
    """Writers put 0 behind a row's last code up to a multiple of 16 bytes: these
    have to be bytes of that row, in a single row and in the last one too."""
    import torch
    u8 = torch.uint8

    def make(codes):
        return gr.Checkpoint(codes, torch.zeros(codes.shape[0], -(-codes.shape[1] // 128), dtype=u8))

    large = torch.zeros(4096, dtype=u8)
    for codes in (torch.zeros(1, 100, dtype=u8),                     # a row without the bytes behind it
                  large[:100].view(1, 100),                          # those behind it are another's
                  large[:17].view(1, 17),
                  torch.as_strided(torch.zeros(49, dtype=u8), (2, 17), (32, 1)),     # the last row ends early
                  torch.as_strided(torch.zeros(4095, dtype=u8), (3, 100), (112, 1), 4095 - 324),
                  torch.zeros(3, 100, dtype=u8)):                    # rows side by side
        with pytest.raises(lm.LionMuonError) as e:
            make(codes)
        assert e.value.status == BAD and "16 bytes" in str(e.value)
    for rows, cols, codes in ((1, 100, torch.zeros(1, 112, dtype=u8)[:, :100]),
                              (1, 17, large.view(16, 256)[3:4, :17]),
                              (1, 128, large[:128].view(1, 128)),
                              (2, 17, torch.as_strided(torch.zeros(64, dtype=u8), (2, 17), (32, 1))),
                              (3, 100, torch.as_strided(torch.zeros(4096, dtype=u8), (3, 100), (112, 1), 4096 - 336)),
                              (0, 100, torch.zeros(0, 100, dtype=u8)), (3, 0, torch.zeros(3, 0, dtype=u8))):
        k = make(codes)
        d = k._desc
        assert k.shape == (rows, cols) and d.ld_codes >= -(-cols // 16) * 16
        if rows and cols:
            end = (rows - 1) * d.ld_codes + -(-cols // 16) * 16
            assert codes.storage_offset() + end <= codes.untyped_storage().nbytes()


def test_checkpoint_is_described_as_its_tensors_are_at_the_call():
    """Tensors whose storage was exchanged (``set_``, ``.data``) or resized since the
    checkpoint was made: the next call gets the new memory, or is refused."""
    import torch
    u8 = torch.uint8

    def place(k):
        return k._desc.codes, k._desc.scales

    codes, scales = torch.zeros(3, 256, dtype=u8), torch.zeros(3, 2, dtype=u8)
    k = gr.Checkpoint(codes, scales)
    assert place(k) == (codes.data_ptr(), scales.data_ptr())
    before, old = codes.data_ptr(), codes.untyped_storage()      # (kept: the new one lies elsewhere)
    codes.set_(torch.zeros(3, 256, dtype=u8))
    scales.data = torch.ones(3, 2, dtype=u8)
    assert place(k) == (codes.data_ptr(), scales.data_ptr()) and codes.data_ptr() != before
    assert k.codes is codes and old.data_ptr() == before
    # another layout is read anew, another shape or type is not the checkpoint any more
    codes.set_(torch.zeros(3, 512, dtype=u8)[:, :256])
    assert k._desc.ld_codes == 512
    for other in (torch.zeros(4, 256, dtype=u8), torch.zeros(3, 255, dtype=u8)):
        codes.data = other
        with pytest.raises(lm.LionMuonError):
            k._desc
    codes.data = torch.as_strided(torch.zeros(768, dtype=u8), (3, 256), (1, 3))
    with pytest.raises(lm.LionMuonError):
        k._desc
    # storage given back and taken again, of tensors passed in and of an allocated one
    codes, scales = torch.zeros(3, 240, dtype=u8), torch.zeros(3, 2, dtype=u8)
    k, own = gr.Checkpoint(codes, scales), gr.Checkpoint.empty(5, 300, "cpu")
    for c in (k, own):
        storage = c.codes.untyped_storage()
        size = storage.nbytes()
        storage.resize_(0)
        assert not c._desc.codes                       # refused by the entry points: null data
        storage.resize_(size)
        d = c._desc
        assert d.codes == storage.data_ptr() == c.codes.data_ptr() and d.scales == c.scales.data_ptr()
