"""Arrays without an alignment requirement (the forwards' h and weights, the prefills' W_UK and W_O) at any
element, in products large enough for the tiles that are copied straight to LDS: such operands go
through registers.

Tolerance against the aligned call: another kernel may take its products and add in another order, so a
rounding to bf16 may fall the other way; at most, then, both carry independent roundings, five each
(query latent, keys, values, probabilities, attention output), rms 1.7e-3: sqrt(10) 1.7e-3 = 5.4e-3 of the
norm, 6e-3 allowed."""
import numpy as np
import pytest

from test_gpu_paged import Layer, Prefill, check_prefill, offsets, shape
from test_gpu_prefill import _run, _setup
from test_gpu_robustness import _case

pytestmark = pytest.mark.gpu

REL = 6e-3


def moved(t, shift):
    """A copy of t whose first element lies `shift` elements past a 16-byte boundary."""
    import torch
    b = torch.empty(t.numel() + 8, dtype=t.dtype, device=t.device)
    b[shift:shift + t.numel()] = t.reshape(-1)
    return b[shift:shift + t.numel()]


@pytest.mark.parametrize("name,n", [("tiny", 300), ("05b", 700), ("1b", 400), ("8b", 3000)])
@pytest.mark.parametrize("shift", [1, 2, 4])
def test_paged_prefill_w_uk(name, n, shift):
    print(f"[unaligned] paged prefill {name} {n} rows, W_UK moved by {shift}", flush=True)
    lay = Layer(shape(name), [n], 64, seed=n + shift)
    q = lay.queries(3)
    lay.d_Wuk = moved(lay.d_Wuk, shift)
    check_prefill(lay, q, offsets([3]), [n], Prefill(lay, q, offsets([3]), offsets([n]))())


@pytest.mark.parametrize("idx,T", [(1, 600), (3, 520)])
@pytest.mark.parametrize("form", ["o+A", "o+folded"])
def test_prefill_weights(idx, T, form):
    import torch
    cfg, c, x = _setup(idx, 1, T)
    o, A = _run(cfg, c, x, form)
    for shift in (1, 4):
        y = dict(x, **{n: moved(x[n], shift) for n in ("Wuk", "Wo", "fold")})
        print(f"[unaligned] prefill cfg{idx} T={T} {form} weights moved by {shift}", flush=True)
        for a, b in zip(_run(cfg, c, y, form), (o, A)):
            assert torch.isfinite(a).all() and (a.float() - b.float()).norm() <= REL * b.float().norm()


@pytest.mark.parametrize("idx,T", [(1, 700), (2, 1100), (3, 513)])
def test_forward_arrays(idx, T):
    import torch
    from paper_2607_27269_amd import _lib as L
    from paper_2607_27269_amd.step import DeviceStep
    cfg, wl = _case(idx, 1, T, None)
    dev = DeviceStep(wl)
    names = [n for n in ("h", "Wq", "Wk", "Wv", "Wo", "Wdq", "Wuq", "Wdkv_kr", "Wuk", "Wuv")
             if getattr(dev, n) is not None]
    outs = []
    for shift in (0, 1, 4):
        print(f"[unaligned] forwards cfg{idx} T={T} moved by {shift}", flush=True)
        x = {n: moved(getattr(dev, n), shift) for n in names}
        p = lambda n: x[n].data_ptr() if n in x else None
        A = torch.full((2,) + tuple(dev.A_t.shape), float("nan"), device=dev.A_t.device)
        tw = L.TeacherW(p("Wq"), p("Wk"), p("Wv"), p("Wo"), dev.inv_freq_t.data_ptr())
        sw = L.StudentW(p("Wdq"), p("Wuq"), p("Wdkv_kr"), p("Wuk"), p("Wuv"), dev.inv_freq_s.data_ptr())
        L.mla_recon_teacher_fwd(dev.ccfg, p("h"), tw, A[0].data_ptr(), dev.ws.data_ptr(), dev.ws_bytes, dev.stream)
        L.mla_recon_student_fwd(dev.ccfg, p("h"), sw, p("Wo"), A[1].data_ptr(), dev.ws.data_ptr(), dev.ws_bytes,
                                dev.stream)
        torch.cuda.synchronize()
        outs.append(A)
    assert torch.isfinite(outs[0]).all()
    for A in outs[1:]:
        for a, b in zip(A, outs[0]):
            assert torch.isfinite(a).all() and (a - b).norm() <= REL * b.norm()
