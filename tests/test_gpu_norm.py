"""si_norm against its formula in 64 bits.

Tolerance of an output: half a step of its type (finfo.eps / 2, relative) for the rounding, and 128 roundings of fp32 (2^-24 each) of the
terms that form it.  A sum over a row is at most 32 additions in a thread and 10 levels above them, so its relative error is below 42 x 2^-24 of
the sum of the terms' magnitudes; a norm takes two such sums, N2 reads what N1 left, and the few operations around them stay within
the rest."""
import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si

TYPES = {"bf16": (torch.bfloat16, si.SI_BF16), "f32": (torch.float32, si.SI_F32)}
KINDS = {"none": si.SI_NORM_NONE, "rms": si.SI_NORM_RMS, "mean": si.SI_NORM_MEAN}
FP32 = 128 * 2.0 ** -24


def norm64(x, m, kind, w, b, eps):
    """N(x) and the magnitude of the terms that form it, given the magnitude m of those that formed x; rows of float64"""
    if kind == "none":
        return x, m
    mu = x.mean(1, keepdims=True) if kind == "mean" else 0.0
    mm = m + (m.mean(1, keepdims=True) if kind == "mean" else 0.0)
    z = x - mu
    rs = 1.0 / np.sqrt((z * z).mean(1, keepdims=True) + eps)
    w = 1.0 if w is None else w
    b = 0.0 if b is None else b
    # an error of the terms moves the second moment too: |z| rs of the element times the rows' mean of rs m
    scale = np.abs(z) * rs * np.sqrt((mm * mm).mean(1, keepdims=True)) * rs
    return z * rs * w + b, (mm * rs + scale) * np.abs(w) + np.abs(b)


def residual64(r, y, gate, a, b, eps, post, w1, b1, pre, w2, b2):
    out, m = 0.0, 0.0
    if y is not None:
        v, mv = norm64(y, np.abs(y), post, w1, b1, eps)
        g = 1.0 if gate is None else gate
        out, m = b * g * v, np.abs(b * g) * mv
    if r is not None:
        out, m = out + a * r, m + np.abs(a * r)
    return (out, m), norm64(out, m, pre, w2, b2, eps)


def close(got, want, m, kind):
    half = torch.finfo(TYPES[kind][0]).eps / 2
    err = np.abs(got.double().cpu().numpy() - want)
    tol = half * np.abs(want) + (1 + half) * FP32 * m
    assert np.all(err <= tol), "worst %.3g of its tolerance" % np.max(err / np.maximum(tol, 1e-300))


def _rows(rng, rows, d, kind, scale, pad, offset=0.0):
    """[rows][d] inside rows of d + pad elements; returns the view and its float64 values"""
    t = torch.from_numpy(rng.standard_normal((rows, d + pad)).astype(np.float32) * scale + offset).to("cuda", TYPES[kind][0])
    return t[:, :d], t[:, :d].double().cpu().numpy()


def run_case(rows, d, r="bf16", y="f32", gate="none", w="bf16", r_out="bf16", out="bf16", post="none", pre="rms", bias=False, pad=0, a=1.0, b=1.0,
             broadcast_gate=False, in_place=False, offset=0.0, eps=1e-5, weights=True, seed=0):
    rng = np.random.default_rng(1000 * rows + d + seed)
    desc = si.si_norm_t(rows=rows, d=d, post=KINDS[post], pre=KINDS[pre], eps=eps, res_scale=a, y_scale=b, w_type=TYPES[w][1])
    keep, val = {}, {}
    for name, kind, scale in (("r", r, 4.0), ("y", y, 0.5), ("gate", gate, 1.0)):
        if kind == "none":
            val[name] = None
            continue
        one = name == "gate" and broadcast_gate
        keep[name], val[name] = _rows(rng, 1 if one else rows, d, kind, scale, pad, offset)
        setattr(desc, name, keep[name].data_ptr())
        setattr(desc, name + "_type", TYPES[kind][1])
        setattr(desc, name + "_stride", 0 if one else d + pad)
    for name, on in (("w_post", post != "none" and weights), ("b_post", post != "none" and bias), ("w_pre", pre != "none" and weights), ("b_pre", pre != "none" and bias)):
        val[name] = None
        if on:
            t = torch.from_numpy((0.2 * rng.standard_normal(d) + (name[0] == "w")).astype(np.float32)).to("cuda", TYPES[w][0])
            keep[name], val[name] = t, t.double().cpu().numpy()
            setattr(desc, name, t.data_ptr())
    for name, kind in (("r_out", r_out), ("out", out)):
        if kind == "none":
            continue
        if in_place and name == "r_out":
            keep[name] = keep["r"]
        else:
            keep[name] = torch.full((rows, d + pad), 77.0, dtype=TYPES[kind][0], device="cuda")[:, :d]
        setattr(desc, name, keep[name].data_ptr())
        setattr(desc, name + "_type", TYPES[kind][1])
        setattr(desc, name + "_stride", d + pad)
    print("si_norm", dict(rows=rows, d=d, r=r, y=y, gate=gate, post=post, pre=pre, pad=pad), flush=True)
    si.si_norm(desc, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    (r64, mr), (o64, mo) = residual64(val["r"], val["y"], val["gate"], float(np.float32(a)), float(np.float32(b)), float(np.float32(eps)), post,
                                      val["w_post"], val["b_post"], pre, val["w_pre"], val["b_pre"])
    if r_out != "none":
        close(keep["r_out"], r64, mr, r_out)
    if out != "none":
        close(keep["out"], o64, mo, out)
    for name, kind in (("r_out", r_out), ("out", out)):
        if kind != "none" and pad and not in_place:
            full = keep[name].as_strided((rows, d + pad), (d + pad, 1))
            assert bool((full[:, d:] == 77.0).all()), "written beyond a row's end"


pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [1, 7, 8, 63, 64, 65, 127, 129, 255, 257, 511, 512, 513, 1000, 2047, 2049, 4096, 4097, 6144, 8191, 8192, 12288, 16384, 20001, 32768])
def test_widths(d):
    run_case(5, d, post="rms", pre="mean", bias=True, gate="bf16", b=0.7)
    run_case(3, d, r="f32", r_out="f32", y="bf16", pre="rms", pad=3)


@pytest.mark.parametrize("rows", [1, 2, 31, 33, 300, 5000])
@pytest.mark.parametrize("d", [72, 1537])
def test_rows(rows, d):
    run_case(rows, d, post="mean", pre="rms", bias=True)


@pytest.mark.parametrize("r", ["bf16", "f32", "none"])
@pytest.mark.parametrize("y", ["bf16", "f32", "none"])
@pytest.mark.parametrize("gate", ["none", "bf16", "f32"])
def test_types_and_missing_terms(r, y, gate):
    if r == "none" and y == "none":
        pytest.skip("refused")
    run_case(9, 321, r=r, y=y, gate=gate, post="rms" if y != "none" else "none", w="f32", r_out="f32", out="f32", a=0.5, b=-1.25, pad=1)


@pytest.mark.parametrize("post", ["none", "rms", "mean"])
@pytest.mark.parametrize("pre", ["none", "rms", "mean"])
@pytest.mark.parametrize("bias", [False, True])
def test_kinds(post, pre, bias):
    run_case(6, 777, post=post, pre=pre, bias=bias, gate="f32")
    run_case(6, 96, post=post, pre=pre, bias=bias, weights=False, out="f32")


def test_one_output_only():
    run_case(4, 500, out="none")
    run_case(4, 500, r_out="none")


def test_in_place_and_a_gate_of_one_row():
    run_case(17, 4099, in_place=True, gate="bf16", broadcast_gate=True, post="rms")


def test_a_mean_far_from_zero():
    """N_mean of rows whose mean is 1000 times their spread: the second moment is taken about the mean."""
    run_case(4, 3001, r="none", y="f32", post="none", pre="mean", r_out="f32", out="f32", offset=500.0)


def test_large_and_small_values():
    for scale in (1e-18, 1e15):
        x = torch.randn((3, 640), device="cuda") * scale
        out = torch.empty_like(x)
        si.si_norm(si.si_norm_t(r=x.data_ptr(), out=out.data_ptr(), r_stride=640, out_stride=640, rows=3, d=640, pre=si.SI_NORM_RMS, eps=0.0,
                                res_scale=1.0), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        v = x.double().cpu().numpy()
        want = v / np.sqrt((v * v).mean(1, keepdims=True))
        close(out, want, np.abs(want) + 1.0, "f32")


def test_a_row_with_nan_keeps_it_to_itself():
    x = torch.randn((4, 200), device="cuda")
    x[2, 5] = float("nan")
    out = torch.empty_like(x)
    si.si_norm(si.si_norm_t(r=x.data_ptr(), out=out.data_ptr(), r_stride=200, out_stride=200, rows=4, d=200, pre=si.SI_NORM_RMS, eps=1e-5,
                            res_scale=1.0), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.isnan(out[2]).all() and torch.isfinite(out[[0, 1, 3]]).all()
