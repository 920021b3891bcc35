"""si_norm with an output in the place of an input, for widths whose last slot overlaps the one before (no multiple of 8, more than 512): what two threads read is
read by both before either writes, with a norm after it and without.  Comparison and tolerances are those of test_gpu_norm.py."""
import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
from test_gpu_norm import KINDS, TYPES, close, residual64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [5, 60, 511, 513, 2049, 4099, 6143, 6151, 9001, 20001])
@pytest.mark.parametrize("r_out,out", [("r", None), ("y", None), ("gate", None), ("r", "y"), ("y", "r"), ("r", "gate"), ("gate", "r"), (None, "r"), (None, "y"), (None, "gate"), ("other", "r"), ("other", "y"),
                                       ("other", "gate")])
def test_an_output_in_an_inputs_place(d, r_out, out):
    for kind in ("bf16", "f32"):
        for post, pre in (("none", "none"), ("none", "rms"), ("mean", "none")):
            check(d, r_out, out, kind, post, pre)


def check(d, r_out, out, kind, post, pre, rows=7):
    rng = np.random.default_rng(d)
    t = {n: torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).to("cuda", TYPES[kind][0]) for n in ("r", "y", "gate")}
    t["other"] = torch.zeros_like(t["r"])
    v = {n: t[n].double().cpu().numpy() for n in ("r", "y", "gate")}
    desc = si.si_norm_t(rows=rows, d=d, post=KINDS[post], pre=KINDS[pre], eps=1e-5, res_scale=0.5, y_scale=2.0)
    for name, place in (("r", "r"), ("y", "y"), ("gate", "gate"), ("r_out", r_out), ("out", out)):
        if place:
            setattr(desc, name, t[place].data_ptr())
            setattr(desc, name + "_type", TYPES[kind][1])
            setattr(desc, name + "_stride", d)
    print("si_norm", dict(d=d, r_out=r_out, out=out, kind=kind, post=post, pre=pre), flush=True)
    si.si_norm(desc, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    (r64, mr), (o64, mo) = residual64(v["r"], v["y"], v["gate"], 0.5, 2.0, float(np.float32(1e-5)), post, None, None, pre, None, None)
    if r_out:
        close(t[r_out], r64, mr, kind)
    if out:
        close(t[out], o64, mo, kind)
    for n in ("r", "y", "gate"):
        if n not in (r_out, out):
            assert np.array_equal(t[n].double().cpu().numpy(), v[n])
