"""The join's gradient from inputs of which some are kept in 8 bits, and with operands and results left out, on the GPU
against the formulas in 64 bits (tolerances: test_gpu_block_join.py)."""
import pytest
import torch
from test_gpu_block_join import F32, check, gradient, make, run, run_bwd, values

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")


PARTS = [(1, 1, 9), (1, 1, 0), (0, 1, 1), (1, 0, 33), (0, 0, 7)]
LEFT_OUT = [(), ("dy",), ("dh",), ("db",), ("dy", "dh"), ("dy", "dh", "db")]


@pytest.mark.parametrize("kept", ["", "h", "b", "hb"])
@pytest.mark.parametrize("dtype,stream", [(torch.bfloat16, F32), (torch.float16, torch.float16)], ids=str)
@pytest.mark.parametrize("left_out,parts", [(x, p) for x in LEFT_OUT for p in PARTS if p[1] or "dy" not in x], ids=str)
def test_parts_from_checkpoints(left_out, parts, dtype, stream, kept):
    post, pre, gate_tokens = parts
    for rows, width in ((33, 72), (70, 1024), (5, 8192)):
        s = make(rows, width, dtype, stream, gate_tokens, post, pre, seed=gate_tokens + rows)
        fwd = run(s)
        inputs, exact = {}, {}
        for n in "hb":
            inputs[n], exact[n] = s[n], s[n].double()
            if n in kept:
                inputs[n] = fdp.Checkpoint8.empty(rows, width)
                fdp.op_checkpoint_save(s[n], inputs[n])
                exact[n] = values(inputs[n])
        if "dy" in left_out:
            s["dy"] = None
        want = gradient(s, fwd.get("r_post"), fwd.get("r_pre"), exact["h"], exact["b"])
        results = {n: None for n in left_out if n != "dy"}
        got = run_bwd(s, fwd, inputs["h"], inputs["b"], into=results)
        check(got, {n: w for n, w in want.items() if n not in results})


def test_refusals_without_db():
    s = make(4, 64, torch.bfloat16, F32, 0, True, True)
    r = torch.ones(4, device="cuda")
    work = torch.empty(fdp.block_join_bwd_workspace_bytes(4, 64), dtype=torch.uint8, device="cuda")
    kept = [fdp.Checkpoint8.empty(4, 64) for _ in range(2)]
    for x, k in zip((s["h"], s["b"]), kept):
        fdp.op_checkpoint_save(x, k)

    def call(**kw):
        d = dict(dy=None, du=s["du"], h=kept[0], b=kept[1], dh=None, db=None, post_gain=s["post"], pre_gain=s["pre"],
                 r_post=r, r_pre=r, workspace=work)
        d.update(kw)
        fdp.op_block_join_bwd(**d)

    call()
    call(b=s["b"], h=s["h"])
    for bad in (dict(b=s["b"].cpu()), dict(b=s["b"][0]), dict(b=None), dict(h=None), dict(du=None),
                dict(du=s["du"].float()), dict(h=fdp.Checkpoint8.empty(4, 72)), dict(b=s["b"].half())):
        with pytest.raises((TypeError, ValueError, fdp.FdError)):
            call(**bad)
