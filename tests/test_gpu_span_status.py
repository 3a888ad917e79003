"""Span attention on a status word that an earlier call has left set."""
import math

import pytest
import torch
from test_gpu_span_attention import BF16, FP16, make

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("T,S", [(700, 500), (40, 6000)])
def test_nothing_seen_after_a_wait_gave_up(T, S, dtype, D):
    """Blocks without work wait for the loads that they began whatever the status word holds (other waits give up at
    once when it is set): zeros come out, every time, and the word stays as it was."""
    s = make([(0, 0)] * T, S, 4, 2, D, dtype)
    out, lse = torch.empty_like(s["q"]), torch.empty(4, T, device="cuda")
    need = max(fdp.span_attention_workspace_bytes(T, S, 4, 2, D, backward=b) for b in (False, True))
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    err = torch.full((1,), 1 << 20, dtype=torch.int32, device="cuda")
    got = {"d" + n: torch.empty_like(s[n]) for n in "qkv"}
    for _ in range(20):
        for x in (out, lse, *got.values()):
            x.fill_(7.0)
        fdp.op_span_attention(s["q"], s["k"], s["v"], s["spans"], out, lse, workspace=work, err=err)
        fdp.op_span_attention_bwd(s["q"], s["k"], s["v"], s["spans"], out, lse, s["dout"], *got.values(),
                                  workspace=work, err=err)
        assert not bool(out.any()) and bool((lse == -math.inf).all())
        assert not any(bool(x.any()) for x in got.values())
    assert int(err) == 1 << 20
