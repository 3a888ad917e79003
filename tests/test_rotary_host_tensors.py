"""op_rotary takes its device from q: with every tensor on the host they agree with one another, and
host addresses must not reach a kernel all the same."""
import pytest
import torch

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")


@pytest.mark.parametrize("with_keys", [False, True])
def test_host_tensors_are_refused(monkeypatch, with_keys):
    plan = fdp.Rotary(64)
    reached = []

    class Lib:
        def fd_op_rotary(self, *args):
            reached.append(args)
            return 0
    monkeypatch.setattr(fdp, "lib", Lib)
    monkeypatch.setattr(fdp, "_raw_stream", lambda device: 0)
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    pos = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA tensor"):
        fdp.op_rotary(plan, pos, q, q, k if with_keys else None, k if with_keys else None)
    assert not reached
    monkeypatch.undo()
