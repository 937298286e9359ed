"""The binding imports and the library loads with a torch that was built without a GPU backend, and finds its streams by torch's
public interface where there is no quicker one."""
import os
import subprocess
import sys

import pytest
import torch

from paper_1802_09113_amd.binding import _raw_stream, ssn_logprobs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WITHOUT_A_BACKEND = """
import torch
for name in [n for n in vars(torch._C) if n.startswith("_cuda_")]:
    delattr(torch._C, name)
import paper_1802_09113_amd.binding as binding
print(binding.lib().ssn_strerror(0))
"""


def test_import_without_a_gpu_backend():
    got = subprocess.run([sys.executable, "-c", WITHOUT_A_BACKEND], cwd=ROOT, capture_output=True, text=True)
    assert got.returncode == 0, got.stderr
    assert "ok" in got.stdout


@pytest.mark.gpu
def test_streams_without_the_table_of_handles(monkeypatch):
    """The same results, on the default stream and on another one, where torch has no accessor of raw handles."""
    Z = torch.randn(3, 5000, device="cuda")
    want = ssn_logprobs(Z, k=3)
    side = torch.cuda.Stream()
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert _raw_stream(Z.get_device()) == torch.cuda.current_stream().cuda_stream
    got = [ssn_logprobs(Z, k=3)]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert _raw_stream(Z.get_device()) == side.cuda_stream
        got.append(ssn_logprobs(Z, k=3))
    torch.cuda.current_stream().wait_stream(side)
    for out in got:
        assert all(torch.equal(out[name], want[name]) for name in want)
