"""rapid3_window_status waits for what runs on every stream of the device, those that the legacy default stream does not wait for too."""
import pytest
import torch

from paper_2509_22323_b200 import binding

pytestmark = pytest.mark.gpu


def test_the_status_waits_for_other_streams():
    q = torch.randn((1, 2, 300, 64), device="cuda").to(torch.bfloat16)
    binding.rapid3_window_attn(q, q, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    done = torch.cuda.Event()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)                               # about a tenth of a second
        out, _ = binding.rapid3_window_attn(q, q, q)
        done.record(side)
    assert not done.query()
    assert binding.rapid3_window_status() == 0
    assert done.query()
    assert torch.isfinite(out).all()
