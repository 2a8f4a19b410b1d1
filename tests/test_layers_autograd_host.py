"""What the layers' operators keep for a backward pass, with stand-ins for the kernels, on the CPU."""
import pytest
import torch

from paper_2008_11343_b200 import operators as O


@pytest.mark.parametrize("mode,kept", [(torch.enable_grad, True), (torch.no_grad, False), (torch.inference_mode, False)])
def test_states_are_kept_for_a_backward_pass_only(monkeypatch, mode, kept):
    asked = []

    def forward(x, gate, state=None, keep=False):
        asked.append(keep)
        return x.detach() * 1.0, x.detach()[:, -1], x.detach() if keep else None

    monkeypatch.setattr(O, "gated_scan_forward", forward)
    x, gate = torch.randn(2, 3, 4, requires_grad=True), torch.randn(2, 3, 4)
    with mode():
        h, last = O.gated_scan(x, gate)                             # x is a leaf that wants gradients, in every mode
        O.gated_scan(x.detach(), gate)
    assert asked == [kept, False] and h.requires_grad == last.requires_grad == kept
