"""What a refusal of the norm's gradient says: the argument that it is about, by its own name (CPU-only: the check of where tensors live is off)."""
import pytest
import torch

from paper_2205_14756_amd import sequence as seq


def test_the_norm_s_gradient_names_its_own_arguments(monkeypatch):
    monkeypatch.setattr(seq, "_on_gpu", lambda *tensors: None)
    x = torch.zeros(4, 64)
    for name, call in (("r", lambda: seq.msla_norm_backward(x[:, ::2], None, x)), ("d_y", lambda: seq.msla_norm_backward(x, None, x[:3])),
                       ("d_y", lambda: seq.msla_norm_backward(x, None, x.half())), ("d_sum", lambda: seq.msla_norm_backward(x, None, x, x[:, :32])),
                       ("x", lambda: seq.msla_norm_forward(x[:, ::2])), ("residual", lambda: seq.msla_norm_forward(x, None, x[:3])),
                       ("sum_out", lambda: seq.msla_norm_forward(x, None, x, sum_out=x[:3]))):
        with pytest.raises(ValueError, match=rf"^msla: {name} must"):
            call()
