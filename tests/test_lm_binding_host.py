"""Sizes that are no 32-bit unsigned numbers never reach the library (no GPU needed: the library and the buffers' addresses are
stand-ins)."""
import pytest
import torch

from paper_2010_08899_b200 import binding as B

CALLS = {
    "layer_norm_fwd": lambda t, rows, d, ld: B.dct_layer_norm_fwd(t, rows, d, ld, None, None, 1e-5, t, ld),
    "layer_norm_fwd, y's stride": lambda t, rows, d, ld: B.dct_layer_norm_fwd(t, rows, d, 8, None, None, 1e-5, t, ld),
    "layer_norm_bwd": lambda t, rows, d, ld: B.dct_layer_norm_bwd(t, 8, t, rows, d, ld, None, t, t, t, 8),
    "layer_norm_bwd, dy's stride": lambda t, rows, d, ld: B.dct_layer_norm_bwd(t, ld, t, rows, d, 8, None, t, t, t, 8),
    "layer_norm_bwd, dx's stride": lambda t, rows, d, ld: B.dct_layer_norm_bwd(t, 8, t, rows, d, 8, None, t, t, t, ld),
    "lm_logprobs_fwd": lambda t, rows, d, ld: B.dct_lm_logprobs_fwd(t, rows, d, ld, 1.0, None, 0, None, t),
    "lm_logprobs_bwd": lambda t, rows, d, ld: B.dct_lm_logprobs_bwd(t, rows, d, 8, 1.0, t, t, None, t, None, t, ld),
    "lm_distill": lambda t, rows, d, ld: B.dct_lm_distill(t, rows, d, ld, 1.0, t, t, 1, 0, None, t),
    "lm_distill, the gradient's stride": lambda t, rows, d, ld: B.dct_lm_distill(t, rows, d, 8, 1.0, t, t, 1, 0, None, t, t, ld),
}


@pytest.mark.parametrize("call", CALLS)
def test_sizes_that_are_no_32_bit_numbers_are_refused(call, monkeypatch):
    class Library:
        def __getattr__(self, name):
            return lambda *args: pytest.fail(f"{name}{args} reached the library")

    monkeypatch.setattr(B, "lib", lambda: Library())
    monkeypatch.setattr(B, "_stream", lambda stream: None)
    span = []
    monkeypatch.setattr(B, "_buf", lambda t, dtype, name, count: span.append(count))
    t = torch.zeros(64)
    for rows, d, ld in ((-1, 8, 8), (2, 8, -8), (-(1 << 32) + 2, 8, 8), ((1 << 32) + 1, 8, 8), (2, 8, (1 << 32) + 8)):
        with pytest.raises(ValueError):
            CALLS[call](t, rows, d, ld)
    assert all(count >= 0 for count in span)
