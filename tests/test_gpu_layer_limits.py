"""Attention, block norms, the embedding and the decoder on them at the limits
of their types, sizes and layouts."""
import numpy as np
import pytest

from tests import _layer as ref
from tests._gpu import say, torch
from tests.test_gpu_step import close, f64

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# the decoder
# ---------------------------------------------------------------------------
def test_decoder_attention_is_float32(monkeypatch):
    """What the decoder's attention returns and its gradients are within the float32 bounds, with one rounding to bfloat16 at
    the end: no probability is rounded on the way."""
    torch()
    from paper_2410_15526_amd import sdp4
    from paper_2410_15526_amd.decoder import Config, Decoder, sequences
    calls = {"sdp4_attention": [], "sdp4_attention_grad": []}
    for name, made in calls.items():
        def watched(*args, made=made, plain=getattr(sdp4, name)):
            plain(*args)
            made.append([f64(x.detach()) if hasattr(x, "detach") else x for x in args])
        monkeypatch.setattr(sdp4, name, watched)
    model = Decoder(Config(batch=3), seed=4)
    tokens, targets = sequences(model.cfg, 3, 0)
    model.backward(tokens, targets, p=0.0)
    forward, backward = calls["sdp4_attention"], calls["sdp4_attention_grad"]
    assert len(forward) == len(backward) == model.cfg.layers
    lengths, last = [model.cfg.seq] * 3, lambda want, bound: bound + ref.V * np.abs(want)  # noqa: E731
    for q, k, v, scale, _, out, lse in forward:
        (want, bound), _ = ref.attention(q, k, v, lengths, scale, "f32")
        close(out, want, last(want, bound), "out")
    for dout, q, k, v, out, lse, scale, _, *grads, _ in backward:
        wants = ref.attention_grad(dout, q, k, v, out, lse, lengths, scale, "f32")
        for got, (want, bound), name in zip(grads, wants, ("dq", "dk", "dv")):
            close(got, want, last(want, bound), name)
