"""What the driver's baselines pass on to the refresh.  CPU only."""

import inspect

import pytest
import torch

from paper_2608_26140_amd.driver import AffixBatch


@pytest.mark.parametrize("call,k", [("direct_reuse", 0), ("full_refresh", 5)])
def test_baselines_pass_their_stream_as_a_stream(call, k):
    batch = AffixBatch.__new__(AffixBatch)
    batch.L, batch.B, batch.device = 5, 2, "cpu"
    seen = {}

    def refresh(anchors, k, drop_non_anchor=False, stream=None, layer_hook=None):
        seen.update(anchors=anchors, k=k, drop=drop_non_anchor, stream=stream)
    batch.refresh = refresh
    stream = object()
    getattr(batch, call)(stream)
    assert seen["k"] == k and seen["drop"] is False and seen["stream"] is stream
    if k:
        assert torch.equal(seen["anchors"], torch.arange(5, dtype=torch.int32).repeat(2, 1))


def calls_with_a_stream():
    from paper_2608_26140_amd import driver as D
    return [(owner, name) for owner in (D, AffixBatch) for name, f in vars(owner).items()
            if inspect.isfunction(f) and not name.startswith("_") and "stream" in inspect.signature(f).parameters
            and name != "recompute_layer"]  # makes no tensor


@pytest.mark.parametrize("positional", [False, True])
def test_calls_make_their_tensors_on_their_stream(monkeypatch, positional):
    """Every call enters its stream's context before anything else."""
    from paper_2608_26140_amd import driver as D

    class Entered(Exception):
        pass

    def on(stream):
        raise Entered(stream)
    monkeypatch.setattr(D, "_on", on)
    calls = calls_with_a_stream()
    assert {"probe", "refresh", "full_refresh", "shift_affix", "decode_step", "decode_schedule"} <= {n for _, n in calls}
    for owner, name in calls:
        f = getattr(owner, name)
        at = list(inspect.signature(f).parameters).index("stream")
        with pytest.raises(Entered) as e:
            if positional:
                f(*range(at), "s")
            else:
                f(*range(at), stream="s")
        assert e.value.args == ("s",), name
