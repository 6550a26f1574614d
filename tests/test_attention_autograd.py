"""CPU: what goes back through ``block_harness.Attention`` is what came forward through it.  The library's calls are replaced by recorders; only
autograd's part is looked at."""
import pytest
import torch

HD, HEADS, KV, ROWS = 8, 4, 2, 8


@pytest.fixture
def calls(monkeypatch):
    """The arguments of each call, by name."""
    from paper_2608_24070_b200 import binding as B

    seen = {}

    def recorder(name):
        def call(*args, **more):
            kept = lambda x: x.detach().clone() if isinstance(x, torch.Tensor) else x
            seen.setdefault(name, []).append(([kept(x) for x in args], {k: kept(x) for k, x in more.items()}))

        return call

    for name in ("slope_rotary", "slope_attention_fwd", "slope_attention_bwd"):
        monkeypatch.setattr(B, name, recorder(name))
    monkeypatch.setattr(B, "slope_attention_bwd_workspace_bytes", lambda *_: 16)
    return seen


def made(**layer):
    from paper_2608_24070_b200 import block_harness as H

    ints = lambda *v: torch.tensor(v, dtype=torch.int32)
    attention = H.Attention(HEADS, KV, 0.5 ** torch.arange(4, dtype=torch.float64), **layer)
    x = [torch.zeros(ROWS, n * HD, dtype=torch.bfloat16, requires_grad=True) for n in (HEADS, KV, KV)]
    where = {"positions": torch.arange(ROWS, dtype=torch.int32), "starts": ints(0, 4, 7), "lengths": ints(4, 3)}
    return attention, x, where


@pytest.mark.parametrize("name", ["positions", "starts", "lengths", "frequencies"])
def test_a_tensor_that_is_written_between_the_passes(calls, name):
    attention, x, where = made()
    out = attention(*x, **where)
    changed = attention.frequencies if name == "frequencies" else where[name]
    changed.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.float().sum().backward()
    assert "slope_attention_bwd" not in calls


def test_a_layer_that_is_changed_between_the_passes(calls):
    """Another table of frequencies, factor, pairing, mask or number of heads is for the calls that follow."""
    attention, x, where = made(factor=1.25, window=3, scale=0.5)
    out = attention(*x, **where)
    frequencies = attention.frequencies
    attention.frequencies, attention.factor, attention.interleaved = frequencies * 2, 2.0, True
    attention.heads, attention.kv_heads = 1, 1
    attention.mask.update(causal=False, window=0, scale=1.0)
    out.float().sum().backward()
    (there, how_there), (back, how_back) = calls["slope_rotary"]
    for a, b in zip(there[2:5], back[2:5]):                        # positions, frequencies, columns of a head
        assert torch.equal(a, b) if isinstance(a, torch.Tensor) else a == b
    assert torch.equal(back[3], frequencies)
    assert how_there == {"factor": 1.25, "interleaved": False} and how_back == {**how_there, "backward": True}
    (_, forward), = calls["slope_attention_fwd"]
    (_, backward), = calls["slope_attention_bwd"]
    assert forward.keys() == backward.keys()
    for k, a in forward.items():
        assert torch.equal(a, backward[k]) if isinstance(a, torch.Tensor) else a == backward[k], k
    assert forward["window"] == 3 and forward["scale"] == 0.5 and forward["causal"] is True


def test_nothing_of_a_batch_is_asked_for_that_is_not_there(calls):
    """Without starts, lengths, positions: equal sequences, no rotation, either way."""
    from paper_2608_24070_b200 import block_harness as H

    _, x, _ = made()
    H.Attention(HEADS, KV)(*x, sequences=2).float().sum().backward()
    assert "slope_rotary" not in calls
    (_, backward), = calls["slope_attention_bwd"]
    assert backward == {"sequences": 2, "starts": None, "lengths": None, "causal": True, "window": 0, "scale": None}


def test_two_passes_forward_with_buffers_of_their_own(calls):
    """Micro-batches: each goes back over its own sequences and positions, in any order."""
    attention, x, where = made()
    other = {k: v.clone() for k, v in where.items()}
    other["positions"] += 100
    other["lengths"] -= 1
    first, second = attention(*x, **where), attention(*x, **other)
    second.float().sum().backward()
    first.float().sum().backward()
    for (_, batch), used in zip(calls["slope_attention_bwd"], (other, where)):
        assert torch.equal(batch["lengths"], used["lengths"]) and torch.equal(batch["starts"], used["starts"])
    for (args, _), used in zip(calls["slope_rotary"][2:], (other, where)):
        assert torch.equal(args[2], used["positions"])


def test_tables_made_in_inference_mode(calls):
    """Positions and frequencies that an evaluation left behind, then a training step; and no graph at all."""
    with torch.inference_mode():
        attention, _, where = made()
        attention(*(torch.zeros(ROWS, n * HD, dtype=torch.bfloat16) for n in (HEADS, KV, KV)), **where)
    _, x, _ = made()
    attention(*x, **where).float().sum().backward()
    forward, backward = calls["slope_rotary"][1:]
    assert torch.equal(forward[0][2], backward[0][2]) and torch.equal(forward[0][3], backward[0][3])
    assert torch.equal(calls["slope_attention_bwd"][0][1]["starts"], where["starts"])
    with torch.no_grad():
        attention(*x, **where)
