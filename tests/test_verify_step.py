"""Verification behind a plan that refuses requests: the oracle by hand, and what kvpr_verify_step refuses before anything touches the GPU."""
import numpy as np
import pytest

from oracle import kvpr_paged_oracle as po


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


def test_nothing_of_a_refused_request_is_kept():
    # two requests of 10 and 16 positions with three rows each and no free page: the second finds none
    plan = po.plan([10, 16], [3, 3], [1, 1], np.array([[0, -1], [1, -1]]), np.zeros(2, int), 0, 16, 6, 2)
    assert plan["refused"] == 1 and plan["seq_len"] == [13, 0] and (plan["slots"][3:] == -1).all()
    logits = np.zeros((6, 4))
    logits[:, 2] = 5
    args = (logits, logits, [2] * 6, plan["row_start"], [0.0, 0.0], [0.0] * 6, [0.5, 0.5], 6)
    assert po.verify(*args, seq_len=plan["seq_len"]) == ([2, 2, 2, -1, -1, -1], [3, 0])
    assert po.verify(*args) == ([2] * 6, [3, 3])                        # without the lengths it cannot know


def test_certain_tokens_stand_by_hand():
    logits = np.zeros((6, 4))
    logits[:, 2] = 5                                                    # the model would always say 2
    tokens, start = [0, 1, 3, 0, 2, 1], [0, 3, 6]
    args = (logits, logits, tokens, start, [0.0, 0.0], [0.0] * 6, [0.5, 0.5], 6)
    # a chunk of three prompt tokens; two certain tokens and a draft that the model does not bear out
    assert po.verify(*args, certain=[3, 2]) == ([1, 3, 2, 2, 2, -1], [3, 2])
    assert po.verify(*args, certain=[0, 9]) == ([2, -1, -1, 2, 1, 2], [1, 3])
    assert po.verify(*args) == ([2, -1, -1, 2, 2, -1], [1, 2])
    assert po.verify(*args, seq_len=[0, 9], certain=[3, 3]) == ([-1, -1, -1, 2, 1, 2], [0, 3])


def _call(k, **change):
    P = 1 << 20                                                       # an aligned address that no refused call touches
    args = dict(target_logits=P, draft_logits=P, logits_type=k.KVPR_F32, ld_target=100, ld_draft=100, vocab=100, tokens=P, row_start=P, seq_len=P, certain=P,
                n_requests=1, n_rows=1, temperature=P, u_accept=P, u_sample=P, len_in=P, len_out=P, kept=P, out_tokens=P, ws_dev=P, ws_bytes=1 << 40)
    return k.kvpr_verify_step(**{**args, **change}, stream=0)


BAD = [("logits_type", 7, "E_INVAL"), ("ld_target", 99, "E_INVAL"), ("ld_draft", 99, "E_INVAL"), ("vocab", 0, "E_RANGE"), ("vocab", (1 << 24) + 1, "E_RANGE"),
       ("n_requests", 0, "E_RANGE"), ("n_requests", 8193, "E_RANGE"), ("n_rows", -1, "E_RANGE"), ("n_rows", 1 << 23, "E_RANGE"), ("len_in", None, "E_INVAL"),
       ("len_out", None, "E_INVAL"), ("ws_bytes", 0, "E_INVAL"), ("target_logits", (1 << 20) + 2, "E_INVAL"), ("ws_dev", (1 << 20) + 8, "E_INVAL")] + \
      [(name, None, "E_INVAL") for name in ("target_logits", "tokens", "row_start", "temperature", "u_accept", "u_sample", "kept", "out_tokens", "ws_dev")]


@pytest.mark.parametrize("name,value,code", BAD)
def test_bad_arguments(k, monkeypatch, name, value, code):
    monkeypatch.setattr(k.binding.torch.cuda, "current_device", lambda: 0)
    with pytest.raises(k.KvprError) as e:
        _call(k, **{name: value})
    assert e.value.code == getattr(k, "KVPR_" + code) and k.kvpr_last_error()


def test_tensors_of_the_wrong_kind(k, monkeypatch):
    import torch
    monkeypatch.setattr(k.binding.torch.cuda, "current_device", lambda: 0)
    for name in ("seq_len", "certain"):
        with pytest.raises(ValueError, match="current device"):
            _call(k, **{name: torch.zeros(16, dtype=torch.int32)})
    for name in ("target_logits", "draft_logits"):
        with pytest.raises(TypeError, match="must be torch.float32"):
            _call(k, **{name: torch.zeros(16, dtype=torch.float16)})
