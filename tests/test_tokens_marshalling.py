"""The token-policy calls' two ways into the library, on the host."""

import pytest
import torch

import paper_1802_01561_amd as vt
from paper_1802_01561_amd import tokens
from paper_1802_01561_amd._lib import lib


def test_outputs_are_taken_from_an_iterator_once(monkeypatch):
    """Where native code declines, the Python path has the same outputs."""
    seen = []

    class Declines:
        clip = 0
        device = staticmethod(lambda: 0)
        stream = staticmethod(lambda device: 0)
        call_clip = staticmethod(lambda fn, gradients, outs, *rest: seen.append((list(gradients), list(outs))))

    monkeypatch.setattr(tokens, "_fast_call", lambda first: Declines)
    workspace = object.__new__(vt.ClipWorkspace)
    workspace.tensor, workspace.nbytes = torch.empty(32768, dtype=torch.uint8), 32768
    g = [torch.ones(3), torch.ones(4)]
    with pytest.raises(ValueError, match="GPU"):  # past the count of the outputs
        vt.vtrace_clip_grad_norm(iter(g), 1.0, out=(t.clone() for t in g), workspace=workspace)
    assert [len(part) for part in seen[0]] == [2, 2]


def test_error_texts_cover_the_token_calls():
    L = lib()
    assert b"vtrace_tokens.h" in L.vtrace_status_string(2)
    assert b"max_norm" in L.vtrace_status_string(4)
    assert b"vtrace_*_workspace_bytes" in L.vtrace_status_string(6)


@pytest.mark.parametrize("wanted", [True, 1, "yes"])
def test_wanted_outputs_by_truth(monkeypatch, wanted):
    """Native code compares with True itself: whatever counts as true reaches it as that."""
    seen = []

    class Declines:
        log_prob_loss = 0
        device = staticmethod(lambda: 0)
        stream = staticmethod(lambda device: 0)
        call_log_prob_loss = staticmethod(lambda *args: seen.append(args))

    monkeypatch.setattr(tokens, "_fast_call", lambda first: Declines)
    workspace = object.__new__(vt.LogProbWorkspace)
    workspace.tensor, workspace.nbytes = torch.empty(32768, dtype=torch.uint8), 32768
    f, b = torch.zeros(2, 3), torch.zeros(3)
    with pytest.raises(ValueError, match="GPU"):
        vt.vtrace_log_prob_loss_grad(f, f, None, f, f, f, b, workspace=workspace, with_vs=wanted, with_pg_advantages=wanted)
    assert seen[0][-7:-4] == (False, True, True) and all(type(x) is bool for x in seen[0][-7:-4])
