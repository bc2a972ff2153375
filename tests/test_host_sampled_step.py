"""Which calls VerifyPass takes around a sampled acceptance.  The library's calls are replaced by recorders on host tensors:
nothing here reaches a GPU."""
import numpy as np
import pytest
import torch

from paper_2507_22424_amd import binding as sv
from paper_2507_22424_amd import runner
from paper_2507_22424_amd import workload as wl

CHAIN = np.arange(-1, 3)


class _Calls:
    """The binding with its device calls taken down instead of made."""

    def __init__(self):
        self.made, self.capturing, self.status = [], False, 0

    def __getattr__(self, name):
        if name in ("sv_workspace_init", "sv_verify_stack", "sv_verify_layer", "sv_action_head_argmax", "sv_relaxed_accept",
                    "sv_token_probs", "sv_sampled_accept", "sv_commit_path", "sv_advance_prefix"):
            return lambda *a, **k: self._made(name, a)
        return getattr(sv, name)

    def _made(self, name, args):
        self.made.append(name)
        if name == "sv_sampled_accept":
            args[-1].copy_(torch.as_tensor(self.status))


@pytest.fixture
def calls(monkeypatch):
    c = _Calls()
    monkeypatch.setattr(runner, "sv", c)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: c.capturing)
    return c


@pytest.fixture
def vp(calls):
    cfg = wl.C2.scaled(name="host-sampled", index=62, n_layers=1, hidden=512, n_heads=4, head_dim=128, mlp_dim=1536, vocab=64, n_bins=32,
                       n_episodes=2, tree_nodes=4, prefix_lo=5, prefix_hi=9, max_depth=3, max_children=1, spine_lo=3)
    vp = runner.VerifyPass(cfg, [5, 9], np.concatenate([CHAIN] * 2), device="cpu", extra_capacity=100)
    vp.workspace.zero_()                             # (the pass's status word among it)
    return vp


def _sample(vp):
    vp.accept_sampled(torch.zeros(8), torch.zeros(2))


def test_sampling_needs_logits_of_the_present_inputs(vp, calls):
    def refused():
        calls.made.clear()
        with pytest.raises(RuntimeError, match="no logits"):
            _sample(vp)
        assert not calls.made

    refused()                                        # no pass yet
    vp.step(4)
    refused()                                        # a pass that wrote none
    vp.forward(want_logits=True)
    _sample(vp)
    _sample(vp)                                      # again, as at another temperature
    vp.set_draft(np.zeros(8))                        # (the pass does not read the draft's tokens)
    _sample(vp)
    vp.accept(4)
    _sample(vp)
    vp.forward(want_logits=False)
    refused()                                        # the logits are an earlier pass's
    for change in (lambda: vp.set_hidden(torch.zeros(8, 512)), lambda: vp.set_tree(np.concatenate([CHAIN] * 2)), vp.commit):
        vp.step(4, want_logits=True)
        _sample(vp)
        change()
        refused()


def test_recorded_passes_are_not_refused(vp, calls):
    """What the caller records is replayed out of sight: the pass, the acceptance, or both."""
    calls.capturing = True
    _sample(vp)                                      # an acceptance to be replayed behind passes yet to come
    vp.step(4)
    calls.capturing = False
    with pytest.raises(RuntimeError, match="no logits"):
        _sample(vp)
    calls.capturing = True
    vp.forward(want_logits=True)
    calls.capturing = False
    vp.set_hidden(torch.zeros(8, 512))               # (and a replay)
    _sample(vp)


def test_sampling_allocates_nothing(vp):
    """Its buffers are the object's from the beginning: a first call may be one that is recorded."""
    held = [t.data_ptr() for t in (vp.probs, vp.accept_status)]
    assert vp.probs.shape == vp.logits.shape and vp.accept_status.shape == (2,)
    vp.forward()
    _sample(vp)
    assert held == [t.data_ptr() for t in (vp.probs, vp.accept_status)]


def test_commit_refuses_an_episode_that_had_nothing_to_draw_from(vp, calls):
    for status, refused in ((0, False), (1, False), (3, True)):          # (1: drawn from the target's row itself)
        vp.forward()
        calls.status = torch.tensor([0, status], dtype=torch.int32)
        vp.accept_sampled(torch.zeros(8), torch.zeros(2))
        calls.made.clear()
        if refused:
            with pytest.raises(RuntimeError, match=r"episodes \[1\]"):
                vp.commit()
            assert not calls.made
            vp.accept(4)                             # what is accepted now was not sampled
        vp.commit()
        assert calls.made[-1] == "sv_advance_prefix"
