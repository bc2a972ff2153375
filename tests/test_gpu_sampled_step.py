"""Sampled acceptance as a step of VerifyPass on an MI355X: whose logits it reads, behind passes and replays."""
import numpy as np
import pytest
import torch

from paper_2507_22424_amd import workload as wl
from paper_2507_22424_amd.runner import VerifyPass

from parity_utils import say

pytestmark = pytest.mark.gpu

B, T, V = 2, 6, 64
PARENT = [-1, 0, 0, 1, 1, 2]


def _pass():
    cfg = wl.C2.scaled(name="bf16-sampled-step", index=63, n_layers=1, hidden=512, n_heads=4, head_dim=128, mlp_dim=1536, vocab=256,
                       n_bins=V, n_episodes=B, tree_nodes=T, prefix_lo=20, prefix_hi=30, max_depth=2, max_children=2, spine_lo=2)
    pl = wl.prefix_lengths(cfg)
    vp = VerifyPass(cfg, pl, np.array(PARENT * B), extra_capacity=4 * T)
    vp.load_layer(0, wl.layer_weights(cfg, 0))
    for b in range(B):
        vp.load_prefix(0, b, *wl.prefix_kv(cfg, b, 0, int(pl[b])))
    head = wl.head_weights(cfg)
    vp.load_head(head["g_final"], head["w_lm"])
    return vp


def _inputs(vp, seed):
    gen = torch.Generator().manual_seed(seed)
    hidden = 0.5 * torch.randn(B * T, vp.wc.hidden, generator=gen)
    draft = vp.wc.vocab - V + torch.randint(0, V, (B * T,), generator=gen)
    return hidden, draft.numpy(), torch.rand(B * T, generator=gen).cuda(), torch.rand(B, generator=gen).cuda()


def _outputs(vp):
    return [t.clone() for t in (vp.probs, vp.accept_mask, vp.accepted_len, vp.best_node, vp.path, vp.out_tokens, vp.accept_status)]


def test_sampling_reads_the_logits_of_the_last_pass_or_refuses():
    """Eager passes and replays of recorded steps, with logits and without, in turn."""
    vp = _pass()
    hidden, draft, ua, ud = _inputs(vp, 0)
    vp.set_hidden(hidden)
    vp.set_draft(draft)
    with_logits, without = vp.capture_step(4, want_logits=True), vp.capture_step(4)
    with pytest.raises(RuntimeError, match="no logits"):
        vp.accept_sampled(ua, ud)
    for rep in range(3):
        say(f"[sampled step] replay {rep}")
        hidden, draft, ua, ud = _inputs(vp, 1 + rep)
        vp.set_hidden(hidden)
        vp.set_draft(draft)
        vp.forward()
        vp.accept_sampled(ua, ud, 0.8)
        want = _outputs(vp)
        assert bool((vp.probs.sum(1) - 1).abs().max() < 1e-5)
        vp.set_hidden(hidden)
        vp.logits.fill_(3.0)
        with pytest.raises(RuntimeError, match="no logits"):
            vp.accept_sampled(ua, ud, 0.8)
        without.replay()
        with pytest.raises(RuntimeError, match="no logits"):
            vp.accept_sampled(ua, ud, 0.8)
        with_logits.replay()
        vp.accept_sampled(ua, ud, 0.8)
        assert all(torch.equal(x, y) for x, y in zip(want, _outputs(vp)))


def test_a_recorded_sampled_step_follows_its_inputs():
    """Pass and sampled acceptance in one graph, their first calls of all inside it but for the pass's; replayed with new
    inputs, eager steps between."""
    vp = _pass()
    hidden, draft, ua, ud = _inputs(vp, 0)
    vp.set_hidden(hidden)
    vp.set_draft(draft)
    vp.forward()
    held = torch.cuda.memory_allocated()
    vp.accept_sampled(ua, ud, 0.8)
    assert torch.cuda.memory_allocated() == held
    vp = _pass()
    vp.set_hidden(hidden)
    vp.forward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vp.forward()
        vp.accept_sampled(ua, ud, 0.8)
    for rep in range(4):
        hidden, draft, a, d = _inputs(vp, 10 + rep)
        ua.copy_(a)
        ud.copy_(d)
        vp.set_hidden(hidden)
        vp.set_draft(draft)
        vp.forward()
        vp.accept_sampled(a, d, 0.8)
        want = _outputs(vp)
        for t in (vp.logits, vp.probs, vp.path, vp.out_tokens, vp.accepted_len, vp.accept_mask):
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, _outputs(vp)))


def test_commit_refuses_rows_without_a_distribution():
    """Logits of an episode that are all masked, or NaN: accept_status says so, and nothing is committed - until another
    acceptance, sampled or not, eager or recorded, takes its place."""
    vp = _pass()
    hidden, draft, ua, ud = _inputs(vp, 0)
    vp.set_hidden(hidden)
    vp.set_draft(draft)
    graph = vp.capture_step(4, want_logits=True)     # older than the first sampled acceptance
    for bad in (float("nan"), -float("inf")):
        for again in (graph.replay, lambda: vp.accept(4), lambda: (vp.forward(), vp.accept_sampled(ua, ud))):
            vp.forward()
            vp.logits[T:] = bad
            vp.accept_sampled(ua, ud)
            assert vp.accept_status.tolist() == [0, 3]
            prefix, bound = vp.kv[0].prefix_len.clone(), vp.kv[0].struct.prefix_len_max
            with pytest.raises(RuntimeError, match="episodes .1."):
                vp.commit()
            assert torch.equal(vp.kv[0].prefix_len, prefix) and vp.kv[0].struct.prefix_len_max == bound
            again()
            assert vp.accept_status.tolist() == [0, 0]
    vp.commit()
    assert torch.equal(vp.kv[0].prefix_len, prefix + vp.accepted_len + 1)
