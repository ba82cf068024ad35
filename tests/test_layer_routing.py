"""The layer's routing methods and the gradient that follows them: which call it is, and that its result fits."""
import numpy as np
import pytest
import torch

from oracle import dynmo_oracle as orc
from paper_2505_14864_amd import binding as B
from paper_2505_14864_amd.layer import RoutedFFNLayer


def host_layer(monkeypatch, T, E, k, mode):
    """A layer without a GPU: torch's pinned memory and events stand aside, and nothing may be launched."""
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, pin_memory=False, **kw: empty(*a, **kw))
    monkeypatch.setattr(torch.cuda, "Event", lambda: None)
    return RoutedFFNLayer(T, 16, 16, E, k, "bf16", mode, device="cpu")


@pytest.mark.parametrize("mode", ["moe", "mod", "early_exit"])
@pytest.mark.parametrize("E", [1, 4])
@pytest.mark.parametrize("allocated", [False, True])
def test_scored_gradient_has_room_for_every_logit(monkeypatch, mode, E, allocated):
    T = 6
    layer, seen = host_layer(monkeypatch, T, E, 1, mode), []
    monkeypatch.setattr(B, "dynmo_route_scored", lambda *a, **kw: None)
    monkeypatch.setattr(B, "dynmo_route_scored_bwd", lambda d, rule, dgate, logits, expert_idx, dlogits: seen.append(dlogits))
    if allocated:
        layer.alloc_backward()
    logits = torch.zeros((T, E), dtype=torch.float32)
    layer.route_scored(logits, B.make_rule())
    got = layer.route_bwd(logits)
    assert seen[0] is got and got.numel() == T * E
    assert layer.droute.shape == ((T, E) if mode == "moe" else (T,))  # the other routings' stays as it is
    assert (got is layer.droute) == (mode == "moe" or E == 1)


def test_the_gradient_is_that_of_the_last_routing(monkeypatch):
    layer, seen = host_layer(monkeypatch, 6, 4, 2, "moe"), []
    for name in ("dynmo_route_topk", "dynmo_route_scored", "dynmo_route_topk_bwd"):
        monkeypatch.setattr(B, name, lambda *a, name=name, **kw: seen.append(name))
    monkeypatch.setattr(B, "dynmo_route_scored_bwd", lambda d, rule, *a, **kw: seen.append(rule))
    logits, rule, other = torch.zeros((6, 4), dtype=torch.float32), B.make_rule(), B.make_rule("sigmoid")

    def gradient_of(*args, **kw):
        seen.clear()
        layer.route_bwd(*args, **kw)
        return seen[0]

    layer.route_scored(logits, rule)
    assert gradient_of(logits) is rule
    # calls of the binding into the layer's buffers: the caller says which
    assert gradient_of(rule=None) == "dynmo_route_topk_bwd"
    assert gradient_of(logits, rule=other) is other
    assert gradient_of(logits) is rule
    layer.route_topk(logits)
    assert gradient_of() == "dynmo_route_topk_bwd"
    assert gradient_of(logits, rule=other) is other


@pytest.mark.parametrize("E", [65, 256])
@pytest.mark.parametrize("T", [(1 << 26) - 3, (1 << 26) - 1])
def test_batches_too_long_for_a_launch_are_refused(E, T):
    """Above 64 experts a workgroup has four tokens, and 2^24 of those are 2^32 threads.  Without a GPU a launch gives another error."""
    d, rule = B.C.byref(B.make_desc(T, 8, 8, E, 2, "bf16")), B.C.byref(B.make_rule())
    assert B.lib().dynmo_route_scored(d, rule, 16, None, 16, 16, None) == -2
    assert B.lib().dynmo_route_scored_bwd(d, rule, 16, 16, 16, 16, None) == -2


@pytest.mark.gpu
def test_gradient_of_a_binding_call_behind_a_scored_routing():
    T, E, k = 40, 6, 2
    rng = np.random.default_rng(5)
    lg, dg = rng.standard_normal((T, E)).astype(np.float32), rng.standard_normal((T, k)).astype(np.float32)
    layer = RoutedFFNLayer(T, 16, 16, E, k, "bf16")
    layer.alloc_backward()
    logits = torch.from_numpy(lg).cuda()
    layer.route_scored(logits, B.make_rule("sigmoid", scale=3.0))
    B.dynmo_route_topk(layer.d, logits, layer.expert_idx, layer.gate_w)
    layer.dgate.copy_(torch.from_numpy(dg))
    idx, gate = orc.route_topk(lg, k)
    ref = orc.route_scored_bwd(dg, lg, idx, "softmax")  # the softmax over the chosen logits is the renormalised one
    assert np.abs(layer.route_bwd(rule=None).cpu().numpy() - ref).max() <= 64 * 2.0 ** -24 * 2 * np.abs(dg).sum(1).max()


@pytest.mark.gpu
@pytest.mark.parametrize("mode", ["moe", "mod", "early_exit"])
def test_scored_routing_of_a_layer_with_a_residual(mode):
    T, E, k = 70, 5, 2
    rng = np.random.default_rng(4)
    lg, dg = rng.standard_normal((T, E)).astype(np.float32), rng.standard_normal((T, k)).astype(np.float32)
    layer = RoutedFFNLayer(T, 16, 16, E, k, "bf16", mode)
    layer.alloc_backward()
    logits = torch.from_numpy(lg).cuda()
    for score, renormalize in (("sigmoid", True), ("softmax", False)):
        layer.route_scored(logits, B.make_rule(score, renormalize=renormalize))
        layer.dgate.copy_(torch.from_numpy(dg))
        idx, _ = orc.route_scored(lg, None, k, score, renormalize=renormalize)
        assert np.array_equal(layer.expert_idx.cpu().numpy(), idx)
        ref = orc.route_scored_bwd(dg, lg, idx, score, renormalize)
        assert np.abs(layer.route_bwd(logits).cpu().numpy() - ref).max() <= 64 * 2.0 ** -24 * 2 * np.abs(dg).sum(1).max()


@pytest.mark.gpu
@pytest.mark.parametrize("E", [8, 40, 100, 256])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("scale", [1.0, 2.3])
def test_gradients_that_renormalised_weights_do_not_pass_on(E, score, scale):
    """One chosen expert has the weight `scale` whatever its logit, and what all of a token's gradients have in common changes nothing: zero, not
    the rounding of a difference.  Where they differ a little the result is as exact as the differences: 64 * 2^-24 of them."""
    T = 45
    rng = np.random.default_rng(E)
    lg = (3 * rng.standard_normal((T, E))).astype(np.float32)

    def grad(idx, dg):
        out = torch.full((T, E), 7.0, dtype=torch.float32, device="cuda")
        B.dynmo_route_scored_bwd(B.make_desc(T, 8, 8, E, idx.shape[1], "bf16"), B.make_rule(score, scale=scale), torch.from_numpy(dg).cuda(),
                                 torch.from_numpy(lg).cuda(), torch.from_numpy(idx).cuda(), out)
        return out.cpu().numpy()

    for k in (1, 5, min(E, 40)):
        idx, _ = orc.route_scored(lg, None, k, score)
        dg = rng.standard_normal((T, k)).astype(np.float32)
        lone = np.full_like(idx, -1)
        lone[np.arange(T), rng.integers(0, k, T)] = idx[:, 0]  # the other slots were dropped
        assert (grad(lone, dg) == 0).all()
        assert (grad(idx, np.repeat(dg[:, :1], k, 1)) == 0).all()
        dg = (100 * rng.standard_normal((T, 1)) + dg).astype(np.float32)
        apart = np.abs(dg.astype(np.float64) - dg[:, :1]).sum(1, keepdims=True)
        assert (np.abs(grad(idx, dg) - orc.route_scored_bwd(dg, lg, idx, score, True, scale)) <= 64 * 2.0 ** -24 * 2 * scale * apart).all()
