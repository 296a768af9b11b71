"""The holders of the few-token calls on the GPU: captures beside eager calls of the same holder."""
import pytest
import torch

from paper_2506_18145_amd import RomError
from tests.test_gpu_few_tokens import ffn_holder, hybrid, randn, routing, states, step_cfg

pytestmark = pytest.mark.gpu


def test_a_forward_captured_first_leaves_eager_calls_their_weights():
    """Fresh holder, one for each pre_norm: the capture's packing has not run when the eager calls in front of a replay read theirs."""
    for pre_norm in (False, True):
        cfg, layer, ffn = ffn_holder(64, 32, 4, 1, "bf16")
        _, _, other = ffn_holder(64, 32, 4, 1, "bf16")
        x = randn(1, 3, 64)
        r = layer.route(x)
        want = other.forward(x, r, pre_norm), other.step(x, r["expert_idx"], r["gate"], pre_norm)
        ffn._ws, ffn._step_ws = other._ws, dict(other._step_ws)
        out, refused = torch.empty_like(x), False
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ffn.forward(x, r, pre_norm, out=out)
            try:
                ffn.step(x, r["expert_idx"], r["gate"], pre_norm)
            except RomError as e:
                refused = "before a capture" in str(e)
        assert refused
        assert torch.equal(ffn.step(x, r["expert_idx"], r["gate"], pre_norm), want[1]) and torch.equal(ffn.forward(x, r, pre_norm), want[0])
        for _ in range(3):
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[0])
            assert torch.equal(ffn.step(x, r["expert_idx"], r["gate"], pre_norm), want[1])


@pytest.mark.parametrize("K", [1, 2])
def test_a_captured_stack_forward_replayed_behind_steps(K):
    cfg = step_cfg(batch=2, top_k=K, gate_mode=K - 1)
    stack = hybrid(cfg)
    x = randn(1, 2, 5, cfg.d_model)
    want = stack.forward(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = stack.forward(x)
    for t in range(3):
        big = step_cfg(batch=60 + 30 * t, top_k=K, gate_mode=K - 1)     # other shapes, larger workspaces
        for group in (0, 64):
            stack.step(randn(t, big.batch, cfg.d_model), *states(big, 7, 3), q4_group=group)
        fill = [torch.full((1 << 20,), -1, dtype=torch.int32, device=x.device) for _ in range(8)]     # takes what was let go
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and all(bool((f == -1).all()) for f in fill)
        del fill


@pytest.mark.parametrize("block", [False, True])
def test_a_captured_plain_step_replayed_behind_4_bit_steps(block):
    cfg, layer, _ = ffn_holder(128, 256, 8, 2, "bf16")
    layer.weights["norm_w"] = torch.ones(128, device="cuda:0")
    step = layer.block_step if block else layer.step
    x = randn(1, 5, 128)
    cs0, ss0 = randn(2, 5, 256, 3, dtype="fp32"), randn(3, 5, 256, 16, dtype="fp32")
    cs, ss = cs0.clone(), ss0.clone()
    want = step(x, cs, ss)                                      # folds the norm's scale, makes the workspace
    want_cs, want_ss = cs.clone(), ss.clone()
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x, cs, ss, out)
    for _ in range(3):
        (layer.block_step_q4 if block else layer.step_q4)(x, cs0.clone(), ss0.clone())       # the same batch, a larger workspace
        fill = [torch.full((n,), -1, dtype=torch.int32, device=x.device) for n in (1 << 12, 1 << 14, 1 << 16, 1 << 18)]
        cs.copy_(cs0), ss.copy_(ss0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(cs, want_cs) and torch.equal(ss, want_ss)
        assert all(bool((f == -1).all()) for f in fill)


@pytest.mark.parametrize("group", [0, 64])
def test_a_stack_step_of_no_sequences(group):
    cfg = step_cfg(batch=0)
    stack = hybrid(cfg)
    x, (cs, ss) = randn(1, 0, cfg.d_model), states(cfg, 2, 3)
    assert stack.step(x, cs, ss, q4_group=group).shape == (0, cfg.d_model)
    layer, ffn = stack.layers[0], stack.ffns[0]
    plain = ffn_holder(cfg.d_model, 32, 4, 1, "bf16")[1]
    assert plain.step_q4(x, cs[0], ss[0]).shape == x.shape and layer.block_step_q4(x, cs[0], ss[0]).shape == x.shape
    idx, gate = torch.empty((0, 1), dtype=torch.int32, device=x.device), torch.empty((0, 1), device=x.device)
    assert ffn.step(x, idx, gate, True, True, group).shape == x.shape
