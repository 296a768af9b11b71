"""The holders of the few-token calls without a GPU: which buffers outlive a captured call, which weights and workspaces are
refused.  Tensors lie on the CPU; the library's size functions are real, the calls that launch are recorded."""
import gc
import weakref
from types import SimpleNamespace

import pytest
import torch

from paper_2506_18145_amd import binding
from paper_2506_18145_amd.build import build_library

E, D, DE, F = 4, 64, 128, 32


class Recorder:
    """The library with its launching calls replaced by ones that succeed and are counted."""

    def __init__(self, lib):
        self.lib, self.calls = lib, []

    def __getattr__(self, name):
        if name.endswith(("_bytes", "_layout")):
            return getattr(self.lib, name)

        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def host(monkeypatch):
    import os
    if not os.path.exists(binding._LIB_PATH):
        build_library()
    h = SimpleNamespace(lib=Recorder(binding.load_library()), capturing=False)
    monkeypatch.setattr(binding, "load_library", lambda: h.lib)
    monkeypatch.setattr(binding, "_current_index", lambda t: t.get_device())
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: h.capturing)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(binding.RomQ4Weight, "pack", lambda w, group=64: SimpleNamespace(
        packed=torch.zeros(binding.rom_q4_bytes(*w.shape, group), dtype=torch.uint8)))
    return h


def layer_of(top_k=1, dtype="bf16"):
    cfg = SimpleNamespace(d_model=D, d_inner=DE, d_state=16, d_conv=4, dt_rank=8, n_experts=E, top_k=top_k, n_experts_xdt=E,
                          dtype=dtype, gate_mode=1 if top_k > 1 else 0)
    zeros = torch.zeros
    return binding.RomLayer(cfg, dict(
        w_router=zeros(E, D), b_router=None, w_in=zeros(E, 2 * DE, D), conv_w=zeros(DE, 4), conv_b=zeros(DE), w_x=zeros(E, 40, DE),
        w_dt=zeros(E, DE, 8), dt_bias=zeros(DE), A_log=zeros(DE, 16), D=zeros(DE), w_out=zeros(E, D, DE), norm_w=torch.ones(D)), device="cpu")


def ffn_of(layer):
    return binding.RomFfnMoe(layer, F, dict(w_gate_up=torch.zeros(E, 2 * F, D), w_down=torch.zeros(E, D, F), norm_w=torch.ones(D)))


def tokens(n, k=1, dtype=torch.bfloat16):
    return torch.zeros(n, D, dtype=dtype), torch.zeros(n, k, dtype=torch.int32), torch.ones(n, k)


# ---------------------------------------------------------------- captures


def test_a_captured_packing_is_not_what_an_eager_call_takes(host):
    """Under capture the packing of gate | up is only recorded: its result is the graph's, and a step asks for an eager call first."""
    ffn = ffn_of(layer_of())
    x, idx, gate = tokens(3)
    routing = dict.fromkeys(("offsets", "perm", "inv_perm"), idx) | {"gate": gate}
    host.capturing = True
    for pre_norm in (False, True):
        with pytest.raises(binding.RomError, match="before a capture"):
            ffn.step(x, idx, gate, pre_norm)
        ffn.forward(x, routing, pre_norm)                       # lays out its weights in front of its products, in every replay
    assert host.lib.calls == ["rom_ffn_pack_gate_up", "rom_ffn_moe_forward"] * 2
    host.capturing = False
    host.lib.calls.clear()
    ffn.step(x, idx, gate, True)
    ffn.forward(x, routing, True)
    assert host.lib.calls == ["rom_ffn_pack_gate_up", "rom_ffn_moe_step", "rom_ffn_moe_forward"]
    host.capturing = True
    ffn.step(x, idx, gate, True)
    with pytest.raises(binding.RomError, match="before a capture"):
        ffn.step(x, idx, gate, False)                           # packed without the norm's scale: another layout


def hybrid_of(n_layers=2):
    layers = [layer_of() for _ in range(n_layers)]
    return binding.RomHybridStack(layers, [ffn_of(ly) for ly in layers])


def states(B, n_layers=None):
    lead = () if n_layers is None else (n_layers,)
    return torch.zeros(*lead, B, DE, 3), torch.zeros(*lead, B, DE, 16)


def let_go(*buffers):
    gc.collect()
    return [r() is None for r in buffers]


def test_a_captured_stack_forward_keeps_its_buffers(host):
    stack = hybrid_of()
    host.capturing = True
    stack.forward(torch.zeros(2, 3, D, dtype=torch.bfloat16))
    host.capturing = False
    used = [weakref.ref(b) for b in (stack._tmp, stack._ffn_ws)]
    stack.step(torch.zeros(40, D, dtype=torch.bfloat16), *states(40, 2))       # another shape, more tokens
    assert let_go(*used) == [False, False]


def test_a_captured_plain_step_keeps_its_workspace(host):
    layer = layer_of(top_k=2)
    x = torch.zeros(4, D, dtype=torch.bfloat16)
    for call in (layer.step, layer.block_step):
        layer._ws = None
        host.capturing = True
        call(x, *states(4))
        host.capturing = False
        used = weakref.ref(layer._ws)
        layer.step_q4(x, *states(4))                            # the same batch needs more with 4-bit projections
        assert layer._ws is not used() and let_go(used) == [False]
        used = weakref.ref(layer._ws)
        layer.forward(torch.zeros(4, 500, D, dtype=torch.bfloat16))
        assert let_go(used) == [True]                           # no capture: nothing piles up


# ---------------------------------------------------------------- what is refused


def raw_ffn_step(dims, gu, down, group=0, dtype=torch.bfloat16, n=3, ws=None):
    x, idx, gate = tokens(n, dims.top_k, dtype)
    ws = torch.zeros(binding.rom_ffn_step_workspace_bytes(dims, F, n), dtype=torch.uint8) if ws is None else ws
    binding.rom_ffn_moe_step(dims, F, gu, down, group, False, 1e-5, False, x, n, idx, gate, torch.empty_like(x), ws)


def packed_of(rows, cols, group=32):
    return torch.zeros(binding.rom_q4_bytes(E, rows, cols, group), dtype=torch.uint8)


def test_weights_of_another_type_of_the_same_size(host):
    for tdtype, others in ((torch.bfloat16, (torch.float16, torch.int16)), (torch.float32, (torch.int32,))):
        dims = layer_of(dtype="bf16" if tdtype is torch.bfloat16 else "fp32").dims
        gu, down = torch.zeros(E, 2 * F, D, dtype=tdtype), torch.zeros(E, D, F, dtype=tdtype)
        raw_ffn_step(dims, gu, down, dtype=tdtype)
        for other in others:
            for w in ((gu.view(other), down), (gu, down.view(other))):
                with pytest.raises(binding.RomError):
                    raw_ffn_step(dims, *w, dtype=tdtype)
        gu, down = packed_of(2 * F, D), packed_of(D, F)
        raw_ffn_step(dims, gu, down, 32, tdtype)
        for w in ((gu.view(tdtype), down), (gu, down.view(torch.int8))):
            with pytest.raises(binding.RomError):
                raw_ffn_step(dims, *w, 32, tdtype)
    q, x = packed_of(64, D), tokens(3)[0]
    out, idx = torch.zeros(3, 64, dtype=x.dtype), torch.zeros(3, 1, dtype=torch.int32)
    binding.rom_q4_project(q, E, 64, D, 32, x, idx, None, None, None, out, None)
    with pytest.raises(binding.RomError):
        binding.rom_q4_project(q.view(torch.bfloat16), E, 64, D, 32, x, idx, None, None, None, out, None)
    assert host.lib.calls == ["rom_ffn_moe_step"] * 4 + ["rom_q4_project"]


def raw_steps(layer, group, weights, B=3):
    """The step and the block step as the C ABI's wrappers take them."""
    x, out, ws = tokens(B, dtype=layer.tdtype)[0], tokens(B, dtype=layer.tdtype)[0], torch.zeros(binding.rom_step_q4_workspace_bytes(layer.dims, B), dtype=torch.uint8)
    cs, ss = states(B)
    return (lambda **kw: binding.rom_step_q4(**dict(dict(dims=layer.dims, weights=weights, q4_group=group, x=x, B=B, conv_state=cs, ssm_state=ss,
                                                         out=out, ws=ws), **kw)),
            lambda **kw: binding.rom_block_step_q4(**dict(dict(dims=layer.dims, weights=weights, q4_group=group, norm_weight=layer.weights["norm_w"],
                                                               eps=1e-5, x=x, B=B, conv_state=cs, ssm_state=ss, out=out, ws=ws), **kw)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_steps_refuse_weights_of_another_group_or_layer(host, dtype):
    """Scales of 128 columns read as those of 32 would be read four times past their end."""
    layer = layer_of(dtype=dtype)
    for held, told in ((128, 32), (32, 128), (64, 32)):
        for call in raw_steps(layer, told, layer.q4_weights(held)):
            with pytest.raises(binding.RomError):
                call()
            call(weights=layer.q4_weights(told))
            for name in ("w_in", "w_out"):
                for bad in (layer.weights[name], layer.q4_weights(told)[name][:-2], None):
                    with pytest.raises(binding.RomError):
                        call(weights=dict(layer.q4_weights(told), **{name: bad}))
    assert host.lib.calls == ["rom_step_q4", "rom_block_step_q4"] * 3


def test_stack_step_refuses_weights_of_another_group(host):
    stack = hybrid_of(3)
    stack.quantize(32).quantize(128)
    B = 3
    x, (cs, ss) = tokens(B)[0], states(B, 3)
    ws, ffn_ws = torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(1 << 20, dtype=torch.uint8)

    def call(blocks, ffns, group):
        binding.rom_hybrid_stack_step(stack.dims, F, blocks, ffns, group, True, 1e-5, x, B, cs, ss, x.clone(), x.clone(), ws, ffn_ws)

    held = {0: (stack.blocks, stack.ffn_structs), 32: stack._q4[32][:2], 128: stack._q4[128][:2]}
    for told in held:
        call(*held[told], told)
        for other in held:
            if other != told:
                for blocks, ffns in ((held[other][0], held[told][1]), (held[told][0], held[other][1])):
                    with pytest.raises(binding.RomError):
                        call(blocks, ffns, told)
    with pytest.raises(binding.RomError):                       # one block of three
        keep = [(ly.q4_weights(32, block=True), ly.weights["norm_w"]) for ly in stack.layers]
        keep[2] = stack.layers[2].q4_weights(128, block=True), keep[2][1]
        call(binding.make_blocks(keep), held[32][1], 32)
    assert host.lib.calls.count("rom_hybrid_stack_step") == 3


class Elsewhere(torch.Tensor):
    """A tensor of another device than the call's."""

    def get_device(self):
        return 7


def test_workspaces_elsewhere_or_with_gaps(host):
    layer = layer_of(top_k=2)
    x, idx, gate = tokens(3, 2)
    gu, down = torch.zeros(E, 2 * F, D, dtype=x.dtype), torch.zeros(E, D, F, dtype=x.dtype)
    q, out = packed_of(64, D), torch.zeros(3, 64, dtype=x.dtype)
    stack = hybrid_of(2)
    stack.quantize(32)
    cs, ss = states(3, 2)
    size = 1 << 20
    calls = [lambda ws: raw_ffn_step(layer.dims, gu, down, ws=ws), lambda ws: binding.rom_q4_project(q, E, 64, D, 32, x, idx, gate, None, None, out, ws)]
    calls += [lambda ws, c=c: c(ws=ws) for c in raw_steps(layer, 32, layer.q4_weights(32))]
    for mine in (lambda ws: (ws, torch.zeros(size, dtype=torch.uint8)), lambda ws: (torch.zeros(size, dtype=torch.uint8), ws)):
        calls.append(lambda ws, mine=mine: binding.rom_hybrid_stack_step(stack.dims, F, *stack._q4[32][:2], 32, True, 1e-5, x, 3, cs, ss, x.clone(),
                                                                          x.clone(), *mine(ws)))
    for call in calls:
        call(torch.zeros(size, dtype=torch.uint8))
        n = len(host.lib.calls)
        for ws in (torch.zeros(size, dtype=torch.uint8).as_subclass(Elsewhere), torch.zeros(size, 2, dtype=torch.uint8)[:, 0]):
            with pytest.raises(binding.RomError):
                call(ws)
        assert len(host.lib.calls) == n


def test_raw_steps_refuse_what_the_holders_refuse(host):
    """The wrappers of the C ABI see types, shapes and devices; the library sees addresses."""
    layer, B = layer_of(), 3
    x, (cs, ss) = tokens(B)[0], states(B)
    bad = [dict(x=x.float()), dict(x=x[:, :32].contiguous()), dict(out=x[:2].clone()), dict(out=x.float()), dict(conv_state=cs.bfloat16()),
           dict(conv_state=cs[:2].contiguous()), dict(ssm_state=ss.transpose(1, 2)), dict(ssm_state=ss.double()), dict(out=x.clone().as_subclass(Elsewhere)),
           dict(ssm_state=ss.clone().as_subclass(Elsewhere)), dict(B=4), dict(weights={k: v if k != "w_in" else v.as_subclass(Elsewhere)
                                                                                       for k, v in layer.q4_weights(32).items()})]
    for call in raw_steps(layer, 32, layer.q4_weights(32)):
        for kw in bad:
            with pytest.raises(binding.RomError):
                call(**kw)
    for group in (0, 32):
        stack = hybrid_of(2)
        stack.quantize(32)
        blocks, ffns = (stack.blocks, stack.ffn_structs) if group == 0 else stack._q4[32][:2]
        cs, ss = states(B, 2)
        base = dict(dims=stack.dims, d_ff=F, blocks=blocks, ffns=ffns, q4_group=group, ffn_pre_norm=True, eps=1e-5, x=x, B=B, conv_state=cs, ssm_state=ss,
                    out=x.clone(), tmp=x.clone(), ws=torch.zeros(1 << 20, dtype=torch.uint8), ffn_ws=torch.zeros(1 << 20, dtype=torch.uint8))
        for kw in (dict(x=x.float()), dict(out=x[:2].clone()), dict(tmp=x[:2].clone()), dict(tmp=x.float()), dict(conv_state=cs[:1].contiguous()), dict(ssm_state=ss[0]),
                   dict(B=4), dict(tmp=x.clone().as_subclass(Elsewhere))):
            with pytest.raises(binding.RomError):
                binding.rom_hybrid_stack_step(**dict(base, **kw))
    assert host.lib.calls.count("rom_step_q4") + host.lib.calls.count("rom_hybrid_stack_step") == 0


def test_steps_of_a_layer_on_another_device(host):
    """x and the states agree with each other; the layer's weights lie elsewhere."""
    layer = layer_of()
    x, (cs, ss) = tokens(3)[0], states(3)
    layer.step_q4(x, cs, ss), layer.block_step_q4(x, cs, ss)
    stack = hybrid_of(2)
    stack.step(x, *states(3, 2)), stack.step(x, *states(3, 2), q4_group=32)
    n = len(host.lib.calls)
    x, cs, ss = (t.as_subclass(Elsewhere) for t in (x, cs, ss))
    stack._tmp = None
    for call in (lambda: layer.step_q4(x, cs, ss, out=x.clone()), lambda: layer.block_step_q4(x, cs, ss, out=x.clone()),
                 lambda: stack.step(x, *(t.as_subclass(Elsewhere) for t in states(3, 2)), out=x.clone()),
                 lambda: stack.step(x, *(t.as_subclass(Elsewhere) for t in states(3, 2)), 32, out=x.clone())):
        with pytest.raises(binding.RomError):
            call()
    assert len(host.lib.calls) == n
    stack.step(tokens(3)[0], *states(3, 2))                     # what a refused call left behind serves the next


# ---------------------------------------------------------------- the C entry of the stack's step


@pytest.fixture
def entry():
    """rom_hybrid_stack_step of RoM + FFN-MoE pairs on addresses that a call which launches nothing does not touch."""
    import ctypes
    import os
    if not os.path.exists(binding._LIB_PATH):
        build_library()
    lib, buf = binding.load_library(), ctypes.create_string_buffer(1 << 16)
    at = (ctypes.addressof(buf) + 255) // 256 * 256
    d = binding.RomDims(D, DE, 16, 4, 8, E, 1, E, 1, 0)

    def call(n=1, B=4, x=at, out=at + 8192, tmp=at + 16384, ffn=True, group=0):
        blocks, ffns = (binding._RomBlock * n)(), (binding._RomFfnWeights * n)()
        for j in range(n):
            blocks[j].w, blocks[j].norm_weight = binding._RomWeights(*([at] * 11)), at
            if ffn:
                ffns[j] = binding._RomFfnWeights(at, at)
        return lib.rom_hybrid_stack_step(ctypes.byref(d), F, blocks, ffns, group, 1, n, ctypes.c_float(1e-5), x, B, at, at, out, tmp, at, 1 << 40,
                                         at + 32768, 1 << 40, None)

    call.at, call.keep = at, buf
    return call


@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("n,ffn", [(1, True), (2, False), (3, True), (1, False), (3, False)])
def test_a_stack_step_is_refused_before_a_state_moves(entry, n, ffn, group):
    """The first block of an even number of them writes tmp: an output that the last one cannot write is seen before."""
    assert entry(n=n, ffn=ffn, group=group, out=entry.at + 8200) == -1
    assert entry(n=n, ffn=ffn, group=group, x=entry.at + 8) == -1


@pytest.mark.parametrize("group", [0, 32])
def test_a_stack_step_of_no_sequences_does_nothing(entry, host, group):
    assert entry(n=3, B=0, x=None, out=None, tmp=None, group=group) == 0       # empty tensors have no address
    assert entry(n=3, B=0, x=entry.at, out=entry.at, tmp=entry.at, group=group) == 0
    stack = hybrid_of(2)
    assert stack.step(tokens(0)[0], *states(0, 2), q4_group=group).shape == (0, D)


def test_plain_4_bit_weights_are_not_packed_from_folded_ones(host):
    """A stack folds its layers' norms into w_in in place: the layer's own step would get the scale that belongs to the block."""
    x, (cs, ss) = tokens(3)[0], states(3)
    layer, early = layer_of(), layer_of()
    early.step_q4(x, cs, ss)                                    # packed from the plain weights
    for ly in (layer, early):
        binding.RomHybridStack([ly], [ffn_of(ly)])
    with pytest.raises(binding.RomError, match="folded"):
        layer.step_q4(x, cs, ss)
    layer.block_step_q4(x, cs, ss), early.step_q4(x, cs, ss)
    apart = layer_of()
    binding.RomHybridStack([apart], [None], fold_in_place=False)
    apart.step_q4(x, cs, ss)


# ---------------------------------------------------------------- workspaces


def test_workspaces_are_sized_by_the_call(host, monkeypatch):
    """One token through wide matrices asks for one token's partial sums; what a size has got is never replaced."""
    asked = []
    empty = torch.empty

    def counted(*size, **kw):
        out = empty(*size, **kw)
        if out.dtype is torch.uint8:
            asked.append(out.numel())
        return out

    q = binding.RomQ4Weight.__new__(binding.RomQ4Weight)
    q.packed, q.n_mats, q.rows, q.cols, q.group = packed_of(1 << 14, D), E, 1 << 14, D, 32
    q.device, q.index, q._ws = torch.device("cpu"), -1, {}
    ffn = ffn_of(layer_of(top_k=2))
    monkeypatch.setattr(torch, "empty", counted)
    need = {"project": lambda n: binding.rom_q4_project_workspace_bytes(q.rows, 2, n),
            "step": lambda n: binding.rom_ffn_step_workspace_bytes(ffn.dims, F, n)}
    for what, call in (("project", lambda n: q.project(tokens(n)[0], *tokens(n, 2)[1:])), ("step", lambda n: ffn.step(*tokens(n, 2), True))):
        for n in (1, 2, 3, 5, 100, 256):
            asked.clear()
            call(n)
            call(n)
            assert len(asked) <= 1 and need[what](n) <= sum(asked) < 2 * need[what](n)      # up to the next power of two
        asked.clear()
        for n in (1, 2, 4, 7, 128, 129, 256, 6):
            call(n)
        assert not asked
    assert need["project"](256) == 256 * need["project"](1)


def test_raw_steps_take_buffers_with_room_for_more(host):
    """B is theirs to say: the tokens, outputs and states of a larger batch, other shapes of as many values."""
    layer, big = layer_of(), 8
    cs, ss = states(big)
    x = torch.zeros(big, 1, D, dtype=torch.bfloat16)
    for call in raw_steps(layer, 32, layer.q4_weights(32)):
        for B in (0, 1, 3):
            call(x=x, out=x.clone(), conv_state=cs, ssm_state=ss, B=B)
    stack = hybrid_of(2)
    cs, ss = states(big, 2)
    binding.rom_hybrid_stack_step(stack.dims, F, stack.blocks, stack.ffn_structs, 0, True, 1e-5, x, 3, cs, ss, x.clone(), x.clone(),
                                  torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(1 << 20, dtype=torch.uint8))
    assert host.lib.calls.count("rom_step_q4") == host.lib.calls.count("rom_block_step_q4") == 3
    for bad in (lambda: layer.step_q4(x, *states(big)), lambda: layer.block_step_q4(x[:3, 0].contiguous(), *states(big)),
                lambda: stack.step(x[:3, 0].contiguous(), cs, ss)):
        with pytest.raises(binding.RomError):                   # a holder's batch is x's
            bad()
