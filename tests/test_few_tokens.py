"""The few-token entry points without a GPU: sizes, refusals (every one before anything is launched), workspaces."""
import ctypes

import pytest

from paper_2506_18145_amd import binding
from paper_2506_18145_amd.build import build_library

F = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(binding._LIB_PATH):
        build_library()
    return binding.load_library()


@pytest.fixture(scope="module")
def addr():
    buf = ctypes.create_string_buffer(1 << 16)
    yield (ctypes.addressof(buf) + 255) // 256 * 256


def dims(**kw):
    base = dict(d_model=64, d_inner=128, d_state=16, d_conv=4, dt_rank=8, n_experts=4, top_k=1, n_experts_xdt=4, dtype=0,
                gate_mode=0)
    base.update(kw)
    return binding.RomDims(**base)


@pytest.mark.parametrize("n,rows,cols,group,want", [
    (1, 8, 8, 32, 16 * 128 // 2 + 16 * 4 * 2), (1, 8, 8, 128, 16 * 128 // 2 + 16 * 2), (3, 24, 136, 64, 3 * 32 * 256 // 2 + 3 * 32 * 4 * 2),
    (64, 16, 128, 32, 64 * (1024 + 128)), (8, 8192, 2048, 64, 8 * 8192 * 2048 // 2 * 17 // 16)])
def test_q4_bytes(lib, n, rows, cols, group, want):
    assert binding.rom_q4_bytes(n, rows, cols, group) == want


@pytest.mark.parametrize("n,rows,cols,group,code", [
    (0, 8, 8, 32, -1), (1, 0, 8, 32, -1), (1, 8, -8, 32, -1), (1, 8, 8, 16, -1), (1, 8, 8, 0, -1), (1, 8, 8, 256, -1),
    (65, 8, 8, 32, -3), (1, 12, 8, 32, -3), (1, 8, 12, 32, -3), (1, (1 << 20) + 8, 8, 32, -3), (1, 8, (1 << 20) + 8, 32, -3),
    (64, 1 << 20, 1 << 20, 32, -3)])
def test_sizes_that_are_refused(lib, addr, n, rows, cols, group, code):
    assert binding.rom_q4_bytes(n, rows, cols, group) == 0
    assert lib.rom_q4_pack(1, addr, n, rows, cols, group, addr + 4096, None) == code
    assert lib.rom_q4_unpack(1, addr, n, rows, cols, group, addr + 4096, None) == code
    assert lib.rom_q4_project(1, addr, n, rows, cols, group, addr, 1, 1, addr, None, None, None, addr + 4096, None, 0, None) == code


def test_conversion_arguments(lib, addr):
    for fn in (lib.rom_q4_pack, lib.rom_q4_unpack):
        assert fn(2, addr, 1, 8, 8, 32, addr + 4096, None) == -1
        assert fn(1, None, 1, 8, 8, 32, addr, None) == -1
        assert fn(1, addr, 1, 8, 8, 32, None, None) == -1
        assert fn(1, addr, 1, 8, 8, 32, addr, None) == -1               # in place
        assert fn(1, addr + 8, 1, 8, 8, 32, addr + 4096, None) == -1
        assert fn(1, addr, 1, 8, 8, 32, addr + 4104, None) == -1


def test_project_arguments(lib, addr):
    base = dict(dtype=1, w=addr, n=4, rows=64, cols=64, group=32, x=addr, N=3, K=1, idx=addr, gate=None, scale=None,
                res=None, out=addr + 4096, ws=None, ws_bytes=0)

    def call(**kw):
        a = dict(base, **kw)
        return lib.rom_q4_project(a["dtype"], a["w"], a["n"], a["rows"], a["cols"], a["group"], a["x"], a["N"], a["K"], a["idx"],
                                  a["gate"], a["scale"], a["res"], a["out"], a["ws"], a["ws_bytes"], None)

    assert call(dtype=2) == -1
    assert call(w=None) == -1 and call(w=addr + 8) == -1
    assert call(x=None) == -1 and call(x=addr + 8) == -1 and call(out=None) == -1 and call(out=addr + 4104) == -1
    assert call(out=addr) == -1                                        # out is x
    assert call(res=addr + 8) == -1
    assert call(N=-1) == -1 and call(K=0) == -1
    assert call(N=257) == -3 and call(K=9) == -3
    assert call(idx=None) == -1                                        # four matrices and no choice
    assert call(idx=None, n=1, K=2) == -1
    assert call(N=0) == 0 and call(N=0, x=None, out=None) == 0
    need = binding.rom_q4_project_workspace_bytes(64, 2, 256)
    assert need > 0
    assert call(N=256, K=2, ws=None, ws_bytes=need) == -1
    assert call(N=256, K=2, ws=addr + 128, ws_bytes=need) == -1
    assert call(N=256, K=2, ws=addr, ws_bytes=need - 1) == -2


def test_project_workspace_of_a_call_serves_every_smaller_one(lib):
    for k in range(1, 9):
        sizes = [binding.rom_q4_project_workspace_bytes(2056, k, n) for n in range(0, 257)]
        assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)
    assert binding.rom_q4_project_workspace_bytes(64, 9, 1) == 0 and binding.rom_q4_project_workspace_bytes(64, 1, 257) == 0


def test_ffn_step_arguments(lib, addr):
    d = dims(top_k=2)
    need = binding.rom_ffn_step_workspace_bytes(d, 32, 8)
    assert need >= 8 * 2 * 32 * 4
    sizes = [binding.rom_ffn_step_workspace_bytes(d, 32, n) for n in range(1, 257)]
    assert sizes == sorted(sizes)
    assert binding.rom_ffn_step_workspace_bytes(d, 32, 257) == 0
    assert binding.rom_ffn_step_workspace_bytes(d, 24, 8) == 0
    w = binding._RomFfnWeights(addr, addr)

    def call(d=d, d_ff=32, w=w, group=0, norm=1, eps=1e-5, x=addr, N=8, idx=addr, gate=addr, out=addr + 8192, ws=addr, nbytes=need):
        return lib.rom_ffn_moe_step(ctypes.byref(d), d_ff, ctypes.byref(w), group, norm, F(eps), 1, x, N, idx, gate, out, ws,
                                    nbytes, None)

    assert call(d_ff=24) == -3 and call(d_ff=0) == -1 and call(d=dims(d_state=8)) == -3
    assert call(group=16) == -1 and call(group=-32) == -1
    assert call(group=32, d_ff=(1 << 19) + 16) == -3
    assert call(w=binding._RomFfnWeights(None, addr)) == -1 and call(w=binding._RomFfnWeights(addr, addr + 8)) == -1
    assert call(eps=-1.0) == -1 and call(eps=float("nan")) == -1
    assert call(N=-1) == -1 and call(N=257, nbytes=1 << 30) == -3 and call(N=0) == 0
    assert call(x=None) == -1 and call(out=addr) == -1 and call(idx=None) == -1 and call(gate=None) == -1
    assert call(x=addr + 8) == -1 and call(out=addr + 8200) == -1 and call(ws=None) == -1 and call(ws=addr + 16) == -1
    assert call(nbytes=need - 1) == -2


def test_step_q4_arguments(lib, addr):
    d, w = dims(), binding._RomWeights(*([addr] * 11))
    plain, need = binding.rom_workspace_bytes(d, 4, 1), binding.rom_step_q4_workspace_bytes(d, 4)
    assert need >= plain > 0
    two = dims(top_k=2)
    assert binding.rom_step_q4_workspace_bytes(two, 256) > binding.rom_workspace_bytes(two, 256, 1)
    assert binding.rom_step_q4_workspace_bytes(d, 257) == 0 and binding.rom_step_q4_workspace_bytes(dims(top_k=9), 4) == 0
    step = lambda group=32, B=4, cs=addr, ss=addr, x=addr, out=addr + 8192, nbytes=need: lib.rom_step_q4(
        ctypes.byref(d), ctypes.byref(w), group, x, B, cs, ss, out, addr, nbytes, None)
    block = lambda group=32, B=4, norm=addr, eps=1e-5, cs=addr, nbytes=need: lib.rom_block_step_q4(
        ctypes.byref(d), ctypes.byref(w), group, norm, F(eps), addr, B, cs, addr, addr + 8192, addr, nbytes, None)
    for f in (step, block):
        assert f(group=0) == -1 and f(group=48) == -1 and f(B=-1) == -1 and f(B=257) == -3 and f(B=0) == 0
        assert f(cs=None) == -1 and f(nbytes=need - 1) == -2
    assert step(out=addr) == -1 and step(x=None) == -1
    assert block(norm=None) == -1 and block(eps=-1.0) == -1


def test_hybrid_step_arguments(lib, addr):
    d = dims()
    blocks, ffns = (binding._RomBlock * 2)(), (binding._RomFfnWeights * 2)()
    for j in range(2):
        blocks[j].w = binding._RomWeights(*([addr] * 11))
        blocks[j].norm_weight = addr
        ffns[j] = binding._RomFfnWeights(addr, addr)
    for group in (0, 32):
        ws = binding.rom_step_q4_workspace_bytes(d, 4) if group else binding.rom_workspace_bytes(d, 4, 1)
        fws = binding.rom_hybrid_step_ffn_workspace_bytes(d, 32, 4, group)
        assert fws > 0

        def call(n=2, B=4, cs=addr, x=addr, out=addr + 8192, tmp=addr + 16384, w=addr, wb=ws, f=addr + 32768, fb=fws, eps=1e-5,
                 g=group, blk=blocks, ff=ffns):
            return lib.rom_hybrid_stack_step(ctypes.byref(d), 32, blk, ff, g, 1, n, F(eps), x, B, cs, addr, out, tmp, w, wb, f, fb, None)

        assert call(n=0) == -1 and call(blk=None) == -1 and call(ff=None) == -1 and call(B=-1) == -1
        assert call(g=7) == -1 and call(eps=-1.0) == -1
        assert call(tmp=None) == -1 and call(tmp=addr) == -1 and call(tmp=addr + 8192) == -1
        assert call(out=addr) == -1 and call(cs=None) == -1 and call(x=None) == -1
        assert call(f=None) == -1 and call(f=addr) == -1 and call(f=addr + 32768 + 16) == -1
        assert call(wb=ws - 1) == -2 and call(fb=fws - 1) == -2
        assert call(B=0) == 0
    assert binding.rom_hybrid_step_ffn_workspace_bytes(d, 32, 257, 32) == 0
    sizes = [binding.rom_hybrid_step_ffn_workspace_bytes(d, 32, b, 0) for b in (1, 8, 255, 256, 257, 300, 1000, 5000)]
    assert sizes == sorted(sizes)
    blocks[1].norm_weight = None                  # a bad second layer is refused before the first one runs
    assert lib.rom_hybrid_stack_step(ctypes.byref(d), 32, blocks, ffns, 0, 1, 2, F(1e-5), addr, 4, addr, addr, addr + 8192,
                                     addr + 16384, addr, 1 << 40, addr + 32768, 1 << 40, None) == -1
