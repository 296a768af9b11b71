"""The few-token operators on the GPU against their 64-bit oracle.

Tolerances.  The final rounding is at most u |result| with u = finfo(T).eps / 2.  An fp32 sum of n products, in any order, is
within n 2^-24 of the sum of the products' sizes; n is the number of columns, with 64 more for scales, gates, norm and SiLU.
Of the FFN-MoE layer: h = SiLU(gate) up is rounded once (u |h|), and summation errors of its two arguments come through its
derivative; the oracle returns both as sizes of the output."""
import numpy as np
import pytest
import torch

from oracle import rom_few_oracle as F
from paper_2506_18145_amd import (RomDims, RomError, RomFfnMoe, RomHybridStack, RomLayer, RomQ4Weight, rom_ffn_moe_step,
                                  rom_ffn_step_workspace_bytes, rom_q4_bytes, rom_q4_pack, rom_q4_project,
                                  rom_q4_project_workspace_bytes)
from rom_synth import RomConfig, make_ffn_weights, make_weights

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def np64(t):
    return t.detach().double().cpu().numpy()


def unit(dtype):
    return torch.finfo(TYPES[dtype]).eps / 2


def randn(seed, *shape, std=1.0, dtype="bf16"):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(TYPES[dtype])


def routing(seed, N, K, E, kind="random"):
    rng = np.random.default_rng(seed)
    if kind == "random":
        idx = np.stack([rng.permutation(E)[:K] for _ in range(N)])
    elif kind == "one":                                        # every slot on one expert
        idx = np.full((N, K), E - 1)
    elif kind == "again":                                      # the same expert twice and more in a row
        idx = rng.integers(0, E, (N, 1)).repeat(K, 1)
    else:                                                      # "missing": some indices name no expert, whole rows of them too
        idx = rng.integers(-2, E + 2, (N, K))
        idx[0] = -1
        idx[-1, 0] = 1 << 30
    gate = rng.uniform(0.05, 1.0, (N, K)).astype(np.float32)
    return torch.from_numpy(idx.astype(np.int32)).to(DEV), torch.from_numpy(gate).to(DEV)


def guarded(n_bytes, fill=0xA5, pad=4096):
    """(whole, the view of n_bytes in its middle): what lies around has to stay."""
    whole = torch.full((n_bytes + 2 * pad,), fill, dtype=torch.uint8, device=DEV)
    return whole, whole[pad:pad + n_bytes]


def untouched(whole, n_bytes, fill=0xA5, pad=4096):
    return bool((whole[:pad] == fill).all()) and bool((whole[pad + n_bytes:] == fill).all())


# ---------------------------------------------------------------- 4 bits


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("E,rows,cols,group", [(1, 8, 8, 32), (3, 24, 136, 64), (2, 16, 128, 128), (2, 40, 200, 32), (1, 8, 1000, 128),
                                               (64, 8, 16, 64), (2, 72, 264, 128)])
def test_pack_and_unpack_bit_for_bit(dtype, E, rows, cols, group):
    w = randn(E * rows + cols, E, rows, cols, dtype=dtype)
    w[0, 0, :8] = torch.tensor([0.0, -0.0, 6.0, 5.0, 3.5, -2.5, 1.25, -0.25], device=DEV)   # ties where 6 is the largest
    w[0, 0, 8:] = w[0, 0, 8:].clamp(-5, 5)
    w[0, 1] = 0.0
    if cols > 8:
        w[0, 2, 9] = float("nan")
        w[0, 3, 10] = float("-inf")
    w[0, 4] *= 1e-38                                            # scales that are subnormal numbers
    w[0, 5] *= 3e37
    need = rom_q4_bytes(E, rows, cols, group)
    whole, packed = guarded(need)
    rom_q4_pack(w, group, packed)
    codes, scales = F.q4_quantize(w.float().cpu().numpy(), group)
    assert np.array_equal(packed.cpu().numpy(), F.q4_layout(codes, scales, group)) and untouched(whole, need)
    values = F.q4_values(codes, scales, group)
    for t in ("fp32", "bf16"):
        n = E * rows * cols * (4 if t == "fp32" else 2)
        whole, out = guarded(n)
        got = RomQ4Weight(packed, E, rows, cols, group)
        from paper_2506_18145_amd import rom_q4_unpack
        rom_q4_unpack(packed, group, out.view(TYPES[t]).view(E, rows, cols))
        want = values if t == "fp32" else F.to_bf16(values.astype(np.float32))
        assert np.array_equal(np64(out.view(TYPES[t]).view(E, rows, cols)), want, equal_nan=True) and untouched(whole, n)
        assert torch.equal(got.unpack(TYPES[t]).view(torch.uint8), out.view(E, rows, -1))


def test_pack_a_whole_layers_weight():
    w = randn(5, 8, 2048, 1024)
    q = RomQ4Weight.pack(w, 64)
    for e, r in ((0, 0), (3, 1000), (7, 2047)):
        codes, scales = F.q4_quantize(w[e:e + 1, r:r + 1].float().cpu().numpy(), 64)
        assert np.array_equal(np64(q.unpack(torch.float32)[e, r]), F.q4_values(codes, scales, 64)[0, 0])


def test_pack_of_every_quotient_of_two_bf16_numbers():
    """Every mantissa of a scale with every bf16 size from 6 s down to 2^-4 s: the code is the one that 64 bits choose."""
    s = (torch.arange(128, 256, device=DEV, dtype=torch.float64) / 128)
    w = torch.arange(128, 256, device=DEV, dtype=torch.float64).repeat(8) * 2.0 ** torch.arange(-11, -3, device=DEV).repeat_interleave(128)
    groups = []
    for part in w.view(-1, 16):                             # 16 sizes, their negatives' mirror and the group's largest
        top = (6 * s).to(torch.bfloat16).double()           # 6 s rounded: its sixth is s again where that is representable
        v = torch.where(part[None, :] <= top[:, None], part[None, :], torch.zeros_like(part)[None, :])
        groups.append(torch.cat([top[:, None], v, -v[:, :15]], dim=1))
    w3 = torch.stack(groups, 1).reshape(1, 128, -1).to(torch.bfloat16)
    q = RomQ4Weight.pack(w3, 32)
    got = q.unpack(torch.float32).double().view(128, -1, 32)
    v = w3.double().view(128, -1, 32)
    scale = (v.abs().amax(-1, keepdim=True) / 6).float().to(torch.bfloat16).double()
    table = torch.tensor(F.E2M1, device=DEV)
    a = v.abs().unsqueeze(-1)
    # the nearest; on a tie (both distances exact in 64 bits) the even code
    d = (a - table * scale.unsqueeze(-1)).abs()
    best = d.amin(-1, keepdim=True)
    code = torch.where((d == best) & (torch.arange(8, device=DEV) % 2 == 0), 0, torch.where(d == best, 1, 2)).argmin(-1)
    assert torch.equal(got, torch.sign(v) * table[code] * scale)


# ---------------------------------------------------------------- routed projection


def q4_of(seed, E, rows, cols, group):
    q = RomQ4Weight.pack(randn(seed, E, rows, cols, std=cols ** -0.5, dtype="fp32"), group)
    return q, np64(q.unpack(torch.float32))


def check_project(q, values, x, idx, gate, row_scale, residual, dtype):
    N, K = idx.shape
    out = torch.full((N, q.rows), float("nan"), dtype=TYPES[dtype], device=DEV)
    ws_bytes = rom_q4_project_workspace_bytes(q.rows, K, N)
    whole, ws = guarded(max(ws_bytes, 256))
    rom_q4_project(q.packed, q.n_mats, q.rows, q.cols, q.group, x, idx, gate, row_scale, residual, out, ws)
    want, size = F.project(np64(x), values, idx.cpu().numpy(), None if gate is None else np64(gate),
                           None if row_scale is None else np64(row_scale), None if residual is None else np64(residual))
    tol = unit(dtype) * np.abs(want) * 1.001 + (q.cols + 64) * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(want)
    err = np.abs(np64(out) - want)
    assert (err <= tol).all(), (float((err - tol).max()), np.argwhere(~(err <= tol))[:5])
    assert untouched(whole, max(ws_bytes, 256))
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,K,E,rows,cols,group,kind", [
    (1, 1, 1, 8, 8, 32, "random"), (1, 1, 8, 64, 256, 64, "random"), (1, 4, 8, 40, 136, 32, "random"), (3, 2, 4, 24, 264, 128, "random"),
    (8, 1, 8, 72, 520, 64, "random"), (5, 1, 3, 16, 128, 128, "missing"), (2, 4, 4, 56, 1000, 64, "again"), (4, 2, 2, 8, 3000, 32, "one"),
    (9, 1, 8, 64, 256, 64, "random"), (5, 2, 4, 40, 136, 32, "missing"), (16, 2, 16, 72, 264, 64, "random"), (17, 1, 4, 136, 520, 128, "one"),
    (33, 8, 64, 24, 96, 32, "random"), (64, 2, 3, 48, 200, 64, "again"), (256, 1, 8, 64, 384, 32, "random"), (256, 8, 16, 32, 128, 128, "missing"),
    (100, 1, 64, 16, 640, 64, "random"), (1, 2, 8, 4104, 136, 64, "random"), (1, 1, 4, 4104, 1160, 128, "random"),
    (1, 2, 4, 4104, 72, 32, "missing"), (255, 2, 2, 24, 72, 64, "random"), (40, 1, 5, 200, 2048, 64, "missing")])
def test_project(dtype, N, K, E, rows, cols, group, kind):
    q, values = q4_of(rows + cols, E, rows, cols, group)
    x = randn(N + cols, N, cols, dtype=dtype)
    idx, gate = routing(N * K + E, N, K, E, kind)
    scale, residual = randn(7, N, dtype="fp32"), randn(8, N, rows, dtype=dtype)
    check_project(q, values, x, idx, None, None, None, dtype)
    check_project(q, values, x, idx, gate, scale, residual, dtype)


@pytest.mark.parametrize("N", [1, 8, 20])
def test_project_with_one_matrix_and_no_choice(N):
    q, values = q4_of(3, 1, 80, 328, 64)
    x = randn(4, N, 328)
    got = q.project(x)
    assert torch.equal(got, q.project(x, torch.zeros((N, 1), dtype=torch.int32, device=DEV)))
    want, size = F.project(np64(x), values, np.zeros((N, 1), int))
    assert (np.abs(np64(got) - want) <= 2.0 ** -8 * np.abs(want) + (328 + 64) * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("N,K", [(3, 2), (8, 1), (30, 2), (30, 1)])
def test_project_residual_may_be_out(N, K):
    q, _ = q4_of(3, 4, 48, 136, 32)
    x, (idx, gate) = randn(4, N, 136), routing(5, N, K, 4)
    res = randn(6, N, 48)
    want = q.project(x, idx, gate, residual=res)
    assert torch.equal(q.project(x, idx, gate, residual=res, out=res), want)


@pytest.mark.parametrize("N,K", [(2, 2), (8, 1), (24, 2), (60, 1)])
def test_a_bad_row_or_matrix_stays_with_its_own(N, K):
    """NaN and infinity in one token, and a NaN group in one expert's row, reach that token and those products only."""
    E, rows, cols = 4, 48, 264
    w = randn(1, E, rows, cols, dtype="fp32")
    w[2, 5, 100] = float("nan")
    q = RomQ4Weight.pack(w, 64)
    x, (idx, gate) = randn(2, N, cols), routing(3, N, K, E)
    clean = q.project(x, idx, gate)
    has = (idx == 2).any(1)
    assert bool(torch.isnan(clean[has][:, 5]).all()) and bool(torch.isfinite(clean[~has]).all())
    assert bool(torch.isfinite(clean[:, [c for c in range(rows) if c != 5]]).all())
    bad = x.clone()
    bad[N - 1, 17] = float("nan")
    if N > 2:
        bad[1, 3] = float("inf")
    got = q.project(bad, idx, gate)
    keep = [n for n in range(N) if n != N - 1 and not (N > 2 and n == 1)]
    assert torch.equal(got[keep].view(torch.int16), clean[keep].view(torch.int16))
    assert bool(torch.isnan(got[N - 1]).all()) and (N <= 2 or not bool(torch.isfinite(got[1]).any()))


@pytest.mark.parametrize("N,K", [(1, 8), (4, 2), (256, 2), (50, 1)])
def test_project_gives_the_same_bits_again(N, K):
    q, _ = q4_of(3, 8, 64, 1024, 64)
    x, (idx, gate) = randn(4, N, 1024), routing(5, N, K, 8)
    want = q.project(x, idx, gate)
    for _ in range(3):
        assert torch.equal(q.project(x, idx, gate), want)


@pytest.mark.parametrize("N,K,dtype", [(12, 1, "bf16"), (12, 2, "bf16"), (200, 1, "bf16"), (12, 2, "fp32")])
def test_a_token_does_not_depend_on_the_others(N, K, dtype):
    cfg, layer, ffn = ffn_holder(192, 320, 4, K, dtype)
    q, _ = q4_of(3, 4, 64, 192, 64)
    x, (idx, gate) = randn(4, N, 192, dtype=dtype), routing(5, N, K, 4)
    other, (idx2, gate2) = randn(6, N, 192, dtype=dtype), routing(7, N, K, 4)
    keep = torch.arange(0, N, 3, device=DEV)
    to = keep.flip(0)                                       # the same tokens elsewhere, among others
    other[to], idx2[to], gate2[to] = x[keep], idx[keep], gate[keep]
    assert torch.equal(q.project(x, idx, gate)[keep], q.project(other, idx2, gate2)[to])
    for group in (0, 64):
        a, b = ffn.step(x, idx, gate, True, True, group), ffn.step(other, idx2, gate2, True, True, group)
        assert torch.equal(a[keep], b[to])


def test_project_refuses_what_does_not_fit():
    q, _ = q4_of(3, 4, 48, 136, 32)
    x, (idx, gate) = randn(4, 3, 136), routing(5, 3, 2, 4)
    for bad in (dict(x=randn(4, 3, 128)), dict(x=x.half()), dict(idx=idx.long()), dict(idx=idx[:2]), dict(gate=gate.double()),
                dict(gate=gate.t()), dict(residual=x), dict(out=torch.empty(3, 48, device=DEV)), dict(x=x.cpu()),
                dict(x=randn(4, 257, 136), idx=routing(1, 257, 1, 4)[0], gate=None), dict(out=x[:, :48])):
        a = dict(x=x, idx=idx, gate=gate, residual=None, out=None)
        a.update(bad)
        with pytest.raises(RomError):
            q.project(a["x"], a["idx"], a["gate"], residual=a["residual"], out=a["out"])
    with pytest.raises(RomError):
        RomQ4Weight(q.packed[1:], 4, 48, 136, 32)
    with pytest.raises(RomError):
        RomQ4Weight.pack(randn(1, 12, 24), 32)                  # rows are no multiple of 8


# ---------------------------------------------------------------- FFN-MoE


def pack_rows(w):
    """[E, 2 f, D] gate rows then up rows -> blocks of 8 gate and 8 up rows"""
    E, r, D = w.shape
    return w.view(E, 2, r // 16, 8, D).transpose(1, 2).reshape(E, r, D).contiguous()


FFN_CASES = [
    (1, 1, 8, 64, 128, "random", 1), (1, 2, 4, 72, 48, "random", 1), (3, 1, 4, 264, 112, "random", 1), (8, 1, 8, 136, 16, "missing", 1),
    (2, 4, 4, 200, 304, "again", 1), (4, 2, 16, 512, 256, "random", 0), (9, 1, 4, 64, 128, "one", 1), (7, 2, 4, 72, 80, "missing", 1),
    (20, 2, 16, 136, 144, "random", 1), (64, 1, 64, 40, 32, "random", 1), (70, 2, 3, 264, 272, "one", 0), (256, 1, 8, 128, 64, "random", 1),
    (256, 2, 16, 64, 48, "missing", 1), (100, 8, 8, 24, 32, "random", 1), (1, 8, 64, 8, 16, "random", 1), (33, 1, 2, 640, 400, "random", 1)]


@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,K,E,D,f,kind,norm", FFN_CASES)
def test_ffn_moe_step(dtype, group, N, K, E, D, f, kind, norm):
    check_ffn(dtype, group, N, K, E, D, f, kind, norm)


# sizes at which the calls take each of the other forms: many slots an expert, many and few row tiles, deep contractions
@pytest.mark.parametrize("dtype,group,N,K,E,D,f,kind,norm", [
    ("bf16", 64, 256, 1, 4, 328, 1424, "missing", 1), ("bf16", 32, 130, 2, 4, 200, 1424, "random", 1), ("bf16", 128, 140, 1, 2, 72, 2064, "one", 0),
    ("bf16", 128, 64, 1, 64, 72, 272, "random", 1), ("bf16", 64, 1, 1, 4, 1160, 48, "random", 1), ("bf16", 64, 9, 2, 4, 136, 2064, "random", 1),
    ("bf16", 0, 256, 1, 4, 200, 1040, "missing", 1), ("bf16", 0, 200, 2, 4, 2056, 48, "random", 0), ("bf16", 0, 9, 1, 8, 72, 1168, "random", 1),
    ("fp32", 0, 64, 1, 64, 264, 144, "random", 1), ("fp32", 64, 64, 1, 64, 264, 144, "random", 1), ("fp32", 0, 9, 1, 4, 2056, 32, "missing", 1)])
def test_ffn_moe_step_in_its_other_forms(dtype, group, N, K, E, D, f, kind, norm):
    check_ffn(dtype, group, N, K, E, D, f, kind, norm)


def check_ffn(dtype, group, N, K, E, D, f, kind, norm):
    gu, down = randn(D, E, 2 * f, D, std=1.5 * D ** -0.5, dtype=dtype), randn(f, E, D, f, std=f ** -0.5, dtype=dtype)
    x = randn(N, N, D, std=1.7, dtype=dtype)
    idx, gate = routing(N + K, N, K, E, kind)
    dims = RomDims(D, 16, 16, 4, 1, E, K, E, 1 if dtype == "bf16" else 0, 0)
    if group:
        q_gu, q_down = RomQ4Weight.pack(pack_rows(gu), group), RomQ4Weight.pack(down, group)
        p_gu, p_down = q_gu.packed, q_down.packed
        back = q_gu.unpack(torch.float32).view(E, f // 8, 2, 8, D).transpose(1, 2).reshape(E, 2 * f, D)
        v_gu, v_down = np64(back), np64(q_down.unpack(torch.float32))
    else:
        p_gu, p_down, v_gu, v_down = pack_rows(gu), down, np64(gu), np64(down)
    need = rom_ffn_step_workspace_bytes(dims, f, N)
    for skip in (True, False):
        whole, ws = guarded(need, fill=0xFF)                    # NaN in every type: nothing may be read before it is written
        out = torch.full((N, D), float("nan"), dtype=TYPES[dtype], device=DEV)
        rom_ffn_moe_step(dims, f, p_gu, p_down, group, norm, 1e-5, skip, x, N, idx, gate, out, ws)
        want, size, carried = F.ffn_step(np64(x), v_gu, v_down, idx.cpu().numpy(), np64(gate), bool(norm), 1e-5, skip)
        u = unit(dtype)
        tol = (u * 1.001 + 2.0 ** -24) * np.abs(want) + u * 1.001 * size + 2.0 ** -24 * ((D + 64) * carried + (f + 64) * size)
        err = np.abs(np64(out) - want)
        assert (err <= tol).all(), (skip, float((err - tol).max()), np.argwhere(~(err <= tol))[:5])
        assert untouched(whole, need, fill=0xFF)


def test_ffn_step_of_a_large_gate_and_of_infinity():
    """SiLU at the ends of fp32: exp overflows and vanishes, the product stays what it is."""
    D, f, E = 64, 32, 1
    gu = torch.zeros(E, 2 * f, D, device=DEV)
    gu[0, :f, 0], gu[0, f:, 1] = 1.0, 1.0
    down = torch.zeros(E, D, f, device=DEV)
    down[0, :f] = torch.eye(f, device=DEV)
    dims = RomDims(D, 16, 16, 4, 1, E, 1, E, 0, 0)
    x = torch.zeros(6, D, device=DEV)
    x[:, 0] = torch.tensor([-1e4, -90.0, 0.0, 90.0, 1e4, 3e38], device=DEV)
    x[:, 1] = 1.0
    idx, gate = torch.zeros((6, 1), dtype=torch.int32, device=DEV), torch.ones((6, 1), device=DEV)
    out = torch.empty_like(x)
    ws = torch.empty(rom_ffn_step_workspace_bytes(dims, f, 6), dtype=torch.uint8, device=DEV)
    rom_ffn_moe_step(dims, f, pack_rows(gu), down, 0, False, 0.0, False, x, 6, idx, gate, out, ws)
    got = np64(out)[:, 0]
    a = np64(x)[:, 0]
    with np.errstate(over="ignore"):
        want = a / (1 + np.exp(-a))
    assert np.all(np.abs(got - want) <= 1e-5 * np.abs(want) + 1e-37), (got, want)


def ffn_holder(D, f, E, K, dtype, seed=0):
    cfg = RomConfig("few", 5, 1, 1, D, 2 * D, 16, 4, 8, E, K, dtype, 1 if K > 1 else 0, weight_std=0.05)
    layer = RomLayer(cfg, make_weights(cfg))
    return cfg, layer, RomFfnMoe(layer, f, make_ffn_weights(cfg, f))


@pytest.mark.parametrize("dtype,K", [("bf16", 1), ("bf16", 2), ("fp32", 2)])
def test_ffn_step_agrees_with_the_layer_on_the_routers_grouping(dtype, K):
    cfg, layer, ffn = ffn_holder(128, 256, 8, K, dtype)
    for n in (1, 6, 40):
        x = randn(n, n, 128, dtype=dtype)
        r = layer.route(x)
        want = ffn.forward(x, r, pre_norm=True, add_skip=True)
        got = ffn.step(x, r["expert_idx"], r["gate"], pre_norm=True, add_skip=True)
        # each of the two is within its own roundings (h, a slot's output, the result) of the layer
        rms = (want - x).float().square().mean().sqrt().item()
        assert (got - want).abs().max().item() <= 8 * unit(dtype) * (want.abs().max().item() + 4 * rms)


def test_ffn_step_refuses_what_does_not_fit():
    cfg, layer, ffn = ffn_holder(64, 32, 4, 2, "bf16")
    x, (idx, gate) = randn(1, 3, 64), routing(2, 3, 2, 4)
    ffn.step(x, idx, gate)
    for bad in (dict(x=x.float()), dict(x=x[:, :32]), dict(idx=idx.long()), dict(idx=idx[:, :1]), dict(gate=gate.half()),
                dict(gate=gate[:2]), dict(q4_group=16), dict(out=x), dict(out=x.float())):
        a = dict(x=x, idx=idx, gate=gate, q4_group=0, out=None)
        a.update(bad)
        with pytest.raises(RomError):
            ffn.step(a["x"], a["idx"], a["gate"], q4_group=a["q4_group"], out=a["out"])
    with pytest.raises(RomError):
        ffn.step(randn(1, 257, 64), *routing(2, 257, 2, 4))
    ws, out = torch.empty(rom_ffn_step_workspace_bytes(ffn.dims, 32, 3), dtype=torch.uint8, device=DEV), torch.empty_like(x)
    gu, down = ffn.packed(False), ffn.w_down
    for bad in (dict(gu=gu[:3]), dict(down=down.float()), dict(group=32), dict(ws=ws[:-1])):
        a = dict(gu=gu, down=down, group=0, ws=ws)
        a.update(bad)
        with pytest.raises(RomError):
            rom_ffn_moe_step(ffn.dims, 32, a["gu"], a["down"], a["group"], False, 1e-5, False, x, 3, idx, gate, out, a["ws"])


@pytest.mark.parametrize("group", [0, 64])
def test_weights_beyond_32_bit_offsets(group):
    """64 experts of 2 x 8192 x 4096: 2^32 gate | up weights; the slots of the last expert against the layer in 64 bits."""
    E, D, f = 64, 4096, 8192
    gu, down = torch.zeros((E, 2 * f, D), dtype=torch.bfloat16, device=DEV), torch.zeros((E, D, f), dtype=torch.bfloat16, device=DEV)
    gu[-1], down[-1] = randn(1, 2 * f, D, std=D ** -0.5), randn(2, D, f, std=f ** -0.5)
    last = gu[-1:].contiguous(), down[-1:].contiguous()
    if group:
        gu, down = RomQ4Weight.pack(gu, group).packed, RomQ4Weight.pack(down, group).packed
        last = tuple(RomQ4Weight.pack(w, group).unpack(torch.float32) for w in last)
    rows, w_down = last[0][0].double().view(f // 8, 2, 8, D), last[1][0].double()
    w_gate, w_up = rows[:, 0].reshape(f, D), rows[:, 1].reshape(f, D)
    dims, u = RomDims(D, 16, 16, 4, 1, E, 1, E, 1, 0), 2.0 ** -8
    for N in (1, 3, 70):
        x, gate, out = randn(N, N, D), torch.ones((N, 1), device=DEV), torch.empty((N, D), dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(rom_ffn_step_workspace_bytes(dims, f, N), dtype=torch.uint8, device=DEV)
        idx = torch.full((N, 1), E - 1, dtype=torch.int32, device=DEV)
        rom_ffn_moe_step(dims, f, gu, down, group, True, 1e-5, True, x, N, idx, gate, out, ws)
        xd = x.double()
        xn = xd / (xd.square().mean(-1, keepdim=True) + 1e-5).sqrt()
        a, b, sa, sb = xn @ w_gate.t(), xn @ w_up.t(), xn.abs() @ w_gate.abs().t(), xn.abs() @ w_up.abs().t()
        silu = a / (1 + torch.exp(-a))
        want, size = xd + (silu * b) @ w_down.t(), (silu * b).abs() @ w_down.abs().t()
        carried = (1.1 * sa * b.abs() + silu.abs() * sb + (silu * b).abs() * (a.abs() + 4)) @ w_down.abs().t()
        tol = (u * 1.001 + 2.0 ** -24) * want.abs() + u * 1.001 * size + 2.0 ** -24 * ((D + 64) * carried + (f + 64) * size)
        assert bool(((out.double() - want).abs() <= tol).all())
        # roundings of 8192 terms do not add up: 1/16 of the bound on h holds a mistake that the worst case would let through
        assert (out.double() - want).norm().item() <= (u * want.abs() + u * size / 16).norm().item()
    del gu, down
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- steps


def states(cfg, seed, n_layers=None):
    lead = () if n_layers is None else (n_layers,)
    return (randn(seed, *lead, cfg.batch, cfg.d_inner, 3, dtype="fp32"), randn(seed + 1, *lead, cfg.batch, cfg.d_inner, 16, dtype="fp32"))


def step_cfg(**kw):
    base = dict(name="few", cfg_id=6, batch=3, seq_len=1, d_model=128, d_inner=256, d_state=16, d_conv=4, dt_rank=8, n_experts=4,
                top_k=1, dtype="bf16", gate_mode=0, step=True, weight_std=0.06)
    base.update(kw)
    return RomConfig(**base)


@pytest.mark.parametrize("block", [False, True])
@pytest.mark.parametrize("kw", [dict(), dict(batch=1, top_k=2, gate_mode=1), dict(batch=20), dict(batch=12, top_k=2, gate_mode=1),
                                dict(dtype="fp32"), dict(dtype="fp32", batch=9, top_k=2), dict(batch=256, routed_xdt=False),
                                dict(d_model=72, d_inner=112, batch=5)])
def test_step_q4_against_the_oracle(kw, block):
    from oracle import rom_oracle as O
    from tests.gpu_util import ELEM_TOL, TOL, rel_err
    cfg = step_cfg(**kw)
    w_np = make_weights(cfg)
    w_np["norm_w"] = np.random.default_rng(1).uniform(0.7, 1.3, cfg.d_model).astype(np.float32)
    layer = RomLayer(cfg, w_np)
    x, (cs, ss) = randn(3, cfg.batch, cfg.d_model, dtype=cfg.dtype), states(cfg, 4)
    cs0, ss0 = np64(cs), np64(ss)
    got = (layer.block_step_q4 if block else layer.step_q4)(x, cs, ss, group=32)
    idx = layer.ws_view("expert_idx", cfg.batch, 1).cpu().numpy()
    ref_w = {k: None if v is None else np64(v) for k, v in layer.weights.items()}
    q = layer.q4_weights(32, block)
    E = cfg.n_experts
    w_in = np64(RomQ4Weight(q["w_in"], E, 2 * cfg.d_inner, cfg.d_model, 32).unpack(torch.float32))
    ref_w["w_out"] = np64(RomQ4Weight(q["w_out"], E, cfg.d_model, cfg.d_inner, 32).unpack(torch.float32))
    if block:        # the packed weight carries the norm's scale: give the oracle one that it multiplies back in
        ref_w["w_in"] = w_in / ref_w["norm_w"]
        ref = O.rom_block_forward(np64(x)[:, None], ref_w, cfg.top_k, cfg.gate_mode, 1e-5, cs0, ss0, expert_idx=idx)
        ref["out"] = ref["out"][:, 0]
    else:
        ref_w["w_in"] = w_in
        ref = O.rom_step(np64(x), ref_w, cfg.top_k, cfg.gate_mode, cs0, ss0, expert_idx=idx)
    assert rel_err(np64(got), ref["out"]) <= TOL[cfg.dtype]
    assert rel_err(np64(cs), ref["conv_state"]) <= TOL[cfg.dtype] and rel_err(np64(ss), ref["ssm_state"]) <= TOL[cfg.dtype]


def hybrid(cfg, n_layers=3, f=96, holes=(1,)):
    layers, ffns = [], []
    for j in range(n_layers):
        w = make_weights(RomConfig(**{**cfg.__dict__, "cfg_id": 10 + j}))
        w["norm_w"] = np.random.default_rng(j).uniform(0.7, 1.3, cfg.d_model).astype(np.float32)
        layers.append(RomLayer(cfg, w))
        fw = make_ffn_weights(RomConfig(**{**cfg.__dict__, "cfg_id": 20 + j}), f)
        ffns.append(None if j in holes else RomFfnMoe(layers[-1], f, fw))
    return RomHybridStack(layers, ffns)


@pytest.mark.parametrize("group", [0, 64])
@pytest.mark.parametrize("kw", [dict(), dict(batch=1, top_k=2, gate_mode=1), dict(batch=20), dict(batch=40), dict(dtype="fp32", batch=2),
                                dict(dtype="fp32", batch=50)])
def test_hybrid_step_is_the_calls_one_by_one(kw, group):
    cfg = step_cfg(**kw)
    stack = hybrid(cfg)
    cs, ss = states(cfg, 7, 3)
    cs1, ss1 = cs.clone(), ss.clone()
    for t in range(2):
        x = randn(30 + t, cfg.batch, cfg.d_model, dtype=cfg.dtype)
        got = stack.step(x, cs, ss, q4_group=group)
        h = x
        for j, (layer, ffn) in enumerate(zip(stack.layers, stack.ffns)):
            h = layer.block_step_q4(h, cs1[j], ss1[j], group) if group else layer.block_step(h, cs1[j], ss1[j])
            slots = cfg.batch * cfg.top_k
            if ffn is None:
                continue
            if group or cfg.dtype == "fp32" or slots <= 8 * min(slots, cfg.n_experts):
                h = ffn.step(h, layer.ws_view("expert_idx", cfg.batch, 1), layer.ws_view("gate", cfg.batch, 1), True, True, group)
            else:
                routing = {n: layer.ws_view(n, cfg.batch, 1) for n in ("offsets", "perm", "inv_perm", "gate")}
                h = ffn.forward(h, routing, True, True)
        assert torch.equal(got, h) and torch.equal(cs, cs1) and torch.equal(ss, ss1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_steps_behind_a_prefill_give_the_whole_sequence(dtype):
    """Prefill of 5 tokens by the stack's forward, 4 steps behind it: the outputs of one forward over 9 tokens."""
    from tests.gpu_util import TOL, rel_err
    cfg = step_cfg(dtype=dtype, batch=2, seq_len=9, step=False, router_bias=(3.0, 0.0, -3.0, -6.0))   # far from ties
    stack = hybrid(cfg, holes=())
    x = randn(1, 2, 9, cfg.d_model, dtype=dtype)
    want = stack.forward(x)
    out, cs, ss = stack.forward(x[:, :5].contiguous(), return_states=True)
    for t in range(5, 9):
        got = stack.step(x[:, t].contiguous(), cs, ss)
        assert rel_err(np64(got), np64(want[:, t])) <= TOL[dtype]


def test_hybrid_step_of_more_sequences_than_few():
    cfg = step_cfg(batch=300)
    stack = hybrid(cfg)
    cs, ss = states(cfg, 7, 3)
    cs1, ss1 = cs.clone(), ss.clone()
    x = randn(9, 300, cfg.d_model)
    got = stack.step(x, cs, ss)
    out, cs2, ss2 = stack.forward(x[:, None].contiguous(), cs1, ss1, return_states=True)
    assert torch.equal(got, out[:, 0]) and torch.equal(cs, cs2) and torch.equal(ss, ss2)
    with pytest.raises(RomError):
        stack.step(x, cs, ss, q4_group=64)


# ---------------------------------------------------------------- graphs, streams


@pytest.mark.parametrize("group", [0, 64])
@pytest.mark.parametrize("kw", [dict(batch=2, top_k=2, gate_mode=1), dict(batch=33)])
def test_hybrid_step_replayed_from_a_graph(kw, group):
    cfg = step_cfg(**kw)
    stack = hybrid(cfg)
    x0 = randn(1, cfg.batch, cfg.d_model)
    cs0, ss0 = states(cfg, 7, 3)
    x, cs, ss = x0.clone(), cs0.clone(), ss0.clone()
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        stack.step(x, cs, ss, group, out)                       # packs and allocates
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stack.step(x, cs, ss, group, out)
    stack.forward(randn(2, 4, 90, cfg.d_model))                 # a larger eager call in between: the graph's memory stays
    cs.copy_(cs0), ss.copy_(ss0)
    want_cs, want_ss = cs0.clone(), ss0.clone()
    for t in range(4):
        x.copy_(randn(50 + t, cfg.batch, cfg.d_model))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = stack.step(x, want_cs, want_ss, group)
        assert torch.equal(got, want) and torch.equal(cs, want_cs) and torch.equal(ss, want_ss)


def test_weights_are_not_packed_by_a_capture():
    cfg, layer, ffn = ffn_holder(64, 32, 4, 1, "bf16")
    x, (idx, gate) = randn(1, 3, 64), routing(2, 3, 1, 4)
    cs, ss = randn(1, 3, 128, 3, dtype="fp32"), randn(2, 3, 128, 16, dtype="fp32")
    want = ffn.step(x, idx, gate)                               # plain weights: nothing to lay out
    refused = []
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ffn.step(x, idx, gate)
        for call in (lambda: ffn.step(x, idx, gate, q4_group=32), lambda: layer.step_q4(x, cs, ss, 32)):
            try:
                call()
            except RomError as e:
                refused.append("before a capture" in str(e))
    graph.replay()
    torch.cuda.synchronize()
    assert refused == [True, True] and torch.equal(out, want)
    assert bool(torch.isfinite(ffn.step(x, idx, gate, q4_group=32)).all())


def test_two_graphs_of_one_holder_replayed_in_turn():
    """Calls of different sizes of the same holders captured into two graphs: they share a workspace and follow each other."""
    cfg, layer, ffn = ffn_holder(128, 256, 8, 2, "bf16")
    q, _ = q4_of(3, 8, 256, 128, 64)
    sets = []
    for N in (30, 3):
        x, (idx, gate) = randn(N, N, 128), routing(N, N, 2, 8)
        ffn.step(x, idx, gate, True, True, 64), q.project(x, idx, gate)
        out, out2 = torch.empty_like(x), torch.empty((N, 256), dtype=x.dtype, device=DEV)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ffn.step(x, idx, gate, True, True, 64, out)
            q.project(x, idx, gate, out=out2)
        sets.append((g, x, idx, gate, out, out2))
    for t in range(4):
        for g, x, idx, gate, out, out2 in sets:
            x.copy_(randn(100 + t, *x.shape))
            idx.copy_(routing(t, x.shape[0], 2, 8)[0])
        for g, *_ in sets:
            g.replay()
        torch.cuda.synchronize()
        for g, x, idx, gate, out, out2 in sets:
            assert torch.equal(out, ffn.step(x, idx, gate, True, True, 64)) and torch.equal(out2, q.project(x, idx, gate))


def test_two_holders_on_two_streams():
    streams = [torch.cuda.Stream() for _ in range(2)]
    held = []
    for j in range(2):
        q, _ = q4_of(3 + j, 8, 256, 1024, 64)
        x, (idx, gate) = randn(4 + j, 40, 1024), routing(5 + j, 40, 2, 8)
        held.append((q, x, idx, gate, q.project(x, idx, gate)))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for j, s in enumerate(streams):
            with torch.cuda.stream(s):
                q, x, idx, gate, _ = held[j]
                got[j].append(q.project(x, idx, gate))
    torch.cuda.synchronize()
    assert all(torch.equal(g, held[j][4]) for j in range(2) for g in got[j])
