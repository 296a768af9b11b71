"""SiLU(gate) * up of the FFN-MoE step where the gate leaves fp32's range, in each of the kernels that apply it.

SiLU(a) is a * sigmoid(a): a gate of -infinity is -infinity times zero, NaN, and +infinity stays."""
import numpy as np
import pytest
import torch

from paper_2506_18145_amd import RomDims, RomQ4Weight, rom_ffn_moe_step, rom_ffn_step_workspace_bytes
from tests.test_gpu_few_tokens import DEV, TYPES, np64, pack_rows, unit

pytestmark = pytest.mark.gpu

GATES = [-1e4, -14.0, -2.0, 0.0, 2.0, 14.0, 1e4, 3e38, -3e38]        # times 6: the last two are infinite


# one token by a workgroup per rows; several slots; many slots of one expert through LDS (bf16, enough rows for the device)
@pytest.mark.parametrize("dtype,group,N,f", [("bf16", 0, 1, 32), ("fp32", 0, 1, 32), ("bf16", 64, 1, 32), ("bf16", 0, 9, 32), ("fp32", 0, 9, 32),
                                             ("bf16", 64, 9, 32), ("fp32", 32, 90, 32), ("bf16", 0, 252, 2048), ("bf16", 64, 252, 4096)])
def test_ffn_step_of_gates_beyond_fp32(dtype, group, N, f):
    D, E, t = 64, 2, TYPES[dtype]
    gu, down = torch.zeros(E, 2 * f, D, device=DEV, dtype=t), torch.zeros(E, D, f, device=DEV, dtype=t)
    gu[:, 0, 0], gu[:, f, 1], down[:, 0, 0] = 6.0, 6.0, 6.0        # exact in 4 bits too
    gu = pack_rows(gu)
    if group:
        gu, down = RomQ4Weight.pack(gu, group).packed, RomQ4Weight.pack(down, group).packed
    dims = RomDims(D, 16, 16, 4, 1, E, 1, E, 1 if dtype == "bf16" else 0, 0)
    for first in range(len(GATES) if N == 1 else 1):
        x = torch.zeros(N, D, device=DEV, dtype=t)
        x[:, 0] = torch.tensor((GATES[first:] + GATES * (N // len(GATES)))[:N], device=DEV).to(t)
        x[:, 1] = 1.0
        idx, gate = (torch.arange(N, device=DEV, dtype=torch.int32) % E).view(N, 1), torch.ones((N, 1), device=DEV)
        out = torch.empty_like(x)
        ws = torch.empty(rom_ffn_step_workspace_bytes(dims, f, N), dtype=torch.uint8, device=DEV)
        rom_ffn_moe_step(dims, f, gu, down, group, False, 0.0, False, x, N, idx, gate, out, ws)
        got, a = np64(out)[:, 0], 6.0 * np64(x)[:, 0]
        end = np.abs(a) > 3.4028235e38
        assert np.all(got[end & (a > 0)] == np.inf) and np.all(np.isnan(got[end & (a < 0)]))
        with np.errstate(over="ignore"):
            want = (36.0 * a / (1 + np.exp(-a)))[~end]
        # h and the result are rounded once each; exp of an argument within 2^-24 of up to 84, and a handful of fp32 roundings
        tol = (2.01 * unit(dtype) + (84 + 16) * 2.0 ** -24) * np.abs(want) + 1e-37
        assert np.all(np.abs(got[~end] - want) <= tol), (got[~end], want)
