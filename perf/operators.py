"""The few-token operators with 16- or 32-bit and 4-bit weights, as a user's program calls them, and in their plain form.

  listed()            the named cases
  draw(rng)           one more case out of the same ranges
  prepare(case, seed) weights (packed, where they are held in 4 bits), tokens and their routing, on the GPU, from the seed alone
  run(state)          one pass; its outputs
  work(case)          bytes and operations that one pass cannot do without
  exact(case, seed)   the same outputs from the definitions in 64 bits

Kinds:
  pack      weights to 4 bits and back: what a load does before the step and, for a prefill, after it
  project   routed matrix-vector products with 4-bit weights (in and out projection of a step)
  ffn       a whole FFN-MoE layer for a few tokens, 16- or 32-bit weights
  ffn_q4    the same layer with 4-bit weights

The 4-bit format, for a stack [n_mats, rows, cols] in groups of G columns: rows are padded to 16, columns to 128.  First
the codes, [n_mats][rows/16][cols/128][q 4][r 16][j 4][4 bytes]: the eight codes of row r, columns 32 j + 8 q + (0 .. 7), low
nibble first.  Then the scales, bf16 [n_mats][rows/16][cols/G][16].  A code is a sign bit over an E2M1 number.
"""
import math
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _case(kind, N, d_in, d_out, E=8, K=1, dtype="bf16", group=64, norm=True, gated=True, skew=False):
    """d_in, d_out: columns and rows of the projection; d_model and d_ff of the FFN-MoE layer."""
    return dict(kind=kind, N=N, d_in=d_in, d_out=d_out, E=E, K=K, dtype=dtype, group=group, norm=norm, gated=gated, skew=skew)


def listed():
    def named(name, *a, **k):
        return dict(_case(*a, **k), name=name)

    return [
        # loading the tiny full-precision research layer's projections
        named("pack_tiny_fp32", "pack", 0, 64, 256, E=4, dtype="fp32", group=32),
        # loading the in projections of one layer of the 1.3B-active model
        named("pack_in_proj", "pack", 0, 2048, 8192),
        # one matrix, one token: the output head's or a shared projection's smallest call, all latency
        named("project_1tok_dense", "project", 1, 1024, 2048, E=1, gated=False),
        # one user's next token through the routed in projection
        named("project_1tok", "project", 1, 2048, 8192, gated=False),
        # a handful of users, two experts each, an odd width, full precision
        named("project_5tok_top2_fp32", "project", 5, 1048, 2072, E=4, K=2, dtype="fp32", group=128),
        # a server's decode step over 256 sequences through the out projection
        named("project_256tok", "project", 256, 4096, 2048),
        # one user's next token through an FFN-MoE layer
        named("ffn_1tok", "ffn", 1, 2048, 4096),
        # beam search: eight tokens, two experts each
        named("ffn_8tok_top2", "ffn", 8, 1024, 2048, E=16, K=2),
        # the tiny full-precision layer
        named("ffn_3tok_fp32", "ffn", 3, 64, 128, E=4, dtype="fp32"),
        # 4 bits: one user's next token
        named("ffn_q4_1tok", "ffn_q4", 1, 2048, 4096),
        # a small server batch
        named("ffn_q4_32tok", "ffn_q4", 32, 2048, 4096, group=32),
        # 256 sequences, 16 experts, top-2, half of all slots on one expert
        named("ffn_q4_256tok_top2", "ffn_q4", 256, 2048, 4096, E=16, K=2, group=128, skew=True),
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) // step * step)


def draw(rng):
    kind = rng.choice(["pack", "project", "project", "ffn", "ffn_q4", "ffn_q4"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    E = rng.choice([1, 2, 4, 8, 8, 16])
    K = min(E, rng.choice([1, 1, 1, 2, 2, 4]))
    group = rng.choice([32, 64, 128])
    N = _log_int(rng, 1, min(256, 512 // K))
    d_in = _log_int(rng, 64, 2048, 8)
    if kind == "ffn":
        E, K, d_in = min(E, 8), min(K, 8), d_in if dtype == "bf16" else d_in // 16 * 8
    if kind.startswith("ffn"):
        return _case(kind, N, d_in, _log_int(rng, 64, 4096, 16), E, K, dtype, group, norm=rng.random() < 0.7, skew=rng.random() < 0.3)
    if kind == "pack":
        return _case(kind, 0, d_in, _log_int(rng, 64, 8192, 8), min(E, 8 if dtype == "bf16" else 4), 1, dtype, group)
    return _case(kind, N, d_in, _log_int(rng, 64, 8192, 8), E, K, dtype, group, gated=rng.random() < 0.5, skew=rng.random() < 0.3)


# ---------------------------------------------------------------- the 4-bit format, in plain operations


def _quantize(w, group):
    """(codes uint8 [E, rows, cols padded to the group], scales bf16 [E, rows, groups]) of w [E, rows, cols]."""
    E, rows, cols = w.shape
    n = -(-cols // group)
    v = torch.nn.functional.pad(w.float(), (0, n * group - cols)).view(E, rows, n, group)
    top = v.abs().amax(-1)
    scale = (top / torch.full_like(top, 6.0)).to(torch.bfloat16)
    s = scale.float().unsqueeze(-1)
    a = v.abs()
    # midpoints between neighbours; a tie goes to the even code, so every second comparison takes the midpoint itself
    code = sum(((a > t * s) if i % 2 == 0 else (a >= t * s)).to(torch.uint8) for i, t in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)))
    code = torch.where((s > 0) & (code > 0), code + 8 * (v < 0).to(torch.uint8), torch.zeros_like(code))
    return code.view(E, rows, n * group), scale


def _pack(codes, scale, group):
    E, rows, c = codes.shape
    rp, cp = -(-rows // 16) * 16, -(-c // 128) * 128
    codes = torch.nn.functional.pad(codes, (0, cp - c, 0, rp - rows))
    b = codes[..., 0::2] | (codes[..., 1::2] << 4)
    b = b.view(E, rp // 16, 16, cp // 128, 4, 4, 4).permute(0, 1, 3, 5, 2, 4, 6).reshape(-1)       # E tile r c j q byte -> E tile c q r j byte
    scale = torch.nn.functional.pad(scale, (0, cp // group - scale.shape[2], 0, rp - rows))
    scale = scale.view(E, rp // 16, 16, cp // group).transpose(2, 3).reshape(-1)
    return torch.cat([b, scale.view(torch.uint8)])


def _values(packed, E, rows, cols, group):
    """float32 [E, rows, cols]: what the packed weights stand for."""
    rp, cp = -(-rows // 16) * 16, -(-cols // 128) * 128
    n = E * rp * cp // 2
    b = packed[:n].view(E, rp // 16, cp // 128, 4, 16, 4, 4).permute(0, 1, 4, 2, 5, 3, 6).reshape(E, rp, cp // 2)
    codes = torch.stack([b & 15, b >> 4], dim=-1).view(-1).int()
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=packed.device)
    v = table.index_select(0, codes).view(E, rp, cp // group, group)
    scale = packed[n:].view(torch.bfloat16).view(E, rp // 16, cp // group, 16).transpose(2, 3).reshape(E, rp, cp // group)
    return (v * scale.float().unsqueeze(-1)).view(E, rp, cp)[:, :rows, :cols]


# ---------------------------------------------------------------- state


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[c["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=DEV) * std

    E, N, K, d_in, d_out = c["E"], c["N"], c["K"], c["d_in"], c["d_out"]
    s = SimpleNamespace(case=dict(c), call=None)
    std = 1.0 / math.sqrt(d_in)
    if c["kind"] == "pack":
        s.w = normal(E, d_out, d_in, std=std).to(t)
        return s
    logits = normal(N, E)
    if c["skew"]:
        logits[:, 0] += 5.0
    top = logits.topk(K, dim=-1)
    s.expert_idx = top.indices.to(torch.int32).contiguous()
    s.gate = torch.softmax(top.values, dim=-1).contiguous() if K > 1 else torch.softmax(logits, dim=-1).gather(1, top.indices).contiguous()
    x = normal(N, d_in)
    s.x = (x / x.square().mean(-1, keepdim=True).sqrt() * (0.5 + torch.rand((N, 1), generator=g, device=DEV))).to(t)
    if c["kind"] == "project":
        s.w = _pack(*_quantize(normal(E, d_out, d_in, std=std).to(t), c["group"]), c["group"])
        s.residual = normal(N, d_out).to(t) if c["gated"] else None      # the out projection adds the block's input
        return s
    # gate and up features in blocks of eight of each, as the layer's packed row order has them
    s.w_gate_up = normal(E, 2 * d_out, d_in, std=std).to(t)
    s.w_down = normal(E, d_in, d_out, std=1.0 / math.sqrt(d_out)).to(t)
    if c["kind"] == "ffn_q4":
        s.w_gate_up = _pack(*_quantize(s.w_gate_up, c["group"]), c["group"])
        s.w_down = _pack(*_quantize(s.w_down, c["group"]), c["group"])
    return s


# ---------------------------------------------------------------- one pass


def _routed(w, x, expert_idx):
    """[N, K, rows]: every token's K experts' products with its row, or with its K rows (x [N, K, cols])."""
    N, K = expert_idx.shape
    if x.dim() == 2:
        y = (w @ x.t().contiguous()).permute(2, 0, 1)                    # [N, E, rows]
        return y.gather(1, expert_idx.long().unsqueeze(-1).expand(N, K, w.shape[1]))
    y = (w @ x.reshape(N * K, -1).t().contiguous()).permute(2, 0, 1)     # [N K, E, rows]
    return y.gather(1, expert_idx.long().view(N * K, 1, 1).expand(N * K, 1, w.shape[1])).view(N, K, -1)


def _plain(s):
    c = s.case
    E, N, K, d_in, d_out, t = c["E"], c["N"], c["K"], c["d_in"], c["d_out"], TYPES[c["dtype"]]
    if c["kind"] == "pack":
        return _values(_pack(*_quantize(s.w, c["group"]), c["group"]), E, d_out, d_in, c["group"]).to(t).contiguous()
    x = s.x.float()
    if c["kind"] == "project":
        y = _routed(_values(s.w, E, d_out, d_in, c["group"]), x, s.expert_idx)
        y = (y * s.gate.unsqueeze(-1) if c["gated"] else y).sum(1)
        return (y + s.residual.float() if c["gated"] else y).to(t)
    q4 = c["kind"] == "ffn_q4"
    xn = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) if c["norm"] else x
    h = _routed(_values(s.w_gate_up, E, 2 * d_out, d_in, c["group"]) if q4 else s.w_gate_up.float(), xn, s.expert_idx)
    h = h.view(N, K, d_out // 8, 2, 8)
    a, b = h[:, :, :, 0].reshape(N, K, d_out), h[:, :, :, 1].reshape(N, K, d_out)
    y = _routed(_values(s.w_down, E, d_in, d_out, c["group"]) if q4 else s.w_down.float(), a * torch.sigmoid(a) * b, s.expert_idx)
    return (x + (y * s.gate.unsqueeze(-1)).sum(1)).to(t)


def _call(s):
    """The call that a user's program makes again and again, its workspace and outputs allocated once."""
    from paper_2506_18145_amd import RomDims, RomQ4Weight, rom_ffn_moe_step, rom_ffn_step_workspace_bytes

    c = s.case
    E, N, K, d_in, d_out = c["E"], c["N"], c["K"], c["d_in"], c["d_out"]
    if c["kind"] == "pack":
        return lambda: RomQ4Weight.pack(s.w, c["group"]).unpack(s.w.dtype)
    if c["kind"] == "project":
        w = RomQ4Weight(s.w, E, d_out, d_in, c["group"])
        out = torch.empty((N, d_out), dtype=s.x.dtype, device=s.x.device)
        return lambda: w.project(s.x, s.expert_idx, gate=s.gate if c["gated"] else None, residual=s.residual, out=out)
    dims = RomDims(d_in, 16, 16, 4, 1, E, K, E, 1 if c["dtype"] == "bf16" else 0, 1 if K > 1 else 0)
    group = c["group"] if c["kind"] == "ffn_q4" else 0
    ws = torch.empty(rom_ffn_step_workspace_bytes(dims, d_out, N), dtype=torch.uint8, device=s.x.device)
    out = torch.empty_like(s.x)

    def step():
        rom_ffn_moe_step(dims, d_out, s.w_gate_up, s.w_down, group, c["norm"], EPS, True, s.x, N, s.expert_idx, s.gate, out, ws)
        return out

    return step


def run(s):
    if not own:
        return _plain(s)
    if s.call is None:
        s.call = _call(s)
    return s.call()


# ---------------------------------------------------------------- work


def work(case):
    """Operations of the picked experts only; weights of an expert that some slot picks, and every other input and output, once."""
    c = case
    E, N, K, d_in, d_out = c["E"], c["N"], c["K"], c["d_in"], c["d_out"]
    es = 2 if c["dtype"] == "bf16" else 4
    q4 = 0.5 + 2.0 / c["group"]
    if c["kind"] == "pack":
        n = E * d_in * d_out
        return {"bytes": n * (2 * es + 2 * q4), "flops": 2 * n}
    reached = E * (1.0 - (1.0 - 1.0 / E) ** (N * K)) if not c["skew"] else 1 + (E - 1) * (1.0 - (1.0 - 1.0 / E) ** (N * (K - 1)))
    reached = min(max(reached, K), E)
    if c["kind"] == "project":
        return {"bytes": reached * d_in * d_out * q4 + N * (d_in + (2 if c["gated"] else 1) * d_out) * es, "flops": 2 * N * K * d_in * d_out}
    per = q4 if c["kind"] == "ffn_q4" else es
    return {"bytes": reached * 3 * d_in * d_out * per + 2 * N * d_in * es, "flops": 6 * N * K * d_in * d_out}


# ---------------------------------------------------------------- the definitions, in 64 bits


def _decode(packed, E, rows, cols, group):
    """float64 [E, rows, cols], each weight looked up at its place in the format."""
    rp, cp = (rows + 15) // 16 * 16, (cols + 127) // 128 * 128
    r = torch.arange(rows, device=packed.device).view(-1, 1)
    k = torch.arange(cols, device=packed.device).view(1, -1)
    lane = (k % 32) // 8 * 16 + r % 16
    at = ((r // 16) * (cp // 128) + k // 128) * 1024 + lane * 16 + (k % 128) // 32 * 4 + (k % 8) // 2
    at_s = ((r // 16) * (cp // group) + k // group) * 16 + r % 16
    scales = packed[E * rp * cp // 2:].view(torch.bfloat16)
    out = torch.empty((E, rows, cols), dtype=torch.float64, device=packed.device)
    for e in range(E):
        byte = packed[e * rp * cp // 2:][at].int()
        code = torch.where(k % 2 == 0, byte & 15, byte >> 4)
        exponent, mantissa = (code >> 1) & 3, (code & 1).double()
        v = torch.where(exponent == 0, mantissa * 0.5, (1 + mantissa * 0.5) * torch.pow(2.0, (exponent - 1).double()))
        out[e] = torch.where(code >= 8, -v, v) * scales[e * rp * (cp // group):][at_s].double()
    return out


def exact(case, seed):
    s, c = prepare(case, seed), case
    E, N, K, d_in, d_out = c["E"], c["N"], c["K"], c["d_in"], c["d_out"]
    if c["kind"] == "pack":
        out = torch.empty((E, d_out, d_in), dtype=torch.float64, device=DEV)
        table = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
        mids = (table[1:] + table[:-1]) / 2
        for e in range(E):
            for k0 in range(0, d_in, c["group"]):
                v = s.w[e, :, k0:k0 + c["group"]].double()
                scale = (v.abs().amax(-1, keepdim=True) / 6).to(torch.bfloat16).double()
                ratio = v.abs() / scale
                low, high = torch.bucketize(ratio, mids), torch.bucketize(ratio, mids, right=True)     # they differ on a tie
                code = torch.where(low % 2 == 0, low, high)
                out[e, :, k0:k0 + c["group"]] = torch.sign(v) * table[code] * scale
        return out
    x, gate, idx = s.x.double(), s.gate.double(), s.expert_idx.long()
    if c["kind"] == "project":
        w = _decode(s.w, E, d_out, d_in, c["group"])
        out = s.residual.double() if c["gated"] else torch.zeros((N, d_out), dtype=torch.float64, device=DEV)
        for e in range(E):
            n, k = (idx == e).nonzero(as_tuple=True)
            y = x[n] @ w[e].t()
            out.index_add_(0, n, y * gate[n, k].unsqueeze(1) if c["gated"] else y)
        return out
    q4 = c["kind"] == "ffn_q4"
    gu = _decode(s.w_gate_up, E, 2 * d_out, d_in, c["group"]) if q4 else s.w_gate_up
    down = _decode(s.w_down, E, d_in, d_out, c["group"]) if q4 else s.w_down
    xn = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() if c["norm"] else x
    out = x.clone()
    f = torch.arange(d_out, device=DEV)
    row = f // 8 * 16 + f % 8
    for e in range(E):
        n, k = (idx == e).nonzero(as_tuple=True)
        y = xn[n] @ gu[e].double().t()
        a = y[:, row] / (1 + torch.exp(-y[:, row])) * y[:, row + 8]
        out.index_add_(0, n, (a @ down[e].double().t()) * gate[n, k].unsqueeze(1))
    return out
