"""The operators around a linear in 8-bit floating point, measured: the residual's addition with the root-mean-square norm
and codes as output, the quantisers of activations (a scale for 128 channels of a token) and of weights (a scale for
128 x 128), and the linear on them.

A case names an operator ("kind"), its sizes and its options.  `prepare` makes what a program that serves a model holds
before the call, `run` makes the call (`own`) or computes the same in elementary torch operations, `exact` states it in 64
bits.  The 16-bit types are those of hidden states; weights are drawn like those of the library's other workloads.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BLOCK = 128          # channels that share a scale
E4M3_MAX = 448.0     # largest finite magnitude of the 8-bit type
TINY = 2.0 ** -100   # a block or row whose largest magnitude is below counts as zero
EPS = 1e-5
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one token between two layers: the latency of a short launch
        {"name": "norm_token", "kind": "norm", "T": 1, "K": 4096, "dtype": "f16", "residual": True, "codes": "e4m3", "y": False},
        # a prompt of odd length, rows that no power of two divides, norm for a router and experts that take 16-bit rows
        {"name": "norm_prompt_777", "kind": "norm", "T": 777, "K": 2064, "dtype": "bf16", "residual": True, "codes": "none", "y": True},
        # a prefill batch in front of an int8 linear
        {"name": "norm_i8_4096", "kind": "norm", "T": 4096, "K": 4096, "dtype": "f16", "residual": True, "codes": "i8", "y": False},
        # the widest hidden states, codes for one linear and rows for another
        {"name": "norm_e4m3_8192", "kind": "norm", "T": 8192, "K": 8192, "dtype": "bf16", "residual": True, "codes": "e4m3", "y": True},
        # the intermediate of a decode batch in front of a down projection
        {"name": "act_decode_33", "kind": "act", "T": 33, "K": 14336, "dtype": "f16"},
        # the intermediate of a prefill batch
        {"name": "act_prefill_4096", "kind": "act", "T": 4096, "K": 14336, "dtype": "bf16"},
        # offline: a small projection with a partial block on both sides
        {"name": "weight_small", "kind": "weight", "K": 2064, "N": 1040},
        # offline: one projection of an expert
        {"name": "weight_expert", "kind": "weight", "K": 4096, "N": 14336},
        # decoding for one user: the weight stream of an attention projection
        {"name": "linear_token", "kind": "linear", "T": 1, "K": 4096, "N": 6144, "dtype": "f16", "act": "none"},
        # decoding for 48 users: the weight stream of an up projection
        {"name": "linear_decode_48", "kind": "linear", "T": 48, "K": 4096, "N": 14336, "dtype": "bf16", "act": "none"},
        # one prompt of odd length, partial blocks, ReLU
        {"name": "linear_prompt_333", "kind": "linear", "T": 333, "K": 2064, "N": 8208, "dtype": "f16", "act": "relu"},
        # a prefill batch
        {"name": "linear_prefill_4096", "kind": "linear", "T": 4096, "K": 4096, "N": 14336, "dtype": "bf16", "act": "none"},
    ]


def _log_int(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return max(lo, min(hi, int(v) // step * step))


def draw(rng):
    kind = rng.choice(("norm", "norm", "norm", "act", "weight", "linear", "linear", "linear"))
    dtype = rng.choice(("f16", "bf16"))
    if kind == "norm":
        codes = rng.choice(("none", "i8", "e4m3"))
        return {"kind": kind, "T": _log_int(rng, 1, 8192), "K": _log_int(rng, 256, 8192, 16), "dtype": dtype,
                "residual": rng.random() < 0.75, "codes": codes, "y": codes == "none" or rng.random() < 0.5}
    if kind == "act":
        return {"kind": kind, "T": _log_int(rng, 1, 4096), "K": _log_int(rng, 256, 14336, 16), "dtype": dtype}
    if kind == "weight":
        return {"kind": kind, "K": _log_int(rng, 256, 8192, 16), "N": _log_int(rng, 256, 7168, 16)}
    return {"kind": kind, "T": _log_int(rng, 1, 4096), "K": _log_int(rng, 256, 8192, 16), "N": _log_int(rng, 256, 7168, 16),
            "dtype": dtype, "act": rng.choice(("none", "relu"))}


# ---- what a program holds before the call --------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _hidden(g, T, K, dtype):
    """Hidden states: normal, with 0.5 % of the channels 20 to 80 times the others."""
    n = max(1, math.ceil(0.005 * K))
    m = torch.ones(K, device=DEV)
    m[torch.randperm(K, generator=g, device=DEV)[:n]] = 20.0 + 60.0 * torch.rand(n, generator=g, device=DEV)
    return (torch.randn(T, K, generator=g, device=DEV) * m).to(dtype)


def _tiled(w):
    """[K, N] as [K blocks, 128, N blocks, 128], zeros past the ends."""
    K, N = w.shape
    kb, nb = -(-K // BLOCK), -(-N // BLOCK)
    return torch.nn.functional.pad(w, (0, nb * BLOCK - N, 0, kb * BLOCK - K)).view(kb, BLOCK, nb, BLOCK)


def _packed_rows(T):
    return -(-T // 16) * 16 + 256


def _packed_weight(wq):
    """[K, N] codes as the matrix kernels take them: [K/16][N, up to 256s][16], K in whole 64s."""
    K, N = wq.shape
    kp, npad = -(-K // 64) * 64, -(-N // 256) * 256
    b = torch.nn.functional.pad(wq.view(torch.int8), (0, npad - N, 0, kp - K))
    return b.view(kp // 16, 16, npad).transpose(1, 2).contiguous().view(-1)


def prepare(case, seed):
    g = _gen(seed, 1)
    kind, K = case["kind"], case["K"]
    st = {"case": case}
    if kind == "weight":
        st["w"] = torch.randn(K, case["N"], generator=g, device=DEV) * 0.02
        st["wq"] = torch.empty(K, case["N"], dtype=torch.float8_e4m3fn, device=DEV)
        st["ws"] = torch.empty(-(-K // BLOCK), -(-case["N"] // BLOCK), device=DEV)
        return st
    T, dtype = case["T"], DTYPES[case["dtype"]]
    st["x"] = _hidden(g, T, K, dtype)
    R, kb = _packed_rows(T), -(-K // BLOCK)
    codes = case.get("codes", "e4m3")
    if codes != "none":
        st["q"] = torch.empty(-(-K // 64) * 64 * R, dtype=torch.int8 if codes == "i8" else torch.float8_e4m3fn, device=DEV)
        st["scale"] = torch.empty(T if codes == "i8" else kb * R, device=DEV)
    if kind == "norm":
        st["g"] = 1.0 + 0.2 * torch.randn(K, generator=g, device=DEV)
        st["r"] = _hidden(g, T, K, dtype) if case["residual"] else None
        st["sum"] = torch.empty_like(st["x"]) if case["residual"] else None
        st["y"] = torch.empty_like(st["x"]) if case["y"] else None
        st["values"] = torch.empty(K // 16, T, 16, dtype=dtype, device=DEV) if codes == "i8" else None
    if kind == "linear":
        N = case["N"]
        w = _tiled(torch.randn(K, N, generator=g, device=DEV) * 0.02)
        st["ws"] = w.abs().amax(dim=(1, 3)) / torch.tensor(E4M3_MAX, device=DEV)
        wq = (w / st["ws"][:, None, :, None]).to(torch.float8_e4m3fn).view(kb * BLOCK, -1)
        st["wq"] = wq.view(torch.uint8)[:K, :N].contiguous().view(torch.float8_e4m3fn)
        st["wp"] = _packed_weight(st["wq"])
        st["out"] = torch.empty(T, N, dtype=dtype, device=DEV)
        st["workspace"] = torch.empty(kb * BLOCK * R + 4 * kb * R + 1024, dtype=torch.uint8, device=DEV)
    return st


# ---- the plain form ------------------------------------------------------------------------------------------------
def _row_blocks(v):
    """[T, K] as [T, K blocks, 128], zeros past the end."""
    T, K = v.shape
    kb = -(-K // BLOCK)
    return torch.nn.functional.pad(v, (0, kb * BLOCK - K)).view(T, kb, BLOCK)


def _e4m3(v, dims):
    """(codes, scales) of blocks over `dims`, in 32 bits."""
    top = torch.tensor(E4M3_MAX, device=DEV)
    a = v.abs().amax(dim=dims, keepdim=True)
    zero = a < TINY
    codes = (v * torch.where(zero, 0.0, top / a)).to(torch.float8_e4m3fn)
    return codes, torch.where(zero, 0.0, a / top)


def _chunks(rows, K):
    """[T, >= K] as the packed operand holds it: [K/16, T, 16]."""
    return rows[:, :K].reshape(rows.shape[0], K // 16, 16).transpose(0, 1)


def _act_codes(v):
    T, K = v.shape
    codes, scale = _e4m3(_row_blocks(v), 2)
    return _chunks(codes.view(torch.uint8).view(T, -1), K).contiguous().view(torch.float8_e4m3fn), scale[:, :, 0].t()


def _plain_norm(st):
    c, x, dtype = st["case"], st["x"], st["x"].dtype
    h = x if st["r"] is None else (x.float() + st["r"].float()).to(dtype)
    m = h.double().square().mean(dim=1, keepdim=True)
    v = h.float() * (1.0 / (m + EPS).sqrt()).float() * st["g"]
    out = []
    if st["r"] is not None:
        out.append(h)
    if c["y"]:
        out.append(v.to(dtype))
    if c["codes"] == "e4m3":
        out += _act_codes(v)
    if c["codes"] == "i8":
        a = v.abs().amax(dim=1, keepdim=True)
        scale = torch.where(a < TINY, 0.0, a / torch.tensor(127.0, device=DEV))
        q = torch.where(a < TINY, 0.0, (v / scale).round())
        out += [_chunks((q * scale).to(dtype), c["K"]), scale[:, 0]]
    return out


def _plain_linear(st):
    c, x = st["case"], st["x"]
    T, K, N = c["T"], c["K"], c["N"]
    codes, scale = _e4m3(_row_blocks(x.float()), 2)
    a = (codes.float() * scale).view(T, -1)[:, :K]
    w = (_tiled(st["wq"].float()) * st["ws"][:, None, :, None]).view(-1, st["ws"].shape[1] * BLOCK)[:K, :N]
    y = a @ w
    return (y.relu() if c["act"] == "relu" else y).to(x.dtype)


def _plain_weight(st):
    K, N = st["w"].shape
    codes, scale = _e4m3(_tiled(st["w"]), (1, 3))
    flat = codes.view(torch.uint8).view(scale.shape[0] * BLOCK, -1)
    return [flat[:K, :N].contiguous().view(torch.float8_e4m3fn), scale[:, 0, :, 0]]


# ---- the calls -----------------------------------------------------------------------------------------------------
def _packed_views(st):
    """Codes and scales of the packed operand, without the rows behind the last token."""
    T, K = st["x"].shape
    R = _packed_rows(T)
    return [st["q"].view(-1, R, 16)[: K // 16, :T], st["scale"].view(-1, R)[:, :T]]


def _own(st):
    import paper_2508_07329_amd as haq

    c = st["case"]
    kind = c["kind"]
    if kind == "weight":
        haq.haq_quant_weight_fp8(st["w"], wq=st["wq"], w_scale=st["ws"])
        return [st["wq"], st["ws"]]
    if kind == "act":
        haq.haq_quant_act_fp8_packed(st["x"], q_packed=st["q"], block_scale=st["scale"])
        return _packed_views(st)
    if kind == "linear":
        act = haq.HAQ_ACT_RELU if c["act"] == "relu" else haq.HAQ_ACT_NONE
        return haq.haq_fp8_linear(st["x"], st["wp"], st["ws"], c["N"], act, out=st["out"], workspace=st["workspace"])
    codes = {"none": haq.HAQ_CODES_NONE, "i8": haq.HAQ_CODES_I8, "e4m3": haq.HAQ_CODES_E4M3}[c["codes"]]
    haq.haq_rmsnorm_quant(st["x"], st["g"], EPS, codes, residual=st["r"], sum_out=st["sum"], y=st["y"], q_packed=st.get("q"),
                          scale=st.get("scale"))
    out = [t for t in (st["sum"], st["y"]) if t is not None]
    if c["codes"] == "e4m3":
        out += _packed_views(st)
    if c["codes"] == "i8":  # the values that the codes stand for
        q = st["q"].view(-1, _packed_rows(c["T"]), 16)[: c["K"] // 16, : c["T"]]
        out += [torch.mul(q, st["scale"][None, :, None], out=st["values"]), st["scale"]]
    return out


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "weight":
        return _plain_weight(state)
    if kind == "act":
        return list(_act_codes(state["x"].float()))
    return _plain_linear(state) if kind == "linear" else _plain_norm(state)


# ---- what one pass cannot do without -------------------------------------------------------------------------------
def work(case):
    K, kb = case["K"], -(-case["K"] // BLOCK)
    if case["kind"] == "weight":
        N = case["N"]
        return {"bytes": 5 * K * N + 4 * kb * -(-N // BLOCK), "flops": 3 * K * N}
    T = case["T"]
    if case["kind"] == "act":
        return {"bytes": 3 * T * K + 4 * T * kb, "flops": 3 * T * K}
    if case["kind"] == "linear":
        N = case["N"]
        return {"bytes": 2 * T * K + K * N + 4 * kb * -(-N // BLOCK) + 2 * T * N, "flops": 2 * T * K * N}
    n = 2 + 4 * case["residual"] + 2 * case["y"] + (case["codes"] != "none")
    scales = {"none": 0, "i8": 4 * T, "e4m3": 4 * T * kb}[case["codes"]]
    return {"bytes": n * T * K + 4 * K + scales, "flops": 8 * T * K}


# ---- in 64 bits ----------------------------------------------------------------------------------------------------
def _nearest_e4m3(v):
    """Values of the 8-bit type nearest to v, ties to the even one: three bits behind the leading one, steps of 2^-9 below 2^-6."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 3)
    return (v / step).round() * step


def _exact_blocks(v, K):
    """Code values and scales of 128 channels each, v [T, K] in 64 bits."""
    kb = -(-K // BLOCK)
    q, s = torch.zeros_like(v), torch.zeros(v.shape[0], kb, dtype=torch.float64, device=DEV)
    for b in range(kb):
        part = v[:, b * BLOCK:(b + 1) * BLOCK]
        s[:, b] = part.abs().amax(dim=1) / E4M3_MAX
        q[:, b * BLOCK:(b + 1) * BLOCK] = _nearest_e4m3(part / s[:, b:b + 1].clamp(min=1e-300))
    return q, s


def exact(case, seed):
    st = prepare(case, seed)
    kind, K = case["kind"], case["K"]
    if kind == "weight":
        w, N = st["w"].double(), case["N"]
        kb, nb = -(-K // BLOCK), -(-N // BLOCK)
        a = torch.zeros(kb, N, dtype=torch.float64, device=DEV)
        for b in range(kb):
            a[b] = w[b * BLOCK:(b + 1) * BLOCK].abs().amax(dim=0)
        s = torch.stack([a[:, b * BLOCK:(b + 1) * BLOCK].amax(dim=1) for b in range(nb)], dim=1) / E4M3_MAX
        full = s.repeat_interleave(BLOCK, 0)[:K].repeat_interleave(BLOCK, 1)[:, :N]
        return [_nearest_e4m3(w / full), s]
    T = case["T"]
    by_chunk = lambda v: v.view(T, K // 16, 16).permute(1, 0, 2)
    if kind == "act":
        q, s = _exact_blocks(st["x"].double(), K)
        return [by_chunk(q), s.t()]
    if kind == "linear":
        q, s = _exact_blocks(st["x"].double(), K)
        a = q * s.repeat_interleave(BLOCK, 1)[:, :K]
        w = st["wq"].double() * st["ws"].double().repeat_interleave(BLOCK, 0)[:K].repeat_interleave(BLOCK, 1)[:, : case["N"]]
        y = a @ w
        return y.clamp(min=0) if case["act"] == "relu" else y
    h = st["x"].double()
    out = []
    if case["residual"]:
        h = (h + st["r"].double()).to(st["x"].dtype).double()  # the residual stream is held in 16 bits
        out.append(h)
    v = h / (h.square().mean(dim=1, keepdim=True) + EPS).sqrt() * st["g"].double()
    if case["y"]:
        out.append(v)
    if case["codes"] == "e4m3":
        q, s = _exact_blocks(v, K)
        out += [by_chunk(q), s.t()]
    if case["codes"] == "i8":
        s = v.abs().amax(dim=1, keepdim=True) / 127
        out += [by_chunk((v / s).round() * s), s[:, 0]]
    return out
