"""Timed cases of the 8-bit integer operators: the norm that leaves codes, the row quantiser, and the product of codes.

A code c of row r stands for c * scale[r].  Rows are tokens (activations) or output channels (weights, stored [out][in]).
  norm        x' = x + delta (float32); y = x' / sqrt(mean(x'^2) + eps) * gain; per row scale = max|y| / 127 as float32,
              code = y / scale rounded to nearest, ties to even.                         -> x', the codes' values, scales
  quantize    the same scale and codes of the rows of x, bf16 or float32.                -> the codes' values, scales
  gemm        a_scale[m] * w_scale[n] * sum_k A[m][k] W[n][k] + bias[n]; kind 0 bf16, 1 float32, 2 bf16 of tanh-GELU,
              3 float32 added, times the row's gate, to what is there.                   -> the result
  geglu       bf16 of tanh-GELU(product with W_gate) * (product with W_up).              -> the result
  transposed  bf16, row m of the product as column col[m] of the output, whose other columns keep their values.  -> the output

The plain forms compute in 32 bits; codes in 64, because a value next to the border of two codes has to fall on its own side.
Codes are returned as the values they stand for, in float32.
"""
import math

import torch

own = False
EPS = 1e-6
SMALLEST = 2.0 ** -126                      # smallest scale
DEV = "cuda"


def listed():
    return [
        # One short prompt (32 tokens) at the text encoder's width: the norm between two products, where latency counts.
        dict(name="norm_prompt", op="norm", M=32, d=4096, delta="bf16"),
        # A batch of 64 prompts of 500 tokens at the encoder's width: bound by memory.
        dict(name="norm_batch", op="norm", M=32000, d=4096, delta="bf16"),
        # An image's tokens at the denoiser's width, no residual pending.
        dict(name="norm_image", op="norm", M=4250, d=1536, delta="none"),
        # The gated activations of a prompt of 77 tokens, on their way into the MLP's output product.
        dict(name="quantize_prompt", op="quantize", M=77, d=10240, x="bf16"),
        # A weight matrix of the encoder, which gets its codes once: float32 rows of odd width.
        dict(name="quantize_weight", op="quantize", M=10240, d=4091, x="f32"),
        # One token through an output product: nothing but the weights' bytes.
        dict(name="gemm_token", op="gemm", M=1, N=4096, K=4096, kind=0, bias=False),
        # A prompt of 32 tokens through the query, key and value products.
        dict(name="gemm_prompt", op="gemm", M=32, N=12288, K=4096, kind=0, bias=False),
        # A prompt of 500 tokens through the MLP's output product into the residual stream.
        dict(name="gemm_long_prompt", op="gemm", M=500, N=4096, K=10240, kind=3, bias=False),
        # Sixteen prompts of 500 tokens through the query, key and value products, the largest case; with a bias and float32 results.
        dict(name="gemm_batch", op="gemm", M=8000, N=12288, K=4096, kind=1, bias=True),
        # A prompt of 77 tokens through the MLP's input products.
        dict(name="geglu_prompt", op="geglu", M=77, N=10240, K=4096),
        # Sixteen prompts of mixed lengths, 2744 tokens in all, through the MLP's input products.
        dict(name="geglu_batch", op="geglu", M=2744, N=10240, K=4096),
        # Ragged prompts' values, written as the attention reads them.
        dict(name="values_ragged", op="transposed", M=1137, N=4096, K=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "quantize", "gemm", "gemm", "geglu", "transposed"])
    if op == "norm":
        return dict(op=op, M=_log(rng, 1, 16384), d=rng.choice([256, 1000, 1536, 2050, 4096, 4097, 5120, 8192]), delta=rng.choice(["none", "bf16", "f32"]))
    if op == "quantize":
        return dict(op=op, M=_log(rng, 1, 16384), d=_log(rng, 64, 14336), x=rng.choice(["bf16", "f32"]))
    K = 128 * _log(rng, 2, 80)
    if op == "gemm":
        M, N = _log(rng, 1, 8000), _log(rng, 64, 12288)
        while M * N * K > 8000 * 12288 * 4096:
            M //= 2
        return dict(op=op, M=M, N=N, K=K, kind=rng.randrange(4), bias=rng.random() < 0.5)
    return dict(op=op, M=_log(rng, 1, 4096), N=_log(rng, 64, 4096 if op == "transposed" else 10240), K=K)


def _codes(g, rows, K):
    """Codes of gaussian rows: four standard deviations are 127."""
    c = torch.randn(rows, K, generator=g, device=DEV, dtype=torch.float32).mul_(32.0).round_().clamp_(-127, 127)
    return c.to(torch.int8)


def _columns(M):
    """Columns of the tokens of ragged prompts packed with every prompt at a multiple of 64: (col [M], columns in all)."""
    lens, left, k = [], M, 0
    while left:
        n = min(left, (77, 200, 33, 131, 500)[k % 5])
        lens.append(n)
        left -= n
        k += 1
    col, at = [], 0
    for n in lens:
        col += range(at, at + n)
        at += -(-n // 64) * 64
    return torch.tensor(col, dtype=torch.int32, device=DEV), at


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=torch.float32)  # noqa: E731
    up8, up128 = lambda n: -(-n // 8) * 8, lambda n: -(-n // 128) * 128  # noqa: E731
    s = dict(case)
    if case["op"] in ("norm", "quantize"):
        M, d = case["M"], case["d"]
        x = torch.zeros(M, up8(d), device=DEV)          # rows start at 16 bytes; gaussian with a few large channels, as a residual stream has them
        x[:, :d] = rand(M, d)
        x[:, torch.randint(0, d, (max(1, d // 512),), generator=g, device=DEV)] *= 12.0
        s["codes"] = torch.zeros(M, up128(d), dtype=torch.int8, device=DEV)
        s["scale"] = torch.zeros(M, device=DEV)
        s["values"] = torch.zeros(M, d, device=DEV)
        if case["op"] == "quantize":
            s["x"] = x.to(torch.bfloat16) if case["x"] == "bf16" else x
            return s
        s["x"], s["gain"], s["x_out"], s["delta"] = x, 1.0 + 0.1 * rand(d), torch.zeros_like(x), None
        if case["delta"] != "none":
            delta = torch.zeros(M, up8(d), device=DEV)
            delta[:, :d] = 0.3 * rand(M, d)
            s["delta"] = delta.to(torch.bfloat16) if case["delta"] == "bf16" else delta
        return s
    M, N, K = case["M"], case["N"], case["K"]
    s["A"], s["a_scale"] = _codes(g, M, K), 0.03 * (1.0 + torch.rand(M, generator=g, device=DEV))
    s["W"], s["w_scale"] = _codes(g, N, K), 0.02 / math.sqrt(K) * (1.0 + torch.rand(N, generator=g, device=DEV))
    if case["op"] == "geglu":
        s["W_up"], s["up_scale"] = _codes(g, N, K), 0.02 / math.sqrt(K) * (1.0 + torch.rand(N, generator=g, device=DEV))
        s["out"] = torch.zeros(M, up8(N), dtype=torch.bfloat16, device=DEV)
    elif case["op"] == "transposed":
        s["col"], width = _columns(M)
        s["out"] = torch.zeros(N, width, dtype=torch.bfloat16, device=DEV)
    else:
        s["bias"] = rand(N) if case["bias"] else None
        s["out"] = torch.zeros(M, up8(N), dtype=torch.float32 if case["kind"] in (1, 3) else torch.bfloat16, device=DEV)
        if case["kind"] == 3:                            # two requests with a gate each
            s["out"][:, :N] = rand(M, N)
            s["gate"], s["row_req"] = rand(2, N), (torch.arange(M, device=DEV) * 3 > M).to(torch.int32)
    # scratch for the shares of a split product; a program keeps one for all its calls
    s["work"] = torch.zeros(32 << 20, dtype=torch.uint8, device=DEV)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _plain_codes(y):
    """Values of the codes of the rows y (float64), and their scales."""
    scale = (y.abs().amax(dim=1) / 127.0).float().clamp_min(SMALLEST)
    code = torch.round(y / scale.double()[:, None]).float()
    return code * scale[:, None], scale


def _plain_product(s, W, w_scale):
    return (s["A"].float() @ W.float().t()) * s["a_scale"][:, None] * w_scale


def _gelu(v):
    return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))


def _plain(s):
    op = s["op"]
    if op == "quantize":
        values, scale = _plain_codes(s["x"][:, :s["d"]].double())
        return {"values": values, "scale": scale}
    if op == "norm":
        x = s["x"][:, :s["d"]]
        if s["delta"] is not None:
            x = x + s["delta"][:, :s["d"]].float()
        y = x.double()
        values, scale = _plain_codes(y * torch.rsqrt(y.square().mean(dim=1, keepdim=True) + EPS) * s["gain"].double())
        return {"x_out": x, "values": values, "scale": scale}
    p = _plain_product(s, s["W"], s["w_scale"])
    if op == "geglu":
        return {"out": (_gelu(p) * _plain_product(s, s["W_up"], s["up_scale"])).to(torch.bfloat16)}
    if op == "transposed":
        s["out"][:, s["col"].long()] = p.t().to(torch.bfloat16)
        return {"out": s["out"]}
    if s["bias"] is not None:
        p = p + s["bias"]
    if s["kind"] == 3:
        s["out"][:, :s["N"]] += s["gate"][s["row_req"].long()] * p
        return {"out": s["out"][:, :s["N"]]}
    return {"out": p if s["kind"] == 1 else (_gelu(p) if s["kind"] == 2 else p).to(torch.bfloat16)}


# ---- the framework's calls ------------------------------------------------------------------------------------------
def _own(s):
    from paper_2510_02838_amd import int8
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    op = s["op"]
    if op in ("norm", "quantize"):
        x, codes, scale = s["x"], s["codes"], s["scale"]
        M, d = s["M"], s["d"]
        if op == "quantize":
            int8.check(int8.dit_op_quantize_i8(None, x.data_ptr(), 0 if s["x"].dtype == torch.bfloat16 else 1, x.shape[1], M, d,
                                               codes.data_ptr(), codes.shape[1], scale.data_ptr()))
            out = {}
        else:
            delta = s["delta"]
            int8.check(int8.dit_op_rmsnorm_i8(None, x.data_ptr(), x.shape[1], ptr(delta), int(delta is not None and delta.dtype == torch.float32),
                                              x.shape[1], s["gain"].data_ptr(), EPS, M, d, s["x_out"].data_ptr(), x.shape[1],
                                              codes.data_ptr(), codes.shape[1], scale.data_ptr()))
            out = {"x_out": s["x_out"][:, :d]}
        torch.mul(codes[:, :d], scale[:, None], out=s["values"])
        return dict(out, values=s["values"], scale=scale)
    A, W, out, work = s["A"], s["W"], s["out"], s["work"]
    M, N, K = s["M"], s["N"], s["K"]
    if op == "geglu":
        int8.check(int8.dit_op_gemm_i8_geglu(None, A.data_ptr(), K, s["a_scale"].data_ptr(), W.data_ptr(), s["w_scale"].data_ptr(),
                                             s["W_up"].data_ptr(), s["up_scale"].data_ptr(), K, M, N, K, out.data_ptr(), out.shape[1],
                                             work.data_ptr(), work.numel()))
        return {"out": out[:, :N]}
    if op == "transposed":
        int8.check(int8.dit_op_gemm_i8_transposed(None, A.data_ptr(), K, s["a_scale"].data_ptr(), W.data_ptr(), K, s["w_scale"].data_ptr(), None,
                                                  M, N, K, out.data_ptr(), out.shape[1], s["col"].data_ptr(), work.data_ptr(), work.numel()))
        return {"out": out}
    resid = s["kind"] == 3
    int8.check(int8.dit_op_gemm_i8(None, A.data_ptr(), K, s["a_scale"].data_ptr(), W.data_ptr(), K, s["w_scale"].data_ptr(), ptr(s["bias"]), M, N, K,
                                   s["kind"], out.data_ptr(), out.shape[1], s["gate"].data_ptr() if resid else None, N if resid else 0,
                                   s["row_req"].data_ptr() if resid else None, work.data_ptr(), work.numel()))
    return {"out": out[:, :N]}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    if case["op"] in ("norm", "quantize"):
        M, d = case["M"], case["d"]
        if case["op"] == "quantize":
            return {"bytes": M * d * ((2 if case["x"] == "bf16" else 4) + 1) + 4 * M, "flops": 3 * M * d}
        return {"bytes": M * d * (4 + {"none": 0, "bf16": 2, "f32": 4}[case["delta"]] + 4 + 1) + 4 * (M + d), "flops": 8 * M * d}
    M, N, K = case["M"], case["N"], case["K"]
    pair = 2 if case["op"] == "geglu" else 1
    out = {0: 2, 1: 4, 2: 2, 3: 8}[case.get("kind", 0)]
    return {"bytes": M * K + pair * N * K + M * N * out + 4 * (M + pair * N), "flops": 2 * pair * M * N * K}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------
def _exact_codes(rows):
    """Row by row in blocks: (values, scales); the scale is the nearest float32, as the definition says."""
    values, scales = torch.empty_like(rows), torch.empty(rows.shape[0], dtype=torch.float64, device=rows.device)
    for a in range(0, rows.shape[0], 2048):
        r = rows[a:a + 2048]
        sc = torch.maximum(r.max(dim=1).values, -r.min(dim=1).values).div(127.0).to(torch.float32).clamp_min(SMALLEST).to(torch.float64)
        scales[a:a + 2048] = sc
        q = r / sc.unsqueeze(1)
        whole = torch.floor(q)
        part = q - whole                                # nearest, ties to the even one
        up = (part > 0.5) | ((part == 0.5) & (torch.remainder(whole, 2.0) == 1.0))
        values[a:a + 2048] = (whole + up.to(torch.float64)) * sc.unsqueeze(1)
    return values, scales


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "quantize"):
        x = s["x"][:, :case["d"]].to(torch.float64)
        if case["op"] == "quantize":
            values, scale = _exact_codes(x)
            return {"values": values, "scale": scale}
        if s["delta"] is not None:
            x = (x + s["delta"][:, :case["d"]].to(torch.float64)).to(torch.float32).to(torch.float64)   # the stream is held in 32 bits
        rms = (torch.einsum("md,md->m", x, x) / case["d"] + EPS).sqrt()
        values, scale = _exact_codes(x / rms.unsqueeze(1) * s["gain"].to(torch.float64))
        return {"x_out": x, "values": values, "scale": scale}

    def product(W, w_scale, a, b):
        return torch.mm(s["A"][a:b].to(torch.float64) * s["a_scale"][a:b, None].to(torch.float64), (W.to(torch.float64) * w_scale[:, None].to(torch.float64)).t().contiguous())

    def gelu(v):
        return v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))

    M, N = case["M"], case["N"]
    out = torch.empty(M, N, dtype=torch.float64, device=DEV)
    for a in range(0, M, 2048):
        b = min(M, a + 2048)
        p = product(s["W"], s["w_scale"], a, b)
        if case["op"] == "geglu":
            p = gelu(p) * product(s["W_up"], s["up_scale"], a, b)
        elif case["op"] == "gemm":
            if s["bias"] is not None:
                p = p + s["bias"].to(torch.float64)
            if case["kind"] == 2:
                p = gelu(p)
            if case["kind"] == 3:
                p = s["out"][a:b, :N].to(torch.float64) + s["gate"].to(torch.float64)[s["row_req"][a:b].long()] * p
        out[a:b] = p
    if case["op"] != "transposed":
        return {"out": out}
    full = s["out"].to(torch.float64)
    full.index_copy_(1, s["col"].long(), out.t().contiguous())
    return {"out": full}
