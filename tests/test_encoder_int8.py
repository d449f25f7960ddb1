"""The Encode stage on 8-bit codes: host logic, and GPU parity with a float64 encoder whose products take the same codes."""
import numpy as np
import pytest

import synth
from helpers import rel_l2
from oracle import encoder_oracle as E

ARCH = synth.ENCODERS["t5_tiny"]


@pytest.fixture(scope="module")
def Q():
    from paper_2510_02838_amd import int8
    return int8


@pytest.fixture(scope="module")
def torch():
    import torch
    torch.cuda.set_device(0)
    return torch


def coded(rows):
    """Values of the codes of float64 rows."""
    s = np.maximum((np.abs(rows).max(axis=1) / 127.0).astype(np.float32), np.float32(2.0 ** -126)).astype(np.float64)[:, None]
    return np.rint(rows / s) * s


class CodedOracle(E.EncoderOracle):
    """Every product of the definition takes codes: of its input's rows and of its weight's output channels.  rounded: what the
    encoder keeps as bf16 (queries, keys, values, attention, activations, branches) is rounded to bf16."""

    def __init__(self, arch, params, rounded=False):
        super().__init__(arch, params)
        self.w = {k: coded(v.T).T for k, v in self.p.items() if k.endswith(".w")}
        self.b = (lambda v: synth.round_bf16(v.astype(np.float32)).astype(np.float64)) if rounded else (lambda v: v)

    def product(self, rows, name):
        return self.b(coded(rows) @ self.w[name])

    def layer(self, x, l, bias, taps=None):
        a, p, pre = self.arch, self.p, f"l{l}"
        H, dh, n = a["n_heads"], a["head_dim"], x.shape[0]
        h = E.rms_norm(x, p[pre + ".ln1.g"])
        q, k, v = (self.product(h, f"{pre}.{m}.w").reshape(n, H, dh) for m in "qkv")
        o = np.stack([E.softmax_rows(q[:, i] @ k[:, i].T + bias[i]) @ v[:, i] for i in range(H)], axis=1).reshape(n, H * dh)
        o = self.b(o)
        x = x + self.product(o, pre + ".o.w")
        h = E.rms_norm(x, p[pre + ".ln2.g"])
        act = self.b(E.gelu_tanh(coded(h) @ self.w[pre + ".wi0.w"]) * (coded(h) @ self.w[pre + ".wi1.w"]))
        y = x + self.product(act, pre + ".wo.w")
        if taps is not None:
            taps.update({pre + ".attn": o, pre + ".x_attn": x, pre + ".act": act, pre + ".x_out": y})
        return y


def test_sizes_and_refusals_without_a_device(Q):
    m = Q.EncoderI8(ARCH, bind=False)
    d, inner, ff, n = ARCH["d_model"], ARCH["n_heads"] * ARCH["head_dim"], ARCH["d_ff"], ARCH["n_layers"]
    rows = 3 * inner + 2 * d + 2 * ff
    assert n * (4 * d * inner + 3 * d * ff + 4 * rows) <= m.code_bytes() <= n * (4 * d * inner + 3 * d * ff + 4 * rows + 10 * 256)
    assert 0 < m.workspace_bytes([30]) < m.workspace_bytes([30, 500])
    assert m.workspace_bytes([0]) == m.workspace_bytes([]) == m.workspace_bytes([1025]) == 0
    lens = (Q.C.c_int * 1)(4)
    assert Q.enc_i8_forward(None, 1, lens, 256, 256, None) == Q.enc_i8_quantize(None, 256, 1 << 30) == 1
    assert Q.enc_i8_forward(m.ctx, 1, lens, 256, 256, None) == Q.enc_i8_quantize(m.ctx, 256, 1 << 30) == 1      # nothing bound
    from paper_2510_02838_amd import encoder as X
    assert X.enc_bind(m.ctx, 1 << 20, 1 << 40, 1 << 20, 1 << 40) == 0                                          # (never dereferenced)
    assert Q.enc_i8_quantize(m.ctx, None, 1 << 30) == Q.enc_i8_quantize(m.ctx, 257, 1 << 30) == 1
    assert Q.enc_i8_quantize(m.ctx, 256, m.code_bytes() - 1) == 3
    assert Q.enc_i8_forward(m.ctx, 1, lens, 256, 256, None) == 1 and b"enc_i8_quantize" in X.enc_last_error(m.ctx)
    m.close()
    big = Q.EncoderI8(dict(ARCH, d_ff=16640), bind=False)
    assert X.enc_bind(big.ctx, 1 << 20, 1 << 40, 1 << 20, 1 << 40) == 0
    assert Q.enc_i8_quantize(big.ctx, 256, 1 << 40) == 5                                                       # rows too long for codes
    big.close()


def make(torch, Q, arch, lens, std=0.05, gain_std=0.1, bias_scale=2.0):
    params = synth.make_params(E.param_shapes(arch), 1, std, 0.0, gain_std)
    params["rel_bias"] = synth.round_bf16(params["rel_bias"] * bias_scale / std)
    params["embed"] = synth.round_bf16(params["embed"] / std)
    toks = synth.make_tokens(lens, arch["vocab"])
    m = Q.EncoderI8(arch)
    m.ensure_workspace(lens)
    m.workspace.fill_(0xFF)                                          # NaN in whatever is read without having been written
    m.init_weights(0, 0.0)
    m.set_params(params)
    m.quantize()
    return params, toks, m, torch.from_numpy(np.concatenate(toks)).cuda()


def bound(arch, params, tok):
    """(what the float64 encoder on codes gives, how far the GPU may be from it.)  Products and codes are exact on both sides; what
    differs is the bf16 roundings, and a code that such a rounding moves to its neighbour moves by a whole step: a value that is off by
    r steps gets another code with probability r, an error of sqrt(r) steps, so that 2^-9 of a value of 30 steps is sqrt(30 / 512) = a
    quarter of a step, and what one layer leaves is enlarged in the next.  How much that comes to for these weights and tokens is
    computed: the same encoder with the roundings in it is one draw of this error, the GPU, which rounds the same values but
    sums in another order, another of the same size.  The two differ from the exact one by e each, and so by at most 2 e
    between them; the probabilities' bf16, which neither oracle rounds, is the 1e-2 of the bf16 encoder's tests."""
    ref, rnd = CodedOracle(arch, params).forward(tok), CodedOracle(arch, params, True).forward(tok)
    return ref, 2.0 * rel_l2(rnd, ref) + 1e-2


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[1], [30], [64, 7, 300], [129, 500, 65]])
def test_forward_against_the_definition_on_codes(torch, Q, lens):
    params, toks, m, d_tok = make(torch, Q, ARCH, lens)
    n = sum(lens)
    out16 = torch.full((n, ARCH["d_model"]), float("nan"), dtype=torch.bfloat16, device="cuda")
    out32 = torch.full((n, ARCH["d_model"]), float("nan"), dtype=torch.float32, device="cuda")
    m.forward(lens, d_tok, out16, out32)
    torch.cuda.synchronize()
    at = 0
    for t, L in zip(toks, lens):
        (ref, most), got = bound(ARCH, params, t), out32[at:at + L].cpu().numpy()
        assert np.isfinite(got).all()
        assert rel_l2(got, ref) <= most, (rel_l2(got, ref), most)
        assert rel_l2(out16[at:at + L].float().cpu().numpy(), got) <= 2.0 ** -8
        at += L
    m.close()


@pytest.mark.gpu
def test_intermediates_neighbours_and_stale_codes(torch, Q):
    lens = [40, 200]
    params, toks, m, d_tok = make(torch, Q, ARCH, lens)
    n, d, inner, ff = sum(lens), ARCH["d_model"], ARCH["n_heads"] * ARCH["head_dim"], ARCH["d_ff"]
    shape = {"l0.attn": (inner, torch.bfloat16), "l0.x_attn": (d, torch.float32), "l0.act": (ff, torch.bfloat16), "l0.x_out": (d, torch.float32),
             "l1.x_out": (d, torch.float32)}
    bufs = {k: torch.zeros((n, w), dtype=t, device="cuda") for k, (w, t) in shape.items()}
    for k, t in bufs.items():
        m.set_tap(k, t)
    out = torch.empty((n, d), device="cuda")
    m.forward(lens, d_tok, None, out)
    torch.cuda.synchronize()
    # Every step from what the step before left: codes and products are exact, what the step keeps is rounded once (and the sums of a
    # product to float32, three roundings of 2^-24 each).
    got = {k: t.double().cpu().numpy() for k, t in bufs.items()}
    ora, x, half = CodedOracle(ARCH, params), params["embed"][np.concatenate(toks)].astype(np.float64), 2.0 ** -8
    branch = ora.product(got["l0.attn"], "l0.o.w")
    assert (np.abs(got["l0.x_attn"] - x - branch) <= 1.001 * half * np.abs(branch) + 2.0 ** -23 * np.abs(x) + 1e-12).all()
    # (a code of the norm's lies on its own side of a border by more than the 64-bit sums differ, save one in a million)
    h = E.rms_norm(got["l0.x_attn"], ora.p["l0.ln2.g"])
    gate, up = ora.product(h, "l0.wi0.w"), ora.product(h, "l0.wi1.w")
    want = E.gelu_tanh(gate) * up
    off = np.abs(got["l0.act"] - want) > 1.001 * half * np.abs(want) + 1e-5 * np.abs(up) + 1e-12
    assert off.any(axis=1).sum() <= 1, off.sum()                     # (at most one row with another code)
    branch = ora.product(got["l0.act"], "l0.wo.w")
    assert (np.abs(got["l0.x_out"] - got["l0.x_attn"] - branch) <= 1.001 * half * np.abs(branch) + 2.0 ** -23 * np.abs(got["l0.x_attn"]) + 1e-12).all()
    final = E.rms_norm(got["l1.x_out"], ora.p["final.g"])
    assert rel_l2(out.cpu().numpy(), final) <= 1e-6
    at = 0
    for t, L in zip(toks, lens):                                     # attention: bf16 inputs and probabilities, as in the bf16 encoder's tests
        tp = {}
        CodedOracle(ARCH, params, True).layer(x[at:at + L], 0, E.position_bias(L, ora.p["rel_bias"]), tp)
        assert rel_l2(got["l0.attn"][at:at + L], tp["l0.attn"]) <= 1e-2
        at += L
    m.clear_taps()
    solo = torch.empty((lens[1], d), device="cuda")
    m.forward([lens[1]], d_tok[lens[0]:], None, solo)
    torch.cuda.synchronize()
    assert torch.equal(solo, out[lens[0]:])
    # a matrix that changes needs new codes, a gain does not
    m.set_tensor("l0.ln1.g", params["l0.ln1.g"])
    m.forward(lens, d_tok, None, out)
    w = params["l1.wo.w"] * 0.5
    m.set_tensor("l1.wo.w", w)
    with pytest.raises(Exception, match="enc_i8_quantize"):
        m.forward(lens, d_tok, None, out)
    m.quantize()
    m.forward(lens, d_tok, None, out)
    torch.cuda.synchronize()
    ref, most = bound(ARCH, dict(params, **{"l1.wo.w": w}), toks[1])
    assert rel_l2(out[lens[0]:].cpu().numpy(), ref) <= most
    m.close()


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[33], [77, 130, 125], [500, 7], [77, 200, 33, 131, 97, 500, 51], [500, 431, 351, 287, 255, 201, 163, 127, 97, 77, 77, 64, 51, 43, 33, 31]])
def test_benchmark_widths(torch, Q, lens):
    """One layer of the widths that the stage tables are timed at, from 33 tokens to 2744, prompts of odd lengths, whose tiles differ from
    those of a prompt alone: one prompt against the definition, the others against themselves alone, bit for bit."""
    arch = dict(synth.ENCODERS["t5_xxl"], n_layers=1, vocab=512)
    params, toks, m, d_tok = make(torch, Q, arch, lens, std=0.0125)
    out = torch.full((sum(lens), arch["d_model"]), float("nan"), device="cuda")
    m.forward(lens, d_tok, None, out)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out).all())
    if len(lens) == 1:
        ref, most = bound(arch, params, toks[0])
        assert rel_l2(out.cpu().numpy(), ref) <= most, (rel_l2(out.cpu().numpy(), ref), most)
    at = 0
    for L in lens:
        solo = torch.full((L, arch["d_model"]), float("nan"), device="cuda")
        m.forward([L], d_tok[at:], None, solo)
        torch.cuda.synchronize()
        assert torch.equal(solo, out[at:at + L]), L
        at += L
    m.close()
