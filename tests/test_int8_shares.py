"""Products of codes in shares of K, in two launches, and transposed on every tile: the calls that the shapes of test_int8.py do not
reach.  Each list says what its shapes take, and a host test holds it to that."""
import os
import subprocess
import sys

import numpy as np
import pytest

import synth
from test_int8 import (BF16, F32, TILES, TWO, Product, columns, gelu64, gelu_bound, product_bound, up,
                       Q, torch)  # noqa: F401 (the last two are fixtures)

SCRATCH = 32 << 20                        # what Product passes

# shape: shares of K, columns of a first launch
SHARED = {(500, 4096, 10240): (2, 0), (102, 9736, 9728): (3, 0), (104, 6200, 10240): (4, 0), (85, 6203, 20480): (4, 0), (339, 3099, 20480): (3, 0),
          (700, 1537, 20480): (3, 0), (241, 3101, 10240): (4, 0)}
SHARED_PAIRS = {(104, 6200, 5120): (2, 0), (257, 1536, 20480): (3, 0), (104, 3080, 10240): (4, 0), (225, 1030, 20480): (4, 0), (397, 1023, 20480): (4, 0),
                (1473, 521, 10240): (2, 0)}
# ... of the second of two launches
SHARED_REST = {(2562, 6654, 5376): (2, 5888), (1130, 8282, 10880): (3, 7168), (1638, 5351, 11904): (4, 4864)}
SHARED_REST_PAIRS = {(3368, 2559, 4992): (2, 2304), (869, 5362, 9856): (3, 4608), (1226, 3516, 10880): (4, 3200)}
# many rows to transpose: tiles of 256 rows with ragged last ones
TALL = {(1928, 2600, 8064): 256128, (3955, 3186, 1536): 256256}


def shares(Q, M, N, K, pair, scratch=SCRATCH):
    """(shares of K of the launch that is split, columns of a first launch): the scratch says how many, 64 KB for each tile and share."""
    plan = (Q.C.c_int * 3)()
    assert Q.dit_op_gemm_i8_tile(M, N, K, pair, scratch, plan) > 0
    need = Q.dit_op_gemm_i8_work_bytes(M, N, K, pair)
    assert need <= SCRATCH
    cols = (2 if pair else 1) * (N - plan[1])
    return (need // (-(-M // 128) * -(-cols // 128) * 65536) if need else 1), plan[1]


def test_the_shapes_take_what_their_lists_say(Q):
    for pair, tables in ((0, (SHARED, SHARED_REST)), (1, (SHARED_PAIRS, SHARED_REST_PAIRS))):
        for table in tables:
            assert {s: shares(Q, *s, pair) for s in table} == table
            assert {n for n, _ in table.values()} == {2, 3, 4}
    assert {s: Q.dit_op_gemm_i8_tile(*s, 0, SCRATCH, None) for s in TALL} == TALL
    assert shares(Q, 128, 2176, Q.MAX_K, 0) == shares(Q, 128, 1088, Q.MAX_K, 1) == (4, 0)
    assert Q.dit_op_gemm_i8_tile(500, 4096, 15360, 0, 0, None) > 1000                                     # (8-wave tiles, unsplit)
    assert shares(Q, 1100, 3100, 20480, 0) == (1, 0) and {shares(Q, n, 3100, 20480, 0)[0] for _, n in PARTS} == {1, 2, 3, 4}
    assert shares(Q, 1100, 1030, 20480, 1) == (1, 0) and {shares(Q, n, 1030, 20480, 1)[0] for _, n in PARTS} == {1, 2, 3, 4}
    # the encoder's query, key and value product at T5-XXL widths: 1793 tokens, where the first launch ends with the keys
    assert shares(Q, 1793, 3 * 4096, 4096, 0) == (1, 2 * 4096)


def test_the_plan_says_the_shares_of_whichever_launch_has_them(Q):
    plan = (Q.C.c_int * 3)()
    for pair, tables in ((0, (SHARED, SHARED_REST)), (1, (SHARED_PAIRS, SHARED_REST_PAIRS))):
        for table in tables:
            for s, (n, first) in table.items():
                Q.dit_op_gemm_i8_tile(*s, pair, SCRATCH, plan)
                assert list(plan[:2]) == [n, first]
                Q.dit_op_gemm_i8_tile(*s, pair, 0, plan)             # (without scratch there are none)
                assert plan[0] == 1


def test_a_workspace_for_a_longer_call_does_for_a_shorter_one(Q):
    """(The products of 401 to 512 tokens split at these widths, those of 513 do not.)"""
    m = Q.EncoderI8(synth.ENCODERS["t5_xxl"], bind=False)
    one = [m.workspace_bytes([n]) for n in range(1, 1025)]
    many = [m.workspace_bytes([256] * k) for k in range(1, 40)]
    assert all(a <= b for w in (one, many) for a, b in zip(w, w[1:]))
    assert one[511] < one[512] and 0 < one[0]
    m.close()


def refusing(tmp_path, body, **env):
    """Runs a child process whose launcher of a tile knows none of them."""
    src, so, child = tmp_path / "refuse.cpp", tmp_path / "librefuse.so", tmp_path / "child.py"
    src.write_text("struct ihipStream_t;\nnamespace dit { struct GemmI8; bool launch_gemm_i8_variant(ihipStream_t*, GemmI8&, int) { return false; } }\n")
    subprocess.run(["g++", "-shared", "-fPIC", str(src), "-o", str(so)], check=True)
    child.write_text(f"import ctypes, torch, synth\nctypes.CDLL({str(so)!r}, mode=ctypes.RTLD_GLOBAL)\nfrom paper_2510_02838_amd import int8 as Q, binding as B\n" + body)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, str(child)], env=dict(os.environ, PYTHONPATH=root, **env), cwd=root, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr


def test_a_tile_that_is_not_built_fails_the_product(tmp_path):
    """The choice offers built tiles only; if it ever does not, a call must not return DIT_OK with nothing written.  (Nothing is launched.)"""
    refusing(tmp_path, """
for M, N, K in ((4, 64, 128), (500, 4096, 10240), (2744, 12288, 128)):       # one launch, shares, two launches
    got = [Q.dit_op_gemm_i8(None, 256, K, 256, 256, K, 256, None, M, N, K, 0, 256, N, None, 0, None, 256, 1 << 25),
           Q.dit_op_gemm_i8_geglu(None, 256, K, 256, 256, 256, 256, 256, K, M, N, K, 256, N, 256, 1 << 25),
           Q.dit_op_gemm_i8_transposed(None, 256, K, 256, 256, K, 256, None, M, N, K, 256, 4096, 256, 256, 1 << 25)]
    assert got == [2, 2, 2], got
""", HIP_VISIBLE_DEVICES="")                                          # (no device: the addresses are none)


@pytest.mark.gpu
def test_a_tile_that_is_not_built_fails_the_encoder(tmp_path):
    refusing(tmp_path, """
torch.cuda.set_device(0)
m = Q.EncoderI8(synth.ENCODERS["t5_tiny"])
m.ensure_workspace([9]); m.workspace.zero_(); m.init_weights(1, 0.05); m.quantize()
out = torch.empty((9, synth.ENCODERS["t5_tiny"]["d_model"]), device="cuda")
try:
    m.forward([9], torch.zeros(9, dtype=torch.int32, device="cuda"), None, out)
    got = 0
except B.DitError as e:
    got = e.status
torch.cuda.synchronize()
assert got == 2, got
""")


def close(got, want, tol):
    d = (got.double() - want).abs()
    assert bool((d <= tol).all()), float((d - tol).max())


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", list(SHARED) + list(SHARED_REST))
def test_products_in_shares_of_k(torch, Q, M, N, K):
    """Every kind, with and without bias and gates, against the formula; and without scratch, unsplit, not a bit differs."""
    P = Product(torch, M, N, K, seed=M + N + K, pad_a=48, pad_w=16)
    p, b = P.exact(), P.bias.double()
    for bias in (True, False):
        v = p + b if bias else p
        dv = product_bound(p, b if bias else 0.0 * b)
        for kind in (0, 1, 2):
            out = P.plain(Q, kind, bias)
            want, tol = (gelu64(v), gelu_bound(v, dv)) if kind == 2 else (v, dv)
            if kind != 1:
                tol = tol + BF16 * (want.abs() + tol)
            close(out[:, :N], want, tol)
            assert bool((out[:, N:] == 9.0).all())
            assert torch.equal(out, P.plain(Q, kind, bias, work=False))
    x = torch.randn(M, up(N, 8) + 8, generator=torch.Generator().manual_seed(2)).cuda()
    gate = torch.randn(3, N + 1, generator=torch.Generator().manual_seed(3)).cuda()
    req = (torch.arange(M) * 3 // M).to(torch.int32).cuda()
    for gt, rr in ((gate, req), (gate, None), (None, None)):
        out = P.plain(Q, 3, out=x.clone(), gate=gt, row_req=rr)
        gv = 1.0 if gt is None else gate[0, :N].double() if rr is None else gate.double()[req.long()][:, :N]
        want = x[:, :N].double() + gv * (p + b)
        close(out[:, :N], want, 1.01 * F32 * want.abs() + abs(gv) * product_bound(p, b))
        assert torch.equal(out[:, N:], x[:, N:])
        assert torch.equal(out, P.plain(Q, 3, out=x.clone(), gate=gt, row_req=rr, work=False))


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", list(SHARED_PAIRS) + list(SHARED_REST_PAIRS))
def test_gated_pairs_in_shares_of_k(torch, Q, M, N, K):
    P = Product(torch, M, N, K, seed=M + N + K, pad_a=16, pad_w=32, pair=True)
    g, u = P.exact(), P.exact(P.W2, P.sw2)
    zero = 0.0 * P.bias.double()
    dg, du = gelu_bound(g, product_bound(g, zero)), product_bound(u, zero)
    want = gelu64(g) * u
    tol = dg * u.abs() + gelu64(g).abs() * du + dg * du
    out = P.pair(Q)
    close(out[:, :N], want, tol + (BF16 + F32) * (want.abs() + tol))
    assert bool((out[:, N:] == 9.0).all())
    assert torch.equal(out, P.pair(Q, work=False))


def check_transposed(torch, Q, M, N, K, kind, bias):
    P = Product(torch, M, N, K, seed=M + N + K, pad_a=16)
    c = columns(M, kind)
    ldo = up(int(c[-1]) + 1, 8) + 16
    col = torch.from_numpy(c.astype(np.int32)).cuda()
    p, b = P.exact(), P.bias.double() if bias else 0.0 * P.bias.double()
    dv = product_bound(p, b)
    out = P.transposed(Q, col, ldo, bias)
    close(out[:, col.long()].t(), p + b, dv + BF16 * ((p + b).abs() + dv))
    rest = torch.ones(ldo, dtype=torch.bool, device="cuda")
    rest[col.long()] = False
    assert bool((out[:, rest] == 9.0).all())
    assert torch.equal(out, P.transposed(Q, col, ldo, bias, work=False))


@pytest.mark.gpu
@pytest.mark.parametrize("kind,bias", [("ragged", True), ("odd", False), ("sparse", True)])
@pytest.mark.parametrize("M,N,K", list(SHARED) + list(SHARED_REST))
def test_transposed_products_in_shares_of_k(torch, Q, M, N, K, kind, bias):
    check_transposed(torch, Q, M, N, K, kind, bias)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,bias", [("ragged", True), ("odd", False)])
@pytest.mark.parametrize("M,N,K", list(TILES.values()) + TWO + list(TALL))
def test_transposed_products_on_every_tile(torch, Q, M, N, K, kind, bias):
    check_transposed(torch, Q, M, N, K, kind, bias)


PARTS = ((0, 1), (3, 33), (40, 100), (100, 256), (300, 350), (11, 600), (400, 700))


@pytest.mark.gpu
def test_a_row_is_the_same_in_any_shares_of_k(torch, Q):
    """A product of 1100 rows, unsplit, and parts of it in other tiles and in 2, 3 and 4 shares of K: not a bit differs."""
    P = Product(torch, 1100, 3100, 20480)
    T = Product(torch, 1100, 1030, 20480, seed=2, pair=True)
    col = torch.arange(1100, dtype=torch.int32, device="cuda")
    full = {k: P.plain(Q, k) for k in (0, 1, 2)}
    pair, tr = T.pair(Q), P.transposed(Q, col, 1104)
    for a, n in PARTS:
        rows = slice(a, a + n)
        for k in (0, 1, 2):
            assert torch.equal(P.plain(Q, k, rows=rows), full[k][rows]), (a, n, k)
        assert torch.equal(T.pair(Q, rows=rows), pair[rows]), (a, n)
        assert torch.equal(P.transposed(Q, col, up(n, 8), rows=rows)[:, :n], tr[:, rows]), (a, n)


@pytest.mark.gpu
@pytest.mark.parametrize("work", [True, False])
def test_longest_sum_on_8_wave_tiles_and_in_shares(torch, Q, work):
    """Every code -128 at the largest K, in 4 shares (sums of 2^14 K / 4 that meet in 32 bits) and unsplit, and at 15360 on an 8-wave tile."""
    for M, N, K in ((128, 2176, Q.MAX_K), (500, 4096, 15360)):
        P = Product(torch, M, N, K)
        P.A.fill_(-128)
        P.W.fill_(-128)
        P.W[1, ::2] = 127
        P.sa.fill_(1.0)
        P.sw.fill_(1.0)
        out = P.plain(Q, 1, bias=False, work=work)[:, :N]
        some = torch.ones(N, dtype=torch.bool, device="cuda")
        some[1] = False
        assert bool((out[:, some] == 16384.0 * K).all()) and bool((out[:, 1] == float(np.float32(128 * 128 * (K // 2) - 128 * 127 * (K // 2)))).all())


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[500, 500, 500, 293], [500, 500, 500, 500, 48]])
def test_encoder_where_the_first_launch_ends_with_the_keys(torch, Q, lens):
    """1793 and 2048 tokens at T5-XXL widths: the query, key and value product's second launch is all transposed columns."""
    arch = dict(synth.ENCODERS["t5_xxl"], n_layers=1, vocab=512)
    m = Q.EncoderI8(arch)
    m.ensure_workspace(lens)
    m.workspace.fill_(0xFF)
    m.init_weights(7, 0.02)
    m.quantize()
    tok = torch.from_numpy(np.concatenate(synth.make_tokens(lens, arch["vocab"]))).cuda()
    out = torch.full((sum(lens), arch["d_model"]), float("nan"), device="cuda")
    m.forward(lens, tok, None, out)
    assert bool(torch.isfinite(out).all())
    at = 0
    for L in lens:
        solo = torch.full((L, arch["d_model"]), float("nan"), device="cuda")
        m.ensure_workspace([L])
        m.forward([L], tok[at:], None, solo)
        torch.cuda.synchronize()
        assert torch.equal(solo, out[at:at + L]), L
        at += L
    m.close()


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(3, 300, 256), (130, 37535, 128), (1137, 4096, 256), (500, 4096, 10240)])
def test_scales_whose_product_leaves_float32(torch, Q, M, N, K):
    """Two legal scales may have a product below the smallest normal number or above the largest; the result need not."""
    P = Product(torch, M, N, K, pair=True)
    P.A.clamp_(min=1)                                                # sums of at least K
    P.W.clamp_(min=1)
    P.W2.clamp_(min=1)
    u, w = P.sa / 0.01, P.sw * 50.0 * K ** 0.5                       # 0.5 .. 1.5
    col = torch.arange(M, dtype=torch.int32, device="cuda")
    for ea, ew in ((-80, -60), (-60, -80), (-126, 100), (80, -120)):
        P.sa, P.sw = torch.ldexp(u, torch.tensor(ea)).clamp_min(2.0 ** -126), torch.ldexp(w, torch.tensor(ew))
        p = P.exact()
        # sum to float32, two products; of these the last may be below 2^-126 (130 x 37535 x 128), where float32 numbers are the multiples
        # of 2^-149 and bf16 ones those of 2^-133, so that a rounding is off by up to half of that
        tol = 3.01 * F32 * p + 2.0 ** -150
        close(P.plain(Q, 1, bias=False)[:, :N], p, tol)
        tol = tol + BF16 * (p + tol) + 2.0 ** -134
        close(P.plain(Q, 0, bias=False)[:, :N], p, tol)
        close(P.transposed(Q, col, up(M, 8), bias=False)[:, :M].t(), p, tol)
    P.A.zero_()
    P.sa, P.sw = torch.ldexp(u, torch.tensor(70)), torch.ldexp(w, torch.tensor(70))
    P.sw2 = P.sw
    for kind in (0, 1, 2):
        assert bool((P.plain(Q, kind, bias=False)[:, :N] == 0.0).all())
        assert torch.equal(P.plain(Q, 1)[:, :N], P.bias.expand(M, N))
    assert bool((P.pair(Q)[:, :N] == 0.0).all()) and bool((P.transposed(Q, col, up(M, 8), bias=False)[:, :M] == 0.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(3, 300, 256), (130, 37535, 128), (176, 17220, 128), (1137, 4096, 256), (500, 4096, 10240), (333, 1000, 1536)])
def test_scales_near_the_largest_number(torch, Q, M, N, K):
    """Rows of numbers up to 2^128 have scales up to 2^121: a sum times one is past float32, the result need not be.  Every form, alone and beside
    rows of ordinary size, of zeros and of 2^-90; a row's result is the same, bit for bit, without the rows beside it."""
    P = Product(torch, M, N, K, pair=True)
    P.A[::5] = 0
    u, w = P.sa / 0.01, P.sw * 50.0 * K ** 0.5                       # 0.5 .. 1.5
    P.sw = torch.ldexp(w, torch.tensor(-124))                        # (2^-126 is the smallest scale)
    P.sw2 = P.sw.flip(0).contiguous()
    P.bias *= 0.25
    every = torch.arange(M, device="cuda")
    e = torch.tensor([-126, 110, 120, 0, -90], device="cuda")[every % 5]
    col = every.to(torch.int32)
    b = P.bias.double()
    for sa in (torch.ldexp(u, torch.tensor(110)), torch.ldexp(u, torch.tensor(120)), torch.ldexp(u, e).clamp_min(2.0 ** -126)):
        P.sa = sa
        p, p2 = P.exact(), P.exact(P.W2, P.sw2)
        dv, d2 = 3.01 * F32 * (p.abs() + abs(b)) + 2.0 ** -150, 3.01 * F32 * p2.abs() + 2.0 ** -150     # (as above: results below 2^-126)
        dp = 3.01 * F32 * p.abs() + 2.0 ** -150
        v = p + b
        out = {k: P.plain(Q, k) for k in (0, 1, 2)}
        close(out[1][:, :N], v, dv)
        close(out[0][:, :N], v, dv + BF16 * (v.abs() + dv) + 2.0 ** -134)
        tr = P.transposed(Q, col, up(M, 8))
        close(tr[:, :M].t(), v, dv + BF16 * (v.abs() + dv) + 2.0 ** -134)
        tol = gelu_bound(v, dv)
        close(out[2][:, :N], gelu64(v), tol + BF16 * (gelu64(v).abs() + tol) + 2.0 ** -134)
        x = torch.randn(M, up(N, 8) + 8, generator=torch.Generator().manual_seed(2)).cuda()
        got = P.plain(Q, 3, bias=False, out=x.clone())
        want = x[:, :N].double() + p
        close(got[:, :N], want, 1.01 * F32 * want.abs() + dp)
        pair = P.pair(Q)
        want = gelu64(p) * p2
        tol = gelu_bound(p, dp)
        tol = tol * p2.abs() + gelu64(p).abs() * d2 + tol * d2
        tol = tol + (BF16 + F32) * (want.abs() + tol) + 2.0 ** -134
        close(pair[:, :N], want, tol)
        for a, n in ((0, 1), (1, 2), (M // 2, M - M // 2)):
            rows = slice(a, a + n)
            for k in (0, 1, 2):
                assert torch.equal(P.plain(Q, k, rows=rows), out[k][rows])
            assert torch.equal(P.pair(Q, rows=rows), pair[rows])
            assert torch.equal(P.transposed(Q, col, up(n, 8), rows=rows)[:, :n], tr[:, rows])


@pytest.mark.gpu
@pytest.mark.parametrize("int8", [False, True])
def test_stage_table_counts_the_weights_that_are_held(capsys, monkeypatch, int8):
    """The codes come on top of the bf16 arena, which stays bound."""
    import json
    from paper_2510_02838_amd import encoder, int8 as Q, stage_profile
    m = Q.EncoderI8(synth.ENCODERS["t5_tiny"], bind=False)
    bf16, codes = encoder.Encoder.weight_bytes(m), m.code_bytes()
    m.close()
    monkeypatch.setattr(sys, "argv", ["stage_profile", "encode", "--encoder", "t5_tiny", "--lens", "32", "--max-batch", "2"] + ["--int8"] * int8)
    stage_profile.main()
    rows = [json.loads(line) for line in capsys.readouterr().out.splitlines()]
    rows = [r for r in rows if r["table"] == "encode"]
    assert len(rows) == 2 and all(r["weight_bytes"] == bf16 + codes * int8 and r["products"] == ("int8" if int8 else "bf16") for r in rows)
    assert all(abs(r["weight_read_floor_ms"] - (codes if int8 else bf16) / 8e9) <= 1e-12 for r in rows)
