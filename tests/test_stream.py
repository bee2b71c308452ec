"""Operators around the residual stream (lookup by token and its gradient, rows in 8 bits, layer norm of such rows) against the fp64
oracle, element by element.

Bounds, in units of u = 2^-24, half a step of fp32 relative to the value.
  lookup       one multiply-add: u |x|; a bf16 output is rounded once more, by 2^-8 of its value
  gradient     a sum of n rows: D = n in calls of up to 1024 tokens, where one wave, or four, add them up; in longer ones a term passes through at most 63
               additions in its piece of the list and the one behind (32 tokens each), a quarter of the run's pieces or 8 of them, and 5
               more where those join, D = min(n, 64 + n / 64 + 8); with the scaling (D + 1) u of the sum of magnitudes, and u of the
               result where it is added to what is there
  8 bits       codes, scales and what is read are exact
  layer norm   a sum over a row: a term passes through up to 32 additions in a lane, 6 in the wave, 4 between waves (16, 6 and 8 in the
               backward pass): D = 44 at most.
               mean: (D + 1) u mean|v| =: m.  v - mean is off by m + u |v - mean|; the terms that are linear in m cancel in the variance, which is
               off by (D + 4) u relative and m^2; rstd by half that and 4 u for its sum, root and quotient
  its gradient xh carries 2 u, g = dy gamma one more; the two means are off by (D + 4) u of the mean magnitudes of their terms; dx is
               formed of three terms by five operations.  Sums over T rows: ceil(T / 256) additions at most in a lane, 3 between rows side by
               side in a wave, 8 waves, 16 and 16 of the 256 partial sums: ceil(T / 256) + 8 + 32 has room for them"""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import stream as os_
from paper_2202_01306_amd import binding as B
from paper_2202_01306_amd import synth

U = 2.0 ** -24
INF, NAN = math.inf, math.nan
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
PC = {"fp32": B.HMY_PREC_FP32, "bf16": B.HMY_PREC_BF16}
CODE = {"int8": B.HMY_CODE_INT8, "e4m3": B.HMY_CODE_E4M3}
HALF = {"fp32": 0.0, "bf16": 2.0 ** -8}
EPS = 1e-5


def say(msg):
    print(msg, flush=True)


def rounded(x, prec):
    x = np.asarray(x, np.float32)
    return synth.round_bf16(x) if prec == "bf16" else x


def groups(d):
    return (d + 31) // 32


def rows_of(x, ld, dtype, fill=NAN, shift=0):
    """[T, ld] in a store that starts `shift` elements in; the first d columns are x, the others must not be looked at."""
    T, d = x.shape
    store = torch.full((T * ld + shift,), fill, device="cuda", dtype=dtype)
    t = store[shift:].view(T, ld)
    t[:, :d] = torch.from_numpy(np.ascontiguousarray(x)).to("cuda").to(dtype)
    return t


def bytes_of(a, ld, fill=0x5a, shift=0):
    T, d = a.shape
    store = torch.full((T * ld + shift,), fill, device="cuda", dtype=torch.uint8)
    t = store[shift:].view(T, ld)
    t[:, :d] = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t


def out_rows(T, ld, dtype, fill=7.0, shift=0):
    return torch.full((T * ld + shift,), fill, device="cuda", dtype=dtype)[shift:].view(T, ld)


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def near(got, ref, bound, what=""):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    fine = np.isfinite(ref)
    np.testing.assert_array_equal(got[~fine], ref[~fine])
    off = np.abs(got[fine] - ref[fine])
    bound = np.broadcast_to(bound, ref.shape)[fine]
    assert np.all(off <= bound), (what, float(off.max()), float((off / np.maximum(bound, 1e-300)).max()))


def scratch(nbytes):
    return torch.full((nbytes,), 0xff, device="cuda", dtype=torch.uint8)


# ---- lookup ----------------------------------------------------------------------------------------

LOOKUPS = [(1, 1, 1, 1, 1, 0, 0), (3, 7, 5, 7, 9, 4, 0), (64, 128, 512, 128, 128, 64, 0), (65, 33, 40, 35, 41, 7, 1), (300, 1600, 77, 1600, 1600, 128, 0),
           (5, 4099, 300, 4100, 4103, 3, 3), (2050, 8, 20, 8, 8, 1, 0), (17, 1024, 50257, 1024, 1025, 1024, 0), (37, 400, 60, 401, 400, 9, 0), (38, 601, 60, 601, 602, 9, 1), (39, 1096, 60, 1096, 1096, 9, 0), (21, 2500, 60, 2500, 2500, 9, 0), (1030, 24, 65537, 27, 24, 0, 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("prec,out", [("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")])
@pytest.mark.parametrize("T,d,V,ldw,ldx,P,shift", LOOKUPS)
def test_lookup_against_64_bits(prec, out, T, d, V, ldw, ldx, P, shift):
    say(f"lookup {prec} {out} T={T} d={d} V={V}")
    rng = np.random.default_rng(T * 131 + d)
    table, pos = rounded(rng.standard_normal((V, d)), prec), rounded(rng.standard_normal((max(P, 1), d)), prec)
    ids = rng.integers(0, V, T)
    ids[1::5], ids[2::9], ids[3::11] = -1, V, -2**31
    places = rng.integers(0, max(P, 1), T)
    places[::7], places[4::13] = -1, P
    td, pd = rows_of(table, ldw, DT[prec], shift=shift), rows_of(pos, ldw, DT[prec], shift=shift)
    for scale in (1.0, math.sqrt(d), -0.3):
        s = float(np.float32(scale))
        for given in ((None, places) if P else (None,)):
            x = out_rows(T, ldx, DT[out], shift=shift)
            B.hmy_k_embed_lookup(PC[prec], PC[out], i32(ids), td, x, T, d, V, ldw, ldx, scale=scale,
                                 positions=None if given is None else i32(given), pos_table=pd if P else None, P=P, ldp=ldw)
            ref = os_.embed_lookup(ids, table, s, given, pos if P else None)
            near(host(x[:, :d]), ref, np.abs(ref) * (U + HALF[out] * (1 + U)) + 2.0 ** -150)
            assert torch.all(x[:, d:] == 7.0)


# ---- its gradient ------------------------------------------------------------------------------------

def text_like(rng, T, V):
    """Tokens of which the r-th most frequent is about 1 / r as frequent as the first."""
    rank = np.clip(np.exp(rng.random(T) * np.log(V + 1)).astype(np.int64) - 1, 0, V - 1)
    return rng.permutation(V)[rank]


def depth(n, T):
    return n if T <= 1024 else np.minimum(n, 64 + n / 64 + 8)


def grad(prec, ids, dx, V, d, ldx, ldt, scale=1.0, accumulate=False, into=None, ws=None, stream=None):
    T = len(ids)
    t = out_rows(V, ldt, torch.float32) if into is None else into
    ws = scratch(B.HMY_EMBED_GRAD_WORKSPACE_BYTES(T, d)) if ws is None else ws
    B.hmy_k_embed_grad(PC[prec], ids, dx, t, T, d, V, ldx, ldt, scale=scale, accumulate=accumulate, workspace=ws, stream=stream)
    return t


GRADS = [(1, 1, 1, 1, 1, 0), (2, 5, 3, 5, 5, 0), (16, 8, 2, 8, 8, 0), (17, 31, 4, 33, 32, 1), (64, 128, 512, 128, 128, 0), (1000, 130, 3, 131, 133, 3), (700, 3000, 90, 3000, 3000, 0), (256, 9000, 40, 9000, 9001, 0), (1024, 2040, 300, 2048, 2040, 0),
         (4096, 64, 50257, 64, 64, 0), (3001, 260, 255, 260, 260, 0), (3001, 20, 256, 20, 20, 0), (1024, 520, 257, 528, 520, 0), (5000, 12, 65535, 12, 12, 0),
         (5000, 12, 65536, 13, 12, 1), (16384, 16, 1000, 16, 16, 0), (16385, 16, 1000, 16, 16, 0), (20000, 9, 70000, 9, 9, 0), (40001, 33, 300, 33, 33, 0),
         (33000, 8, 1, 8, 8, 0), (18000, 4, 16777300, 4, 4, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("T,d,V,ldx,ldt,shift", GRADS)
def test_gradient_of_a_table_against_64_bits(prec, T, d, V, ldx, ldt, shift):
    say(f"grad {prec} T={T} d={d} V={V}")
    rng = np.random.default_rng(T * 7 + V)
    ids = text_like(rng, T, V)
    if T > 8:
        ids[rng.random(T) < 0.05] = -1
        ids[3::17] = V                                   # names no row either
    dx = rounded(rng.standard_normal((T, d)), prec)
    dd = rows_of(dx, ldx, DT[prec], shift=shift)
    scale = -1.7
    s = float(np.float32(scale))
    named = np.unique(ids[(ids >= 0) & (ids < V)])
    ref, size, n = os_.embed_grad(np.searchsorted(named, ids) if V > 1 << 20 else ids, dx, len(named) if V > 1 << 20 else V, s)
    if V > 1 << 20:
        bad = (ids < 0) | (ids >= V)
        ref, size, n = os_.embed_grad(np.where(bad, -1, np.searchsorted(named, ids)), dx, len(named), s)
    bound = (depth(n, len(ids))[:, None] + 1) * U * size
    t = grad(prec, i32(ids), dd, V, d, ldx, ldt, scale)
    again = grad(prec, i32(ids), dd, V, d, ldx, ldt, scale)
    assert torch.equal(t, again)                         # one order, whatever order workgroups run in
    assert torch.all(t[:, d:] == 7.0)
    if V > 1 << 20:
        near(host(t[torch.from_numpy(named).cuda(), :d]), ref, bound)
        assert int(torch.count_nonzero(t[:, :d].abs().sum(1))) == len(named)
    else:
        near(host(t[:, :d]), ref, bound)
        assert torch.all(t[torch.from_numpy(np.nonzero(n == 0)[0]).cuda(), :d] == 0.0)
    # added to what is there: rows without a token keep every bit
    old = torch.randn(V, ldt, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    t = grad(prec, i32(ids), dd, V, d, ldx, ldt, scale, accumulate=True, into=old.clone())
    rows = torch.from_numpy(named).cuda()
    base = host(old[rows, :d])
    want = base + (ref if V > 1 << 20 else ref[named])
    near(host(t[rows, :d]), want, (bound if V > 1 << 20 else bound[named]) + U * np.abs(want))
    untouched = torch.ones(V, dtype=torch.bool, device="cuda")
    untouched[rows] = False
    assert torch.equal(t[untouched], old[untouched]) and torch.equal(t[:, d:], old[:, d:])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 15, 16, 17, 100, 256, 257, 1000, 1024, 1025, 8192, 8193, 16384, 17000])
@pytest.mark.parametrize("kind", ["one", "none", "ascending", "descending", "last", "blocks"])
def test_gradient_of_lists_where_it_can_go_wrong(T, kind):
    say(f"grad {kind} T={T}")
    V, d = 40000, 12
    at = np.arange(T)
    ids = {"one": np.full(T, 7), "none": np.where(at % 2, -1, V + at), "ascending": at % V, "descending": V - 1 - at, "last": np.full(T, V - 1),
           "blocks": at // 16 * 3}[kind]
    dx = np.random.default_rng(T).standard_normal((T, d)).astype(np.float32)
    ref, size, n = os_.embed_grad(ids, dx, V)
    t = grad("fp32", i32(ids), rows_of(dx, d, torch.float32), V, d, d, d)
    near(host(t), ref, (depth(n, T)[:, None] + 1) * U * size)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [3, 20, 300])
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("least,seed", [(257, 1), (257, 2), (257, 3), (1500, 4), (3000, 5), (8300, 6), (8300, 7), (12000, 8)])
def test_gradient_of_runs_of_every_length(prec, d, least, seed):
    """Runs that begin and end around the ends of pieces of 16 and 32 tokens, up to some that go through eight, nine and many of them."""
    say(f"grad runs {prec} d={d} least={least} seed={seed}")
    rng = np.random.default_rng(seed)
    piece = 16 if least < 8192 else 32
    lengths = [1, 1, 1, 2, 3, piece - 1, piece, piece + 1, 2 * piece - 1, 2 * piece, 2 * piece + 1, 3 * piece, 3 * piece + 5, 8 * piece, 9 * piece - 1, 9 * piece,
               10 * piece + 3, 11 * piece + 1, 40 * piece + 7, 70 * piece]
    runs = []
    while sum(runs) < least:
        runs.append(int(rng.choice(lengths)))
    names = np.sort(rng.choice(3000, len(runs), replace=False))
    ids = rng.permutation(np.repeat(names, runs))
    ids = np.concatenate([ids, np.full(int(rng.integers(0, 40)), -1)])
    assert (len(ids) <= 8192) == (piece == 16) and len(ids) > 256
    dx = rounded(rng.standard_normal((len(ids), d)), prec)
    ref, size, n = os_.embed_grad(ids, dx, 3000)
    dd = rows_of(dx, d, DT[prec])
    t = grad(prec, i32(ids), dd, 3000, d, d, d)
    bound = (depth(n, len(ids))[:, None] + 1) * U * size
    near(host(t), ref, bound)
    old = torch.randn(3000, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6))
    t = grad(prec, i32(ids), dd, 3000, d, d, d, accumulate=True, into=old.clone())
    near(host(t), ref + host(old), bound + U * np.abs(ref + host(old)))


@pytest.mark.gpu
@pytest.mark.parametrize("V", [200, 70000])
def test_gradient_of_so_many_tokens_that_the_sort_scans_its_counts(V):
    T, d = 300001, 2
    rng = np.random.default_rng(V)
    ids = text_like(rng, T, V)
    ids[::50] = -1
    dx = rng.standard_normal((T, d)).astype(np.float32)
    ref, size, n = os_.embed_grad(ids, dx, V)
    near(host(grad("fp32", i32(ids), rows_of(dx, d, torch.float32), V, d, d, d)), ref, (depth(n, len(ids))[:, None] + 1) * U * size)


@pytest.mark.gpu
@pytest.mark.parametrize("prec,T,d,ldx,shift", [("fp32", 2100, 16001, 16003, 1), ("bf16", 2100, 32001, 32001, 0), ("fp32", 9001, 3730, 3731, 0), ("bf16", 9001, 7463, 7463, 1)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_more_rows_than_the_caches_hold(prec, T, d, ldx, shift, accumulate):
    """128 MiB of dx and more: whole numbers, whose sums fp32 holds."""
    say(f"grad large {prec} T={T} d={d} accumulate={accumulate}")
    V = 300
    rng = np.random.default_rng(T + d)
    ids = text_like(rng, T, V)
    ids[5::40] = -1
    dx = rng.integers(-9, 10, (T, d), dtype=np.int8)     # up to 9 * 9001 in a sum, below 2^24
    ref = np.stack([dx[ids == v].sum(0, dtype=np.int64) for v in range(V)])
    dd = rows_of(dx.astype(np.float32), ldx, DT[prec], shift=shift)
    old = torch.full((V, d), 3.0, device="cuda") if accumulate else None
    t = grad(prec, i32(ids), dd, V, d, ldx, d, scale=2.0, accumulate=accumulate, into=old)
    assert torch.equal(t, torch.from_numpy(2 * ref + 3 * accumulate).float().cuda())


@pytest.mark.gpu
def test_gradient_of_the_positions_is_the_same_call():
    T, d, P = 700, 40, 128
    rng = np.random.default_rng(1)
    places = np.arange(T) % P
    places[::9] = -1
    dx = rng.standard_normal((T, d)).astype(np.float32)
    ref, size, n = os_.embed_grad(places, dx, P)
    near(host(grad("fp32", i32(places), rows_of(dx, d, torch.float32), P, d, d, d)), ref, (depth(n, T)[:, None] + 1) * U * size)


@pytest.mark.gpu
def test_gradient_of_rows_that_hold_no_numbers():
    """A NaN or an infinity stays in the row of its token and in its column; padding's are not looked at."""
    T, d, V = 200, 16, 50
    rng = np.random.default_rng(3)
    ids = rng.integers(0, V, T)
    ids[[10, 50]] = -1
    ids[[20, 21]] = 5, 9
    dx = rng.standard_normal((T, d)).astype(np.float32)
    dx[10], dx[50] = NAN, INF
    dx[20, 3], dx[21, 4] = NAN, INF
    t = host(grad("fp32", i32(ids), rows_of(dx, d, torch.float32), V, d, d, d))
    off = np.argwhere(~np.isfinite(t))
    assert off.tolist() == [[5, 3], [9, 4]] and np.isnan(t[5, 3]) and t[9, 4] == INF


# ---- rows in 8 bits ----------------------------------------------------------------------------------

def stream_rows(rng, T, d, prec="fp32"):
    x = rng.standard_normal((T, d)) * np.exp(rng.normal(0, 2, (T, 1)))
    x[:, ::37] *= 40.0
    return rounded(x, prec)


def hard_groups(prec, d=96):
    rng = np.random.default_rng(8)
    x = np.zeros((40, d), np.float32)
    x[1] = -0.0
    x[2] = 1e-45                                         # the least number there is
    x[3] = 2.0 ** -126
    x[4] = 2.0 ** -120 * rng.standard_normal(d)
    x[5] = 3.4e38
    x[6] = np.float32(2.0 ** 127)
    x[7, 5], x[7, 40] = NAN, 1.0
    x[8, 70], x[8, 40] = INF, 1.0
    x[9, 0] = -INF
    for r, top in enumerate((127.0, 448.0)):             # at the border of a scale and next to it, with ties between two codes
        for k, a in enumerate((top, np.nextafter(np.float32(top), np.float32(0)), np.nextafter(np.float32(top), np.float32(1e9)), top * 2.0 ** 20, 2 * top)):
            row = 10 + 5 * r + k
            x[row] = np.linspace(-1, 1, d) * top
            x[row, ::32] = a
            x[row, 1::32], x[row, 2::32], x[row, 3::32] = 0.5, 1.5, -2.5
    x[20] = np.arange(d) - 48 + 0.5
    x[21] = (np.arange(d) - 48) * 2.0 ** -10
    x[22] = 2.0 ** (-np.arange(d) % 40.0)                # most of it below what the scale resolves
    x[23] = 448.0 * 2.0 ** -(np.arange(d) % 20.0)
    x[24, 0], x[24, 1:] = 448.0, np.arange(1, d) * 2.0 ** -10   # among the least of the format's numbers, and ties there
    for r in range(25, 40):
        x[r] = rng.standard_normal(d) * 10.0 ** rng.integers(-38, 38)
    with np.errstate(over="ignore"):
        return rounded(x, prec)


def packed(x, prec, code, ldx=None, ldc=None, lds=None, shift=0, stream=None):
    T, d = x.shape
    ldx, ldc, lds = ldx or d, ldc or d, lds or groups(d)
    codes, scales = bytes_of(np.zeros((T, 0), np.uint8), ldc, shift=shift), bytes_of(np.zeros((T, 0), np.uint8), lds, shift=shift)
    B.hmy_k_pack8(PC[prec], CODE[code], rows_of(x, ldx, DT[prec], shift=shift), codes, scales, T, d, ldx, ldc, lds, stream=stream)
    return codes, scales


def check_packed(x, prec, code, codes, scales):
    T, d = x.shape
    want, two = os_.pack8(x, code)
    np.testing.assert_array_equal(scales[:, :groups(d)].cpu().numpy(), two)
    np.testing.assert_array_equal(codes[:, :d].cpu().numpy(), want)
    assert torch.all(codes[:, d:] == 0x5a) and torch.all(scales[:, groups(d):] == 0x5a)


MOVES = [(1, 1, 1, 1, 1, 0), (1, 8, 8, 8, 1, 0), (3, 31, 33, 31, 2, 1), (4, 32, 32, 32, 1, 0), (5, 33, 35, 40, 3, 3), (64, 128, 128, 128, 4, 0),
         (7, 1601, 1603, 1607, 51, 5), (300, 1024, 1024, 1024, 32, 0), (2, 8193, 8193, 8193, 257, 0), (1000, 40, 40, 41, 2, 0), (33, 4096, 4100, 4096, 130, 2),
         (37, 400, 401, 400, 13, 0), (38, 601, 601, 603, 19, 1), (39, 1096, 1096, 1096, 35, 0), (21, 2500, 2500, 2500, 79, 0), (130, 4400, 4400, 4400, 138, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("T,d,ldx,ldc,lds,shift", MOVES)
def test_rows_to_8_bits_and_back(prec, code, T, d, ldx, ldc, lds, shift):
    say(f"pack8 {prec} {code} T={T} d={d}")
    x = stream_rows(np.random.default_rng(T + d), T, d, prec)
    codes, scales = packed(x, prec, code, ldx, ldc, lds, shift)
    check_packed(x, prec, code, codes, scales)
    ref = os_.unpack8(codes[:, :d].cpu().numpy(), scales[:, :groups(d)].cpu().numpy(), code)
    for out in ("fp32", "bf16"):
        y = out_rows(T, ldx, DT[out], shift=shift)
        B.hmy_k_unpack8(PC[out], CODE[code], codes, scales, y, T, d, ldc, lds, ldx)
        np.testing.assert_array_equal(host(y[:, :d]), ref)
        assert torch.all(y[:, d:] == 7.0)


@pytest.mark.gpu
@pytest.mark.parametrize("prec,T,d,ld,shift", [("fp32", 8200, 4099, 4099, 1), ("bf16", 42000, 1601, 1603, 0), ("fp32", 1400000, 24, 24, 0), ("bf16", 10000000, 7, 7, 1), ("fp32", 131072, 256, 260, 0)])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_more_rows_to_8_bits_than_the_caches_hold(prec, code, T, d, ld, shift):
    """128 MiB of rows and more in one call give what calls of few rows each give."""
    say(f"pack8 large {prec} {code} T={T} d={d}")
    x = torch.randn(T * ld + shift, device="cuda", generator=torch.Generator(device="cuda").manual_seed(d)).to(DT[prec])[shift:].view(T, ld)
    x[:, ::5] *= 30.0
    g, step = groups(d), T // 3 + 1

    def pack(lo, hi, codes, scales):
        B.hmy_k_pack8(PC[prec], CODE[code], x[lo:hi], codes[lo:hi], scales[lo:hi], hi - lo, d, ld, d, g)

    whole, parts = [[torch.full((T, n), 0x5a, device="cuda", dtype=torch.uint8) for n in (d, g)] for _ in range(2)]
    pack(0, T, *whole)
    for lo in range(0, T, step):
        pack(lo, min(T, lo + step), *parts)
    assert torch.equal(whole[0], parts[0]) and torch.equal(whole[1], parts[1])


@pytest.mark.gpu
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_groups_where_8_bits_can_go_wrong(prec, code):
    x = hard_groups(prec)
    codes, scales = packed(x, prec, code)
    check_packed(x, prec, code, codes, scales)
    y = out_rows(*x.shape, torch.float32)
    B.hmy_k_unpack8(0, CODE[code], codes, scales, y, *x.shape, x.shape[1], groups(x.shape[1]), x.shape[1])
    with np.errstate(over="ignore"):                     # the largest fp32 numbers are rounded to 2^128, which is infinity as fp32
        ref = os_.unpack8(codes.cpu().numpy(), scales.cpu().numpy(), code).astype(np.float32)
    np.testing.assert_array_equal(host(y), ref)
    assert torch.isnan(y[7, :32]).all() and y[7, 40] == 1.0 and torch.isnan(y[8, 64:]).all() and torch.isnan(y[9, :32]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_every_code_and_every_scale_is_read_as_it_is_defined(code):
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 8, 1)
    with np.errstate(over="ignore"):
        ref = os_.unpack8(codes, scales, code).astype(np.float32)
    for out in ("fp32", "bf16"):
        y = out_rows(256, 256, DT[out])
        B.hmy_k_unpack8(PC[out], CODE[code], bytes_of(codes, 256), bytes_of(scales, 8), y, 256, 256, 256, 8, 256)
        want = torch.from_numpy(ref).to(DT[out]).double().numpy()
        np.testing.assert_array_equal(host(y), want)


# ---- layer norm ------------------------------------------------------------------------------------------

D = 44
NORMS = [(1, 1, 1, 0), (3, 7, 9, 1), (5, 33, 40, 0), (64, 128, 128, 0), (9, 512, 512, 0), (10, 513, 515, 3), (70, 1024, 1024, 0), (13, 1025, 1025, 0),
         (11, 1600, 1601, 1), (10, 1280, 1280, 0), (9, 1500, 1500, 0), (8, 1300, 1301, 0), (7, 5130, 5130, 0), (6, 7000, 7001, 1), (9, 2048, 2048, 0), (7, 2049, 2056, 0), (6, 4096, 4096, 0), (5, 4099, 4103, 2), (4, 8192, 8192, 0), (3, 8185, 8191, 5),
         (2500, 65, 65, 0), (3001, 8, 8, 0), (2777, 31, 33, 1), (2049, 32, 32, 0), (2600, 64, 64, 0), (3000, 100, 101, 0), (2500, 129, 129, 2), (2200, 260, 260, 0), (8200, 700, 700, 0), (5000, 1024, 1024, 0), (1100, 4096, 4096, 0)]


def dx_bound(dy, v, mean, rstd, gamma, dx, res=None):
    g, xh, r = np.abs(dy * gamma), np.abs((v - mean[:, None]) * rstd[:, None]), rstd[:, None]
    inner = dx if res is None else dx - res
    return U * (r * (6 * g + (D + 6) * g.mean(1, keepdims=True) + xh * (D + 10) * (g * xh).mean(1, keepdims=True)) + 4 * np.abs(inner) + np.abs(dx))


class Norm:
    def __init__(self, prec, code, T, d, ld, shift=0, seed=0):
        rng = np.random.default_rng(T * 3 + d + seed)
        self.prec, self.code, self.T, self.d, self.ld, self.shift, self.G = prec, code, T, d, ld, shift, groups(d)
        x = stream_rows(rng, T, d) + 0.2
        codes, scales = os_.pack8(x, code)
        self.v = os_.unpack8(codes, scales, code)
        self.codes, self.scales = bytes_of(codes, ld, shift=shift), bytes_of(scales, self.G, shift=shift)
        self.gamma, self.beta = rounded(rng.standard_normal(d) * 0.3 + 1, prec), rounded(rng.standard_normal(d) * 0.2, prec)
        self.dy = rounded(rng.standard_normal((T, d)), prec)
        self.res = rng.standard_normal((T, d)).astype(np.float32)
        vector = lambda a: rows_of(a[None], d, DT[prec], shift=shift)[0]
        self.g, self.b = vector(self.gamma), vector(self.beta)

    def forward(self, keep_x=True, stats=True, stream=None):
        self.y = out_rows(self.T, self.ld, DT[self.prec], shift=self.shift)
        self.x = out_rows(self.T, self.ld, torch.float32, shift=self.shift) if keep_x else None
        self.mean, self.rstd = (torch.full((self.T,), 7.0, device="cuda") for _ in range(2)) if stats else (None, None)
        B.hmy_k_layernorm8_fwd(PC[self.prec], CODE[self.code], self.codes, self.scales, self.g, self.b, self.y, self.mean, self.rstd, self.T,
                               self.d, self.ld, self.G, self.ld, EPS, x=self.x, ldx=self.ld, stream=stream)
        return self.y

    def check_forward(self):
        y, m, r = os_.layernorm(self.v, self.gamma.astype(np.float64), self.beta.astype(np.float64), EPS)
        var = 1 / r ** 2
        dm = (D + 1) * U * np.abs(self.v).mean(1)
        dr = 0.5 * ((D + 4) * U + dm ** 2 / var) + 4 * U     # relative
        t = np.abs(self.v - m[:, None])
        near(host(self.mean), m, dm, "mean")
        near(host(self.rstd), r, r * dr, "rstd")
        bound = np.abs(self.gamma) * (r[:, None] * (t * (dr[:, None] + 3 * U) + dm[:, None])) + U * np.abs(y)
        near(host(self.y[:, :self.d]), y, bound + HALF[self.prec] * (np.abs(y) + bound), "y")
        assert torch.all(self.y[:, self.d:] == 7.0)
        if self.x is not None:
            np.testing.assert_array_equal(host(self.x[:, :self.d]), self.v)
            assert torch.all(self.x[:, self.d:] == 7.0)

    def backward(self, res=True, rounded_too=True, sums=True, accumulate=False, into=None, in_place=False, ws=None, stream=None, dx=None):
        T, d, ld = self.T, self.d, self.ld
        self.dyd = rows_of(self.dy, ld, DT[self.prec], shift=self.shift)
        self.resd = rows_of(self.res, ld, torch.float32, fill=7.0, shift=self.shift) if res else None
        self.dx = self.resd if in_place else out_rows(T, ld, torch.float32, shift=self.shift)
        self.dx_e = out_rows(T, ld, DT[self.prec], shift=self.shift) if rounded_too else None
        self.sums = [torch.full((d,), 7.0, device="cuda") for _ in range(3)] if into is None else into
        ws = scratch(B.HMY_NORM8_WORKSPACE_BYTES(d)) if ws is None else ws
        B.hmy_k_layernorm8_bwd(PC[self.prec], CODE[self.code], self.dyd, self.codes, self.scales, self.mean, self.rstd, self.g, self.dx, self.sums[0],
                               self.sums[1], T, d, ld, self.G, ld, ld, res=self.resd, ldr=ld, dx_e=self.dx_e, lde=ld,
                               dres_sum=self.sums[2] if sums and res else None, accumulate=accumulate, workspace=ws, stream=stream)
        return [t for t in (self.dx, self.dx_e, *self.sums) if t is not None]

    def check_backward(self, res=True, sums=True, base=None):
        mean, rstd = host(self.mean), host(self.rstd)
        gamma, dy = self.gamma.astype(np.float64), self.dy.astype(np.float64)
        r64 = self.res.astype(np.float64) if res else None
        dx, dg, db, dr = os_.layernorm_grad(dy, self.v, mean, rstd, gamma, r64)
        xh = (self.v - mean[:, None]) * rstd[:, None]
        bound = dx_bound(dy, self.v, mean, rstd, gamma, dx, r64)
        near(host(self.dx[:, :self.d]), dx, bound, "dx")
        assert torch.all(self.dx[:, self.d:] == 7.0)
        if self.dx_e is not None:
            assert torch.equal(self.dx_e[:, :self.d], self.dx[:, :self.d].to(DT[self.prec])) and torch.all(self.dx_e[:, self.d:] == 7.0)
        n = math.ceil(self.T / 256) + 8 + 32
        for name, t, ref, size, own in (("dgamma", self.sums[0], dg, np.abs(dy * xh).sum(0), 4), ("dbeta", self.sums[1], db, np.abs(dy).sum(0), 0),
                                        ("dres", self.sums[2], dr, np.abs(r64).sum(0) if res else None, 0)):
            if ref is None or (name == "dres" and not sums):
                assert torch.all(t == (7.0 if base is None else base))
                continue
            want = ref + (0 if base is None else base)
            near(host(t), want, (n + own) * U * size + U * np.abs(want), name)


@pytest.mark.gpu
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("T,d,ld,shift", NORMS)
def test_layer_norm_of_rows_in_8_bits_and_its_gradient(prec, code, T, d, ld, shift):
    say(f"norm8 {prec} {code} T={T} d={d}")
    n = Norm(prec, code, T, d, ld, shift)
    n.forward()
    n.check_forward()
    first = [t.clone() for t in n.backward()]
    n.check_backward()
    for a, b in zip(first, n.backward()):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(40, 96), (300, 1024), (20, 3000), (9, 6001)])
def test_layer_norm_any_subset_of_outputs(T, d):
    n = Norm("bf16", "int8", T, d, d + 3)
    n.forward(keep_x=False)
    n.check_forward()
    y = n.y.clone()
    n.forward(keep_x=True, stats=False)
    assert torch.equal(y, n.y)
    n.forward()
    for kw in (dict(res=False), dict(res=False, rounded_too=False), dict(rounded_too=False), dict(sums=False)):
        n.backward(**kw)
        n.check_backward(res=kw.get("res", True), sums=kw.get("sums", True))
    # in place of the residual connection's gradient, and added to what is there
    n.backward(in_place=True, accumulate=True, into=[torch.full((d,), 3.0, device="cuda") for _ in range(3)])
    n.check_backward(base=3.0)


@pytest.mark.gpu
def test_layer_norm_of_rows_that_hold_no_numbers():
    """A group that was packed with a NaN makes its row NaN and no other."""
    T, d = 70, 200
    n = Norm("fp32", "int8", T, d, d)
    n.scales[11, 2] = 255
    n.v[11, 64:96] = NAN
    n.forward()
    keep = np.arange(T) != 11
    y, x = host(n.y), host(n.x)
    assert np.isnan(y[11]).all() and np.isfinite(y[keep]).all()
    assert np.isnan(x[11, 64:96]).all() and np.isfinite(x[11, :64]).all() and np.isnan(host(n.mean)[11])
    n.backward()
    dx = host(n.dx)
    assert np.isnan(dx[11]).all() and np.isfinite(dx[keep]).all() and torch.isnan(n.sums[0]).all() and torch.isfinite(n.sums[1]).all()


@pytest.mark.gpu
def test_layer_norm_of_equal_columns():
    """Variance 0: the rows are beta, and the gradient is what eps leaves."""
    T, d = 5, 640
    n = Norm("fp32", "int8", T, d, d)
    n.codes[:, :d], n.scales[:] = 64, 127
    n.v[:] = 64.0
    n.forward()
    n.check_forward()
    assert torch.equal(n.y, n.b.expand(T, d))
    n.backward()
    n.check_backward()


# ---- together, in graphs, on streams, at the ends of the range ---------------------------------------------

class Step:
    """Tokens to the stream, the stream to a checkpoint, the checkpoint through a layer norm, and all of it backward."""

    def __init__(self, seed, T=600, d=256, V=1000, P=64, prec="bf16", code="int8"):
        rng = np.random.default_rng(seed)
        self.T, self.d, self.V, self.P, self.prec, self.code = T, d, V, P, prec, code
        self.ids = text_like(rng, T, V)
        self.ids[-20:] = -1
        self.places = np.where(self.ids >= 0, np.arange(T) % P, -1)
        self.table, self.pos = rounded(rng.standard_normal((V, d)), prec), rounded(rng.standard_normal((P, d)), prec)
        self.gamma, self.beta = rounded(rng.standard_normal(d) + 1, prec), rounded(rng.standard_normal(d), prec)
        self.dy, self.res = rounded(rng.standard_normal((T, d)), prec), rng.standard_normal((T, d)).astype(np.float32)
        dev = lambda a: torch.from_numpy(a).cuda().to(DT[prec])
        self.dev = [i32(self.ids), i32(self.places), dev(self.table), dev(self.pos), dev(self.gamma), dev(self.beta), dev(self.dy), torch.from_numpy(self.res).cuda()]
        f = lambda *s: torch.full(s, 7.0, device="cuda")
        self.x, self.codes, self.scales = f(T, d), torch.zeros(T, d, dtype=torch.uint8, device="cuda"), torch.zeros(T, groups(d), dtype=torch.uint8, device="cuda")
        self.y, self.v, self.mean, self.rstd = f(T, d).to(DT[prec]), f(T, d), f(T), f(T)
        self.dx, self.dgamma, self.dbeta, self.dres, self.dtable, self.dpos = f(T, d), f(d), f(d), f(d), f(V, d), f(P, d)
        self.ws = [scratch(B.HMY_NORM8_WORKSPACE_BYTES(d)), scratch(B.HMY_EMBED_GRAD_WORKSPACE_BYTES(T, d))]

    def run(self, stream=None):
        ids, places, table, pos, gamma, beta, dy, res = self.dev
        T, d, G, p, c = self.T, self.d, groups(self.d), PC[self.prec], CODE[self.code]
        B.hmy_k_embed_lookup(p, 0, ids, table, self.x, T, d, self.V, d, d, scale=16.0, positions=places, pos_table=pos, P=self.P, ldp=d, stream=stream)
        B.hmy_k_pack8(0, c, self.x, self.codes, self.scales, T, d, d, d, G, stream=stream)
        B.hmy_k_layernorm8_fwd(p, c, self.codes, self.scales, gamma, beta, self.y, self.mean, self.rstd, T, d, d, G, d, EPS, x=self.v, ldx=d, stream=stream)
        B.hmy_k_layernorm8_bwd(p, c, dy, self.codes, self.scales, self.mean, self.rstd, gamma, self.dx, self.dgamma, self.dbeta, T, d, d, G, d, d, res=res,
                               ldr=d, dres_sum=self.dres, workspace=self.ws[0], stream=stream)
        B.hmy_k_embed_grad(0, ids, self.dx, self.dtable, T, d, self.V, d, d, scale=16.0, workspace=self.ws[1], stream=stream)
        B.hmy_k_embed_grad(0, places, self.dx, self.dpos, T, d, self.P, d, d, workspace=self.ws[1], stream=stream)

    def outputs(self):
        return [self.x, self.codes, self.scales, self.y, self.v, self.mean, self.rstd, self.dx, self.dgamma, self.dbeta, self.dres, self.dtable, self.dpos]

    def refill(self, other):
        for a, b in zip(self.dev, other.dev):
            a.copy_(b)


@pytest.mark.gpu
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_a_step_from_tokens_to_the_gradient_of_their_table(code):
    s = Step(4, code=code)
    s.run()
    x = os_.embed_lookup(s.ids, s.table, 16.0, s.places, s.pos)
    near(host(s.x), x, U * np.abs(x))
    codes, scales = os_.pack8(host(s.x), code)
    np.testing.assert_array_equal(s.codes.cpu().numpy(), codes)
    np.testing.assert_array_equal(s.scales.cpu().numpy(), scales)
    v = os_.unpack8(codes, scales, code)
    np.testing.assert_array_equal(host(s.v), v)
    y, m, r = os_.layernorm(v, s.gamma.astype(np.float64), s.beta.astype(np.float64), EPS)
    dm = (D + 1) * U * np.abs(v).mean(1)
    near(host(s.mean), m, dm)
    dx, dg, db, dr = os_.layernorm_grad(s.dy.astype(np.float64), v, host(s.mean), host(s.rstd), s.gamma.astype(np.float64), s.res.astype(np.float64))
    near(host(s.dx), dx, dx_bound(s.dy.astype(np.float64), v, host(s.mean), host(s.rstd), s.gamma.astype(np.float64), dx, s.res.astype(np.float64)))
    for out, at, V, scale in ((s.dtable, s.ids, s.V, 16.0), (s.dpos, s.places, s.P, 1.0)):
        ref, size, n = os_.embed_grad(at, host(s.dx), V, scale)
        near(host(out), ref, (depth(n, s.T)[:, None] + 1) * U * size)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(600, 256), (17000, 48), (30, 2500)])
def test_captured_and_replayed(T, d):
    say(f"graph T={T} d={d}")
    s, others = Step(1, T=T, d=d), [Step(k, T=T, d=d) for k in (2, 3)]
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run(stream=torch.cuda.current_stream().cuda_stream)
    for k in range(4):
        o = others[k % 2]
        o.run()                                          # eager work between replays, with workspaces of its own
        s.refill(o)
        for t in s.outputs():
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(s.outputs(), o.outputs()):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_two_graphs_that_share_workspaces_one_after_the_other():
    a, b = Step(1), Step(2, T=400, d=128)
    big = [scratch(B.HMY_NORM8_WORKSPACE_BYTES(256)), scratch(B.HMY_EMBED_GRAD_WORKSPACE_BYTES(600, 256))]
    want = []
    for s in (a, b):
        s.run()
        want.append([t.clone() for t in s.outputs()])
        s.ws = big
    torch.cuda.synchronize()
    made = []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run(stream=torch.cuda.current_stream().cuda_stream)
        made.append(g)
    for k in (0, 1, 1, 0, 0, 1):
        s = (a, b)[k]
        for t in s.outputs():
            t.fill_(3)
        made[k].replay()
        torch.cuda.synchronize()
        for x, y in zip(s.outputs(), want[k]):
            assert torch.equal(x, y)


@pytest.mark.gpu
def test_two_streams_with_workspaces_each():
    steps = [Step(k, T=3000, d=512) for k in (1, 2)]
    want = []
    for s in steps:
        s.run()
        want.append([t.clone() for t in s.outputs()])
        for t in s.outputs():
            t.fill_(3)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(3):
        for s, q in zip(steps, streams):
            s.run(stream=q.cuda_stream)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        for a, b in zip(s.outputs(), w):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_rows_side_by_side_in_one_array():
    """Checkpoint and scales in one array of bytes, and a gradient beside the gradient that it reads."""
    T, d = 50, 96
    x = stream_rows(np.random.default_rng(2), T, d)
    store = torch.full((T, 128), 0x5a, dtype=torch.uint8, device="cuda")
    codes, scales = store, store[:, 100:]
    B.hmy_k_pack8(0, 0, rows_of(x, d, torch.float32), codes, scales, T, d, d, 128, 128)
    want, two = os_.pack8(x, "int8")
    got = store.cpu().numpy()
    np.testing.assert_array_equal(got[:, :d], want)
    np.testing.assert_array_equal(got[:, 100:103], two)
    assert (got[:, d:100] == 0x5a).all() and (got[:, 103:] == 0x5a).all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits_and_more_tiles_than_workgroups():
    """2^32 elements and more: 2^20 + 3 rows of 4096 columns, the last of them looked at."""
    T, d = (1 << 20) + 3, 4096
    x = torch.zeros(T, d, device="cuda", dtype=torch.bfloat16)
    rng = np.random.default_rng(5)
    at = [0, 1, (1 << 19) - 1, 1 << 19, (1 << 20) - 1, 1 << 20, T - 1]
    some = stream_rows(rng, len(at), d, "bf16")
    x[at] = torch.from_numpy(some).cuda().bfloat16()
    codes, scales = torch.full((T, d), 9, device="cuda", dtype=torch.uint8), torch.full((T, groups(d)), 9, device="cuda", dtype=torch.uint8)
    B.hmy_k_pack8(1, 0, x, codes, scales, T, d, d, d, groups(d))
    want, two = os_.pack8(some, "int8")
    np.testing.assert_array_equal(codes[at].cpu().numpy(), want)
    np.testing.assert_array_equal(scales[at].cpu().numpy(), two)
    assert int(codes.count_nonzero()) == int(np.count_nonzero(want))
    x.fill_(7)
    B.hmy_k_unpack8(1, 0, codes, scales, x, T, d, d, groups(d), d)
    np.testing.assert_array_equal(host(x[at]), os_.unpack8(want, two, "int8"))
    assert int((x == 7).sum()) == int((os_.unpack8(want, two, "int8") == 7).sum())
    gamma, beta = torch.ones(d, device="cuda", dtype=torch.bfloat16), torch.full((d,), 0.5, device="cuda", dtype=torch.bfloat16)
    mean, rstd = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    B.hmy_k_layernorm8_fwd(1, 0, codes, scales, gamma, beta, x, mean, rstd, T, d, d, groups(d), d, EPS)
    y, m, r = os_.layernorm(os_.unpack8(want, two, "int8"), 1.0, 0.5, EPS)
    np.testing.assert_allclose(host(x[at]), y, rtol=2.0 ** -7, atol=2.0 ** -8)
    assert int((x == 0.5).all(1).sum()) == T - len(at)
    dx = torch.empty(T, d, device="cuda")
    dg, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    B.hmy_k_layernorm8_bwd(1, 0, x, codes, scales, mean, rstd, gamma, dx, dg, db, T, d, d, groups(d), d, d, workspace=scratch(B.HMY_NORM8_WORKSPACE_BYTES(d)))
    args = (host(x[at]), os_.unpack8(want, two, "int8"), host(mean[at]), host(rstd[at]), np.ones(d))
    ref = os_.layernorm_grad(*args)[0]
    near(host(dx[at]), ref, dx_bound(*args, ref))
    near(host(db), np.full(d, 0.5 * (T - len(at))) + host(x[at]).sum(0), (math.ceil(T / 256) + 40) * U * 0.6 * T)
    del dx, codes
    # rows far apart, in the table and out of it
    table = torch.zeros(66000, 65600, device="cuda", dtype=torch.bfloat16)
    table[:, :64] = torch.arange(66000, device="cuda")[:, None] % 251
    ids = torch.tensor([65999, 3, 65535, -1, 65999], dtype=torch.int32, device="cuda")
    out = torch.full((5, 64), 7.0, device="cuda")
    B.hmy_k_embed_lookup(1, 0, ids, table, out, 5, 64, 66000, 65600, 64)
    assert out[:, 0].tolist() == [65999 % 251, 3, 65535 % 251, 0, 65999 % 251]
    into = table.view(torch.float32)
    into.zero_()
    B.hmy_k_embed_grad(0, ids, out, into, 5, 64, 66000, 64, 32800, accumulate=True, workspace=scratch(B.HMY_EMBED_GRAD_WORKSPACE_BYTES(5, 64)))
    assert into[65999, 0] == 2 * (65999 % 251) and into[3, 63] == 3 and int(into.count_nonzero()) == 64 * 3


# ---- without a GPU --------------------------------------------------------------------------------------------

def test_structs_and_sizes_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ["hmy_embed_lookup_desc", "hmy_embed_grad_desc", "hmy_rows8_desc", "hmy_layernorm8_desc", "hmy_layernorm8_grad_desc"]
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hmy.h"\nint main(void){' +
                   "".join(f'printf("%zu\\n", sizeof({n}));' +
                           "".join(f'printf("%zu\\n", offsetof({n}, {f}));' for f, _ in getattr(B, n)._fields_) for n in names) +
                   'printf("%d %d %d %d %d\\n", HMY_MAX_SORTED, HMY_CODE_INT8, HMY_CODE_E4M3, HMY_ROWS8_GROUP, HMY_MAX_NORM8_COLUMNS);'
                   'printf("%llu %llu\\n", (unsigned long long)HMY_EMBED_GRAD_WORKSPACE_BYTES(16777215, 4097), (unsigned long long)HMY_NORM8_WORKSPACE_BYTES(8192));'
                   'return 0;}')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    out = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for n in names:
        S = getattr(B, n)
        want += [ctypes.sizeof(S)] + [getattr(S, f).offset for f, _ in S._fields_]
    want += [B.HMY_MAX_SORTED, B.HMY_CODE_INT8, B.HMY_CODE_E4M3, B.HMY_ROWS8_GROUP, B.HMY_MAX_NORM8_COLUMNS]
    want += [B.HMY_EMBED_GRAD_WORKSPACE_BYTES(16777215, 4097), B.HMY_NORM8_WORKSPACE_BYTES(8192)]
    assert out == want


A = 1 << 24    # addresses that are looked at for alignment and overlap only, this far apart


def at(k):
    return (k + 1) * A


def lookup(**kw):
    a = dict(prec=0, out_prec=0, ids=at(0), table=at(1), x=at(2), T=4, d=10, V=6, ldw=10, ldx=10, positions=at(3), pos_table=at(4), P=3, ldp=10)
    a.update(kw)
    B.hmy_k_embed_lookup(**a)


def gradient(**kw):
    a = dict(prec=0, ids=at(0), dx=at(1), dtable=at(2), T=4, d=10, V=6, ldx=10, ldt=10, workspace=at(3), workspace_bytes=1 << 20)
    a.update(kw)
    B.hmy_k_embed_grad(**a)


def pack(**kw):
    a = dict(prec=0, code=0, x=at(0), codes=at(1), scales=at(2), T=4, d=40, ldx=40, ldc=40, lds=2)
    a.update(kw)
    B.hmy_k_pack8(**a)


def unpack(**kw):
    a = dict(prec=0, code=0, x=at(0), codes=at(1), scales=at(2), T=4, d=40, ldx=40, ldc=40, lds=2)
    a.update(kw)
    B.hmy_k_unpack8(**a)


def norm(**kw):
    a = dict(prec=0, code=0, codes=at(0), scales=at(1), gamma=at(2), beta=at(3), y=at(4), mean=at(5), rstd=at(6), T=4, d=40, ldc=40, lds=2, ldy=40,
             eps=1e-5, x=at(7), ldx=40)
    a.update(kw)
    B.hmy_k_layernorm8_fwd(**a)


def norm_grad(**kw):
    a = dict(prec=0, code=0, dy=at(0), codes=at(1), scales=at(2), mean=at(3), rstd=at(4), gamma=at(5), dx=at(6), dgamma=at(7), dbeta=at(8), T=4, d=40,
             ldc=40, lds=2, ldy=40, ldx=40, res=at(9), ldr=40, dx_e=at(10), lde=40, dres_sum=at(11), workspace=at(12), workspace_bytes=1 << 20)
    a.update(kw)
    B.hmy_k_layernorm8_bwd(**a)


@pytest.mark.parametrize("call,bad", [
    *[(lookup, kw) for kw in (dict(ids=None), dict(table=None), dict(x=None), dict(T=0), dict(T=-3), dict(d=0), dict(d=(1 << 24) + 1, ldw=1 << 25, ldx=1 << 25, ldp=1 << 25),
                              dict(V=0), dict(P=-1), dict(P=0), dict(pos_table=None), dict(pos_table=None, P=0), dict(ldw=9), dict(ldx=9), dict(ldp=9), dict(ldx=-10),
                              dict(ldx=1 << 60), dict(prec=2), dict(out_prec=-1), dict(scale=NAN), dict(scale=INF), dict(ids=at(0) + 2), dict(positions=at(3) + 1),
                              dict(table=at(1) + 2), dict(x=at(2) + 2), dict(prec=1, table=at(1) + 1), dict(x=at(1)), dict(x=at(1) - 40), dict(x=at(4)), dict(x=at(0)), dict(x=at(3)))],
    *[(gradient, kw) for kw in (dict(ids=None), dict(dx=None), dict(dtable=None), dict(workspace=None), dict(T=0), dict(T=(1 << 24) + 1, workspace_bytes=1 << 40), dict(d=0),
                                dict(V=0), dict(V=2 ** 31 - 1), dict(ldx=9), dict(ldt=9), dict(ldt=1 << 60), dict(prec=2), dict(scale=NAN), dict(accumulate=2),
                                dict(ids=at(0) + 1), dict(dx=at(1) + 2), dict(dtable=at(2) + 2), dict(workspace=at(3) + 8), dict(workspace_bytes=65536 + 128 + 79),
                                dict(dtable=at(1)), dict(dtable=at(0) - 200), dict(dtable=at(3)), dict(workspace=at(1)), dict(workspace=at(0)),
                                dict(T=1 << 24, d=1 << 24, ldx=1 << 24, ldt=1 << 24, ids=1 << 52, dx=1 << 53, dtable=1 << 56, workspace=1 << 57, workspace_bytes=1 << 50))],
    *[(f, kw) for f in (pack, unpack) for kw in (dict(x=None), dict(codes=None), dict(scales=None), dict(T=0), dict(d=0), dict(ldx=39), dict(ldc=39), dict(lds=1), dict(lds=1 << 60),
                                                 dict(prec=2), dict(code=2), dict(code=-1), dict(x=at(0) + 2), dict(prec=1, x=at(0) + 1), dict(x=at(1)), dict(x=at(2)),
                                                 dict(d=(1 << 24) + 1, ldx=1 << 25, ldc=1 << 25, lds=1 << 25))],
    (pack, dict(codes=at(2) - 8)),
    *[(norm, kw) for kw in (dict(codes=None), dict(scales=None), dict(gamma=None), dict(beta=None), dict(y=None), dict(T=0), dict(d=0), dict(d=8193, ldc=9000, lds=300, ldy=9000, ldx=9000),
                            dict(ldc=39), dict(lds=1), dict(ldy=39), dict(ldx=39), dict(prec=5), dict(code=3), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF),
                            dict(gamma=at(2) + 2), dict(beta=at(3) + 2), dict(y=at(4) + 1), dict(mean=at(5) + 2), dict(rstd=at(6) + 1), dict(x=at(7) + 2), dict(y=at(0)), dict(x=at(4)),
                            dict(x=at(1)), dict(mean=at(6)), dict(y=at(2)), dict(rstd=at(4) + 16))],
    *[(norm_grad, kw) for kw in (dict(codes=None), dict(scales=None), dict(mean=None), dict(rstd=None), dict(gamma=None), dict(dy=None), dict(dx=None), dict(dgamma=None), dict(dbeta=None),
                                 dict(workspace=None), dict(T=0), dict(d=0), dict(d=8193, ldc=9000, lds=300, ldy=9000, ldx=9000, ldr=9000, lde=9000, workspace_bytes=1 << 30), dict(ldc=39), dict(lds=1), dict(ldy=39),
                                 dict(ldx=39), dict(ldr=39), dict(lde=39), dict(prec=2), dict(code=2), dict(accumulate=2), dict(res=None), dict(workspace_bytes=256 * 12 * 40 - 1),
                                 dict(workspace=at(12) + 4), dict(dx=at(6) + 2), dict(dy=at(0) + 1), dict(res=at(9) + 2), dict(dx_e=at(10) + 2), dict(gamma=at(5) + 2), dict(mean=at(3) + 2),
                                 dict(dgamma=at(7) + 1), dict(dx=at(0)), dict(dx=at(9), ldx=44), dict(dx=at(9) + 4), dict(dx_e=at(6)), dict(dx_e=at(0)), dict(dgamma=at(8)), dict(dres_sum=at(7)),
                                 dict(workspace=at(1)), dict(dbeta=at(12)), dict(dx=at(1)), dict(dgamma=at(5)))],
])
def test_refusals(call, bad):
    with pytest.raises(B.HmyError) as e:
        call(**bad)
    assert e.value.code == B.HMY_E_INVALID and len(str(e.value)) > 30


def test_no_description_at_all():
    for f in ("hmy_k_embed_lookup", "hmy_k_embed_grad", "hmy_k_pack8", "hmy_k_unpack8", "hmy_k_layernorm8_fwd", "hmy_k_layernorm8_bwd"):
        assert getattr(B.lib, f)(None, None) == B.HMY_E_INVALID


@pytest.mark.parametrize("call", [gradient, norm_grad])
def test_a_workspace_by_its_address_wants_its_size(call):
    with pytest.raises(B.HmyError, match="workspace_bytes") as e:
        call(workspace_bytes=None)
    assert e.value.code == B.HMY_E_INVALID


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_oracle_of_8_bits(code):
    """Every value is off by at most what the header says, every number of the format is read back as itself, scales are the least."""
    x = hard_groups("fp32").astype(np.float64)
    codes, scales = os_.pack8(x, code)
    v = os_.unpack8(codes, scales, code)
    fine = np.repeat(scales != 255, 32, 1)
    assert np.array_equal(np.isnan(v), ~fine)
    two = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, 1)
    step = 0.5 * two if code == "int8" else np.maximum(np.abs(x) * 2.0 ** -4, two * 2.0 ** -10)
    assert np.all(np.abs(v - x)[fine] <= step[fine])
    a = np.abs(x).reshape(len(x), -1, 32).max(2)
    ok = (scales != 255) & (scales > 1)
    assert np.all(a[ok] <= os_.TOP[code] * 2.0 ** (scales[ok] - 127.0)) and np.all(a[ok] > os_.TOP[code] * 2.0 ** (scales[ok] - 128.0))
    again = os_.pack8(np.where(fine, v, 0.0), code)
    assert np.array_equal(os_.unpack8(*again, code)[fine], v[fine])
    if code == "e4m3":
        bits = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
        np.testing.assert_array_equal(os_.numbers(code), bits)
        q = np.concatenate([x[23], x[24], -x[24]])
        np.testing.assert_array_equal(os_._nearest(q, code), torch.from_numpy(q).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_oracle_gradients_are_differences():
    rng = np.random.default_rng(3)
    T, d, V = 9, 12, 5
    v, gamma, beta, res, dy = rng.standard_normal((T, d)), rng.standard_normal(d), rng.standard_normal(d), rng.standard_normal((T, d)), rng.standard_normal((T, d))
    dv, dg, db = rng.standard_normal((T, d)), rng.standard_normal(d), rng.standard_normal(d)
    _, m, r = os_.layernorm(v, gamma, beta, EPS)
    dx, gg, gb, dr = os_.layernorm_grad(dy, v, m, r, gamma, res)
    f = lambda h: float((os_.layernorm(v + h * dv, gamma + h * dg, beta + h * db, EPS)[0] * dy).sum() + (res * (v + h * dv)).sum())
    h = 1e-6
    # a central difference: h^2 f''' / 6 and the rounding of f over h
    assert abs((f(h) - f(-h)) / (2 * h) - ((dx * dv).sum() + gg @ dg + gb @ db)) < 1e-7
    np.testing.assert_allclose(dr, res.sum(0), rtol=1e-15)
    ids, table, dt = rng.integers(-1, V + 1, T), rng.standard_normal((V, d)), rng.standard_normal((V, d))
    pos, dp = rng.standard_normal((4, d)), rng.standard_normal((4, d))
    places = rng.integers(-1, 5, T)
    g, p = os_.embed_grad(ids, dy, V, 1.5)[0], os_.embed_grad(places, dy, 4)[0]
    f = lambda h: float((os_.embed_lookup(ids, table + h * dt, 1.5, places, pos + h * dp) * dy).sum())
    assert abs((f(1.0) - f(-1.0)) / 2 - ((g * dt).sum() + (p * dp).sum())) < 1e-12   # linear
