"""Operators around the residual stream at the ends of what they accept: many rows, long runs, many rounds, rows side by side.

Bounds as in test_stream.py, but where a sum's depth is given here."""
import numpy as np
import pytest
import torch

from paper_2202_01306_amd import binding as B
from tests.test_stream import DT, PC, Norm, U, dx_bound, grad, gradient, host, i32, near, os_, rows_of, say


# ---- a table's gradient: tables of very many rows ----------------------------------------------------------

@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no memory: accepted calls would be launched")
@pytest.mark.parametrize("T", [1, 10, 256, 257, 300, 1024, 1025, 9000])
@pytest.mark.parametrize("V", [(1 << 30) + 100, 2 ** 31 - 2])
def test_tables_of_many_rows_are_accepted_whatever_the_number_of_tokens(T, V):
    """A call that passes all checks ends at the launch, for want of a device."""
    with pytest.raises(B.HmyError) as e:
        gradient(T=T, d=1, V=V, ldx=1, ldt=1, dtable=1 << 40)
    assert e.value.code != B.HMY_E_INVALID, str(e.value)


@pytest.mark.parametrize("T", [1, 256, 257, 1024, 9000])
def test_more_workgroups_than_a_launch_has_are_refused_whatever_the_number_of_tokens(T):
    """2^22 rows of 2^17 columns: four rows of 1024 columns a wave are 2^27 waves."""
    d, V = 1 << 17, 1 << 22
    with pytest.raises(B.HmyError, match="too large together") as e:
        gradient(T=T, d=d, V=V, ldx=d, ldt=d, dx=1 << 50, dtable=1 << 52, workspace=1 << 54, workspace_bytes=1 << 40)
    assert e.value.code == B.HMY_E_INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", [(256, (1 << 30) + 100), (10, 2 ** 31 - 2), (257, 2 ** 31 - 2)])
def test_tables_of_many_rows(T, V):
    """Every row written once: those that tokens name with their sums of whole numbers, all others with zeros."""
    say(f"grad T={T} V={V}")
    rng = np.random.default_rng(T)
    ids = rng.integers(0, V, T)
    ids[-7:] = V - 1, 0, -1, V - 1, V - 2, 1 << 30, 63
    dx = rng.integers(1, 9, (T, 1)).astype(np.float32)
    t = grad("fp32", i32(ids), rows_of(dx, 1, torch.float32), V, 1, 1, 1)
    named = np.unique(ids[ids >= 0])
    want = np.array([dx[ids == v].sum() for v in named], np.float32)
    assert torch.equal(t[torch.from_numpy(named).cuda(), 0].cpu(), torch.from_numpy(want))
    assert sum(int(p.count_nonzero()) for p in t.view(-1).split(1 << 28)) == len(named)


# ---- a table's gradient: long runs ----------------------------------------------------------------------------

# A term goes through at most 63 additions in its piece of the list and the one behind, 64 among the parts of its run, 64 among sums of 64
# parts, 32 among sums of 64 of those (2^24 tokens are 2^19 parts, a quarter of them a wave's), 2 and 3 more where these and the waves meet,
# and the scaling: 229 roundings, however long the run is.
LONG = 229


@pytest.mark.gpu
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,V,d", [(1 << 20, 1, 8), ((1 << 20) + 77, 2, 5), (1 << 22, 2, 8), (1 << 24, 1, 4), (1 << 24, 2, 8), ((1 << 24) - 1, 5, 3)])
def test_long_runs_of_terms_that_round_the_same_way(prec, accumulate, T, V, d):
    """Equal terms in a column, as of a bias: a rounding repeats itself instead of cancelling."""
    say(f"grad long {prec} T={T} V={V} d={d} accumulate={accumulate}")
    gen = torch.Generator(device="cuda").manual_seed(T + V)
    ids = torch.randint(0, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
    terms = torch.tensor([0.1, 0.9, 3.3, 0.7, 1 / 7, 1.1, 1 / 3, 0.013][:d], device="cuda").to(torch.float32 if prec == "fp32" else torch.bfloat16)
    dx = terms.expand(T, d).contiguous()
    into = torch.full((V, d), 2.5, device="cuda") if accumulate else torch.full((V, d), 7.0, device="cuda")
    ws = torch.full((B.HMY_EMBED_GRAD_WORKSPACE_BYTES(T, d),), 0xff, device="cuda", dtype=torch.uint8)
    B.hmy_k_embed_grad(PC[prec], ids, dx, into, T, d, V, d, d, scale=1.5, accumulate=accumulate, workspace=ws)
    n = torch.bincount(ids.long(), minlength=V).double().cpu().numpy()
    size = 1.5 * n[:, None] * terms.double().cpu().numpy()[None]
    want = size + 2.5 * accumulate
    off = np.abs(into.double().cpu().numpy() - want)
    bound = LONG * U * size + U * want
    assert np.all(off <= bound), float((off / bound).max())


# ---- layer norm of rows in 8 bits: several rounds of rows --------------------------------------------------------

def slots_of(d):
    """Rows that a workgroup of the backward pass has at a time."""
    return 8 // (1 if d <= 1024 else 2 if d <= 2048 else 4 if d <= 4096 else 8) * (8 if d <= 32 else 4 if d <= 64 else 2 if d <= 128 else 1)


@pytest.mark.gpu
@pytest.mark.parametrize("prec,code", [("fp32", "int8"), ("bf16", "e4m3")])
@pytest.mark.parametrize("T,d,ld,shift", [(3001, 1100, 1100, 0), (2500, 2048, 2051, 1), (1300, 2500, 2500, 0), (700, 4099, 4100, 3), (600, 8192, 8192, 0), (5001, 1023, 1023, 0),
                                          (40001, 24, 24, 0), (33000, 5, 6, 1), (20003, 50, 53, 2), (10001, 100, 100, 0)])
def test_layer_norm_backward_in_three_rounds_and_a_ragged_one(prec, code, T, d, ld, shift):
    """Rows fetched ahead, waves of a row that exchange sums round after round, sums carried from one round to the next."""
    say(f"norm8 rounds {prec} {code} T={T} d={d}")
    assert 2 * 256 * slots_of(d) < T and T % (256 * slots_of(d))
    n = Norm(prec, code, T, d, ld, shift)
    n.forward()
    n.check_forward()
    first = [t.clone() for t in n.backward()]
    n.check_backward()
    for a, b in zip(first, n.backward()):
        assert torch.equal(a, b)
    n.backward(in_place=True, accumulate=True, into=[torch.full((d,), 3.0, device="cuda") for _ in range(3)])
    n.check_backward(base=3.0)
    assert torch.equal(n.dx[:, :d], first[0][:, :d])
    n.backward(res=False, rounded_too=False)
    n.check_backward(res=False)


# ---- layer norm of rows in 8 bits: column sums over many rows --------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("prec,T,d,accumulate", [("fp32", 1 << 28, 8, False), ("bf16", (1 << 24) + 9, 24, True), ("bf16", 1 << 25, 100, False), ("bf16", (1 << 22) + 1, 300, True),
                                                 ("bf16", (1 << 20) + 3, 1100, False), ("fp32", (1 << 20) + 5, 2100, False), ("bf16", (1 << 20) + 3, 4100, True)])
def test_column_sums_over_rows_that_round_the_same_way(prec, T, d, accumulate):
    """Equal rows.  A term goes through at most 256 additions in a lane, one for each 256 of its rows, 3 between rows side by side, 8 between a
    workgroup's, 16 and 16 of the 256 partial sums; products with what the codes stand for are exact."""
    say(f"norm8 sums {prec} T={T} d={d} accumulate={accumulate}")
    dt = torch.float32 if prec == "fp32" else torch.bfloat16
    at = torch.arange(d, device="cuda")
    v = (at * 37 % 251 - 125).to(torch.int8)
    row = (0.1 + 0.8 * (at * 13 % 101) / 101).to(dt)
    with_res = d <= 24
    codes, dy = v.expand(T, d).contiguous(), row.expand(T, d).contiguous()
    scales = torch.full((T, (d + 31) // 32), 127, device="cuda", dtype=torch.uint8)
    mean, rstd = torch.zeros(T, device="cuda"), torch.ones(T, device="cuda")
    res = (row.float() + 0.3).expand(T, d).contiguous() if with_res else None
    dx = res if with_res else torch.empty(T, d, device="cuda")
    sums = [torch.full((d,), 2.5 if accumulate else 7.0, device="cuda") for _ in range(3)]
    r = (row.float() + 0.3).double().cpu().numpy()
    ws = torch.full((B.HMY_NORM8_WORKSPACE_BYTES(d),), 0xff, device="cuda", dtype=torch.uint8)
    B.hmy_k_layernorm8_bwd(PC[prec], B.HMY_CODE_INT8, dy, codes, scales, mean, rstd, torch.ones(d, device="cuda", dtype=dt), dx, sums[0], sums[1], T, d, d,
                           (d + 31) // 32, d, d, res=res, ldr=d, dres_sum=sums[2] if with_res else None, accumulate=accumulate, workspace=ws)
    y, x = row.double().cpu().numpy(), v.double().cpu().numpy()
    rounds = -(-T // (256 * slots_of(d)))
    n = 256 + -(-rounds // 256) + 3 + 8 + 32
    for t, terms in zip(sums, [y * x, y] + ([r] if with_res else [])):
        want = T * terms + 2.5 * accumulate
        off = np.abs(t.double().cpu().numpy() - want)
        bound = n * U * T * np.abs(terms) + U * np.abs(want)
        assert np.all(off <= bound), float((off[bound > 0] / bound[bound > 0]).max())


# ---- rows side by side in one array ----------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("T,d", [(50, 97), (300, 33), (70, 5), (40, 1025), (20, 2501), (30, 4099)])
def test_a_gradient_beside_the_gradient_that_it_reads(prec, T, d):
    """Layer norm backward with res and dx, and dy of fp32, as ranges of columns of one array; odd widths, whose last unit begins in the one before."""
    say(f"norm8 beside {prec} T={T} d={d}")
    n = Norm(prec, "int8", T, d, d)
    n.forward()
    ld = 3 * d + 11
    store = torch.full((T, ld), 7.0, device="cuda")
    res, dx = store[:, 3:], store[:, d + 3:]             # no column between them
    store[:, 3:d + 3] = torch.from_numpy(n.res).cuda()
    dy, ldy = (store[:, 2 * d + 6:], ld) if prec == "fp32" else (rows_of(n.dy, d, DT[prec]), d)
    dy[:, :d] = torch.from_numpy(n.dy).cuda()
    before = store.clone()
    sums = [torch.full((d,), 7.0, device="cuda") for _ in range(3)]
    ws = torch.full((B.HMY_NORM8_WORKSPACE_BYTES(d),), 0xff, device="cuda", dtype=torch.uint8)
    B.hmy_k_layernorm8_bwd(PC[prec], B.HMY_CODE_INT8, dy, n.codes, n.scales, n.mean, n.rstd, n.g, dx, sums[0], sums[1], T, d, d, n.G, ldy, ld, res=res, ldr=ld,
                           dres_sum=sums[2], workspace=ws)
    args = (n.dy.astype(np.float64), n.v, host(n.mean), host(n.rstd), n.gamma.astype(np.float64))
    ref = os_.layernorm_grad(*args, n.res.astype(np.float64))[0]
    near(host(dx[:, :d]), ref, dx_bound(*args, ref, n.res.astype(np.float64)))
    alone = n.backward()
    assert torch.equal(dx[:, :d], alone[0][:, :d]) and all(torch.equal(a, b) for a, b in zip(sums, n.sums))
    dx[:, :d] = 7.0
    assert torch.equal(store, before)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [60, 700, 1500, 9001])
@pytest.mark.parametrize("d", [3, 37, 261])
@pytest.mark.parametrize("accumulate", [False, True])
def test_a_tables_gradient_beside_the_rows_that_it_adds_up(T, d, accumulate):
    """dtable and dx as ranges of columns of one array."""
    say(f"grad beside T={T} d={d} accumulate={accumulate}")
    rng = np.random.default_rng(T + d)
    V = T // 3
    ids = rng.integers(-1, V + 1, T)
    ids[ids == 5] = 6                                    # a row that no token names
    dx = rng.integers(-9, 10, (T, d)).astype(np.float32)
    ld = 2 * d + 5
    store = torch.full((T, ld), 7.0, device="cuda")
    rows, table = store[:, 2:], store[:, d + 2:]
    rows[:, :d] = torch.from_numpy(dx).cuda()
    before = store.clone()
    grad("fp32", i32(ids), rows, V, d, ld, ld, scale=0.5, accumulate=accumulate, into=table)
    want, _, named = os_.embed_grad(ids, dx, V, 0.5)
    np.testing.assert_array_equal(host(table[:V, :d]), want + 7.0 * accumulate)   # whole numbers and halves: exact
    table[:V, :d] = 7.0
    assert torch.equal(store, before)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [3, 37, 400, 1601])
def test_rows_of_a_lookup_beside_the_rows_of_its_table(d):
    T, V = 90, 70
    rng = np.random.default_rng(d)
    values = rng.standard_normal((V, d)).astype(np.float32)
    ids = rng.integers(-1, V + 1, T)
    ld = 2 * d + 1
    store = torch.full((T, ld), 7.0, device="cuda")
    store[:V, :d] = torch.from_numpy(values).cuda()
    before = store.clone()
    x = store[:, d:]
    B.hmy_k_embed_lookup(0, 0, i32(ids), store, x, T, d, V, ld, ld, scale=2.0)
    np.testing.assert_array_equal(host(x[:, :d]), os_.embed_lookup(ids, values, 2.0))
    x[:, :d] = 7.0
    assert torch.equal(store, before)


# ---- offsets beyond 32 bits, the longest lists -------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("prec,out,T,d,ldx", [("bf16", "bf16", (1 << 20) + 3, 4096, 4096), ("fp32", "fp32", (1 << 20) + 1, 1025, 4100), ("bf16", "fp32", (1 << 30) + 5, 16, 16)])
def test_rows_of_a_lookup_beyond_32_bits(prec, out, T, d, ldx):
    """2^32 elements and more, with as many units of a lane in the last one."""
    say(f"lookup far {prec} {out} T={T} d={d}")
    V = 251
    table = torch.randn(V, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(d)).to(DT[prec])
    ids = torch.arange(T, device="cuda", dtype=torch.int32) % (V + 2) - 1   # none, 0 .. V - 1, none
    x = torch.full((T, ldx), 7.0, device="cuda", dtype=DT[out])
    B.hmy_k_embed_lookup(PC[prec], PC[out], ids, table, x, T, d, V, d, ldx, scale=0.25)
    zero = torch.zeros(1, d, device="cuda", dtype=DT[prec])
    want = (torch.cat([zero, table, zero]).float() * 0.25).to(DT[out])      # a power of two: exact
    step = (V + 2) * max(1, (1 << 26) // ((V + 2) * d))
    for r in range(0, T, step):
        part = x[r:r + step]
        assert torch.equal(part[:, :d], want.repeat(step // (V + 2), 1)[:len(part)])
        assert ldx == d or torch.all(part[:, d:] == 7.0)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,ldx", [(600, 64, 1 << 23), (8000, 64, (1 << 20) + 1), (70001, 64, 65600), (70001, 640, 65600)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_rows_that_a_gradient_adds_up_beyond_32_bits(T, d, ldx, accumulate):
    """Rows far apart: in one launch, ranked, sorted, and by streaming loads."""
    say(f"grad far T={T} d={d} accumulate={accumulate}")
    V = 90
    gen = torch.Generator(device="cuda").manual_seed(T + d)
    dx = torch.full((T, ldx), 99.0, device="cuda", dtype=torch.bfloat16)
    dx[:, :d] = torch.randint(-9, 10, (T, d), device="cuda", generator=gen).bfloat16()
    ids = torch.randint(-1, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
    into = torch.full((V, d), 3.0, device="cuda")
    ws = torch.full((B.HMY_EMBED_GRAD_WORKSPACE_BYTES(T, d),), 0xff, device="cuda", dtype=torch.uint8)
    B.hmy_k_embed_grad(1, ids, dx, into, T, d, V, ldx, d, accumulate=accumulate, workspace=ws)
    x, at = host(dx[:, :d]), ids.cpu().numpy()
    want = np.stack([x[at == v].sum(0) for v in range(V)]) + 3.0 * accumulate   # whole numbers below 2^24
    np.testing.assert_array_equal(host(into), want)


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,d", [(B.HMY_MAX_SORTED, 100000, 2), (B.HMY_MAX_SORTED - 3, 200, 3), (1 << 22, 2 ** 31 - 2, 1), ((1 << 23) + 1023, 1 << 24, 1)])
def test_gradient_of_the_longest_lists(T, V, d):
    """Up to 2^24 tokens, one to four passes of the sort: whole numbers, whose sums fp32 holds."""
    say(f"grad T={T} V={V} d={d}")
    gen = torch.Generator(device="cuda").manual_seed(V % 1000)
    rank = torch.exp(torch.rand(T, device="cuda", generator=gen, dtype=torch.float64) * np.log(V + 1.0)).long().sub_(1).clamp_(0, V - 1)
    ids = ((rank * 7919 + 17) % V).to(torch.int32)                          # spread over the table
    ids[5::50] = -1
    ids[-1] = V - 1
    dx = torch.randint(-4, 5, (T, d), device="cuda", generator=gen).float()
    t = torch.full((V, d), 7.0, device="cuda")
    ws = torch.full((B.HMY_EMBED_GRAD_WORKSPACE_BYTES(T, d),), 0xff, device="cuda", dtype=torch.uint8)
    B.hmy_k_embed_grad(0, ids, dx, t, T, d, V, d, d, workspace=ws)
    at, x = ids.cpu().numpy(), host(dx)
    named, inverse = np.unique(at[at >= 0], return_inverse=True)
    rows = torch.from_numpy(named).cuda()
    for c in range(d):
        np.testing.assert_array_equal(host(t[rows, c]), np.bincount(inverse, weights=x[at >= 0, c], minlength=len(named)))
    t[rows] = 0.0
    assert all(int(p.count_nonzero()) == 0 for p in t.view(-1).split(1 << 28))
