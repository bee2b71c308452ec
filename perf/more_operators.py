"""Performance cases of the operators around the residual stream, through the single-kernel entry points.

The stream's rows [T, d]: what goes into them, what is kept of them for the backward pass, and what reads it there.

  lookup     rows of a table by token, scaled, with rows of positions added
  grad       the gradient of a table: rows of the stream's gradient added up by token
  pack8      rows in 8 bits, a power of two for each 32 columns
  unpack8    and back
  norm8      layer norm of rows that are held in 8 bits, with the rows themselves for the residual connection
  norm8_bwd  its backward pass, with the reductions over rows

`own` false: their plain form in torch; true: the framework's kernels.  `listed()` names the cases, `draw()` gives more
of the same ranges.
"""
import math

import numpy as np
import torch
import torch.nn.functional as F

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
PREC = {"fp32": 0, "bf16": 1}
BYTES = {"fp32": 4, "bf16": 2}
CODES = {"int8": 0, "e4m3": 1}
GROUP = 32
EPS = 1e-5


def _lookup(name, T, d, V, table, out, scale, positions):
    return dict(name=name, kind="lookup", T=T, d=d, V=V, table=table, out=out, scale=scale, positions=positions, ld=d)


def _grad(name, T, d, V, dx, scale, parts):
    return dict(name=name, kind="grad", T=T, d=d, V=V, dx=dx, scale=scale, parts=parts, ld=d)


def _rows8(kind, name, T, d, code, rows, ld):
    return dict(name=name, kind=kind, T=T, d=d, code=code, rows=rows, ld=ld)


def _norm8(name, T, d, code, prec, keep_x):
    return dict(name=name, kind="norm8", T=T, d=d, code=code, prec=prec, keep_x=keep_x, ld=d)


def _norm8_bwd(name, T, d, code, prec, res, rounded, ld, parts):
    return dict(name=name, kind="norm8_bwd", T=T, d=d, code=code, prec=prec, res=res, rounded=rounded, ld=ld, parts=parts)


def listed():
    return [
        # one short sequence of the tiny decoder: nothing but latency
        _lookup("lookup_tiny", 64, 128, 512, "fp32", "fp32", 1.0, 64),
        # the benchmark workload's minibatch, its table times the root of its width, sequences with padding behind them
        _lookup("lookup_minibatch", 32768, 1024, 50257, "bf16", "fp32", 32.0, 1024),
        # two microbatches of the benchmark workload: the first writes the table's gradient, the second adds to it
        _grad("grad_two_microbatches", 4096, 1024, 50257, "fp32", 1.0, 2),
        # the encoder workload's whole minibatch in one call: the most tokens, the longest runs of one token
        _grad("grad_minibatch", 131072, 1024, 30522, "fp32", 1.0, 1),
        # a tiny microbatch's checkpoint
        _rows8("pack8", "pack8_tiny", 128, 128, "int8", "fp32", 128),
        # the largest decoder's minibatch as a checkpoint: the most work
        _rows8("pack8", "pack8_wide_minibatch", 32768, 4096, "int8", "fp32", 4096),
        # an odd width in rows without any alignment, 8-bit floats, for bf16 products
        _rows8("unpack8", "unpack8_odd", 5003, 1601, "e4m3", "bf16", 1603),
        # the benchmark workload's minibatch read back
        _rows8("unpack8", "unpack8_minibatch", 32768, 1024, "int8", "fp32", 1024),
        # one sequence of the tiny decoder
        _norm8("norm8_tiny", 64, 128, "int8", "fp32", True),
        # one microbatch of the benchmark workload: where a block's recomputation starts
        _norm8("norm8_microbatch", 4096, 1024, "int8", "bf16", True),
        # the same microbatch backward, with everything that a block wants of it
        _norm8_bwd("norm8_bwd_microbatch", 4096, 1024, "int8", "bf16", True, True, 1024, 1),
        # wide rows, an odd number of them, in two parts that add to one gradient
        _norm8_bwd("norm8_bwd_wide", 8191, 4096, "e4m3", "bf16", True, False, 4096, 2),
    ]


def draw(rng):
    """Rows from 1 to 131072, widths from 24 to 8192, tables of 64 to 100000 rows, products up to the benchmark workload's minibatch."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = 32768 * 1024
    kind = rng.choice(["lookup", "grad", "pack8", "unpack8", "norm8", "norm8_bwd"])
    d = spread(24, 8192)
    if rng.random() < 0.6:
        d = (d + 31) // 32 * 32
    T = spread(1, min(131072, most // d))
    ld = rng.choice([d, d, (d + 63) // 64 * 64, d + rng.randrange(1, 20)])
    c = dict(kind=kind, T=T, d=d, ld=ld)
    prec = rng.choice(["fp32", "bf16"])
    if kind in ("lookup", "grad"):
        c["V"] = spread(64, min(100000, 50257 * 1024 // d))
        c["scale"] = rng.choice([1.0, math.sqrt(d), 0.5])
    else:
        c["code"] = rng.choice(["int8", "e4m3"])
    if kind == "lookup":
        c.update(table=prec, out=rng.choice(["fp32", prec]), positions=rng.choice([0, spread(1, 4096)]))
    elif kind == "grad":
        c.update(dx=prec, parts=rng.choice([1, 2]))
    elif kind in ("pack8", "unpack8"):
        c["rows"] = prec
    elif kind == "norm8":
        c.update(prec=prec, keep_x=rng.random() < 0.5)
    else:
        c.update(prec=prec, res=rng.random() < 0.7, rounded=prec == "bf16" and rng.random() < 0.7, parts=rng.choice([1, 2]))
    return c


# ---- what a program has in hand ------------------------------------------------------------

class _State:
    pass


def _groups(d):
    return (d + GROUP - 1) // GROUP


def _chances(V):
    """Of the tokens by rank: token r about 1 / r as often as the first, as in text."""
    return np.diff(np.log(np.arange(1, V + 2)) / math.log(V + 1))


def prepare(case, seed):
    s = _State()
    s.case = case
    kind, T, d, ld = case["kind"], case["T"], case["d"], case["ld"]
    s.T, s.d, s.ld, s.G = T, d, ld, _groups(d)
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 13)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    uniform = lambda *shape: torch.rand(*shape, device="cuda", generator=g)

    def rows(values, dtype):
        """[T, ld] of which the first d columns are the values."""
        t = torch.zeros(T, ld, device="cuda", dtype=dtype)
        t[:, :d] = values
        return t

    def stream():
        """The residual stream as a trained model has it: rows of different size, a few columns that stand out."""
        x = normal(T, d).mul_(0.5 + 2.0 * uniform(T, 1)).add_(0.1)
        x *= torch.where(uniform(d) < 0.01, 30.0, 1.0)
        return x

    if kind in ("lookup", "grad"):
        V = s.V = case["V"]
        s.scale, s.parts = case["scale"], case.get("parts", 1)
        n = T * s.parts
        rank = torch.exp(uniform(n) * math.log(V + 1)).long().sub_(1).clamp_(0, V - 1)
        ids = torch.randperm(V, device="cuda", generator=g)[rank].to(torch.int32)
        if n >= 32:
            ids[uniform(n) < 0.02] = -1           # padding behind sequences
        s.ids = ids
    if kind == "lookup":
        s.table = normal(V, d).mul_(0.02).to(DTYPES[case["table"]])
        s.P = case["positions"]
        s.pos_table = normal(s.P, d).mul_(0.02).to(DTYPES[case["table"]]) if s.P else None
        # sequences packed one behind the other: positions start again wherever one ends, padding has none
        at = torch.arange(T, device="cuda") - 7
        s.positions = torch.where(s.ids >= 0, at % max(1, s.P), -1).to(torch.int32) if s.P else None
        s.x = torch.zeros(T, ld, device="cuda", dtype=DTYPES[case["out"]])
    elif kind == "grad":
        s.dx = [rows(normal(T, d).mul_(1e-3), DTYPES[case["dx"]]) for _ in range(s.parts)]
        s.part_ids = [s.ids[p * T:(p + 1) * T].clone() for p in range(s.parts)]
        s.dtable = torch.zeros(V, d, device="cuda")
        s.workspace = torch.empty(65536 + 32 * T + 8 * d * ((T + 15) // 16), dtype=torch.uint8, device="cuda")
    else:
        s.code = case["code"]
        s.codes = torch.zeros(T, ld, device="cuda", dtype=torch.uint8)
        s.scales = torch.zeros(T, s.G, device="cuda", dtype=torch.uint8)
    if kind == "pack8":
        s.x = rows(stream(), DTYPES[case["rows"]])
    if kind in ("unpack8", "norm8", "norm8_bwd"):
        for r in range(0, T, 8192):
            part = normal(min(8192, T - r), d).mul_(0.5 + 2.0 * uniform(min(8192, T - r), 1)).add_(0.1)
            part[:, ::97] *= 30.0
            codes, scales = _plain_codes(part, s.code)
            s.codes[r:r + 8192, :d], s.scales[r:r + 8192] = codes, scales
    if kind == "unpack8":
        s.x = torch.zeros(T, ld, device="cuda", dtype=DTYPES[case["rows"]])
    if kind in ("norm8", "norm8_bwd"):
        E = DTYPES[case["prec"]]
        s.gamma, s.beta = (normal(d).mul_(0.2).add_(1.0)).to(E), normal(d).mul_(0.1).to(E)
        s.mean, s.rstd = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    if kind == "norm8":
        s.y = torch.zeros(T, ld, device="cuda", dtype=E)
        s.x = torch.zeros(T, ld, device="cuda") if case["keep_x"] else None
    if kind == "norm8_bwd":
        s.parts = min(case["parts"], T)
        for r in range(0, T, 8192):                # what the forward pass left
            x = _values64(s, r, r + 8192)
            m = x.mean(1)
            s.mean[r:r + 8192] = m.float()
            s.rstd[r:r + 8192] = torch.rsqrt((x - m[:, None]).square().mean(1) + EPS).float()
        s.dy = rows(normal(T, d).mul_(1e-2), E)
        s.res = rows(normal(T, d).mul_(1e-2).add_(1e-3), torch.float32) if case["res"] else None
        s.dx = torch.zeros(T, ld, device="cuda")
        s.dx_e = torch.zeros(T, ld, device="cuda", dtype=E) if case["rounded"] else None
        s.dgamma, s.dbeta = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
        s.dres_sum = torch.zeros(d, device="cuda") if case["res"] else None
        s.workspace = torch.empty(256 * 3 * d, device="cuda")
    return s


def _cuts(s):
    """The parts that a minibatch's rows are worked through in."""
    edges = [s.T * p // s.parts for p in range(s.parts + 1)]
    return list(zip(edges[:-1], edges[1:]))


# ---- the plain forms -------------------------------------------------------------------------

def _plain_lookup(s):
    named = (s.ids >= 0) & (s.ids < s.V)
    x = torch.where(named[:, None], s.table[s.ids.long().clamp(0, s.V - 1)].float() * s.scale, 0.0)
    if s.P:
        placed = (s.positions >= 0) & (s.positions < s.P)
        x = x + torch.where(placed[:, None], s.pos_table[s.positions.long().clamp(0, s.P - 1)].float(), 0.0)
    s.x[:, :s.d] = x.to(s.x.dtype)
    return [s.x]


def _plain_grad(s):
    s.dtable.zero_()
    for ids, dx in zip(s.part_ids, s.dx):
        named = (ids >= 0) & (ids < s.V)
        part = torch.where(named[:, None], dx[:, :s.d].float() * s.scale, 0.0)
        s.dtable.index_add_(0, ids.long().clamp(0, s.V - 1), part)
    return [s.dtable]


def _plain_codes(x, code):
    """Rows in fp32 -> codes [T, d] and scales [T, groups], as bytes."""
    T, d = x.shape
    x = F.pad(x, (0, _groups(d) * GROUP - d)).view(T, -1, GROUP)
    a = x.abs().amax(2)
    part, power = torch.frexp(a)                   # a = part 2^power, part in [1/2, 1)
    if code == "int8":                             # the least e with a <= 127 2^e
        e = power - torch.where(part <= 127 / 128, 7, 6)
    else:                                          # a <= 448 2^e
        e = power - torch.where(part <= 448 / 512, 9, 8)
    e = e.clamp(min=-126)
    q = torch.ldexp(x, -e[:, :, None])
    fine = torch.isfinite(a)
    q = torch.where(fine[:, :, None], q, 0.0)
    q = torch.round(q).to(torch.int8).view(torch.uint8) if code == "int8" else q.to(torch.float8_e4m3fn).view(torch.uint8)
    return q.view(T, -1)[:, :d], torch.where(fine, e + 127, 255).to(torch.uint8)


def _plain_values(codes, scales, code, d):
    q = codes[:, :d].contiguous().view(torch.int8 if code == "int8" else torch.float8_e4m3fn).float()
    two = torch.where(scales == 255, math.nan, torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127))
    return q * two.repeat_interleave(GROUP, 1)[:, :d]


def _as_held(s):
    """The codes as the numbers that they are, in units of their group's scale."""
    return s.codes.view(torch.int8 if s.code == "int8" else torch.float8_e4m3fn)


def _plain_pack8(s):
    codes, s.scales[:] = _plain_codes(s.x[:, :s.d].float(), s.code)
    s.codes[:, :s.d] = codes
    return [_as_held(s), s.scales]


def _plain_unpack8(s):
    s.x[:, :s.d] = _plain_values(s.codes, s.scales, s.code, s.d).to(s.x.dtype)
    return [s.x]


def _plain_norm8(s):
    x = _plain_values(s.codes, s.scales, s.code, s.d)
    m = x.mean(1)
    c = x - m[:, None]
    r = torch.rsqrt(c.square().mean(1) + EPS)
    s.y[:, :s.d] = (s.gamma.float() * (c * r[:, None]) + s.beta.float()).to(s.y.dtype)
    s.mean[:], s.rstd[:] = m, r
    if s.x is None:
        return [s.y, s.mean, s.rstd]
    s.x[:, :s.d] = x
    return [s.y, s.mean, s.rstd, s.x]


def _bwd_outputs(s):
    return [t for t in (s.dx, s.dgamma, s.dbeta, s.dx_e, s.dres_sum) if t is not None]


def _plain_norm8_bwd(s):
    d = s.d
    s.dgamma.zero_(), s.dbeta.zero_()
    for a, b in _cuts(s):
        xh = (_plain_values(s.codes[a:b], s.scales[a:b], s.code, d) - s.mean[a:b, None]) * s.rstd[a:b, None]
        dy = s.dy[a:b, :d].float()
        g = dy * s.gamma.float()
        dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * s.rstd[a:b, None]
        if s.res is not None:
            dx = dx + s.res[a:b, :d]
        s.dx[a:b, :d] = dx
        if s.dx_e is not None:
            s.dx_e[a:b, :d] = dx.to(s.dx_e.dtype)
        s.dgamma += (dy * xh).sum(0)
        s.dbeta += dy.sum(0)
    if s.res is not None:
        s.dres_sum[:] = s.res[:, :d].sum(0)
    return _bwd_outputs(s)


# ---- the framework's calls ---------------------------------------------------------------------

def _own_lookup(s):
    from paper_2202_01306_amd import binding as B
    B.hmy_k_embed_lookup(PREC[s.case["table"]], PREC[s.case["out"]], s.ids, s.table, s.x, s.T, s.d, s.V, s.d, s.ld, scale=s.scale,
                         positions=s.positions, pos_table=s.pos_table, P=s.P, ldp=s.d)
    return [s.x]


def _own_grad(s):
    from paper_2202_01306_amd import binding as B
    for p in range(s.parts):
        B.hmy_k_embed_grad(PREC[s.case["dx"]], s.part_ids[p], s.dx[p], s.dtable, s.T, s.d, s.V, s.ld, s.d, scale=s.scale,
                           accumulate=p > 0, workspace=s.workspace)
    return [s.dtable]


def _own_pack8(s):
    from paper_2202_01306_amd import binding as B
    B.hmy_k_pack8(PREC[s.case["rows"]], CODES[s.code], s.x, s.codes, s.scales, s.T, s.d, s.ld, s.ld, s.G)
    return [_as_held(s), s.scales]


def _own_unpack8(s):
    from paper_2202_01306_amd import binding as B
    B.hmy_k_unpack8(PREC[s.case["rows"]], CODES[s.code], s.codes, s.scales, s.x, s.T, s.d, s.ld, s.G, s.ld)
    return [s.x]


def _own_norm8(s):
    from paper_2202_01306_amd import binding as B
    B.hmy_k_layernorm8_fwd(PREC[s.case["prec"]], CODES[s.code], s.codes, s.scales, s.gamma, s.beta, s.y, s.mean, s.rstd, s.T, s.d,
                           s.ld, s.G, s.ld, EPS, x=s.x, ldx=s.ld)
    return [s.y, s.mean, s.rstd] + ([] if s.x is None else [s.x])


def _own_norm8_bwd(s):
    from paper_2202_01306_amd import binding as B
    part = lambda t, a, b: None if t is None else t[a:b]
    for a, b in _cuts(s):
        B.hmy_k_layernorm8_bwd(PREC[s.case["prec"]], CODES[s.code], s.dy[a:b], s.codes[a:b], s.scales[a:b], s.mean[a:b], s.rstd[a:b],
                               s.gamma, s.dx[a:b], s.dgamma, s.dbeta, b - a, s.d, s.ld, s.G, s.ld, s.ld, res=part(s.res, a, b), ldr=s.ld,
                               dx_e=part(s.dx_e, a, b), lde=s.ld, dres_sum=s.dres_sum, accumulate=a > 0, workspace=s.workspace)
    return _bwd_outputs(s)


_PLAIN = dict(lookup=_plain_lookup, grad=_plain_grad, pack8=_plain_pack8, unpack8=_plain_unpack8, norm8=_plain_norm8,
              norm8_bwd=_plain_norm8_bwd)
_OWN = dict(lookup=_own_lookup, grad=_own_grad, pack8=_own_pack8, unpack8=_own_unpack8, norm8=_own_norm8, norm8_bwd=_own_norm8_bwd)


def run(state):
    return (_OWN if own else _PLAIN)[state.case["kind"]](state)


def work(case):
    kind, T, d = case["kind"], case["T"], case["d"]
    n = T * d
    if kind in ("lookup", "grad"):
        distinct = float((1.0 - (1.0 - _chances(case["V"])) ** T).sum())     # rows of the table that T tokens name
    if kind == "lookup":
        E = BYTES[case["table"]]
        places = min(T, case["positions"])
        return {"bytes": n * BYTES[case["out"]] + (distinct + places) * d * E + 4 * T * (2 if places else 1), "flops": 2.0 * n}
    if kind == "grad":
        # every part reads its rows; the first writes the whole table, the others read and write the rows that they name
        later = case["parts"] - 1
        return {"bytes": case["parts"] * (n * BYTES[case["dx"]] + 4 * T) + (case["V"] + 2 * later * distinct) * d * 4,
                "flops": 2.0 * n * case["parts"]}
    held = n + T * _groups(d)
    if kind in ("pack8", "unpack8"):
        return {"bytes": held + n * BYTES[case["rows"]], "flops": 3.0 * n}
    E = BYTES[case["prec"]]
    if kind == "norm8":
        return {"bytes": held + n * (E + (4 if case["keep_x"] else 0)) + 8 * T, "flops": 8.0 * n}
    return {"bytes": held + n * (E + 4 + (4 if case["res"] else 0) + (E if case["rounded"] else 0)) + 8 * T, "flops": 14.0 * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _exact_lookup(s):
    out = torch.zeros(s.T, s.ld, device="cuda", dtype=torch.float64)
    has = torch.nonzero((s.ids >= 0) & (s.ids < s.V)).squeeze(1)
    out[has, :s.d] = s.scale * s.table.double()[s.ids[has].long()]
    if s.P:
        has = torch.nonzero((s.positions >= 0) & (s.positions < s.P)).squeeze(1)
        out[has, :s.d] += s.pos_table.double()[s.positions[has].long()]
    return [out]


def _exact_grad(s):
    out = torch.zeros(s.V, s.d, device="cuda", dtype=torch.float64)
    for ids, dx in zip(s.part_ids, s.dx):
        for r in range(0, s.T, 16384):
            has = torch.nonzero((ids[r:r + 16384] >= 0) & (ids[r:r + 16384] < s.V)).squeeze(1) + r
            out.index_put_((ids[has].long(),), dx[has, :s.d].double() * s.scale, accumulate=True)
    return [out]


def _values64(s, r, e):
    """Rows r .. e as their codes and scales say, each code looked up in its format's table."""
    bits = torch.arange(256, device="cuda")
    if s.code == "int8":
        table = torch.where(bits < 128, bits, bits - 256).double()
    else:                                          # sign, four bits of exponent around 7, three of mantissa; all ones: no number
        sign, power, part = 1.0 - 2.0 * (bits >> 7), bits >> 3 & 15, (bits & 7).double()
        table = sign * torch.where(power == 0, part / 8 * 2.0 ** -6, (1 + part / 8) * 2.0 ** (power - 7).double())
        table[(bits & 127) == 127] = math.nan
    two = 2.0 ** (s.scales[r:e].double() - 127)
    return table[s.codes[r:e, :s.d].long()] * two[:, torch.arange(s.d, device="cuda") // GROUP]


def _exact_pack8(s):
    x = s.x[:, :s.d].double()
    top = 127.0 if s.code == "int8" else 448.0
    held = torch.zeros(s.T, s.ld, device="cuda", dtype=torch.float32)
    for i in range(s.G):
        part = x[:, i * GROUP:(i + 1) * GROUP]
        a = part.abs().amax(1)
        e = torch.ceil(torch.log2(torch.where(a > 0, a / top, 2.0 ** -126))).clamp(min=-126)
        e = torch.where(a > top * 2.0 ** e, e + 1, e)
        q = part / (2.0 ** e)[:, None]
        if s.code == "int8":
            q = torch.round(q)
        else:
            step = 2.0 ** (torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
            q = torch.round(q / step) * step
        held[:, i * GROUP:i * GROUP + part.shape[1]] = q.float()
    return [held.to(torch.int8) if s.code == "int8" else held, None]


def _exact_unpack8(s):
    out = torch.zeros(s.T, s.ld, device="cuda", dtype=torch.float64)
    for r in range(0, s.T, 8192):
        out[r:r + 8192, :s.d] = _values64(s, r, r + 8192)
    return [out]


def _exact_norm8(s):
    y, held = (torch.zeros(s.T, s.ld, device="cuda", dtype=torch.float64) for _ in range(2))
    mean, rstd = (torch.zeros(s.T, device="cuda", dtype=torch.float64) for _ in range(2))
    for r in range(0, s.T, 8192):
        x = _values64(s, r, r + 8192)
        held[r:r + 8192, :s.d] = x
        var, m = torch.var_mean(x, 1, correction=0)
        mean[r:r + 8192], rstd[r:r + 8192] = m, (var + EPS) ** -0.5
        y[r:r + 8192, :s.d] = s.gamma.double() * (x - m[:, None]) / torch.sqrt(var + EPS)[:, None] + s.beta.double()
    return [y, mean, rstd] + ([] if s.x is None else [held])


def _exact_norm8_bwd(s):
    dx = torch.zeros(s.T, s.ld, device="cuda", dtype=torch.float64)
    dgamma, dbeta, dres = (torch.zeros(s.d, device="cuda", dtype=torch.float64) for _ in range(3))
    for r in range(0, s.T, 4096):
        e = r + 4096
        xh = (_values64(s, r, e) - s.mean[r:e, None].double()) * s.rstd[r:e, None].double()
        dy = s.dy[r:e, :s.d].double()
        dxh = dy * s.gamma.double()
        lean = (dxh @ torch.ones(s.d, 1, device="cuda", dtype=torch.float64) + xh * (dxh * xh).sum(1, keepdim=True)) / s.d
        dx[r:e, :s.d] = s.rstd[r:e, None].double() * (dxh - lean)
        if s.res is not None:
            dx[r:e, :s.d] += s.res[r:e, :s.d].double()
            dres += s.res[r:e, :s.d].double().sum(0)
        dgamma += (dy * xh).sum(0)
        dbeta += dy.sum(0)
    return [dx, dgamma, dbeta] + ([dx] if s.dx_e is not None else []) + ([dres] if s.res is not None else [])


_EXACT = dict(lookup=_exact_lookup, grad=_exact_grad, pack8=_exact_pack8, unpack8=_exact_unpack8, norm8=_exact_norm8,
              norm8_bwd=_exact_norm8_bwd)


def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["kind"]](s)
