"""Performance cases of the operators at the two ends of the vocabulary: what turns hidden states into
the sampler's logits, what turns its tokens into the next step's input, and how the table that both
read is trained and refreshed.

A case is a plain dict; ``op`` names the operator, the other fields its sizes and types:

  head   logits[T, V] = h[T, H] . W[V, H]^T, W held in 4 bits with a scale for each group of columns
         (T hidden rows of type ``h``, logits of type ``out``)
  embed  out[t] = scale * W[token[t]], a row of zeros for a token outside the vocabulary; ``table``
         is bf16, f32, or w4 (the 4-bit table of the head)
  grad   dW[v] = scale * sum of dout[t] over the t with token[t] = v, all V rows (``h`` the type of
         dout, ``out`` the type of dW)
  quant  the 4-bit form of a table W of type ``h``, returned as the values it stands for, type ``out``

The 4-bit table.  Rows are split into blocks of 128 columns (the last one filled up), a block into 16
dwords; dword 4 g + j holds columns 32 j + 8 g .. + 7 of the block, element e = 0..7.
  fmt int  integers -7..7 with a bfloat16 scale for each ``group`` columns.  With bytes s0000mmm (sign,
           magnitude), A those of elements 0..3 and B of 4..7, lowest byte first: A | rotl32(B, 4)
  fmt mx   E2M1 numbers (element e in bits 4 e .. 4 e + 3) with a scale 2^(x - 127), x one byte, for
           each 32 columns
Scales are [V, blocks * 128 / group], also filled up.
"""
from __future__ import annotations

import math

import torch

own = False

SCALE = 1.25  # of lookups and their gradients: exact in every type
PAD = 0.1     # share of positions without a token (id -1), as padded batches and rejected drafts have


def listed():
    def head(name, T, V, H, fmt, group, h="bf16", out="bf16"):
        return dict(name=name, op="head", T=T, V=V, H=H, fmt=fmt, group=group, h=h, out=out)

    def embed(name, T, V, H, table, out="bf16", fmt="int", group=128):
        return dict(name=name, op="embed", T=T, V=V, H=H, table=table, out=out, fmt=fmt, group=group)

    def grad(name, T, V, H, h, out):
        return dict(name=name, op="grad", T=T, V=V, H=H, h=h, out=out)

    def quant(name, V, H, fmt, group, h="bf16", out="bf16"):
        return dict(name=name, op="quant", V=V, H=H, fmt=fmt, group=group, h=h, out=out)

    return [
        # one user, a small model: latency
        head("head_t1_int", 1, 32768, 2048, "int", 128),
        # a few users, float32 hidden states and logits
        head("head_t4_f32_int", 4, 32768, 4096, "int", 64, "f32", "f32"),
        # a decode step over a large vocabulary
        head("head_t16_mx", 16, 262144, 8192, "mx", 32),
        # a vocabulary that is not padded, small groups, a number of requests that fills no tile
        head("head_odd_t37_int", 37, 200003, 2880, "int", 32),
        # a decode step of a serving batch
        head("head_t64_int", 64, 131072, 4096, "int", 128),
        # the target rows of a verification, 64 requests of four drafts each
        head("head_t320_mx", 320, 131072, 4096, "mx", 32),
        # the tokens of a verification step: latency
        embed("embed_t320_bf16", 320, 131072, 4096, "bf16"),
        # the prompts of a batch, from the table that the head reads
        embed("embed_t8192_w4", 8192, 131072, 4096, "w4"),
        # a small model's training step
        grad("grad_t2048_f32", 2048, 32768, 2048, "f32", "f32"),
        # an ordinary training step: tokens by Zipf's law, padding among them
        grad("grad_t16384_bf16", 16384, 131072, 4096, "bf16", "f32"),
        # the serving table refreshed from the trained one
        quant("quant_int_bf16", 131072, 4096, "int", 128),
        quant("quant_mx_f32", 32768, 2048, "mx", 32, "f32", "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["head", "head", "head", "embed", "grad", "quant"])
    fmt = rng.choice(["int", "mx"])
    group = 32 if fmt == "mx" else rng.choice([32, 64, 128])
    step = max(group, rng.choice([32, 128, 128, 128]))
    H = max(1024, _log_int(rng, 1024, 8192) // step * step)
    V = _log_int(rng, 32000, 262144)
    V = rng.choice([V, V | 1, (V + 63) // 64 * 64])
    t = lambda *k: rng.choice(k)  # noqa: E731
    if op == "head":
        h = t("bf16", "bf16", "f32")
        T = _log_int(rng, 1, 320 if h == "bf16" else 64)
        while T * V * H > 320 * 131072 * 4096 / 2:
            T = (T + 1) // 2
        return dict(op=op, T=T, V=V, H=H, fmt=fmt, group=group, h=h, out=t("bf16", "f32"))
    if op == "embed":
        return dict(op=op, T=_log_int(rng, 1, 16384), V=V, H=min(H, 4096), table=t("bf16", "f32", "w4"),
                    out=t("bf16", "f32"), fmt=fmt, group=group)
    while V * H > 131072 * 4096:
        V = V // 2
    if op == "grad":
        return dict(op=op, T=_log_int(rng, 1, 16384), V=V, H=H, h=t("bf16", "f32"), out=t("bf16", "f32"))
    return dict(op=op, V=V, H=H, fmt=fmt, group=group, h=t("bf16", "f32"), out=t("bf16", "f32"))


_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------
# The 4-bit table in elementary operations
# ---------------------------------------------------------------------------
def _filled(x, n):
    """x with zeros up to n columns."""
    return x if x.shape[1] == n else torch.nn.functional.pad(x, (0, n - x.shape[1]))


def _scales(w, fmt, group):
    """The scale of each group, float32 [V, H / group]: amax / 7 rounded to float32 and then to
    bfloat16, or the power of two under amax, less the two binades that E2M1 has above one."""
    top = w.view(w.shape[0], -1, group).abs().amax(2).float()
    if fmt == "int":
        return (top.double() / 7).float().to(torch.bfloat16).float()
    return torch.ldexp(torch.ones_like(top), (torch.frexp(top)[1] - 3).clamp(-127, 127))


def _magnitudes(w, s, fmt, group):
    """|w / s| rounded to the format's numbers (nearest, ties to the even code), float32.  The quotient is
    taken in 64 bits: it decides between two codes."""
    q = w.view(w.shape[0], -1, group).abs().double().div_(s[:, :, None].clamp_min(2.0 ** -149).double())
    if fmt == "int":
        return q.round_().clamp_(max=7).view(w.shape).float()
    q = q.float()  # float32 or bfloat16 over a power of two: exact
    step = torch.where(q < 2, 0.5, torch.where(q < 4, 1.0, 2.0))
    return (q.div_(step).round_().mul_(step)).clamp_(max=6).view(w.shape)


def _quantise(w, fmt, group):
    """(codes uint8 [V, 64 blocks], scales) of a table."""
    V, H = w.shape
    nb = (H + 127) // 128
    s = _scales(w, fmt, group)
    m = _magnitudes(w, s, fmt, group)
    if fmt == "mx":  # 0, .5, 1, 1.5, 2, 3, 4, 6 are codes 0..7
        m = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4))
    c = _filled(m.to(torch.uint8) | torch.signbit(w).to(torch.uint8) << 3, nb * 128)
    c = c.view(V, nb, 4, 4, 8).transpose(2, 3)  # [.., g, j, element]
    if fmt == "mx":
        c = c[..., 0::2] | c[..., 1::2] << 4
        x = (torch.frexp(s)[1] + 126).to(torch.uint8)
    else:
        a, b = c[..., :4], c[..., 4:]
        c = (a & 7) | (a >> 3) << 7 | (b & 7) << 4 | (b >> 3).roll(1, -1) << 3
        x = s.to(torch.bfloat16)
    return c.contiguous().view(V, nb * 64), _filled(x, nb * 128 // group).contiguous()


def _values(codes, scales, fmt, group, H):
    """The numbers that a 4-bit table stands for, float32 [.., H]."""
    V = codes.shape[0]
    c = codes.view(V, -1, 4, 4, 4)
    if fmt == "mx":
        n = torch.stack([c & 15, c >> 4], -1).view(V, -1, 4, 4, 8).transpose(2, 3).reshape(V, -1)[:, :H]
        m = (n & 7).float()
        m = torch.where(m < 4, m / 2, torch.where(m < 6, m - 2, 2 * m - 8))
        v = torch.where(n >= 8, -m, m)
        s = torch.ldexp(torch.ones((), device=v.device), scales.int() - 127)
    else:
        n = torch.cat([(c & 7) | c >> 7 << 3, (c >> 4 & 7) | c.roll(-1, -1) & 8], -1)
        n = n.transpose(2, 3).reshape(V, -1)[:, :H]
        m = (n & 7).float()
        v = torch.where(n >= 8, -m, m)
        s = scales.float()
    return (v.reshape(V, -1, group) * s[:, :H // group, None]).view(V, H)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 11)
    return g


def _tokens(g, T, V):
    """Ids by Zipf's law over a shuffled vocabulary, a share of them -1."""
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1).long().clamp_(0, V - 1)
    ids = torch.randperm(V, generator=g, device="cuda")[rank]
    return torch.where(torch.rand(T, generator=g, device="cuda") < PAD, -1, ids).to(torch.int32)


def _normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=g)


def _inputs(case, seed):
    g, op, H, V = _gen(seed), case["op"], case["H"], case["V"]
    d = {}
    if op == "head":
        d["h"] = _normal(g, (case["T"], H), _TYPE[case["h"]])  # normalised hidden states
    if op in ("embed", "grad"):
        d["tokens"] = _tokens(g, case["T"], V)
    if op == "grad":
        d["dout"] = _normal(g, (case["T"], H), _TYPE[case["h"]], 1e-3)
        return d
    w = _normal(g, (V, H), _TYPE[case["h"] if op == "quant" else "f32" if case.get("table") == "f32" else "bf16"], 0.02)
    if op == "quant" or op == "embed" and case["table"] != "w4":
        d["w"] = w
    else:
        d["codes"], d["scales"] = _quantise(w, case["fmt"], case["group"])
    return d


def prepare(case, seed):
    state = dict(case=case, **_inputs(case, seed))
    if own:  # what a serving or training loop keeps: the table's handle, workspaces and output buffers
        from paper_2607_20475_amd import binding as ssb

        op, H, V, dt = case["op"], case["H"], case["V"], _TYPE.get(case["out"])
        new = lambda *s: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        if "codes" in state:
            state["w4"] = ssb.W4(state["codes"], state["scales"], V, H, case["fmt"], case["group"])
        if op == "head":
            state["out"] = new(case["T"], V)
            state["ws"] = ssb.head_workspace(state["h"])
        elif op == "embed":
            state["out"] = new(case["T"], H)
        elif op == "grad":
            state["out"] = new(V, H)
            state["ws"] = ssb.embed_grad_workspace(case["T"], V, H)
        else:
            state["w4"] = ssb.W4.empty(V, H, case["fmt"], case["group"])
            state["out"] = new(V, H)
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state):
    case = state["case"]
    op, dt = case["op"], _TYPE[case["out"]]
    if own:
        from paper_2607_20475_amd import binding as ssb

        if op == "head":
            return ssb.head_w4(state["h"], state["w4"], out=state["out"], ws=state["ws"])
        if op == "embed":
            return ssb.embed(state["tokens"], state.get("w4") or state["w"], scale=SCALE, out=state["out"])
        if op == "grad":
            return ssb.embed_grad(state["dout"], state["tokens"], case["V"], scale=SCALE, out=state["out"], ws=state["ws"])
        ssb.quantize_w4(state["w"], state["w4"], values=state["out"])
        return state["out"]
    if op == "head":
        W = _values(state["codes"], state["scales"], case["fmt"], case["group"], case["H"])
        return (state["h"].float() @ W.T).to(dt)
    if op == "quant":
        w = state["w"]
        s = _scales(w, case["fmt"], case["group"])
        m = _magnitudes(w, s, case["fmt"], case["group"]).view(w.shape[0], -1, case["group"]) * s[:, :, None]
        return torch.where(w < 0, -m.view(w.shape), m.view(w.shape)).to(dt)
    tok = state["tokens"].long()
    there = (tok >= 0) & (tok < case["V"])
    at = torch.where(there, tok, 0)
    if op == "embed":
        if "codes" in state:
            rows = _values(state["codes"][at], state["scales"][at], case["fmt"], case["group"], case["H"])
        else:
            rows = state["w"][at].float()
        return torch.where(there[:, None], rows * SCALE, 0.0).to(dt)
    dout = torch.where(there[:, None], state["dout"].float(), 0.0)
    dW = torch.zeros(case["V"], case["H"], device="cuda").index_add_(0, at, dout)
    return dW.mul_(SCALE).to(dt)


def work(case):
    op, V, H = case["op"], case["V"], case["H"]
    T = case.get("T", 0)
    size = {"bf16": 2, "f32": 4}
    w4 = lambda rows: rows * (H // 2 + H // case["group"] * (1 if case["fmt"] == "mx" else 2))  # noqa: E731
    if op == "head":
        return {"bytes": w4(V) + T * H * size[case["h"]] + T * V * size[case["out"]], "flops": 2 * T * V * H}
    rows = T * (1 - PAD)  # a repeated token's row is read once
    rows = min(rows, V * (1 - math.exp(-rows / V)))
    if op == "embed":
        read = w4(rows) if case["table"] == "w4" else rows * H * size[case["table"]]
        return {"bytes": read + T * 4 + T * H * size[case["out"]], "flops": T * H}
    if op == "grad":
        return {"bytes": T * (1 - PAD) * H * size[case["h"]] + T * 4 + V * H * size[case["out"]], "flops": T * H}
    return {"bytes": V * H * (size[case["h"]] + size[case["out"]]) + w4(V), "flops": 2 * V * H}


# ---------------------------------------------------------------------------
# The same results in 64 bits
# ---------------------------------------------------------------------------
def _table64(codes, scales, case):
    """The 4-bit table's numbers, dword by dword."""
    H, fmt = case["H"], case["fmt"]
    word = codes.contiguous().view(torch.int32).long() & 0xFFFFFFFF  # [V, 16 blocks]
    col = torch.arange(H, device="cuda")
    k = col % 128
    at = col // 128 * 16 + k % 32 // 8 * 4 + k // 32
    e = k % 8
    out = torch.empty(codes.shape[0], H, dtype=torch.float64, device="cuda")
    if fmt == "mx":
        number = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
        number = torch.cat([number, -number])
    else:
        number = torch.arange(8, dtype=torch.float64, device="cuda")
        number = torch.cat([number, -number])
    step = max(1, (1 << 26) // H)
    for r in range(0, codes.shape[0], step):
        w = word[r:r + step][:, at]
        if fmt == "mx":
            n = w >> (4 * e) & 15
            s = torch.exp2(scales[r:r + step].double() - 127)
        else:
            turned = (w >> 4 | w << 28) & 0xFFFFFFFF
            byte = torch.where(e < 4, w, turned) >> (8 * (e % 4))
            n = (byte & 7) + (byte >> 7 & 1) * 8
            s = scales[r:r + step].double()
        out[r:r + step] = number[n] * s[:, col // case["group"]]
    return out


def exact(case, seed):
    d, op, V, H = _inputs(case, seed), case["op"], case["V"], case["H"]
    if op == "head":
        return d["h"].double() @ _table64(d["codes"], d["scales"], case).T
    if op == "quant":
        w, G = d["w"], case["group"]
        out = torch.empty(V, H, dtype=torch.float64, device="cuda")
        half = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device="cuda")
        number = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
        for r in range(0, V, 8192):
            x = w[r:r + 8192].double().unflatten(1, (-1, G))
            top = x.abs().amax(2, keepdim=True)
            if case["fmt"] == "int":  # the scale is defined by its roundings: to float32, then to bfloat16
                s = (top / 7).float().to(torch.bfloat16).double()
                q = torch.where(s > 0, x / s, 0.0).round()
                y = q * s
            else:
                s = torch.exp2(torch.floor(torch.log2(top)).clamp_min(-125) - 2)
                a = x.abs() / s
                up, down = torch.bucketize(a, half, right=True), torch.bucketize(a, half)
                n = torch.where(up % 2 == 0, up, down)  # between two codes: the even one
                y = number[n] * s * x.sign()
            out[r:r + 8192] = y.flatten(1)
        return out
    tok = d["tokens"].cpu().long()
    hits = [(t, v) for t, v in enumerate(tok.tolist()) if 0 <= v < V]
    t, v = (torch.tensor([p[i] for p in hits], dtype=torch.long, device="cuda") for i in (0, 1))
    if op == "embed":
        out = torch.zeros(case["T"], H, dtype=torch.float64, device="cuda")
        out[t] = (_table64(d["codes"][v], d["scales"][v], case) if "codes" in d else d["w"][v].double()) * SCALE
        return out
    by = torch.argsort(v, stable=True)
    t, v = t[by], v[by]
    rows, n = torch.unique_consecutive(v, return_counts=True)
    out = torch.zeros(V, H, dtype=torch.float64, device="cuda")
    out[rows] = torch.segment_reduce(d["dout"][t].double(), "sum", lengths=n, axis=0) * SCALE if len(rows) else 0.0
    return out
