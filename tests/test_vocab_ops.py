"""The operators at the two ends of the vocabulary (4-bit head, lookup, its gradient, quantiser):
small cases against plain implementations in 64 bits, refusals, and a run of them together.

Tolerances.  A rounding to a type is off by at most half a step, u = eps / 2 relative.  The head's
products are exact; a matrix instruction adds 32 of them, and a row is H / 32 (float32 hidden states:
3 H / 32) instructions and at most 24 joins long, each addition off by at most 2^-23 of the sum of
magnitudes S, whether it rounds or cuts: (32 + P H / 32 + 24) 2^-23 S.  The gradient's sums of n rows
are n additions of float32, 2^-24 each.
"""
import ctypes as C

import numpy as np
import pytest
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF16, F32 = torch.bfloat16, torch.float32
KINDS = [("int", 128), ("int", 64), ("int", 32), ("mx", 32)]
E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])


def say(*a):
    print(*a, flush=True)


# ---------------------------------------------------------------------------
# Plain implementations (numpy, 64 bits)
# ---------------------------------------------------------------------------
def pack(n, fmt):
    """Dwords of codes n [V, H] (sign and magnitude in four bits: s mmm), by the layout's words."""
    V, H = n.shape
    nb = (H + 127) // 128
    out = np.zeros((V, nb * 16), np.uint32)
    for k in range(H):
        b, c = divmod(k, 128)
        j, g, e = c // 32, c % 32 // 8, c % 8
        x = n[:, k].astype(np.uint64)
        if fmt == "mx":
            w = x << np.uint64(4 * e)
        else:
            byte = (x >> np.uint64(3)) << np.uint64(7) | x & np.uint64(7)
            w = byte << np.uint64(8 * (e % 4))
            if e >= 4:
                w = w << np.uint64(4) | w >> np.uint64(28)
        out[:, b * 16 + 4 * g + j] |= (w & np.uint64(0xFFFFFFFF)).astype(np.uint32)
    return out.view(np.uint8).reshape(V, nb * 64)


def numbers(n, fmt):
    if fmt == "mx":
        return E2M1[n]
    m = (n & 7).astype(np.float64)
    return np.where(n & 8, -m, m)


def random_table(rng, V, H, fmt, group, fill=0xFF):
    """(codes, scales) as the library takes them, and the table's values [V, H]; what pads the last block
    is `fill`: it must not count."""
    n = rng.integers(0, 16, (V, H)).astype(np.int64)
    nb = (H + 127) // 128
    codes = pack(n, fmt)
    pad = nb * 128 - H
    if pad:
        junk = np.full((V, nb * 128), 15, np.int64)
        junk[:, :H] = n
        codes = pack(junk, fmt)
    groups, padded = H // group, nb * 128 // group
    if fmt == "mx":
        x = rng.integers(115, 125, (V, padded)).astype(np.uint8)
        x[:, groups:] = fill
        s = np.exp2(x[:, :groups].astype(np.float64) - 127)
        scales = torch.from_numpy(x)
    else:
        sc = torch.from_numpy(rng.uniform(0.001, 0.02, (V, padded)).astype(np.float32)).to(BF16)
        sc[:, groups:] = float("nan")
        s = sc[:, :groups].double().numpy()
        scales = sc
    return torch.from_numpy(codes), scales, numbers(n, fmt) * np.repeat(s, group, 1)


def quantise(w, fmt, group):
    """(codes n [V, H] s mmm, scales [V, H / group]) by the definition, in 64 bits."""
    V, H = w.shape
    x = w.astype(np.float64).reshape(V, -1, group)
    with np.errstate(all="ignore"):
        top = np.abs(x).max(2)
        fine = np.isfinite(top)
        if fmt == "int":
            s = torch.from_numpy(np.where(fine, top, 0) / 7).float().to(BF16).double().numpy()
            q = np.abs(x) / s[:, :, None]
            m = np.where(s[:, :, None] > 0, np.minimum(np.rint(q), 7), 0)
        else:
            e = np.where(top > 0, np.floor(np.log2(np.where(fine & (top > 0), top, 1))), -1000)
            s = np.exp2(np.maximum(e - 2, -127))
            q = np.abs(x) / s[:, :, None]
            half = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0])
            up, down = (q[..., None] >= half).sum(-1), (q[..., None] > half).sum(-1)
            m = np.where(up % 2 == 0, up, down)
        m = np.where(fine[:, :, None], m, 0).astype(np.int64)
        n = m | np.where(np.signbit(x) & fine[:, :, None], 8, 0)
    return n.reshape(V, H), np.where(fine, s, np.nan)


def as64(t):
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------------------
# Without a GPU: layout, sizes, refusals
# ---------------------------------------------------------------------------
@pytest.fixture(scope="module")
def lib():
    import os

    from paper_2607_20475_amd import build as b
    if not os.path.exists(b.LIB_PATH):
        b.build()
    from paper_2607_20475_amd import binding
    return binding.lib()


def test_layout_of_the_performance_cases_is_the_documented_one():
    """The plain form's packing and values (what perf/operators.py feeds to both sides)."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("perf_operators", path)
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    rng = np.random.default_rng(0)
    for fmt, group in KINDS:
        w = rng.normal(0, 0.02, (9, 3 * 128 + max(group, 32))).astype(np.float32)[:, : 3 * 128 + group % 128]
        n, s = quantise(w, fmt, group)
        codes, scales = M._quantise(torch.from_numpy(w), fmt, group)
        assert np.array_equal(codes.numpy(), pack(n, fmt)), (fmt, group)
        v = M._values(codes, scales, fmt, group, w.shape[1])
        assert np.array_equal(as64(v), numbers(n, fmt) * np.repeat(s, group, 1))


def test_table_sizes(lib):
    from paper_2607_20475_amd import binding as b
    size = lambda V, H, fmt, group: (  # noqa: E731
        lib.ss_w4_codes_bytes(C.byref(b._W4(V=V, H=H, fmt=fmt, group=group))),
        lib.ss_w4_scales_bytes(C.byref(b._W4(V=V, H=H, fmt=fmt, group=group))))
    assert size(10, 256, 0, 128) == (10 * 128, 10 * 4)
    assert size(10, 160, 0, 32) == (10 * 128, 10 * 16)
    assert size(10, 160, 1, 32) == (10 * 128, 10 * 8)
    assert size(1 << 20, 8192, 1, 32) == (1 << 32, 1 << 28)
    for bad in [(0, 256, 0, 128), ((1 << 20) + 1, 256, 0, 128), (10, 0, 0, 128), (10, 192, 0, 128), (10, 96, 0, 64),
                (10, 40, 0, 32), (10, 256, 0, 16), (10, 256, 1, 64), (10, 48, 1, 32), (10, 256, 2, 32),
                (10, (1 << 16) + 128, 0, 128), (-1, 256, 0, 128)]:
        assert size(*bad) == (0, 0), bad
    assert lib.ss_w4_codes_bytes(None) == 0


def test_head_arguments_are_checked_before_launch(lib):
    from paper_2607_20475_amd import binding as b
    fake = 0x10000  # never dereferenced: validation fails first

    def call(h=fake, dtype=1, T=4, ld_h=256, V=100, H=256, fmt=0, group=128, codes=fake, scales=fake, out=fake,
             out_dtype=1, ld=100, ws=fake, ws_bytes=1 << 20):
        t = b._W4(V=V, H=H, fmt=fmt, group=group, codes=codes, scales=scales)
        return lib.ss_head_w4(h, dtype, T, ld_h, C.byref(t), out, out_dtype, ld, ws, ws_bytes, None)

    for bad in [dict(h=None), dict(dtype=2), dict(T=-1), dict(T=(1 << 20) + 1), dict(ld_h=255), dict(V=0), dict(H=192),
                dict(fmt=3), dict(group=16), dict(codes=None), dict(codes=fake + 8), dict(scales=None),
                dict(scales=fake + 2), dict(out=None), dict(out_dtype=-1), dict(ld=99), dict(ws=None)]:
        assert call(**bad) == -1, bad
    assert lib.ss_head_w4(fake, 1, 4, 256, None, fake, 1, 100, fake, 1 << 20, None) == -1
    n = lib.ss_head_w4_bytes(4, 256, 0)
    assert call(dtype=0, ws_bytes=n - 1) == -3
    assert call(ws=fake + 8) == -3
    assert call(T=0, h=None, out=None, ws=None) == 0  # no rows: nothing to do
    assert lib.ss_head_w4_bytes(-1, 256, 0) == 0 and lib.ss_head_w4_bytes(4, 0, 0) == 0
    assert lib.ss_head_w4_bytes(4, 256, 2) == 0


def test_lookup_arguments_are_checked_before_launch(lib):
    from paper_2607_20475_amd import binding as b
    fake = 0x10000

    def call(tokens=fake, T=4, table=fake, dtype=1, V=100, H=60, ld=60, out=fake, out_dtype=0, ld_out=60):
        return lib.ss_embed(tokens, T, table, dtype, V, H, ld, 1.0, out, out_dtype, ld_out, None)

    for bad in [dict(tokens=None), dict(T=-1), dict(T=(1 << 20) + 1), dict(table=None), dict(dtype=2), dict(V=0),
                dict(H=0), dict(H=(1 << 16) + 1), dict(ld=59), dict(out=None), dict(out_dtype=5), dict(ld_out=59)]:
        assert call(**bad) == -1, bad
    assert call(T=0, tokens=None, table=None, out=None) == 0
    t = b._W4(V=100, H=256, fmt=0, group=128, codes=fake, scales=fake)
    assert lib.ss_embed_w4(fake, 4, C.byref(t), 1.0, fake, 0, 255, None) == -1
    assert lib.ss_embed_w4(None, 4, C.byref(t), 1.0, fake, 0, 256, None) == -1
    assert lib.ss_embed_w4(fake, 4, None, 1.0, fake, 0, 256, None) == -1
    assert lib.ss_embed_w4(None, 0, C.byref(t), 1.0, None, 0, 256, None) == 0
    t.codes = fake + 4
    assert lib.ss_embed_w4(fake, 4, C.byref(t), 1.0, fake, 0, 256, None) == -1


def test_gradient_arguments_are_checked_before_launch(lib):
    fake = 0x10000
    n = lib.ss_embed_grad_bytes(4, 100, 60)

    def call(dout=fake, dtype=1, T=4, ld=60, tokens=fake, V=100, H=60, out=fake, out_dtype=0, ld_out=60, ws=fake,
             ws_bytes=n):
        return lib.ss_embed_grad(dout, dtype, T, ld, tokens, V, H, 1.0, out, out_dtype, ld_out, 0, ws, ws_bytes, None)

    for bad in [dict(dout=None), dict(dtype=2), dict(T=-1), dict(T=(1 << 20) + 1), dict(ld=59), dict(tokens=None),
                dict(V=0), dict(V=(1 << 20) + 1), dict(H=0), dict(out=None), dict(out_dtype=2), dict(ld_out=59),
                dict(ws=None)]:
        assert call(**bad) == -1, bad
    assert call(ws_bytes=n - 1) == -3
    assert call(ws=fake + 4) == -3
    assert lib.ss_embed_grad_bytes(4, 0, 60) == 0 and lib.ss_embed_grad_bytes(-1, 10, 60) == 0


def test_quantiser_arguments_are_checked_before_launch(lib):
    from paper_2607_20475_amd import binding as b
    fake = 0x10000

    def call(w=fake, dtype=1, ld=256, V=100, H=256, fmt=0, group=128, codes=fake, scales=fake, values=None, vdt=0, ldv=0):
        t = b._W4(V=V, H=H, fmt=fmt, group=group, codes=codes, scales=scales)
        return lib.ss_quant_w4(w, dtype, ld, C.byref(t), values, vdt, ldv, None)

    for bad in [dict(w=None), dict(dtype=2), dict(ld=255), dict(V=0), dict(H=100), dict(fmt=2), dict(group=8),
                dict(codes=None), dict(scales=None), dict(codes=fake + 1), dict(values=fake, ldv=255),
                dict(values=fake, vdt=3, ldv=256)]:
        assert call(**bad) == -1, bad


def test_wrappers_refuse_what_they_cannot_pass_on():
    from paper_2607_20475_amd import binding as b
    with pytest.raises(b.SSError, match="neither"):
        b.W4.empty(4, 128, "fp8", 128, device="cpu")
    with pytest.raises(b.SSError, match="no int table"):
        b.W4.empty(4, 192, "int", 128, device="cpu")
    t = b.W4.empty(4, 160, "int", 32, device="cpu")
    assert t.codes.shape == (4, 128) and t.scales.shape == (4, 8)
    with pytest.raises(b.SSError, match="codes"):
        b.W4(t.codes[:, :64], t.scales, 4, 160, "int", 32)
    with pytest.raises(b.SSError, match="scales"):
        b.W4(t.codes, t.scales.float(), 4, 160, "int", 32)
    with pytest.raises(b.SSError, match="not on a GPU"):
        b.head_w4(torch.zeros(2, 160, dtype=BF16), t)
    with pytest.raises(b.SSError, match="not on a GPU"):
        b.embed(torch.zeros(2, dtype=torch.int32), t)
    with pytest.raises(b.SSError, match="tokens"):
        b.embed(torch.zeros(2, dtype=torch.int64), t)
    with pytest.raises(b.SSError, match="unit column stride"):
        b.embed_grad(torch.zeros(6, 4).t(), torch.zeros(4, dtype=torch.int32), 10)
    with pytest.raises(b.SSError, match="unit column stride"):  # broadcast rows
        b.embed_grad(torch.zeros(1, 6).expand(4, 6), torch.zeros(4, dtype=torch.int32), 10)


def test_a_table_keeps_the_arrays_it_was_made_with():
    """Calls pass the addresses that a table was made with: neither they nor its sizes can be changed under it, and an
    array that has moved is refused (before its place is looked at by a kernel)."""
    from paper_2607_20475_amd import binding as b
    t = b.W4.empty(4, 256, "int", 128, device="cpu")
    for name, value in [("codes", torch.zeros(4, 128, dtype=torch.uint8)), ("scales", torch.zeros(4, 2, dtype=BF16)),
                        ("V", 5), ("H", 128), ("fmt", "mx"), ("group", 64)]:
        with pytest.raises(AttributeError):
            setattr(t, name, value)
    b._table(t, -1)  # (a CPU tensor's device index)
    t.codes.fill_(3)
    b._table(t, -1)
    t.codes.set_(torch.zeros(4, 128, dtype=torch.uint8))
    with pytest.raises(b.SSError, match="moved"):
        b._table(t, -1)
    t = b.W4.empty(4, 256, "int", 128, device="cpu")
    t.scales.set_(torch.zeros(4, 2, dtype=BF16))
    with pytest.raises(b.SSError, match="moved"):
        b._table(t, -1)


def test_sizes_reach_the_library_as_they_are():
    """Sizes that 32 bits do not hold, or that are no whole numbers, are refused: cut to 32 bits or to whole numbers
    they would name other tables, with fewer rows or scales than the kernels read."""
    from paper_2607_20475_amd import binding as b
    wrap = 1 << 32
    codes, scales = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 4, dtype=BF16)
    for V, H, group in [(4 + wrap, 128, 32), (4, 128 + wrap, 32), (4, 128, 32 + wrap), (4, 128, 32 - wrap), (4, 128, 32.5),
                        (4.5, 128, 32), (4, 128.25, 32), ("4", 128, 32), (None, 128, 32), (float("nan"), 128, 32)]:
        with pytest.raises(b.SSError):
            b.W4.empty(V, H, "int", group, device="cpu")
        with pytest.raises(b.SSError):
            b.W4(codes, scales, V, H, "int", group)
    with pytest.raises(b.SSError):
        b.W4(codes, scales[:, :3].contiguous(), 4, 128, "int", 32.5)
    t = b.W4(codes, scales, np.int64(4), np.int64(128), "int", np.int64(32))
    assert (t._struct.V, t._struct.H, t._struct.group) == (t.V, t.H, t.group) == (4, 128, 32)
    for T, V, H in [(5 + wrap, 10, 8), (5, 10 + wrap, 8), (5, 10, 8 + wrap), (5, 10.5, 8)]:
        with pytest.raises(b.SSError):
            b.embed_grad_workspace(T, V, H, device="cpu")
    with pytest.raises(b.SSError, match="V = "):
        b.embed_grad(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), 10 + wrap)
    # rows beyond 2^32, without their memory: a view of one row
    tall = torch.zeros(1, 32, dtype=BF16).expand(wrap + 4, 32)
    with pytest.raises(b.SSError, match="32 bits"):
        b._rows(tall, "table", -1)
    with pytest.raises(b.SSError, match="32 bits"):
        b._tokens(torch.empty(wrap + 4, dtype=torch.int32, device="meta"), -1)
    with pytest.raises(b.SSError):
        b.head_workspace(tall)


def test_a_workspace_has_the_bytes_that_it_is_taken_for():
    """Elements times their size is the room behind the pointer only where they follow one another."""
    from paper_2607_20475_amd import binding as b
    ws = torch.zeros(64, 32, dtype=torch.int32)
    assert b._space(ws, -1) == (ws.data_ptr(), 64 * 32 * 4)
    assert b._space(ws[8:], -1) == (ws.data_ptr() + 8 * 32 * 4, 56 * 32 * 4)
    for bad in (ws[:1, :1].expand(64, 1024), ws[:, ::2], ws.t(), ws[:, :16]):
        with pytest.raises(b.SSError, match="contiguous"):
            b._space(bad, -1)


def test_what_a_call_asks_for_is_not_passed_over():
    """A format, group or type that differs from the table or output that is handed in."""
    from paper_2607_20475_amd import binding as b
    t = b.W4.empty(4, 256, "mx", 32, device="cpu")
    w = torch.zeros(4, 256)
    for bad in (dict(fmt="int"), dict(group=64), dict(fmt="mx", group=128)):
        with pytest.raises(b.SSError, match="table is mx in groups of 32"):
            b.quantize_w4(w, t, **bad)
    for good in (dict(), dict(fmt="mx"), dict(group=32), dict(fmt="mx", group=32)):
        with pytest.raises(b.SSError, match="not on a GPU"):
            b.quantize_w4(w, t, **good)


@pytest.mark.gpu
def test_the_type_of_a_gradient_is_not_passed_over(ssb):
    d, tok = torch.ones(3, 8, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    out = torch.zeros(2, 8, dtype=BF16, device="cuda")
    with pytest.raises(ssb.SSError, match="out must be"):
        ssb.embed_grad(d, tok, 2, out=out, dtype=F32)
    assert ssb.embed_grad(d, tok, 2, out=out, dtype=BF16) is out and (out[0] == 3).all()
    assert (ssb.embed_grad(d, tok, 2, out=out, accumulate=True)[0] == 6).all()
    assert ssb.embed_grad(d, tok, 2).dtype == F32 and ssb.quantize_w4(torch.ones(2, 128, device="cuda")).group == 128


# ---------------------------------------------------------------------------
# On the GPU
# ---------------------------------------------------------------------------
@pytest.fixture(scope="module")
def ssb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_20475_amd import binding
    binding.lib()
    return binding


def strided(t, extra, shift=0):
    """t on the GPU as rows `extra` columns further apart, `shift` elements into an allocation of sentinels."""
    R, n = t.shape
    base = torch.full((R * (n + extra) + shift + 8,), 77.0, dtype=t.dtype, device="cuda")
    v = base[shift:shift + R * (n + extra)].view(R, n + extra)
    v[:, :n] = t.cuda()
    return v[:, :n], base


HEAD = [
    # T, V, H: one token and one row, tiles that end inside, every number of token tiles, partial blocks
    (1, 1, 32), (1, 65, 128), (2, 15, 64), (3, 16, 96), (5, 63, 160), (15, 64, 384), (16, 257, 640), (16, 1000, 1152),
    (17, 70, 128), (31, 300, 224), (32, 64, 256), (33, 257, 288), (48, 130, 512), (50, 513, 640), (64, 256, 384),
    (65, 259, 96), (100, 1025, 256), (129, 33, 1056), (200, 2100, 128), (1, 5000, 2048), (7, 40, 8192), (40, 20, 8192),
]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", KINDS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_head_against_64_bits(ssb, fmt, group, dtype):
    rng = np.random.default_rng(31 + group)
    for i, (T, V, H) in enumerate(HEAD):
        if H % group:
            H = (H + group - 1) // group * group
        codes, scales, W = random_table(rng, V, H, fmt, group)
        table = ssb.W4(codes.cuda(), scales.cuda(), V, H, fmt, group)
        h = torch.from_numpy(rng.normal(0, 1, (T, H)).astype(np.float32)).to(dtype)
        for out_dtype, extra, shift in ((BF16, 0, 0), (F32, 3, 1), (BF16, 4, 4)):
            say(f"[head] {fmt}{group} {dtype} T={T} V={V} H={H} out={out_dtype} extra={extra}")
            hs, _ = strided(h, extra, shift)
            out, base = strided(torch.zeros(T, V, dtype=out_dtype), extra, shift)
            r = ssb.head_w4(hs, table, out=out)
            torch.cuda.synchronize()
            assert r.data_ptr() == out.data_ptr()
            h64 = as64(h)
            ref, S = h64 @ W.T, np.abs(h64) @ np.abs(W).T
            P = 3 if dtype == F32 else 1
            tol = (32 + P * H / 32 + 24) * 2.0 ** -23 * S * (1 + U[out_dtype]) + U[out_dtype] * np.abs(ref) + 1e-30
            err = np.abs(as64(out) - ref)
            assert (err <= tol).all(), (T, V, H, out_dtype, float((err / tol).max()))
            rest = base[shift:shift + T * (V + extra)].view(T, V + extra)[:, V:]
            assert (rest == 77).all() and (base[:shift] == 77).all() and (base[shift + T * (V + extra):] == 77).all()


LARGE = [
    # V, H: one unit of eight blocks a row; ends inside a unit, inside a block; columns that do not fit LDS at 16 rows (and
    # end inside a block); more waves than a row has units, and tiles that waves share unevenly
    (131077, 128), (131072, 1024), (50007, 2080), (200003, 1152), (26229, 4224), (26245, 8032), (33003, 6144),
]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", KINDS)
@pytest.mark.parametrize("dtype,T", [(BF16, 1), (BF16, 6), (BF16, 16), (F32, 1), (F32, 4)])
def test_head_of_large_tables(ssb, fmt, group, dtype, T):
    """Tables that fill the chip with few hidden rows, against 64 bits on the GPU (the table's values by the lookup, which
    is exact in float32)."""
    g = torch.Generator(device="cuda")
    for V, H in LARGE:
        H = (H + group - 1) // group * group
        g.manual_seed(V + H)
        nb = (H + 127) // 128
        codes = torch.randint(0, 256, (V, 64 * nb), dtype=torch.uint8, device="cuda", generator=g)
        if fmt == "mx":
            scales = torch.randint(115, 125, (V, nb * 4), dtype=torch.uint8, device="cuda", generator=g)
            scales[:, H // 32:] = 255
        else:
            scales = torch.empty(V, nb * 128 // group, device="cuda").uniform_(0.001, 0.02, generator=g).to(BF16)
            scales[:, H // group:] = float("nan")
        table = ssb.W4(codes, scales, V, H, fmt, group)
        say(f"[head large] {fmt}{group} {dtype} T={T} V={V} H={H}")
        h = torch.empty(T, H + 3, device="cuda").normal_(generator=g).to(dtype)[:, 1:H + 1]  # rows at odd addresses
        if T >= 4:
            h[1, H // 2], h[2, H - 1] = float("inf"), float("nan")  # stay in their rows
        out = torch.full((T, V + 1), 77.0, device="cuda")
        ssb.head_w4(h, table, out=out[:, :V])
        if T >= 4:
            assert not torch.isfinite(out[1:3, :V]).any()
            h[1:3] = 0
            out[1:3, :V] = 0
        W = ssb.embed(torch.arange(V, dtype=torch.int32, device="cuda"), table, dtype=F32)
        h64 = h.double()
        for r in range(0, V, 32768):
            w = W[r:r + 32768].double()
            ref, S = h64 @ w.T, h64.abs() @ w.abs().T
            tol = (32 + (3 if dtype == F32 else 1) * H / 32 + 24) * 2.0 ** -23 * S + U[F32] * ref.abs()
            assert ((out[:, r:min(r + 32768, V)].double() - ref).abs() <= tol).all(), (V, H)
        assert (out[:, V] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", KINDS)
@pytest.mark.parametrize("dtype,T", [(BF16, 9), (BF16, 20), (BF16, 41), (BF16, 64), (BF16, 100), (F32, 11), (F32, 27), (F32, 70)])
def test_head_of_large_tables_with_more_rows(ssb, fmt, group, dtype, T):
    """The same with every number of token tiles, for tables that give each compute unit less than a workgroup, more
    than one, and many (columns end inside a block and inside a chunk)."""
    g = torch.Generator(device="cuda")
    for V, H in ((12301, 1824), (30011, 800), (40003, 928), (95003, 544), (131077, 672), (161103, 1184)):
        H = (H + group - 1) // group * group
        g.manual_seed(V + H)
        nb = (H + 127) // 128
        codes = torch.randint(0, 256, (V, 64 * nb), dtype=torch.uint8, device="cuda", generator=g)
        if fmt == "mx":
            scales = torch.randint(115, 125, (V, nb * 4), dtype=torch.uint8, device="cuda", generator=g)
            scales[:, H // 32:] = 255
        else:
            scales = torch.empty(V, nb * 128 // group, device="cuda").uniform_(0.001, 0.02, generator=g).to(BF16)
            scales[:, H // group:] = float("nan")
        table = ssb.W4(codes, scales, V, H, fmt, group)
        say(f"[head large] {fmt}{group} {dtype} T={T} V={V} H={H}")
        h = torch.empty(T, H, device="cuda").normal_(generator=g).to(dtype)
        h[1, H // 2], h[2, H - 1] = float("inf"), float("nan")  # stay in their rows
        out = torch.full((T, V + 3), 77.0, device="cuda")
        ssb.head_w4(h, table, out=out[:, :V])
        assert not torch.isfinite(out[1:3, :V]).any()
        h[1:3] = 0
        out[1:3, :V] = 0
        W = ssb.embed(torch.arange(V, dtype=torch.int32, device="cuda"), table, dtype=F32)
        h64 = h.double()
        for r in range(0, V, 32768):
            w = W[r:r + 32768].double()
            ref, S = h64 @ w.T, h64.abs() @ w.abs().T
            tol = (32 + (3 if dtype == F32 else 1) * H / 32 + 24) * 2.0 ** -23 * S + U[F32] * ref.abs()
            assert ((out[:, r:min(r + 32768, V)].double() - ref).abs() <= tol).all(), (V, H)
        assert (out[:, V:] == 77).all()


FORMS = [
    # float32 hidden states?, T, V, H: every form of the head's kernels, and both sides of the rules between them.  More than
    # 16 rows: four tiles of table rows a wave (and their last columns apart), two, one; workgroups of 16, 14 and 12 waves
    (0, 64, 131072, 608), (0, 64, 131065, 608), (0, 320, 131072, 608), (0, 41, 131072, 608), (0, 41, 131065, 608),
    (0, 32, 131072, 608), (0, 20, 131065, 608), (0, 20, 12301, 608), (0, 29, 161103, 608), (0, 29, 95003, 608),
    (0, 64, 65521, 608), (0, 64, 161103, 608), (0, 64, 95003, 608),
    # up to 16 rows: short rows, a table row more than the other kernel's first round, columns that fit LDS and that do not
    (0, 16, 131077, 384), (0, 16, 131077, 512), (0, 9, 32768, 4096), (0, 9, 32769, 4096), (0, 16, 131072, 1056),
    (0, 1, 131077, 1024), (0, 8, 16384, 8192), (0, 16, 16384, 8192), (0, 16, 40003, 6144), (0, 11, 4097, 608), (0, 3, 33001, 608),
    # float32 hidden states
    (1, 4, 131077, 1024), (1, 4, 33003, 6144), (1, 11, 131077, 672), (1, 9, 257, 96), (1, 9, 257, 640), (1, 20, 257, 640),
    (1, 33, 40003, 160),
]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", KINDS)
@pytest.mark.parametrize("part", range(4))
def test_every_form_of_the_head(ssb, fmt, group, part):
    """bfloat16 and float32 logits, rows of hidden states and logits at aligned and at odd addresses, against 64 bits."""
    g = torch.Generator(device="cuda")
    for f32, T, V, H in FORMS[part::4]:
        H = (H + group - 1) // group * group
        g.manual_seed(T + V + H)
        nb = (H + 127) // 128
        codes = torch.randint(0, 256, (V, 64 * nb), dtype=torch.uint8, device="cuda", generator=g)
        if fmt == "mx":
            scales = torch.randint(115, 125, (V, nb * 4), dtype=torch.uint8, device="cuda", generator=g)
            scales[:, H // 32:] = 255
        else:
            scales = torch.empty(V, nb * 128 // group, device="cuda").uniform_(0.001, 0.02, generator=g).to(BF16)
            scales[:, H // group:] = float("nan")
        table = ssb.W4(codes, scales, V, H, fmt, group)
        h = torch.empty(T, H, device="cuda").normal_(generator=g).to(F32 if f32 else BF16)
        W = ssb.embed(torch.arange(V, dtype=torch.int32, device="cuda"), table, dtype=F32)
        h64 = h.double()
        ref, S = torch.empty(T, V, dtype=torch.float64, device="cuda"), torch.empty(T, V, dtype=torch.float64, device="cuda")
        for r in range(0, V, 32768):
            w = W[r:r + 32768].double()
            ref[:, r:r + 32768], S[:, r:r + 32768] = h64 @ w.T, h64.abs() @ w.abs().T
        slack = (32 + (3 if f32 else 1) * H / 32 + 24) * 2.0 ** -23 * S
        for extra, shift in ((0, 0), (3, 1)):
            hs, _ = strided(h, extra, shift)
            for out_dtype in (BF16, F32):
                say(f"[forms] {fmt}{group} {h.dtype} T={T} V={V} H={H} out={out_dtype} extra={extra}")
                base = torch.full((T * (V + extra) + shift + 8,), 77.0, dtype=out_dtype, device="cuda")
                rows = base[shift:shift + T * (V + extra)].view(T, V + extra)
                ssb.head_w4(hs, table, out=rows[:, :V])
                tol = slack * (1 + U[out_dtype]) + U[out_dtype] * ref.abs()
                assert ((rows[:, :V].double() - ref).abs() <= tol).all()
                assert (rows[:, V:] == 77).all() and (base[:shift] == 77).all() and (base[shift + T * (V + extra):] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", [("mx", 32), ("int", 128)])
def test_rows_beyond_32_bits_bit_for_bit(ssb, fmt, group):
    """A table of 4.5 GB against tables of some of its rows.  Sums of multiples of a half below 2^18: exact in any order."""
    g = torch.Generator(device="cuda").manual_seed(16)
    V, H = 1 << 20, 8704
    nb = H // 128
    codes = torch.empty(V, 64 * nb, dtype=torch.uint8, device="cuda")
    for r in range(0, V, 1 << 17):
        codes[r:r + (1 << 17)] = torch.randint(0, 256, (1 << 17, 64 * nb), dtype=torch.uint8, device="cuda", generator=g)
    scales = (torch.full((V, nb * 4), 127, dtype=torch.uint8, device="cuda") if fmt == "mx"
              else torch.ones(V, nb, dtype=BF16, device="cuda"))
    big = ssb.W4(codes, scales, V, H, fmt, group)
    at = [slice(0, 100), slice(493440, 493600), slice(986800, 987000), slice(V - 100, V)]  # 2^32 bytes lie at row 986895
    few = [ssb.W4(codes[s].clone(), scales[s].clone(), s.stop - s.start, H, fmt, group) for s in at]
    for dtype, T in ((BF16, 2), (BF16, 20), (BF16, 64), (F32, 2), (F32, 20)):
        say(f"[4 GB exact] {fmt}{group} {dtype} T={T}")
        h = torch.randint(-4, 5, (T, H), device="cuda", generator=g).to(dtype)
        out = ssb.head_w4(h, big, dtype=F32)
        for s, t in zip(at, few):
            W = ssb.embed(torch.arange(t.V, dtype=torch.int32, device="cuda"), t, dtype=F32)
            want = h.double() @ W.double().T
            assert torch.equal(out[:, s].double(), want) and torch.equal(ssb.head_w4(h, t, dtype=F32), out[:, s])


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", KINDS)
def test_the_widest_rows(ssb, fmt, group):
    """Rows of 65536 columns, the most there are, through every operator; tables that fill the chip and that do not."""
    g = torch.Generator(device="cuda").manual_seed(5)
    H = 65536
    for V in (37, 2049):
        w = torch.empty(V, H, device="cuda").normal_(generator=g)
        table = ssb.quantize_w4(w, fmt=fmt, group=group, values=w)
        W = ssb.embed(torch.arange(V, dtype=torch.int32, device="cuda"), table, dtype=F32)
        assert torch.equal(W, w)
        for dtype, T in ((BF16, 1), (BF16, 16), (BF16, 33), (F32, 1), (F32, 3), (F32, 17)):
            say(f"[wide] {fmt}{group} V={V} {dtype} T={T}")
            h = torch.empty(T, H, device="cuda").normal_(generator=g).to(dtype)
            out = ssb.head_w4(h, table, dtype=F32)
            ref, S = h.double() @ W.double().T, h.double().abs() @ W.double().abs().T
            tol = (32 + (3 if dtype == F32 else 1) * H / 32 + 24) * 2.0 ** -23 * S + U[F32] * ref.abs()
            assert ((out.double() - ref).abs() <= tol).all(), (V, dtype, T)
    tokens = torch.tensor([4, -1, 4, 36, 0] + [7] * 70, dtype=torch.int32, device="cuda")
    d = torch.empty(len(tokens), H, device="cuda").normal_(generator=g)
    grad = ssb.embed_grad(d, tokens, 37)
    for v, where in ((4, [0, 2]), (36, [3]), (0, [4]), (7, list(range(5, 75)))):
        ref, S = d[where].double().sum(0), d[where].double().abs().sum(0)
        assert ((grad[v].double() - ref).abs() <= (len(where) + 1) * 2.0 ** -24 * S).all()
    named = torch.zeros(37, dtype=torch.bool, device="cuda")
    named[[4, 36, 0, 7]] = True
    assert (grad[~named] == 0).all()


@pytest.mark.gpu
def test_one_token_at_every_position(ssb):
    """The longest run: every position names one id, beside positions that name none."""
    T, H = 1 << 20, 8
    d = torch.randint(-8, 9, (T, H), device="cuda").to(BF16)  # sums of integers: exact below 2^24
    tokens = torch.full((T,), 99, dtype=torch.int32, device="cuda")
    tokens[::1000] = -1
    out = ssb.embed_grad(d, tokens, 100)
    ref = d[tokens == 99].double().sum(0)
    assert torch.equal(out[99].double(), ref) and (out[:99] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 40])
def test_head_takes_float32_whole(ssb, T):
    """Hidden states that differ beyond bfloat16: the result keeps what float32 has.  A table row of a single one
    returns the state itself, bit for bit."""
    rng = np.random.default_rng(2)
    V, H = 256, 256
    n = np.zeros((V, H), np.int64)
    n[np.arange(V), np.arange(V)] = 1
    one = torch.ones(V, 2, dtype=BF16)
    table = ssb.W4(torch.from_numpy(pack(n, "int")).cuda(), one.cuda(), V, H, "int", 128)
    h = (rng.normal(0, 1, (T, H)) * np.exp2(rng.integers(-60, 60, (T, H)))).astype(np.float32)
    out = ssb.head_w4(torch.from_numpy(h).cuda(), table)
    assert np.array_equal(out.cpu().numpy(), h)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4, 70])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_head_keeps_rows_and_columns_apart(ssb, T, dtype):
    """Infinities and NaN of one hidden row or one table row stay there."""
    rng = np.random.default_rng(3)
    for fmt, group in KINDS:
        V, H = 130, 256
        codes, scales, W = random_table(rng, V, H, fmt, group)
        if fmt == "mx":
            scales[77, 3] = 255
        else:
            scales[77, 0] = float("nan")
        h = torch.from_numpy(rng.normal(0, 1, (T, H)).astype(np.float32)).to(dtype)
        h[1, 5], h[2, 9], h[T - 1, 0] = float("inf"), float("nan"), -float("inf")
        out = ssb.head_w4(h.cuda(), ssb.W4(codes.cuda(), scales.cuda(), V, H, fmt, group), dtype=F32)
        got = torch.isfinite(out).cpu().numpy()
        want = np.ones((T, V), bool)
        want[:, 77] = False
        want[[1, 2, T - 1]] = False
        assert np.array_equal(got, want), (fmt, group)
        assert torch.isnan(out[2]).all()


@pytest.mark.gpu
def test_head_extreme_scales(ssb):
    """Powers of two over the range that bfloat16 has as normal numbers, and integer scales down to its subnormals."""
    V, H = 16, 64
    n = np.full((V, H), 2, np.int64)  # 1.0 in E2M1, 2 as an integer
    x = np.tile(np.array([[2, 3, 20, 60, 100, 126, 127, 128, 150, 180, 200, 220, 240, 250, 251, 247]], np.uint8).T, (1, 4))
    h = torch.ones(1, H, dtype=BF16)
    out = ssb.head_w4(h.cuda(), ssb.W4(torch.from_numpy(pack(n, "mx")).cuda(), torch.from_numpy(x).cuda(), V, H, "mx", 32),
                      dtype=F32)
    with np.errstate(over="ignore"):  # 64 * 2^123 and 64 * 2^124 are infinities in float32, as in the result
        assert np.array_equal(out.cpu().numpy()[0], (H * np.exp2(x[:, 0].astype(np.float64) - 127)).astype(np.float32))
    s = torch.from_numpy(np.exp2(np.linspace(-133, 110, V).round())).to(BF16)[:, None].repeat(1, 2)
    out = ssb.head_w4(h.cuda(), ssb.W4(torch.from_numpy(pack(n, "int")).cuda(), s.cuda(), V, H, "int", 64), dtype=F32)
    assert np.array_equal(as64(out)[0], as64(s)[:, 0] * 2 * H)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_lookup_against_64_bits(ssb, dtype, out_dtype):
    rng = np.random.default_rng(5)
    for T, V, H, extra, shift in [(1, 1, 1, 0, 0), (5, 7, 8, 0, 0), (9, 33, 100, 3, 1), (64, 50, 2048, 0, 0),
                                  (33, 1000, 2049, 0, 0), (300, 20, 4104, 8, 8), (2, 3, 5000, 1, 3)]:
        table = torch.from_numpy(rng.normal(0, 1, (V, H)).astype(np.float32)).to(dtype)
        tok = rng.integers(0, V, T).astype(np.int32)
        tok[rng.random(T) < 0.2] = -1
        tok[-1] = V - 1
        if T > 3:
            tok[:3] = V, 2 ** 31 - 1, -2 ** 31
        say(f"[lookup] {dtype}->{out_dtype} T={T} V={V} H={H} extra={extra}")
        tt, _ = strided(table, extra, shift)
        out, base = strided(torch.zeros(T, H, dtype=out_dtype), extra, shift)
        ssb.embed(torch.from_numpy(tok).cuda(), tt, scale=1.5, out=out)
        there = (tok >= 0) & (tok < V)
        ref = np.where(there[:, None], as64(table)[np.where(there, tok, 0)] * 1.5, 0)
        # one product rounded to float32, one rounding to the output
        assert (np.abs(as64(out) - ref) <= np.abs(ref) * (U[out_dtype] + 2.0 ** -24 * (1 + U[out_dtype]))).all()
        rest = base[shift:shift + T * (H + extra)].view(T, H + extra)[:, H:]
        assert (rest == 77).all() and (base[:shift] == 77).all() and (base[shift + T * (H + extra):] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", KINDS)
def test_lookup_in_4_bits(ssb, fmt, group):
    rng = np.random.default_rng(6)
    for T, V, H, out_dtype in [(1, 1, group, F32), (40, 9, 3 * 128 + group % 128, BF16), (300, 77, 4096, F32),
                               (5, 600, 2944, BF16)]:
        codes, scales, W = random_table(rng, V, H, fmt, group)
        table = ssb.W4(codes.cuda(), scales.cuda(), V, H, fmt, group)
        tok = rng.integers(-2, V + 2, T).astype(np.int32)
        say(f"[lookup] {fmt}{group} T={T} V={V} H={H}")
        out = ssb.embed(torch.from_numpy(tok).cuda(), table, scale=0.3, dtype=out_dtype)
        there = (tok >= 0) & (tok < V)
        ref = np.where(there[:, None], W[np.where(there, tok, 0)] * float(np.float32(0.3)), 0)
        assert (np.abs(as64(out) - ref) <= np.abs(ref) * (U[out_dtype] + 2.0 ** -24 * (1 + U[out_dtype]))).all()


def grad64(dout, tok, V, scale):
    ref, S, n = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1])), np.zeros(V)
    for t, v in enumerate(tok):
        if 0 <= v < V:
            ref[v] += dout[t] * scale
            S[v] += np.abs(dout[t] * scale)
            n[v] += 1
    return ref, S, n


@pytest.mark.gpu
def test_offsets_beyond_32_bits(ssb):
    """Tables, gradients and logits of more than 4 GB: their last rows, against the same rows of a small call."""
    g = torch.Generator(device="cuda")
    g.manual_seed(15)
    V, H = 560000, 4096
    say("[4 GB] lookup")
    table = torch.zeros(V, H, dtype=BF16, device="cuda")
    table[-40:].normal_(generator=g)
    tok = torch.tensor([V - 1, 5, V - 40, V, V - 7], dtype=torch.int32, device="cuda")
    out = ssb.embed(tok, table)
    assert torch.equal(out[[0, 2, 4]], table[[V - 1, V - 40, V - 7]]) and not out[[1, 3]].any()
    say("[4 GB] gradient")
    d = torch.empty(5, H, device="cuda").normal_(generator=g)
    dW = torch.full((V, H), 3.0, device="cuda")
    ssb.embed_grad(d, tok, V, out=dW)
    assert torch.equal(dW[[V - 1, 5, V - 40, V - 7]], d[[0, 1, 2, 4]])
    dW[[V - 1, 5, V - 40, V - 7]] = 0
    assert int(torch.count_nonzero(dW)) == 0
    del table, dW
    say("[4 GB] quantiser, head, lookup in 4 bits")
    V, H = 1 << 20, 8704
    w = torch.zeros(V, H, dtype=BF16, device="cuda")
    w[-100:].normal_(generator=g)
    t = ssb.quantize_w4(w, fmt="mx", group=32)
    small = ssb.quantize_w4(w[-100:].contiguous(), fmt="mx", group=32)
    assert torch.equal(t.codes[-100:], small.codes) and torch.equal(t.scales[-100:], small.scales)
    del w
    for T in (2, 20):
        h = torch.empty(T, H, dtype=BF16, device="cuda").normal_(generator=g)
        big, few = ssb.head_w4(h, t, dtype=F32), ssb.head_w4(h, small, dtype=F32)
        # a sum of one row's products in another order
        assert (big[:, -100:] - few).abs().max() <= (32 + H / 32 + 24) * 2.0 ** -22 * 6 * H
        assert int(torch.count_nonzero(big[:, :-100])) == 0 and big[:, -100:].abs().min() > 0
    tok = torch.arange(V - 100, V, dtype=torch.int32, device="cuda")
    assert torch.equal(ssb.embed(tok, t), ssb.embed(tok - (V - 100), small))
    del t, big, few
    say("[4 GB] logits")
    T, H = 2300, 32
    w = torch.empty(V, H, dtype=BF16, device="cuda").normal_(generator=g)
    t = ssb.quantize_w4(w, fmt="int", group=32)
    h = torch.empty(T, H, dtype=BF16, device="cuda").normal_(generator=g)
    big = ssb.head_w4(h, t)
    small = ssb.W4(t.codes[-64:].clone(), t.scales[-64:].clone(), 64, H, "int", 32)
    assert torch.equal(big[-30:, -64:], ssb.head_w4(h[-30:], small))


GRAD = [
    # T, V, H, how the tokens fall
    (0, 5, 16, "even"), (1, 1, 1, "even"), (1, 300, 8, "even"), (7, 513, 60, "even"), (128, 4, 64, "even"),
    (129, 2, 72, "one"), (500, 257, 100, "few"), (1000, 700, 40, "zipf"), (1000, 3, 2056, "few"), (640, 256, 33, "blocks"),
    (3000, 40, 24, "zipf"), (2500, 1, 16, "one"), (300, 600, 16, "none"), (900, 300, 2052, "runs"), (809, 220, 4100, "short"), (1025, 1025, 8, "even"), (5000, 9000, 16, "sorted"),
    (200100, 500, 8, "even"),
]


def grad_tokens(rng, T, V, how):
    if how == "one":
        return np.full(T, V - 1, np.int32)
    if how == "none":
        return rng.choice(np.array([-1, V, 2 ** 31 - 1, -2 ** 31], np.int64), T).astype(np.int32)
    if how == "few":
        tok = rng.integers(0, min(V, 3), T)
    elif how == "zipf":
        tok = np.minimum((np.exp(rng.random(T) * np.log(V + 1)) - 1).astype(np.int64), V - 1)
    elif how == "short":  # runs of 32 and its neighbours
        tok = np.repeat(np.arange(20) * 11, [32, 33, 31, 1, 32, 32, 33, 33, 2, 62, 96, 97, 5, 31, 33, 64, 65, 32, 32, 63])[:T]
    elif how == "runs":  # of 64 and its neighbours, and twice that
        tok = np.repeat(np.arange(12) * 25, [64, 1, 63, 65, 64, 128, 2, 129, 127, 64, 65, 128])[:T]
    elif how == "blocks":  # runs of exactly 128 and its neighbours
        tok = np.repeat(np.arange(5), [128, 129, 127, 128, 128])[:T]
    else:
        tok = rng.integers(0, V, T)
    if how == "sorted":
        tok = np.sort(tok)
    tok = tok.astype(np.int32)
    if how not in ("blocks", "runs", "short"):
        tok[rng.random(T) < 0.1] = -1
    return tok


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_gradient_against_64_bits(ssb, dtype, out_dtype):
    rng = np.random.default_rng(7)
    for i, (T, V, H, how) in enumerate(GRAD):
        dout = torch.from_numpy(rng.normal(0, 1, (T, H)).astype(np.float32)).to(dtype)
        tok = grad_tokens(rng, T, V, how)
        extra, shift = (0, 0) if i % 2 else (3, 1)
        say(f"[grad] {dtype}->{out_dtype} T={T} V={V} H={H} {how} extra={extra}")
        ref, S, n = grad64(as64(dout), tok, V, 0.75)
        slack = (n[:, None] + 2) * 2.0 ** -24 * S
        ds, _ = strided(dout, extra, shift)
        t = torch.from_numpy(tok).cuda()
        out, base = strided(torch.full((V, H), 5.0, dtype=out_dtype), extra, shift)
        ssb.embed_grad(ds, t, V, scale=0.75, out=out)
        err = np.abs(as64(out) - ref)
        tol = slack * (1 + U[out_dtype]) + U[out_dtype] * np.abs(ref)
        assert (err <= tol).all(), (T, V, H, how)
        rest = base[shift:shift + V * (H + extra)].view(V, H + extra)[:, H:]
        assert (rest == 77).all() and (base[:shift] == 77).all() and (base[shift + V * (H + extra):] == 77).all()
        # the same call, the same bits; added to what is there, the rows without a token untouched
        again = ssb.embed_grad(ds, t, V, scale=0.75, dtype=out_dtype)
        assert torch.equal(again, out)
        start = torch.from_numpy(rng.normal(0, 1, (V, H)).astype(np.float32)).to(out_dtype)
        start[n == 0] = float("nan")
        acc = start.cuda()
        ssb.embed_grad(ds, t, V, scale=0.75, out=acc, accumulate=True)
        keep = torch.from_numpy(n == 0)
        assert torch.isnan(acc.cpu()[keep]).all()
        sum64 = as64(start)[n > 0] + ref[n > 0]
        tol = ((slack[n > 0] + 2.0 ** -24 * np.abs(sum64)) * (1 + U[out_dtype]) + U[out_dtype] * np.abs(sum64)) * (1 + 2 ** -20)
        assert (np.abs(as64(acc)[n > 0] - sum64) <= tol).all(), (T, V, H, how)


@pytest.mark.gpu
def test_gradient_is_the_lookups(ssb):
    """<lookup(W + E) - lookup(W), d> = <E, gradient(d)>: the lookup is linear, so the difference is exact but for
    rounding (small integers: none at all)."""
    rng = np.random.default_rng(8)
    T, V, H = 400, 90, 96
    W, E = (torch.from_numpy(rng.integers(-8, 9, (V, H)).astype(np.float32)).cuda() for _ in range(2))
    d = torch.from_numpy(rng.integers(-8, 9, (T, H)).astype(np.float32)).cuda()
    tok = torch.from_numpy(grad_tokens(rng, T, V, "zipf")).cuda()
    diff = ssb.embed(tok, W + E, scale=0.5) - ssb.embed(tok, W, scale=0.5)
    assert float((diff.double() * d.double()).sum()) == float(
        (E.double() * ssb.embed_grad(d, tok, V, scale=0.5).double()).sum())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", KINDS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantiser_by_its_definition(ssb, fmt, group, dtype):
    rng = np.random.default_rng(9)
    for V, H, extra, shift in [(1, group, 0, 0), (50, 3 * 128 + group % 128, 3, 1), (257, 1024, 8, 8), (3, 4096, 0, 0)]:
        w = rng.normal(0, 0.02, (V, H)).astype(np.float32)
        if V >= 50:
            w[3] = 0
            w[4, : group] = 1e-44
            w[5] *= 1e-36
            w[6] *= 1e38
            w[7] *= np.exp2(-100.0).astype(np.float32)
            w[8, 5], w[9, H - 1], w[10, 0] = np.nan, np.inf, -np.inf
            # ties: halves of a scale of one, and numbers next to them
            w[11] = rng.choice(np.arange(-7, 7.5, 0.5), H)
            w[11, ::group] = 7
            w[12] = np.nextafter(w[11], np.float32(100))
            w[12, ::group] = 7
            w[13] = np.nextafter(w[11], np.float32(-100))
            w[13, ::group] = 7
            w[14] = rng.choice(np.array([0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.9], np.float32), H)
            w[15] = -np.abs(w[15])
            w[16] = rng.integers(-200, 200, H) * np.float32(0.37)
        w = torch.from_numpy(w).to(dtype)
        n, s = quantise(w.double().numpy(), fmt, group)
        ws, _ = strided(w, extra, shift)
        for values_dtype in (None, F32, BF16):
            say(f"[quant] {fmt}{group} {dtype} V={V} H={H} values={values_dtype}")
            table = ssb.W4.empty(V, H, fmt, group)
            table.codes.fill_(0x55)
            values, base = (None, None) if values_dtype is None else strided(torch.zeros(V, H, dtype=values_dtype), extra, shift)
            assert ssb.quantize_w4(ws, table, values=values) is table
            assert np.array_equal(table.codes.cpu().numpy(), pack(n, fmt)), np.nonzero((table.codes.cpu().numpy() != pack(n, fmt)).any(1))
            got = table.scales.cpu()
            got = np.where(got.numpy() == 255, np.nan, np.exp2(got.double().numpy() - 127)) if fmt == "mx" else as64(got)
            assert np.array_equal(got[:, : H // group], s, equal_nan=True)
            if values is not None:
                exact = torch.from_numpy(numbers(n, fmt) * np.repeat(s, group, 1))
                assert torch.equal(torch.nan_to_num(values.cpu().double(), nan=9e9), torch.nan_to_num(
                    exact.float().to(values_dtype).double(), nan=9e9))
                rest = base[shift:shift + V * (H + extra)].view(V, H + extra)[:, H:]
                assert (rest == 77).all()
        new = ssb.quantize_w4(ws, fmt=fmt, group=group)
        assert torch.equal(new.codes, table.codes)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", KINDS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_written_over_the_weights(ssb, fmt, group, dtype):
    """`values` may be the weights themselves: the table and the numbers of a call with another array."""
    g = torch.Generator(device="cuda").manual_seed(17)
    for V, H, extra in ((37, 160, 0), (50, 4096, 8), (9, 2944, 3)):
        H = (H + group - 1) // group * group
        w, _ = strided(torch.empty(V, H, dtype=dtype, device="cuda").normal_(0, 0.02, generator=g), extra)
        apart = torch.empty(V, H, dtype=dtype, device="cuda")
        want = ssb.quantize_w4(w, fmt=fmt, group=group, values=apart)
        got = ssb.quantize_w4(w, fmt=fmt, group=group, values=w)
        assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales) and torch.equal(w, apart)


@pytest.mark.gpu
def test_wrappers_refuse_on_the_gpu(ssb):
    t = ssb.W4.empty(64, 256, "int", 128)
    h = torch.zeros(4, 256, dtype=BF16, device="cuda")
    tok = torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in [lambda: ssb.head_w4(h[:, :128], t), lambda: ssb.head_w4(h.half(), t),
                 lambda: ssb.head_w4(h, t, out=torch.zeros(4, 63, dtype=BF16, device="cuda")),
                 lambda: ssb.head_w4(h, t, out=torch.zeros(64, 4, dtype=BF16, device="cuda").t()),
                 lambda: ssb.head_w4(h, t, ws=torch.zeros(16, dtype=torch.uint8, device="cuda")),
                 lambda: ssb.embed(tok[::2], t), lambda: ssb.embed(tok.long(), t),
                 lambda: ssb.embed(tok, t, out=torch.zeros(4, 256, dtype=torch.float16, device="cuda")),
                 lambda: ssb.embed_grad(h, tok[:3], 10), lambda: ssb.embed_grad(h, tok, 10, accumulate=True),
                 lambda: ssb.embed_grad(h, tok, 10, ws=torch.zeros(16, dtype=torch.uint8, device="cuda")),
                 lambda: ssb.quantize_w4(h, t), lambda: ssb.quantize_w4(h[:, :100], fmt="mx", group=32)]:
        with pytest.raises(ssb.SSError):
            call()


@pytest.mark.gpu
def test_no_rows(ssb):
    t = ssb.W4.empty(64, 256, "int", 128)
    e = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert ssb.head_w4(torch.zeros(0, 256, dtype=BF16, device="cuda"), t).shape == (0, 64)
    assert ssb.embed(e, t).shape == (0, 256)
    out = torch.full((10, 256), 3.0, device="cuda")
    ssb.embed_grad(torch.zeros(0, 256, device="cuda"), e, 10, out=out, accumulate=True)
    assert (out == 3).all()
    ssb.embed_grad(torch.zeros(0, 256, device="cuda"), e, 10, out=out)
    assert (out == 0).all()


def loop_inputs(ssb, B, V, H, fmt, group):
    """A table, its 4-bit form, and sampling parameters: greedy and stochastic requests side by side."""
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    W = torch.empty(V, H, dtype=BF16, device="cuda").normal_(0, 0.05, generator=g)
    mode = torch.where(torch.arange(B, device="cuda") % 2 == 0, ssb.GREEDY, ssb.TEMP | ssb.TOPK).to(torch.int32)
    prm = ssb.Params(B, V, mode=mode, temperature=torch.full((B,), 0.7, device="cuda"),
                     top_k=torch.full((B,), 20, dtype=torch.int32, device="cuda"),
                     seed=torch.arange(B, device="cuda"), position=torch.zeros(B, dtype=torch.int64, device="cuda"))
    return W, ssb.quantize_w4(W, fmt=fmt, group=group), prm


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group,B", [("int", 128, 8), ("mx", 32, 24)])
def test_decode_loop_eager_and_replayed(ssb, fmt, group, B):
    """Lookup, (an identity for the model,) head, sampler, and again; the loop captured in a graph gives the same
    tokens on every replay, with eager work between them."""
    V, H, steps = 3000, 512, 3
    W, table, prm = loop_inputs(ssb, B, V, H, fmt, group)
    first = torch.arange(B, dtype=torch.int32, device="cuda") * 7
    ws = ssb.workspace(ssb.OP_SAMPLE, B, V, 0, 64, ssb.F32)
    hws = ssb.head_workspace(torch.empty(B, H, dtype=BF16, device="cuda"))
    logits = [torch.empty(B, V, device="cuda") for _ in range(steps)]

    def loop():
        tok, seen = first, []
        for s in range(steps):
            x = ssb.embed(tok, table, scale=4.0)
            ssb.head_w4(x, table, out=logits[s], ws=hws)
            tok = ssb.sample(logits[s], prm, 64, ws=ws)[0]
            seen.append(tok)
        return seen

    say(f"[loop] eager {fmt}{group} B={B}")
    want = [t.clone() for t in loop()]
    torch.cuda.synchronize()
    table64 = as64(ssb.embed(torch.arange(V, dtype=torch.int32, device="cuda"), table, dtype=F32))
    tok = first.cpu().numpy()
    for s in range(steps):  # greedy rows: the leading logit of the 64-bit product, up to its rounding
        x = as64((torch.from_numpy(table64[tok] * 4)).to(BF16))
        ref = x @ table64.T
        got = want[s].cpu().numpy()
        for b in range(0, B, 2):
            assert ref[b, got[b]] >= ref[b].max() - 1e-4 * np.abs(ref[b]).max()
        tok = got
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loop()
    torch.cuda.current_stream().wait_stream(side)
    say("[loop] capture")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = loop()
    for rep in range(3):
        say(f"[loop] replay {rep}")
        for t in got:
            t.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        eager = loop()
        assert all(torch.equal(a, b) for a, b in zip(want, eager))


@pytest.mark.gpu
def test_verification_takes_the_heads_logits(ssb):
    """Draft rows through the head into ss_verify_sparse; its padded tokens through the lookup."""
    B, L, V, H = 4, 3, 2500, 384
    W, table, _ = loop_inputs(ssb, B, V, H, "int", 64)
    prm = ssb.Params(B, V, mode=torch.full((B,), ssb.GREEDY, dtype=torch.int32, device="cuda"),
                     seed=torch.arange(B, device="cuda"), position=torch.zeros(B, dtype=torch.int64, device="cuda"))
    h = torch.empty(B * (L + 1), H, dtype=BF16, device="cuda").normal_()
    logits = ssb.head_w4(h, table)
    best = logits.float().argmax(1).view(B, L + 1)
    draft = best[:, :L].clone()
    draft[1, 1] = (draft[1, 1] + 1) % V  # request 1 is rejected at its second draft
    tokens, n, _ = ssb.verify_sparse(logits.view(B, L + 1, V), draft[:, :, None].int().contiguous(),
                                     torch.ones(B, L, 1, device="cuda"), draft.int().contiguous(), prm, 64)
    assert n.tolist() == [3, 1, 3, 3]
    rows = ssb.embed(tokens.view(-1), table, dtype=F32).view(B, L + 1, H)
    assert (rows[1, 2:] == 0).all() and (rows[1, :2].abs().sum(1) > 0).all()
    want = ssb.embed(best.int().view(-1), table, dtype=F32).view(B, L + 1, H)
    assert torch.equal(rows[0], want[0]) and torch.equal(rows[1, :2], want[1, :2])


@pytest.mark.gpu
def test_training_step_refreshes_the_serving_table(ssb):
    """Gradient, update, new 4-bit form: all captured, replayed twice; a plain 64-bit step beside it."""
    T, V, H = 300, 400, 256
    rng = np.random.default_rng(13)
    W0 = torch.from_numpy(rng.normal(0, 0.05, (V, H)).astype(np.float32))
    W = W0.cuda()
    tok = grad_tokens(rng, T, V, "zipf")
    t = torch.from_numpy(tok).cuda()
    d = torch.from_numpy(rng.normal(0, 0.01, (T, H)).astype(np.float32))
    dd = d.cuda()
    table = ssb.W4.empty(V, H, "mx", 32)
    gws, dW = ssb.embed_grad_workspace(T, V, H), torch.empty(V, H, device="cuda")

    def step():
        ssb.embed_grad(dd, t, V, scale=2.0, out=dW, ws=gws)
        W.sub_(dW)
        ssb.quantize_w4(W, table)
        return ssb.embed(t, table, scale=2.0, dtype=F32)

    step()
    torch.cuda.synchronize()
    W.copy_(W0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    ref = as64(W0)
    g64 = grad64(as64(d), tok, V, 2.0)[0]
    for rep in range(3):
        graph.replay()
        torch.cuda.synchronize()
        ref = ref - g64
        assert np.abs(as64(W) - ref).max() <= 1e-5 * max(1, np.abs(ref).max())
        n, s = quantise(W.cpu().numpy().astype(np.float64), "mx", 32)
        vals = numbers(n, "mx") * np.repeat(s, 32, 1)
        there = tok >= 0
        assert np.array_equal(as64(out), np.where(there[:, None], vals[np.where(there, tok, 0)] * 2, 0))
        torch.zeros(1000, device="cuda").sum()


@pytest.mark.gpu
def test_two_streams_with_their_own_workspaces(ssb):
    rng = np.random.default_rng(14)
    V, H = 5000, 1024
    codes, scales, _ = random_table(rng, V, H, "int", 128)
    table = ssb.W4(codes.cuda(), scales.cuda(), V, H, "int", 128)
    hs = [torch.empty(T, H, device="cuda").normal_() for T in (5, 40)]
    toks = [torch.randint(0, V, (700,), device="cuda", dtype=torch.int32) for _ in range(2)]
    ds = [torch.empty(700, H, device="cuda").normal_() for _ in range(2)]
    want = [(ssb.head_w4(h, table), ssb.embed_grad(d, t, V)) for h, d, t in zip(hs, ds, toks)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for rep in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = (ssb.head_w4(hs[i], table), ssb.embed_grad(ds[i], toks[i], V))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
