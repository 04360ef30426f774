"""Products with 4-bit weights and the 4-bit paged cache on values at the ends of their types, and at the ends of their
buffers; formats and bounds of tests/int4_ref.py."""
import numpy as np
import pytest
import torch

from paper_2602_18447_amd import binding as cb
from tests import int4_ref as R
from tests.test_gpu_int4 import DEV, Cache, Ctx, _append_case, _attn_check, _gen, _w4_case

pytestmark = pytest.mark.gpu
NAN_HALF = torch.tensor([0x7E00], dtype=torch.int16).view(torch.float16)[0]


# ---------------------------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("Hq, Hkv, L, S, n", [(4, 2, (13, 0), (12, 9), None), (1, 1, (5,), (12,), (10,)), (12, 3, (40, 7, 0), (1, 12, 30), (1, 11, 30))])
def test_append_a_row_with_a_nan_is_stored_as_nan(Hq, Hkv, L, S, n):
    """s and z are 0x7E00 and every code 0: the row reads back as NaN.  The other rows are what they are without it."""
    gen = _gen(50)
    c = Cache(gen, Hkv, L, S)
    x = torch.randn(c.T, Hq + 2 * Hkv, 128, generator=gen, device=DEV)
    nan, inf = float("nan"), float("inf")
    other = torch.tensor([-0x3FFFFF], dtype=torch.int32).view(torch.float32).item()             # with a sign and a payload
    k, v = x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    bad_k = torch.zeros(c.T, Hkv, dtype=torch.bool)
    bad_v = torch.zeros(c.T, Hkv, dtype=torch.bool)
    for bad, rows, t, h, at, value in ((bad_v, v, 1, 0, 7, nan), (bad_v, v, 3, Hkv - 1, 127, other), (bad_v, v, 4, 0, slice(None), nan), (bad_k, k, 2, 0, 3, nan),
                                       (bad_k, k, 4, Hkv - 1, 64, other), (bad_k, k, 5, 0, slice(None), nan), (bad_v, v, 10, 0, 0, nan), (bad_k, k, 11, Hkv - 1, 90, nan)):
        rows[t, h, at] = value
        bad[t, h] = True
    v[7, 0, 5], v[7, 0, 6], v[8, 0, 9] = inf, nan, -inf
    bad_v[7, 0] = True
    q, kk, vv = (torch.empty(c.T, h, 128, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv))
    kr, vr = (torch.empty(c.T, Hkv, 128, device=DEV) for _ in range(2))
    want = c.pages[0].cpu()
    hn = None if n is None else np.asarray(n, dtype=np.int32)
    dn = None if n is None else torch.from_numpy(hn).to(DEV)
    with Ctx(Hq, Hkv) as ctx:
        cb.confspec_op_kv4_append(ctx, c.kv, c.batch, 0, x, dn, hn, q, kk, vv, qkv_stride=(Hq + 2 * Hkv) * 128)
        cb.confspec_op_kv4_read(ctx, c.kv, c.batch, 0, kr, vr)
        torch.cuda.synchronize()
    assert torch.equal(torch.isnan(kk).any(-1).cpu(), bad_k) and torch.equal(torch.isnan(vv).any(-1).cpu(), bad_v)
    none = torch.zeros(128, dtype=torch.int64)
    for rows, bad, got, is_v in ((kk.cpu(), bad_k, kr.cpu(), False), (vv.cpu(), bad_v, vr.cpu(), True)):
        cc, ss, zz = R.quantise(torch.where(bad[..., None], torch.zeros_like(rows), rows))
        for b in range(len(L)):
            for i in range(S[b] if n is None else n[b]):
                t, row = int(c.cu[b]) + i, L[b] + i
                for h in range(Hkv):
                    stored = (none, NAN_HALF, NAN_HALF) if bad[t, h] else (cc[t, h], ss[t, h], zz[t, h])
                    R.write_row(want, int(c.table[b, row // 16]), h, row % 16, *stored, is_v)
                    assert bool(torch.isnan(got[t, h]).all()) if bad[t, h] else bool(torch.isfinite(got[t, h]).all()), (b, i, h)
    assert torch.equal(want, c.pages[0].cpu())


@pytest.mark.parametrize("L, S", [((40,), (1,)), ((40, 100), (3, 1)), ((5003, 60), (2, 40)), ((20,) * 6, (100,) * 6)])
@pytest.mark.parametrize("is_v", [False, True])
def test_attention_over_a_row_stored_as_nan(L, S, is_v):
    """Every row of its trace and head is NaN, and no other."""
    gen = _gen(51)
    Hq, Hkv, j = 40, 8, 19
    c = Cache(gen, Hkv, L, S)
    q = torch.randn(c.T, Hq, 128, generator=gen, device=DEV).bfloat16()
    k, v = (torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16() for _ in range(2))
    with Ctx(Hq, Hkv) as ctx:
        good = _attn_check(ctx, c, Hq, Hkv, q, k, v).view(c.T, Hq, 128)
        none = torch.zeros(128, dtype=torch.int64, device=DEV)
        R.write_row(c.pages[0], int(c.table[0, j // 16]), 3, j % 16, none, NAN_HALF.to(DEV), NAN_HALF.to(DEV), is_v)
        out = torch.empty(c.T, Hq, 128, dtype=torch.bfloat16, device=DEV)
        cb.confspec_op_kv4_attention(ctx, c.kv, c.batch, 0, q, k, v, out, c.scratch(ctx))
        torch.cuda.synchronize()
    seen = torch.zeros(c.T, Hq, dtype=torch.bool, device=DEV)
    seen[:S[0], 15:20] = True
    assert bool(torch.isnan(out[seen]).all()) and torch.equal(out[~seen], good[~seen])


def test_append_a_zero_has_no_sign():
    """Rows whose minimum or range rounds to a zero half from below: bytes as the plain form has them."""
    def edit(x, Hq, Hkv):
        for rows in (x[:, Hq + Hkv:], x[:1, Hq:Hq + Hkv]):             # (keys at position 0 are not turned)
            for t in range(rows.shape[0]):
                rows[t] = torch.rand(Hkv, 128, generator=_gen(t), device=DEV) * 1e-3
        v = x[:, Hq + Hkv:]
        v[0, :, 3] = -1e-9                                             # z from (-2^-25, 0)
        v[1, :, 100] = -2.0 ** -26
        v[2] = 1.5 * 2.0 ** -25                                        # z is 2^-24, beyond the maximum: s from below 0
        v[3] = -2.0 ** -26
        v[4] = -0.0
        v[5] = -1e-9
        v[5, :, 9] = 1e-9
        x[0, Hq:Hq + Hkv, 70] = -1e-9
    _append_case(3, 3, (0,), (6,), None, 52, edit=edit)


# ---------------------------------------------------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------------------------------------------------
W4_TILES = [(1, 48, 416, 32, 0), (4, 5136, 416, 32, 1), (7, 144, 1600, 64, 1), (16, 4112, 640, 128, 0), (12, 32, 160, 32, 2), (20, 272, 1088, 64, 0), (40, 2576, 640, 128, 1),
            (17, 8208, 416, 32, 0), (32, 4112, 1088, 64, 2), (48, 7200, 640, 128, 0), (70, 12304, 416, 32, 1), (100, 6160, 1088, 64, 0), (128, 12304, 640, 128, 0)]


@pytest.mark.parametrize("M, N, K, group, epi", W4_TILES)
def test_w4_infinite_activations(M, N, K, group, epi):
    """An infinity times a weight that is not 0 is an infinity: what the definition has, element by element."""
    gen = _gen(53)
    codes, s, z, w = R.w4_quantise_case(gen, N, K, group, DEV)
    a = torch.randn(M, K, generator=gen, device=DEV).bfloat16()
    inf = float("inf")
    a[0, 5] = inf
    if M > 3:
        a[1, K - 1], a[2, 9], a[2, K - 20], a[3, 33] = -inf, inf, inf, float("nan")
    if M > 16:
        a[16, K // 2] = -inf
    resid = torch.randn(M, N, generator=gen, device=DEV) if epi == cb.EPI_RESID_F32 else None
    packed = torch.empty(cb.confspec_w4_bytes(N, K, group), dtype=torch.uint8, device=DEV)
    out = torch.empty(M, N // 2, dtype=torch.bfloat16, device=DEV) if epi == cb.EPI_SWIGLU else torch.empty(M, N, device=DEV)
    with Ctx() as ctx:
        cb.confspec_w4_pack(ctx, codes, s, z, N, K, group, packed, gate_up=epi == cb.EPI_SWIGLU)
        cb.confspec_op_w4_gemm(ctx, a, packed, resid, out, M, N, K, group, epi)
    zero = torch.zeros_like(a)
    fin = torch.isfinite(a)
    y, tol = R.w4_gemm(torch.where(fin, a, zero), w, s, z, group)
    for m, k in torch.nonzero(~fin).tolist():
        y[m] += a[m, k].double() * w[:, k]                             # (an infinity, or NaN where the weight is 0)
    if epi == cb.EPI_SWIGLU:
        y, tol = R.swiglu(y, tol)
    elif epi == cb.EPI_RESID_F32:
        y = y + resid.double()
        tol = tol + 2.0 ** -24 * y.abs()
    got, fin = out.double(), torch.isfinite(y)
    assert not bool(fin[0].any()) and bool(torch.isinf(y[0]).any())
    assert bool(((got - y).abs() <= tol)[fin].all())
    assert torch.equal(torch.isnan(got), torch.isnan(y)) and torch.equal(got[torch.isinf(y)], y[torch.isinf(y)])


@pytest.mark.parametrize("M, N, K, group, epi", [c for c in W4_TILES if c[4] != 2])
def test_w4_activations_near_the_largest(M, N, K, group, epi):
    """31 times an activation and its sums pass the range of fp32, the result does not."""
    _w4_case(M, N, K, group, epi, 54, scale_a=1e37)


# ---------------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("Hq, Hkv, L, S", [(4, 2, (50, 3), (100, 2)), (12, 2, (5003,), (70,)), (40, 8, (20,) * 6, (100,) * 6), (4, 4, (0,), (300,)), (8, 1, (0, 33), (1, 33)),
                                           (40, 8, (0,) * 4, (200,) * 4)])
@pytest.mark.parametrize("weights", ["even", "first_alone", "context_alone"])
def test_attention_infinite_values_of_tokens_seen(Hq, Hkv, L, S, weights):
    """A weight is positive, so a column with an infinity is that infinity, with both of them or a NaN it is NaN: in every row that
    sees the token, however many tokens later and however small the weight is in fp32."""
    gen = _gen(55)
    c = Cache(gen, Hkv, L, S)
    q = torch.randn(c.T, Hq, 128, generator=gen, device=DEV)
    k = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV)
    v = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    last = Hkv - 1
    n = S[0]
    bad = [(0, 5, float("inf")), (0, 77, -float("inf")), (n // 3, 40, float("inf")), (n // 2, 41, -float("inf")), (n - 1, 77, float("inf")), (n // 4, 100, float("nan")),
           (n // 4, 5, float("inf"))]
    if weights == "first_alone":                                       # the others' weights are 2^-400 of the first token's
        q, k = torch.zeros_like(q), torch.zeros_like(k)
        q[..., 0], k[..., 0], k[0, :, 0] = 40.0, -40.0, 40.0
        if n > 4:
            k[1, :, 0], bad[0] = 40.0, (2, 5, float("inf"))
    elif weights == "context_alone":                                   # and here the context's largest scores are far above
        q, k = q * 60.0, k * 0.0
    q, k = q.bfloat16(), k.bfloat16()
    want = torch.zeros(c.T, 128, dtype=torch.float64, device=DEV)
    with Ctx(Hq, Hkv) as ctx:
        outs = []
        for put in (False, True):
            for (t, col), value in {(t, col): value for t, col, value in bad}.items() if put else ():
                v[t, last, col] = value
                want[t:n, col] += value
            out = torch.empty(c.T, Hq, 128, dtype=torch.bfloat16, device=DEV)
            cb.confspec_op_kv4_attention(ctx, c.kv, c.batch, 0, q, k, v, out, c.scratch(ctx))
            outs.append(out.double())
        torch.cuda.synchronize()
    want = want[:, None].expand(-1, Hq, -1).clone()
    want[:, :last * (Hq // Hkv)] = 0.0
    plain = want == 0.0
    assert torch.equal(outs[1][plain], outs[0][plain]) and bool(torch.isfinite(outs[0]).all())
    assert torch.equal(torch.isnan(outs[1]), torch.isnan(want))
    sure = torch.isinf(want)
    assert torch.equal(outs[1][sure], want[sure])


# ---------------------------------------------------------------------------------------------------------------------
# the largest calls, and what lies behind the buffers
# ---------------------------------------------------------------------------------------------------------------------
def test_read_of_the_largest_batch():
    """2^22 tokens of 25 heads, whose rows lie in two pages over and over."""
    T, Hkv = 1 << 22, 25
    if torch.cuda.mem_get_info()[0] < 125e9:
        pytest.skip("needs 125 GB of free device memory")
    pages = R.random_pages(_gen(56), 1, 2, Hkv, DEV)
    cu, lens = np.asarray([0, T], dtype=np.int32), np.asarray([0], dtype=np.int32)
    table = (torch.arange(T // 16, device=DEV, dtype=torch.int32) % 2).view(1, -1).contiguous()
    d = [torch.from_numpy(cu).to(DEV), torch.from_numpy(lens).to(DEV), torch.zeros(T, dtype=torch.int32, device=DEV)]
    kv = cb.make_kv4(pages, table, 2, 16, T // 16)
    batch, keep = cb.make_batch(d[2], d[0], d[1], cu, lens)
    k, v = (torch.empty(T, Hkv, 128, device=DEV) for _ in range(2))
    k[-1] = v[-1] = float("nan")
    with Ctx(Hkv, Hkv) as ctx:
        cb.confspec_op_kv4_read(ctx, kv, batch, 0, k, v)
        torch.cuda.synchronize()
    for got, (codes, s, z) in zip((k, v), R.read_pages(pages[0].reshape(-1, R.PAGE))):
        want = (z[..., None] + s[..., None] * codes).float().view(2, Hkv, 16, 128).transpose(1, 2).reshape(32, Hkv, 128)
        for part in got.view(-1, 32, Hkv, 128).split(1 << 13):
            assert bool((part == want).all())
    del k, v, got, part
    torch.cuda.empty_cache()


@pytest.mark.parametrize("Hq, Hkv, L, S", [(12, 2, (2048,), (1,)), (12, 2, (3000, 70, 900), (1, 5, 3)), (40, 8, (4000,) * 9, (1,) * 9), (6, 1, (9000, 17), (150, 3)), (34, 2, (70,) * 12, tuple(range(30, 54, 2)))])
def test_nothing_is_written_behind_the_buffers(Hq, Hkv, L, S):
    """Scratch of exactly the size asked for and every output, with bytes behind them that stay as they were."""
    gen = _gen(57)
    c = Cache(gen, Hkv, L, S)
    width = (Hq + 2 * Hkv) * 128
    qkv = torch.randn(c.T, width, generator=gen, device=DEV)
    guard = 4096

    def room(n_bytes):
        return torch.full((n_bytes + guard,), 0xA5, dtype=torch.uint8, device=DEV)

    rows = c.T * 128
    with Ctx(Hq, Hkv) as ctx:
        need = cb.confspec_op_kv4_attention_scratch_bytes(ctx, c.batch)
        sizes = dict(q=2 * rows * Hq, k=2 * rows * Hkv, v=2 * rows * Hkv, out=2 * rows * Hq, kr=4 * rows * Hkv, vr=4 * rows * Hkv, scratch=need)
        buf = {name: room(n) for name, n in sizes.items()}
        cb.confspec_op_kv4_append(ctx, c.kv, c.batch, 0, qkv, None, None, buf["q"], buf["k"], buf["v"], qkv_stride=width)
        cb.confspec_op_kv4_read(ctx, c.kv, c.batch, 0, buf["kr"], buf["vr"])
        cb.confspec_op_kv4_attention(ctx, c.kv, c.batch, 0, buf["q"], buf["k"], buf["v"], buf["out"], buf["scratch"][:need] if need else None)
        torch.cuda.synchronize()
    for name, n in sizes.items():
        assert bool((buf[name][n:] == 0xA5).all()), name
    q, k, v = (buf[name][:sizes[name]].view(torch.bfloat16).view(c.T, -1, 128) for name in ("q", "k", "v"))
    ref, tol = R.attention(c.pages[0], c.table, q, k, v, c.cu, c.lens, Hq, Hkv)
    got = buf["out"][:sizes["out"]].view(torch.bfloat16).view(c.T, Hq * 128).double()
    assert bool(((got - ref).abs() <= tol).all())


@pytest.mark.parametrize("N, K, group, gate_up", [(16, 32, 32, False), (48, 416, 32, True), (144, 1600, 64, False), (272, 640, 128, True)])
def test_pack_writes_its_bytes_and_no_other(N, K, group, gate_up):
    codes, s, z, _ = R.w4_quantise_case(_gen(58), N, K, group, DEV)
    n = cb.confspec_w4_bytes(N, K, group)
    first, second = (torch.full((n + 4096,), fill, dtype=torch.uint8, device=DEV) for fill in (0x00, 0xFF))
    with Ctx() as ctx:
        for dst in (first, second):
            cb.confspec_w4_pack(ctx, codes, s, z, N, K, group, dst[:n], gate_up=gate_up)
    assert torch.equal(first[:n], second[:n])
    assert bool((first[n:] == 0x00).all()) and bool((second[n:] == 0xFF).all())
