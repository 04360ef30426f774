"""What a generation step in 4 bits is made of, as cases to be timed: products of a few rows with 4-bit weights, the
append of rotated keys and values to a paged cache held in 4 bits (and the rows read back), and the attention over it.

Shapes are those of the two models of the benchmark (width 1536, 12 query heads on 2 key/value heads; width 5120, 40 on 8)
and generic ones around them; a head has 128 elements, a cache block 16 tokens.

Formats.  A weight is s * (c - z) with a code c of 4 bits and half-precision s, z for every group of 32, 64 or 128 along k.
A cache row (token, head) is z + s * c with half-precision s, z of its own.  A page of the cache holds 16 tokens of one
head in 2176 bytes: key codes, value codes, (s, z) of the keys, (s, z) of the values; `_pack_pages` writes it out.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
HD, BLOCK, PAGE = 128, 16, 2176
THETA = 1.0e6
STORE, RESID, SWIGLU = 0, 1, 2
HEADS = ((12, 2), (40, 8), (8, 8), (16, 4), (16, 1), (6, 3))


def listed():
    return [
        # output projection of the small model, one user's token: the smallest product, all latency
        dict(name="w4_small_out_m1", do="w4", M=1, N=1536, K=1536, group=128, epi=RESID),
        # gate/up projection of the large model, one token
        dict(name="w4_large_gate_up_m1", do="w4", M=1, N=55296, K=5120, group=128, epi=SWIGLU),
        # down projection of the large model, eight traces, fine groups
        dict(name="w4_large_down_m8", do="w4", M=8, N=5120, K=27648, group=64, epi=RESID),
        # QKV projection of the large model on a batch of drafted tokens
        dict(name="w4_large_qkv_m72", do="w4", M=72, N=7168, K=5120, group=32, epi=STORE),
        # one user's token joins the cache of the small model
        dict(name="append_one", do="append", Hq=12, Hkv=2, B=1, L_lo=2048, L_hi=2048, S_lo=1, S_hi=1, partial=False),
        # a serving batch of the large model, one token each, contexts of any length
        dict(name="append_b64_token", do="append", Hq=40, Hkv=8, B=64, L_lo=100, L_hi=16384, S_lo=1, S_hi=1, partial=False),
        # verified steps of which a part is accepted, far into a long chain of thought
        dict(name="append_steps_partial", do="append", Hq=12, Hkv=2, B=32, L_lo=30000, L_hi=40000, S_lo=17, S_hi=128, partial=True),
        # a chunk of prefill on the large model
        dict(name="append_prefill", do="append", Hq=40, Hkv=8, B=8, L_lo=0, L_hi=777, S_lo=512, S_hi=512, partial=False),
        # one user's token on a context of ordinary length
        dict(name="attn_one", do="attn", Hq=12, Hkv=2, B=1, L_lo=2048, L_hi=2048, S_lo=1, S_hi=1),
        # a full serving batch of the large model, one token each, long contexts of uneven length
        dict(name="attn_b48_long", do="attn", Hq=40, Hkv=8, B=48, L_lo=2000, L_hi=16384, S_lo=1, S_hi=1),
        # a few drafted tokens in every trace
        dict(name="attn_b32_drafts", do="attn", Hq=12, Hkv=2, B=32, L_lo=500, L_hi=8192, S_lo=1, S_hi=7),
        # verification of whole steps
        dict(name="attn_b16_steps", do="attn", Hq=12, Hkv=2, B=16, L_lo=512, L_hi=8192, S_lo=32, S_hi=256),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))

    do = rng.choice(("w4", "append", "attn"))
    top = max(_price(c) for c in listed() if c["do"] == do)
    while True:
        if do == "w4":
            group = rng.choice((32, 64, 128))
            c = dict(do=do, M=log_int(1, 128), N=16 * log_int(8, 3456), K=group * max(1, log_int(256, 27648) // group), group=group,
                     epi=rng.choice((STORE, RESID, SWIGLU)))
        else:
            Hq, Hkv = rng.choice(HEADS)
            L_hi = log_int(1, 16384 if do == "attn" else 40000)
            L_lo = L_hi if rng.random() < 0.25 else int(L_hi * rng.uniform(0.0, 0.9))
            S_hi = rng.choice((1, log_int(2, 8), log_int(9, 256)))
            S_lo = S_hi if rng.random() < 0.3 else max(1, int(S_hi * rng.uniform(0.1, 0.9)))
            c = dict(do=do, Hq=Hq, Hkv=Hkv, B=log_int(1, 64), L_lo=L_lo, L_hi=L_hi, S_lo=S_lo, S_hi=S_hi)
            if do == "append":
                c["partial"] = rng.random() < 0.5
        if _price(c) <= top:
            return c


# ---------------------------------------------------------------------------------------------------------------------
# what follows from the case alone
# ---------------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Context lengths, suffix lengths and appended counts of the traces."""
    r = random.Random("lengths" + repr(sorted((k, v) for k, v in case.items() if k != "name")))
    L = [r.randint(case["L_lo"], case["L_hi"]) for _ in range(case["B"])]
    S = [r.randint(case["S_lo"], case["S_hi"]) for _ in range(case["B"])]
    n = [r.randint(1, s) if case.get("partial") else s for s in S]
    return L, S, n


def work(case):
    if case["do"] == "w4":
        M, N, K = case["M"], case["N"], case["K"]
        out = M * N if case["epi"] == SWIGLU else 4 * M * N * (2 if case["epi"] == RESID else 1)
        return {"bytes": N * K // 2 + N * (K // case["group"]) * 4 + 2 * M * K + out, "flops": 2 * M * N * K}
    L, S, n = _lengths(case)
    Hq, Hkv, T = case["Hq"], case["Hkv"], sum(S)
    row = HD + 8                                # a cache row of one head: codes of key and value, two pairs of halves
    if case["do"] == "append":
        return {"bytes": T * (Hq + 2 * Hkv) * HD * (4 + 2) + sum(n) * Hkv * (2 * row + 2 * HD * 4),
                "flops": 6 * T * (Hq + Hkv) * HD + 8 * sum(n) * Hkv * HD}
    return {"bytes": sum(L) * Hkv * row + T * (2 * Hq + 2 * Hkv) * HD * 2,
            "flops": sum(4 * HD * Hq * s * (l + (s + 1) // 2) for l, s in zip(L, S))}


def _price(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 4e14 + (case["B"] * 3e-7 if "B" in case else 0)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _word_order(codes, order):
    """Last axis of 8 codes -> one 32-bit word; code e goes to nibble order[e]."""
    w = torch.zeros(codes.shape[:-1], dtype=torch.int32, device=codes.device)
    for e, nib in enumerate(order):
        w |= codes[..., e].to(torch.int32) << (4 * nib)
    return w


K_ORDER = (0, 4, 1, 5, 2, 6, 3, 7)
V_ORDER = (0, 1, 2, 3, 4, 5, 6, 7)


def _pack_pages(kc, ks, kz, vc, vs, vz):
    """Codes [n, 16, 128] (n = blocks x heads, uint8) and halves [n, 16] -> pages [n, 2176] (uint8)."""
    n = kc.shape[0]
    kw = _word_order(kc.view(n, BLOCK, 4, 4, 8), K_ORDER)                    # [n, token, i, c]: elements 32 i + 8 c ..
    kw = kw.permute(0, 3, 1, 2).reshape(n, 256)                              # stored [c, token, i]
    vw = _word_order(vc.view(n, 4, 4, 16, 8), V_ORDER)                       # [n, t / 4, t % 4, w]: elements 8 w ..
    vw = vw.permute(0, 1, 3, 2).reshape(n, 256)                              # stored [t / 4, w, t % 4]
    kp = torch.stack((ks, kz), -1).reshape(n, 32).contiguous().view(torch.int32)
    vp = torch.stack((vs, vz), -1).reshape(n, 32).contiguous().view(torch.int32)
    return torch.cat((kw, vw, kp, vp), 1).contiguous().view(torch.uint8)


def _quantise_rows(x):
    """Rows x [..., 128] (float64 holding bf16 values) -> codes, s, z (halves)."""
    x = x.clamp(-65504.0, 65504.0)
    z = x.amin(-1).to(torch.float32).half()
    s = ((x.amax(-1) - z.double()) / 15.0).to(torch.float32).half()
    sd = s.double().unsqueeze(-1)
    c = torch.where(sd > 0, torch.round((x - z.double().unsqueeze(-1)) / torch.where(sd > 0, sd, 1.0)), 0.0).clamp(0, 15)
    return c.to(torch.uint8), s, z


def _fill_pages(gen, n_blocks, Hkv):
    """A cache whose keys have channels with means of their own, as rotated keys do, and whose values are centred."""
    pages = torch.empty(n_blocks * Hkv, PAGE, dtype=torch.uint8, device=DEVICE)
    mean = torch.randn(Hkv, 1, HD, generator=gen, device=DEVICE) * 0.8
    step = max(1, (1 << 25) // (Hkv * BLOCK * HD))
    for a in range(0, n_blocks, step):
        m = min(step, n_blocks - a)
        k = (torch.randn(m, Hkv, BLOCK, HD, generator=gen, device=DEVICE) * 0.7 + mean).bfloat16().float()
        v = (torch.randn(m, Hkv, BLOCK, HD, generator=gen, device=DEVICE) * 0.5).bfloat16().float()
        parts = []
        for x in (k, v):
            x = x.view(m * Hkv, BLOCK, HD)
            z = x.amin(-1).half()
            s = ((x.amax(-1) - z.float()) / 15.0).half()
            parts += [torch.round((x - z.float().unsqueeze(-1)) / s.float().unsqueeze(-1)).clamp(0, 15).to(torch.uint8), s, z]
        pages[a * Hkv:(a + m) * Hkv] = _pack_pages(*parts)
    return pages


def _cu(S):
    return np.concatenate([[0], np.cumsum(S)]).astype(np.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 7919 + 17)
    st = dict(case=case)
    if case["do"] == "w4":
        M, N, K, g = case["M"], case["N"], case["K"], case["group"]
        st["a"] = torch.randn(M, K, generator=gen, device=DEVICE).bfloat16()
        # round-to-nearest codes of normal weights fall in a bell; zero points lie around the middle
        c = torch.empty(N, K // 2, dtype=torch.uint8, device=DEVICE)
        rows = max(1, (1 << 25) // K)
        for r in range(0, N, rows):
            x = torch.randn(min(rows, N - r), K, generator=gen, device=DEVICE).mul_(2.8).add_(7.5).round_().clamp_(0, 15).to(torch.uint8)
            c[r:r + rows] = x[:, 0::2] | (x[:, 1::2] << 4)
        st["codes"] = c
        st["scales"] = ((torch.rand(N, K // g, generator=gen, device=DEVICE) + 0.5) * (0.35 / math.sqrt(K))).half()
        st["zeros"] = torch.randint(5, 11, (N, K // g), generator=gen, device=DEVICE).half()
        st["resid"] = torch.randn(M, N, generator=gen, device=DEVICE) if case["epi"] == RESID else None
        st["out"] = torch.empty(M, N // 2, dtype=torch.bfloat16, device=DEVICE) if case["epi"] == SWIGLU else \
            torch.empty(M, N, dtype=torch.float32, device=DEVICE)
        if own:
            _own_w4(st)
        return st
    L, S, n = _lengths(case)
    Hq, Hkv, B, T = case["Hq"], case["Hkv"], case["B"], sum(S)
    cap = [(l + s + BLOCK - 1) // BLOCK for l, s in zip(L, S)]
    n_blocks, width = sum(cap) + 3, max(cap)
    order = torch.randperm(n_blocks, generator=gen, device=DEVICE).cpu().numpy().astype(np.int32)
    table = np.zeros((B, width), dtype=np.int32)
    at = 0
    for b, m in enumerate(cap):
        table[b, :m] = order[at:at + m]
        at += m
    st.update(L=L, S=S, n=n, T=T, h_table=table, n_blocks=n_blocks, width=width, h_cu=_cu(S), h_len=np.asarray(L, dtype=np.int32))
    st["pages"] = _fill_pages(gen, n_blocks, Hkv)
    for key, host in (("table", table), ("cu", st["h_cu"]), ("len", st["h_len"])):
        st[key] = torch.from_numpy(host).to(DEVICE)
    if case["do"] == "attn":
        st["q"] = (torch.randn(T, Hq, HD, generator=gen, device=DEVICE) * 1.3).bfloat16()
        st["k"] = (torch.randn(T, Hkv, HD, generator=gen, device=DEVICE) * 0.8).bfloat16()
        st["v"] = (torch.randn(T, Hkv, HD, generator=gen, device=DEVICE) * 0.5).bfloat16()
        st["out"] = torch.empty(T, Hq * HD, dtype=torch.bfloat16, device=DEVICE)
    else:
        st["qkv"] = torch.randn(T, (Hq + 2 * Hkv) * HD, generator=gen, device=DEVICE)
        st["q"] = torch.empty(T, Hq, HD, dtype=torch.bfloat16, device=DEVICE)
        st["k"] = torch.empty(T, Hkv, HD, dtype=torch.bfloat16, device=DEVICE)
        st["v"] = torch.empty(T, Hkv, HD, dtype=torch.bfloat16, device=DEVICE)
        st["h_cu_n"] = _cu(n)
        st["h_n"] = np.asarray(n, dtype=np.int32)
        st["cu_n"] = torch.from_numpy(st["h_cu_n"]).to(DEVICE)
        st["dev_n"] = torch.from_numpy(st["h_n"]).to(DEVICE)
        st["k_rows"] = torch.empty(sum(n), Hkv, HD, dtype=torch.float32, device=DEVICE)
        st["v_rows"] = torch.empty(sum(n), Hkv, HD, dtype=torch.float32, device=DEVICE)
        # token of the batch and cache row of every appended token
        tok = np.concatenate([st["h_cu"][b] + np.arange(m) for b, m in enumerate(n)])
        trace = np.repeat(np.arange(B), n)
        pos = np.concatenate([l + np.arange(m) for l, m in zip(L, n)])
        st["tok"] = torch.from_numpy(tok).to(DEVICE)
        st["blk"] = torch.from_numpy(table[trace, pos // BLOCK].astype(np.int64)).to(DEVICE)
        st["slot"] = torch.from_numpy(pos % BLOCK).to(DEVICE)
        st["pos"] = torch.from_numpy(np.concatenate([l + np.arange(s) for l, s in zip(L, S)])).to(DEVICE)
    if own:
        _own_kv(st)
    return st


# ---------------------------------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------------------------------
class _Ctx:
    """A context for the life of the state."""

    def __init__(self, cb, Hq, Hkv):
        self.cb = cb
        self.ptr = cb.confspec_create(cb.make_model_cfg(1, 128 * Hq, Hq, Hkv, HD, 256, 1024, THETA, 1e-6, "bf16"), 0)

    def __del__(self):
        self.cb.confspec_destroy(self.ptr)


def _own_w4(st):
    from paper_2602_18447_amd import binding as cb
    c = st["case"]
    st["cb"], st["ctx"] = cb, _Ctx(cb, 2, 1)
    st["w4"] = torch.empty(cb.confspec_w4_bytes(c["N"], c["K"], c["group"]), dtype=torch.uint8, device=DEVICE)
    cb.confspec_w4_pack(st["ctx"].ptr, st["codes"], st["scales"], st["zeros"], c["N"], c["K"], c["group"], st["w4"],
                        gate_up=c["epi"] == SWIGLU)


def _own_kv(st):
    from paper_2602_18447_amd import binding as cb
    c = st["case"]
    st["cb"], st["ctx"] = cb, _Ctx(cb, c["Hq"], c["Hkv"])
    st["kv"] = cb.make_kv4(st["pages"], st["table"], st["n_blocks"], BLOCK, st["width"])
    st["ids"] = torch.zeros(st["T"], dtype=torch.int32, device=DEVICE)
    st["batch"], st["keep"] = cb.make_batch(st["ids"], st["cu"], st["len"], st["h_cu"], st["h_len"])
    if c["do"] == "append":
        st["rows"], st["keep_n"] = cb.make_batch(st["ids"], st["cu_n"], st["len"], st["h_cu_n"], st["h_len"])
    else:
        need = cb.confspec_op_kv4_attention_scratch_bytes(st["ctx"].ptr, st["batch"])
        st["scratch"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEVICE)


def _run_own(st):
    c, cb, ctx = st["case"], st["cb"], st["ctx"].ptr
    if c["do"] == "w4":
        cb.confspec_op_w4_gemm(ctx, st["a"], st["w4"], st["resid"], st["out"], c["M"], c["N"], c["K"], c["group"], c["epi"])
        return st["out"]
    if c["do"] == "append":
        cb.confspec_op_kv4_append(ctx, st["kv"], st["batch"], 0, st["qkv"], st["dev_n"], st["h_n"], st["q"], st["k"], st["v"])
        cb.confspec_op_kv4_read(ctx, st["kv"], st["rows"], 0, st["k_rows"], st["v_rows"])
        return dict(q=st["q"], k=st["k"], v=st["v"], k_rows=st["k_rows"], v_rows=st["v_rows"])
    cb.confspec_op_kv4_attention(ctx, st["kv"], st["batch"], 0, st["q"], st["k"], st["v"], st["out"], st["scratch"])
    return st["out"]


# ---------------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _unpack_words(w, order):
    """Words [...] -> codes [..., 8] as fp32."""
    sh = torch.tensor([4 * n for n in order], dtype=torch.int32, device=w.device)
    return ((w.unsqueeze(-1) >> sh) & 15).float()


def _unpack_pages(p):
    """Pages [n, 2176] -> keys and values [n, 16, 128] fp32."""
    n = p.shape[0]
    w = p.view(torch.int32)
    kc = _unpack_words(w[:, :256].view(n, 4, 16, 4), K_ORDER)                 # [n, c, token, i, 8]
    kc = kc.permute(0, 2, 3, 1, 4).reshape(n, BLOCK, HD)
    vc = _unpack_words(w[:, 256:512].view(n, 4, 16, 4), V_ORDER)              # [n, t / 4, w, t % 4, 8]
    vc = vc.permute(0, 1, 3, 2, 4).reshape(n, BLOCK, HD)
    par = p[:, 2048:].contiguous().view(torch.float16).float().view(n, 2, BLOCK, 2)
    return (par[:, 0, :, 1:] + par[:, 0, :, :1] * kc, par[:, 1, :, 1:] + par[:, 1, :, :1] * vc)


def _plain_w4(st):
    c = st["case"]
    M, N, K, g = c["M"], c["N"], c["K"], c["group"]
    w = torch.empty(N, K // 2, 2, dtype=torch.float32, device=DEVICE)
    w[..., 0] = (st["codes"] & 15).float()
    w[..., 1] = (st["codes"] >> 4).float()
    w = w.view(N, K // g, g)
    w = (w - st["zeros"].float().unsqueeze(-1)) * st["scales"].float().unsqueeze(-1)
    y = st["a"].float() @ w.view(N, K).t()
    if c["epi"] == RESID:
        return st["resid"] + y
    if c["epi"] == SWIGLU:
        gate, up = y[:, :N // 2], y[:, N // 2:]
        return (gate / (1.0 + torch.exp(-gate)) * up).bfloat16()
    return y


def _plain_append(st):
    c = st["case"]
    Hq, Hkv, T = c["Hq"], c["Hkv"], st["T"]
    x = st["qkv"].view(T, Hq + 2 * Hkv, HD)
    # angles of far positions and values next to a border between two codes need 64 bits
    inv = THETA ** (-2.0 * torch.arange(HD // 2, dtype=torch.float64, device=DEVICE) / HD)
    ang = st["pos"].double().unsqueeze(-1) * inv
    cos, sin = torch.cos(ang).unsqueeze(1), torch.sin(ang).unsqueeze(1)
    r = x[:, :Hq + Hkv].double()
    lo, hi = r[..., :HD // 2], r[..., HD // 2:]
    rot = torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), -1).float().bfloat16()
    q, k, v = rot[:, :Hq], rot[:, Hq:], x[:, Hq + Hkv:].bfloat16()
    kc, ks, kz = _quantise_rows(k[st["tok"]].double())
    vc, vs, vz = _quantise_rows(v[st["tok"]].double())
    # into the pages: words and halves of one token of every head
    words = st["pages"].view(st["n_blocks"], Hkv, PAGE).view(torch.int32)
    halves = st["pages"].view(st["n_blocks"], Hkv, PAGE).view(torch.float16)
    m = len(st["tok"])
    blk, slot = st["blk"], st["slot"]
    b3, h3 = blk.view(m, 1, 1), torch.arange(Hkv, device=DEVICE).view(1, Hkv, 1)
    kw = _word_order(kc.view(m, Hkv, 4, 4, 8), K_ORDER).permute(0, 1, 3, 2).reshape(m, Hkv, 16)       # [c, i]
    ki = (torch.arange(4, device=DEVICE).view(4, 1) * 64 + torch.arange(4, device=DEVICE)).view(1, 1, 16) + slot.view(m, 1, 1) * 4
    words[b3, h3, ki] = kw
    vw = _word_order(vc.view(m, Hkv, 16, 8), V_ORDER)
    vi = 256 + (slot // 4).view(m, 1, 1) * 64 + torch.arange(16, device=DEVICE).view(1, 1, 16) * 4 + (slot % 4).view(m, 1, 1)
    words[b3, h3, vi] = vw
    b2, h2, s2 = blk.view(m, 1), torch.arange(Hkv, device=DEVICE).view(1, Hkv), slot.view(m, 1)
    for base, s, z in ((1024, ks, kz), (1056, vs, vz)):
        halves[b2, h2, base + 2 * s2] = s
        halves[b2, h2, base + 2 * s2 + 1] = z
    # and back: the values that the stored rows stand for
    kr = kz.float().unsqueeze(-1) + ks.float().unsqueeze(-1) * _unpack_words(words[b3, h3, ki].view(m, Hkv, 4, 4), K_ORDER) \
        .permute(0, 1, 3, 2, 4).reshape(m, Hkv, HD)
    vr = vz.float().unsqueeze(-1) + vs.float().unsqueeze(-1) * _unpack_words(words[b3, h3, vi], V_ORDER).reshape(m, Hkv, HD)
    return dict(q=q, k=k, v=v, k_rows=kr, v_rows=vr)


def _plain_attn(st):
    c = st["case"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    G = Hq // Hkv
    pages = st["pages"].view(st["n_blocks"], Hkv, PAGE)
    out = st["out"]
    for b in range(c["B"]):
        L, S, t0 = st["L"][b], st["S"][b], int(st["h_cu"][b])
        nb = (L + BLOCK - 1) // BLOCK
        k = st["k"][t0:t0 + S].float().transpose(0, 1)
        v = st["v"][t0:t0 + S].float().transpose(0, 1)
        if nb:
            kc, vc = _unpack_pages(pages[st["table"][b, :nb].long()].reshape(nb * Hkv, PAGE))
            kc = kc.view(nb, Hkv, BLOCK, HD).transpose(0, 1).reshape(Hkv, nb * BLOCK, HD)[:, :L]
            vc = vc.view(nb, Hkv, BLOCK, HD).transpose(0, 1).reshape(Hkv, nb * BLOCK, HD)[:, :L]
            k, v = torch.cat((kc, k), 1), torch.cat((vc, v), 1)
        q = st["q"][t0:t0 + S].float().view(S, Hkv, G, HD).permute(1, 2, 0, 3).reshape(Hkv, G * S, HD)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(HD))
        seen = torch.arange(L + S, device=DEVICE).view(1, -1) <= L + torch.arange(S, device=DEVICE).view(-1, 1)
        s = s.view(Hkv, G, S, L + S).masked_fill(~seen, float("-inf"))
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.matmul(p.view(Hkv, G * S, L + S), v.contiguous()) / p.sum(-1).view(Hkv, G * S, 1)
        out[t0:t0 + S] = o.view(Hkv, G, S, HD).permute(2, 0, 1, 3).reshape(S, Hq * HD).bfloat16()
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"w4": _plain_w4, "append": _plain_append, "attn": _plain_attn}[state["case"]["do"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_page_rows(page_bytes):
    """The 16 keys and values of pages [n, 2176] in float64, element by element as the format says."""
    n = page_bytes.shape[0]
    p = page_bytes.to(torch.int64)
    nib = torch.stack((p[:, :2048] & 15, p[:, :2048] >> 4), -1).view(n, 4096)   # nibble i of the page at 4 i bits
    t = torch.arange(16, device=p.device).view(16, 1)
    d = torch.arange(128, device=p.device).view(1, 128)
    e = d % 8
    k_at = ((((d % 32) // 8) * 16 + t) * 4 + d // 32) * 8 + e // 2 + 4 * (e % 2)
    v_at = 2048 + (((t // 4) * 16 + d // 8) * 4 + t % 4) * 8 + e
    par = page_bytes[:, 2048:].contiguous().view(torch.float16).double()
    rows = []
    for at, base in ((k_at, 0), (v_at, 32)):
        code = nib[:, at.reshape(-1)].view(n, 16, 128).double()
        rows.append(par[:, base + 1:base + 32:2].unsqueeze(-1) + par[:, base:base + 32:2].unsqueeze(-1) * code)
    return rows


def exact(case, seed):
    global own
    mine, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = mine
    f64 = torch.float64
    if case["do"] == "w4":
        N, K, g = case["N"], case["K"], case["group"]
        a = st["a"].to(f64)
        y = torch.empty(case["M"], N, dtype=f64, device=DEVICE)
        step = max(16, (1 << 26) // K)
        for r in range(0, N, step):
            c = st["codes"][r:r + step]
            w = torch.stack((c % 16, torch.div(c, 16, rounding_mode="floor")), 2).reshape(c.shape[0], K).to(f64)
            s = st["scales"][r:r + step].to(f64).repeat_interleave(g, 1)
            z = st["zeros"][r:r + step].to(f64).repeat_interleave(g, 1)
            y[:, r:r + step] = torch.matmul(a, (s * w - s * z).t())
        if case["epi"] == RESID:
            y += st["resid"].to(f64)
        if case["epi"] == SWIGLU:
            y = y[:, :N // 2] * torch.sigmoid(y[:, :N // 2]) * y[:, N // 2:]
        return y
    Hq, Hkv, B = case["Hq"], case["Hkv"], case["B"]
    if case["do"] == "append":
        x = st["qkv"].to(f64).view(st["T"], Hq + 2 * Hkv, HD)
        i = torch.arange(HD // 2, device=DEVICE, dtype=f64)
        turn = torch.polar(torch.ones((), dtype=f64, device=DEVICE), st["pos"].to(f64)[:, None, None] * torch.exp(-i * (2.0 / HD) * math.log(THETA)))
        z = torch.complex(x[..., :HD // 2], x[..., HD // 2:])
        z[:, :Hq + Hkv] *= turn
        y = torch.cat((z.real, z.imag), -1)
        # what the cache holds are the 16-bit rows, quantised
        rows = []
        for h0 in (Hq, Hq + Hkv):
            r = y[:, h0:h0 + Hkv][st["tok"]].float().bfloat16().to(f64)
            low, high = r.min(-1, keepdim=True).values, r.max(-1, keepdim=True).values
            low = low.half().to(f64)
            step = ((high - low) / 15).float().half().to(f64)
            rows.append(low + step * torch.clamp(torch.round((r - low) / step), 0, 15))
        return dict(q=y[:, :Hq], k=y[:, Hq:Hq + Hkv], v=y[:, Hq + Hkv:], k_rows=rows[0], v_rows=rows[1])
    G = Hq // Hkv
    if work(case)["flops"] > 3e12:
        return None
    pages = st["pages"].view(st["n_blocks"], Hkv, PAGE)
    out = torch.empty(st["T"], Hq * HD, dtype=f64, device=DEVICE)
    for b in range(B):
        L, S, t0 = st["L"][b], st["S"][b], int(st["h_cu"][b])
        blocks = torch.from_numpy(st["h_table"][b, :(L + 15) // 16].astype(np.int64)).to(DEVICE)
        for h in range(Hkv):
            k, v = _exact_page_rows(pages[blocks, h]) if L else (torch.empty(0, HD, dtype=f64, device=DEVICE),) * 2
            k = torch.cat((k.reshape(-1, HD)[:L], st["k"][t0:t0 + S, h].to(f64)))
            v = torch.cat((v.reshape(-1, HD)[:L], st["v"][t0:t0 + S, h].to(f64)))
            q = st["q"][t0:t0 + S, h * G:(h + 1) * G].to(f64).reshape(S * G, HD)
            s = torch.mm(q, k.t()) / math.sqrt(HD)
            last = (L + torch.arange(S, device=DEVICE)).repeat_interleave(G)
            s[torch.arange(L + S, device=DEVICE)[None, :] > last[:, None]] = -math.inf
            o = torch.mm(torch.softmax(s, -1), v)
            out[t0:t0 + S, h * G * HD:(h + 1) * G * HD] = o.view(S, G * HD)
    return out
