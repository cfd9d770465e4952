"""Performance cases of the decode operators: the 4-bit paged latent cache (append, read back, single-token
attention) and the 4-bit matrix-vector products of the decode-time projections.

Every case runs in two forms.  The plain form (`own = False`) spells the operator out in elementary torch
operations in 32 bits; the other form makes the calls of `paper_2609_07008_b200.binding` that a program makes.

Cached rows.  A page holds 64 rows of one segment (a document, or the suffix a request has generated so far) as
26 units of 16 bytes per row, unit-major: byte u * 1024 + row * 16 + i of the page is byte i of unit u of the row.
  units 0-15   latent dims 32 u .. 32 u + 31 as 4-bit codes n + 8: dim 32 u + 8 w + 2 i + e is the four bits at
               16 e + 4 i of the unit's 32-bit word w
  units 16-17  scale bytes: group g (latent dims 16 g .. 16 g + 15) is byte 4 (g >> 3) + (g & 3) of unit
               16 + ((g >> 2) & 1);  byte b stands for 2^((b >> 3) - 20) * (1 + (b & 7) / 8), 255 for NaN
  units 18-25  the 64 rope dims (bf16), rotated at the row's index in its segment
A code n with scale s stands for n * s, which is a bf16 number.
"""
import math

import numpy as np
import torch

own = False

D_LATENT, D_ROPE, D_QK = 512, 64, 576
PAGE_ROWS, UNITS, PAGE_BYTES = 64, 26, 26 * 64 * 16
ROW_BYTES = UNITS * 16
ROPE_BASE = 10000.0
SM_SCALE = 1.0 / math.sqrt(192.0)
GROUP = 16

# heads, output groups, rows of each group's W_a block, rows of W_b: the serving shapes of this repository
SHAPES = {"tiny": (16, 2, 256, 1024), "flash": (64, 8, 1024, 4096), "pro": (128, 16, 1024, 7168)}


# ------------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decode step of a batch: one new row per running request, rows scattered over 64 pages
        dict(name="append_step_64", op="append", segs=64, new_lo=1, new_hi=1, old_lo=100, old_hi=9000, geo=1),
        # documents of a long request enter the cache (64 documents of ragged length, from index 0)
        dict(name="append_docs_64", op="append", segs=64, new_lo=1025, new_hi=4096, old_lo=0, old_hi=0, geo=2),
        # one cached document of odd length is expanded for the online step
        dict(name="read_doc_777", op="read", segs=1, new_lo=777, new_hi=777, old_lo=0, old_hi=0, geo=3),
        # all documents of the 256K-context request are expanded into the packed stream of the online step
        dict(name="read_docs_256k", op="read", segs=64, new_lo=4096, new_hi=4096, old_lo=0, old_hi=0, geo=4),
        # the smallest call: one request, one short document and its question, one token, 16 heads
        dict(name="attn_small_1x1000", op="attn", heads=16, seqs=1, q_len=1, pool=1, doc_lo=1000, doc_hi=1000,
             per_seq=1, suf_lo=65, suf_hi=65, geo=5),
        # one request over the 256K-context set of 64 relocated documents, 64 heads, one token
        dict(name="attn_flash_256k", op="attn", heads=64, seqs=1, q_len=1, pool=64, doc_lo=4096, doc_hi=4096,
             per_seq=64, suf_lo=2048, suf_hi=2048, geo=6),
        # a running batch: ragged requests of two to three documents out of a pool that they share
        dict(name="attn_flash_batch_64", op="attn", heads=64, seqs=64, q_len=1, pool=96, doc_lo=1024, doc_hi=4096,
             per_seq=3, suf_lo=1, suf_hi=700, geo=7),
        # 128 heads, two tokens per request (one drafted ahead), long private contexts
        dict(name="attn_pro_batch_16_draft", op="attn", heads=128, seqs=16, q_len=2, pool=64, doc_lo=3500,
             doc_hi=4600, per_seq=4, suf_lo=33, suf_hi=2000, geo=8),
        # W_b of the 64-head shape for one token
        dict(name="matvec_wb_flash_1", op="matvec", mats=1, n_out=4096, k=8192, tok=1, group=128),
        # per-head value projections W_uv for five tokens (64 small matrices in one call)
        dict(name="matvec_wuv_flash_5", op="matvec", mats=64, n_out=128, k=512, tok=5, group=64),
        # per-group W_a for one token of the small shape: latency
        dict(name="matvec_wa_tiny_1", op="matvec", mats=2, n_out=256, k=1024, tok=1, group=32),
        # W_b of the 128-head shape for a batch of sixteen
        dict(name="matvec_wb_pro_16", op="matvec", mats=1, n_out=7168, k=16384, tok=16, group=128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "read", "attn", "attn", "attn", "matvec", "matvec"])
    geo = rng.randrange(1, 1 << 20)
    if op in ("append", "read"):
        segs = _log_int(rng, 1, 128)
        hi = _log_int(rng, 1, min(8192, max(2, 180000 // segs)))
        lo = max(1, hi // rng.choice([1, 2, 5]))
        old = 0 if rng.random() < 0.4 else _log_int(rng, 1, 9000 if segs <= 64 else 1000)
        return dict(op=op, segs=segs, new_lo=lo, new_hi=hi, old_lo=old // 3, old_hi=old, geo=geo)
    if op == "attn":
        heads = rng.choice([16, 64, 128, 8 * rng.randrange(1, 17)])
        q_len = rng.choice([1, 1, 1, 2, 3, 4])
        seqs = _log_int(rng, 1, 64)
        budget = 56_000_000 // (heads * q_len)              # (row, key) pairs of the call stay below the largest case
        per_seq = _log_int(rng, 1, 12)
        doc_hi = max(2, min(8000, budget // (seqs * per_seq)))
        doc_hi = max(2, _log_int(rng, max(2, doc_hi // 12), doc_hi))
        doc_lo = max(1, doc_hi // rng.choice([1, 2, 7]))
        suf_hi = q_len + _log_int(rng, 1, 600)
        return dict(op=op, heads=heads, seqs=seqs, q_len=q_len, pool=per_seq + rng.randrange(0, per_seq * seqs + 1),
                    doc_lo=doc_lo, doc_hi=doc_hi, per_seq=per_seq, suf_lo=q_len, suf_hi=suf_hi, geo=geo)
    heads, groups, o_rank, d_model = SHAPES[rng.choice(["tiny", "flash", "pro"])]
    mats, n_out, k = rng.choice([(heads, 128, 512), (groups, o_rank, 1024), (1, d_model, groups * o_rank),
                                 (1, 16 * rng.randrange(1, 300), 128 * rng.randrange(1, 100))])
    return dict(op=op, mats=mats, n_out=n_out, k=k, tok=_log_int(rng, 1, 16), group=rng.choice([32, 64, 128]))


# ------------------------------------------------------------------------------------------------------------
# geometry: depends on the case alone, so that the work of a case is a number
# ------------------------------------------------------------------------------------------------------------
def _seg_geometry(case):
    r = np.random.default_rng(np.random.PCG64(case["geo"]))
    new = r.integers(case["new_lo"], case["new_hi"] + 1, size=case["segs"])
    old = r.integers(case["old_lo"], case["old_hi"] + 1, size=case["segs"])
    return new.tolist(), old.tolist()


def _attn_geometry(case):
    """Segments 0 .. pool - 1 are the documents, the rest one suffix per request.  Per request: its segments in
    request order with the offset each appears at, and the position of its first query token."""
    r = np.random.default_rng(np.random.PCG64(case["geo"]))
    lens = r.integers(case["doc_lo"], case["doc_hi"] + 1, size=case["pool"]).tolist()
    items, pos0 = [], []
    for b in range(case["seqs"]):
        docs = r.permutation(case["pool"])[:case["per_seq"]]
        if case["per_seq"] == 3 and b % 2:
            docs = docs[:2]
        run, mine = 0, []
        for d in docs.tolist():
            mine.append((d, run))
            run += lens[d]
        suffix = int(r.integers(case["suf_lo"], case["suf_hi"] + 1))
        mine.append((len(lens), run))
        lens.append(suffix)
        items.append(mine)
        pos0.append(run + suffix - case["q_len"])
    return lens, items, pos0


def work(case):
    if case["op"] in ("append", "read"):
        n = sum(_seg_geometry(case)[0])
        row = D_QK * 2 + ROW_BYTES
        # append: the new rows in, the cached form out, and that read back as the rows that later steps see
        return {"bytes": n * row * (2 if case["op"] == "append" else 1), "flops": n * 4 * D_QK}
    if case["op"] == "attn":
        lens, items, pos0 = _attn_geometry(case)
        rows = case["seqs"] * case["q_len"] * case["heads"]
        used = {s for mine in items for s, _ in mine}
        keys = sum(min(max(p + t - d + 1, 0), lens[s]) for mine, p in zip(items, pos0) for s, d in mine
                   for t in range(case["q_len"]))
        return {"bytes": sum(lens[s] for s in used) * ROW_BYTES + rows * (D_QK * 2 + D_LATENT * 2 + 4),
                "flops": keys * case["heads"] * 2 * (D_QK + D_LATENT)}
    m, n, k, t = case["mats"], case["n_out"], case["k"], case["tok"]
    return {"bytes": m * n * k // 2 + m * n * (k // case["group"]) * 2 + t * m * (k + n) * 2, "flops": 2 * t * m * n * k}


# ------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 11)
    return g


def _context(heads, groups, o_rank=256, d_model=1024):
    from paper_2609_07008_b200 import binding as rk
    return rk, rk.Context(heads, groups, o_rank, d_model, [8 * g for g in range(groups)], SM_SCALE, ROPE_BASE)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _page_table(lens, seed):
    """Pages of every segment out of one shuffled pool."""
    counts = [(n + PAGE_ROWS - 1) // PAGE_ROWS for n in lens]
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    ids = np.random.default_rng(np.random.PCG64(seed + 5)).permutation(int(off[-1]) + 3)[:int(off[-1])]
    return off, ids


def _scale_bytes(amax):
    """Nearest scale byte (ties to even) of amax / 7; amax float32.  The division is by a tensor: by a Python
    number it may become a product with the rounded reciprocal, which moves ties."""
    u = (amax / torch.full_like(amax, 7.0)).contiguous().view(torch.int32)
    u = u + 0x7FFFF + ((u >> 20) & 1)
    return ((u >> 20) - (107 << 3)).clamp(0, 254)


def _scale_values(byte):
    v = ((byte.to(torch.int32) + (107 << 3)) << 20).view(torch.float32)
    return torch.where(byte == 255, torch.full_like(v, float("nan")), v)


def _quantise(c):
    """c [..., 512] float32 -> codes [..., 32, 16] in -7..7 (float32), scale bytes [..., 32] (int32)."""
    x = c.unflatten(-1, (32, GROUP))
    byte = _scale_bytes(x.abs().amax(-1))
    return torch.round(x / _scale_values(byte)[..., None]).clamp(-7, 7), byte


def _random_pages(n_pages, g):
    """Pages full of cached rows: latents N(0, 1) in 4 bits, rope dims N(0, 1)."""
    pages = torch.empty((n_pages, PAGE_BYTES), dtype=torch.uint8, device="cuda")
    shift = torch.tensor([[4 * i + 16 * e for e in (0, 1)] for i in range(4)], device="cuda")
    for lo in range(0, n_pages, 1024):
        p = min(1024, n_pages - lo)
        c = torch.randn((p, PAGE_ROWS, D_LATENT), generator=g, device="cuda").to(torch.bfloat16).float()
        code, byte = _quantise(c)
        nib = (code + 8).to(torch.int64).reshape(p, PAGE_ROWS, 16, 4, 4, 2)
        words = (nib << shift).sum((-1, -2))
        words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)      # [p, row, unit, word]
        out = pages[lo:lo + p].view(p, UNITS, PAGE_ROWS, 16)
        out[:, :16] = words.view(torch.uint8).transpose(1, 2)
        sb = byte.to(torch.uint8).reshape(p, PAGE_ROWS, 4, 2, 4).permute(0, 3, 1, 2, 4).reshape(p, 2, PAGE_ROWS, 16)
        out[:, 16:18] = sb
        rope = torch.randn((p, PAGE_ROWS, D_ROPE), generator=g, device="cuda").to(torch.bfloat16)
        out[:, 18:] = rope.view(torch.uint8).reshape(p, PAGE_ROWS, 8, 16).transpose(1, 2)
    return pages


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] in ("append", "read"):
        new, old = _seg_geometry(case)
        lens = [a + b for a, b in zip(new, old)]
        off, ids = _page_table(lens, seed)
        s.update(new=new, old=old, lens=lens, off=off, ids_host=ids, ids=_i32(ids), n=sum(new))
        s["new_off"] = _i32(np.concatenate([[0], np.cumsum(new)]))
        if case["op"] == "append":
            s["pages"] = torch.zeros((len(ids) + 3, PAGE_BYTES), dtype=torch.uint8, device="cuda")
            # the down-projection gives latent and rope part of a token in one row; the latent is normalised apart
            s["c"] = torch.randn((s["n"], D_LATENT), generator=g, device="cuda").to(torch.bfloat16)
            s["k_rope"] = torch.randn((s["n"], D_QK), generator=g, device="cuda").to(torch.bfloat16)[:, D_LATENT:]
        else:
            s["pages"] = _random_pages(len(ids) + 3, g)
        if own:
            rk, s["ctx"] = _context(64, 8)
            s["table"] = rk.CacheTable(_i32(lens), _i32(off), s["ids"])
        return s
    if case["op"] == "attn":
        lens, items, pos0 = _attn_geometry(case)
        off, ids = _page_table(lens, seed)
        h = case["heads"]
        s.update(lens=lens, items=items, pos0=pos0, off=off, ids=_i32(ids), pages=_random_pages(len(ids) + 3, g))
        s["q"] = (torch.randn((case["seqs"], case["q_len"], h, D_QK), generator=g, device="cuda") * 1.2).to(torch.bfloat16)
        if own:
            rk, s["ctx"] = _context(h, h // 8)
            s["table"] = rk.CacheTable(_i32(lens), _i32(off), s["ids"])
            seq_off = np.concatenate([[0], np.cumsum([len(m) for m in items])])
            q_pos = [[p + t for t in range(case["q_len"])] for p in pos0]
            tiles = sum((lens[i] + 127) // 128 for m in items for i, _ in m)
            s["plan"] = s["ctx"].rk_decode_plan(s["table"], len(s["pages"]), _i32(seq_off), _i32([i for m in items for i, _ in m]),
                                                _i32([d for m in items for _, d in m]), _i32(q_pos), max_tiles=tiles)
        return s
    m, n, k, t, grp = case["mats"], case["n_out"], case["k"], case["tok"], case["group"]
    w = (torch.randn((m, n, k), generator=g, device="cuda") * 0.02).to(torch.bfloat16)
    s["x"] = torch.randn((t, m, k), generator=g, device="cuda").to(torch.bfloat16)
    if own:
        rk, s["ctx"] = _context(64, 8)
        s["w4"] = s["ctx"].rk_quant4(w, grp)
    else:
        x = w.float().unflatten(-1, (k // grp, grp))
        top = x.abs().amax(-1)
        s["scale"] = (top / torch.full_like(top, 7.0)).to(torch.bfloat16)
        sc = s["scale"].float()[..., None]
        code = (torch.round(x / sc).clamp(-7, 7) + 8).to(torch.uint8).reshape(m, n, k // 2, 2)
        s["code"] = code[..., 0] | (code[..., 1] << 4)
    return s


# ------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------
def _turn(x, ang):
    """Rotates interleaved pairs of x [..., 64] by the angles ang [..., 32] (float64), in float32."""
    co, si = torch.cos(ang).float(), torch.sin(ang).float()
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * co - b * si, a * si + b * co], -1).flatten(-2)


def _theta():
    return torch.pow(torch.tensor(ROPE_BASE, dtype=torch.float64, device="cuda"),
                     -torch.arange(0, D_ROPE, 2, dtype=torch.float64, device="cuda") / D_ROPE)


def _cached_rows(pages, ids, first, count):
    """Rows first .. first + count - 1 of a segment whose pages are `ids`: [count, 576] float32."""
    lo = first // PAGE_ROWS
    hi = (first + count + PAGE_ROWS - 1) // PAGE_ROWS
    p = pages[ids[lo:hi].long()].view(hi - lo, UNITS, PAGE_ROWS, 16).transpose(1, 2)
    p = p.reshape((hi - lo) * PAGE_ROWS, UNITS, 16)[first - lo * PAGE_ROWS:first - lo * PAGE_ROWS + count]
    words = p[:, :16].contiguous().view(torch.int32)                                     # [rows, unit, word]
    shift = torch.tensor([[4 * i + 16 * e for e in (0, 1)] for i in range(4)], dtype=torch.int32, device="cuda")
    code = ((words[..., None, None] >> shift) & 15).reshape(count, 32, GROUP).float() - 8.0
    byte = p[:, 16:18].reshape(count, 2, 4, 4).transpose(1, 2).reshape(count, 32)
    rope = p[:, 18:].reshape(count, 128).contiguous().view(torch.bfloat16).float()
    return torch.cat([(code * _scale_values(byte)[..., None]).flatten(1), rope], 1)


def _plain_append(s):
    theta, out, at = _theta(), [], 0
    for new, old in zip(s["new"], s["old"]):
        code, byte = _quantise(s["c"][at:at + new].float())
        pos = torch.arange(old, old + new, dtype=torch.float64, device="cuda")
        rope = _turn(s["k_rope"][at:at + new].float(), pos[:, None] * theta)
        out.append(torch.cat([(code * _scale_values(byte)[..., None]).flatten(1), rope], 1))
        at += new
    return torch.cat(out).to(torch.bfloat16)


def _plain_read(s):
    return torch.cat([_cached_rows(s["pages"], s["ids"][s["off"][i]:s["off"][i + 1]], old, new)
                      for i, (new, old) in enumerate(zip(s["new"], s["old"]))]).to(torch.bfloat16)


def _plain_attn(s):
    case, theta = s["case"], _theta()
    h, ql = case["heads"], case["q_len"]
    out = torch.empty((case["seqs"], ql, h, D_LATENT), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((case["seqs"], ql, h), dtype=torch.float32, device="cuda")
    for b, mine in enumerate(s["items"]):
        q = s["q"][b].float().reshape(ql * h, D_QK)
        pos = torch.arange(s["pos0"][b], s["pos0"][b] + ql, device="cuda").repeat_interleave(h)
        logits, values = [], []
        for seg, delta in mine:
            k = _cached_rows(s["pages"], s["ids"][s["off"][seg]:s["off"][seg + 1]], 0, s["lens"][seg])
            qd = torch.cat([q[:, :D_LATENT], _turn(q[:, D_LATENT:], -float(delta) * theta)], 1)
            l = (qd @ k.t()) * SM_SCALE
            at = delta + torch.arange(s["lens"][seg], device="cuda")
            logits.append(torch.where(at[None, :] <= pos[:, None], l, torch.full_like(l, float("-inf"))))
            values.append(k[:, :D_LATENT])
        l = torch.cat(logits, 1)
        mx = l.amax(1, keepdim=True)
        p = torch.exp(l - mx)
        tot = p.sum(1, keepdim=True)
        out[b] = ((p @ torch.cat(values)) / tot).to(torch.bfloat16).view(ql, h, D_LATENT)
        lse[b] = (mx + torch.log(tot)).view(ql, h)
    return out, lse


def _plain_matvec(s):
    c, grp = s["code"], s["case"]["group"]
    w = torch.stack([c & 15, c >> 4], -1).flatten(-2).float() - 8.0
    w = (w.unflatten(-1, (-1, grp)) * s["scale"].float()[..., None]).flatten(-2)          # [mats, n_out, k]
    return torch.matmul(w, s["x"].float().permute(1, 2, 0)).permute(2, 0, 1).to(torch.bfloat16).contiguous()


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"append": _plain_append, "read": _plain_read, "attn": _plain_attn, "matvec": _plain_matvec}[op](s)
    if op == "append":
        s["ctx"].rk_cache4_append(s["pages"], s["table"], s["c"], s["k_rope"], s["new_off"])
        return s["ctx"].rk_cache4_read(s["pages"], s["table"], s["new_off"], s["n"])
    if op == "read":
        return s["ctx"].rk_cache4_read(s["pages"], s["table"], s["new_off"], s["n"])
    if op == "attn":
        return s["ctx"].rk_cache4_attn(s["pages"], s["plan"], s["q"])
    return s["ctx"].rk_matvec4(s["w4"], s["x"])


# ------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits, from the inputs' bytes
# ------------------------------------------------------------------------------------------------------------
def _rotate64(v, angle):
    z = torch.view_as_complex(v.double().unflatten(-1, (-1, 2)).contiguous())
    return torch.view_as_real(z * torch.polar(torch.ones_like(angle), angle)).flatten(-2)


def _unpack64(pages, ids, first, count):
    """Row by index: unit u of row r of a page starts at byte u * 1024 + r * 16."""
    r = torch.arange(first, first + count, device="cuda")
    page = ids.long()[r // 64]
    flat = pages.reshape(-1)
    base = page * PAGE_BYTES + (r % 64) * 16
    d = torch.arange(D_LATENT, device="cuda")
    # dim d: unit d / 32, word (d % 32) / 8, in the word bit 4 * ((d % 8) / 2) + 16 * (d % 2)
    bit = 4 * ((d % 8) // 2) + 16 * (d % 2)
    byte_at = (d // 32) * 1024 + ((d % 32) // 8) * 4 + bit // 8
    code = (flat[base[:, None] + byte_at].to(torch.int64) >> (bit % 8)) & 15
    gi = d // 16
    sb = flat[base[:, None] + (16 + (gi // 4) % 2) * 1024 + 4 * (gi // 8) + gi % 4].to(torch.int64)
    scale = torch.ldexp(1.0 + (sb % 8).double() / 8.0, sb // 8 - 20)
    scale[sb == 255] = float("nan")
    e = torch.arange(D_ROPE, device="cuda")
    lo = base[:, None] + (18 + e // 8) * 1024 + (e % 8) * 2
    bits = flat[lo].to(torch.int32) | (flat[lo + 1].to(torch.int32) << 8)
    rope = (bits << 16).view(torch.float32).double()
    return torch.cat([(code - 8).double() * scale, rope], 1)


def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    freq = ROPE_BASE ** (-2.0 * torch.arange(32, dtype=torch.float64, device="cuda") / D_ROPE)
    if case["op"] == "append":
        out, at = torch.empty((s["n"], D_QK), dtype=torch.float64, device="cuda"), 0
        for new, old in zip(s["new"], s["old"]):
            for lo in range(0, new, 4096):
                n = min(4096, new - lo)
                x = s["c"][at:at + n].double().view(n, 32, 16)
                top = x.abs().amax(2)
                mant, ex = torch.frexp(top / torch.full_like(top, 7.0))       # mant in [1/2, 1)
                step = torch.ldexp(torch.round(mant * 16.0), ex - 4).clamp(2.0 ** -20, 3584.0)
                out[at:at + n, :D_LATENT] = (torch.round(x / step[..., None]).clamp(-7, 7) * step[..., None]).flatten(1)
                j = torch.arange(old + lo, old + lo + n, device="cuda").double()
                out[at:at + n, D_LATENT:] = _rotate64(s["k_rope"][at:at + n], j[:, None] * freq)
                at += n
        return out
    if case["op"] == "read":
        return torch.cat([_unpack64(s["pages"], s["ids"][s["off"][i]:s["off"][i + 1]], old, new)
                          for i, (new, old) in enumerate(zip(s["new"], s["old"]))])
    if case["op"] == "attn":
        h, ql = case["heads"], case["q_len"]
        if work(case)["flops"] > 4e13:
            return None
        out, lse = [], []
        for b, mine in enumerate(s["items"]):
            q = s["q"][b].double()                                            # [ql, h, 576]
            num = torch.zeros((ql, h, D_LATENT), dtype=torch.float64, device="cuda")
            den = torch.zeros((ql, h), dtype=torch.float64, device="cuda")
            top = torch.full((ql, h), float("-inf"), dtype=torch.float64, device="cuda")
            for seg, delta in mine:
                rows = _unpack64(s["pages"], s["ids"][s["off"][seg]:s["off"][seg + 1]], 0, s["lens"][seg])
                qr = _rotate64(q[..., D_LATENT:], (-delta * freq).expand(ql, h, 32).contiguous())
                score = SM_SCALE * (q[..., :D_LATENT] @ rows[:, :D_LATENT].t() + qr @ rows[:, D_LATENT:].t())
                for t in range(ql):
                    seen = min(max(s["pos0"][b] + t - delta + 1, 0), s["lens"][seg])
                    score[t, :, seen:] = float("-inf")
                higher = torch.maximum(top, score.amax(-1))
                safe = torch.where(torch.isinf(higher), torch.zeros_like(higher), higher)
                shrink = torch.exp(top - safe)
                p = torch.exp(score - safe[..., None])
                num = num * shrink[..., None] + p @ rows[:, :D_LATENT]
                den = den * shrink + p.sum(-1)
                top = higher
            out.append(num / den[..., None])
            lse.append(top + torch.log(den))
        return torch.stack(out), torch.stack(lse)
    m, n, k, grp = case["mats"], case["n_out"], case["k"], case["group"]
    w = (torch.randn((m, n, k), generator=_gen(seed), device="cuda") * 0.02).to(torch.bfloat16).double()
    y = torch.empty((case["tok"], m, n), dtype=torch.float64, device="cuda")
    for b in range(m):
        x = w[b].view(n, k // grp, grp)
        top = x.abs().amax(2)
        step = (top / torch.full_like(top, 7.0)).to(torch.bfloat16).double()[..., None]
        y[:, b] = s["x"][:, b].double() @ (torch.round(x / step).clamp(-7, 7) * step).flatten(1).t()
    return y
