"""The operators of an attention layer in 8-bit formats with a scale for each block, as cases
that can be timed and compared: the page tables of a serving step, the paged e4m3 cache (written
and read), and the e4m3 product that makes the projections around it.

One case is one call of one operator.  `run` computes it in its plain form (elementary torch
operations in 32 bits), or, where `own` is true, through the framework's public calls.  Sizes are
those of the repository's workloads (8B decoders: 32 query and 8 KV heads of 128, widths 4096,
6144, 12288, 14336, 28672; blocks of 8 and 16 rows; contexts up to 32768), of its tests (heads of
64) and generic odd ones.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _plan(name, batch, lo, hi, new_lo, new_hi, page, wave=False, pool=1.0):
    return {"name": name, "kind": "plan", "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi,
            "page": page, "wave": wave, "pool": pool}


def _append(name, batch, lo, hi, new_lo, new_hi, page, heads=8, dh=128, dtype="bf16"):
    return {"name": name, "kind": "append", "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi,
            "page": page, "heads": heads, "dh": dh, "dtype": dtype}


def _attend(name, batch, lo, hi, new_lo, new_hi, page, causal, q_heads=32, heads=8, dh=128, dtype="bf16"):
    return {"name": name, "kind": "attend", "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi,
            "page": page, "causal": causal, "q_heads": q_heads, "heads": heads, "dh": dh, "dtype": dtype}


def _quantize(name, rows, cols, block_rows, dtype="bf16"):
    return {"name": name, "kind": "quantize", "rows": rows, "cols": cols, "block_rows": block_rows, "dtype": dtype}


def _matmul(name, m, n, k, dtype="bf16"):
    return {"name": name, "kind": "matmul", "m": m, "n": n, "k": k, "dtype": dtype}


def listed():
    return [
        # the next block of a serving batch enters its tables: pages are there or one more is taken
        _plan("plan_b32_k8", 32, 512, 4096, 8, 8, 64),
        # a whole batch ends and as many prompts take its pages: the largest tables
        _plan("plan_wave_b256", 256, 1, 4096, 1, 2048, 16, wave=True),
        # the rows of a decode step enter the cache, most of them into a page that holds earlier rows
        _append("append_b32_k8", 32, 512, 4096, 8, 8, 64),
        # prompts of odd lengths enter the cache
        _append("append_prefill_b4", 4, 0, 900, 1001, 3001, 64),
        # one user's decode step: a block of 16 rows over 2048 positions
        _attend("attend_b1_l2048_k16", 1, 2048, 2048, 16, 16, 64, "one"),
        # a serving batch of ragged contexts in small pages, short blocks, the other 16-bit type
        _attend("attend_b32_ragged_k8", 32, 512, 4096, 8, 8, 16, "one", dtype="fp16"),
        # prompts of odd lengths, one of them behind a cached prefix
        _attend("attend_prefill_b3", 3, 0, 1500, 801, 4001, 64, "all"),
        # the SwiGLU outputs of a prompt of odd length, a scale for each row and 128 columns
        _quantize("quantize_rows_2001", 2001, 14336, 1),
        # a gate/up weight matrix, a scale for each 128 x 128 block
        _quantize("quantize_weight", 28672, 4096, 128),
        # gate/up of one block of 16 rows: the weights' bytes are all there is
        _matmul("matmul_m16", 16, 28672, 4096),
        # the down projection of a small batch with an odd number of rows, 32-bit sums out
        _matmul("matmul_m203_fp32", 203, 4096, 14336, "fp32"),
        # gate/up of a prompt of 4096 rows: the matrix unit is all there is
        _matmul("matmul_m4096", 4096, 28672, 4096),
    ]


def _logint(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(("plan", "append", "attend", "quantize", "matmul"), (12, 16, 36, 12, 24))[0]
    if kind == "quantize":
        br = rng.choice((1, 1, 128))
        cols = 16 * _logint(rng, 4, 896)
        c = _quantize("", _logint(rng, 1, min(28672, 117000000 // cols)), cols, br, rng.choice(("bf16", "fp16", "fp32")))
    elif kind == "matmul":
        k = 16 * _logint(rng, 8, 896)
        n = _logint(rng, 64, 28672)
        if rng.random() < 0.6:  # projection widths are whole blocks more often than not
            n = max(128, n // 128 * 128)
            k = max(128, k // 128 * 128)
        c = _matmul("", _logint(rng, 1, min(4096, 4096 * 28672 * 4096 // (n * k))), n, k, rng.choice(("bf16", "bf16", "fp16", "fp32")))
    else:
        page = rng.choice((16, 32, 64, 128))
        wave = kind == "plan" and rng.random() < 0.4
        if wave or (kind != "plan" and rng.random() < 0.3):  # prompts
            batch = _logint(rng, 1, 256 if kind == "plan" else 4)
            lo, hi = 0, _logint(rng, 1, 4096 if kind == "plan" else 1500)
            new_hi = _logint(rng, 17, 4096 // max(1, batch // 64) if kind == "plan" else 5000 // batch)
            new_lo = rng.randint(1, new_hi)
        else:                                                # blocks of a serving batch
            batch = _logint(rng, 1, 256 if kind == "plan" else 48)
            hi = _logint(rng, 1, min(32768, 131072 // batch) if kind != "plan" else 8192)
            lo = rng.randint(0, hi)
            new_hi = rng.choice((1, 1, 4, 8, 13, 16, 32))
            new_lo = rng.choice((0, 1, new_hi, new_hi))      # 0: some sequences sit the step out
        if kind == "plan":
            c = _plan("", batch, lo, hi, new_lo, new_hi, page, wave, rng.choice((1.0, 1.0, 0.9)))
        else:
            dh = rng.choice((128, 128, 64))
            heads, group = rng.choice(((8, 4), (8, 4), (8, 1), (4, 8), (2, 2), (1, 16), (8, 5)))
            dtype = rng.choice(("bf16", "bf16", "fp16"))
            if kind == "append":
                c = _append("", batch, lo, hi, new_lo, new_hi, page, heads, dh, dtype)
            else:
                c = _attend("", batch, lo, hi, new_lo, new_hi, page, rng.choice(("all", "one", "none")), heads * group,
                            heads, dh, dtype)
    del c["name"]
    return c


# ---- inputs


def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + stream)
    return g


def _lens(case):
    """Cached tokens and new rows of each sequence: the same for every seed, so that the work is."""
    r = random.Random(case["lo"] * 131071 + case["hi"] * 31 + case["batch"] * 7 + case["new_hi"])
    lens = [(r.randint(case["lo"], case["hi"]), r.randint(case["new_lo"], case["new_hi"])) for _ in range(case["batch"])]
    return lens if any(n for _, n in lens) else [(lens[0][0], case["new_hi"])] + lens[1:]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pages_of(n, page):
    return -(-n // page)


def _values(g, std, *shape):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g)


def _codes(g, *shape):
    """e4m3 codes of normal values that use the format's range as a scaled block does."""
    return _values(g, 110.0, *shape).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _tables(case, seed, held):
    """Tables of sequences that hold `held[b]` pages each, in random order, and the pages left."""
    page, batch = case["page"], case["batch"]
    lens = _lens(case)
    width = max(1, max(_pages_of(c + n, page) for c, n in lens))
    if case.get("wave"):
        need = sum(_pages_of(n, page) for _, n in lens)
        n_pages = max(sum(held), int(need * case["pool"])) + 1
    else:
        need = sum(max(0, _pages_of(c + n, page) - h) for (c, n), h in zip(lens, held))
        n_pages = sum(held) + int(need * case.get("pool", 1.0)) + 1
    perm = torch.randperm(n_pages, generator=_gen(seed, 3), device=DEV).to(torch.int32)
    table = torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
    h = torch.tensor(held, device=DEV)
    mask = torch.arange(width, device=DEV)[None, :] < h[:, None]
    table[mask] = perm[:sum(held)]
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    free[:n_pages - sum(held)] = perm[sum(held):]
    return n_pages, table, free, n_pages - sum(held)


def _layout(case, seed):
    """A step's tables as a plan leaves them: every page that the new rows need is there."""
    page, lens = case["page"], _lens(case)
    n_pages, table, _, _ = _tables(case, seed, [_pages_of(c + n, page) for c, n in lens])
    starts = [0]
    for _, n in lens:
        starts.append(starts[-1] + n)
    st = {"n_pages": n_pages, "table": table, "row_start": _ints(starts), "kv_len": _ints([c + n for c, n in lens]),
          "rows": starts[-1]}
    b = torch.repeat_interleave(torch.arange(case["batch"], device=DEV), torch.tensor([n for _, n in lens], device=DEV),
                                output_size=starts[-1])
    j = torch.arange(starts[-1], device=DEV) - st["row_start"][b]
    p = torch.tensor([c for c, _ in lens], device=DEV)[b] + j
    st["slots"] = (table[b, p // page].long() * page + p % page).to(torch.int32)
    return st


def _cache(case, seed, st):
    """Pages of random codes with a power of two for each page and head, as cached values have."""
    n, H, page, dh = st["n_pages"], case["heads"], case["page"], case["dh"]
    g = _gen(seed, 4)
    st["k_codes"], st["v_codes"] = _codes(g, n, H, page, dh), _codes(g, n, H, dh, page)
    for name in ("k_exp", "v_exp"):
        st[name] = torch.randint(-8, -5, (n, H), dtype=torch.int8, device=DEV, generator=g)


def prepare(case, seed):
    st = {"kind": case["kind"], "case": dict(case)}
    if case["kind"] == "plan":
        lens, page = _lens(case), case["page"]
        held = [_pages_of(c, page) for c, _ in lens]
        n_pages, table, free, count = _tables(case, seed, held)
        rows = sum(n for _, n in lens)
        st.update(n_pages=n_pages, table=table, free_list=free, free_count=_ints([count]), held=_ints(held),
                  cached=_ints([c for c, _ in lens]), n_new=_ints([n for _, n in lens]), rows=rows + 5,
                  release=torch.ones(case["batch"], dtype=torch.uint8, device=DEV) if case["wave"] else None)
        if own:
            from paper_2509_04185_amd import PageTable
            st["pages"] = PageTable(table, st["held"], st["cached"], free, st["free_count"], page)
        return st
    if case["kind"] in ("append", "attend"):
        st.update(_layout(case, seed))
        _cache(case, seed, st)
        g = _gen(seed, 5)
        if case["kind"] == "append":  # values about as large as the cached ones, some rows larger
            for name in ("k", "v"):
                x = _values(g, 1.0, st["rows"], case["heads"], case["dh"])
                x *= torch.exp(_values(g, 0.7, st["rows"], 1, 1))
                st[name] = x.to(TYPES[case["dtype"]])
        else:
            st["q"] = _values(g, 1.0, st["rows"], case["q_heads"], case["dh"]).to(TYPES[case["dtype"]])
            lens = _lens(case)
            st["n_causal"] = {"all": None, "none": _ints([0] * len(lens)),
                              "one": _ints([min(1, n) for _, n in lens])}[case["causal"]]
            st["max_new"] = max(n for _, n in lens)
            st["max_kv"] = max(c + n for c, n in lens)
        if own:
            from paper_2509_04185_amd import PagedKV, PagedStep
            st["kv"] = PagedKV(st["k_codes"], st["v_codes"], st["k_exp"], st["v_exp"])
            st["step"] = PagedStep(st["table"], st["row_start"], st["kv_len"], st["slots"], case["page"])
        return st
    g = _gen(seed, 6)
    if case["kind"] == "quantize":
        x = _values(g, 1.0, case["rows"], case["cols"])
        x *= torch.exp(_values(g, 1.0, 1, case["cols"]))  # some columns are much larger than others
        st["x"] = x.to(TYPES[case["dtype"]])
        return st
    m, n, k = case["m"], case["n"], case["k"]
    kb = _pages_of(k, 128)
    st.update(a=_codes(g, m, k), b=_codes(g, n, k),
              a_scale=torch.empty((kb, m), device=DEV).uniform_(0.5e-2, 2e-2, generator=g),
              b_scale=torch.empty((_pages_of(n, 128), kb), device=DEV).uniform_(0.5e-4, 2e-4, generator=g))
    return st


# ---- one pass: the framework's calls, or the plain forms


def run(st):
    kind, case = st["kind"], st["case"]
    if kind == "plan":
        if own:
            s = st["pages"].plan(st["n_new"], st["rows"], release=st["release"])
            row_start, kv_len, slots = s.row_start, s.kv_len, s.slots
        else:
            row_start, kv_len, slots = _plain_plan(st, case["page"])
        return {"row_start": row_start, "kv_len": kv_len, "slots": slots, "table": st["table"], "held": st["held"],
                "cached": st["cached"], "free_list": st["free_list"], "free_count": st["free_count"]}
    if kind == "append":
        if own:
            st["kv"].append(st["step"], st["k"], st["v"])
        else:
            _plain_append(st["k"], st["k_codes"], st["k_exp"], st["slots"], case["page"])
            _plain_append(st["v"], st["v_codes"].transpose(2, 3), st["v_exp"], st["slots"], case["page"])
        return {"k": st["k_codes"].view(torch.float8_e4m3fn), "v": st["v_codes"].view(torch.float8_e4m3fn),
                "k_exp": st["k_exp"], "v_exp": st["v_exp"]}
    if kind == "attend":
        if own:
            return st["kv"].attend(st["step"], st["q"], n_causal=st["n_causal"], max_kv=st["max_kv"])
        return _plain_attend(st, case)
    if kind == "quantize":
        if own:
            from paper_2509_04185_amd import scaled_quantize
            codes, scale = scaled_quantize(st["x"], block_rows=case["block_rows"])
        else:
            codes, scale = _plain_quantize(st["x"], case["block_rows"])
        return {"codes": codes.view(torch.float8_e4m3fn), "scale": scale}
    if own:
        from paper_2509_04185_amd import scaled_matmul
        return scaled_matmul(st["a"], st["a_scale"], st["b"], st["b_scale"], out_dtype=TYPES[case["dtype"]])
    return _plain_matmul(st, TYPES[case["dtype"]])


def _plain_plan(st, page):
    table, held, cached, n_new, free, count = (st[k] for k in ("table", "held", "cached", "n_new", "free_list", "free_count"))
    batch, width = table.shape
    n_pages, rows = free.shape[0], st["rows"]
    col = torch.arange(width, device=DEV)[None, :]
    if st["release"] is not None:  # pages of sequences that ended go back, in the order of the tables
        gone = st["release"] != 0
        back = gone[:, None] & (col < held[:, None])
        at = torch.where(back, back.reshape(-1).cumsum(0).reshape(batch, width) - 1 + count, n_pages)
        free.copy_(torch.cat((free, free[:1])).scatter(0, at.reshape(-1), table.reshape(-1))[:n_pages])
        count += back.sum().to(torch.int32)
        table.masked_fill_(gone[:, None], -1)
        held.masked_fill_(gone, 0)
        cached.masked_fill_(gone, 0)
    total = cached + n_new
    fits = total <= width * page
    need = torch.where(fits, ((total + page - 1) // page - held).clamp_min(0), 0)
    end = need.cumsum(0)
    ok = fits & ((need == 0) | (end <= count))
    need = torch.where(ok, need, 0)
    start = end - need
    base = count - need.sum()
    at = (base + start)[:, None] + col - held[:, None]
    fresh = (col >= held[:, None]) & (col < (held + need)[:, None])
    table.copy_(torch.where(fresh, free[at.clamp(0, n_pages - 1)], table))
    held += need.to(torch.int32)
    count.copy_(base)
    row_start = torch.cat((torch.zeros(1, dtype=torch.int64, device=DEV), n_new.cumsum(0))).to(torch.int32)
    kv_len = torch.where(ok, total, 0).to(torch.int32)
    t = torch.arange(rows, device=DEV, dtype=torch.int32)
    b = torch.searchsorted(row_start[1:].contiguous(), t, right=True).clamp_max(batch - 1)
    p = cached[b] + t - row_start[b]
    slot = table[b, (p // page).clamp(0, width - 1)] * page + p % page
    slots = torch.where(ok[b] & (t < row_start[-1]), slot, -1).to(torch.int32)
    return row_start, kv_len, slots


def _exponent(amax):
    """Smallest e in [-100, 100] with amax <= 448 * 2^e."""
    f, e = torch.frexp(amax)
    return torch.where(amax > 0, e - 9 + (f > 0.875).to(e.dtype), -100).clamp(-100, 100)


def _pow2(e):
    """2^e in float32 for whole numbers e in [-126, 127], made from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _round8(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _plain_append(x, codes, exps, slots, page):
    """codes: [pages][heads][page][dim] (any strides); rows x [rows][heads][dim]."""
    n_pages, H = exps.shape
    row_page, row_off = (slots // page).long(), (slots % page).long()
    x = x.float()
    amax = torch.zeros((n_pages, H), device=DEV)
    amax = amax.scatter_reduce(0, row_page[:, None].expand(-1, H), x.abs().amax(-1), "amax")
    kept = torch.full((n_pages,), page, device=DEV).scatter_reduce(0, row_page, row_off, "amin")
    touched = torch.unique(row_page)
    old = exps[touched].int()
    keeps = kept[touched] > 0
    new = torch.where(keeps[:, None], torch.maximum(old, _exponent(amax[touched])), _exponent(amax[touched]))
    sub = codes[touched].contiguous()
    was = sub.view(torch.float8_e4m3fn).float()
    again = _round8(was * _pow2((old - new).clamp_min(-126))[:, :, None, None]).view(torch.uint8)
    first = torch.arange(page, device=DEV)[None, :] < kept[touched][:, None]
    sub = torch.where(first[:, None, :, None], again, sub)
    codes[touched] = sub
    exps[touched] = new.to(torch.int8)
    e = exps[row_page].int()[:, :, None]
    codes[row_page, :, row_off] = _round8(x * _pow2(-e)).view(torch.uint8)


def _plain_attend(st, case):
    page, H, dh, nq = case["page"], case["heads"], case["dh"], case["q_heads"]
    rs, kv_len, table, q = st["row_start"].long(), st["kv_len"].long(), st["table"].long(), st["q"]
    B, rows, G, N = table.shape[0], q.shape[0], nq // H, st["max_new"]
    P = _pages_of(st["max_kv"], page)
    L = P * page
    n = rs[1:] - rs[:-1]
    j = torch.arange(N, device=DEV)
    at = (rs[:-1, None] + j).clamp_max(max(0, rows - 1))
    qp = q[at].float().reshape(B, N, H, G, dh).permute(0, 2, 1, 3, 4).reshape(B, H, N * G, dh)
    pages = table[:, :P].clamp_min(0)
    ke, ve = _pow2(st["k_exp"][pages]), _pow2(st["v_exp"][pages])  # [B][P][H]
    k = st["k_codes"][pages].view(torch.float8_e4m3fn).float() * ke[..., None, None]         # [B][P][H][page][dh]
    v = st["v_codes"][pages].view(torch.float8_e4m3fn).float() * ve[..., None, None]         # [B][P][H][dh][page]
    kt = k.permute(0, 2, 4, 1, 3).reshape(B, H, dh, L).contiguous()
    v = v.permute(0, 2, 1, 4, 3).reshape(B, H, L, dh).contiguous()
    s = torch.matmul(qp, kt) * (1.0 / math.sqrt(dh))
    causal = n if st["n_causal"] is None else st["n_causal"].long()
    end = torch.where(j[None, :] < causal[:, None], (kv_len - n)[:, None] + j + 1, kv_len[:, None])
    end = torch.where(j[None, :] < n[:, None], end, 0)
    end = end[:, None, :, None].expand(B, 1, N, G).reshape(B, 1, N * G, 1)
    seen = torch.arange(L, device=DEV) < end
    s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    o = o.reshape(B, H, N, G, dh).permute(0, 2, 1, 3, 4).reshape(B, N, nq, dh)
    t = torch.arange(rows, device=DEV)
    b = torch.searchsorted(rs[1:].contiguous(), t, right=True)
    return o[b, t - rs[b]].to(q.dtype)


def _plain_quantize(x, block_rows):
    rows, cols = x.shape
    kb, rb = _pages_of(cols, 128), _pages_of(rows, block_rows)
    x = torch.nn.functional.pad(x.float(), (0, kb * 128 - cols, 0, rb * block_rows - rows))
    blocks = x.reshape(rb, block_rows, kb, 128)
    e = _exponent(blocks.abs().amax(3).amax(1))
    codes = _round8(blocks * _pow2(-e)[:, None, :, None])
    codes = codes.view(torch.uint8).reshape(rb * block_rows, kb * 128)[:rows, :cols].contiguous()
    scale = _pow2(e)
    return codes, scale.t().contiguous() if block_rows == 1 else scale


def _plain_matmul(st, dtype):
    a, b = st["a"].view(torch.float8_e4m3fn).float(), st["b"].view(torch.float8_e4m3fn).float()
    (m, k), n = a.shape, b.shape[0]
    a *= st["a_scale"].t().repeat_interleave(128, 1)[:, :k]
    b *= st["b_scale"].repeat_interleave(128, 1)[:, :k].repeat_interleave(128, 0)[:n]
    return torch.matmul(a, b.t()).to(dtype)


# ---- what a pass cannot do without


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n, es = case["rows"] * case["cols"], 4 if case["dtype"] == "fp32" else 2
        return {"bytes": n * (es + 1) + 4 * (n // (128 * case["block_rows"])), "flops": 2 * n}
    if kind == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        es = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": m * k + n * k + es * m * n + 4 * m * k // 128, "flops": 2 * m * n * k}
    lens, page = _lens(case), case["page"]
    rows = sum(n for _, n in lens)
    if kind == "plan":
        taken = sum(_pages_of(c * (not case["wave"]) + n, page) - (0 if case["wave"] else _pages_of(c, page)) for c, n in lens)
        given = sum(_pages_of(c, page) for c, _ in lens) if case["wave"] else 0
        return {"bytes": 4 * (rows + 6 * case["batch"] + 2 * taken + 3 * given), "flops": 4 * rows + 8 * case["batch"]}
    H, dh = case["heads"], case["dh"]
    if kind == "append":
        touched = sum(_pages_of(c + n, page) - c // page for c, n in lens if n)
        return {"bytes": 2 * rows * H * dh * 3 + 4 * rows + 4 * touched * H, "flops": 4 * rows * H * dh}
    pairs = 0
    for c, n in lens:
        nc = {"all": n, "one": min(1, n), "none": 0}[case["causal"]]
        pairs += sum(range(c + 1, c + nc + 1)) + (n - nc) * (c + n)
    keys = sum(c + n for c, n in lens if n)
    pages = sum(_pages_of(c + n, page) for c, n in lens if n)
    return {"bytes": 2 * keys * H * dh + pages * (4 + 2 * H) + 4 * rows * case["q_heads"] * dh,
            "flops": 4 * pairs * case["q_heads"] * dh}


# ---- the same in 64 bits, from the definitions


def _two_to(e):
    """2^e in float64 for whole numbers e in [-200, 200], from a table made on the host."""
    return torch.tensor([math.ldexp(1.0, i) for i in range(-200, 201)], dtype=torch.float64, device=DEV)[e.long() + 200]


def _of_codes(codes):
    """Values of e4m3 codes, from a table of all 256: sign, 4 exponent bits of bias 7, 3 mantissa bits."""
    vals = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        vals.append(-v if c >= 128 else v)
    return torch.tensor(vals, dtype=torch.float64, device=DEV)[codes.long()]


def _nearest8(y):
    """The e4m3 value nearest to y, ties to the even code, at most 448 in size."""
    a = y.abs()
    _, e = torch.frexp(a)
    step = _two_to((e - 1).clamp_min(-6) - 3)
    return torch.where(y < 0, -1.0, 1.0) * (torch.round(a / step) * step).clamp_max(448.0)


def _fits(amax):
    """2^e for the smallest e in [-100, 100] with amax <= 448 * 2^e, by trying every e."""
    powers = _two_to(torch.arange(-100, 101, device=DEV))
    return powers[torch.searchsorted(448.0 * powers, amax.double().contiguous()).clamp_max(200)]


def _exact_append(x, codes, exps, slots, lens, page):
    """codes [pages][heads][page][dim] as values, sequence by sequence and page by page."""
    vals = _of_codes(codes)
    at = 0
    host = slots.tolist()
    for _, n in lens:
        r = 0
        while r < n:
            pg, off = divmod(host[at + r], page)
            m = min(page - off, n - r)
            rows = x[at + r:at + r + m].double().permute(1, 0, 2)
            scale = _fits(rows.abs().amax((1, 2)))
            if off:
                old = _two_to(exps[pg])
                scale = torch.maximum(scale, old)
                vals[pg, :, :off] = _nearest8(vals[pg, :, :off] * (old / scale)[:, None, None])
            vals[pg, :, off:off + m] = _nearest8(rows / scale[:, None, None])
            r += m
        at += n
    return vals


def exact(case, seed):
    kind = case["kind"]
    if kind == "plan":
        return None  # whole numbers only
    st = prepare(case, seed)
    if kind == "quantize":
        br, x = case["block_rows"], st["x"]
        rows, cols = x.shape
        kb, rb = _pages_of(cols, 128), _pages_of(rows, br)
        scale = torch.empty((rb, kb), dtype=torch.float64, device=DEV)
        vals = torch.empty((rows, cols), dtype=torch.float64, device=DEV)
        for c in range(kb):
            part = x[:, 128 * c:128 * c + 128].double()
            top = part.abs().amax(1)
            if br > 1:
                full = torch.zeros(rb * br, dtype=torch.float64, device=DEV)
                full[:rows] = top
                top = full.reshape(rb, br).amax(1)
            scale[:, c] = _fits(top)
            vals[:, 128 * c:128 * c + 128] = _nearest8(part / scale[:, c].repeat_interleave(br)[:rows, None])
        return {"codes": vals, "scale": scale.t().contiguous() if br == 1 else scale}
    if kind == "matmul":
        a, b = _of_codes(st["a"]), _of_codes(st["b"])
        out = torch.zeros((case["m"], case["n"]), dtype=torch.float64, device=DEV)
        wide = torch.arange(case["n"], device=DEV) // 128
        for c in range(_pages_of(case["k"], 128)):
            part = slice(128 * c, min(case["k"], 128 * c + 128))
            out += (a[:, part] @ b[:, part].t()) * (st["a_scale"][c].double()[:, None] * st["b_scale"][:, c].double()[wide])
        return out
    lens, page = _lens(case), case["page"]
    if kind == "append":
        k = _exact_append(st["k"], st["k_codes"], st["k_exp"], st["slots"], lens, page)
        v = _exact_append(st["v"], st["v_codes"].transpose(2, 3), st["v_exp"], st["slots"], lens, page)
        return {"k": k, "v": v.transpose(2, 3).contiguous(), "k_exp": None, "v_exp": None}
    H, dh, nq = case["heads"], case["dh"], case["q_heads"]
    out = torch.zeros((st["rows"], nq, dh), dtype=torch.float64, device=DEV)
    row = 0
    for b, (c, n) in enumerate(lens):
        if n == 0:
            continue
        L = c + n
        pages = st["table"][b, :_pages_of(L, page)].long()
        nc = {"all": n, "one": min(1, n), "none": 0}[case["causal"]]
        for h in range(H):
            k = _of_codes(st["k_codes"][pages, h]) * _two_to(st["k_exp"][pages, h])[:, None, None]
            v = _of_codes(st["v_codes"][pages, h]) * _two_to(st["v_exp"][pages, h])[:, None, None]
            k, v = k.reshape(-1, dh)[:L], v.transpose(1, 2).reshape(-1, dh)[:L]
            for g in range(nq // H):
                q = st["q"][row:row + n, h * (nq // H) + g].double()
                s = (q @ k.t()) / math.sqrt(dh)
                hidden = torch.ones((nc, n), dtype=torch.bool, device=DEV).triu(1)
                s[:nc, c:].masked_fill_(hidden, -math.inf)
                out[row:row + n, h * (nq // H) + g] = torch.softmax(s, -1) @ v
        row += n
    return out
