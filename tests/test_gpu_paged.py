"""The paged e4m3 cache on the GPU against plain 64-bit forms (ops_ref.py): tables and slots
(whole numbers, equal), the write (codes and exponents, equal), attention (within the bound that
its types give), alone and together."""
import math

import numpy as np
import pytest
import torch

import ops_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, FP = torch.bfloat16, torch.float16


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def host(t):
    return t.cpu().numpy()


# ---- tables and slots ---------------------------------------------------------------------


def check_plan(pages, state, n_new, rows, release=None):
    """One plan on the GPU and on the host arrays `state`; returns the state after it."""
    step = pages.plan(ints(n_new), rows, release=None if release is None else
                      torch.tensor(release, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    table, held, cached, free, count, starts, kv, slots = R.plan(*state, n_new, release, rows, pages.page_size)
    assert np.array_equal(host(pages.table), table)
    assert np.array_equal(host(pages.held), held)
    assert np.array_equal(host(pages.cached), cached)
    assert int(pages.free_count) == count
    assert np.array_equal(host(pages.free_list)[:count], free[:count])
    assert np.array_equal(host(step.row_start), starts)
    assert np.array_equal(host(step.kv_len), kv)
    assert np.array_equal(host(step.slots), slots)
    return table, held, cached, free, count


def state_of(p):
    return host(p.table), host(p.held), host(p.cached), host(p.free_list), int(p.free_count)


@pytest.mark.parametrize("batch,max_len,n_pages,page,top", [
    (1, 64, 4, 16, 20),        # one sequence
    (5, 300, 40, 32, 60),      # a few; the pool runs out
    (64, 1000, 900, 16, 90),   # a wave of lanes
    (65, 500, 4000, 16, 40),   # one more
    (300, 2100, 3000, 64, 200),  # more entries than one workgroup takes
    (1500, 700, 9000, 128, 30),  # more sequences than threads of the scans
], ids=lambda v: str(v))
def test_plan_over_many_steps(batch, max_len, n_pages, page, top):
    from paper_2509_04185_amd import PageTable
    print(f"[gpu] plan: {batch} sequences, {n_pages} pages of {page}", flush=True)
    rng = np.random.default_rng(batch * 7 + page)
    pages = PageTable.empty(batch, max_len, n_pages, page)
    perm = rng.permutation(n_pages)
    pages.free_list.copy_(ints(perm))
    for step in range(8):
        n_new = rng.integers(0, top + 1, batch) * (rng.random(batch) < 0.8)
        release = (rng.random(batch) < 0.3).astype(np.uint8) if step % 2 else None
        if step == 3:
            release[:] = 1
        state = check_plan(pages, state_of(pages), n_new, int(n_new.sum()) + (step % 3) * 5, release)
        # every page is held once or free
        table, held, _, free, count = state
        all_pages = np.concatenate([table[b, :held[b]] for b in range(batch)] + [free[:count]])
        assert np.array_equal(np.sort(all_pages), np.arange(n_pages))
        kv = np.array(host(pages.cached))
        commit = (rng.random(batch) * (n_new + 1)).astype(np.int64)
        served = held * page >= kv + n_new
        pages.cached += ints(np.where(served, np.minimum(commit, n_new), 0))


def test_plan_refuses_sequences_not_steps():
    """Negative lengths, lengths beyond the table and a short pool leave those sequences out; the
    rest are served, a sequence that needs no page even behind one that got none."""
    from paper_2509_04185_amd import PageTable
    pages = PageTable.empty(6, 64, 5, 16)
    pages.cached.copy_(ints([0, -3, 0, 0, 0, 0]))
    state = check_plan(pages, state_of(pages), np.array([30, 5, 65, -2, 16, 0]), 120)
    assert host(pages.held).tolist() == [2, 0, 0, 0, 1, 0]
    # two pages left: sequence 3 gets them, 4 needs one more than is left, 0 has room in its pages
    pages.cached.copy_(ints([30, 0, 0, 0, 16, 0]))
    check_plan(pages, state_of(pages), np.array([2, 0, 0, 32, 16, 1]), 60)
    assert host(pages.held).tolist() == [2, 0, 0, 2, 1, 0]


def test_plan_rows_shorter_than_the_step():
    """Fewer rows than the lengths add up to: the slots that there are, nothing behind them."""
    from paper_2509_04185_amd import PageTable
    pages = PageTable.empty(3, 200, 30, 16)
    buf = pages.plan(ints([40, 40, 40]), 50).slots
    ref = R.plan(-np.ones((3, 13)), np.zeros(3), np.zeros(3), np.arange(30), 30, np.array([40, 40, 40]), None, 50, 16)
    assert np.array_equal(host(buf), ref[-1])
    assert pages.plan(ints([0, 0, 0]), 0).slots.numel() == 0


# ---- write into the cache ------------------------------------------------------------------


def make_cache(n_pages, page, heads, dh, seed, spread=3):
    """A cache of random codes (no NaN) and exponents, and the same as host arrays."""
    from paper_2509_04185_amd import PagedKV
    g = torch.Generator().manual_seed(seed)
    kv = PagedKV.empty(n_pages, page, heads, dh)
    for t in (kv.k_codes, kv.v_codes):
        x = (torch.randn(t.shape, generator=g) * 110).clamp(-448, 448).to(torch.float8_e4m3fn)
        t.copy_(x.view(torch.uint8))
    for t in (kv.k_exp, kv.v_exp):
        t.copy_(torch.randint(-7 - spread, -6, t.shape, generator=g, dtype=torch.int8))
    return kv


def make_step(lens, page, n_pages, seed, pad=0, width=None, rows=None):
    """A step by hand: (cached, new) per sequence, pages in random order."""
    from paper_2509_04185_amd import PagedStep
    rng = np.random.default_rng(seed)
    need = [-(-(c + n) // page) for c, n in lens]
    width = width or max(1, max(need))
    perm = rng.permutation(n_pages)
    assert sum(need) <= n_pages
    table, at = np.full((len(lens), width), -1, np.int64), 0
    starts = np.concatenate([[0], np.cumsum([n for _, n in lens])]).astype(np.int64)
    slots = np.full(int(starts[-1]) + pad, -1, np.int64)
    for b, (c, n) in enumerate(lens):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
        p = np.arange(c, c + n)
        slots[starts[b]:starts[b + 1]] = table[b, p // page] * page + p % page
    kv_len = np.array([c + n for c, n in lens])
    step = PagedStep(ints(table), ints(starts), ints(kv_len), ints(slots), page)
    return step, table, starts, kv_len, slots


def check_append(lens, page, heads, dh, dtype, seed=0, edit=None, strided=False, pad=3, spread=3):
    n_pages = sum(-(-(c + n) // page) for c, n in lens) + 3
    kv = make_cache(n_pages, page, heads, dh, seed, spread)
    step, table, starts, kv_len, slots = make_step(lens, page, n_pages, seed, pad)
    g = torch.Generator().manual_seed(seed + 1)
    rows = len(slots)
    x = torch.randn((rows, 2 * heads + 3, dh), generator=g) * torch.exp(torch.randn((rows, 1, 1), generator=g))
    x = x.to(dtype)
    if edit:
        edit(x)
    x = x.to(DEV)
    k, v = x[:, :heads], x[:, heads:2 * heads]
    if not strided:
        k, v = k.contiguous(), v.contiguous()
    want = []
    for codes, exps, t in ((kv.k_codes, kv.k_exp, k), (kv.v_codes.transpose(2, 3), kv.v_exp, v)):
        vals, e = R.VALUES[host(codes)], host(exps).astype(np.int64)
        R.append(vals, e, R.f64(t), starts, slots, page)
        want.append((vals, e))
    kv.append(step, k, v)
    torch.cuda.synchronize()
    for (vals, e), codes, exps in zip(want, (kv.k_codes, kv.v_codes.transpose(2, 3)), (kv.k_exp, kv.v_exp)):
        assert np.array_equal(host(exps), e)
        assert np.array_equal(R.VALUES[host(codes)], vals, equal_nan=True)
    return kv


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_append_ragged(page, dtype):
    print(f"[gpu] append, pages of {page}, {dtype}", flush=True)
    lens = [(0, 1), (page - 1, 1), (page, 1), (5, 0), (page - 1, 2), (3, 3 * page + 1), (2 * page - 7, 8), (0, page)]
    check_append(lens, page, 3, 128, dtype, seed=page)


@pytest.mark.parametrize("heads,dh", [(1, 64), (8, 128), (2, 64)])
@pytest.mark.parametrize("strided", [False, True])
def test_append_shapes(heads, dh, strided):
    check_append([(70, 9), (0, 130), (31, 1)], 64, heads, dh, BF, seed=heads, strided=strided)


def test_append_exponent_grows_and_rounds_again():
    """Kept codes are rounded again when a larger row enters their page, up to the full range."""
    def edit(x):
        x[0:3] *= 2.0 ** 20       # the kept codes lose all but their largest
        x[3:5] = 0                # nothing but zeros: the page's exponent stays
        x[5:9] *= 2.0 ** -30
    kv = check_append([(9, 3), (20, 2), (0, 4), (33, 1)], 16, 2, 64, BF, seed=5, edit=edit, spread=20)
    assert int(kv.k_exp.max()) > 8


def test_append_infinities_nan_zero_and_the_ends_of_the_range():
    def edit(x):
        x[0, :, :3] = torch.tensor([math.inf, -math.inf, math.nan], dtype=x.dtype)
        x[1] = math.nan           # no finite value in the page: exponent -100
        x[2] = 0
        x[3] = 3e38               # beyond 448 * 2^100: saturates
        x[4, :, :4] = torch.tensor([1e-38, -1e-39, 2e-38, 0.0], dtype=x.dtype)
        x[4, :, 4:] = 0
        x[5, :, :] = 448.0        # exactly at the border of an exponent
        x[6, :, :] = 450.0
    check_append([(0, 1), (0, 1), (0, 1), (0, 1), (0, 1), (0, 1), (0, 1), (7, 2)], 16, 2, 64, BF, seed=6, edit=edit)


def test_append_every_rounding():
    """Every e4m3 value, every midpoint and their neighbours in bf16, in one page."""
    vals = np.unique(R.VALUES[np.isfinite(R.VALUES)])
    mids = (vals[1:] + vals[:-1]) / 2
    x = np.concatenate([vals, mids, mids * (1 + 2.0 ** -8), mids * (1 - 2.0 ** -8)])
    x = np.concatenate([x, np.full(-len(x) % 128, 448.0)])
    n = len(x) // 128

    def edit(t):
        t[:n] = torch.tensor(x).reshape(n, 1, 128).to(t.dtype)
        t[0, :, 0] = 448.0
    check_append([(0, n)], 16, 2, 128, BF, seed=8, edit=edit, pad=0)


def test_append_leaves_out_bad_slots():
    """Slots outside the cache are skipped with their page; nothing else changes."""
    from paper_2509_04185_amd import PagedKV, PagedStep
    kv = make_cache(4, 16, 2, 64, 1)
    before = [t.clone() for t in (kv.k_codes, kv.v_codes, kv.k_exp, kv.v_exp)]
    x = torch.ones((6, 2, 64), dtype=BF, device=DEV)
    for slots, starts in (([-1] * 6, [0, 3, 6]), ([64, 65, 66, 10 ** 9, 2 ** 31 - 1, -5], [0, 3, 6]),
                          ([0, 1, 2, 3, 4, 5], [0, 0, 0]), ([0, 1, 2, 3, 4, 5], [-4, -2, -1])):
        step = PagedStep(ints(np.zeros((2, 1))), ints(starts), ints([3, 3]), ints(slots), 16)
        kv.append(step, x, x)
    torch.cuda.synchronize()
    for t, old in zip((kv.k_codes, kv.v_codes, kv.k_exp, kv.v_exp), before):
        assert torch.equal(t, old)
    assert isinstance(kv, PagedKV)


# ---- attention -----------------------------------------------------------------------------


def check_attend(lens, page, heads, group, dh, dtype, causal="all", seed=0, pad=2, edit=None, edit_q=None, scale=None,
                 max_kv=None, strided=False, spread=3, edit_table=None, served=None, only=None):
    n_pages = sum(-(-(c + n) // page) for c, n in lens) + 2
    kv = make_cache(n_pages, page, heads, dh, seed, spread)
    step, table, starts, kv_len, slots = make_step(lens, page, n_pages, seed, pad)
    # what no sequence has written is the worst there is: NaN codes behind every sequence's end
    for b, (c, n) in enumerate(lens):
        if (c + n) % page:
            pg, off = int(table[b, (c + n) // page]), (c + n) % page
            kv.k_codes[pg, :, off:] = 0x7f
            kv.v_codes[pg, :, :, off:] = 0xff
    if edit:
        edit(kv, table)
    if edit_table:
        edit_table(table)
        step.table.copy_(ints(table))
    if served is not None:
        kv_len = np.where(served, kv_len, 0)
        step.kv_len.copy_(ints(kv_len))
    g = torch.Generator().manual_seed(seed + 2)
    rows, nq = len(slots), heads * group
    q = torch.randn((rows, nq + (3 if strided else 0), dh), generator=g).to(dtype)
    if edit_q:
        edit_q(q)
    q = q.to(DEV)[:, :nq]
    n_causal = {"all": None, "one": [min(1, n) for _, n in lens], "none": [0] * len(lens),
                "half": [n // 2 for _, n in lens]}[causal]
    out = torch.full((rows, nq + 2, dh), 7.0, dtype=dtype, device=DEV)
    got = kv.attend(step, q, n_causal=None if n_causal is None else ints(n_causal), scale=scale, max_kv=max_kv,
                    out=out[:, :nq] if strided else None)
    torch.cuda.synchronize()
    real = int(starts[-1])
    if strided:
        assert bool((out[:, nq:] == 7).all()) and bool((out[real:] == 7).all())
    want, bound = R.attend(R.f64(q), host(kv.k_codes), host(kv.v_codes), host(kv.k_exp), host(kv.v_exp), table, starts,
                           kv_len, n_causal, scale or 1 / math.sqrt(dh), page, dtype, only=only)
    rows = list(range(real)) if only is None else sorted(only)
    share = R.worst(R.f64(got)[rows], want[rows], bound[rows])
    print(f"    largest error {share:.3f} of its bound", flush=True)
    assert share <= 1.0
    return got, want


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_attend_lengths_around_pages_and_stages(page, dtype):
    """One row each over 1 .. a few hundred keys, around the ends of pages and of key stages."""
    print(f"[gpu] attend, pages of {page}, {dtype}", flush=True)
    lens = [(c, 1) for c in (0, 1, 14, 15, 16, 30, 31, 62, 63, 64, 127, 128, 254, 255, 256, 300, 511, 512)]
    check_attend(lens, page, 2, 2, 128, dtype, seed=page)


@pytest.mark.parametrize("heads,group,dh", [(1, 1, 64), (2, 4, 128), (1, 16, 128), (3, 5, 64), (8, 1, 128), (1, 71, 64)])
@pytest.mark.parametrize("causal", ["all", "one", "none", "half"])
def test_attend_heads_and_masks(heads, group, dh, causal):
    lens = [(100, 7), (0, 3), (40, 0), (65, 1), (513, 16)]
    check_attend(lens, 32, heads, group, dh, BF, causal, seed=group)


@pytest.mark.parametrize("batch", [63, 64, 65, 130, 4200])
def test_many_sequences(batch):
    """More sequences than a wave looks at at once, some without rows."""
    lens = [((7 * b) % 90, (5 * b) % 4) for b in range(batch)]
    check_append(lens, 16, 1, 64, BF, seed=batch)
    check_attend(lens, 16, 1, 2, 64, BF, "one", seed=batch)


@pytest.mark.parametrize("lens", [[(0, 300)], [(37, 129), (0, 64), (900, 65)], [(0, 1), (0, 2), (3000, 40)]],
                         ids=lambda v: str(v))
@pytest.mark.parametrize("dh", [64, 128])
def test_attend_prompts(lens, dh):
    check_attend(lens, 64, 2, 2, dh, BF, "all", seed=len(lens), strided=True)
    check_attend(lens, 16, 1, 4, dh, FP, "half", seed=len(lens) + 1)


@pytest.mark.parametrize("heads,group,dh,page,dtype", [(8, 4, 128, 64, BF), (8, 1, 64, 16, FP), (4, 8, 128, 32, FP),
                                                       (8, 5, 64, 128, BF)], ids=lambda v: str(v))
def test_attend_long_prompts(heads, group, dh, page, dtype):
    """Prompts of thousands of rows, some behind a cached prefix: rows at the ends of tiles and
    sequences against the plain form, all of them finite."""
    lens = [(0, 1), (700, 1333), (0, 0), (33, 1500), (0, 17)]
    ends = np.cumsum([n for _, n in lens])
    near = [e + d for e in ends for d in (-2, -1, 0, 1)] + [32 * i + d for i in range(0, 85, 9) for d in (-1, 0)]
    only = {int(r) for r in near if 0 <= r < ends[-1]}
    for causal in ("all", "half"):
        got, _ = check_attend(lens, page, heads, group, dh, dtype, causal, seed=heads + group, only=only)
        assert bool(torch.isfinite(got[:int(ends[-1])]).all())


@pytest.mark.parametrize("max_kv", [1, 64, 256, 257, 1000, 5008])
def test_attend_any_split(max_kv):
    """The hint only decides how the keys are split: too small or too large, the same result."""
    check_attend([(5000, 8), (3, 8), (700, 8)], 64, 2, 4, 128, BF, "one", seed=3, max_kv=max_kv, strided=True)


def test_attend_unserved_missing_and_empty_rows():
    """A sequence that was not served gives zeros; pages missing from the table are not seen."""
    served = np.array([True, False, True, True])
    for max_kv in (16, 304):
        got, want = check_attend([(70, 4), (90, 4), (0, 2), (300, 3)], 16, 2, 2, 64, BF, "one", seed=9, served=served,
                                 max_kv=max_kv)
        assert bool((got[4:8] == 0).all())

    def lose(table):
        table[0, 1], table[0, 3] = -1, 10 ** 6
        table[2, 0] = -7               # all that sequence 2 has
        table[3, :4] = -1              # a whole stage
    got, want = check_attend([(70, 4), (90, 4), (0, 2), (300, 3)], 16, 2, 2, 64, FP, "none", seed=10, edit_table=lose)
    assert bool((got[8:10] == 0).all())


def test_attend_nan_reaches_only_rows_that_see_it():
    """NaN keys and values inside a block: rows in front of them stay clean, rows that see them are NaN
    (a value in its own dimension only)."""
    def edit(kv, table):
        kv.v_codes[int(table[0, 4]), 0, 5, 3] = 0x7f       # position 67, dim 5, head 0
        kv.k_codes[int(table[1, 0]), 1, 9, 2] = 0xff       # position 9 of the second sequence, head 1
    got, want = check_attend([(60, 12), (4, 9)], 16, 2, 2, 64, BF, "all", seed=11, edit=edit)
    nan = torch.isnan(got[:21]).cpu().numpy()
    assert nan[:12].sum() == 2 * 5 and nan[7:12, :2, 5].all()
    assert nan[12:].sum() == 2 * 4 * 64 and nan[12 + 5:, 2:].all()


def test_attend_nan_query_and_large_scores():
    def edit_q(q):
        q[1] = math.nan
        q[2] *= 300          # one key takes all the weight
        q[3] = 0             # all keys alike
        q[4] *= 1e-3
    check_attend([(200, 8)], 64, 2, 2, 128, BF, "none", seed=12, edit_q=edit_q)
    check_attend([(200, 8)], 64, 2, 2, 128, BF, "none", seed=12, scale=-0.3)


def test_attend_exponents_far_apart():
    """Runs of one stage whose values differ by more than fp16 holds, and pages of zeros."""
    def edit(kv, table):
        kv.v_exp[int(table[0, 0])] = 20
        kv.v_exp[int(table[0, 1])] = -30
        kv.v_exp[int(table[0, 2])] = -100
        kv.v_codes[int(table[0, 2])] = 0
        kv.k_exp[int(table[0, 3])] = -100
        kv.k_exp[int(table[0, 1])] = -2
    check_attend([(90, 6)], 16, 2, 2, 64, BF, "one", seed=13, edit=edit)

    def low(kv, table):   # one page of the stage holds all the weight and the smallest values
        kv.v_exp[int(table[0, 0])] = 30
        kv.v_exp[int(table[0, 1])] = -20
        kv.k_codes[int(table[0, 0])] = 0
        kv.k_codes[int(table[0, 1])] = 0x78

    def q(x):
        x[:] = 1.0
        x[:, :, 0] = 2.0
    check_attend([(30, 2)], 16, 1, 2, 64, BF, "none", seed=14, edit=low, edit_q=q)


def test_attend_the_ends_of_the_exponents():
    def edit(kv, table):
        kv.v_exp[:] = 100
        kv.k_exp[:] = -100
    check_attend([(90, 6)], 64, 2, 2, 64, BF, "one", seed=15, edit=edit)

    def small(kv, table):
        kv.v_exp[:] = -100
    check_attend([(90, 6)], 64, 2, 2, 64, BF, "one", seed=16, edit=small)


def test_attend_pages_shared_and_repeated():
    """Two sequences with a common prefix, and a page that one sequence reads twice."""
    def share(table):
        table[1, :4] = table[0, :4]
        table[2, 3] = table[2, 1]
    check_attend([(100, 3), (80, 2), (70, 5)], 16, 2, 4, 64, BF, "all", seed=17, edit_table=share)


def test_offsets_beyond_32_bits():
    """A cache of 5 GB codes: rows written to and read from its last pages."""
    from paper_2509_04185_amd import PagedKV, PagedStep
    n_pages, page, H, dh = 80000, 64, 8, 128
    kv = PagedKV.empty(n_pages, page, H, dh)
    g = torch.Generator().manual_seed(21)
    rows = 100
    x = torch.randn((rows, 3 * H, dh), generator=g).to(BF).to(DEV)
    table = np.array([[n_pages - 1, n_pages - 2]])
    p = np.arange(rows)
    step = PagedStep(ints(table), ints([0, rows]), ints([rows]), ints(table[0, p // page] * page + p % page), page)
    kv.append(step, x[:, H:2 * H], x[:, 2 * H:])
    got = kv.attend(step, x[:, :H])
    # the same in a small cache
    small = PagedKV.empty(2, page, H, dh)
    s2 = PagedStep(ints([[1, 0]]), ints([0, rows]), ints([rows]), ints((1 - p // page) * page + p % page), page)
    small.append(s2, x[:, H:2 * H], x[:, 2 * H:])
    want = small.attend(s2, x[:, :H])
    torch.cuda.synchronize()
    tail = rows - page   # rows of the second page, which is page 0 of the small cache
    same = [torch.equal(kv.k_codes[-1], small.k_codes[1]), torch.equal(kv.v_codes[-1], small.v_codes[1]),
            torch.equal(kv.k_codes[-2, :, :tail], small.k_codes[0, :, :tail]),
            torch.equal(kv.v_codes[-2, :, :, :tail], small.v_codes[0, :, :, :tail]),
            torch.equal(kv.k_exp[-2:], small.k_exp), torch.equal(kv.v_exp[-2:], small.v_exp), torch.equal(got, want)]
    assert same == [True] * 7


# ---- together ------------------------------------------------------------------------------


def test_steps_of_a_serving_batch():
    """Prompts, then blocks with commits, then a sequence that ends and another in its place: after
    every step the attention equals that over the keys and values of a plain list."""
    from paper_2509_04185_amd import PagedKV, PageTable
    page, H, G, dh, B = 16, 2, 2, 64, 3
    pages = PageTable.empty(B, 200, 30, page)
    kv = PagedKV.empty(30, page, H, dh)
    kv.k_codes.fill_(0x7f)
    kv.v_codes.fill_(0x7f)
    g = torch.Generator().manual_seed(31)
    steps = [([33, 0, 18], None, [33, 0, 18]), ([8, 21, 8], None, [1, 21, 0]), ([8, 8, 8], None, [3, 1, 8]),
             ([8, 40, 8], [0, 1, 0], [8, 40, 1]), ([1, 1, 1], None, [1, 1, 1])]
    state = state_of(pages)
    vals = {n: (np.full((30, H, page, dh), np.nan), np.zeros((30, H), np.int64)) for n in "kv"}
    for i, (n_new, release, commit) in enumerate(steps):
        print(f"    step {i}", flush=True)
        rows = sum(n_new) + 3
        x = torch.randn((rows, H * (G + 2), dh), generator=g).to(BF).to(DEV)
        q, k, v = x[:, :H * G], x[:, H * G:H * (G + 1)], x[:, H * (G + 1):]
        step = pages.plan(ints(n_new), rows,
                          release=None if release is None else torch.tensor(release, dtype=torch.uint8, device=DEV))
        kv.append(step, k, v)
        got = kv.attend(step, q, n_causal=ints(commit))
        torch.cuda.synchronize()
        *state, starts, kv_len, slots = R.plan(*state, np.array(n_new), release, rows, page)
        for n, t in (("k", k), ("v", v)):
            R.append(*vals[n], R.f64(t), starts, slots, page)
        assert np.array_equal(R.VALUES[host(kv.k_codes)], vals["k"][0], equal_nan=True)
        assert np.array_equal(R.VALUES[host(kv.v_codes)].swapaxes(2, 3), vals["v"][0], equal_nan=True)
        want, bound = R.attend(R.f64(q), host(kv.k_codes), host(kv.v_codes), vals["k"][1], vals["v"][1], state[0],
                               starts, kv_len, commit, 1 / math.sqrt(dh), page, BF)
        assert R.worst(R.f64(got)[:sum(n_new)], want[:sum(n_new)], bound[:sum(n_new)]) <= 1.0
        pages.cached += ints(commit)
        state[2] = state[2] + np.array(commit)


def test_layer_of_a_context_in_pages():
    """A context's own cache moved into pages: its exported keys and values appended, and the
    attention of its last block against the one that its forward computed ("q" and "attn" of the
    last layer, over bf16 keys and values).

    Bound: a key, a value and a query change by at most r = 2^-4 (e4m3) or 2^-8 (bf16) of
    themselves, or by half of the smallest code 2^-10 at their page's scale.  A score then moves
    by at most d = sum |q| |k| (r_q + r_k + r_q r_k) + the small codes' share, every weight by a
    factor of at most exp(2 d), and a value as stated."""
    import synth
    from paper_2509_04185_amd import PagedKV, PageTable, Sbd
    s = synth.TINY
    w = synth.make_weights(s, 6100, device=DEV)
    lib = Sbd(s, w, max_batch=1, max_seq_len=128, max_block=8)
    n, k, page = 70, 8, 16
    rng = np.random.default_rng(6100)
    lib.prefill(0, rng.integers(0, s.vocab - 1, n))
    toks = np.full((1, k), s.mask_id)
    toks[0, 0] = 5
    lib.block_forward([0], toks)
    H, nq, dh = s.n_kv_heads, s.n_q_heads, s.head_dim
    q2 = lib.region("q").view(2, -1, nq * dh)[:, :k].float().sum(0)   # rotated, times log2(e) / sqrt(dh)
    o2 = lib.region("attn").view(2, -1, nq * dh)[:, :k].float().sum(0)
    kk, vv = (t[s.n_layers - 1] for t in lib.kv_export(0, 0, n + k))
    pages, kv = PageTable.empty(1, 128, 8, page), PagedKV.empty(8, page, H, dh)
    kv.append(pages.plan(ints([n]), n), kk[:n], vv[:n])
    pages.cached += n
    step = pages.plan(ints([k]), k)
    kv.append(step, kk[n:], vv[n:])
    got = kv.attend(step, q2.view(k, nq, dh).to(BF), n_causal=ints([1]), scale=math.log(2.0))
    torch.cuda.synchronize()
    got, o2, q = R.f64(got), R.f64(o2).reshape(k, nq, dh), R.f64(q2).reshape(k, nq, dh)
    K, V = R.f64(kk), R.f64(vv)
    ks, vs = (2.0 ** (float(t.max()) - 10) for t in (kv.k_exp, kv.v_exp))
    worst = 0.0
    for j in range(k):
        end = n + 1 if j < 1 else n + k
        for h in range(nq):
            kh, vh, x = K[:end, h // (nq // H)], V[:end, h // (nq // H)], q[j, h]
            p = np.exp((kh @ x) * math.log(2.0))
            p /= p.sum()
            rq, rk = 2.0 ** -8, 2.0 ** -4
            d = float(((np.abs(kh) @ np.abs(x)) * (rq + rk + rq * rk) + ks * np.abs(x).sum() * (1 + rq)).max()) * math.log(2.0)
            f = math.exp(2 * d)
            bound = (f * (1 + rk) - 1) * (p @ np.abs(vh)) + f * vs + 2.0 ** -8 * np.abs(got[j, h]) + 1e-3 * np.abs(o2[j, h])
            worst = max(worst, float((np.abs(got[j, h] - o2[j, h]) / bound).max()))
    print(f"    largest difference {worst:.3f} of its bound, {np.linalg.norm(got - o2) / np.linalg.norm(o2):.4f} in all", flush=True)
    assert worst <= 1.0
    lib.close()
