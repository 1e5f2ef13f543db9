"""The paged 8-bit cache on the GPU: tables, storing, reading back, decode and prefill attention against 64-bit arithmetic (page_ref)."""
import numpy as np
import pytest
import torch

import page_ref as ref
from paper_2603_22910_amd import binding as ek

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MHA, GQA, NARROW = (4, 4, 128), (8, 2, 128), (12, 2, 64)


class Batch:
    """A batch with its rows on the CPU beside the GPU's cache."""

    def __init__(self, layer, batch, max_pages=40, n_pages=200, seed=0, out_dtype="bf16", scale=0.0):
        self.hq, self.hkv, self.d = layer
        self.shape = ek.make_shape(*layer, 0, "bf16", out_dtype, scale)
        self.scale = scale or self.d ** -0.5
        self.batch, self.gen = batch, torch.Generator().manual_seed(seed)
        self.table = ek.PageTable.empty(batch, max_pages, n_pages, DEV)
        self.table.free_list.copy_(torch.randperm(n_pages, generator=self.gen, dtype=torch.int32))
        self.cache = ek.PageCache.empty(self.shape, batch, n_pages, DEV)
        self.rows = [[torch.empty(0, self.hkv, self.d, dtype=torch.bfloat16) for _ in range(2)] for _ in range(batch)]
        self.plan = None

    def random(self, *size, scale=1.0):
        return (torch.randn(*size, generator=self.gen) * scale).to(torch.bfloat16)

    def grow(self, n_new, rows=None, slack=0, stream=None):
        """Appends random rows (or the given ones); returns slots and positions."""
        total = sum(n_new)
        new = rows or [self.random(total + slack, self.hkv, self.d) for _ in range(2)]
        self.plan = ek.PagePlan.empty(self.batch, total + slack, DEV)
        self.slot, self.pos = (torch.full((max(1, total + slack),), 77, dtype=torch.int32, device=DEV) for _ in range(2))
        ek.pages_grow(self.shape, self.table, torch.tensor(n_new, dtype=torch.int32, device=DEV), self.plan, row_slot=self.slot, row_pos=self.pos)
        ek.page_append(self.shape, self.table, self.cache, self.plan, *(x.flatten(1).to(DEV) for x in new))
        at = 0
        for b, n in enumerate(n_new):
            for s in range(2):
                self.rows[b][s] = torch.cat([self.rows[b][s], new[s][at:at + n]])
            at += n
        return self

    def held(self, b):
        return [ref.held(x) for x in self.rows[b]]

    def workspace(self, rows=None):
        n = ek.page_workspace_bytes(self.shape, self.batch, self.plan.max_rows if rows is None else rows)
        return torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)             # NaN wherever it is read before it is written

    def out(self, rows):
        t = torch.float32 if self.shape.out_dtype == ek.F32 else torch.bfloat16
        return torch.full((rows, self.hq, self.d), 3.0, dtype=t, device=DEV), torch.full((rows, self.hq), 3.0, device=DEV)

    def decode(self, q, **kw):
        out, lse = self.out(self.batch)
        ek.page_decode_attn(self.shape, self.table, self.cache, self.plan, q.to(DEV), out, lse, self.workspace(), **kw)
        return out.cpu(), lse.cpu()

    def prefill(self, q, **kw):
        out, lse = self.out(max(1, self.plan.max_rows))
        ek.page_prefill_attn(self.shape, self.table, self.cache, self.plan, q.to(DEV), out, lse, self.workspace(), **kw)
        return out.cpu(), lse.cpu()

    def check(self, got, lse, q, b, positions, p_half, cap=0.0, slopes=None, prefix=0):
        k, v = self.held(b)
        want = ref.attend(q, k, v, positions, self.scale, cap, slopes, prefix)
        out_half = ref.HALF_F32 if got.dtype == torch.float32 else ref.HALF_BF16
        tol, tol_lse = ref.tolerances(*want, len(k), self.d, out_half, p_half, cap)
        assert torch.isfinite(got).all()
        assert ((got.double() - want[0]).abs() <= tol).all(), float(((got.double() - want[0]).abs() / tol).max())
        assert ((lse.double() - want[1]).abs() <= tol_lse).all(), float(((lse.double() - want[1]).abs() / tol_lse).max())


SLOPES = lambda hq: torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)])
# probabilities enter the second product as a pair of bf16 numbers in decode (2^-16 of each is lost), as one in prefill
P_PAIR, P_ONE = ref.HALF_BF16 ** 2, ref.HALF_BF16


# ---- tables
def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("batch,lens,new", [(1, (0, 1), (1, 2)), (3, (0, 300), (0, 400)), (70, (100, 140), (0, 3)), (300, (0, 600), (0, 40)),
                                            (1500, (0, 200), (0, 3)), (9, (0, 1), (700, 2000))])
@pytest.mark.parametrize("in_place", [False, True])
def test_grow_and_slots(batch, lens, new, in_place):
    rng = np.random.default_rng(batch)
    len0, n_new = rng.integers(*lens, batch), rng.integers(*new, batch)
    full = len0 // 128
    n_pages, total = int(full.sum() + ((len0 + n_new) // 128 - full).sum()) + 5, int(n_new.sum())
    order = rng.permutation(n_pages)
    table = np.full((batch, 40), -1, dtype=np.int64)
    at = 0
    for b in range(batch):
        table[b, :full[b]] = order[at:at + full[b]]
        at += full[b]
    free = np.concatenate([order[at:], np.zeros(at, dtype=np.int64)])
    want = ref.grow(len0.tolist(), n_new.tolist(), free, n_pages - at, table)
    t = ek.PageTable(i32(table), i32(len0), i32(free), i32([n_pages - at]))
    plan = ek.PagePlan.empty(batch, total + 3, DEV)
    slot, pos = (torch.full((total + 3,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    out = (t.seq_len, t.n_free) if in_place else (torch.empty_like(t.seq_len), torch.empty_like(t.n_free))
    for _ in range(1 if in_place else 2):                     # from separate arrays the same step can be taken again
        ek.pages_grow(ek.make_shape(*GQA, 0, "bf16"), t, i32(n_new), plan, out[0], out[1], slot, pos)
        assert plan.status() == 0
        for got, expected in zip((out[0], out[1], t.table, plan.row_start, slot[:total], pos[:total]), want):
            assert np.array_equal(got.cpu().numpy().reshape(-1), np.asarray(expected).reshape(-1))
        assert (slot[total:] == 77).all() and (pos[total:] == 77).all()
    # slots of whole sequences, from any position, in any number of rows
    t.seq_len = out[0]
    len1 = want[0]
    first = rng.integers(0, 3, batch)
    count = np.minimum(np.maximum(len1 - first, 0), 300) + 1      # one past the end where the sequence is short
    starts = np.concatenate([[0], np.cumsum(count)])
    got = torch.full((int(starts[-1]) + 4,), 77, dtype=torch.int32, device=DEV)
    ek.pages_slots(t, i32(starts), i32(first), got)
    expected = []
    for b in range(batch):
        for p in range(first[b], first[b] + count[b]):
            expected.append(-2 ** 31 if p >= len1[b] else want[2][b, p // 128] * 128 + p % 128 if p // 128 < len1[b] // 128 else -1 - (b * 128 + p % 128))
    assert np.array_equal(got.cpu().numpy()[:len(expected)], expected) and (got[len(expected):] == 77).all()


@pytest.mark.parametrize("change,status", [(dict(n_new=[5, -1, 3]), ek.PLAN_BAD_LENGTH), (dict(len0=[5, -3, 3]), ek.PLAN_BAD_LENGTH),
                                           (dict(len0=[5, 4 * 128 + 128, 3]), ek.PLAN_BAD_LENGTH), (dict(n_free=[-1]), ek.PLAN_BAD_LENGTH),
                                           (dict(n_free=[99]), ek.PLAN_BAD_LENGTH), (dict(n_new=[5, 640, 3]), ek.PLAN_TABLE_FULL),
                                           (dict(n_new=[5, 2 ** 31 - 1, 3]), ek.PLAN_TABLE_FULL), (dict(n_free=[1]), ek.PLAN_NO_PAGES),
                                           (dict(max_rows=280), ek.PLAN_TOO_MANY_ROWS)])
def test_a_step_that_does_not_fit_changes_nothing(change, status):
    x = dict(len0=[130, 0, 3], n_new=[0, 280, 3], n_free=[6], max_rows=1000)
    x.update(change)
    t = ek.PageTable(torch.full((3, 4), -1, dtype=torch.int32, device=DEV), i32(x["len0"]), i32(list(range(8))), i32(x["n_free"]))
    t.table[0, 0] = 7
    before = [a.clone() for a in (t.table, t.seq_len, t.free_list, t.n_free)]
    plan = ek.PagePlan.empty(3, x["max_rows"], DEV)
    slot = torch.full((x["max_rows"],), 77, dtype=torch.int32, device=DEV)
    shape = ek.make_shape(*GQA, 0, "bf16")
    ek.pages_grow(shape, t, i32(x["n_new"]), plan, row_slot=slot)
    assert plan.status() == status and (plan.row_start == 0).all() and (slot == 77).all()
    assert all(torch.equal(a, b) for a, b in zip(before, (t.table, t.seq_len, t.free_list, t.n_free)))
    # a layer's calls with such a plan: nothing is stored, attention is over what was there
    c = ek.PageCache.empty(shape, 3, 8, DEV)
    for a in (c.k, c.v, c.k_exp, c.v_exp):
        a.zero_()
    c.k_exp.fill_(127), c.v_exp.fill_(127), c.k_tail.zero_(), c.v_tail.fill_(2.0)
    rows = torch.ones(x["max_rows"], 256, dtype=torch.bfloat16, device=DEV)
    ek.page_append(shape, t, c, plan, rows, rows)
    assert not c.k.any() and (c.v_tail == 2.0).all()
    out = torch.full((x["max_rows"], 8, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(ek.page_workspace_bytes(shape, 3, x["max_rows"]), dtype=torch.uint8, device=DEV)
    ek.page_prefill_attn(shape, t, c, plan, out.clone(), out, None, ws)
    assert (out == 3.0).all()
    ek.page_decode_attn(shape, t, c, plan, out[:3].clone(), out, None, ws)
    if "len0" not in change:                                    # 130 tokens: a page of zeros and two rows of 2
        assert torch.allclose(out[0].float(), torch.full((8, 128), 4.0 / 130, device=DEV), rtol=2.0 ** -8, atol=0)


def test_release_gives_the_pages_back():
    b = Batch(GQA, 5, n_pages=30).grow([300, 128, 0, 1000, 127])
    t = b.table
    table, free = t.table.clone(), t.free_list.clone()
    n = int(t.n_free)
    ek.pages_release(t, i32([1, 0, 1, -1, 0]))
    assert t.seq_len.tolist() == [0, 128, 0, 0, 127] and int(t.n_free) == n + 9
    assert torch.equal(t.free_list[n:n + 9], torch.cat([table[0, :2], table[3, :7]])) and torch.equal(t.free_list[:n], free[:n])
    assert (t.table[0] == -1).all() and (t.table[3] == -1).all() and torch.equal(t.table[1], table[1])
    before = [x.clone() for x in (t.table, t.seq_len, t.free_list, t.n_free)]
    t.n_free.fill_(30)                                          # as if all pages were free already: one more cannot come back
    ek.pages_release(t, i32([0, 1, 0, 0, 0]))
    t.n_free.copy_(before[3])
    assert all(torch.equal(x, y) for x, y in zip(before, (t.table, t.seq_len, t.free_list, t.n_free)))
    b.rows[0], b.rows[3] = ([torch.empty(0, b.hkv, b.d, dtype=torch.bfloat16)] * 2 for _ in range(2))
    b.grow([400, 5, 0, 20, 1])
    q = b.random(5, b.hq, b.d)
    out, lse = b.decode(q)
    for i in (0, 1, 3, 4):
        b.check(out[i:i + 1], lse[i:i + 1], q[i:i + 1], i, [len(b.rows[i][0]) - 1], P_PAIR)


# ---- what is held
def special_rows(n, h, d, gen):
    x = torch.randn(n, h, d, generator=gen) * torch.exp(3 * torch.randn(n, h, 1, generator=gen))
    x = x.to(torch.bfloat16)
    x[128:256] = 0
    x[256:384] *= 2.0 ** -125                                   # down to numbers below the normal ones, and past the least scale
    x[384:512] *= 2.0 ** 100
    x[512:640, 0] = torch.arange(0, 128 * d).reshape(128, d).to(torch.int16).view(torch.bfloat16)      # every pattern from 0
    x[3, 0, 5], x[70, 0, 1], x[71, 0, 2] = float("nan"), 448.0, -449.0
    x[640, 0, 0], x[641, 0, 1] = float("inf"), float("-inf")
    x[770:790, 0, :8] = torch.tensor([448.0, 1.75, 3.5, 450.0, float("nan"), float("inf"), 2.0 ** -9, -0.0])
    return x


@pytest.mark.parametrize("layer", [MHA, GQA, NARROW, (5, 1, 64)])
@pytest.mark.parametrize("out_dtype", ["bf16", "f32"])
def test_rows_are_held_and_read_back_exactly(layer, out_dtype):
    b = Batch(layer, 4, out_dtype=out_dtype)
    lens = [900, 0, 128, 77]
    rows = [special_rows(sum(lens), b.hkv, b.d, b.gen) for _ in range(2)]
    b.grow(lens, rows)
    assert b.plan.status() == ek.PLAN_NOT_FINITE
    t = torch.float32 if out_dtype == "f32" else torch.bfloat16
    for order in (torch.arange(sum(lens)), torch.randperm(sum(lens), generator=b.gen), torch.arange(sum(lens)).flip(0), torch.arange(5, 480),
                  torch.tensor([3] * 40 + [899])):
        slot = torch.cat([b.slot[order.to(DEV)], i32([-2 ** 31, 200 * 128, -1 - 4 * 128])])
        out = [torch.full((len(slot), b.hkv * b.d), 3.0, dtype=t, device=DEV) for _ in range(2)]
        ek.page_read(b.shape, b.table, b.cache, slot, *out)
        for s in range(2):
            want = torch.cat([b.held(i)[s] for i in range(4)])[order].flatten(1)
            assert torch.equal(out[s][:-3].double().cpu(), want)
            assert (out[s][-3:] == 3.0).all()                   # slots that do not exist


@pytest.mark.parametrize("layer", [GQA, NARROW])
def test_what_is_held_does_not_depend_on_the_pieces(layer):
    whole, pieces = (Batch(layer, 3, seed=5) for _ in range(2))
    lens = [517, 128, 300]
    rows = [[torch.randn(n, whole.hkv, whole.d, generator=whole.gen).to(torch.bfloat16) for n in lens] for _ in range(2)]
    whole.grow(lens, [torch.cat(x) for x in rows])
    at = [0, 0, 0]
    for step in ([1, 127, 100], [126, 0, 30], [0, 1, 170], [3, 0, 0], [300, 0, 0], [87, 0, 0]):
        pieces.grow(step, [torch.cat([rows[s][b][at[b]:at[b] + n] for b, n in enumerate(step)] + [torch.full((9, whole.hkv, whole.d), float("nan"))])
                           .to(torch.bfloat16) for s in range(2)], slack=9)
        at = [x + n for x, n in zip(at, step)]
        assert pieces.plan.status() == 0
    assert at == lens and torch.equal(pieces.table.seq_len, whole.table.seq_len)
    for b, n in enumerate(lens):
        i, j = (x.table.table[b, :n // 128].long() for x in (whole, pieces))
        for name in ("k", "v", "k_exp", "v_exp"):
            assert torch.equal(getattr(whole.cache, name)[i], getattr(pieces.cache, name)[j]), name
        for name in ("k_tail", "v_tail"):
            assert torch.equal(getattr(whole.cache, name)[b, :n % 128], getattr(pieces.cache, name)[b, :n % 128])


# ---- attention
LENGTHS = [0, 1, 2, 63, 64, 65, 127, 128, 129, 191, 192, 256, 300, 1100]


@pytest.mark.parametrize("layer", [MHA, GQA, NARROW, (5, 1, 64), (40, 2, 128), (7, 7, 64)])
@pytest.mark.parametrize("mode", ["plain", "cap", "slopes", "both"])
def test_decode(layer, mode):
    b = Batch(layer, len(LENGTHS), out_dtype="f32" if mode in ("plain", "both") else "bf16", scale=0.25 if mode == "slopes" else 0.0).grow(LENGTHS)
    cap = 5.0 if mode in ("cap", "both") else 0.0
    slopes = SLOPES(b.hq) if mode in ("slopes", "both") else None
    q = b.random(len(LENGTHS), b.hq, b.d, scale=2.0)
    out, lse = b.decode(q, softcap=cap, slopes=None if slopes is None else slopes.to(DEV))
    assert (out[0] == 0).all() and (lse[0] == -float("inf")).all()
    for i in range(1, len(LENGTHS)):
        b.check(out[i:i + 1], lse[i:i + 1], q[i:i + 1], i, [LENGTHS[i] - 1], P_PAIR, cap, slopes)


@pytest.mark.parametrize("lens", [[1], [40 * 128 + 127], [3000, 10, 2999], [700] * 200], ids=["one", "full", "three", "many"])
def test_decode_splits(lens):
    b = Batch(GQA, len(lens), n_pages=1100).grow(lens)
    q = b.random(len(lens), b.hq, b.d)
    out, lse = b.decode(q)
    for i in sorted({0, len(lens) // 2, len(lens) - 1}):
        b.check(out[i:i + 1], lse[i:i + 1], q[i:i + 1], i, [lens[i] - 1], P_PAIR)
    again, _ = b.decode(q)
    assert torch.equal(again, out)


@pytest.mark.parametrize("cap", [1e-3, 1.0, 1e6])
def test_caps_far_below_and_above_the_scores(cap):
    b = Batch(GQA, 2).grow([200, 90])
    q = b.random(2, b.hq, b.d)
    out, lse = b.decode(q, softcap=cap)
    for i, n in enumerate((200, 90)):
        b.check(out[i:i + 1], lse[i:i + 1], q[i:i + 1], i, [n - 1], P_PAIR, cap if cap < 10 else 0.0)       # 1e6: (s / cap)^2 / 3 is nothing


@pytest.mark.parametrize("cap", [60.0, 12.0, 3.0])
def test_prefill_and_decode_with_scores_below_a_third_of_the_cap_three_quarters_and_beyond(cap):
    """One form of the cap for each; largest score of a wave's 64 x 48 about 16."""
    b = Batch(GQA, 2).grow([700, 130])
    q = b.random(830, b.hq, b.d, scale=3.0)
    out, lse = b.prefill(q, softcap=cap)
    at = 0
    for i, n in enumerate((700, 130)):
        b.check(out[at:at + n], lse[at:at + n], q[at:at + n], i, list(range(n)), P_ONE, cap)
        at += n
    out, lse = b.decode(q[:2], softcap=cap)
    for i, n in enumerate((700, 130)):
        b.check(out[i:i + 1], lse[i:i + 1], q[i:i + 1], i, [n - 1], P_PAIR, cap)


def test_long_chunks_and_many_blocks():
    """Blocks of 384 columns, whole and with keys split, beside a sequence of few columns: some rows of each."""
    for layer, ctx, new, n_pages in (((16, 8, 64), (0, 100, 0), (6200, 3, 77), 60), ((8, 1, 64), (0, 41000, 500), (0, 260, 20), 400)):
        b = Batch(layer, 3, max_pages=330, n_pages=n_pages)
        if any(ctx):
            b.grow(ctx)
        b.grow(new)
        q = b.random(sum(new), b.hq, b.d)
        out, lse = b.prefill(q)
        at = 0
        for i, (c, n) in enumerate(zip(ctx, new)):
            for r in sorted({0, 1, n // 3, n // 2, n - 130, n - 1}):
                if 0 <= r < n:
                    b.check(out[at + r:at + r + 1], lse[at + r:at + r + 1], q[at + r:at + r + 1], i, [c + r], P_ONE)
            at += n


def test_a_query_of_nan_stays_alone():
    b = Batch(GQA, 1).grow([500])
    q = b.random(500, b.hq, b.d)
    clean, clean_lse = b.prefill(q)
    q[77, 3] = float("nan")
    out, lse = b.prefill(q)
    assert torch.isnan(out[77, 3]).all() and torch.isnan(lse[77, 3])
    out[77, 3], lse[77, 3] = clean[77, 3], clean_lse[77, 3]
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


def test_a_plan_of_another_step_does_nothing():
    """Shapes of other head counts, another max_rows, a buffer that no step has written."""
    b = Batch(GQA, 2).grow([300, 40])
    q = b.random(340, b.hq, b.d).to(DEV)
    k = torch.ones(340, 256, dtype=torch.bfloat16, device=DEV)
    before = b.cache.k_tail.clone()
    wide = ek.make_shape(16, 2, 128, 0, "bf16")
    other = ek.PagePlan(b.plan.buf, 2, 339)
    blank = ek.PagePlan(torch.zeros_like(b.plan.buf), 2, 340)
    for shape, plan in ((wide, b.plan), (b.shape, other), (b.shape, blank)):
        out = torch.full((340, shape.n_q_heads, 128), 3.0, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(ek.page_workspace_bytes(shape, 2, plan.max_rows), dtype=torch.uint8, device=DEV)
        qq = q.repeat_interleave(shape.n_q_heads // 8, 1)
        ek.page_decode_attn(shape, b.table, b.cache, plan, qq, out, None, ws)
        ek.page_prefill_attn(shape, b.table, b.cache, plan, qq, out, None, ws)
        ek.page_append(shape, b.table, b.cache, plan, k, k)
        assert (out == 3.0).all() and torch.equal(torch.nan_to_num(b.cache.k_tail.float()), torch.nan_to_num(before.float()))


def test_two_calls_at_once_share_a_plan():
    b = Batch(GQA, 3).grow([3000, 700, 129])
    q = [b.random(3, b.hq, b.d).to(DEV) for _ in range(2)]
    want = [b.decode(x) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs, ws = [b.out(3) for _ in range(2)], [b.workspace() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, st in enumerate(streams):
            ek.page_decode_attn(b.shape, b.table, b.cache, b.plan, q[i], *outs[i], ws[i], stream=st)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i][0].cpu(), want[i][0]) and torch.equal(outs[i][1].cpu(), want[i][1])


PREFILL = {"one": ([0], [1]), "short": ([0, 5], [17, 3]), "page": ([0, 128, 100], [128, 128, 28]), "odd": ([0, 200, 0, 131], [301, 77, 0, 1]),
           "behind": ([2500, 10, 0], [3, 40, 129]), "blocks": ([0, 70], [900, 390])}


@pytest.mark.parametrize("layer", [MHA, GQA, NARROW, (5, 1, 64), (40, 2, 128)])
@pytest.mark.parametrize("case", PREFILL)
def test_prefill(layer, case):
    ctx, new = PREFILL[case]
    mode = list(PREFILL).index(case) % 3
    b = Batch(layer, len(ctx), out_dtype="f32" if mode == 1 else "bf16")
    if any(ctx):
        b.grow(ctx)
    b.grow(new, slack=3)
    cap, slopes = (4.0 if mode == 2 else 0.0), SLOPES(b.hq) if mode == 1 else None
    q = b.random(sum(new) + 3, b.hq, b.d, scale=2.0)
    out, lse = b.prefill(q, softcap=cap, slopes=None if slopes is None else slopes.to(DEV))
    at = 0
    for i, (c, n) in enumerate(zip(ctx, new)):
        if n:
            b.check(out[at:at + n], lse[at:at + n], q[at:at + n], i, list(range(c, c + n)), P_ONE, cap, slopes)
        at += n
    assert (out[at:] == 3.0).all() and (lse[at:] == 3.0).all()


@pytest.mark.parametrize("layer", [GQA, NARROW])
@pytest.mark.parametrize("prefix", [[0, 0, 0], [1, 64, 10 ** 9], [100, 129, 130], [-5, 300, 250]])
def test_prefill_with_a_prefix(layer, prefix):
    b = Batch(layer, 3).grow([0, 20, 200]).grow([260, 300, 5])
    q = b.random(565, b.hq, b.d)
    out, lse = b.prefill(q, prefix_len=i32(prefix))
    at = 0
    for i, (c, n) in enumerate(((0, 260), (20, 300), (200, 5))):
        b.check(out[at:at + n], lse[at:at + n], q[at:at + n], i, list(range(c, c + n)), P_ONE, prefix=max(0, min(prefix[i], c + n)))
        at += n


def test_scores_that_grow_and_fall_by_thousands():
    """References of the softmax far apart from block to block, in both directions."""
    b = Batch(GQA, 2)
    lens = [600, 600]
    k = torch.randn(1200, b.hkv, b.d, generator=b.gen)
    k *= torch.cat([torch.arange(600) / 12.0, 50 - torch.arange(600) / 12.0])[:, None, None]
    b.grow(lens, [k.to(torch.bfloat16), b.random(1200, b.hkv, b.d)])
    q = b.random(1200, b.hq, b.d, scale=8.0)
    out, lse = b.prefill(q)
    for i in range(2):
        b.check(out[600 * i:600 * i + 600], lse[600 * i:600 * i + 600], q[600 * i:600 * i + 600], i, list(range(600)), P_ONE)
    out, lse = b.decode(q[:2])
    for i in range(2):
        b.check(out[i:i + 1], lse[i:i + 1], q[i:i + 1], i, [599], P_PAIR)


def test_tokens_that_are_not_seen_may_hold_anything():
    """Later tokens of the chunk with NaN and infinities (held as zeros and the largest numbers), tail rows behind the last one, free pages."""
    b = Batch(GQA, 2)
    for x in (b.cache.k, b.cache.v, b.cache.k_exp, b.cache.v_exp):
        x.fill_(0xff)
    b.cache.k_tail.fill_(float("nan")), b.cache.v_tail.fill_(float("nan"))
    rows = [b.random(330, b.hkv, b.d) for _ in range(2)]
    for x in rows:
        x[150:200] = float("nan")
        x[290:300] = float("inf")
    b.grow([300, 30], rows)
    q = b.random(330, b.hq, b.d)
    out, lse = b.prefill(q)
    # the block of tokens 128 .. 255 keeps its scale, NaN are zeros there; queries in front of the infinities do not meet them
    b.check(out[:290], lse[:290], q[:290], 0, list(range(290)), P_ONE)
    b.check(out[300:], lse[300:], q[300:], 1, list(range(30)), P_ONE)


def test_table_entries_outside_the_pool_are_skipped():
    b = Batch(GQA, 2).grow([400, 150])
    b.table.table[0, 1], b.table.table[1, 0] = 200, -1
    keep = [torch.cat([torch.arange(0, 128), torch.arange(256, 400)]), torch.arange(128, 150)]
    q = b.random(550, b.hq, b.d)
    out, lse = b.decode(q[:2])
    pre, pre_lse = b.prefill(q)
    for i, n in enumerate((400, 150)):
        k, v = (x[keep[i]] for x in b.held(i))
        for o, s, qq, half in ((out[i:i + 1], lse[i:i + 1], q[i:i + 1], P_PAIR), (pre[(399, 549)[i]][None], pre_lse[(399, 549)[i]][None], q[(399, 549)[i]][None], P_ONE)):
            want = ref.attend(qq, k, v, [len(k) - 1], b.scale)
            tol, tol_lse = ref.tolerances(*want, n, b.d, ref.HALF_BF16, half)
            assert ((o.double() - want[0]).abs() <= tol).all() and ((s.double() - want[1]).abs() <= tol_lse).all()
    assert (pre[400:528] == 0).all() and (pre_lse[400:528] == -float("inf")).all()        # rows that see nothing


def test_pages_past_4_gb():
    b = Batch((8, 8, 128), 1, max_pages=8, n_pages=40000)
    b.table.free_list[:6] = i32([39999, 1, 33000, 16500, 32767, 32768])
    b.table.n_free.fill_(6)
    b.grow([6 * 128 + 5])
    q = b.random(773, b.hq, b.d)
    out, lse = b.decode(q[:1])
    b.check(out, lse, q[:1], 0, [772], P_PAIR)
    out, lse = b.prefill(q)
    b.check(out, lse, q, 0, list(range(773)), P_ONE)
    got = [torch.empty(773, 1024, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ek.page_read(b.shape, b.table, b.cache, b.slot, *got)
    assert all(torch.equal(g.double().cpu(), h.flatten(1)) for g, h in zip(got, b.held(0)))


@pytest.mark.parametrize("in_place", [False, True])
def test_prefill_of_many_sequences_of_all_lengths(in_place):
    """More sequences than the step's workgroup has threads; few and many columns, with and without split keys; outputs equal whether the lengths
    are written in place or elsewhere."""
    rng = np.random.default_rng(4)
    batch = 1300
    new = np.where(rng.random(batch) < 0.9, rng.integers(0, 3, batch), rng.integers(50, 140, batch)).tolist()
    b = Batch((8, 2, 64), batch, max_pages=12, n_pages=2600)
    b.grow(rng.integers(0, 300, batch).tolist())
    before = b.table.seq_len.clone()
    b.grow(new)
    if not in_place:
        n_new, len1, n_free = i32(new), b.table.seq_len.clone(), b.table.n_free.clone()
        taken = sum(int(x) for x in (len1 // 128 - before // 128).tolist())
        b.table.seq_len = before
        b.table.n_free = n_free + taken                        # the same step from the same state: the same pages again
        table = b.table.table.clone()
        ek.pages_grow(b.shape, b.table, n_new, b.plan, torch.empty_like(before), torch.empty_like(n_free))
        assert torch.equal(table, b.table.table)
    q = b.random(sum(new), b.hq, b.d)
    out, lse = b.prefill(q)
    at = 0
    for i, n in enumerate(new):
        if n and (n > 3 or i % 100 == 0):
            total = len(b.rows[i][0])
            b.check(out[at:at + n], lse[at:at + n], q[at:at + n], i, list(range(total - n, total)), P_ONE)
        at += n


# ---- together
def test_a_captured_step_follows_its_sequences():
    """grow, append and decode in one graph, replayed over the end of a block, with eager work in between; a twin takes the steps eagerly."""
    captured, eager = (Batch(GQA, 3, seed=9).grow([120, 0, 255]) for _ in range(2))
    new = [torch.empty(3, 256, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    q = torch.empty(3, 8, 128, dtype=torch.bfloat16, device=DEV)
    one = i32([1, 1, 1])
    side = torch.cuda.Stream()

    def step(b, out, lse, plan, ws):
        ek.pages_grow(b.shape, b.table, one, plan)
        ek.page_append(b.shape, b.table, b.cache, plan, *new)
        ek.page_decode_attn(b.shape, b.table, b.cache, plan, q, out, lse, ws)

    state = {}
    for b in (captured, eager):
        plan = ek.PagePlan.empty(3, 3, DEV)
        state[b] = (*b.out(3), plan, torch.full((ek.page_workspace_bytes(b.shape, 3, 3),), 0xff, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured, *state[captured])
    for i in range(12):
        for x in (*new, q):
            x.copy_(captured.random(*x.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(eager, *state[eager])
        torch.cuda.synchronize()
        assert torch.equal(captured.table.seq_len, eager.table.seq_len) and int(captured.table.seq_len[0]) == 121 + i
        assert torch.equal(captured.table.table, eager.table.table)
        assert all(torch.equal(x, y) for x, y in zip(state[captured][:2], state[eager][:2])), i
        assert torch.isfinite(state[captured][0]).all()


def test_a_prompt_in_chunks_then_tokens_and_back_to_a_layer_cache():
    """The set as a server uses it, on a stream of its own: chunks, decode steps, a sequence ended and its pages taken over; then the rows are
    read into a LayerCache, over which the framework's decode gives the same as decode over the pages."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = Batch(GQA, 3, n_pages=14)
        for new in ([150, 500, 0], [0, 300, 40], [130, 0, 88]):
            b.grow(new)
            q = b.random(sum(new), b.hq, b.d)
            out, lse = b.prefill(q)
            at = 0
            for i, n in enumerate(new):
                if n:
                    total = len(b.rows[i][0])
                    b.check(out[at:at + n], lse[at:at + n], q[at:at + n], i, list(range(total - n, total)), P_ONE)
                at += n
        ek.pages_release(b.table, i32([0, 1, 0]))
        b.rows[1] = [torch.empty(0, b.hkv, b.d, dtype=torch.bfloat16)] * 2
        for _ in range(3):
            b.grow([1, 1, 1])
            q = b.random(3, b.hq, b.d)
            out, lse = b.decode(q)
            for i in range(3):
                b.check(out[i:i + 1], lse[i:i + 1], q[i:i + 1], i, [len(b.rows[i][0]) - 1], P_PAIR)
        lens = b.table.seq_len.tolist()
        starts = np.concatenate([[0], np.cumsum(lens)])
        slots = torch.empty(int(starts[-1]), dtype=torch.int32, device=DEV)
        ek.pages_slots(b.table, i32(starts), i32([0, 0, 0]), slots)
        rows = [torch.empty(int(starts[-1]), b.hkv * b.d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        ek.page_read(b.shape, b.table, b.cache, slots, *rows)
        layer = ek.LayerCache(*rows, b.hkv * b.d, int(starts[-1]), starts[:-1], lens, lens)
        full = ek.make_shape(b.hq, b.hkv, b.d, b.hkv * b.d, "bf16")
        ws = torch.empty(ek.workspace_bytes(full, 3, int(starts[-1])), dtype=torch.uint8, device=DEV)
        other, other_lse = b.out(3)
        ek.decode_attn(full, layer, layer, None, None, q.to(DEV), other, other_lse, ws)
    side.synchronize()
    assert (other.cpu().float() - out.float()).abs().max() <= 2 * ref.HALF_BF16 * out.float().abs().max()
    assert (other_lse.cpu() - lse).abs().max() <= 1e-4


def test_everything_is_refused_while_another_gpu_is_the_current_one(monkeypatch):
    """Views of tables and caches that were made before, too; nothing is launched."""
    b = Batch(GQA, 2).grow([130, 5])
    q, (out, lse), space = b.random(2, b.hq, b.d).to(DEV), b.out(2), b.workspace()
    which = torch.zeros(2, dtype=torch.int32, device=DEV)
    ek.page_decode_attn(b.shape, b.table, b.cache, b.plan, q, out, lse, space)
    torch.cuda.synchronize()
    monkeypatch.setitem(ek._DTYPES, "device", lambda: 1)
    for call in (lambda: ek.pages_release(b.table, which), lambda: ek.page_decode_attn(b.shape, b.table, b.cache, b.plan, q, out, lse, space),
                 lambda: ek.page_append(b.shape, b.table, b.cache, b.plan, None, None), lambda: b.table.as_c(), lambda: b.plan.as_c(),
                 lambda: b.cache.as_c(b.shape, b.table)):
        with pytest.raises(ValueError, match="current GPU is cuda:1"):
            call()
    monkeypatch.undo()
    with pytest.raises(ValueError, match="workspace"):
        ek.page_decode_attn(b.shape, b.table, b.cache, b.plan, q, out, lse, space.cpu())
    assert int(b.table.seq_len[0]) == 130


def test_shares_of_more_halves_than_32_bits_hold():
    """Sequences may share pages: 4096 of 2^19 halves each, one share for all of them.  The share's size stays within 2^26, more than any sequence has."""
    batch, pages = 4096, 1 << 18
    shape = ek.make_shape(1024, 1024, 64, 0, "bf16")
    table = ek.PageTable(torch.empty(batch, pages, dtype=torch.int32, device=DEV), torch.full((batch,), pages * 128, dtype=torch.int32, device=DEV),
                         torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    plan = ek.PagePlan.empty(batch, 8, DEV)
    n_new = torch.zeros(batch, dtype=torch.int32, device=DEV)
    n_new[0] = n_new[7] = 4                                  # 4 columns each: two blocks of few
    ek.pages_grow(shape, table, n_new, plan)
    words = plan._words()[:16].tolist()
    assert words[0] == 0 and words[2] == 1 << 26             # status, halves of a decode share
    assert words[3] == batch + 2 and words[14] >= 2          # a share for each sequence's pages, tails of two of them; blocks of few columns
    assert int(table.seq_len[0]) == pages * 128 + 4


@pytest.mark.parametrize("layer,ctx,new,plain,capped", [
    ((32, 32, 64), 0, 3600, 256, 256),                      # 320 blocks of 384, 480 of 256, whose longest ends earlier
    ((32, 8, 64), 16384, 600, 384, 256),                    # few blocks, their keys split
    ((32, 8, 64), 7, 600, 128, 128),
    ((16, 16, 128), 100, 1290, 128, 128),
    ((8, 8, 128), 0, 16400, 256, 256),                      # 344 and 520 blocks: the longest of 384 would take 257 x 2.5 us, all of 256 take 574
    ((32, 32, 64), 0, 8192, 384, 256)])                     # 704 and 1024 blocks
def test_blocks_of_every_size_with_and_without_a_cap(layer, ctx, new, plain, capped):
    """Two dozen of a prompt's rows, the first and last ones and those at the blocks' edges among them."""
    pages = (ctx + new) // 128 + 1
    b = Batch(layer, 1, max_pages=pages, n_pages=pages, scale=0.25)
    if ctx:
        b.grow([ctx])
    b.grow([new])
    words = b.plan._words()[:16].tolist()
    assert (words[4], words[8]) == (plain, capped)
    q = b.random(new, b.hq, b.d)
    some = sorted({0, 1, 31, 32, 63, 64, 95, 96, 127, 128, 255, 256, 383, 384, new // 2, new - 130, new - 129, new - 2, new - 1})
    prefix = i32([ctx + 100])
    for kw in (dict(), dict(softcap=8.0), dict(slopes=SLOPES(b.hq).to(DEV), softcap=8.0), dict(prefix_len=prefix), dict(prefix_len=prefix, softcap=8.0)):
        out, lse = b.prefill(q, **kw)
        slopes = kw.get("slopes")
        b.check(out[some], lse[some], q[some], 0, [ctx + i for i in some], P_ONE, kw.get("softcap", 0.0), None if slopes is None else slopes.cpu(),
                prefix=ctx + 100 if "prefix_len" in kw else 0)


@pytest.mark.parametrize("batch", [1, 300, 1024, 1025, 4096])
def test_plans_for_decode_alone(batch):
    """max_rows = 0: nobody grows, lengths and decode's items stand; a token more than none is refused."""
    b = Batch((4, 2, 64), batch, max_pages=2, n_pages=batch).grow([1 + i % 130 for i in range(batch)])
    lens = b.table.seq_len.clone()
    b.plan = ek.PagePlan.empty(batch, 0, DEV)
    none = torch.zeros(batch, dtype=torch.int32, device=DEV)
    ek.pages_grow(b.shape, b.table, none, b.plan)
    assert b.plan.status() == 0 and torch.equal(b.table.seq_len, lens) and not b.plan.row_start.any()
    q = b.random(batch, b.hq, b.d)
    out, lse = b.decode(q)
    for i in (0, batch // 2, batch - 1):
        b.check(out[i:i + 1], lse[i:i + 1], q[i:i + 1], i, [i % 130], P_PAIR)
    none[batch - 1] = 1
    ek.pages_grow(b.shape, b.table, none, b.plan)
    assert b.plan.status() == ek.PLAN_TOO_MANY_ROWS and torch.equal(b.table.seq_len, lens)
