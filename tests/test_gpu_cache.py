"""The calls around the key / value cache on the GPU, against plain 64-bit forms, and a run of them together."""
import math
import random

import pytest
import torch

from paper_2603_14549_b200 import binding as A
from paper_2603_14549_b200 import workloads as W
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HEAD = 128


@pytest.fixture(scope="module")
def ctx():
    c = A.asap_init(0, max_total_tokens=8192, max_B=8, max_H=4, max_D=512)
    yield c
    A.asap_free(c)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


# ------------------------------------------------------------------------------------------------ rotation
def _freq(plan):
    return torch.tensor([plan.turns[i] * 2 * math.pi / 2.0 ** 64 for i in range(plan.n_pairs)], dtype=torch.float64, device=DEV)


def _close_rotation(got, ref, x, dtype, mag):
    # cosine and sine to 2^-22, the products and their sum in fp32, one rounding to the element type
    size = x.double().abs().amax(-1, keepdim=True) * 2 * mag
    tol = torch.finfo(dtype).eps / 2 * ref.abs() + 2.0 ** -20 * size + torch.finfo(dtype).tiny * torch.finfo(dtype).eps
    assert ((got.double() - ref).abs() <= tol).all(), ((got.double() - ref).abs() / tol).max().item()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("n,dim,rot,scaling", [(1, 128, 128, "none"), (3, 128, 20, "linear"), (67, 128, 64, "yarn"), (5, 256, 256, "ntk"),
                                               (2500, 64, 32, "bands"), (9, 80, 6, "none"), (4, 8, 8, "none"), (7, 96, 96, "yarn")])
def test_rotation(ctx, dtype, layout, n, dim, rot, scaling):
    plan = A.asap_rope_make(rot, layout=layout, scaling=scaling, factor=4.0, theta=10000.0 if n != 5 else 1e6)
    g = gen(n * 1000 + dim)
    fused = torch.randn(n, 5 + 2 * 3, dim, device=DEV, generator=g).to(dtype)
    q, k, v = fused[:, :5], fused[:, 5:8], fused[:, 8:]
    far = [0, 2 ** 31 - 1, -(2 ** 31), -1, 1, 131071, 1000003]
    pos = i32([far[i] if i < len(far) else random.Random(i).randrange(1 << 20) for i in range(n)])
    rows = n + 11
    where = random.Random(n).sample(range(rows), n)
    if n > 2:
        where[1], where[2] = -1, rows                   # padded rows write nothing
    q_out = torch.full((n, 5, dim), 7.0, dtype=dtype, device=DEV)
    k_cache = torch.full((3, rows, dim), 7.0, dtype=dtype, device=DEV).transpose(0, 1)     # stored head by head
    v_cache = torch.full((rows, 3, dim), 7.0, dtype=dtype, device=DEV)
    n0 = A.asap_launch_count(ctx)
    A.asap_rope(ctx, plan, A.RopeArgs(pos, [A.RopeTensor(q, q_out), A.RopeTensor(k, k_cache, mapped=True),
                                            A.RopeTensor(v, v_cache, mapped=True, rotate=False)], dst_row=i32(where)))
    assert A.asap_launch_count(ctx) == n0 + 1
    f = _freq(plan)
    _close_rotation(q_out, R.rotate(q, pos, rot, layout, f, plan.magnitude), q, dtype, plan.magnitude)
    put = [i for i in range(n) if 0 <= where[i] < rows]
    at = torch.tensor([where[i] for i in put], device=DEV)
    put = torch.tensor(put, device=DEV)
    _close_rotation(k_cache[at], R.rotate(k, pos, rot, layout, f, plan.magnitude)[put], k[put], dtype, plan.magnitude)
    assert torch.equal(v_cache[at], v[put])
    assert torch.equal(q_out[..., rot:], q[..., rot:])
    rest = torch.ones(rows, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert (k_cache[rest] == 7).all() and (v_cache[rest] == 7).all()


@pytest.mark.parametrize("layout,rot", [("half", 128), ("interleaved", 128), ("half", 20), ("interleaved", 6)])
def test_rotation_in_place_and_back(ctx, layout, rot):
    plan = A.asap_rope_make(rot, layout=layout)
    x = torch.randn(33, 4, HEAD, device=DEV, generator=gen(1)).to(torch.float16)
    pos = i32(list(range(1000, 1033)))
    out = torch.empty_like(x)
    A.asap_rope(ctx, plan, A.RopeArgs(pos, [A.RopeTensor(x, out)]))
    y = x.clone()
    A.asap_rope(ctx, plan, A.RopeArgs(pos, [A.RopeTensor(y, y)]))
    assert torch.equal(y, out)
    z = torch.empty_like(y)
    A.asap_rope(ctx, plan, A.RopeArgs(pos, [A.RopeTensor(y, z)], inverse=True))
    _close_rotation(z, R.rotate(y, pos, rot, layout, _freq(plan), inverse=True), y, x.dtype, 1.0)
    # two roundings of values up to the pair's length
    assert ((z.double() - x.double()).abs() <= 2.0 ** -9 * (x.double().abs().amax(-1, keepdim=True) * 1.5)).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_parts_of_a_packed_projection_turn_in_place(ctx, layout):
    """Queries and keys between each other's rows, the values beside them as they were."""
    packed = torch.randn(37, 6 + 2 + 2, HEAD, device=DEV, generator=gen(7)).to(torch.bfloat16)
    before, pos, plan = packed.clone(), i32(list(range(37))), A.asap_rope_make(64, layout=layout)
    q, k = packed[:, :6], packed[:, 6:8]
    A.asap_rope(ctx, plan, A.RopeArgs(pos, [A.RopeTensor(q, q), A.RopeTensor(k, k)]))
    A.asap_check(ctx)
    _close_rotation(packed[:, :8], R.rotate(before[:, :8], pos, 64, layout, _freq(plan)), before[:, :8], packed.dtype, 1.0)
    assert torch.equal(packed[:, 8:], before[:, 8:])


def test_far_positions_keep_their_angles(ctx):
    """Positions up to the last int32, where an angle taken in 32 bits would be off by whole turns."""
    x = torch.randn(6, 2, HEAD, device=DEV, generator=gen(2)).to(torch.bfloat16)
    pos = i32([2 ** 31 - 1, 2 ** 31 - 2, 123456789, 16777217, 16777219, 3])
    plan = A.asap_rope_make(HEAD)
    out = torch.empty_like(x)
    A.asap_rope(ctx, plan, A.RopeArgs(pos, [A.RopeTensor(x, out)]))
    _close_rotation(out, R.rotate(x, pos, HEAD, "half", _freq(plan)), x, x.dtype, 1.0)


def test_the_largest_number_of_rows(ctx):
    """2^31 - 1 rows of one source row, whose count cannot be rounded up to whole blocks in 32 bits."""
    n, plan = 2 ** 31 - 1, A.asap_rope_make(8)
    x = torch.randn(1, 1, 8, device=DEV, generator=gen(5)).to(torch.bfloat16).expand(n, 1, 8)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    out = torch.zeros(n, 1, 8, dtype=torch.bfloat16, device=DEV)
    A.asap_rope(ctx, plan, A.RopeArgs(pos, [A.RopeTensor(x, out)]))
    A.asap_check(ctx)
    at = torch.cat([torch.arange(5000, device=DEV), torch.randint(0, n, (20000,), device=DEV, generator=gen(6)), torch.arange(n - 5000, n, device=DEV)])
    _close_rotation(out[at], R.rotate(x[at], pos[at], 8, "half", _freq(plan)), x[at], torch.bfloat16, 1.0)
    del pos, out
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------ attention
class Case:
    """Random sequences in a cache whose unused rows hold NaN."""

    def __init__(self, lens, nq, H, kv, dtype, layout="rows", groups=None, seed=0, weights=True, slack=0):
        rng = random.Random(seed)
        self.len, self.nq, B = list(lens), list(nq), len(lens)
        g = gen(seed)
        row = rng.randrange(3)
        self.groups = []
        for b0, b1, pl in groups or []:
            self.groups.append((b0, b1, row, pl))
            row += pl + rng.randrange(3)
        order = list(range(B))
        rng.shuffle(order)
        self.start = [0] * B
        for b in order:
            self.start[b] = row
            row += lens[b] + rng.randrange(3)
        rows = max(row, 1) + slack
        shape = {"rows": (rows, kv, HEAD), "pairs": (rows, 2, kv, HEAD), "heads": (kv, rows, HEAD)}[layout]
        nan = lambda: torch.full(shape, float("nan"), dtype=dtype, device=DEV)           # noqa: E731
        if layout == "pairs":
            both = nan()
            self.k, self.v = both[:, 0], both[:, 1]
        else:
            self.k, self.v = (nan().transpose(0, 1), nan().transpose(0, 1)) if layout == "heads" else (nan(), nan())
        for s, n in [(s, n) for s, n in zip(self.start, self.len)] + [(s, n) for _, _, s, n in self.groups]:
            for t in (self.k, self.v):
                t[s:s + n] = torch.randn(n, kv, HEAD, device=DEV, generator=g).to(dtype)
        n_q = sum(nq)
        fused = torch.randn(n_q, H + 1, HEAD, device=DEV, generator=g).to(dtype)
        self.q = fused[:, :H]                                     # a view of a wider projection
        self.out = torch.full((n_q, H, HEAD), 7.0, dtype=dtype, device=DEV)
        self.lse = torch.full((n_q, H), 7.0, device=DEV)
        self.weights = torch.rand(rows, device=DEV, generator=g) if weights else None
        self.q_cu = [0]
        for n in nq:
            self.q_cu.append(self.q_cu[-1] + n)
        cu = None
        if self.groups:
            cu = i32([self.groups[0][0]] + [b1 for _, b1, _, _ in self.groups])
        self.dev = dict(start=i32(self.start), len=i32(self.len), q_cu=i32(self.q_cu), group_cu=cu,
                        prefix_start=i32([p for _, _, p, _ in self.groups]) if self.groups else None,
                        prefix_len=i32([p for _, _, _, p in self.groups]) if self.groups else None)
        self.bounds = dict(max_len=max(lens), max_q=max(max(nq), 1), max_prefix=max([p for _, _, _, p in self.groups], default=0))

    def args(self, **kw):
        d = dict(self.dev, **self.bounds, lse=self.lse, weights=self.weights)
        d.update(kw)
        return A.CacheAttention(self.q, self.k, self.v, self.out, **d)

    def run(self, ctx, stream=None, **kw):
        args = self.args(**kw)
        scratch = torch.full((A.asap_cache_attention_scratch_bytes(ctx, args),), 0x7f, dtype=torch.uint8, device=DEV)
        A.asap_cache_attention(ctx, args, scratch, stream)
        return args, scratch

    def ref(self, **kw):
        return R.attention(self.q, self.k, self.v, self.start, self.len, self.q_cu, self.groups, **kw)

    def check(self, ctx, **kw):
        before = None if self.weights is None else self.weights.clone()
        self.run(ctx)
        A.asap_check(ctx)
        ref = self.ref(**kw)
        n_keys = max(self.len) + self.bounds["max_prefix"]
        R.check_attention(self.out, self.lse, ref, self.q.dtype, n_keys)
        if before is not None:
            R.check_weights(self.weights, before, ref, sum(self.nq))
        return ref


CASES = {
    "one_row": dict(lens=[1], nq=[1], H=1, kv=1),
    "tile_edges": dict(lens=[63, 64, 65, 127, 128, 129, 15, 16, 17], nq=[1] * 9, H=4, kv=4),
    "empty_and_short": dict(lens=[0, 1, 2, 0, 300], nq=[1] * 5, H=6, kv=2),
    "no_query_rows": dict(lens=[50, 70, 90], nq=[1, 0, 2], H=4, kv=2),
    "odd_ratio": dict(lens=[333, 20], nq=[1, 1], H=14, kv=2),
    "one_kv_head": dict(lens=[700, 5], nq=[1, 1], H=16, kv=1),
    "wide_ratio": dict(lens=[200], nq=[3], H=40, kv=1),
    "several_rows": dict(lens=[300, 77, 40], nq=[5, 9, 40], H=4, kv=2),
    "rows_before_their_keys": dict(lens=[3, 0, 10], nq=[7, 4, 10], H=2, kv=2),
    "whole_prompt": dict(lens=[400, 130], nq=[400, 130], H=2, kv=1),
    "many_splits": dict(lens=[20000], nq=[1], H=8, kv=2),
    "groups": dict(lens=[10, 0, 33, 64, 1], nq=[1] * 5, H=4, kv=4, groups=[(0, 3, 100), (3, 5, 257)]),
    "group_gaps": dict(lens=[10, 20, 33, 64, 1], nq=[1, 2, 0, 3, 1], H=4, kv=2, groups=[(1, 2, 0), (2, 4, 65)]),
    "group_of_many": dict(lens=[7] * 40, nq=[1] * 40, H=8, kv=2, groups=[(0, 40, 1000)]),
    "group_rows": dict(lens=[70, 100, 33], nq=[70, 64, 33], H=4, kv=4, groups=[(0, 3, 500)]),
    "group_rows_gqa": dict(lens=[40, 90], nq=[33, 90], H=6, kv=2, groups=[(0, 2, 300)]),
    "prefix_only": dict(lens=[0, 0, 0], nq=[1, 3, 1], H=4, kv=1, groups=[(0, 3, 129)]),
    "many_items": dict(lens=[150, 40, 70, 200, 33, 256], nq=[150, 33, 70, 181, 33, 130], H=24, kv=24, groups=[(0, 2, 300), (2, 6, 1000)]),
    "many_items_gqa": dict(lens=[100] * 30, nq=[17] * 30, H=32, kv=8, groups=[(0, 30, 700)]),
    "tiles_of_an_odd_ratio": dict(lens=[60, 200], nq=[5, 9], H=14, kv=2, groups=[(0, 2, 400)]),
    "sixteen_rows": dict(lens=[30] * 16, nq=[1] * 16, H=4, kv=4, groups=[(0, 16, 3000)]),
    "nine_rows_each": dict(lens=[700, 45, 9], nq=[9, 9, 9], H=4, kv=4),
    "two_heads_together": dict(lens=[500, 17, 4500], nq=[2, 3, 1], H=12, kv=4),
    "four_heads_together": dict(lens=[500, 33, 15, 16, 17, 5000], nq=[1] * 6, H=16, kv=8),
    "sixty_four_pairs": dict(lens=[300, 1, 64, 1025], nq=[2, 1, 2, 2], H=32, kv=8),
    "late_rows": dict(lens=[2, 1], nq=[9, 5], H=2, kv=2, groups=[(0, 2, 70)]),
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("name", CASES)
def test_attention(ctx, name, dtype):
    layout = ["rows", "pairs", "heads"][len(name) % 3]
    Case(**CASES[name], dtype=dtype, layout=layout, seed=len(name) * 7 + sum(map(ord, name))).check(ctx)


@pytest.mark.parametrize("layout", ["rows", "pairs", "heads"])
def test_every_layout_gives_the_same_bits(ctx, layout):
    c = Case(**CASES["groups"], dtype=torch.bfloat16, seed=3)
    c.run(ctx)
    d = Case(**CASES["groups"], dtype=torch.bfloat16, seed=3, layout=layout)
    d.k.copy_(c.k); d.v.copy_(c.v); d.q.copy_(c.q)
    d.run(ctx)
    assert torch.equal(c.out, d.out) and torch.equal(c.lse, d.lse) and torch.equal(c.weights, d.weights)


def test_without_query_offsets_weights_and_lse(ctx):
    c = Case(lens=[100, 31, 7], nq=[1, 1, 1], H=4, kv=2, dtype=torch.bfloat16, seed=4)
    c.run(ctx)
    first = c.out.clone()
    c.out.fill_(7)
    args = A.CacheAttention(c.q, c.k, c.v, c.out, c.dev["start"], c.dev["len"], max_len=100)
    scratch = torch.empty(A.asap_cache_attention_scratch_bytes(ctx, args), dtype=torch.uint8, device=DEV)
    A.asap_cache_attention(ctx, args, scratch)
    assert torch.equal(first, c.out)


@pytest.mark.parametrize("nq", [1, 20], ids=["streamed", "tiles"])
def test_weights_where_every_prefix_is_empty(ctx, nq):
    """Groups whose prefixes have no rows (yet): the bound of the prefixes is zero, and the own rows get their weights all the same."""
    c = Case(lens=[900, 300, 31, 700], nq=[nq] * 4, H=8, kv=2, dtype=torch.bfloat16, seed=40, groups=[(0, 1, 0), (1, 3, 0), (3, 4, 0)])
    assert c.bounds["max_prefix"] == 0
    c.check(ctx)


@pytest.mark.parametrize("nq", [1, 20], ids=["streamed", "tiles"])
def test_weights_where_no_sequence_has_rows_of_its_own(ctx, nq):
    c = Case(lens=[0, 0, 0], nq=[nq] * 3, H=8, kv=2, dtype=torch.bfloat16, seed=41, groups=[(0, 1, 500), (1, 3, 77)])
    assert c.bounds["max_len"] == 0
    c.check(ctx)


def test_scale_and_loose_bounds(ctx):
    c = Case(lens=[100, 31], nq=[1, 2], H=4, kv=2, dtype=torch.bfloat16, seed=5, slack=5000)
    before = c.weights.clone()
    c.run(ctx, scale=0.3, max_len=5000, max_q=3)
    A.asap_check(ctx)
    ref = c.ref(scale=0.3)
    R.check_attention(c.out, c.lse, ref, torch.bfloat16, 100)
    R.check_weights(c.weights, before, ref, 3)


def test_out_may_be_a_strided_view(ctx):
    c = Case(lens=[100, 31], nq=[1, 2], H=4, kv=2, dtype=torch.float16, seed=6)
    c.run(ctx)
    wide = torch.full((3, 7, HEAD), 7.0, dtype=torch.float16, device=DEV)
    first = c.out
    c.out = wide[:, 2:6]
    c.run(ctx)
    assert torch.equal(first, c.out) and (wide[:, :2] == 7).all() and (wide[:, 6:] == 7).all()


@pytest.mark.parametrize("nq", [[1, 2], [40, 90]], ids=["streamed", "tiles"])
@pytest.mark.parametrize("what", ["rows", "heads"])
def test_queries_may_be_a_broadcast_view(ctx, nq, what):
    c = Case(lens=[100, 131], nq=nq, H=4, kv=2, dtype=torch.bfloat16, seed=8)
    one = torch.randn(1 if what == "rows" else sum(nq), 4 if what == "rows" else 1, HEAD, device=DEV, generator=gen(8)).to(torch.bfloat16)
    c.q = one.expand(sum(nq), 4, HEAD)
    c.check(ctx)


@pytest.mark.parametrize("weights", [False, True], ids=["", "weights"])
def test_many_partial_results_of_many_rows(ctx, weights):
    """Enough rows for two warps a head in the join, and long sequences cut into more pieces than those take at a time."""
    c = Case(lens=[30000] + [20] * 49, nq=[1] * 50, H=24, kv=4, dtype=torch.float16, seed=16, weights=weights, groups=[(1, 3, 9000)])
    c.check(ctx)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")], ids=["nan", "inf", "-inf"])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("name,H,kv,nq", [("few", 2, 2, 5), ("many", 4, 2, 70)])
def test_a_query_row_does_not_see_later_rows(ctx, value, which, name, H, kv, nq):
    """Key or value rows that only later query rows admit hold infinities or NaN: the rows before them keep every bit, and the rows
    that admit them get what the formula gives."""
    c = Case(lens=[150], nq=[nq], H=H, kv=kv, dtype=torch.bfloat16, seed=8, weights=False)
    c.run(ctx)
    good = c.out.clone()
    t = nq - 3
    row = c.start[0] + c.len[0] - 3
    getattr(c, which)[row, :, 5] = value
    c.run(ctx)
    assert torch.equal(c.out[:t], good[:t])
    if which == "v":
        ref = c.ref()
        assert torch.equal(torch.isnan(c.out), torch.isnan(ref[0])) and torch.equal(torch.isinf(c.out), torch.isinf(ref[0]))
        fine = torch.isfinite(ref[0])
        assert ((c.out.double() - ref[0]).abs()[fine] <= (2.0 ** -8 * ref[0].abs() + 2.0 ** -7 * ref[3])[fine]).all()
    elif value != value:
        assert torch.isnan(c.out[t:]).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=["nan", "inf"])
def test_values_of_late_rows_where_items_follow_each_other(ctx, value):
    """Items of two row tiles between items of one, several to a block, most with an infinity or NaN in a value row that only their last query
    rows admit: each item's mark reaches its own rows, and only those."""
    nq = [[200, 30, 40, 60, 20, 35][i % 6] for i in range(280)]
    c = Case(lens=[n + i % 5 for i, n in enumerate(nq)], nq=nq, H=4, kv=4, dtype=torch.bfloat16, seed=51, weights=False)
    hit = [i for i in range(280) if i % 6 != 3]
    row = torch.tensor([c.start[b] + c.len[b] - 3 for b in hit], device=DEV)
    admits = torch.zeros(sum(nq), dtype=torch.bool, device=DEV)
    for b in hit:
        admits[c.q_cu[b + 1] - 3:c.q_cu[b + 1]] = True
    c.v[row, :, 5] = 0.0
    c.run(ctx)
    good = c.out.clone()
    assert torch.isfinite(good).all()
    c.v[row, :, 5] = value
    want = good.clone()
    want[admits, :, 5] = value
    for _ in range(5):
        c.out.fill_(7)
        c.run(ctx)
        A.asap_check(ctx)
        assert torch.equal(c.out.nan_to_num(123.0, 456.0), want.nan_to_num(123.0, 456.0))


STREAMED = {
    "few_keys": dict(lens=[2, 3, 5, 17, 33, 9], nq=[1] * 6, H=8, kv=8),
    "one_head": dict(lens=[200, 7, 60], nq=[2, 1, 1], H=14, kv=2),
    "two_sets_of_rows": dict(lens=[150, 31], nq=[3, 2], H=40, kv=8),
    "two_heads_together": dict(lens=[120, 40], nq=[2, 2], H=16, kv=4),
    "four_heads_together": dict(lens=[190, 20, 3], nq=[1] * 3, H=16, kv=16),
    "prefix": dict(lens=[10, 20, 3, 40], nq=[1] * 4, H=8, kv=4, groups=[(0, 4, 100)]),
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("name", STREAMED)
def test_streamed_rows_lose_nothing_but_the_last_rounding(ctx, name, dtype):
    """Up to 16 stacked rows: the output is off by its own rounding, as if the probabilities had 32 bits.  (Small logits: a probability's relative
    error from its logit, 2^-15 of the logit's size as for the weights, is then far below a step of the element type.)  Rounded to the element
    type the probabilities would be off by up to half a step each, 2^-8 or 2^-11 of theirs."""
    c = Case(**STREAMED[name], dtype=dtype, seed=60, weights=False)
    c.run(ctx, scale=0.005)
    A.asap_check(ctx)
    out, _, _, pv, size = c.ref(scale=0.005)
    eps, sub = torch.finfo(dtype).eps, torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2
    # the two terms (a step, and half a step of that), 32-bit sums, and the smallest numbers of the type as elsewhere
    rel = eps * eps / 2 + 2.0 ** -15 * float(size.max()) + 2.0 ** -16 + 2.0 ** -15
    assert rel < 2.0 ** -13
    tol = eps / 2 * out.abs() * (1 + eps) + rel * pv + sub * (1 + 8.0 * 200)
    bad = ~((c.out.double() - out).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), ((c.out.double() - out).abs() / tol).max().item())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")], ids=["inf", "-inf"])
@pytest.mark.parametrize("H,kv,nq,n", [(2, 2, 1, 1), (8, 8, 1, 300), (8, 2, 2, 150), (10, 1, 1, 70), (4, 2, 70, 200)],
                         ids=["one_key", "four_heads", "two_heads", "one_head", "tiles"])
def test_rows_that_admit_an_infinite_value(ctx, value, dtype, H, kv, nq, n):
    """A value with an infinite element among the keys of every row, the one of the largest logit (a probability that the type holds exactly if it is
    1) or another: that element of the output is infinite, the others keep every bit."""
    for which in (0, n // 2):
        c = Case(lens=[n, 40], nq=[nq, 1], H=H, kv=kv, dtype=dtype, seed=54, weights=False)
        if which == 0:
            c.k[c.start[0]] = c.q[0, ::H // kv] * 0.25
        c.v[c.start[0] + which, :, 5] = 0.0
        c.run(ctx, scale=0.02)
        good = c.out.clone()
        assert torch.isfinite(good).all()
        c.v[c.start[0] + which, :, 5] = value
        c.run(ctx, scale=0.02)
        A.asap_check(ctx)
        want = good.clone()
        want[:nq, :, 5] = value
        assert torch.equal(c.out, want)


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")], ids=["inf", "-inf", "nan"])
@pytest.mark.parametrize("H,kv,nq", [(2, 2, 5), (16, 2, 1), (4, 2, 70)], ids=["few", "one", "many"])
def test_rows_that_admit_an_infinite_key(ctx, value, H, kv, nq):
    """A key with an infinite element: rows whose logit is minus infinity give it no probability, and rows whose logit is plus infinity or NaN are NaN,
    in the output and in lse.  The others keep every bit."""
    c = Case(lens=[150, 90], nq=[nq, 2], H=H, kv=kv, dtype=torch.bfloat16, seed=52, weights=False)
    c.run(ctx)
    good, good_lse = c.out.clone(), c.lse.clone()
    key = c.len[0] - nq                                          # the first row's own: all rows of the sequence admit it
    c.k[c.start[0] + key, :, 5] = value
    c.run(ctx)
    A.asap_check(ctx)
    with_it = (c.q[:nq, :, 5].double() * value) != -math.inf      # (NaN counts)
    assert value != value or (0 < int(with_it.sum()) < with_it.numel())
    assert torch.isnan(c.out[:nq][with_it]).all() and torch.isnan(c.lse[:nq][with_it]).all()
    assert torch.equal(c.out[nq:], good[nq:]) and torch.equal(c.lse[nq:], good_lse[nq:])
    # without it: the same as the formula over the other keys, a logit of minus infinity in its place
    ref = c.ref()
    fine = ~with_it
    assert torch.isfinite(ref[0][:nq][fine]).all()
    assert ((c.out[:nq].double() - ref[0][:nq]).abs() <= 2.0 ** -8 * ref[0][:nq].abs() + 2.0 ** -7 * ref[3][:nq])[fine].all()
    assert ((c.lse[:nq].double() - ref[1][:nq]).abs()[fine] <= 2.0 ** -15 * (1 + ref[1][:nq].abs()[fine])).all()


def test_nan_queries_stay_in_their_rows(ctx):
    c = Case(lens=[150, 80], nq=[3, 1], H=4, kv=2, dtype=torch.bfloat16, seed=9, weights=False, groups=[(0, 2, 90)])
    c.run(ctx)
    good, lse = c.out.clone(), c.lse.clone()
    c.q[1, 2] = float("nan")
    c.run(ctx)
    hit = torch.zeros(4, 4, dtype=torch.bool, device=DEV)
    hit[1, 2] = True
    assert torch.isnan(c.out[hit]).all() and torch.isnan(c.lse[hit]).all()
    assert torch.equal(c.out[~hit], good[~hit]) and torch.equal(c.lse[~hit], lse[~hit])


def test_large_logits(ctx):
    """Logits of thousands, rising along the keys: the running maximum moves in every tile, and the other rows' sums vanish."""
    c = Case(lens=[500, 300], nq=[1, 40], H=4, kv=2, dtype=torch.bfloat16, seed=10)
    ramp = torch.arange(c.k.shape[0], device=DEV).float()[:, None, None] / 5
    c.k.copy_((c.k.float() * ramp).to(c.k.dtype))
    c.check(ctx)


def test_weights_are_the_same_bits_every_time(ctx):
    c = Case(lens=[300, 70, 33, 500], nq=[1, 2, 1, 1], H=8, kv=2, dtype=torch.bfloat16, seed=11, groups=[(0, 3, 400)])
    base = c.weights.clone()
    runs = []
    for _ in range(3):
        c.weights.copy_(base)
        c.run(ctx)
        runs.append((c.out.clone(), c.lse.clone(), c.weights.clone()))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))
    gone = torch.isnan(c.k[:, 0, 0])                   # rows of nobody
    assert torch.equal(c.weights[gone], base[gone])


@pytest.mark.parametrize("spoil", ["len", "start", "q", "prefix", "group"])
def test_a_bad_sequence_is_skipped(ctx, spoil):
    c = Case(lens=[100, 31, 64], nq=[1, 2, 1], H=4, kv=2, dtype=torch.bfloat16, seed=12, groups=[(0, 1, 50), (1, 3, 70)])
    base = c.weights.clone()
    ref = c.ref()
    skipped = {"len": [1], "start": [1], "q": [1, 2], "prefix": [1, 2], "group": [0, 1, 2]}[spoil]
    kw = {}
    if spoil == "len":
        c.dev["len"][1] = 10000
    elif spoil == "start":
        c.dev["start"][1] = -5
    elif spoil == "q":
        kw["max_q"] = 1                                 # sequence 1 has two query rows, and so its group of two has three
    elif spoil == "prefix":
        c.dev["prefix_len"][1] = -1
    else:
        c.dev["group_cu"][1] = 9                        # both groups' ranges
    c.run(ctx, **kw)
    with pytest.raises(A.AsapError) as e:
        A.asap_check(ctx)
    assert e.value.status == -6
    dead = torch.tensor([any(c.q_cu[b] <= r < c.q_cu[b + 1] for b in skipped) for r in range(4)], device=DEV)
    assert (c.out[dead] == 7).all() and (c.lse[dead] == 7).all()
    live = ~dead
    assert ((c.out.double() - ref[0]).abs()[live] <= (2.0 ** -8 * ref[0].abs() + 2.0 ** -7 * ref[3])[live]).all()
    for b in skipped:
        assert torch.equal(c.weights[c.start[b]:c.start[b] + c.len[b]], base[c.start[b]:c.start[b] + c.len[b]])


def test_capture_replay_and_another_stream(ctx):
    """A captured call takes the lengths that the arrays hold when it is replayed, on another stream as well."""
    c = Case(lens=[300, 70, 33], nq=[1, 1, 1], H=8, kv=2, dtype=torch.bfloat16, seed=13, groups=[(0, 2, 400)], slack=200)
    c.k.copy_(torch.nan_to_num(c.k)); c.v.copy_(torch.nan_to_num(c.v))
    args = c.args(max_len=400)
    scratch = torch.empty(A.asap_cache_attention_scratch_bytes(ctx, args), dtype=torch.uint8, device=DEV)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        A.asap_cache_attention(ctx, args, scratch)
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            A.asap_cache_attention(ctx, args, scratch)
    for lens in ([300, 70, 33], [1, 0, 200], [17, 333, 64]):
        c.len = lens
        c.start = [min(x, c.k.shape[0] - n) for x, n in zip(c.start, lens)]
        c.dev["len"].copy_(i32(lens)); c.dev["start"].copy_(i32(c.start))
        c.weights.zero_()
        graph.replay()
        torch.cuda.synchronize()
        A.asap_check(ctx)
        ref = c.ref()
        R.check_attention(c.out, c.lse, ref, torch.bfloat16, 800)
    other = torch.cuda.Stream()
    first = c.out.clone()
    c.out.fill_(7)
    torch.cuda.synchronize()
    A.asap_cache_attention(ctx, args, scratch, other)
    other.synchronize()
    assert torch.equal(first, c.out)


@pytest.mark.parametrize("H,kv,groups", [(8, 2, [(0, 2, 400)]), (8, 8, None), (8, 2, None)], ids=["tiles", "streamed", "few"])
def test_weights_of_a_replayed_call(ctx, H, kv, groups):
    """The weights under the lengths that a replay finds, added to what the rows had."""
    c = Case(lens=[300, 70, 33], nq=[1, 1, 1] if kv == 2 else [9, 2, 3], H=H, kv=kv, dtype=torch.bfloat16, seed=53, groups=groups, slack=200)
    c.k.copy_(torch.nan_to_num(c.k)); c.v.copy_(torch.nan_to_num(c.v))
    args = c.args(max_len=400)
    scratch = torch.empty(A.asap_cache_attention_scratch_bytes(ctx, args), dtype=torch.uint8, device=DEV)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        A.asap_cache_attention(ctx, args, scratch)
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            A.asap_cache_attention(ctx, args, scratch)
    rows = c.k.shape[0]
    own = sum(p for _, _, _, p in c.groups) + 10                  # (own rows behind the prefixes, apart from each other)
    for lens in ([300, 70, 33], [1, 0, 200], [17, 333, 64], [0, 0, 0]):
        c.len, c.start = lens, [own + sum(lens[:b]) for b in range(3)]
        assert c.start[2] + lens[2] <= rows
        c.dev["len"].copy_(i32(lens)); c.dev["start"].copy_(i32(c.start))
        before = torch.rand(rows, device=DEV, generator=gen(sum(lens)))
        c.weights.copy_(before)
        graph.replay()
        torch.cuda.synchronize()
        A.asap_check(ctx)
        ref = c.ref()
        R.check_attention(c.out, c.lse, ref, torch.bfloat16, 800)
        R.check_weights(c.weights, before, ref, sum(c.nq))


def test_a_padded_batch(ctx):
    """Query rows behind the last sequence's, as a batch of fixed size has them, stay as they are, whatever they hold."""
    c = Case(lens=[100, 31, 64], nq=[1, 2, 20], H=4, kv=2, dtype=torch.bfloat16, seed=21, groups=[(0, 2, 90)])
    c.run(ctx)
    first = (c.out.clone(), c.lse.clone())
    d = Case(lens=[100, 31, 64], nq=[1, 2, 20], H=4, kv=2, dtype=torch.bfloat16, seed=21, groups=[(0, 2, 90)])
    pad = torch.full((5, 4, HEAD), float("nan"), dtype=torch.bfloat16, device=DEV)
    d.q = torch.cat([c.q, pad])
    d.out, d.lse = torch.full((28, 4, HEAD), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((28, 4), 7.0, device=DEV)
    d.run(ctx)
    A.asap_check(ctx)
    assert torch.equal(d.out[:23], first[0]) and torch.equal(d.lse[:23], first[1]) and torch.equal(d.weights, c.weights)
    assert (d.out[23:] == 7).all() and (d.lse[23:] == 7).all()


@pytest.mark.parametrize("spoil", ["q_cu", "group_cu"])
def test_offsets_that_do_not_ascend_skip_the_call(ctx, spoil):
    c = Case(lens=[100, 31, 64, 20], nq=[2, 3, 1, 40], H=4, kv=2, dtype=torch.bfloat16, seed=22, groups=[(0, 1, 50), (1, 4, 70)])
    base = c.weights.clone()
    if spoil == "q_cu":
        c.dev["q_cu"][2] = 1
    else:
        c.dev["group_cu"].copy_(i32([2, 1, 4]))
    c.run(ctx)
    with pytest.raises(A.AsapError) as e:
        A.asap_check(ctx)
    assert e.value.status == -6
    assert (c.out == 7).all() and (c.lse == 7).all() and torch.equal(c.weights, base)


def test_two_contexts_on_two_streams(ctx):
    """Calls on contexts and scratch of their own may overlap."""
    other = A.asap_init(0, 64, 1, 1, HEAD)
    try:
        cases = [Case(lens=[900, 70, 400], nq=[1, 1, 1], H=32, kv=8, dtype=torch.bfloat16, seed=s, groups=[(0, 3, 800)]) for s in (23, 24)]
        for c in cases:
            c.run(ctx)
        A.asap_check(ctx)
        want = [(c.out.clone(), c.lse.clone()) for c in cases]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        work = []
        for c, x in zip(cases, (ctx, other)):
            args = c.args()
            work.append((args, torch.empty(A.asap_cache_attention_scratch_bytes(x, args), dtype=torch.uint8, device=DEV), x))
            c.out.fill_(7)
        torch.cuda.synchronize()
        for _ in range(20):
            for (args, scratch, x), s in zip(work, streams):
                A.asap_cache_attention(x, args, scratch, s)
        for (_, _, x), s in zip(work, streams):
            A.asap_check(x, s)
        torch.cuda.synchronize()
        assert all(torch.equal(c.out, w[0]) and torch.equal(c.lse, w[1]) for c, w in zip(cases, want))
    finally:
        A.asap_free(other)


def test_back_to_back_calls_of_different_shapes(ctx):
    """Calls that follow each other without a wait, through the same scratch: each launch sequence keeps out of the way of the one before."""
    cases = [Case(**CASES[n], dtype=torch.bfloat16, seed=30 + i) for i, n in enumerate(["many_items", "groups", "many_splits", "one_row", "sixteen_rows",
                                                                                       "four_heads_together", "whole_prompt", "prefix_only"])]
    args = [c.args() for c in cases]
    scratch = torch.empty(max(A.asap_cache_attention_scratch_bytes(ctx, a) for a in args), dtype=torch.uint8, device=DEV)
    want = []
    for c, a in zip(cases, args):
        A.asap_cache_attention(ctx, a, scratch)
        A.asap_check(ctx)
        want.append((c.out.clone(), c.lse.clone()))
    rng = random.Random(31)
    for _ in range(6):
        order = list(range(len(cases)))
        rng.shuffle(order)
        for c in cases:
            c.out.fill_(7)
        for i in order:
            A.asap_cache_attention(ctx, args[i], scratch)
        torch.cuda.synchronize()
        assert all(torch.equal(c.out, w[0]) and torch.equal(c.lse, w[1]) for c, w in zip(cases, want))
    A.asap_check(ctx)


def test_offsets_past_32_bits(ctx):
    """A cache of more than 2^31 elements, the sequence and its prefix at its end."""
    rows, kv = 1 << 20, 32
    k = torch.empty(rows, kv, HEAD, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    assert k.numel() > 2 ** 31
    c = Case(lens=[70, 200], nq=[1, 1], H=32, kv=32, dtype=torch.bfloat16, seed=14, groups=[(0, 2, 150)], weights=False)
    n = c.k.shape[0]
    k[rows - n:], v[rows - n:] = c.k, c.v
    c.run(ctx)
    first = c.out.clone()
    c.out.fill_(7)
    c.k, c.v = k, v
    c.dev["start"] += rows - n
    c.dev["prefix_start"] += rows - n
    c.run(ctx)
    A.asap_check(ctx)
    assert torch.equal(first, c.out)


def test_many_sequences(ctx):
    rng = random.Random(15)
    c = Case(lens=[rng.randrange(0, 40) for _ in range(900)], nq=[1] * 900, H=2, kv=1, dtype=torch.bfloat16, seed=15,
             groups=[(i * 45, i * 45 + 45, rng.randrange(0, 90)) for i in range(20)])
    c.check(ctx)


# ------------------------------------------------------------------------------------------------ eviction
def _evict_case(seed, lens, special=False, gap=3):
    rng = random.Random(seed)
    start, row = [], rng.randrange(3)
    for n in lens:
        start.append(row)
        row += n + rng.randrange(gap)
    rows = row + 2
    w = torch.rand(rows, generator=torch.Generator().manual_seed(seed)).pow(3) * 5
    if special:
        pick = [0.0, -0.0, float("nan"), float("inf"), -float("inf"), 1.0, 1e-40, -1.0]
        w = torch.tensor([rng.choice(pick) for _ in range(rows)])
    pos = torch.zeros(rows, dtype=torch.int32)
    for s, n in zip(start, lens):
        p = sorted(rng.sample(range(-5, 3 * n + 5), n))
        pos[s:s + n] = torch.tensor(p, dtype=torch.int32)
    return start, rows, w, pos


def _bits(t):
    return t.view(torch.int32)


@pytest.mark.parametrize("in_place", [False, True], ids=["apart", "in_place"])
@pytest.mark.parametrize("special", [False, True], ids=["random", "special"])
@pytest.mark.parametrize("lens,keep,sink,recent,row", [([0, 1, 5, 40, 33], 5, 1, 2, 16), ([2000, 700, 1025, 31], 640, 4, 64, 272),
                                                       ([9000], 8999, 0, 0, 4096), ([300, 300], 1, 0, 1, 48), ([65, 64, 63], 64, 30, 34, 256),
                                                       ([150, 400], 129, 129, 0, 768), ([70001], 4096, 4, 512, 64),
                                                       ([6000, 20000, 5, 6144], 700, 4, 50, 16), ([400000], 3000, 2, 10, 16)])
def test_eviction(ctx, lens, keep, sink, recent, row, special, in_place):
    start, rows, w, pos = _evict_case(len(lens) * 31 + keep, lens, special)
    B = len(lens)
    src = [torch.randint(0, 255, (rows, row), dtype=torch.uint8, device=DEV, generator=gen(i)) for i in range(3)]
    before = [t.clone() for t in src]
    dw, dp = w.to(DEV), pos.to(DEV)
    keep_idx, new_len = torch.full((B, keep), 77, dtype=torch.int32, device=DEV), i32(lens)
    expect = [R.evict(w[s:s + n].tolist(), pos[s:s + n].tolist(), keep, sink, recent) for s, n in zip(start, lens)]
    if in_place:
        dst, ow, op, dst_start = src, dw, dp, list(start)
        args = A.CacheEvict(i32(start), new_len, max(lens), keep, dw, dp, keep_idx, new_len, src=src, dst=src, dst_weights=dw, dst_pos=dp,
                            sink=sink, recent=recent)
    else:
        dst_start = [b * keep + 1 for b in range(B)]
        dst = [torch.full((B * keep + 3, row), 9, dtype=torch.uint8, device=DEV) for _ in src]
        ow, op = torch.full((B * keep + 3,), 9.0, device=DEV), torch.full((B * keep + 3,), 9, dtype=torch.int32, device=DEV)
        args = A.CacheEvict(i32(start), i32(lens), max(lens), keep, dw, dp, keep_idx, new_len, src=src, dst=dst, dst_start=i32(dst_start),
                            dst_weights=ow, dst_pos=op, sink=sink, recent=recent)
    want = [t.clone() for t in dst]
    want_w, want_p = ow.clone(), op.clone()
    A.asap_cache_evict(ctx, args)
    A.asap_check(ctx)
    assert new_len.tolist() == [len(e) for e in expect]
    for b, e in enumerate(expect):
        assert keep_idx[b].tolist() == e + [-1] * (keep - len(e)), b
        at = torch.tensor(e, device=DEV, dtype=torch.long) + start[b]
        to = slice(dst_start[b], dst_start[b] + len(e))
        for t, x in zip(want, before):
            t[to] = x[at]
        want_w[to], want_p[to] = w.to(DEV)[at], pos.to(DEV)[at]
    assert all(torch.equal(t, x) for t, x in zip(dst, want))          # and every other row as it was
    assert torch.equal(_bits(ow), _bits(want_w)) and torch.equal(op, want_p)


@pytest.mark.parametrize("special", [False, True], ids=["random", "special"])
@pytest.mark.parametrize("lens,keep", [([20000, 31, 7000], 900), ([60000, 50001], 4096)])
def test_long_evictions_without_clusters(ctx, monkeypatch, lens, keep, special):
    """A device that cannot place a cluster of eight large blocks: one block ranks a long sequence, and gives what the cluster gives."""
    monkeypatch.setenv("ASAP_EVICT_CLUSTER", "0")
    single = A.asap_init(0, 64, 1, 1, HEAD)
    start, rows, w, pos = _evict_case(len(lens) + keep, lens, special)
    got, names = [], []
    try:
        for c in (ctx, single):
            keep_idx, new_len = torch.full((len(lens), keep), 77, dtype=torch.int32, device=DEV), i32([0] * len(lens))
            A.asap_profile(c, True)
            A.asap_cache_evict(c, A.CacheEvict(i32(start), i32(lens), max(lens), keep, w.to(DEV), pos.to(DEV), keep_idx, new_len, sink=3, recent=40))
            A.asap_check(c)
            names.append(list(A.asap_profile_read(c)))
            A.asap_profile(c, False)
            got.append((keep_idx.tolist(), new_len.tolist()))
    finally:
        A.asap_free(single)
    assert names == [["evict_select_cluster"], ["evict_select"]]
    assert got[0] == got[1]
    for b, (s, n) in enumerate(zip(start, lens)):
        e = R.evict(w[s:s + n].tolist(), pos[s:s + n].tolist(), keep, 3, 40)
        assert got[1][0][b] == e + [-1] * (keep - len(e)) and got[1][1][b] == len(e)


def test_eviction_of_a_large_batch_with_one_long_sequence(ctx):
    """A block per sequence, and one whose keys do not fit its shared memory."""
    lens = [55000] + [60 + i for i in range(79)]
    start, rows, w, pos = _evict_case(21, lens)
    dw, dp, new_len = w.to(DEV), pos.to(DEV), i32(lens)
    keep_idx, ow = torch.empty(80, 64, dtype=torch.int32, device=DEV), torch.full((rows,), 9.0, device=DEV)
    A.asap_cache_evict(ctx, A.CacheEvict(i32(start), new_len, 55000, 64, dw, dp, keep_idx, new_len, dst_weights=ow, sink=2, recent=10))
    A.asap_check(ctx)
    for b, n in enumerate(lens):
        e = R.evict(w[start[b]:start[b] + n].tolist(), pos[start[b]:start[b] + n].tolist(), 64, 2, 10)
        assert keep_idx[b].tolist() == e + [-1] * (64 - len(e)) and int(new_len[b]) == len(e), b
        assert torch.equal(ow[start[b]:start[b] + len(e)].cpu(), w[torch.tensor(e) + start[b]]), b


def test_eviction_without_positions_or_tensors(ctx):
    lens = [100, 7, 260]
    start, rows, w, _ = _evict_case(5, lens)
    dw = w.to(DEV)
    keep_idx, new_len, op = torch.empty(3, 50, dtype=torch.int32, device=DEV), i32([0, 0, 0]), torch.zeros(rows, dtype=torch.int32, device=DEV)
    A.asap_cache_evict(ctx, A.CacheEvict(i32(start), i32(lens), 260, 50, dw, None, keep_idx, new_len, dst_pos=op, sink=2, recent=10))
    for b, n in enumerate(lens):
        e = R.evict(w[start[b]:start[b] + n].tolist(), list(range(n)), 50, 2, 10)
        assert keep_idx[b].tolist() == e + [-1] * (50 - len(e)) and int(new_len[b]) == len(e)
        assert op[start[b]:start[b] + len(e)].tolist() == e


def test_eviction_of_tensors_given_as_iterators(ctx):
    """Tensors that a generator hands out are moved like those of a list."""
    lens = [100, 80]
    start, rows, w, pos = _evict_case(11, lens)
    src, dst = [torch.randn(rows, 8, device=DEV, generator=gen(i)) for i in range(2)], [torch.full((rows, 8), 9.0, device=DEV) for _ in range(2)]
    keep_idx, new_len = torch.empty(2, 20, dtype=torch.int32, device=DEV), i32([0, 0])
    args = A.CacheEvict(i32(start), i32(lens), 100, 20, w.to(DEV), pos.to(DEV), keep_idx, new_len, src=iter(src), dst=(t for t in dst))
    assert args.c.n_tensors == 2
    A.asap_cache_evict(ctx, args)
    A.asap_check(ctx)
    for b in range(2):
        at = slice(start[b], start[b] + 20)
        assert all(torch.equal(d[at], s[start[b] + keep_idx[b].long()]) for s, d in zip(src, dst))


def test_eviction_of_weights_in_place_beside_tensors_apart(ctx):
    lens = [300, 7, 1200]
    start, rows, w, pos = _evict_case(9, lens)
    dw, dp = w.to(DEV), pos.to(DEV)
    src = torch.randn(rows, 16, device=DEV)
    dst = torch.full((rows, 16), 9.0, device=DEV)
    keep_idx, new_len = torch.empty(3, 90, dtype=torch.int32, device=DEV), i32([0, 0, 0])
    A.asap_cache_evict(ctx, A.CacheEvict(i32(start), i32(lens), 1200, 90, dw, dp, keep_idx, new_len, src=[src], dst=[dst], dst_weights=dw,
                                         dst_pos=dp, sink=1, recent=5))
    A.asap_check(ctx)
    want = dst.clone().fill_(9.0)
    for s, n in zip(start, lens):
        e = R.evict(w[s:s + n].tolist(), pos[s:s + n].tolist(), 90, 1, 5)
        at = torch.tensor(e) + s
        assert torch.equal(dw[s:s + len(e)].cpu(), w[at]) and torch.equal(dp[s:s + len(e)].cpu(), pos[at])
        assert torch.equal(dw[s + len(e):s + n].cpu(), w[s + len(e):s + n])
        want[s:s + len(e)] = src[at.to(DEV)]
    assert torch.equal(dst, want)


@pytest.mark.parametrize("spoil", ["len", "start", "dst"])
def test_eviction_skips_a_bad_sequence(ctx, spoil):
    lens = [100, 70, 90]
    start, rows, w, pos = _evict_case(6, lens)
    s, n, d = i32(start), i32(lens), i32([0, 50, 100])
    if spoil == "len":
        n[1] = 101
    elif spoil == "start":
        s[1] = rows - 69
    else:
        d[1] = 101
    src = torch.randn(rows, 8, device=DEV)
    dst = torch.full((150, 8), 9.0, device=DEV)
    keep_idx, new_len = torch.empty(3, 50, dtype=torch.int32, device=DEV), i32([7, 7, 7])
    A.asap_cache_evict(ctx, A.CacheEvict(s, n, 100, 50, w.to(DEV), pos.to(DEV), keep_idx, new_len, src=[src], dst=[dst], dst_start=d))
    with pytest.raises(A.AsapError) as e:
        A.asap_check(ctx)
    assert e.value.status == -6
    assert new_len.tolist() == [50, 7, 50] and (keep_idx[1] == -1).all() and (dst[50:100] == 9).all()
    assert not (dst[:50] == 9).any() and not (dst[100:] == 9).any()


@pytest.mark.parametrize("special", [False, True], ids=["random", "special"])
@pytest.mark.parametrize("cap,sink,recent", [(1, 0, 0), (40, 4, 10), (700, 0, 0), (5000, 4, 100), (64, 0, 63)])
def test_slot_is_the_row_that_eviction_would_drop(ctx, cap, sink, recent, special):
    B = 5
    rng = random.Random(cap)
    lens = [cap, cap, 0, cap - 1, cap]
    start = [b * cap for b in range(B)]
    w = torch.rand(B * cap, generator=torch.Generator().manual_seed(cap))
    if special:
        w = torch.tensor([rng.choice([0.0, -0.0, float("nan"), float("inf"), 2.0]) for _ in range(B * cap)])
    pos = torch.tensor([p for _ in range(B) for p in rng.sample(range(3 * cap), cap)], dtype=torch.int32)
    new_pos = [3 * cap + 1] * B
    dw, dp, dl, row = w.to(DEV), pos.to(DEV), i32(lens), i32([-9] * B)
    A.asap_cache_slot(ctx, A.CacheSlot(i32(start), dl, cap, dw, dp, i32(new_pos), row, sink=sink, recent=recent))
    A.asap_check(ctx)
    for b in range(B):
        if lens[b] < cap:
            slot = lens[b]
        else:
            s = slice(start[b], start[b] + cap)
            slot = R.rank(w[s].tolist(), pos[s].tolist(), cap, sink, recent, new_pos[b] - 1)[-1]
        assert int(row[b]) == start[b] + slot, b
        w[start[b] + slot], pos[start[b] + slot] = 0.0, new_pos[b]
        lens[b] = min(lens[b] + 1, cap)
    assert dl.tolist() == lens and torch.equal(_bits(dw.cpu()), _bits(w)) and torch.equal(dp.cpu(), pos)


def test_slot_skips_a_bad_sequence(ctx):
    dw, dp, dl, row = torch.ones(30, device=DEV), torch.arange(30, dtype=torch.int32, device=DEV), i32([11, 10, -1]), i32([5, 5, 5])
    A.asap_cache_slot(ctx, A.CacheSlot(i32([0, 21, 0]), dl, 10, dw, dp, i32([40, 40, 40]), row))
    with pytest.raises(A.AsapError):
        A.asap_check(ctx)
    assert row.tolist() == [-1, -1, -1] and dl.tolist() == [11, 10, -1] and (dw == 1).all()


def test_slots_of_caches_about_to_be_full(ctx):
    """The call fills the last free row: the length that it writes is the one that tells a full cache, and no thread may take it for the
    length before.  Row 0 is the lowest ranked one, which a thread that saw a full cache would choose."""
    B, cap = 3000, 700
    dw, dp = torch.rand(B * cap, device=DEV, generator=gen(3)) + 1, torch.arange(cap, dtype=torch.int32, device=DEV).repeat(B)
    dw[::cap] = 0.5
    start, dl, row = torch.arange(B, dtype=torch.int32, device=DEV) * cap, torch.empty(B, dtype=torch.int32, device=DEV), torch.empty(B, dtype=torch.int32, device=DEV)
    args = A.CacheSlot(start, dl, cap, dw, dp, i32([cap + 5] * B), row)
    want_w, want_p = dw.clone(), dp.clone()
    want_w[cap - 1::cap], want_p[cap - 1::cap] = 0.0, cap + 5
    for _ in range(30):
        dl.fill_(cap - 1)
        row.fill_(-9)
        A.asap_cache_slot(ctx, args)
        assert torch.equal(row, start + cap - 1) and (dl == cap).all() and torch.equal(dw, want_w) and torch.equal(dp, want_p)
    want_w[cap - 1::cap] = 2.0                          # now they are full, and row 0 goes
    dw.copy_(want_w)
    A.asap_cache_slot(ctx, args)
    A.asap_check(ctx)
    assert torch.equal(row, start) and (dl == cap).all() and (dw[::cap] == 0).all() and (dp[::cap] == cap + 5).all()


# ------------------------------------------------------------------------------------------------ all of them together
def test_prune_then_decode_with_eviction(ctx):
    """A pruned prompt's cache is compacted, then questions are answered token by token: every new row is rotated into its slot, attends
    over its image's shared rows and its own, adds to the weights, and full caches give up their lowest ranked row.  A second model of
    the cache in 64 bits follows every step."""
    batch = W.tiny(B=2, n_vis=[120, 90], text_lens=[6, 9], H=4, keep_k=32, seed=900, centres=6)
    inp = A.make_inputs(batch, DEV)
    out = A.alloc_outputs(inp, 32, fill=True)
    A.asap_prune_step(ctx, inp, A.Params(keep_k=32), out)
    cu = out.out_cu_seqlens.tolist()
    H, kv, rows = 4, 4, cu[2] + 6 * 24
    kc = torch.zeros(rows, kv, HEAD, dtype=torch.bfloat16, device=DEV)
    vc = torch.zeros_like(kc)
    A.asap_compact_kv(ctx, out.src_row, out.out_cu_seqlens[2:], [inp.k, W.draw_values(batch, 901).to(DEV)], [kc, vc])
    B, cap, steps = 6, 24, 60
    start = [cu[2] + b * cap for b in range(B)]
    length = i32([0] * B)
    weights, pos = torch.zeros(rows, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    first = [int(out.out_pos[cu[1] - 1]) + 1] * 4 + [int(out.out_pos[cu[2] - 1]) + 1] * 2
    new_pos, row = i32(first), i32([0] * B)
    plan = A.asap_rope_make(HEAD)
    qkv = torch.empty(B, 3 * H, HEAD, dtype=torch.bfloat16, device=DEV)
    q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
    qr, o, lse = torch.empty(B, H, HEAD, dtype=torch.bfloat16, device=DEV), torch.empty(B, H, HEAD, dtype=torch.bfloat16, device=DEV), torch.empty(B, H, device=DEV)
    groups = [(0, 4, 0, cu[1]), (4, 6, cu[1], cu[2] - cu[1])]
    slot = A.CacheSlot(i32(start), length, cap, weights, pos, new_pos, row, sink=2, recent=5)
    rope = A.RopeArgs(new_pos, [A.RopeTensor(q, qr), A.RopeTensor(k, kc, mapped=True), A.RopeTensor(v, vc, mapped=True, rotate=False)], dst_row=row)
    att = A.CacheAttention(qr, kc, vc, o, i32(start), length, max_len=cap, group_cu=i32([0, 4, 6]), prefix_start=i32([0, cu[1]]),
                           prefix_len=i32([cu[1], cu[2] - cu[1]]), max_prefix=max(cu[1], cu[2] - cu[1]), lse=lse, weights=weights)
    scratch = torch.empty(A.asap_cache_attention_scratch_bytes(ctx, att), dtype=torch.uint8, device=DEV)
    model_pos, reused = [[] for _ in range(B)], 0
    g = gen(902)
    for step in range(steps):
        qkv.copy_(torch.randn(qkv.shape, device=DEV, generator=g))
        before = weights.clone()
        expect_row = []
        for b in range(B):                                     # the 64-bit model's slot, from the weights as they are
            if len(model_pos[b]) < cap:
                expect_row.append(start[b] + len(model_pos[b]))
                model_pos[b].append(first[b] + step)
            else:
                r = R.rank(before[start[b]:start[b] + cap].tolist(), model_pos[b], cap, 2, 5, first[b] + step - 1)[-1]
                expect_row.append(start[b] + r)
                model_pos[b][r] = first[b] + step
                reused += 1
        A.asap_cache_slot(ctx, slot)
        A.asap_rope(ctx, plan, rope)
        A.asap_cache_attention(ctx, att, scratch)
        assert row.tolist() == expect_row
        assert length.tolist() == [len(p) for p in model_pos]
        before[torch.tensor(expect_row, device=DEV)] = 0.0
        _close_rotation(kc[row.long()], R.rotate(k, new_pos, HEAD, "half", _freq(plan)), k, torch.bfloat16, 1.0)
        ref = R.attention(qr, kc, vc, start, length.tolist(), list(range(B + 1)), groups)
        R.check_attention(o, lse, ref, torch.bfloat16, 200)
        R.check_weights(weights, before, ref, B)
        new_pos += 1
    A.asap_check(ctx)
    assert reused > 100
    for b in range(B):
        assert pos[start[b]:start[b] + cap].tolist() == model_pos[b]
    # cut the caches back in place and answer once more
    keep_idx = torch.empty(B, 10, dtype=torch.int32, device=DEV)
    w0, k0, v0 = weights.clone(), kc.clone(), vc.clone()
    A.asap_cache_evict(ctx, A.CacheEvict(i32(start), length, cap, 10, weights, pos, keep_idx, length, src=[kc, vc], dst=[kc, vc],
                                         dst_weights=weights, dst_pos=pos, sink=2, recent=5))
    for b in range(B):
        e = R.evict(w0[start[b]:start[b] + cap].tolist(), model_pos[b], 10, 2, 5)
        assert keep_idx[b].tolist() == e and int(length[b]) == 10
        at = torch.tensor(e, device=DEV) + start[b]
        assert torch.equal(kc[start[b]:start[b] + 10], k0[at]) and torch.equal(vc[start[b]:start[b] + 10], v0[at])
        assert torch.equal(weights[start[b]:start[b] + 10], w0[at]) and pos[start[b]:start[b] + 10].tolist() == [model_pos[b][i] for i in e]
    before = weights.clone()
    A.asap_cache_attention(ctx, att, scratch)
    ref = R.attention(qr, kc, vc, start, [10] * B, list(range(B + 1)), groups)
    R.check_attention(o, lse, ref, torch.bfloat16, 200)
    R.check_weights(weights, before, ref, B)
    A.asap_check(ctx)


def _decode(ctx, steps, wait, H, kv, seqs, groups, weights):
    """Slot, rotation and attention `steps` times, every call's arrays written by the call before it; with `wait` the host waits for each call."""
    cap, pre = 30, 200
    rows, G = len(groups) * pre + seqs * cap, len(groups)
    g = gen(77)
    kc, vc = torch.randn(rows, kv, HEAD, device=DEV, generator=g).to(torch.bfloat16), torch.randn(rows, kv, HEAD, device=DEV, generator=g).to(torch.bfloat16)
    start, length = i32([G * pre + b * cap for b in range(seqs)]), i32([b % cap for b in range(seqs)])
    w, pos = torch.zeros(rows, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    for b in range(seqs):
        pos[G * pre + b * cap:G * pre + (b + 1) * cap] = torch.arange(cap, dtype=torch.int32, device=DEV)
    new_pos, row = [i32([cap + s] * seqs) for s in range(steps)], i32([0] * seqs)
    qkv = torch.randn(steps, seqs, H + 2 * kv, HEAD, device=DEV, generator=g).to(torch.bfloat16)
    qr, out, lse = torch.empty(seqs, H, HEAD, dtype=torch.bfloat16, device=DEV), torch.empty(steps, seqs, H, HEAD, dtype=torch.bfloat16, device=DEV), torch.empty(seqs, H, device=DEV)
    plan, calls, scratch = A.asap_rope_make(HEAD), [], None
    kw = dict(group_cu=i32([0] + [b1 for _, b1 in groups]), prefix_start=i32([i * pre for i in range(G)]), prefix_len=i32([pre - i for i in range(G)]),
              max_prefix=pre) if groups else {}
    for s in range(steps):
        q, k, v = qkv[s, :, :H], qkv[s, :, H:H + kv], qkv[s, :, H + kv:]
        slot = A.CacheSlot(start, length, cap, w, pos, new_pos[s], row, sink=1, recent=3)
        rope = A.RopeArgs(new_pos[s], [A.RopeTensor(q, qr), A.RopeTensor(k, kc, mapped=True), A.RopeTensor(v, vc, mapped=True, rotate=False)], dst_row=row)
        att = A.CacheAttention(qr, kc, vc, out[s], start, length, max_len=cap, lse=lse, weights=w if weights else None, **kw)
        if scratch is None:
            scratch = torch.empty(A.asap_cache_attention_scratch_bytes(ctx, att), dtype=torch.uint8, device=DEV)
        calls += [lambda x=slot: A.asap_cache_slot(ctx, x), lambda x=rope: A.asap_rope(ctx, plan, x), lambda x=att: A.asap_cache_attention(ctx, x, scratch)]
    torch.cuda.synchronize()
    for call in calls:
        call()
        if wait:
            torch.cuda.synchronize()
    A.asap_check(ctx)
    return out, lse, w, pos, length, kc, vc


@pytest.mark.parametrize("weights", [False, True], ids=["", "weights"])
@pytest.mark.parametrize("H,kv,seqs,groups", [(8, 2, 12, [(0, 12)]), (16, 16, 40, [(0, 18), (18, 40)]), (8, 8, 1, []), (32, 8, 2, []), (4, 4, 30, [(0, 3), (3, 30)])],
                         ids=["tiles", "more_tiles", "one_request", "two_requests", "both"])
def test_steps_that_nobody_waits_between(ctx, H, kv, seqs, groups, weights):
    """Lengths, rows, queries and keys that a call has just written are what the next one reads, through the same buffers step after step."""
    steps = 40
    want = _decode(ctx, steps, True, H, kv, seqs, groups, weights)
    for _ in range(4):
        got = _decode(ctx, steps, False, H, kv, seqs, groups, weights)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("nq", [[1, 1], [20, 40]], ids=["streamed", "tiles"])
def test_a_wait_that_runs_out_is_reported_and_the_context_recovers(ctx, nq):
    # (long enough that every block has more tiles than its ring holds: some wait cannot be satisfied at once)
    c = Case(lens=[30000, 20000], nq=nq, H=32, kv=32, dtype=torch.bfloat16, seed=16, weights=False)
    c.run(ctx)
    good = c.out.clone()
    A.asap_debug_wait_limit(ctx, 1)
    c.run(ctx)
    with pytest.raises(A.AsapError) as e:
        A.asap_check(ctx)
    assert e.value.status == -6 and "cache attention" in str(e.value)
    c.out.fill_(7)
    c.run(ctx)
    A.asap_check(ctx)
    assert torch.equal(c.out, good)


GIVING_UP = {
    "one_head": dict(lens=[30000, 9000], nq=[1, 1], H=14, kv=2),
    "rows_eight_and_up": dict(lens=[20000, 3000], nq=[3, 2], H=40, kv=8),
    "two_heads_together": dict(lens=[4000] * 40, nq=[2] * 40, H=16, kv=4),
    "four_heads_together": dict(lens=[3000] * 60, nq=[1] * 60, H=32, kv=32),
    "tiles_and_streams": dict(lens=[2000] * 12, nq=[1] * 6 + [40] * 6, H=32, kv=8, groups=[(0, 8, 3000), (8, 12, 500)]),
    "short_items": dict(lens=[70] * 100, nq=[3] * 100, H=32, kv=8, groups=[(0, 60, 400), (60, 100, 130)]),
}


@pytest.mark.parametrize("weights", [False, True], ids=["", "weights"])
@pytest.mark.parametrize("name", GIVING_UP)
def test_a_wait_that_gives_up_is_never_silent(ctx, name, weights):
    """Limits from a clock to more than any wait takes, so that waits of every kind run out, in some blocks and warps and not in others: the
    call comes to an end and is reported, or its results are right to the last bit."""
    c = Case(**GIVING_UP[name], dtype=torch.bfloat16, seed=50, weights=weights)
    base = c.weights.clone() if weights else None
    args = c.args()
    scratch = torch.full((A.asap_cache_attention_scratch_bytes(ctx, args),), 0x7f, dtype=torch.uint8, device=DEV)

    def go():
        c.out.fill_(7)
        c.lse.fill_(7)
        if weights:
            c.weights.copy_(base)
        A.asap_cache_attention(ctx, args, scratch)
        return [t.clone() for t in (c.out, c.lse, c.weights) if t is not None]

    want = go()
    A.asap_check(ctx)
    reported = 0
    for limit in [1, 10, 40, 100, 250, 500, 800, 1200, 2000, 4000, 8000, 16000, 50000, 200000, 10 ** 9]:
        A.asap_debug_wait_limit(ctx, limit)
        got = go()
        try:
            A.asap_check(ctx)
        except A.AsapError as e:
            assert e.status == -6 and "cache attention" in str(e) and limit < 10 ** 9
            reported += 1
            continue
        assert all(torch.equal(a, b) for a, b in zip(got, want)), limit
    assert reported > 0
    assert all(torch.equal(a, b) for a, b in zip(go(), want))
    A.asap_check(ctx)
