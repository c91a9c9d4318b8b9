"""The work of the operators around a key/value cache: rotary positions with the rows appended to the cache, attention of
new tokens over a cache with shared prefixes and accumulated attention weights, and eviction by those weights.

A case names an operator, its sizes and how ragged they are; `prepare` makes the tensors that a program holds before the call,
`run` makes one pass, in elementary torch operations or, with `own`, through the library.  All lengths follow from the case
alone, all values from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

HEAD = 128
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_context = None


def listed():
    return [
        # one new token of one request: the latency of a decoder layer's rotation and append
        dict(name="rope_token", op="rope", rows=1, heads=32, kv_heads=32, rot=128, layout="half", scaling="none", factor=1.0,
             theta=10000.0, far=700, append=True, cache=1024, dtype="bf16"),
        # one new token each of a batch at far positions: interleaved pairs, part of the head, frequencies scaled by bands
        dict(name="rope_batch_far", op="rope", rows=67, heads=32, kv_heads=8, rot=64, layout="interleaved", scaling="yarn", factor=16.0,
             theta=10000.0, far=500000, append=True, cache=4096, dtype="fp16"),
        # the prompts of eight image conversations, from the fused projection into the cache
        dict(name="rope_prompt", op="rope", rows=24531, heads=32, kv_heads=32, rot=128, layout="half", scaling="linear", factor=2.0,
             theta=10000.0, far=3171, append=False, cache=24531, dtype="bf16"),
        # one request after pruning to 192 visual tokens, weights accumulated: the smallest decode step
        dict(name="attend_one", op="attend", seqs=1, groups=0, heads=32, kv_heads=32, lo=267, hi=267, pre_lo=0, pre_hi=0, q_lo=1, q_hi=1,
             layout="rows", weights=True, dtype="bf16", ragged=1),
        # a decode step of 64 pruned AnyRes prompts (576 of 2880 visual tokens kept), weights accumulated for eviction
        dict(name="attend_pruned", op="attend", seqs=64, groups=0, heads=32, kv_heads=32, lo=643, hi=1100, pre_lo=0, pre_hi=0, q_lo=1,
             q_hi=1, layout="rows", weights=True, dtype="bf16", ragged=2),
        # a few long conversations, eight key/value heads, keys and values interleaved in one buffer, fp16
        dict(name="attend_long", op="attend", seqs=5, groups=0, heads=32, kv_heads=8, lo=2000, hi=60000, pre_lo=0, pre_hi=0, q_lo=1,
             q_hi=1, layout="pairs", weights=False, dtype="fp16", ragged=3),
        # many questions about a few images: each group shares the image's rows, every question decodes, weights accumulated
        dict(name="attend_questions", op="attend", seqs=61, groups=6, heads=32, kv_heads=32, lo=9, hi=300, pre_lo=611, pre_hi=2915, q_lo=1,
             q_hi=1, layout="rows", weights=True, dtype="bf16", ragged=4),
        # the same questions when they arrive: several text rows each against the shared image
        dict(name="attend_question_rows", op="attend", seqs=13, groups=2, heads=32, kv_heads=32, lo=16, hi=256, pre_lo=2915, pre_hi=2915,
             q_lo=16, q_hi=256, layout="rows", weights=False, dtype="bf16", ragged=5),
        # a long shared document in front of a large batch, eight key/value heads stored head by head
        dict(name="attend_shared_long", op="attend", seqs=128, groups=1, heads=32, kv_heads=8, lo=1, hi=500, pre_lo=16001, pre_hi=16001,
             q_lo=1, q_hi=1, layout="heads", weights=False, dtype="bf16", ragged=6),
        # caches of a batch cut back to 640 rows each by accumulated weight
        dict(name="evict_batch", op="evict", seqs=24, lo=500, hi=2300, keep=640, sink=4, recent=64, kv_heads=32, dtype="bf16", ragged=7),
        # two long caches cut back to 4096 rows
        dict(name="evict_long", op="evict", seqs=2, lo=30001, hi=60001, keep=4096, sink=4, recent=512, kv_heads=8, dtype="bf16", ragged=8),
        # full caches of 64 requests: one slot each for the next token
        dict(name="slot_batch", op="slot", seqs=64, capacity=1152, sink=4, recent=128, fill=1.0, ragged=9),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "attend", "attend", "attend", "evict", "slot"])
    ragged = rng.randrange(1 << 20)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if kind == "rope":
        kv = rng.choice([1, 4, 8, 32])
        append = rng.random() < 0.6
        rows = _log_int(rng, 1, 256) if append else _log_int(rng, 100, 20000)
        return dict(op="rope", rows=rows, heads=32, kv_heads=kv, rot=rng.choice([20, 32, 64, 96, 128]),
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "ntk", "yarn", "bands"]),
                    factor=rng.choice([2.0, 4.0, 8.0]), theta=rng.choice([1e4, 5e5]), far=_log_int(rng, 1000, 1000000), append=append,
                    cache=rows + rng.randrange(1, 3000), dtype=dtype)
    if kind == "attend":
        heads, kv = rng.choice([(32, 32), (40, 40), (32, 8), (32, 4), (28, 4), (16, 1)])
        shared = rng.random() < 0.5
        q_hi = rng.choice([1, 1, 1, 3, 40])
        seqs = _log_int(rng, 1, 80 if q_hi < 40 else 12)
        budget = (1 << 26) // (kv * HEAD)                     # rows that hold 128 MB of keys
        lo = _log_int(rng, 1, 400)
        hi = max(lo, min(_log_int(rng, 16, 30000), budget // seqs))
        pre = _log_int(rng, 32, min(8000, budget)) if shared else 0
        return dict(op="attend", seqs=seqs, groups=rng.randrange(1, min(seqs, max(1, budget // max(pre, 1)), 6) + 1) if shared else 0, heads=heads,
                    kv_heads=kv, lo=lo, hi=hi, pre_lo=max(1, pre // 3) if shared else 0, pre_hi=pre, q_lo=1, q_hi=q_hi,
                    layout=rng.choice(["rows", "pairs", "heads"]), weights=rng.random() < 0.5, dtype=dtype, ragged=ragged)
    if kind == "evict":
        kv = rng.choice([4, 8, 32])
        seqs = _log_int(rng, 1, 32)
        hi = min(_log_int(rng, 300, 60000), (1 << 26) // (kv * HEAD) // seqs)
        keep = max(80, int(hi * rng.uniform(0.2, 0.8)))
        return dict(op="evict", seqs=seqs, lo=max(1, hi // 3), hi=hi, keep=keep, sink=rng.choice([0, 1, 4]), recent=rng.randrange(0, 70),
                    kv_heads=kv, dtype=dtype, ragged=ragged)
    return dict(op="slot", seqs=_log_int(rng, 1, 512), capacity=_log_int(rng, 100, 20000), sink=rng.choice([0, 4]),
                recent=rng.randrange(0, 90), fill=rng.choice([0.9, 1.0, 1.0]), ragged=ragged)


# ---------------------------------------------------------------------------------------------- sizes that follow from a case
def _lengths(n, lo, hi, rng):
    return [rng.randint(lo, hi) for _ in range(n)]


def _attend_sizes(c):
    """Rows of every sequence and prefix, where they lie in the cache, and the query rows."""
    rng = random.Random(c["ragged"])
    B, G = c["seqs"], c["groups"]
    nq = _lengths(B, c["q_lo"], c["q_hi"], rng)
    own_len = [max(n, q) for n, q in zip(_lengths(B, c["lo"], c["hi"], rng), nq)]       # the new rows are in the cache already
    pre = _lengths(G, c["pre_lo"], c["pre_hi"], rng)
    cuts = sorted(rng.sample(range(1, B), G - 1)) if G > 1 else []
    group_cu = [0] + cuts + [B] if G else []
    row, pre_start, start = 0, [], []
    for n in pre:
        pre_start.append(row)
        row += n
    order = list(range(B))
    rng.shuffle(order)                                        # requests come and go: their slabs lie in no order
    start = [0] * B
    for b in order:
        start[b] = row
        row += own_len[b] + rng.randint(0, 7)                 # room for the next tokens
    return dict(nq=nq, len=own_len, pre=pre, group_cu=group_cu, pre_start=pre_start, start=start, rows=row)


def _evict_sizes(c):
    rng = random.Random(c["ragged"])
    lens = _lengths(c["seqs"], c["lo"], c["hi"], rng)
    start, row = [], 0
    for n in lens:
        start.append(row)
        row += n + rng.randint(0, 5)
    return dict(len=lens, start=start, rows=row)


def _slot_sizes(c):
    rng = random.Random(c["ragged"])
    cap = c["capacity"]
    lens = [cap if rng.random() < c["fill"] else rng.randint(max(1, cap // 2), cap) for _ in range(c["seqs"])]
    return dict(len=lens, start=[b * cap for b in range(c["seqs"])], rows=c["seqs"] * cap)


def work(case):
    c, e = case, 2
    if c["op"] == "rope":
        elements = c["rows"] * (c["heads"] + 2 * c["kv_heads"]) * HEAD
        return {"bytes": 2 * e * elements + 8 * c["rows"], "flops": 3 * c["rows"] * (c["heads"] + c["kv_heads"]) * c["rot"]}
    if c["op"] == "attend":
        s = _attend_sizes(c)
        keys = sum(s["len"]) + sum(s["pre"])
        n_q = sum(s["nq"])
        pairs = sum(q * (n - q) + q * (q + 1) // 2 for q, n in zip(s["nq"], s["len"]))
        for g, p in enumerate(s["pre"]):
            pairs += p * sum(s["nq"][s["group_cu"][g]:s["group_cu"][g + 1]])
        return {"bytes": 2 * e * keys * c["kv_heads"] * HEAD + 2 * e * n_q * c["heads"] * HEAD + 4 * n_q * c["heads"]
                + (8 * keys if c["weights"] else 0), "flops": 4 * HEAD * c["heads"] * pairs}
    if c["op"] == "evict":
        s = _evict_sizes(c)
        kept = sum(min(n, c["keep"]) for n in s["len"])
        return {"bytes": 2 * 2 * e * kept * c["kv_heads"] * HEAD + 8 * sum(s["len"]) + 12 * kept, "flops": 0}
    s = _slot_sizes(c)
    return {"bytes": 8 * sum(s["len"]) + 24 * c["seqs"], "flops": 0}


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def _rope_plan(c):
    from paper_2603_14549_b200 import binding as A
    return A.asap_rope_make(c["rot"], layout=c["layout"], theta=c["theta"], scaling=c["scaling"], factor=c["factor"],
                            original_positions=4096)


def _handle():
    """The library context that a program keeps."""
    global _context
    from paper_2603_14549_b200 import binding as A
    if _context is None:
        _context = A.asap_init(torch.cuda.current_device(), 64, 1, 1, HEAD)
    return A, _context


def _cache(c, rows, g):
    """Keys and values [rows, kv_heads, 128] as row-major tensors, as halves of one buffer, or head by head."""
    dtype, kv = DTYPES[c["dtype"]], c["kv_heads"]
    if c.get("layout") == "pairs":
        both = _normal((rows, 2, kv, HEAD), dtype, g)
        return both[:, 0], both[:, 1]
    if c.get("layout") == "heads":
        return _normal((kv, rows, HEAD), dtype, g).transpose(0, 1), _normal((kv, rows, HEAD), dtype, g).transpose(0, 1)
    return _normal((rows, kv, HEAD), dtype, g), _normal((rows, kv, HEAD), dtype, g)


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = {"case": c}
    if c["op"] == "rope":
        rng = random.Random(int(seed) * 7919 + c["rows"])
        dtype, H, kv, n = DTYPES[c["dtype"]], c["heads"], c["kv_heads"], c["rows"]
        fused = _normal((n, H + 2 * kv, HEAD), dtype, g)
        st["q"], st["k"], st["v"] = fused[:, :H], fused[:, H:H + kv], fused[:, H + kv:]
        if c["append"]:
            st["pos"] = _i32([rng.randrange(c["far"]) for _ in range(n)])
            st["dst"] = _i32(rng.sample(range(c["cache"]), n))
        else:
            st["pos"] = torch.arange(n, dtype=torch.int32, device="cuda") % c["far"]
            st["dst"] = torch.arange(n, dtype=torch.int32, device="cuda") + (c["cache"] - n)
        st["q_out"] = torch.empty(n, H, HEAD, dtype=dtype, device="cuda")
        st["k_cache"] = _normal((c["cache"], kv, HEAD), dtype, g)
        st["v_cache"] = _normal((c["cache"], kv, HEAD), dtype, g)
        if own:
            A, st["ctx"] = _handle()
            st["plan"] = _rope_plan(c)
            st["args"] = A.RopeArgs(st["pos"], [A.RopeTensor(st["q"], st["q_out"]),
                                                A.RopeTensor(st["k"], st["k_cache"], mapped=True),
                                                A.RopeTensor(st["v"], st["v_cache"], mapped=True, rotate=False)], dst_row=st["dst"])
        else:
            st["freq"], st["mag"] = _frequencies(c)
        return st
    if c["op"] == "attend":
        s = _attend_sizes(c)
        n_q, H = sum(s["nq"]), c["heads"]
        dtype = DTYPES[c["dtype"]]
        st["q"] = _normal((n_q, H, HEAD), dtype, g)
        st["k"], st["v"] = _cache(c, s["rows"], g)
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(n_q, H, dtype=torch.float32, device="cuda")
        st["weights"] = torch.rand(s["rows"], device="cuda", generator=g) if c["weights"] else None
        st["start"], st["len"] = _i32(s["start"]), _i32(s["len"])
        st["q_cu"] = _i32(np.concatenate([[0], np.cumsum(s["nq"])]).tolist())
        st["max"] = (max(s["len"]), max(s["nq"]), max(s["pre"], default=0))
        st["group_cu"] = st["pre_start"] = st["pre_len"] = None
        if c["groups"]:
            st["group_cu"], st["pre_start"], st["pre_len"] = _i32(s["group_cu"]), _i32(s["pre_start"]), _i32(s["pre"])
            cu = np.concatenate([[0], np.cumsum(s["nq"])])
            st["max_group_q"] = int(max(cu[s["group_cu"][i + 1]] - cu[s["group_cu"][i]] for i in range(c["groups"])))
        if own:
            A, st["ctx"] = _handle()
            st["args"] = A.CacheAttention(st["q"], st["k"], st["v"], st["out"], st["start"], st["len"], max_len=st["max"][0],
                                          q_cu=st["q_cu"], max_q=st["max"][1], group_cu=st["group_cu"], prefix_start=st["pre_start"],
                                          prefix_len=st["pre_len"], max_prefix=st["max"][2], lse=st["lse"], weights=st["weights"])
            st["scratch"] = torch.empty(A.asap_cache_attention_scratch_bytes(st["ctx"], st["args"]), dtype=torch.uint8, device="cuda")
        return st
    s = _evict_sizes(c) if c["op"] == "evict" else _slot_sizes(c)
    st["weights"] = torch.rand(s["rows"], device="cuda", generator=g).pow(4) * 20      # a few rows hold most of the weight
    st["start"], st["len"] = _i32(s["start"]), _i32(s["len"])
    st["pos"] = torch.zeros(s["rows"], dtype=torch.int32, device="cuda")
    for b, n in enumerate(s["len"]):
        step = torch.randint(1, 3, (n,), device="cuda", generator=g)                   # earlier evictions left gaps
        st["pos"][s["start"][b]:s["start"][b] + n] = torch.cumsum(step, 0).int()
    st["max_len"] = max(s["len"])
    if c["op"] == "slot":
        last = torch.tensor([s["start"][b] + n - 1 for b, n in enumerate(s["len"])], device="cuda")
        st["new_pos"] = st["pos"][last] + 1
        st["row"] = torch.empty(c["seqs"], dtype=torch.int32, device="cuda")
        if own:
            A, st["ctx"] = _handle()
            st["args"] = A.CacheSlot(st["start"], st["len"], c["capacity"], st["weights"], st["pos"], st["new_pos"], st["row"],
                                     sink=c["sink"], recent=c["recent"])
        return st
    st["k"], st["v"] = _cache(c, s["rows"], g)
    B, keep = c["seqs"], c["keep"]
    st["dst_start"] = torch.arange(B, dtype=torch.int32, device="cuda") * keep
    st["k_out"] = torch.zeros(B * keep, c["kv_heads"], HEAD, dtype=st["k"].dtype, device="cuda")
    st["v_out"] = torch.zeros_like(st["k_out"])
    st["weights_out"] = torch.zeros(B * keep, device="cuda")
    st["pos_out"] = torch.zeros(B * keep, dtype=torch.int32, device="cuda")
    st["keep_idx"] = torch.empty(B, keep, dtype=torch.int32, device="cuda")
    st["new_len"] = torch.empty(B, dtype=torch.int32, device="cuda")
    if own:
        A, st["ctx"] = _handle()
        st["args"] = A.CacheEvict(st["start"], st["len"], st["max_len"], keep, st["weights"], st["pos"], st["keep_idx"], st["new_len"],
                                  src=[st["k"], st["v"]], dst=[st["k_out"], st["v_out"]], dst_start=st["dst_start"],
                                  dst_weights=st["weights_out"], dst_pos=st["pos_out"], sink=c["sink"], recent=c["recent"])
    return st


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        from paper_2603_14549_b200 import binding as A
        op = state["case"]["op"]
        if op == "rope":
            A.asap_rope(state["ctx"], state["plan"], state["args"])
        elif op == "attend":
            A.asap_cache_attention(state["ctx"], state["args"], state["scratch"])
        elif op == "evict":
            A.asap_cache_evict(state["ctx"], state["args"])
        else:
            A.asap_cache_slot(state["ctx"], state["args"])
        return _outputs(state)
    return {"rope": _plain_rope, "attend": _plain_attend, "evict": _plain_evict, "slot": _plain_slot}[state["case"]["op"]](state)


def _outputs(st):
    names = {"rope": ("q_out", "k_cache", "v_cache"), "attend": ("out", "lse", "weights"),
             "evict": ("keep_idx", "new_len", "k_out", "v_out", "weights_out", "pos_out"), "slot": ("row", "len", "weights", "pos")}
    return {n: st[n] for n in names[st["case"]["op"]]}


def _frequencies(c):
    """Turns per position of every pair, in 64 bits, and the factor of the rotated values."""
    n, theta, f, orig = c["rot"] // 2, c["theta"], c["factor"], 4096
    i = torch.arange(n, dtype=torch.float64, device="cuda")
    if c["scaling"] == "ntk":
        theta = theta * f ** (c["rot"] / (c["rot"] - 2))
    turns = theta ** (-i / n) / (2 * math.pi)
    mag = 1.0
    if c["scaling"] == "linear":
        turns = turns / f
    if c["scaling"] == "yarn":
        # pairs that turn more than 32 times over the original length keep their frequency, those under one turn are divided
        at = lambda rotations: n * math.log(orig / (rotations * 2 * math.pi)) / math.log(theta)   # noqa: E731
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), 2 * n - 1)
        ramp = ((i - low) / max(high - low, 0.001)).clamp(0, 1)
        turns = turns * (1 - ramp) + turns / f * ramp
        mag = 0.1 * math.log(f) + 1.0
    if c["scaling"] == "bands":
        # the same in terms of turns over the original length: kept above 4, divided under 1, linear between
        smooth = ((orig * turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        turns = turns * smooth + turns / f * (1 - smooth)
    return turns, mag


def _plain_rotate(x, cos, sin, rot, layout):
    x = x.float()
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rope(st):
    c = st["case"]
    turns = st["pos"].double()[:, None] * st["freq"]
    angle = (turns - turns.round()) * (2 * math.pi)
    cos, sin = ((f * st["mag"]).float()[:, None, :] for f in (angle.cos(), angle.sin()))
    st["q_out"].copy_(_plain_rotate(st["q"], cos, sin, c["rot"], c["layout"]))
    dst = st["dst"].long()
    st["k_cache"][dst] = _plain_rotate(st["k"], cos, sin, c["rot"], c["layout"]).to(st["k"].dtype)
    st["v_cache"][dst] = st["v"]
    return _outputs(st)


def _plain_attend(st):
    """Queries padded per sequence (own rows) and per group (shared rows); logits of both side by side, one softmax."""
    c, q = st["case"], st["q"]
    n_q, H, kv = q.shape[0], c["heads"], c["kv_heads"]
    B, rep = c["seqs"], H // kv
    dev = q.device
    max_len, max_q, max_pre = st["max"]
    q_cu, start, length = st["q_cu"].long(), st["start"].long(), st["len"].long()
    rows = torch.arange(n_q, device=dev)
    seq = torch.searchsorted(q_cu, rows, right=True) - 1
    t = rows - q_cu[seq]
    nq = q_cu[1:] - q_cu[:-1]
    key = torch.arange(max_len, device=dev)
    at = (start[:, None] + key.clamp(max=max_len)).clamp(max=st["k"].shape[0] - 1)
    inside = key < length[:, None]
    qf = q.float().view(n_q, kv, rep, HEAD)
    padded = torch.zeros(B, max_q, kv, rep, HEAD, device=dev)
    padded[seq, t] = qf
    k = torch.where(inside[:, :, None, None], st["k"][at].float(), 0.0)
    s = torch.matmul(padded.permute(0, 2, 1, 3, 4).reshape(B, kv, max_q * rep, HEAD), k.permute(0, 2, 3, 1))
    del k
    s = s.view(B, kv, max_q, rep, max_len).permute(0, 2, 1, 3, 4)[seq, t].reshape(n_q, H, max_len) / math.sqrt(HEAD)
    admitted = key <= (length - nq)[seq][:, None] + t[:, None]
    s = torch.where((admitted & inside[seq])[:, None, :], s, -math.inf)
    if c["groups"]:
        G = c["groups"]
        group_cu, p_start, p_len = st["group_cu"].long(), st["pre_start"].long(), st["pre_len"].long()
        grp = torch.searchsorted(group_cu, seq, right=True) - 1
        u = rows - q_cu[group_cu[grp]]
        max_u = st["max_group_q"]
        pkey = torch.arange(max_pre, device=dev)
        p_at = (p_start[:, None] + pkey).clamp(max=st["k"].shape[0] - 1)
        p_in = pkey < p_len[:, None]
        padded = torch.zeros(G, max_u, kv, rep, HEAD, device=dev)
        padded[grp, u] = qf
        k = torch.where(p_in[:, :, None, None], st["k"][p_at].float(), 0.0)
        sp = torch.matmul(padded.permute(0, 2, 1, 3, 4).reshape(G, kv, max_u * rep, HEAD), k.permute(0, 2, 3, 1))
        del k
        sp = sp.view(G, kv, max_u, rep, max_pre).permute(0, 2, 1, 3, 4)[grp, u].reshape(n_q, H, max_pre) / math.sqrt(HEAD)
        s = torch.cat([s, torch.where(p_in[grp][:, None, :], sp, -math.inf)], -1)
        del sp
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = torch.exp(s - top)
    del s
    total = p.sum(-1, keepdim=True)
    st["lse"].copy_((torch.log(total) + top)[..., 0])
    p = p / torch.where(total > 0, total, 1.0)
    v = torch.where(inside[:, :, None, None], st["v"][at].float(), 0.0)
    padded = torch.zeros(B, max_q, kv, rep, max_len, device=dev)
    padded[seq, t] = p[..., :max_len].view(n_q, kv, rep, max_len)
    o = torch.matmul(padded.permute(0, 2, 1, 3, 4).reshape(B, kv, max_q * rep, max_len), v.permute(0, 2, 1, 3))
    o = o.view(B, kv, max_q, rep, HEAD).permute(0, 2, 1, 3, 4)[seq, t].reshape(n_q, H, HEAD)
    del v
    if c["weights"]:
        w = torch.zeros(B, max_len, device=dev).index_add_(0, seq, p[..., :max_len].sum(1) / H)
        st["weights"][at[inside]] += w[inside]
    if c["groups"]:
        v = torch.where(p_in[:, :, None, None], st["v"][p_at].float(), 0.0)
        padded = torch.zeros(G, max_u, kv, rep, max_pre, device=dev)
        padded[grp, u] = p[..., max_len:].view(n_q, kv, rep, max_pre)
        op = torch.matmul(padded.permute(0, 2, 1, 3, 4).reshape(G, kv, max_u * rep, max_pre), v.permute(0, 2, 1, 3))
        o = o + op.view(G, kv, max_u, rep, HEAD).permute(0, 2, 1, 3, 4)[grp, u].reshape(n_q, H, HEAD)
        if c["weights"]:
            w = torch.zeros(G, max_pre, device=dev).index_add_(0, grp, p[..., max_len:].sum(1) / H)
            st["weights"][p_at[p_in]] += w[p_in]
    st["out"].copy_(o)
    return _outputs(st)


def _ranked(st, n, newest):
    """Rows of every sequence, best first: the first `sink`, those of the last `recent` positions, the others by weight; lower row
    first among equals.  Rows past a sequence come last."""
    c = st["case"]
    key = torch.arange(n, device=newest.device)
    length = st["len"].long()
    at = (st["start"].long()[:, None] + key).clamp(max=st["pos"].shape[0] - 1)
    pos, w = st["pos"][at].long(), st["weights"][at]
    held = (key < c["sink"]) | (pos > newest[:, None] - c["recent"])
    rank = torch.where(held, math.inf, w)
    rank = torch.where(key < length[:, None], rank, -math.inf)
    return torch.sort(rank, dim=1, descending=True, stable=True).indices, at


def _plain_evict(st):
    c = st["case"]
    n, keep = st["max_len"], c["keep"]
    length = st["len"].long()
    key = torch.arange(n, device=length.device)
    at = (st["start"].long()[:, None] + key).clamp(max=st["pos"].shape[0] - 1)
    newest = torch.where(key < length[:, None], st["pos"][at].long(), -(1 << 40)).amax(1)
    order, at = _ranked(st, n, newest)
    new_len = length.clamp(max=keep)
    slot = torch.arange(keep, device=length.device)
    used = slot < new_len[:, None]
    width = min(n, keep)
    first = torch.full((length.shape[0], keep), n, device=length.device)
    first[:, :width] = order[:, :width]
    kept = torch.where(used, first, n).sort(1).values
    st["keep_idx"].copy_(torch.where(used, kept, -1))
    st["new_len"].copy_(new_len)
    src = (st["start"].long()[:, None] + kept)[used]
    dst = (st["dst_start"].long()[:, None] + slot)[used]
    st["k_out"][dst] = st["k"][src]
    st["v_out"][dst] = st["v"][src]
    st["weights_out"][dst] = st["weights"][src]
    st["pos_out"][dst] = st["pos"][src]
    return _outputs(st)


def _plain_slot(st):
    c = st["case"]
    n = c["capacity"]
    length = st["len"].long()
    order, _ = _ranked(st, n, st["new_pos"].long() - 1)
    full = length >= n
    slot = torch.where(full, order[:, n - 1], length)
    row = st["start"].long() + slot
    st["row"].copy_(row)
    st["len"].copy_(torch.where(full, length, length + 1))
    st["weights"][row] = 0.0
    st["pos"][row] = st["new_pos"]
    return _outputs(st)


# ---------------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["op"] == "rope":
        n, rot = c["rows"], c["rot"]
        f, half = c["factor"], c["rot"] // 2
        base = c["theta"] * (f ** (rot / (rot - 2)) if c["scaling"] == "ntk" else 1.0)
        w = np.array([base ** (-2.0 * i / rot) for i in range(half)])
        mag = 1.0
        if c["scaling"] == "linear":
            w = w / f
        elif c["scaling"] == "yarn":
            lo = max(math.floor(rot * math.log(4096 / (32 * 2 * math.pi)) / (2 * math.log(base))), 0)
            hi = min(math.ceil(rot * math.log(4096 / (2 * math.pi)) / (2 * math.log(base))), rot - 1)
            g = np.clip((np.arange(half) - lo) / max(hi - lo, 0.001), 0, 1)
            w, mag = w / f * g + w * (1 - g), 0.1 * math.log(f) + 1
        elif c["scaling"] == "bands":
            g = np.clip((4096 * w / (2 * math.pi) - 1) / 3, 0, 1)
            w = w / f * (1 - g) + w * g
        z = torch.polar(torch.full((n, half), mag, dtype=torch.float64, device="cuda"),
                        st["pos"].double()[:, None] * torch.tensor(w, device="cuda"))[:, None, :]

        def turn(x):
            x = x.double()
            pair = torch.complex(x[..., :half], x[..., half:rot]) if c["layout"] == "half" else \
                torch.complex(x[..., 0:rot:2].contiguous(), x[..., 1:rot:2].contiguous())
            y = pair * z
            out = x.clone()
            if c["layout"] == "half":
                out[..., :half], out[..., half:rot] = y.real, y.imag
            else:
                out[..., 0:rot:2], out[..., 1:rot:2] = y.real, y.imag
            return out
        k_cache, v_cache = st["k_cache"].double(), st["v_cache"].double()
        k_cache[st["dst"].long()] = turn(st["k"])
        v_cache[st["dst"].long()] = st["v"].double()
        return {"q_out": turn(st["q"]), "k_cache": k_cache, "v_cache": v_cache}
    if c["op"] == "attend":
        s = _attend_sizes(c)
        rep = c["heads"] // c["kv_heads"]
        out = torch.zeros(sum(s["nq"]), c["heads"], HEAD, dtype=torch.float64, device="cuda")
        lse = torch.zeros(sum(s["nq"]), c["heads"], dtype=torch.float64, device="cuda")
        weights = st["weights"].double() if c["weights"] else None
        group = [next(i for i in range(c["groups"]) if s["group_cu"][i + 1] > b) if c["groups"] else -1 for b in range(c["seqs"])]
        row = 0
        for b, (n, m) in enumerate(zip(s["nq"], s["len"])):
            idx = torch.arange(s["start"][b], s["start"][b] + m, device="cuda")
            p = 0
            if group[b] >= 0:
                p = s["pre"][group[b]]
                idx = torch.cat([torch.arange(s["pre_start"][group[b]], s["pre_start"][group[b]] + p, device="cuda"), idx])
            hidden = torch.arange(p + m, device="cuda")[None, :] > torch.arange(n, device="cuda")[:, None] + (p + m - n)
            total = torch.zeros(p + m, dtype=torch.float64, device="cuda")
            for h in range(c["kv_heads"]):
                hs = slice(h * rep, (h + 1) * rep)
                x = torch.einsum("thd,jd->htj", st["q"][row:row + n, hs].double(), st["k"][idx, h].double()) * HEAD ** -0.5
                x = x.masked_fill(hidden, -math.inf)
                lse[row:row + n, hs] = torch.logsumexp(x, -1).T
                a = torch.softmax(x, -1)
                out[row:row + n, hs] = torch.einsum("htj,jd->thd", a, st["v"][idx, h].double())
                total += a.sum((0, 1)) / c["heads"]
            if weights is not None:
                weights[idx] += total
            row += n
        return {"out": out, "lse": lse, "weights": weights}
    # eviction computes no value: it says which rows stay, and moves them
    s = _evict_sizes(c) if c["op"] == "evict" else _slot_sizes(c)
    weight, pos = st["weights"].double().cpu().numpy().copy(), st["pos"].cpu().numpy().copy()

    def best_first(b, newest):
        rows = np.arange(s["len"][b])
        held = (rows < c["sink"]) | (pos[s["start"][b] + rows] > newest - c["recent"])
        return np.lexsort((rows, np.where(held, 0.0, -weight[s["start"][b] + rows]), ~held))
    if c["op"] == "slot":
        row, length = np.zeros(c["seqs"], np.int32), np.array(s["len"], np.int32)
        for b, new in enumerate(st["new_pos"].tolist()):
            if s["len"][b] < c["capacity"]:
                slot, length[b] = s["len"][b], s["len"][b] + 1
            else:
                slot = best_first(b, new - 1)[-1]
            row[b] = s["start"][b] + slot
            weight[row[b]], pos[row[b]] = 0.0, new
        return {"row": row, "len": length, "weights": weight, "pos": pos}
    B, keep = c["seqs"], c["keep"]
    keep_idx, new_len = np.full((B, keep), -1, np.int32), np.array([min(n, keep) for n in s["len"]], np.int32)
    k_out, v_out = st["k_out"].double(), st["v_out"].double()
    w_out, p_out = np.zeros(B * keep), np.zeros(B * keep, np.int32)
    for b, m in enumerate(new_len):
        kept = np.sort(best_first(b, pos[s["start"][b]:s["start"][b] + s["len"][b]].max())[:m])
        keep_idx[b, :m] = kept
        src = torch.from_numpy(s["start"][b] + kept).cuda()
        k_out[b * keep:b * keep + m], v_out[b * keep:b * keep + m] = st["k"][src].double(), st["v"][src].double()
        w_out[b * keep:b * keep + m], p_out[b * keep:b * keep + m] = weight[s["start"][b] + kept], pos[s["start"][b] + kept]
    return {"keep_idx": keep_idx, "new_len": new_len, "k_out": k_out, "v_out": v_out, "weights_out": w_out, "pos_out": p_out}
