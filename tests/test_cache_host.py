"""What the calls around the key / value cache decide on the host, without a GPU: struct layouts, rotation plans, refusals."""
import ctypes as C
import math
import types

import pytest
import torch

from paper_2603_14549_b200 import binding as A
from paper_2603_14549_b200 import build
from tests.test_library_abi import _struct_fields


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return A.load_library()


@pytest.fixture()
def ctx():
    """A context of zeros: enough for calls that are refused, which look at nothing but their arguments and leave an error text."""
    return C.create_string_buffer(1 << 16)


@pytest.mark.parametrize("cname,cls", [
    ("asap_rope_plan", A.CRopePlan), ("asap_rope_tensor", A.CRopeTensor), ("asap_rope_args", A.CRopeArgs),
    ("asap_cache_attention_args", A.CCacheAttentionArgs), ("asap_cache_evict_args", A.CCacheEvictArgs),
    ("asap_cache_slot_args", A.CCacheSlotArgs)])
def test_binding_struct_matches_header(cname, cls):
    assert _struct_fields(cname) == [f[0] for f in cls._fields_]


def _freq(plan):
    return [plan.turns[i] * 2 * math.pi / 2.0 ** 64 for i in range(plan.n_pairs)]


@pytest.mark.parametrize("rot", [2, 20, 128, 256])
def test_plain_linear_and_ntk_frequencies(lib, rot):
    plain = [10000.0 ** (-2 * i / rot) for i in range(rot // 2)]
    close = lambda got, want: all(abs(g - w) <= 1e-14 * w + 1e-18 for g, w in zip(got, want, strict=True))     # noqa: E731
    assert close(_freq(A.asap_rope_make(rot)), plain)
    assert close(_freq(A.asap_rope_make(rot, scaling="linear", factor=4)), [f / 4 for f in plain])
    if rot > 2:
        base = 10000.0 * 8 ** (rot / (rot - 2))
        assert close(_freq(A.asap_rope_make(rot, scaling="ntk", factor=8)), [base ** (-2 * i / rot) for i in range(rot // 2)])
    plan = A.asap_rope_make(rot, layout="interleaved")
    assert plan.n_pairs == rot // 2 and plan.interleaved == 1 and plan.magnitude == 1.0


def test_yarn_and_bands_keep_fast_pairs_and_divide_slow_ones(lib):
    plain = _freq(A.asap_rope_make(128))
    yarn = A.asap_rope_make(128, scaling="yarn", factor=16, original_positions=4096)
    bands = A.asap_rope_make(128, scaling="bands", factor=16, original_positions=4096)
    assert abs(yarn.magnitude - (0.1 * math.log(16) + 1)) < 1e-6 and bands.magnitude == 1.0
    low = math.floor(64 * math.log(4096 / (32 * 2 * math.pi)) / math.log(10000))
    high = math.ceil(64 * math.log(4096 / (2 * math.pi)) / math.log(10000))
    for i, (p, y, b) in enumerate(zip(plain, _freq(yarn), _freq(bands))):
        share = min(max((i - low) / (high - low), 0), 1)
        assert abs(y - (p * (1 - share) + p / 16 * share)) <= 1e-14 * p
        turns = 4096 * p / (2 * math.pi)
        keep = min(max((turns - 1) / 3, 0), 1)
        assert abs(b - (p * keep + p / 16 * (1 - keep))) <= 1e-14 * p


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=258), dict(rot_dim=64, theta=1.0), dict(rot_dim=64, theta=float("nan")),
                                dict(rot_dim=64, scaling="linear", factor=0.5), dict(rot_dim=64, scaling="yarn", factor=float("nan")),
                                dict(rot_dim=2, scaling="ntk", factor=2), dict(rot_dim=64, scaling="bands", factor=2, fast=1.0, slow=1.0),
                                dict(rot_dim=64, scaling="yarn", factor=2, original_positions=0)])
def test_plans_that_are_refused(lib, kw):
    with pytest.raises(A.AsapError):
        A.asap_rope_make(**kw)


def _refused(lib, ctx, name, args, status, *more):
    st = getattr(lib, name)(ctx, *more, C.byref(args), *([] if name != "asap_cache_attention" else [4096, 1 << 40]), None)
    assert st == status, (st, lib.asap_last_error(ctx))
    assert lib.asap_last_error(ctx)


def _rope(**kw):
    t = (A.CRopeTensor * 1)(A.CRopeTensor(1 << 20, 2 << 20, 4, 1, 0, 0, 512, 128, 512, 128))
    for f in list(kw):
        if f.startswith("t_"):
            setattr(t[0], f[2:], kw.pop(f))
    a = A.CRopeArgs(3, 128, 0, 0, 1, 0, 4096, None, t)
    a.owner = t
    for f, v in kw.items():
        setattr(a, f, v)
    return a


@pytest.mark.parametrize("status,kw", [
    (-1, dict(n_rows=-1)), (-5, dict(head_dim=100)), (-5, dict(head_dim=264)), (-1, dict(head_dim=64)), (-5, dict(dtype=2)),
    (-1, dict(n_tensors=0)), (-1, dict(n_tensors=5)), (-1, dict(pos=None)), (-1, dict(t_heads=0)), (-1, dict(t_src=None)),
    (-1, dict(t_mapped=1)), (-2, dict(t_src=(1 << 20) + 2)), (-2, dict(t_src_row=513)), (-1, dict(t_dst_row=504)),
    (-1, dict(t_dst_head=64)), (-1, dict(t_src_row=-8)), (-1, dict(t_dst=(1 << 20) + 16)), (-1, dict(t_dst=1 << 20, t_dst_row=1024)),
    (-1, dict(t_src_row=1 << 40))])
def test_rotations_that_are_refused(lib, ctx, status, kw):
    plan = A.asap_rope_make(128)
    _refused(lib, ctx, "asap_rope", _rope(**kw), status, C.byref(plan))


@pytest.mark.parametrize("status,src,dst", [(-1, 3 << 20, 2 << 20), (-1, 2 << 20, 4 << 20), (-1, 3 << 20, 1 << 20)])
def test_two_tensors_of_a_rotation_that_meet_are_refused(lib, ctx, status, src, dst):
    a = _rope(n_tensors=2)
    a.owner = t = (A.CRopeTensor * 2)(a.owner[0], A.CRopeTensor(src, dst, 4, 1, 0, 0, 512, 128, 512, 128))
    a.tensors = t
    _refused(lib, ctx, "asap_rope", a, status, C.byref(A.asap_rope_make(128)))


def test_heads_beyond_the_counters_are_refused(lib, ctx):
    _refused(lib, ctx, "asap_rope", _rope(t_heads=65537, n_rows=1), -5, C.byref(A.asap_rope_make(128)))


def test_a_rotation_without_rows_does_nothing(lib, ctx):
    plan = A.asap_rope_make(128)
    assert lib.asap_rope(ctx, C.byref(plan), C.byref(_rope(n_rows=0, pos=None, t_src=None, t_dst=None)), None) == 0


def _attend(**kw):
    a = A.CCacheAttentionArgs(B=2, H=8, kv_heads=2, head_dim=128, dtype=0, n_q=2, max_q=1, max_len=100, max_prefix=0, n_groups=0,
                              cache_rows=1000, scale=0.0, q_row=1024, q_head=128, out_row=1024, out_head=128, kv_row=256, kv_head=128,
                              start=4096, len=4096, q=1 << 20, k=1 << 21, v=1 << 23, out=1 << 24)
    for f, v in kw.items():
        setattr(a, f, v)
    return a


@pytest.mark.parametrize("status,kw", [
    (-1, dict(B=0)), (-1, dict(n_q=0)), (-1, dict(max_q=0)), (-1, dict(max_q=3)), (-5, dict(head_dim=64)), (-5, dict(dtype=7)),
    (-1, dict(kv_heads=3)), (-1, dict(max_len=1001)), (-1, dict(max_len=-1)), (-1, dict(n_groups=1)), (-1, dict(n_groups=3)),
    (-5, dict(B=1025, n_q=1025)), (-1, dict(scale=-1.0)), (-1, dict(scale=float("nan"))), (-1, dict(q=None)), (-1, dict(len=None)),
    (-1, dict(n_q=3)), (-2, dict(k=(1 << 21) + 8)), (-2, dict(kv_row=260)), (-1, dict(kv_row=64)), (-1, dict(kv_head=0)),
    (-1, dict(out_row=1000)), (-1, dict(out=1 << 20)), (-1, dict(out=1 << 21)), (-1, dict(q_row=-8)), (-1, dict(kv_row=1 << 40))])
def test_attention_that_is_refused(lib, ctx, status, kw):
    _refused(lib, ctx, "asap_cache_attention", _attend(**kw), status)


def test_scratch_of_attention(lib, ctx):
    size = lambda **kw: lib.asap_cache_attention_scratch_bytes(ctx, C.byref(_attend(**kw)))      # noqa: E731
    assert size() > 0 and size(weights=4096) >= size() + 2 * 8 * 100 * 4
    assert size(B=0) == 0 and size(kv_heads=3) == 0 and lib.asap_cache_attention_scratch_bytes(None, C.byref(_attend())) == 0
    st = lib.asap_cache_attention(ctx, C.byref(_attend()), 4096, size() - 1, None)
    assert st == -3
    assert lib.asap_cache_attention(ctx, C.byref(_attend()), None, 1 << 40, None) == -3
    assert lib.asap_cache_attention(ctx, C.byref(_attend()), 4096 + 16, 1 << 40, None) == -3


@pytest.mark.parametrize("kw", [dict(head_dim=64), dict(head_dim=256), dict(dtype=7), dict(B=1025, n_q=1025), dict(B=1000, n_q=1000, n_groups=30), dict(max_q=3),
                                dict(max_q=0), dict(n_groups=3), dict(n_groups=-1), dict(max_len=1001), dict(max_prefix=1001), dict(cache_rows=0), dict(H=65537, kv_heads=1),
                                dict(B=2 ** 31 - 1, n_q=2 ** 31 - 1, n_groups=1), dict(n_q=1 << 23, H=128, q_cu=4096), dict(n_q=2 ** 31 - 1, max_q=2 ** 31 - 1, H=65536),
                                dict(B=1000, n_q=1000, H=1 << 16, kv_heads=1 << 16, max_len=2 ** 31 - 1, cache_rows=2 ** 31 - 1),
                                dict(B=1023, H=513, kv_heads=1, n_q=1, max_len=38_600_000, cache_rows=38_600_000, weights=4096)])
def test_scratch_of_sizes_that_attention_refuses(lib, ctx, kw):
    assert lib.asap_cache_attention_scratch_bytes(ctx, C.byref(_attend(**kw))) == 0
    assert b"asap_cache_attention" in lib.asap_last_error(None)
    st = lib.asap_cache_attention(ctx, C.byref(_attend(**kw)), 4096, 1 << 40, None)
    assert st in (-1, -5)


@pytest.mark.parametrize("scratch", [torch.empty(1 << 16, dtype=torch.uint8), torch.empty(1 << 16, dtype=torch.uint8, device="meta"),
                                     torch.empty(64, 64, dtype=torch.uint8, device="meta").t()], ids=["cpu", "meta", "strided"])
def test_scratch_that_is_no_contiguous_tensor_of_the_device_is_refused(lib, ctx, monkeypatch, scratch):
    """... before the library is called: on the GPU its address would be a bad one."""
    class Never:
        def __getattr__(self, name):
            raise AssertionError("the library was called")

    monkeypatch.setattr(A, "_lib", Never())
    a = _attend()
    device = torch.device("meta") if not scratch.is_contiguous() else torch.device("cuda", 0)
    with pytest.raises(ValueError):
        A.asap_cache_attention(ctx, types.SimpleNamespace(device=device, ref=C.addressof(a), c=a), scratch, stream=0)


def _evict(**kw):
    src, dst = (C.c_void_p * 2)(1 << 20, 1 << 22), (C.c_void_p * 2)(1 << 24, 1 << 26)
    for f in list(kw):
        if f in ("src0", "src1", "dst0", "dst1"):
            (src if f[0] == "s" else dst)[int(f[-1])] = kw.pop(f)
    a = A.CCacheEvictArgs(B=2, max_len=100, keep=50, sink=4, recent=10, rows=1000, dst_rows=1000, n_tensors=2, row_bytes=256, start=4096,
                          len=4096, weights=8192, keep_idx=1 << 14, new_len=4096, src=src, dst=dst)
    a.owner = (src, dst)
    for f, v in kw.items():
        setattr(a, f, v)
    return a


@pytest.mark.parametrize("status,kw", [
    (-1, dict(B=0)), (-1, dict(keep=0)), (-1, dict(max_len=0)), (-1, dict(sink=-1)), (-1, dict(sink=41)), (-1, dict(recent=2 ** 31 - 1)),
    (-5, dict(n_tensors=65)), (-5, dict(n_tensors=-1)), (-2, dict(row_bytes=24)), (-2, dict(row_bytes=0)), (-1, dict(weights=None)),
    (-1, dict(src0=None)), (-2, dict(dst1=(1 << 26) + 8)), (-5, dict(dst0=1 << 20)), (-1, dict(dst0=(1 << 20) + 256)),
    (-1, dict(dst0=1 << 22)), (-1, dict(dst1=(1 << 24) + 256)), (-1, dict(dst0=1 << 20, dst1=1 << 22, dst_start=4096)),
    (-1, dict(dst0=1 << 20, dst1=1 << 22, dst_rows=500)), (-1, dict(dst_weights=8192 + 16)), (-1, dict(dst_weights=8192, dst_start=4096)),
    (-1, dict(pos=1 << 30, dst_pos=(1 << 30) + 4)), (-5, dict(B=65536))])
def test_evictions_that_are_refused(lib, ctx, status, kw):
    _refused(lib, ctx, "asap_cache_evict", _evict(**kw), status)


@pytest.mark.parametrize("kw", [dict(keep=2 ** 30 + 1), dict(max_len=2 ** 31 - 1)])
def test_evictions_beyond_the_counters_are_refused(lib, ctx, kw):
    _refused(lib, ctx, "asap_cache_evict", _evict(**kw), -5)


def test_slots_beyond_the_counters_are_refused(lib, ctx):
    a = A.CCacheSlotArgs(B=2, capacity=2 ** 31 - 1, sink=4, recent=10, rows=1000, start=4096, len=4096, weights=8192, pos=8192, new_pos=4096, row=4096)
    _refused(lib, ctx, "asap_cache_slot", a, -5)


def test_attention_weights_of_more_blocks_than_a_launch_has_are_refused(lib, ctx):
    # 1023 sequences of up to 38,600,000 keys, 16 keys a block: 2,467,987,500 blocks
    _refused(lib, ctx, "asap_cache_attention", _attend(B=1023, H=513, kv_heads=1, n_q=1, max_q=1, max_len=38_600_000, cache_rows=38_600_000, q_cu=4096,
                                                       q_row=513 * 128, out_row=513 * 128, kv_row=128, k=1 << 40, v=1 << 41, weights=4096), -5)


@pytest.mark.parametrize("kw", [dict(B=0), dict(capacity=0), dict(sink=90, recent=10), dict(sink=-1), dict(weights=None), dict(row=None)])
def test_slots_that_are_refused(lib, ctx, kw):
    a = A.CCacheSlotArgs(B=2, capacity=100, sink=4, recent=10, rows=1000, start=4096, len=4096, weights=8192, pos=8192, new_pos=4096, row=4096)
    for f, v in kw.items():
        setattr(a, f, v)
    _refused(lib, ctx, "asap_cache_slot", a, -1)


def test_a_null_context_is_refused(lib):
    plan = A.asap_rope_make(128)
    assert lib.asap_rope(None, C.byref(plan), C.byref(_rope()), None) == -1
    assert lib.asap_cache_attention(None, C.byref(_attend()), 4096, 1 << 40, None) == -1
    assert lib.asap_cache_evict(None, C.byref(_evict()), None) == -1
    assert lib.asap_cache_slot(None, None, None) == -1
