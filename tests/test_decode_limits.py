"""Where the calls of the attention side of a decoder block end: caches that no kernel may be given, places that may not be shared, sizes of a
launch, counts past 32 bits, and values at the ends of their types."""
import json
import os
import subprocess
import sys
import textwrap
import types

import numpy as np
import pytest
import torch

from paper_2605_19561_amd import binding, build
from test_launch_host import STUB

DEV = "cuda:0"
BF, F8, E8 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu
gpu = pytest.mark.gpu


@pytest.fixture(params=["native", "interpreted"])
def either_way(request, monkeypatch):
    """The binding's C++ module, and its own Python in the place of that."""
    if request.param == "interpreted":
        monkeypatch.setattr(binding, "_host", binding._Interpreted)
    return request.param


def calls_with(cache, device):
    """The two calls that take a cache, all their other arguments in order."""
    x = torch.zeros((3, 2, 64), dtype=BF, device=device)
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)
    return {"append": lambda: binding.torq_cache_append(cache, x, x, torch.full((3,), -1, dtype=torch.int64, device=device)),
            "attention": lambda: binding.torq_paged_attention(x, cache, i(3, 2), i(3), 1.0, out=torch.zeros_like(x),
                                                              workspace=torch.zeros(1 << 20, dtype=torch.uint8, device=device))}


def host_cache():
    return binding.KVCache(*(torch.zeros((4, 2, 16, 64), dtype=BF) for _ in "kv"))


def cache_elsewhere(cache):
    """The same one as if it lay on another GPU."""
    there = torch.device("cuda", 1)
    return types.SimpleNamespace(kv_handle=cache.kv_handle, kv_device=1, k=types.SimpleNamespace(device=there), _struct=cache._struct,
                                 format=cache.format, heads=cache.heads, head_dim=cache.head_dim, page_size=cache.page_size)


@pytest.mark.parametrize("call", ["append", "attention"])
@pytest.mark.parametrize("elsewhere", [False, True])
def test_no_kernel_is_given_a_cache_of_the_host_or_of_another_device(monkeypatch, call, elsewhere):
    # every other argument passes as if it were on the device, and the library is one that takes note of its calls
    launched = []
    note = lambda *args: launched.append(args) or 0
    cache = cache_elsewhere(host_cache()) if elsewhere else host_cache()
    if elsewhere:
        cache.kv_handle = 0x1000
    monkeypatch.setattr(binding, "_host", binding._Interpreted)
    monkeypatch.setattr(binding, "_dev", lambda t, dtype, what: t.data_ptr())
    monkeypatch.setattr(binding, "_rows", lambda t, dtype, dims, what: t.data_ptr())
    monkeypatch.setattr(binding, "_stream", lambda stream=None: 0)
    monkeypatch.setattr(binding, "lib", lambda: types.SimpleNamespace(torq_cache_append=note, torq_paged_attention=note))
    with pytest.raises(ValueError, match="cache"):
        calls_with(cache, "cpu")[call]()
    assert not launched


@gpu
@pytest.mark.parametrize("call", ["append", "attention"])
def test_device_tensors_with_a_cache_of_the_host_or_of_another_device(either_way, call):
    with pytest.raises(ValueError, match="cache"):
        calls_with(host_cache(), DEV)[call]()
    here = binding.KVCache(*(torch.zeros((4, 2, 16, 64), dtype=BF, device=DEV) for _ in "kv"))
    calls_with(here, DEV)[call]()
    with pytest.raises(ValueError, match="cache"):
        calls_with(cache_elsewhere(here), DEV)[call]()


def test_workspace_sizes_need_no_cache_on_the_gpu():
    assert binding.torq_paged_attention_workspace_bytes(host_cache(), 8, 3, 4000) > 0


def test_a_cache_cannot_be_given_other_tensors():
    # the calls go by the addresses that it was made with: with another k in its place they would use the old one, freed
    cache = host_cache()
    k, other = cache.k, torch.zeros((4, 2, 16, 64), dtype=BF)
    for name, value in (("k", other), ("v", other), ("k_scales", None), ("v_scales", None), ("heads", 1), ("head_dim", 32), ("page_size", 32),
                        ("format", binding.TORQ_FMT_MXFP8)):
        with pytest.raises(AttributeError):
            setattr(cache, name, value)
    assert cache.k is k and cache.k_scales is None and (cache.heads, cache.head_dim, cache.page_size) == (2, 64, 16)
    assert cache._struct.k == k.data_ptr()


# ---- places that may not be shared -------------------------------------------------------------

def test_the_norms_two_outputs_are_two_arrays(launches):
    # each would overwrite the other's rows
    assert len(launches("""
        P2 = C.c_void_p(1 << 21)
        call = lambda x, r, ro, out, M=4: L.torq_add_rms_norm(x, r, P, M, 256, 1e-5, 8, ro, out, None, None)
        assert call(P, P2, P, P) == call(P, P2, P2, P2) == binding.TORQ_EINVAL
        assert call(P, P2, P2, P) == call(P, P2, P, P2) == call(P, None, None, P) == call(P, P2, P, P, M=0) == OK
        """)) == 3


@gpu
def test_one_tensor_for_the_norms_two_outputs(either_way):
    x, r, w = torch.randn((3, 64), device=DEV).to(BF), torch.randn((3, 64), device=DEV).to(BF), torch.ones(64, dtype=BF, device=DEV)
    before = x.clone()
    with pytest.raises(binding.TorqError) as e:
        binding.torq_add_rms_norm(x, r, w, 1e-5, residual_out=x, out=x)
    assert e.value.status == binding.TORQ_EINVAL and torch.equal(x, before)


@gpu
@pytest.mark.parametrize("fmt", [binding.TORQ_FMT_BF16, binding.TORQ_FMT_MXFP8])
def test_a_slot_named_twice_spoils_no_other(fmt):
    # what it holds itself is undefined; the slots beside it, and the tokens passed over, are as without it
    T, heads, dim, pages = 600, 4, 64, 40
    x = torch.randn((T, 2, heads, dim), device=DEV).to(BF)
    slots = torch.randperm(pages * 16, device=DEV)[:T]
    twice, several = slots.clone(), slots[5].clone()
    twice[300], twice[17], twice[599], twice[100:110] = several, several, several, -1
    alone = slots.clone()
    alone[torch.tensor([5, 300, 17, 599] + list(range(100, 110)), device=DEV)] = -1

    def filled(at):
        cache = binding.KVCache.empty(pages, heads, 16, dim, fmt)
        arrays = [t for t in (cache.k, cache.v, cache.k_scales, cache.v_scales) if t is not None]
        for t in arrays:
            t.view(torch.uint8).fill_(0x33)
        binding.torq_cache_append(cache, x[:, 0], x[:, 1], at)
        return [t.view(torch.uint8) for t in arrays]
    for got, want in zip(filled(twice), filled(alone)):
        got[several // 16, :, several % 16] = want[several // 16, :, several % 16] = 0
        assert torch.equal(got, want)


# ---- sizes of a launch -------------------------------------------------------------------------
# The runtime refuses launches whose workgroups times threads reach 2^32 along a dimension.  A stand-in for it takes note of what is asked
# of it; addresses are made up, and nothing goes to them.

@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("stub")
    taken = "hipError_t hipLaunchKernel(const void *f, dim3 g, dim3, void **, size_t lds, hipStream_t) {"
    noted = "hipError_t hipLaunchKernel(const void *f, dim3 g, dim3 b, void **args, size_t lds, hipStream_t) {\n" \
            '  fprintf(events, "{\\"threads\\": %u, \\"fourth\\": %lld}\\n", b.x, *(long long *)args[fourth]);'
    assert taken in STUB
    source = STUB.replace(taken, noted).replace('extern "C" {', 'static int fourth = 0;\nextern "C" {\nvoid stub_argument(int n) { fourth = n; }', 1)
    src, so = str(tmp / "stub.cpp"), str(tmp / "libstub.so")
    open(src, "w").write(source)
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", src, "-o", so], check=True)
    return so


@pytest.fixture
def launches(stand_in, tmp_path):
    """Runs code with L, the library, and P, an address; returns (workgroups along x and y, threads, the argument that was asked for, the
    kernel)."""
    def run(body, argument=0):
        if not os.path.exists(build.LIB):
            build.build()
        events = str(tmp_path / "events")
        code = f"""
import ctypes as C
stub = C.CDLL({stand_in!r}, mode=C.RTLD_GLOBAL)
stub.stub_open({events.encode()!r}); stub.stub_argument({argument})
from paper_2605_19561_amd import binding
L, P, OK = binding.lib(), C.c_void_p(1 << 20), binding.TORQ_OK
""" + textwrap.dedent(body) + "\nstub.stub_close()\n"
        subprocess.run([sys.executable, "-c", code], check=True, timeout=120, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
        lines = [json.loads(line) for line in open(events)]
        return [(g["grid"], b["threads"], b["fourth"], g["launch"]) for b, g in zip(lines[::2], lines[1::2])]
    return run


@pytest.mark.parametrize("d", [32, 256, 1024, 2048, 8192, 32768])
def test_norm_launches_stay_within_the_runtimes_limit(launches, d):
    # (the kernel's fourth argument is its number of rows)
    sizes = [1, 1000, 1 << 22, 1 << 24, (1 << 28) + 37, 1 << 31]
    got = launches(f"""
        for M in {sizes}:
            assert L.torq_add_rms_norm(P, None, P, M, {d}, 1e-5, 8, None, P, None, None) == OK
        """, argument=3)
    assert all(grid[0] * threads < 1 << 32 for grid, threads, *_ in got)
    for M in sizes:
        rows = 0
        while rows < M:
            rows += got.pop(0)[2]
        assert rows == M
    assert not got


@gpu
@pytest.mark.parametrize("fmt", [binding.TORQ_FMT_BF16, binding.TORQ_FMT_MXFP8])
def test_norm_of_more_rows_than_one_launch_takes(fmt):
    M, d, step = (1 << 28) + 37, 32, 1 << 25          # 16 rows a workgroup, 2^24 workgroups and some
    weight = (1 + 0.25 * torch.randn(d, device=DEV)).to(BF)
    x = torch.empty((M, d), dtype=BF, device=DEV)
    for i in range(0, M, step):
        x[i:i + step].normal_()
    # the same rows by calls that a launch takes whole
    want = []
    for i in range(0, M, step):
        want.append(binding.torq_add_rms_norm(x[i:i + step], None, weight, 1e-5, fmt)[:2])
    out, scales, _ = binding.torq_add_rms_norm(x, None, weight, 1e-5, fmt, out=x if fmt == binding.TORQ_FMT_BF16 else None)
    for n, (o, s) in enumerate(want):
        rows = slice(n * step, (n + 1) * step)
        assert torch.equal(out[rows].view(torch.uint8), o.view(torch.uint8)), n
        assert s is None or torch.equal(scales[rows].view(torch.uint8), s.view(torch.uint8)), n
    # and the last of them against the formula
    if fmt == binding.TORQ_FMT_MXFP8:
        tail = x[-100:].double()
        y = tail / (tail.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * weight.double()
        unit = 2.0 ** (scales[-100:].view(torch.uint8).double() - 127)
        assert ((out[-100:].double() * unit - y).abs() <= (2.0 ** -4 + 2.0 ** -15) * y.abs() + unit * 2.0 ** -10).all()


@pytest.mark.parametrize("kv_heads,heads,dim", [(1, 1, 8), (1, 24, 64), (1, 40, 256), (4, 8, 128)])
def test_attention_launches_stay_within_the_runtimes_limit(launches, kv_heads, heads, dim):
    # with tables of a page, of 16 tiles and of 32, as many requests as the call takes and about as many as a launch
    got = launches(f"""
        asked = 0
        for width in (1, 32, 64):
            columns = {kv_heads} * -(-({heads} // {kv_heads}) // 16)
            most = min(0x7FFFFFFF // {heads}, 0x7FFFFFFF // (width // 2 + 8) // columns)
            for B in (most, (1 << 24) // columns, (1 << 24) // columns - 1, (1 << 22) + 3):
                cache = binding._KVCacheStruct(P, P, None, None, 10, {kv_heads} * 16 * {dim}, 16 * {dim}, {dim}, 8, {kv_heads}, {dim}, 16)
                need = L.torq_paged_attention_workspace_bytes(C.byref(cache), {heads}, min(B, most), width)
                status = L.torq_paged_attention(C.byref(cache), P, 128, 128, {heads}, P, width, width, P, min(B, most), 1.0, P, P, need, None)
                assert status == OK
        """)
    assert len(got) >= 12 and all(grid[0] * threads < 1 << 32 for grid, threads, *_ in got)


@gpu
def test_attention_of_more_requests_than_one_launch_takes_workgroups():
    # a request's only token, or none: its output is that token's value
    B, pages = (1 << 24) + 5, 3
    cache = binding.KVCache(*(torch.randn((pages, 1, 16, 8), device=DEV).to(BF) for _ in "kv"))
    tables = torch.randint(0, pages, (B, 1), dtype=torch.int32, device=DEV)
    lengths = torch.randint(0, 2, (B,), dtype=torch.int32, device=DEV)
    q = torch.randn((B, 1, 8), dtype=BF, device=DEV)
    got = binding.torq_paged_attention(q, cache, tables, lengths, 1.0)
    assert torch.equal(got[:, 0], cache.v[:, 0, 0][tables[:, 0].long()] * lengths[:, None])


def attention_kernels(launches, cases):
    """The kernel of each call: cases of (kv_heads, heads, head_dim, requests, tokens that the tables hold, format)."""
    return [kernel for _, _, _, kernel in launches(f"""
        for kv, heads, dim, B, tokens, fmt in {cases}:
            cache = binding._KVCacheStruct(P, P, P, P, 10, kv * 16 * dim, 16 * dim, dim, fmt, kv, dim, 16)
            need = L.torq_paged_attention_workspace_bytes(C.byref(cache), heads, B, tokens // 16)
            assert L.torq_paged_attention(C.byref(cache), P, dim, dim, heads, P, tokens // 16, tokens // 16, P, B, 1.0, P, P, need, None) == OK
        """)]


@pytest.mark.parametrize("fmt", [binding.TORQ_FMT_BF16, binding.TORQ_FMT_MXFP8])
def test_waves_with_columns_of_their_own_have_one(launches, fmt):
    # tables for up to 512 tokens: a launch a call.  Where a request has one column the waves take turns at it as they do for a single request,
    # and so they do where the last of them would have none, but for a few in MXFP8 and in the shortest tables of head_dim 256
    mx = fmt == binding.TORQ_FMT_MXFP8
    full, most, half = (4, 8, 16, 20), (3, 7, 15, 18), (2, 5)
    cases = lambda dim, heads, *tokens: [(kv, 8 * kv, dim, 4096, t, fmt) for kv in heads for t in tokens]
    for dim, own, turns in ((64, cases(64, full + most * mx, 64, 128, 256), cases(64, (1,) + half + most * (not mx), 128, 256) + cases(64, full, 288, 512)),
                            (128, cases(128, full + most * mx, 64, 128, 160) + cases(128, full, 256) * mx,
                             cases(128, (1,) + half + most * (not mx), 128, 256) + cases(128, full, 192, 256) * (not mx) + cases(128, full, 288, 512)),
                            (256, cases(256, full + most + half * (not mx), 64, 192) + cases(256, full, 208, 256, 512),
                             cases(256, (1,) + half * mx, 64, 192) + cases(256, (1, 3) + half, 208, 256, 512))):
        single, *kernels = attention_kernels(launches, [(1, 8, dim, 1, 512, fmt)] + turns + own)
        assert kernels[:len(turns)] == [single] * len(turns), dim
        assert set(kernels[len(turns):]) != {single} and len(set(kernels[len(turns):])) == 1, dim


def test_idle_waves_do_not_take_columns_of_mxfp8(launches):
    # 24 query heads of 256 are two columns: for one key head half of the waves would have none
    for kv, B, alone in ((1, 128, False), (1, 512, False), (2, 128, True), (3, 32, False), (3, 128, True), (8, 16, True)):
        single, _, many, _ = attention_kernels(launches, [(1, 8, 256, 1, 4000, 9), (kv, 24 * kv, 256, B, 4000, 9)])
        assert (many != single) == alone, (kv, B)


def test_head_dim_256_has_a_column_a_wave_where_whole_rounds_of_the_cus_do(launches):
    # a CU has one workgroup at a time: half a round would leave half of them without; whether a table has a page to spare says nothing
    cases = [(64, 8, 192, 8, True), (60, 8, 192, 8, False), (64, 8, 208, 8, False), (64, 8, 256, 8, False), (64, 8, 272, 8, False), (128, 8, 256, 8, True),
             (128, 8, 272, 8, True), (128, 8, 512, 8, True), (128, 8, 528, 8, False), (160, 8, 272, 8, False), (256, 8, 272, 8, True), (256, 2, 192, 8, True),
             (256, 2, 256, 8, False), (64, 8, 256, 9, False), (128, 8, 256, 9, True), (136, 8, 272, 9, False)]
    kernels = attention_kernels(launches, [(1, 8, 256, 1, 512, 8), (1, 8, 256, 1, 512, 9)] + [(kv, 4 * kv, 256, B, tokens, fmt) for B, kv, tokens, fmt, _ in cases])
    for (B, kv, tokens, fmt, own), kernel in zip(cases, kernels[2:]):
        assert (kernel != kernels[fmt - 8]) == own, (B, kv, tokens, fmt)


# ---- values at the ends of their types ---------------------------------------------------------

def two_tokens(score, value, dim=64):
    """The output of a token of score 0 and value 1 beside one of that score and value, one launch and in runs."""
    k, v = torch.zeros((1, 1, 16, dim), dtype=BF, device=DEV), torch.ones((1, 1, 16, dim), dtype=BF, device=DEV)
    k[0, 0, 1, 0], v[0, 0, 1] = score, value
    q = torch.zeros((1, 1, dim), dtype=BF, device=DEV)
    q[0, 0, 0] = 1
    two = torch.tensor([2], dtype=torch.int32, device=DEV)
    outs = [binding.torq_paged_attention(q, binding.KVCache(k, v), torch.zeros((1, width), dtype=torch.int32, device=DEV), two, 1.0) for width in (1, 200)]
    assert torch.equal(*outs) or all(torch.isnan(o).all() for o in outs)
    assert (outs[0] == outs[0][0, 0, 0]).all() or torch.isnan(outs[0]).all()
    return float(outs[0][0, 0, 0])


@gpu
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("value", [2.0 ** 100, 2.0 ** 118, 2.0 ** 120, 2.0 ** 127, -2.0 ** 127])
def test_a_weight_of_nothing_leaves_out_values_of_any_size(dim, value):
    # exp(-300) is nothing in 32 bits (and 1e-130 by the formula): the other token's value alone
    assert two_tokens(-300.0, value, dim) == 1.0
    # a weight that is something: p value + 1, to the output's rounding and 2^-16 of the term
    for score in (-40.0, -60.0, -80.0):
        p = 2.718281828459045 ** score
        want, term = (1.0 + p * value) / (1.0 + p), p * abs(value)
        assert abs(two_tokens(score, value, dim) - want) <= 2.0 ** -8 * abs(want) + (2.0 ** -15 + 2.0 ** -17) * term + 2.0 ** -20


@gpu
@pytest.mark.parametrize("score", [0.0, -1.0, -8.0, -40.0, -80.0])
def test_an_infinite_value_stays_infinite_under_any_weight(score):
    # weights with low bits and without (that of score 0 is 1)
    assert two_tokens(score, float("inf")) == float("inf") and two_tokens(score, -float("inf")) == -float("inf")


# ---- counts past 32 bits -----------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("before,B,width", [(2 ** 31 - 5, 1, 1000), (2 ** 31 - 1, 3, 70), (2 ** 30 + 2 ** 29, 520, 1 << 20), (2 ** 31 - 1, 2, 0)])
def test_a_cursor_stays_at_the_end_of_its_type(before, B, width, in_place):
    # pages wanted beyond what 32 bits count: the list has long run out, and says so
    i32 = dict(dtype=torch.int32, device=DEV)
    held, lengths, free, cursor = torch.zeros(B, **i32), torch.full((B,), 2 ** 31 - 1, **i32), torch.arange(9, **i32), torch.full((1,), before, **i32)
    tables = torch.full((B, width), 77, **i32)
    slots, after = binding.torq_block_tables(held, lengths, free, cursor, tables, 16, 40, cursor_out=cursor if in_place else None)
    assert after.tolist() == [min(before + B * width, 2 ** 31 - 1)]
    had = max(0, len(free) - before)
    assert tables.flatten()[:had].tolist() == list(range(before, before + had)) and (tables.flatten()[had:] == -1).all()
    assert slots.tolist() == [((before + i // 16) * 16 + i % 16 if i // 16 < had else -1) for i in range(40)]


def test_workspace_sizes_go_up_and_down_with_requests_and_tables():
    # what the header says of them: a workspace for the largest sizes is not one for all
    need = binding.lib().torq_paged_attention_workspace_bytes
    size = lambda B, width, kv=1, dim=64: need(binding.C.byref(binding._KVCacheStruct(1, 1, None, None, 10, kv * 16 * dim, 16 * dim, dim, 8, kv, dim, 16)), kv, B, width)
    assert size(1, 32) == 0 < size(1, 33) < size(1, 128)                     # a wider table, more
    assert size(16, 63, 8, 128) == size(16, 64, 8, 128) == 0 < size(16, 65, 8, 128)
    assert size(15, 64, 8, 128) > size(16, 64, 8, 128)                       # fewer requests, more
    assert size(1, 65, 8, 128) < size(4, 65, 8, 128) < size(300, 65, 8, 128) <= 66 << 20


@gpu
def test_every_mxfp8_value_as_attention_reads_it():
    # one token a request, whose value is its output: every element under every scale byte, as bf16
    codes, bytes_ = torch.arange(256, dtype=torch.uint8), torch.arange(256, dtype=torch.uint8)
    elements, scales = codes.view(F8).double(), bytes_.view(E8).double()
    want = (scales[:, None] * elements).float().to(BF)                       # (no value has more bits than fp32 holds)
    e = torch.zeros((256, 1, 16, 256), dtype=torch.uint8, device=DEV)
    s = torch.full((256, 1, 16, 8), 127, dtype=torch.uint8, device=DEV)
    v, v_scales = e.clone(), s.clone()
    v[:, 0, 0], v_scales[:, 0, 0] = codes.to(DEV), bytes_[:, None].to(DEV)
    cache = binding.KVCache(e.view(F8), v.view(F8), s.view(E8), v_scales.view(E8))
    got = binding.torq_paged_attention(torch.zeros((256, 1, 256), dtype=BF, device=DEV), cache, torch.arange(256, dtype=torch.int32, device=DEV)[:, None].contiguous(),
                                       torch.ones(256, dtype=torch.int32, device=DEV), 1.0)[:, 0].cpu()
    same = (got == want) | (got.isnan() & want.isnan())
    assert same.all(), [(int(b), int(c), float(got[b, c]), float(want[b, c])) for b, c in (~same).nonzero()[:8]]
    assert float(want[0, 0x78]) == 2.0 ** -119 and want[255].isnan().all() and float(want[3, 1]) == 2.0 ** -133


@gpu
@pytest.mark.parametrize("byte", [0, 1, 2, 3, 60, 127, 200, 254])
def test_keys_under_every_kind_of_scale(byte):
    # keys of 1 and 1/2 times the scale, a query that brings the scores to 1 and 1/2 (byte 0: 2^-127 and 2^-128, which are no normal bf16 values)
    e = torch.zeros((1, 1, 16, 32), dtype=torch.uint8, device=DEV)
    s = torch.full((1, 1, 16, 1), 127, dtype=torch.uint8, device=DEV)
    k, v, k_scales = e.clone(), e.clone(), s.clone()
    k[0, 0, 0, 5], k[0, 0, 1, 5], v[0, 0, 0], v[0, 0, 1], k_scales[0, 0, :2] = 0x38, 0x30, 0x38, 0x40, byte
    q = torch.zeros((1, 1, 32), dtype=BF, device=DEV)
    q[0, 0, 5] = 2.0 ** (127 - byte)
    cache = binding.KVCache(k.view(F8), v.view(F8), k_scales.view(E8), s.view(E8))
    got = binding.torq_paged_attention(q, cache, torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.full((1,), 2, dtype=torch.int32, device=DEV), 1.0)
    p = 1 / (1 + 2.718281828459045 ** -0.5)
    want = p + 2 * (1 - p)
    assert ((got.double() - want).abs() <= (2.0 ** -9 + 2.0 ** -12) * 2 * want).all()
    k_scales[0, 0, 1] = 255
    assert binding.torq_paged_attention(q, cache, torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.full((1,), 2, dtype=torch.int32, device=DEV), 1.0).isnan().all()


@gpu
def test_scores_of_minus_infinity_weigh_nothing():
    assert two_tokens(-float("inf"), 5.0) == 1.0
    k, v = torch.zeros((1, 1, 16, 64), dtype=BF, device=DEV), torch.ones((1, 1, 16, 64), dtype=BF, device=DEV)
    k[..., 3] = -float("inf")
    q = torch.ones((1, 1, 64), dtype=BF, device=DEV)
    for width in (1, 200):
        got = binding.torq_paged_attention(q, binding.KVCache(k, v), torch.zeros((1, width), dtype=torch.int32, device=DEV), torch.full((1,), 9, dtype=torch.int32, device=DEV), 1.0)
        assert not got.any()


@gpu
def test_norm_of_rows_past_fp32():
    # squares whose sum fp32 does not hold; half of that is held
    w = torch.ones(256, dtype=BF, device=DEV)
    x = torch.full((2, 256), 2.0 ** 62, device=DEV).to(BF)
    x[1] = 2.0 ** 59
    out = binding.torq_add_rms_norm(x, None, w, 1e-5)[0].double()
    assert not out[0].any() and ((out[1] - 1).abs() <= 2.0 ** -8 + 2.0 ** -16).all()


# ---- sizes from which another form of a kernel runs --------------------------------------------

@gpu
@pytest.mark.parametrize("M,d,fmt,place", [(8192, 4096, 8, None), (8192, 4096, 9, "residual"), (8192, 4096, 8, "x"), (4099, 8192, 8, "residual"), (250000, 128, 8, None),
                                           (250000, 128, 9, "x"), (500001, 64, 9, None), (65000, 512, 8, "residual"), (1100, 28672, 9, "x"), (2050, 16384, 8, None)])
def test_norm_of_more_than_the_cache_holds(M, d, fmt, place):
    # over 120 MiB of inputs: read, and the residual written, with the non-temporal hint
    assert 4 * M * d > 120 << 20
    x, r, w = (torch.randn((M, d), device=DEV) * 3).to(BF), torch.randn((M, d), device=DEV).to(BF), (1 + 0.2 * torch.randn(d, device=DEV)).to(BF)
    x[:, ::19] *= 20
    a, b = x.clone(), r.clone()
    out, scales, total = binding.torq_add_rms_norm(a, b, w, 1e-5, fmt, residual_out={"x": a, "residual": b, None: None}[place])
    assert place is None or total is (a if place == "x" else b)
    if place != "x":
        assert torch.equal(a, x)
    if place != "residual":
        assert torch.equal(b, r)
    part = 2.0 ** -16                                # fp32's part of y, as of smaller rows
    for i in range(0, M, max(1, (1 << 25) // d)):
        rows = slice(i, i + max(1, (1 << 25) // d))
        s = x[rows].double() + r[rows].double()
        y = s / (s.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * w.double()
        assert ((total[rows].double() - s).abs() <= (2.0 ** -8 + 2.0 ** -23) * s.abs()).all()
        if fmt == binding.TORQ_FMT_BF16:
            assert ((out[rows].double() - y).abs() <= (2.0 ** -8 + part) * y.abs() + 1e-38).all()
            continue
        unit = 2.0 ** (scales[rows].view(torch.uint8).double() - 127)
        amax = y.abs().unflatten(-1, (-1, 32)).amax(-1)
        assert (amax * (1 - part) <= 448 * unit).all() and (amax * (1 + part) > 224 * unit).all()
        unit = unit.repeat_interleave(32, -1)
        assert ((out[rows].double() * unit - y).abs() <= (2.0 ** -4 + 2 * part) * y.abs() + unit * 2.0 ** -10).all()


def check_tables(held, lengths, page, width, before, tokens, pages=None):
    """torq_block_tables against running sums over arrays of the host, in 64 bits."""
    held, lengths = np.asarray(held, dtype=np.int64), np.asarray(lengths, dtype=np.int64)
    B = len(held)
    had, have = np.minimum(-(-held // page), width), np.minimum(-(-lengths // page), width)
    need, new = np.maximum(have - had, 0), np.maximum(lengths - held, 0)
    g = np.random.default_rng(B + page)
    pages = int(need.sum()) + before + 3 if pages is None else pages
    free, tables = g.permutation(pages).astype(np.int32), g.integers(0, pages, (B, width)).astype(np.int32)
    first, want = before + np.cumsum(need) - need, tables.copy()
    for b in np.nonzero(need)[0]:
        at = first[b] + np.arange(need[b])
        want[b, had[b]:have[b]] = np.where(at < pages, free[np.minimum(at, pages - 1)], -1)
    ends = np.cumsum(new)
    token = np.arange(tokens)
    owner = np.minimum(np.searchsorted(ends, token, side="right"), B - 1)
    position = held[owner] + token - (ends - new)[owner]
    entry = want[owner, np.minimum(position // page, max(width - 1, 0))].astype(np.int64)
    slots = np.where((token < ends[-1]) & (position // page < width) & (entry >= 0), entry * page + position % page, -1)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)
    t, cursor = dev(tables), torch.full((1,), before, dtype=torch.int32, device=DEV)
    got, after = binding.torq_block_tables(dev(held), dev(lengths), dev(free), cursor, t, page, tokens)
    assert np.array_equal(t.cpu().numpy(), want) and np.array_equal(got.cpu().numpy(), slots) and after.tolist() == [before + int(need.sum())]


@gpu
@pytest.mark.parametrize("held,lengths,page,width,tokens", [
    ([0, 100, 7, 0], [700000, 500001, 7, 90], 16, 44000, None), ([0, 100, 7, 0], [700000, 500001, 7, 90], 16, 44000, (1 << 20) + 77), ([5] * 3, [1 << 19] * 3, 1, 1 << 19, None),
    ([16, 0], [40, 20], 16, (1 << 20) + 3, None), ([16, 0, 3], [1 << 25, 20, 9], 16, (1 << 20) + 3, 50)])
def test_block_tables_of_more_than_a_million(held, lengths, page, width, tokens):
    # 2^20 tokens or entries of a row: sums in 64 bits
    tokens = int(np.maximum(np.array(lengths) - np.array(held), 0).sum()) if tokens is None else tokens
    assert tokens >= 1 << 20 or width > 1 << 20
    check_tables(held, lengths, page, width, 4, tokens)


@gpu
@pytest.mark.parametrize("B", [1024, 1025, 2500, 7001])
@pytest.mark.parametrize("more", ["one", "two", "first", "second", "third"])
def test_block_tables_of_many_requests_that_go_on_by_a_token(B, more):
    # 1024 requests at a time: entries written by their own lanes, except where one of the 1024 has more than two
    g = np.random.default_rng(B)
    held = g.integers(0, 100, B)
    new = np.full(B, 2 if more == "two" else 1)
    if more in ("first", "second", "third"):
        at = 1024 * ("first", "second", "third").index(more) + 5
        new[at if at < B else B - 1] = 300
        new[g.integers(0, B, B // 9)] = 0
    check_tables(held, held + new, 16, 30, 3, int(new.sum()))
    check_tables(held, held + new, 16, 30, 3, int(new.sum()) + 700, pages=40)
