"""What the binding of the paged-cache calls and of the log probabilities refuses, and what it hands on.  The library calls
themselves are replaced; nothing here needs a GPU."""
import ctypes
import gc
import os
import subprocess
import sys
from dataclasses import replace

import pytest
import torch

from paper_2511_17560_b200 import a3
from paper_2511_17560_b200 import workloads as W
from tests import paged_reference as R


@pytest.fixture
def eng(monkeypatch):
    """An engine on the CPU whose library calls only note what they are given."""
    a3._load()
    calls, kept = [], []

    def replace_call(name, packed):
        def note(h, cache, fields, stream):
            calls.append(packed.unpack(ctypes.string_at(fields, packed.size)))
            return 0

        put(name, note, ctypes.c_int, 4 if packed is not R.LOGIT_ROWS else 3)

    def put(name, fn, result, n, *rest):
        f = fn if n != 3 else lambda h, fields, stream: fn(h, None, fields, stream)
        kept.append(ctypes.CFUNCTYPE(result, *[ctypes.c_void_p] * n, *rest)(f))
        monkeypatch.setitem(a3._entry, name, ctypes.cast(kept[-1], ctypes.c_void_p).value)

    for name, packed in [("a3_paged_append", R.PAGED_ROWS), ("a3_paged_attention", R.PAGED_QUERIES), ("a3_token_logprobs", R.LOGIT_ROWS)]:
        replace_call(name, packed)
    put("a3_paged_attention_workspace_bytes", lambda h, cache, n_seqs, max_pages: 512 if n_seqs > 1 else 0, ctypes.c_size_t, 2, ctypes.c_int, ctypes.c_int)
    monkeypatch.setattr(a3, "_stream", lambda: 0)
    e = a3.A3.__new__(a3.A3)
    e.shape, e._h, e._ws, e.device = replace(W.TINY, n_q_heads=4, n_kv_heads=2), ctypes.c_void_p(), None, torch.device("cpu")
    e.calls, e.kept = calls, kept
    return e


def pages(dtype=torch.bfloat16, n=3, size=16, heads=2, d=64):
    return torch.zeros((n, size, heads, d), dtype=torch.uint8 if dtype == torch.float8_e4m3fn else dtype).view(dtype)


def i32(*x):
    return torch.tensor(x, dtype=torch.int32)


def refused(call, *args, **kw):
    with pytest.raises(a3.A3Error) as e:
        call(*args, **kw)
    assert e.value.status == -1


def test_cache_layouts():
    k = pages()
    c = a3.PagedCache(k, pages())
    assert (c.desc.page_stride, c.desc.n_pages, c.desc.page_size, c.desc.type) == (16 * 2 * 64 * 2, 3, 16, 0)
    both = torch.zeros((3, 2, 16, 2, 64), dtype=torch.bfloat16)
    assert a3.PagedCache(both[:, 0], both[:, 1]).desc.page_stride == 2 * 16 * 2 * 64 * 2
    s, f8 = torch.ones(2), torch.float8_e4m3fn
    c = a3.PagedCache(pages(f8), pages(f8), s, s)
    assert (c.desc.page_stride, c.desc.type) == (16 * 2 * 64, 1)
    for args in [(k, pages(n=4)), (k, pages(torch.float16)), (pages(torch.float16),) * 2, (k, k, s, s), (pages(f8), pages(f8)), (pages(f8), pages(f8), s, None),
                 (pages(f8), pages(f8), s, torch.ones(3)), (pages(f8), pages(f8), s, s.double()), (k[:, ::2], k[:, ::2]), (k[0], k[0]),
                 (k.transpose(1, 2),) * 2, (k, both[:, 0]), (k[:0], k[:0])]:
        refused(a3.PagedCache, *args)


def test_append_arguments(eng):
    cache, table = a3.PagedCache(pages(), pages()), torch.zeros((2, 2), dtype=torch.int32)
    wide = torch.zeros((5, 8, 64), dtype=torch.bfloat16)
    q, k, v, seq = wide[:, :4], wide[:, 4:6], wide[:, 6:], i32(0, 0, 1, 1, -1)
    out = eng.paged_append(cache, table, seq, seq, k, v, q_rows=q)
    args = eng.calls[-1]
    assert out.shape == (5, 4, 64) and out.is_contiguous()
    assert args == (table.data_ptr(), seq.data_ptr(), seq.data_ptr(), 0, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), 512, 512, 512, 256,
                    2, 2, 5, 1)
    assert eng.paged_append(cache, table, seq, seq, k, v, rotate=False) is None
    assert eng.calls[-1][4] == eng.calls[-1][7] == 0 and eng.calls[-1][15] == 0
    eng.paged_append(cache, table, seq[:1], seq[:1], k[:1], v[:1], q_rows=q[:1])
    assert eng.calls[-1][8:12] == (256, 128, 128, 256) and eng.calls[-1][14] == 1
    calls = len(eng.calls)
    flat = torch.zeros((5, 64, 2), dtype=torch.bfloat16).transpose(1, 2)
    for kw in [dict(page_table=table.long()), dict(page_table=table[0]), dict(page_table=torch.zeros((2, 4), dtype=torch.int32)[:, ::2]), dict(row_seq=seq[:4]), dict(row_seq=seq.long()), dict(row_slot=seq[::2]),
               dict(row_pos=seq[:2]), dict(row_pos=seq.float()), dict(k_rows=k.float()), dict(k_rows=k[:4]), dict(k_rows=flat), dict(v_rows=q),
               dict(v_rows=v[..., :32]), dict(q_rows=k), dict(k_rows=k.flatten(1)), dict(v_rows=v[0]), dict(q_rows=q.flatten(1)), dict(q_rows=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(q_rows=None, q_out=out), dict(q_out=out.float()), dict(q_out=out[:4]),
               dict(cache=a3.PagedCache(pages(heads=4), pages(heads=4))), dict(cache=a3.PagedCache(pages(d=128), pages(d=128)))]:
        refused(eng.paged_append, **{**dict(cache=cache, page_table=table, row_seq=seq, row_slot=seq, k_rows=k, v_rows=v, q_rows=q), **kw})
    assert len(eng.calls) == calls


def test_attention_arguments(eng):
    cache, table, lens = a3.PagedCache(pages(), pages()), torch.zeros((3, 2), dtype=torch.int32), i32(5, 0, 32)
    q = torch.zeros((3, 6, 64), dtype=torch.bfloat16)[:, 1:5]
    out, lse = eng.paged_attention(cache, table, lens, q, want_lse=True)
    args = eng.calls[-1]
    assert out.shape == (3, 4, 64) and lse.shape == (3, 4) and lse.dtype == torch.float32
    assert args[:5] == (table.data_ptr(), lens.data_ptr(), q.data_ptr(), out.data_ptr(), lse.data_ptr()) and args[6:10] == (512, 384, 3, 2)
    assert abs(args[10] - 64 ** -0.5) < 1e-8
    given = torch.empty((3, 4, 64), dtype=torch.bfloat16)
    out, lse = eng.paged_attention(cache, table, lens, q, scale=0.5, out=given)
    assert out is given and lse is None and eng.calls[-1][10] == 0.5 and eng.calls[-1][4] == 0
    eng.paged_attention(cache, table[:1], lens[:1], q[:1])
    assert eng.calls[-1][5:7] == (0, 0)  # no workspace where none is needed
    calls = len(eng.calls)
    for kw in [dict(cache_len=lens[:2]), dict(cache_len=lens.long()), dict(cache_len=lens[None]), dict(page_table=table.long()), dict(page_table=table[:2]),
               dict(q_rows=q.float()), dict(q_rows=q.flatten(1)), dict(q_rows=q[:2]), dict(q_rows=q[:, :2]), dict(q_rows=q[..., :32]), dict(out=given[:2]), dict(out=given.float()),
               dict(cache=a3.PagedCache(pages(heads=1), pages(heads=1)))]:
        refused(eng.paged_attention, **{**dict(cache=cache, page_table=table, cache_len=lens, q_rows=q), **kw})
    assert len(eng.calls) == calls


def test_logprob_arguments(eng):
    x = torch.zeros((3, 80), dtype=torch.bfloat16)
    logprob, entropy, ids, lps = eng.token_logprobs(x[:, 1:70], i32(0, 1, -1), 4)
    assert logprob.shape == entropy.shape == (3,) and ids.shape == lps.shape == (3, 4) and ids.dtype == torch.int32
    assert eng.calls[-1][6:] == (80, 1, 3, 69, 4)
    logprob, entropy, ids, lps = eng.token_logprobs(x)
    assert logprob is ids is lps is None and eng.calls[-1][1:3] == (0, 0) and eng.calls[-1][4:6] == (0, 0) and eng.calls[-1][10] == 0
    calls = len(eng.calls)
    for args in [(x[0],), (x.double(),), (x.t(),), (x[:, ::2],), (x[:, :0],), (x, i32(0, 1)), (x, i32(0, 1, 2).long()), (x, i32(0, 1, 2)[None])]:
        refused(eng.token_logprobs, *args)
    assert len(eng.calls) == calls


def test_arguments_of_other_kinds_and_statuses(eng, monkeypatch):
    cache, table, lens = a3.PagedCache(pages(), pages()), torch.zeros((3, 2), dtype=torch.int32), i32(5, 0, 32)
    q, x = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 80))
    for bad in (None, 3, "x", [1, 2, 3], x.numpy()):
        refused(eng.paged_append, cache, table, bad, lens, q[:, :2], q[:, 2:])
        refused(eng.paged_append, cache, table, lens, lens, bad, q[:, 2:])
        refused(eng.paged_attention, cache, bad, lens, q)
        refused(eng.paged_attention, cache, table, lens, bad)
        refused(eng.token_logprobs, bad)
        if bad is not None:
            refused(eng.paged_append, cache, table, lens, lens, q[:, :2], q[:, 2:], row_pos=bad)
            refused(eng.paged_append, cache, table, lens, lens, q[:, :2], q[:, 2:], q_rows=bad)
            refused(eng.paged_attention, cache, table, lens, q, out=bad)
            refused(eng.token_logprobs, x, bad)
    refused(eng.token_logprobs, x, None, 1 << 31)
    for n in ("x", 1 << 70):
        with pytest.raises((TypeError, OverflowError)):
            eng.token_logprobs(x, None, n)
    with pytest.raises(TypeError):
        eng.paged_attention(cache, table, lens, q, scale="x")
    refused(eng.paged_append, cache, table.to_sparse(), lens, lens, q[:, :2], q[:, 2:])
    assert eng.calls == []
    fails = ctypes.CFUNCTYPE(ctypes.c_int, *[ctypes.c_void_p] * 4)(lambda *a: -3)
    monkeypatch.setitem(a3._entry, "a3_paged_attention", ctypes.cast(fails, ctypes.c_void_p).value)
    with pytest.raises(a3.A3Error) as e:
        eng.paged_attention(cache, table, lens, q)
    assert e.value.status == -3 and "a3_paged_attention" in str(e.value)


def test_results_are_the_callers_alone(eng):
    """No tensor outlives its last use, and none is freed before: counted on tensors that the calls allocate and on those that they are given."""
    cache, table, lens = a3.PagedCache(pages(), pages()), torch.zeros((3, 2), dtype=torch.int32), i32(5, 0, 32)
    q, x = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 80))
    given = torch.empty_like(q)
    before = [sys.getrefcount(o) for o in (table, lens, q, x, given)]
    for _ in range(50):
        out, lse = eng.paged_attention(cache, table, lens, q, want_lse=True)
        assert sys.getrefcount(out) == sys.getrefcount(lse) == 2
        assert eng.paged_attention(cache, table, lens, q, out=given)[0] is given
        assert eng.paged_append(cache, table, lens, lens, q[:, :2], q[:, 2:], q_rows=q, q_out=given) is given
        assert all(sys.getrefcount(o) == 2 + 1 for o in eng.token_logprobs(x, lens, 4))  # the list's iterator holds it too
        refused(eng.paged_attention, cache, table, lens, x)
    del out, lse
    gc.collect()  # frames of the refusals
    assert before == [sys.getrefcount(o) for o in (table, lens, q, x, given)]


def test_structs_match_the_header(tmp_path):
    """The packed forms have the header's size and order: each field's place as the C compiler sees it."""
    fields = {"a3_paged_rows": ("page_table row_seq row_slot row_pos q_rows k_rows v_rows q_out q_stride k_stride v_stride q_out_stride n_seqs max_pages M "
                                "rotate", R.PAGED_ROWS),
              "a3_paged_queries": ("page_table cache_len q_rows out lse_out ws ws_bytes q_stride n_seqs max_pages scale reserved", R.PAGED_QUERIES),
              "a3_logit_rows": ("logits targets logprob_out entropy_out top_ids_out top_logprobs_out row_stride type M vocab n_top", R.LOGIT_ROWS)}
    lines = ['printf("%zu\\n", sizeof(a3_paged_cache));'] + [f'printf("%zu\\n", offsetof(a3_paged_cache, {f}));' for f, _ in a3.PagedCacheDesc._fields_]
    want = [ctypes.sizeof(a3.PagedCacheDesc)] + [getattr(a3.PagedCacheDesc, f).offset for f, _ in a3.PagedCacheDesc._fields_]
    for name, (names, packed) in fields.items():
        lines += [f'printf("%zu\\n", sizeof({name}));'] + [f'printf("%zu\\n", offsetof({name}, {f}));' for f in names.split()]
        # the place of a field is where the only byte that is not zero lies
        want.append(packed.size)
        for i in range(len(names.split())):
            values = [0] * len(names.split())
            values[i] = 1
            data = packed.pack(*values)
            at = next(k for k, b in enumerate(data) if b)
            want.append(at // 4 * 4)
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "a3.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-std=c99", "-I", inc, str(src), "-o", str(exe)], check=True)
    assert [int(s) for s in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == want


def test_null_handles():
    lib = a3._load()
    assert lib.a3_paged_attention_workspace_bytes(None, None, 1, 1) == 0
    assert lib.a3_paged_append(None, None, None, None) == -1
    assert lib.a3_paged_attention(None, None, None, None) == -1
    assert lib.a3_token_logprobs(None, None, None) == -1


@pytest.mark.parametrize("spoil,message", [("sys.modules['paper_2511_17560_b200.a3_calls'] = None", "missing or made for another torch"),
                                           ("torch.__version__ = '2.0.0+other'", "is made for torch")])
def test_the_rest_of_the_binding_needs_no_compiled_calls(spoil, message):
    """Without a3_calls.so, or with one made for another torch, everything but the decoding calls works; those say what is wrong."""
    code = f"""
import sys
import torch
{spoil}
from paper_2511_17560_b200 import a3
assert a3.recompute_count(0.5, 10, 10) > 0 and a3.launch_count() == 0
e = a3.A3.__new__(a3.A3)
e._h, e.device, e._ws = a3.C.c_void_p(), torch.device("cpu"), None
for _ in range(2):
    try:
        e.token_logprobs(torch.zeros((3, 80)))
    except ImportError as error:
        assert {message!r} in str(error) and "paper_2511_17560_b200.build" in str(error), error
    else:
        raise AssertionError("no ImportError")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", code], cwd=root, check=True)


def test_compiled_calls_are_made_anew_for_another_torch(monkeypatch, tmp_path):
    from paper_2511_17560_b200 import build

    stamp = tmp_path / "torch"
    monkeypatch.setattr(build, "CALLS_FOR", str(stamp))
    monkeypatch.setattr(build, "_stale", lambda target, deps: False)
    assert build.calls_stale()
    stamp.write_text(str(torch.__version__))
    assert not build.calls_stale()
    monkeypatch.setattr(torch, "__version__", "2.0.0+other")
    assert build.calls_stale()


def test_cache_of_single_pages_entries_and_heads():
    """Where there is one page, one entry or one KV head, the stride of that dimension says nothing about where elements lie."""
    bf = torch.bfloat16
    one_head = torch.zeros((3, 1, 16, 64), dtype=bf).transpose(1, 2)  # [3][16][1][64]
    assert one_head.stride() == (1024, 64, 1024, 1)
    c = a3.PagedCache(one_head, pages(heads=1))
    assert (c.desc.page_stride, c.n_kv_heads, c.page_size) == (16 * 64 * 2, 1, 16)
    one_entry = torch.zeros((3, 2, 1, 64), dtype=bf).transpose(1, 2)  # [3][1][2][64]
    assert a3.PagedCache(one_entry, pages(size=1)).desc.page_stride == 2 * 64 * 2
    apart = torch.zeros((4, 2, 16, 2, 64), dtype=bf)
    assert a3.PagedCache(apart[:1, 0], pages(n=1)).desc.page_stride == 16 * 2 * 64 * 2  # no second page to be apart from
    for k, v in [(apart[:, 0], pages(n=4)), (pages().transpose(1, 2).contiguous().transpose(1, 2), pages())]:
        refused(a3.PagedCache, k, v)


def test_more_alternatives_than_there_can_be_are_refused_before_anything_is_allocated(eng, monkeypatch):
    """n_top beyond what the library takes goes to the library, whose status it is, without results of that size."""
    given = []

    def refuses(h, fields, stream):
        given.append(R.LOGIT_ROWS.unpack(ctypes.string_at(fields, R.LOGIT_ROWS.size)))
        return -2

    f = ctypes.CFUNCTYPE(ctypes.c_int, *[ctypes.c_void_p] * 3)(refuses)
    monkeypatch.setitem(a3._entry, "a3_token_logprobs", ctypes.cast(f, ctypes.c_void_p).value)
    x = torch.zeros((4096, 8))
    for n in (33, (1 << 31) - 1):  # 2^43 elements
        with pytest.raises(a3.A3Error) as e:
            eng.token_logprobs(x, None, n)
        assert e.value.status == -2 and given[-1][-1] == n and given[-1][4:6] == (0, 0)
