"""Refusals of the paged-cache operators and of sampling: every check runs on the host
before any HIP call, so these need no GPU (the pointers are numbers that are never
followed)."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2608_19889_amd as ops
from paper_2608_19889_amd import axon as ax

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # a "device pointer"
F, B = ax.AXON_F32, ax.AXON_BF16
BIG = 1 << 50
NAN, INF = float("nan"), float("inf")


def ints(*v):
    return (ctypes.c_int32 * len(v))(*v)


PAGES = dict(k=P, v=2 * P, dtype=B, kv_heads=2, head_dim=64, page_size=16, num_pages=9)
BATCH = dict(seqs=3, table_stride=4, d_cu=P, h_cu=ints(0, 2, 2, 6), d_lens=P, d_table=P)
PREFIX = dict(groups=2, table_stride=4, d_cu=P, h_cu=ints(0, 1, 3), d_lens=P, d_table=P)
APPEND = dict(tokens=6, heads=4, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, q_out=2 * P, ldqo=256, inv=P, rot=64,
              interleaved=0, scale=1.0, offsets=P, stream=None)
ATTEND = dict(tokens=6, heads=4, q=P, ldq=256, scale=0.125, out=2 * P, ldo=256, lse=P, ws=P, ws_bytes=BIG, stream=None)
SAMPLE = dict(rows=4, vocab=50, z=P, dtype=F, ld=50, u=P, d_t=None, t=1.0, d_k=None, k=0, d_p=None, p=1.0, d_m=None,
              m=0.0, tokens=P, logps=P, ws=P, ws_bytes=BIG, stream=None)

SHARED_BAD = [  # of both operators on the cache
    ("pages", dict(dtype=3), ax.AXON_E_DTYPE, "the cache must be"),
    ("pages", dict(k=None), ax.AXON_E_INVALID, "key cache is NULL"),
    ("pages", dict(v=P + 8), ax.AXON_E_INVALID, "value cache is not aligned"),
    ("pages", dict(kv_heads=0), ax.AXON_E_INVALID, "kv_heads"),
    ("pages", dict(kv_heads=3), ax.AXON_E_INVALID, "heads"),
    ("pages", dict(head_dim=96), ax.AXON_E_INVALID, "head_dim"),
    ("pages", dict(page_size=8), ax.AXON_E_INVALID, "page_size"),
    ("pages", dict(page_size=24), ax.AXON_E_INVALID, "page_size"),
    ("pages", dict(page_size=0), ax.AXON_E_INVALID, "page_size"),
    ("pages", dict(num_pages=0), ax.AXON_E_INVALID, "num_pages"),
    ("batch", dict(seqs=0), ax.AXON_E_INVALID, "seqs"),
    ("batch", dict(seqs=4097), ax.AXON_E_INVALID, "seqs"),
    ("batch", dict(table_stride=0), ax.AXON_E_CAPACITY, "d_block_table"),
    ("batch", dict(table_stride=1 << 27), ax.AXON_E_CAPACITY, "d_block_table"),
    ("batch", dict(d_table=None), ax.AXON_E_INVALID, "d_block_table is NULL"),
    ("batch", dict(d_lens=None), ax.AXON_E_INVALID, "d_lens"),
    ("batch", dict(d_lens=P + 2), ax.AXON_E_INVALID, "d_lens"),
    ("batch", dict(d_cu=None), ax.AXON_E_INVALID, "d_cu_seqlens"),
    ("batch", dict(h_cu=None), ax.AXON_E_INVALID, "h_cu_seqlens"),
    ("batch", dict(h_cu=ints(1, 2, 2, 6)), ax.AXON_E_INVALID, r"cu_seqlens\[0\]"),
    ("batch", dict(h_cu=ints(0, 3, 2, 6)), ax.AXON_E_INVALID, "falls at entry 2"),
    ("batch", dict(h_cu=ints(0, 2, 2, 7)), ax.AXON_E_INVALID, "end at 7"),
    ("batch", dict(d_cu=None, h_cu=None), ax.AXON_E_INVALID, "6 tokens for 3 sequences"),
    ("call", dict(tokens=-1), ax.AXON_E_INVALID, "tokens"),
    ("call", dict(tokens=(1 << 30) + 1), ax.AXON_E_INVALID, "tokens"),
    ("call", dict(heads=3), ax.AXON_E_INVALID, "heads"),
    ("call", dict(heads=-2), ax.AXON_E_INVALID, "heads"),
    ("call", dict(heads=4098), ax.AXON_E_INVALID, "heads"),
    ("call", dict(q=None), ax.AXON_E_INVALID, "q is NULL"),
    ("call", dict(q=P + 1), ax.AXON_E_INVALID, "q is not aligned"),
    ("call", dict(ldq=255), ax.AXON_E_INVALID, "stride of q"),
    ("call", dict(scale=NAN), ax.AXON_E_INVALID, "scale"),
    ("call", dict(scale=INF), ax.AXON_E_INVALID, "scale"),
]
APPEND_BAD = [
    ("call", dict(k=None), ax.AXON_E_INVALID, "k is NULL"),
    ("call", dict(v=P + 1), ax.AXON_E_INVALID, "v is not aligned"),
    ("call", dict(ldk=127), ax.AXON_E_INVALID, "stride of k"),
    ("call", dict(ldv=0), ax.AXON_E_INVALID, "stride of v"),
    ("call", dict(q_out=None), ax.AXON_E_INVALID, "q_out is NULL"),
    ("call", dict(ldqo=10), ax.AXON_E_INVALID, "stride of q_out"),
    ("call", dict(q_out=P, ldqo=300), ax.AXON_E_INVALID, "q's buffer"),
    ("call", dict(rot=63), ax.AXON_E_INVALID, "rot"),
    ("call", dict(rot=66), ax.AXON_E_INVALID, "rot"),
    ("call", dict(rot=-2), ax.AXON_E_INVALID, "rot"),
    ("call", dict(inv=None), ax.AXON_E_INVALID, "d_inv_freq"),
    ("call", dict(inv=P + 4), ax.AXON_E_INVALID, "d_inv_freq"),
    ("call", dict(interleaved=2), ax.AXON_E_INVALID, "interleaved"),
    ("call", dict(offsets=P + 1), ax.AXON_E_INVALID, "d_offsets"),
]
ATTEND_BAD = [
    ("call", dict(heads=0), ax.AXON_E_INVALID, "heads"),
    ("call", dict(out=None), ax.AXON_E_INVALID, "out is NULL"),
    ("call", dict(ldo=255), ax.AXON_E_INVALID, "stride of out"),
    ("call", dict(out=P, ldo=300), ax.AXON_E_INVALID, "q's buffer"),
    ("call", dict(lse=P + 2), ax.AXON_E_INVALID, "d_lse"),
    ("batch", dict(table_stride=(1 << 30) // PAGES["page_size"]), ax.AXON_E_CAPACITY, "too many for one call"),
    ("prefix", dict(groups=-1), ax.AXON_E_INVALID, "groups"),
    ("prefix", dict(groups=4097), ax.AXON_E_INVALID, "groups"),
    ("prefix", dict(table_stride=0), ax.AXON_E_CAPACITY, "d_prefix_table"),
    ("prefix", dict(d_table=None), ax.AXON_E_INVALID, "d_prefix_table"),
    ("prefix", dict(d_lens=None), ax.AXON_E_INVALID, "d_prefix_lens"),
    ("prefix", dict(d_cu=None), ax.AXON_E_INVALID, "d_cu_groups"),
    ("prefix", dict(h_cu=None), ax.AXON_E_INVALID, "h_cu_groups"),
    ("prefix", dict(h_cu=ints(0, 1, 4)), ax.AXON_E_INVALID, "cu_groups end at 4"),
    ("prefix", dict(h_cu=ints(0, 2, 1)), ax.AXON_E_INVALID, "cu_groups falls"),
]
SAMPLE_BAD = [
    (dict(rows=-1), ax.AXON_E_INVALID, "rows"),
    (dict(rows=65536), ax.AXON_E_INVALID, "rows"),
    (dict(vocab=0), ax.AXON_E_INVALID, "vocab"),
    (dict(vocab=(1 << 22) + 1, ld=1 << 23), ax.AXON_E_INVALID, "vocab"),
    (dict(z=None), ax.AXON_E_INVALID, "logits is NULL"),
    (dict(z=P + 2), ax.AXON_E_INVALID, "logits is not aligned"),
    (dict(dtype=0), ax.AXON_E_DTYPE, "logits"),
    (dict(ld=49), ax.AXON_E_INVALID, "stride of logits"),
    (dict(u=None), ax.AXON_E_INVALID, "d_uniform"),
    (dict(t=-0.5), ax.AXON_E_INVALID, "temperature"),
    (dict(t=NAN), ax.AXON_E_INVALID, "temperature"),
    (dict(d_t=P + 1), ax.AXON_E_INVALID, "d_temperature"),
    (dict(k=-1), ax.AXON_E_INVALID, "top_k"),
    (dict(d_k=P + 2), ax.AXON_E_INVALID, "d_top_k"),
    (dict(p=0.0), ax.AXON_E_INVALID, "top_p"),
    (dict(p=1.5), ax.AXON_E_INVALID, "top_p"),
    (dict(p=NAN), ax.AXON_E_INVALID, "top_p"),
    (dict(d_p=P + 2), ax.AXON_E_INVALID, "d_top_p"),
    (dict(m=-0.1), ax.AXON_E_INVALID, "min_p"),
    (dict(m=1.1), ax.AXON_E_INVALID, "min_p"),
    (dict(d_m=P + 3), ax.AXON_E_INVALID, "d_min_p"),
    (dict(tokens=None), ax.AXON_E_INVALID, "d_tokens"),
    (dict(logps=None), ax.AXON_E_INVALID, "d_logps"),
]


def structures(where, change):
    s = {"pages": dict(PAGES), "batch": dict(BATCH), "prefix": dict(PREFIX)}
    if where in s:
        s[where].update(change)
    return [t(*s[n].values()) for t, n in ((ax.AxonKvPages, "pages"), (ax.AxonKvBatch, "batch"),
                                           (ax.AxonKvPrefix, "prefix"))]


def refused(status, code, text):
    with pytest.raises(ax.AxonError, match=text) as e:
        ax._check(status)
    assert e.value.code == code


@pytest.mark.parametrize("where,change,code,text", SHARED_BAD + APPEND_BAD)
def test_append_refusals(where, change, code, text):
    pages, batch, _ = structures(where, change)
    call = {**APPEND, **(change if where == "call" else {})}
    refused(ax.lib().axon_rope_append(pages, batch, *call.values()), code, text)


@pytest.mark.parametrize("where,change,code,text", SHARED_BAD + ATTEND_BAD)
def test_attention_refusals(where, change, code, text):
    pages, batch, prefix = structures(where, change)
    call = {**ATTEND, **(change if where == "call" else {})}
    refused(ax.lib().axon_prefix_attention(pages, batch, prefix, *call.values()), code, text)


def test_missing_structures_are_refused():
    pages, batch, prefix = structures("", {})
    L = ax.lib()
    refused(L.axon_rope_append(None, batch, *APPEND.values()), ax.AXON_E_INVALID, "pages is NULL")
    refused(L.axon_rope_append(pages, None, *APPEND.values()), ax.AXON_E_INVALID, "batch is NULL")
    refused(L.axon_prefix_attention(None, batch, prefix, *ATTEND.values()), ax.AXON_E_INVALID, "pages is NULL")
    refused(L.axon_prefix_attention(pages, None, prefix, *ATTEND.values()), ax.AXON_E_INVALID, "batch is NULL")
    for args in ((None, batch, prefix), (pages, None, prefix)):
        assert L.axon_prefix_attention_workspace(*args, 6, 4) == 0


@pytest.mark.parametrize("change,code,text", SAMPLE_BAD)
def test_sample_refusals(change, code, text):
    refused(ax.lib().axon_sample_tokens(*{**SAMPLE, **change}.values()), code, text)


def large_call(tokens, heads, kv, hd, keys, groups=0, cu=None, page=16, prefix_keys=None):
    """(workspace, the refusal of a call with no workspace): ``groups`` even groups of the sequences"""
    seqs = tokens if cu is None else len(cu) - 1
    host = None if cu is None else ints(*cu)
    pages = ax.AxonKvPages(P, 2 * P, B, kv, hd, page, 1 << 20)
    batch = ax.AxonKvBatch(seqs, -(-keys // page), None if cu is None else P, host, P, P)
    sums = ints(*(i * seqs // max(groups, 1) for i in range(groups + 1)))
    shared = ax.AxonKvPrefix(groups, -(-(prefix_keys or keys) // page), P, sums, P, P) if groups else None
    L = ax.lib()
    need = L.axon_prefix_attention_workspace(pages, batch, shared, tokens, heads)
    with pytest.raises(ax.AxonError) as e:
        ax._check(L.axon_prefix_attention(pages, batch, shared, tokens, heads, P, heads * hd, 1.0, P, heads * hd, None,
                                          None, BIG, None))
    return need, e.value


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads", [8, 128, 256, 320, 512, 4096])
@pytest.mark.parametrize("groups", [0, 1, 100, 4096])
def test_the_documented_sizes_are_taken(groups, heads, hd):
    """4096 single tokens of any heads over 8 kv heads and tables of 2^18 keys."""
    need, e = large_call(4096, heads, 8, hd, 1 << 18, groups)
    assert 0 < need < 1 << 39 and e.code == ax.AXON_E_INVALID and "workspace is NULL" in str(e)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("groups", [0, 1])
def test_a_long_prompt_is_taken(groups, hd):
    need, e = large_call(200000, 64, 8, hd, 200000, groups, cu=[0, 200000], prefix_keys=1 << 20)
    assert 0 < need < 1 << 39 and e.code == ax.AXON_E_INVALID and "workspace is NULL" in str(e)
    # many rows over short tables, few over a long one
    need, e = large_call(4096, 64, 8, hd, 64, 1, prefix_keys=1 << 23)
    assert need > 0 and e.code == ax.AXON_E_INVALID and "workspace is NULL" in str(e)


def test_a_call_too_large_is_refused_before_its_workspace():
    for call in (dict(tokens=6, heads=4, kv=2, hd=64, keys=1 << 30, cu=[0, 2, 2, 6]),
                 dict(tokens=4096, heads=1024, kv=1024, hd=64, keys=1 << 20),
                 dict(tokens=1 << 30, heads=4096, kv=1024, hd=128, keys=1 << 16, cu=[0, 1 << 30])):
        need, e = large_call(**call)
        assert need == 0 and e.code == ax.AXON_E_CAPACITY and "too many for one call" in str(e), call


def test_binding_refuses_what_it_cannot_hand_over():
    x = torch.zeros(4, 8)
    i = torch.zeros(4, 1, dtype=torch.int32)
    for call in (lambda: ops.sample_tokens(x, x[0]), lambda: ops.prefix_attention(x, x, x, i, i),
                 lambda: ops.rope_append(None, x, x, x, x, i, i, stream=0)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()


def test_binding_layouts(monkeypatch):
    """Shapes that the structures cannot express, before anything is handed over."""
    k = torch.zeros(6, 2, 64)
    cache = torch.zeros(9, 2, 16, 64)
    with pytest.raises(ValueError, match="must be"):
        ax._head_rows(k, 3, 64, torch.float32, "k")
    with pytest.raises(ValueError, match="must be"):
        ax._head_rows(k[0], None, 64, torch.float32, "k")
    with pytest.raises(ValueError, match="must be"):
        ax._head_rows(k, 2, 64, torch.bfloat16, "k")
    fused = torch.zeros(6, 5, 64)
    t, ld = ax._head_rows(fused[:, 1:3], 2, 64, torch.float32, "k")
    assert t.data_ptr() == fused[:, 1:].data_ptr() and ld == 5 * 64
    other = torch.zeros(2, 6, 64).transpose(0, 1)
    t, ld = ax._head_rows(other, 2, 64, torch.float32, "k")
    assert t.is_contiguous() and ld == 128
    with pytest.raises(ValueError, match="contiguous heads"):
        ax._head_rows(other, 2, 64, torch.float32, "out", out=True)
    with pytest.raises(ValueError, match="contiguous heads"):
        ax._head_rows(k[:1].expand(6, 2, 64), 2, 64, torch.float32, "out", out=True)
    with pytest.raises(ValueError, match="one type"):
        ax._pages_arg(cache, cache.bfloat16())
    with pytest.raises(ValueError, match="one type"):
        ax._pages_arg(cache, cache[1:])
    with pytest.raises(ValueError, match="contiguous"):
        ax._pages_arg(cache.transpose(1, 2), cache.transpose(1, 2))
    with pytest.raises(ValueError, match="float32"):
        ax._pages_arg(cache.half(), cache.half())
    with pytest.raises(ValueError, match="int32"):
        ax._table(torch.zeros(3, 2), torch.zeros(3, dtype=torch.int32), "block_table", "lens")
    with pytest.raises(ValueError, match="lens must hold 3"):
        ax._table(torch.zeros(3, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), "block_table", "lens")
    with pytest.raises(ValueError, match="must have 4 entries"):
        ax._sums([0, 1], None, 3, "cu_seqlens", k)
    with pytest.raises(ValueError, match="top_k must hold"):
        ax._setting(torch.zeros(4), 4, torch.int32, "top_k")


@pytest.mark.parametrize("k,taken", [(0, 0), (7, 7), ((1 << 31) - 1, (1 << 31) - 1), (1 << 31, (1 << 31) - 1),
                                     ((1 << 32) + 5, (1 << 31) - 1), ((1 << 63) - 1, (1 << 31) - 1),
                                     (-1, -1), (-(1 << 32), -(1 << 31)), (5 - (1 << 32), -(1 << 31))])
def test_top_k_past_32_bits_keeps_its_meaning(k, taken):
    """All are kept, or the call refused: not the number that the low 32 bits make."""
    assert ax._setting(k, 4, torch.int32, "top_k") == (None, taken)
    if k < 0:
        call = {**SAMPLE, "k": ax._setting(k, 4, torch.int32, "top_k")[1]}
        refused(ax.lib().axon_sample_tokens(*call.values()), ax.AXON_E_INVALID, "top_k must be >= 0")


def test_structures_match_the_c_compiler(tmp_path):
    names = {"axon_kv_pages": ax.AxonKvPages, "axon_kv_batch": ax.AxonKvBatch, "axon_kv_prefix": ax.AxonKvPrefix}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "axon.h"', "int main(void) {"]
    for st, cls in names.items():
        lines.append(f'  printf("{st} size %zu\\n", sizeof({st}));')
        lines += [f'  printf("{st} {n} %zu\\n", offsetof({st}, {n}));' for n, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["  return 0;\n}"]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    got = {tuple(x.split()[:2]): int(x.split()[2]) for x in out.splitlines()}
    for st, cls in names.items():
        assert got[(st, "size")] == ctypes.sizeof(cls)
        for n, _ in cls._fields_:
            assert got[(st, n)] == getattr(cls, n).offset


def test_docstrings_say_that_autograd_sees_nothing():
    for f in (ops.rope_append, ops.prefix_attention, ops.sample_tokens):
        assert "autograd" in f.__doc__ and "``stream``" in f.__doc__
