"""What a served step holds and which of the library's calls it makes (no GPU needed: the calls
are recorded instead of made)."""

import pytest
import torch

from paper_2506_20194_amd import duo, serve

HEADS, KV, HD, D, PAGE = 8, 2, 64, 96, 16


@pytest.fixture()
def calls(duo_lib, monkeypatch):
    """serve.attention without a device: the names and arguments of its calls."""
    made = []
    like = lambda n, w: torch.zeros(n, w, dtype=torch.bfloat16)
    results = dict(
        duo_kv_append=lambda *a, **k: None, duo_linear=lambda x, W, R=None: like(len(x), len(W)), duo_rope_at=lambda X, *a, **k: X,
        duo_head_norm_rope=lambda X, *a, **k: X, duo_kv_read=lambda cache, slots: (like(1, 1), like(1, 1)),
        duo_attention_paged=lambda q, *a, **k: q, duo_attention_chunk=lambda q, *a, **k: q, duo_attention_packed=lambda q, *a, **k: q)
    for name, f in results.items():
        monkeypatch.setattr(duo, name, lambda *a, _n=name, _f=f, **k: made.append((_n, a, k)) or _f(*a, **k))
    return made


def cache_of(fmt="bf16", pages=40):
    return duo.KVCache.empty(pages, PAGE, KV, HD, fmt, "cpu")


def weights(**more):
    W = {nm: torch.zeros(n * HD, D, dtype=torch.bfloat16) for nm, n in (("q", HEADS), ("k", KV), ("v", KV))}
    return {**W, **more}


def attend(cache, step, W=None, **cfg):
    cfg = dict(dict(heads=HEADS, theta=1e4, eps=1e-5), **cfg)
    return serve.attention(torch.zeros(step.m, D, dtype=torch.bfloat16), W or weights(), cfg, cache, step)


@pytest.mark.parametrize("before,new", [([37, 0, 5], [60, 3, 100]), ([1, 1], [2, 300]), ([16, 0], [0, 20])])
def test_whole_sequences_are_those_of_the_table_at_the_start(calls, monkeypatch, before, new):
    """Slots and offsets of the whole sequences belong to the step from its start on: a table that
    is changed afterwards, as for a later step, does not change them, and nothing is
    made of host data inside the block, which may be captured into a graph or run on another stream."""
    monkeypatch.setattr(serve, "MANY_ROWS_16", 0)
    cache = cache_of()
    table = torch.randperm(40, generator=torch.Generator().manual_seed(1))[:len(new) * 20 // len(new) * len(new)].int()
    table = table[:len(new) * (len(table) // len(new))].view(len(new), -1)
    was = table.clone()
    step = serve.Step(cache, table, before, new)
    table.fill_(-1)
    with monkeypatch.context() as m:
        m.setattr(torch, "tensor", lambda *a, **k: pytest.fail("host data inside the block"))
        attend(cache, step)
    (_, (_, slots), _), = [c for c in calls if c[0] == "duo_kv_read"]
    after = [b + n for b, n in zip(before, new)]
    want = [int(was[s, t // PAGE]) * PAGE + t % PAGE for s, n in enumerate(after) for t in range(n)]
    assert slots.dtype == torch.int64 and slots.tolist() == want
    (_, _, k), = [c for c in calls if c[0] == "duo_attention_packed"]
    assert k["cu_k"].dtype == torch.int32 and k["cu_k"].tolist() == [sum(after[:i]) for i in range(len(after) + 1)]


def test_prompts_are_their_own_whole_sequences(calls):
    cache = cache_of()
    step = serve.Step(cache, torch.arange(40, dtype=torch.int32).view(2, 20), [0, 0], [70, 9])
    attend(cache, step)
    assert [c[0] for c in calls if "attention" in c[0] or "read" in c[0]] == ["duo_attention_packed"]
    assert calls[-1][2]["cu_k"] is None and step.all_slots is step.slots


@pytest.mark.parametrize("one", ["q_norm", "k_norm"])
def test_norms_go_together(calls, one):
    """Gains for the heads of queries or of keys alone: which norm the other ones should have is not said."""
    cache = cache_of()
    step = serve.Step(cache, torch.arange(40, dtype=torch.int32).view(1, 40), [0], [5])
    with pytest.raises(ValueError, match="q_norm and k_norm"):
        attend(cache, step, weights(**{one: torch.ones(HD)}))
    assert not calls
    attend(cache, step, weights(q_norm=torch.ones(HD), k_norm=torch.ones(HD)))
    assert calls[3][0] == "duo_kv_append" and calls[3][2]["eps"] == 1e-5


# new tokens and tokens before them, K/V heads, cache: over which rows the attention goes.  Times of both ways on the
# left and right of each (attention over the pages, rows read back), heads of 128, in microseconds.
WAYS = [
    ("int8", 8, [16384 - 64], [64], "packed"),            # 85 and 78
    ("int8", 8, [4096 - 16] * 4, [16] * 4, "packed"),     # 66 and 54
    ("int8", 8, [2048 - 8], [8], "packed"),               # 31 and 27
    ("int4", 8, [4096 - 32], [32], "packed"),             # 50 and 36
    ("int8", 8, [16384 - 4], [4], "chunk"),               # 37 and 56 (16 bits)
    ("int8", 8, [512 - 4] * 8, [4] * 8, "chunk"),         # 26 and 29
    ("int8", 8, [32768 - 32], [32], "chunk"),             # 92 and 99
    ("int8", 8, [8192 - 64] * 4, [64] * 4, "packed"),     # 137 and 126
    ("int8", 8, [65536 - 64], [64], "chunk"),             # 220 and 233
    ("int8", 8, [65536 - 128], [128], "packed"),          # 398 and 351
    ("int4", 32, [16384 - 256] * 4, [256] * 4, "chunk"),  # 412 and 681
    ("int8", 8, [1536] + [999] * 3, [512, 1, 1, 1], "packed"),           # 105 and 59
    ("int8", 8, [7168] + [3999] * 7, [1024] + [1] * 7, "chunk"),         # 333 and 320
    ("int8", 8, [0, 3300] + [5999] * 46, [1024, 700] + [1] * 46, "chunk"),  # 323 and 648
    ("int8", 8, [0, 0], [9, 300], "packed"),
    ("bf16", 8, [2048 - 64], [64], "packed"),             # 41 and 31
    ("bf16", 8, [4096 - 16], [16], "packed"),             # 41 and 33
    ("bf16", 8, [512 - 4] * 8, [4] * 8, "chunk"),         # 24 and 25
    ("bf16", 8, [16384 - 64], [64], "chunk"),             # 71 and 82
    ("bf16", 8, [65536 - 512], [512], "chunk"),           # 1087 and 1235
    ("bf16", 8, [16384 - 2048], [2048], "packed"),        # 1013 and 971
    ("bf16", 8, [768] * 2 + [499] * 14, [256] * 2 + [1] * 14, "packed"),  # 74 and 43
    ("bf16", 8, [0, 0], [9, 300], "packed"),
]


@pytest.mark.parametrize("fmt,kv,before,new,way", WAYS)
def test_ways(calls, fmt, kv, before, new, way):
    """Chunks take the way that is faster for their sizes (64 query heads, or 32 on 32)."""
    heads = 64 if kv == 8 else 32
    after = [b + n for b, n in zip(before, new)]
    cache = duo.KVCache.empty(4, 256, kv, 128, fmt, "cpu")
    step = serve.Step(cache, torch.zeros(len(new), -(-max(after) // 256), dtype=torch.int32), before, new)
    W = {nm: torch.zeros(n * 128, 8, dtype=torch.bfloat16) for nm, n in (("q", heads), ("k", kv), ("v", kv))}
    serve.attention(torch.zeros(step.m, 8, dtype=torch.bfloat16), W, dict(heads=heads, theta=1e4, eps=1e-5), cache, step)
    assert calls[-1][0] == "duo_attention_" + way
