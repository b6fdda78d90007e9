"""Decode with drafted tokens over a 4-bit cache, end to end: pages and rows from the device's lengths, append, attention, penalties,
verification, step after step; and one such step captured and replayed."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from paper_2505_21889_b200 import drafted

pytestmark = pytest.mark.gpu


def _prompts(users, vocab, seed):
    rng = np.random.default_rng(seed)
    return [np.tile(rng.integers(0, vocab, 9), 6)[:n].tolist() for n in rng.integers(17, 54, users)]


@pytest.mark.parametrize("temperature", [0.0, 0.8])
@pytest.mark.parametrize("drafts", [0, 1, 4, 9])
def test_generated_text_and_cache(drafts, temperature):
    """What the steps leave is what one pass over the generated text gives: the cache bit for bit, and, decoded greedily, every token the
    likeliest of its row up to the rounding of bf16 logits (2^-8 of values below 16, from attention outputs that differ by
    rounding: 0.1).  Pages are taken as they are needed and all come back."""
    model = drafted.Model(3, 504, 8, 2, 64, 300)
    prompts = _prompts(6, 504, drafts)
    session, said, totals = drafted.run(model, prompts, 40, drafts, temperature, seed=5, cache_bits=4)
    assert all(40 <= len(t) <= 40 + drafts for t in said) and totals["steps"] <= 40
    texts = [p + t for p, t in zip(prompts, said)]
    whole = drafted.Session4(model, texts, session.history.shape[1] - max(len(t) for t in texts))
    tokens = torch.cat([whole.history[s, :n] for s, n in enumerate(whole.lens)])
    _, out = whole.attend(tokens, np.zeros(len(texts), np.int32), whole.lens)
    logits = model.logits(tokens, out).float()
    torch.cuda.synchronize()
    assert int(whole.status.item()) == 0 and int(session.status.item()) == 0
    row = 0
    for s, (p, t) in enumerate(zip(prompts, said)):
        n = len(p) + len(t) - 1                                           # the last token's row is not in the cache yet
        at, slots = torch.arange(n) // 16, torch.arange(n) % 16
        held = session.table[s][session.table[s] >= 0]
        assert len(held) == -(-n // 16) or len(held) <= -(-(n + drafts + 1) // 16)
        for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
            a, b = getattr(session.cache, name), getattr(whole.cache, name)
            assert torch.equal(a[session.table[s, at].long(), :, slots], b[whole.table[s, at].long(), :, slots])
        if temperature == 0:
            said_by = logits[row + len(p) - 1:row + n]
            chosen = said_by.gather(1, torch.tensor(t, device="cuda")[:, None])[:, 0]
            assert (said_by.amax(1) - chosen).max() <= 0.1
        row += n + 1
    pages = len(session.free)
    assert session.num_free.item() == pages - int((session.table >= 0).sum())
    session.finish()
    assert session.num_free.item() == pages and sorted(session.free.tolist()) == list(range(pages)) and (session.table == -1).all()


def test_penalties_keep_from_repeating():
    """A model that goes round in eights does not where repetition costs more than its preference, with either cache."""
    model = drafted.Model(4, 304, 4, 4, 128, 400)
    prompts = _prompts(3, 304, 1)
    for bits in (16, 4):
        _, free, _ = drafted.run(model, prompts, 60, 4, cache_bits=bits)
        _, held, _ = drafted.run(model, prompts, 60, 4, cache_bits=bits, penalties=dict(presence=40.0))
        assert all(len(set(t)) < 40 for t in free) and all(len(set(t[:60])) == 60 for t in held)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (28, 4, 128)])
def test_captured_step(hq, hkv, d):
    """Tables, append, attention, logits and verification as one graph: the same bits as the calls, also after the lengths moved on."""
    users, most, vocab, width = 5, 4, 1000, 20
    g = torch.Generator(device="cuda").manual_seed(d)
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = efim.Cache4.empty(users * width, hkv, d, hq, 0.5, 0.5)
    rope, norm = efim.Rope(10000.0, d, 16 * width), efim.QkNorm(None, None)
    table, free = torch.full((users, width), -1, **i32), torch.randperm(users * width, generator=g, device="cuda").to(torch.int32)
    count, status = torch.tensor([users * width], **i32), torch.zeros(1, **i32)
    cached, new, ctx = (torch.zeros(users, **i32) for _ in range(3))
    rows = users * most
    indptr, positions, sequences = torch.zeros(users + 1, **i32), torch.zeros(rows, **i32), torch.zeros(rows, **i32)
    slots = torch.zeros(rows, dtype=torch.int64, device="cuda")
    qkv = torch.randn(rows, (hq + 2 * hkv) * d, generator=g, device="cuda").bfloat16()
    q, k, v = qkv.split([hq * d, hkv * d, hkv * d], 1)
    q_out, out = (torch.zeros(rows, hq, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    head = torch.randn(vocab, hq * d, generator=g, device="cuda").bfloat16()
    history = torch.randint(vocab, (users, 16 * width), generator=g, **i32)
    tokens = torch.randint(vocab, (rows,), generator=g, **i32)
    logits = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    accepted, following, emitted = torch.zeros(users, **i32), torch.zeros(users, **i32), torch.zeros(users, most, **i32)
    ws = torch.empty(efim.efim_kv4_decode_workspace_bytes(cache, users, most, 16 * width), dtype=torch.uint8, device="cuda")
    tables_ws = torch.empty(efim.efim_step_tables_workspace_bytes(users), dtype=torch.uint8, device="cuda")
    batch = efim.Batch.from_device(cached, new, indptr, table, rows)
    repetition = torch.full((users,), 1.2, device="cuda")

    def step():
        efim.efim_step_tables(cached, new, table, free, count, indptr, positions, slots, sequences, workspace=tables_ws, status=status)
        efim.efim_kv4_append(cache, batch, norm, rope, q, k, v, q_out, status)
        efim.efim_kv4_decode_attn(cache, users, ctx, 16 * width, table, q_out, out, q_indptr=indptr, max_new_len=most, workspace=ws, status=status)
        torch.matmul(out.view(rows, -1), head.t(), out=logits)
        efim.efim_adjust_logits(indptr, logits, history=history, lengths=ctx, tokens=tokens, repetition=repetition, status=status)
        efim.efim_verify_drafts(indptr, tokens, logits, accepted, following, out_tokens=emitted, status=status)

    def lengths(seed):
        r = np.random.default_rng(seed)
        n = r.integers(0, most + 1, users)
        cached.copy_(torch.tensor(r.integers(0, 16 * width - most, users)))
        new.copy_(torch.tensor(n))
        ctx.copy_(cached + new)

    results = [table, count, indptr, positions, slots, sequences, q_out, out, logits, accepted, following, emitted, cache.k_codes, cache.v_codes,
               cache.k_scales, cache.v_scales, status]
    starts = [x.clone() for x in results]
    def restart():
        for x, y in zip(results, starts):
            x.copy_(y)
    for x in (cache.k_scales, cache.v_scales):                              # what was appended earlier on
        x.fill_(0x30)
    table.copy_(free.view(users, width))
    starts = [x.clone() for x in results]
    lengths(0)
    step()                                                                   # (first looks at the device are not captured)
    graph = torch.cuda.CUDAGraph()
    restart()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2):
        lengths(seed)
        restart()
        step()
        want = [x.clone() for x in results]
        restart()
        graph.replay()
        assert status.item() == 0
        for x, y in zip(results, want):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
