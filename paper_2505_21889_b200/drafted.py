"""Decode of the generated middle with drafted tokens, through one layer with q/k norms: what a serving loop does around the
library when infilled code repeats its prefix and suffix.  Per step, for all users together:

  drafts     efim_draft_lookup        what followed the history's last tokens earlier on
  k/v, q     efim_qk_norm_append      the pending token and its drafts: norms, rotation, pages (views of one projection's output)
  attention  efim_append_prefill_attn over everything before each of them
  logits     one matrix product of this toy model
  decision   efim_verify_drafts       accepted drafts and the next token, greedily or by given random numbers

With a cache held in 4 bits pages and rows come from the lengths on the device (efim_step_tables), and efim_kv4_append and
efim_kv4_decode_attn stand in place of the middle two: calls that read no lengths on the host, and so can be captured.  This loop, with either
cache, reads back what each step accepted and keeps the histories' lengths on the host.  Penalties go between logits and decision
(efim_adjust_logits).

The accepted drafts' keys and values stay, the next step writes over the others'.  Without drafts the same loop decodes one token a
step.  The "model" is a layer whose projections are tables by token id (random weights: what it says means nothing).

    python -m paper_2505_21889_b200.drafted --users 16 --tokens 128 --drafts 4 --temperature 0.7 [--cache-bits 4 --repetition 1.1]
"""
import argparse
import json

import numpy as np
import torch

from . import binding as efim
from efim_synth import token_tables, infill_sessions, TOK_P, TOK_S, TOK_M


class Model:
    """One layer: token id -> q, k, v heads in one row, norm weights, an output matrix onto the vocabulary."""

    def __init__(self, seed, vocab, num_q_heads, num_kv_heads, head_dim, max_position, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.shape = num_q_heads, num_kv_heads, head_dim
        self.vocab, self.device = vocab, device
        tables = [torch.from_numpy(t.view(np.int16)).view(torch.bfloat16).reshape(vocab, -1)
                  for t in token_tables(seed, vocab, num_q_heads, num_kv_heads, head_dim)]
        self.qkv = torch.cat(tables, 1).to(device)
        weights = [(1 + 0.1 * torch.randn(head_dim, generator=g)).bfloat16().to(device) for _ in range(2)]
        self.norm = efim.QkNorm(*weights, eps=1e-6)
        self.rope = efim.Rope(10000.0, head_dim, max_position, False, device)
        width = num_q_heads * head_dim
        self.head = (torch.randn(vocab, width, generator=g) * 8 / width ** 0.5).bfloat16().to(device)
        # text that repeats itself: mostly a token is followed by the next one of its eight
        t = torch.arange(vocab, device=device)
        self.follow = t // 8 * 8 + (t + 1) % 8 if vocab % 8 == 0 else (t + 1) % vocab

    def logits(self, tokens, attended):
        out = attended.view(len(tokens), -1) @ self.head.t()
        out[torch.arange(len(tokens), device=self.device), self.follow[tokens.long()]] += 9.0
        return out


class Session:
    """Users' histories, pages and lengths on one layer."""

    def __init__(self, model, prompts, room, penalties=None):
        self.model, self.room = model, room
        self.penalties = {name: torch.full((len(prompts),), x, device=model.device) for name, x in (penalties or {}).items()}
        self.prompt_len = torch.tensor([len(p) for p in prompts], dtype=torch.int32).to(model.device)
        self.lens = np.array([len(p) for p in prompts], np.int64)         # of the histories, the pending token included
        users, top = len(prompts), int(self.lens.max()) + room
        history = torch.zeros(users, top, dtype=torch.int32)
        for s, p in enumerate(prompts):
            history[s, :len(p)] = torch.as_tensor(p, dtype=torch.int32)
        self.history = history.to(model.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=model.device)
        pages = -(-top // 16)
        self.make_cache(users, pages, torch.randperm(users * pages, generator=torch.Generator().manual_seed(1)).to(torch.int32))

    def make_cache(self, users, pages, order):
        hq, hkv, d = self.model.shape
        self.table = order.view(users, pages).to(self.model.device)
        pools = (torch.zeros(users * pages, hkv, 16, d, dtype=torch.bfloat16, device=self.model.device) for _ in range(2))
        self.cache = efim.Cache(*pools, hq)

    def attend(self, tokens, cached, new):
        """Appends `new` tokens per user behind `cached` ones and attends.  -> rows of heads"""
        hq, hkv, d = self.model.shape
        batch = efim.Batch(cached, new, self.table, self.model.device)
        q, k, v = self.model.qkv[tokens.long()].split([hq * d, hkv * d, hkv * d], 1)
        q_out = torch.empty(len(tokens), hq, d, dtype=torch.bfloat16, device=self.model.device)
        out = torch.empty_like(q_out)
        efim.efim_qk_norm_append(self.cache, batch, self.model.norm, self.model.rope, q, k, v, q_out, self.status)
        ws = torch.empty(efim.efim_prefill_workspace_bytes(self.cache, batch), dtype=torch.uint8, device=self.model.device)
        efim.efim_append_prefill_attn(self.cache, batch, q_out, out, None, 0.0, ws, self.status)
        return batch, out

    def prefill(self):
        """Keys and values of every token but the last, which is pending."""
        rows = [self.history[s, :n - 1] for s, n in enumerate(self.lens)]
        self.attend(torch.cat(rows), np.zeros(len(rows), np.int32), self.lens - 1)

    def step(self, drafts, temperature, generator, max_ngram=4):
        """-> tokens that each user goes on with (lists)"""
        users, device = len(self.lens), self.model.device
        lens = torch.as_tensor(self.lens, dtype=torch.int32).to(device)
        rows, found = self.look_up(lens, drafts, max_ngram)
        indptr, tokens, out = self.forward(lens, rows, found)
        logits = self.model.logits(tokens, out)
        if self.penalties:
            efim.efim_adjust_logits(indptr, logits, history=self.history, lengths=lens, prompt_len=self.prompt_len, tokens=tokens,
                                    status=self.status, **self.penalties)
        accepted, following = (torch.empty(users, dtype=torch.int32, device=device) for _ in range(2))
        emitted = torch.empty(users, drafts + 1, dtype=torch.int32, device=device)
        chance = {}
        if temperature > 0:
            chance = dict(uniform=torch.rand(len(tokens), device=device, generator=generator),
                          noise=torch.empty(users, self.model.vocab, device=device).exponential_(generator=generator),
                          temperature=torch.full((users,), temperature, device=device))
        efim.efim_verify_drafts(indptr, tokens, logits, accepted, following, out_tokens=emitted, status=self.status, **chance)
        # the histories go on; what the verification refused is written over by the next step
        got = accepted.long() + 1
        place = torch.arange(drafts + 1, device=device)
        at = (lens.long()[:, None] + place).clamp(max=self.history.shape[1] - 1)
        keep = place < got[:, None]
        self.history.scatter_(1, at, torch.where(keep, emitted, self.history.gather(1, at)))
        self.lens = self.lens + got.cpu().numpy()
        return [row[:n] for row, n in zip(emitted.tolist(), got.tolist())]

    def look_up(self, lens, drafts, max_ngram):
        """-> pending token and drafts of each user, how many drafts there are"""
        users, device = len(self.lens), self.model.device
        pending = self.history.gather(1, (lens.long() - 1)[:, None])
        found = torch.zeros(users, dtype=torch.int32, device=device)
        if drafts > 0:
            tail = torch.empty(users, drafts, dtype=torch.int32, device=device)
            efim.efim_draft_lookup(self.history, lens, 1, max_ngram, tail, found, self.status)
            rows = torch.cat([pending, tail], 1)
        else:
            rows = pending
        return rows, found

    def forward(self, lens, rows, found):
        """One step of the layer.  -> row offsets, tokens, attended rows"""
        new = 1 + found.cpu().numpy()                                    # the host plans the attention by these lengths
        tokens = rows[torch.arange(rows.shape[1], device=rows.device) <= found[:, None]]
        batch, out = self.attend(tokens, self.lens - 1, new)
        return batch.d_q_indptr, tokens, out


class Session4(Session):
    """The same over a cache in 4 bits, with pages taken from a stack of free ones as the sequences grow."""

    def make_cache(self, users, pages, order):
        hq, hkv, d = self.model.shape
        self.table = torch.full((users, pages), -1, dtype=torch.int32, device=self.model.device)
        self.cache = efim.Cache4.empty(users * pages, hkv, d, hq, device=self.model.device)
        self.free = order.to(self.model.device)
        self.num_free = torch.tensor([len(order)], dtype=torch.int32).to(self.model.device)

    def grow(self, cached, new, rows):
        """Pages for the new tokens.  -> the batch, and for each of its rows the sequence and the place among its new tokens"""
        indptr = torch.empty(len(cached) + 1, dtype=torch.int32, device=cached.device)
        positions, sequences = (torch.empty(rows, dtype=torch.int32, device=cached.device) for _ in range(2))
        efim.efim_step_tables(cached, new, self.table, self.free, self.num_free, indptr, positions, None, sequences, status=self.status)
        batch = efim.Batch.from_device(cached, new, indptr, self.table, rows)
        sequence = sequences.clamp(min=0).long()
        return batch, sequence, (positions - cached[sequence]).clamp(min=0).long()

    def append(self, batch, tokens):
        hq, hkv, d = self.model.shape
        q, k, v = self.model.qkv[tokens.long()].split([hq * d, hkv * d, hkv * d], 1)
        q_out = torch.zeros(len(tokens), hq, d, dtype=torch.bfloat16, device=self.model.device)
        efim.efim_kv4_append(self.cache, batch, self.model.norm, self.model.rope, q, k, v, q_out, self.status)
        return q_out

    def attend(self, tokens, cached, new):
        device = self.model.device
        self.grow(*(torch.as_tensor(x, dtype=torch.int32).to(device) for x in (cached, new)), 0)
        batch = efim.Batch(cached, new, self.table, device)
        q = self.append(batch, tokens)
        ws = torch.empty(efim.efim_kv4_prefill_workspace_bytes(self.cache, batch), dtype=torch.uint8, device=device)
        efim.efim_kv4_append_prefill_attn(self.cache, batch, q, q, workspace=ws, status=self.status)
        return batch, q

    def forward(self, lens, rows, found):
        users, most = rows.shape
        batch, sequence, place = self.grow(lens - 1, 1 + found, users * most)
        tokens = rows[sequence, place]
        q = self.append(batch, tokens)
        longest = 16 * self.table.shape[1]
        ws = torch.empty(efim.efim_kv4_decode_workspace_bytes(self.cache, users, most, longest), dtype=torch.uint8, device=rows.device)
        efim.efim_kv4_decode_attn(self.cache, users, lens + found, longest, self.table, q, q, q_indptr=batch.d_q_indptr, max_new_len=most,
                                  workspace=ws, status=self.status)
        return batch.d_q_indptr, tokens, q

    def finish(self):
        """Every sequence is over: its pages are free again."""
        efim.efim_release_pages(torch.zeros_like(self.prompt_len), self.table, self.free, self.num_free, status=self.status)


def run(model, prompts, tokens, drafts, temperature=0.0, seed=0, max_ngram=4, cache_bits=16, penalties=None):
    """Every user generates at least `tokens` tokens.  penalties: numbers by name (repetition, presence, frequency).
    -> (session, lists of tokens, totals)"""
    session = (Session4 if cache_bits == 4 else Session)(model, prompts, tokens + 2 * (drafts + 1), penalties)
    generator = torch.Generator(device=model.device).manual_seed(seed)
    session.prefill()
    said = [[] for _ in prompts]
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    steps = 0
    start.record()
    limit = session.lens + tokens
    while (session.lens < limit).any():
        before = session.lens.copy()
        for s, got in enumerate(session.step(drafts, temperature, generator, max_ngram)):
            if before[s] < limit[s]:
                said[s] += got
            else:
                session.lens[s] = before[s]                               # that user has enough
        steps += 1
    end.record()
    torch.cuda.synchronize()
    if int(session.status.item()) != 0:
        raise RuntimeError(f"device status 0x{int(session.status.item()):x}")
    made = sum(len(t) for t in said)
    return session, said, dict(users=len(prompts), cache_bits=cache_bits, drafts=drafts, temperature=temperature, steps=steps, tokens=made,
                               tokens_per_user_step=made / (steps * len(prompts)), ms=start.elapsed_time(end))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--users", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=128)
    ap.add_argument("--drafts", type=int, nargs="+", default=[0, 4])
    ap.add_argument("--temperature", type=float, default=0.0)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--heads", type=int, nargs=2, default=(32, 8), metavar=("HQ", "HKV"))
    ap.add_argument("--cache-bits", type=int, default=16, choices=(16, 4))
    for name in ("repetition", "presence", "frequency"):
        ap.add_argument("--" + name, type=float, help="penalty of tokens that occurred")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    prompts = [[TOK_P] + t["prefix"] + [TOK_S] + t["suffix"] + [TOK_M]
               for user in infill_sessions(a.seed, a.users, 1, a.vocab) for t in user]
    torch.cuda.set_device(0)
    longest = max(len(p) for p in prompts) + a.tokens + 2 * (max(a.drafts) + 1)
    model = Model(a.seed, a.vocab, a.heads[0], a.heads[1], 128, longest)
    more = dict(cache_bits=a.cache_bits, penalties={n: getattr(a, n) for n in ("repetition", "presence", "frequency") if getattr(a, n) is not None})
    for drafts in a.drafts:
        run(model, prompts, 4, drafts, a.temperature, a.seed, **more)      # warm-up
        print(json.dumps(run(model, prompts, a.tokens, drafts, a.temperature, a.seed, **more)[2]), flush=True)


if __name__ == "__main__":
    main()
