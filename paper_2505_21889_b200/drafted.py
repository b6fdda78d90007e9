"""Decode of the generated middle with drafted tokens, through one layer with q/k norms: what a serving loop does around the
library when infilled code repeats its prefix and suffix.  Per step, for all users together:

  drafts     efim_draft_lookup        what followed the history's last tokens earlier on
  k/v, q     efim_qk_norm_append      the pending token and its drafts: norms, rotation, pages (views of one projection's output)
  attention  efim_append_prefill_attn over everything before each of them
  logits     one matrix product of this toy model
  decision   efim_verify_drafts       accepted drafts and the next token, greedily or by given random numbers

The accepted drafts' keys and values stay, the next step writes over the others'.  Without drafts the same loop decodes one token a
step.  The "model" is a layer whose projections are tables by token id (random weights: what it says means nothing).

    python -m paper_2505_21889_b200.drafted --users 16 --tokens 128 --drafts 4 --temperature 0.7
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

    def __init__(self, model, prompts, room):
        hq, hkv, d = model.shape
        self.model, self.room = model, room
        self.lens = np.array([len(p) for p in prompts], np.int64)         # of the histories, the pending token included
        users, top = len(prompts), int(self.lens.max()) + room
        history = torch.zeros(users, top, dtype=torch.int32)
        for s, p in enumerate(prompts):
            history[s, :len(p)] = torch.as_tensor(p, dtype=torch.int32)
        self.history = history.to(model.device)
        pages = -(-top // 16)
        order = torch.randperm(users * pages, generator=torch.Generator().manual_seed(1))
        self.table = order.view(users, pages).to(torch.int32).to(model.device)
        pools = (torch.zeros(users * pages, hkv, 16, d, dtype=torch.bfloat16, device=model.device) for _ in range(2))
        self.cache = efim.Cache(*pools, hq)
        self.status = torch.zeros(1, dtype=torch.int32, device=model.device)

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
        pending = self.history.gather(1, (lens.long() - 1)[:, None])
        found = torch.zeros(users, dtype=torch.int32, device=device)
        if drafts > 0:
            tail = torch.empty(users, drafts, dtype=torch.int32, device=device)
            efim.efim_draft_lookup(self.history, lens, 1, max_ngram, tail, found, self.status)
            rows = torch.cat([pending, tail], 1)
        else:
            rows = pending
        new = 1 + found.cpu().numpy()                                    # the host plans the attention by these lengths
        tokens = rows[torch.arange(drafts + 1, device=device) <= found[:, None]]
        batch, out = self.attend(tokens, self.lens - 1, new)
        logits = self.model.logits(tokens, out)
        accepted, following = (torch.empty(users, dtype=torch.int32, device=device) for _ in range(2))
        emitted = torch.empty(users, drafts + 1, dtype=torch.int32, device=device)
        chance = {}
        if temperature > 0:
            chance = dict(uniform=torch.rand(len(tokens), device=device, generator=generator),
                          noise=torch.empty(users, self.model.vocab, device=device).exponential_(generator=generator),
                          temperature=torch.full((users,), temperature, device=device))
        efim.efim_verify_drafts(batch.d_q_indptr, tokens, logits, accepted, following, out_tokens=emitted, status=self.status, **chance)
        # the histories go on; what the verification refused is written over by the next step
        got = accepted.long() + 1
        place = torch.arange(drafts + 1, device=device)
        at = (lens.long()[:, None] + place).clamp(max=self.history.shape[1] - 1)
        keep = place < got[:, None]
        self.history.scatter_(1, at, torch.where(keep, emitted, self.history.gather(1, at)))
        self.lens = self.lens + got.cpu().numpy()
        return [row[:n] for row, n in zip(emitted.tolist(), got.tolist())]


def run(model, prompts, tokens, drafts, temperature=0.0, seed=0, max_ngram=4):
    """Every user generates at least `tokens` tokens.  -> (session, lists of tokens, totals)"""
    session = Session(model, prompts, tokens + 2 * (drafts + 1))
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
    return session, said, dict(users=len(prompts), drafts=drafts, temperature=temperature, steps=steps, tokens=made,
                               tokens_per_user_step=made / (steps * len(prompts)), ms=start.elapsed_time(end))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--users", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=128)
    ap.add_argument("--drafts", type=int, nargs="+", default=[0, 4])
    ap.add_argument("--temperature", type=float, default=0.0)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--heads", type=int, nargs=2, default=(32, 8), metavar=("HQ", "HKV"))
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    prompts = [[TOK_P] + t["prefix"] + [TOK_S] + t["suffix"] + [TOK_M]
               for user in infill_sessions(a.seed, a.users, 1, a.vocab) for t in user]
    torch.cuda.set_device(0)
    longest = max(len(p) for p in prompts) + a.tokens + 2 * (max(a.drafts) + 1)
    model = Model(a.seed, a.vocab, a.heads[0], a.heads[1], 128, longest)
    for drafts in a.drafts:
        run(model, prompts, 4, drafts, a.temperature, a.seed)              # warm-up
        print(json.dumps(run(model, prompts, a.tokens, drafts, a.temperature, a.seed)[2]), flush=True)


if __name__ == "__main__":
    main()
