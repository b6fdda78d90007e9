"""Timed cases of the operators around a step with drafted tokens: drafts looked up in a sequence's own history, q/k norms with
rotation and append, verification of the drafts.  Each case goes through its plain form (elementary torch operations, fp32) or,
with `own`, through the library."""
import math
import random

import torch

own = False

EPS = 1e-6


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one user, one generated token: the smallest append there is
        dict(name="norm_decode_one", op="norm", seqs=1, new_lo=1, new_hi=1, ctx_lo=2300, ctx_hi=2300, hq=32, hkv=8, dim=128,
             interleaved=False, lengths=1),
        # a decode step of 64 users of a grouped-query coder model
        dict(name="norm_decode_users", op="norm", seqs=64, new_lo=1, new_hi=1, ctx_lo=1024, ctx_hi=16384, hq=28, hkv=4, dim=128,
             interleaved=False, lengths=2),
        # a step of 16 users with up to eight drafted tokens each, small heads, pairs side by side
        dict(name="norm_drafts", op="norm", seqs=16, new_lo=1, new_hi=9, ctx_lo=300, ctx_hi=4000, hq=4, hkv=4, dim=64,
             interleaved=True, lengths=3),
        # a turn: 16 increments of 32 to 256 tokens, as many kv heads as query heads
        dict(name="norm_turn", op="norm", seqs=16, new_lo=32, new_hi=256, ctx_lo=2048, ctx_hi=8192, hq=32, hkv=32, dim=128,
             interleaved=False, lengths=4),
        # suffixes recomputed after a cache miss: the largest append
        dict(name="norm_miss", op="norm", seqs=8, new_lo=3200, new_hi=3200, ctx_lo=5120, ctx_hi=5120, hq=32, hkv=8, dim=128,
             interleaved=False, lengths=5),
        # one user, four tokens drafted from the history (no distribution of their own)
        dict(name="verify_one", op="verify", seqs=1, lo=4, hi=4, vocab=32768, kind="bf16", dense=False, lengths=6),
        # 16 users, four tokens each from a draft model
        dict(name="verify_users", op="verify", seqs=16, lo=4, hi=4, vocab=131072, kind="bf16", dense=True, lengths=7),
        # ragged numbers of drafts (none among them), an odd vocabulary, fp32 logits
        dict(name="verify_ragged", op="verify", seqs=37, lo=0, hi=7, vocab=100003, kind="f32", dense=False, lengths=8),
        # a full server: 256 users, five rows each, draft model of the same vocabulary
        dict(name="verify_many", op="verify", seqs=256, lo=4, hi=4, vocab=131072, kind="bf16", dense=True, lengths=9),
        # drafts for one user
        dict(name="lookup_one", op="lookup", seqs=1, ctx_lo=2300, ctx_hi=2300, ngram=4, drafts=4, lengths=10),
        # drafts for a mixed batch
        dict(name="lookup_users", op="lookup", seqs=64, ctx_lo=1024, ctx_hi=16384, ngram=3, drafts=8, lengths=11),
        # drafts for a full server with long contexts
        dict(name="lookup_long", op="lookup", seqs=256, ctx_lo=4096, ctx_hi=32768, ngram=8, drafts=8, lengths=12),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("norm", "verify", "verify", "lookup"))
    lengths = rng.randrange(1 << 20)
    if op == "norm":
        hkv, group = rng.choice(((1, 16), (4, 1), (4, 7), (8, 4), (8, 5), (32, 1), (3, 3)))
        dim = rng.choice((64, 128))
        total = _log_int(rng, 1, min(20000, 150000000 // ((group + 2) * hkv * dim)))
        seqs = _log_int(rng, 1, min(total, 256))
        hi = max(1, total // seqs)
        return dict(op=op, seqs=seqs, new_lo=rng.randint(1, hi), new_hi=hi, ctx_lo=rng.randint(0, 500), ctx_hi=_log_int(rng, 500, 8192),
                    hq=hkv * group, hkv=hkv, dim=dim, interleaved=rng.random() < 0.3, lengths=lengths)
    if op == "verify":
        vocab = _log_int(rng, 1000, 131072)
        hi = _log_int(rng, 1, 9) - 1
        seqs = _log_int(rng, 1, 256)
        kind = rng.choice(("bf16", "bf16", "f32", "probs"))
        while seqs * (hi + 1) * vocab > (1280 if kind == "bf16" else 640) * 131072:
            seqs //= 2
        return dict(op=op, seqs=seqs, lo=rng.randint(0, hi), hi=hi, vocab=vocab, kind=kind,
                    dense=rng.random() < 0.5, lengths=lengths)
    hi = _log_int(rng, 64, 32768)
    return dict(op=op, seqs=_log_int(rng, 1, min(256, 4700000 // hi)), ctx_lo=rng.randint(2, hi), ctx_hi=hi, ngram=rng.randint(1, 8),
                drafts=rng.randint(1, 16), lengths=lengths)


def _ints(case, seqs, lo, hi, tag):
    r = random.Random(case["lengths"] * 4 + tag)
    return [r.randint(lo, hi) for _ in range(seqs)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    return dict(norm=_prepare_norm, verify=_prepare_verify, lookup=_prepare_lookup)[case["op"]](case, seed)


def _rope_table(dim, positions):
    theta = 10000.0 ** (-2.0 * torch.arange(dim // 2, dtype=torch.float64) / dim)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * theta
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _prepare_norm(case, seed):
    """One projection's output [tokens, (hq + 2 hkv) dim], pages of a shuffled pool, the norms' weights."""
    g = _gen(seed)
    b, hq, hkv, d = case["seqs"], case["hq"], case["hkv"], case["dim"]
    cached = _ints(case, b, case["ctx_lo"], case["ctx_hi"], 0)
    new = _ints(case, b, case["new_lo"], case["new_hi"], 1)
    pages = [(c + n + 15) // 16 for c, n in zip(cached, new)]
    # the pool holds the pages that the step writes; the table's other entries, which it does not read, are -1
    first = [c // 16 for c in cached]
    mine = [p - f for p, f in zip(pages, first)]
    perm = torch.randperm(sum(mine) + 3, generator=g, device="cuda").to(torch.int32)
    table = torch.full((b, max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s in range(b):
        table[s, first[s]:pages[s]] = perm[at:at + mine[s]]
        at += mine[s]
    tokens = sum(new)
    qkv = torch.randn(tokens, (hq + 2 * hkv) * d, generator=g, device="cuda", dtype=torch.bfloat16)
    pool = (sum(mine) + 3, hkv, 16, d)
    st = dict(case=case, qkv=qkv, k_pool=torch.randn(pool, generator=g, device="cuda", dtype=torch.bfloat16),
              v_pool=torch.randn(pool, generator=g, device="cuda", dtype=torch.bfloat16),
              q_weight=(1 + 0.2 * torch.randn(d, generator=g, device="cuda")).bfloat16(),
              k_weight=(1 + 0.2 * torch.randn(d, generator=g, device="cuda")).bfloat16(),
              cached=_i32(cached), new=_i32(new), table=table, rope_table=_rope_table(d, max(c + n for c, n in zip(cached, new))).cuda(),
              h_cached=cached, h_new=new, q_out=torch.empty(tokens, hq, d, dtype=torch.bfloat16, device="cuda"))
    st["indptr"] = torch.cat([_i32([0]), st["new"].cumsum(0).to(torch.int32)])
    return st


def _draft_rows(case):
    """Rows of each sequence: its pending token and its drafts."""
    return [k + 1 for k in _ints(case, case["seqs"], case["lo"], case["hi"], 0)]


def _prepare_verify(case, seed):
    """Target logits with one likely token a row, drafts that mostly are that token (or draws of a draft model that is near the
    target), random numbers, temperatures of 0.6 to 1 and a greedy user in eight."""
    g = _gen(seed)
    rows, v = _draft_rows(case), case["vocab"]
    b, r = len(rows), sum(rows)
    logits = 2.5 * torch.randn(r, v, generator=g, device="cuda")
    likely = torch.randint(v, (r,), generator=g, device="cuda")
    # log of the row's mass is about log(v) + 2.5^2 / 2: the likely token gets some 0.2 to 0.99 of it
    lift = math.log(v) + 3.1 + 3.0 * torch.rand(r, generator=g, device="cuda") - 1.0
    logits[torch.arange(r, device="cuda"), likely] = lift
    indptr = torch.tensor([0] + rows, device="cuda").cumsum(0).to(torch.int32)
    st = dict(case=case, indptr=indptr, uniform=torch.rand(r, generator=g, device="cuda"),
              noise=torch.empty(b, v, device="cuda").exponential_(generator=g).clamp_(min=1e-30))
    if case["dense"]:
        near = logits + 0.5 * torch.randn(r, v, generator=g, device="cuda")
        near[torch.arange(r, device="cuda"), likely] = lift - 0.3
        st["draft_probs"] = torch.softmax(near, 1)
        drawn = (st["draft_probs"] / torch.empty_like(near).exponential_(generator=g)).argmax(1)
        del near
    else:
        other = torch.randint(v, (r,), generator=g, device="cuda")
        drawn = torch.where(torch.rand(r, generator=g, device="cuda") < 0.9, likely, other)
    # the draft that row i proposes is the step's token i + 1
    st["tokens"] = torch.roll(drawn, 1).to(torch.int32)
    if case["kind"] == "probs":
        st["target"] = torch.softmax(logits, 1)
    else:
        st["target"] = logits.bfloat16() if case["kind"] == "bf16" else logits
        t = 0.6 + 0.4 * torch.rand(b, generator=g, device="cuda")
        st["temperature"] = torch.where(torch.arange(b, device="cuda") % 8 == 5, torch.zeros_like(t), t)
    most = max(rows)
    st["accepted"] = torch.empty(b, dtype=torch.int32, device="cuda")
    st["next"] = torch.empty(b, dtype=torch.int32, device="cuda")
    st["out"] = torch.empty(b, most, dtype=torch.int32, device="cuda")
    st["logprobs"] = torch.empty(b, most, device="cuda")
    return st


def _prepare_lookup(case, seed):
    """Histories of a small working vocabulary that now and then repeat an earlier stretch, and end in the middle of one."""
    g = _gen(seed)
    lens = _ints(case, case["seqs"], case["ctx_lo"], case["ctx_hi"], 0)
    b, top = len(lens), max(lens)
    hist = torch.randint(2000, (b, top), generator=g, device="cuda", dtype=torch.int32)
    ends = torch.tensor(lens, device="cuda")
    for n in (3, 9):                                    # the last 3, then 9 tokens occur before, at another place each
        n = min(n, min(lens) // 2)
        back = (ends - n).clamp(min=0)
        src = (torch.rand(b, generator=g, device="cuda") * (back - n).clamp(min=1)).long()
        at = torch.arange(n, device="cuda")
        row = torch.arange(b, device="cuda")[:, None]
        hist[row, src[:, None] + at] = hist[row, back[:, None] + at]
    return dict(case=case, history=hist, lengths=ends.to(torch.int32),
                drafts=torch.empty(b, case["drafts"], dtype=torch.int32, device="cuda"),
                draft_len=torch.empty(b, dtype=torch.int32, device="cuda"))


# ------------------------------------------------------------------ one pass
def run(state):
    forms = _OWN if own else _PLAIN
    return forms[state["case"]["op"]](state)


def _library(st):
    """The library's descriptors of a state, made on the first pass and kept, as a serving loop keeps them."""
    if "own" not in st:
        import paper_2505_21889_b200 as efim
        st["own"], st["status"] = efim, torch.zeros(1, dtype=torch.int32, device="cuda")
        case = st["case"]
        if case["op"] == "norm":
            st["cache"] = efim.Cache(st["k_pool"], st["v_pool"], case["hq"])
            st["batch"] = efim.Batch(st["h_cached"], st["h_new"], st["table"])
            st["rope"] = efim.Rope.from_table(st["rope_table"], case["interleaved"])
            st["norm"] = efim.QkNorm(st["q_weight"], st["k_weight"], EPS)
            st["split"] = st["qkv"].split([case["hq"] * case["dim"], case["hkv"] * case["dim"], case["hkv"] * case["dim"]], 1)
    return st["own"]


def _own_norm(st):
    efim = _library(st)
    q, k, v = st["split"]
    efim.efim_qk_norm_append(st["cache"], st["batch"], st["norm"], st["rope"], q, k, v, st["q_out"], st["status"])
    return dict(q=st["q_out"], k_pool=st["k_pool"], v_pool=st["v_pool"])


def _own_verify(st):
    efim = _library(st)
    efim.efim_verify_drafts(st["indptr"], st["tokens"], st["target"], st["accepted"], st["next"], uniform=st["uniform"],
                            noise=st["noise"], draft_probs=st.get("draft_probs"), temperature=st.get("temperature"),
                            target_is_probs=st["case"]["kind"] == "probs", out_tokens=st["out"], out_logprobs=st["logprobs"],
                            status=st["status"])
    return dict(accepted=st["accepted"], next=st["next"], out=st["out"], logprobs=st["logprobs"])


def _own_lookup(st):
    efim = _library(st)
    efim.efim_draft_lookup(st["history"], st["lengths"], 1, st["case"]["ngram"], st["drafts"], st["draft_len"], st["status"])
    return dict(drafts=st["drafts"], draft_len=st["draft_len"])


def _plain_norm(st):
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    tokens = st["qkv"].shape[0]
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), st["new"], output_size=tokens)
    pos = st["cached"][seq] + torch.arange(tokens, device="cuda") - st["indptr"][seq]
    cos, sin = st["rope_table"][pos][:, None, :].split(d // 2, 2)
    x = st["qkv"].float().view(tokens, hq + 2 * hkv, d)

    def normed(x, weight):
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * weight.float()
        if case["interleaved"]:
            a, b = x[:, :, 0::2], x[:, :, 1::2]
            return torch.stack([a * cos - b * sin, b * cos + a * sin], 3).flatten(2).bfloat16()
        a, b = x.split(d // 2, 2)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], 2).bfloat16()

    page, slot = st["table"][seq, pos // 16].long(), pos % 16
    st["k_pool"][page, :, slot] = normed(x[:, hq:hq + hkv], st["k_weight"])
    st["v_pool"][page, :, slot] = x[:, hq + hkv:].bfloat16()
    return dict(q=normed(x[:, :hq], st["q_weight"]), k_pool=st["k_pool"], v_pool=st["v_pool"])


def _plain_verify(st):
    case, indptr = st["case"], st["indptr"].long()
    r, b = st["target"].shape[0], len(indptr) - 1
    row = torch.arange(r, device="cuda")
    seq = torch.searchsorted(indptr, row, right=True) - 1
    target, q = st["target"].float(), st.get("draft_probs")
    if case["kind"] == "probs":
        p, greedy = target, torch.zeros(b, dtype=torch.bool, device="cuda")
    else:
        greedy = st["temperature"] <= 0
        w = torch.exp((target - target.amax(1, keepdim=True)) * (1 / torch.where(greedy, 1, st["temperature"]))[seq, None])
        p = w / w.sum(1, keepdim=True)
    # acceptance: row i looks at the token after it, if that is of the same sequence
    has_draft = row + 1 < indptr[seq + 1]
    x = st["tokens"].long()[(row + 1).clamp(max=r - 1)]
    px = p.gather(1, x[:, None])[:, 0]
    qx = q.gather(1, x[:, None])[:, 0] if q is not None else 1.0
    best = target.argmax(1)
    ok = has_draft & torch.where(greedy[seq], best == x, st["uniform"] * qx < px)
    stop = torch.full((b,), r, device="cuda").scatter_reduce(0, seq, torch.where(ok, r, row), "amin")
    accepted = stop - indptr[:-1]
    # the next token: from what the draft's distribution leaves of the target's, or from the target's
    ps, rejected = p[stop], has_draft[stop][:, None]
    if q is not None:
        left = (ps - q[stop]).clamp(min=0)
    else:
        left = torch.where(torch.arange(ps.shape[1], device="cuda") == x[stop][:, None], 0, ps)
    left = torch.where(rejected & (left > 0).any(1, keepdim=True), left, ps)
    nxt = torch.where(greedy, best[stop], (left / st["noise"]).argmax(1))
    # what the sequence goes on with: its accepted drafts and the next token
    col = torch.arange(st["out"].shape[1], device="cuda")
    at = (indptr[:-1, None] + col).clamp(max=r - 1)
    after, last = col < accepted[:, None], col == accepted[:, None]
    out = torch.where(after, x[at], torch.where(last, nxt[:, None], -1))
    logprobs = torch.where(after, px[at].log(), torch.where(last, ps.gather(1, nxt[:, None]).log(), 0.0))
    return dict(accepted=accepted.int(), next=nxt.int(), out=out.int(), logprobs=logprobs)


def _plain_lookup(st):
    case, hist, n = st["case"], st["history"], st["case"]["ngram"]
    b, top = hist.shape
    lens = st["lengths"].long()[:, None]
    ngram = torch.arange(n, device="cuda")
    # what stands before each end e, last token first, against the history's own last tokens; -1 before its start
    padded = torch.cat([torch.full((b, n), -1, dtype=hist.dtype, device="cuda"), hist], 1)
    before = padded.unfold(1, n, 1).flip(2)                                      # [b, e, n]: tokens e - 1, e - 2, ...
    tail = padded.gather(1, (lens + n - 1 - ngram).clamp(min=0))
    same = torch.where((before == tail[:, None, :]) & (before >= 0), n, ngram).amin(2)   # the first place that differs
    end = torch.arange(top + 1, device="cuda")
    key = torch.where((end >= 1) & (end < lens) & (same > 0), same * (top + 1) + end, 0)
    best = key.amax(1, keepdim=True)
    e = best % (top + 1)
    drafts = hist.gather(1, e + torch.arange(case["drafts"], device="cuda") % (lens - e))
    return dict(drafts=torch.where(best > 0, drafts, -1), draft_len=torch.where(best[:, 0] > 0, case["drafts"], 0).int())


_OWN = dict(norm=_own_norm, verify=_own_verify, lookup=_own_lookup)
_PLAIN = dict(norm=_plain_norm, verify=_plain_verify, lookup=_plain_lookup)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "norm":
        tokens = sum(_ints(case, case["seqs"], case["new_lo"], case["new_hi"], 1))
        values = tokens * (case["hq"] + 2 * case["hkv"]) * case["dim"]
        return dict(bytes=4 * values + 4 * tokens * case["dim"], flops=8 * values)
    if case["op"] == "verify":
        rows, v = _draft_rows(case), case["vocab"]
        # About 0.8 of these drafts are accepted: a sequence needs the rows up to its first refusal, the draft's distribution
        # of that row if it is a refusal, and its random numbers (not where it is greedy: one in eight has logits).
        needed = sum(sum(0.8 ** i for i in range(n)) for n in rows)
        refused = sum(1 - 0.8 ** (n - 1) for n in rows)
        size = 2 if case["kind"] == "bf16" else 4
        if case["kind"] == "probs":                     # only the row at the stop is read whole
            needed = len(rows)
        noise = len(rows) if case["kind"] == "probs" else sum(s % 8 != 5 for s in range(len(rows)))
        return dict(bytes=v * (size * needed + 4 * noise + (4 * refused if case["dense"] else 0)), flops=v * 5 * needed)
    tokens = sum(_ints(case, case["seqs"], case["ctx_lo"], case["ctx_hi"], 0))
    return dict(bytes=4 * tokens + 4 * case["seqs"] * (case["drafts"] + 2), flops=tokens)


# ------------------------------------------------------------------ 64-bit definitions
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(st)
    if case["op"] == "verify":
        return _exact_verify(st)
    return None                                         # whole numbers only


def _exact_norm(st):
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    half = d // 2
    if case["interleaved"]:
        first, second = torch.arange(0, d, 2, device="cuda"), torch.arange(1, d, 2, device="cuda")
    else:
        first, second = torch.arange(half, device="cuda"), torch.arange(half, d, device="cuda")
    k_pool, v_pool = st["k_pool"].double(), st["v_pool"].double()
    q = torch.empty(st["q_out"].shape, dtype=torch.float64, device="cuda")
    start = 0
    for s, (c, n) in enumerate(zip(st["h_cached"], st["h_new"])):
        x = st["qkv"][start:start + n].double().reshape(n, hq + 2 * hkv, d)
        place = torch.arange(c, c + n, device="cuda")
        table = st["rope_table"][c:c + n].double()
        turn = torch.complex(table[:, :half], table[:, half:])[:, None, :]
        page, slot = st["table"][s, place // 16].long(), place % 16

        def turned(x, weight):
            x = x / (x.square().sum(-1, keepdim=True) / d + EPS).sqrt() * weight.double()
            z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
            y = torch.empty_like(x)
            y[..., first], y[..., second] = z.real, z.imag
            return y
        q[start:start + n] = turned(x[:, :hq], st["q_weight"])
        k_pool[page, :, slot] = turned(x[:, hq:hq + hkv], st["k_weight"])
        v_pool[page, :, slot] = x[:, hq + hkv:]
        start += n
    return dict(q=q, k_pool=k_pool, v_pool=v_pool)


def _exact_verify(st):
    """Sequence by sequence, row by row, as the rule reads; only the log-probabilities are computed numbers."""
    case = st["case"]
    bounds, tokens, uniform = st["indptr"].tolist(), st["tokens"].tolist(), st["uniform"].double().tolist()
    temperature = st["temperature"].tolist() if "temperature" in st else [None] * case["seqs"]
    logprobs = torch.zeros(st["logprobs"].shape, dtype=torch.float64)
    for s in range(case["seqs"]):
        for i, row in enumerate(range(bounds[s], bounds[s + 1])):
            t = st["target"][row].double()
            if case["kind"] == "probs":
                logp = t.log()
            else:
                logp = torch.log_softmax(t / temperature[s] if temperature[s] else t, 0)
            draft = tokens[row + 1] if row + 1 < bounds[s + 1] else None
            q = st["draft_probs"][row].double() if "draft_probs" in st else None
            if draft is not None:
                if temperature[s] == 0:
                    taken = int(t.argmax()) == draft
                else:
                    taken = uniform[row] * (float(q[draft]) if q is not None else 1.0) < math.exp(float(logp[draft]))
                if taken:
                    logprobs[s, i] = logp[draft]
                    continue
            p = logp.exp()
            left = p
            if draft is not None and q is not None:
                left = (p - q).clamp(min=0)
            elif draft is not None:
                left = p.clone()
                left[draft] = 0
            if not float(left.max()) > 0:
                left = p
            pick = t if temperature[s] == 0 else left / st["noise"][s].double()
            logprobs[s, i] = logp[int(pick.argmax())]
            break
    return dict(accepted=None, next=None, out=None, logprobs=logprobs.cuda())
