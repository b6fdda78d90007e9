"""Timed cases of a step over a KV cache held in 4 bits: the append that quantises, pages read back, attention of one or several
new tokens a sequence, block tables and slot maps from request lengths, logits with penalties, biases and grammar masks.  Each case
goes through its plain form (elementary torch operations, fp32) or, with `own`, through the library."""
import math
import random

import torch

own = False

EPS = 1e-6
K_SCALE, V_SCALE = 0.5, 0.25                # of the pools: powers of two


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one generated token of 64 users of a grouped-query coder model; what was stored is read back
        dict(name="append_decode", op="append", seqs=64, new_lo=1, new_hi=1, ctx_lo=1024, ctx_hi=16384, hq=28, hkv=4, dim=128,
             interleaved=False, norm=False, lengths=1),
        # 16 users with up to eight drafted tokens each, normalised q and k heads, small heads, pairs side by side
        dict(name="append_drafts", op="append", seqs=16, new_lo=1, new_hi=9, ctx_lo=300, ctx_hi=4000, hq=4, hkv=4, dim=64,
             interleaved=True, norm=True, lengths=2),
        # suffixes recomputed after a cache miss: the largest append
        dict(name="append_miss", op="append", seqs=8, new_lo=3200, new_hi=3200, ctx_lo=5120, ctx_hi=5120, hq=32, hkv=8, dim=128,
             interleaved=False, norm=True, lengths=3),
        # one user, one generated token: the smallest attention
        dict(name="attend_one", op="attend", seqs=1, new_lo=1, new_hi=1, ctx_lo=2300, ctx_hi=2300, hq=32, hkv=8, dim=128, lengths=4),
        # a decode step of 64 users, contexts of very different lengths
        dict(name="attend_users", op="attend", seqs=64, new_lo=1, new_hi=1, ctx_lo=1024, ctx_hi=16384, hq=32, hkv=8, dim=128, lengths=5),
        # a step with up to four drafted tokens a user
        dict(name="attend_drafts", op="attend", seqs=37, new_lo=1, new_hi=5, ctx_lo=500, ctx_hi=8000, hq=28, hkv=4, dim=128, lengths=6),
        # a turn: increments of 32 to 256 tokens over 2k to 8k cached ones
        dict(name="attend_turn", op="attend", seqs=16, new_lo=32, new_hi=256, ctx_lo=2048, ctx_hi=8192, hq=32, hkv=8, dim=128, lengths=7),
        # pages and slots of a step of 16 users with up to eight drafted tokens each
        dict(name="tables_drafts", op="tables", seqs=16, new_lo=1, new_hi=9, ctx_lo=300, ctx_hi=16000, width=1024, lengths=8),
        # pages and slots of the prompts of 512 requests that come in at once
        dict(name="tables_prompts", op="tables", seqs=512, new_lo=32, new_hi=512, ctx_lo=0, ctx_hi=8192, width=1024, lengths=9),
        # penalties for one user, fp32 logits, an odd vocabulary
        dict(name="logits_one", op="logits", seqs=1, lo=1, hi=1, vocab=32003, kind="f32", ctx_lo=2300, ctx_hi=2300, mask=False, bias=16,
             lengths=10),
        # 16 users with four drafted tokens each, a grammar and biases
        dict(name="logits_users", op="logits", seqs=16, lo=5, hi=5, vocab=131072, kind="bf16", ctx_lo=1024, ctx_hi=16384, mask=True, bias=300,
             lengths=11),
        # a full server: 256 users, up to five rows each
        dict(name="logits_many", op="logits", seqs=256, lo=1, hi=5, vocab=131072, kind="bf16", ctx_lo=1024, ctx_hi=16384, mask=True, bias=32,
             lengths=12),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "attend", "tables", "logits", "logits"))
    lengths = rng.randrange(1 << 20)
    if op == "append":
        hkv, group = rng.choice(((1, 16), (4, 1), (4, 7), (8, 4), (8, 5), (32, 1), (3, 3)))
        dim = rng.choice((64, 128))
        total = _log_int(rng, 1, min(20000, 150000000 // ((group + 2) * hkv * dim)))
        seqs = _log_int(rng, 1, min(total, 256))
        hi = max(1, total // seqs)
        return dict(op=op, seqs=seqs, new_lo=rng.randint(1, hi), new_hi=hi, ctx_lo=rng.randint(0, 500), ctx_hi=_log_int(rng, 500, 8192),
                    hq=hkv * group, hkv=hkv, dim=dim, interleaved=rng.random() < 0.3, norm=rng.random() < 0.5, lengths=lengths)
    if op == "attend":
        hkv, group = rng.choice(((1, 16), (4, 1), (4, 7), (8, 4), (8, 5), (32, 1), (3, 3), (2, 24)))
        dim = rng.choice((64, 128))
        new = rng.choice((1, 1, _log_int(rng, 2, 9), _log_int(rng, 10, 256)))
        hi = _log_int(rng, 16, 16384)
        top = 64 * 16384 * 8 * 128 // (hi * hkv * dim)                     # as many cached values as the largest listed case
        scores = 16 * 256 * 32 * 8448 // (new * hkv * group * (hi + new))   # and scores
        return dict(op=op, seqs=_log_int(rng, 1, max(1, min(64, top, scores))), new_lo=rng.randint(1, new), new_hi=new, ctx_lo=rng.randint(0, hi),
                    ctx_hi=hi, hq=hkv * group, hkv=hkv, dim=dim, lengths=lengths)
    if op == "tables":
        hi = _log_int(rng, 1, 512)
        ctx = _log_int(rng, 16, 16000)
        return dict(op=op, seqs=_log_int(rng, 1, 512), new_lo=rng.randint(0, hi), new_hi=hi, ctx_lo=rng.randint(0, ctx), ctx_hi=ctx,
                    width=(ctx + hi + 15) // 16 + rng.randint(0, 64), lengths=lengths)
    vocab = _log_int(rng, 1000, 131072)
    hi = rng.randint(1, 9)
    seqs = _log_int(rng, 1, 256)
    kind = rng.choice(("bf16", "bf16", "f32"))
    while seqs * hi * vocab > (768 if kind == "bf16" else 384) * 131072:
        seqs //= 2
    top = _log_int(rng, 1, 16384)
    return dict(op=op, seqs=seqs, lo=rng.randint(1, hi), hi=hi, vocab=vocab, kind=kind, ctx_lo=rng.randint(1, top), ctx_hi=top,
                mask=rng.random() < 0.5, bias=_log_int(rng, 1, 300) - 1, lengths=lengths)


def _ints(case, seqs, lo, hi, tag):
    r = random.Random(case["lengths"] * 4 + tag)
    return [r.randint(lo, hi) for _ in range(seqs)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _indptr(counts):
    return torch.tensor([0] + list(counts), device="cuda").cumsum(0).to(torch.int32)


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    return dict(append=_prepare_append, attend=_prepare_attend, tables=_prepare_tables, logits=_prepare_logits)[case["op"]](case, seed)


def _rope_table(dim, positions):
    theta = 10000.0 ** (-2.0 * torch.arange(dim // 2, dtype=torch.float64) / dim)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * theta
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _prepare_append(case, seed):
    """One projection's output [tokens, (hq + 2 hkv) dim]; a pool of the pages that the step writes, in any order."""
    g = _gen(seed)
    b, hq, hkv, d = case["seqs"], case["hq"], case["hkv"], case["dim"]
    cached = _ints(case, b, case["ctx_lo"], case["ctx_hi"], 0)
    new = _ints(case, b, case["new_lo"], case["new_hi"], 1)
    pages = [(c + n + 15) // 16 for c, n in zip(cached, new)]
    first = [c // 16 for c in cached]
    mine = [p - f for p, f in zip(pages, first)]
    perm = torch.randperm(sum(mine), generator=g, device="cuda").to(torch.int32)
    table = torch.full((b, max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s in range(b):
        table[s, first[s]:pages[s]] = perm[at:at + mine[s]]
        at += mine[s]
    tokens = sum(new)
    qkv = torch.randn(tokens, (hq + 2 * hkv) * d, generator=g, device="cuda")
    qkv *= 1 + 3 * (torch.rand(qkv.shape[1], generator=g, device="cuda") < 0.05)       # channels that stand out
    st = dict(case=case, qkv=qkv.bfloat16(), cached=_i32(cached), new=_i32(new), indptr=_indptr(new), h_cached=cached, h_new=new,
              table=table, rope_table=_rope_table(d, max(c + n for c, n in zip(cached, new))).cuda(),
              q_weight=(1 + 0.2 * torch.randn(d, generator=g, device="cuda")).bfloat16(),
              k_weight=(1 + 0.2 * torch.randn(d, generator=g, device="cuda")).bfloat16(),
              q_out=torch.empty(tokens, hq, d, dtype=torch.bfloat16, device="cuda"))
    st.update(_pools(g, sum(mine), hkv, d))
    st["pages"] = torch.arange(sum(mine), dtype=torch.int32, device="cuda")
    st["k_read"], st["v_read"] = (torch.empty(sum(mine), hkv, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return st


def _pools(g, pages, hkv, d):
    """Codes of any value, scales of blocks whose largest value is about 1 to 4."""
    st = {}
    for x in "kv":
        st[x + "_codes"] = torch.randint(256, (pages, hkv, 16, d // 2), generator=g, device="cuda", dtype=torch.uint8)
        scale = (0.15 + 0.5 * torch.rand(pages, hkv, 16, d // 16, generator=g, device="cuda")) / (K_SCALE if x == "k" else V_SCALE)
        st[x + "_scales"] = scale.to(torch.float8_e4m3fn).view(torch.uint8)
    return st


def _prepare_attend(case, seed):
    """A shuffled pool, new tokens already in it, block tables with -1 past each sequence's end."""
    g = _gen(seed)
    b, hq, hkv, d = case["seqs"], case["hq"], case["hkv"], case["dim"]
    cached = _ints(case, b, case["ctx_lo"], case["ctx_hi"], 0)
    new = _ints(case, b, case["new_lo"], case["new_hi"], 1)
    pages = [(c + n + 15) // 16 for c, n in zip(cached, new)]
    perm = torch.randperm(sum(pages), generator=g, device="cuda").to(torch.int32)
    table = torch.full((b, max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s in range(b):
        table[s, :pages[s]] = perm[at:at + pages[s]]
        at += pages[s]
    q = torch.randn(sum(new), hq, d, generator=g, device="cuda").bfloat16()
    return dict(case=case, q=q, out=torch.empty_like(q), table=table, cached=_i32(cached), new=_i32(new), indptr=_indptr(new),
                ctx=_i32([c + n for c, n in zip(cached, new)]), h_cached=cached, h_new=new, **_pools(g, sum(pages), hkv, d))


def _prepare_tables(case, seed):
    """Tables that hold the pages of the cached tokens (and now and then one more, left by a refused draft); a stack of free pages."""
    g = _gen(seed)
    b, width = case["seqs"], case["width"]
    cached = _ints(case, b, case["ctx_lo"], case["ctx_hi"], 0)
    new = _ints(case, b, case["new_lo"], case["new_hi"], 1)
    tokens = sum(new)
    have = (_i32(cached) + 15) // 16 + (torch.rand(b, generator=g, device="cuda") < 0.3)
    place = torch.arange(width, device="cuda")
    pages = torch.randperm(b * width, generator=g, device="cuda").to(torch.int32)
    table = torch.where(place < have[:, None], pages.view(b, width), -1)
    free = torch.randperm(b * width, generator=g, device="cuda").to(torch.int32) + b * width
    count = sum((c + n + 15) // 16 - (c + 15) // 16 for c, n in zip(cached, new)) + b
    room = tokens + case["seqs"]                                            # rows of a step of fixed size, some of them unused
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(case=case, cached=_i32(cached), new=_i32(new), table=table, free=free, count=_i32([min(count, b * width)]), room=room,
                table_out=torch.empty(b, width, **i32), count_out=torch.empty(1, **i32), indptr=torch.empty(b + 1, **i32),
                positions=torch.empty(room, **i32), sequences=torch.empty(room, **i32),
                slots=torch.empty(room, dtype=torch.int64, device="cuda"))


def _prepare_logits(case, seed):
    """Histories of a working vocabulary that repeats itself, a prompt of about half of each; grammars that let pass all, or one token in
    fifty; biases of both signs, some of them -inf."""
    g = _gen(seed)
    rows = _ints(case, case["seqs"], case["lo"], case["hi"], 0)
    lens = _ints(case, case["seqs"], case["ctx_lo"], case["ctx_hi"], 1)
    b, r, v = len(rows), sum(rows), case["vocab"]
    logits = 3 * torch.randn(r, v, generator=g, device="cuda")
    words = torch.randint(v, (b, max(1, min(v, 2000))), generator=g, device="cuda", dtype=torch.int32)
    pick = (torch.rand(b, max(lens), generator=g, device="cuda") ** 2 * words.shape[1]).long()
    st = dict(case=case, logits=logits.bfloat16() if case["kind"] == "bf16" else logits, indptr=_indptr(rows), history=words.gather(1, pick),
              lens=_i32(lens), prompt=_i32([n // 2 for n in lens]),
              repetition=1 + 0.3 * torch.rand(b, generator=g, device="cuda"),
              frequency=0.2 * torch.rand(b, generator=g, device="cuda"), presence=0.5 * torch.rand(b, generator=g, device="cuda"))
    seq = torch.repeat_interleave(torch.arange(b, device="cuda"), torch.tensor(rows, device="cuda"), output_size=r)
    st["tokens"] = words[seq, torch.randint(words.shape[1], (r,), generator=g, device="cuda")]
    st["out"] = torch.empty_like(st["logits"])
    if case["bias"]:
        n = min(case["bias"], v)
        st["bias_indptr"] = _indptr([n] * b)
        st["bias_tokens"] = torch.rand(b, v, generator=g, device="cuda").topk(n, 1)[1].flatten().to(torch.int32)
        st["bias"] = torch.where(torch.rand(b * n, generator=g, device="cuda") < 0.1, -math.inf, 2 * torch.randn(b * n, generator=g, device="cuda"))
    if case["mask"]:
        width = (v + 31) // 32
        some = torch.rand(r, 1, generator=g, device="cuda") < 0.5
        bit = torch.ones(1, dtype=torch.int64, device="cuda") << torch.randint(32, (r, width), generator=g, device="cuda")
        few = torch.where(torch.rand(r, width, generator=g, device="cuda") < 0.6, bit, 0)
        st["mask"] = torch.where(some, few, 0xffffffff).to(torch.uint32).view(torch.int32)
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    forms = _OWN if own else _PLAIN
    return forms[state["case"]["op"]](state)


def _library(st):
    """The library's descriptors of a state and its workspace, made on the first pass and kept, as a serving loop keeps them."""
    if "own" not in st:
        import paper_2505_21889_b200 as efim
        st["own"], st["status"] = efim, torch.zeros(1, dtype=torch.int32, device="cuda")
        case = st["case"]

        def bytes_of(n):
            return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
        if case["op"] in ("append", "attend"):
            st["cache"] = efim.Cache4(st["k_codes"], st["v_codes"], st["k_scales"], st["v_scales"], case["hq"], K_SCALE, V_SCALE)
            st["batch"] = efim.Batch(st["h_cached"], st["h_new"], st["table"])
        if case["op"] == "append":
            st["rope"] = efim.Rope.from_table(st["rope_table"], case["interleaved"])
            st["norm"] = efim.QkNorm(st["q_weight"], st["k_weight"], EPS) if case["norm"] else None
            st["split"] = st["qkv"].split([case["hq"] * case["dim"], case["hkv"] * case["dim"], case["hkv"] * case["dim"]], 1)
        if case["op"] == "attend":
            st["most"] = max(c + n for c, n in zip(st["h_cached"], st["h_new"]))
            if case["new_hi"] <= 9:
                st["ws"] = bytes_of(efim.efim_kv4_decode_workspace_bytes(st["cache"], case["seqs"], case["new_hi"], st["most"]))
            else:
                st["ws"] = bytes_of(efim.efim_kv4_prefill_workspace_bytes(st["cache"], st["batch"]))
        if case["op"] == "tables":
            st["ws"] = bytes_of(efim.efim_step_tables_workspace_bytes(case["seqs"]))
    return st["own"]


def _own_append(st):
    efim = _library(st)
    q, k, v = st["split"]
    efim.efim_kv4_append(st["cache"], st["batch"], st["norm"], st["rope"], q, k, v, st["q_out"], st["status"])
    efim.efim_kv4_unpack(st["cache"], st["pages"], st["k_read"], st["v_read"], st["status"])
    return dict(q=st["q_out"], k=st["k_read"], v=st["v_read"])


def _own_attend(st):
    efim, case = _library(st), st["case"]
    if case["new_hi"] == 1:
        efim.efim_kv4_decode_attn(st["cache"], case["seqs"], st["ctx"], st["most"], st["table"], st["q"], st["out"], workspace=st["ws"],
                                  status=st["status"])
    elif case["new_hi"] <= 9:
        efim.efim_kv4_decode_attn(st["cache"], case["seqs"], st["ctx"], st["most"], st["table"], st["q"], st["out"],
                                  q_indptr=st["indptr"], max_new_len=case["new_hi"], workspace=st["ws"], status=st["status"])
    else:
        efim.efim_kv4_append_prefill_attn(st["cache"], st["batch"], st["q"], st["out"], workspace=st["ws"], status=st["status"])
    return dict(out=st["out"])


def _own_tables(st):
    efim = _library(st)
    efim.efim_step_tables(st["cached"], st["new"], st["table"], st["free"], st["count"], st["indptr"], st["positions"], st["slots"],
                          st["sequences"], block_table_out=st["table_out"], num_free_out=st["count_out"], workspace=st["ws"],
                          status=st["status"])
    return dict(table=st["table_out"], count=st["count_out"], indptr=st["indptr"], positions=st["positions"], slots=st["slots"],
                sequences=st["sequences"])


def _own_logits(st):
    efim = _library(st)
    bias = (st["bias_indptr"], st["bias_tokens"], st["bias"]) if "bias" in st else None
    efim.efim_adjust_logits(st["indptr"], st["logits"], st["out"], history=st["history"], lengths=st["lens"], prompt_len=st["prompt"],
                            tokens=st["tokens"], repetition=st["repetition"], frequency=st["frequency"], presence=st["presence"], bias=bias,
                            mask=st.get("mask"), status=st["status"])
    return dict(logits=st["out"])


def _codes_of(x, scale):
    """What a pool of this scale holds of x [.., dims].  In 64 bits: a value on the border between two goes to the right one."""
    x = x.double().unflatten(-1, (-1, 16)) / scale
    s = (x.abs().amax(-1, keepdim=True) / 6).clamp(2.0 ** -9, 448.0).float().to(torch.float8_e4m3fn).double()
    y = x / s
    a = y.abs()
    # the borders between the values 0, 0.5, 1, 1.5, 2, 3, 4, 6; a border itself goes to the neighbour with the even code
    held = 0.5 * ((a > 0.25).double() + (a >= 0.75) + (a > 1.25) + (a >= 1.75)) + (a > 2.5).double() + (a >= 3.5) + 2 * (a > 5).double()
    return (torch.where(y < 0, -held, held) * s * scale).flatten(-2)


def _plain_append(st):
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    tokens = st["qkv"].shape[0]
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), st["new"], output_size=tokens)
    pos = st["cached"][seq] + torch.arange(tokens, device="cuda") - st["indptr"][seq]
    table = st["rope_table"][pos][:, None, :]
    x = st["qkv"].float().view(tokens, hq + 2 * hkv, d)

    def turned(x, weight):
        cos, sin = table.to(x.dtype).split(d // 2, 2)
        if case["norm"]:
            x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * weight.to(x.dtype)
        if case["interleaved"]:
            a, b = x[:, :, 0::2], x[:, :, 1::2]
            return torch.stack([a * cos - b * sin, b * cos + a * sin], 3).flatten(2).bfloat16()
        a, b = x.split(d // 2, 2)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], 2).bfloat16()

    k, v = _values(st, "k", K_SCALE).bfloat16(), _values(st, "v", V_SCALE).bfloat16()
    page, slot = st["table"][seq, pos // 16].long(), pos % 16
    k[page, :, slot] = _codes_of(turned(x[:, hq:hq + hkv].double(), st["k_weight"]), K_SCALE).bfloat16()
    v[page, :, slot] = _codes_of(x[:, hq + hkv:], V_SCALE).bfloat16()
    return dict(q=turned(x[:, :hq], st["q_weight"]), k=k, v=v)


def _values(st, x, scale, pages=None):
    """Held values of a pool, or of some pages of it, in fp32: [pages, kv heads, 16, dims]."""
    codes, scales = st[x + "_codes"], st[x + "_scales"]
    if pages is not None:
        codes, scales = codes[pages], scales[pages]
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    both = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).flatten(-2)
    return (both.unflatten(-1, (-1, 16)) * (scales.view(torch.float8_e4m3fn).float() * scale)[..., None]).flatten(-2)


def _plain_attend(st):
    case = st["case"]
    b, hq, hkv, d = case["seqs"], case["hq"], case["hkv"], case["dim"]
    tokens, most = st["q"].shape[0], max(st["h_new"])
    seq = torch.repeat_interleave(torch.arange(b, device="cuda"), st["new"], output_size=tokens)
    i = torch.arange(tokens, device="cuda") - st["indptr"][seq]
    q = torch.zeros(b, most, hq, d, device="cuda")
    q[seq, i] = st["q"].float()
    q = q.view(b, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).flatten(2, 3)              # [b, hkv, group * new, d]
    pages = st["table"].long().clamp(min=0)
    k, v = (_values(st, x, s, pages).transpose(1, 2).flatten(2, 3) for x, s in (("k", K_SCALE), ("v", V_SCALE)))
    scores = (q @ k.transpose(2, 3)) * d ** -0.5
    key = torch.arange(k.shape[2], device="cuda")
    seen = key <= (st["cached"][:, None] + torch.arange(most, device="cuda"))[:, :, None]       # [b, new, keys]
    seen &= (key < st["ctx"][:, None])[:, None]
    scores = scores.unflatten(2, (-1, most)).masked_fill_(~seen[:, None, None], -math.inf)
    scores = torch.exp_(scores.sub_(scores.amax(-1, keepdim=True)))
    total = scores.sum(-1, keepdim=True)
    out = (scores.flatten(2, 3) @ v).unflatten(2, (-1, most)) / total
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)                                              # [b, new, hq, d]
    return dict(out=out[seq, i].bfloat16())


def _plain_tables(st):
    case, table, room = st["case"], st["table"], st["room"]
    b, width = table.shape
    cached, new = st["cached"].long(), st["new"].long()
    place = torch.arange(width, device="cuda")
    wanted = (place >= ((cached + 15) // 16)[:, None]) & (place < ((cached + new + 15) // 16)[:, None]) & (table < 0)
    rank = wanted.flatten().cumsum(0) - 1
    got = wanted.flatten() & (rank < st["count"])
    pages = st["free"][(st["count"] - 1 - rank).clamp(min=0)]
    table = torch.where(got, pages, table.flatten()).view(b, width)
    indptr = torch.cat([torch.zeros_like(new[:1]), new.cumsum(0)])
    row = torch.arange(room, device="cuda")
    seq = (torch.searchsorted(indptr, row, right=True) - 1).clamp(max=b - 1)
    inside = row < indptr[-1]
    pos = cached[seq] + row - indptr[seq]
    page = table[seq, (pos // 16).clamp(max=width - 1)].long()
    slots = torch.where(inside & (page >= 0), page * 16 + pos % 16, -1)
    return dict(table=table, count=(st["count"] - wanted.sum()).clamp(min=0).int(), indptr=indptr.int(),
                positions=torch.where(inside, pos, -1).int(), slots=slots, sequences=torch.where(inside, seq, -1).int())


def _plain_logits(st):
    case, v = st["case"], st["case"]["vocab"]
    r, b = st["logits"].shape[0], case["seqs"]
    indptr, hist = st["indptr"].long(), st["history"].long()
    row = torch.arange(r, device="cuda")
    seq = torch.searchsorted(indptr, row, right=True) - 1
    at = torch.arange(hist.shape[1], device="cuda")
    written = (at >= st["prompt"][:, None]) & (at < st["lens"][:, None])
    counts = torch.zeros(b, v, dtype=torch.int32, device="cuda").scatter_add_(1, hist, written.int())
    prompt = torch.zeros(b, v, dtype=torch.int32, device="cuda").scatter_add_(1, hist, (at < st["prompt"][:, None]).int())
    # a row also counts the drafts before it: the tokens behind its sequence's first, up to its own
    back = row[:, None] - torch.arange(case["hi"], device="cuda")
    counts = counts[seq].scatter_add_(1, st["tokens"].long()[back.clamp(min=0)], (back > indptr[seq][:, None]).int())
    x = st["logits"].float()
    each = lambda name: st[name][seq][:, None]  # noqa: E731
    x = torch.where((counts > 0) | (prompt[seq] > 0), torch.where(x > 0, x / each("repetition"), x * each("repetition")), x)
    x = x - each("frequency") * counts - each("presence") * (counts > 0)
    if "bias" in st:
        dense = torch.zeros(b, v, device="cuda")
        dense[torch.arange(b, device="cuda").repeat_interleave(len(st["bias"]) // b), st["bias_tokens"].long()] = st["bias"]
        x = x + dense[seq]
    if "mask" in st:
        j = torch.arange(v, device="cuda")
        x = torch.where((st["mask"][:, j // 32] >> (j % 32).int()) & 1 > 0, x, -math.inf)
    return dict(logits=x.to(st["logits"].dtype))


_OWN = dict(append=_own_append, attend=_own_attend, tables=_own_tables, logits=_own_logits)
_PLAIN = dict(append=_plain_append, attend=_plain_attend, tables=_plain_tables, logits=_plain_logits)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    b = case["seqs"]
    if case["op"] == "append":
        new = _ints(case, b, case["new_lo"], case["new_hi"], 1)
        cached = _ints(case, b, case["ctx_lo"], case["ctx_hi"], 0)
        q, kv = sum(new) * case["hq"] * case["dim"], sum(new) * 2 * case["hkv"] * case["dim"]
        slots = sum((c + n + 15) // 16 - c // 16 for c, n in zip(cached, new)) * 16
        read = slots * 2 * case["hkv"] * case["dim"]                        # pages, written to or not, read back
        return dict(bytes=4 * q + kv * (2 + 9 / 16) + read * (2 + 9 / 16) + 4 * sum(new) * case["dim"], flops=8 * (q + kv))
    if case["op"] == "attend":
        new = _ints(case, b, case["new_lo"], case["new_hi"], 1)
        cached = _ints(case, b, case["ctx_lo"], case["ctx_hi"], 0)
        keys = sum(c + n for c, n in zip(cached, new))
        pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(cached, new))
        return dict(bytes=keys * case["hkv"] * case["dim"] * 2 * 9 / 16 + 4 * sum(new) * case["hq"] * case["dim"],
                    flops=4 * pairs * case["hq"] * case["dim"])
    if case["op"] == "tables":
        rows = sum(_ints(case, b, case["new_lo"], case["new_hi"], 1)) + b
        return dict(bytes=8 * b * case["width"] + 16 * rows + 12 * b, flops=0)
    rows = sum(_ints(case, b, case["lo"], case["hi"], 0))
    tokens = sum(_ints(case, b, case["ctx_lo"], case["ctx_hi"], 1))
    size = 2 if case["kind"] == "bf16" else 4
    return dict(bytes=rows * case["vocab"] * (2 * size + (0.125 if case["mask"] else 0)) + 4 * tokens + 8 * b * case["bias"],
                flops=2 * rows * case["vocab"])


# ------------------------------------------------------------------ 64-bit definitions
def exact(case, seed):
    if case["op"] == "tables":
        return None                                     # whole numbers only
    st = prepare(case, seed)
    return dict(append=_exact_append, attend=_exact_attend, logits=_exact_logits)[case["op"]](st)


def _e2m1(code):
    """The value of a code, by its sign, exponent and mantissa bits."""
    exponent, mantissa = (code >> 1) & 3, (code & 1).double()
    size = torch.where(exponent == 0, mantissa / 2, (1 + mantissa / 2) * (1 << exponent) / 2)
    return torch.where(code >= 8, -size, size)


def _e4m3(byte):
    byte = byte.long()
    exponent, mantissa = (byte >> 3) & 15, (byte & 7).double()
    return torch.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * (1 << exponent) * 2.0 ** -10)


def _exact_values(codes, scales, scale):
    codes = codes.long()
    x = torch.stack([_e2m1(codes % 16), _e2m1(codes // 16)], -1).reshape(*scales.shape, 16)
    return (x * _e4m3(scales)[..., None] * scale).reshape(*codes.shape[:-1], -1)


def _nearest(x, values):
    """The nearest of some ascending values, of two alike the one at an even place."""
    hi = torch.searchsorted(values, x.contiguous()).clamp(1, len(values) - 1)
    lo = hi - 1
    down, up = x - values[lo], values[hi] - x
    return torch.where((down < up) | ((down == up) & (lo % 2 == 0)), values[lo], values[hi])


def _exact_held(x, scale):
    e4m3 = _e4m3(torch.arange(127, device="cuda"))
    e2m1 = _e2m1(torch.arange(8, device="cuda"))
    x = x.reshape(*x.shape[:-1], -1, 16) / scale
    s = _nearest(x.abs().amax(-1), 6 * e4m3).clamp(min=6 * 2.0 ** -9)[..., None] * 0.5 / 3      # (6 times the scale: no quotient is rounded)
    s = s.float().double()
    return (torch.sign(x) * _nearest(x.abs() / s, e2m1) * s * scale).flatten(-2)


def _exact_append(st):
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    half = d // 2
    if case["interleaved"]:
        first, second = torch.arange(0, d, 2, device="cuda"), torch.arange(1, d, 2, device="cuda")
    else:
        first, second = torch.arange(half, device="cuda"), torch.arange(half, d, device="cuda")
    k = _exact_values(st["k_codes"], st["k_scales"], K_SCALE)
    v = _exact_values(st["v_codes"], st["v_scales"], V_SCALE)
    q = torch.empty(st["q_out"].shape, dtype=torch.float64, device="cuda")
    start = 0
    for s, (c, n) in enumerate(zip(st["h_cached"], st["h_new"])):
        x = st["qkv"][start:start + n].double().reshape(n, hq + 2 * hkv, d)
        place = torch.arange(c, c + n, device="cuda")
        table = st["rope_table"][c:c + n].double()
        turn = torch.complex(table[:, :half], table[:, half:])[:, None, :]
        page, slot = st["table"][s, place // 16].long(), place % 16

        def turned(x, weight):
            if case["norm"]:
                x = x / (x.square().sum(-1, keepdim=True) / d + EPS).sqrt() * weight.double()
            z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
            y = torch.empty_like(x)
            y[..., first], y[..., second] = z.real, z.imag
            return y
        q[start:start + n] = turned(x[:, :hq], st["q_weight"])
        # keys are rounded to bf16, then to the block's values
        k[page, :, slot] = _exact_held(turned(x[:, hq:hq + hkv], st["k_weight"]).bfloat16().double(), K_SCALE)
        v[page, :, slot] = _exact_held(x[:, hq + hkv:], V_SCALE)
        start += n
    return dict(q=q, k=k, v=v)


def _exact_attend(st):
    case = st["case"]
    group, d = case["hq"] // case["hkv"], case["dim"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    start = 0
    for s, (c, n) in enumerate(zip(st["h_cached"], st["h_new"])):
        pages = st["table"][s, :(c + n + 15) // 16].long()
        for h in range(case["hkv"]):
            k, v = (_exact_values(st[x + "_codes"][pages, h], st[x + "_scales"][pages, h], scale).reshape(-1, d)[:c + n]
                    for x, scale in (("k", K_SCALE), ("v", V_SCALE)))
            q = st["q"][start:start + n, h * group:(h + 1) * group].double()
            scores = torch.einsum("ngd,kd->gnk", q, k) / math.sqrt(d)
            ahead = torch.ones(n, c + n, dtype=torch.bool, device="cuda").triu(c + 1)
            out[start:start + n, h * group:(h + 1) * group] = torch.einsum("gnk,kd->ngd", scores.masked_fill(ahead, -math.inf).softmax(-1), v)
        start += n
    return dict(out=out)


def _exact_logits(st):
    case, v = st["case"], st["case"]["vocab"]
    bounds, lens, prompt = st["indptr"].tolist(), st["lens"].tolist(), st["prompt"].tolist()
    out = torch.empty(st["logits"].shape, dtype=torch.float64, device="cuda")
    places = torch.arange(v, device="cuda")
    for s in range(case["seqs"]):
        rho, alpha, beta = (float(st[name][s]) for name in ("repetition", "frequency", "presence"))
        before = torch.bincount(st["history"][s, :prompt[s]], minlength=v)
        n = torch.bincount(st["history"][s, prompt[s]:lens[s]], minlength=v).double()
        for row in range(bounds[s], bounds[s + 1]):
            if row > bounds[s]:
                n[int(st["tokens"][row])] += 1
            x = st["logits"][row].double()
            x = torch.where(n + before > 0, torch.where(x > 0, x / rho, x * rho), x) - alpha * n - beta * (n > 0)
            if "bias" in st:
                lo, hi = st["bias_indptr"][s], st["bias_indptr"][s + 1]
                x[st["bias_tokens"][lo:hi].long()] += st["bias"][lo:hi].double()
            if "mask" in st:
                word = st["mask"][row].long() % (1 << 32)
                x[(word[places // 32] >> (places % 32)) % 2 == 0] = -math.inf
            out[row] = x
    return dict(logits=out)
