"""Two operators of batched decoding as measurable cases, each beside its plain form.

  attend   attention of a batch's query rows over the session's paged cache, where the sequences share a long prefix (a
           system prompt, one prompt with many continuations, or a tree of both): the pages that several block tables
           name are read once for all rows that see them
  rules    decoding rules on the rows of an exit head: penalties for repeated tokens, additive biases, temperature and
           bit masks of the allowed tokens, giving the adjusted logits or their softmax, and the arg max

`own` chooses between the plain form (elementary torch operations in 32 bits) and the library's calls.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

PAGE = 64
#        query heads, KV heads, head_dim: the head shapes of the repository's test models and of its benchmark models
HEADS = {"tiny": (4, 4, 64), "small": (8, 2, 64), "8b": (32, 8, 128), "70b": (64, 8, 128)}

ATTEND = {"kind": "attend", "dtype": "bf16", "branch": 0, "groups": 1, "ragged": True}
RULES = {"kind": "rules", "dtype": "f32", "probs": True, "argmax": True, "penalties": True, "bias": 0, "masks": False, "ragged": False}


def listed():
    attend = [
        # four samples of one short prompt, a token each: bound by launches and latency
        dict(name="attend_4_short", heads="8b", batch=4, prefix=500, suffix=40, rows=1),
        # eight requests of a small model (head_dim 64), blocks of five rows, a prefix that ends inside a page
        dict(name="attend_8_small", heads="small", batch=8, prefix=1503, suffix=130, rows=5),
        # thirty-two samples behind one 8k prompt, one token each: the ordinary decoding step
        dict(name="attend_32_8k", heads="8b", batch=32, prefix=8192, suffix=400, rows=1),
        # sixteen requests behind one system prompt, a verify block of nine rows each
        dict(name="attend_16_verify", heads="8b", batch=16, prefix=4100, suffix=600, rows=9),
        # a tree: one system prompt, four conversations, six samples of each, on the wide model's heads
        dict(name="attend_24_tree", heads="70b", batch=24, prefix=6000, branch=2100, groups=4, suffix=200, rows=3),
        # a serving batch behind a long document, blocks of nine rows
        dict(name="attend_64_32k", heads="8b", batch=64, prefix=32768, suffix=500, rows=9),
    ]
    rules = [
        # one row of the repository's small test vocabulary, greedy: the smallest call
        dict(name="rules_1_small", seqs=1, rows=1, vocab=1000, hist=40, probs=False),
        # one request, one token: sampling with every rule on
        dict(name="rules_1_full", seqs=1, rows=1, vocab=128256, hist=2048, bias=40, masks=True),
        # a verify step of sixteen requests, nine rows each, every row with the mask of its place in a grammar
        dict(name="rules_16_verify", seqs=16, rows=9, vocab=128256, hist=1500, bias=20, masks=True, ragged=True),
        # greedy decoding of sixty-four requests with long histories
        dict(name="rules_64_greedy", seqs=64, rows=1, vocab=128256, hist=16000, probs=False, ragged=True),
        # half-width logits of an odd vocabulary
        dict(name="rules_24_bf16", seqs=24, rows=4, vocab=32003, hist=700, dtype="bf16", bias=300, ragged=True),
        # a large batch of sampled requests
        dict(name="rules_512_probs", seqs=512, rows=1, vocab=128256, hist=600, ragged=True, argmax=False),
    ]
    return [{**ATTEND, **c} for c in attend] + [{**RULES, **c} for c in rules]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    if rng.random() < 0.5:
        c = dict(ATTEND, heads=rng.choice(["8b", "8b", "8b", "70b", "small"]))
        c["batch"], c["rows"] = _log_int(rng, 1, 64), rng.choice([1, 1, 2, 4, 9, rng.randint(1, 17)])
        c["prefix"] = 0 if rng.random() < 0.08 else _log_int(rng, 20, 32768)
        c["suffix"] = _log_int(rng, 1, 700)
        c["ragged"] = rng.random() < 0.8
        if c["batch"] >= 6 and rng.random() < 0.3:
            c["groups"], c["branch"] = rng.randint(2, c["batch"] // 2), _log_int(rng, 70, 2000)
        if rng.random() < 0.1:      # the reference-precision models: short contexts, few sequences
            c.update(heads="tiny", dtype="f32", batch=min(c["batch"], 4), prefix=min(c["prefix"], 300), suffix=min(c["suffix"], 100),
                     rows=min(c["rows"], 9), groups=1, branch=0)
        most = work(dict(listed()[5]))
        while True:
            w = work(c)
            if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"]:
                return c
            c["prefix"], c["branch"], c["suffix"] = c["prefix"] // 2, c["branch"] // 2, max(1, c["suffix"] // 2)
    c = dict(RULES, vocab=rng.choice([1000, 32000, 32003, 50257, 128256, _log_int(rng, 300, 128256)]))
    c["rows"] = rng.choice([1, 1, 1, 4, 9, rng.randint(1, 17)])
    c["seqs"] = _log_int(rng, 1, max(1, 512 // c["rows"]))
    c["hist"] = _log_int(rng, 1, 16000)
    c["dtype"] = "bf16" if rng.random() < 0.25 else "f32"
    c["probs"], c["argmax"] = rng.random() < 0.6, rng.random() < 0.7
    c["penalties"], c["masks"], c["ragged"] = rng.random() < 0.8, rng.random() < 0.4, rng.random() < 0.6
    c["bias"] = 0 if rng.random() < 0.5 else _log_int(rng, 1, 300)
    return c


# ---- sizes of a case (the same for every seed) --------------------------------------------------------------------------

def _spread(n, nominal, ragged, lo, salt):
    """n lengths around `nominal`; ragged ones from about a quarter to almost twice of it."""
    if not ragged:
        return [max(lo, nominal)] * n
    r = np.random.default_rng(n * 1009 + nominal * 31 + salt)
    return [int(min(2 * nominal, max(lo, round(nominal * f)))) for f in np.exp(r.normal(-0.15, 0.5, n))]


def _parts(c):
    """Per sequence: (branch number, own positions, rows).  A sequence's context is prefix | branch | own positions, and its rows
    are the last ones of it."""
    rows = [max(1, r) for r in _spread(c["batch"], c["rows"], c["ragged"] and c["rows"] > 4, 1, 5)]
    rows = [min(r, c["rows"]) for r in rows]
    suffix = _spread(c["batch"], c["suffix"], c["ragged"], 1, 7)
    return [(b * c["groups"] // c["batch"], max(suffix[b], rows[b]), rows[b]) for b in range(c["batch"])]


def work(case):
    c = case
    if c["kind"] == "attend":
        hq, hkv, d = HEADS[c["heads"]]
        es = 4 if c["dtype"] == "f32" else 2
        parts = _parts(c)
        shared = c["prefix"] + c["branch"]
        positions = c["prefix"] + (c["branch"] * c["groups"] if c["branch"] else 0) + sum(n for _, n, _ in parts)
        n_rows = sum(m for _, _, m in parts)
        seen = sum(m * (shared + n) - m * (m - 1) // 2 for _, n, m in parts)
        return {"bytes": positions * hkv * d * 2 * es + 2 * n_rows * hq * d * es, "flops": 4 * hq * d * seen}
    n_rows = c["seqs"] * c["rows"]
    values = n_rows * c["vocab"]
    read = values * (2 if c["dtype"] == "bf16" else 4) + (values // 8 if c["masks"] else 0)
    if c["penalties"]:
        read += sum(_spread(c["seqs"], c["hist"], c["ragged"], 1, 3)) * 4
    return {"bytes": read + values * 4 + c["bias"] * c["seqs"] * 8, "flops": values * (8 if c["probs"] else 5)}


# ---- attention ----------------------------------------------------------------------------------------------------------

def _attend_inputs(c, seed):
    """Logical K and V of every part of the tree and the query rows, from the seed alone."""
    hq, hkv, d = HEADS[c["heads"]]
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 11)
    parts = _parts(c)

    def kv(n):
        k = torch.randn((n, hkv, d), generator=g, device="cuda", dtype=torch.float32)
        v = torch.randn((n, hkv, d), generator=g, device="cuda", dtype=torch.float32)
        return k.to(dt), v.to(dt)

    prefix = kv(c["prefix"])
    branches = [kv(c["branch"]) for _ in range(c["groups"] if c["branch"] else 0)]
    suffixes = [kv(n) for _, n, _ in parts]
    # queries of about one and a half times the keys' length: weights that differ by a few powers of e over a context
    q = (1.5 * torch.randn((sum(m for _, _, m in parts), hq, d), generator=g, device="cuda", dtype=torch.float32)).to(dt)
    return parts, prefix, branches, suffixes, q


def _attend_session(c, seed, st):
    """A session whose sequences share the prefix and the branches, holding the case's K and V in one layer."""
    import paper_2510_01336_amd as hs
    hq, hkv, d = HEADS[c["heads"]]
    cfg = SimpleNamespace(n_layers=3, d_model=64, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, d_ffn=64, vocab=512, exit_draft=1,
                          exit_inter=2, rope_theta=1e4, rms_eps=1e-5, dtype=c["dtype"], sigma=0.02)
    r = np.random.default_rng([seed, 77])
    shared = c["prefix"] + c["branch"]
    common = r.integers(0, cfg.vocab, c["prefix"]).astype(np.int32)
    branch = [r.integers(0, cfg.vocab, c["branch"]).astype(np.int32) for _ in range(c["groups"])]
    for grp, t in enumerate(branch):
        t[:1] = 100 + grp                             # (branches part where they begin)
    prompts = []
    for j, (grp, n, _) in enumerate(st.parts):
        tail = r.integers(0, cfg.vocab, n).astype(np.int32)
        tail[0] = j % cfg.vocab                       # (sequences part where their own positions begin)
        prompts.append(np.concatenate([common, branch[grp], tail]))
    model = hs.Model(cfg, 1)
    most = max(len(p) for p in prompts) + 2
    pages = -(-most // PAGE) + sum(-(-(n + c["branch"] + 2 * PAGE) // PAGE) + 1 for _, n, _ in st.parts)
    sess = hs.Session(model, c["batch"], most, max(2, c["rows"] + 1), pages)
    sess.prefill_seq(0, prompts[0])
    leader = {}
    for b, (grp, _, _) in enumerate(st.parts):
        leader.setdefault(grp, b)
    later = [b for b in leader.values() if b != 0]
    if later:                                         # the first sequence of every branch behind the prefix ...
        sess.prefill_shared([0] * c["batch"], [prompts[b] if b in later else None for b in range(c["batch"])])
    rest = [b for b in range(c["batch"]) if b not in leader.values()]
    if rest:                                          # ... and the others behind their branch
        sess.prefill_shared([leader[grp] for grp, _, _ in st.parts], [prompts[b] if b in rest else None for b in range(c["batch"])])
    layer = 1
    for b, (grp, n, _) in enumerate(st.parts):
        own_from = sess.shared_pages(b) * PAGE if b else 0           # (what it shares is written by another sequence)
        k = torch.cat([st.prefix[0]] + ([st.branches[grp][0]] if c["branch"] else []) + [st.suffixes[b][0]])
        v = torch.cat([st.prefix[1]] + ([st.branches[grp][1]] if c["branch"] else []) + [st.suffixes[b][1]])
        if b in leader.values() and b:
            own_from = min(own_from, c["prefix"] // PAGE * PAGE)
        sess.write_kv(b, layer, own_from, k[own_from:].float().cpu().numpy(), v[own_from:].float().cpu().numpy())
    rows = [m for _, _, m in st.parts]
    sess.attend_begin(rows, [shared + n - m for _, n, m in st.parts])
    return SimpleNamespace(model=model, sess=sess, layer=layer)


def _plain_attend(st):
    c = st.case
    hq, hkv, d = HEADS[c["heads"]]
    rep = hq // hkv
    shared_k, shared_v = st.prefix[0].float(), st.prefix[1].float()
    out, r0 = torch.empty_like(st.q), 0
    for b, (grp, n, m) in enumerate(st.parts):
        ks, vs = [shared_k], [shared_v]
        if c["branch"]:
            ks.append(st.branches[grp][0].float())
            vs.append(st.branches[grp][1].float())
        k = torch.cat(ks + [st.suffixes[b][0].float()]).permute(1, 0, 2).contiguous()       # [KV head, position, dim]
        v = torch.cat(vs + [st.suffixes[b][1].float()]).permute(1, 0, 2).contiguous()
        total = k.shape[1]
        q = st.q[r0:r0 + m].float().reshape(m, hkv, rep, d).permute(1, 0, 2, 3).reshape(hkv, m * rep, d)
        s = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        row = torch.arange(m * rep, device="cuda") // rep
        s = s.masked_fill(torch.arange(total, device="cuda")[None, None, :] > (total - m + row)[None, :, None], -math.inf)
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.bmm(p, v) / p.sum(-1, keepdim=True)
        out[r0:r0 + m] = o.reshape(hkv, m, rep, d).permute(1, 0, 2, 3).reshape(m, hq, d).to(out.dtype)
        r0 += m
    return out


def _exact_attend(c, seed):
    parts, prefix, branches, suffixes, q = _attend_inputs(c, seed)
    hq, hkv, d = HEADS[c["heads"]]
    rep = hq // hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    first = 0
    for (grp, n, m), own_kv in zip(parts, suffixes):
        pieces = [prefix] + ([branches[grp]] if branches else []) + [own_kv]
        for h in range(hkv):
            k = torch.cat([x[0][:, h] for x in pieces]).double()
            v = torch.cat([x[1][:, h] for x in pieces]).double()
            for i0 in range(0, m):
                keep = k.shape[0] - m + i0 + 1
                z = (q[first + i0, h * rep:(h + 1) * rep].double() @ k[:keep].T) * d ** -0.5
                out[first + i0, h * rep:(h + 1) * rep] = torch.softmax(z, dim=1) @ v[:keep]
        first += m
    return out


# ---- rules --------------------------------------------------------------------------------------------------------------

def _rules_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 104729 + 5)
    V, S = c["vocab"], c["seqs"]
    n_rows = S * c["rows"]
    st = SimpleNamespace(case=dict(c))
    # an exit head's logits: most of them within a few units, a handful of likely tokens above
    x = torch.randn((n_rows, V), generator=g, device="cuda", dtype=torch.float32) * 2.2
    top = torch.randint(0, V, (n_rows, 8), generator=g, device="cuda")
    x.scatter_add_(1, top, 6.0 * torch.rand((n_rows, 8), generator=g, device="cuda"))
    st.logits = x.to(torch.bfloat16) if c["dtype"] == "bf16" else x
    st.row_start = torch.arange(0, n_rows + 1, c["rows"], dtype=torch.int32, device="cuda")
    st.tokens = st.first_len = st.prompt_len = st.repetition = st.frequency = st.presence = None
    st.bias_start = st.bias_token = st.bias_value = st.allowed = st.allowed_row = None

    def some(lo, hi):
        return lo + (hi - lo) * torch.rand(S, generator=g, device="cuda")

    if c["penalties"]:
        lens = _spread(S, c["hist"], c["ragged"], 1, 3)
        # text repeats itself: few tokens make up most of a history
        u = torch.rand((S, max(lens) + c["rows"]), generator=g, device="cuda")
        st.tokens = (u.pow(4) * V).to(torch.int32).clamp_(max=V - 1)
        st.first_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        st.prompt_len = (st.first_len.float() * some(0.2, 0.9)).to(torch.int32)
        st.repetition, st.frequency, st.presence = some(1.0, 1.4), some(0.0, 0.4), some(0.0, 0.8)
    st.temperature = some(0.6, 1.3)
    if c["bias"]:
        n = c["bias"]
        st.bias_start = torch.arange(0, S * n + 1, n, dtype=torch.int32, device="cuda")
        # distinct tokens of a sequence: one of every run of the vocabulary
        if n <= V:
            run = V // n
            at = torch.arange(n, device="cuda")[None, :] * run + torch.randint(0, run, (S, n), generator=g, device="cuda")
        else:
            at = torch.randint(0, V, (S, n), generator=g, device="cuda")
        st.bias_token = at.to(torch.int32).reshape(-1).contiguous()
        st.bias_value = 4.0 * torch.randn(S * n, generator=g, device="cuda")
    if c["masks"]:
        words = -(-V // 32)
        # places in a grammar: a number, an identifier, free text, and one where nothing may follow
        bits = torch.randint(-2 ** 31, 2 ** 31, (n_rows, words), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
        kind = torch.arange(n_rows, device="cuda") % 4
        rare = torch.randint(0, words, (n_rows, words), generator=g, device="cuda") < 30
        bits = torch.where((kind == 1)[:, None] & ~rare, torch.zeros_like(bits), bits)
        bits = torch.where((kind == 2)[:, None], torch.full_like(bits, -1), bits)
        if n_rows > 8:
            bits[7] = 0
        st.allowed = bits
        st.allowed_row = torch.arange(n_rows, dtype=torch.int32, device="cuda")
        st.allowed_row[n_rows // 2:n_rows // 2 + (1 if n_rows > 8 else 0)] = -1        # a row that anything may follow
    return st


def _plain_rules(st):
    c = st.case
    V, S, m = c["vocab"], c["seqs"], c["rows"]
    x = st.logits.float()
    seq = torch.arange(S, device="cuda").repeat_interleave(m)
    if c["penalties"]:
        ix = torch.arange(st.tokens.shape[1], device="cuda")[None, :]
        known = ix < st.first_len[:, None]
        tok = st.tokens.long()
        whole = torch.zeros((S, V), dtype=torch.int32, device="cuda").scatter_add_(1, tok, known.int())
        said = torch.zeros((S, V), dtype=torch.int32, device="cuda").scatter_add_(1, tok, (known & (ix >= st.prompt_len[:, None])).int())
        whole, said = whole[seq], said[seq]
        if m > 1:                                     # row i also sees the i tokens in front of it
            i = torch.arange(m - 1, device="cuda")[None, :]
            at = st.first_len.long()[:, None] + i
            extra = tok.gather(1, at)[seq]
            count = (i < (torch.arange(S * m, device="cuda") % m)[:, None]).int()
            whole.scatter_add_(1, extra, count)
            said.scatter_add_(1, extra, count)
        rho = st.repetition[seq][:, None]
        x = torch.where(whole > 0, torch.where(x > 0, x / rho, x * rho), x)
        x = x - st.frequency[seq][:, None] * said.float()
        x = x - st.presence[seq][:, None] * (said > 0).float()
    if c["bias"]:
        dense = torch.zeros((S, V), device="cuda")
        dense[torch.arange(S, device="cuda").repeat_interleave(c["bias"]), st.bias_token.long()] = st.bias_value
        x = x + dense[seq]
    x = x / st.temperature[seq][:, None]
    if c["masks"]:
        ids = torch.arange(V, device="cuda")
        words = st.allowed[st.allowed_row.clamp(min=0).long()]
        ok = ((words[:, ids // 32] >> (ids % 32)) & 1).bool() | (st.allowed_row < 0)[:, None]
        x = torch.where(ok, x, torch.full_like(x, -math.inf))
    best = x.amax(-1, keepdim=True)
    out = []
    if c["probs"]:
        e = torch.where(x > -math.inf, torch.exp(x - torch.where(best > -math.inf, best, torch.zeros_like(best))), torch.zeros_like(x))
        total = e.sum(-1, keepdim=True)
        out.append(e / torch.where(total > 0, total, torch.ones_like(total)))
    else:
        out.append(x)
    if c["argmax"]:
        ids = torch.arange(V, device="cuda", dtype=torch.int32)
        first = torch.where((x == best) & (x > -math.inf), ids[None, :], V).amin(-1)
        out.append(torch.where(first < V, first, -1).to(torch.int32))
    return out


def _exact_rules(c, seed):
    st = _rules_inputs(c, seed)
    V, m = c["vocab"], c["rows"]
    values = torch.empty(st.logits.shape, dtype=torch.float64, device="cuda")
    token = []
    for r in range(c["seqs"] * m):
        b, i = divmod(r, m)
        z = st.logits[r].double()
        if c["penalties"]:
            n = int(st.first_len[b]) + i
            past, new = st.tokens[b, :n].long(), st.tokens[b, int(st.prompt_len[b]):n].long()
            rho = float(st.repetition[b])
            met = torch.unique(past)
            z[met] = torch.where(z[met] > 0, z[met] / rho, z[met] * rho)
            which, times = torch.unique(new, return_counts=True)
            z[which] -= float(st.frequency[b]) * times.double() + float(st.presence[b])
        if c["bias"]:
            lo = b * c["bias"]
            z[st.bias_token[lo:lo + c["bias"]].long()] += st.bias_value[lo:lo + c["bias"]].double()
        z = z / float(st.temperature[b])
        if c["masks"] and int(st.allowed_row[r]) >= 0:
            word = st.allowed[int(st.allowed_row[r])]
            bit = (word[:, None] >> torch.arange(32, device="cuda")[None, :]) & 1
            z[bit.reshape(-1)[:V] == 0] = -math.inf
        alive = bool((z > -math.inf).any())
        if c["argmax"]:
            token.append(int((z == z.max()).nonzero()[0]) if alive else -1)
        values[r] = (torch.softmax(z, 0) if alive else torch.zeros_like(z)) if c["probs"] else z
    out = [values]
    if c["argmax"]:
        out.append(torch.tensor(token, dtype=torch.int32, device="cuda"))
    return out


# ---- the calls ----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    c = dict(case)
    if c["kind"] == "attend":
        st = SimpleNamespace(case=c)
        st.parts, st.prefix, st.branches, st.suffixes, st.q = _attend_inputs(c, seed)
        if own:
            st.user = _attend_session(c, seed, st)
        return st
    st = _rules_inputs(c, seed)
    if own:
        import paper_2510_01336_amd as hs
        st.rules = hs.LogitRules(c["vocab"], st.row_start, tokens=st.tokens, first_len=st.first_len, prompt_len=st.prompt_len,
                                 repetition=st.repetition, frequency=st.frequency, presence=st.presence, temperature=st.temperature,
                                 bias_start=st.bias_start, bias_token=st.bias_token, bias_value=st.bias_value, allowed=st.allowed,
                                 allowed_row=st.allowed_row)
    return st


def run(state):
    c = state.case
    if c["kind"] == "attend":
        return state.user.sess.attend(state.user.layer, state.q) if own else _plain_attend(state)
    if not own:
        return _plain_rules(state)
    call = state.rules.probs if c["probs"] else state.rules.logits
    out = call(state.logits, argmax=c["argmax"])
    return list(out) if c["argmax"] else [out]


def exact(case, seed):
    return _exact_attend(case, seed) if case["kind"] == "attend" else _exact_rules(case, seed)
