"""GPU: the decoding rules -- ee_logit_rules against its definition (adjusted logits bit for bit, softmax in 64 bits), and the
rules of a session in every call that decides on tokens."""
import numpy as np
import pytest
import torch

import synth
import paper_2510_01336_amd as hs
from hs_common import bf16_small, gpu_side
from rules_common import adjust, pack, pick, softmax

pytestmark = pytest.mark.gpu


def make(rng, m, vocab, hist, penalties=True, bias=0, masks=False, empty=(), dtype=torch.float32, same_prompt=False):
    """Random rows, their rules and the rows' own pieces as host values.  m: rows of every sequence."""
    S, M = len(m), sum(m)
    x = rng.normal(0, 3, (M, vocab)).astype(np.float32)
    if vocab > 4:
        x[:, 1] = x[:, 3] = x.max(1)                        # exact ties at the top
    x = torch.from_numpy(x).to(dtype).float().numpy()
    p = dict(x=x, m=m, vocab=vocab, lens=[0] * S, nprompt=[0] * S, rho=np.ones(S, np.float32), freq=np.zeros(S, np.float32),
             pres=np.zeros(S, np.float32), temp=rng.uniform(0.5, 1.5, S).astype(np.float32), bias=[[] for _ in m], mask=None, rowmask=None)
    p["tokens"] = None
    if penalties:
        p["lens"] = [int(v) for v in rng.integers(0, hist + 1, S)]
        p["lens"][0] = hist
        room = hist + max(m) + 1
        t = (rng.random((S, room)) ** 3 * (vocab + 2)).astype(np.int32) - 1          # some ids outside the vocabulary
        p["tokens"], p["nprompt"] = t, [int(v * f) for v, f in zip(p["lens"], rng.random(S))]
        p["rho"] = rng.uniform(0.7, 1.8, S).astype(np.float32)
        p["freq"], p["pres"] = rng.uniform(-0.2, 0.7, S).astype(np.float32), rng.uniform(-0.3, 0.9, S).astype(np.float32)
    if bias:
        for b in range(S):
            n = int(rng.integers(0, bias + 1)) if b else bias
            p["bias"][b] = [(int(t), float(np.float32(v))) for t, v in zip(rng.integers(-1, vocab + 1, n), rng.normal(0, 3, n))]
    if masks:
        p["mask"] = rng.random((M + 1, vocab)) < rng.random((M + 1, 1))
        p["mask"][np.arange(M + 1), rng.integers(0, vocab, M + 1)] = True
        for r in empty:
            p["mask"][r] = False
        p["rowmask"] = rng.permutation(M).astype(np.int32)
        p["rowmask"][::5] = -1                              # no mask
        if len(empty):
            p["rowmask"][1:1 + len(empty)] = empty
        p["rowmask"][-1] = M + 7                            # outside the table: no mask either
    return p


def device_rules(p, dev="cuda"):
    def t(a, dt):
        return None if a is None else torch.tensor(np.asarray(a), dtype=dt, device=dev)
    start = np.concatenate([[0], np.cumsum(p["m"])])
    kw = dict(temperature=t(p["temp"], torch.float32))
    if p["tokens"] is not None:
        kw.update(tokens=t(p["tokens"], torch.int32), first_len=t(p["lens"], torch.int32), prompt_len=t(p["nprompt"], torch.int32),
                  repetition=t(p["rho"], torch.float32), frequency=t(p["freq"], torch.float32), presence=t(p["pres"], torch.float32))
    if any(p["bias"]):
        kw.update(bias_start=t(np.concatenate([[0], np.cumsum([len(b) for b in p["bias"]])]), torch.int32),
                  bias_token=t([e[0] for b in p["bias"] for e in b], torch.int32), bias_value=t([e[1] for b in p["bias"] for e in b], torch.float32))
    if p["mask"] is not None:
        kw.update(allowed=t(pack(p["mask"]), torch.int32), allowed_row=t(p["rowmask"], torch.int32))
    return hs.LogitRules(p["vocab"], t(start, torch.int32), **kw)


def reference(p, dtype):
    rows, r = [], 0
    for b, m in enumerate(p["m"]):
        for i in range(m):
            h = p["tokens"][b][:min(p["lens"][b] + i, p["tokens"].shape[1])] if p["tokens"] is not None else []
            mask = p["mask"][p["rowmask"][r]] if p["mask"] is not None and 0 <= p["rowmask"][r] < len(p["mask"]) else None
            rows.append(adjust(p["x"][r], h, p["nprompt"][b], p["rho"][b], p["freq"][b], p["pres"][b], p["temp"][b], p["bias"][b], mask, dtype))
            r += 1
    return np.array(rows).reshape(-1, p["vocab"])


def check(p, x, rules=None, out=None):
    rules = rules or device_rules(p)
    ref32, ref64 = reference(p, np.float32), reference(p, np.float64)
    z, tok = rules.logits(x, argmax=True, out=out)
    z, tok = z.cpu().numpy().copy(), tok.cpu().numpy()
    assert np.array_equal(z, ref32)
    assert tok.tolist() == [pick(v) for v in ref32]
    q, tok2 = rules.probs(x, argmax=True)
    q = q.cpu().numpy().astype(np.float64)
    assert np.array_equal(tok, tok2.cpu().numpy())
    # a logit of size L carries up to six roundings of intermediates no larger than 2 L + 10 over the temperature: |error| <= 6 * 2^-24 * that; the
    # exponential multiplies its relative error, the sum and the two factors add under 200 roundings (chains of at most 150 terms)
    size = (2 * np.abs(p["x"]).max() + 10 + max([abs(e[1]) for b in p["bias"] for e in b] + [0])) / p["temp"].min() * 1.8
    rel = 2 * 6 * 2.0 ** -24 * size + 200 * 2.0 ** -24
    for r in range(len(q)):
        w = softmax(ref64[r])
        assert np.all(np.abs(q[r] - w) <= rel * w + 1e-37), r
    # the same without the tokens, and again: equal to the bit
    assert torch.equal(rules.probs(x), rules.probs(x)) and np.array_equal(rules.logits(x).cpu().numpy(), ref32)


CASES = [
    # rows of every sequence, vocabulary, history, biases, masks
    ([1], 1, 3, 0, False), ([1], 7, 0, 2, True), ([1], 1000, 40, 0, False), ([3, 0, 2], 31, 20, 3, True), ([5], 4099, 700, 50, True),
    ([1] * 20, 1000, 90, 5, True), ([9, 1, 4, 9], 32003, 300, 20, True), ([2] * 40, 4096, 50, 0, False), ([1], 128256, 3000, 40, True),
    ([17], 50257, 100, 0, True), ([1] * 70, 32000, 300, 0, False), ([3] * 60, 8192, 30, 4, True), ([1] * 300, 20001, 64, 0, True)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{max(c[0])}_v{c[1]}_h{c[2]}_b{c[3]}_{int(c[4])}")
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_rules_against_the_definition(case, dtype):
    m, vocab, hist, bias, masks = case
    rng = np.random.default_rng(vocab + 7 * len(m))
    if dtype == torch.bfloat16 and sum(m) > 80:
        m = m[:20]
    p = make(rng, m, vocab, hist, True, bias, masks, empty=(2,) if sum(m) > 6 else (), dtype=dtype)
    check(p, torch.from_numpy(p["x"]).cuda().to(dtype))


@pytest.mark.parametrize("what", ["nothing", "temperature", "mask", "bias"])
def test_rules_one_at_a_time(what):
    rng = np.random.default_rng(3)
    p = make(rng, [2, 1], 5001, 0, penalties=False, bias=9 if what == "bias" else 0, masks=what == "mask")
    if what == "nothing":
        p["temp"][:] = 1
    check(p, torch.from_numpy(p["x"]).cuda())


@pytest.mark.parametrize("vocab", [1000, 4099, 40000])
def test_strided_and_unaligned_rows(vocab):
    """Rows of a larger buffer, out of step with the vector loads; what lies around the rows stays."""
    rng = np.random.default_rng(vocab)
    p = make(rng, [3, 2], vocab, 60, True, 4, True)
    for off, extra in ((1, 3), (0, 8), (4, 4), (2, 1)):
        big = torch.full((5, off + vocab + extra), 9.0, device="cuda")
        x = big[:, off:off + vocab]
        x.copy_(torch.from_numpy(p["x"]))
        out_big = torch.full((5, off + vocab + extra), 7.0, device="cuda")
        check(p, x, out=out_big[:, off:off + vocab])
        assert (out_big[:, :off] == 7).all() and (out_big[:, off + vocab:] == 7).all() and (big[:, off + vocab:] == 9).all()
        # in place
        rules = device_rules(p)
        ref = rules.probs(x.contiguous())
        got = rules.probs(x, out=x)
        assert got.data_ptr() == x.data_ptr() and torch.equal(got, ref)


def test_rows_of_no_sequence_are_left_alone():
    rng = np.random.default_rng(5)
    for vocab in (900, 9000):
        p = make(rng, [2, 3], vocab, 30)
        x = torch.from_numpy(rng.normal(0, 1, (9, vocab)).astype(np.float32)).cuda()
        x[2:7] = torch.from_numpy(p["x"])
        rules = device_rules(p)
        rules._kept["row_start"] += 2                        # rows 2..6 of nine
        for call in (rules.logits, rules.probs):
            out = torch.full((9, vocab), 5.0, device="cuda")
            got, tok = call(x, argmax=True, out=out)
            keep = tok.clone()
            assert (got[:2] == 5).all() and (got[7:] == 5).all()
        z = rules.logits(x, out=torch.full((9, vocab), 5.0, device="cuda"))
        assert np.array_equal(z[2:7].cpu().numpy(), reference(p, np.float32))
        assert keep[2:7].tolist() == [pick(v) for v in reference(p, np.float32)]


def test_what_masked_places_hold_does_not_matter():
    rng = np.random.default_rng(6)
    p = make(rng, [1, 2], 6000, 50, masks=True)
    p["rowmask"][:] = [0, 1, 2]
    clean = device_rules(p).probs(torch.from_numpy(p["x"]).cuda(), argmax=True)
    dirty = p["x"].copy()
    hidden = ~p["mask"][:3]
    dirty[hidden] = rng.choice([np.nan, np.inf, -np.inf, 3.4e38, -3.4e38], hidden.sum()).astype(np.float32)
    got = device_rules(p).probs(torch.from_numpy(dirty).cuda(), argmax=True)
    assert torch.equal(clean[0], got[0]) and torch.equal(clean[1], got[1])


def test_rows_of_lowest_values():
    """All logits at the lowest finite value are equal and count as such; all at -inf are nothing."""
    vocab = 5000
    x = torch.full((2, vocab), torch.finfo(torch.float32).min, device="cuda")
    x[1] = -torch.inf
    rules = hs.LogitRules(vocab, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"))
    q, tok = rules.probs(x, argmax=True)
    assert tok.tolist() == [0, -1]
    assert (q[1] == 0).all() and torch.allclose(q[0], torch.full_like(q[0], 1 / vocab), rtol=200 * 2.0 ** -24, atol=0)


def test_history_longer_than_its_room():
    """A length past the room of the list counts what the room holds."""
    rng = np.random.default_rng(8)
    p = make(rng, [4], 500, 20)
    rules = device_rules(p)
    p["lens"] = [p["tokens"].shape[1] - 2]
    rules._kept["first_len"].fill_(p["lens"][0])
    z = rules.logits(torch.from_numpy(p["x"]).cuda())
    assert np.array_equal(z.cpu().numpy(), reference(p, np.float32))


def test_captured_and_replayed():
    """A captured call sees the histories and rows as they are at every replay."""
    rng = np.random.default_rng(9)
    p = make(rng, [1, 3], 9001, 80, True, 3, True)
    x, rules = torch.from_numpy(p["x"]).cuda(), device_rules(p)
    rules.probs(x, argmax=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, tok = rules.probs(x, argmax=True)
    for step in range(4):
        x.copy_(torch.from_numpy(rng.normal(0, 3, p["x"].shape).astype(np.float32)))
        rules._kept["first_len"] += 1 if step else 0
        graph.replay()
        want, wtok = rules.probs(x, argmax=True)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(tok, wtok)


def test_other_streams_and_two_calls_at_once():
    rng = np.random.default_rng(10)
    p = make(rng, [9] * 8, 32000, 500, True, 3, True)
    x, rules = torch.from_numpy(p["x"]).cuda(), device_rules(p)
    want = rules.probs(x)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(rules.probs(x))
    torch.cuda.synchronize()
    assert all(torch.equal(want, g) for g in got)


def test_pieces_that_do_not_meet_are_scaled_afterwards():
    """With no wait for the other pieces of a row most pieces are left to the last launch: the same bits, arg max included."""
    rng = np.random.default_rng(12)
    for m, vocab in (([1], 128256), ([9, 0, 9], 32003), ([1] * 100, 50000)):
        p = make(rng, m, vocab, 100, True, 5, True, empty=(2,) if sum(m) > 6 else ())
        x, rules = torch.from_numpy(p["x"]).cuda(), device_rules(p)
        want = rules.probs(x, argmax=True)
        try:
            hs.ee_debug_rules_looks(0)
            for _ in range(3):
                got = rules.probs(x, argmax=True)
                assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        finally:
            hs.ee_debug_rules_looks(-1)
    with pytest.raises(hs.EEError):
        hs.ee_debug_rules_looks(-2)


def test_binding_refuses():
    start = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    rules = hs.LogitRules(100, start)
    f = lambda *s: torch.zeros(*s, device="cuda")
    for bad in (f(2, 99), f(100), f(2, 100).double(), f(2, 100).cpu(), f(100, 2).T):
        with pytest.raises(ValueError):
            rules.probs(bad)
    with pytest.raises(ValueError):
        rules.probs(f(2, 100), out=f(2, 100).half())
    with pytest.raises(ValueError):
        hs.LogitRules(100, start, repetition=f(2))
    with pytest.raises(ValueError):
        hs.LogitRules(100, start, first_len=f(1))
    with pytest.raises(ValueError):
        hs.LogitRules(100, start, allowed=torch.zeros((1, 3), dtype=torch.int32, device="cuda"))
    with pytest.raises(hs.EEError):
        hs.LogitRules(100, start, repetition=f(1)).probs(f(2, 100))          # a penalty without a history
    out, tok = rules.probs(f(0, 100), argmax=True)
    assert out.shape == (0, 100) and tok.shape == (0,)


def test_histories_that_overlap_are_refused():
    """One history expanded over the sequences, or windows of one list, would be read from one room after another; of a single sequence any
    stride is good."""
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    one, start, first = torch.full((40,), 7, dtype=torch.int32, device="cuda"), ints([0, 1, 2]), ints([40, 40])
    rep = torch.full((2,), 2.0, device="cuda")
    for tokens in (one[None].expand(2, 40), one.unfold(0, 20, 20 // 2)[:2]):
        with pytest.raises(ValueError):
            hs.LogitRules(100, start, tokens=tokens, first_len=first, repetition=rep)
    x = torch.ones(1, 100, device="cuda")
    got = hs.LogitRules(100, ints([0, 1]), tokens=one[None].expand(1, 40), first_len=first[:1], repetition=rep[:1]).logits(x)
    want = x.clone()
    want[0, 7] = 0.5
    assert torch.equal(got, want)


# ---- the rules of a session ------------------------------------------------------------------------------------------

RULES = [dict(repetition=1.3, frequency=0.4, presence=0.5), dict(temperature=0.8, bias={5: 2.0, 17: -3.0, 900: 1.0}, repetition=0.9),
         None, dict(frequency=-0.2, presence=0.1, repetition=1.1)]


def _allowed(vocab, seed):
    return np.random.default_rng(seed).random(vocab) < 0.5


def session(cfg, seed, B, max_ctx, max_rows, rules=RULES, masks=(1,)):
    model, sess = gpu_side(cfg, seed, B, max_ctx, max_rows)
    sess.enable_rules(8)
    put(sess, B, rules, masks, cfg.vocab)
    return model, sess


def put(sess, B, rules, masks, vocab):
    for b in range(B):
        r = rules[b % len(rules)]
        if r is not None:
            sess.set_rules(b, **r, allowed=_allowed(vocab, b) if b in masks else None)


def apply(x, b, text, n_prompt, vocab, masks=(1,), extra=None, rules=RULES):
    r = rules[b % len(rules)]
    if r is None:
        return np.asarray(x, np.float32)
    mask = _allowed(vocab, b) if b in masks else None
    if extra is not None:
        mask = extra if mask is None else mask & extra
    return adjust(x, text, n_prompt, r.get("repetition", 1), r.get("frequency", 0), r.get("presence", 0), r.get("temperature", 1),
                  list(r.get("bias", {}).items()), mask)


@pytest.mark.parametrize("cfg", [synth.tiny_config(), bf16_small(vocab=1024)], ids=["f32", "bf16"])
def test_session_rules_in_every_head(cfg):
    """Prompt, decoding, drafting and both verifications under rules: the logits of the same calls without rules (a second session
    in lockstep), adjusted row by row with the history of the row's position, give the tokens."""
    B, ctx, k = 4, [40, 70, 23, 9], 4
    prompts = [synth.gen_prompt(cfg.vocab, n, 300 + n) for n in ctx]
    model, sess = session(cfg, 99, B, 200, 20)
    plain = hs.Session(model, B, 200, 20)
    for s in (sess, plain):
        s.enable_logits(True)
    first = sess.prefill(prompts)
    plain.prefill(prompts)
    raw, got = plain.last_logits(), sess.last_logits()
    ends = np.cumsum(ctx) - 1 if cfg.dtype != "f32" else None
    if ends is not None:
        for b in range(B):
            z = apply(raw[ends[b]], b, prompts[b], ctx[b], cfg.vocab)
            assert np.array_equal(got[ends[b]], z) and int(first[b]) == pick(z)
    text = [list(p) + [int(f)] for p, f in zip(prompts, first)]

    # decoding, one token per call
    for _ in range(3):
        tok = sess.decode_ar(1)[:, 0]
        got = sess.last_logits()
        for b in range(B):
            text[b].append(int(tok[b]))
            assert int(tok[b]) == pick(got[b])
    # several tokens in one call are those of single calls
    keep = [len(t) for t in text]
    many = sess.decode_ar(4)
    for b in range(B):
        sess.rollback(b, 0b111, keep[b] - 1)
    single = np.concatenate([sess.decode_ar(1) for _ in range(4)], axis=1)
    assert np.array_equal(many, single)
    for b in range(B):
        text[b] += [int(t) for t in single[b]]
    # a block: verified at L_i and at L_f with the logits of a plain session that holds the same context
    rng = np.random.default_rng(4)
    S = rng.integers(0, cfg.vocab, (B, k)).astype(np.int32)
    for b in range(B):
        S[b, 0] = text[b][-2]                                  # (a token of the history comes again inside the block)
    before = [len(t) for t in text]
    assert [sess.tokens(b).tolist() for b in range(B)] == text
    sess.draft_inject(S)
    a, nxt = sess.verify_intermediate()
    z_i, hid = sess.last_logits(), sess.last_hidden()
    n_prompt = ctx
    row = 0
    for b in range(B):
        v = [pick(z_i[row + j]) for j in range(k + 1)]
        want = 0
        while want < k and v[want] == S[b, want]:
            want += 1
        assert (int(a[b]), int(nxt[b])) == (want, v[want])
        # masked and biased tokens show in the rows themselves
        if b == 1:
            off = ~_allowed(cfg.vocab, 1)
            assert np.all(np.isneginf(z_i[row:row + k + 1][:, off])) and np.isfinite(z_i[row:row + k + 1][:, ~off]).all()
        row += k + 1
    # the same block without rules: its logits, adjusted, are the ruled ones bit for bit (same kernels, same operands)
    for b in range(B):
        sess.rollback(b, 0b011, before[b] - 1)
        sess.clear_rules(b)
    sess.draft_inject(S)
    sess.verify_intermediate()
    raw = sess.last_logits()
    row = 0
    for b in range(B):
        for j in range(k + 1):
            z = apply(raw[row], b, text[b] + S[b, :j].tolist(), n_prompt[b], cfg.vocab)
            assert np.array_equal(z, z_i[row]), (b, j)
            row += 1
    # the full verification, likewise: first without rules, then with them on the same tentative tokens
    for b in range(B):
        sess.rollback(b, 0b011, before[b] - 1)
    put(sess, B, RULES, (1,), cfg.vocab)
    out = []
    for ruled in (True, False):
        sess.draft_inject(S)
        sess.verify_intermediate()
        V = [sess.tokens(b).tolist()[before[b]:] for b in range(B)]
        if not ruled:
            for b in range(B):
                sess.clear_rules(b)
        f, fn, com = sess.verify_full()
        out.append((V, f, fn, com, sess.last_logits()))
        if ruled:
            for b in range(B):
                sess.rollback(b, 0b111, before[b] - 1)
    assert out[0][0] == out[1][0]
    row = 0
    for b, V in enumerate(out[0][0]):
        for j in range(len(V) + 1):
            z = apply(out[1][4][row], b, text[b] + V[:j], n_prompt[b], cfg.vocab)
            assert np.array_equal(z, out[0][4][row]), (b, j)
            if j == int(out[0][1][b]):
                assert int(out[0][2][b]) == pick(z)
            row += 1
    plain.close(); sess.close(); model.close()


@pytest.mark.parametrize("cfg", [synth.tiny_config(gamma=(1.0, 0.3, 0.3)), synth.tiny_config(n_layers=6, exit_draft=1, exit_inter=2, exit_extra=(4,),
                                                                                          gamma=(1.0, 0.3, 0.3))], ids=["two_levels", "three_levels"])
def test_loop_stream_equals_decoding_under_the_same_rules(cfg):
    from paper_2510_01336_amd.loop import hispec_generate, hispec_generate_levels
    B, n_new, k = 3, 40, 4
    prompts = [synth.gen_prompt(cfg.vocab, n, 40 + n) for n in (30, 17, 5)]
    # (the loop steps all sequences until the slowest has n_new tokens: where the exits disagree under its rules it commits one token in
    # four, or with a further level 24, drafts, while another sequence may gain five a draft)
    room = min(8000, 40 * 5 * (24 if cfg.exit_extra else 6) + 400)
    model, sess = session(cfg, 4242, B, room, 60)
    first = sess.prefill(prompts)
    ar = sess.decode_ar(n_new)
    assert len(set(ar[0].tolist())) > 1
    sess.prefill(prompts)
    if cfg.exit_extra:
        toks, st = hispec_generate_levels(sess, n_new, k, [4, 6])
    else:
        toks, st = hispec_generate(sess, n_new, k, n_i=6)
    assert np.array_equal(toks, ar)
    # rules change what is said, and taking them back restores it
    for b in range(B):
        sess.clear_rules(b)
    sess.prefill(prompts)
    free = sess.decode_ar(n_new)
    assert not np.array_equal(free[0], ar[0])
    fresh = hs.Session(model, B, room, 60)
    fresh.prefill(prompts)
    assert np.array_equal(fresh.decode_ar(n_new), free)
    fresh.close(); sess.close(); model.close()


@pytest.mark.parametrize("cfg", [synth.tiny_config(), bf16_small()], ids=["f32", "bf16"])
def test_row_masks(cfg):
    """Masks of single rows: a mask of one token decides its row, rows behind the masks are free, one call uses them up."""
    B, k = 2, 4
    prompts = [synth.gen_prompt(cfg.vocab, n, n) for n in (20, 31)]
    model, sess = gpu_side(cfg, 11, B, 160, 20)
    sess.enable_rules()
    for b in range(B):
        sess.set_rules(b, temperature=0.9)
    one = lambda *toks: np.eye(cfg.vocab, dtype=bool)[list(toks)]
    sess.row_masks(0, one(7))
    first = sess.prefill(prompts)
    assert int(first[0]) == 7 and sess.tokens(0)[-1] == 7
    free = sess.decode_ar(3)                                    # (used up)
    for b in range(B):
        sess.rollback(b, 0b111, len(prompts[b]))
    sess.row_masks(1, one(3, 4))
    got = sess.decode_ar(3)
    assert got[1, :2].tolist() == [3, 4] and np.array_equal(got[0], free[0])
    for b in range(B):
        sess.rollback(b, 0b111, len(prompts[b]))
    sess.row_masks(0, one(9, 8, 7, 6))
    S = sess.draft(k)
    assert S[0].tolist() == [9, 8, 7, 6]
    sess.row_masks(0, one(9, 8, 50))
    a, n = sess.verify_intermediate()
    assert (int(a[0]), int(n[0])) == (2, 50)
    sess.row_masks(0, one(9, 5))
    f, fn, com = sess.verify_full()
    assert com[0] == [9, 5]
    # an own mask and a row's mask both hold; what allows nothing is refused and changes nothing
    half = np.arange(cfg.vocab) < 100
    sess.set_rules(0, allowed=half)
    with pytest.raises(hs.EEError) as e:
        sess.row_masks(0, one(200))
    assert e.value.code == -1
    two = one(60) | one(200)
    sess.row_masks(0, two)
    assert int(sess.decode_ar(1)[0, 0]) == 60
    assert int(sess.decode_ar(1)[0, 0]) < 100
    # ee_rules_set takes masks of rows back
    sess.row_masks(0, one(61))
    sess.set_rules(0, temperature=0.9)
    sess.row_masks(0, one(61))
    sess.row_masks(0, np.zeros((0, cfg.vocab), bool))
    sess.close(); model.close()


def test_sampling_calls_under_rules():
    """The distributions of drafting and verification are the softmax of the adjusted logits, and tokens come from them."""
    cfg, B, k = synth.tiny_config(), 2, 4
    prompts = [synth.gen_prompt(cfg.vocab, n, n) for n in (25, 40)]
    rules = [dict(repetition=1.2, frequency=0.3, presence=0.2, temperature=0.7), dict(temperature=1.4, presence=0.6)]
    model, sess = session(cfg, 5, B, 160, 20, rules, (0, 1))
    sess.enable_sampling()
    sess.enable_logits(True)
    text = [list(p) + [int(t)] for p, t in zip(prompts, sess.prefill(prompts))]
    u = np.random.default_rng(0).random((B, k)).astype(np.float32)
    S = sess.draft_sample(k, u)
    for b in range(B):
        P = sess.read_dist(0, b, 0, k).astype(np.float64)
        assert (P[:, ~_allowed(cfg.vocab, b)] == 0).all() and np.allclose(P.sum(1), 1, atol=1e-5)
        for j in range(k):
            c = np.concatenate([[0], np.cumsum(P[j])])
            assert c[S[b, j]] - 1e-5 <= u[b, j] <= c[S[b, j] + 1] + 1e-5, (b, j)
    a, n = sess.verify_intermediate_rs(u, u[:, 0].copy())
    target = sess.last_logits()
    for b in range(B):
        sess.rollback(b, 0b011, len(text[b]) - 1)
        sess.clear_rules(b)
    sess.draft_inject(S)
    sess.verify_intermediate()
    raw, row = sess.last_logits(), 0
    for b in range(B):
        for j in range(k + 1):
            z = apply(raw[row], b, text[b] + S[b, :j].tolist(), len(prompts[b]), cfg.vocab, (0, 1), rules=rules)
            w = softmax(z)
            assert np.all(np.abs(target[row] - w) <= 1e-5 * w + 1e-30), (b, j)
            row += 1
    sess.close(); model.close()


def test_rules_at_the_8b_vocabulary():
    """Two layers' worth of the 8B width with the whole vocabulary: nine rows each of three sequences, logits bit for bit."""
    cfg, k, B = synth.llama8b_config(n_layers=3, exit_draft=1, exit_inter=2), 8, 3
    prompts = [synth.gen_prompt(cfg.vocab, n, n) for n in (60, 100, 31)]
    model, sess = session(cfg, 1, B, 200, 20)
    sess.enable_logits(True)
    text = [list(p) + [int(t)] for p, t in zip(prompts, sess.prefill(prompts))]
    S = np.random.default_rng(0).integers(0, cfg.vocab, (B, k)).astype(np.int32)
    sess.draft_inject(S)
    sess.verify_intermediate()
    ruled = sess.last_logits().copy()
    for b in range(B):
        sess.rollback(b, 0b011, len(text[b]) - 1)
        sess.clear_rules(b)
    sess.draft_inject(S)
    sess.verify_intermediate()
    raw = sess.last_logits()
    for r in range(B * (k + 1)):
        b, j = divmod(r, k + 1)
        assert np.array_equal(apply(raw[r], b, text[b] + S[b, :j].tolist(), len(prompts[b]), cfg.vocab), ruled[r]), r
    sess.close(); model.close()


def test_session_refusals_and_states():
    cfg = bf16_small()
    model, sess = gpu_side(cfg, 3, 2, 100, 12)
    for call in (lambda: sess.set_rules(0), lambda: hs.ee_rules_rows(sess.handle, 0, np.zeros((0, 32), np.uint32))):
        with pytest.raises(hs.EEError) as e:
            call()
        assert e.value.code == -2                                 # not attached
    with pytest.raises(hs.EEError):
        hs.ee_rules_bytes(sess.handle, -1)
    n = hs.ee_rules_bytes(sess.handle, 3)
    buf = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    ptr = buf.data_ptr() + (-buf.data_ptr()) % 256
    for args in ((3, ptr + 4, n), (3, ptr, n - 1), (-1, ptr, n)):
        with pytest.raises(hs.EEError) as e:
            hs.ee_rules_attach(sess.handle, *args)
        assert e.value.code == -1
    hs.ee_rules_attach(sess.handle, 3, ptr, n)
    with pytest.raises(hs.EEError) as e:
        hs.ee_rules_attach(sess.handle, 3, ptr, n)
    assert e.value.code == -2
    nan, inf = float("nan"), float("inf")
    for bad in (dict(repetition=0.0), dict(repetition=-1.0), dict(repetition=nan), dict(temperature=0.0), dict(temperature=inf),
                dict(frequency=nan), dict(presence=inf), dict(bias={1: 1.0, 2: 1.0, 3: 1.0, 4: 1.0}), dict(bias={-1: 1.0}),
                dict(bias={cfg.vocab: 1.0}), dict(bias={2: -inf}), dict(allowed=np.zeros(cfg.vocab, bool))):
        with pytest.raises(hs.EEError) as e:
            sess.set_rules(1, **bad)
        assert e.value.code == -1, bad
    with pytest.raises(hs.EEError):
        sess.set_rules(2)
    with pytest.raises(ValueError):
        sess.set_rules(0, allowed=np.ones(cfg.vocab - 1, bool))
    with pytest.raises(hs.EEError) as e:
        sess.row_masks(0, np.ones((1, cfg.vocab), bool))           # no rules yet
    assert e.value.code == -2
    sess.set_rules(0, temperature=2.0)
    with pytest.raises(hs.EEError) as e:
        sess.row_masks(0, np.ones((13, cfg.vocab), bool))
    assert e.value.code == -1
    # the call whose scratch is static refuses while rules hold, and works again without
    sess.prefill([synth.gen_prompt(cfg.vocab, 20, 1), synth.gen_prompt(cfg.vocab, 9, 2)])
    sess.draft(3)
    with pytest.raises(hs.EEError) as e:
        sess.verify_intermediate_static()
    assert e.value.code == -2
    sess.clear_rules(0)
    sess.verify_intermediate_static()
    # an idle slot takes no part
    sess.set_rules(1, presence=0.5)
    sess.verify_full()
    sess.release(1)
    assert sess.decode_ar(2)[1].tolist() == [-1, -1]
    sess.prefill_seq(1, synth.gen_prompt(cfg.vocab, 50, 3))
    sess.decode_ar(2)
    sess.close(); model.close()
