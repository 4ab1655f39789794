"""GPU: attention over pages that sequences share -- ee_attend against its formula in 64 bits, and the calls of a session that take
this form against the oracle and against the forms that read every sequence's pages by themselves."""
import numpy as np
import pytest
import torch

import synth
import paper_2510_01336_amd as hs
from hs_common import TOL, OracleSide, bf16_d128, bf16_small, check_state, gpu_side, max_rel, run_round

pytestmark = pytest.mark.gpu

PAGE = 64


@pytest.fixture(autouse=True)
def builtin_choice():
    yield
    hs.ee_debug_shared_attention(-1)


def config(hq, hkv, D, dtype="bf16"):
    return synth.EEConfig(n_layers=3, d_model=64, n_q_heads=hq, n_kv_heads=hkv, head_dim=D, d_ffn=64, vocab=512, exit_draft=1, exit_inter=2,
                          dtype=dtype)


class Planted:
    """A session whose sequences have the given contexts -- paths into a tree of runs, {name: positions} -- with random K and V
    in one layer; sequences share what the paths share."""

    def __init__(self, cfg, runs, paths, max_rows=24, seed=0, layer=1, pages=0, spread=1.0):
        self.cfg, self.layer = cfg, layer
        self.rng = rng = np.random.default_rng(seed)
        self.model = hs.Model(cfg, 1)
        tok, kv = {}, {}
        for i, (name, n) in enumerate(runs.items()):
            tok[name] = rng.integers(0, cfg.vocab, n).astype(np.int32)
            tok[name][:1] = i                                    # (runs part where they begin)
            kv[name] = [self.rounded(rng.normal(0, spread, (n, cfg.n_kv_heads, cfg.head_dim))) for _ in range(2)]
        prompts = [np.concatenate([tok[r] for r in p]) for p in paths]
        self.lens = [len(p) for p in prompts]
        B = len(paths)
        self.sess = hs.Session(self.model, B, max(self.lens) + 20, max_rows, pages)
        self.sess.prefill_seq(0, prompts[0])
        for b in range(1, B):
            # the earlier sequence with the longest common path
            same = [next((i for i, (x, y) in enumerate(zip(paths[a], paths[b])) if x != y), min(len(paths[a]), len(paths[b]))) for a in range(b)]
            self.sess.prefill_shared([int(np.argmax(same))] * B, [prompts[c] if c == b else None for c in range(B)])
        self.K = [np.concatenate([kv[r][0] for r in p]) for p in paths]
        self.V = [np.concatenate([kv[r][1] for r in p]) for p in paths]
        for b in range(B):
            self.sess.write_kv(b, layer, 0, self.K[b], self.V[b])

    def rounded(self, x):
        t = torch.from_numpy(np.asarray(x, np.float32))
        return (t.to(torch.bfloat16).float() if self.cfg.dtype == "bf16" else t).numpy()

    def query(self, rows, scale=1.5):
        c = self.cfg
        return self.rounded(self.rng.normal(0, scale, (sum(rows), c.n_q_heads, c.head_dim)))

    def tensor(self, q):
        return torch.from_numpy(q).cuda().to(torch.bfloat16 if self.cfg.dtype == "bf16" else torch.float32)

    def check(self, q, rows, pos0, got):
        """Against the formula in 64 bits.  bf16: a weight rounded by at most 2^-8 of itself moves the normalised sum by at most 2^-8 of
        sum w |v - o|, the output is rounded by at most 2^-8 of itself; scores are off by less than 2^-24 * 2 D of sum |q||k|, far below;
        2^-10 of slack.  fp32: chains of at most a few hundred roundings on the sums, 2^-24 * 400 of sum w |v|, and of the scores' size."""
        c = self.cfg
        rep = c.n_q_heads // c.n_kv_heads
        got = got.float().cpu().numpy().astype(np.float64)
        r = 0
        for b, m in enumerate(rows):
            for i in range(m):
                n = pos0[b] + i + 1
                for h in range(c.n_q_heads):
                    k, v = self.K[b][:n, h // rep].astype(np.float64), self.V[b][:n, h // rep].astype(np.float64)
                    s = k @ q[r, h].astype(np.float64) / np.sqrt(c.head_dim)
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    o = w @ v
                    if c.dtype == "bf16":
                        tol = 2.0 ** -8 * (w @ np.abs(v - o) + np.abs(o)) * (1 + 2.0 ** -2) + 2.0 ** -10 * (w @ np.abs(v))
                    else:
                        tol = 2.0 ** -24 * (400 + 4 * np.abs(s).max() * c.head_dim) * (w @ np.abs(v))
                    bad = np.abs(got[r, h] - o) > tol
                    assert not bad.any(), (b, i, h, got[r, h][bad][:4], o[bad][:4])
                r += 1

    def attend(self, rows, pos0=None, **kw):
        q = self.query(rows)
        at = pos0 if pos0 is not None else [n - m for n, m in zip(self.lens, rows)]
        for mode in (0, 1, -1):                                  # never together, together wherever pages are shared, the built-in choice
            hs.ee_debug_shared_attention(mode)
            self.sess.attend_begin(rows, pos0)
            got = self.sess.attend(self.layer, self.tensor(q), **kw)
            self.check(q, rows, at, got)
        return q, got

    def close(self):
        self.sess.close(); self.model.close()


HEADS = [(8, 2, 64), (32, 8, 128), (64, 8, 128), (3, 3, 128), (16, 1, 64), (10, 2, 128)]


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_shared_prefix_against_the_formula(heads):
    """One prefix that ends inside a page, ragged tails and rows; then other rows and positions of the same session."""
    runs = {"p": 700, "a": 9, "b": 64, "c": 130, "d": 1, "e": 300}
    P = Planted(config(*heads), runs, [("p", t) for t in "abcde"])
    P.attend([1, 1, 1, 1, 1])
    P.attend([3, 9, 17, 1, 0])
    P.attend([2, 0, 5, 0, 24])
    P.attend([4, 4, 4, 4, 4], [0, 60, 640, 64, 690])             # rows inside the prefix: fewer whole pages in front of them
    P.attend([0, 1, 0, 0, 0])
    P.close()


@pytest.mark.parametrize("prefix", [0, 1, 63, 64, 65, 127, 128, 129, 1000])
def test_lengths_around_the_page_edges(prefix):
    runs = {"p": prefix, "a": 1, "b": 63, "c": 64, "d": 65, "e": 2}
    paths = [("p", t) for t in "abcde"]
    P = Planted(config(8, 2, 64), runs, paths)
    P.attend([1] * 5)
    rows = [min(n, 5) for n in P.lens]
    P.attend(rows)
    P.attend([1] * 5, [0] * 5)                                  # the first position: a context of one
    P.close()


def test_a_tree_of_prefixes():
    runs = {"r": 260, "x": 200, "y": 100, "xx": 70, "z": 30}
    runs.update({f"t{i}": n for i, n in enumerate([1, 33, 64, 70, 5, 90, 2, 140])})
    paths = [("r", "x", "xx", "t0"), ("r", "x", "xx", "t1"), ("r", "x", "t2"), ("r", "y", "t3"), ("r", "y", "t4"), ("z", "t5"), ("r", "t6"), ("r", "x", "xx", "t7")]
    for heads in ((8, 2, 64), (32, 8, 128)):
        P = Planted(config(*heads), runs, paths)
        P.attend([1] * 8)
        P.attend([9, 1, 3, 9, 2, 7, 1, 5])
        P.close()


def test_long_contexts_are_split_and_many_sequences():
    """A prefix of many pages (items of several cuts), and as many sequences as fill several blocks of tiles."""
    runs = {"p": 9000, "a": 200, "b": 3}
    P = Planted(config(32, 8, 128), runs, [("p", "a"), ("p", "b")], spread=0.7)
    P.attend([1, 1])
    P.attend([17, 5])
    P.close()
    runs = {"p": 900, **{f"t{i}": 1 + 7 * i for i in range(40)}}
    P = Planted(config(8, 2, 64), runs, [("p", f"t{i}") for i in range(40)])
    P.attend([1] * 40)
    P.attend([1 + i % 9 for i in range(40)])
    P.close()


def test_offsets_behind_32_bits():
    """A page pool whose last layer lies more than 2^32 elements into the cache; a copied page keeps every layer's contents."""
    P = Planted(config(32, 8, 128), {"p": 300, "a": 20, "b": 90}, [("p", "a"), ("p", "b")], layer=2, pages=20000)
    assert 2 * 20000 * 8 * 2 * PAGE * 128 > 2 ** 32
    P.attend([1, 1])
    P.attend([9, 3])
    before = [P.sess.read_kv(1, l, 0, 200) for l in range(3)]
    P.sess.rollback(1, 0b111, 200)
    P.sess.decode_ar(1)                                         # position 200 on is written: the shared page is copied
    assert P.sess.shared_pages(1) == 3
    for l, want in enumerate(before):
        for x, y in zip(P.sess.read_kv(1, l, 0, 200), want):
            assert np.array_equal(x, y), l
    for x, y in zip(P.sess.read_kv(0, 2, 0, 300), (P.K[0], P.V[0])):
        assert np.array_equal(np.asarray(x).reshape(-1), y[:300].reshape(-1))
    P.close()


def test_nothing_shared_and_one_sequence():
    runs = {"a": 100, "b": 700, "c": 5}
    P = Planted(config(32, 8, 128), runs, [("a",), ("b",), ("c",)])
    P.attend([1, 1, 1])
    P.attend([9, 20, 5])
    P.close()
    P = Planted(config(8, 2, 64), {"a": 3000}, [("a",)])
    P.attend([1])
    P.attend([24])
    P.close()


def test_large_scores():
    """Scores of several hundred: the running maximum carries the sums, one position may take all the weight."""
    runs = {"p": 500, "a": 90, "b": 20}
    P = Planted(config(8, 2, 64), runs, [("p", "a"), ("p", "b")], spread=6.0)
    P.attend([3, 3])
    P.close()


def test_what_lies_behind_the_rows_does_not_matter():
    """NaN in dead positions of the sequences' own pages, and live positions behind the rows asked for."""
    cfg = config(32, 8, 128)
    P = Planted(cfg, {"p": 200, "a": 70, "b": 10}, [("p", "a"), ("p", "b")])
    for b in range(2):
        P.sess.poison_dead_kv(b)
    q, got = P.attend([4, 4])
    bad = np.full((30, cfg.n_kv_heads, cfg.head_dim), np.nan, np.float32)
    P.sess.write_kv(0, 1, 240, bad, bad)                        # behind rows 200 .. 239
    P.attend([24, 2], [216, 200])
    P.close()


@pytest.mark.parametrize("dtype, mode", [("bf16", -1), ("bf16", 1), ("f32", -1)])
def test_strides_streams_and_graphs(dtype, mode):
    cfg = config(8, 2, 64, dtype)
    P = Planted(cfg, {"p": 150, "a": 30, "b": 8, "c": 1}, [("p", "a"), ("p", "b"), ("p", "c")])
    rows = [3, 2, 1]
    q, _ = P.attend(rows)
    t = P.tensor(q)
    hs.ee_debug_shared_attention(mode)
    P.sess.attend_begin(rows)
    want = P.sess.attend(1, t)
    # rows of a wider buffer, in and out; what lies between them stays
    wide = torch.full((6, 12, 64), 3.0, dtype=t.dtype, device="cuda")
    wide[:, 2:10] = t
    out_wide = torch.full((6, 12, 64), 7.0, dtype=t.dtype, device="cuda")
    got = P.sess.attend(1, wide[:, 2:10], out=out_wide[:, 1:9])
    assert torch.equal(got, want) and (out_wide[:, 0] == 7).all() and (out_wide[:, 9:] == 7).all()
    # another stream than the session's, with work in front of and behind the call
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = torch.zeros_like(t)
        late.copy_(t)
        other = P.sess.attend(1, late) + 0
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, want)
    # captured on the session's stream and replayed with other rows
    model = hs.Model(cfg, 1, stream=side)
    torch.cuda.synchronize()
    model.close()
    P.close()
    with torch.cuda.stream(side):
        P = Planted(cfg, {"p": 150, "a": 30, "b": 8, "c": 1}, [("p", "a"), ("p", "b"), ("p", "c")])
        q, _ = P.attend(rows)
        static = P.tensor(q)
        hs.ee_debug_shared_attention(mode)
        P.sess.attend_begin(rows)
        P.sess.attend(1, static)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = P.sess.attend(1, static)
        for _ in range(4):
            q = P.query(rows)
            static.copy_(P.tensor(q))
            graph.replay()
            eager = P.sess.attend(1, static)
            torch.cuda.synchronize()
            assert torch.equal(out, eager)
            P.check(q, rows, [n - m for n, m in zip(P.lens, rows)], out)
        P.close()


def test_reference_precision():
    cfg = config(4, 4, 64, "f32")
    P = Planted(cfg, {"p": 100, "a": 30, "b": 1}, [("p", "a"), ("p", "b")])
    P.attend([1, 1])
    P.attend([9, 4])
    P.attend([2, 2], [0, 63])
    P.close()
    P = Planted(config(6, 2, 40, "f32"), {"p": 70, "a": 30, "b": 1}, [("p", "a"), ("p", "b")])
    P.attend([5, 3])
    P.close()


def test_refusals():
    cfg = config(8, 2, 64)
    P = Planted(cfg, {"p": 100, "a": 30, "b": 1}, [("p", "a"), ("p", "b")], max_rows=8)
    s = P.sess
    q = torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda")

    def code(f):
        with pytest.raises(hs.EEError) as e:
            f()
        return e.value.code
    assert code(lambda: hs.ee_attend(s.handle, 1, q.data_ptr(), hs.EE_BF16, 512, q.data_ptr() + 4096, 512)) == -2      # no begin yet
    for rows, pos in (([9, 1], None), ([-1, 1], None), ([0, 0], None), ([1, 1], [130, 0]), ([1, 1], [-1, 0]), ([2, 1], [129, 0])):
        assert code(lambda: s.attend_begin(rows, pos)) == -1, (rows, pos)
    s.attend_begin([2, 1])
    out = torch.empty_like(q)
    good = (s.handle, 1, q.data_ptr(), hs.EE_BF16, 512, out.data_ptr(), 512)
    for i, v in ((1, -1), (1, 3), (3, hs.EE_F32), (4, 511), (4, 516), (5, q.data_ptr()), (6, 500), (2, q.data_ptr() + 2), (5, out.data_ptr() + 8)):
        bad = list(good); bad[i] = v
        assert code(lambda: hs.ee_attend(*bad)) == -1, (i, v)
    hs.ee_attend(*good)
    for t in (q[:2], q.float(), q.cpu(), q.transpose(1, 2)):
        with pytest.raises(ValueError):
            s.attend(1, t)
    # anything that moves the session on ends it
    for move in (lambda: s.rollback(0, 0b111, 120), lambda: s.draft(2), lambda: s.verify_intermediate(), lambda: s.verify_full(), lambda: s.decode_ar(1),
                 lambda: s.prefill_seq(1, np.arange(70, dtype=np.int32))):
        s.attend_begin([2, 1])
        move()
        assert code(lambda: hs.ee_attend(*good)) == -2
    # a pending draft block: group 1 holds more positions than the others
    s.draft(3)
    s.attend_begin([2, 1])
    hs.ee_attend(s.handle, 0, *good[2:])
    assert code(lambda: hs.ee_attend(*good)) == -1
    s.release(1)
    assert code(lambda: s.attend_begin([1, 1])) == -2
    s.attend_begin([1, 0])
    with pytest.raises(hs.EEError):
        hs.ee_debug_shared_attention(2)
    P.close()


# ---- calls of a session ------------------------------------------------------------------------------------------------

def prompts_of(vocab, prefix, tails):
    common = synth.gen_prompt(vocab, prefix, 5)
    out = []
    for i, n in enumerate(tails):
        t = synth.gen_prompt(vocab, n, 60 + i)
        t[0] = i
        out.append(np.concatenate([common, t]).astype(np.int32))
    return out


@pytest.mark.parametrize("cfg", [bf16_small(), bf16_d128()], ids=["d64", "d128"])
def test_rounds_against_the_oracle(cfg):
    """Draft, verification and rollback rounds with the shared form forced follow the oracle, page edges included."""
    tails = [9, 50, 1, 63]
    prompts = prompts_of(cfg.vocab, 140, tails)
    B, cap = len(tails), 400
    O = OracleSide(cfg, 31, plain_twin=True)
    model, sess = gpu_side(cfg, 31, B, cap, 24)
    sess.enable_logits(True)
    hs.ee_debug_shared_attention(1)
    first = [int(sess.prefill_seq(0, prompts[0]))] + [int(t) for t in sess.prefill_shared([-1, 0, 0, 0], [None] + prompts[1:])[1:]]
    ref, _ = O.prefill(prompts, cap)
    if first != [int(t) for t in ref]:
        pytest.skip("a first token inside the margin")
    rng = np.random.default_rng(5)
    for i in range(4):
        run_round(O, sess, 6, 0.7, rng, i % 2 == 1, TOL["bf16"])
        assert hs.ee_debug_last_attention(sess.handle) == 3
        check_state(O, sess)
        for b in range(B):
            sess.poison_dead_kv(b)
    sess.close(); model.close()


def test_shared_and_separate_forms_agree():
    """The same rounds with the form forced on and off, sequential passes over page edges among them: logits to bf16 accuracy, and
    repeated runs of one form to the bit."""
    cfg = bf16_d128()
    prompts = prompts_of(cfg.vocab, 200, [54, 20, 3])           # the first sequence crosses a page edge while it decodes
    model, sess = gpu_side(cfg, 3, 3, 600, 30)
    sess.enable_logits(True)
    sess.prefill_seq(0, prompts[0])
    sess.prefill_shared([-1, 0, 0], [None, prompts[1], prompts[2]])
    lens = sess.lengths()[:, 0]

    def run(mode):
        hs.ee_debug_shared_attention(mode)
        out = []
        S = np.random.default_rng(1).integers(0, cfg.vocab, (3, 12)).astype(np.int32)
        sess.draft_inject(S)
        sess.verify_intermediate()
        out.append(sess.last_logits().copy())
        assert hs.ee_debug_last_attention(sess.handle) == (3 if mode else hs.ee_debug_last_attention(sess.handle))
        for b in range(3):
            sess.rollback(b, 0b111, int(lens[b]))
        toks = sess.decode_ar(12)
        out.append(sess.last_logits().copy())
        out.append(toks)
        for b in range(3):
            sess.rollback(b, 0b111, int(lens[b]))
        return out
    on, off, again = run(1), run(0), run(1)
    assert all(np.array_equal(x, y) for x, y in zip(on, again))
    assert max_rel(on[0], off[0]) <= 2e-2
    if np.array_equal(on[2], off[2]):
        assert max_rel(on[1], off[1]) <= 2e-2
    assert (on[2][:, 0] == off[2][:, 0]).sum() >= 2
    # scratch in the static array: the same bits
    hs.ee_debug_shared_attention(1)
    S = np.random.default_rng(2).integers(0, cfg.vocab, (3, 5)).astype(np.int32)
    res = []
    for call in (sess.verify_intermediate, sess.verify_intermediate_static):
        sess.draft_inject(S)
        a, n = call()
        res.append((a.copy(), n.copy(), sess.last_logits().copy(), sess.last_hidden().copy()))
        for b in range(3):
            sess.rollback(b, 0b011, int(lens[b]))
    assert all(np.array_equal(x, y) for x, y in zip(*res))
    sess.close(); model.close()


def test_samples_of_one_prompt_under_rules():
    """The operators as they serve together: continuations of one prompt in sequences that share its pages, each under its own rules, drafted,
    verified and committed by the sampling calls; the loop's streams differ, stay inside their masks, and the pool gets its pages back."""
    from paper_2510_01336_amd.loop import hispec_generate_sampling
    cfg = bf16_d128()
    prompt = synth.gen_prompt(cfg.vocab, 300, 9)
    B, n_new = 6, 24
    model, sess = gpu_side(cfg, 3, B, 900, 30)
    total = sess.free_pages()
    sess.enable_sampling()
    sess.enable_rules(4)
    allowed = [np.random.default_rng(b).random(cfg.vocab) < 0.6 for b in range(B)]
    for b in range(B):
        sess.set_rules(b, temperature=0.6 + 0.2 * b, presence=0.3 * b, repetition=1.1, bias={b: -5.0}, allowed=allowed[b])
    sess.prefill_seq(0, prompt)
    sess.prefill_shared([0] * B, [None] + [prompt] * (B - 1))
    assert [sess.shared_pages(b) for b in range(B)] == [4] * B
    toks, st = hispec_generate_sampling(sess, n_new, 4, 6, np.random.default_rng(0))
    assert toks.shape == (B, n_new) and st.full_verifies > 0
    for b in range(B):
        assert allowed[b][toks[b]].all()
        assert sess.shared_pages(b) == 4
        assert sess.tokens(b)[:300].tolist() == prompt.tolist()
    assert len({t.tobytes() for t in toks}) == B
    for b in range(B):
        sess.release(b)
    assert sess.free_pages() == total
    sess.close(); model.close()


def test_built_in_choice():
    """Where many sequences share much a call takes the shared form by itself, where little is shared it does not; both agree."""
    cfg = config(32, 8, 128)
    model = hs.Model(cfg, 1)
    for B, prefix, taken in ((48, 2600, True), (3, 300, False)):
        prompts = prompts_of(cfg.vocab, prefix, [20 + b for b in range(B)])
        sess = hs.Session(model, B, prefix + 100, 4)
        sess.enable_logits(True)
        sess.prefill_seq(0, prompts[0])
        sess.prefill_shared([-1] + [0] * (B - 1), [None] + prompts[1:])
        lens = sess.lengths()[:, 0]
        logits = []
        for mode in (-1, 0):
            hs.ee_debug_shared_attention(mode)
            sess.decode_ar(1)
            assert (hs.ee_debug_last_attention(sess.handle) == 3) == (taken and mode == -1), (B, mode)
            logits.append(sess.last_logits().copy())
            for b in range(B):
                sess.rollback(b, 0b111, int(lens[b]))
        assert max_rel(*logits) <= 2e-2
        sess.close()
    model.close()


def test_arena_without_room_for_the_tables():
    """In the smallest arena a session shares pages and decodes as ever, by sequences; attention of given rows is refused."""
    cfg = bf16_d128()
    model = hs.Model(cfg, 4)
    prompts = prompts_of(cfg.vocab, 700, [30, 5])
    hs.ee_debug_shared_attention(1)
    full = hs.ee_session_bytes(model.handle, 2, 2000, 8, 0)
    with pytest.raises(hs.EEError) as e:
        hs.Session(model, 2, 2000, 8, arena_bytes=4096)
    least = int(str(e.value).split("<")[1])                      # (of passes of 512 rows, without the tables)
    assert least < full
    toks = []
    for size, form in ((full, True), (least, False)):
        sess = hs.Session(model, 2, 2000, 8, arena_bytes=size)
        sess.enable_logits(True)
        sess.prefill_seq(0, prompts[0])
        sess.prefill_shared([-1, 0], [None, prompts[1]])
        assert sess.shared_pages(1) == 10
        if form:
            sess.attend_begin([1, 1])
        else:
            with pytest.raises(hs.EEError) as e:
                sess.attend_begin([1, 1])
            assert e.value.code == -3
        sess.decode_ar(1)
        assert (hs.ee_debug_last_attention(sess.handle) == 3) == form
        toks.append(sess.last_logits().copy())
        sess.close()
    assert max_rel(*toks) <= 2e-2
    model.close()
