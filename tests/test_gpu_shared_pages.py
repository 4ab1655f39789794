"""GPU: sequences that share the pages of a common prefix (ee_prefill_shared) -- against the oracle and against sessions that
share nothing, through everything that reads, writes and gives back pages."""
import numpy as np
import pytest

import synth
import paper_2510_01336_amd as hs
from hs_common import TOL, OracleSide, bf16_small, check_state, gpu_side, max_rel, run_round

pytestmark = pytest.mark.gpu

PAGE = 64


def tree(vocab, prefix, tails, seed=0):
    common = synth.gen_prompt(vocab, prefix, 900 + seed)
    out = []
    for i, n in enumerate(tails):
        t = synth.gen_prompt(vocab, n, 50 + i + 100 * seed)
        t[0] = i                                                # (parts where it begins)
        out.append(np.concatenate([common, t]).astype(np.int32))
    return out


@pytest.mark.parametrize("cfg", [synth.tiny_config(), bf16_small()], ids=["f32", "bf16"])
def test_shared_prompts_against_the_oracle(cfg):
    """Prompts of one 150-token prefix: prompt logits, cached K and V, and rounds of draft, verification and rollback follow the oracle."""
    tails = [9, 70, 1, 33]
    prompts = tree(cfg.vocab, 150, tails)
    B, cap = len(tails), 400
    O = OracleSide(cfg, 31, plain_twin=True)
    model, sess = gpu_side(cfg, 31, B, cap, 24)
    sess.enable_logits(True)
    first = [int(sess.prefill_seq(0, prompts[0]))]
    before = sess.free_pages()
    rest = sess.prefill_shared([-1, 0, 0, 0], [None] + prompts[1:])
    assert rest[0] == -1
    first += [int(t) for t in rest[1:]]
    assert [sess.shared_pages(b) for b in range(B)] == [2] * B
    own = [-(-(len(p) + 1) // PAGE) - 2 for p in prompts[1:]]
    assert before - sess.free_pages() == sum(own)
    ref, margins = O.prefill(prompts, cap)
    tol = TOL[cfg.dtype]
    for b in range(B):
        if margins[b] > 1e-2:
            assert first[b] == int(ref[b])
    # continue from the oracle's own first token where a near-tie went the other way: same texts on both sides
    for b in range(B):
        if first[b] != int(ref[b]):
            pytest.skip("a first token inside the margin")
    for b in range(B):
        for layer in range(cfg.n_layers):
            k, v = sess.read_kv(b, layer, 0, len(prompts[b]))
            for side in O.sides():
                c = side.seqs[b].cache
                n = len(prompts[b])
                assert max_rel(k, c.K[layer][:n].reshape(k.shape)) <= tol and max_rel(v, c.V[layer][:n].reshape(v.shape)) <= tol
    rng = np.random.default_rng(5)
    for i in range(3):
        run_round(O, sess, 4, 0.7, rng, i % 2 == 1, tol)
        check_state(O, sess)
        for b in range(B):
            sess.poison_dead_kv(b)
    sess.close(); model.close()


@pytest.mark.parametrize("cfg", [synth.tiny_config(gamma=(1.0, 0.3, 0.3)), bf16_small(gamma=(1.0, 0.3, 0.3))], ids=["f32", "bf16"])
def test_streams_of_shared_and_separate_sequences(cfg):
    """Greedy streams and loops of sequences that share a prefix equal those of sequences of their own (fp32: all, bf16: what the
    first token agrees on, to 2e-2 in the logits)."""
    from paper_2510_01336_amd.loop import hispec_generate
    prompts = tree(cfg.vocab, 200, [5, 40, 64])
    model, sess = gpu_side(cfg, 77, 3, 1000, 40)
    solo = hs.Session(model, 3, 1000, 40)
    for s in (sess, solo):
        s.enable_logits(True)
    want = solo.prefill(prompts)
    z_want = solo.last_logits()
    sess.prefill_seq(0, prompts[0])
    got = sess.prefill_shared([-1, 0, 0], [None, prompts[1], prompts[2]])
    z = sess.last_logits()
    if cfg.dtype == "bf16":                                     # (the last 512-row piece of a build is kept: its last row ends the last prompt)
        assert max_rel(z[-1], z_want[-1]) <= 2e-2
    else:
        assert np.array_equal(got[1:], want[1:])
        a, b = sess.decode_ar(30), solo.decode_ar(30)
        assert np.array_equal(a, b)
        for s in (sess, solo):
            for i, p in enumerate(prompts):
                s.rollback(i, 0b111, len(p))
        t1, _ = hispec_generate(sess, 30, 4, n_i=6)
        assert np.array_equal(t1, a)
    solo.close(); sess.close(); model.close()


@pytest.mark.parametrize("cfg", [synth.tiny_config(), bf16_small()], ids=["f32", "bf16"])
def test_rollback_into_a_shared_page_writes_a_copy(cfg):
    """Two sequences hold the same pages; one goes back into them and says something else.  The other's cache stays as it was, bit for bit."""
    prompt = tree(cfg.vocab, 250, [8])[0]
    model, sess = gpu_side(cfg, 8, 2, 400, 24, True, True)
    sess.prefill_seq(0, prompt)
    sess.prefill_shared([-1, 0], [None, prompt])
    assert sess.shared_pages(1) == 4
    kv = [sess.read_kv(0, l, 0, len(prompt)) for l in range(cfg.n_layers)]
    for back in (200, 130, 64, 10):                             # inside a page, at its edge, near the beginning
        sess.rollback(1, 0b111, back)
        free = sess.free_pages()
        assert sess.shared_pages(1) == back // PAGE + 1
        sess.poison_dead_kv(1)                                   # (the shared page stays)
        S = np.random.default_rng(back).integers(0, cfg.vocab, (2, 3)).astype(np.int32)
        sess.draft_inject(S)
        sess.verify_intermediate()
        sess.verify_full()
        assert sess.shared_pages(1) == back // PAGE
        for l in range(cfg.n_layers):
            k, v = sess.read_kv(0, l, 0, len(prompt))
            assert np.array_equal(k, kv[l][0]) and np.array_equal(v, kv[l][1])
            k, v = sess.read_kv(1, l, 0, back)
            assert np.array_equal(k, kv[l][0][:back]) and np.array_equal(v, kv[l][1][:back])
        sess.rollback(0, 0b111, len(prompt))
        sess.prefill_shared([-1, 0], [None, prompt])
    # the source goes back into its own shared pages: it gets the copy, the other keeps the pages
    other = [sess.read_kv(1, l, 0, len(prompt)) for l in range(cfg.n_layers)]
    sess.rollback(0, 0b111, 100)
    sess.decode_ar(2)
    assert sess.shared_pages(0) == 1
    for l in range(cfg.n_layers):
        k, v = sess.read_kv(1, l, 0, len(prompt))
        assert np.array_equal(k, other[l][0]) and np.array_equal(v, other[l][1])
    sess.close(); model.close()


def test_pages_come_back():
    """Releases, restarts and prompts that share with their own past: the pool's count is that of the distinct pages held."""
    cfg = bf16_small()
    prompts = tree(cfg.vocab, 300, [20, 90, 5])
    model, sess = gpu_side(cfg, 9, 3, 600, 10)
    total = sess.free_pages()

    def pages(n):
        return -(-n // PAGE)
    sess.prefill_seq(0, prompts[0])
    sess.prefill_shared([0, 0, 0], [None, prompts[1], prompts[2]])
    held = pages(len(prompts[0]) + 1) + sum(pages(len(p) + 1) - 4 for p in prompts[1:])
    assert sess.free_pages() == total - held and [sess.shared_pages(b) for b in range(3)] == [4, 4, 4]
    sess.release(0)                                             # the source leaves, its prefix stays with the others
    held -= pages(len(prompts[0]) + 1) - 4
    assert sess.free_pages() == total - held and sess.shared_pages(1) == 4
    # a conversation goes on: the new prompt begins like the sequence's own context
    longer = np.concatenate([sess.tokens(1), synth.gen_prompt(cfg.vocab, 100, 4)]).astype(np.int32)
    sess.prefill_shared([-1, 1, -1], [None, longer, None])
    held += pages(len(longer) + 1) - pages(len(prompts[1]) + 1)
    assert sess.free_pages() == total - held and sess.shared_pages(1) == 4
    # everybody restarts from everybody, the sources among them
    sess.prefill_shared([1, 2, 1], [longer, prompts[1], longer])
    n = (len(longer) - 1) // PAGE
    assert sess.shared_pages(0) == sess.shared_pages(2) == n - (n > len(longer) // PAGE)
    for b in range(3):
        sess.release(b)
    assert sess.free_pages() == total
    sess.close(); model.close()


def test_edges_and_refusals():
    cfg = bf16_small()
    model, sess = gpu_side(cfg, 10, 3, 200, 10)
    p = synth.gen_prompt(cfg.vocab, 129, 1)
    q = p.copy(); q[63] = (q[63] + 1) % cfg.vocab
    with pytest.raises(hs.EEError) as e:
        sess.prefill_shared([1, -1, -1], [p, None, None])
    assert e.value.code == -2                                   # its source has no context
    for src in ([3, -1, -1], [-2, -1, -1]):
        with pytest.raises(hs.EEError) as e:
            sess.prefill_shared(src, [p, None, None])
        assert e.value.code == -1
    with pytest.raises(hs.EEError):
        sess.prefill_shared([-1] * 3, [None] * 3)
    with pytest.raises(ValueError):
        sess.prefill_shared([-1] * 3, [p[:0], None, None])
    with pytest.raises(ValueError):
        sess.prefill_shared([-1], [p])
    with pytest.raises(hs.EEError):
        sess.shared_pages(3)
    sess.prefill_shared([-1, -1, -1], [p, None, None])           # no source: an ordinary prompt
    assert sess.shared_pages(0) == 0
    sess.prefill_shared([-1, 0, 0], [None, q, p[:64]])           # parts at the first page's last token; a page long: its last token has to run
    assert [sess.shared_pages(b) for b in range(3)] == [0, 0, 0]
    sess.prefill_shared([-1, 0, 0], [None, p[:65], p])           # a page and one token; the whole prompt again
    assert [sess.shared_pages(b) for b in range(3)] == [2, 1, 2]
    before = (sess.lengths().tolist(), [sess.tokens(b).tolist() for b in range(3)], sess.free_pages())
    bad = p.copy(); bad[70] = cfg.vocab
    for prompts in ([bad, None, None], [synth.gen_prompt(cfg.vocab, 300, 2), None, None]):
        with pytest.raises(hs.EEError):
            sess.prefill_shared([0, -1, -1], prompts)
        assert (sess.lengths().tolist(), [sess.tokens(b).tolist() for b in range(3)], sess.free_pages()) == before
    sess.close()
    # a pool that holds the prompts only because they share; a copy-on-write that finds no page leaves the session as it was
    sess = hs.Session(model, 3, 200, 10, 5)
    sess.prefill_seq(0, p)
    sess.prefill_shared([-1, 0, 0], [None, p, p])
    assert sess.free_pages() == 0
    sess.rollback(1, 0b111, 100)                                # into shared page 1: frees its third page
    assert sess.free_pages() == 1
    sess.release(2)
    sess.prefill_shared([-1, -1, 0], [None, None, p])
    before = (sess.lengths().tolist(), sess.free_pages())
    assert before[1] == 1
    sess.rollback(0, 0b111, 100)
    sess.rollback(2, 0b111, 110)                                # three sequences in one page: two copies at least, and there are pages for them
    sess.draft(2)
    assert [sess.shared_pages(b) for b in range(3)] == [1, 1, 1]
    sess.close()
    sess = hs.Session(model, 2, 200, 10, 4)
    sess.prefill_seq(0, p[:127])
    sess.prefill_shared([-1, 0], [None, p[:127]])
    assert sess.free_pages() == 1 and sess.shared_pages(1) == 1
    sess.close(); model.close()


def test_capacity_of_a_copy():
    """A sequence that would need a page for its copy and finds none is refused; nothing changes."""
    cfg = bf16_small()
    model, sess = gpu_side(cfg, 10, 2, 200, 10)
    sess.close()
    p = synth.gen_prompt(cfg.vocab, 190, 1)
    sess = hs.Session(model, 2, 200, 10, 5)
    sess.prefill_seq(0, p[:191])                                # three pages
    sess.prefill_shared([-1, 0], [None, p[:190]])                # two shared, one of its own
    assert sess.free_pages() == 1
    sess.rollback(1, 0b111, 100)                                # its own page comes back
    assert sess.free_pages() == 2
    assert sess.decode_ar(1).shape == (2, 1)                    # the copy, and no page for the other yet
    assert sess.free_pages() == 1 and sess.shared_pages(1) == 1
    sess.close()
    sess = hs.Session(model, 2, 200, 10, 3)
    sess.prefill_seq(0, p[:120])                                # two pages of three
    sess.prefill_shared([-1, 0], [None, p[:100]])                # one shared, one of its own: none left
    assert sess.free_pages() == 0
    sess.rollback(1, 0b111, 20)                                 # back into the shared page: its own comes back
    sess.rollback(0, 0b111, 30)                                 # ... and the source into the same page
    assert sess.free_pages() == 2 and sess.shared_pages(0) == sess.shared_pages(1) == 1
    sess.decode_ar(1)
    assert sess.free_pages() == 1 and sess.shared_pages(0) == 0
    sess.close()
    sess = hs.Session(model, 2, 200, 10, 2)
    sess.prefill_seq(0, p[:70])
    sess.rollback(0, 0b111, 66)
    with pytest.raises(hs.EEError) as e:
        sess.prefill_shared([-1, 0], [None, p[:66]])             # one shared page and one too many
    assert e.value.code == -3
    sess.close(); model.close()


def test_two_copies_of_one_page():
    """Two sequences rolled back into the page that they share: the first gets a copy, the other keeps the page, and one free page is enough."""
    cfg = bf16_small()
    p, other = synth.gen_prompt(cfg.vocab, 190, 1), synth.gen_prompt(cfg.vocab, 80, 2)
    model = hs.Model(cfg, 10)
    roomy, tight = hs.Session(model, 3, 200, 10), hs.Session(model, 3, 200, 10, 4)
    toks = []
    for sess in (roomy, tight):
        sess.prefill_seq(0, p[:120])
        sess.prefill_shared([-1, 0, -1], [None, p[:100], None])
        sess.rollback(0, 0b111, 30)
        sess.rollback(1, 0b111, 20)
        sess.prefill_seq(2, other)
        assert sess.shared_pages(0) == sess.shared_pages(1) == 1
        if sess is tight:
            assert sess.free_pages() == 1
        toks.append(sess.decode_ar(4))
        assert sess.shared_pages(0) == sess.shared_pages(1) == 0
    assert tight.free_pages() == 0 and np.array_equal(*toks)
    roomy.close(); tight.close(); model.close()
