"""Several continuations of one prompt, with the operators of include/sssd_kv8.h and sssd_op_logprobs together: the prompt is admitted once and forked, every step makes room,
stores, attends over the shared prefix, samples, scores its tokens, and from time to time the better continuations take the places of the others; the pool is compacted and moved to another
size on the way.  Every step is compared with 64 bits on what the cache holds, sequence by sequence."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from kv8_reference import attend
from paper_2411_05894_amd import binding as sv
from paper_2411_05894_amd import kv8

DEV = "cuda:0"
U = 2.0 ** -24


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Model:
    """Layers of QKV product, rotation, cache and attention, each adding to a hidden row, and a vocabulary."""

    def __init__(self, layers, nq, nkv, d, hidden, vocab, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.nq, self.nkv, self.d, self.hidden, self.vocab, self.layers = nq, nkv, d, hidden, vocab, layers
        self.embed = torch.randn(vocab, hidden, generator=g, device=DEV)
        self.qkv = [sv.sssd_op_pack_weight((torch.randn((nq + 2 * nkv) * d, hidden, generator=g, device=DEV) * 0.1).to(torch.bfloat16)) for _ in range(layers)]
        self.out = [sv.sssd_op_pack_weight((torch.randn(hidden, nq * d, generator=g, device=DEV) * 0.1).to(torch.bfloat16)) for _ in range(layers)]
        self.head = sv.sssd_op_pack_weight((torch.randn(vocab, hidden, generator=g, device=DEV) * 0.05).to(torch.bfloat16))
        self.rope = kv8.Rope(d, 10000.0, device=DEV)

    def product(self, x, w, n):
        return sv.sssd_op_gemm(*sv.sssd_op_pack_activation(x), w, x.shape[0], n, x.shape[1])

    def rows(self, tokens, book, lens, attention, first=0):
        """tokens [B][n] -> logits [B * n][vocab]; attention(layer, q, out) after the rows are stored."""
        B, n = tokens.shape
        x = self.embed[tokens.long()].view(B * n, -1)
        for layer in range(self.layers):
            qkv = self.product(x, self.qkv[layer], (self.nq + 2 * self.nkv) * self.d).view(B, n, self.nq + 2 * self.nkv, self.d)
            q, k, v = qkv.split([self.nq, self.nkv, self.nkv], 2)
            book.cache.sssd_kv8_append(layer, k, v, lens, first=first, rope=self.rope, q=q, q_out=q)
            out = torch.zeros(B, n, self.nq, self.d, device=DEV)
            attention(layer, q, out)
            x = x + self.product(out.view(B * n, -1), self.out[layer], self.hidden)
        return self.product(x, self.head, self.vocab)


def held(cache, layer, lens, rows):
    kk, vv = (torch.zeros(len(lens), rows, cache.n_kv_heads, cache.head_dim, device=DEV) for _ in range(2))
    cache.sssd_kv8_read(layer, None, ints(lens), kk, vv)
    return kk.double(), vv.double()


@pytest.mark.parametrize("fmt,n", [("e4m3", 1), ("int8", 1), ("e4m3", 4)])
def test_best_of_eight(fmt, n):
    B, max_seq, vocab = 8, 256, 1008
    model = Model(2, 8, 2, 64, 128, vocab, 3)
    cache = kv8.Kv8Cache(2, 8, 2, 64, B, max_seq, fmt, n_pages=40, device=DEV)
    book = kv8.Kv8Pages(cache)
    g = torch.Generator(device=DEV).manual_seed(4)
    prompt = torch.randint(0, vocab, (1, 75), generator=g, device=DEV, dtype=torch.int32)
    lens = ints([0] * B)
    book.sssd_kv8_reserve(75, lens[:1].contiguous())
    for at in range(0, 75, 25):                                # the prompt, through slot 0, a piece at a time
        here = ints([at])
        model.rows(prompt[:, at:at + 25], book, here, lambda layer, q, out: cache.sssd_kv8_attention(layer, q, here, out))
    lens[0] = 75
    book.sssd_kv8_fork(ints([0] * B), lens)
    assert lens.tolist() == [75] * B
    score, history = torch.zeros(B, device=DEV), [[] for _ in range(B)]
    tokens = torch.randint(0, vocab, (B, n), generator=g, device=DEV, dtype=torch.int32)
    starts, shared, workspace = ints([0, B]), ints([75]), cache.sssd_kv8_shared_workspace(B, n)
    uniform = torch.rand(200, B * n, generator=g, device=DEV)
    for step in range(18):
        was = lens.tolist()
        book.sssd_kv8_reserve(n, lens)

        def attention(layer, q, out):
            cache.sssd_kv8_attention_shared(layer, q, lens, out, starts, shared, workspace)
            kk, vv = held(cache, layer, [a + n for a in was], max_seq)
            for b in range(B):
                want, mass, most = attend(q[b], kk[b, :was[b] + n], vv[b, :was[b] + n], was[b])
                assert ((out[b].double() - want).abs() <= mass * (2 * most * (2.0 ** -22 + 256 * U) + 2.0 ** -20)).all(), (step, layer, b)
        logits = model.rows(tokens, book, lens, attention)
        sampled = sv.sssd_op_sample(logits, sv.SamplingParams(1.0, 50, 1.0), uniform[step])
        lp, ranks, entropy, ids, top = sv.sssd_op_logprobs(logits, sampled[:, None].contiguous(), n_top=3)
        want = torch.log_softmax(logits.double(), 1)
        assert ((lp.double() - torch.gather(want, 1, sampled[:, None].long())).abs() <= 200 * U).all()       # |x| of some tens, sums of some tens of terms
        assert (ranks < 50).all() and torch.equal(ids[:, 0].long(), logits.argmax(1)) and (entropy > 0).all()
        score += lp.view(B, n).sum(1)
        lens += n                                              # all rows of the step are kept
        for b in range(B):
            history[b] += tokens[b].tolist()
        tokens = sampled.view(B, n)
        if step % 5 == 4:                                      # the better half goes on, twice each
            order = torch.argsort(score, descending=True, stable=True).tolist()
            origins = list(range(B))
            for loser, winner in zip(order[B // 2:], order[:B // 2]):
                origins[loser] = winner
            before = [held(cache, layer, lens.tolist(), max_seq) for layer in range(2)]
            at = lens.tolist()
            book.sssd_kv8_fork(ints(origins), lens)
            assert lens.tolist() == [at[o] for o in origins]
            for layer in range(2):
                after = held(cache, layer, lens.tolist(), max_seq)
                assert all(torch.equal(y, x[origins]) for x, y in zip(before[layer], after))
            pick = torch.tensor(origins, device=DEV)
            score, tokens, history = score[pick].clone(), tokens[pick].contiguous(), [list(history[o]) for o in origins]
        if step in (6, 12):
            before = [held(cache, layer, lens.tolist(), max_seq) for layer in range(2)]
            if step == 6:
                in_use = ints([0])
                book.sssd_kv8_compact(in_use=in_use)
                assert (book.refs[:in_use.item()] > 0).all() and (book.refs[in_use.item():] == 0).all()
            else:                                              # a larger pool
                larger = kv8.Kv8Cache(2, 8, 2, 64, B, max_seq, fmt, n_pages=64, device=DEV)
                other = kv8.Kv8Pages(larger)
                book.sssd_kv8_compact(to=other)
                assert cache.sssd_kv8_sync() == sv.SSSD_OK
                cache, book = larger, other
            for layer in range(2):
                after = held(cache, layer, lens.tolist(), max_seq)
                assert all(torch.equal(x, y) for x, y in zip(before[layer], after))
    assert cache.sssd_kv8_sync() == sv.SSSD_OK
    # what a continuation holds is what its own tokens alone give, written by the same steps without its neighbours
    alone = kv8.Kv8Cache(2, 8, 2, 64, 1, max_seq, fmt, device=DEV)
    single = kv8.Kv8Pages(alone)
    b = int(torch.argmax(score))
    for at in range(0, 75, 25):
        here = ints([at])
        single.sssd_kv8_reserve(25, here)
        model.rows(prompt[:, at:at + 25], single, here, lambda layer, q, out: alone.sssd_kv8_attention(layer, q, here, out))
    for i in range(0, len(history[b]), n):
        here = ints([75 + i])
        single.sssd_kv8_reserve(n, here)
        model.rows(ints([history[b][i:i + n]]), single, here, lambda layer, q, out: alone.sssd_kv8_attention(layer, q, here, out))
    total = 75 + len(history[b])
    assert lens.tolist()[b] == total
    (k0, _), (k1, _) = held(cache, 0, lens.tolist(), max_seq), held(alone, 0, [total], max_seq)
    assert torch.equal(k0[b], k1[0])                           # layer 0 sees tokens and positions alone


def test_a_step_replays_while_sequences_come_and_go():
    """Room, store and attention of a step in one graph; between replays slots are forked and emptied, the groups' arrays changed, other work done eagerly."""
    B, n, nq, nkv, d = 6, 3, 8, 2, 64
    cache = kv8.Kv8Cache(1, nq, nkv, d, B, 300, "e4m3", n_pages=60, device=DEV)
    book = kv8.Kv8Pages(cache)
    g = torch.Generator(device=DEV).manual_seed(9)
    lens, counts = ints([0] * B), ints([n] * B)
    first = torch.randn(1, 130, nkv, d, generator=g, device=DEV)
    book.sssd_kv8_reserve(130, lens[:1].contiguous())
    cache.sssd_kv8_append(0, first, first, lens[:1].contiguous())
    lens[0] = 130
    book.sssd_kv8_fork(ints([0, 0, 0, 0, -1, -1]), lens)
    counts[4:] = 0
    starts, shared, workspace = ints([0, 4, 6]), ints([130, 0]), cache.sssd_kv8_shared_workspace(B, n)
    q, k, v = (torch.zeros(B, n, h, d, device=DEV) for h in (nq, nkv, nkv))
    out = torch.zeros_like(q)

    def step():
        book.sssd_kv8_reserve(n, lens, counts)
        cache.sssd_kv8_append(0, k, v, lens, counts=counts)
        cache.sssd_kv8_attention_shared(0, q, lens, out, starts, shared, workspace, counts=counts)
    keep = [t.clone() for t in (book.table, book.refs, cache.cache)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t, x in zip((book.table, book.refs, cache.cache), keep):
        t.copy_(x)
    origins = [None, [0, 1, 1, 1, 3, -1], [0, 0, 0, 0, 0, 0], [0, 1, 2, -1, -1, -1], None]
    for turn, who in enumerate(origins):
        if who is not None:
            book.sssd_kv8_fork(ints(who), lens)
            live = [b for b, o in enumerate(who) if o >= 0]
            counts.copy_(ints([n if o >= 0 else 0 for o in who]))
            starts.copy_(ints([0, len(live), 6]))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        out.fill_(5.5)
        graph.replay()
        was = lens.tolist()
        other = torch.randn(500, 500, device=DEV) @ torch.randn(500, 500, device=DEV)
        assert other.isfinite().all() and cache.sssd_kv8_sync() == sv.SSSD_OK
        c = counts.tolist()
        kk, vv = held(cache, 0, [a + m for a, m in zip(was, c)], 300)
        for b in range(B):
            assert (out[b, c[b]:] == 5.5).all()
            if c[b]:
                want, mass, most = attend(q[b], kk[b, :was[b] + n], vv[b, :was[b] + n], was[b])
                assert ((out[b].double() - want).abs() <= mass * (2 * most * (2.0 ** -22 + 256 * U) + 2.0 ** -20)).all(), (turn, b)
        lens += counts
