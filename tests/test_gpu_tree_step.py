"""Steps with drafted trees as a server runs them: K and V of the nodes written, attention over the cache in every layer, the
vocabulary projection, verification and the accepted paths' rows moved together, over several steps of the same cache.

Each operator's results are held against its definition, from the inputs it got.  What is left in the cache after the
steps has to be what the accepted tokens alone would have left, and a captured step has to give what the eager one gives."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu

HEADS, GROUP, D, LAYERS, V, PAGE = 2, 2, 64, 2, 48, 16
WIDTH = HEADS * GROUP * D
NODES = [7, 1, 40, 3, 12]
FIRST = [0, 30, 5, 127, 64]
SCALE = D ** -0.5


class Model:
    """A toy: rows of an embedding, products with vectors instead of matrices, so that a row does not depend on its batch."""

    def __init__(self, seed):
        g = T.gen(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.embed = r(V, WIDTH).bfloat16()
        self.wq, self.wk, self.wv = (1 + 0.3 * r(LAYERS, n) for n in (WIDTH, HEADS * D, HEADS * D))
        self.head = (r(V, WIDTH) / 8).bfloat16()
        self.norm = torch.ones(WIDTH, dtype=torch.bfloat16, device="cuda")
        self.head_q, self.head_scale = torch.empty(V, WIDTH, dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
        B.dspark_lm_head_quantize(self.head, self.head_q, self.head_scale)

    def keys(self, layer, x):
        n = HEADS * D
        return ((x[:, :n].float() * self.wk[layer]).bfloat16().view(-1, HEADS, D), (x[:, n:].float() * self.wv[layer]).bfloat16().view(-1, HEADS, D))


class Step:
    """Buffers of a step of a fixed layout, and the step itself: only launches, so that it can be captured."""

    def __init__(self, model, cache):
        self.model, self.cache = model, cache
        n, R = sum(NODES), len(NODES)
        self.off, self.first, self.next_first = T.offsets(NODES), T.i32(FIRST), T.i32(FIRST)
        self.tokens, self.parents = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
        self.draft, self.u, self.u_last = torch.zeros(n, V, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(R, device="cuda")
        self.accepted = torch.zeros(R, dtype=torch.int32, device="cuda")
        self.out_tokens, self.path = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
        self.status = T.status()
        self.workspace = B.workspace(B.dspark_tree_attention_workspace_bytes(n, HEADS * GROUP, HEADS, D))
        self.xq, self.xs = torch.empty(n, WIDTH, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        self.logits = torch.empty(n, V, device="cuda")
        self.attended = [torch.empty(n, HEADS * GROUP, D, dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
        self.queries = [None] * LAYERS

    def run(self):
        m, c = self.model, self.cache.handle
        x = m.embed[self.tokens.long()]
        for l in range(LAYERS):
            k, v = m.keys(l, x)
            B.dspark_kv_write(c, k, v, self.first, self.off, layer=l, dev_status=self.status)
            q = (x.float() * m.wq[l]).bfloat16().view(-1, HEADS * GROUP, D)
            self.queries[l] = q
            B.dspark_tree_attention(q, c, self.first, self.off, parents=self.parents, scale=SCALE, out=self.attended[l], layer=l,
                                    dev_status=self.status, workspace=self.workspace)
            x = (x.float() + self.attended[l].view(-1, WIDTH).float()).bfloat16()
        B.dspark_rms_norm_quant(x, m.norm, 1e-6, out_q=self.xq, out_scale=self.xs)
        B.dspark_lm_head_int8(self.xq, self.xs, m.head_q, m.head_scale, out_logits=self.logits, dev_status=self.status)
        self.target = torch.softmax(self.logits, 1)
        B.dspark_verify_tree(self.target, self.draft, self.tokens, self.parents, self.off, self.u, self.u_last, accepted_len=self.accepted,
                             out_tokens=self.out_tokens, out_path=self.path, dev_status=self.status)
        B.dspark_kv_commit(c, self.first, self.off, self.accepted, self.path, out_first=self.next_first, dev_status=self.status)


def feed(step, roots, seed):
    """Trees drafted from random rows, into the step's buffers; (tokens, parents) of the nodes."""
    g = T.gen(seed)
    n = sum(NODES)
    draft = torch.softmax(torch.randn(n, V, generator=g, device="cuda"), 1)
    parents = T.random_parents(NODES, seed)
    off = step.off.tolist()
    tokens = [0] * n
    for r, count in enumerate(NODES):
        tokens[off[r]] = roots[r]
        for i in range(1, count):
            tokens[off[r] + i] = int(torch.multinomial(draft[off[r] + parents[off[r] + i]], 1, generator=g))
    step.tokens.copy_(T.i32(tokens))
    step.parents.copy_(T.i32(parents))
    step.draft.copy_(draft)
    step.u.copy_(torch.rand(n, generator=g, device="cuda"))
    step.u_last.copy_(torch.rand(len(NODES), generator=g, device="cuda"))
    return tokens, parents


def make(kind, seed, model):
    cache = T.Cache([f + 6 * n for f, n in zip(FIRST, NODES)], PAGE, HEADS, D, kind, layers=LAYERS, seed=seed)
    g = T.gen(seed + 50)
    history = []
    for r, n in enumerate(FIRST):                             # what is there before: rows of tokens, in both layers
        toks = torch.randint(0, V, (n,), generator=g, device="cuda")
        history.append(toks.tolist())
        if n:
            for l in range(LAYERS):
                cache.put(r, range(n), *model.keys(l, model.embed[toks]), layer=l)
    return Step(model, cache), history


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
def test_steps(kind):
    model = Model(3)
    eager, history = make(kind, 4, model)
    captured, _ = make(kind, 4, model)
    blank = captured.cache.snapshot()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        captured.run()
    assert T.same(captured.cache.snapshot(), blank)           # a capture runs nothing
    first, roots, accepted_all = list(FIRST), [1, 2, 3, 4, 5], 0
    off = eager.off.tolist()
    for s in range(5):
        for step in (eager, captured):
            step.first.copy_(T.i32(first))
            tokens, parents = feed(step, roots, 100 + s)
        before = eager.cache.snapshot()
        eager.run()
        graph.replay()
        torch.cuda.synchronize()
        assert int(eager.status.item()) == 0 and int(captured.status.item()) == 0
        # the captured step: the same bits
        for a, b in ((eager.logits, captured.logits), (eager.accepted, captured.accepted), (eager.out_tokens, captured.out_tokens),
                     (eager.path, captured.path), (eager.next_first, captured.next_first)):
            assert torch.equal(a, b)
        assert T.same(eager.cache.snapshot(), captured.cache.snapshot())
        # verification, from the step's own probabilities
        acc, out, path = T.verify(eager.target, eager.draft, tokens, parents, off, eager.u.tolist(), eager.u_last.tolist())
        assert (acc, out, path) == (eager.accepted.tolist(), eager.out_tokens.tolist(), eager.path.tolist())
        assert eager.next_first.tolist() == [f + 1 + a for f, a in zip(first, acc)]
        # attention, over the cache as it was before the paths were moved: written anew from what the step wrote
        twin, _ = make(kind, 4, model)
        for t, b in zip((twin.cache.k, twin.cache.v), before):
            t.view(torch.uint8).copy_(b.view_as(t.view(torch.uint8)))
        for t, b in zip((twin.cache.ks, twin.cache.vs), before[2:]):
            if t is not None:
                t.view(torch.int32).copy_(b)
        x = model.embed[eager.tokens.long()]
        for l in range(LAYERS):
            k, v = model.keys(l, x)
            for r, n in enumerate(NODES):
                twin.cache.put(r, range(first[r], first[r] + n), k[off[r]: off[r + 1]], v[off[r]: off[r + 1]], layer=l)
            want, bound, _, _ = T.attention(twin.cache, eager.queries[l], first, off, parents, SCALE, l)
            err = (eager.attended[l].double() - want).abs()
            assert bool((err <= bound).all()), float((err / bound).max())
            x = (x.float() + eager.attended[l].view(-1, WIDTH).float()).bfloat16()
        # what is certain now
        for r in range(len(NODES)):
            history[r] += [tokens[off[r]]] + out[off[r]: off[r] + acc[r]]
            roots[r] = out[off[r] + acc[r]]
            first[r] += 1 + acc[r]
            assert len(history[r]) == first[r]
        accepted_all += sum(acc)
    assert accepted_all > 5                                   # paths were moved
    # the first layer's rows depend on their token alone: those of the history, bit for bit
    twin, _ = make(kind, 4, model)
    for r, toks in enumerate(history):
        twin.cache.put(r, range(len(toks)), *model.keys(0, model.embed[torch.tensor(toks, device="cuda")]))
        for a, b in zip(eager.cache.values(r, range(len(toks))), twin.cache.values(r, range(len(toks)))):
            assert torch.equal(a, b)


def test_two_steps_at_once():
    """Two streams, each with its own cache, buffers and workspace, give what each gives alone."""
    model = Model(5)
    alone, both = [], []
    for seed in (1, 2):
        step, _ = make("int8", seed, model)
        feed(step, [1, 2, 3, 4, 5], seed)
        step.run()
        torch.cuda.synchronize()
        alone.append(step)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for seed in (1, 2):
        step, _ = make("int8", seed, model)
        feed(step, [1, 2, 3, 4, 5], seed)
        both.append(step)
    torch.cuda.synchronize()
    for _ in range(4):                                        # the same step again: nothing depends on the times
        for step, stream in zip(both, streams):
            with torch.cuda.stream(stream):
                step.run()
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        assert int(a.status.item()) == 0 and int(b.status.item()) == 0
        assert torch.equal(a.logits, b.logits) and torch.equal(a.out_tokens, b.out_tokens) and torch.equal(a.next_first, b.next_first)
        assert T.same(a.cache.snapshot(), b.cache.snapshot())
