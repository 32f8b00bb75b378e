"""The example's session off the default stream and in a graph."""
import pytest
import torch

from gpu_helpers import ensure_built

pytestmark = pytest.mark.gpu
LAYERS, HEADS, KV, HD, PAGE = 2, 8, 2, 64, 16


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


def session(**kw):
    from paper_2609_34045_gb300.kv4_session import Session
    f = dict(n_users=5, max_ctx=200, n_pages=60, page_tokens=PAGE, max_tokens=64)
    f.update(kw)
    return Session(LAYERS, HEADS, KV, HD, **f)


def rows(n, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, h, HD, generator=g).to(torch.bfloat16).cuda() for h in (HEADS, KV, KV)]


def some_passes(busy):
    """Prompts, a step and a fork; before every pass the stream is given work (`busy`) that its inputs have to wait for."""
    s, out = session(), []
    for i, counts in enumerate(({0: 33, 1: 7, 2: 50}, {0: 1, 1: 1, 2: 1}, {0: 1, 3: 1})):
        step = s.begin(counts)
        for layer in range(LAYERS):
            q, k, v = rows(sum(counts.values()), 10 * i + layer)
            late = [torch.zeros_like(x) for x in (q, k, v)]
            busy()
            for a, b in zip(late, (q, k, v)):
                a.copy_(b)
            out.append(s.attend(layer, step, *late))
            for a in late:
                a.zero_()
        if i == 1:
            s.fork([0], [3])
    s.free([1])
    live = s.compact()
    return [o.cpu() for o in out] + [live.cpu(), s.table.cpu(), s.status.cpu()]


def test_a_session_on_another_stream():
    want = some_passes(lambda: None)
    x = torch.randn(2048, 2048, device="cuda")

    def busy():
        y = x
        for _ in range(20):
            y = torch.matmul(y, x) * 0.02
        return y

    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = some_passes(busy)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and len(want) == len(got)
    assert got[-1].item() == 0


def test_a_captured_layer_of_a_pass():
    """The calls of a pass are in the graph, which reads its inputs anew."""
    s = session()
    step = s.begin({0: 20, 2: 1})
    q, k, v = rows(21, 1)
    for layer in range(LAYERS):
        s.attend(layer, step, q, k, v)
    q2, k2, v2 = rows(21, 2)
    want = s.attend(1, step, q2, k2, v2).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s.attend(1, step, q, k, v)
    for a, b in zip((q, k, v), (q2, k2, v2)):
        a.copy_(b)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and s.status.item() == 0


def test_a_full_pool_stops_a_pass_before_it_begins():
    """Users go on where they were once there is room again, with the outputs of a session that was never short."""
    from paper_2609_34045_gb300.kv4_session import NoRoom

    def passes(s, short):
        out = []
        for i, counts in enumerate(({0: 30, 1: 17, 2: 16}, {0: 2, 1: 1}, {0: 1, 2: 3})):
            if i == 2 and short:
                tables = s.table.clone(), s.lengths.clone(), s.refs.clone()
                for bad in (counts, {1: 1, 0: 17}, {2: 1}):
                    with pytest.raises(NoRoom):
                        s.begin(bad)
                assert all(torch.equal(a, b) for a, b in zip(tables, (s.table, s.lengths, s.refs)))
            if i == 2:
                s.free([1])
            step = s.begin(counts)
            out.append([s.attend(layer, step, *rows(sum(counts.values()), 3 * i + layer)) for layer in range(LAYERS)])
        assert s.status.item() == 0
        return out

    full, roomy = session(n_pages=5), session()
    assert all(torch.equal(a, b) for x, y in zip(passes(full, True), passes(roomy, False)) for a, b in zip(x, y))


def test_a_full_pool_stops_a_fork():
    from paper_2609_34045_gb300.kv4_session import NoRoom
    s = session(n_pages=4)
    s.begin({0: 40, 1: 3})
    before = s.table.clone(), s.lengths.clone(), s.refs.clone()
    with pytest.raises(NoRoom):
        s.fork([0], [1])  # (new pages are taken before old ones are given back)
    assert all(torch.equal(a, b) for a, b in zip(before, (s.table, s.lengths, s.refs)))
    s.free([1])
    s.fork([0], [1])
    assert s.lengths.tolist()[:2] == [40, 40] and s.refs.tolist() == [2, 2, 1, 1] and s.status.item() == 0
