"""ptq_kv_cache_copy_pages against torch's indexing, byte by byte."""
import pytest
import torch

import paper_2601_19675_amd as ptq

pytestmark = pytest.mark.gpu


def cache(pages, heads, page, row, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    b = lambda *s: torch.randint(0, 256, s, device="cuda", generator=g, dtype=torch.uint8)
    # scales of any bits, NaN among them
    return b(2, pages, heads, page, row), b(2, pages, heads, page, 4).view(torch.float32).squeeze(-1), b(2, pages, heads, page)


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("heads,page,row", [(8, 32, 128), (1, 1, 8), (3, 1, 24), (5, 16, 40), (1, 256, 256), (7, 4, 56), (32, 64, 64), (1, 2, 16)])
def test_within_a_cache(heads, page, row):
    pages = 41
    c = cache(pages, heads, page, row, 1)
    order = torch.randperm(pages, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    source, target = order[:20].to(torch.int32), order[20:40].to(torch.int32)
    want = [x.clone() for x in c]
    for x in want:
        x[:, target.long()] = x[:, source.long()]
    ptq.ptq_kv_cache_copy_pages(*c, source, *c, target)
    assert same(c, want)


@pytest.mark.parametrize("n", [1, 2, 500])
def test_to_another_cache_of_another_size(n):
    a, b = cache(600, 2, 8, 96, 3), cache(501, 2, 8, 96, 4)
    source = ints([(i * 7) % 600 for i in range(n)])      # (a page may go to several places)
    source[-1] = source[0]
    target = ints([500 - i for i in range(n)])
    want = [x.clone() for x in b]
    before = [x.clone() for x in a]
    for x, y in zip(want, a):
        x[:, target.long()] = y[:, source.long()]
    ptq.ptq_kv_cache_copy_pages(*a, source, *b, target)
    assert same(b, want) and same(a, before)


def test_numbers_that_are_no_pages_are_passed_over():
    a, b = cache(6, 3, 4, 32, 5), cache(4, 3, 4, 32, 6)
    want = [x.clone() for x in b]
    source, target = ints([0, -1, 6, 5, 2, 2 ** 31 - 1, 3]), ints([0, 1, 1, 4, -1, 2, 3])
    for x, y in zip(want, a):
        x[:, 0], x[:, 3] = y[:, 0], y[:, 3]
    ptq.ptq_kv_cache_copy_pages(*a, source, *b, target)
    assert same(b, want)
    ptq.ptq_kv_cache_copy_pages(*a, ints([]), *b, ints([]))
    assert same(b, want)


def test_replayed_and_on_another_stream():
    c = cache(12, 2, 16, 64, 7)
    source, target = ints([0, 1]), ints([10, 11])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ptq.ptq_kv_cache_copy_pages(*c, source, *c, target)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ptq.ptq_kv_cache_copy_pages(*c, source, *c, target)
    for i in range(4):
        source.copy_(ints([i, i + 1]))
        target.copy_(ints([11 - i, 6]))
        want = [x.clone() for x in c]
        for x in want:
            x[:, target.long()] = x[:, source.long()]
        graph.replay()
        torch.cuda.synchronize()
        assert same(c, want), i
