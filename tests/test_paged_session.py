"""PagedLayer's own bookkeeping (pages, rows, positions), on the CPU with the library's calls stubbed."""
import numpy as np
import pytest

from paper_2605_05219_amd import binding as B, paged as PG
from paper_2605_05219_amd.paged_session import PagedLayer


@pytest.fixture
def made(monkeypatch):
    """made(rows, n_pages): a layer of pages of 16 rows whose requests hold `rows`; layer.calls gets the arguments of its evictions."""
    import torch
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *size, device=None, **kw: empty(*size, **kw))

    def make(rows, n_pages):
        layer = PagedLayer(4, 2, 64, len(rows), n_pages, page_rows=16)
        layer.calls = []
        monkeypatch.setattr(PG, "attn_evict", lambda *args: layer.calls.append(args))
        for r, n in enumerate(rows):
            layer.pages[r] = layer._take(-(-n // 16))
            layer.rows[r] = layer.pos[r] = n
        return layer
    return make


def whole(layer, n_pages):
    """Every page is free or one request's."""
    held = [p for pages in layer.pages for p in pages]
    assert sorted(layer.free + held) == list(range(n_pages))
    assert all(len(p) * layer.P >= n for p, n in zip(layer.pages, layer.rows))


@pytest.mark.parametrize("rows,budget,keep,after", [
    ([150], 100, 200, [150]), ([150, 300, 90], 100, 200, [150, 200, 90]), ([150], 100, 150, [150]), ([150, 20], 100, 80, [80, 20]),
    ([100], 100, 80, [100]),
])
def test_an_eviction_leaves_no_request_with_more_rows_than_it_held(made, rows, budget, keep, after):
    layer = made(rows, 80)
    dropped = layer.evict(budget, keep, first=2, recent=8)
    assert list(layer.rows) == after and dropped == sum(rows) - sum(after)
    assert list(layer.pos) == rows
    assert len(layer.calls) == (after != rows)
    for call in layer.calls:                    # rows, keep, first, recent; the index has room for what is kept
        assert [min(a, b) for a, b in zip(call[1], call[2])] == [x for x, n in zip(after, rows) if x != n]
        assert call[-2].numel() == layer.H_kv * sum(min(a, b) for a, b in zip(call[1], call[2]))
    whole(layer, 80)


def test_pages_of_an_eviction_that_fails_are_free_again(made, monkeypatch):
    layer = made([150, 150], 24)                # 20 pages held, 4 free: enough for one request's copy, not for both
    free, pages = sorted(layer.free), [list(p) for p in layer.pages]
    with pytest.raises(RuntimeError, match="out of pages"):
        layer.evict(100, 48, first=2, recent=8)
    whole(layer, 24)
    assert sorted(layer.free) == free and layer.pages == pages and list(layer.rows) == [150, 150] and not layer.calls

    def refuse(*args):
        raise B.GdnError(-10, "attn_evict")
    monkeypatch.setattr(PG, "attn_evict", refuse)
    layer.rows[1] = 90
    with pytest.raises(B.GdnError):
        layer.evict(100, 48, first=2, recent=8)
    whole(layer, 24)
    assert sorted(layer.free) == free and layer.pages == pages and list(layer.rows) == [150, 90]


@pytest.mark.parametrize("keep,first,recent,want", [(60, 4, 64, (4, 56)), (3, 4, 64, (3, 0)), (0, 4, 64, (0, 0)), (68, 4, 64, (4, 64)), (100, 4, 64, (4, 64))])
def test_an_eviction_to_few_rows_keeps_of_the_first_and_the_last_what_there_is_room_for(made, keep, first, recent, want):
    layer = made([150, 200], 80)
    layer.evict(100, keep, first=first, recent=recent)
    (call,) = layer.calls
    assert list(call[2]) == [keep] * 2 and list(call[3]) == [want[0]] * 2 and list(call[4]) == [want[1]] * 2
    assert list(layer.rows) == [keep] * 2
    whole(layer, 80)


def test_a_step_that_fails_loses_no_page_and_no_row(made, monkeypatch):
    import torch
    layer = made([15, 31], 6)                   # 3 pages held, 3 free

    def refuse(*args):
        raise B.GdnError(-3, "refused")
    monkeypatch.setattr(PG, "attn_rope_append", refuse)
    q, k = torch.zeros(80, 4, 64), torch.zeros(80, 2, 64)
    with pytest.raises(RuntimeError, match="out of pages"):
        layer.step(q, k, k, [30, 50])
    with pytest.raises(B.GdnError):
        layer.step(q[:4], k[:4], k[:4], [2, 2])
    assert list(layer.rows) == list(layer.pos) == [15, 31]
    whole(layer, 6)
