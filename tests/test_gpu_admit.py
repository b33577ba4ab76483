"""isd_admit against a dictionary model of the allocator (needs a B200)."""
import numpy as np
import pytest
import torch

import paper_2604_11035_b200 as isd_pkg
from paper_2604_11035_b200.binding import ST_BAD_SLOT, ST_MAP_FULL, ST_POOL_EXHAUSTED, ST_SLOT_CAPACITY

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAGE = 16
STATE = ("ctx_len", "n_ver", "block_tok", "q_row0", "page_table", "free_stack", "free_top", "active", "slot_status")


class Batch:
    def __init__(self, B, stride, width, pages, free, seed=0):
        self.B, self.N, self.Q, self.width, self.pages = B, stride, 2 * stride - 1, width, pages
        rng = np.random.default_rng(seed)
        i = lambda *s: rng.integers(-5, 99, s).astype(np.int32)  # noqa: E731  (what is left behind must not matter)
        stack = np.full(pages, -1, np.int32)
        stack[:free] = rng.permutation(pages)[:free]
        self.s = dict(ctx_len=i(B), n_ver=i(B), block_tok=i(B, self.Q), q_row0=i(B), page_table=i(B, width), free_stack=stack,
                      free_top=np.array([free], np.int32), active=np.zeros(B, np.uint8), slot_status=i(B))
        self.st = {k: torch.from_numpy(v.copy()).to(DEV) for k, v in self.s.items()}
        self.st["q_stats"] = torch.zeros(B, stride - 1, 2, device=DEV)
        self.isd = isd_pkg.Isd(batch=B, stride=stride, n_q_heads=4, n_kv_heads=4, vocab=64, max_pages_per_slot=width, num_pages=pages,
                               logits_dtype="f32", mask_token_id=61)

    def admit(self, slots, lens, cap=None, names=("slot_map", "tok_req", "tok_pos")):
        n = len(slots)
        cap = int(sum(max(0, x) for x in lens)) if cap is None else cap
        anchors = np.arange(n, dtype=np.int32) + 500
        maps = isd_pkg.alloc_admit_maps(n, cap, DEV)
        for k in list(maps):
            maps[k].fill_(-9)
            if k not in names and k not in ("result", "cu_len"):
                maps[k] = None
        t = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
        self.isd.isd_admit(self.st, t(slots), t(lens), t(anchors), maps)
        want = self.model(slots, lens, anchors, cap)
        for k, v in want.items():
            if maps.get(k) is not None:
                assert np.array_equal(maps[k].cpu().numpy(), v), (k, maps[k].cpu().numpy(), v)
        for k in STATE:
            assert np.array_equal(self.st[k].cpu().numpy(), self.s[k]), k
        return maps, want

    def model(self, slots, lens, anchors, cap):
        s, n = self.s, len(slots)
        result, cu = np.zeros(n, np.int32), np.zeros(n + 1, np.int32)
        smap, req, pos = np.full(cap, -9, np.int64), np.full(cap, -9, np.int32), np.full(cap, -9, np.int32)
        top, asked, toks, served, used = int(s["free_top"][0]), 0, 0, 0, 0
        was_active, seen = s["active"].copy(), set()
        for i, (b, ln) in enumerate(zip(slots, lens)):
            cu[i] = used
            if not 0 <= b < self.B or was_active[b] or b in seen:
                result[i] = ST_BAD_SLOT
                continue
            seen.add(b)
            want = (ln + self.Q + PAGE - 1) // PAGE
            if ln < 0 or want > self.width:
                result[i] = ST_SLOT_CAPACITY
                continue
            first = asked
            asked, toks = asked + want, toks + ln
            if asked > top:
                result[i] = ST_POOL_EXHAUSTED
            elif toks > cap:
                result[i] = ST_MAP_FULL
            else:
                ids = [int(s["free_stack"][top - 1 - first - j]) for j in range(want)]
                s["page_table"][b, :want] = ids
                s["ctx_len"][b], s["n_ver"][b], s["q_row0"][b], s["slot_status"][b], s["active"][b] = ln, 0, 0, 0, 1
                s["block_tok"][b] = [anchors[i]] + [61] * (self.Q - 1)
                p = np.arange(ln)
                smap[used:used + ln] = np.array(ids, np.int64)[p // PAGE] * PAGE + p % PAGE
                req[used:used + ln], pos[used:used + ln] = i, p
                used += ln
                served += want
        cu[n] = used
        s["free_top"][0] = top - served
        return dict(result=result, cu_len=cu, slot_map=smap, tok_req=req, tok_pos=pos)


@pytest.mark.parametrize("lens", [[0], [1], [15], [16], [700], [0, 0, 5, 0], [13, 300, 1, 16, 0, 47]])
@pytest.mark.parametrize("stride", [1, 4])
def test_admits_in_request_order(lens, stride):
    b = Batch(9, stride, 60, 300, 250)
    b.admit([7, 2, 0, 8, 5, 1][:len(lens)], lens)


def test_nothing_to_admit():
    b = Batch(3, 2, 8, 20, 20)
    b.admit([], [])


@pytest.mark.parametrize("n,B", [(256, 300), (1024, 1100), (1500, 1500), (2500, 2600), (1024, 4096), (70, 4097)])
def test_many_requests(n, B):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 200, n)
    b = Batch(B, 3, 14, 40000, int(((lens + 5 + 15) // 16).sum() * 0.93), seed=n)
    _, want = b.admit(list(rng.permutation(B)[:n]), list(lens))
    assert (want["result"] == ST_POOL_EXHAUSTED).any() and (want["result"] == 0).any()


def test_bad_requests_change_nothing_else():
    b = Batch(8, 2, 6, 64, 40)
    b.admit([3], [20])
    #  in use | out of range | negative length | too long | twice (first counts, also when it is refused) | fine
    _, want = b.admit([3, -1, 8, 2, 4, 4, 5, 5, 6], [5, 5, 5, -1, 100, 10, 9, 9, 30])
    assert want["result"].tolist() == [ST_BAD_SLOT] * 3 + [ST_SLOT_CAPACITY] * 2 + [ST_BAD_SLOT, 0, ST_BAD_SLOT, 0]
    assert b.isd.isd_read_status() == 0


def test_lengths_near_the_ends_of_32_bits():
    b = Batch(4, 2, 6, 64, 40)
    _, want = b.admit([0, 1, 2, 3], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 20, 3], cap=64)
    assert want["result"].tolist() == [ST_SLOT_CAPACITY] * 3 + [0]


def test_requests_for_more_than_two_to_the_31_pages():
    """1024 slots of two million pages each: what a round of them asks for passes 32 bits."""
    B, width, pages = 1100, (1 << 21) + 4096, 64
    i32 = dict(dtype=torch.int32, device=DEV)
    st = dict(ctx_len=torch.zeros(B, **i32), n_ver=torch.zeros(B, **i32), block_tok=torch.zeros(B, 3, **i32), q_row0=torch.zeros(B, **i32),
              q_stats=torch.zeros(B, 1, 2, device=DEV), page_table=torch.empty(B, width, **i32), free_stack=torch.arange(pages, **i32),
              free_top=torch.full((1,), pages, **i32), active=torch.zeros(B, dtype=torch.uint8, device=DEV), slot_status=torch.zeros(B, **i32))
    isd = isd_pkg.Isd(batch=B, stride=2, n_q_heads=4, n_kv_heads=4, vocab=64, max_pages_per_slot=width, num_pages=pages, logits_dtype="f32")
    lens = torch.full((B,), width * PAGE - 3, **i32)
    lens[0], lens[1050:] = 20, 5
    maps = isd_pkg.alloc_admit_maps(B, 100, DEV)
    isd.isd_admit(st, torch.arange(B, **i32), lens, torch.zeros(B, **i32), maps)
    assert maps["result"].tolist() == [0] + [ST_POOL_EXHAUSTED] * (B - 1)
    assert int(st["free_top"]) == pages - 2 and st["active"].nonzero().flatten().tolist() == [0]
    assert st["page_table"][0, :2].tolist() == [63, 62] and int(maps["cu_len"][B]) == 20


def test_maps_that_are_too_short_or_left_out():
    b = Batch(8, 2, 6, 64, 60)
    _, want = b.admit([0, 1, 2], [20, 30, 5], cap=40)
    assert want["result"].tolist() == [0, ST_MAP_FULL, ST_MAP_FULL]
    b.admit([1, 2], [30, 5], names=("tok_pos",))
    b.admit([3, 4], [30, 5], names=())
    b.admit([5, 6], [0, 5], cap=0)


def test_release_and_admit_again_keeps_every_page():
    b = Batch(6, 2, 10, 40, 40)
    rng = np.random.default_rng(1)
    for _ in range(6):
        free_slots = [i for i in range(6) if not b.s["active"][i]]
        k = int(rng.integers(0, len(free_slots) + 1))
        b.admit(list(rng.permutation(free_slots)[:k]), list(rng.integers(0, 120, k)))
        live = [i for i in range(6) if b.s["active"][i]]
        gone = torch.tensor([i for i in live if rng.random() < 0.5], dtype=torch.int32, device=DEV)
        if gone.numel():
            b.isd.isd_release(b.st, gone)
        b.s = {k: b.st[k].cpu().numpy() for k in STATE}
        held = [int(p) for i in range(6) if b.s["active"][i] for p in b.s["page_table"][i, :(b.s["ctx_len"][i] + 3 + 15) // 16]]
        free = b.s["free_stack"][:b.s["free_top"][0]].tolist()
        assert sorted(held + free) == list(range(40))


def test_captured_admission_replays():
    b = Batch(4, 2, 10, 64, 50)
    t = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    slots, lens, anchors, maps = t([2, 0]), t([33, 18]), t([5, 6]), isd_pkg.alloc_admit_maps(2, 80, DEV)
    start = {k: b.st[k].clone() for k in STATE}
    b.isd.isd_admit(b.st, slots, lens, anchors, maps)
    first = [maps[k].clone() for k in maps] + [b.st[k].clone() for k in STATE]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.isd.isd_admit(b.st, slots, lens, anchors, maps)
    for _ in range(2):
        for k in STATE:
            b.st[k].copy_(start[k])
        for k in maps:
            maps[k].fill_(-1)
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip([maps[k] for k in maps] + [b.st[k] for k in STATE], first))


def test_refusals():
    b = Batch(4, 2, 10, 64, 50)
    t = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    maps = isd_pkg.alloc_admit_maps(2, 80, DEV)
    ok = [t([0, 1]), t([3, 3]), t([1, 1])]
    for i, x in ((0, t([0])), (1, t([3, 3]).long()), (2, t([1, 1]).cpu())):
        with pytest.raises(isd_pkg.IsdError):
            b.isd.isd_admit(b.st, *[x if j == i and i else (ok[j] if j or i else x) for j in range(3)], maps)
    with pytest.raises(isd_pkg.IsdError):
        b.isd.isd_admit(b.st, *ok, {**maps, "tok_pos": maps["tok_pos"][:5]})
