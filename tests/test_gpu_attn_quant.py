"""isd_attn_quant against a 64-bit statement of attention over the decoded cache (needs a B200)."""
import numpy as np
import pytest
import torch

import paper_2604_11035_b200 as isd_pkg
from paper_2604_11035_b200.binding import ST_BAD_PAGE_ID, ST_SLOT_CAPACITY
from quant_ref import Cache, D, PAGE, TILE, attention, attention_bounds, pack, random_cache, unpack

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Problem:
    """A batch over a random 4-bit cache: slots' contexts and proposals under verification as given."""

    def __init__(self, ctx, n_ver, stride, hq, hkv, seed=0, k_sigma=0.5, spare=3, max_pages=None, sm_scale=0.0):
        self.B, self.N, self.Q, self.hq, self.hkv = len(ctx), stride, 2 * stride - 1, hq, hkv
        self.ctx, self.n_ver = np.array(ctx), np.array(n_ver)
        rng = np.random.default_rng(seed)
        self.have = (self.ctx + self.Q + PAGE - 1) // PAGE
        self.pages = int(self.have.sum()) + spare
        self.width = max_pages or int(self.have.max())
        order = rng.permutation(self.pages)
        self.table = np.full((self.B, self.width), -1, np.int32)
        at = 0
        for b, n in enumerate(self.have):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.cache = random_cache(self.pages, hkv, seed + 1, k_sigma)
        g = torch.Generator().manual_seed(seed + 2)
        self.q = torch.randn(self.B, self.Q, hq, D, generator=g).bfloat16()
        self.k_new, self.v_new = ((torch.randn(self.B, self.Q, hkv, D, generator=g) * 0.5).bfloat16() for _ in range(2))
        self.active = np.ones(self.B, np.uint8)
        self.sm_scale = sm_scale
        self.scale = sm_scale or 1 / np.sqrt(D)

    def to_gpu(self):
        i32 = dict(dtype=torch.int32, device=DEV)
        self.st = dict(ctx_len=torch.tensor(self.ctx, **i32), n_ver=torch.tensor(self.n_ver, **i32), block_tok=torch.zeros(self.B, self.Q, **i32),
                       q_row0=torch.zeros(self.B, **i32), q_stats=torch.zeros(self.B, self.N - 1, 2, device=DEV),
                       page_table=torch.from_numpy(self.table).to(DEV), free_stack=torch.zeros(self.pages, **i32), free_top=torch.zeros(1, **i32),
                       active=torch.from_numpy(self.active).to(DEV), slot_status=torch.zeros(self.B, **i32))
        self.pool = torch.from_numpy(pack(self.cache)).to(DEV)
        self.out = torch.full((self.B, self.Q, self.hq, D), 77.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((self.B, self.Q, self.hq), 77.0, device=DEV)
        self.isd = isd_pkg.Isd(batch=self.B, stride=self.N, n_q_heads=self.hq, n_kv_heads=self.hkv, vocab=64, sm_scale=self.sm_scale,
                               max_pages_per_slot=self.width, num_pages=self.pages, logits_dtype="f32")
        self.dev = [x.to(DEV) for x in (self.q, self.k_new, self.v_new)]
        return self

    def call(self):
        self.isd.isd_attn_quant(self.st, *self.dev, self.pool, self.out, self.lse)

    def slot_values(self, b):
        """Appends slot b's block to the reference cache; its K, V [Hkv, ctx + q_len, 128] and q_len."""
        n, ctx = int(self.n_ver[b]) + self.N, int(self.ctx[b])
        for r in range(n):
            p = ctx + r
            self.cache.store(self.table[b, p // PAGE], p % PAGE, self.k_new[b, r].float().numpy(), self.v_new[b, r].float().numpy())
        for p in range(ctx + n, (ctx + n + PAGE - 1) // PAGE * PAGE):
            self.cache.empty(self.table[b, p // PAGE], p % PAGE)
        pages = [self.cache.values(p) for p in self.table[b, :(ctx + n + PAGE - 1) // PAGE]]
        K, V = (np.concatenate([x[i] for x in pages], 1)[:, :ctx + n] for i in range(2))
        return K, V, n

    def check(self, slots=None, pool=True):
        out, lse = self.out.float().cpu().numpy().astype(np.float64), self.lse.cpu().numpy().astype(np.float64)
        worst = 0.0
        for b in range(self.B):
            if not self.active[b]:
                assert (out[b] == 77).all() and (lse[b] == 77).all(), b
                continue
            K, V, n = self.slot_values(b)
            if slots is not None and b not in slots:
                continue
            o, l, absv, mag = attention(self.q[b, :n].double().numpy(), K, V, int(self.ctx[b]), self.scale)
            tol_o, tol_l = attention_bounds(o, l, absv, mag)
            eo, el = np.abs(out[b, :n] - o), np.abs(lse[b, :n] - l)
            assert (eo <= tol_o).all(), (b, eo.max(), (eo / tol_o).max())
            assert (el <= tol_l).all(), (b, el.max(), (el / tol_l).max())
            assert (out[b, n:] == 77).all() and (lse[b, n:] == 77).all(), b
            worst = max(worst, (eo / tol_o).max())
        if pool:
            got, want = unpack(self.pool.cpu().numpy()), unpack(pack(self.cache))
            tail = self.tail()
            for i in range(2):
                assert np.array_equal(got[0][i][~tail], want[0][i][~tail])  # codes of emptied tokens are not stated
                assert np.array_equal(got[1][i], want[1][i]) and np.array_equal(got[2][i], want[2][i])
        return worst

    def tail(self):
        """[pages, heads, 16] tokens that the append emptied"""
        t = np.zeros((self.pages, self.hkv, PAGE), bool)
        for b in range(self.B):
            end = int(self.ctx[b] + self.n_ver[b]) + self.N
            if self.active[b] and end % PAGE:
                t[self.table[b, end // PAGE], :, end % PAGE:] = True
        return t


@pytest.mark.parametrize("ctx,n_ver,stride,hq,hkv", [
    ([256], [0], 4, 8, 2),                              # the tiny workload's heads
    ([0], [0], 1, 8, 8),                                # a first token: one key
    ([0, 1, 15, 16, 17, 127, 128, 129], [0] * 8, 1, 32, 8),   # single tokens, borders of pages and tiles
    ([113, 100, 300, 0], [3, 0, 2, 3], 4, 40, 8),       # five query heads to a kv head: rows that are not a power of two
    ([1000, 33, 512], [7, 0, 7], 8, 32, 8),             # 60, 32 and 60 rows
    ([700, 250], [15, 4], 16, 32, 8),                   # 124 rows
    ([130, 40], [15, 0], 16, 16, 16),                   # one query head to a kv head: 31 rows
    ([95], [1], 2, 28, 1),                              # 28 query heads to one kv head
    ([77], [0], 1, 128, 1),                             # 128 rows of one token
    ([2047, 2033, 2040], [3, 1, 3], 4, 24, 8),          # blocks across the border of a tile
])
def test_matches_plain_attention(ctx, n_ver, stride, hq, hkv):
    p = Problem(ctx, n_ver, stride, hq, hkv, seed=len(ctx)).to_gpu()
    p.call()
    assert p.isd.isd_read_status() == 0
    p.check()


def test_long_contexts_split_over_many_ctas():
    p = Problem([20000, 5, 7777], [3, 0, 1], 4, 8, 2, seed=5).to_gpu()
    p.call()
    p.check()


def test_ragged_batch_fills_the_machine():
    rng = np.random.default_rng(3)
    p = Problem(rng.integers(0, 700, 120), rng.integers(0, 4, 120), 4, 16, 4, seed=6)
    p.active[[0, 17, 119]] = 0
    p.to_gpu()
    p.call()
    p.check()


def test_more_slots_than_the_shared_memory_plan_holds():
    rng = np.random.default_rng(4)
    p = Problem(rng.integers(0, 40, 1100), rng.integers(0, 2, 1100), 2, 2, 1, seed=7).to_gpu()
    p.call()
    p.check(slots=set(range(0, 1100, 37)) | {1099})


@pytest.mark.parametrize("grow", [0.05, 1.0, 12.0])
def test_scores_that_grow_along_the_context(grow):
    """Keys get louder with the position: the running maximum is raised again and again, by little and by much."""
    p = Problem([900, 1300], [3, 0], 4, 8, 2, seed=8)
    for b in range(2):
        for j, page in enumerate(p.table[b, :int(p.have[b])]):
            p.cache.s[0, page] = np.array(p.cache.s[0, page] * (1 + grow * j))
    from quant_ref import bf16_round
    p.cache.s[0] = bf16_round(p.cache.s[0]).astype(np.float64)
    p.to_gpu()
    p.call()
    p.check()


def test_scores_that_fall_and_tiny_and_huge_values():
    p = Problem([900, 400], [3, 0], 4, 8, 2, seed=9)
    p.cache.s[0, p.table[0, 0]] *= 64.0      # the first page dominates: later probabilities underflow
    p.cache.s[1, p.table[1, :20]] *= 2.0 ** 80
    p.cache.s[1, p.table[1, 20:24]] = 0.0
    p.to_gpu()
    p.call()
    p.check()


def test_scale_argument_and_no_log_sums():
    p = Problem([300, 20], [0, 1], 2, 8, 2, seed=10, sm_scale=0.3).to_gpu()
    p.call()
    p.check()
    out = p.out.clone()
    p.isd.isd_attn_quant(p.st, *p.dev, p.pool, p.out.fill_(5.0), None)
    valid = torch.zeros(2, p.Q, dtype=torch.bool, device=DEV)
    for b in range(2):
        valid[b, :int(p.n_ver[b]) + p.N] = True
    assert torch.equal(p.out[valid], out[valid]) and bool((p.out[~valid] == 5).all())


def test_what_no_row_sees_does_not_matter():
    """Pages that nobody owns, tokens behind the block and other slots' pages hold NaN scales and zeros."""
    p = Problem([100, 260], [0, 3], 4, 8, 2, seed=11, spare=9)
    p.to_gpu()
    end = p.ctx + p.n_ver + p.N
    used = np.zeros((p.pages, PAGE), bool)
    for b in range(2):
        for t in range(int(end[b])):
            used[p.table[b, t // PAGE], t % PAGE] = True
    poison = torch.from_numpy(~used).to(DEV)
    meta = p.pool[:, :, 2048:].contiguous().view(torch.int16).view(p.pages, p.hkv, 4, 16)
    meta[poison[:, None, None, :].expand_as(meta)] = 0x7FC0
    p.pool[:, :, 2048:] = meta.view(p.pages, p.hkv, 64).view(torch.uint8)
    p.call()
    assert p.isd.isd_read_status() == 0
    p.check(pool=False)


def test_a_nan_in_the_cache_reaches_those_who_see_it_alone():
    p = Problem([200, 200], [3, 3], 4, 8, 2, seed=12)
    p.k_new[0, 2, 0, 9] = float("nan")  # seen by rows 2.. of slot 0, heads of kv head 0
    p.to_gpu()
    p.call()
    out, lse = p.out.float(), p.lse
    assert torch.isnan(out[0, 2:, :4]).all() and torch.isnan(lse[0, 2:, :4]).all()
    assert not torch.isnan(out[0, :2]).any() and not torch.isnan(out[0, :, 4:]).any() and not torch.isnan(out[1]).any()
    assert not torch.isnan(lse[0, :2]).any() and not torch.isnan(lse[0, :, 4:]).any()


@pytest.mark.parametrize("stride", [1, 4, 16])
def test_a_nan_value_scale_spoils_outputs_and_no_log_sums(stride):
    """One in the cached part (all rows see it), one in the block (rows from its own on)."""
    p = Problem([300, 200], [0, 0], stride, 8, 2, seed=17)
    clean = Problem([300, 200], [0, 0], stride, 8, 2, seed=17).to_gpu()
    clean.call()
    p.cache.s[1, p.table[0, 3], 1, 5] = np.nan
    p.v_new[1, stride - 1, 0, 7] = float("nan")
    p.to_gpu()
    p.call()
    out, lse = p.out.float(), p.lse
    assert torch.equal(lse[:, :stride], clean.lse[:, :stride])
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, :stride, 4:] = True
    bad[1, stride - 1, :4] = True
    assert torch.equal(torch.isnan(out), bad)
    assert torch.equal(p.out[~bad], clean.out[~bad])


@pytest.mark.parametrize("stride", [1, 4, 16])
@pytest.mark.parametrize("power", [28, 60, 100])
def test_scores_far_beyond_any_probability(power, stride):
    """The largest score takes all the weight: its lead over the second (checked here) is far above the rounding of the scores, an
    fp32 sum of 128 products (129 * 2^-24 of the sum of magnitudes)."""
    p = Problem([500], [0], stride, 8, 2, seed=18)
    p.cache.s[0] *= 2.0 ** power
    p.k_new = (p.k_new.float() * 2.0 ** power).bfloat16()
    p.to_gpu()
    p.call()
    assert p.isd.isd_read_status() == 0
    K, W, n = p.slot_values(0)
    out, lse = p.out.double().cpu().numpy(), p.lse.double().cpu().numpy()
    x = p.q[0].double().numpy()
    checked = 0
    for r in range(n):
        for h in range(8):
            a, mag = K[h // 4, :500 + r + 1] @ x[r, h], np.abs(K[h // 4, :500 + r + 1]) @ np.abs(x[r, h])
            top = np.argsort(a)[-2:]
            err = 144 * 2.0 ** -24 * mag.max()
            assert abs(lse[0, r, h] - a[top[1]] * p.scale) <= err * p.scale + 2.0 ** -20 * abs(a[top[1]]) * p.scale
            if a[top[1]] - a[top[0]] > 4 * err and power >= 28:  # then the second's weight is exp(-2^6) at most
                want = W[h // 4, top[1]]
                assert (np.abs(out[0, r, h] - want) <= 3 * 2.0 ** -8 * np.abs(want) + 1e-20).all(), (r, h)
                checked += 1
    assert checked >= n * 8 * 3 // 4


def test_a_nan_in_a_query_stays_in_its_row():
    p = Problem([300], [3], 4, 8, 2, seed=13)
    p.q[0, 3, 5, 0] = float("nan")
    p.q[0, 4, 2, 0] = float("inf")
    p.to_gpu()
    p.call()
    bad = torch.zeros(1, p.Q, p.hq, dtype=torch.bool)
    bad[0, 3, 5] = bad[0, 4, 2] = True
    assert torch.equal(torch.isnan(p.out.float()).all(-1).cpu(), bad)
    assert torch.equal(torch.isnan(p.out.float()).any(-1).cpu(), bad)


def test_bad_pages_and_lengths_stop_their_slot_alone():
    p = Problem([50, 60, 70, 80], [0, 0, 0, 0], 2, 8, 2, seed=14)
    p.table[1, 2] = p.pages
    p.ctx[2] = p.width * PAGE  # the block would pass the table's row
    p.active[[1, 2]] = 0       # (for the reference only)
    p.to_gpu()
    p.st["active"].fill_(1)
    p.call()
    assert p.isd.isd_read_status() == ST_BAD_PAGE_ID | ST_SLOT_CAPACITY
    assert p.st["slot_status"].tolist() == [0, ST_BAD_PAGE_ID, ST_SLOT_CAPACITY, 0]
    p.check(pool=False)


def test_pages_behind_four_gigabytes():
    p = Problem([70, 33], [1, 0], 2, 32, 8, seed=15)
    far = (1 << 32) // (8 * TILE) + 7
    small = pack(p.cache)
    p.pages_small = p.pages
    table = p.table.copy()
    p.to_gpu()
    pool = torch.zeros(far + p.pages, 8, TILE, dtype=torch.uint8, device=DEV)
    pool[far:] = torch.from_numpy(small).to(DEV)
    p.st["page_table"] = torch.from_numpy(np.where(table >= 0, table + far, -1).astype(np.int32)).to(DEV)
    isd = isd_pkg.Isd(batch=2, stride=2, n_q_heads=32, n_kv_heads=8, vocab=64, max_pages_per_slot=p.width, num_pages=far + p.pages,
                      logits_dtype="f32")
    isd.isd_attn_quant(p.st, *p.dev, pool, p.out, p.lse)
    assert isd.isd_read_status() == 0
    p.pool = pool[far:]
    p.check()


@pytest.mark.parametrize("stride,hq", [(1, 4), (4, 8)])
def test_a_context_beyond_two_to_the_24_tokens(stride, hq):
    """One page stands for all but the last of a context's pages, so that the plain statement can count its sixteen tokens as often."""
    ctx, Q = (1 << 24) + 21, 2 * stride - 1
    many = ctx // PAGE
    p = Problem([ctx % PAGE + PAGE], [0], stride, hq, 1, seed=19, k_sigma=0.1)
    last = p.table[0, 1:].copy()
    table = np.concatenate([np.full(many, p.table[0, 0], np.int32), last])
    p.to_gpu()
    p.st["ctx_len"].fill_(ctx)
    p.st["page_table"] = torch.from_numpy(table[None].copy()).to(DEV)
    isd = isd_pkg.Isd(batch=1, stride=stride, n_q_heads=hq, n_kv_heads=1, vocab=64, max_pages_per_slot=len(table), num_pages=p.pages,
                      logits_dtype="f32")
    isd.isd_attn_quant(p.st, *p.dev, p.pool, p.out, p.lse)
    assert isd.isd_read_status() == 0
    K, V, n = p.slot_values(0)  # [1, 16 + 5 + n, 128]
    weight = np.concatenate([np.full(PAGE, float(many)), np.ones(K.shape[1] - PAGE)])
    out, lse = p.out[0].double().cpu().numpy(), p.lse[0].double().cpu().numpy()
    x = p.q[0].double().numpy()
    for r in range(n):
        L = PAGE + ctx % PAGE + r + 1
        a = x[r] @ K[0, :L].T * p.scale
        e = np.exp(a - a.max(-1, keepdims=True)) * weight[:L]
        t = e.sum(-1, keepdims=True)
        want, wl = (e / t) @ V[0, :L], (a.max(-1, keepdims=True) + np.log(t))[:, 0]
        mag = (np.abs(x[r]) @ np.abs(K[0, :L]).T).max(-1) * p.scale
        # (a CTA's chain of additions is 2^24 / 148 keys long: 2^17 roundings of 2^-24 at most instead of 2^11, below 2^-7 in all)
        to, tl = attention_bounds(want, wl, (e / t) @ np.abs(V[0, :L]), mag)
        extra = 2.0 ** -7
        assert (np.abs(out[r] - want) <= to + extra * ((e / t) @ np.abs(V[0, :L]))).all()
        assert (np.abs(lse[r] - wl) <= tl + extra).all()


def test_stream_repeat_and_captured_replay_give_the_same_bits():
    p = Problem([3000, 64, 900], [3, 0, 2], 4, 32, 8, seed=16).to_gpu()
    p.call()
    first = p.out.clone(), p.lse.clone(), p.pool.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        p.out.fill_(77)
        p.call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            p.call()
    torch.cuda.synchronize()
    assert torch.equal(p.out, first[0])
    for _ in range(3):
        p.out.fill_(77)
        p.lse.fill_(77)
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((p.out, p.lse, p.pool), first))
    p.check()


def test_step_on_the_quantised_cache_verifies_and_commits_like_isd_step():
    """Verification and commit do not depend on the attention: the same state, logits and step number give the same results."""
    from paper_2604_11035_b200 import workloads as wl
    w = wl.Workload("q", batch=5, stride=4, n_q_heads=8, n_kv_heads=2, vocab=4096, ctx_min=20, ctx_max=90, peaked_frac=0.7, steps=3, q_mode=1, seed=4)
    states, isds, outs = [], [], []
    for _ in range(2):
        st = wl.make_state(w, DEV)
        states.append(st)
        isds.append(isd_pkg.isd_for_workload(w, st))
        outs.append(isd_pkg.alloc_verify_out(w.batch, w.stride, DEV))
    pool = [torch.zeros(states[1]["num_pages"], 2, TILE, dtype=torch.uint8, device=DEV) for _ in range(2)]
    att = [torch.zeros(w.batch, w.Q, 8, D, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    prev = None
    for t in range(3):
        q, k, v = wl.make_qkv(w, t, DEV)
        lg = wl.make_logits(w, t, states[0]["ctx_len"])
        a = isds[0].step_args(q=q, k_new=k, v_new=v, k_pool=states[0]["k_pool"], v_pool=states[0]["v_pool"], attn_out=att[0], attn_lse=None,
                              logits_cur=lg, q_prev_logits=prev, out=outs[0])
        isds[0].isd_step(states[0], a, t)
        layers = isds[1].quant_layer_args([dict(q=q, k_new=k, v_new=v, kv_pool=pool[i], attn_out=att[1 + i]) for i in range(2)])
        isds[1].isd_step_quant(states[1], layers, lg, prev, outs[1], t)
        for n in ("accept", "accept_len", "n_emit", "repl_tok", "out_tok", "new_prop_tok"):
            assert torch.equal(outs[0][n], outs[1][n]), (t, n)
        for n in ("ctx_len", "n_ver", "block_tok", "page_table", "free_top"):
            assert torch.equal(states[0][n], states[1][n]), (t, n)
        assert torch.equal(att[1], att[2])
        prev = lg


def test_refusals():
    p = Problem([50], [0], 2, 8, 2).to_gpu()
    p.call()
    q, k, v = p.dev
    for args in ((q.float(), k, v, p.pool, p.out, p.lse), (q, k[:, :1], v, p.pool, p.out, p.lse), (q, k, v, p.pool[:-1], p.out, p.lse),
                 (q, k, v, p.pool.view(torch.int8), p.out, p.lse), (q, k, v, p.pool, p.out, p.lse.double()), (q.cpu(), k, v, p.pool, p.out, p.lse),
                 (None, k, v, p.pool, p.out, p.lse)):
        with pytest.raises(isd_pkg.IsdError):
            p.isd.isd_attn_quant(p.st, *args)
