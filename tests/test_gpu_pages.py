"""The pool's pages on the GPU against the one-page-at-a-time form of pages_ref.py: whole numbers and copies, all equal."""
import random

import pytest
import torch

import pages_ref as ref
from paper_2609_39068_b200 import binding

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


class Pool:
    """B slots over P pages: some rows share the pages of others, some pages are pruned, some are held from outside."""

    def __init__(self, seed, B, P, width, longest, shapes=((3, 16), (5,)), dtypes=(torch.bfloat16, torch.float32), alias=0.3, absent=0.1):
        r = random.Random(seed)
        self.rng, self.B, self.P, self.width = r, B, P, width
        free = list(range(P))
        r.shuffle(free)
        self.lens, self.table = [], []
        for i in range(B):
            n = r.choice([0, r.randint(0, longest), r.randint(0, longest)])
            row = [-1] * width
            other = r.randrange(i) if i and r.random() < alias else -1
            share = 0 if other < 0 else r.randint(0, min(n, self.lens[other]) // 16)
            for b in range(ref.pages(n)):
                if b < share:
                    row[b] = self.table[other][b]
                elif r.random() >= absent and free:
                    row[b] = free.pop()
            self.lens.append(n), self.table.append(row)
        self.refs = [0] * P
        for row, n in zip(self.table, self.lens):
            for e in row[:ref.pages(n)]:
                if e >= 0:
                    self.refs[e] += 1
        for e in r.sample(range(P), P // 10):
            self.refs[e] += 1
        g = torch.Generator().manual_seed(seed)
        self.buffers = [torch.randint(0, 255, (P,) + s + (4,), generator=g, dtype=torch.uint8).view(t).cuda() for s, t in zip(shapes, dtypes)]
        self.p = binding.make_params(B, 4, 4, 64, width, P, 1)
        self.ws = binding.alloc_pages_workspace(self.p)

    def on_gpu(self):
        return torch.tensor(self.table, **I32), torch.tensor(self.lens, **I32), torch.tensor(self.refs, **I32)

    def update(self, new_lens, parent=None, in_place=False, status=0):
        t, n, c = self.on_gpu()
        want = ref.update(self.table, self.lens, self.refs, new_lens, parent)
        before = [b.clone() for b in self.buffers]
        outs = (t, n, c) if in_place else (torch.full_like(t, -9), torch.full_like(n, -9), torch.full_like(c, -9))
        left = torch.zeros(1, **I32)
        binding.se_pages_update(self.p, t, n, c, torch.tensor(new_lens, **I32), *outs, left, self.ws,
                                parent=None if parent is None else torch.tensor(parent, **I32), buffers=self.buffers)
        assert binding.se_last_device_status(self.ws) == (binding.SE_DEV_NO_PAGES if want[3] < 0 else status)
        assert outs[0].tolist() == want[0]
        assert outs[1].tolist() == want[1]
        assert outs[2].tolist() == want[2]
        assert left.tolist() == [want[3]]
        for b, x in zip(self.buffers, before):
            for f, to in want[4]:
                x[to] = x[f]
            assert torch.equal(b.view(torch.uint8), x.view(torch.uint8))
        assert int(self.ws[256:].view(torch.int32)[256:256 + 64].abs().sum()) == 0        # counts of changes are zero again
        self.table, self.lens, self.refs = want[0], want[1], want[2]
        return want

    def compact(self, in_place=False):
        t, n, c = self.on_gpu()
        want = ref.compact(self.table, self.lens, self.refs)
        before = [b.clone() for b in self.buffers]
        to, co = (t, c) if in_place else (torch.full_like(t, -9), torch.full_like(c, -9))
        where, live = torch.full_like(c, -9), torch.zeros(1, **I32)
        binding.se_pages_compact(self.p, t, n, c, to, co, where, live, self.ws, buffers=binding.page_buffers(self.buffers))
        assert binding.se_last_device_status(self.ws) == 0
        assert to.tolist() == want[0] and co.tolist() == want[1] and where.tolist() == want[2] and live.tolist() == [want[3]]
        for b, x in zip(self.buffers, before):
            y = x.clone()
            for f, k in want[4]:
                y[k] = x[f]
            assert torch.equal(b.view(torch.uint8), y.view(torch.uint8))
        self.table, self.refs = want[0], want[1]
        return want

    def random_step(self):
        r = self.rng
        parent = [r.choice([s, s, s, r.randrange(self.B), -1]) for s in range(self.B)]
        old = [0 if s < 0 else self.lens[s] for s in parent]
        new = [max(0, min(16 * self.width, n + r.choice([0, 1, 1, 5, 40, -1, -20, -n]))) for n in old]
        return parent, new


@pytest.mark.parametrize("seed,B,P,width,longest", [(1, 1, 4, 3, 40), (2, 5, 60, 9, 100), (3, 64, 1500, 30, 400), (4, 200, 3000, 20, 250),
                                                    (5, 3, 20000, 700, 11000),
                                                    (6, 8192, 30000, 6, 60)])
def test_many_steps(seed, B, P, width, longest):
    """Steps after one another, each on what the last one left: forks, ends, cuts, growth, and compaction in between."""
    pool = Pool(seed, B, P, width, longest)
    copies = moves = 0
    for k in range(8):
        parent, new = pool.random_step()
        copies += len(pool.update(new, parent)[4])
        if k % 3 == 2:
            moves += len(pool.compact(in_place=k == 5)[4])
        pool.update([min(16 * width, n + 1) for n in pool.lens], in_place=k % 2 == 0)
    assert B < 5 or (copies > 0 and moves > 0)


def test_beams_share_and_part():
    pool = Pool(7, 6, 40, 8, 1, alias=0, absent=0)
    pool.table, pool.lens, pool.refs = [[-1] * 8 for _ in range(6)], [0] * 6, [0] * 40
    pool.update([40, 0, 0, 0, 0, 0])                                # a prompt of 40 tokens: three pages, the last one open
    got = pool.update([40] * 6, [0] * 6)                            # six beams: two shared pages, five copies of the last
    assert len(got[4]) == 5 and got[2][got[0][0][0]] == 6 and got[2][got[0][0][2]] == 1
    got = pool.update([41, 41, 0, 0, 0, 0], [3, 3, -1, -1, -1, -1])  # two beams go on from the fourth
    assert len(got[4]) == 1 and sum(c > 0 for c in got[2]) == 4
    got = pool.update([32, 33, 0, 0, 0, 0])                         # whole pages stay shared, nothing is copied
    assert got[4] == [] and got[2][got[0][0][0]] == 2
    got = pool.update([20, 33, 0, 0, 0, 0])                         # a cut inside a page that the other row holds whole
    assert len(got[4]) == 1 and got[4][0][0] == got[0][1][1]


def test_not_enough_pages_changes_nothing():
    pool = Pool(9, 8, 30, 12, 60, alias=0.5)
    got = pool.update([192] * 8)
    assert got[3] < 0
    got = pool.update([192] * 8, in_place=True)
    assert got[3] < 0
    pool.update([n + 1 for n in pool.lens])                         # the scratch is clean


def test_odd_page_sizes_and_one_buffer_of_many():
    pool = Pool(11, 20, 300, 12, 150, shapes=((1,), (7,), (1025,), (3, 64), (4096,)), dtypes=(torch.float32,) * 5)
    for _ in range(3):
        parent, new = pool.random_step()
        pool.update(new, parent)
    pool.compact()


def test_full_and_empty_pools():
    pool = Pool(13, 4, 16, 8, 64, alias=0, absent=0)
    pool.table, pool.lens, pool.refs = [[4 * r + b if b < 4 else -1 for b in range(8)] for r in range(4)], [64] * 4, [1] * 16
    pool.compact()
    assert pool.update([65, 64, 64, 64])[3] == -1                   # no page is left
    assert pool.update([0, 65, 65, 65])[3] == 1                     # freed pages count
    pool.update([0] * 4)
    pool.compact()
    assert pool.refs == [0] * 16


def test_reports():
    pool = Pool(15, 3, 40, 8, 100, alias=0, absent=0)
    pool.lens, pool.table, pool.refs = [33, 40, 16], [[0, 1, 2] + [-1] * 5, [3, 4, 5] + [-1] * 5, [6] + [-1] * 7], [1] * 7 + [0] * 33
    t, n, c = pool.on_gpu()
    left = torch.zeros(1, **I32)
    # slot 0 and 2 ask for what there is not, slot 1 goes on
    for new, parent, bad in (([129, 41, -1], None, [0, 2]), ([5, 41, 5], [7, 1, -2], [0, 2])):
        to, no, co = torch.full_like(t, -9), torch.full_like(n, -9), torch.full_like(c, -9)
        binding.se_pages_update(pool.p, t, n, c, torch.tensor(new, **I32), to, no, co, left, pool.ws,
                                parent=None if parent is None else torch.tensor(parent, **I32), buffers=pool.buffers)
        assert binding.se_last_device_status(pool.ws) == binding.SE_DEV_BAD_LENGTH
        assert no.tolist() == [33, 41, 16] and to.tolist() == pool.table and co.tolist() == pool.refs and left.tolist() == [33]
    t[1, 1] = 40                                                    # no page of the pool
    binding.se_pages_update(pool.p, t, n, c, n, to, no, co, left, pool.ws, buffers=pool.buffers)
    assert binding.se_last_device_status(pool.ws) == binding.SE_DEV_BAD_PAGE_ID
    assert to.tolist() == t.tolist() and co.tolist() == pool.refs


def test_faulty_slots_stay_as_they_are():
    """Rows and lengths bit for bit, entries behind the length included; what shares their pages goes on with copies."""
    pool = Pool(19, 5, 40, 8, 100, alias=0, absent=0)
    tail = [7, 99, -5]
    pool.lens, pool.refs = [33, 33, 16 * 8 + 1, 20, -3], [2, 2, 2] + [1] * 2 + [0] * 35
    pool.table = [[0, 1, 2, -1, -1] + tail, [0, 1, 2, -1, -1] + tail, [8, 9, 10, 11, 12] + tail, [3, 4, -1, -1, -1] + tail, [-1, 6, 6, 6, 6] + tail]
    t, n, c = pool.on_gpu()
    left = torch.zeros(1, **I32)
    # slot 0 asks for too much, slots 2 and 4 have no length, slot 3 wants to go on from slot 2; slot 1 goes on from page 2, which slot 0 holds
    new, parent = [400, 34, 8, 8, 8], [0, 1, 2, 2, 4]
    before = [b.clone() for b in pool.buffers]
    to, no, co = torch.full_like(t, -9), torch.full_like(n, -9), torch.full_like(c, -9)
    binding.se_pages_update(pool.p, t, n, c, torch.tensor(new, **I32), to, no, co, left, pool.ws, parent=torch.tensor(parent, **I32),
                            buffers=pool.buffers)
    assert binding.se_last_device_status(pool.ws) == binding.SE_DEV_BAD_LENGTH
    assert no.tolist() == [33, 34] + pool.lens[2:]
    assert to.tolist() == [pool.table[0], [0, 1, 5] + [-1] * 5] + pool.table[2:]
    assert co.tolist() == [2, 2, 1, 1, 1, 1] + [0] * 34 and left.tolist() == [34]
    for b, x in zip(pool.buffers, before):
        x[5] = x[2]
        assert torch.equal(b.view(torch.uint8), x.view(torch.uint8))
    # without parents, in place
    binding.se_pages_update(pool.p, to, no, co, torch.tensor([-1, 34, 5, 20, 5], **I32), to, no, co, left, pool.ws, buffers=pool.buffers)
    assert binding.se_last_device_status(pool.ws) == binding.SE_DEV_BAD_LENGTH
    assert no.tolist() == [33, 34] + pool.lens[2:] and co.tolist() == [2, 2, 1, 1, 1, 1] + [0] * 34
    assert to.tolist() == [pool.table[0], [0, 1, 5] + [-1] * 5] + pool.table[2:3] + [[3, 4] + [-1] * 6] + pool.table[4:]
    # compaction leaves rows without a length alone
    where = torch.full_like(c, -9)
    binding.se_pages_compact(pool.p, to, no, co, torch.empty_like(t), torch.empty_like(c), where, left, pool.ws, buffers=pool.buffers)
    assert binding.se_last_device_status(pool.ws) == binding.SE_DEV_BAD_LENGTH and left.tolist() == [6]


def test_replayed_from_a_graph():
    pool = Pool(17, 16, 400, 12, 150)
    t, n, c = pool.on_gpu()
    new, left = n + 1, torch.zeros(1, **I32)
    args = [pool.p, t, n, c, new, t, n, c, left, pool.ws]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            binding.se_pages_update(*args, buffers=pool.buffers)
            new.add_(1)
    for _ in range(20):
        g.replay()
    torch.cuda.synchronize()
    assert binding.se_last_device_status(pool.ws) == 0
    table, lens, refs = pool.table, pool.lens, pool.refs
    for _ in range(20):
        table, lens, refs, free, _ = ref.update(table, lens, refs, [x + 1 for x in lens])
    assert n.tolist() == lens and t.tolist() == table and c.tolist() == refs and left.tolist() == [free]
