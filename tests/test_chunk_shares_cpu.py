"""How the blocks of chunks are given out (csrc/chunk_rows.h), modelled in whole numbers: the
blocks that are dealt out and the shares of the count together cover every tile of every block
once, what a block's cost says is at least what it has, parts of a block lie in shares
one behind the other and in places of their own, and the join is told how many there are."""

import random

import pytest

QB, COST, LEAST, SNAP, KB = 128, 128, 512, 512, 64


class Seq:
    def __init__(self, lq, length, blocks, deal, qpb, window, sinks):
        self.lq, self.len = lq, length
        self.dealt = blocks // deal * deal if deal else 0
        self.nb = blocks - self.dealt
        self.first = max(length - lq, 0)
        self.most = window + sinks + qpb + 192 if window else 2 ** 31 - 1
        self.linear = 0 if self.most < self.first else min((self.most - self.first) // qpb, self.nb)
        self.qpb = qpb

    def cost(self, n):
        return (self.first + (n + 1) * self.qpb if n < self.linear else self.most) + COST

    def upto(self, n):
        m = min(n, self.linear)
        return m * (self.first + COST) + m * (m + 1) // 2 * self.qpb + (n - m) * (self.most + COST)


def tiles_of(q, n, qpb, window, sinks):
    pos0, rows = q.len - q.lq + n * qpb, min(qpb, q.lq - n * qpb)
    end, first = pos0 + rows - 1, max(pos0 - window + 1, 0) if window else 0
    few = (min(sinks, first) + KB - 1) // KB
    return 0 if end < 0 else few + (end + KB) // KB - max(first // KB, few)


def check(r):
    kv, group, nseq = r.choice([1, 2, 8]), r.choice([1, 2, 3, 5, 8, 10, 40, 130, 200]), r.choice([1, 2, 5, 40, 70])
    nsub = -(-group // QB)
    qpb, heads = QB // -(-group // nsub), kv * nsub
    window, sinks, least = r.choice([0, 0, 1, 20, 100, 1000, 5000]), r.choice([0, 4, 100, 3000]), r.choice([0, 64])
    grid = r.choice([8, 16, 64, 512])
    deal = grid // heads if grid % heads == 0 else 0
    seqs = []
    for _ in range(nseq):
        lq, n = r.choice([0, 1, 3, r.randint(0, 40), r.randint(0, 600)]), r.choice([0, 1, 5, r.randint(0, 300), r.randint(0, 20000)])
        seqs.append(Seq(lq, n, -(-lq // qpb) if lq * group > least else 0, deal, qpb, window, sinks))
    for q in seqs:
        dealt = sorted((b % heads, q.nb + q.dealt - 1 - (k * deal + (deal - 1 - b // heads if k & 1 else b // heads)))
                       for k in range(q.dealt // deal if deal else 0) for b in range(grid))
        assert dealt == [(h, n) for h in range(heads) for n in range(q.nb, q.nb + q.dealt)]
        for n in range(min(q.nb, 20)):
            assert q.upto(n + 1) - q.upto(n) == q.cost(n)
    total = sum(q.upto(q.nb) * heads for q in seqs)
    shares = min(grid, -(-total // LEAST))
    if not shares:
        return
    size, more = divmod(total, shares)
    begin = lambda i: i * size + min(i, more)
    share_of = lambda u: u // (size + 1) if u < more * (size + 1) else more + (u - more * (size + 1)) // size
    near = lambda c: min(SNAP, c // 2, size // 2)

    def locate(u):
        for s, q in enumerate(seqs):
            each = q.upto(q.nb)
            if u >= each * heads:
                u -= each * heads
                continue
            h, u = divmod(u, each)
            n = max(x for x in range(q.nb) if q.upto(x) <= u)
            return s, h, n, u - q.upto(n)

    def snapped(u):
        if u >= total:
            return total
        s, _, n, at = locate(u)
        c = seqs[s].cost(n)
        return u - at if at <= near(c) else u - at + c if c - at <= near(c) else u

    cover, tasks, places = {}, {}, set()
    for sh in range(shares):
        u, u1 = snapped(begin(sh)), snapped(begin(sh + 1))
        assert u <= u1
        while u < u1:
            s, h, n, at = locate(u)
            q = seqs[s]
            c, block = q.cost(n), u - at
            to = min(c, u1 - block)
            u = block + to
            T = tiles_of(q, n, qpb, window, sinks)
            assert T * KB <= c - COST + KB - 1
            tile = lambda x: min(max(-(-(x - COST) // KB), 0), T)
            t0, t1 = tile(at), tile(to)
            if t0 == t1 and not (T == 0 and at == 0):
                continue
            cover.setdefault((s, h, n), []).append((sh, t0, t1))
            if t1 - t0 < T:
                assert (sh, t0 == 0) not in places
                places.add((sh, t0 == 0))
                if t0 == 0:
                    tasks[sh] = (s, h, n), share_of(block + min(COST + (T - 1) * KB + 1, c - near(c)) - 1) - sh + 1
    for s, q in enumerate(seqs):
        for h in range(heads):
            for n in range(q.nb):
                parts, at = cover[s, h, n], 0
                for _, a, b in parts:
                    assert a == at
                    at = b
                assert at == tiles_of(q, n, qpb, window, sinks)
                first = parts[0][0]
                assert [p[0] for p in parts] == list(range(first, first + len(parts)))
                if len(parts) > 1:
                    assert tasks[first] == ((s, h, n), len(parts))


@pytest.mark.parametrize("block", range(6))
def test_cover(block):
    for i in range(60):
        check(random.Random(1000 * block + i))
