"""Pages of a step against a plain form on the host: who gets pages, who gives them back, where tokens lie."""
import random

import pytest
import torch

import paper_2511_11248_amd as tman
from gpu_helpers import dev

pytestmark = pytest.mark.gpu
ERR_INDEX = -10


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=dev())


def plain(table, page, lens, more, stack, left, n_tokens):
    """(table, new_lens, left, q_start, slots, positions, owners, stack), everything as lists; tables are long enough."""
    table, stack = [list(r) for r in table], list(stack)
    pages = lambda n: -(-n // page)  # noqa: E731
    for b, (n, m) in enumerate(zip(lens, more)):
        for e in range(pages(n + m), pages(n)):
            stack[left] = table[b][e]
            left += 1
    asked_pages = asked_tokens = 0
    new_lens, starts, slots, positions, owners, top = [], [0], [], [], [], left
    for b, (n, m) in enumerate(zip(lens, more)):
        need = max(0, pages(n + m) - pages(n))
        asked_pages += need
        asked_tokens += max(0, m)
        granted = m > 0 and asked_tokens <= n_tokens and (need == 0 or asked_pages <= left)
        if granted:
            for e in range(need):
                top -= 1
                table[b][pages(n) + e] = stack[top]
            for j in range(n, n + m):
                slots.append(table[b][j // page] * page + j % page)
                positions.append(j)
                owners.append(b)
        new_lens.append(n + m if granted or m < 0 else n)
        starts.append(len(slots))
    rest = [-1] * (n_tokens - len(slots))
    return table, new_lens, top, starts, slots + rest, positions + rest, owners + rest, stack


class Step:
    def __init__(self, seed, lens, more, page, free, n_tokens, slack=0):
        r = random.Random(seed)
        self.page, self.lens, self.more, self.free, self.n_tokens = page, lens, more, free, n_tokens
        used = [-(-n // page) for n in lens]
        wide = max(-(-max(n, n + m, 1) // page) for n, m in zip(lens, more)) + 1
        ids = list(range(sum(used) + free + 3))
        r.shuffle(ids)
        self.table = [[ids.pop() for _ in range(u)] + [77] * (wide - u) for u in used]
        self.stack = [ids.pop() for _ in range(free)] + [-5] * (sum(used) + slack)

    def run(self, in_place=False, outputs="slots positions owners", call=None, stream=None):
        B = len(self.lens)
        t = dict(table=ints(self.table), lens=ints(self.lens), more=ints(self.more), stack=ints(self.stack), left=ints([self.free]),
                 q_start=ints([9] * (B + 1)))
        t["new_lens"] = t["lens"] if in_place else ints([9] * B)
        t["new_left"] = t["left"] if in_place else ints([9])
        for name, kind in (("slots", torch.int64), ("positions", torch.int32), ("owners", torch.int32)):
            t[name] = torch.full((self.n_tokens,), 9, dtype=kind, device=dev()) if name in outputs else None
        need = tman.tman_kv_plan_workspace_bytes(B, self.n_tokens)
        ws = torch.full((need,), 0xa5, dtype=torch.uint8, device=dev()) if need else None
        tman.tman_kv_plan(t["table"], self.page, t["lens"], t["more"], t["stack"], t["left"], t["new_lens"], t["new_left"], t["q_start"],
                          t["slots"], t["positions"], t["owners"], ws, n_tokens=self.n_tokens, stream=stream)
        return t

    def check(self, **how):
        t = self.run(**how)
        assert tman.tman_device_status() == 0
        want = plain(self.table, self.page, self.lens, self.more, self.stack, self.free, self.n_tokens)
        for name, w in zip(("table", "new_lens", "new_left", "q_start", "slots", "positions", "owners", "stack"), want):
            if t[name] is not None:
                got = t[name].tolist()
                assert got == ([w] if name == "new_left" else w), name
        return t


def changes(seed, B, most, tokens):
    r = random.Random(seed)
    lens = [r.randint(0, most) for _ in range(B)]
    more = [r.choice([0, 1, 1, r.randint(1, tokens), -n, -min(n, r.randint(0, 40))]) for n in lens]
    return lens, more


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("B,most,tokens", [(1, 100, 50), (8, 300, 1), (8, 300, 200), (63, 700, 40), (64, 50, 5), (65, 2000, 300), (1024, 90, 3),
                                           (1025, 90, 4), (3000, 200, 40), (9000, 40, 2)])
@pytest.mark.parametrize("share", [2.0, 0.5, 0.0])
def test_sequences_and_pages(page, B, most, tokens, share):
    """Small calls (one launch) and large ones (two); enough pages, too few, none."""
    lens, more = changes(B + page, B, most, tokens)
    need = sum(max(0, -(-(n + m) // page) + (-n // page)) for n, m in zip(lens, more))
    N = max(1, sum(max(0, m) for m in more))
    Step(B, lens, more, page, int(need * share), N + 5).check()


@pytest.mark.parametrize("n_tokens", [1, 10, 4096, 4097, 6000])
def test_a_bound_on_tokens_refuses_those_behind_it(n_tokens):
    lens, more = [5, 0, 17, 3, 900], [3, 0, 8, 4000, 1100]
    Step(1, lens, more, 16, 1000, n_tokens).check()


@pytest.mark.parametrize("large", [False, True])
def test_in_place_and_without_outputs(large):
    lens, more = changes(7, 40, 300, 4000 if large else 30)
    N = max(1, sum(max(0, m) for m in more))
    Step(2, lens, more, 32, 900 if large else 60, N).check(in_place=True)
    Step(3, lens, more, 32, 900 if large else 60, N).check(in_place=True, outputs="positions")
    Step(3, lens, more, 32, 900 if large else 60, N).check(outputs="none")


def test_pages_that_come_back_are_given_again():
    t = Step(5, [64, 10], [-64, 60], 16, 0, 60).check()
    assert t["new_left"].tolist() == [0] and t["new_lens"].tolist() == [0, 70]


def test_many_steps_keep_every_page_once():
    """A server's life: pages are either free or in one sequence's table, all of them, always."""
    r = random.Random(3)
    B, page, pool, wide = 30, 16, 200, 40
    table, lens, stack, left = ints([[0] * wide] * B), ints([0] * B), ints(list(range(pool))), ints([pool])
    q_start, n = ints([0] * (B + 1)), 400
    slots = torch.empty(n, dtype=torch.int64, device=dev())
    for _ in range(60):
        now = lens.tolist()
        more = [r.choice([1, 1, 1, r.randint(0, 60), -x if r.random() < 0.3 else 0]) for x in now]
        more = [min(m, wide * page - x) for m, x in zip(more, now)]
        tman.tman_kv_plan(table, page, lens, ints(more), stack, left, lens, left, q_start, slots)
        assert tman.tman_device_status() == 0
        held = [p for row, x in zip(table.tolist(), lens.tolist()) for p in row[:-(-x // page)]]
        assert sorted(held + stack.tolist()[:left.item()]) == list(range(pool))
        total = q_start.tolist()[-1]
        assert len(set(slots.tolist()[:total])) == total and set(slots.tolist()[total:]) <= {-1}


@pytest.mark.parametrize("large", [False, True])
def test_what_is_out_of_range_is_cut_and_reported(large):
    N = 5000 if large else 50
    # a length beyond the table, below zero; more goes than is there; a table that is too short; a stack that is full
    s = Step(1, [20, 20, 20], [1, 1, 1], 16, 4, N)
    wide = len(s.table[0])
    for lens, more in (([10 ** 9, 20, 20], [1, 1, 1]), ([-3, 20, 20], [1, 1, 1]), ([20, 20, 20], [-21, 1, 1]), ([20, 20, 20], [2 ** 31 - 1, 1, 1])):
        s.lens, s.more = lens, more
        t = s.run()
        assert tman.tman_device_status() == ERR_INDEX and tman.tman_device_status() == 0
        assert t["q_start"].tolist()[1:] == [t["q_start"].tolist()[1], t["q_start"].tolist()[1] + 1, t["q_start"].tolist()[1] + 2]
        assert all(0 <= n <= wide * 16 for n in t["new_lens"].tolist())
    s = Step(1, [64, 20], [-64, 1], 16, 4, N)
    s.stack = s.stack[:6]
    t = s.run()
    assert tman.tman_device_status() == ERR_INDEX
    assert t["stack"].tolist()[4:6] == s.table[0][:2] and t["new_left"].tolist() == [6]
    s = Step(1, [20], [20], 16, 4, N)
    s.free = 99999
    s.run()
    assert tman.tman_device_status() == ERR_INDEX
