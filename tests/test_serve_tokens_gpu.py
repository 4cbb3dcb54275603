"""The service's own bookkeeping (device), with a step in place of the model's whose tokens are known: next = f(token, position).  Every
sequence has to be fed its own last token whatever slot it moves to, and no request may keep the others from being served."""
import types

import pytest
import torch

from paper_2511_11729_amd import binding as hb
from paper_2511_11729_amd import serve

pytestmark = pytest.mark.gpu
DEV, P = "cuda:0", 16


def follow(token, position):
    return (token * 31 + position * 7 + 11) % 997


class Steps:
    """Stands for a context: remembers which sequences ran and what they were fed."""

    def __init__(self):
        self.server, self.log = None, []

    def decode_step(self, *, batch, kv_len, token_ids, next_token, stream, position=None, **kw):
        with torch.cuda.stream(stream):
            at = kv_len if position is None else position
            next_token[:batch] = follow(token_ids[:batch].long(), at[:batch].long()).int()
        stream.synchronize()
        self.log.append([(seq[2] + seq[3], seq[3], int(token_ids[b])) for b, seq in enumerate(self.server.running)])

    def decode_step_tracked(self, *, track, decay, workspace, **kw):
        self.decode_step(**kw)

    def kv_attend_workspace_bytes(self, batch, max_len):
        return 256

    def kv_record_init(self, **kw):
        pass

    kv_evict = kv_record_init


def service(chunks, max_batch=4, max_len=2000, **kw):
    """A pool of `chunks` times 16 pages, and a server on it."""
    block, row = 64 << 10, 256
    size = chunks * 2 * block
    slab = torch.zeros(size, dtype=torch.uint8, device=DEV)
    pool = hb.Pool(slab, size, block_bytes=block, n_layers=1, kv_row_bytes=row)
    assert pool.stats().n_chunks * pool.stats().pages_per_block == 16 * chunks
    ctx = Steps()
    m = types.SimpleNamespace(vocab=16, hidden=16, n_kv=1)
    ctx.server = serve.DecodeServer(ctx, pool, m, max_batch=max_batch, max_len=max_len, stream=torch.cuda.Stream(), **kw)
    return ctx.server, ctx, pool


def fed(log, total, prompt):
    """What the sequence of `prompt` tokens that ends with `total` of them was fed, step after step."""
    got = [(had, tok) for step in log for key, had, tok in step if key == total]
    assert [had for had, _ in got] == list(range(prompt, prompt + len(got)))      # one token after another, none twice
    return [tok for _, tok in got]


def chain(prompt, n):
    tok, out = 0, []
    for i in range(n):
        out.append(tok)
        tok = follow(tok, prompt + i)
    return out


def test_a_sequence_is_fed_its_own_token_in_whatever_slot_it_is():
    server, ctx, pool = service(8)
    requests = [(20, 3), (37, 30), (11, 13), (64, 9), (5, 21), (90, 2), (33, 1), (7, 14), (50, 5)]
    server.submit(requests)
    while server.step() is not None:
        pass
    assert server.finished == len(requests)
    for prompt, out in requests:
        assert fed(ctx.log, prompt + out, prompt) == chain(prompt, out), (prompt, out)


def test_requests_that_come_later_and_streams_that_change():
    server, ctx, pool = service(8, max_batch=3)
    requests = [(16 + 3 * i, 2 + (5 * i) % 13) for i in range(20)]
    assert len({p + o for p, o in requests}) == 20
    streams = [server.stream, torch.cuda.Stream()]
    left = list(requests)
    for step in range(400):
        if left and step % 3 == 0:
            server.submit([left.pop(0)])
        if step % 5 == 4:
            server.use_stream(streams[step // 5 % 2])
        if server.step() is None and not left:
            break
    assert server.finished == 20
    for prompt, out in requests:
        assert fed(ctx.log, prompt + out, prompt) == chain(prompt, out), (prompt, out)


@pytest.mark.parametrize("budget", [None, serve.KvBudget(keep=48, slack=8, sink=2, recent=12)], ids=["whole", "budget"])
def test_a_sequence_that_was_sent_back_goes_on_from_its_own_token(budget):
    server, ctx, pool = service(8, max_batch=3, budget=budget)
    requests = [(30, 40), (41, 35), (25, 33), (10, 7)]
    server.submit(requests)
    alloc, step = pool.alloc_pages, 0

    def none_left(n):
        if 4 <= step < 30 and (step < 20 or n == 1):               # pages run out, first for prompts too
            raise hb.HarliError(hb.HARLI_ERR_OOM, "none left")
        return alloc(n)
    pool.alloc_pages = none_left
    while step < 300 and (server.queue or server.running):
        server.step()
        step += 1
    assert server.preempted >= 3 and server.finished == 4
    for prompt, out in requests:
        assert fed(ctx.log, prompt + out, prompt) == chain(prompt, out), (prompt, out)


def test_a_prompt_that_the_pool_can_never_hold_does_not_hold_up_the_others():
    server, ctx, pool = service(1)                                 # 16 pages: 256 tokens
    server.submit([(10, 3), (256, 4), (255, 1), (1000, 5), (20, 6)])
    for _ in range(40):
        server.step()
        server.stream.synchronize()                                # (what was freed can be had again)
    assert not server.queue and not server.running
    assert server.finished == 3 and server.refused == 2 and server.admitted == 3
    assert pool.stats().kv_pages_live == 0 or pool.stats().pending_frees > 0


@pytest.mark.parametrize("budget", [None, serve.KvBudget(keep=48, slack=32, sink=2, recent=12)], ids=["whole", "budget"])
def test_a_sequence_that_outgrew_the_pool_and_was_sent_back_does_not_hold_up_the_others(budget):
    server, ctx, pool = service(1, max_batch=2, budget=budget)
    server.submit([(60, 900)])
    for _ in range(200):                                           # 256 tokens and more, inside a budget in at most six pages
        server.step()
    alloc = pool.alloc_pages

    def none_left(n):
        raise hb.HarliError(hb.HARLI_ERR_OOM, "none left")
    pool.alloc_pages = none_left
    for _ in range(40):
        server.step()
    pool.alloc_pages = alloc
    assert server.preempted == 1 and not server.running
    assert server.refused == 1 and not server.queue                # its history is longer than 256 tokens
    server.submit([(20, 6), (30, 4)])
    for _ in range(20):
        server.step()
        server.stream.synchronize()
    assert server.finished == 2


@pytest.mark.parametrize("budget", [dict(keep=32), dict(keep=67), dict(keep=20, sink=4, recent=17), dict(keep=64, sink=0, recent=65),
                                    dict(keep=80, sink=-1), dict(keep=80, recent=-1), dict(keep=80, decay=1.5), dict(keep=80, decay=-0.1),
                                    dict(keep=80, decay=float("nan"))], ids=str)
def test_budgets_that_cannot_keep_what_they_promise_are_refused(budget):
    with pytest.raises(ValueError):
        service(1, budget=serve.KvBudget(**budget))


@pytest.mark.parametrize("keep", [1, 2, 5, 8, 32, 67, 68, 69, 512])
def test_the_protection_of_a_small_budget_fits_it(keep):
    budget = serve.KvBudget.of(keep)
    assert budget.keep == keep and 1 <= budget.recent <= 64 and 0 <= budget.sink <= 4 and budget.sink + budget.recent <= keep
    service(1, budget=budget)
    if keep >= 68:
        assert budget == serve.KvBudget(keep)
