"""Tracked decode steps against the oracle, and the calls of a budgeted cache together: steps that record weights, sampled tokens,
evictions, and steps that go on from the shorter cache.  Outputs and weights meet the bars of the plain step (tests/test_decode_gpu.py);
what eviction and sampling choose has to be exactly the oracle's choice on what the device held."""
import dataclasses

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import budget_oracle as BO
from oracle import harli_oracle as O
from paper_2511_11729_amd import binding as hb
from paper_2511_11729_amd import serve
from tests.gpu_util import DEV, DecodeCase, assert_close, shapes_of
from tests.test_decode_gpu import F32_BAR
from tests.test_serve_gpu import small

pytestmark = pytest.mark.gpu
P = 16
REC = [("w", np.float32), ("p", np.int32)]


def records_of(case):
    """Empty records for every page of the case's pool, and a workspace for its steps."""
    st = case.pool.stats()
    track = torch.full((case.m.n_layers, st.n_chunks * st.pages_per_block, case.m.n_kv, P, 2), 12345, dtype=torch.int32, device=DEV)
    ws = torch.empty(case.ctx.kv_attend_workspace_bytes(case.B, case.ctx.cfg.max_seq_len), dtype=torch.uint8, device=DEV)
    return track, ws


def host(track):
    return track.cpu().numpy().view(REC)[..., 0]


def where(table, b, n):
    t = np.arange(n)
    return table[b, t // P], t % P


def oracle_step(case, img, x, kv_len, table, position, records, decay):
    """One step of every layer from a slab image and records: (hidden, [layer] weights per sequence)."""
    kv = O.PagedKV(case.geom, case.m.elem_bytes, case.m.n_kv, case.m.head_dim, slab=case._decode_img(img))
    sh, weights = shapes_of(case.m), []
    x = np.asarray(x, np.float64)
    for l, W in enumerate(case.layers_np):
        q, k, v = O._qkv_new_token(x, W, sh, np.asarray(position))
        o, ws = np.empty(q.shape), []
        for b, n in enumerate(kv_len):
            kv.write(table[b], l, int(n), k[b], v[b])
            K, V = kv.gather(table[b], l, int(n) + 1)
            page, slot = where(table, b, int(n) + 1)
            o[b], w, _ = BO.attend_weights(q[b], K, V, records["w"][l, page, :, slot], decay, 0)
            ws.append(w)
        weights.append(ws)
        x = O._post_attention(x, o, W, sh)
    return x, weights


def check_weights(got, want, kv_len, table, position, bar):
    for l, ws in enumerate(want):
        for b, w in enumerate(ws):
            page, slot = where(table, b, int(kv_len[b]) + 1)
            assert_close(got["w"][l, page, :, slot], w, "weights of layer %d, sequence %d" % (l, b), **bar)
            assert np.all(got["p"][l, page[-1], :, slot[-1]] == position[b])


@pytest.mark.parametrize("dtype,heads,batch", [("bf16", (4, 4, 64), 3), ("bf16", (8, 2, 128), 5), ("bf16", (7, 1, 128), 3), ("bf16", (4, 2, 64), 40),
                                               ("f32", (4, 4, 64), 3), ("f32", (6, 2, 48), 4)])
def test_tracked_step_meets_the_oracle_and_appends_where_the_plain_step_does(dtype, heads, batch):
    w = wl.workload(0)
    m = dataclasses.replace(w.model, dtype=dtype, n_layers=2, n_q=heads[0], n_kv=heads[1], head_dim=heads[2])
    lengths = np.asarray([0, 300, 37, 16, 129] * 8, np.int32)[:batch]
    case = DecodeCase(w, m, lengths, block_bytes=256 << 10)
    track, ws = records_of(case)
    case.ctx.kv_record_init(batch=case.B, n_tokens=case.kv_len_dev, page_table=case.table_dev, max_pages=case.max_pages,
                            max_kv_len=int(lengths.max()), track=track)
    position = lengths + np.arange(batch) * 100
    pos_dev = torch.from_numpy(position.astype(np.int32)).to(DEV)
    torch.cuda.synchronize()
    before = host(track)
    y = torch.empty(case.B, m.hidden, device=DEV)
    case.ctx.decode_step_tracked(batch=case.B, kv_len=case.kv_len_dev, page_table=case.table_dev, max_pages=case.max_pages,
                                 max_kv_len=int(lengths.max()) + 1, x_in=case.x_dev, x_out=y, track=track, workspace=ws, position=pos_dev, decay=1.0)
    torch.cuda.synchronize()
    case.ctx.check()
    bar = F32_BAR if dtype == "f32" else {}
    ref, weights = oracle_step(case, case.img0, case.x_np, lengths, case.table, position, before, 1.0)
    assert_close(y.cpu().numpy(), ref, "hidden state", **bar)
    check_weights(host(track), weights, lengths, case.table, position, bar)
    # without positions: the plain step's output (other order of the sums) and its cache
    img = case.slab_image()
    case.slab.copy_(torch.from_numpy(case.img0.view(np.uint8)))
    case.ctx.decode_step_tracked(batch=case.B, kv_len=case.kv_len_dev, page_table=case.table_dev, max_pages=case.max_pages,
                                 max_kv_len=int(lengths.max()) + 1, x_in=case.x_dev, x_out=y, track=track, workspace=ws)
    torch.cuda.synchronize()
    assert_close(y.cpu().numpy(), case.run_oracle(), "hidden state at the cache's own positions", **bar)
    case.check_cache(*((1e-4, 2e-5) if dtype == "f32" else ()))
    assert np.array_equal(np.flatnonzero(img != case.img0), np.flatnonzero(case.slab_image() != case.img0))


def test_tracked_step_is_captured_and_replayed_and_long_uneven_batches_take_the_list_of_chunks():
    """More than 4096 workgroups of attention and 256 MB of traffic: the chunks go out as a list."""
    w = wl.workload(0)
    m = dataclasses.replace(w.model, dtype="bf16", n_layers=1, n_q=32, n_kv=32, head_dim=128, hidden=256, ffn=320)
    lengths = np.asarray([3000] + [40 + 3 * i for i in range(19)], np.int32)
    case = DecodeCase(w, m, lengths)
    assert -(-3001 // 256) * 20 * 32 > 4096 and 20 * 3001 * 32 * 128 * 4 > 256 << 20
    track, ws = records_of(case)
    case.ctx.kv_record_init(batch=case.B, n_tokens=case.kv_len_dev, page_table=case.table_dev, max_pages=case.max_pages, max_kv_len=3000, track=track)
    torch.cuda.synchronize()
    start = track.clone()
    y, y_g = torch.empty(case.B, m.hidden, device=DEV), torch.empty(case.B, m.hidden, device=DEV)
    args = dict(batch=case.B, kv_len=case.kv_len_dev, page_table=case.table_dev, max_pages=case.max_pages, max_kv_len=3001, x_in=case.x_dev, track=track,
                workspace=ws, decay=0.5)
    case.ctx.decode_step_tracked(x_out=y, **args)
    torch.cuda.synchronize()
    case.ctx.check()
    ref, weights = oracle_step(case, case.img0, case.x_np, lengths, case.table, lengths, host(start), 0.5)
    assert_close(y.cpu().numpy(), ref, "hidden state")
    check_weights(host(track), weights, lengths, case.table, lengths, {})
    want = track.clone()
    st = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        case.ctx.decode_step_tracked(x_out=y_g, stream=st, **args)
    for _ in range(3):
        track.copy_(start)
        case.slab.copy_(torch.from_numpy(case.img0.view(np.uint8)))
        y_g.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y_g) and torch.equal(track, want)
    del g


def test_steps_samples_and_evictions_together():
    """Three sequences over 28 steps with a budget of 32 tokens: every call is checked against the oracle on what the device held
    before it."""
    w = wl.workload(0)
    m = dataclasses.replace(w.model, dtype="bf16", n_layers=2, n_q=4, n_kv=2, vocab=512)
    prompts = np.asarray([40, 9, 33], np.int32)
    case = DecodeCase(w, m, prompts, full_model=True, block_bytes=64 << 10, extra_chunks=4)
    B, steps, keep, slack, sink, recent = 3, 28, 32, 4, 2, 6
    table = np.full((B, 8), -1, np.int32)
    fresh = iter(case.pool.alloc_pages(B * 8))
    for b in range(B):
        held = [int(i) for i in case.table[b] if i >= 0]
        table[b] = (held + [next(fresh) for _ in range(8)])[:8]
    track, _ = records_of(case)
    ctx = hb.Context(case.pool, n_layers=2, hidden=m.hidden, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn=m.ffn, rms_eps=m.rms_eps, rope_base=m.rope_base,
                     max_batch=B, max_seq_len=128, layers=case.layers_dev, emb=case.emb_dev, g_final=case.gf_dev, w_lm=case.wlm_dev, vocab=m.vocab)
    ws = torch.empty(ctx.kv_attend_workspace_bytes(B, 128), dtype=torch.uint8, device=DEV)
    sws = torch.empty(hb.sample_workspace_bytes(B, m.vocab), dtype=torch.uint8, device=DEV)
    i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).to(DEV)  # noqa: E731
    pages = dict(batch=B, page_table=i32(table), max_pages=8, max_kv_len=128, track=track)
    ctx.kv_record_init(n_tokens=i32(prompts), **pages)
    n, position, evicted = prompts.copy(), prompts.copy(), 0
    tok = wl.make_token_ids(dataclasses.replace(w, model=m), (B,))
    logits, hidden = torch.empty(B, m.vocab, device=DEV), torch.empty(B, m.hidden, device=DEV)
    token, r = torch.empty(B, dtype=torch.int32, device=DEV), np.random.default_rng(0)
    settings = dict(temperature=np.array([0.9, 1.2, 0.0], np.float32), top_k=np.array([0, 40, 5], np.int32), top_p=np.array([0.9, 1.0, 1.0], np.float32))
    for step in range(steps):
        img, before = case.slab_image(), host(track)
        ctx.decode_step_tracked(kv_len=i32(n), position=i32(position), token_ids=i32(tok), logits=logits, x_out=hidden, workspace=ws, decay=0.9, **pages)
        u = r.random(B).astype(np.float32)
        hb.sample(logits, torch.from_numpy(u).to(DEV), token, workspace=sws, **{k: torch.from_numpy(v).to(DEV) for k, v in settings.items()})
        torch.cuda.synchronize()
        ctx.check()
        x = np.asarray(case.extras_np["emb"], np.float64)[tok]
        ref, weights = oracle_step(case, img, x, n, table, position, before, 0.9)
        assert_close(hidden.cpu().numpy(), ref, "hidden state of step %d" % step)
        check_weights(host(track), weights, n, table, position, {})
        z = logits.cpu().numpy()
        assert_close(z, O.rmsnorm(ref, case.extras_np["gf"], m.rms_eps) @ np.asarray(case.extras_np["wlm"], np.float64).T, "logits of step %d" % step)
        tok = token.cpu().numpy()
        assert tok.tolist() == [BO.sample_token(z[b], float(u[b]), **{k: v[b].item() for k, v in settings.items()})[0] for b in range(B)]
        n, position = n + 1, position + 1
        if np.any(n >= keep + slack):
            img, before = case.slab_image(), host(track)
            want_img, want = img.copy(), before.copy()
            to = np.where(n >= keep + slack, keep, n)
            for b in range(B):
                page, slot = where(table, b, int(n[b]))
                for l in range(2):
                    for c in range(2):
                        rec = before[l, page, c, slot]
                        for a, t in BO.evict_moves(rec["w"], rec["p"], to[b], position[b], sink, recent):
                            want[l, page[t], c, slot[t]] = rec[a]
                            for kv in (0, 1):
                                src, dst = (case.geom.head_offset(int(page[i]), l, kv, c, int(slot[i]), 128) // 2 for i in (a, t))
                                want_img[dst: dst + 64] = img[src: src + 64]
                            evicted += 1
            left = torch.empty(B, dtype=torch.int32, device=DEV)
            ctx.kv_evict(n_tokens=i32(n), keep=i32(to), position=i32(position), sink=sink, recent=recent, n_left=left, **pages)
            torch.cuda.synchronize()
            ctx.check()
            assert np.array_equal(case.slab_image(), want_img) and host(track).tobytes() == want.tobytes()
            assert left.tolist() == to.tolist()
            n = to.astype(np.int32)
    assert evicted > 50 and n.max() < keep + slack


def test_refusals_of_a_tracked_step():
    w = wl.workload(0)
    m = dataclasses.replace(w.model, dtype="bf16")
    case = DecodeCase(w, m, np.asarray([20, 5], np.int32), block_bytes=64 << 10)
    track, ws = records_of(case)
    good = dict(batch=2, kv_len=case.kv_len_dev, page_table=case.table_dev, max_pages=case.max_pages, max_kv_len=21, x_in=case.x_dev, track=track, workspace=ws)
    for kw in (dict(track=None), dict(track=track.data_ptr() + 8), dict(workspace=None), dict(workspace=ws[64:]), dict(workspace=ws[:256]), dict(decay=1.1),
               dict(decay=float("nan")), dict(batch=0), dict(max_kv_len=0), dict(kv_len=None), dict(x_in=None)):
        with pytest.raises(hb.HarliError) as e:
            case.ctx.decode_step_tracked(**dict(good, **kw))
        assert e.value.status == hb.HARLI_ERR_INVALID, kw
    torch.cuda.synchronize()
    case.ctx.check()
    assert np.array_equal(case.slab_image(), case.img0) and bool((track == 12345).all())


# --------------------------------------------------------------------------------------------- the service
def serving(sampling=None, budget=None, steps=300):
    args, w, m, ft, pool, ctx, ft_step, sizes, keep = small()
    sD = torch.cuda.Stream()
    server = serve.DecodeServer(ctx, pool, m, max_batch=args.max_batch, max_len=args.max_len, stream=sD, slab=keep[0], sampling=sampling, budget=budget)
    arrivals = wl.make_arrivals(w, steps, targets=(2, 6, 12, 4), mean_out=40, prompt=("uniform", 5, 120))
    seen, most, kv_pages = [], 0, 0
    for reqs in arrivals:
        server.submit(reqs)
        r = server.step()
        if r is not None:
            r[0].synchronize()
            seen.append(server.tok[: r[1]].cpu())
            most = max([most] + [s[1] for s in server.running])
            kv_pages = max(kv_pages, pool.stats().kv_pages_live)
            for b, s in enumerate(server.running):            # the table names just the pages a sequence holds, enough for its next token
                assert server.table[b, : len(s[0])].tolist() == s[0] and np.all(server.table[b, len(s[0]):] == -1)
                assert s[1] < len(s[0]) * P and server.kv[b] == s[1]
    torch.cuda.synchronize()
    ctx.check(sD)
    server.drain()
    pool.alloc_pages(0)
    assert pool.stats().kv_pages_live == 0
    return server, seen, most, kv_pages


def same(a, b):
    return len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


def test_service_with_sampled_tokens():
    argmax = serving()[1]
    assert same(argmax, serving(serve.Sampling(temperature=0.0))[1]) and same(argmax, serving(serve.Sampling(top_k=1))[1])
    drawn = serving(serve.Sampling(temperature=1.0, top_p=0.95, seed=3))[1]
    assert same(drawn, serving(serve.Sampling(temperature=1.0, top_p=0.95, seed=3))[1])
    assert not same(drawn, argmax) and not same(drawn, serving(serve.Sampling(temperature=1.0, top_p=0.95, seed=4))[1])
    assert all(bool(((0 <= t) & (t < 512)).all()) for t in drawn)


def test_service_inside_a_budget_gives_pages_back():
    budget = serve.KvBudget(keep=48, slack=8, sink=2, recent=12)
    server, seen, most, pages = serving(budget=budget)
    free, _, longest, free_pages = serving()
    assert server.finished == free.finished and len(seen) > 200       # the same service
    assert server.evicted > 100 and free.evicted == 0
    assert pages < free_pages
    # a prompt may arrive longer than the budget; after its first step it is cut
    assert most < 48 + 8 and longest > 100
    for s in (dict(keep=0), dict(keep=5, slack=0)):
        with pytest.raises(ValueError):
            serving(budget=serve.KvBudget(**s))


def test_a_sequence_that_is_sent_back_returns_with_all_tokens_it_has_had():
    args, w, m, ft, pool, ctx, ft_step, sizes, keep = small()
    server = serve.DecodeServer(ctx, pool, m, max_batch=2, max_len=args.max_len, stream=torch.cuda.Stream(), slab=keep[0],
                                budget=serve.KvBudget(keep=40, slack=16, sink=2, recent=8))
    server.submit([(60, 40)])
    server.step()[0].synchronize()
    assert server.running[0][1:4] == [40, 39, 61] and server.evicted == 21     # cached, left, had
    alloc = pool.alloc_pages

    def none_left(n):
        raise hb.HarliError(hb.HARLI_ERR_OOM, "none left")
    pool.alloc_pages = none_left                       # the page for a 49th token
    for _ in range(8):
        server.step()[0].synchronize()
    assert server.preempted == 1 and not server.running and list(server.queue) == [(69, 31)]
    pool.alloc_pages = alloc
    server.step()[0].synchronize()
    assert server.running[0][1:4] == [40, 30, 70]      # its next token has position 69
    ctx.check(server.stream)
    server.drain()


def test_a_budget_for_longer_sequences_than_an_eviction_takes_is_refused():
    args, w, m, ft, pool, ctx, ft_step, sizes, keep = small()
    with pytest.raises(ValueError):
        serve.DecodeServer(ctx, pool, m, max_batch=1, max_len=(1 << 18) + 1, stream=torch.cuda.Stream(), budget=serve.KvBudget(keep=40))


@pytest.mark.parametrize("heads,batch", [((28, 4, 128), 48), ((5, 1, 128), 190)], ids=str)
def test_uneven_batches_of_groups_on_the_matrix_units_take_the_list_of_chunks(heads, batch):
    w = wl.workload(0)
    m = dataclasses.replace(w.model, dtype="bf16", n_layers=1, n_q=heads[0], n_kv=heads[1], head_dim=heads[2], hidden=256, ffn=320)
    lengths = np.asarray([3000] + [1 + 3 * (i % 60) for i in range(batch - 1)], np.int32)
    case = DecodeCase(w, m, lengths)
    assert -(-3001 // 128) * batch * m.n_kv > 4096 and batch * 3001 * m.n_kv * 128 * 4 > 256 << 20
    track, ws = records_of(case)
    case.ctx.kv_record_init(batch=case.B, n_tokens=case.kv_len_dev, page_table=case.table_dev, max_pages=case.max_pages, max_kv_len=3000, track=track)
    torch.cuda.synchronize()
    before = host(track)
    y = torch.empty(case.B, m.hidden, device=DEV)
    case.ctx.decode_step_tracked(batch=case.B, kv_len=case.kv_len_dev, page_table=case.table_dev, max_pages=case.max_pages, max_kv_len=3001,
                                 x_in=case.x_dev, x_out=y, track=track, workspace=ws)
    torch.cuda.synchronize()
    case.ctx.check()
    ref, weights = oracle_step(case, case.img0, case.x_np, lengths, case.table, lengths, before, 1.0)
    assert_close(y.cpu().numpy(), ref, "hidden state")
    check_weights(host(track), weights, lengths, case.table, lengths, {})
