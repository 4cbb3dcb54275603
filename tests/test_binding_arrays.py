"""What the binding refuses before a call takes an array for something it is not (CPU only): device code would read a wrong type's halves, or
past the end, or the host's memory.  Tensors of the host stand for the device's here, and the library is not called."""
import ctypes

import pytest

from paper_2511_11729_amd import binding as hb

torch = pytest.importorskip("torch")
CALLS = ("harli_sample", "harli_kv_attend", "harli_kv_record_init", "harli_kv_evict", "harli_decode_step_tracked")


@pytest.fixture
def host(monkeypatch):
    """Lets the host's tensors pass for the device's; the list of what the library would have been given."""
    seen = []
    monkeypatch.setattr(hb, "_INT", torch.IntTensor)
    monkeypatch.setattr(hb, "_FLOAT", torch.FloatTensor)
    monkeypatch.setattr(hb, "_workspace", lambda who, t: (t.data_ptr(), t.nbytes))
    for name in CALLS:
        monkeypatch.setattr(hb.lib(), name, lambda *a: seen.append(a) or 0)
    return seen


def arrays(B=4, V=6):
    f, i = torch.zeros(B), torch.zeros(B, dtype=torch.int32)
    return dict(logits=torch.zeros(B, V), uniform=f, token=i, workspace=torch.zeros(4096, dtype=torch.uint8), temperature=f.clone(), top_k=i.clone(),
                top_p=f.clone(), min_p=f.clone(), logprob=f.clone())


SAMPLE = ("uniform", "token", "temperature", "top_k", "top_p", "min_p", "logprob")


@pytest.mark.parametrize("name", SAMPLE)
def test_sample_refuses_arrays_of_other_types_lengths_and_steps(name, host):
    good = arrays()[name]
    other = torch.float32 if good.dtype == torch.int32 else torch.int32
    for bad in (good.long(), good.double(), good.to(other), good.half(), good[:3], torch.zeros(8, dtype=good.dtype)[::2], torch.zeros(0, dtype=good.dtype),
                torch.zeros(1, dtype=good.dtype).expand(4)):
        with pytest.raises(ValueError, match=name) as e:
            hb.sample(**dict(arrays(), **{name: bad}))
        assert isinstance(e.value, hb.HarliError) and e.value.status == hb.HARLI_ERR_INVALID
    assert not host
    hb.sample(**arrays())
    hb.sample(**dict(arrays(), **{name: torch.zeros(9, dtype=good.dtype)}))
    assert len(host) == 2


def test_arrays_of_the_host_are_refused(monkeypatch):
    reached = []
    for name in CALLS:
        monkeypatch.setattr(hb.lib(), name, lambda *a: reached.append(a) or 0)
    with pytest.raises(ValueError, match="device"):
        hb.sample(**arrays())
    for name, kw in calls().items():
        with pytest.raises(hb.HarliError, match="device"):
            getattr(context(), name)(**kw)
    assert not reached


def test_a_workspace_that_is_smaller_than_it_says_is_refused():
    for t in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(4096, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="workspace"):
            hb._workspace("sample", t)


def test_one_row_of_logits_may_have_any_distance_to_the_next(host):
    one = arrays(B=1)
    for logits in (torch.zeros(6, 1).t(), torch.zeros(1, 1, 6)[:, 0], torch.zeros(6).expand(1, 6)):
        hb.sample(**dict(one, logits=logits))
    assert [hb.SampleBatch.from_buffer_copy(b).ld >= 6 for b, _ in host] == [True] * 3


# ---- the calls of a budgeted cache
B, PAGES, L, N_Q, N_KV, D = 3, 5, 2, 4, 2, 8


def context():
    ctx = object.__new__(hb.Context)
    ctx.handle = ctypes.c_void_p()
    ctx.cfg = hb.ModelCfg(L, 16, N_Q, N_KV, D, 16, 0, 1e-6, 1e4, hb.HARLI_BF16, B, 64, 0, 0)
    ctx.record_bytes, ctx.row_values = 8 * L * 20 * N_KV * 16, N_Q * D
    return ctx


def calls():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    table = dict(batch=B, page_table=i(B, PAGES), max_pages=PAGES, max_kv_len=40, track=i(L, 20, N_KV, 16, 2))
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    return {"kv_attend": dict(table, layer=0, q=torch.zeros(B, N_Q, D), out=torch.zeros(B, N_Q, D), n_tokens=i(B), position=i(B), workspace=ws),
            "kv_record_init": dict(table, n_tokens=i(B)),
            "kv_evict": dict(table, n_tokens=i(B), keep=i(B), position=i(B), n_left=i(B)),
            "decode_step_tracked": dict(table, kv_len=i(B), position=i(B), workspace=ws, x_in=torch.zeros(B, 16), x_out=torch.zeros(B, 16))}


@pytest.mark.parametrize("call,name", [(c, n) for c, a in calls().items() for n, t in a.items()
                                       if torch.is_tensor(t) and n not in ("workspace", "x_in", "x_out")])
def test_cache_calls_refuse_arrays_of_other_types_lengths_and_steps(call, name, host):
    good = calls()[call][name]
    wide = torch.zeros(good.shape[:-1] + (2 * good.shape[-1],), dtype=good.dtype)[..., ::2]
    for bad in (good.long(), good.double(), good.half(), good.flatten()[:-1], wide):
        with pytest.raises(hb.HarliError, match=name) as e:
            getattr(context(), call)(**dict(calls()[call], **{name: bad}))
        assert e.value.status == hb.HARLI_ERR_INVALID
    assert not host


def test_what_the_library_is_given_is_what_the_structs_hold(host):
    for name, kw in calls().items():
        getattr(context(), name)(**kw)
    attend, record, evict, step = (a[1] for a in host)
    kw = calls()["kv_attend"]
    want = hb.AttendBatch(B, 1, 16, 32, 48, 64, PAGES, 40, hb.Tracking(80, 0.5, 96, 112, 128))
    assert hb._pack_attend(B, 1, 16, 32, 48, 64, PAGES, 40, 80, 0.5, 96, 112, 128) == bytes(want)
    a = hb.AttendBatch.from_buffer_copy(attend)
    assert (a.batch, a.layer, a.max_pages, a.max_kv_len, a.track.decay) == (B, 0, PAGES, 40, 1.0) and a.track.workspace_bytes == kw["workspace"].nbytes
    assert all((a.q, a.out, a.n_tokens, a.page_table, a.track.records, a.track.position))
    r, e = hb.RecordBatch.from_buffer_copy(record), hb.EvictBatch.from_buffer_copy(evict)
    assert (r.batch, r.max_pages, r.max_kv_len, e.batch, e.max_pages, e.max_kv_len, e.sink, e.recent) == (B, PAGES, 40, B, PAGES, 40, 0, 0)
    assert all((r.n_tokens, r.page_table, r.records, e.n_tokens, e.keep, e.position, e.page_table, e.records, e.n_left))
    s, t = hb.DecodeBatch.from_buffer_copy(step), hb.Tracking.from_buffer_copy(host[3][2])
    assert (s.batch, s.max_pages, s.max_kv_len) == (B, PAGES, 40) and s.x_in and s.x_out and not s.token_ids and not s.logits and not s.next_token
    assert s.kv_len and s.page_table and t.records and t.position and t.workspace and t.workspace_bytes == kw["workspace"].nbytes


def test_records_may_be_words_of_either_type(host):
    track = calls()["kv_evict"]["track"].float()
    context().kv_evict(**dict(calls()["kv_evict"], track=track))
    assert hb.EvictBatch.from_buffer_copy(host[0][1]).records == track.data_ptr()
    with pytest.raises(hb.HarliError, match="track"):
        context().kv_evict(**dict(calls()["kv_evict"], track=track.flatten()[1:]))
