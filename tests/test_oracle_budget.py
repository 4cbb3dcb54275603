"""The oracle of the budgeted cache and of sampling against brute force and against properties of the definitions; and what the entry
points refuse before anything touches a device (CPU only)."""
import ctypes
import itertools
import math

import numpy as np
import pytest

from oracle import budget_oracle as O
from paper_2511_11729_amd import binding as hb


def test_weights_of_one_step_add_up_to_the_query_heads_and_outputs_stay_inside_the_values():
    r = np.random.default_rng(1)
    q, K, V = r.normal(size=(6, 8)), r.normal(size=(11, 2, 8)), r.normal(size=(11, 2, 8))
    out, w, P = O.attend_weights(q, K, V, r.random((11, 2)), 0.0, 11)
    assert np.allclose(w.sum(0), 3.0) and np.allclose(P.sum(1), 1.0)
    assert np.all(out <= V.max(0).repeat(3, 0) + 1e-12) and np.all(out >= V.min(0).repeat(3, 0) - 1e-12)
    two = O.attend_weights(q, K, V, w, 0.5, 11)[1]
    assert np.allclose(two[:-1], 1.5 * w[:-1]) and np.allclose(two[-1], w[-1])       # the newest token's record begins anew


@pytest.mark.parametrize("keep,sink,recent", [(0, 0, 0), (1, 0, 0), (3, 1, 1), (4, 2, 3), (5, 0, 2), (7, 0, 0)])
def test_eviction_keeps_the_best_set_and_moves_as_little_as_any_choice_of_places(keep, sink, recent):
    r = np.random.default_rng(keep)
    for _ in range(20):
        n = 7
        weight, position = r.integers(0, 4, n) / 2.0, r.permutation(9)[:n]
        moves = O.evict_moves(weight, position, keep, 9, sink, recent)
        slots = list(range(n))
        for a, b in moves:
            assert a >= keep > b
            slots[b] = a
        guarded = {t for t in range(n) if position[t] < sink or position[t] >= 9 - recent}
        key = lambda t: (t in guarded, 0.0 if t in guarded else weight[t], -t)  # noqa: E731
        best = max(itertools.combinations(range(n), min(keep, n)), key=lambda s: sorted(map(key, s), reverse=True)) if keep else ()
        assert set(slots[:keep]) == set(best)
        assert len(moves) == sum(t >= keep for t in best)


def test_filters_keep_prefixes_and_the_draw_inverts_the_distribution():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.25, 0.05]))
    assert O.sample_kept(z)[0] == [1, 3, 2, 0, 4]
    assert O.sample_kept(z, top_k=2)[0] == [1, 3]
    assert O.sample_kept(z, top_p=0.66)[0] == [1, 3, 2]
    assert O.sample_kept(z, top_p=0.66, top_k=3)[0] == [1, 3]                         # of 0.85: 0.561 is reached with two
    assert O.sample_kept(z, min_p=0.5)[0] == [1, 3, 2]
    assert O.sample_kept(z, temperature=0.0)[0] == [1]
    assert O.sample_kept([3.0, 3.0, 1.0, 3.0], top_k=2)[0] == [0, 1]                  # equal ones by index
    got = [O.sample_token(z, u)[0] for u in (0.0, 0.0999, 0.1001, 0.4999, 0.5001, 0.6999, 0.9499, 0.9501, 0.999999)]
    assert got == [0, 0, 1, 1, 2, 2, 3, 4, 4]
    assert O.sample_token([-math.inf, math.nan], 0.5) == (-1, -math.inf)
    assert O.sample_token([1.0, math.inf, math.inf], 0.7) == (2, math.log(0.5))


def refused(word, fn, *a):
    assert fn(*a) == hb.HARLI_ERR_INVALID
    assert word in hb.lib().harli_last_error().decode()


def test_sample_refuses_bad_arguments_on_the_host():
    l = hb.lib()
    good = dict(batch=2, vocab=100, logits=4096, ld=100, uniform=4096, token=4096, workspace=4096, workspace_bytes=hb.sample_workspace_bytes(2, 100))

    def call(**kw):
        return ctypes.byref(hb.SampleBatch(**dict(good, **kw))), None

    refused("null", l.harli_sample, None, None)
    for n in (0, 65536):
        refused("batch", l.harli_sample, *call(batch=n))
    for v in (0, -1, (1 << 20) + 1):
        refused("vocabulary", l.harli_sample, *call(vocab=v))
        assert hb.sample_workspace_bytes(2, v) == 0
    for name in ("logits", "uniform", "token"):
        refused("required", l.harli_sample, *call(**{name: None}))
    refused("apart", l.harli_sample, *call(ld=99))
    refused("workspace", l.harli_sample, *call(workspace=None))
    refused("workspace", l.harli_sample, *call(workspace=4096 + 64))
    refused("workspace", l.harli_sample, *call(workspace_bytes=good["workspace_bytes"] - 1))
    assert hb.sample_workspace_bytes(0, 100) == 0


def test_cache_calls_refuse_a_null_context():
    l = hb.lib()
    for name, cls in (("harli_kv_attend", hb.AttendBatch), ("harli_kv_evict", hb.EvictBatch), ("harli_kv_record_init", hb.RecordBatch)):
        refused("null", getattr(l, name), None, ctypes.byref(cls()), None)
    refused("null", l.harli_decode_step_tracked, None, None, None, None)
    assert l.harli_kv_attend_workspace_bytes(None, 1, 1) == 0


def test_logits_that_are_not_rows_of_fp32_are_refused():
    torch = pytest.importorskip("torch")
    z = torch.zeros(4, 6)
    for bad in (z.t(), z[:, ::2], z.double(), z[0], z[None]):
        with pytest.raises(ValueError):
            hb.sample(bad, z, z, workspace=z)
