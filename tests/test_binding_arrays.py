"""What the binding refuses before a call takes an array for something it is not (CPU only): device code would read a wrong type's halves, or
past the end."""
import ctypes

import pytest

from paper_2511_11729_amd import binding as hb

torch = pytest.importorskip("torch")


def arrays(B=4, V=6):
    f, i = torch.zeros(B), torch.zeros(B, dtype=torch.int32)
    return dict(logits=torch.zeros(B, V), uniform=f, token=i, workspace=torch.zeros(4096, dtype=torch.uint8), temperature=f.clone(), top_k=i.clone(),
                top_p=f.clone(), min_p=f.clone(), logprob=f.clone())


SAMPLE = ("uniform", "token", "temperature", "top_k", "top_p", "min_p", "logprob")


@pytest.mark.parametrize("name", SAMPLE)
def test_sample_refuses_arrays_of_other_types_lengths_and_steps(name):
    good = arrays()[name]
    other = torch.float32 if good.dtype == torch.int32 else torch.int32
    for bad in (good.long(), good.double(), good.to(other), good.half(), good[:3], torch.zeros(8, dtype=good.dtype)[::2], torch.zeros(0, dtype=good.dtype),
                torch.zeros(1, dtype=good.dtype).expand(4)):
        with pytest.raises(ValueError, match=name) as e:
            hb.sample(**dict(arrays(), **{name: bad}))
        assert isinstance(e.value, hb.HarliError) and e.value.status == hb.HARLI_ERR_INVALID


def test_sample_refuses_arrays_that_are_not_on_the_device():
    with pytest.raises(ValueError, match="device"):
        hb.sample(**arrays())


def test_sample_refuses_a_workspace_that_is_smaller_than_it_says(monkeypatch):
    monkeypatch.setattr(hb, "_on_device", lambda *a: None)
    with pytest.raises(ValueError, match="workspace"):
        hb.sample(**dict(arrays(), workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 20)))


def test_one_row_of_logits_may_have_any_distance_to_the_next(monkeypatch):
    seen = []
    monkeypatch.setattr(hb, "_on_device", lambda *a: None)
    monkeypatch.setattr(hb.lib(), "harli_sample", lambda b, st: seen.append(b._obj.ld) or 0)
    one = arrays(B=1)
    for logits in (torch.zeros(6, 1).t(), torch.zeros(1, 1, 6)[:, 0], torch.zeros(6).expand(1, 6)):
        hb.sample(**dict(one, logits=logits))
    assert all(ld >= 6 for ld in seen) and len(seen) == 3
