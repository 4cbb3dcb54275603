"""Decode steps on caches with keys that score -inf: zeros of the softmax, also where a wave or a whole chunk has nothing else."""
import dataclasses

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import harli_oracle as O
from tests.gpu_util import DecodeCase, assert_close, shapes_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(4, 4, 64), (2, 2, 128), (8, 2, 128), (7, 1, 128)], ids=str)
def test_keys_of_minus_infinity(heads):
    w = wl.workload(0)
    m = dataclasses.replace(w.model, dtype="bf16", n_layers=1, n_q=heads[0], n_kv=heads[1], head_dim=heads[2])
    lengths = np.asarray([300, 300, 40, 2900, 129], np.int32)
    group, d = m.n_q // m.n_kv, m.head_dim

    def alike(case):
        # one rotary pair of the query is the same in all heads of a group: there is an element that all of them have with one sign
        wq = case.layers_np[0]["wq"].reshape(m.n_kv, group, d, m.hidden)
        wq[:, :, [0, d // 2]] = wq[:, :1, [0, d // 2]]
        case.layers_np[0]["wq"] = wq.reshape(m.n_q * d, m.hidden)
    case = DecodeCase(w, m, lengths, block_bytes=256 << 10, tweak=alike)
    q = O._qkv_new_token(case.x_np, case.layers_np[0], shapes_of(m), lengths)[0]
    masked = ((0, 64, 128), (1, 0, 256), (2, 0, 39), (3, 0, 2304), (4, 1, 128))
    for b, lo, hi in masked:
        for c in range(m.n_kv):
            mine = q[b, c * group: (c + 1) * group]
            same = np.abs(mine).min(0) * (np.abs(np.sign(mine).sum(0)) == group)
            e = int(same.argmax())
            assert same[e] > 1e-3
            bits = 0xff80 if mine[0, e] > 0 else 0x7f80
            for t in range(lo, hi):
                case.img0[case.geom.head_offset(int(case.table[b, t // 16]), 0, 0, c, t % 16, 2 * d) // 2 + e] = bits
    case.slab.copy_(torch.from_numpy(case.img0.view(np.uint8)))
    got = case.run_gpu()
    with np.errstate(invalid="ignore"):
        want = case.run_oracle()
    assert np.isfinite(want).all()
    assert_close(got, want, "hidden state")
