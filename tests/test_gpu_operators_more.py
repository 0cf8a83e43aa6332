"""More of the operators beside the paged attention: calls that fail on the device, rows that one key dominates, tables much wider
than the batch, selections over several pieces.  Bounds as at the head of test_gpu_operators.py unless a test derives its own."""
import numpy as np
import pytest
import torch

from oracle import operators as oo
from paper_2411_09317_b200 import binding as pie
from paper_2411_09317_b200 import synth
from tests.test_gpu_operators import DEV, Pool, check_prompt, down, real, refused, rows, table_for, up

pytestmark = pytest.mark.gpu
F16, BF16 = synth.F16, synth.BF16


# ============================================================================================ weights calls that fail
class WeightsCase:
    """A resident batch with a running account; call() adds one step's weights to it."""

    def __init__(self, p, lens, seed, width=None, spare=7):
        self.p, self.lens, self.S = p, np.array(lens, np.int32), len(lens)
        self.data = p.random(seed)
        p.fill(self.data)
        self.table = table_for(lens, p.blocks, seed, width)
        self.q = rows(seed, self.S, p.hq, p.d, p.dtype)
        self.stride, self.scale = max(lens) + spare, p.d ** -0.5
        self.before = np.random.default_rng(seed).random((self.S, p.hkv, self.stride)).astype(np.float32)
        self.w, self.dq, self.tab = up(self.before), up(self.q), up(self.table)
        self.ctx = up(self.lens)
        self.out = torch.zeros((self.S, p.hq, p.d), dtype=torch.int16, device=DEV)

    def call(self, ctx=None, **kw):
        pie.pie_decode_attention_weights(self.p.h, 0, self.dq.data_ptr(), self.out.data_ptr(), self.tab.data_ptr(), self.table.shape[1],
                                         (self.ctx if ctx is None else ctx).data_ptr(), self.S, self.scale, self.w.data_ptr(), self.stride, **kw)

    def unchanged(self):
        return np.array_equal(self.w.cpu().numpy().view(np.uint32), self.before.view(np.uint32))

    def check(self, steps=1):
        got, kv, p = self.w.cpu().numpy().astype(np.float64), self.p.values(self.data), self.p
        for s, n in enumerate(self.lens):
            ids = self.table[s, :(n + 15) // 16]
            k, v = (kv[ids, :, i].transpose(0, 2, 1, 3).reshape(-1, p.hkv, p.d)[:n] for i in (0, 1))
            added = steps * oo.attention_weights(real(self.q[s], p.dtype), k, self.scale)
            want = self.before[s, :, :n] + added
            assert np.all(np.abs(got[s, :, :n] - want) <= 1.3e-4 * added + 2.0 ** -23 * steps * np.abs(want) + 1e-30), s
            assert np.array_equal(got[s, :, n:], self.before[s, :, n:].astype(np.float64))
            for h in range(p.hq):
                want, _, size = oo.attend(real(self.q[s, h], p.dtype), k[:, h * p.hkv // p.hq], v[:, h * p.hkv // p.hq], self.scale)
                check_prompt(p.dtype, down(self.out[s, h], p.dtype), want, size, (s, h))


@pytest.mark.parametrize("d,dtype,fp8", [(64, F16, False), (128, BF16, False), (128, F16, True)])
@pytest.mark.parametrize("lens", [[40, 50], [700, 30, 333]])
def test_weights_of_a_call_that_misses_a_block_stay_as_they_were(d, dtype, fp8, lens):
    """No host tables: the kernel finds the gap.  Nothing is added to any sum, the next call says why, and once the block is back
    the same call adds every sequence's weights once."""
    with Pool(4, 2, d, dtype, sum((n + 15) // 16 for n in lens), host_slots=64, fp8=fp8) as p:
        c = WeightsCase(p, lens, 800)
        away = [int(c.table[0, 1])]
        pie.pie_swap_out(p.h, 0, away)
        pie.pie_sync(p.h)
        c.call()
        refused(pie.PIE_ERR_NOT_RESIDENT, pie.pie_sync, p.h)
        assert c.unchanged()
        pie.pie_swap_in(p.h, 0, away)
        c.call()
        c.call()
        pie.pie_sync(p.h)
        c.check(steps=2)


@pytest.mark.parametrize("seqs", [3, 1100])
def test_weights_of_a_call_with_a_context_beyond_its_table_stay_as_they_were(seqs):
    """1100 sequences: the plan of a kernel of its own."""
    lens = [1 + (5 * i) % 30 for i in range(seqs)]
    with Pool(2, 1, 64, F16, sum((n + 15) // 16 for n in lens), seqs=seqs) as p:
        c = WeightsCase(p, lens, 810, spare=100)
        bad = c.lens.copy()
        bad[seqs // 2] = 16 * c.table.shape[1] + 1
        bad = up(bad)
        c.call(ctx=bad)
        refused(pie.PIE_ERR_INVALID, pie.pie_sync, p.h)
        assert c.unchanged()
        c.call()
        pie.pie_sync(p.h)
        c.check()
