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
            if n == 0:
                assert not down(self.out[s], p.dtype).any() and np.array_equal(got[s], self.before[s].astype(np.float64))
                continue
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


@pytest.mark.parametrize("d,dtype", [(64, F16), (128, BF16)])
def test_weights_keep_what_a_decayed_account_holds(d, dtype):
    """Sums that have decayed to subnormal numbers, of tokens whose probability is below 2^-126 (a key 200 nats above them): 0 is added
    and every bit stays, by which an eviction still tells them apart."""
    n, hq, hkv = 70, 4, 2
    with Pool(hq, hkv, d, dtype, (n + 15) // 16, seqs=1) as p:
        q, k, v, scale = sink_rows(930, n, hq, hkv, d, dtype, 200.0, 20)
        kv = np.zeros((p.blocks * 16, hkv, 2, d), np.uint16)
        kv[:n, :, 0], kv[:n, :, 1] = k, v
        p.fill(np.ascontiguousarray(kv.reshape(p.blocks, 16, hkv, 2, d).transpose(0, 2, 3, 1, 4)))
        before = (np.arange(hkv * n).reshape(1, hkv, n) * 2.0 ** -149).astype(np.float32)
        tab, ctx, dq, w = up(np.arange(p.blocks, dtype=np.int32)[None]), up(np.array([n], np.int32)), up(q[:1]), up(before)
        out = torch.zeros_like(dq)
        pie.pie_decode_attention_weights(p.h, 0, dq.data_ptr(), out.data_ptr(), tab.data_ptr(), p.blocks, ctx.data_ptr(), 1, scale, w.data_ptr(), n)
        pie.pie_sync(p.h)
    got, others = w.cpu().numpy(), np.arange(n) != 20
    assert np.array_equal(got[:, :, others].view(np.uint32), before[:, :, others].view(np.uint32))
    assert np.all(np.abs(got[:, :, 20] - hq / hkv) <= 1.3e-4 * hq / hkv)


# ================================================================================== rows that one key dominates (fp16 range)
def sink_rows(seed, n, hq, hkv, d, dtype, nats, at):
    """q, k, v bits and the scale: the key at `at` lies `nats` (give or take a half) above all others, and its value is 0."""
    rng = np.random.default_rng(seed)
    q, k = np.zeros((n, hq, d)), np.zeros((n, hkv, d))
    q[:, :, 0] = 8.0
    k[:, :, 0] = rng.uniform(-1.0, 1.0, (n, hkv))
    k[at, :, 0] = 2.0 * nats
    k[:, :, 1:] = rng.standard_normal((n, hkv, d - 1))
    bits = lambda x: synth.f32_to_16_bits(x.astype(np.float32), dtype)  # noqa: E731
    v = np.abs(rng.standard_normal((n, hkv, d)))
    v[at] = 0.0
    return bits(q), bits(k), bits(v), 1.0 / 16


def sink_bound(dtype, want, size, weights, v, below):
    """As check_prompt, and for P in fp16 what a probability may lose below the type's smallest step: `below` of the largest."""
    u, tiny = (2.0 ** -11, 2.0 ** -25) if dtype == F16 else (2.0 ** -8, 2.0 ** -134)
    return (u + 4e-4) * size + u * np.abs(want) + tiny + below * weights.max() * np.abs(v).sum(axis=0)


@pytest.mark.parametrize("d,dtype", [(128, F16), (64, F16), (128, BF16)])
@pytest.mark.parametrize("nats,at", [(5.5, 200), (12.0, 0), (14.0, 0), (16.0, 0), (16.0, 131), (17.4, 0), (18.5, 0), (17.4, 4000)])
def test_prompt_rows_that_one_key_dominates(d, dtype, nats, at):
    """Thousands of keys far below one whose value is 0: what they add up to is the whole output."""
    n, hq, hkv = 4001, 4, 2
    q, k, v, scale = sink_rows(900, n, hq, hkv, d, dtype, nats, at)
    dq, dk, dv = up(q), up(k), up(v)
    out = torch.zeros_like(dq)
    with Pool(hq, hkv, d, dtype, 1) as p:
        pie.pie_prompt_attention(p.h, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), out.data_ptr(), np.array([0, n], np.int32), 1, scale)
        pie.pie_sync(p.h)
    q, k, v, got = real(q, dtype), real(k, dtype), real(v, dtype), down(out, dtype)
    for i in [0, 1, at, 127, 128, 300, 1000, 2047, 3000, n - 1]:
        for h in range(hq):
            want, w, size = oo.attend(q[i, h], k[:i + 1, h // 2], v[:i + 1, h // 2], scale)
            bound = sink_bound(dtype, want, size, w, v[:i + 1, h // 2], 2.0 ** -32 if dtype == F16 else 0.0)
            err = np.abs(got[i, h] - want)
            assert np.all(err <= bound), (i, h, float((err / bound).max()))


def e4m3_bytes(x):
    return torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


@pytest.mark.parametrize("d,dtype,fp8", [(128, F16, False), (64, F16, False), (128, BF16, False), (128, F16, True), (128, BF16, True)])
@pytest.mark.parametrize("nats,at", [(12.0, 0), (15.0, 700), (17.4, 0), (19.0, 1)])
def test_decode_rows_that_one_key_dominates(d, dtype, fp8, nats, at):
    """The same from the cache, with and without weights; P (1 at most) is scaled by 2^15, so that half of fp16's smallest step is
    2^-40 of the largest probability."""
    n, hq, hkv = 1000, 4, 2
    q, k, v, scale = sink_rows(910, n, hq, hkv, d, dtype, nats, at)
    q = q[:1]
    with Pool(hq, hkv, d, dtype, (n + 15) // 16, fp8=fp8, seqs=1, split_tokens=1024) as p:
        kv = np.zeros((p.blocks * 16, hkv, 2, d), np.uint8 if fp8 else np.uint16)
        for i, x in enumerate((k, v)):
            kv[:n, :, i] = e4m3_bytes(real(x, dtype) / p.scales[i]) if fp8 else x
        data = np.ascontiguousarray(kv.reshape(p.blocks, 16, hkv, 2, d).transpose(0, 2, 3, 1, 4))
        p.fill(data)
        tab, ctx, dq = up(np.arange(p.blocks, dtype=np.int32)[None]), up(np.array([n], np.int32)), up(q)
        w, outs = torch.zeros((1, hkv, n), dtype=torch.float32, device=DEV), [torch.zeros_like(dq) for _ in range(2)]
        args = (tab.data_ptr(), p.blocks, ctx.data_ptr())
        pie.pie_decode_attention_weights(p.h, 0, dq.data_ptr(), outs[0].data_ptr(), *args, 1, scale, w.data_ptr(), n)
        pie.pie_decode_attention(p.h, 0, dq.data_ptr(), outs[1].data_ptr(), *args, 1, scale)
        pie.pie_sync(p.h)
        assert torch.equal(outs[0], outs[1])
        stored = p.values(data).transpose(0, 3, 1, 2, 4).reshape(-1, hkv, 2, d)[:n]
    want_w = oo.attention_weights(real(q[0], dtype), stored[:, :, 0], scale)
    assert np.all(np.abs(w[0].cpu().numpy() - want_w) <= 1.3e-4 * want_w + 1e-30)
    for h in range(hq):
        want, weights, size = oo.attend(real(q[0, h], dtype), stored[:, h // 2, 0], stored[:, h // 2, 1], scale)
        bound = sink_bound(dtype, want, size, weights, stored[:, h // 2, 1], 2.0 ** -40 if fp8 or dtype == F16 else 0.0)
        err = np.abs(down(outs[0][0, h], dtype) - want)
        assert np.all(err <= bound), (h, float((err / bound).max()))


@pytest.mark.parametrize("d,dtype", [(128, F16), (64, F16), (128, BF16)])
@pytest.mark.parametrize("nats,at", [(5.5, 200), (12.0, 0), (16.0, 300), (17.4, 0), (17.4, 999)])
def test_chunk_rows_that_one_key_dominates(d, dtype, nats, at):
    """The same for a chunk of 70 tokens at the end of 1000 cached ones (P up to 2^15 in fp16, as for whole prompts)."""
    n, chunk, hq, hkv = 1000, 70, 4, 2
    q, k, v, scale = sink_rows(920, n, hq, hkv, d, dtype, nats, at)
    q = q[n - chunk:]
    with Pool(hq, hkv, d, dtype, (n + 15) // 16, seqs=1) as p:
        kv = np.zeros((p.blocks * 16, hkv, 2, d), np.uint16)
        kv[:n, :, 0], kv[:n, :, 1] = k, v
        p.fill(np.ascontiguousarray(kv.reshape(p.blocks, 16, hkv, 2, d).transpose(0, 2, 3, 1, 4)))
        tab, lens, off = np.arange(p.blocks, dtype=np.int32)[None], np.array([n], np.int32), np.array([0, chunk], np.int32)
        dtab, dlens, doff, dq = up(tab), up(lens), up(off), up(q)
        out = torch.zeros_like(dq)
        pie.pie_prefill_attention(p.h, 0, dq.data_ptr(), out.data_ptr(), dtab.data_ptr(), p.blocks, dlens.data_ptr(), doff.data_ptr(), lens, off, 1,
                                  scale)
        pie.pie_sync(p.h)
    q, k, v, got = real(q, dtype), real(k, dtype), real(v, dtype), down(out, dtype)
    for i in [0, 1, 33, chunk - 1]:
        m = n - chunk + i + 1
        for h in range(hq):
            want, w, size = oo.attend(q[i, h], k[:m, h // 2], v[:m, h // 2], scale)
            err = np.abs(got[i, h] - want)
            bound = sink_bound(dtype, want, size, w, v[:m, h // 2], 2.0 ** -32 if dtype == F16 else 0.0)
            assert np.all(err <= bound), (i, h, float((err / bound).max()))


# ============================================================================== tables and strides much wider than the batch
@pytest.mark.parametrize("hq,hkv,d,dtype,fp8", [(8, 2, 64, F16, False), (8, 8, 128, BF16, False), (4, 1, 128, F16, True)])
@pytest.mark.parametrize("lens,width", [([333], 2048), ([1, 700, 0, 45], 2048), ([50] * 9, 8000)])
def test_weights_of_short_sequences_in_a_wide_table(hq, hkv, d, dtype, fp8, lens, width):
    """The table and the rows of the account are made for 32 768 tokens and more; entries behind a sequence's blocks name no block."""
    with Pool(hq, hkv, d, dtype, sum((n + 15) // 16 for n in lens), fp8=fp8) as p:
        c = WeightsCase(p, lens, 830, width=width, spare=16 * width)
        c.call()
        c.call()
        pie.pie_sync(p.h)
        c.check(steps=2)


class EvictCase:
    """One eviction of random blocks, weights as given, into wider tables and strides; check() against the oracle's choice."""

    def __init__(self, p, lens, w, budget, recent, in_place, seed, width=None):
        self.p, self.lens, self.w, self.in_place = p, lens, w, in_place
        need = sum((n + 15) // 16 for n in lens)
        data = p.random(seed)
        p.fill(data)
        table = table_for(lens, need, seed, width)
        dst = table if in_place else table_for([min(n, budget) for n in lens], p.blocks - need, seed + 1, width, first=need)
        dt, dd, dw, ctx = up(table), up(dst), up(w), up(np.array(lens, np.int32))
        out = dw if in_place else torch.full(w.shape, -7.0, dtype=torch.float32, device=DEV)
        kept = torch.full((len(lens), p.hkv, budget), 12345, dtype=torch.int32, device=DEV)
        pie.pie_kv_evict(p.h, 0, dt.data_ptr(), table.shape[1], ctx.data_ptr(), len(lens), dw.data_ptr(), w.shape[2], budget, recent,
                         dst_block_table_dev=None if in_place else dd.data_ptr(), dst_max_blocks=0 if in_place else dst.shape[1],
                         weights_out=None if in_place else out.data_ptr(), weights_out_stride=0 if in_place else w.shape[2],
                         new_lens_dev=ctx.data_ptr(), kept_dev=kept.data_ptr())
        pie.pie_sync(p.h)
        want, want_w = data.copy(), w.copy() if in_place else np.full(w.shape, -7.0, np.float32)
        got_k = kept.cpu().numpy()
        for s, n in enumerate(lens):
            m = min(n, budget)
            for h in range(p.hkv):
                chosen = oo.keep(w[s, h], n, budget, recent)
                assert got_k[s, h].tolist() == chosen + [-1] * (budget - m), (s, h)
                to, c = np.arange(m), np.array(chosen, np.int64)
                want[dst[s, to // 16], h, :, to % 16] = data[table[s, c // 16], h, :, c % 16]
                want_w[s, h, :m], want_w[s, h, m:n] = w[s, h, c], 0.0
        assert np.array_equal(p.raw(), want)
        assert np.array_equal(out.cpu().numpy().view(np.uint32), want_w.view(np.uint32))
        assert ctx.cpu().numpy().tolist() == [min(n, budget) for n in lens]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,width,budget", [([700], 2048, 100), ([333, 20, 0, 1200], 7500, 90)])
def test_evict_short_sequences_in_a_wide_table(in_place, fp8, lens, width, budget):
    """2048 blocks a row: sixteen weights a thread for a short sequence; 7500: the blocks' slots are looked up again."""
    blocks = sum((n + 15) // 16 + (min(n, budget) + 15) // 16 for n in lens)
    with Pool(4, 2, 128, F16, blocks, fp8=fp8) as p:
        w = np.exp(2 * np.random.default_rng(6).standard_normal((len(lens), 2, 16 * width))).astype(np.float32)
        EvictCase(p, lens, w, budget, 11, in_place, 340, width=width)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("name", ["zeros", "few values", "odd", "rising", "falling", "close"])
@pytest.mark.parametrize("budget,recent", [(600, 100), (9000, 0), (17000, 300)])
def test_evict_selection_over_several_pieces(in_place, name, budget, recent):
    """20 000 tokens, more than the selecting threads hold at a time, with hundreds of weights that share the first digits or are
    equal: all digits are searched, and the places left for equal weights end in the first, second or third piece."""
    n, hkv = 20000, 2
    rng, shape = np.random.default_rng(9), (1, hkv, n + 3)
    t = np.arange(n + 3)
    w = {"zeros": np.zeros(shape), "few values": rng.integers(0, 3, shape) * 1.5,
         "odd": rng.choice([0.0, -0.0, np.nan, np.inf, -np.inf, 1.0, -1.0, 1e-40], shape),
         "rising": np.broadcast_to(1 + t * 2.0 ** -23, shape), "falling": np.broadcast_to(2 - t * 2.0 ** -23, shape),
         "close": 1 + rng.integers(0, 5000, shape) * 2.0 ** -23}[name]
    with Pool(2, hkv, 64, F16, 1250 + (budget + 15) // 16, seqs=1) as p:
        EvictCase(p, [n], np.ascontiguousarray(w, dtype=np.float32), budget, recent, in_place, 350)


def test_decode_with_a_tiny_value_scale():
    """8-bit values times 2^-118, bf16: the outputs are those of the scale 1 times 2^-118 (what falls below 2^-126 may be 0)."""
    n, hq, hkv, d = 300, 4, 2, 128
    outs = []
    for v_scale in (1.0, 2.0 ** -118):
        with Pool(hq, hkv, d, BF16, (n + 15) // 16, fp8=True, seqs=1, v_scale=v_scale) as p:
            p.fill(p.random(940))
            tab, ctx, dq = up(np.arange(p.blocks, dtype=np.int32)[None]), up(np.array([n], np.int32)), up(rows(941, 1, hq, d, BF16))
            out = torch.zeros_like(dq)
            pie.pie_decode_attention(p.h, 0, dq.data_ptr(), out.data_ptr(), tab.data_ptr(), p.blocks, ctx.data_ptr(), 1, d ** -0.5)
            pie.pie_sync(p.h)
            outs.append(down(out, BF16))
    assert np.abs(outs[0]).max() > 0.01 and np.all(np.abs(outs[1] - outs[0] * 2.0 ** -118) <= 2.0 ** -126)
