"""Rotary positions with the cache write, attention over whole prompts, decode attention with accumulated weights and eviction,
through the C ABI against the fp64 oracle.

Bounds (u = half a step of the type, relative: bf16 2^-8, fp16 2^-11, E4M3 2^-4):
  rotation   u |want| for the one rounding, plus 1e-6 (|a| + |b|): the angle's conversion to fp32 (2^-25 of half a turn, 9.4e-8
             radians), sincospif and three fp32 operations (2^-23 each) stay below 6e-7; subnormals: half of the smallest one
  attention  a probability is rounded once (u) and carries the score's error: fp32 accumulation of D <= 128 products,
             128 x 2^-24 x scale x sum |q k| <= 7.6e-6 x 8 for N(0, 1) inputs, in numerator and denominator, and an exponential
             of at most 1e-4: (u + 4e-4) sum p |v| in all; then u |want| for the result
  weights    no 16-bit rounding: 2 x (6.1e-5 + 2^-22) of each head's probability, fp32 sums: 1.3e-4 of what was added + 2^-23 |want|
"""
import numpy as np
import pytest
import torch

from oracle import operators as oo
from paper_2411_09317_b200 import binding as pie
from paper_2411_09317_b200 import synth
from tests.gpu_helpers import PoolCase
from tests.helpers import Case

pytestmark = pytest.mark.gpu
F16, BF16 = synth.F16, synth.BF16
U = {F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F16: 2.0 ** -25, BF16: 2.0 ** -134}
DEV = torch.device("cuda:0")


def up(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).to(DEV)


def real(bits, dtype):
    return synth.bits16_to_f32(np.asarray(bits).view(np.uint16), dtype).astype(np.float64)


def down(t, dtype):
    return real(t.cpu().numpy(), dtype)


def rows(seed, n, h, d, dtype, gain=1.0):
    return synth.tensor_bits(seed, synth.STREAM_KNEW, (n, h, d), dtype, gain)


class Pool:
    """A pool of one or more layers with every block on the GPU; ids are 0 .. n - 1."""

    def __init__(self, hq, hkv, d, dtype, blocks, seqs=16, layers=1, host_slots=0, fp8=False, k_scale=0.25, v_scale=0.5, **kw):
        self.hq, self.hkv, self.d, self.dtype, self.blocks, self.fp8 = hq, hkv, d, dtype, blocks, fp8
        self.scales = (k_scale, v_scale) if fp8 else (1.0, 1.0)
        self.h = pie.pie_pool_create(n_layers=layers, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype, n_logical_blocks=blocks,
                                     max_seqs=seqs, n_gpu_slots=layers * blocks, n_host_slots=host_slots, kv_fp8=int(fp8), **kw)
        if fp8:
            pie.pie_set_kv_scales(self.h, k_scale, v_scale)
        pie.pie_block_alloc(self.h, blocks)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        if self.h:
            pie.pie_pool_destroy(self.h)
            self.h = None

    def fill(self, data, layer=0):
        """data: [blocks][Hkv][2][16][D] 16-bit patterns or E4M3 bytes"""
        for b in range(self.blocks):
            pie.pie_block_write(self.h, layer, b, data[b])

    def raw(self, layer=0):
        kind = np.uint8 if self.fp8 else np.uint16
        return np.stack([pie.pie_block_read(self.h, layer, b).view(kind).reshape(self.hkv, 2, 16, self.d) for b in range(self.blocks)])

    def values(self, raw):
        if not self.fp8:
            return real(raw, self.dtype)
        x = torch.from_numpy(raw.copy()).view(torch.float8_e4m3fn).double().numpy()
        x[:, :, 0] *= self.scales[0]
        x[:, :, 1] *= self.scales[1]
        return x

    def random(self, seed):
        if self.fp8:
            return np.stack([synth.kv_unit_bytes(seed, 0, b, self.blocks, self.hkv, self.d) for b in range(self.blocks)])
        return np.stack([synth.kv_unit_bits(seed, 0, b, self.blocks, self.hkv, self.d, self.dtype) for b in range(self.blocks)])


def table_for(lens, blocks, seed=1, width=None, first=0):
    """Scattered block ids, [S][width]; entries behind a sequence's blocks name no block."""
    need = [(n + 15) // 16 for n in lens]
    order = np.random.default_rng(seed).permutation(blocks)[:sum(need)] + first
    t = np.full((len(lens), width or max(max(need), 1)), -1, np.int32)
    at = 0
    for s, n in enumerate(need):
        t[s, :n] = order[at:at + n]
        at += n
    return t


def refused(status, call, *args, **kw):
    with pytest.raises(pie.PieError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value


# ======================================================================================================== rotary + write
def frequencies(rotary, theta=10000.0):
    return theta ** (-np.arange(0, rotary, 2) / rotary)


def run_rope(p, seed, share, start, axes, rotary, adjacent=False, amplitude=1.0, packed=False, in_place=False, positions=None,
             write=True, k_out=True, gain=1.0):
    n = int(sum(share))
    axis = np.arange(rotary // 2) * axes // (rotary // 2)
    freq = frequencies(rotary)
    pie.pie_set_rope(p.h, rotary, axis, freq, adjacent=int(adjacent), amplitude=amplitude)
    q, k, v = rows(seed, n, p.hq, p.d, p.dtype, gain), rows(seed + 1, n, p.hkv, p.d, p.dtype, gain), rows(seed + 2, n, p.hkv, p.d, p.dtype, gain)
    seq = np.repeat(np.arange(len(share)), share).astype(np.int32)
    place = (start + np.concatenate([np.arange(c) for c in share])).astype(np.int32) if n else np.zeros(0, np.int32)
    if positions is None:
        rng = np.random.default_rng(seed)
        positions = rng.integers(-1000, 1 << 30, (axes, n)).astype(np.int32)
    table = table_for([start + c for c in share], p.blocks)
    before = p.raw()
    if packed:
        qkv = up(np.concatenate([q, k, v], axis=1))
        dq, dk, dv = qkv[:, :p.hq], qkv[:, p.hq:p.hq + p.hkv], qkv[:, p.hq + p.hkv:]
    else:
        dq, dk, dv = up(q), up(k), up(v)
    sentinel = 0x5a5a
    oq = dq if in_place else torch.full((n + 3, p.hq, p.d), sentinel, dtype=torch.int16, device=DEV)
    ok = dk if in_place else torch.full((n + 3, p.hkv, p.d), sentinel, dtype=torch.int16, device=DEV)
    dpos, dseq, dplace, dtab = up(positions), up(seq), up(place), up(table)
    pie.pie_rope_kv_write(p.h, 0, dq.data_ptr(), oq.data_ptr(), dk.data_ptr(), ok.data_ptr() if k_out else None, dv.data_ptr(), dpos.data_ptr(),
                          dseq.data_ptr(), dplace.data_ptr(), n, dtab.data_ptr() if write else None, table.shape[1], len(share),
                          q_stride=dq.stride(0) if packed else 0, k_stride=dk.stride(0) if packed else 0, v_stride=dv.stride(0) if packed else 0)
    pie.pie_sync(p.h)
    for name, bits, got in (("q", q, oq), ("k", k, ok)):
        want, size = oo.rotate(real(bits, p.dtype), positions, axis, freq, adjacent, amplitude)
        if name == "k":
            k_want, k_size = want, size
            if not k_out:
                assert in_place or bool((got == sentinel).all())
                continue
        err = np.abs(down(got[:n], p.dtype) - want)
        bound = U[p.dtype] * np.abs(want) + 1e-6 * size + TINY[p.dtype]
        assert np.all(err <= bound), (name, float((err / bound).max()))
        rest = np.asarray(bits)[:, :, rotary:]
        assert np.array_equal(got[:n].cpu().numpy().view(np.uint16)[:, :, rotary:], rest)      # passed through, bit for bit
        if not in_place:
            assert bool((got[n:] == sentinel).all())                                            # rows behind the last token
    after = p.raw()
    want = p.values(before) if n == 0 or not write else None
    if not write:
        assert np.array_equal(before, after)
        return
    touched = np.zeros(before.shape[:1] + (16,), bool)
    blk, row = table[seq, place // 16], place % 16
    touched[blk, row] = True
    same = before == after
    assert np.all(same.transpose(0, 3, 1, 2, 4)[~touched])
    if n == 0:
        return
    got_k, got_v = after[blk, :, 0, row], after[blk, :, 1, row]
    if p.fp8:
        code_k, code_v = (torch.from_numpy(x.copy()).view(torch.float8_e4m3fn).double().numpy() for x in (got_k, got_v))
        for code, x, size, sc in ((code_k, k_want, k_size, p.scales[0]), (code_v, real(v, p.dtype), 0.0, p.scales[1])):
            want = np.clip(x / sc, -448, 448)
            assert np.all(np.abs(code - want) <= 2.0 ** -4 * np.abs(want) + (1e-6 * size + 1e-6 * np.abs(x)) / sc + 2.0 ** -10)
    else:
        err = np.abs(real(got_k, p.dtype) - k_want)
        assert np.all(err <= U[p.dtype] * np.abs(k_want) + 1e-6 * k_size + TINY[p.dtype])
        assert np.array_equal(got_v, v)
        if k_out and not in_place:
            assert np.array_equal(got_k, ok[:n].cpu().numpy().view(np.uint16))                  # the cache holds the same bits


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 4, 64, F16), (32, 8, 128, BF16), (6, 2, 128, F16), (7, 1, 64, BF16)])
@pytest.mark.parametrize("share,start", [([1], 0), ([1, 1, 1, 1, 1], 47), ([3, 0, 40, 1], 13), ([700, 333], 5)])
@pytest.mark.parametrize("axes,adjacent,packed", [(1, False, False), (3, False, True), (4, True, False)])
def test_rope_write(hq, hkv, d, dtype, share, start, axes, adjacent, packed):
    with Pool(hq, hkv, d, dtype, 80) as p:
        p.fill(p.random(3))
        run_rope(p, 20, share, start, axes, d, adjacent=adjacent, packed=packed)


@pytest.mark.parametrize("rotary", [16, 48, 64, 112, 128])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rope_part_of_the_head(rotary, adjacent):
    with Pool(4, 2, 128, F16, 8) as p:
        p.fill(p.random(4))
        run_rope(p, 30, [17, 9], 3, 2, rotary, adjacent=adjacent, amplitude=1.25)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("share", [[1], [60, 1, 19]])
def test_rope_into_an_8bit_cache(dtype, share):
    with Pool(8, 2, 128, dtype, 16, fp8=True) as p:
        p.fill(p.random(5))
        run_rope(p, 40, share, 7, 3, 64, packed=True)
        run_rope(p, 41, share, 7, 1, 128, gain=64.0)      # saturates at 448 times the scale


def test_rope_in_place_and_without_some_outputs():
    with Pool(8, 2, 128, BF16, 16) as p:
        p.fill(p.random(6))
        run_rope(p, 50, [33, 7], 0, 1, 128, in_place=True)
        run_rope(p, 51, [33, 7], 0, 1, 128, k_out=False)
        run_rope(p, 52, [33, 7], 0, 1, 128, write=False)
        run_rope(p, 53, [0], 0, 1, 128)
        # q alone, k alone
        x, pos = up(rows(54, 5, 8, 128, BF16)), up(np.arange(5, dtype=np.int32))
        y = torch.empty_like(x)
        pie.pie_rope_kv_write(p.h, 0, x.data_ptr(), y.data_ptr(), None, None, None, pos.data_ptr(), None, None, 5, None, 0, 0)
        z = torch.empty((5, 2, 128), dtype=torch.int16, device=DEV)
        xk = x[:, :2].contiguous()
        pie.pie_rope_kv_write(p.h, 0, None, None, xk.data_ptr(), z.data_ptr(), None, pos.data_ptr(), None, None, 5, None, 0, 0)
        pie.pie_sync(p.h)
        assert torch.equal(y[:, :2], z)


@pytest.mark.parametrize("positions", [[0], [-1], [(1 << 31) - 1], [-(1 << 31)], [999_983]])
def test_rope_extreme_positions(positions):
    with Pool(2, 2, 128, F16, 2) as p:
        p.fill(p.random(7))
        run_rope(p, 60, [1], 31, 1, 128, positions=np.array([positions], np.int32))


def test_rope_flags_missing_blocks_and_writes_the_others():
    with Pool(4, 2, 64, F16, 6, host_slots=8) as p:
        data = p.random(8)
        p.fill(data)
        pie.pie_set_rope(p.h, 64, [0] * 32, frequencies(64))
        table = np.array([[0, 1], [2, 3]], np.int32)
        pie.pie_swap_out(p.h, 0, [1])
        pie.pie_sync(p.h)
        n = 6
        q, k, v = rows(70, n, 4, 64, F16), rows(71, n, 2, 64, F16), rows(72, n, 2, 64, F16)
        pos = up(np.zeros((1, n), np.int32))
        args = [up(x) for x in (q, k, v)]
        oq, ok = torch.zeros_like(args[0]), torch.zeros_like(args[1])
        for seq, place, status in (([0, 0, 1, 1, 0, 1], [0, 16, 3, 20, 31, 31], pie.PIE_ERR_NOT_RESIDENT),
                                   ([0, 2, 1, -1, 0, 1], [0, 1, 32, 4, -1, 5], pie.PIE_ERR_INVALID)):
            oq.zero_()
            dseq, dplace, dtab = up(np.array(seq, np.int32)), up(np.array(place, np.int32)), up(table)
            pie.pie_rope_kv_write(p.h, 0, args[0].data_ptr(), oq.data_ptr(), args[1].data_ptr(), ok.data_ptr(), args[2].data_ptr(), pos.data_ptr(),
                                  dseq.data_ptr(), dplace.data_ptr(), n, dtab.data_ptr(), 2, 2)
            refused(status, pie.pie_sync, p.h)
            assert np.array_equal(oq.cpu().numpy().view(np.uint16), q)          # position 0 turns nothing: every row is there
            raw = p.raw()
            for s, t, i in zip(seq, place, range(n)):
                if 0 <= s < 2 and 0 <= t < 32 and table[s, t // 16] != 1:
                    assert np.array_equal(raw[table[s, t // 16], :, 0, t % 16], k[i]) and np.array_equal(raw[table[s, t // 16], :, 1, t % 16], v[i])
            assert np.array_equal(raw[1], data[1])


def test_rope_refusals():
    with Pool(4, 2, 64, F16, 4) as p:
        x = torch.zeros(1 << 14, dtype=torch.int16, device=DEV)
        i32 = torch.zeros(64, dtype=torch.int32, device=DEV)
        a, q, qo, k, ko, v = x.data_ptr(), x.data_ptr(), x.data_ptr() + 4096, x.data_ptr() + 8192, x.data_ptr() + 12288, x.data_ptr() + 16384
        i = i32.data_ptr()

        def call(q=q, qo=qo, k=k, ko=ko, v=v, pos=i, seq=i, place=i, n=2, bt=i, mb=1, s=1, layer=0, **kw):
            pie.pie_rope_kv_write(p.h, layer, q, qo, k, ko, v, pos, seq, place, n, bt, mb, s, **kw)

        refused(pie.PIE_ERR_INVALID, call)                                     # before pie_set_rope
        for bad in ((0, [], []), (80, [0] * 40, [1.0] * 40), (16, [9] * 8, [1.0] * 8), (16, [0] * 8, [np.inf] * 8)):
            refused(pie.PIE_ERR_INVALID, pie.pie_set_rope, p.h, *bad)
        refused(pie.PIE_ERR_UNSUPPORTED, pie.pie_set_rope, p.h, 8, [0] * 4, [1.0] * 4)
        for amp in (0.0, -1.0, float("nan"), float("inf")):
            refused(pie.PIE_ERR_INVALID, pie.pie_set_rope, p.h, 16, [0] * 8, [1.0] * 8, amplitude=amp)
        pie.pie_set_rope(p.h, 64, [0] * 32, frequencies(64))
        for kw in (dict(q=q + 2), dict(ko=ko + 8), dict(v=None), dict(k=None, ko=None), dict(seq=None), dict(place=None), dict(pos=None),
                   dict(qo=None), dict(q=None), dict(bt=None, ko=None), dict(n=-1), dict(mb=0), dict(s=0), dict(q_stride=255), dict(q_stride=260),
                   dict(k_stride=64), dict(v_stride=120), dict(qo=q + 512), dict(ko=k + 256), dict(qo=k), dict(ko=v), dict(ko=qo),
                   dict(qo=q, q_stride=512), dict(q=None, qo=None, k=None, ko=None, bt=None), dict(pos=i + 2), dict(seq=i + 1), dict(place=i + 2),
                   dict(bt=i + 2), dict(q_stride=1 << 40)):
            refused(pie.PIE_ERR_INVALID, call, **kw)
        refused(pie.PIE_ERR_RANGE, call, layer=1)
        refused(pie.PIE_ERR_RANGE, call, layer=-1)
        call(n=0)
        pie.pie_sync(p.h)
        assert int(x.abs().sum()) == 0


# =============================================================================================================== prompts
def run_prompt(hq, hkv, d, dtype, lens, seed, packed=False, scale=None, gain=1.0, poison=None, k_gain=1.0, sample=None):
    n = int(sum(lens))
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q, k, v = rows(seed, n, hq, d, dtype, gain), rows(seed + 1, n, hkv, d, dtype, k_gain), rows(seed + 2, n, hkv, d, dtype)
    if poison is not None:
        poison(k, v, off)
    scale = d ** -0.5 if scale is None else scale
    extra = 5
    out = torch.full((n + extra, hq, d), 0x7e01 if dtype == F16 else 0x7fc1, dtype=torch.int16, device=DEV)   # NaN: every row is written
    # rows behind the last sequence hold NaN as well: nothing may read them into a result
    pad = lambda x: np.concatenate([x, np.full((extra,) + x.shape[1:], 0x7e00 if dtype == F16 else 0x7fc0, np.uint16)])  # noqa: E731
    if packed:
        qkv = up(np.concatenate([pad(q), pad(k), pad(v)], axis=1))
        dq, dk, dv = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:
        dq, dk, dv = up(pad(q)), up(pad(k)), up(pad(v))
    with Pool(hq, hkv, d, dtype, 1) as p:
        pie.pie_prompt_attention(p.h, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), out.data_ptr(), off, len(lens), scale,
                                 q_stride=dq.stride(0), k_stride=dk.stride(0), v_stride=dv.stride(0))
        pie.pie_sync(p.h)
    got = down(out[:n], dtype)
    assert bool((out[n:] == (0x7e01 if dtype == F16 else 0x7fc1)).all())
    return got, (real(q, dtype), real(k, dtype), real(v, dtype), off, scale)


def check_prompt(dtype, got, want, size, what=""):
    err = np.abs(got - want)
    bound = (U[dtype] + 4e-4) * size + U[dtype] * np.abs(want) + TINY[dtype]
    assert np.all(np.isfinite(got)) and np.all(err <= bound), (what, float((err / bound).max()), np.argwhere(~(err <= bound))[:4])


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 4, 64, F16), (4, 1, 128, BF16), (2, 2, 128, F16), (8, 1, 128, BF16), (3, 1, 64, BF16),
                                            (5, 1, 128, F16), (12, 2, 128, BF16), (7, 1, 64, F16), (2, 2, 64, BF16)])
@pytest.mark.parametrize("lens", [[1], [2, 1, 3], [45], [128], [129, 0, 1, 257, 64, 0], [511, 130]])
def test_prompt_lengths_and_groups(hq, hkv, d, dtype, lens):
    got, args = run_prompt(hq, hkv, d, dtype, lens, 100, packed=len(lens) > 1)
    check_prompt(dtype, got, *oo.prompt_attention(*args))


@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 1, 128, BF16), (2, 2, 64, F16), (8, 1, 128, F16)])
def test_prompt_of_many_stages(hq, hkv, d, dtype):
    """Long enough for every buffer of the kernel to be used several times; sampled rows."""
    lens = [1, 2500, 1033]
    got, (q, k, v, off, scale) = run_prompt(hq, hkv, d, dtype, lens, 110)
    assert np.all(np.isfinite(got))
    rng = np.random.default_rng(2)
    for i in [0, 1, 128, 1000, 2500, 2501, 3533] + rng.integers(0, sum(lens), 30).tolist():
        s = int(np.searchsorted(off, i, side="right")) - 1
        for h in range(hq):
            want, _, size = oo.attend(q[i, h], k[off[s]:i + 1, h * k.shape[1] // hq], v[off[s]:i + 1, h * k.shape[1] // hq], scale)
            check_prompt(dtype, got[i, h], want, size, (i, h))


@pytest.mark.parametrize("scale,k_gain", [(0.0, 1.0), (-0.09, 1.0), (0.09, 16.0), (1e-6, 1.0)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_prompt_scales(dtype, scale, k_gain):
    """Zero, negative and tiny scales; keys so large that the softmax is all but a maximum.  The score's fp32 error grows with
    its size: 128 x 2^-24 x scale x sum |q k| = 1.1e-4 x k_gain of a probability, in numerator and denominator."""
    got, args = run_prompt(4, 2, 128, dtype, [300, 77], 120, scale=scale, k_gain=k_gain)
    want, size = oo.prompt_attention(*args)
    err = np.abs(got - want)
    bound = (U[dtype] + 1e-4 + 3e-4 * max(1.0, k_gain)) * size + U[dtype] * np.abs(want) + TINY[dtype]
    assert np.all(err <= bound), float((err / bound).max())


@pytest.mark.parametrize("dtype,d", [(F16, 128), (BF16, 128), (BF16, 64)])
@pytest.mark.parametrize("value", ["nan", "inf", "-inf", "largest"])
def test_prompt_masked_places_cannot_reach_a_row(dtype, d, value):
    """NaN and infinities in the keys and values of later tokens, and of other sequences, change nothing; rows that see such a
    value get what the definition gives (NaN or the infinity in the value's own column)."""
    bits = {"nan": 0x7e00 if dtype == F16 else 0x7fc0, "inf": 0x7c00 if dtype == F16 else 0x7f80, "-inf": 0xfc00 if dtype == F16 else 0xff80,
            "largest": 0x7bff if dtype == F16 else 0x7f7f}[value]
    lens, at = [200, 300, 64], {0: 150, 1: 17, 2: 63}

    def poison_v(k, v, off):
        for s, t in at.items():
            v[off[s] + t, :, 5] = bits

    clean, args = run_prompt(4, 2, d, dtype, lens, 130)
    got, _ = run_prompt(4, 2, d, dtype, lens, 130, poison=poison_v)
    for s, t in at.items():
        o, e = args[3][s], args[3][s + 1]
        assert np.array_equal(got[o:o + t], clean[o:o + t])
        assert np.array_equal(np.delete(got[o + t:e], 5, axis=2), np.delete(clean[o + t:e], 5, axis=2))
        seen = got[o + t:e, :, 5]
        if value == "nan":
            assert np.all(np.isnan(seen))
        elif value != "largest":
            assert np.all(seen == (np.inf if value == "inf" else -np.inf))

    def poison_k(k, v, off):
        for s, t in at.items():
            k[off[s] + t] = bits

    got, _ = run_prompt(4, 2, d, dtype, lens, 130, poison=poison_k)
    for s, t in at.items():
        o, e = args[3][s], args[3][s + 1]
        assert np.array_equal(got[o:o + t], clean[o:o + t])
        assert value != "nan" or np.all(np.isnan(got[o + t:e]))


@pytest.mark.parametrize("value", [0x7fc0, 0xff80])
def test_prompt_values_not_finite_in_every_item(value):
    """Many more items than CTAs, of one tile and of two in every order, each with NaN or -inf in the last value of its sequence: a
    row but the last is as without it, the last one gets the value in its column."""
    lens = [(1, 130, 20, 3, 257, 32, 9, 64, 65, 2)[i % 10] for i in range(400)]
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)

    def poison(k, v, off):
        v[off[1:] - 1, :, 3] = value

    clean, _ = run_prompt(8, 2, 64, BF16, lens, 150)
    got, _ = run_prompt(8, 2, 64, BF16, lens, 150, poison=poison)
    last = np.zeros(len(got), bool)
    last[off[1:] - 1] = True
    assert np.array_equal(got[~last], clean[~last])
    assert np.array_equal(np.delete(got[last], 3, axis=2), np.delete(clean[last], 3, axis=2))
    assert np.all(np.isnan(got[last][:, :, 3]) if value == 0x7fc0 else got[last][:, :, 3] == -np.inf)


def test_prompt_repeats_bit_for_bit_and_on_two_pools_at_once():
    """The same inputs give the same bits, alone and with a second pool's call running beside it on its own stream."""
    lens = [700, 1, 333, 64]
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    n, hq, hkv, d = int(off[-1]), 8, 2, 128
    q, k, v = (up(rows(140 + i, n, h, d, BF16)) for i, h in enumerate((hq, hkv, hkv)))
    with Pool(hq, hkv, d, BF16, 1) as a, Pool(hq, hkv, d, BF16, 1) as b:
        outs = [torch.zeros_like(q) for _ in range(6)]
        torch.cuda.synchronize()
        for i, o in enumerate(outs):
            pie.pie_prompt_attention((a if i % 2 == 0 else b).h, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), off, 4, d ** -0.5)
        pie.pie_sync(a.h)
        pie.pie_sync(b.h)
        for o in outs[1:]:
            assert torch.equal(o, outs[0])


def test_prompt_refusals():
    with Pool(4, 2, 64, F16, 1) as p:
        x = torch.zeros(1 << 15, dtype=torch.int16, device=DEV)
        a = x.data_ptr()

        def call(q=a, k=a + 8192, v=a + 16384, o=a + 24576, off=(0, 3, 8), n=2, **kw):
            pie.pie_prompt_attention(p.h, q, k, v, o, np.array(off, np.int32), n, 0.1, **kw)

        for kw in (dict(off=(1, 3, 8)), dict(off=(0, 5, 3)), dict(n=-1), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=a + 2),
                   dict(o=a + 24584), dict(q_stride=128), dict(k_stride=132), dict(v_stride=64), dict(o=a), dict(o=a + 2048), dict(o=a + 8192),
                   dict(o=a + 16384)):
            refused(pie.PIE_ERR_INVALID, call, **kw)
        call(off=(0, 0, 0))
        call(n=0)
        pie.pie_sync(p.h)
        assert int(x.abs().sum()) == 0


# ============================================================================================================== weights
def run_weights(hq, hkv, d, dtype, lens, seed, fp8=False, stride_extra=3, steps=2, split=0, append=False):
    case = Case(1, hq, hkv, d, dtype, lens, seed=seed, placement="random", shuffle_table=True, kv_fp8=fp8)
    pc = PoolCase(case, all_on_gpu=True, split_tokens=split)
    stride = max(max(lens), 1) + stride_extra
    before = np.random.default_rng(seed).random((len(lens), hkv, stride)).astype(np.float32)
    w = up(before)
    plain = torch.zeros_like(pc.out[0])
    kn = vn = None
    if append:
        kn, vn = up(rows(seed + 1, len(lens), hkv, d, dtype)), up(rows(seed + 2, len(lens), hkv, d, dtype))
    new = dict(k_new=None if kn is None else kn.data_ptr(), v_new=None if vn is None else vn.data_ptr())
    for _ in range(steps):
        pie.pie_decode_attention_weights(pc.pool, 0, pc.q[0].data_ptr(), pc.out[0].data_ptr(), pc.bt.data_ptr(), case.block_table.shape[1],
                                         pc.ctx.data_ptr(), case.S, case.scale, w.data_ptr(), stride, **new)
    pie.pie_decode_attention(pc.pool, 0, pc.q[0].data_ptr(), plain.data_ptr(), pc.bt.data_ptr(), case.block_table.shape[1], pc.ctx.data_ptr(),
                             case.S, case.scale, **new)
    pie.pie_sync(pc.pool)
    assert split == 0 or torch.equal(plain, pc.out[0])       # the same chunks: the same bits
    got = w.cpu().numpy().astype(np.float64)
    kv = Pool.values(pc_view(pc, hkv, d, dtype, fp8), np.stack([pc.read_unit(0, b).reshape(hkv, 2, 16, d) for b in range(case.NB)]))
    for s, n in enumerate(lens):
        k = kv[case.block_table[s, :(n + 15) // 16], :, 0].transpose(0, 2, 1, 3).reshape(-1, hkv, d)[:n]
        added = steps * oo.attention_weights(case.q_f(0)[s], k, case.scale)
        want = before[s, :, :n] + added
        err = np.abs(got[s, :, :n] - want)
        bound = 1.3e-4 * added + 2.0 ** -23 * steps * np.abs(want) + 1e-30
        assert np.all(err <= bound), (s, float((err / bound).max()))
        assert np.array_equal(got[s, :, n:], before[s, :, n:].astype(np.float64))
        v = kv[case.block_table[s, :(n + 15) // 16], :, 1].transpose(0, 2, 1, 3).reshape(-1, hkv, d)[:n]
        for h in range(hq):
            row = down(pc.out[0][s, h], dtype)
            if n == 0:
                assert not row.any()
                continue
            out, _, size = oo.attend(case.q_f(0)[s, h], k[:, h * hkv // hq], v[:, h * hkv // hq], case.scale)
            check_prompt(dtype, row, out, size, (s, h))
    pc.close()
    return got


def pc_view(pc, hkv, d, dtype, fp8):
    v = Pool.__new__(Pool)
    v.fp8, v.dtype, v.scales, v.h = fp8, dtype, (pc.c.k_scale, pc.c.v_scale), None
    return v


@pytest.mark.parametrize("hq,hkv,d,dtype,fp8", [(8, 4, 64, F16, False), (8, 2, 128, BF16, False), (2, 2, 128, F16, False), (8, 1, 128, F16, False),
                                                (6, 2, 64, BF16, False), (5, 1, 128, BF16, False), (8, 2, 128, BF16, True), (4, 4, 128, F16, True),
                                                (7, 1, 128, F16, True)])
@pytest.mark.parametrize("lens", [[1], [0, 15, 16, 17, 0], [700, 1, 2047, 513]])
def test_weights(hq, hkv, d, dtype, fp8, lens):
    run_weights(hq, hkv, d, dtype, lens, 200, fp8=fp8)


def test_weights_short_chunks_and_append():
    a = run_weights(8, 2, 128, BF16, [300, 33, 1], 210, split=16, append=True)
    b = run_weights(8, 2, 128, BF16, [300, 33, 1], 210, split=16, append=True)
    assert np.array_equal(a, b)
    run_weights(4, 2, 128, F16, [300, 33, 1], 211, fp8=True, split=32, append=True)


def test_weights_of_a_batch_beyond_the_in_kernel_plan():
    run_weights(2, 1, 64, F16, [(7 * i) % 40 for i in range(1100)], 220, steps=1)


def test_weights_after_blocks_have_come_back_in_other_slots():
    """The same bits whether or not the blocks were swapped out and in between."""
    lens = [400, 90]
    case = Case(1, 8, 2, 128, F16, lens, seed=230, placement="identity")
    got = []
    for swap in (False, True):
        pc = PoolCase(case, all_on_gpu=True, n_gpu_slots=2 * case.NB)
        w = torch.zeros((2, 2, 400), dtype=torch.float32, device=DEV)
        if swap:
            ids = np.arange(case.NB, dtype=np.int32)
            pie.pie_swap_out(pc.pool, 0, ids)
            pie.pie_swap_in(pc.pool, 0, ids[::-1].copy())
        pie.pie_decode_attention_weights(pc.pool, 0, pc.q[0].data_ptr(), pc.out[0].data_ptr(), pc.bt.data_ptr(), case.block_table.shape[1],
                                         pc.ctx.data_ptr(), 2, case.scale, w.data_ptr(), 400)
        pie.pie_sync(pc.pool)
        got.append((w.cpu().numpy(), pc.out[0].cpu().numpy()))
        pc.close()
    assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1])


def test_weights_refusals_and_a_row_that_is_too_short():
    case = Case(1, 4, 2, 64, F16, [40, 20], seed=240)
    pc = PoolCase(case, all_on_gpu=True)
    w = torch.zeros((2, 2, 40), dtype=torch.float32, device=DEV)

    def call(stride=40, wp=w.data_ptr(), **kw):
        pie.pie_decode_attention_weights(pc.pool, 0, pc.q[0].data_ptr(), pc.out[0].data_ptr(), pc.bt.data_ptr(), case.block_table.shape[1],
                                         pc.ctx.data_ptr(), 2, case.scale, wp, stride, **kw)

    refused(pie.PIE_ERR_INVALID, call, wp=None)
    refused(pie.PIE_ERR_INVALID, call, wp=w.data_ptr() + 2)
    refused(pie.PIE_ERR_INVALID, call, stride=0)
    refused(pie.PIE_ERR_INVALID, call, stride=39, block_table_host=case.block_table, ctx_lens_host=case.ctx_lens)
    pie.pie_sync(pc.pool)
    assert float(w.abs().sum()) == 0
    call(stride=25)                                     # without host lengths the kernel drops what has no room, and says so
    refused(pie.PIE_ERR_INVALID, pie.pie_sync, pc.pool)
    flat = w.cpu().numpy().ravel()
    assert np.all(flat[4 * 25:] == 0) and np.all(flat[70:75] == 0) and np.all(flat[95:100] == 0) and np.all(flat[:70] > 0)
    pc.close()


# ================================================================================================================ evict
def run_evict(hq, hkv, d, dtype, lens, budget, recent, seed, fp8=False, in_place=False, weights=None, kept=True, alias_lens=False, w_in_place=None):
    need = [(n + 15) // 16 for n in lens]
    blocks = max(sum(need), 1)
    dst_need = [(min(n, budget) + 15) // 16 for n in lens]
    total = blocks + (0 if in_place else max(sum(dst_need), 1))
    w_in_place = in_place if w_in_place is None else w_in_place
    with Pool(hq, hkv, d, dtype, total, fp8=fp8, seqs=max(len(lens), 1)) as p:
        data = p.random(seed)
        p.fill(data)
        table = table_for(lens, blocks, seed)
        dst = table if in_place else table_for([min(n, budget) for n in lens], total - blocks, seed + 1, first=blocks)
        stride, out_stride = max(max(lens), 1) + 5, max(max(lens), 1) + 5 if w_in_place else budget + 2
        rng = np.random.default_rng(seed)
        w = np.exp(2 * rng.standard_normal((len(lens), hkv, stride))).astype(np.float32) if weights is None else weights(rng, (len(lens), hkv, stride))
        dw, ctx = up(w), up(np.array(lens, np.int32))
        w_out = dw if w_in_place else torch.full((len(lens), hkv, out_stride), -7.0, dtype=torch.float32, device=DEV)
        dk = torch.full((len(lens), hkv, budget), 12345, dtype=torch.int32, device=DEV)
        new = ctx if alias_lens else torch.full((len(lens),), -1, dtype=torch.int32, device=DEV)
        dt, ddst = up(table), up(dst)
        pie.pie_kv_evict(p.h, 0, dt.data_ptr(), table.shape[1], ctx.data_ptr(), len(lens), dw.data_ptr(), stride, budget, recent,
                         dst_block_table_dev=None if in_place else ddst.data_ptr(), dst_max_blocks=0 if in_place else dst.shape[1],
                         weights_out=None if w_in_place else w_out.data_ptr(), weights_out_stride=0 if w_in_place else out_stride,
                         new_lens_dev=new.data_ptr(), kept_dev=dk.data_ptr() if kept else None)
        pie.pie_sync(p.h)
        raw, got_w, got_k = p.raw(), w_out.cpu().numpy(), dk.cpu().numpy()
        want, want_w = data.copy(), (w if w_in_place else np.full((len(lens), hkv, out_stride), -7.0, np.float32)).copy()
        for s, n in enumerate(lens):
            m = min(n, budget)
            for h in range(hkv):
                chosen = oo.keep(w[s, h], n, budget, recent)
                if kept:
                    assert got_k[s, h].tolist() == chosen + [-1] * (budget - m), (s, h)
                to = np.arange(m)
                c = np.array(chosen, np.int64)
                want[dst[s, to // 16], h, :, to % 16] = data[table[s, c // 16], h, :, c % 16]
                want_w[s, h, :m] = w[s, h, c]
                want_w[s, h, m:min(n, want_w.shape[2])] = 0.0
        assert np.array_equal(raw, want)
        assert np.array_equal(got_w.view(np.uint32), want_w.view(np.uint32))
        assert new.cpu().numpy().tolist() == [min(n, budget) for n in lens]
        if not w_in_place:
            assert np.array_equal(dw.cpu().numpy().view(np.uint32), w.view(np.uint32))


@pytest.mark.parametrize("hq,hkv,d,dtype,fp8", [(8, 4, 64, F16, False), (8, 2, 128, BF16, False), (2, 2, 128, F16, True)])
@pytest.mark.parametrize("lens,budget,recent", [([1], 1, 0), ([2, 1, 0], 1, 1), ([33, 17, 16, 40, 3], 16, 5), ([700, 64, 65, 0, 300], 64, 64),
                                                ([700, 64, 65, 0, 300], 64, 0), ([1200, 2500], 1000, 100), ([90, 100], 200, 10)])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(hq, hkv, d, dtype, fp8, lens, budget, recent, in_place):
    run_evict(hq, hkv, d, dtype, lens, budget, recent, 300, fp8=fp8, in_place=in_place)


def test_evict_in_place_over_many_blocks():
    """Rows travel far and every batch overwrites rows that later batches have passed: long sequences, few and many kept."""
    run_evict(4, 2, 128, F16, [5000, 4097], 4000, 7, 310, in_place=True)
    run_evict(4, 2, 64, BF16, [9000], 1111, 1000, 311, in_place=True)


@pytest.mark.parametrize("in_place,fp8,alias", [(True, False, False), (False, True, True), (True, True, True), (False, False, False)])
def test_evict_of_more_pairs_than_sms(in_place, fp8, alias):
    """More (sequence, KV head) pairs than one wave of the selecting CTAs takes."""
    lens = [(37 * i) % 300 for i in range(90)] + [1500]
    run_evict(8, 4, 128, F16, lens, 90, 11, 313, fp8=fp8, in_place=in_place, alias_lens=alias)
    run_evict(8, 8, 64 if not fp8 else 128, BF16, [700] * 40, 650, 0, 314, fp8=fp8, in_place=in_place, alias_lens=alias)


def test_evict_with_one_of_the_two_in_place():
    run_evict(4, 2, 128, F16, [333, 20], 100, 10, 312, in_place=True, w_in_place=False)
    run_evict(4, 2, 128, F16, [333, 20], 100, 10, 312, in_place=False, w_in_place=True)


@pytest.mark.parametrize("name", ["zeros", "few values", "signs", "odd", "rising", "falling", "subnormal"])
def test_evict_weights_of_every_kind(name):
    """Ties, signs, both zeros, NaN, infinities, sorted weights, values that differ in the last bits only."""
    def weights(rng, shape):
        n = shape[-1]
        base = {"zeros": np.zeros(shape), "few values": rng.integers(0, 3, shape) * 1.5, "signs": rng.standard_normal(shape),
                "odd": rng.choice([0.0, -0.0, np.nan, np.inf, -np.inf, 1.0, -1.0, 1e-40], shape),
                "rising": np.broadcast_to(1 + np.arange(n) * 2.0 ** -23, shape), "falling": np.broadcast_to(2 - np.arange(n) * 2.0 ** -23, shape),
                "subnormal": rng.integers(0, 50, shape) * 2.0 ** -149}[name]
        return np.ascontiguousarray(base, dtype=np.float32)

    run_evict(4, 2, 64, F16, [600, 130, 100, 520], 100, 30, 320, weights=weights)
    run_evict(4, 2, 64, F16, [600, 130, 100, 520], 100, 0, 321, weights=weights, in_place=True)


def test_evict_optional_outputs_and_aliased_lengths():
    run_evict(4, 2, 64, F16, [60, 130, 0, 7], 50, 20, 330, kept=False)
    run_evict(4, 2, 64, F16, [60, 130, 0, 7], 50, 20, 331, alias_lens=True, in_place=True)


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_with_a_budget_beyond_every_table(in_place):
    """The largest budget: every sequence keeps everything; out of place that is a copy."""
    lens = [40, 0, 21]
    with Pool(4, 2, 64, F16, 10) as p:
        data = p.random(345)
        p.fill(data)
        tab, dst = np.array([[0, 1, 2], [0, 0, 0], [3, 4, 0]], np.int32), np.array([[5, 6, 7], [0, 0, 0], [8, 9, 0]], np.int32)
        w0 = np.random.default_rng(1).random((3, 2, 48)).astype(np.float32)
        w, w_out = up(w0), torch.zeros((3, 2, 48), dtype=torch.float32, device=DEV)
        dt, dd, ctx = up(tab), up(dst), up(np.array(lens, np.int32))
        new = torch.zeros(3, dtype=torch.int32, device=DEV)
        pie.pie_kv_evict(p.h, 0, dt.data_ptr(), 3, ctx.data_ptr(), 3, w.data_ptr(), 48, 2 ** 31 - 1, 2 ** 31 - 1 if in_place else 0,
                         dst_block_table_dev=None if in_place else dd.data_ptr(), dst_max_blocks=0 if in_place else 3,
                         weights_out=w_out.data_ptr(), weights_out_stride=48, new_lens_dev=new.data_ptr())
        pie.pie_sync(p.h)
        assert new.cpu().numpy().tolist() == lens
        want = data.copy()
        for s, n in enumerate(lens):
            assert np.array_equal(w_out[s, :, :n].cpu().numpy(), w0[s, :, :n])
            if not in_place:
                t = np.arange(n)
                want[dst[s, t // 16], :, :, t % 16] = data[tab[s, t // 16], :, :, t % 16]
        assert np.array_equal(p.raw(), want)


def test_evict_leaves_a_sequence_alone_that_is_not_all_there():
    with Pool(4, 2, 64, F16, 12, host_slots=16) as p:
        data = p.random(340)
        p.fill(data)
        table = np.array([[0, 1, 2], [3, 4, 5], [6, 7, -1]], np.int32)
        lens = np.array([48, 40, 32], np.int32)
        pie.pie_swap_out(p.h, 0, [4])
        pie.pie_sync(p.h)
        w0 = np.random.default_rng(0).random((3, 2, 48)).astype(np.float32)

        def call(ctx=lens, stride=48, tab=table):
            w, kept = up(w0), torch.full((3, 2, 20), 9, dtype=torch.int32, device=DEV)
            new = torch.zeros(3, dtype=torch.int32, device=DEV)
            dt, dc = up(tab), up(ctx)
            pie.pie_kv_evict(p.h, 0, dt.data_ptr(), tab.shape[1], dc.data_ptr(), 3, w.data_ptr(), stride, 20, 4, new_lens_dev=new.data_ptr(),
                             kept_dev=kept.data_ptr())
            with pytest.raises(pie.PieError) as e:
                pie.pie_sync(p.h)
            return e.value.status, w.cpu().numpy(), kept.cpu().numpy(), new.cpu().numpy()

        status, w, kept, new = call()
        assert status == pie.PIE_ERR_NOT_RESIDENT
        assert new.tolist() == [20, 40, 20] and np.all(kept[1] == -1) and np.all(kept[[0, 2]] >= 0)
        assert np.array_equal(w[1], w0[1]) and not np.array_equal(w[0], w0[0])
        raw = p.raw()
        for b in (3, 4, 5):
            assert np.array_equal(raw[b], data[b])
        # a length beyond the table, and a negative one
        p.fill(data)
        status, w, kept, new = call(ctx=np.array([49, -1, 32], np.int32))
        assert status == pie.PIE_ERR_INVALID and new.tolist() == [49, -1, 20] and np.array_equal(w[:2], w0[:2])
        raw = p.raw()
        assert np.array_equal(raw[:6], data[:6])


def test_evict_refusals():
    with Pool(4, 2, 64, F16, 4) as p:
        i32 = torch.zeros(64, dtype=torch.int32, device=DEV)
        w = torch.zeros((1, 2, 32), dtype=torch.float32, device=DEV)
        i = i32.data_ptr()

        def call(bt=i, mb=2, ctx=i + 64, n=1, wp=w.data_ptr(), stride=32, budget=4, recent=2, layer=0, **kw):
            pie.pie_kv_evict(p.h, layer, bt, mb, ctx, n, wp, stride, budget, recent, **kw)

        for kw in (dict(bt=None), dict(mb=0), dict(ctx=None), dict(n=-1), dict(wp=None), dict(stride=0), dict(budget=0), dict(recent=-1),
                   dict(recent=5), dict(dst_block_table_dev=i + 128, dst_max_blocks=0), dict(dst_block_table_dev=i, dst_max_blocks=1),
                   dict(weights_out=w.data_ptr(), weights_out_stride=16), dict(weights_out=w.data_ptr() + 64, weights_out_stride=0),
                   dict(weights_out=w.data_ptr() + 64, weights_out_stride=16), dict(weights_out=w.data_ptr() - 64, weights_out_stride=16),
                   dict(bt=i + 2), dict(ctx=i + 66), dict(wp=w.data_ptr() + 2), dict(new_lens_dev=i + 129), dict(kept_dev=i + 130),
                   dict(dst_block_table_dev=i + 129, dst_max_blocks=1), dict(weights_out=w.data_ptr() + 1026, weights_out_stride=32)):
            refused(pie.PIE_ERR_INVALID, call, **kw)
        refused(pie.PIE_ERR_RANGE, call, layer=1)
        call(n=0)
        pie.pie_sync(p.h)


# ======================================================================================= captured graphs, other streams
def test_calls_into_a_capture_are_refused():
    with Pool(4, 2, 64, F16, 4) as base:
        stream = torch.cuda.Stream()
        h = pie.pie_pool_create(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=F16, n_logical_blocks=4, max_seqs=2, n_gpu_slots=4,
                                n_host_slots=0, own_streams=0, compute_stream=stream.cuda_stream, copy_in_stream=stream.cuda_stream,
                                copy_out_stream=stream.cuda_stream)
        pie.pie_block_alloc(h, 4)
        pie.pie_set_rope(h, 64, [0] * 32, frequencies(64))
        pie.pie_sync(h)
        x = torch.zeros(1 << 15, dtype=torch.int16, device=DEV)
        i, f = torch.zeros(64, dtype=torch.int32, device=DEV), torch.zeros(64, dtype=torch.float32, device=DEV)
        a = x.data_ptr()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            x.add_(0)
            refused(pie.PIE_ERR_UNSUPPORTED, pie.pie_rope_kv_write, h, 0, a, a, a + 8192, a + 8192, a + 16384, i.data_ptr(), i.data_ptr(),
                    i.data_ptr(), 1, i.data_ptr(), 1, 1)
            refused(pie.PIE_ERR_UNSUPPORTED, pie.pie_prompt_attention, h, a, a + 8192, a + 16384, a + 24576, np.array([0, 2], np.int32), 1, 0.1)
            refused(pie.PIE_ERR_UNSUPPORTED, pie.pie_decode_attention_weights, h, 0, a, a + 8192, i.data_ptr(), 1, i.data_ptr(), 1, 0.1, f.data_ptr(), 16)
            refused(pie.PIE_ERR_UNSUPPORTED, pie.pie_kv_evict, h, 0, i.data_ptr(), 1, i.data_ptr() + 64, 1, f.data_ptr(), 16, 4, 2)
        g.replay()
        torch.cuda.synchronize()
        pie.pie_prompt_attention(h, a, a + 8192, a + 16384, a + 24576, np.array([0, 2], np.int32), 1, 0.1)   # works again
        pie.pie_sync(h)
        pie.pie_pool_destroy(h)
        del g
        assert base.h


# ============================================================================================================ the sequence
@pytest.mark.parametrize("dtype,fp8", [(BF16, False), (F16, False), (F16, True)])
def test_serve_prompts_decode_evict_and_go_on(dtype, fp8):
    """As a serving loop uses them: rotate and write the prompts (three axes), attend over them, decode some tokens while the
    weights add up, cut every head's cache to a budget, give the freed blocks back, swap the rest out and in, decode on.  Every
    output against fp64 over the cache's own stored values; the eviction against the oracle's choice."""
    hq, hkv, d, budget, recent, steps = 8, 2, 128, 96, 16, 5
    lens = np.array([150, 70, 211], np.int32)
    S, width = 3, 16
    scale = d ** -0.5
    axis, freq = np.arange(64) % 3, frequencies(128)
    with Pool(hq, hkv, d, dtype, S * width, host_slots=S * width, fp8=fp8) as p:
        table = np.random.default_rng(7).permutation(S * width).reshape(S, width).astype(np.int32)
        dtab = up(table)
        pie.pie_set_rope(p.h, 128, axis, freq)
        off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        n = int(off[-1])
        q, k, v = rows(400, n, hq, d, dtype), rows(401, n, hkv, d, dtype), rows(402, n, hkv, d, dtype)
        seq = np.repeat(np.arange(S), lens).astype(np.int32)
        place = np.concatenate([np.arange(x) for x in lens]).astype(np.int32)
        positions = np.stack([place // 12, place % 12 // 4, place % 4]).astype(np.int32)
        dq, dk, dv, dseq, dplace, dpos = up(q), up(k), up(v), up(seq), up(place), up(positions)
        oq, ok, out = torch.empty_like(dq), torch.empty_like(dk), torch.empty_like(dq)
        pie.pie_rope_kv_write(p.h, 0, dq.data_ptr(), oq.data_ptr(), dk.data_ptr(), ok.data_ptr(), dv.data_ptr(), dpos.data_ptr(), dseq.data_ptr(),
                              dplace.data_ptr(), n, dtab.data_ptr(), width, S)
        pie.pie_prompt_attention(p.h, oq.data_ptr(), ok.data_ptr(), dv.data_ptr(), out.data_ptr(), off, S, scale)
        pie.pie_sync(p.h)
        check_prompt(dtype, down(out, dtype), *oo.prompt_attention(down(oq, dtype), down(ok, dtype), real(v, dtype), off, scale))

        w = torch.zeros((S, hkv, 16 * width), dtype=torch.float32, device=DEV)
        added = [np.zeros((hkv, 16 * width)) for _ in range(S)]
        ctx = lens.copy()

        def decode(step, ctx, rotary_pos):
            q1, k1, v1 = rows(500 + step, S, hq, d, dtype), rows(600 + step, S, hkv, d, dtype), rows(700 + step, S, hkv, d, dtype)
            b = [up(x) for x in (q1, k1, v1, np.broadcast_to(rotary_pos, (3, S)).astype(np.int32), np.arange(S, dtype=np.int32),
                                 (ctx - 1).astype(np.int32), ctx.astype(np.int32))]
            qo, o = torch.empty_like(b[0]), torch.empty_like(b[0])
            pie.pie_rope_kv_write(p.h, 0, b[0].data_ptr(), qo.data_ptr(), b[1].data_ptr(), None, b[2].data_ptr(), b[3].data_ptr(), b[4].data_ptr(),
                                  b[5].data_ptr(), S, dtab.data_ptr(), width, S)
            pie.pie_decode_attention_weights(p.h, 0, qo.data_ptr(), o.data_ptr(), dtab.data_ptr(), width, b[6].data_ptr(), S, scale, w.data_ptr(),
                                             16 * width)
            pie.pie_sync(p.h)
            kv = p.values(p.raw())
            got, qr = down(o, dtype), down(qo, dtype)
            for s in range(S):
                c = int(ctx[s])
                both = kv[table[s, :(c + 15) // 16]].transpose(2, 0, 3, 1, 4).reshape(2, -1, hkv, d)[:, :c]
                for h in range(hq):
                    want, _, size = oo.attend(qr[s, h], both[0][:, h // 4], both[1][:, h // 4], scale)
                    check_prompt(dtype, got[s, h], want, size, (step, s, h))
                added[s][:, :c] += oo.attention_weights(qr[s], both[0], scale)

        for step in range(steps):
            ctx = ctx + 1
            decode(step, ctx, place.max() + step)
        got_w = w.cpu().numpy()
        for s in range(S):
            assert np.all(np.abs(got_w[s] - added[s]) <= 1.3e-4 * added[s] + 2.0 ** -21 * added[s] + 1e-30)

        before, dctx = p.raw(), up(ctx.astype(np.int32))
        kept = torch.zeros((S, hkv, budget), dtype=torch.int32, device=DEV)
        pie.pie_kv_evict(p.h, 0, dtab.data_ptr(), width, dctx.data_ptr(), S, w.data_ptr(), 16 * width, budget, recent, new_lens_dev=dctx.data_ptr(),
                         kept_dev=kept.data_ptr())
        pie.pie_sync(p.h)
        after, got_k = p.raw(), kept.cpu().numpy()
        for s in range(S):
            for h in range(hkv):
                chosen = np.array(oo.keep(got_w[s, h], int(ctx[s]), budget, recent))
                assert got_k[s, h, :len(chosen)].tolist() == chosen.tolist()
                to = np.arange(len(chosen))
                assert np.array_equal(after[table[s, to // 16], h, :, to % 16], before[table[s, chosen // 16], h, :, chosen % 16])
                moved = np.zeros(16 * width)
                moved[:len(chosen)] = added[s][h, chosen]
                added[s][h] = moved
        ctx = np.minimum(ctx, budget)
        assert dctx.cpu().numpy().tolist() == ctx.tolist()
        used = np.unique(np.concatenate([table[s, :(int(ctx[s]) + steps + 15) // 16] for s in range(S)]))
        pie.pie_block_free(p.h, np.setdiff1d(np.arange(S * width), used))
        pie.pie_swap_out(p.h, 0, used)
        pie.pie_swap_in(p.h, 0, used[::-1].copy())
        p_blocks, p.blocks = p.blocks, S * width

        def raw_used():
            out = np.zeros(after.shape, after.dtype)
            for b in used:
                out[b] = pie.pie_block_read(p.h, 0, int(b)).view(after.dtype).reshape(hkv, 2, 16, d)
            return out

        p.raw = lambda layer=0: raw_used()
        for step in range(steps):
            ctx = ctx + 1
            decode(steps + step, ctx, place.max() + steps + step)
        got_w = w.cpu().numpy()
        for s in range(S):
            assert np.all(np.abs(got_w[s] - added[s]) <= 1.3e-4 * added[s] + 2.0 ** -20 * added[s] + 1e-30)
        p.blocks = p_blocks


# ============================================================================================= offsets that pass 32 bits
def test_far_end_of_a_large_pool():
    """A pool of 4.6 GB: rotary write, weights and eviction in blocks whose elements' offsets do not fit 32 bits."""
    hq, hkv, d, blocks = 8, 8, 128, 70000
    with Pool(hq, hkv, d, F16, blocks, seqs=2) as p:
        lens = [100, 37]
        ids = [blocks - 1 - i for i in range(20)]
        table = np.array([ids[:8], ids[8:16]], np.int32)
        seq, place = np.repeat([0, 1], lens).astype(np.int32), np.concatenate([np.arange(n) for n in lens]).astype(np.int32)
        n = sum(lens)
        k, v, q = rows(400, n, hkv, d, F16), rows(401, n, hkv, d, F16), rows(402, 2, hq, d, F16)
        freq = frequencies(d)
        pie.pie_set_rope(p.h, d, [0] * (d // 2), freq)
        dk, dv, dq, dpos, dseq, dplace, dtab = up(k), up(v), up(q), up(place), up(seq), up(place), up(table)
        pie.pie_rope_kv_write(p.h, 0, None, None, dk.data_ptr(), None, dv.data_ptr(), dpos.data_ptr(), dseq.data_ptr(), dplace.data_ptr(), n,
                              dtab.data_ptr(), 8, 2)
        out, w, ctx = torch.zeros_like(dq), torch.zeros((2, hkv, 128), dtype=torch.float32, device=DEV), up(np.array(lens, np.int32))
        pie.pie_decode_attention_weights(p.h, 0, dq.data_ptr(), out.data_ptr(), dtab.data_ptr(), 8, ctx.data_ptr(), 2, d ** -0.5, w.data_ptr(), 128)
        kept = torch.zeros((2, hkv, 40), dtype=torch.int32, device=DEV)
        pie.pie_sync(p.h)
        raw = lambda b: pie.pie_block_read(p.h, 0, int(b)).view(np.uint16).reshape(hkv, 2, 16, d)  # noqa: E731
        before = {b: raw(b) for b in ids}
        kr, size = oo.rotate(real(k, F16), place[None], np.zeros(d // 2, np.int64), freq, False, 1.0)
        got_w, off = w.cpu().numpy(), [0, 100, 137]
        for s, c in enumerate(lens):
            at = np.arange(c)
            got_k = np.stack([before[table[s, t // 16]][:, 0, t % 16] for t in at])
            assert np.all(np.abs(real(got_k, F16) - kr[off[s]:off[s + 1]]) <= U[F16] * np.abs(kr[off[s]:off[s + 1]]) + 1e-6 * size[off[s]:off[s + 1]] + TINY[F16])
            assert np.array_equal(np.stack([before[table[s, t // 16]][:, 1, t % 16] for t in at]), v[off[s]:off[s + 1]])
            want = oo.attention_weights(real(q[s], F16), real(got_k, F16), d ** -0.5)
            assert np.all(np.abs(got_w[s, :, :c] - want) <= 1.3e-4 * want + 1e-30)
        pie.pie_kv_evict(p.h, 0, dtab.data_ptr(), 8, ctx.data_ptr(), 2, w.data_ptr(), 128, 40, 5, kept_dev=kept.data_ptr())
        pie.pie_sync(p.h)
        for h in range(hkv):
            chosen = oo.keep(got_w[0, h], 100, 40, 5)
            assert kept[0, h].tolist() == chosen
            for j, t in enumerate(chosen):
                assert np.array_equal(raw(table[0, j // 16])[h, :, j % 16], before[table[0, t // 16]][h, :, t % 16])


def test_prompt_rows_beyond_32_bits():
    """Query and output arrays of more than 2^32 bytes and 2^31 elements: the last sequences against the same ones alone."""
    hq, hkv, d = 64, 8, 128
    lens = [128] * 2080
    n = sum(lens)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    assert n * hq * d > 1 << 31
    g = torch.Generator(device=DEV).manual_seed(7)
    q, k, v = (torch.randn((n, h, d), generator=g, device=DEV, dtype=torch.bfloat16) for h in (hq, hkv, hkv))
    out = torch.empty_like(q)
    with Pool(hq, hkv, d, BF16, 1) as p:
        torch.cuda.synchronize()
        pie.pie_prompt_attention(p.h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), off, len(lens), d ** -0.5)
        pie.pie_sync(p.h)
        part = slice(n - 3 * 128, n)
        q2, k2, v2 = (x[part].clone() for x in (q, k, v))
        alone = torch.empty_like(q2)
        torch.cuda.synchronize()
        pie.pie_prompt_attention(p.h, q2.data_ptr(), k2.data_ptr(), v2.data_ptr(), alone.data_ptr(), np.array([0, 128, 256, 384], np.int32), 3, d ** -0.5)
        pie.pie_sync(p.h)
    assert torch.equal(out[part], alone)
    bits = lambda x: real(x.view(torch.int16).cpu().numpy(), BF16)  # noqa: E731
    check_prompt(BF16, bits(alone[:128]), *oo.prompt_attention(bits(q2[:128]), bits(k2[:128]), bits(v2[:128]), np.array([0, 128], np.int32), d ** -0.5))
