"""The serving operators beside the paged cache, as cases that can be timed and compared: each in its plain form (elementary
torch operations in 32 bits) and as a user's program calls it in this package.

  rope     rotary positions with one to three axes (time, height, width) on q and k, and the write of the rotated k and of v
           into the paged cache: ``pie_set_rope`` + ``pie_rope_kv_write``
  prompt   causal attention over whole prompts, packed one after the other, grouped heads: ``pie_prompt_attention``
  weights  one layer's decode attention that also adds every cached token's attention weight to a running sum per
           (sequence, KV head, token): ``pie_decode_attention_weights``
  evict    per (sequence, KV head): keep the newest ``recent`` tokens and, of the older ones, those with the largest accumulated
           weights, and move their keys, values and weights to the front of a shorter sequence: ``pie_kv_evict``

Head counts and types are those of the package's own workloads (Llama-2-7B: 32 / 32 heads of 128, fp16; Llama-3-8B: 32 / 8 of
128, bf16; Llama-3-70B: 64 / 8 of 128, bf16; a small shape of 8 / 4 heads of 64).  Cache blocks are the package's slots:
[n_kv_heads][K, V][16 tokens][head_dim], 16-bit or E4M3 bytes.
"""
import math

import numpy as np
import torch

own = False

#: name -> (query heads, KV heads, head_dim, 16-bit type)
SHAPES = {"small": (8, 4, 64, "f16"), "mha": (32, 32, 128, "f16"), "gqa4": (32, 8, 128, "bf16"), "gqa8": (64, 8, 128, "bf16")}
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
K_SCALE, V_SCALE = 0.25, 0.5   # what a stored E4M3 byte is multiplied by, for keys and for values


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a decode step of a small batch: one new token per sequence, latency counts
        {"name": "rope decode 8", "op": "rope", "shape": "gqa4", "fp8": False, "seqs": 8, "tokens": 8, "start": 4100, "axes": 1,
         "rotary": 128, "adjacent": False, "packed": True, "far": 0},
        # a chunk of three prompts with images into an 8-bit cache, sliced out of the fused projection's output
        {"name": "rope chunk fp8", "op": "rope", "shape": "gqa4", "fp8": True, "seqs": 3, "tokens": 2045, "start": 37, "axes": 3,
         "rotary": 128, "adjacent": False, "packed": True, "far": 0},
        # a long video prompt, positions far out, half of the head rotated
        {"name": "rope video 16k", "op": "rope", "shape": "gqa8", "fp8": False, "seqs": 1, "tokens": 16411, "start": 0, "axes": 3,
         "rotary": 64, "adjacent": True, "packed": False, "far": 900001},
        # one short prompt alone: latency
        {"name": "prompt 45", "op": "prompt", "shape": "small", "seqs": 1, "longest": 45, "shortest": 45, "packed": False},
        # the prompts that a scheduler puts into one step: ragged, from one token up, sliced out of the fused projection
        {"name": "prompt ragged 16", "op": "prompt", "shape": "gqa4", "seqs": 16, "longest": 1500, "shortest": 1, "packed": True},
        # one long document
        {"name": "prompt 10007", "op": "prompt", "shape": "gqa4", "seqs": 1, "longest": 10007, "shortest": 10007, "packed": False},
        # one sequence alone: latency
        {"name": "weights 1 x 333", "op": "weights", "shape": "gqa4", "fp8": False, "seqs": 1, "longest": 333, "shortest": 333},
        # a batch over an 8-bit cache
        {"name": "weights 64 fp8", "op": "weights", "shape": "gqa4", "fp8": True, "seqs": 64, "longest": 2000, "shortest": 1},
        # a batch of longer contexts, one query head per KV head
        {"name": "weights 32 mha", "op": "weights", "shape": "mha", "fp8": False, "seqs": 32, "longest": 4000, "shortest": 500},
        # one short sequence halved
        {"name": "evict 700", "op": "evict", "shape": "small", "fp8": False, "seqs": 1, "longest": 700, "shortest": 700,
         "budget": 256, "recent": 64},
        # a ragged batch over an 8-bit cache: some sequences are within the budget already
        {"name": "evict 24 fp8", "op": "evict", "shape": "gqa4", "fp8": True, "seqs": 24, "longest": 3500, "shortest": 200,
         "budget": 999, "recent": 100},
        # a batch of long contexts cut to a quarter
        {"name": "evict 32 mha", "op": "evict", "shape": "mha", "fp8": False, "seqs": 32, "longest": 4096, "shortest": 3500,
         "budget": 1024, "recent": 512},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "prompt", "weights", "evict"])
    shape = rng.choice(sorted(SHAPES))
    hq, hkv, d, _ = SHAPES[shape]
    fp8 = d == 128 and rng.random() < 0.4
    if op == "rope":
        axes = rng.choice([1, 2, 3])
        return {"op": op, "shape": shape, "fp8": fp8, "seqs": rng.randint(1, 9), "tokens": _log_uniform(rng, 1, 12000), "start": rng.randint(0, 300),
                "axes": axes, "rotary": rng.choice([d, d // 2]), "adjacent": rng.random() < 0.5, "packed": rng.random() < 0.5,
                "far": rng.choice([0, rng.randint(1, 1 << 20)])}
    if op == "prompt":
        # the padded squares of the plain form stay below the long document's
        longest = _log_uniform(rng, 1, 6000)
        seqs = rng.randint(1, max(1, min(24, 40_000_000 * 32 // hq // (longest * longest))))
        return {"op": op, "shape": shape, "seqs": seqs, "longest": longest, "shortest": rng.randint(0, longest), "packed": rng.random() < 0.5}
    if op == "weights":
        longest = _log_uniform(rng, 1, 16000)
        seqs = rng.randint(1, max(1, min(96, 70_000 * 32 // hkv // longest)))
        return {"op": op, "shape": shape, "fp8": fp8, "seqs": seqs, "longest": longest, "shortest": rng.randint(0, longest)}
    longest = _log_uniform(rng, 2, 16000)
    seqs = rng.randint(1, max(1, min(48, 32_000 * 32 // hkv // longest)))
    budget = rng.randint(1, longest)
    return {"op": op, "shape": shape, "fp8": fp8, "seqs": seqs, "longest": longest, "shortest": rng.randint(0, longest), "budget": budget,
            "recent": rng.randint(0, budget)}


def _lengths(case):
    """The batch's lengths: the longest first, the others spread between the two ends (a function of the case alone)."""
    n, lo, hi = case["seqs"], case["shortest"], case["longest"]
    return [hi] + [lo + (hi - lo) * ((7919 * i) % 104729) // 104729 for i in range(1, n)]


def _frequencies(rotary):
    """1 / theta^(2 i / rotary), in double."""
    return 500000.0 ** (-np.arange(0, rotary, 2, dtype=np.float64) / rotary)


def _pair_axis(case):
    """Which axis turns which pair: a quarter of the pairs for the first of three axes and three eighths for each other one, in
    consecutive sections - or dealt out in turn where the pairs are adjacent elements."""
    pairs, axes = case["rotary"] // 2, case["axes"]
    if case["adjacent"]:
        return np.arange(pairs, dtype=np.int32) % axes
    cuts = {1: [pairs], 2: [pairs // 4, pairs], 3: [pairs // 4, pairs // 4 + 3 * pairs // 8, pairs]}[axes]
    return np.searchsorted(np.asarray(cuts), np.arange(pairs), side="right").astype(np.int32)


# -------------------------------------------------------------------------------------------------------------- prepare
class _Pool:
    """The package's handle over a cache that the program owns; it lives as long as the state."""

    def __init__(self, case, cache, max_seqs):
        from paper_2411_09317_b200 import binding
        hq, hkv, d, kind = SHAPES[case["shape"]]
        self.binding = binding
        stream = torch.cuda.current_stream().cuda_stream
        self.handle = binding.pie_pool_create(
            n_layers=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=binding.PIE_F16 if kind == "f16" else binding.PIE_BF16,
            n_logical_blocks=cache.shape[0], max_seqs=max(1, max_seqs), n_gpu_slots=cache.shape[0], n_host_slots=0, kv_fp8=int(case.get("fp8", False)),
            gpu_base=cache.data_ptr(), own_streams=0, compute_stream=stream, copy_in_stream=stream, copy_out_stream=stream)
        if case.get("fp8"):
            binding.pie_set_kv_scales(self.handle, K_SCALE, V_SCALE)
        ids = binding.pie_block_alloc(self.handle, cache.shape[0])
        _, slots = binding.pie_get_placement(self.handle, 1, cache.shape[0])
        assert np.array_equal(slots[0], ids)   # a block's slot is its own number: what the plain form goes by

    def __del__(self):
        if getattr(self, "handle", None):
            self.binding.pie_pool_destroy(self.handle)
            self.handle = None


def _cache(case, n_blocks, gen, filled):
    """Blocks of keys and values: 16-bit normal values (keys with a few strong channels, as trained keys have), or E4M3 codes."""
    hq, hkv, d, kind = SHAPES[case["shape"]]
    shape = (n_blocks, hkv, 2, 16, d)
    if not filled:
        if case["fp8"]:
            return torch.zeros(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        return torch.zeros(shape, dtype=TYPES[kind], device="cuda")
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    x[:, :, 0, :, : d // 16] *= 3.0
    if case["fp8"]:
        x[:, :, 0] /= K_SCALE
        x[:, :, 1] /= V_SCALE
        return x.to(torch.float8_e4m3fn)
    return x.to(TYPES[kind])


def _tables(lengths, gen, first=0):
    """Block ids of each sequence in scattered order, as [sequences][blocks of the longest], and the number of blocks."""
    blocks = [max(1, -(-n // 16)) for n in lengths]
    order = torch.randperm(sum(blocks), generator=gen, device="cuda").to(torch.int32) + first
    table = torch.zeros((len(blocks), max(blocks)), dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(blocks):
        table[s, :n] = order[at:at + n]
        at += n
    return table, at


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    hq, hkv, d, kind = SHAPES[case["shape"]]
    dtype = TYPES[kind]
    st = {"case": case, "scale": 1.0 / math.sqrt(d)}

    def fresh(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)

    def projected(n):
        """q, k, v of n tokens: slices of one projection's rows, or tensors of their own."""
        if case["packed"]:
            qkv = fresh(n, hq + 2 * hkv, d)
            return qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        return fresh(n, hq, d), fresh(n, hkv, d), fresh(n, hkv, d)

    if case["op"] == "rope":
        n, seqs, start = case["tokens"], case["seqs"], case["start"]
        share = [n // seqs + (1 if s < n % seqs else 0) for s in range(seqs)]
        table, n_blocks = _tables([start + c for c in share], gen)
        seq = torch.repeat_interleave(torch.arange(seqs, device="cuda"), torch.tensor(share, device="cuda"))
        first = torch.tensor([0] + share[:-1], device="cuda").cumsum(0)
        pos = start + torch.arange(n, device="cuda") - first[seq]
        # text: the cache position; images and video: a frame every 196 tokens, a grid of 14 x 14 in it
        far = case["far"] + int(torch.randint(0, 1000, (1,), generator=gen, device="cuda")) * (case["far"] > 0)
        along = [pos + far] if case["axes"] == 1 else [pos // 196 + far, pos % 196 // 14 + far, pos % 14 + far][: case["axes"]]
        st.update(table=table, seq=seq.to(torch.int32), pos=pos.to(torch.int32), positions=torch.stack(along).to(torch.int32).contiguous(),
                  frequencies=_frequencies(case["rotary"]), pair_axis=_pair_axis(case), cache=_cache(case, n_blocks, gen, False),
                  q_out=torch.empty((n, hq, d), dtype=dtype, device="cuda"), k_out=torch.empty((n, hkv, d), dtype=dtype, device="cuda"))
        st["q"], st["k"], st["v"] = projected(n)
        st["frequencies_dev"] = torch.from_numpy(st["frequencies"]).cuda()
        st["pair_axis_dev"] = torch.from_numpy(st["pair_axis"]).cuda().long()
        if own:
            st["pool"] = _Pool(case, st["cache"], seqs)
            st["pool"].binding.pie_set_rope(st["pool"].handle, case["rotary"], st["pair_axis"], st["frequencies"],
                                            adjacent=int(case["adjacent"]))
        return st

    lengths = _lengths(case)
    st["lengths"] = lengths
    if case["op"] == "prompt":
        n = sum(lengths)
        st["q"], st["k"], st["v"] = projected(n)
        st["offsets"] = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        st["out"] = torch.empty((n, hq, d), dtype=dtype, device="cuda")
        seq = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), torch.tensor(lengths, device="cuda"))
        st["seq"] = seq
        st["pos"] = torch.arange(n, device="cuda") - torch.from_numpy(st["offsets"]).cuda().long()[seq]
        if own:
            st["pool"] = _Pool(case, torch.zeros((1, hkv, 2, 16, d), dtype=dtype, device="cuda"), len(lengths))
        return st

    table, n_blocks = _tables(lengths, gen)
    st["table"], st["ctx"] = table, torch.tensor(lengths, dtype=torch.int32, device="cuda")
    width = max(lengths)
    if case["op"] == "weights":
        st["cache"] = _cache(case, n_blocks, gen, True)
        st["q"], st["out"] = fresh(len(lengths), hq, d), torch.empty((len(lengths), hq, d), dtype=dtype, device="cuda")
        st["sums"] = torch.rand((len(lengths), hkv, width + 3), generator=gen, device="cuda")   # what earlier steps have added
    else:
        # the destination: fresh blocks behind the source's (a shared prefix stays as it is)
        kept = [min(n, case["budget"]) for n in lengths]
        st["dst_table"], n_dst = _tables(kept, gen, first=n_blocks)
        cache = _cache(case, n_blocks + n_dst, gen, True)
        (cache.view(torch.uint8) if case["fp8"] else cache)[n_blocks:] = 0
        st["cache"], st["dst"] = cache, cache[n_blocks:]
        # accumulated weights: a few heavy tokens, a long tail
        st["sums"] = torch.exp(2.5 * torch.randn((len(lengths), hkv, width + 3), generator=gen, device="cuda") - 4.0)
        st["sums_out"] = torch.zeros((len(lengths), hkv, case["budget"]), device="cuda")
        st["kept"] = torch.full((len(lengths), hkv, case["budget"]), -1, dtype=torch.int32, device="cuda")
        st["new_ctx"] = torch.zeros(len(lengths), dtype=torch.int32, device="cuda")
    if own:
        st["pool"] = _Pool(case, st["cache"], len(lengths))
    return st


# ------------------------------------------------------------------------------------------------------------------ run
def run(st):
    if own:
        return {"rope": _own_rope, "prompt": _own_prompt, "weights": _own_weights, "evict": _own_evict}[st["case"]["op"]](st)
    return {"rope": _plain_rope, "prompt": _plain_prompt, "weights": _plain_weights, "evict": _plain_evict}[st["case"]["op"]](st)


def _own_rope(st):
    p = st["pool"]
    q, k, v = st["q"], st["k"], st["v"]
    p.binding.pie_rope_kv_write(p.handle, 0, q.data_ptr(), st["q_out"].data_ptr(), k.data_ptr(), st["k_out"].data_ptr(), v.data_ptr(),
                                st["positions"].data_ptr(), st["seq"].data_ptr(), st["pos"].data_ptr(), q.shape[0], st["table"].data_ptr(),
                                st["table"].shape[1], st["table"].shape[0], q_stride=q.stride(0), k_stride=k.stride(0), v_stride=v.stride(0))
    return {"q": st["q_out"], "k": st["k_out"], "cache": st["cache"]}


def _own_prompt(st):
    p = st["pool"]
    q, k, v = st["q"], st["k"], st["v"]
    p.binding.pie_prompt_attention(p.handle, q.data_ptr(), k.data_ptr(), v.data_ptr(), st["out"].data_ptr(), st["offsets"],
                                   len(st["lengths"]), st["scale"], q_stride=q.stride(0), k_stride=k.stride(0), v_stride=v.stride(0))
    return st["out"]


def _own_weights(st):
    p = st["pool"]
    p.binding.pie_decode_attention_weights(p.handle, 0, st["q"].data_ptr(), st["out"].data_ptr(), st["table"].data_ptr(),
                                           st["table"].shape[1], st["ctx"].data_ptr(), len(st["lengths"]), st["scale"],
                                           st["sums"].data_ptr(), st["sums"].shape[2])
    return {"out": st["out"], "weights": st["sums"]}


def _own_evict(st):
    p = st["pool"]
    p.binding.pie_kv_evict(p.handle, 0, st["table"].data_ptr(), st["table"].shape[1], st["ctx"].data_ptr(), len(st["lengths"]),
                           st["sums"].data_ptr(), st["sums"].shape[2], st["case"]["budget"], st["case"]["recent"],
                           dst_block_table_dev=st["dst_table"].data_ptr(), dst_max_blocks=st["dst_table"].shape[1],
                           weights_out=st["sums_out"].data_ptr(), weights_out_stride=st["sums_out"].shape[2],
                           new_lens_dev=st["new_ctx"].data_ptr(), kept_dev=st["kept"].data_ptr())
    return {"cache": st["dst"], "kept": st["kept"], "lengths": st["new_ctx"], "weights": st["sums_out"]}


def _plain_rope(st):
    case = st["case"]
    # angles in double: far positions lose their fraction in 32 bits
    angle = st["positions"].double()[st["pair_axis_dev"]].t() * st["frequencies_dev"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x):
        y = x.float()
        r, half = case["rotary"], case["rotary"] // 2
        a, b = (y[..., 0:r:2], y[..., 1:r:2]) if case["adjacent"] else (y[..., :half], y[..., half:r])
        a, b = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack([a, b], dim=-1).flatten(-2) if case["adjacent"] else torch.cat([a, b], dim=-1)
        return torch.cat([turned, y[..., r:]], dim=-1)

    q, k, v, cache = turn(st["q"]), turn(st["k"]), st["v"], st["cache"]
    block, row = st["table"][st["seq"].long(), st["pos"].long() // 16].long(), st["pos"].long() % 16
    if case["fp8"]:
        raw = cache.view(torch.uint8)
        raw[block, :, 0, row] = (k / K_SCALE).clamp(-448, 448).to(cache.dtype).view(torch.uint8)
        raw[block, :, 1, row] = (v.float() / V_SCALE).clamp(-448, 448).to(cache.dtype).view(torch.uint8)
    else:
        cache[block, :, 0, row] = k.to(cache.dtype)
        cache[block, :, 1, row] = v
    st["q_out"].copy_(q)
    st["k_out"].copy_(k)
    return {"q": st["q_out"], "k": st["k_out"], "cache": cache}


def _plain_prompt(st):
    hq, hkv, d, _ = SHAPES[st["case"]["shape"]]
    seqs, width = len(st["lengths"]), max(st["lengths"])
    if sum(st["lengths"]) == 0:
        return st["out"]

    def padded(x):
        y = torch.zeros((seqs, width, x.shape[1], d), device="cuda")
        y[st["seq"], st["pos"]] = x.float()
        return y

    q = padded(st["q"]).view(seqs, width, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, hq // hkv * width, d)
    k, v = (padded(st[n]).permute(0, 2, 1, 3) for n in "kv")
    at = torch.arange(width, device="cuda")
    s = torch.matmul(q, k.transpose(2, 3)).mul_(st["scale"]).view(seqs, hkv, hq // hkv, width, width)
    s.masked_fill_(at[None, :] > at[:, None], -math.inf)     # (columns behind a sequence's end are behind its rows too)
    s = s.sub_(s.amax(-1, keepdim=True)).exp_()
    out = torch.matmul(s.div_(s.sum(-1, keepdim=True)).view(seqs, hkv, hq // hkv * width, width), v)
    out = out.view(seqs, hkv, hq // hkv, width, d).permute(0, 3, 1, 2, 4).reshape(seqs, width, hq, d)
    st["out"].copy_(out[st["seq"], st["pos"]])
    return st["out"]


def _blocks(cache, ids):
    """Blocks by number (8-bit ones are picked out as bytes)."""
    return cache.view(torch.uint8)[ids].view(cache.dtype) if cache.element_size() == 1 else cache[ids]


def _gathered(st, real):
    """Keys and values [sequences][KV heads][tokens][head_dim] of the padded batch, read through the block table."""
    hq, hkv, d, _ = SHAPES[st["case"]["shape"]]
    x = _blocks(st["cache"], st["table"].long()).to(real)                  # [S][blocks][Hkv][2][16][D]
    x = x.permute(3, 0, 2, 1, 4, 5).reshape(2, x.shape[0], hkv, -1, d)
    if st["case"]["fp8"]:
        x[0] *= K_SCALE
        x[1] *= V_SCALE
    return x[0], x[1]


def _plain_weights(st):
    hq, hkv, d, _ = SHAPES[st["case"]["shape"]]
    seqs, width = len(st["lengths"]), max(st["lengths"])
    k, v = _gathered(st, torch.float32)
    there = (torch.arange(k.shape[2], device="cuda")[None] < st["ctx"][:, None])[:, None, None]
    q = st["q"].float().view(seqs, hkv, hq // hkv, d)
    s = (torch.matmul(q, k.transpose(2, 3)) * st["scale"]).masked_fill(~there, -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.where(there, (s - top).exp(), 0.0)
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    st["out"].copy_(torch.matmul(p, v).view(seqs, hq, d))
    st["sums"][:, :, :width] += p.sum(2)[:, :, :width]
    return {"out": st["out"], "weights": st["sums"]}


def _plain_evict(st):
    case = st["case"]
    hq, hkv, d, _ = SHAPES[case["shape"]]
    budget, recent = case["budget"], case["recent"]
    width = max(st["lengths"])
    ctx = st["ctx"].long()[:, None, None]
    at = torch.arange(width, device="cuda")[None, None]
    w = st["sums"][:, :, :width]
    # 0: a token that stays whatever its weight; 1: one that competes; 2: none
    fixed = (at < ctx) & ((at >= ctx - recent) | (ctx <= budget))
    key = torch.where(fixed, math.inf, torch.where(at < ctx, w, -math.inf))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices      # ties: the lowest position first
    new = torch.minimum(ctx, torch.tensor(budget, device="cuda"))
    first = order[:, :, :budget]
    n = min(budget, width)
    place = torch.arange(n, device="cuda")[None, None]
    kept = torch.sort(torch.where(place < new, first, width), dim=-1).values
    valid = place < new
    kept = torch.where(valid, kept, 0)
    s = torch.arange(len(st["lengths"]), device="cuda")[:, None, None].expand_as(kept)
    h = torch.arange(hkv, device="cuda")[None, :, None].expand_as(kept)
    src = st["table"].long()[s, kept // 16]
    raw = st["cache"].view(torch.uint8) if case["fp8"] else st["cache"]
    rows = raw[src, h, :, kept % 16]                                           # [S][Hkv][n][2][D]
    dst = st["dst_table"].long()[s, (place // 16).clamp(max=st["dst_table"].shape[1] - 1).expand_as(kept)]
    put = valid.expand_as(kept)
    raw[dst[put], h[put], :, (place % 16).expand_as(kept)[put]] = rows[put]
    st["sums_out"][:, :, :n] = torch.where(valid, torch.gather(w, 2, kept), st["sums_out"][:, :, :n])
    st["kept"].fill_(-1)
    st["kept"][:, :, :n] = torch.where(valid, kept, -1).to(torch.int32)
    st["new_ctx"].copy_(new[:, 0, 0])
    return {"cache": st["dst"], "kept": st["kept"], "lengths": st["new_ctx"], "weights": st["sums_out"]}


# ----------------------------------------------------------------------------------------------------------------- work
def work(case):
    hq, hkv, d, _ = SHAPES[case["shape"]]
    element = 1 if case.get("fp8") else 2
    if case["op"] == "rope":
        n = case["tokens"]
        moved = 2 * n * d * (2 * hq + 3 * hkv) + n * d * 2 * hkv * element
        return {"bytes": moved + 4 * n * (case["axes"] + 2), "flops": 3 * n * case["rotary"] * (hq + hkv)}
    lengths = _lengths(case)
    if case["op"] == "prompt":
        return {"bytes": 2 * sum(lengths) * d * (2 * hq + 2 * hkv), "flops": sum(2 * n * (n + 1) * hq * d for n in lengths)}
    if case["op"] == "weights":
        t = sum(lengths)
        return {"bytes": t * hkv * 2 * d * element + 2 * 4 * t * hkv + 4 * len(lengths) * hq * d + 4 * (t // 16 + len(lengths)), "flops": 4 * t * hq * d}
    kept = sum(min(n, case["budget"]) for n in lengths)
    return {"bytes": 4 * sum(lengths) * hkv + kept * hkv * (2 * 2 * d * element + 4 + 4), "flops": sum(lengths) * hkv}


# ---------------------------------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The definitions in double, sequence by sequence and head by head."""
    return {"rope": _exact_rope, "prompt": _exact_prompt, "weights": _exact_weights, "evict": _exact_evict}[case["op"]](case, seed)


def _inputs(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _exact_rope(case, seed):
    st = _inputs(case, seed)
    half = case["rotary"] // 2
    turned = {}
    for name in "qk":
        y = st[name].double().clone()
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if case["adjacent"] else (i, half + i)
            angle = (st["positions"][int(st["pair_axis"][i])].double() * float(st["frequencies"][i]))[:, None]
            x = torch.complex(y[:, :, a], y[:, :, b]) * torch.polar(torch.ones_like(angle), angle)
            y[:, :, a], y[:, :, b] = x.real, x.imag
        turned[name] = y
    cache = st["cache"].double()
    for s in range(case["seqs"]):
        mine = (st["seq"] == s).nonzero()[:, 0]
        where = st["pos"][mine].long()
        ids = st["table"][s].long()[where // 16]
        scales = (K_SCALE, V_SCALE) if case["fp8"] else (1.0, 1.0)
        cache[ids, :, 0, where % 16] = turned["k"][mine] / scales[0]
        cache[ids, :, 1, where % 16] = st["v"][mine].double() / scales[1]
    return {"q": turned["q"], "k": turned["k"], "cache": cache}


def _exact_prompt(case, seed):
    st = _inputs(case, seed)
    hq, hkv, d, _ = SHAPES[case["shape"]]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(st["lengths"]):
        o = int(st["offsets"][s])
        hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
        for h in range(hq):
            q, k, v = st["q"][o:o + n, h].double(), st["k"][o:o + n, h * hkv // hq].double(), st["v"][o:o + n, h * hkv // hq].double()
            out[o:o + n, h] = torch.softmax((q @ k.t() * st["scale"]).masked_fill_(hidden, -math.inf), dim=-1) @ v
    return out


def _exact_weights(case, seed):
    st = _inputs(case, seed)
    hq, hkv, d, _ = SHAPES[case["shape"]]
    g = hq // hkv
    out, sums = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda"), st["sums"].double()
    scales = (K_SCALE, V_SCALE) if case["fp8"] else (1.0, 1.0)
    for s, n in enumerate(st["lengths"]):
        if n == 0:
            continue
        x = _blocks(st["cache"], st["table"][s, :-(-n // 16)].long()).double()   # [blocks][Hkv][2][16][D]
        k, v = (x[:, :, i].transpose(0, 1).reshape(hkv, -1, d)[:, :n] * scales[i] for i in (0, 1))
        p = torch.softmax(torch.einsum("hgd,htd->hgt", st["q"][s].double().view(hkv, g, d), k) * st["scale"], dim=-1)
        out[s] = torch.einsum("hgt,htd->hgd", p, v).reshape(hq, d)
        sums[s, :, :n] += p.sum(1)
    return {"out": out, "weights": sums}


def _exact_evict(case, seed):
    """Whole positions and moved values: chosen here by repeated comparison with the budget-th largest weight."""
    st = _inputs(case, seed)
    hq, hkv, d, _ = SHAPES[case["shape"]]
    budget, recent = case["budget"], case["recent"]
    sums = st["sums"].double().cpu().numpy()
    base = st["cache"].shape[0] - st["dst"].shape[0]
    src, out, w_out = st["cache"][:base], st["dst"].double(), st["sums_out"].double().cpu().numpy()
    kept = np.full(st["kept"].shape, -1, dtype=np.int32)
    for s, n in enumerate(st["lengths"]):
        m = min(n, budget)
        for h in range(hkv):
            chosen = np.arange(n)
            if n > budget:
                older, places = sums[s, h, :n - recent], budget - recent
                chosen = np.arange(0)
                if places:
                    edge = np.partition(older, len(older) - places)[len(older) - places]
                    above = np.nonzero(older > edge)[0]
                    chosen = np.concatenate([above, np.nonzero(older == edge)[0][:places - len(above)]])
                chosen = np.sort(np.concatenate([chosen, np.arange(n - recent, n)]))
            kept[s, h, :m] = chosen
            w_out[s, h, :m] = sums[s, h, chosen]
            c, to = torch.from_numpy(chosen).cuda(), torch.arange(m, device="cuda")
            block = _blocks(src[:, h], st["table"][s, c // 16].long())
            out[st["dst_table"][s, to // 16].long() - base, h, :, to % 16] = block[to, :, c % 16].double()
    return {"cache": out, "kept": torch.from_numpy(kept), "lengths": np.minimum(st["lengths"], budget).astype(np.int32), "weights": torch.from_numpy(w_out)}
