"""The 4-bit paged cache on the device against a plain 64-bit implementation (paged_reference.py): codes bit for bit, attention
within bounds derived from its arithmetic, and everything that is refused."""
import numpy as np
import pytest

import paged_reference as R
from paper_2408_08146_amd import KoalaError, PagedCache, alloc_paged_cache, rope_tables, tree_masks
from koala_synth.trees import make_tree

pytestmark = pytest.mark.gpu


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def rounded(x, bf16):
    """What of x [..] a tensor of the type holds, as float32 numpy."""
    import torch
    t = torch.from_numpy(np.asarray(x, np.float32))
    return t.to(torch.bfloat16).float().numpy() if bf16 else t.numpy()


def check_pools(t, ref):
    for name in ref.pool:
        got = t[name].cpu().numpy()
        assert (got == ref.pool[name]).all(), (name, np.argwhere(got != ref.pool[name])[:5])


# ------------------------------------------------------------------------------------------------- append and read
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("dh,heads,kv,page,batch,rows,lengths", [
    (128, 4, 4, 64, 1, 1, [0]), (128, 8, 2, 16, 3, 7, [0, 15, 33]), (64, 4, 1, 32, 2, 26, [5, 64]), (64, 3, 3, 16, 5, 17, [1, 2, 16, 31, 0]),
    (128, 1, 1, 256, 2, 70, [250, 3]), (128, 0, 2, 128, 2, 3, [127, 128])])
def test_append_writes_the_codes_of_the_definition(bf16, dh, heads, kv, page, batch, rows, lengths):
    import torch
    rng = np.random.default_rng(dh + rows)
    ref = R.Cache(rng, 2, batch, kv, page, dh, lengths, rows)
    cache, t, length = ref.device()
    cos, sin = rope_tables(max(lengths) + rows, dh)
    qkv = rounded(rng.standard_normal((batch, rows, heads + 2 * kv, dh)) * np.exp(rng.standard_normal((1, 1, 1, dh))), bf16)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = dev(qkv, dt)
    q_out = torch.full((batch, rows, heads, dh), 7.0, dtype=dt, device="cuda")
    cache.append(1, x[:, :, :heads] if heads else None, x[:, :, heads:heads + kv], x[:, :, heads + kv:], q_out if heads else None, cos, sin)
    c, s = cos.cpu().numpy(), sin.cpu().numpy()
    ref.append(1, qkv[:, :, heads:heads + kv], qkv[:, :, heads + kv:], c[:, None], s[:, None])
    check_pools(t, ref)
    assert (length.cpu().numpy() == ref.len).all()
    for b in range(batch):
        for i in range(rows):
            want = R.rotate(qkv[b, i, :heads], c[lengths[b] + i], s[lengths[b] + i])
            assert (q_out[b, i].float().cpu().numpy() == rounded(want, bf16)).all()
    # and read back, one layer and all
    start = np.maximum(np.array(lengths, np.int32) - 2, 0)
    for layer in (1, None):
        for out_dt in (torch.bfloat16, torch.float32):
            shape = (batch, rows, kv, dh) if layer is not None else (2, batch, rows, kv, dh)
            k, v = (torch.empty(shape, dtype=out_dt, device="cuda") for _ in range(2))
            cache.read(layer, dev(start), k, v)
            for name, out in (("k", k), ("v", v)):
                got = out.double().cpu().numpy().reshape(-1, batch, rows, kv, dh)
                for li, l in enumerate([layer] if layer is not None else [0, 1]):
                    for b in range(batch):
                        assert (got[li, b] == ref.values(name, l, b, start[b], rows)).all()


def test_append_tree_depths_and_padding():
    import torch
    rng = np.random.default_rng(3)
    tree = make_tree([3, 2], [1, 3, 4])
    depth = [0]
    for p in tree.parent[1:]:
        depth.append(depth[p] + 1)
    lengths, n_new = [30, 0, 7], [8, 0, 3]
    ref = R.Cache(rng, 1, 3, 2, 16, 128, lengths, 8)
    cache, t, _ = ref.device()
    cos, sin = rope_tables(40, 128)
    k, v = (rng.standard_normal((3, 8, 2, 128)).astype(np.float32) for _ in range(2))
    q = torch.randn(3, 8, 4, 128, device="cuda")
    q_out = torch.full_like(q, 7.0)
    cache.append(0, q, dev(k), dev(v), q_out, cos, sin, depth=dev(np.array(depth, np.int32)), n_new=dev(np.array(n_new, np.int32)))
    ref.append(0, k, v, cos.cpu().numpy()[:, None], sin.cpu().numpy()[:, None], depth, n_new)
    check_pools(t, ref)
    got = q_out.cpu().numpy()
    for b in range(3):
        for i in range(8):
            want = R.rotate(q[b, i].cpu().numpy(), cos[lengths[b] + depth[i]].cpu().numpy(), sin[lengths[b] + depth[i]].cpu().numpy())
            assert (got[b, i] == (want if i < n_new[b] else 7.0)).all()


def test_append_rounds_ties_extremes_and_values_that_are_not_finite_as_defined():
    rng = np.random.default_rng(4)
    special = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0, -0.0, 6.0, 7.0, 7.0000005, 7.5, 8.0, 1e-30, 1e-38, 1e-45, 3e38, 2.0 ** -98, 2.0 ** -100], np.float32)
    v = np.zeros((1, 64, 1, 64), np.float32)
    for i in range(64):
        v[0, i, 0] = rng.choice(special[:12 if i < 32 else 20], 64) * rng.choice([-1, 1], 64) * (np.float32(2.0) ** rng.integers(-6, 6) if i < 32 else 1)
    v[0, 60, 0, 5], v[0, 61, 0, 40], v[0, 62, 0, 0], v[0, 63] = np.inf, np.nan, -np.inf, 0
    k = v[:, ::-1].copy()
    ref = R.Cache(rng, 1, 1, 1, 16, 64, [0], 64)
    cache, t, _ = ref.device()
    cos, sin = rope_tables(64, 64)
    cos, sin = cos * 0 + 1, sin * 0      # turned by nothing, the keys' codes are those of the values given
    cache.append(0, None, dev(k), dev(v), None, cos, sin)
    with np.errstate(all="ignore"):
        ref.append(0, k, v, cos.cpu().numpy()[:, None], sin.cpu().numpy()[:, None])
    check_pools(t, ref)


def test_rows_without_a_place_are_left_out():
    """Positions past the rotary table, slots past the page table, page numbers outside the pool and negative lengths."""
    import torch
    rng = np.random.default_rng(5)
    ref = R.Cache(rng, 1, 4, 1, 16, 64, [30, 5, 0, 10], 2, shuffle=False)
    ref.table = ref.table[:, :2].copy()          # 32 slots each
    ref.table[1] = [-1, 1000]
    ref.len[2] = -3
    cache, t, _ = ref.device()
    cos, sin = rope_tables(12, 64)               # positions 0 .. 11
    k, v = (rng.standard_normal((4, 4, 1, 64)).astype(np.float32) for _ in range(2))
    cache.append(0, None, dev(k), dev(v), None, cos, sin)
    c, s = cos.cpu().numpy(), sin.cpu().numpy()
    for i in range(2):                           # only sequence 3, positions 10 and 11, has a place
        for name, x in (("k", R.rotate(k[3, i], c[10 + i], s[10 + i])), ("v", v[3, i])):
            code, scale = R.encode(x)
            ref.put(name, 0, 3, 10 + i, code)
            ref.put(name + "_scale", 0, 3, 10 + i, scale)
    check_pools(t, ref)
    ko, vo = (torch.full((4, 3, 1, 64), 7.0, device="cuda") for _ in range(2))
    cache.read(0, dev(np.array([31, 0, 2 ** 31 - 1, -2], np.int32)), ko, vo)
    got = ko.double().cpu().numpy()
    assert (got[0, 0] == ref.values("k", 0, 0, 31, 1)[0]).all() and not got[0, 1:].any() and not got[1].any() and not got[2].any()
    assert not got[3, :2].any() and (got[3, 2] == ref.values("k", 0, 3, 0, 1)[0]).all()


# ------------------------------------------------------------------------------------------------- attention
def bound(ref, layer, q, scale, bf16):
    """Largest error of an output element, a bfloat16 output's own rounding apart.  fp32: every sum, product and power of two rounds at 2^-24 of its terms; scores are sums
    of dh terms (their rounding moves weights by 2 dh 2^-24 sum |q k| scale at most, counted once a term and twice for numerator and
    denominator), outputs sums over the keys, whose rounding grows with the 32-key steps that follow one another.  bfloat16:
    a probability's rounding to 11 bits is 2^-12 of it at most."""
    eps = 2.0 ** -24
    k = np.nan_to_num(R.decode(ref.pool["k"][layer], ref.pool["k_scale"][layer]))
    v = np.nan_to_num(R.decode(ref.pool["v"][layer], ref.pool["v_scale"][layer]))
    s_abs = np.abs(q).sum(-1).max() * np.abs(k).max() * scale
    n = max(ref.len.max(), 0) + q.shape[1]
    rel = 2 * q.shape[-1] * eps * s_abs + (n / 32 + 64) * eps + (2.0 ** -12 if bf16 else 0)
    return rel * np.abs(v).max()


def agrees(ref, layer, q, scale, bf16, got, want):
    """fp32: within the bound of the 64-bit value; bfloat16: a rounding of some number within it (rounding keeps order)."""
    tol = bound(ref, layer, q, scale, bf16)
    lo, hi = (rounded(want - tol, bf16).astype(np.float64), rounded(want + tol, bf16).astype(np.float64)) if bf16 else (want - tol, want + tol)
    return ((lo <= got) & (got <= hi)) | (np.isnan(got) & np.isnan(want))


def causal(batch, T):
    return [[[j <= i for j in range(T)] for i in range(T)]] * batch


def run_attend(ref, q, bf16, mask=None, scale=None, max_len=0, layer=0, strided=False):
    import torch
    cache, t, _ = ref.device()
    x = dev(q, torch.bfloat16 if bf16 else torch.float32)
    if strided:     # rows inside wider ones
        wide = torch.full((*x.shape[:2], x.shape[2] + 3, x.shape[3]), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, :, 1:1 + x.shape[2]] = x
        x = wide[:, :, 1:1 + x.shape[2]]
    out = torch.full(q.shape, 7.0, dtype=x.dtype, device="cuda")
    cache.attend(layer, x, out, mask=mask, scale=scale, max_len=max_len)
    check_pools(t, ref)
    return out.double().cpu().numpy()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("dh,heads,kv,page,rows,lengths", [
    (128, 2, 2, 16, 1, [0]), (128, 2, 2, 16, 1, [1]), (128, 4, 2, 16, 1, [15, 16, 31, 32]), (64, 8, 1, 64, 1, [700, 1, 33]),
    (128, 2, 1, 32, 16, [97]), (128, 1, 1, 16, 17, [40, 3]), (64, 6, 2, 128, 26, [300]), (128, 8, 1, 64, 33, [129, 64]),
    (128, 1, 1, 256, 64, [5, 260]), (64, 2, 2, 16, 64, [1000]), (128, 4, 4, 64, 3, [2500]), (64, 40, 8, 32, 2, [61, 62, 63, 64, 65, 66, 67]),
    (128, 16, 1, 64, 60, [90]), (64, 64, 1, 16, 1, [257])])
def test_attention_of_causal_rows(bf16, dh, heads, kv, page, rows, lengths):
    rng = np.random.default_rng(dh + heads + rows)
    ref = R.Cache(rng, 2, len(lengths), kv, page, dh, lengths, rows)
    q = rounded(rng.standard_normal((len(lengths), rows, heads, dh)), bf16).astype(np.float64)
    scale = dh ** -0.5
    want = ref.attend(1, q, causal(len(lengths), rows), scale)
    got = run_attend(ref, q, bf16, layer=1, strided=rows % 2 == 1)
    assert agrees(ref, 1, q, scale, bf16, got, want).all()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("topk,widths,lengths,per_seq", [([2, 2], [1, 2, 4], [64], False), ([4, 2, 2, 1, 1], [1, 4, 8, 6, 4, 3], [100, 37], False),
                                                         ([10, 5, 3, 2], [1, 10, 20, 18, 15], [7, 0, 250], True)])
def test_attention_of_trees(bf16, topk, widths, lengths, per_seq):
    tree = make_tree(topk, widths)
    T, B = tree.n_nodes, len(lengths)
    rng = np.random.default_rng(T)
    ref = R.Cache(rng, 1, B, 2, 32, 128, lengths, T)
    q = rounded(rng.standard_normal((B, T, 4, 128)), bf16).astype(np.float64)
    mask = tree_masks(tree)
    bits = [[int(m) >> j & 1 for j in range(T)] for m in mask.tolist()]
    want = ref.attend(0, q, [bits] * B, 0.1)
    got = run_attend(ref, q, bf16, mask=mask[None].expand(B, T).contiguous() if per_seq else mask, scale=0.1)
    assert agrees(ref, 0, q, 0.1, bf16, got, want).all()


@pytest.mark.parametrize("bf16", [True, False])
def test_rows_whose_mask_leaves_nothing_and_masks_of_any_form(bf16):
    """Random masks, some rows seeing nothing (with a context and without), bits past the rows set; a masked slot never counts."""
    rng = np.random.default_rng(8)
    T, lengths = 37, [0, 70, 0]
    ref = R.Cache(rng, 1, 3, 2, 16, 64, lengths, T)
    q = rounded(rng.standard_normal((3, T, 2, 64)), bf16).astype(np.float64)
    bits = rng.integers(0, 2, (3, T, T)).astype(bool)
    bits[0, 5] = bits[1, 6] = bits[2, :] = False
    words = [[sum(1 << j for j in range(T) if bits[b, i, j]) | (1 << 63) | (1 << T) for i in range(T)] for b in range(3)]
    mask = dev(np.array(words, np.uint64).view(np.int64))
    want = ref.attend(0, q, bits, 0.125)
    got = run_attend(ref, q, bf16, mask=mask, scale=0.125)
    assert not got[0, 5].any() and not got[2].any()
    assert agrees(ref, 0, q, 0.125, bf16, got, want).all()


@pytest.mark.parametrize("bf16", [True, False])
def test_not_a_number_reaches_the_rows_that_see_it_and_no_other(bf16):
    rng = np.random.default_rng(9)
    T, C = 20, 50
    ref = R.Cache(rng, 1, 1, 1, 16, 128, [C], T)
    bits = np.tril(np.ones((T, T), bool))
    bits[12:, 4] = bits[9, 3] = False
    ref.put("v_scale", 0, 0, C + 4, np.array([[127, 255, 127, 127]], np.uint8))      # a block of a value: rows 4 .. 11
    ref.put("k_scale", 0, 0, C + 15, np.array([[255, 127, 127, 127]], np.uint8))     # a key: rows 15 ..
    # slots past the end hold anything, not-a-number too
    for s in range(C + T, 80):
        ref.put("v_scale", 0, 0, s, np.full((1, 4), 255, np.uint8))
        ref.put("k_scale", 0, 0, s, np.full((1, 4), 255, np.uint8))
    q = rounded(rng.standard_normal((1, T, 2, 128)), bf16).astype(np.float64)
    words = [sum(1 << j for j in range(T) if bits[i, j]) for i in range(T)]
    got = run_attend(ref, q, bf16, mask=dev(np.array(words, np.uint64).view(np.int64)))
    want = ref.attend(0, q, [bits], 128 ** -0.5)
    assert np.isnan(want[0, 4:12, :, 32:64]).all() and not np.isnan(want[0, 4:12, :, :32]).any() and np.isnan(want[0, 15:]).all()
    assert (np.isnan(got) == np.isnan(want)).all()
    assert agrees(ref, 0, q, 128 ** -0.5, bf16, got, want).all()
    # in the context every row sees it
    ref.put("v_scale", 0, 0, 3, np.array([[255, 127, 127, 127]], np.uint8))
    got = run_attend(ref, q, bf16, mask=dev(np.array(words, np.uint64).view(np.int64)))
    assert np.isnan(got[..., :32]).all()


def test_a_dominant_late_key_and_scores_far_apart():
    """The running maximum moves at the end of a long context; weights underflow on both sides of it."""
    rng = np.random.default_rng(10)
    ref = R.Cache(rng, 1, 1, 1, 64, 64, [1500], 2)
    q = rounded(rng.standard_normal((1, 2, 1, 64)) * 20, False).astype(np.float64)
    code, s = R.encode(np.sign(q[0, 0]).astype(np.float32) * 6)
    ref.put("k", 0, 0, 1400, code)
    ref.put("k_scale", 0, 0, 1400, s + 1)
    want = ref.attend(0, q, causal(1, 2), 0.125)
    got = run_attend(ref, q, False, scale=0.125)
    assert agrees(ref, 0, q, 0.125, False, got, want).all()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("lo,hi", [(27, 60), (95, 112), (130, 150), (200, 230), (27, 230)])
def test_values_of_any_magnitude(bf16, lo, hi):
    """Exponents far outside fp16's range, all of them or some among others; every 32 dimensions are compared on their own scale."""
    rng = np.random.default_rng(lo + hi)
    for rows in (3, 20):
        ref = R.Cache(rng, 1, 2, 1, 16, 128, [150, 10], rows)
        e = rng.integers(lo, hi, ref.pool["v_scale"].shape[-1])          # a block of the head is of one magnitude, give or take
        ref.pool["v_scale"][:] = np.clip(e + rng.integers(-2, 3, ref.pool["v_scale"].shape), 27, 250)
        q = rounded(rng.standard_normal((2, rows, 2, 128)), bf16).astype(np.float64)
        want = ref.attend(0, q, causal(2, rows), 0.09)
        got = run_attend(ref, q, bf16, scale=0.09)
        full = ref.pool["v"], ref.pool["v_scale"]
        for block in range(4):
            d = slice(32 * block, 32 * block + 32)
            ref.pool["v"], ref.pool["v_scale"] = full[0][..., 16 * block:16 * block + 16], full[1][..., block:block + 1]
            assert agrees(ref, 0, q, 0.09, bf16, got[..., d], want[..., d]).all(), (rows, block)
        ref.pool["v"], ref.pool["v_scale"] = full


@pytest.mark.parametrize("max_len", [1, 31, 32, 33, 64, 100, 1000])
def test_slots_at_and_past_max_len_are_not_read(max_len):
    rng = np.random.default_rng(11)
    ref = R.Cache(rng, 1, 2, 1, 16, 64, [90, 20], 5)
    for s in range(max_len, 95):
        if s < 95:
            ref.put("v_scale", 0, 0, s, np.full((1, 2), 255, np.uint8))
    q = rng.standard_normal((2, 5, 1, 64)).astype(np.float32).astype(np.float64)
    want = ref.attend(0, q, causal(2, 5), 0.125, max_len=max_len)
    got = run_attend(ref, q, False, scale=0.125, max_len=max_len)
    assert agrees(ref, 0, q, 0.125, False, got, want).all()


def test_more_sequences_than_a_wave_has_lanes():
    rng = np.random.default_rng(12)
    lengths = [int(v) for v in rng.integers(0, 90, 150)]
    ref = R.Cache(rng, 1, 150, 1, 16, 64, lengths, 2)
    q = rng.standard_normal((150, 2, 2, 64)).astype(np.float32).astype(np.float64)
    want = ref.attend(0, q, causal(150, 2), 0.125)
    got = run_attend(ref, q, False, scale=0.125)
    assert agrees(ref, 0, q, 0.125, False, got, want).all()


def test_page_numbers_whose_bytes_pass_32_bits():
    """A pool of 4.4 GB of keys: the sequence's pages lie at its end."""
    import torch
    page, kv, dh = 256, 8, 128
    n = 34000
    rng = np.random.default_rng(13)
    pools = alloc_paged_cache(1, n, page, kv, dh)
    assert pools["k"].numel() > 2 ** 32
    table = torch.tensor([[n - 1, n - 3]], dtype=torch.int32, device="cuda")
    length = torch.tensor([300], dtype=torch.int32, device="cuda")
    cache = PagedCache(pools["k"], pools["v"], pools["k_scale"], pools["v_scale"], table, length)
    small = R.Cache(rng, 1, 1, kv, page, dh, [300], 4, shuffle=False)
    for name in small.pool:
        for i, p in enumerate((n - 1, n - 3)):
            pools[name][0, p] = dev(small.pool[name][0, i])
    cos, sin = rope_tables(310, dh)
    k, v = (rng.standard_normal((1, 4, kv, dh)).astype(np.float32) for _ in range(2))
    cache.append(0, None, dev(k), dev(v), None, cos, sin)
    small.append(0, k, v, cos.cpu().numpy()[:, None], sin.cpu().numpy()[:, None])
    q = rng.standard_normal((1, 4, kv, dh)).astype(np.float32).astype(np.float64)
    out = torch.empty(q.shape, device="cuda")
    cache.attend(0, dev(q, torch.float32), out)
    want = small.attend(0, q, causal(1, 4), dh ** -0.5)
    assert agrees(small, 0, q, dh ** -0.5, False, out.double().cpu().numpy(), want).all()
    cache.commit(dev(np.array([2], np.int32)), dev(np.array([[0, 2, 3]], np.int32)))
    small.commit([2], [[0, 2, 3]])
    ko, vo = (torch.empty(1, 304, kv, dh, device="cuda") for _ in range(2))
    cache.read(0, None, ko, vo)
    assert (ko[0].double().cpu().numpy() == small.values("k", 0, 0, 0, 304)).all()
    assert (vo[0].double().cpu().numpy() == small.values("v", 0, 0, 0, 304)).all() and length.item() == 303


def test_attention_is_the_same_twice_and_on_another_stream():
    import torch
    rng = np.random.default_rng(14)
    ref = R.Cache(rng, 1, 3, 2, 32, 128, [900, 10, 333], 5)
    cache, _, _ = ref.device()
    q = torch.randn(3, 5, 4, 128, device="cuda").bfloat16()
    a, b, c = (torch.empty_like(q) for _ in range(3))
    cache.attend(0, q, a)
    cache.attend(0, q, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache.attend(0, q, c, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, b) and torch.equal(a, c)
    assert len(cache._workspaces._by_stream) == 2


# ------------------------------------------------------------------------------------------------- commit, graphs
@pytest.mark.parametrize("dh,in_place", [(128, True), (64, False)])
def test_commit_moves_the_accepted_rows_in_every_layer(dh, in_place):
    import torch
    rng = np.random.default_rng(15)
    lengths = [0, 13, 30, 64, 5]
    path = np.array([[0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10], [0, 1, 4, 5, 20, -1, -1, -1, -1, -1, -1], [0] + [-1] * 10,
                     [0, 7, 8, 9, 10, 11, 12, 13, 14, 15, 39], [0, 2, 3, 4, 5, 6, 7, 8, 9, 30, -1]], np.int32)
    accept = np.array([10, 4, 0, 10, 9], np.int32)
    ref = R.Cache(rng, 3, 5, 2, 16, dh, lengths, 40)
    cache, t, length = ref.device()
    new_len = None if in_place else torch.empty(5, dtype=torch.int32, device="cuda")
    cache.commit(dev(accept), dev(path), new_len=new_len)
    before = ref.len.copy()
    ref.commit(accept.tolist(), path.tolist())
    check_pools(t, ref)
    assert (length.cpu().numpy() == (ref.len if in_place else before)).all()
    if not in_place:
        assert (new_len.cpu().numpy() == ref.len).all()


def test_an_iteration_captured_in_a_graph_replays():
    """Append, attend and commit of a growing sequence: every replay against the eager calls on a second cache."""
    import torch
    rng = np.random.default_rng(16)
    ref = R.Cache(rng, 1, 2, 2, 16, 64, [3, 40], 60)
    caches = [ref.device() for _ in range(2)]
    cos, sin = rope_tables(120, 64)
    qkv = torch.randn(2, 4, 8, 64, device="cuda")
    qo, out = torch.zeros(2, 2, 4, 4, 64, device="cuda"), torch.zeros(2, 2, 4, 4, 64, device="cuda")
    accept, path = dev(np.array([2, 0], np.int32)), dev(np.array([[0, 2, 3], [0, -1, -1]], np.int32))

    def step(i):
        c = caches[i][0]
        c.append(0, qkv[:, :, :4], qkv[:, :, 4:6], qkv[:, :, 6:], qo[i], cos, sin)
        c.attend(0, qo[i], out[i])
        c.commit(accept, path)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(0)
    torch.cuda.current_stream().wait_stream(side)
    step(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(0)
    for i in range(4):
        qkv.copy_(torch.randn_like(qkv))
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1]) and torch.equal(caches[0][2], caches[1][2]), i
        for name in ref.pool:
            assert torch.equal(caches[0][1][name], caches[1][1][name])


# ------------------------------------------------------------------------------------------------- refusals
def status(call):
    try:
        call()
    except KoalaError as e:
        return e.status
    return 0


def test_what_is_refused():
    import torch
    pools = alloc_paged_cache(2, 4, 16, 2, 64)
    for p in pools.values():
        p.zero_()
    table, length = torch.zeros(3, 4, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    make = lambda pool=pools, t=table, n=length: PagedCache(pool["k"], pool["v"], pool["k_scale"], pool["v_scale"], t, n)
    c = make()
    SHAPE, ALIGN, UNSUP, WS = -2, -3, -5, -6
    assert status(lambda: make(t=table.long())) == UNSUP and status(lambda: make(n=length[:2])) == SHAPE
    assert status(lambda: make(pool=dict(pools, v=pools["k"][:1]))) == SHAPE
    assert status(lambda: make(pool=dict(pools, k_scale=pools["v"]))) == SHAPE
    odd = alloc_paged_cache(1, 4, 24, 2, 64)
    assert status(lambda: make(odd).read(0, None, torch.empty(1, 1, 2, 64, device="cuda"), torch.empty(1, 1, 2, 64, device="cuda"))) == UNSUP
    assert status(lambda: make(alloc_paged_cache(1, 4, 16, 2, 32))) == UNSUP
    f = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    cos, sin = rope_tables(64, 64)
    k = f(3, 2, 2, 64)
    ok = dict(layer=0, q=f(3, 2, 4, 64), k=k, v=f(3, 2, 2, 64), q_out=f(3, 2, 4, 64), rope_cos=cos, rope_sin=sin)
    app = lambda **o: status(lambda: c.append(**dict(ok, **o)))
    assert app() == 0
    assert app(layer=2) == SHAPE and app(layer=-1) == SHAPE
    assert app(k=f(4, 2, 2, 64), v=f(4, 2, 2, 64), q=None, q_out=None) == SHAPE          # more sequences than the cache has
    assert app(v=f(3, 2, 2, 64, dt=torch.bfloat16)) == SHAPE and app(v=f(3, 2, 1, 64)) == SHAPE
    assert app(q=f(3, 2, 4, 64, dt=torch.bfloat16)) == UNSUP and app(k=f(3, 2, 2, 64, dt=torch.float16), v=f(3, 2, 2, 64, dt=torch.float16)) == UNSUP
    assert app(rope_sin=sin[:5]) == SHAPE and app(n_new=torch.zeros(2, dtype=torch.int32, device="cuda")) == SHAPE
    assert app(depth=torch.zeros(2, dtype=torch.int64, device="cuda")) == UNSUP
    assert app(q_out=f(3, 2, 4, 65)[..., :64]) == SHAPE
    assert app(k=f(3, 2, 2, 64).expand(3, 2, 2, 64)[:, :1].expand(3, 2, 2, 64)) == SHAPE  # rows on top of each other
    off = f(3 * 2 * 2 * 64 + 1)[1:].view(3, 2, 2, 64)
    assert app(k=off) == ALIGN
    q, out = f(3, 2, 4, 64), f(3, 2, 4, 64)
    att = lambda *a, **o: status(lambda: c.attend(*a, **o))
    assert att(0, q, out) == 0
    assert att(0, f(3, 65, 4, 64), f(3, 65, 4, 64)) == SHAPE and att(0, f(3, 2, 3, 64), f(3, 2, 3, 64)) == SHAPE
    assert att(0, q, f(3, 2, 4, 64, dt=torch.bfloat16)) == UNSUP and att(0, q, out, scale=0.0) == SHAPE and att(0, q, out, scale=float("nan")) == SHAPE
    assert att(0, q, out, scale=float("inf")) == SHAPE and att(0, q, out, max_len=-1) == SHAPE and att(5, q, out) == SHAPE
    assert att(0, q, out, mask=torch.zeros(3, dtype=torch.int64, device="cuda")) == SHAPE
    assert att(0, f(3, 2, 4, 128), f(3, 2, 4, 128)) == SHAPE
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    com = lambda *a, **o: status(lambda: c.commit(*a, **o))
    assert com(i32(4), i32(4, 3)) == SHAPE and com(i32(2), i32(3, 3)) == SHAPE and com(i32(2), i32(2, 3).long()) == UNSUP
    assert com(i32(2), i32(2, 3), new_len=i32(3)) == SHAPE
    rd = lambda *a: status(lambda: c.read(*a))
    assert rd(0, None, f(3, 1, 2, 64), f(3, 2, 2, 64)) == SHAPE and rd(2, None, f(3, 1, 2, 64), f(3, 1, 2, 64)) == SHAPE
    assert rd(None, None, f(3, 1, 2, 64), f(3, 1, 2, 64)) == SHAPE and rd(0, i32(2), f(3, 1, 2, 64), f(3, 1, 2, 64)) == SHAPE
    # the library's own checks, past the binding's
    lib, ref = c.lib, c._ref
    p = q.data_ptr()
    assert lib.koala_paged_attend(ref, 0, 0, 3, 2, 0, 4, p, 256, 0, 0, 1.0, 0, out.data_ptr(), p, 16) == WS
    assert lib.koala_paged_attend(ref, 0, 0, 3, 2, 0, 4, p, 256, 0, 0, 1.0, 0, out.data_ptr(), 0, 1 << 40) == -1
    assert lib.koala_paged_attend(ref, 0, 0, 3, 2, 7, 4, p, 256, 0, 0, 1.0, 0, out.data_ptr(), p, 1 << 40) == UNSUP
    assert lib.koala_paged_attend(ref, 0, 0, 3, 2, 0, 4, p + 4, 256, 0, 0, 1.0, 0, out.data_ptr(), p, 1 << 40) == ALIGN
    assert lib.koala_paged_attend(None, 0, 0, 3, 2, 0, 4, p, 256, 0, 0, 1.0, 0, out.data_ptr(), p, 1 << 40) == -1
    assert lib.koala_paged_commit(ref, 0, 3, p, p, 0, p) == SHAPE and lib.koala_paged_commit(ref, 0, 3, 0, p, 1, p) == -1
    assert lib.koala_paged_workspace_bytes(None, None) == -1
