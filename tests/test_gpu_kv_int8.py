"""GPU: keys and values into a cache of 8-bit integers and back, against the 64-bit definition, for every layout the calls describe."""
import pytest
import torch

import int8_ref as ref
import paper_2607_12121_b200 as fd

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rnd(*shape, seed=0, dt="bf16"):
    g = torch.Generator(device="cuda").manual_seed(sum(shape) + seed)
    return (torch.randn(*shape, generator=g, device="cuda") * torch.exp(torch.randn(*shape[:-1], 1, generator=g, device="cuda"))).to(TYPES[dt])


def _cache(groups, tokens, heads, dh, layout="step", pad=0):
    """Codes and scales of keys and values, filled with what nobody wrote: views [groups, tokens, heads, head_dim] of the layout."""
    if layout == "step":                                        # [B, 2, N, heads, head_dim]
        c = torch.full((groups, 2, tokens, heads, dh + pad), 55, dtype=torch.int8, device="cuda")[..., :dh]
        s = torch.full((groups, 2, tokens, heads), 9.0, device="cuda")
        return [(c[:, i], s[:, i]) for i in (0, 1)]
    if layout == "heads_first":                                 # [B, heads, N, head_dim] each
        return [(torch.full((groups, heads, tokens, dh + pad), 55, dtype=torch.int8, device="cuda")[..., :dh].transpose(1, 2),
                 torch.full((groups, heads, tokens), 9.0, device="cuda").transpose(1, 2)) for _ in range(2)]
    assert layout == "tokens_first"                             # [N, B, heads, head_dim] each
    return [(torch.full((tokens, groups, heads, dh + pad), 55, dtype=torch.int8, device="cuda")[..., :dh].transpose(0, 1),
             torch.full((tokens, groups, heads), 9.0, device="cuda").transpose(0, 1)) for _ in range(2)]


def _index(slots, count, seed=0):
    g = torch.Generator(device="cuda").manual_seed(slots + seed)
    return torch.randperm(slots, generator=g, device="cuda")[:count].sort().values.int()


def _flat(t):
    return t.reshape(-1, *t.shape[2:])                          # slots in front (a copy where the layout needs one)


def _untouched(codes, scale, slots):
    assert bool((_flat(codes)[slots] == 55).all()) and bool((_flat(scale)[slots] == 9.0).all())


def _value(codes, scale):
    return codes.double() * scale.double()[..., None]


SHAPES = [(1, 1, 1, 1), (1, 3, 2, 8), (2, 37, 4, 64), (3, 20, 16, 72), (1, 150, 12, 128), (2, 11, 3, 40), (2, 9, 2, 256), (1, 33, 5, 7), (2, 17, 1, 250), (1, 2, 65, 16),
          (1, 40, 24, 96)]


@pytest.mark.parametrize("layout", ["step", "heads_first", "tokens_first"])
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("source", ["rows", "slots"])
@pytest.mark.parametrize("groups,tokens,heads,dh", SHAPES)
def test_store_then_load(groups, tokens, heads, dh, source, dt, layout):
    slots = groups * tokens
    count = max(1, slots * 5 // 8)
    index = _index(slots, count)
    (k8, ks), (v8, vs) = _cache(groups, tokens, heads, dh, layout)
    if source == "rows":                                        # slices of a fused projection's output
        qkv = _rnd(count, 3 * heads * dh, dt=dt)
        k, v = (qkv[:, i * heads * dh: (i + 1) * heads * dh].unflatten(1, (heads, dh)) for i in (1, 2))
        want = k, v
    else:
        step = _rnd(groups, 2, tokens, heads, dh, dt=dt)
        k, v = step[:, 0], step[:, 1]
        want = _flat(k)[index.long()], _flat(v)[index.long()]
    fd.fd_kv_store_int8(k, k8, ks, v, v8, vs, index=index)
    rest = torch.ones(slots, dtype=torch.bool, device="cuda")
    rest[index.long()] = False
    for codes, scale, w in ((k8, ks, want[0]), (v8, vs, want[1])):
        ref.check_codes(_flat(codes)[index.long()], _flat(scale)[index.long()], w.double())
        _untouched(codes, scale, rest)
    # all of it into the step's layout, and some of it, in any order and one slot twice, into rows
    for back in TYPES.values():
        kv = torch.full((groups, 2, tokens, heads, dh), 3.0, dtype=back, device="cuda")
        fd.fd_kv_load_int8(k8, ks, kv[:, 0], v8, vs, kv[:, 1])
        for got, codes, scale in ((kv[:, 0], k8, ks), (kv[:, 1], v8, vs)):
            w = _value(codes, scale)
            ref.near(got, w, ref.U32 * w.abs())
        some = torch.cat([index.flip(0), index[:1]])
        rows = torch.full((count + 1, heads, 2 * dh), 3.0, dtype=back, device="cuda")
        fd.fd_kv_load_int8(v8, vs, rows[..., dh:], index=some)
        w = _value(_flat(v8), _flat(vs))[some.long()]
        ref.near(rows[..., dh:], w, ref.U32 * w.abs())
        assert bool((rows[..., :dh] == 3.0).all())


@pytest.mark.parametrize("dh", [64, 72, 60])
@pytest.mark.parametrize("used", [-1, 0, 1, 29, 30, 99])
def test_rows_used(used, dh):
    groups, tokens, heads = 2, 40, 3
    index, n = _index(80, 30), max(0, min(30, used))
    count, status = torch.tensor([used], dtype=torch.int32, device="cuda"), torch.full((1,), 5, dtype=torch.int32, device="cuda")
    (k8, ks), _ = _cache(groups, tokens, heads, dh)
    k = _rnd(30, heads, dh)
    fd.fd_kv_store_int8(k, k8, ks, index=index, rows_used=count, status_out=status)
    rest = torch.ones(80, dtype=torch.bool, device="cuda")
    rest[index[:n].long()] = False
    _untouched(k8, ks, rest)
    if n:
        ref.check_codes(_flat(k8)[index[:n].long()], _flat(ks)[index[:n].long()], k[:n].double())
    rows = torch.full((30, heads, dh), 3.0, device="cuda")
    fd.fd_kv_load_int8(k8, ks, rows, index=index, rows_used=count, status_out=status)
    w = _value(_flat(k8), _flat(ks))[index.long()]
    if n:
        ref.near(rows[:n], w[:n], ref.U32 * w[:n].abs())
    assert bool((rows[n:] == 3.0).all()) and int(status) == 0
    whole = torch.full((groups, tokens, heads, dh), 3.0, device="cuda")     # at the slots' own places
    fd.fd_kv_load_int8(k8, ks, whole, index=index, rows_used=count)
    assert bool((_flat(whole)[rest] == 3.0).all())
    assert torch.equal(_flat(whole)[index[:n].long()], rows[:n])


@pytest.mark.parametrize("dh", [128, 72, 50])
def test_refused_indices(dh):
    """Numbers that are no slot, and in a store one that is not above the one before it: skipped and reported, the others done."""
    heads, tokens = 2, 25
    status = torch.full((1,), 5, dtype=torch.int32, device="cuda")
    for index, bad in (([0, 3, 3, 8], [2]), ([-1, 2, 4, 50], [0, 3]), ([5, 9, 7, 20], [2]), ([2 ** 31 - 1, 4, 6, -2 ** 31], [0, 1, 3])):
        (k8, ks), _ = _cache(2, tokens, heads, dh)
        k, idx = _rnd(4, heads, dh), torch.tensor(index, dtype=torch.int32, device="cuda")
        fd.fd_kv_store_int8(k, k8, ks, index=idx, status_out=status)
        assert int(status) == fd.FD_ERR_STATE
        good = [i for i in range(4) if i not in bad]
        at = idx[good].long()
        ref.check_codes(_flat(k8)[at], _flat(ks)[at], k[good].double())
        rest = torch.ones(50, dtype=torch.bool, device="cuda")
        rest[at] = False
        _untouched(k8, ks, rest)
    rows = torch.full((4, heads, dh), 3.0, device="cuda")
    fd.fd_kv_load_int8(k8, ks, rows, index=torch.tensor([50, 6, -1, 6], dtype=torch.int32, device="cuda"), status_out=status)
    assert int(status) == fd.FD_ERR_STATE and bool((rows[[0, 2]] == 3.0).all()) and torch.equal(rows[1], rows[3])
    fd.fd_kv_load_int8(k8, ks, rows, index=torch.tensor([0, 6, 0, 6], dtype=torch.int32, device="cuda"), status_out=status)
    assert int(status) == 0


@pytest.mark.parametrize("dh", [64, 72, 128, 30])
def test_extreme_heads(dh):
    k = torch.zeros(7, 2, dh, device="cuda")
    k[1, 0, 0], k[2, 1, dh - 1], k[3, 0, 1], k[4, 0, 2], k[5], k[6, 1, 0] = float("nan"), float("inf"), 3.4e38, 2.0 ** -120, -2.0, float("-inf")
    k8, ks = torch.full((1, 7, 2, dh), 55, dtype=torch.int8, device="cuda"), torch.full((1, 7, 2), 9.0, device="cuda")
    fd.fd_kv_store_int8(k, k8, ks)
    bad = torch.zeros(7, 2, dtype=torch.bool, device="cuda")
    bad[1, 0] = bad[2, 1] = bad[6, 1] = True
    ref.check_codes(k8[0][~bad], ks[0][~bad], k[~bad].double())
    assert bool(ks[0][bad].isnan().all()) and bool((k8[0][bad] == 0).all())
    back = torch.empty_like(k)
    fd.fd_kv_load_int8(k8, ks, back)
    assert torch.equal(back.isnan().all(dim=2), bad) and torch.equal(back.isnan().any(dim=2), bad)


@pytest.mark.parametrize("off", [1, 4])
@pytest.mark.parametrize("dh", [64, 128])
def test_unaligned_rows_and_codes(off, dh):
    store = _rnd(20, 3 * dh + off)
    k = store[:, off: off + 3 * dh].unflatten(1, (3, dh))
    codes = torch.full((20, 3 * dh + off), 55, dtype=torch.int8, device="cuda")
    k8, ks = codes[:, off:].unflatten(1, (3, dh))[None], torch.empty(1, 20, 3, device="cuda")
    fd.fd_kv_store_int8(k, k8, ks)
    ref.check_codes(k8[0], ks[0], k.double())
    assert bool((codes[:, :off] == 55).all())
    back = torch.zeros_like(store)
    fd.fd_kv_load_int8(k8, ks, back[:, off:].unflatten(1, (3, dh)))
    w = _value(k8[0], ks[0]).flatten(1)
    ref.near(back[:, off:], w, ref.U32 * w.abs())
    assert bool((back[:, :off] == 0).all())


def test_codes_past_32_bits():
    groups, tokens, heads, dh, far = 2, 5, 2, 64, 5_000_000_000  # the second request's codes start 5e9 bytes behind the first's
    base = torch.zeros(far + tokens * heads * dh, dtype=torch.int8, device="cuda")
    k8 = base.as_strided((groups, tokens, heads, dh), (far, heads * dh, dh, 1))
    ks, k = torch.empty(groups, tokens, heads, device="cuda"), _rnd(groups * tokens, heads, dh)
    fd.fd_kv_store_int8(k, k8, ks)
    ref.check_codes(_flat(k8), _flat(ks), k.double())
    back = torch.empty_like(k)
    fd.fd_kv_load_int8(k8, ks, back)
    w = _value(_flat(k8), _flat(ks))
    ref.near(back, w, ref.U32 * w.abs())


def test_another_stream_and_graph():
    k, (k8, ks) = _rnd(40, 4, 64), _cache(1, 60, 4, 64)[0]
    index, used = _index(60, 40), torch.tensor([40], dtype=torch.int32, device="cuda")
    back = torch.zeros(1, 60, 4, 64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fd.fd_kv_store_int8(k, k8, ks, index=index, rows_used=used)
        fd.fd_kv_load_int8(k8, ks, back)
    for count, seed in ((40, 1), (17, 2)):
        k.copy_(_rnd(40, 4, 64, seed=seed))
        used.fill_(count)
        graph.replay()
        torch.cuda.synchronize()
        at = index[:count].long()
        ref.check_codes(_flat(k8)[at], _flat(ks)[at], k[:count].double())
        w = _value(k8, ks)
        ref.near(back, w, ref.U32 * w.abs())
