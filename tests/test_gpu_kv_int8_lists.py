"""GPU: lists of a store that are not strictly ascending.  A row counts if its index is a slot above the index before it; a slot that several such
rows name holds the last one's codes and scales, all of them."""
import pytest
import torch

import int8_ref as ref
import paper_2607_12121_b200 as fd

pytestmark = pytest.mark.gpu


def _last(index, slots):
    """How many rows count, and the slots that they name with the last row that does, in the order of the slots."""
    count = [i for i, s in enumerate(index) if 0 <= s < slots and not (i > 0 and index[i - 1] >= s)]
    last = {index[i]: i for i in count}
    return len(count), sorted(last), [last[s] for s in sorted(last)]


def _run(index, slots, heads, dh, source="rows", used=None, sets=2, dt=torch.bfloat16, replay=False):
    n = len(index)
    count = n if used is None else used
    g = torch.Generator(device="cuda").manual_seed(n + heads + dh)
    rows = torch.randn(2, n if source == "rows" else slots, heads, dh, generator=g, device="cuda").to(dt)
    codes = torch.full((2, 1, slots, heads, dh), 55, dtype=torch.int8, device="cuda")
    scale = torch.full((2, 1, slots, heads), 9.0, device="cuda")
    idx, status = torch.tensor(index, dtype=torch.int32, device="cuda"), torch.full((1,), 5, dtype=torch.int32, device="cuda")
    word = None if used is None else torch.tensor([used], dtype=torch.int32, device="cuda")
    src = [t if source == "rows" else t[None] for t in rows]
    second = (src[1], codes[1], scale[1]) if sets == 2 else ()

    def store(**kw):
        fd.fd_kv_store_int8(src[0], codes[0], scale[0], *second, index=idx, rows_used=word, **kw)

    if replay:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            store(status_out=status)
        graph.replay()
    else:
        store(status_out=status)
    counted, named, last = _last(index[:count], slots)
    assert int(status) == (0 if counted == count else fd.FD_ERR_STATE)
    at = torch.tensor(named, dtype=torch.long, device="cuda")
    rest = torch.ones(slots, dtype=torch.bool, device="cuda")
    rest[at] = False
    for half in range(2):
        c, s = codes[half, 0], scale[half, 0]
        if half < sets and named:
            ref.check_codes(c[at], s[at], rows[half][last if source == "rows" else at].double())
        untouched = rest if half < sets else torch.ones_like(rest)
        assert bool((c[untouched] == 55).all()) and bool((s[untouched] == 9.0).all())
    before = codes.clone(), scale.clone()                       # the same again, without the word: the same slots get the same
    store()
    assert torch.equal(codes, before[0]) and torch.equal(scale, before[1])


@pytest.mark.parametrize("index", [[5, 3, 5], [5, -1, 5], [0, 1, 2, 0, 1, 2], [3, 5, 3, 4, 5], [7, 50, 7], [2 ** 31 - 1, 4, 6, 4, 6], [9, 9, 9], [4, 3, 2, 1, 0],
                                   [-2 ** 31, 0, -1, 0, 1], [0], [49], [50], [-1]])
@pytest.mark.parametrize("heads,dh", [(1, 8), (3, 64), (16, 72), (5, 50), (12, 128), (2, 250)])
def test_short_lists(index, heads, dh):
    _run(index, 50, heads, dh)
    _run(index, 50, heads, dh, "slots", sets=1, dt=torch.float32)


def _long(n, slots, kind):
    g = torch.Generator().manual_seed(n + len(kind))
    up = torch.randperm(slots, generator=g)[:n].sort().values
    if kind == "two numberings":                                # of two requests, each from zero
        up = torch.cat([torch.arange(n // 2), torch.arange(n - n // 2)])
    elif kind == "random":
        up = torch.randint(-2, slots + 2, (n,), generator=g)
    elif kind == "one returns":                                 # the first slot once more, far behind
        up[n - 2] = up[0]
    elif kind == "repeats":
        up = torch.arange(n) // 2 % slots
    elif kind == "a hole":
        up[n // 3] = -1
    elif kind == "swaps":                                       # every 97th pair of neighbours the wrong way round
        for i in range(5, n - 1, 97):
            up[[i, i + 1]] = up[[i + 1, i]]
    elif kind == "first is last":
        up[0] = slots - 1
    elif kind == "holes":                                       # every 256th row, a run of rows, and the end name no slot
        up[256::256] = -1
        up[n // 2: n // 2 + 300] = -1
        up[n - n // 3:] = -1
    elif kind == "halves swapped":
        up = torch.cat([up[n // 2:], up[: n // 2]])
    elif kind == "thrice":                                      # the same slots three times over
        up = torch.cat([up[: n // 3]] * 3 + [up[n // 3: n // 3 + n - n // 3 * 3]])
    return up.tolist()


@pytest.mark.parametrize("kind", ["ascending", "two numberings", "random", "one returns", "repeats", "a hole", "swaps", "first is last", "holes", "halves swapped", "thrice"])
@pytest.mark.parametrize("n,slots,heads,dh", [(4099, 6000, 12, 128), (3001, 3300, 1, 64), (20011, 40000, 2, 40), (2500, 5000, 65, 16), (3001, 4000, 3, 50), (700, 900, 24, 96)])
def test_long_lists(n, slots, heads, dh, kind):
    """Lists over many CTAs, with slots that come back near and far."""
    _run(_long(n, slots, kind), slots, heads, dh)


@pytest.mark.parametrize("used", [0, 1, 77, 999, 1000])
@pytest.mark.parametrize("kind", ["ascending", "random", "one returns"])
def test_rows_behind_the_used_ones_do_not_count(used, kind):
    index = _long(1000, 1500, kind)
    _run(index, 1500, 4, 64, used=used, replay=True)
    _run(index, 1500, 3, 30, used=used, source="slots")


@pytest.mark.parametrize("offset", [0, 1, 2, 3])
def test_lists_that_begin_anywhere(offset):
    """The list as a slice of a longer one, at every alignment of its address."""
    whole = torch.tensor([7] * offset + _long(2003, 2500, "one returns"), dtype=torch.int32, device="cuda")
    k = torch.randn(2003, 2, 64, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    k8, ks = torch.full((1, 2500, 2, 64), 55, dtype=torch.int8, device="cuda"), torch.full((1, 2500, 2), 9.0, device="cuda")
    fd.fd_kv_store_int8(k, k8, ks, index=whole[offset:])
    counted, named, last = _last(whole[offset:].tolist(), 2500)
    assert counted == 2002 and len(named) == 2002               # (all but the row that names the first slot again)
    at = torch.tensor(named, device="cuda")
    ref.check_codes(k8[0, at], ks[0, at], k[last].double())


@pytest.mark.parametrize("captured", [False, True])
def test_lists_written_just_before(captured):
    """Lists and their lengths that change from call to call in the same memory without a wait between, ascending and not; other calls of the library
    stand before and behind."""
    n, slots, heads, dh, steps = 3000, 4000, 6, 64, 24
    g = torch.Generator(device="cuda").manual_seed(3)
    kinds = ["ascending", "two numberings", "thrice", "ascending", "repeats", "one returns"]
    lists = [torch.tensor(_long(n, slots, kinds[i % len(kinds)]), dtype=torch.int32, device="cuda") for i in range(steps)]
    lengths = [torch.tensor([n - 100 * i], dtype=torch.int32, device="cuda") for i in range(steps)]
    xs = [torch.randn(n, 2 * heads * dh, generator=g, device="cuda").bfloat16() for _ in range(3)]
    x, y8, y_s = torch.empty_like(xs[0]), torch.empty(n, 2 * heads * dh, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
    index, used = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    codes = torch.empty(2, 1, slots, heads, dh, dtype=torch.int8, device="cuda")
    scale, back = torch.empty(2, 1, slots, heads, device="cuda"), torch.empty(2, 1, slots, heads, dh, device="cuda")
    k, v = (x[:, i * heads * dh: (i + 1) * heads * dh].unflatten(1, (heads, dh)) for i in (0, 1))

    def work():
        fd.fd_quantize_int8_rows(x, y8, y_s, rows_used=used)
        fd.fd_kv_store_int8(k, codes[0], scale[0], v, codes[1], scale[1], index=index, rows_used=used)
        fd.fd_kv_load_int8(codes[0], scale[0], back[0], codes[1], scale[1], back[1])

    graph = None
    if captured:
        x.copy_(xs[0]), index.copy_(lists[0]), used.copy_(lengths[0]), codes.fill_(55), scale.fill_(9.0)
        work()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            work()
    kept = []
    for i in range(steps):
        x.copy_(xs[i % 3]), codes.fill_(55), scale.fill_(9.0), index.copy_(lists[i]), used.copy_(lengths[i])
        graph.replay() if captured else work()
        kept.append((codes.clone(), scale.clone(), back.clone()))
    for i, (codes_, scale_, back_) in enumerate(kept):
        counted, named, last = _last(lists[i].tolist()[: n - 100 * i], slots)
        at, rest = torch.tensor(named, device="cuda"), torch.ones(slots, dtype=torch.bool, device="cuda")
        rest[at] = False
        rows = xs[i % 3].unflatten(1, (2, heads, dh))
        for half in range(2):
            ref.check_codes(codes_[half, 0, at], scale_[half, 0, at], rows[last, half].double())
            assert bool((codes_[half, 0, rest] == 55).all()) and bool((scale_[half, 0, rest] == 9.0).all())
        value = codes_.double() * scale_.double()[..., None]
        ref.near(back_, value, ref.U32 * value.abs())
