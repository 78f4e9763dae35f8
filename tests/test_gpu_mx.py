"""The 4-bit path against plain 64-bit arithmetic (block_reference): conversions exactly, products within the rounding of fp32 sums.

Tolerances.  u = 2^-24.  The held values' products are exact.  A matrix instruction adds 64 of them, in whatever order at most 64 additions
for a term, and n / 64 instructions follow each other: 64 + n / 64 additions, each off by at most a step of the partial sum (2 u of it;
the matrix cores may cut instead of rounding), and one more for the bias.  The FFN's hidden rows are
rounded to 4 bits from fp32: where a hidden value lies within its own error of a border, it may fall on either side, and the output may
be off by that step times the weight."""
import numpy as np
import pytest
import torch

from paper_2502_16927_amd import binding as B
import block_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": B.F32, "bf16": B.BF16}


def up(t):
    return t.double().cpu().numpy()


def scale_place(blocks):
    b = np.arange(blocks)
    return (b // 8) * 8 + (b % 2) * 4 + (b % 8) // 2


def quantised(src):
    """Codes and scales of the library, as numpy: codes [rows, cols], scale bytes in block order, and the buffers."""
    rows, cols = src.shape
    codes = torch.full((rows, cols // 2), 0xEE, dtype=torch.uint8, device=DEV)
    scales = torch.full((B.mx_scale_bytes(cols) // 8, rows, 8), 0xEE, dtype=torch.uint8, device=DEV)
    B.bigmac_mx_quantize(rows, cols, B.BF16 if src.dtype == torch.bfloat16 else B.F32, src, codes, scales)
    c, s = codes.cpu().numpy().astype(np.int64), scales.cpu().numpy().astype(np.int64).transpose(1, 0, 2).reshape(rows, -1)
    used = scale_place(cols // 32)
    assert (np.delete(s, used, 1) == 0).all(), "unused scale bytes"
    return np.stack([c & 15, c >> 4], 2).reshape(rows, cols), s[:, used], codes, scales


def check_rows(src):
    rows, cols = src.shape
    want_codes, want_scales, want = R.quantise(up(src))
    got_codes, got_scales, codes, scales = quantised(src)
    assert np.array_equal(got_scales, want_scales)
    assert np.array_equal(got_codes, want_codes)
    for t in ("f32", "bf16"):
        back = torch.full((rows, cols), 7.0, dtype=TYPE[t], device=DEV)
        B.bigmac_mx_dequantize(rows, cols, codes, scales, CODE[t], back)
        assert np.array_equal(up(back), want, equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 64), (3, 96), (65, 288), (130, 1024), (7, 4096), (513, 320), (2, 8224)])
def test_rows_to_four_bits_and_back(rows, cols, dtype):
    g = torch.Generator(device=DEV).manual_seed(rows + cols)
    src = torch.randn((rows, cols), generator=g, device=DEV) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=g, device=DEV).float())
    check_rows(src.to(TYPE[dtype]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_borders_ties_zeros_and_extremes(dtype):
    """Every middle between two held values, its neighbours, largest magnitudes at and next to powers of two, zeros of both signs, the
    smallest and the largest numbers of the type, blocks with an infinity or NaN beside whole ones."""
    t = TYPE[dtype]
    grid = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7])
    rows = []
    for power in (-140, -133, -128, -126, -125, -100, -3, 0, 1, 90, 120):
        for top in (4.0, 6.0, 7.5, 1.0, 2.0):
            base = torch.tensor(np.concatenate([grid[grid <= top], [top]]) * 2.0 ** power, dtype=torch.float64).to(t)
            near = torch.cat([base, torch.nextafter(base.float(), torch.tensor(float("inf"))).to(t), -base])
            block = torch.zeros(96, dtype=t)
            block[:min(96, near.numel())] = near[:96]
            block[block.abs() > abs(float(base[-1]))] = base[-1]
            rows.append(block)
    rows.append(torch.zeros(96, dtype=t))
    rows.append(-torch.zeros(96, dtype=t))
    rows.append(torch.full((96,), torch.finfo(t).max, dtype=t))
    rows.append(torch.full((96,), torch.finfo(t).tiny, dtype=t))
    for bad in (float("inf"), float("-inf"), float("nan")):
        r = torch.linspace(-5, 5, 96).to(t)
        r[40] = bad
        rows.append(r)
    check_rows(torch.stack(rows).to(DEV))


def pack(w):
    groups, n_in, n_out = w.shape
    packed = torch.full((B.mx_packed_bytes(groups, n_in, n_out),), 0xEE, dtype=torch.uint8, device=DEV)
    B.bigmac_mx_pack(groups, n_in, n_out, B.BF16 if w.dtype == torch.bfloat16 else B.F32, w, packed)
    return packed


def held(w):
    """Held values of weights [groups, n_in, n_out]: blocks along n_in."""
    return np.swapaxes(R.quantise(np.swapaxes(up(w), 1, 2).copy())[2], 1, 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups,n_in,n_out", [(1, 64, 64), (3, 192, 64), (2, 320, 192), (5, 1024, 128)])
def test_weights_packed_and_unpacked(groups, n_in, n_out, dtype):
    g = torch.Generator(device=DEV).manual_seed(n_in)
    w = (torch.randn((groups, n_in, n_out), generator=g, device=DEV) * 0.02).to(TYPE[dtype])
    w[0, :32, 5] = 0.0
    w[groups - 1, n_in - 3, n_out - 1] = float("inf")
    packed = pack(w)
    for t in ("f32", "bf16"):
        back = torch.empty((groups, n_in, n_out), dtype=TYPE[t], device=DEV)
        B.bigmac_mx_unpack(groups, n_in, n_out, packed, CODE[t], back)
        assert np.array_equal(up(back), held(w), equal_nan=True)
    again = pack(torch.nan_to_num(back, nan=float("inf")))
    assert torch.equal(again, packed)                                # held values are held as themselves


def offsets_of(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def product(x, counts, w, bias=None, out="f32", spare=0):
    """bigmac_mx_product on quantised rows; counts None: dense.  spare: rows of the buffers behind the last group."""
    groups, n_in, n_out = w.shape
    rows = x.shape[0]
    _, _, codes, scales = quantised(x)
    dims = B.make_mx_dims(rows, groups, n_in, n_out, CODE[out])
    ws = torch.full((max(B.mx_workspace_bytes(dims), 256),), 0xEE, dtype=torch.uint8, device=DEV)
    got = torch.full((rows, n_out), 7.0, dtype=TYPE[out], device=DEV)
    B.bigmac_mx_product(dims, codes, scales, None if counts is None else offsets_of(counts), pack(w), bias, got, ws)
    return got


def check_product(counts, n_in, n_out, out="f32", bias=False, spare=0, dense=False, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    groups, rows = len(counts), int(sum(counts)) + spare
    x = torch.randn((rows, n_in), generator=g, device=DEV).to(torch.bfloat16)
    w = (torch.randn((groups, n_in, n_out), generator=g, device=DEV) * torch.exp2(torch.randint(-4, 5, (groups, n_in, 1), generator=g, device=DEV).float())).to(torch.bfloat16)
    b = torch.randn((groups, n_out), generator=g, device=DEV).to(torch.bfloat16) if bias else None
    got = up(product(x, None if dense else counts, w, b, out))
    xq, wq = R.quantise(up(x))[2], held(w)
    at = 0
    for e, n in enumerate(counts):
        a = xq[at:at + n]
        want, size = a @ wq[e], np.abs(a) @ np.abs(wq[e])
        if bias:
            want, size = want + up(b)[e], size + np.abs(up(b)[e])
        limit = 2 * (65 + n_in / 64) * R.U32 * size + R.HALF_STEP[out] * np.abs(want) * (1 + 2.0 ** -10)
        off = np.abs(got[at:at + n] - want)
        assert (off <= limit).all(), f"group {e} of {n} rows: {int((off > limit).sum())} of {off.size} off, worst {np.nanmax(off / limit)} of the limit"
        at += n
    assert (got[at:] == 7.0).all(), "rows behind the last group"


# row counts around the tiles' edges, groups without rows at the start, in between and at the end, inputs that end inside a chunk
@pytest.mark.parametrize("n_in,n_out", [(64, 64), (192, 320), (256, 64), (320, 128), (1024, 192), (4096, 64)])
@pytest.mark.parametrize("counts", [[1], [0, 1, 0], [31, 32, 33, 0], [5, 0, 63, 64, 65, 1], [127, 128, 129], [300, 0, 1, 270]], ids=str)
def test_ragged_products(counts, n_in, n_out):
    print(f"products of {counts} rows, {n_in} -> {n_out}", flush=True)
    check_product(counts, n_in, n_out, seed=n_in)
    check_product(counts, n_in, n_out, out="bf16", bias=True, spare=37, seed=n_in + 1)


@pytest.mark.parametrize("rows", [1, 2, 33, 64, 100, 129, 1000])
def test_dense_products(rows):
    check_product([rows], 576, 448, dense=True, bias=rows % 2 == 0, out="bf16" if rows > 64 else "f32")


# row counts around every sub-tile's edge; groups for tiles of 64 rows and enough for tiles of 128
EDGES = [0, 1, 31, 32, 33, 64, 65, 96, 97, 127, 128, 129, 200, 5, 0, 160]


@pytest.mark.parametrize("n_in,n_out", [(64, 64), (320, 192), (1088, 64), (512, 320)])
@pytest.mark.parametrize("times", [8, 13])
def test_tiles_of_64_and_128_rows(n_in, n_out, times):
    counts = EDGES * times
    print(f"products of {sum(counts)} rows in {len(counts)} groups, {n_in} -> {n_out}", flush=True)
    check_product(counts, n_in, n_out, seed=n_in)
    check_product(counts, n_in, n_out, out="bf16", bias=True, spare=70, seed=n_in + 1)


def test_one_row_and_few_rows_over_many_inputs():
    """A quarter of the inputs per wavefront: inputs that end inside a chunk, fewer chunks for one wavefront than for another."""
    for n_in in (2048, 2112, 2304, 4160):
        for counts in ([1], [33], [3, 0, 40]):
            check_product(counts, n_in, 128, out="f32", bias=True, seed=n_in)
            check_product(counts, n_in, 64, out="bf16", dense=len(counts) == 1, seed=n_in)


def test_many_groups():
    rng = np.random.default_rng(3)
    check_product(list(rng.integers(0, 5, 700)), 64, 64)


def test_large_ragged_product_against_an_exact_one():
    """Thousands of rows over uneven groups: the values are small integers, every product and sum is exact."""
    g = torch.Generator(device=DEV).manual_seed(4)
    counts = [1500, 0, 3, 700, 2049, 31]
    held_ints = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0], device=DEV)
    pick = lambda *shape: held_ints[torch.randint(0, 6, shape, generator=g, device=DEV)] * (torch.randint(0, 2, shape, generator=g, device=DEV) * 2 - 1)  # noqa: E731
    rows, n_in, n_out = sum(counts), 1088, 640
    x, w = pick(rows, n_in), pick(len(counts), n_in, n_out)
    x[:, ::32], w[:, ::32] = 6.0, 4.0                                # every block's scale is 1
    got = product(x.to(torch.bfloat16), counts, w.to(torch.bfloat16), out="f32")
    at = 0
    for e, n in enumerate(counts):
        assert torch.equal(got[at:at + n], (x[at:at + n].double() @ w[e].double()).float()), e
        at += n


def test_a_row_that_is_not_finite_stays_alone():
    g = torch.Generator(device=DEV).manual_seed(8)
    x = torch.randn((70, 256), generator=g, device=DEV).to(torch.bfloat16)
    w = torch.randn((2, 256, 128), generator=g, device=DEV).to(torch.bfloat16)
    want = product(x, [40, 30], w)
    x[5, 100], x[60, 0] = float("nan"), float("inf")
    got = product(x, [40, 30], w)
    keep = [r for r in range(70) if r not in (5, 60)]
    assert torch.equal(got[keep], want[keep]) and torch.isnan(got[5]).all() and torch.isnan(got[60]).all()


@pytest.mark.parametrize("rows", [70, 6000])
@pytest.mark.parametrize("offsets", [lambda n: [0, 2 * n, 3 * n, 3 * n], lambda n: [0, n, 0, n], lambda n: [-n, 0, n, 2 * n], lambda n: [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0],
                                     lambda n: [n, n - 1, n - 2, 0]], ids=["past", "back", "negative", "extremes", "descending"])
def test_offsets_that_are_not_offsets(rows, offsets):
    """The product bounds every access by the rows and the map's size: what lies in front of and behind the buffers keeps its values."""
    n_in, n_out, groups = 128, 320, 3
    x = torch.ones((rows, n_in), dtype=torch.bfloat16, device=DEV)
    _, _, codes, scales = quantised(x)
    w = pack(torch.ones((groups, n_in, n_out), dtype=torch.bfloat16, device=DEV))
    dims = B.make_mx_dims(rows, groups, n_in, n_out, B.F32)
    size = B.mx_workspace_bytes(dims)
    ws = torch.full((size + 8192,), 0xEE, dtype=torch.uint8, device=DEV)
    out = torch.full((rows + 512, n_out), 7.0, device=DEV)
    at = torch.tensor(offsets(rows), dtype=torch.int64).to(torch.int32).to(DEV)
    print(f"offsets {offsets(rows)}, {rows} rows", flush=True)
    B.bigmac_mx_product(dims, codes, scales, at, w, None, out[256:256 + rows], ws[4096:4096 + size])
    assert (out[:256] == 7.0).all() and (out[256 + rows:] == 7.0).all(), "beside the rows"
    assert (ws[:4096] == 0xEE).all() and (ws[4096 + size:] == 0xEE).all(), "beside the workspace"
    inside = out[256:256 + rows]
    assert ((inside == 7.0) | (inside == n_in)).all()


# ------------------------------------------------------------------ the experts' FFN

class Ffn:
    def __init__(self, T, k, N, r, h, counts, bias, order=B.ORDER_DCCA, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.counts, rows = counts, T * k
        self.dims = B.make_dims(T, r if order == B.ORDER_CDAC else 4 * r, h if order == B.ORDER_CDAC else r, N, k, h, order=order)
        rand = lambda std, *shape: (torch.randn(shape, generator=g, device=DEV) * std).to(torch.bfloat16)  # noqa: E731
        self.x, w1, w2 = rand(1.0, rows, r), rand(2.0 / r ** 0.5, N, r, h), rand(0.02, N, h, r)
        self.b1, self.b2 = (rand(0.3, N, h), rand(0.02, N, r)) if bias else (None, None)
        self.w1, self.w2, self.h1, self.h2 = pack(w1), pack(w2), held(w1), held(w2)
        self.offsets = offsets_of(counts)
        self.out = torch.full((rows, r), 7.0, dtype=torch.bfloat16, device=DEV)
        self.ws = torch.full((B.workspace_bytes(self.dims, B.WS_MX_GROUPED_FFN),), 0xEE, dtype=torch.uint8, device=DEV)

    def run(self, stream=None):
        B.bigmac_mx_grouped_ffn(self.dims, self.x, self.offsets, self.w1, self.w2, self.out, self.ws, b1=self.b1, b2=self.b2, stream=stream)

    def check(self):
        rows = sum(self.counts)
        want, limit = R.ffn(up(self.x)[:rows], self.counts, self.h1, self.h2, None if self.b1 is None else up(self.b1), None if self.b2 is None else up(self.b2))
        off = np.abs(up(self.out)[:rows] - want)
        assert (off <= limit).all(), f"{int((off > limit).sum())} of {off.size} off, worst {np.nanmax(off / limit)} of the limit"
        assert (self.out[rows:] == 7.0).all(), "rows behind the last expert"
        # the tolerance for hidden values next to a border is an exception, not the rule
        assert np.mean(limit > 0.05 * np.sqrt(np.mean(want ** 2))) < 0.2


@pytest.mark.parametrize("T,k,N,r,h,counts", [
    (1, 1, 1, 64, 64, [1]),
    (1, 2, 4, 128, 256, [0, 1, 1, 0]),
    (32, 8, 8, 192, 448, [40, 0, 31, 33, 64, 1, 86, 1]),
    (40, 4, 4, 320, 640, [70, 64, 20, 6]),
    (200, 2, 3, 256, 576, [129, 0, 271]),
    (64, 2, 2, 1024, 128, [128, 0]),
    (20, 1, 2, 2112, 64, [7, 13]),
    (12, 1, 2, 128, 2176, [0, 12]),
    (sum(EDGES) * 4, 2, 128, 192, 320, EDGES * 8),
    (400, 2, 8, 128, 4096, [129, 64, 65, 63, 1, 0, 200, 278]),
], ids=lambda v: str(v)[:40])
@pytest.mark.parametrize("bias", [False, True])
def test_experts(T, k, N, r, h, counts, bias):
    print(f"experts T {T} k {k} N {N} r {r} h {h} {counts}", flush=True)
    f = Ffn(T, k, N, r, h, counts, bias, seed=r)
    f.run()
    f.check()


def test_experts_of_the_fine_grained_order_and_dropped_pairs():
    """win = d, hid = r; fewer rows than T k (a capacity dropped some): the rest of o_perm stays as it was."""
    f = Ffn(50, 2, 4, 256, 192, [20, 3, 0, 41], True, order=B.ORDER_CDAC)
    f.run()
    f.check()


def test_experts_on_another_stream_and_in_a_graph():
    f = Ffn(60, 4, 6, 256, 512, [100, 0, 33, 64, 42, 1], True)
    f.run()
    f.check()
    want = f.out.clone()
    s = torch.cuda.Stream()
    f.out.fill_(7.0)
    torch.cuda.synchronize()
    f.run(stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(f.out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f.run()
    for replay in range(4):
        f.out.fill_(7.0)
        f.ws.fill_(0xEE)
        _ = (f.x.float() * 2).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(f.out, want), replay


# ------------------------------------------------------------------ hidden blocks whose 32 inputs are all negative

def ffn_limit(x, counts, w1, w2, b1):
    """Like R.ffn with the activation held to include/bigmac.h: a hidden value is off by at most 2^-15 of the largest of its block, besides
    what its input's own error makes of it (a product of n inputs adds 64 + n / 64 times in fp32, each off by 2 u of the partial sum at
    most, and once for the bias; GELU taken at both ends of that, and inside 1.13 times it where the two ends enclose GELU's minimum)."""
    outs, limits, at = [], [], 0
    xq = R.quantise(x)[2]
    for e, n in enumerate(counts):
        a = xq[at:at + n]
        pre, size = a @ w1[e] + b1[e], np.abs(a) @ np.abs(w1[e]) + np.abs(b1[e])
        delta = 2 * (66 + a.shape[1] / 64) * R.U32 * size
        h = R.gelu(pre)
        off = np.maximum(np.abs(R.gelu(pre + delta) - h), np.abs(R.gelu(pre - delta) - h))
        off = np.where(np.abs(pre + 0.7518) < 0.5, 1.13 * delta, off)
        off = off + 2.0 ** -15 * np.repeat(np.abs(h).reshape(n, h.shape[1] // 32, 32).max(2), 32, 1)
        q, sign = R.quantise(h)[2], np.where(h < 0, -1.0, 1.0)
        moved = np.zeros_like(q)
        for direction in (1.0, -1.0):
            moved = np.maximum(moved, np.abs(R.quantise(sign * np.maximum(np.abs(h) + direction * off, 0.0))[2] - q))
        want, osize = q @ w2[e], np.abs(q) @ np.abs(w2[e])
        outs.append(want)
        limits.append(2 * (65 + h.shape[1] / 64) * R.U32 * osize + R.HALF_STEP["bf16"] * np.abs(want) * (1 + 2.0 ** -10) + (1 + R.HALF_STEP["bf16"]) * (moved @ np.abs(w2[e])))
        at += n
    return np.concatenate(outs), np.concatenate(limits)


# where the blocks' inputs lie: the tail out to where GELU leaves the range of 4-bit blocks' scales, the border between the two forms of the
# activation (largest magnitude 2^-5: inputs about -2.25 or 0.061), blocks of tiny inputs beside far ones
TAILS = [(-2.6, -2.0), (-3.5, -2.2), (-4.8, -4.2), (-5.5, -5.0), (-6.5, -6.0), (-7.5, -7.0), (-9.0, -8.5), (-12.3, -11.9), (0.04, 0.07), (-7.0, 1e-4), (-0.05, 0.05), (-1.0, 1.0)]


@pytest.mark.parametrize("T,k,N,r,counts", [
    (40, 2, 4, 128, [1, 31, 0, 40]),                                 # tiles of 32 rows
    (20, 1, 1, 2112, [17]),                                          # inputs split over the wavefronts, rows behind the last
    (1536, 2, 4, 192, [700, 801, 97, 1400]),                         # more rows: the larger tiles
    (12288, 1, 2, 64, [5000, 7000]),
], ids=["few", "split", "many", "more"])
@pytest.mark.parametrize("bias", [True, False])
def test_experts_with_hidden_blocks_of_the_tail(T, k, N, r, counts, bias):
    """bias False: the same places by weights of an input that is 1 in every row, as 4 bits hold them."""
    g = torch.Generator(device=DEV).manual_seed(r)
    h = 32 * 2 * len(TAILS)                                          # an even and an odd block of every range
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    lo, hi = (torch.tensor(v, device=DEV).repeat_interleave(2).repeat_interleave(32) for v in zip(*TAILS))
    b1 = (lo + (hi - lo) * torch.rand((N, h), generator=g, device=DEV)).to(torch.bfloat16)
    x = rand(T * k, r).to(torch.bfloat16)
    w1 = (rand(N, r, h) * (0.1 * (hi - lo) / r ** 0.5)).to(torch.bfloat16)
    if not bias:
        x[:, :32], x[:, 0], w1[:, :32] = 0.0, 1.0, 0.0
        w1[:, 0] = b1
        b1 = torch.from_numpy(held(w1)[:, 0]).to(torch.bfloat16).to(DEV)
    # every block's hidden values count alike in the output
    weight = 1.0 / torch.from_numpy(np.abs(R.gelu(up(b1))).reshape(N, -1, 32).max(2)).to(DEV).repeat_interleave(32, 1)
    w2 = (rand(N, h, r) * weight[:, :, None]).to(torch.bfloat16)
    dims = B.make_dims(T, 4 * r, r, N, k, h)
    out = torch.full((T * k, r), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((B.workspace_bytes(dims, B.WS_MX_GROUPED_FFN),), 0xEE, dtype=torch.uint8, device=DEV)
    print(f"experts with tail blocks, T {T} k {k} N {N} r {r} h {h} {counts}, bias {bias}", flush=True)
    B.bigmac_mx_grouped_ffn(dims, x, offsets_of(counts), pack(w1), pack(w2), out, ws, b1=b1 if bias else None)
    rows = sum(counts)
    want, limit = ffn_limit(up(x)[:rows], counts, held(w1), held(w2), up(b1) if bias else np.zeros((N, h)))
    off = np.abs(up(out)[:rows] - want)
    scale = np.sqrt(np.mean(want ** 2))
    print(f"off at most {off.max() / scale:.2e} of the RMS, limits {limit.mean() / scale:.2e} in the mean", flush=True)
    assert (off <= limit).all(), f"{int((off > limit).sum())} of {off.size} off, worst {np.nanmax(off / limit)} of the limit"
    assert (out[rows:] == 7.0).all(), "rows behind the last expert"
    assert np.mean(limit > 0.05 * scale) < 0.2


@pytest.mark.parametrize("ragged", [False, True])
def test_product_of_rows_past_32_bit_offsets(ragged):
    """16 GiB of rows, 4 GiB of their codes: the last ones against an exact product (small integers, every block's scale 1)."""
    rows, n, n_in, n_out = (1 << 21) + 300, 200, 4096, 64
    g = torch.Generator(device=DEV).manual_seed(12)
    whole = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0], device=DEV)
    pick = lambda *shape: whole[torch.randint(0, 6, shape, generator=g, device=DEV)] * (torch.randint(0, 2, shape, generator=g, device=DEV) * 2 - 1)  # noqa: E731
    x = torch.zeros((rows, n_in), dtype=torch.bfloat16, device=DEV)
    x[-n:] = pick(n, n_in).to(torch.bfloat16)
    x[:, ::32] = 6.0
    w = pick(2 if ragged else 1, n_in, n_out)
    w[:, ::32] = 4.0
    codes = torch.empty((rows, n_in // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((B.mx_scale_bytes(n_in) // 8, rows, 8), dtype=torch.uint8, device=DEV)
    print(f"product of {rows} rows", flush=True)
    B.bigmac_mx_quantize(rows, n_in, B.BF16, x, codes, scales)
    dims = B.make_mx_dims(rows, len(w), n_in, n_out, B.F32)
    out = torch.empty((rows, n_out), device=DEV)
    B.bigmac_mx_product(dims, codes, scales, offsets_of([rows - 77, 77]) if ragged else None, pack(w.to(torch.bfloat16)), None, out, B.alloc_bytes(B.mx_workspace_bytes(dims)))
    first, last = w[0].double().cpu(), w[-1].double().cpu()
    tail = x[-n:].double().cpu()
    want = tail @ first
    if ragged:
        want[-77:] = tail[-77:] @ last
    assert torch.equal(out[-n:].double().cpu(), want)
    assert (out[:-n].double() == (6.0 * first[::32].sum(0)).to(DEV)).all()
    back = torch.empty((rows, n_in), dtype=torch.bfloat16, device=DEV)
    B.bigmac_mx_dequantize(rows, n_in, codes, scales, B.BF16, back)
    assert torch.equal(back[-n:], x[-n:]) and torch.equal(back[1 << 20], x[1 << 20])


@pytest.mark.parametrize("T,r", [(24, 128), (20, 2112), (700, 128), (6000, 64)])
def test_a_row_does_not_depend_on_its_neighbours_blocks(T, r):
    """Rows beside others whose hidden blocks lie in GELU's tail: the same bits as beside others that do not."""
    g = torch.Generator(device=DEV).manual_seed(T)
    h = 320
    x = torch.randn((T, r), generator=g, device=DEV).to(torch.bfloat16)
    x[:, :32] = 0.0
    w1 = (torch.randn((1, r, h), generator=g, device=DEV) / r ** 0.5).to(torch.bfloat16)
    w1[:, :32] = 0.0
    w1[:, 0] = -8.0
    w2 = pack(torch.randn((1, h, r), generator=g, device=DEV).to(torch.bfloat16))
    w1 = pack(w1)
    dims = B.make_dims(T, 4 * r, r, 1, 1, h)
    ws = B.alloc_bytes(B.workspace_bytes(dims, B.WS_MX_GROUPED_FFN))
    outs = []
    for deep in (False, True):
        x[1::3, 0] = 1.0 if deep else 0.0
        out = torch.empty((T, r), dtype=torch.bfloat16, device=DEV)
        B.bigmac_mx_grouped_ffn(dims, x, offsets_of([T]), w1, w2, out, ws)
        outs.append(out)
    keep = [i for i in range(T) if i % 3 != 1]
    assert torch.equal(outs[0][keep], outs[1][keep]) and not torch.equal(outs[0][1::3], outs[1][1::3])
