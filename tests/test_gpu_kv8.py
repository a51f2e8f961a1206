"""The paged 8-bit cache on the GPU against its float64 oracle: appended bytes bit for bit, attention within the bar that the
oracle module derives, and what a serving program does with both."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O
from paper_2503_18773_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda:0"


def half(rng, dtype, *shape, scale=1.0):
    """Normal values of a half type, as a CPU tensor; a few large channels, as activations have."""
    x = rng.standard_normal(shape) * scale
    x[..., rng.integers(0, shape[-1], 2)] *= 8
    return torch.from_numpy(x).to(DT[dtype])


def f64(t):
    return t.double().cpu().numpy()


def cu_of(counts, start=0):
    return torch.tensor(np.concatenate([[start], start + np.cumsum(counts)]), dtype=torch.int32, device=DEV)


class Pair:
    """The library's cache and the oracle's, filled alike."""

    def __init__(self, batch, hq, hkv, dim, code, dtype, columns, seed=0, spare=3, table=None):
        self.rng = np.random.default_rng(seed)
        self.dim, self.hq, self.hkv, self.dtype, self.batch = dim, hq, hkv, dtype, batch
        pages = batch * columns + spare
        if table is None:
            table = self.rng.permutation(pages)[:batch * columns].reshape(batch, columns)
        self.o = O.Cache(batch, hkv, dim, code, dtype, pages, table)
        self.g = B.PagedKV8Cache(batch, hq, hkv, code, pages, table, head_dim=dim, dtype=DT[dtype])
        for t, x in zip(self.g.buffers, (0x7F, 0x7F, 0xFF, 0xFF, 0xFF, 0xFF)):   # e4m3's NaN; NaN scales and residual rows
            t.fill_(x)

    def append(self, counts, rot=None, interleaved=False, start=0, behind=0, scale=1.0, q=False, make=None, advance=True, same=False):
        """One step through both.  Returns q's rows as rotated (float64 oracle)."""
        rows = start + sum(counts) + behind
        make = make or (lambda h: half(self.rng, self.dtype, rows, h, self.dim, scale=scale))
        k, v, qq = make(self.hkv), make(self.hkv), make(self.hq) if q else None
        cu = None if start == behind == 0 and all(c == 1 for c in counts) else cu_of(counts, start)
        most, at = max(max(counts), 1), start
        rotation = None if rot is None else B.Rotation(rot.to(DEV), interleaved=interleaved)
        kd, vd = k.to(DEV), v.to(DEV)
        if q:
            qd = qq.to(DEV)
            q_out = qd if same else torch.full_like(qd, 7.0)
            self.g.append(kd, vd, q=qd, q_out=q_out, cu_tokens=cu, max_tokens=most, rotation=rotation)
        else:
            self.g.append(kd, vd, cu_tokens=cu, max_tokens=most, rotation=rotation)
        want_q = f64(qq) if q and same else np.full((rows, self.hq, self.dim), 7.0)
        for b, n in enumerate(counts):
            kb = f64(k[at:at + n])
            pos = np.clip(np.arange(self.o.lens[b], self.o.lens[b] + n), 0, 10 ** 9 if rot is None else rot.shape[0] - 1)
            if rot is not None and n:
                t = rot.numpy()[pos]
                r = rot.shape[1] // 2
                kb = O.rotate(kb, t[:, :r], t[:, r:], interleaved, self.dtype)
                if q:
                    want_q[at:at + n] = O.rotate(f64(qq[at:at + n]), t[:, :r], t[:, r:], interleaved, self.dtype)
            if n:
                self.o.append(b, kb, f64(v[at:at + n]))
            at += n
        if advance:
            self.g.advance(cu, rows=rows, max_tokens=most)
            self.o.lens = [x + n for x, n in zip(self.o.lens, counts)]
        return (q_out, want_q) if q else None

    def same(self):
        """Every byte of the cache, NaN where nothing was written."""
        kc, vc, ks, vs, kr, vr = self.g.buffers
        kind = torch.int8 if self.g.code == "int8" else torch.float8_e4m3fn
        shape = self.o.k_codes.shape
        for got, want in ((kc.view(kind).reshape(shape), self.o.k_codes),
                          (vc.view(kind).reshape(shape[0], shape[1], shape[3], 128).transpose(2, 3), self.o.v_codes),
                          (ks.view(torch.float32).reshape(shape[:2]), self.o.k_scales), (vs.view(torch.float32).reshape(shape[:2]), self.o.v_scales),
                          (kr.view(DT[self.dtype]).reshape(self.o.k_res.shape), self.o.k_res), (vr.view(DT[self.dtype]).reshape(self.o.v_res.shape), self.o.v_res)):
            got = got.float().cpu().numpy().astype(np.float64)
            if kind == torch.int8 and want is self.o.k_codes or kind == torch.int8 and want is self.o.v_codes:
                got = np.where(np.isnan(want) & (got == 127), np.nan, got)
            assert np.array_equal(got, want, equal_nan=True)
        assert self.g.seq_lens.tolist() == self.o.lens

    def attend(self, counts, scale=None, start=0, behind=0, splits=None, prefix=None, slopes=None, cap=0.0, window=0, q=None, check=True, stream=None):
        """The step's queries (the newest `counts` of what both caches hold and the step brings) through both."""
        rows = start + sum(counts) + behind
        scale = 1 / np.sqrt(self.dim) if scale is None else scale
        q = half(self.rng, self.dtype, rows, self.hq, self.dim) if q is None else q
        cu = None if start == behind == 0 and all(c == 1 for c in counts) else cu_of(counts, start)
        out = torch.full((rows, self.hq, self.dim), 7.0, dtype=DT[self.dtype], device=DEV)
        dev = lambda x, t: None if x is None else torch.tensor(x, dtype=t, device=DEV)   # noqa: E731
        self.g.attn(q.to(DEV), scale, out, cu_tokens=cu, max_tokens=max(max(counts), 1), max_len=max(self.o.lens) + max(counts), softcap=cap,
                    slopes=dev(slopes, torch.float32), window=window, prefix_lens=dev(prefix, torch.int32), num_splits=splits)
        got, at = f64(out), start
        if check:
            assert (got[:start] == 7).all() and (got[start + sum(counts):] == 7).all()
        for b, n in enumerate(counts):
            if n and check:
                length = self.o.lens[b] + n
                want, spread, products, whole = O.attention(self.o, b, f64(q[at:at + n]), self.o.lens[b], scale, cap, slopes, window,
                                                            0 if prefix is None else min(max(prefix[b], 0), length))
                far = np.abs(got[at:at + n] - want) - O.bar(want, spread, products, whole, self.dim, length, self.dtype)
                assert far.max() <= 0, (b, n, length, far.max(), np.unravel_index(far.argmax(), far.shape))
            at += n
        return out


TABLE = B.Rotation.table(6000, 128, device="cpu")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_appended_bytes(code, dtype, dim):
    """Ragged steps of any sizes, some empty, rows of nobody in front and behind: every byte as the oracle has it."""
    p = Pair(4, 6, 2, dim, code, dtype, 6, seed=1)
    for i, counts in enumerate([(1, 1, 1, 1), (126, 0, 128, 300), (1, 127, 1, 1), (1, 1, 1, 1), (0, 130, 255, 84), (1, 1, 128, 1)]):
        for interleaved, r in [(bool(i % 2), (16, 32, 64)[i % 3])]:
            rot = torch.cat([TABLE[:, :r // 2], TABLE[:, 64:64 + r // 2]], 1).contiguous()
            got, want = p.append(counts, rot, interleaved, start=3 * (i % 2), behind=i % 3, q=True, same=i == 4)
            assert np.array_equal(f64(got), want), i
        p.same()
    assert p.g.status.item() == 0


def test_appended_bytes_whole_rotation_and_none():
    p = Pair(2, 4, 1, 128, "e4m3", "bf16", 9, seed=2)
    got, want = p.append((700, 129), TABLE, q=True)
    assert np.array_equal(f64(got), want)
    p.append((77, 300))
    p.append((300, 1))
    p.same()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_blocks_of_zeros_tiny_and_huge_values(code, dtype):
    """Scale 0, subnormals, the half type's largest, negative zeros, ties of the division."""
    p = Pair(1, 2, 1, 64, code, dtype, 6, seed=3)
    t = torch.finfo(DT[dtype])
    for x in (0.0, t.smallest_normal / 4, t.max, 2.0 ** -9):
        block = torch.zeros(128, 1, 64, dtype=DT[dtype])
        if x:
            block = (torch.randint(-8, 9, (128, 1, 64), generator=torch.Generator().manual_seed(4)) / 8.0 * x).to(DT[dtype])
            block[5, 0, 7] = x
        p.append((128,), make=lambda h: block if h == 1 else half(p.rng, dtype, 128, h, 64))   # noqa: B023
    p.same()


def test_steps_in_pieces_and_at_once_leave_the_same_bytes():
    """and so does every order of work inside the call: the same call twice."""
    rng = np.random.default_rng(5)
    k, v = half(rng, "bf16", 777, 3, 128).to(DEV), half(rng, "bf16", 777, 3, 128).to(DEV)
    rot = B.Rotation(TABLE.to(DEV))
    caches = []
    for pieces in ([777], [1] * 3 + [124, 1, 256, 130] + [1] * 263, [777]):
        c = B.PagedKV8Cache(1, 3, 3, "e4m3", 7, [[6, 5, 0, 1, 2, 3]], dtype=torch.bfloat16)
        for i, n in enumerate(pieces):
            at = sum(pieces[:i])
            c.append(k[at:at + n], v[at:at + n], cu_tokens=cu_of([n]), max_tokens=n, rotation=rot)
            c.advance(cu_of([n]), rows=n, max_tokens=n)
        caches.append(c)
    for c in caches[1:]:
        for x, y in zip(caches[0].buffers[:4], c.buffers[:4]):
            assert torch.equal(x, y)
        for x, y in zip(caches[0].buffers[4:], c.buffers[4:]):   # (rows behind the length are anything)
            rows = lambda t: t.view(torch.int16).reshape(3, 128, 128)[:, :777 % 128]   # noqa: E731
            assert torch.equal(rows(x), rows(y))


def test_rows_with_strides_and_queries_in_place():
    """Parts of one projection's output; tensors laid out head by head; positions of their own."""
    rng = np.random.default_rng(6)
    T, Hq, H, D = 200, 8, 2, 64
    qkv = half(rng, "fp16", T, Hq + 2 * H, D).to(DEV)
    pos = torch.from_numpy(rng.integers(0, 6000, T).astype(np.int32)).to(DEV)
    rot = B.Rotation(torch.cat([TABLE[:, :32], TABLE[:, 64:96]], 1).contiguous().to(DEV), positions=pos)
    parts = [qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]]
    whole = [x.contiguous() for x in parts]
    by_head = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in parts]
    results = []
    for q, k, v in (whole, parts, by_head):
        c = B.PagedKV8Cache(2, Hq, H, "int8", 4, [[0, 1], [2, 3]], head_dim=D)
        q_out = torch.empty_like(q)
        c.append(k, v, q=q, q_out=q_out, cu_tokens=cu_of([150, 50]), max_tokens=150, rotation=rot)
        out = torch.empty(T, Hq, D, dtype=torch.float16, device=DEV)
        c.attn(q_out, 0.125, out, cu_tokens=cu_of([150, 50]), max_tokens=150)
        results.append([q_out.clone(), out] + [b.clone() for b in c.buffers])
    c = B.PagedKV8Cache(2, Hq, H, "int8", 4, [[0, 1], [2, 3]], head_dim=D)
    c.append(parts[1], parts[2], q=parts[0], q_out=parts[0], cu_tokens=cu_of([150, 50]), max_tokens=150, rotation=rot)
    results.append([parts[0], results[0][1]] + c.buffers)
    for r in results[1:]:
        for x, y in zip(results[0], r):
            assert torch.equal(x, y)
    t = TABLE.numpy()[pos.cpu().numpy()]
    want = O.rotate(f64(whole[0]), t[:, :32], t[:, 64:96], False, "fp16")
    assert np.array_equal(f64(results[0][0]), want)


def test_bad_lists_tables_and_positions_are_left_out_and_said():
    p = Pair(4, 2, 1, 64, "int8", "fp16", 2, seed=7)
    p.append((100, 100, 100, 100))
    # sequence 1's page for its first block is missing: bit 1, the rest of the step goes on
    p.g.block_table[1, 0] = p.o.table[1, 0] = 99999
    p.append((30, 30, 30, 30))
    p.same()
    assert p.g.status.item() == 2
    out = p.attend((1, 1, 1, 1))
    assert p.g.status.item() == 3 and out.isfinite().all()
    # lists that do not fit: more rows than said, beyond the rows there are, backwards, negative; a negative length
    p.g.status.zero_()
    before = [b.clone() for b in p.g.buffers]
    k = half(p.rng, "fp16", 8, 1, 64).to(DEV)
    q = half(p.rng, "fp16", 8, 2, 64).to(DEV)
    lens = p.g.seq_lens.clone()
    for cu in ([0, 5, 5, 5, 5], [6, 9, 9, 9, 9], [5, 3, 3, 3, 3], [-2, 0, 0, 0, 0]):
        cu = torch.tensor(cu, dtype=torch.int32, device=DEV)
        out = torch.full((8, 2, 64), 7.0, dtype=torch.float16, device=DEV)
        for call in (lambda: p.g.append(k, k, cu_tokens=cu, max_tokens=4), lambda: p.g.attn(q, 0.1, out, cu_tokens=cu, max_tokens=4),   # noqa: B023
                     lambda: p.g.attn(q, 0.1, out, cu_tokens=cu, max_tokens=4, num_splits=2), lambda: p.g.advance(cu, rows=8, max_tokens=4)):   # noqa: B023
            call()
            assert p.g.status.item() == 4
            p.g.status.zero_()
        assert (out == 7).all()
    for bad in (-5, 2 ** 31 - 1):
        p.g.seq_lens.copy_(lens)
        p.g.seq_lens[3] = bad
        one = torch.full((4, 2, 64), 7.0, dtype=torch.float16, device=DEV)
        p.g.attn(q[:4], 0.1, one)
        p.g.advance()
        assert p.g.status.item() == 5 and (one[3] == 7).all() and (one[:3] != 7).any() and p.g.seq_lens[3] == bad   # (bit 0: the missing page)
        p.g.status.zero_()
    assert all(torch.equal(x, y) for x, y in zip(before, p.g.buffers))
    # positions outside of the table: the nearest in it
    rot = TABLE[:, :32].contiguous()
    for pos in (-3, 6000):
        got = [torch.empty_like(q) for _ in range(2)]
        for at, o in ((pos, got[0]), (min(max(pos, 0), 5999), got[1])):
            r = B.Rotation(rot.to(DEV), positions=torch.full((8,), at, dtype=torch.int32, device=DEV))
            p.g.seq_lens.zero_()
            p.g.append(k, k, q=q, q_out=o, cu_tokens=cu_of([2, 2, 2, 2]), max_tokens=2, rotation=r)
            assert p.g.status.item() == (8 if at == pos else 0)
            p.g.status.zero_()
        assert torch.equal(*got)


LENGTHS = [(0, 1), (126, 1), (127, 1), (128, 1), (129, 1), (511, 1), (640, 1), (1300, 1)]


@pytest.mark.parametrize("splits", [None, 1, 3, 40])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_one_token_a_sequence(code, dtype, dim, splits):
    p = Pair(len(LENGTHS), 8, 2, dim, code, dtype, 11, seed=8)
    p.append([n for n, _ in LENGTHS])
    p.append([1] * len(LENGTHS), advance=False)
    p.attend([1] * len(LENGTHS), splits=splits)
    p.attend([1] * len(LENGTHS), splits=splits, cap=5.0, window=200, prefix=[0, 5, 130, 1, 128, 9999, 600, 3], slopes=[0.5, 0.0, -0.02, 0.1, 1.0, 0.01, 2.0, 0.3])
    assert p.g.status.item() == 0


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (5, 1), (16, 1), (17, 1), (40, 2), (64, 8)])
@pytest.mark.parametrize("tokens", [1, 2, 5, 30])
def test_groups_of_any_size(hq, hkv, tokens):
    """Sixteen rows to a product, 128 to a tile: rows that fill them, do not, and go over."""
    p = Pair(3, hq, hkv, 128, "int8", "fp16", 4, seed=9)
    p.append((256 - tokens, 70, 200))
    p.append((tokens, tokens, 1), advance=False)
    for splits in (None, 2):
        p.attend((tokens, tokens, 1), splits=splits)
        p.attend((tokens, tokens, 1), splits=splits, window=90, cap=20.0, prefix=[7, 0, 201], start=2, behind=3)


@pytest.mark.parametrize("splits", [None, 1, 2, 5])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_prompts_and_pieces_of_prompts(code, dtype, dim, splits):
    p = Pair(4, 4, 2, dim, code, dtype, 8, seed=10)
    p.append((0, 300, 128, 512))
    counts = (400, 0, 129, 333)
    p.append(counts, advance=False)
    p.attend(counts, splits=splits, start=5, behind=9)
    p.attend(counts, splits=splits, cap=3.0)
    p.attend(counts, splits=splits, window=130, slopes=[0.1, 0.02, 0.5, -0.01])
    p.attend(counts, splits=splits, prefix=[150, 0, 1000, 5], window=40)
    assert p.g.status.item() == 0


@pytest.mark.parametrize("splits", [None, 1])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_prompts_in_one_split_of_large_tiles(code, dtype, dim, splits):
    """More small tiles (4 sequences, 8 heads, 15 tiles of 32 rows: 480) than a call of one split is given: large ones write the outputs themselves."""
    p = Pair(4, 8, 8, dim, code, dtype, 8, seed=23)
    p.append((0, 300, 128, 512))
    counts = (460, 0, 129, 333)
    p.append(counts, advance=False)
    p.attend(counts, splits=splits, start=5, behind=9)
    p.attend(counts, splits=splits, cap=3.0, scale=-0.2)
    p.attend(counts, splits=splits, window=130, slopes=[0.1, 0.02, 0.5, -0.01, 0.0, 1.0, 0.3, 0.004])
    p.attend(counts, splits=splits, prefix=[150, 0, 1000, 5], window=40)
    assert p.g.status.item() == 0


@pytest.mark.parametrize("scale", [0.0, -0.125, 1.0, 3.0])
def test_scales_of_any_sign_and_peaked_weights(scale):
    p = Pair(2, 4, 2, 64, "int8", "fp16", 5, seed=11)
    p.append((300, 500))
    for counts in ((1, 1), (90, 60)):
        p.append(counts, advance=False)
        p.attend(counts, scale=scale)
        p.attend(counts, scale=scale, cap=30.0)


@pytest.mark.parametrize("counts", [(1, 1), (70, 40)])
@pytest.mark.parametrize("first", [0.0, 1e-4, 300.0])
def test_blocks_whose_values_differ_in_size(first, counts):
    """A first block of zeros, tiny or large values, then zeros, then others: a block's scale is no one else's, and a block of zeros counts
    with its weights."""
    p = Pair(2, 4, 2, 64, "e4m3", "bf16", 8, seed=12)
    for size in (first, 0.0, 1.0, 1e-5, 50.0, 0.0):
        p.append((128, 128), make=lambda h: half(p.rng, "bf16", 256, h, 64, scale=size))   # noqa: B023
    p.append(counts, advance=False, scale=0.01)
    p.attend(counts, scale=0.0)       # every token weighs the same
    p.attend(counts)
    p.attend(counts, window=100, splits=3)


def test_rows_that_see_nothing_are_zeros():
    p = Pair(2, 4, 2, 128, "int8", "fp16", 3, seed=13)
    p.append((127, 254))
    p.append((1, 2))                          # (nothing left in the residuals)
    p.g.block_table.fill_(-1)
    p.o.table[:] = -1
    p.g.seq_lens.copy_(torch.tensor([127, 254], dtype=torch.int32))
    p.o.lens = [127, 254]
    for splits in (1, 4):
        assert (p.attend((1, 2), splits=splits) == 0).all()
    p.g.seq_lens.copy_(torch.tensor([28, 156], dtype=torch.int32))
    p.o.lens = [28, 156]
    for splits in (1, 4):
        assert (p.attend((100, 100), splits=splits) == 0).all()
    assert p.g.status.item() == 1


def test_a_pool_whose_offsets_pass_32_bits():
    """Pages of 2 x 4.6 GB; the last ones are used."""
    pages = 36000
    c = B.PagedKV8Cache(2, 8, 8, "int8", pages, [[0, pages - 1, 7], [pages - 2, pages - 3, 8]],
                        buffers=[torch.empty(pages * 8 * n, dtype=torch.uint8, device=DEV) for n in (128 * 128, 128 * 128, 4, 4)]
                        + [torch.zeros(2 * 8 * 128 * 256, dtype=torch.uint8, device=DEV) for _ in range(2)])
    small = B.PagedKV8Cache(2, 8, 8, "int8", 6, [[0, 3, 4], [1, 2, 5]])
    rng = np.random.default_rng(14)
    k, v, q = (half(rng, "fp16", 600, 8, 128).to(DEV) for _ in range(3))
    outs = []
    for x in (c, small):
        cu = cu_of([280, 320])
        x.append(k, v, cu_tokens=cu, max_tokens=320)
        out = torch.empty(600, 8, 128, dtype=torch.float16, device=DEV)
        outs.append(x.attn(q, 0.1, out, cu_tokens=cu, max_tokens=320))
        x.advance(cu, rows=600, max_tokens=320)
        x.append(k[:2], v[:2])
        outs.append(x.attn(q[:2], 0.1, torch.empty_like(out[:2])))
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


def test_a_long_context():
    """A single sequence of 40000 tokens, by one query and by twenty."""
    p = Pair(1, 4, 1, 128, "e4m3", "fp16", 314, seed=15)
    p.append((40000,), TABLE)
    for n in (1, 20):
        p.append((n,), advance=False)
        p.attend((n,))
        p.attend((n,), window=9000, prefix=[1000], cap=50.0)


@pytest.mark.parametrize("batch,hkv,tokens", [(2, 8, 1), (5, 2, 1), (16, 8, 1), (60, 1, 1), (64, 2, 2), (70, 1, 1), (40, 8, 1)])
def test_ragged_batches_whose_splits_are_dealt_by_length(batch, hkv, tokens):
    """Lengths from nothing to 6000 tokens in wide tables; more workgroups than compute units and fewer; rows of nobody."""
    rng = np.random.default_rng(21)
    lens = [int(6000 * rng.random() ** 3) for _ in range(batch)]
    lens[0], lens[-1] = 6000, 0
    kept = sorted({0, 1, batch // 2, batch - 1})   # (held against the oracle; the others have lengths alone)
    p = Pair(batch, 2 * hkv, hkv, 64, "e4m3", "fp16", 48, seed=22)
    for t in p.g.buffers[:2]:
        t.zero_()
    p.g.k_scales.view(torch.float32).fill_(1.0)
    p.g.v_scales.view(torch.float32).fill_(1.0)
    for t in p.g.buffers[4:]:
        t.zero_()
    p.append([n if b in kept else 0 for b, n in enumerate(lens)])
    p.g.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    step = [tokens if b != 1 else 0 for b in range(batch)]
    k = half(rng, "fp16", sum(step), hkv, 64)
    v = half(rng, "fp16", sum(step), hkv, 64)
    q = half(rng, "fp16", sum(step), 2 * hkv, 64).to(DEV)
    cu = cu_of(step)
    p.g.append(k.to(DEV), v.to(DEV), cu_tokens=cu, max_tokens=tokens)
    outs = []
    for splits in (None, 1, 2, 3, 7):
        for window in (0, 900):
            out = torch.full_like(q, 7.0)
            p.g.attn(q, 0.125, out, cu_tokens=cu, max_tokens=tokens, window=window, num_splits=splits)
            outs.append((window, f64(out)))
    assert p.g.status.item() == 0
    at = np.cumsum([0] + step)
    for b in kept:
        if step[b]:
            rows = slice(at[b], at[b + 1])
            p.o.lens[b] = lens[b]
            p.o.append(b, f64(k[rows]), f64(v[rows]))
            for window, got in outs:
                want, spread, products, whole = O.attention(p.o, b, f64(q[rows]), lens[b], 0.125, window=window)
                far = np.abs(got[rows] - want) - O.bar(want, spread, products, whole, 64, lens[b] + tokens, "fp16")
                assert far.max() <= 0, (b, lens[b], window)


def test_a_stream_of_its_own_and_two_at_once():
    """Two caches on two streams, steps of both under way at the same time."""
    pairs = [Pair(3, 8, 2, 128, "int8", "fp16", 5, seed=s) for s in (16, 17)]
    streams = [torch.cuda.Stream() for _ in pairs]
    data = []
    for p in pairs:
        p.append((300, 400, 500))
        k, v, q = (half(p.rng, "fp16", 3, h, 128).to(DEV) for h in (2, 2, 8))
        data.append((k, v, q, torch.empty_like(q), torch.empty_like(q)))
    torch.cuda.synchronize()
    for _ in range(5):
        for p, (k, v, q, out, _) in zip(pairs, data):   # first on the current stream
            p.g.append(k, v)
            p.g.attn(q, 0.1, out, num_splits=3)
    torch.cuda.synchronize()
    for _ in range(5):
        for p, st, (k, v, q, _, out) in zip(pairs, streams, data):
            with torch.cuda.stream(st):
                p.g.append(k, v)
                p.g.attn(q, 0.1, out, num_splits=3)
            p.g.attn(q, 0.1, out, num_splits=3, stream=st)
    torch.cuda.synchronize()
    for _, _, _, one, two in data:
        assert torch.equal(one, two)


def test_the_first_call_may_be_another_streams():
    """The workspace's counters are zeros for it, over memory that was not, whatever is under way on the current stream."""
    p, like = (Pair(3, 8, 2, 128, "int8", "fp16", 5, seed=21) for _ in range(2))
    for x in (p, like):
        x.append((300, 400, 500))
        x.append((1, 1, 1), advance=False)
    q = half(p.rng, "fp16", 3, 8, 128).to(DEV)
    want, got = torch.empty_like(q), torch.empty_like(q)
    like.g.attn(q, 0.1, want, num_splits=3)
    _, ws = like.g.workspace(3, 1, like.g.max_len, 3)
    other, x = torch.cuda.Stream(), torch.ones(4096, 4096, device=DEV)
    used = torch.full_like(ws, 255)
    torch.cuda.synchronize()
    del used
    for _ in range(20):
        y = x @ x
    p.g.attn(q, 0.1, got, num_splits=3, stream=other)
    torch.cuda.synchronize()
    assert y[0, 0].item() == 4096 and torch.equal(want, got)


def test_a_workspace_does_not_grow_inside_of_a_capture():
    p = Pair(2, 8, 2, 128, "e4m3", "bf16", 5, seed=22)
    p.append((300, 600))
    p.append((1, 1), advance=False)
    q = half(p.rng, "bf16", 2, 8, 128).to(DEV)
    want, got = torch.empty_like(q), torch.zeros_like(q)
    for ready in (False, True):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.zero_()
            if ready:
                p.g.attn(q, 0.1, got, num_splits=3)
            else:
                with pytest.raises(ValueError, match="before it is captured"):
                    p.g.attn(q, 0.1, got, num_splits=3)
        p.g.attn(q, 0.1, want, num_splits=3)
    for _ in range(3):
        graph.replay()
        p.g.attn(q, 0.1, want, num_splits=3)
        torch.cuda.synchronize()
        assert torch.equal(want, got) and want.abs().max().item() > 0
        got.zero_()


def test_decoding_in_a_graph():
    """Two layers that share table and lengths: a step captured once and replayed over a block's end, the program's own work between
    the replays, against the same steps one by one."""
    steps, batch = 12, 3
    rng = np.random.default_rng(18)
    rot = B.Rotation(TABLE.to(DEV))
    ks = [[half(rng, "bf16", batch, 2, 128).to(DEV) for _ in range(4)] for _ in range(steps)]
    qs = [[half(rng, "bf16", batch, 8, 128).to(DEV) for _ in range(2)] for _ in range(steps)]
    start = [half(rng, "bf16", 700, 2, 128).to(DEV) for _ in range(4)]

    def program():
        table = torch.arange(12, dtype=torch.int32, device=DEV).reshape(batch, 4)
        lens = torch.zeros(batch, dtype=torch.int32, device=DEV)
        layers = [B.PagedKV8Cache(batch, 8, 2, "e4m3", 12, table, dtype=torch.bfloat16, seq_lens=lens) for _ in range(2)]
        cu = cu_of([250, 200, 250])
        for i, c in enumerate(layers):
            c.append(start[2 * i], start[2 * i + 1], cu_tokens=cu, max_tokens=250, rotation=rot)
        layers[0].advance(cu, rows=700, max_tokens=250)
        kv = [torch.empty_like(x) for x in ks[0]]
        q = [torch.empty_like(x) for x in qs[0]]
        out = [torch.zeros_like(x) for x in qs[0]]

        def step():
            for i, c in enumerate(layers):
                c.append(kv[2 * i], kv[2 * i + 1], q=q[i], q_out=q[i], rotation=rot)
                c.attn(q[i], 0.088, out[i], max_len=512)
            layers[0].advance()
        return layers, kv, q, out, step

    outs, states = [], []
    for graphed in (False, True):
        layers, kv, q, out, step = program()
        if graphed:
            lens = layers[0].seq_lens.clone()
            step()   # (as captures want it: once before; the workspace is there then)
            layers[0].seq_lens.copy_(lens)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            layers[0].seq_lens.copy_(lens)
        got = []
        for s in range(steps):
            for x, y in zip(kv + q, ks[s] + qs[s]):
                x.copy_(y)
            graph.replay() if graphed else step()
            got += [x.clone() for x in out]
            torch.cuda.synchronize()
        outs.append(got)
        states.append([layers[0].seq_lens] + [b for c in layers for b in c.buffers[:4]])
        assert layers[0].seq_lens.tolist() == [262, 212, 262] and layers[1].status.item() == 0
    assert all(torch.equal(x, y) for x, y in zip(*outs)) and all(torch.equal(x, y) for x, y in zip(*states))


def test_a_model_serves_a_batch():
    """Prompts in pieces, decoding, drafted tokens of which some are taken back: a serving program's calls in a row, each against the oracle."""
    p = Pair(3, 8, 2, 128, "int8", "bf16", 8, seed=19)
    table = TABLE
    for counts in ((256, 100, 0), (256, 28, 300), (40, 128, 5)):
        q, want = p.append(counts, table, q=True, advance=False)
        assert np.array_equal(f64(q), want)
        p.attend(counts, q=q.cpu())
        cu = cu_of(counts)
        p.g.advance(cu, rows=sum(counts), max_tokens=max(counts))
        p.o.lens = [x + n for x, n in zip(p.o.lens, counts)]
    for _ in range(3):
        q, _ = p.append((1, 1, 1), table, q=True, advance=False)
        p.attend((1, 1, 1), q=q.cpu(), window=300)
        p.g.advance()
        p.o.lens = [x + 1 for x in p.o.lens]
    # five drafted tokens, of which two, none and four stay: the lengths are the program's own
    q, _ = p.append((5, 5, 5), table, q=True, advance=False)
    p.attend((5, 5, 5), q=q.cpu(), prefix=[10, 0, 50])
    p.o.lens = [x + n for x, n in zip(p.o.lens, (2, 0, 4))]
    p.g.seq_lens.copy_(torch.tensor(p.o.lens, dtype=torch.int32))
    q, _ = p.append((1, 1, 1), table, q=True, advance=False)
    p.attend((1, 1, 1), q=q.cpu())
    p.same()
    assert p.g.status.item() == 0


def test_attention_reads_queries_behind_any_stride_and_repeats_itself():
    p = Pair(2, 8, 2, 64, "e4m3", "fp16", 6, seed=20)
    p.append((200, 700))
    for counts in ((1, 1), (60, 9)):
        p.append(counts, advance=False)
        rows = sum(counts)
        q = half(p.rng, "fp16", rows, 8, 64).to(DEV)
        wide = torch.zeros(rows, 12, 64, dtype=torch.float16, device=DEV)
        wide[:, 2:10] = q
        cu = None if counts == (1, 1) else cu_of(counts)
        outs = [p.g.attn(x, 0.1, torch.empty_like(q), cu_tokens=cu, max_tokens=max(counts), num_splits=s)
                for s in (1, 4) for x in (q, q, wide[:, 2:10], q.transpose(0, 1).contiguous().transpose(0, 1))]
        assert all(torch.equal(outs[i], outs[i // 4 * 4]) for i in range(8))


def test_the_entry_points_without_the_class():
    """Plain addresses through the C interface, no status word."""
    L = B.lib()
    c = B.PagedKV8Cache(1, 2, 1, "int8", 2, [[1, 0]], head_dim=64)
    c.desc.status = None
    k = torch.ones(130, 1, 64, dtype=torch.float16, device=DEV)
    q = torch.ones(130, 2, 64, dtype=torch.float16, device=DEV)
    out = torch.zeros_like(q)
    cu = cu_of([130])
    st = torch.cuda.current_stream().cuda_stream
    rows = B.bd_rows(k.data_ptr(), 64, 64)
    assert L.bd_paged8_append(ctypes.byref(c.desc), ctypes.byref(rows), ctypes.byref(rows), None, None, cu.data_ptr(), 130, 130, None, st) == 0
    s, qr = B.bd_scores(0.125, 0.0, None, None, 0), B.bd_rows(q.data_ptr(), 128, 64)
    assert L.bd_paged8_attn(ctypes.byref(c.desc), ctypes.byref(qr), cu.data_ptr(), 130, 130, ctypes.byref(s), 1, None, out.data_ptr(), st) == 0
    assert L.bd_paged8_advance(ctypes.byref(c.desc), cu.data_ptr(), 130, 130, st) == 0
    assert (out - 1).abs().max().item() <= 2 ** -10 and c.seq_lens.item() == 130
