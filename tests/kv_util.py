"""Shared helpers of the paged-cache tests: pools, page tables and their copies for the oracle."""
import numpy as np

F32_U, BF16_U, E4M3_U = 2.0 ** -24, 2.0 ** -8, 2.0 ** -4  # relative half steps


def bf16(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16)


def make_table(rng, lens, page_size, spare=2):
    """Page table [B, width] with the pages in random order, -1 past each end, and the page count."""
    need = [-(-n // page_size) for n in lens]
    ids = rng.permutation(sum(need) + spare)
    width = max(1, max(need, default=1))
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, sum(need) + spare


class Pool:
    """A cache on the GPU and the same values on the host.  Every slot that no
    sequence uses is poisoned with NaN."""

    def __init__(self, torch, sdq, rng, lens, heads, page_size, dim, dtype="bf16", layout="hnd", track=False, poison=True):
        self.table, pages = make_table(rng, lens, page_size)
        self.lens, self.page_size, self.heads, self.dim, self.pages = list(lens), page_size, heads, dim, pages
        shape = (pages, heads, page_size, dim)
        self.e4m3 = dtype == "e4m3"
        k, v = (torch.from_numpy(rng.standard_normal(shape).astype(np.float32)) for _ in range(2))
        k[..., ::7] *= 3
        used = np.zeros((pages, page_size), bool)
        for b, n in enumerate(lens):
            t = np.arange(n)
            used[self.table[b][t // page_size], t % page_size] = True
        unused = torch.from_numpy(~used)[:, None, :].expand(pages, heads, page_size)
        self.ks = self.vs = None
        nan = float("nan") if poison else 0.0
        if self.e4m3:
            k, v = (t * 40 for t in (k, v))
            self.ks, self.vs = (torch.from_numpy(rng.uniform(0.5, 1.5, shape[:3]).astype(np.float32) / 40).masked_fill(unused, nan) for _ in range(2))
            k, v = (t.clamp(-448, 448).masked_fill(unused[..., None], nan).to(torch.float8_e4m3fn) for t in (k, v))
        else:
            k, v = (t.masked_fill(unused[..., None], nan).to(torch.bfloat16) for t in (k, v))
        self.k, self.v = k.float().numpy().copy(), v.float().numpy().copy()
        self.position = rng.integers(0, 1000, shape[:3]).astype(np.int32) if track else None
        self.weight = rng.exponential(1.0, shape[:3]).astype(np.float32) if track else None

        def place(t):
            t = t.cuda()
            if layout == "nhd":  # [pages, page_size, heads, dim] in memory
                raw = t.view(torch.uint8) if self.e4m3 else t
                return raw.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3).view(t.dtype)
            if layout == "wide":  # rows and heads with gaps between them, NaN in the gaps
                raw = t.view(torch.uint8) if self.e4m3 else t
                big = torch.full((pages + 1, heads + 1, page_size + 1, dim + 16), 0x7F if self.e4m3 else float("nan"), dtype=raw.dtype, device="cuda")
                big[:pages, :heads, :page_size, :dim] = raw
                return big[:pages, :heads, :page_size, :dim].view(t.dtype) if not self.e4m3 else big.view(torch.float8_e4m3fn)[:pages, :heads, :page_size, :dim]
            return t

        dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
        put = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.cache = sdq.KVCache(place(k), place(v), put(self.ks), put(self.vs), dev(self.position), dev(self.weight))
        self.table_gpu = torch.from_numpy(self.table).cuda()
        self.lens_gpu = torch.tensor(self.lens, dtype=torch.int32).cuda()

    def rows(self, oracle, which, b, head):
        pool, scale = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        return oracle.gather(pool, self.table[b], self.lens[b], head, self.page_size, None if scale is None else scale.numpy())


def attn_tolerance(ref, T, D, out_u, split_u):
    """Error bounds of the attention kernel's outputs, from its arithmetic.
    Scores: D products and their sum in fp32 (D + 4 roundings of the sum of the
    magnitudes: the products, their order of addition, a scale per row and the
    softmax scale), then exp2 of a difference (a rounding of the score, one of
    the maximum, the instruction's own).  Probabilities: twice that (numerator
    and sum), the sum's additions (each lane adds at most T / 4 of them, waves and
    ranges join at most T / 32 + 64), 16 for the exponentials.  Outputs: the
    terms of p, the additions, the final rounding."""
    dz = (D + 4) * F32_U * ref["score_size"] + 4 * F32_U * (np.abs(np.where(np.isfinite(ref["lse"]), ref["lse"], 0)) + ref["score_size"])
    sums = (T / 4 + T / 32 + 80) * F32_U
    rel = 2 * dz + 2 * sums + 16 * F32_U
    out = (rel + split_u)[:, None] * ref["out_size"] + out_u * np.abs(ref["out"]) + 1e-30
    lse = dz + sums + 8 * F32_U + 4 * F32_U * np.abs(np.where(np.isfinite(ref["lse"]), ref["lse"], 0))
    p = rel[:, None] * ref["p"]
    return out, lse, p
