"""Batches over a paged cache for the tests: NumPy inputs whose values are exact in
the working type, the calls on the GPU, and how far a result may be.

Every slot that no run owns holds NaN, and so do query rows of no sequence; table
entries past a run's tokens hold -1.
"""
import numpy as np
import torch

from oracle import cache as oracle_cache
from oracle.rounding import round_bf16
from paper_2609_13804_amd import binding as sp

U32 = 2.0 ** -24                       # half a step of float32, relative
HALF_STEP = {"f32": U32, "bf16": 2.0 ** -8}


def torch_type(dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def device(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to("cuda", torch_type(dtype))


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def offsets(counts):
    return np.concatenate([[0], np.cumsum(np.asarray(counts, np.int64))])


class Batch:
    """counts, lens: rows and tokens of every sequence; prefix: tokens of every group's
    prefix, cuts: the groups' sequences (len(prefix) + 1 of them)."""

    def __init__(self, counts, lens, heads=(8, 2), D=128, page=16, dtype="bf16", layout="packed", prefix=(),
                 cuts=(), seed=0, spare=3, pad=0, q_scale=2.0):
        rng = np.random.default_rng(seed)
        self.exact_type = (lambda a: np.asarray(a, np.float32).astype(np.float64)) if dtype == "f32" else \
            (lambda a: round_bf16(np.asarray(a, np.float64)))
        self.counts, self.lens = list(counts), list(lens)
        self.prefix, self.cuts = list(prefix), list(cuts)
        self.Hq, self.Hk = heads
        self.D, self.page, self.dtype, self.layout = D, page, dtype, layout
        self.S, self.rng = len(self.counts), rng
        most = max(self.counts, default=0)
        self.per_seq = most + pad if layout == "padded" else 0
        self.first = [s * self.per_seq for s in range(self.S)] if layout == "padded" else \
            [int(f) for f in offsets(self.counts)[:-1]]
        self.rows = self.S * self.per_seq if layout == "padded" else int(sum(self.counts)) + pad
        self.seq_info = np.asarray(self.counts if layout == "padded" else offsets(self.counts), np.int32)
        runs = self.lens + self.prefix
        need = [-(-n // page) for n in runs]
        self.pages = sum(need) + spare
        order = rng.permutation(self.pages)
        at = offsets(need)
        pages = [order[at[i]:at[i + 1]] for i in range(len(runs))]
        wide = max(need, default=0) + 2
        fill = lambda rows: np.asarray([list(r) + [-1] * (wide - len(r)) for r in rows], np.int32).reshape(
            len(rows), wide)
        self.tables, self.prefix_tables = fill(pages[:self.S]), fill(pages[self.S:])
        shape = (self.pages, self.Hk, page, D)
        self.k_cache, self.v_cache = np.full(shape, np.nan), np.full(shape, np.nan)
        for table, n in zip(pages, runs):
            for p in range(n):
                where = table[p // page], slice(None), p % page
                self.k_cache[where] = self.exact_type(rng.standard_normal((self.Hk, D)))
                self.v_cache[where] = self.exact_type(rng.standard_normal((self.Hk, D)))
        self.q = self.values((self.rows, self.Hq, D), q_scale)
        self.scale = float(np.float32(D ** -0.5))

    def live(self):
        return np.concatenate([np.arange(f, f + n) for f, n in zip(self.first, self.counts)] +
                              [np.zeros(0, np.int64)]).astype(np.int64)

    def values(self, shape, scale=1.0):
        """Rows of the batch; NaN in the rows of no sequence."""
        out = np.full(shape, np.nan)
        rows = self.live()
        out[rows] = self.exact_type(scale * self.rng.standard_normal((len(rows),) + shape[1:]))
        return out

    # ---- the calls' structs (kept alive here)
    def code(self):
        return sp.SP_F32 if self.dtype == "f32" else sp.SP_BF16

    def upload(self, max_rows=None, max_len=None, max_prefix=None):
        self.d_info, self.d_lens, self.d_tables = ints(self.seq_info), ints(self.lens), ints(self.tables)
        self.d_k, self.d_v = device(self.k_cache, self.dtype), device(self.v_cache, self.dtype)
        self.dims = sp.cache_dims(self.Hq, self.Hk, self.D, self.code(), self.page, self.pages)
        layout = sp.SP_LAYOUT_PADDED if self.layout == "padded" else sp.SP_LAYOUT_PACKED
        self.c_rows = sp.cache_rows(self.rows, layout, self.per_seq, self.d_info,
                                    max(self.counts, default=0) if max_rows is None else max_rows)
        self.c_runs = sp.cache_runs(self.d_tables, self.d_lens,
                                    max(self.lens, default=0) if max_len is None else max_len)
        self.c_prefix = self.d_off = None
        if self.prefix:
            self.d_ptables, self.d_plens = ints(self.prefix_tables), ints(self.prefix)
            self.d_off = ints(self.cuts)
            self.c_prefix = sp.cache_runs(self.d_ptables, self.d_plens,
                                          max(self.prefix) if max_prefix is None else max_prefix)

    def attend(self, see_all=False, lse=True, ld_extra=0, stream=None, check=True):
        """(o [rows, heads, D] float64, lse) with 7.0 in the places that were not written."""
        ld = self.Hq * self.D + ld_extra
        q = torch.full((self.rows, ld), float("nan"), dtype=torch_type(self.dtype), device="cuda")
        q[:, :self.Hq * self.D] = device(self.q, self.dtype).view(self.rows, -1)
        o = torch.full((self.rows, self.Hq, self.D), 7.0, dtype=torch_type(self.dtype), device="cuda")
        z = torch.full((self.rows, self.Hq), 7.0, dtype=torch.float32, device="cuda") if lse else None
        nbytes = sp.stepprune_cache_workspace_bytes(self.dims, self.c_rows, self.c_runs, self.c_prefix)
        assert nbytes > 0
        ws = torch.full((nbytes,), 0xff, dtype=torch.uint8, device="cuda")     # NaN wherever nothing is written
        ws[:256] = 0
        torch.cuda.synchronize()
        sp.stepprune_cache_attend(self.dims, q, ld, self.c_rows, self.c_runs, self.c_prefix, self.d_off,
                                  self.scale, sp.SP_ATTEND_ALL if see_all else 0, self.d_k, self.d_v, o, z, ws,
                                  nbytes, stream=stream)
        torch.cuda.synchronize()
        if check:
            code = sp.stepprune_read_device_error(ws)
            assert code == sp.SP_DEV_OK, code
        self.ws = ws
        return o.double().cpu().numpy(), None if z is None else z.double().cpu().numpy()

    # ---- what comes out, and how far it may be
    def oracle(self, see_all=False, v_cache=None):
        return oracle_cache.attend(self.q, self.k_cache, self.v_cache if v_cache is None else v_cache, self.first,
                                   self.counts, self.tables, self.lens, self.scale, self.prefix_tables, self.prefix,
                                   self.cuts, see_all)

    def bounds(self, o, lse, see_all=False):
        """How far o and lse may be from the definition, element by element.

        A score is a float32 sum of D products: off by at most (D + 2) U32 times the sum
        of their sizes, which is below |q| |k|; scaling and the exponent's product add 4
        U32 of its own size, below scale |q| |k| too; so e = (D + 6) U32 scale |q| max |k|.
        A weight is then off by a factor within exp(e), and by 2^-21 for the exponential
        (2 in the last place, and rescalings); its sum over N keys by N U32 more, and so
        is the sum over the values; joining up to 64 parts adds 128 U32.  A weight is
        rounded to the working type before it meets its value (float32: it is there
        already).  All of that is relative to A = sum_j p_j |v_j|; the output is rounded
        once.  lse takes e, the sum's error and 4 U32 of its size."""
        A, _ = self.oracle(see_all, np.abs(self.v_cache))
        norm = np.nanmax(np.sqrt((self.k_cache ** 2).sum(-1))) if np.isfinite(self.k_cache).any() else 0.0
        e = (self.D + 6) * U32 * self.scale * np.sqrt((self.q ** 2).sum(-1)) * norm
        N = max(self.lens, default=0) + max(self.prefix, default=0)
        sums = 2 * (N + 128) * U32 + 2.0 ** -20
        weight = HALF_STEP[self.dtype] if self.dtype == "bf16" else 0.0
        rel = np.expm1(2 * e) + sums + weight
        tol_o = (A * rel[..., None] * (1 + HALF_STEP[self.dtype]) + HALF_STEP[self.dtype] * np.abs(o) + 1e-30)
        tol_l = e + sums + 4 * U32 * np.abs(np.where(np.isfinite(lse), lse, 0.0))
        return tol_o, tol_l

    def check(self, got_o, got_lse, see_all=False):
        o, lse = self.oracle(see_all)
        tol_o, tol_l = self.bounds(o, lse, see_all)
        rows = self.live()
        other = np.setdiff1d(np.arange(self.rows), rows)
        assert (got_o[other] == 7.0).all()                    # rows of no sequence are left alone
        d = np.abs(got_o[rows] - o[rows])
        assert (d <= tol_o[rows]).all(), (np.nanmax(d / tol_o[rows]), np.isnan(d).any())
        if got_lse is not None:
            assert (got_lse[other] == 7.0).all()
            empty = np.isneginf(lse[rows])
            assert (np.isneginf(got_lse[rows]) == empty).all()
            dl = np.abs(np.where(empty, 0.0, got_lse[rows]) - np.where(empty, 0.0, lse[rows]))
            assert (dl <= tol_l[rows]).all(), np.nanmax(dl / tol_l[rows])
