"""Helpers of the prompt-pass tests: packed sequences with their inputs, the
library's calls on them, and the comparison with the fp64 oracle."""
import numpy as np
import torch

from oracle import prompt as O
from paper_2607_16673_amd import binding as B

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def starts_of(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32)


class Prompt:
    """Random inputs of a prefill on the GPU.  `before` and `behind`: rows of no sequence."""

    def __init__(self, lens, heads=2, k_heads=None, dk=128, dv=128, dtype="bf16", family="gdn", fused=False, fresh=False,
                 seed=0, before=0, behind=0, alpha=None, beta=None):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g)
        self.lens, self.family, self.dt = list(lens), family, DT[dtype]
        self.B, self.H, self.Hk, self.dk, self.dv = len(lens), heads, k_heads or heads, dk, dv
        self.starts = starts_of(lens, before)
        T = self.T = int(self.starts[-1]) + behind
        widths = [self.Hk * dk, self.Hk * dk, heads * dv]
        unit = lambda: torch.nn.functional.normalize(rand(T, self.Hk, dk), dim=-1).flatten(1)
        parts = [unit(), unit(), rand(T, heads * dv)]
        if fused:  # behind 16 elements of something else
            row = torch.cat([rand(T, 16)] + parts, 1).to(self.dt).cuda()
            parts = row[:, 16:].split(widths, 1)
        else:
            parts = [p.to(self.dt).cuda() for p in parts]
        self.q, self.k = (p.unflatten(1, (self.Hk, dk)) for p in parts[:2])
        self.v = parts[2].unflatten(1, (heads, dv))
        gate = lambda x: x.float().contiguous().cuda()
        self.alpha = None if family == "deltanet" else gate(torch.sigmoid(2 + 3 * torch.rand(T, heads, generator=g))
                                                            if alpha is None else alpha(T, heads, g))
        self.beta = None if family == "decay" else gate(torch.sigmoid(rand(T, heads)) if beta is None else beta(T, heads, g))
        self.state = None if fresh else (0.1 * rand(self.B, heads, dk, dv)).cuda()
        self.start = torch.from_numpy(self.starts).cuda()

    def outputs(self, fill=7.0):
        return (torch.full((self.T, self.H, self.dv), fill, dtype=self.dt, device="cuda"),
                torch.full((self.B, self.H, self.dk, self.dv), fill, device="cuda"),
                torch.full((self.B,), 99, dtype=torch.int32, device="cuda"))

    def workspace(self):
        return B.prefill_workspace(self.q, self.v, self.B, family=self.family)

    def run(self, out=None, state_out=None, status=None, **over):
        made = self.outputs()
        out = made[0] if out is None else out
        state_out = made[1] if state_out is None else state_out
        status = made[2] if status is None else status
        kw = dict(state=self.state, workspace=self.workspace(), status=status, family=self.family)
        kw.update(over)
        B.sla_prefill(self.q, self.k, self.v, self.alpha, self.beta, self.start, out, state_out, **kw)
        return out, state_out, status

    def exact(self):
        return O.prefill(f64(self.state), f64(self.q), f64(self.k), f64(self.v), f64(self.alpha), f64(self.beta),
                         self.starts, self.family)

    def check(self, got, want=None):
        """Outputs, states and status against the oracle.

        State and fp32 outputs: the library's fp32 bar, 1e-5 of the largest value.  A
        token's sums of d_k products and of up to 64 corrections are off by some
        2^-24 sqrt(d_k + 64) = 8e-7 of their terms, a decay of 64 factors by 64 x
        2^-24 = 4e-6 at most, and the steps are contractions, so errors of a token
        do not grow over later ones.  bf16 outputs: half a step, 2^-8 of the value,
        and 2^-14 of the largest for sums of products that keep 16 bits (2^-17 of
        their terms)."""
        out, state_out, status = got
        o, s = self.exact() if want is None else want
        torch.cuda.synchronize()
        assert status.eq(0).all()
        close(state_out, s)
        inside = ~np.isnan(o).all((1, 2))
        assert (f64(out)[~inside] == 7.0).all(), "rows of no sequence were written"
        close(out[torch.from_numpy(inside).cuda()], o[inside])


def close(got, want):
    """|got - want| within a rounding of got's type and the sums' error (Prompt.check)."""
    x = f64(got)
    assert np.isfinite(x).all()
    top = float(np.max(np.abs(want))) if want.size else 0.0
    bound = 1e-5 * top if got.dtype == torch.float32 else 2.0 ** -8 * np.abs(want) + 2.0 ** -14 * top
    assert (np.abs(x - want) <= bound).all(), float(np.max(np.abs(x - want) / np.maximum(bound, 1e-300)))
