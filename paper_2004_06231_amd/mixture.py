"""Mixture of EiNets (Sec. 4.2: one EiNet per cluster, the cluster proportions as coefficients) whose samples are routed
to their components.

The density of a sample needs every component (einet_mixture_logp).  Everything else a component does for the samples
that are its own: they are sorted by component (einet_sort), carried to contiguous rows (einet_dispatch), each component
works on its rows, and what it answers is carried back, weighted where a sample has several components (einet_combine).
Which components a sample has is decided by its posterior (einet_route), or drawn from it (einet_choose).
"""
import contextlib
import math

from .binding import (einet_choose, einet_combine, einet_dispatch, einet_mixture_logp, einet_route, einet_route_backward,
                      einet_sort)


class Mixture:
    """components: bound EiNet models over the same variables; log_coef: float32 [n_components] or None for equal ones.
    streams: torch streams that the components' work is spread over (the current stream alone by default); a model that is
    several components has all its work on one of them."""

    def __init__(self, components, log_coef=None, streams=None):
        import torch
        self._torch = torch
        self.components = list(components)
        assert self.components, "a mixture needs a component"
        self.device = self.components[0].device
        n = len(self.components)
        self.log_coef = self._torch.full((n,), -math.log(n), dtype=self._torch.float32, device=self.device)
        if log_coef is not None:
            self.log_coef.copy_(self._torch.as_tensor(log_coef))
        self.streams = list(streams or [])
        # (a model's workspace holds one call at a time: its calls follow each other on one stream)
        self._first_of_model = [next(i for i, o in enumerate(self.components) if o is m) for m in self.components]

    @contextlib.contextmanager
    def _beside_each_other(self):
        """Yields a function of a component's number: the context in which its work is enqueued.  The work starts behind
        what the current stream holds, and the current stream goes on behind all of it."""
        if not self.streams:
            yield lambda c: contextlib.nullcontext()
            return
        here = self._torch.cuda.current_stream(self.device)
        for s in self.streams:
            s.wait_stream(here)
        try:
            yield lambda c: self._torch.cuda.stream(self.streams[self._first_of_model[c] % len(self.streams)])
        finally:
            for s in self.streams:
                here.wait_stream(s)

    def component_logp(self, x, mask=None):
        """[n_components, N] log-densities of every sample under every component; mask: uint8 [D] or [N, D] or None."""
        N = x.shape[0]
        rows = self._torch.empty(len(self.components), N, dtype=self._torch.float32, device=self.device)
        with self._beside_each_other() as at:
            for c, m in enumerate(self.components):
                with at(c):
                    for b in range(0, N, m.max_batch):
                        e = min(N, b + m.max_batch)
                        m.logp(x[b:e], mask[b:e] if mask is not None and mask.dim() == 2 else mask, rows[c, b:e])
        return rows

    def logp(self, x, mask=None):
        """[N] log-density of the mixture."""
        if x.shape[0] == 0:
            return self._torch.empty(0, dtype=self._torch.float32, device=self.device)
        return einet_mixture_logp(self.component_logp(x, mask), self.log_coef)

    def route(self, x, mask=None, top=1, renormalise=True):
        """ids [N, top], weights [N, top], logp [N]: the most probable components of every sample given its observed variables."""
        return einet_route(self.component_logp(x, mask), self.log_coef, top, renormalise)

    def _segments(self, ids):
        """place, and (component, first row, last row + 1) of the components that have rows.  Synchronises: how many samples a
        component gets is an argument of the calls that follow."""
        first, place = einet_sort(ids, len(self.components))
        bounds = first.tolist()
        return place, [(c, bounds[c], bounds[c + 1]) for c in range(len(self.components)) if bounds[c] < bounds[c + 1]]

    def em_epoch(self, x, mask=None, batch=None, step=0.5, u=None, ids=None, **em):
        """One pass of hard EM: every sample goes to one component, which runs einet_em_epoch on its samples in their order.
        The component is the most probable one, or with u (float32 [N] uniforms) drawn from the posterior, or given by ids
        (int32 [N]; -1: the sample is left out, as is one that no component has a density for).  The coefficients move by
        `step` towards the posteriors' means over the samples before the pass (Eq. 7-9 with the mixture's own E-step).  Returns
        ids and, per sample, the log-density under its component at the time it was visited (0 for those left out).  batch, em:
        as in einet_em_epoch."""
        N = x.shape[0]
        logp = self._torch.zeros(N, dtype=self._torch.float32, device=self.device)
        if N == 0:
            return self._torch.empty(0, dtype=self._torch.int32, device=self.device), logp
        rows = self.component_logp(x, mask)
        if ids is None:
            if u is None:
                ids = einet_route(rows, self.log_coef, 1)[0].view(N)
            else:
                # (log-densities are in the thousands, where float32 would round the coefficients away: the sums, and their
                # differences from the largest of the components that take part, are formed in float64 as einet_route does)
                t = rows.double() + self.log_coef.double()[:, None]
                t = self._torch.where(t.isnan(), -math.inf, t)
                largest = t.amax(0)
                rest = t - self._torch.where(largest.isfinite(), largest, 0.0)
                ids = einet_choose(rest.float().t().contiguous(), u)[0]
        place, segments = self._segments(ids.view(N, 1))
        counts = einet_route_backward(rows, self.log_coef, None, None, None, self._torch.ones_like(logp))[1]
        mine = einet_dispatch(x, place)
        masks = einet_dispatch(mask, place) if mask is not None and mask.dim() == 2 else None
        visited = self._torch.empty(N, 1, dtype=self._torch.float32, device=self.device)
        with self._beside_each_other() as at:
            for c, lo, hi in segments:
                with at(c):
                    self.components[c].em_epoch(mine[lo:hi], masks[lo:hi] if masks is not None else mask, batch=batch, step=step,
                                                logp=visited[lo:hi], **em)
        total = counts.sum()
        shares = self._torch.where(total > 0, counts / total, self.log_coef.exp())
        self.log_coef.copy_(self._torch.log((1.0 - step) * self.log_coef.exp() + step * shares))
        einet_combine(visited, place, out=logp.view(N, 1))
        return ids, logp

    def _draw(self, segments, rows, u, noise, x=None, mask=None):
        """Fills `rows` [n, D, C] with the components' samples: segment by segment, max_batch rows at a time."""
        with self._beside_each_other() as at:
            for c, lo, hi in segments:
                m = self.components[c]
                st = m.structure()
                n_u = int(st["num_partitions"]) + int(st["num_regions"])
                with at(c):
                    for b in range(lo, hi, m.max_batch):
                        e = min(hi, b + m.max_batch)
                        m.sample(e - b, u[:n_u, b:e].contiguous(), None if noise is None else noise[b:e],
                                 None if x is None else x[b:e], mask[b:e] if mask is not None and mask.dim() == 2 else mask, rows[b:e])

    def choices(self):
        """Rows of the uniforms that a sample from any of the components needs."""
        return max(int(m.structure()["num_partitions"]) + int(m.structure()["num_regions"]) for m in self.components)

    def sample(self, u_component, u, noise=None, temperature=1.0, top_p=1.0):
        """[N, D, C] samples of the mixture.  u_component: float32 [N] uniforms that draw the components from the coefficients
        (which temperature and top_p sharpen); u: float32 [choices(), N], noise: float32 [N, D, C] or None, both as in
        einet_sample, in the order of the samples sorted by component."""
        N = u_component.shape[0]
        m = self.components[0]
        shape = (int(m.structure()["num_vars"]), m.channels)
        ids, _ = einet_choose(self.log_coef[None].expand(N, -1), u_component, temperature=temperature, top_p=top_p)
        place, segments = self._segments(ids.view(N, 1))
        rows = self._torch.empty((N,) + shape, dtype=self._torch.float32, device=self.device)
        self._draw(segments, rows, u, noise)
        return einet_combine(rows, place)

    def inpaint(self, x, mask, u, noise=None, top=1):
        """[N, D, C]: the observed variables (mask 1; uint8 [D] or [N, D]) as they are, the others as the `top` most probable
        components given the observed ones complete them, weighted by their shares of the posterior (zeros where no component has a
        density for the observed ones).  u: float32
        [choices(), N * top], noise: float32 [N * top, D, C] or None for leaf means, both as in einet_sample, in the order of
        the slots sorted by component."""
        ids, weights, _ = self.route(x, mask, top)
        place, segments = self._segments(ids)
        mine = einet_dispatch(x, place)
        masks = einet_dispatch(mask, place) if mask.dim() == 2 else mask
        rows = self._torch.empty_like(mine)
        self._draw(segments, rows, u, noise, mine, masks)
        out = einet_combine(rows, place, weights)
        # (a weighted sum of an observed value with itself is off by a rounding)
        observed = (mask if mask.dim() == 2 else mask[None])[:, :, None] != 0
        return self._torch.where(observed, x, out)
