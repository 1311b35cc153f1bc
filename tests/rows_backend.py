"""The oracle's tape backend with the row operators: layer normalisation, dropout, sampling (float64 NumPy arrays)."""
import numpy as np

from oracle import rows as R
from oracle_backend import OracleBackend


class RowsBackend(OracleBackend):
    def dropout(self, x, y, ratio, rng, site, residual=None):
        self.calls.append(("dropout", site))
        keep = self._keep(x, ratio, rng, site)
        y[...] = np.where(keep, x / (1.0 - ratio), 0.0) + (0.0 if residual is None else residual)

    @staticmethod
    def _keep(x, ratio, rng, site):
        if ratio == 0.0:
            return np.ones(x.shape, bool)
        return R.mask(x.shape[0], x.shape[1], ratio, int(rng[0]) % 2 ** 64, int(rng[1]), site)

    def rng_advance(self, rng, steps):
        rng[1] += steps

    def layer_norm_fwd(self, x, y, gamma, beta, eps, mean, rstd):
        self.calls.append(("layer_norm_fwd", None))
        y[...], mean[...], rstd[...] = R.layer_norm(x, gamma, beta, eps)

    def layer_norm_bwd(self, dy, x, mean, rstd, dx, gamma, dgamma, dbeta):
        self.calls.append(("layer_norm_bwd", None))
        for out, v in zip((dx, dgamma, dbeta), R.layer_norm_bwd(dy, x, mean, rstd, gamma)):
            if out is not None:
                out[...] = v

    def residual_norm_fwd(self, x, residual, s, y, gamma, beta, eps, mean, rstd, ratio, rng, site):
        self.calls.append(("residual_norm_fwd", site))
        s[...] = residual + np.where(self._keep(x, ratio, rng, site), x / (1.0 - ratio), 0.0)
        y[...], mean[...], rstd[...] = R.layer_norm(s, gamma, beta, eps)

    def residual_norm_bwd(self, dy, ds, s, mean, rstd, dresidual, dx, gamma, dgamma, dbeta, ratio, rng, site):
        self.calls.append(("residual_norm_bwd", site))
        t, dg, db = R.layer_norm_bwd(dy, s, mean, rstd, gamma)
        t = t if ds is None else t + ds
        for out, v in ((dresidual, t), (dx, np.where(self._keep(s, ratio, rng, site), t / (1.0 - ratio), 0.0)), (dgamma, dg), (dbeta, db)):
            if out is not None:
                out[...] = v

    def sample(self, logits, u, out, temperature=None, top_k=None, top_p=None, min_p=None):
        self.calls.append(("sample", None))
        out[...] = R.sample(logits, u, temperature, top_k, top_p, min_p)
