"""The oracle's tape backend with the gated recurrence, scaled embeddings and adjusted logits (float64 NumPy arrays)."""
import numpy as np

from oracle import recurrent as R
from rows_backend import RowsBackend


class RecurrentBackend(RowsBackend):
    @staticmethod
    def _halves(z, n_steps):
        z = z.reshape(n_steps, z.shape[0] // n_steps, z.shape[1])
        H = z.shape[2] // 2
        return z[:, :, :H], z[:, :, H:]

    def gated_scan_fwd(self, z, y, h0, h_last, keep, lengths, kind, n_steps):
        self.calls.append(("gated_scan_fwd", keep))
        out, states, _ = R.gated_scan(*self._halves(z, n_steps), h0, kind, lengths)
        y[...] = out.reshape(y.shape)
        h_last[...] = states[-1]
        return states[:-1:16] if keep else None

    def gated_scan_bwd(self, z, states, dy, dz, dh_last, dh0, lengths, kind, n_steps):
        self.calls.append(("gated_scan_bwd", None))
        gate, x = self._halves(z, n_steps)
        (dg, dx, d0), _ = R.gated_scan_bwd(gate, x, states[0], dy.reshape(gate.shape), dh_last, kind, lengths)
        dz[...] = np.concatenate([dg, dx], 2).reshape(dz.shape)
        if dh0 is not None:
            dh0[...] = d0

    def embed_scaled_fwd(self, table, ids, out, scale):
        self.calls.append(("embed_scaled_fwd", None))
        out[...] = R.embed_scaled(table, ids, scale)

    def embed_sorted_bwd(self, ids, dout, dtable, scale, accumulate):
        self.calls.append(("embed_sorted_bwd", accumulate))
        g, _ = R.embed_scaled_bwd(ids, dout, len(dtable), scale)
        dtable[...] = dtable + g if accumulate else g

    def logits_adjust(self, logits, out, **k):
        self.calls.append(("logits_adjust", None))
        if k.get("allowed") is not None:
            k["allowed"] = np.asarray(k["allowed"]).astype(np.int32)
        out[...] = R.adjust(logits, **k)[0]

    def text(self, ids, n_steps, more):
        return np.concatenate([ids.reshape(n_steps, -1), np.zeros((more, len(ids) // n_steps), np.int64)])


def gated_params(rng, V=11, H=6, layers=2):
    P = {"E": rng.standard_normal((V, H)) / np.sqrt(H), "W_out": rng.standard_normal((V, H)) / np.sqrt(H), "b_out": 0.1 * rng.standard_normal(V),
         "gamma": 1 + 0.1 * rng.standard_normal(H), "beta": 0.1 * rng.standard_normal(H)}
    for k in map(str, range(layers)):
        P.update({"W" + k: rng.standard_normal((2 * H, H)) / np.sqrt(H), "b" + k: np.concatenate([1 + 0.3 * rng.standard_normal(H), 0.1 * rng.standard_normal(H)]),
                  "gamma" + k: 1 + 0.1 * rng.standard_normal(H), "beta" + k: 0.1 * rng.standard_normal(H)})
    return P
